"""Limits of the calls on a paged whole-token cache that are found on the host.  Addresses here are made up and never dereferenced."""
import ctypes as C

import pytest

import paper_2506_18226_b200 as A
from paper_2506_18226_b200 import binding as B

P = 0x10000000      # a 256-byte aligned address


def _rotary(head_dim, pairs, halves):
    r = B.AdsaRotary()
    assert A.load().adsa_rotary_init(C.byref(r), head_dim, 1, (C.c_int32 * 1)(pairs), halves, 1, 0.0) == 0
    return r


@pytest.mark.parametrize("halves", [0, 1])
@pytest.mark.parametrize("heads", [2**23, 2**25, 2**26, 2**27 + 5, 2**31 - 1])
def test_more_heads_than_a_grid_holds_are_refused(heads, halves):
    """Their units (up to one an element) pass 32 bits."""
    r = _rotary(64, 32, halves)
    assert A.load().adsa_rope_axes(C.byref(r), 0, P + 2, 64, 64, P, 1, heads, P + 2, 64, 64, None) == B.EINVAL
    kv = B.AdsaPagedKv(P, P, 0, 10, 2, 16, 64, 64)
    assert A.load().adsa_paged_append(C.byref(kv), P, 1, 3, P, None, 1, P + 2, 128, 64, P, 128, 64, C.byref(r), P, P, heads, 0, 64, P, 0, 64,
                                      None, None) == B.EINVAL


def _shell_without_a_gpu(grid, monkeypatch):
    """A SharedPromptShell whose step does nothing but count, and note on which device it would run."""
    import contextlib

    import torch
    from paper_2506_18226_b200.shell import SharedPromptShell, ShellConfig
    current = ["cuda:0"]

    @contextlib.contextmanager
    def device(dev):
        current.append(str(dev))
        yield
        current.pop()

    monkeypatch.setattr(torch.cuda, "device", device)

    class Counting(SharedPromptShell):
        def __init__(self):
            self.cfg = ShellConfig(n_layers=1, dim=64, n_heads=1, ffn_hidden=64, vocab=8, n_text=1, grid_h=grid, grid_w=grid, n_images=2)
            self.dev, self.use_graphs, self.graph, self.kernel_calls, self.steps = torch.device("cuda:1"), False, None, 0, []
            self.next_cell = None
            self.ids_host, self.tokens = torch.zeros(grid * grid, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)

        def _step(self):
            self.steps.append(current[-1])

        def _prefill(self, text_emb):
            self._step()

    return Counting()


def test_the_shared_prompt_shell_stops_at_the_end_of_its_grid(monkeypatch):
    """A step beyond it would look up a position and random numbers that the device does not have."""
    sh = _shell_without_a_gpu(3, monkeypatch)
    for cell in (0, 1, 8):
        with pytest.raises(ValueError, match="prefill first"):
            sh.decode_step(cell)
    sh.next_cell = 1                                                              # as after a prefill
    for cell in range(1, 9):
        for other in (0, cell - 1, cell + 1, 9, -1):
            if other != cell:
                with pytest.raises(ValueError):
                    sh.decode_step(other)
        assert sh.decode_step(cell) is sh.tokens
    for cell in (8, 9, 10):
        with pytest.raises(ValueError):
            sh.decode_step(cell)
    assert len(sh.steps) == 8


def test_the_shared_prompt_shell_runs_on_its_own_device(monkeypatch):
    """Whatever device is the current one: a kernel launched there could not reach the shell's buffers."""
    sh = _shell_without_a_gpu(2, monkeypatch)
    sh.prefill(None)
    sh.next_cell = 1
    sh.decode_step(1)
    assert sh.steps == ["cuda:1", "cuda:1"]


def test_the_shared_prompt_shell_refuses_a_condition_of_no_rows():
    from paper_2506_18226_b200.shell import SharedPromptShell, ShellConfig
    with pytest.raises(ValueError, match="condition"):
        SharedPromptShell(ShellConfig(n_layers=1, dim=64, n_heads=1, ffn_hidden=64, vocab=8, n_text=0, grid_h=2, grid_w=2, n_images=1))


@pytest.mark.parametrize("wrong", [b"torch 1.", b"Python 2."])
def test_a_binding_built_against_another_torch_or_python_is_built_again(wrong, tmp_path, monkeypatch):
    """Its file is as new as its sources all the same."""
    import os
    import shutil

    from paper_2506_18226_b200 import build
    good = build.build_marshal()
    mine = str(tmp_path / "adsa_marshal.so")
    monkeypatch.setattr(build, "MARSHAL", mine)
    built = []

    def compiler(command):
        built.append(command)
        shutil.copyfile(good, command[command.index("-o") + 1])

    monkeypatch.setattr(build.subprocess, "check_call", compiler)
    shutil.copyfile(good, mine)
    assert build.build_marshal() == mine and not built
    with open(good, "rb") as f:
        whole = f.read()
    word = wrong.split()[0] + b" "
    at = whole.index(word, whole.index(b"adsa_marshal built against "))
    with open(mine, "wb") as f:
        f.write(whole[:at] + wrong + whole[at + len(wrong):])
    assert os.path.getmtime(mine) >= os.path.getmtime(build.MARSHAL_SOURCE)
    assert build.build_marshal() == mine and len(built) == 1
    with open(mine, "rb") as f:
        assert f.read() == whole


@pytest.mark.parametrize("token,head", [(0, 64), (128, 0), (63, 256), (-60, 256), (256, 32), (256, -62)])
def test_outputs_whose_rows_overlap_are_refused(token, head):
    """An expanded tensor turned in place would be turned several times, by threads that race."""
    r = _rotary(64, 32, 0)
    assert A.load().adsa_rope_axes(C.byref(r), 0, P, token, head, P, 3, 2, P, token, head, None) == B.EINVAL
    kv = B.AdsaPagedKv(P, P, 0, 10, 2, 16, 64, 64)
    assert A.load().adsa_paged_append(C.byref(kv), P, 1, 3, P, None, 3, P, 128, 64, P, 128, 64, C.byref(r), P, P, 2, token, head, P, token, head,
                                      None, None) == B.EINVAL
