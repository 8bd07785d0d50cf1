"""What SharedPromptShell.given refuses of its ids before any state changes or anything is launched (no GPU: a shell without its buffers)."""
import pytest
import torch

from paper_2506_18226_b200.shell import SharedPromptShell, ShellConfig


def shell(next_cell=3):
    sh = SharedPromptShell.__new__(SharedPromptShell)
    sh.cfg = ShellConfig(n_layers=1, dim=128, n_heads=2, ffn_hidden=256, vocab=512, n_text=4, grid_h=4, grid_w=4, n_images=3)
    sh.next_cell = next_cell
    sh.dev = torch.device("cpu")
    return sh


@pytest.mark.parametrize("bad", [-1, 512, 2 ** 31, -2 ** 40, 2 ** 32 + 5, 2 ** 62])
@pytest.mark.parametrize("at", [(0, 0), (3, 1), (4, 2)])
def test_ids_outside_the_vocabulary(bad, at):
    ids = torch.zeros(5, 3, dtype=torch.int64)
    ids[at] = bad
    sh = shell()
    with pytest.raises(ValueError, match="vocabulary"):
        sh.given(ids)
    assert sh.next_cell == 3
    if -2 ** 31 <= bad < 2 ** 31:
        with pytest.raises(ValueError, match="vocabulary"):
            sh.given(ids.to(torch.int32))


@pytest.mark.parametrize("ids", [torch.zeros(5, 3), torch.zeros(5, 3, dtype=torch.bool), torch.zeros(5, 3, dtype=torch.bfloat16), torch.tensor(7),
                                 torch.zeros(5, dtype=torch.int32), torch.zeros(1, 5, 3, dtype=torch.int32)])
def test_ids_that_are_no_whole_numbers_by_cell_and_image(ids):
    sh = shell()
    with pytest.raises(ValueError, match="whole numbers"):
        sh.given(ids)
    assert sh.next_cell == 3


@pytest.mark.parametrize("next_cell,shape", [(None, (5, 3)), (3, (0, 3)), (3, (5, 2)), (3, (14, 3))])
def test_ids_that_cannot_follow(next_cell, shape):
    sh = shell(next_cell)
    with pytest.raises(ValueError, match="cannot follow"):
        sh.given(torch.zeros(shape, dtype=torch.int32))
    assert sh.next_cell == next_cell
