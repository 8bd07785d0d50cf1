"""The decoder around the calls between a prompt and its tokens: conditions of different lengths, given tokens, top_p and min_p."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _cfg(**kw):
    from paper_2506_18226_b200.shell import ShellConfig
    return ShellConfig(**dict(dict(n_layers=2, dim=128, n_heads=2, ffn_hidden=256, vocab=512, n_text=70, grid_h=6, grid_w=6, n_images=3, top_k=50), **kw))


def _text(cfg, rows, seed):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return torch.randn(*rows, cfg.dim, generator=g, device="cuda:0").to(torch.bfloat16)


def _close(a, b):
    # a layer stores some eight activations of a row in bfloat16, each off by 2^-8 at most; two layers and the last norm: 17 2^-8 of
    # them if all errors add up, against themselves
    a, b = a.float(), b.float()
    assert float((a - b).norm() / b.norm()) <= 17 * 2.0 ** -8


def test_conditions_of_one_length_end_to_end_and_by_rows():
    from paper_2506_18226_b200.shell import SharedPromptShell
    cfg = _cfg()
    text = _text(cfg, (2, cfg.n_text), 3)
    a, b = SharedPromptShell(cfg, seed=1, use_graphs=False), SharedPromptShell(cfg, seed=1, use_graphs=False)
    a.prefill(text)
    b.prefill((text[0], text[1]))
    _close(b.logits, a.logits)
    assert torch.equal(a.prefix_rows, b.prefix_rows) and int(b.status) == 0
    # the same rows in the cache, up to the rounding of what is made from the attention's outputs
    _close(b.k_pool, a.k_pool)
    _close(b.v_pool, a.v_pool)


def test_conditions_of_different_lengths():
    """Each half as in a decoder of its own, whose conditions are both of that length."""
    from paper_2506_18226_b200.shell import SharedPromptShell
    cfg = _cfg()
    lens = (70, 9)
    cond, null = _text(cfg, (lens[0],), 4), _text(cfg, (lens[1],), 5)
    sh = SharedPromptShell(cfg, seed=2, use_graphs=False)
    sh.prefill((cond, null))
    assert sh.prefix_rows.tolist() == list(lens)
    n = cfg.n_images
    halves = [sh.logits[:n].clone(), sh.logits[n:].clone()]
    for i, (t, half) in enumerate(zip((cond, null), halves)):
        alone = SharedPromptShell(_cfg(n_text=lens[i]), seed=2, use_graphs=False)
        alone.prefill(torch.stack([t, t]))
        _close(half, alone.logits[:n])
    for cell in range(1, 5):
        sh.decode_step(cell)
    assert int(sh.status) == 0
    sh.prefill(_text(cfg, (2, cfg.n_text), 6))                             # and of one length again
    assert sh.prefix_rows.tolist() == [cfg.n_text] * 2


@pytest.mark.parametrize("m", [1, 2, 7, 20])
def test_given_tokens_enter_as_decoded_ones_do(m):
    from paper_2506_18226_b200.shell import SharedPromptShell
    cfg = _cfg()
    text = _text(cfg, (2, cfg.n_text), 7)
    ids = torch.randint(0, cfg.vocab, (m, cfg.n_images), generator=torch.Generator().manual_seed(m), dtype=torch.int32)
    a, b = SharedPromptShell(cfg, seed=3, use_graphs=False), SharedPromptShell(cfg, seed=3)
    for sh in (a, b):
        sh.prefill(text)
        sh.decode_step(1)
    for i in range(m):                                                     # fed one by one
        a.tokens.copy_(ids[i])
        a.decode_step(2 + i)
    b.given(ids)
    _close(b.logits, a.logits)
    assert torch.equal(a.n_before, b.n_before) and torch.equal(a.cell, b.cell) and a.next_cell == b.next_cell
    _close(b.k_pool, a.k_pool)
    for sh in (a, b):                                                      # and on from there, by eager steps and by the graph
        sh.tokens.copy_(ids[0])
        sh.decode_step(2 + m)
    _close(b.logits, a.logits)
    torch.cuda.synchronize()
    assert torch.equal(b.ids_host[1:1 + m], ids) and int(b.status) == 0


def test_given_tokens_that_cannot_follow_are_refused():
    from paper_2506_18226_b200.shell import SharedPromptShell
    cfg = _cfg()
    sh = SharedPromptShell(cfg, seed=4, use_graphs=False)
    ids = torch.zeros(3, cfg.n_images, dtype=torch.int32)
    with pytest.raises(ValueError):
        sh.given(ids)
    sh.prefill(_text(cfg, (2, cfg.n_text), 8))
    for bad in (ids[:0], ids[:, :2], torch.zeros(36, cfg.n_images, dtype=torch.int32)):
        with pytest.raises(ValueError):
            sh.given(bad)
    with pytest.raises(ValueError):
        sh.prefill((_text(cfg, (71,), 1), _text(cfg, (3,), 1)))
    with pytest.raises(ValueError):
        sh.given(ids)                                                      # (a refused prefill leaves none)


@pytest.mark.parametrize("shell", ["SharedPromptShell", "LlamaGenShell"])
def test_top_p_and_min_p(shell):
    """Drawn by adsa_sample from the step's own logits and numbers; the same ids from graphs and eager steps."""
    import paper_2506_18226_b200 as A
    from paper_2506_18226_b200 import shell as S
    cfg = _cfg(n_text=8, top_p=0.8, min_p=0.05)
    both = []
    for graphs in (True, False):
        sh = getattr(S, shell)(cfg, seed=5, use_graphs=graphs)
        sh.prefill(_text(cfg, (2,) if shell == "SharedPromptShell" else (cfg.batch,), 9)[:, None].expand(-1, cfg.n_text, -1).contiguous())
        for cell in range(1, 12):
            sh.decode_step(cell)
            n = cfg.n_images
            want = A.sample(sh.logits[:n], sh.uniforms[cell], uncond=sh.logits[n:], guidance=cfg.cfg_scale, top_k=cfg.top_k, top_p=0.8, min_p=0.05)
            assert torch.equal(sh.tokens, want)
        torch.cuda.synchronize()
        both.append(sh.ids_host[:12].clone())
    assert torch.equal(*both)
