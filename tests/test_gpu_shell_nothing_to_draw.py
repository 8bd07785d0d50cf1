"""An image whose logits are NaN has no token to draw (id -1); its decoder goes on, and the other images are as they are without it."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("graphs", [False, True])
@pytest.mark.parametrize("shell", ["SharedPromptShell", "LlamaGenShell"])
def test_an_image_without_a_token(shell, graphs):
    from paper_2506_18226_b200 import shell as S
    cfg = S.ShellConfig(n_layers=2, dim=128, n_heads=2, ffn_hidden=256, vocab=512, n_text=8, grid_h=6, grid_w=6, n_images=3, top_k=50, top_p=0.8)
    rows = 2 if shell == "SharedPromptShell" else cfg.batch
    g = torch.Generator(device="cuda:0").manual_seed(1)
    text = torch.randn(rows, cfg.n_text, cfg.dim, generator=g, device="cuda:0").to(torch.bfloat16)
    ids = []
    for bad in (False, True):
        sh = getattr(S, shell)(cfg, seed=5, use_graphs=graphs)
        sh.prefill(text)
        for cell in range(1, 6):
            if bad and cell == 2:
                sh.logits[1].fill_(math.nan)                               # (as if the step before had made them)
                sh._draw(sh.logits, sh.uniforms[1].contiguous())
                sh.ids_host[1].copy_(sh.tokens)
            sh.decode_step(cell)
        torch.cuda.synchronize()
        ids.append(sh.ids_host[:6].clone())
    assert ids[1][1, 1] == -1 and (ids[1][2:] >= 0).all() and (ids[1][2:] < cfg.vocab).all()
    assert torch.equal(ids[0][:, [0, 2]], ids[1][:, [0, 2]])
    # the image goes on from id 0
    sh = getattr(S, shell)(cfg, seed=5, use_graphs=graphs)
    sh.prefill(text)
    sh.decode_step(1)
    sh.tokens[1] = 0
    for cell in range(2, 6):
        sh.decode_step(cell)
    torch.cuda.synchronize()
    assert torch.equal(sh.ids_host[2:6, 1], ids[1][2:, 1])


@pytest.mark.parametrize("shell", ["SharedPromptShell", "LlamaGenShell"])
def test_all_images_without_a_token(shell):
    from paper_2506_18226_b200 import shell as S
    cfg = S.ShellConfig(n_layers=1, dim=128, n_heads=2, ffn_hidden=256, vocab=512, n_text=8, grid_h=6, grid_w=6, n_images=2, top_k=50, min_p=0.1)
    rows = 2 if shell == "SharedPromptShell" else cfg.batch
    sh = getattr(S, shell)(cfg, seed=5)
    sh.prefill(torch.full((rows, cfg.n_text, cfg.dim), math.nan, dtype=torch.bfloat16, device="cuda:0"))
    assert (sh.tokens == -1).all()
    for cell in range(1, 4):
        assert (sh.decode_step(cell) == -1).all()
    torch.cuda.synchronize()
