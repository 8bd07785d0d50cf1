"""What the calls on a paged whole-token cache and the shell around them refuse on the GPU, and their largest sizes."""
import pytest
import torch

from test_gpu_shared_prefix import DEV

pytestmark = pytest.mark.gpu


def test_rope_axes_refuses_more_heads_than_32_bits_count():
    """2^32 + 1 heads would be one."""
    import paper_2506_18226_b200 as A
    x = torch.ones(1, 1, 2, dtype=torch.bfloat16, device=DEV).expand(1, 2**32 + 1, 2)
    with pytest.raises(ValueError, match="rope_axes: sizes out of range"):
        A.rope_axes(A.Rotary(2, (1,)), x, torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.bfloat16, device=DEV).expand(1, 2**32 + 1, 2))


def test_arguments_that_no_call_would_read_are_refused():
    """A prefix without its table would be left out of the softmax, an output without its input never written."""
    import paper_2506_18226_b200 as A
    i32 = dict(dtype=torch.int32, device=DEV)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV)
    pool = torch.zeros(5, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    table, n, one = torch.zeros(4, 2, **i32), torch.zeros(4, **i32), torch.zeros(1, **i32)
    for kw in (dict(prefix_rows=one), dict(group_start=torch.tensor([0, 4], **i32)), dict(prefix_rows=one, group_start=torch.tensor([0, 4], **i32))):
        with pytest.raises(ValueError, match="shared_prefix_attn: .* need prefix_table"):
            A.shared_prefix_attn(x, pool, pool, table, n, **kw)
    table[:, 0] = torch.arange(4)
    with pytest.raises(ValueError, match="paged_append: q_out needs q"):
        A.paged_append(x, x, pool, pool.clone(), table, n, q_out=x.clone())


def test_the_shared_prompt_shell_takes_long_conditions():
    """More rows than one attention call has queries for: the logits after the condition agree with the shell that keeps private
    caches, as two bf16 evaluations of one decoder do, and the first steps follow."""
    from paper_2506_18226_b200.shell import LlamaGenShell, SharedPromptShell, ShellConfig
    cfg = ShellConfig(n_layers=2, dim=128, n_heads=2, ffn_hidden=256, vocab=512, n_text=2100, grid_h=2, grid_w=2, n_images=2, top_k=50,
                      budget_fraction=1.0)
    g = torch.Generator(device=DEV).manual_seed(6)
    text = torch.randn(2, cfg.n_text, cfg.dim, generator=g, device=DEV).to(torch.bfloat16)
    a, b = LlamaGenShell(cfg, seed=2, use_graphs=False), SharedPromptShell(cfg, seed=2)
    a.prefill(text.repeat_interleave(cfg.n_images, 0).contiguous())
    b.prefill(text)
    for cell in range(1, 4):
        x, y = a.logits.double(), b.logits.double()
        assert float((x - y).norm() / x.norm()) <= 3e-2 and float((x * y).sum() / (x.norm() * y.norm())) >= 0.999
        a.tokens.copy_(b.tokens)
        a.decode_step(cell)
        b.decode_step(cell)
    assert int(b.status) == 0


def test_expanded_tensors_are_read_and_not_written():
    import paper_2506_18226_b200 as A
    rot = A.Rotary(64, (32,))
    x, pos = torch.randn(1, 2, 64, device=DEV).to(torch.bfloat16), torch.arange(5, dtype=torch.int32, device=DEV)[:, None]
    wide = x.expand(5, 2, 64)
    assert torch.equal(A.rope_axes(rot, wide, pos), A.rope_axes(rot, wide.contiguous(), pos))
    for bad in (wide, x[:, :1].expand(1, 2, 64).expand(5, 2, 64)):
        with pytest.raises(A.AdsaError):
            A.rope_axes(rot, wide, pos, out=bad)
    one = x[:1].as_strided((1, 2, 64), (0, 64, 1))                                # a stride that nothing takes
    want = A.rope_axes(rot, x, pos[3:4])
    assert torch.equal(A.rope_axes(rot, one, pos[3:4], out=one), want) and torch.equal(x, want)
    pool, table = torch.zeros(5, 2, 16, 64, dtype=torch.bfloat16, device=DEV), torch.arange(5, dtype=torch.int32, device=DEV)[:, None].contiguous()
    with pytest.raises(A.AdsaError):
        A.paged_append(wide, wide, pool, pool.clone(), table, torch.zeros(5, dtype=torch.int32, device=DEV), rotary=rot, pos=pos, q=wide, q_out=wide)


@pytest.mark.parametrize("rows,room", [(6, 0), (6, 2000), (80, 30000)])
def test_a_step_captured_over_two_streams(rows, room):
    """q is turned on one stream while k and v enter the cache on another; the attention waits for both, the norm for it."""
    import paper_2506_18226_b200 as A
    from test_gpu_shared_prefix import _gen, _randn, attn_case
    g = _gen(rows + room)
    c = attn_case(g, [30] * rows, [200], [0, rows], 2, 2, 64, 16, torch.bfloat16, room=room)
    i32 = dict(dtype=torch.int32, device=DEV)
    rot, pos = A.Rotary(64, (16, 16)), torch.full((rows, 2), 7, **i32)
    q, k, v = _randn(g, rows, 4, 64), _randn(g, rows, 2, 64), _randn(g, rows, 2, 64)
    x, w = _randn(g, rows, 256), _randn(g, 256)
    before = torch.full((rows,), 29, **i32)
    turned, out, x_out, h = torch.empty_like(q), torch.empty_like(q), torch.empty_like(x), torch.empty_like(x)
    ws = A.shared_prefix_workspace(q, c["k_pool"], c["page_table"], c["prefix_table"])
    side = torch.cuda.Stream()

    def step():
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        A.paged_append(k, v, c["k_pool"], c["v_pool"], c["page_table"], before, rotary=rot, pos=pos)
        with torch.cuda.stream(side):
            A.rope_axes(rot, q, pos, out=turned)
        main.wait_stream(side)
        A.shared_prefix_attn(**dict(c, q=turned), out=out, workspace=ws)
        A.norm_residual(out.view(rows, 256), x, w, x_out=x_out, h=h)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(6):
        for t in (q, k, v, x):
            t.copy_(_randn(g, *t.shape))
        step()
        want = [t.clone() for t in (turned, out, x_out, h)]
        for t in (turned, out, x_out, h):
            t.fill_(3.0)
        for n in range(i + 1):                                                    # several replays one behind the other
            graph.replay()
        for t, u in zip((turned, out, x_out, h), want):
            assert torch.equal(t, u)
