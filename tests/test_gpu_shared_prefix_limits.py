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
