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
