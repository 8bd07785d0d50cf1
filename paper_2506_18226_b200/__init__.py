"""B200-native ADSA decode attention: CUDA kernels behind a C-ABI (libadsa.so) plus a thin binding."""
from .binding import (  # noqa: F401
    AdsaBuffers,
    AdsaConfig,
    AdsaEngine,
    AdsaError,
    EXPORTS,
    Rotary,
    cfg_sample,
    decode_attn_static,
    load,
    norm_residual,
    paged_append,
    rmsnorm,
    rope_axes,
    shared_prefix_attn,
    shared_prefix_workspace,
    strerror,
    swiglu,
    workspace_bytes,
)
from .build import build_lib, build_marshal  # noqa: F401
