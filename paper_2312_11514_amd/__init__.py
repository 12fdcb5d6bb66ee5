"""MI355X-native sparse-FFN hot path of "LLM in a flash" (arXiv 2312.11514).

The product is the C-ABI library declared in include/lif.h (HIP kernels for gfx950);
this package is the thin ctypes binding over it: Layer (an FFN layer) and KVCache (a paged key-value cache with its attention).  There is no CPU fallback: importing
`binding` without a built liblif.so raises.
"""
from .binding import (  # noqa: F401
    LifError, Layer, load_library, LIF_OK, LIF_INVALID_ARG, LIF_BAD_STATE, LIF_CAPACITY, LIF_HIP_ERROR,
    LIF_F32, LIF_F16, LIF_BF16, FFN_SKIP_DEAD, FFN_FULL_BUNDLE, PRED_LOWRANK, PRED_GATE, KERNEL_NAMES, profile_read, profile_handoff,
    profile_handoff_bytes, NORM_NONE, NORM_RMS, NORM_LAYER, ROTARY_HALF, ROTARY_INTERLEAVED, ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE,
    ROPE_RAMP,
)
from .kv import KVCache, rope_frequencies  # noqa: F401
