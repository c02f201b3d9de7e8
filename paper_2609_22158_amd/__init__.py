"""StepKV compression pass on AMD Instinct MI355X (gfx950).

The pass lives in libstepkv.so (hand-written HIP kernels behind the C ABI of
include/stepkv.h); ``binding`` is its ctypes binding. Importing this package
loads nothing; the first binding call loads the library and raises if it has
not been built. ``cache4`` is the binding of the 4-bit cache
(include/stepkv_cache4.h) and of the attention that reads it.
"""
from . import binding, cache4  # noqa: F401
from .binding import (  # noqa: F401
    Params,
    Problem,
    StepKVError,
    StepTracker,
    TextTracker,
    budget_from_ratio,
    compact,
    compact_shared,
    compress,
    decode_attention,
    decode_stats,
    load,
    priority,
    retained_rows,
    saliency,
    saliency_from_lse,
    score,
    score_shared,
    select,
    select_shared,
    step_utilities,
    text_cues,
    window_lse,
)
from .cache4 import (  # noqa: F401
    Cache4,
    advance4,
    append4,
    compact4,
    decode_attention4,
    decode_sparse4,
    read4,
    select_blocks4,
)
