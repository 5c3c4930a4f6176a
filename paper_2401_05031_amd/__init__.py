"""MI355X-native token-adapted transformer encoder (OTAS token adaptation): Python binding of the
C ABI in include/otas.h, include/otas_decode.h and include/otas_sched.h.  Argument marshalling only; every step runs in the HIP library."""
from .binding import (  # noqa: F401
    OTAS_F32, OTAS_BF16, OTAS_FLAG_SIZE_BIAS, OTAS_FLAG_TRACE, OTAS_PROMPT_REPLACE, OTAS_PROMPT_GROW, OtasError, Context, Scheduler, OTAS_GAMMA_SKIP, OTAS_GAMMA_UNDECIDED, lib_path, load_library,
    Rotary, Score, HeadNorm, KVCache, KVCache4, OTAS_CACHE4_GROUP, OTAS_ROTARY_HALF, OTAS_ROTARY_INTERLEAVED, OTAS_ROTARY_PLAIN, OTAS_ROTARY_LINEAR, OTAS_ROTARY_BASE,
    OTAS_ROTARY_BY_PARTS, OTAS_DECODE_ARGUMENTS, OTAS_MAX_LONG_SEQ, OTAS_MAX_TREE_NODES,
    otas_schedule, otas_strerror, otas_sched_rate_table, OTAS_CLOCK_PROBE_MAX_SAMPLES,
)
