"""MI355X-native quantized matrix-product path (quant_int, dot'_int, fused
epilogues) of arxiv 1805.12096.  The work is done by hand-written gfx950 HIP
kernels behind a C boundary (include/mq.h, include/mq_seq.h); this package is the thin binding."""
from . import binding, seq
from .binding import *  # noqa: F401,F403
from .seq import *  # noqa: F401,F403

__all__ = binding.__all__ + seq.__all__
