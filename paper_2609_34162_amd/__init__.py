"""MI355X-native data-parallel optimizer update (SlideDP's hot path):
aggregate R ranks' BF16 gradients, clip by the global L2 norm, mixed-precision
AdamW on FP32 master/moments, BF16 re-emit -- hand-written HIP for gfx950
behind the C ABI in include/sdp.h.  ``sdp`` is the ctypes binding; ``ops`` is
that of include/sdp_ops.h and include/sdp_layer.h, the training operators beside
the update (norm and rotation of queries and keys, grouped products of experts,
distillation loss; embedding, norms around a block, routing and the rows to the
experts and back)."""
from . import sdp  # noqa: F401  (raises ImportError if libsdp.so is not built)
from . import ops  # noqa: F401

__all__ = ["ops", "sdp"]
