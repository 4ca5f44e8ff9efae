"""SubGraph-Stationary SubNet inference on B200: ctypes binding of the CUDA library plus the
seeded workload generators.  The CUDA library is loaded on first use, never at import."""
from . import workload  # noqa: F401
from .binding import (SGS_BF16, SGS_DISTILL_TOP_MAX, SGS_E4M3, SGS_E5M2, SGS_F32, SGS_POLICY_AVGNET, SGS_POLICY_INTERSECTION, SGS_STRICT_ACCURACY, SGS_STRICT_LATENCY, SGS_TOP_LOGITS_MAX, AuxArgs, AuxDesc, CacheStats, ConvDesc, ConvI8Desc, DistillDesc, LinearF8Desc, QuantizeF8Desc, Scheduler, SgsError, StreamOpts, StreamStats, SuperNet, TopLogitsDesc,  # noqa: F401
                      aux_op, conv2d_sliced, conv2d_sliced_i8, conv2d_sliced_static, debug_expire_f8_wait, debug_expire_team_wait, debug_expire_wait, device_status, device_status_clear, distill, distill_backward, lib, linear_f8, measure_fma_peak, quantize_f8, top_logits)
