"""SQuant weight-quantization solver for MI355X (gfx950): HIP kernels behind a C ABI."""
from .binding import (OUT_INT8, OUT_INT4, OUT_F32, OUT_BF16, OUTPUTS, squant_quantize_ex,  # noqa: F401
                      squant_quantize_batched_ex, squant_output_bytes, squant_activation_ranges,
                      squant_quantize_network, MODE_E, MODE_EK, MODE_EKC, MODE_EC, MODES, BatchPlan, SQuantError,  # noqa: F401
                      squant_batched_workspace_bytes, squant_max_channel_elems, squant_quantize,
                      squant_quantize_batched, squant_status_string, squant_version)
from .linear import (ACT_GELU, ACT_NONE, ACT_RELU, ACT_SILU, ACTS, IGNORE_INDEX, KEEP_FULL, KEEP_INT8, KEEP_NONE,  # noqa: F401
                     KEEPS, quantized_cross_entropy, quantized_linear, squant_codes_t, squant_cross_entropy,
                     squant_cross_entropy_backward, squant_linear, squant_linear_backward)
from .attention import (QuantizedCache, packed_attention, squant_attention, squant_attention_backward,  # noqa: F401
                        squant_cache_attention, squant_cache_read, squant_cache_t, squant_cache_write, squant_heads_t,
                        squant_packed_t, squant_paged_t)
