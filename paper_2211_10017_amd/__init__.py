"""MI355X-native sparsely activated expert FFN layer with weight-only int4/int8 experts.

The work is done by the HIP library behind ``include/moe_wq.h``; ``binding`` marshals torch
device pointers into its C entry points (loaded on first use, and failing loudly if the
library has not been built).  ``workloads`` holds the seeded synthetic input generators.
"""

from . import adapters, binding, exchange, layer, mx4_layer, optimizer, router, workloads  # noqa: E402,F401
from .layer import MoEExpertLayer  # noqa: E402,F401
from .mx4_layer import MoEMx4Layer  # noqa: E402,F401
from .router import balance_loss  # noqa: E402,F401
from .exchange import combine_tokens, permute_tokens  # noqa: E402,F401
from .adapters import AdapterIndex, LowRankAdapters, adapt, adapter_index  # noqa: E402,F401
from .optimizer import AdamW  # noqa: E402,F401
from .binding import (MoeError, moe_combine, moe_gate_topk, moe_grouped_ffn_wq,  # noqa: E402,F401
                      moe_grouped_ffn_wq_workspace_bytes, moe_permute, moe_permute_workspace_bytes,
                      moe_quantize_experts)
from .binding import (moe_balance_loss, moe_balance_loss_backward, moe_grouped_ffn_mx4,  # noqa: E402,F401
                      moe_grouped_ffn_mx4_workspace_bytes, moe_grouped_gemm_mx4, moe_mx4_dequantize, moe_mx4_quantize_experts,
                      moe_mx4_quantize_rows)
from .binding import (moe_adamw, moe_adamw_state, moe_adapters, moe_adapters_backward, moe_adapters_backward_workspace_bytes,  # noqa: E402,F401
                      moe_combine_backward, moe_permute_backward)
