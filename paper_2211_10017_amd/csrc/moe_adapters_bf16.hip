// Adapters in bf16.
#include "moe_adapters_kernel.h"

namespace moe {

int launch_adapter_bf16(const AdapterArgs &p, int x_dtype, int out_dtype, hipStream_t s, const char *what) { return launch_adapter<MOE_BF16>(p, x_dtype, out_dtype, s, what); }

}  // namespace moe
