// Adapters in bf16: gradients of rows.
#include "moe_adapters_kernel.h"

namespace moe {

int launch_adapter_backward_bf16(const AdapterArgs &p, int x_dtype, hipStream_t s, const char *what)
{
    return with_dtype(x_dtype, [&](auto x) { return launch_types<decltype(x)::value, MOE_BF16, MOE_BF16, false>(p, s, what); });
}

}  // namespace moe
