// Adapters in fp16: gradients of rows.
#include "moe_adapters_kernel.h"

namespace moe {

int launch_adapter_backward_f16(const AdapterArgs &p, int x_dtype, hipStream_t s, const char *what)
{
    return with_dtype(x_dtype, [&](auto x) { return launch_types<decltype(x)::value, MOE_F16, MOE_F16, false>(p, s, what); });
}

}  // namespace moe
