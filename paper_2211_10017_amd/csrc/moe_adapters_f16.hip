// Adapters in fp16: rows in, rows beside them.
#include "moe_adapters_kernel.h"

namespace moe {

int launch_adapter_forward_f16(const AdapterArgs &p, int out_dtype, hipStream_t s, const char *what)
{
    return with_dtype(out_dtype, [&](auto o) {
        constexpr int O = decltype(o)::value;
        return p.y ? launch_types<MOE_F16, MOE_F16, O, true>(p, s, what) : launch_types<MOE_F16, MOE_F16, O, false>(p, s, what);
    });
}

}  // namespace moe
