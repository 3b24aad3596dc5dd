// Adapters in fp16.
#include "moe_adapters_kernel.h"

namespace moe {

int launch_adapter_f16(const AdapterArgs &p, int x_dtype, int out_dtype, hipStream_t s, const char *what) { return launch_adapter<MOE_F16>(p, x_dtype, out_dtype, s, what); }

}  // namespace moe
