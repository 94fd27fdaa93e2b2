// Products with 4-bit weights, x in 16-bit floats (bfloat16): the kernels of q4_kernels.h.
#include "q4_kernels.h"

namespace fscnn {

template <> hipError_t launch_q4_type<FSCNN_BF16>(const Q4Args &a, int parts, hipStream_t st)
{
    return launch_narrow<FSCNN_BF16>(a, parts, st);
}

}  // namespace fscnn
