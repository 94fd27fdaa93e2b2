// Products with 4-bit weights, x in 8-bit integers: the kernels of q4_kernels.h.
#include "q4_kernels.h"

namespace fscnn {

template <> hipError_t launch_q4_type<FSCNN_I8>(const Q4Args &a, int parts, hipStream_t st)
{
    return launch_narrow<FSCNN_I8>(a, parts, st);
}

}  // namespace fscnn
