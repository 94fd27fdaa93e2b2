// Products with 4-bit weights, x in 32-bit floats: the kernels of q4_kernels.h.
#include "q4_kernels.h"

namespace fscnn {

template <> hipError_t launch_q4_type<FSCNN_F32>(const Q4Args &a, int parts, hipStream_t st)
{
    constexpr int XT = FSCNN_F32;
    if (parts > 1 || a.M > 16) {
        if (a.M <= 16) return launch_rows<XT, 4, 1, 8>(a, parts, st);
        if (a.M <= 32) return launch_rows<XT, 4, 2, 8>(a, parts, st);
        if (a.M <= 64) return launch_rows<XT, 2, 4, 4>(a, parts, st);
        return launch_tiles<XT, 2, 2, 1, 4, 1>(a, st);
    }
    return launch_rows<XT, 1, 1, 16>(a, 1, st);
}

}  // namespace fscnn
