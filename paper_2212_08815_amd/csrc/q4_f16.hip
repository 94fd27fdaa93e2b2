// Products with 4-bit weights, x in 16-bit floats (fp16): the kernels of q4_kernels.h.
#include "q4_kernels.h"

namespace fscnn {

template <> hipError_t launch_q4_type<FSCNN_F16>(const Q4Args &a, int parts, hipStream_t st)
{
    constexpr int XT = FSCNN_F16;
    if (a.M <= 16) return launch_rows<XT, 1, 1, 16>(a, parts, st);
    if (a.M <= 32) return launch_rows<XT, 1, 2, 8>(a, parts, st);
    if (a.M <= 64) return launch_rows<XT, 1, 4, 8>(a, parts, st);
    if ((long long)((a.M + 127) / 128) * ((a.K + 127) / 128) < 400) return launch_tiles<XT, 2, 1, 1, 4, 2>(a, st);
    return launch_tiles<XT, 4, 1, 1, 4, 1>(a, st);
}

}  // namespace fscnn
