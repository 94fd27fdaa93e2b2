// Products with 4-bit weights, x in 32-bit floats: the kernels of q4_kernels.h.
#include "q4_kernels.h"

namespace fscnn {

template <> hipError_t launch_q4_type<FSCNN_F32>(const Q4Args &a, int parts, hipStream_t st)
{
    constexpr int XT = FSCNN_F32;
    const Q4Choice c = f32_choice(a.tiles, a.blocks, a.M, parts);
    switch (c.kernel) {
        case Q4Choice::kStaged: return c.waves == 16 ? launch_staged<XT, 16>(a, st) : launch_staged<XT, 8>(a, st);
        case Q4Choice::kRows: return launch_rows<XT, 8>(a, st);
        default: return c.shape == 32 ? launch_tiles<XT, 1, 8, 1, false, false>(a, parts, st) : launch_tiles<XT, 2, 8, 1, false, false>(a, parts, st);
    }
}

}  // namespace fscnn
