// Products with 4-bit weights, x in 32-bit floats: the kernels of q4_kernels.h.
#include "q4_kernels.h"

namespace fscnn {

template <> hipError_t launch_q4_type<FSCNN_F32>(const Q4Args &a, int parts, hipStream_t st)
{
    constexpr int XT = FSCNN_F32;
    // every row's three parts in one operand; else a wave's own parts (few rows, little work) or a tile's, made once for 256 rows of weights
    switch (f32_choice(a.tiles, a.blocks, a.M, parts).kernel) {
        case F32Choice::kStaged: return a.blocks >= 64 && a.tiles <= 256 ? launch_staged<XT, 16>(a, st) : launch_staged<XT, 8>(a, st);
        case F32Choice::kRows: return launch_rows<XT, 8>(a, st);
        case F32Choice::kTile32: return launch_tiles<XT, 1, 8, 1, false, false>(a, parts, st);
        default: return launch_tiles<XT, 2, 8, 1, false, false>(a, parts, st);
    }
}

}  // namespace fscnn
