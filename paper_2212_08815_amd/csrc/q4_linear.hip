// y = act(x W^T + b) with 4-bit weights (internal.h has their order).  The simple form: a wave per row of x and tile of 16 weight rows, a
// quarter of a wave per 8 columns of each step of 32; the four quarters' sums are added at the end.
#include <type_traits>

#include "internal.h"
#include "lowbits.h"

namespace fscnn {

namespace {

struct Q4Args {
    const uint32_t *codes, *scales;
    const void *x;
    const float *x_scale, *bias;
    void *y;
    long long ldx, ldy;
    int K, C, M, blocks, group, x_type, y_type, x_cols, act;
};

__global__ void __launch_bounds__(64) linear_kernel(const Q4Args a)
{
    const int lane = threadIdx.x, row = lane & 15, quarter = lane >> 4;
    const long long tile = blockIdx.x;
    for (int m = blockIdx.y; m < a.M; m += gridDim.y) {
        const int ng = kQ4Block / a.group;
        float sum = 0.0f;
        for (int b = 0; b < a.blocks; ++b) {
            for (int s = 0; s < 4; ++s) {
                const uint32_t w = a.codes[((tile * a.blocks + b) * 64 + lane) * 4 + s];
                const int g = b * ng + s * 32 / a.group;
                const uint32_t sz = a.scales[(tile * a.blocks * ng + g) * 16 + row];
                const int zero = (int)(sz & 15);
                const float scale = __builtin_bit_cast(float, sz & ~15u);
                const int col = b * kQ4Block + s * 32 + quarter * 8;
                float f = 0.0f;
                int whole = 0;
                for (int j = 0; j < 8; ++j) {
                    const int v = (int)(w >> (j < 4 ? 8 * j : 8 * (j - 4) + 4) & 15) - zero;
                    if (col + j >= a.C) continue;
                    const long long at = (long long)m * a.ldx + col + j;
                    if (a.x_type == FSCNN_I8) whole += v * static_cast<const int8_t *>(a.x)[at];
                    else f = __builtin_fmaf((float)v, load_float(a.x, at, a.x_type), f);
                }
                if (a.x_type == FSCNN_I8 && col < a.C) f = (float)whole * a.x_scale[(long long)m * a.x_cols + (a.x_cols == 1 ? 0 : g)];
                sum = __builtin_fmaf(scale, f, sum);
            }
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        const long long k = tile * 16 + row;
        if (quarter == 0 && k < a.K) store_float(a.y, (long long)m * a.ldy + k, a.y_type, act_apply(sum + (a.bias ? a.bias[k] : 0.0f), a.act));
    }
}

}  // namespace

hipError_t launch_linear_q4(const fscnn_q4 *q, const void *x, int x_type, long long ldx, const float *x_scale, int x_scale_cols, int M,
                            const float *bias, int act, void *y, int y_type, long long ldy, hipStream_t st)
{
    const Q4Args a = {q->codes, q->scales, x, x_scale, bias, y, ldx, ldy, q->K, q->C, M, (int)q4_blocks(q->C), q->group, x_type, y_type, x_scale_cols, act};
    const long long tiles = q4_tiles(q->K);
    if (tiles * 64 > 0xffffffffLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL(linear_kernel, dim3((unsigned)tiles, M < 65535 ? M : 65535), dim3(64), 0, st, a);
    return hipGetLastError();
}

}  // namespace fscnn
