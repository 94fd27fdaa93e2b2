// y = act(x W^T + b) with 4-bit weights (internal.h has their order, q4_tile.h the operands).
//
// rows_kernel: a work-group of W waves owns 16 NT rows of weights and up to 16 MT rows of x.  Weights are the matrix cores' left operand, straight
// from memory into registers (16 bytes a lane hold 16 rows x 128 columns); rows of x the right one, from the L2.  The waves divide the blocks of
// 128 columns, each keeps fp32 sums of its own, which are added at the end through LDS in the order of the waves.
#include <type_traits>

#include "internal.h"
#include "q4_tile.h"

namespace fscnn {

namespace {

struct Q4Args {
    const u4v *codes;
    const uint32_t *scales;
    const char *x;
    const float *x_scale, *bias;
    void *y;
    long long ldx, ldy;                       // ldx in bytes
    int K, C, M, blocks, tiles, steps, y_type, x_cols, act;   // steps: of 32 columns a group
};

// Four adjacent outputs of a row, from column k on; those from K on are not there
__device__ inline void store_outputs(const Q4Args &a, int token, int k, q4f4 v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = act_apply(v[i] + (a.bias && k + i < a.K ? a.bias[k + i] : 0.0f), a.act);
    const long long at = (long long)token * a.ldy + k;
    if (k + 4 <= a.K) {
        if (a.y_type == FSCNN_F32) __builtin_memcpy(static_cast<float *>(a.y) + at, &v, 16);
        else {
            uint32_t h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                h[i] = a.y_type == FSCNN_F16 ? __builtin_bit_cast(unsigned short, (_Float16)v[i]) : __builtin_bit_cast(unsigned short, (__bf16)v[i]);
            const u2v w = {h[0] | h[1] << 16, h[2] | h[3] << 16};
            __builtin_memcpy(static_cast<unsigned short *>(a.y) + at, &w, 8);
        }
    } else {
        for (int i = 0; i < 4; ++i)
            if (k + i < a.K) store_float(a.y, at + i, a.y_type, v[i]);
    }
}

template <int XT, int NT, int MT, int W> __global__ void __launch_bounds__(W * 64) rows_kernel(const Q4Args a)
{
    using X = XOp<XT>;
    constexpr bool kInt = XT == FSCNN_I8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col16 = lane & 15, quarter = lane >> 4;
    const int tile0 = blockIdx.x * NT, m0 = blockIdx.y * (16 * MT);
    const u4v *codes[NT];
    const uint32_t *scales[NT];
    const int groups = a.blocks * 4 / a.steps;
#pragma unroll
    for (int t = 0; t < NT; ++t) {            // (tiles past the last one repeat it, and so do rows of x: their outputs are not stored)
        const long long tile = tile0 + t < a.tiles ? tile0 + t : a.tiles - 1;
        codes[t] = a.codes + tile * a.blocks * 64 + lane;
        scales[t] = a.scales + tile * groups * 16 + 4 * quarter;
    }
    const char *rows[MT];
    int token[MT];
#pragma unroll
    for (int u = 0; u < MT; ++u) {
        token[u] = m0 + 16 * u + col16 < a.M ? m0 + 16 * u + col16 : a.M - 1;
        rows[u] = a.x + token[u] * a.ldx;
    }
    q4f4 total[NT][MT] = {};
    auto block = [&](int b, auto tail) {
        u4v w[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) w[t] = codes[t][(long long)b * 64];
        typename X::Acc acc[NT][MT] = {}, sum[MT] = {};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            typename X::Op op[MT][X::kParts];
#pragma unroll
            for (int u = 0; u < MT; ++u)
                X::parts(load_columns<XT, decltype(tail)::value>(rows[u], b * kQ4Block + s * 32 + quarter * 8, a.C), op[u]);
#pragma unroll
            for (int u = 0; u < MT; ++u)
#pragma unroll
                for (int p = 0; p < X::kParts; ++p) sum[u] = X::mfma(X::ones(), op[u][p], sum[u]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const typename X::Op q = X::codes(w[t][s]);
#pragma unroll
                for (int u = 0; u < MT; ++u)
#pragma unroll
                    for (int p = 0; p < X::kParts; ++p) acc[t][u] = X::mfma(q, op[u][p], acc[t][u]);
            }
            if ((s + 1) % a.steps == 0) {     // the group's end
                const int g = b * 4 / a.steps + s / a.steps;
                float xs[MT];
#pragma unroll
                for (int u = 0; u < MT; ++u) xs[u] = kInt && a.x_cols > 1 && g < a.x_cols ? a.x_scale[(long long)token[u] * a.x_cols + g] : 1.0f;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const u4v sz = *reinterpret_cast<const u4v *>(scales[t] + (long long)g * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float f = __builtin_bit_cast(float, sz[i] & ~15u);
#pragma unroll
                        for (int u = 0; u < MT; ++u) {
                            float v;
                            if constexpr (kInt) v = (float)(acc[t][u][i] - (int)(sz[i] & 15) * sum[u][i]) * xs[u];
                            else v = __builtin_fmaf(-(float)(sz[i] & 15), sum[u][i], acc[t][u][i]);
                            total[t][u][i] = __builtin_fmaf(f, v, total[t][u][i]);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < MT; ++u) acc[t][u] = {};
                }
#pragma unroll
                for (int u = 0; u < MT; ++u) sum[u] = {};
            }
        }
    };
    const int whole = a.C / kQ4Block;
    int b = wave;
    for (; b < whole; b += W) block(b, std::false_type{});
    if (b < a.blocks) block(b, std::true_type{});

    __shared__ q4f4 sums[W][NT * MT][64];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int u = 0; u < MT; ++u) sums[wave][t * MT + u][lane] = total[t][u];
    __syncthreads();
    for (int e = wave; e < NT * MT; e += W) {
        q4f4 v = sums[0][e][lane];
        for (int i = 1; i < W; ++i) v += sums[i][e][lane];
        const int m = m0 + e % MT * 16 + col16, k = (tile0 + e / MT) * 16 + 4 * quarter;
        if (m >= a.M || k >= a.K) continue;
        if (kInt && a.x_cols == 1) v *= a.x_scale[m];
        store_outputs(a, m, k, v);
    }
}

template <int XT, int NT, int MT, int W> hipError_t launch_rows(const Q4Args &a, hipStream_t st)
{
    const long long gx = (a.tiles + NT - 1) / NT, gy = ((long long)a.M + 16 * MT - 1) / (16 * MT);
    if (gx * W * 64 > 0xffffffffLL || gy > 65535) return hipErrorInvalidValue;
    hipLaunchKernelGGL((rows_kernel<XT, NT, MT, W>), dim3((unsigned)gx, (unsigned)gy), dim3(W * 64), 0, st, a);
    return hipGetLastError();
}

template <int XT> hipError_t launch_type(Q4Args a, hipStream_t st)
{
    // (rows of x in launches of as many as a grid's second dimension holds)
    for (long long m = 0; m < a.M; m += 1 << 21) {
        Q4Args b = a;
        b.M = a.M - m < 1 << 21 ? (int)(a.M - m) : 1 << 21;
        b.x += m * a.ldx;
        if (b.x_scale) b.x_scale += m * a.x_cols;
        b.y = static_cast<char *>(a.y) + m * a.ldy * (a.y_type == FSCNN_F32 ? 4 : 2);
        const hipError_t e = b.M <= 16 ? launch_rows<XT, 1, 1, 8>(b, st) : b.M <= 32 ? launch_rows<XT, 2, 2, 8>(b, st) : launch_rows<XT, 4, 4, 4>(b, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_linear_q4(const fscnn_q4 *q, const void *x, int x_type, long long ldx, const float *x_scale, int x_scale_cols, int M,
                            const float *bias, int act, void *y, int y_type, long long ldy, hipStream_t st)
{
    const int bytes = x_type == FSCNN_F32 ? 4 : x_type == FSCNN_I8 ? 1 : 2;
    const Q4Args a = {reinterpret_cast<const u4v *>(q->codes), q->scales, static_cast<const char *>(x), x_scale, bias, y, ldx * bytes, ldy, q->K, q->C, M,
                      (int)q4_blocks(q->C), (int)q4_tiles(q->K), q->group / 32, y_type, x_scale_cols, act};
    switch (x_type) {
        case FSCNN_F32: return launch_type<FSCNN_F32>(a, st);
        case FSCNN_F16: return launch_type<FSCNN_F16>(a, st);
        case FSCNN_BF16: return launch_type<FSCNN_BF16>(a, st);
        default: return launch_type<FSCNN_I8>(a, st);
    }
}

}  // namespace fscnn
