// y = act(x W^T + b) with 4-bit weights (internal.h has their order, q4_tile.h the operands).
//
// rows_kernel (few rows of x): a work-group of W waves owns up to 16 MT rows of x and 16 NT rows of weights.  Both go straight from memory into the
// matrix cores' operands (16 bytes a lane hold the codes of 16 rows x 128 columns).  The waves divide the blocks of
// 128 columns, each keeps fp32 sums of its own, which are added at the end through LDS in the order of the waves.
//
// tile_kernel (many rows of x): a work-group of WM x WN waves owns 32 MT WM rows of x and 32 NT WN rows of weights.  A block of 128 columns of its rows
// of x is in LDS while the next one is on its way there (16 bytes a lane, without registers); codes come from memory into registers a block
// ahead.  What a wave does per block of 128: 8 MT NT products of 32 x 32 x 16, codes to operands, and a multiply-add per output and group, since a
// group's sum is multiplied by its scale in fp32.
#include <type_traits>

#include "internal.h"
#include "lds_dma.h"
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
    int dma, mt, nt;                          // tile_kernel: x may go to LDS without registers; tiles of the launch
};

__device__ inline void store_output(const Q4Args &a, int m, int k, float v, float bias)
{
    store_float(a.y, m * a.ldy + k, a.y_type, act_apply(v + bias, a.act));
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
        scales[t] = a.scales + tile * groups * 16 + col16;
    }
    const char *rows[MT];
#pragma unroll
    for (int u = 0; u < MT; ++u) {
        const int m = m0 + 16 * u + col16;
        rows[u] = a.x + (m < a.M ? m : a.M - 1) * a.ldx;
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
                for (int p = 0; p < X::kParts; ++p) sum[u] = X::mfma(op[u][p], X::ones(), sum[u]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const typename X::Op q = X::codes(w[t][s]);
#pragma unroll
                for (int u = 0; u < MT; ++u)
#pragma unroll
                    for (int p = 0; p < X::kParts; ++p) acc[t][u] = X::mfma(op[u][p], q, acc[t][u]);
            }
            if ((s + 1) % a.steps == 0) {     // the group's end
                const int g = b * 4 / a.steps + s / a.steps;
                q4f4 xs[MT];
#pragma unroll
                for (int u = 0; u < MT; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        xs[u][i] = 1.0f;
                        if (kInt && a.x_cols > 1) {
                            const int m = m0 + 16 * u + 4 * quarter + i;
                            if (m < a.M && g < a.x_cols) xs[u][i] = a.x_scale[(long long)m * a.x_cols + g];
                        }
                    }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const uint32_t sz = scales[t][(long long)g * 16];
                    const float f = __builtin_bit_cast(float, sz & ~15u), z = -(float)(sz & 15);
#pragma unroll
                    for (int u = 0; u < MT; ++u) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float v;
                            if constexpr (kInt) v = (float)(acc[t][u][i] - (int)(sz & 15) * sum[u][i]) * xs[u][i];
                            else v = __builtin_fmaf(z, sum[u][i], acc[t][u][i]);
                            total[t][u][i] = __builtin_fmaf(f, v, total[t][u][i]);
                        }
                        acc[t][u] = {};
                    }
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
        const int m = m0 + e % MT * 16 + 4 * quarter, k = (tile0 + e / MT) * 16 + col16;
        if (k >= a.K) continue;
        const float bias = a.bias ? a.bias[k] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (m + i < a.M) store_output(a, m + i, k, kInt && a.x_cols == 1 ? v[i] * a.x_scale[m + i] : v[i], bias);
    }
}

// The 32 x 32 products: 16 columns in 16 bits, 32 in 8
template <int XT> struct Tile {
    using Acc = q4f16;
    static constexpr int kChunk = 8, kChunks = 16;        // columns in 16 bytes; 16-byte chunks of a row's block
    __device__ static Acc mfma(u4v x, u4v w, Acc c)
    {
        if constexpr (XT == FSCNN_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(q4h8, x), __builtin_bit_cast(q4h8, w), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(q4b8, x), __builtin_bit_cast(q4b8, w), c, 0, 0, 0);
    }
};
template <> struct Tile<FSCNN_I8> {
    using Acc = q4i16;
    static constexpr int kChunk = 16, kChunks = 8;
    __device__ static Acc mfma(u4v x, u4v w, Acc c)
    {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(q4i4, x), __builtin_bit_cast(q4i4, w), c, 0, 0, 0);
    }
};

// Work-group id -> one of a run of ids that share an XCD and its L2
__device__ inline int xcd_neighbours(int bid, int nblk)
{
    const int q = nblk >> 3, rem = nblk & 7, xcd = bid & 7, slot = bid >> 3;
    return xcd < rem ? xcd * (q + 1) + slot : rem * (q + 1) + (xcd - rem) * q + slot;
}

// STEPS: of 32 columns a group.  x in LDS: rows of kChunks 16-byte chunks a part, chunk c of row r at c ^ f(r), so that the 16 lanes that read a chunk of
// adjacent rows find it in all banks
template <int XT, int MT, int NT, int WM, int WN, int STEPS> __global__ void __launch_bounds__(WM * WN * 64, XT == FSCNN_F32 ? 1 : 2) tile_kernel(const Q4Args a)
{
    using X = XOp<XT>;
    using T = Tile<XT>;
    constexpr bool kInt = XT == FSCNN_I8;
    constexpr int kRows = 32 * MT * WM, kThreads = WM * WN * 64, kParts = X::kParts, kCh = T::kChunks;
    constexpr int kPer = kRows * kCh / kThreads;          // chunks a thread brings
    constexpr int kBuf = kRows * kCh * kParts;            // chunks of a buffer
    static_assert(kPer * kThreads == kRows * kCh, "a whole number of chunks a thread");
    __shared__ u4v lds[2 * kBuf];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, wm = wave / WN, wn = wave % WN;
    // panels of 8 tiles of x: work-groups that run together share both operands
    const int lid = xcd_neighbours(blockIdx.x, a.mt * a.nt), panel = lid / (8 * a.nt), in = lid % (8 * a.nt);
    const int tall = a.mt - panel * 8 < 8 ? a.mt - panel * 8 : 8;
    const int m0 = (panel * 8 + in % tall) * kRows, n0 = in / tall * (32 * NT * WN) + wn * (32 * NT);
    auto swizzle = [](int r) { return kCh == 16 ? r & 15 : r >> 1 & 7; };

    const u4v *codes[NT];
    const uint32_t *scales[NT];
    const int groups = a.blocks * 4 / STEPS;
#pragma unroll
    for (int t = 0; t < NT; ++t) {            // (tiles past the last one repeat it: their outputs are not stored)
        int tile = (n0 + 32 * t + (lane & 31)) >> 4;
        tile = tile < a.tiles ? tile : a.tiles - 1;
        codes[t] = a.codes + (long long)tile * a.blocks * 64 + (lane & 15) + 32 * half;
        scales[t] = a.scales + (long long)tile * groups * 16 + (lane & 15);
    }
    const int live = a.M - m0 < kRows ? a.M - m0 : kRows;
    const char *x = a.x + m0 * a.ldx;
    // (with a.dma, kRows * ldx is below 2^31; rows that are not there are out of the descriptor's range and read as zeros)
    const unsigned long long xa = (unsigned long long)x;
    const int4v rsrc = {(int)(uint32_t)xa, (int)(uint32_t)(xa >> 32), (int)((live - 1) * a.ldx + a.C * (16 / T::kChunk)), 0x00020000};
    int from[kPer];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u4v *)lds;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int at = (wave * kPer + i) * 64 + lane, r = at / kCh, c = at % kCh ^ swizzle(r);
        from[i] = r < live ? (int)(r * a.ldx) + c * 16 : (int)0x80000000;
    }
    typename X::Raw raw[XT == FSCNN_I8 ? 2 * kPer : kPer];
    // brings block b's rows of x on their way; what goes through registers is put into LDS by commit()
    auto direct = [&](int b) { return XT != FSCNN_F32 && a.dma && (b + 1) * kQ4Block <= a.C; };
    auto fetch = [&](int b) {
        if (direct(b)) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                lds_dma_dwordx4(rsrc, lds0 + ((b & 1) * kBuf + (wave * kPer + i) * 64) * 16, from[i] + b * (kCh * 16));
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int at = (wave * kPer + i) * 64 + lane, r = at / kCh, c = at % kCh ^ swizzle(r), col = b * kQ4Block + c * T::kChunk;
                const char *row = x + r * a.ldx;
                if constexpr (kInt) {
                    raw[2 * i] = raw[2 * i + 1] = typename X::Raw{};
                    if (r < live) {
                        raw[2 * i] = load_columns<XT, true>(row, col, a.C);
                        raw[2 * i + 1] = load_columns<XT, true>(row, col + 8, a.C);
                    }
                } else {
                    raw[i] = typename X::Raw{};
                    if (r < live) raw[i] = load_columns<XT, true>(row, col, a.C);
                }
            }
        }
    };
    auto commit = [&](int b) {
        if (direct(b)) return;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            u4v *to = lds + (b & 1) * kBuf + (wave * kPer + i) * 64 + lane;
            if constexpr (kInt) *to = u4v{raw[2 * i][0], raw[2 * i][1], raw[2 * i + 1][0], raw[2 * i + 1][1]};
            else {
                u4v part[kParts];
                X::parts(raw[i], part);
#pragma unroll
                for (int p = 0; p < kParts; ++p) to[p * kRows * kCh] = part[p];
            }
        }
    };
    u4v next[NT][2];
    uint32_t word[NT][4 / STEPS];
    auto load_weights = [&](int b) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int e = 0; e < 2; ++e) next[t][e] = codes[t][(long long)b * 64 + 16 * e];
#pragma unroll
            for (int g = 0; g < 4 / STEPS; ++g) word[t][g] = scales[t][((long long)b * (4 / STEPS) + g) * 16];
        }
    };
    q4f16 total[MT][NT] = {};
    const int row0 = wm * (32 * MT) + (lane & 31);
    const u4v *mine = lds + row0 * kCh;

    fetch(0);
    load_weights(0);
    commit(0);
    for (int b = 0; b < a.blocks; ++b) {
        wait_vmcnt<0>();                      // block b is in LDS, its codes in registers
        __syncthreads();
        u4v now[NT][2];
        uint32_t sz[NT][4 / STEPS];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            now[t][0] = next[t][0];
            now[t][1] = next[t][1];
#pragma unroll
            for (int g = 0; g < 4 / STEPS; ++g) sz[t][g] = word[t][g];
        }
        const bool more = b + 1 < a.blocks;
        if (more) {
            fetch(b + 1);
            load_weights(b + 1);
        }
        const u4v *from_lds = mine + (b & 1) * kBuf;
#pragma unroll
        for (int g = 0; g < 4 / STEPS; ++g) {
            typename T::Acc acc[MT][NT] = {};
            typename X::Zero z[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) z[t] = X::zero(sz[t][g]);
#pragma unroll
            for (int s = g * STEPS; s < (g + 1) * STEPS; ++s) {
                if constexpr (kInt) {
                    u4v op[MT];
#pragma unroll
                    for (int u = 0; u < MT; ++u) op[u] = from_lds[u * 32 * kCh + ((2 * s + half) ^ swizzle(row0))];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const u2v w0 = X::weights(now[t][0][s], z[t]), w1 = X::weights(now[t][1][s], z[t]);
#pragma unroll
                        for (int u = 0; u < MT; ++u) acc[u][t] = T::mfma(op[u], u4v{w0[0], w0[1], w1[0], w1[1]}, acc[u][t]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        u4v w[NT];
#pragma unroll
                        for (int t = 0; t < NT; ++t) w[t] = X::weights(now[t][e][s], z[t]);
#pragma unroll
                        for (int p = 0; p < kParts; ++p)
#pragma unroll
                            for (int u = 0; u < MT; ++u) {
                                const u4v op = from_lds[p * kRows * kCh + u * 32 * kCh + ((4 * s + 2 * half + e) ^ swizzle(row0))];
#pragma unroll
                                for (int t = 0; t < NT; ++t) acc[u][t] = T::mfma(op, w[t], acc[u][t]);
                            }
                    }
                }
            }
            // the group's end
            const int group = b * (4 / STEPS) + g;
#pragma unroll
            for (int u = 0; u < MT; ++u) {
                float xs[16];
                if (kInt && a.x_cols > 1) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int m = m0 + wm * (32 * MT) + u * 32 + 8 * (i >> 2) + 4 * half + (i & 3);
                        xs[i] = m < a.M && group < a.x_cols ? a.x_scale[(long long)m * a.x_cols + group] : 0.0f;
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const float f = __builtin_bit_cast(float, sz[t][g] & ~15u);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float v = (float)acc[u][t][i];
                        if (kInt && a.x_cols > 1) v *= xs[i];
                        total[u][t][i] = __builtin_fmaf(f, v, total[u][t][i]);
                    }
                }
            }
            // (a second group's sums at the same time would not fit the registers)
#pragma unroll
            for (int u = 0; u < MT; ++u)
#pragma unroll
                for (int t = 0; t < NT; ++t) asm volatile("" : "+v"(total[u][t]));
        }
        if (more) commit(b + 1);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int k = n0 + 32 * t + (lane & 31);
        if (k >= a.K) continue;
        const float bias = a.bias ? a.bias[k] : 0.0f;
#pragma unroll
        for (int u = 0; u < MT; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int m = m0 + wm * (32 * MT) + u * 32 + 8 * (i >> 2) + 4 * half + (i & 3);
                if (m < a.M) store_output(a, m, k, kInt && a.x_cols == 1 ? total[u][t][i] * a.x_scale[m] : total[u][t][i], bias);
            }
    }
}

template <int XT, int NT, int MT, int W> hipError_t launch_rows(const Q4Args &a, hipStream_t st)
{
    const long long gx = (a.tiles + NT - 1) / NT, gy = ((long long)a.M + 16 * MT - 1) / (16 * MT);
    if (gx * W * 64 > 0xffffffffLL || gy > 65535) return hipErrorInvalidValue;
    hipLaunchKernelGGL((rows_kernel<XT, NT, MT, W>), dim3((unsigned)gx, (unsigned)gy), dim3(W * 64), 0, st, a);
    return hipGetLastError();
}

template <int XT, int MT, int NT, int WM, int WN> hipError_t launch_tiles(Q4Args a, hipStream_t st)
{
    constexpr int rows = 32 * MT * WM, threads = WM * WN * 64;
    const long long mt = ((long long)a.M + rows - 1) / rows, nt = (a.K + 32LL * NT * WN - 1) / (32 * NT * WN);
    if (mt * nt * threads > 0xffffffffLL || 8 * nt > 0x7fffffffLL) return hipErrorInvalidValue;
    a.mt = (int)mt;
    a.nt = (int)nt;
    // 16-byte loads into LDS, offsets of a tile's rows below 2^31
    a.dma = !(((uintptr_t)a.x | (uintptr_t)a.ldx) & 15) && a.ldx * rows < 0x7fff0000LL;
    const dim3 grid((unsigned)(mt * nt)), block(threads);
    if (a.steps == 1) hipLaunchKernelGGL((tile_kernel<XT, MT, NT, WM, WN, 1>), grid, block, 0, st, a);
    else if (a.steps == 2) hipLaunchKernelGGL((tile_kernel<XT, MT, NT, WM, WN, 2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((tile_kernel<XT, MT, NT, WM, WN, 4>), grid, block, 0, st, a);
    return hipGetLastError();
}

template <int XT> hipError_t launch_type(Q4Args a, hipStream_t st)
{
    // (rows of x in launches that a grid holds)
    constexpr long long kMost = 1 << 18;
    for (long long m = 0; m < a.M; m += kMost) {
        Q4Args b = a;
        b.M = a.M - m < kMost ? (int)(a.M - m) : (int)kMost;
        b.x += m * a.ldx;
        if (b.x_scale) b.x_scale += m * a.x_cols;
        b.y = static_cast<char *>(a.y) + m * a.ldy * (a.y_type == FSCNN_F32 ? 4 : 2);
        hipError_t e;
        if (b.M <= 16) e = launch_rows<XT, 1, 1, 8>(b, st);
        else if (b.M <= 32) e = launch_rows<XT, 2, 2, 8>(b, st);
        else if (b.M <= 64) e = launch_rows<XT, 4, 4, 4>(b, st);
        else e = launch_tiles<XT, 2, 2, XT == FSCNN_F32 ? 1 : 2, XT == FSCNN_F32 ? 4 : 2>(b, st);
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
                      (int)q4_blocks(q->C), (int)q4_tiles(q->K), q->group / 32, y_type, x_scale_cols, act, 0, 0, 0};
    switch (x_type) {
        case FSCNN_F32: return launch_type<FSCNN_F32>(a, st);
        case FSCNN_F16: return launch_type<FSCNN_F16>(a, st);
        case FSCNN_BF16: return launch_type<FSCNN_BF16>(a, st);
        default: return launch_type<FSCNN_I8>(a, st);
    }
}

}  // namespace fscnn
