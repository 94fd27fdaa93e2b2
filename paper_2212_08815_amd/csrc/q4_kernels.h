// The kernels of y = act(x W^T + b) with 4-bit weights (internal.h has their order, q4_tile.h the operands), for one type of x a translation unit.
//
// rows_kernel (one or two rows of x; fp32 also six to 16 of little work) and staged_kernel (up to 16 rows, in fp32 five): a work-group of W waves owns
// 16 rows of weights, whose codes go straight from memory into the matrix cores' operands (16 bytes a lane hold 16 rows x 128 columns), as do
// the rows of x or, in staged_kernel, from LDS.  The waves divide the blocks of 128 columns, each keeps fp32 sums of its own, which are
// added at the end through LDS.  What bounds them: a launch and two trips to memory where the weights are few (4096 x 4096, one row of bf16: 3.7 us,
// 2.3 TB/s), else vector instructions and the codes' way (25088 x 4096, one row of fp32: 13.6 us, 3.9 TB/s).
//
// tile_kernel (many rows of x): WN waves, a set, own 32 MT rows of x and 32 WN rows of weights.  A block of 128 columns of the rows of x is in LDS
// while the next one is on its way there (16 bytes a lane, without registers where x is aligned); codes come from memory into registers a
// block ahead.  WK sets may divide the blocks; their sums are added through LDS.  What a wave does per block (16 bits, MT = 4): 32 products of
// 32 x 32 x 16, 1024 clocks of the matrix core, 19 vector instructions for every 8 codes a lane, 152, and 64 multiply-adds, since a
// group's sum is multiplied by its scale in fp32; with addresses and staging 263.  So what counts is how few of the latter there are for a
// product: hence 128 rows of x per decoded weight.  4096 rows of 4096 x 12288, bf16: 416 us, 0.99 PFLOP/s.  Matrix cores are busy 47 % of the
// clocks there, vector instructions as long again; decoding takes 13 %, scales 7, the rows' way to LDS 11, stores 10, LDS reads 4.
// Decoding for twice the rows at once, codes two blocks ahead, products and vector instructions interleaved by hand, and one barrier a block with the next block's first
// operands read beside the last products brought 1 % or less, or lost.
#pragma once
#include <type_traits>

#include "internal.h"
#include "lds_dma.h"
#include "q4_choice.h"
#include "q4_tile.h"

namespace fscnn {

struct Q4Args {
    const u4v *codes;
    const uint32_t *scales;
    const char *x;
    const float *x_scale, *bias;
    void *y;
    float *sums;                              // tile_kernel: [gridDim.y][M][16 tiles], where work-groups divide the blocks
    long long ldx, ldy;                       // ldx in bytes
    int K, C, M, blocks, tiles, steps, y_type, x_cols, act;   // steps: of 32 columns a group
    int x_type;
    int mt, nt;                               // tile_kernel: tiles of the launch
};

namespace {

__device__ inline bool finite(float v) { return fabsf(v) < __builtin_inff(); }

// The sum of an output from the definition, entry by entry, in 64 bits, where no product or sum is too large: a row of x, its scales, and codes
// and scales from the weight row's first on.  By a whole wave: four columns a lane, the lanes' sums added in a fixed order.  (No more than
// four, and in functions that are not inlined and call no others: the kernels' own registers are what counts, and none uses a stack.)
__device__ __attribute__((always_inline)) inline float sum_again(const char *row, int x_type, const float *x_scale, int x_cols, const uint32_t *codes,
                                                                  const uint32_t *scales, int C, int group)
{
    double sum = 0.0;
#pragma unroll 1
    for (int c = (threadIdx.x & 63) * 4; c < C; c += 256) {
        const int g = c / group;
        // (four codes of a parity: code_bit)
        const uint32_t word = codes[(c >> 7) * 256LL + (c >> 3 & 3) * 64 + (c >> 5 & 3)] >> (c & 4), sz = scales[g * 16LL];
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = c + j < C ? c + j : c;
            x[j] = x_type == FSCNN_I8 ? (float)reinterpret_cast<const int8_t *>(row)[at] : load_float(row, at, x_type);
        }
        const double s = (double)__builtin_bit_cast(float, sz & ~15u), xs = x_scale ? (double)x_scale[x_cols > 1 ? g : 0] : 1.0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < C) sum += x[j] * xs * (((int)(word >> code_bit(j) & 15) - (int)(sz & 15)) * s);
        if (__any(sum != sum)) break;        // NaN stays
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    return (float)sum;
}

__device__ __attribute__((noinline)) float one_again(const char *row, int x_type, const float *x_scale, int x_cols, const uint32_t *codes,
                                                           const uint32_t *scales, int C, int group)
{
    return sum_again(row, x_type, x_scale, x_cols, codes, scales, C, group);
}

// Whether a row of x holds a NaN; by a whole wave
__device__ __attribute__((always_inline)) inline int has_nan(const char *row, int x_type, int C)
{
    int nan = 0;
#pragma unroll 1
    for (int c = threadIdx.x & 63; !__any(nan) && c - (int)(threadIdx.x & 63) < C; c += 256)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = load_float(row, c + 64 * j < C ? c + 64 * j : C - 1, x_type);
            nan |= x != x;
        }
    return __any(nan);
}

__device__ __attribute__((noinline)) int nan_in_row(const char *row, int x_type, int C) { return has_nan(row, x_type, C); }

// v of the wave's lanes, each the sum of output (m, k) if it is one (`real`): those that are not finite are made again.  A kernel's may be that
// where the definition's is finite (codes times x, or a group's sum before it meets its scale, past the largest float), or NaN where it is
// infinite (an infinite x in three parts, or less the zero point's share).  bf16, 4096 columns: 64 x 4096 outputs 16 us, 0.15 ms if those of one row are
// made again; 4096 x 12288 415 us, 160 ms if all are, 0.9 if all are NaN.  Looking for them costs up to 2 % (0.1 us of the smallest calls).
__device__ inline float mended(const Q4Args &a, bool real, int m, int k, float v)
{
    int looked = -1, nan = 0;                 // the row of x that was looked at last, for a NaN: its sums are NaN as they are
    for (unsigned long long todo = __ballot(real && !finite(v)); __builtin_expect(todo != 0, 0); todo &= todo - 1) {
        const int lane = __builtin_ctzll(todo), mm = __builtin_amdgcn_readlane(m, lane), kk = __builtin_amdgcn_readlane(k, lane);
        if (mm != looked && a.x_type != FSCNN_I8) nan = nan_in_row(a.x + mm * a.ldx, a.x_type, a.C);
        looked = mm;
        if (nan) continue;
        const long long tile = kk >> 4;
        const float s = one_again(a.x + mm * a.ldx, a.x_type, a.x_scale ? a.x_scale + (long long)mm * a.x_cols : nullptr, a.x_cols,
                                  reinterpret_cast<const uint32_t *>(a.codes) + (tile * a.blocks * 256 + (kk & 15) * 4),
                                  a.scales + (tile * a.blocks * (64 >> (a.steps >> 1)) + (kk & 15)), a.C, a.steps * 32);
        if ((int)(threadIdx.x & 63) == lane) v = s;
    }
    return v;
}

// The activation, which leaves NaN as it is (act_apply's ReLU gives 0 for it, as the convolutions have it)
__device__ inline float activated(float v, int act)
{
    float y = (act == 1) & (v <= 0.0f) ? 0.0f : v;
    if (__builtin_expect((act & ~1) != 0, 0)) y = v > 0.0f ? v : v * __builtin_bit_cast(float, act);
    return y;
}

// Lane l's output l % 32 of a row of x and 32 weight rows (codes, scales: of the first one on, which is a tile's first), of those that `bad` has a bit
// for, by a wave.  NaN where the row of x holds one.
__device__ __attribute__((noinline)) float row_again(uint32_t bad, const char *row, int x_type, const float *x_scale, int x_cols, const uint32_t *codes,
                                                     const uint32_t *scales, int blocks, int C, int group)
{
    float v = __builtin_nanf("");
    if (x_type != FSCNN_I8 && has_nan(row, x_type, C)) bad = 0;
#pragma unroll 1
    for (bad = __builtin_amdgcn_readfirstlane(bad); bad; bad &= bad - 1) {
        const int at = __builtin_ctz(bad);
        const long long tile = (at >> 4) * (long long)blocks;
        const float s = sum_again(row, x_type, x_scale, x_cols, codes + (tile * 256 + (at & 15) * 4), scales + (tile * (128 / group) * 16 + (at & 15)), C, group);
        if ((int)(threadIdx.x & 31) == at) v = s;
    }
    return v;
}

__device__ inline void store_output(const Q4Args &a, int m, int k, float v, float bias)
{
    store_float(a.y, m * a.ldy + k, a.y_type, activated(v + bias, a.act));
}

// The scales of a group of rows m to m + 3 of x, where x has one for each group
template <int XT> __device__ inline q4f4 row_scales(const Q4Args &a, int m, int group)
{
    q4f4 xs = {1.0f, 1.0f, 1.0f, 1.0f};
    if (XT == FSCNN_I8 && a.x_cols > 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) xs[i] = m + i < a.M && group < a.x_cols ? a.x_scale[(long long)(m + i) * a.x_cols + group] : 0.0f;
    }
    return xs;
}

// A group's end in the 16-row kernels: its sum without the zero point's share, times its scale (and, in 8 bits, those of x).  acc, sum: products with
// the codes and with ones
template <int XT, class Acc> __device__ inline q4f4 add_group(const q4f4 &xs, uint32_t word, const Acc &acc, const Acc &sum, q4f4 total)
{
    const float f = __builtin_bit_cast(float, word & ~15u), z = -(float)(word & 15);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v;
        if constexpr (XT == FSCNN_I8) {
            v = (float)(acc[i] - (int)(word & 15) * sum[i]) * xs[i];
        } else {
            v = __builtin_fmaf(z, sum[i], acc[i]);
        }
        total[i] = __builtin_fmaf(f, v, total[i]);
    }
    return total;
}

// The outputs of 16 rows of weights from the sums of W waves, [W][64 lanes][4 rows of the operand], PARTS rows of which are one of x: added in the
// order of parts and waves
template <int XT, int PARTS, int W> __device__ inline void store_sums(const Q4Args &a, const float *sums, int tile)
{
    for (int e0 = 0; e0 < a.M * 16; e0 += W * 64) {
        const int e = e0 + threadIdx.x, m = e >> 4, k = tile * 16 + (e & 15);
        const bool real = m < a.M && k < a.K;
        float f = 0.0f, bias = 0.0f;
        if (real) {
            if (a.bias) bias = a.bias[k];     // (on its way beside the reads of LDS)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                const int row = m * PARTS + p, at = ((row >> 2) * 16 + (e & 15)) * 4 + (row & 3);
#pragma unroll
                for (int w = 0; w < W; ++w) f += sums[w * 256 + at];
            }
            if (XT == FSCNN_I8 && a.x_cols == 1) f *= a.x_scale[m];
        }
        f = mended(a, real, m, k, f);
        if (real) store_output(a, m, k, f, bias);
    }
}

// 16 rows of weights, W waves
template <int XT, int W, int STEPS> __global__ void __launch_bounds__(W * 64) rows_kernel(const Q4Args a)
{
    using X = XOp<XT>;
    constexpr int kGroups = 4 / STEPS;        // of a block
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col16 = lane & 15, quarter = lane >> 4, tile = blockIdx.x;
    const u4v *codes = a.codes + (long long)tile * a.blocks * 64 + lane;
    const uint32_t *scales = a.scales + (long long)tile * a.blocks * (kGroups * 16) + col16;
    const char *row = a.x + (col16 < a.M ? col16 : a.M - 1) * a.ldx;   // (rows past the last one repeat it: their outputs are not stored)
    struct Weights {
        u4v w;
        uint32_t sz[kGroups];
    };
    auto load_weights = [&](int b, Weights &v) {
        v.w = codes[(long long)b * 64];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) v.sz[g] = scales[((long long)b * kGroups + g) * 16];
    };
    typename X::Raw raw[4];
    auto load_x = [&](int b, int s, auto tail) { raw[s] = load_columns<XT, decltype(tail)::value>(row, b * kQ4Block + s * 32 + quarter * 8, a.C); };
    q4f4 total = {};
    // block b; its loads are done or on their way, those of block `then` are issued here if there is one
    auto block = [&](int b, int then, const Weights &v, Weights &next, auto has) {
        if constexpr (decltype(has)::value) load_weights(then, next);
        q4f4 xs[kGroups];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) xs[g] = row_scales<XT>(a, 4 * quarter, b * kGroups + g);
        typename X::Acc acc = {}, sum = {};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            typename X::Op op[X::kParts];
            X::parts(raw[s], op);
            if constexpr (decltype(has)::value) load_x(then, s, std::false_type{});
            if constexpr (X::kParts > 1) {    // (a product with ones costs more here than to subtract zero points, and the parts' sums lose a digit)
                const typename X::Op q = X::weights(v.w[s], X::zero(v.sz[s / STEPS]));
#pragma unroll
                for (int p = 0; p < X::kParts; ++p) acc = X::mfma(op[p], q, acc);
            } else {
                sum = X::mfma(op[0], X::ones(), sum);
                acc = X::mfma(op[0], X::codes(v.w[s]), acc);
            }
            if ((s + 1) % STEPS == 0) {       // the group's end
                total = add_group<XT>(xs[s / STEPS], X::kParts > 1 ? v.sz[s / STEPS] & ~15u : v.sz[s / STEPS], acc, sum, total);
                acc = sum = typename X::Acc{};
                // (a second group's sums at the same time would take more registers)
                asm volatile("" : "+v"(total));
            }
        }
    };
    const int whole = a.C / kQ4Block;         // (the last block may be a part of one)
    Weights v, next;
    int b = wave;
    if (b < whole) {
        load_weights(b, v);
#pragma unroll
        for (int s = 0; s < 4; ++s) load_x(b, s, std::false_type{});
        for (; b + W < whole; b += W) {
            block(b, b + W, v, next, std::true_type{});
            v = next;
        }
        block(b, 0, v, next, std::false_type{});
        b += W;
    }
    if (b < a.blocks) {
        load_weights(b, v);
#pragma unroll
        for (int s = 0; s < 4; ++s) load_x(b, s, std::true_type{});
        block(b, 0, v, next, std::false_type{});
    }
    __shared__ q4f4 sums[W][64];
    sums[wave][lane] = total;
    __syncthreads();
    store_sums<XT, 1, W>(a, reinterpret_cast<const float *>(sums), tile);
}

// Few rows of x: all of them, each of their parts, are the 16 rows of one operand, so that a row of x costs a third of a product and not three.  The
// operand is made once for a work-group: `cols` columns at a time lie in LDS, rows 16 bytes more than that apart (a multiple of 256 bytes:
// the 16 rows of a chunk are in all banks).  16 rows of weights, W waves that divide the blocks; their sums are added as rows_kernel adds them.
template <int XT> using RowOp = XOp<XT == FSCNN_F32 ? FSCNN_BF16 : XT>;
template <int XT, int W, int STEPS> __global__ void __launch_bounds__(W * 64) staged_kernel(const Q4Args a, int cols)
{
    using X = XOp<XT>;
    using R = RowOp<XT>;
    constexpr int kGroups = 4 / STEPS, kBytes = XT == FSCNN_I8 ? 1 : 2, kParts = X::kParts;
    extern __shared__ __align__(256) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col16 = lane & 15, quarter = lane >> 4, tile = blockIdx.x, pitch = cols * kBytes + 16;
    const u4v *codes = a.codes + (long long)tile * a.blocks * 64 + lane;
    const uint32_t *scales = a.scales + (long long)tile * a.blocks * (kGroups * 16) + col16;
    struct Weights {
        u4v w;
        uint32_t sz[kGroups];
    };
    auto load_weights = [&](int b, Weights &v) {
        b = b < a.blocks ? b : a.blocks - 1;
        v.w = codes[(long long)b * 64];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) v.sz[g] = scales[((long long)b * kGroups + g) * 16];
    };
    const int rows = a.M * kParts;            // at most 16; the operand's others repeat the last one
    const char *mine = lds + (col16 < rows ? col16 : rows - 1) * pitch + quarter * (8 * kBytes);
    q4f4 total = {};
    // Codes are two blocks ahead, in three slots.  (Every step loads, past the last block that one again: the waits count loads.)
    Weights v[3];
    int b = wave;
    for (int c0 = 0; c0 < a.blocks * kQ4Block; c0 += cols) {
        load_weights(b, v[0]);
        load_weights(b + W, v[1]);
        if (c0) __syncthreads();
        const int end = a.blocks * kQ4Block - c0 < cols ? a.blocks * kQ4Block - c0 : cols;
        const int inside = a.C - c0 < end ? (a.C - c0) & ~7 : end;   // columns in whole chunks of 8; then those that end in C, and zeros
        auto put = [&](int m, int c, const typename X::Raw &raw) {
            typename X::Op op[kParts];
            X::parts(raw, op);
#pragma unroll
            for (int p = 0; p < kParts; ++p) *reinterpret_cast<typename X::Op *>(lds + (m * kParts + p) * pitch + c * kBytes) = op[p];
        };
        const int chunks = inside / 8, each = chunks * a.M;
        for (int i = threadIdx.x; i < each; i += W * 64 * 4) {       // four loads on their way
            typename X::Raw raw[4];
            int m[4], c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = i + j * (W * 64) < each ? i + j * (W * 64) : i;
                m[j] = at / chunks;
                c[j] = (at - m[j] * chunks) * 8;
                raw[j] = load_columns<XT, false>(a.x + m[j] * a.ldx, c0 + c[j], a.C);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j == 0 || i + j * (W * 64) < each) put(m[j], c[j], raw[j]);
        }
        for (int i = threadIdx.x; i < (end - inside) / 8 * a.M; i += W * 64) {
            const int m = i % a.M, c = inside + i / a.M * 8;
            put(m, c, load_columns<XT, true>(a.x + m * a.ldx, c0 + c, a.C));
        }
        __syncthreads();
        auto block = [&](const Weights &now, Weights &after) {
            load_weights(b + 2 * W, after);
            q4f4 xs[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) xs[g] = row_scales<XT>(a, 4 * quarter, b * kGroups + g);
            const char *from = mine + (b * kQ4Block - c0) * kBytes;
            typename R::Op op[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) op[s] = *reinterpret_cast<const typename R::Op *>(from + s * (32 * kBytes));
            typename R::Acc acc = {}, sum = {};
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                sum = R::mfma(op[s], R::ones(), sum);
                acc = R::mfma(op[s], R::codes(now.w[s]), acc);
                if ((s + 1) % STEPS == 0) {
                    total = add_group<XT>(xs[s / STEPS], now.sz[s / STEPS], acc, sum, total);
                    acc = sum = typename R::Acc{};
                }
            }
            b += W;
            return b * kQ4Block < c0 + end;
        };
        if (b * kQ4Block < c0 + end)
            while (block(v[0], v[2]) && block(v[1], v[0]) && block(v[2], v[1])) {}
    }
    __syncthreads();
    q4f4 *const sums = reinterpret_cast<q4f4 *>(lds);   // [W][64 lanes]
    sums[wave * 64 + lane] = total;
    __syncthreads();
    store_sums<XT, kParts, W>(a, reinterpret_cast<const float *>(sums), tile);
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

// STEPS: of 32 columns a group.  DMA: rows of x are 16 bytes aligned, offsets in a tile below 2^31.  GS: x (8 bits) has a scale for each group.
// x in LDS: rows of kChunks 16-byte chunks a part, chunk c of row r at c ^ f(r), so that the 16 lanes that read a chunk of adjacent rows find
// it in all banks.
template <int XT, int MT, int WN, int WK, int STEPS, bool DMA, bool GS>
__global__ void __launch_bounds__(WN * WK * 64, XT == FSCNN_F32 ? 1 : 2) tile_kernel(const Q4Args a)
{
    using X = XOp<XT>;
    using T = Tile<XT>;
    constexpr bool kInt = XT == FSCNN_I8;
    constexpr int kRows = 32 * MT, kSet = WN * 64, kParts = X::kParts, kCh = T::kChunks, kGroups = 4 / STEPS;
    constexpr int kAnyAlu = 6;                            // of sched_barrier: vector and scalar arithmetic may pass
    constexpr int kSteps = kInt ? 4 : 8, kStepsOfGroup = kSteps / kGroups;   // products of a block, of a group
    constexpr int kPer = kRows * kCh / kSet;              // chunks a thread brings
    constexpr int kBuf = kRows * kCh * kParts;            // chunks of a buffer
    constexpr int kScales = GS ? 2 * kGroups * kRows / 4 : 0;
    constexpr int kSums = (WK - 1) * kSet * MT * 4;  // in 16 bytes, at the end
    constexpr int kChunksOfSet = 2 * kBuf + kScales;
    static_assert(kPer * kSet == kRows * kCh, "a whole number of chunks a thread");
    static_assert(!GS || kRows <= kSet, "a thread a row");
    constexpr int kPitch = 32 * WN + 8, kArea = 32 * kPitch;   // of outputs, in floats: rows 4 apart half of the banks apart
    constexpr int kNeed = kSums * 4 > 2 * kArea ? kSums : (2 * kArea + 3) / 4;
    __shared__ u4v lds[kChunksOfSet * WK > kNeed ? kChunksOfSet * WK : kNeed];
    __shared__ int odd;                       // some sums are not finite
    if (threadIdx.x == 0) odd = 0;            // (there is a barrier before it is read or set)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wk = wave / WN, in_set = wave % WN, half = lane >> 5;
    // panels of 8 tiles of x: work-groups that run together share both operands
    const int lid = xcd_neighbours(blockIdx.x, a.mt * a.nt), panel = lid / (8 * a.nt), in = lid % (8 * a.nt);
    const int tall = a.mt - panel * 8 < 8 ? a.mt - panel * 8 : 8;
    const int m0 = (panel * 8 + in % tall) * kRows, n0 = in / tall * (32 * WN) + in_set * 32;
    auto swizzle = [](int r) { return kCh == 16 ? r & 15 : r >> 1 & 7; };

    // codes and scales: a base for the wave, which moves from block to block, and what a lane is away from it
    const int first = (n0 >> 4) < a.tiles ? n0 >> 4 : a.tiles - 1;
    // (this work-group's blocks: b0 up to b1)
    const int b0 = (int)((long long)a.blocks * blockIdx.y / gridDim.y), b1 = (int)((long long)a.blocks * (blockIdx.y + 1) / gridDim.y);
    const char *codes = reinterpret_cast<const char *>(a.codes) + ((long long)first * a.blocks + b0 + wk) * 1024;
    const char *scales = reinterpret_cast<const char *>(a.scales) + ((long long)first * a.blocks + b0 + wk) * (kGroups * 64);
    // (tiles past the last one repeat it: their outputs are not stored)
    const int behind = (n0 + (lane & 31)) >> 4 < a.tiles ? ((n0 + (lane & 31)) >> 4) - first : a.tiles - 1 - first;
    const uint32_t code_at = behind * a.blocks * 1024 + ((lane & 15) + 32 * half) * 16, scale_at = behind * a.blocks * (kGroups * 64) + (lane & 15) * 4;
    const int live = a.M - m0 < kRows ? a.M - m0 : kRows;
    const char *x = a.x + m0 * a.ldx;
    u4v *const set = lds + wk * kChunksOfSet;
    float *const set_scales = reinterpret_cast<float *>(set + 2 * kBuf);
    const int slot = in_set * kPer * 64 + lane;           // of the thread's first chunk; the others follow 64 apart
    int from[DMA ? kPer : 1];
    if constexpr (DMA) {
        // (rows that are not there are out of the descriptor's range and read as zeros)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int at = slot + i * 64, r = at / kCh, c = at % kCh ^ swizzle(r);
            from[i] = r < live ? (int)(r * a.ldx) + c * 16 : (int)0x80000000;
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u4v *)set + in_set * kPer * 1024;
    // a block of the rows of x by way of registers (rows that are not there repeat the last one: their outputs are not stored)
    struct Chunk { typename X::Raw r[kInt ? 2 : 1]; };
    auto load_chunk = [&](int b, int i, auto tail) {
        constexpr bool kTail = decltype(tail)::value;
        const int at = slot + i * 64, r = at / kCh, c = at % kCh ^ swizzle(r), col = b * kQ4Block + c * T::kChunk;
        const char *row = x + (r < live ? r : live - 1) * a.ldx;
        Chunk v;
        v.r[0] = load_columns<XT, kTail>(row, col, a.C);
        if constexpr (kInt) v.r[1] = load_columns<XT, kTail>(row, col + 8, a.C);
        return v;
    };
    auto put_chunk = [&](int buf, int i, const Chunk &v) {
        u4v *to = set + buf * kBuf + slot + i * 64;
        if constexpr (kInt) *to = u4v{v.r[0][0], v.r[0][1], v.r[1][0], v.r[1][1]};
        else {
            u4v part[kParts];
            X::parts(v.r[0], part);
#pragma unroll
            for (int p = 0; p < kParts; ++p) to[p * kRows * kCh] = part[p];
        }
    };
    Chunk raw[DMA ? 1 : kPer];
    float xs_next[GS ? kGroups : 1];
    struct Weights {
        u4v w[2];
        uint32_t sz[kGroups];
    } now, next;
    auto load_weights = [&](Weights &v) {
#pragma unroll
        for (int e = 0; e < 2; ++e) v.w[e] = *reinterpret_cast<const u4v *>(codes + (code_at + 256 * e));
#pragma unroll
        for (int g = 0; g < kGroups; ++g) v.sz[g] = *reinterpret_cast<const uint32_t *>(scales + (scale_at + 64 * g));
        codes += WK * 1024;
        scales += WK * (kGroups * 64);
    };
    // brings block b on its way to buffer `buf`; what goes through registers is put there by commit()
    auto fetch = [&](int b, int buf) {
        if constexpr (DMA) {
            if ((b + 1) * kQ4Block <= a.C) {
                const unsigned long long xa = (unsigned long long)x + (unsigned)b * (kCh * 16);
                const int4v rsrc = {(int)(uint32_t)xa, (int)(uint32_t)(xa >> 32), (int)((live - 1) * a.ldx + a.C * (16 / T::kChunk)) - b * (kCh * 16), 0x00020000};
#pragma unroll
                for (int i = 0; i < kPer; ++i) lds_dma_dwordx4(rsrc, lds0 + buf * (kBuf * 16) + i * 1024, from[i]);
            } else {
#pragma unroll 1
                for (int i = 0; i < kPer; ++i) put_chunk(buf, i, load_chunk(b, i, std::true_type{}));
            }
        } else {
            if ((b + 1) * kQ4Block <= a.C) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) raw[i] = load_chunk(b, i, std::false_type{});
            } else {
#pragma unroll
                for (int i = 0; i < kPer; ++i) raw[i] = load_chunk(b, i, std::true_type{});
            }
        }
        if constexpr (GS) {
            const int r = in_set * 64 + lane;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int group = b * kGroups + g;
                xs_next[g] = r < live && group < a.x_cols ? a.x_scale[(long long)(m0 + r) * a.x_cols + group] : 0.0f;
            }
        }
    };
    auto commit = [&](int buf) {
        if constexpr (!DMA) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) put_chunk(buf, i, raw[i]);
        }
        if constexpr (GS) {
            const int r = in_set * 64 + lane;
            if (r < kRows)
#pragma unroll
                for (int g = 0; g < kGroups; ++g) set_scales[(buf * kGroups + g) * kRows + r] = xs_next[g];
        }
    };
    q4f16 total[MT] = {};
    const int row0 = lane & 31;
    const int turns = (b1 - b0 + WK - 1) / WK;

    if (b0 + wk < b1) {
        load_weights(next);
        fetch(b0 + wk, 0);
        commit(0);
    }
    for (int turn = 0; turn < turns; ++turn) {
        const int b = b0 + turn * WK + wk, buf = turn & 1;
        wait_vmcnt<0>();                      // the block is in LDS, its codes in registers
        now = next;
        // step st of the block: the weights' operand
        auto decode = [&](int st) {
            const typename X::Zero z = X::zero(now.sz[st / kStepsOfGroup]);
            if constexpr (kInt) {
                const u2v w0 = X::weights(now.w[0][st], z), w1 = X::weights(now.w[1][st], z);
                return u4v{w0[0], w0[1], w1[0], w1[1]};
            } else {
                return X::weights(now.w[st & 1][st >> 1], z);
            }
        };
        const u4v *from_lds = set + buf * kBuf + row0 * kCh;
        // part p of the rows of x at that step
        auto read = [&](int st, int p, u4v *op) {
            const int chunk = kInt ? 2 * st + half : 4 * (st >> 1) + 2 * half + (st & 1);
#pragma unroll
            for (int u = 0; u < MT; ++u) op[u] = from_lds[p * kRows * kCh + u * 32 * kCh + (chunk ^ swizzle(row0))];
        };
        u4v op[2][MT], w[2];
        w[0] = decode(0);
        lds_only_barrier();
        if (b >= b1) continue;                // (the last turn of some sets)
        const bool more = b + WK < b1;
        if (more) {
            fetch(b + WK, buf ^ 1);
            load_weights(next);
        }
        read(0, 0, op[0]);
        typename T::Acc acc[MT] = {};
        // one part of one step after the other; what the next one needs is read and made beside the products
#pragma unroll
        for (int i = 0; i < kSteps * kParts; ++i) {
            const int st = i / kParts, p = i % kParts;
            const bool last = i + 1 == kSteps * kParts;
            if (!last) read((i + 1) / kParts, (i + 1) % kParts, op[(i + 1) & 1]);
            __builtin_amdgcn_sched_barrier(kAnyAlu);   // (else the reads sink to their uses, to save registers)
#pragma unroll
            for (int u = 0; u < MT; ++u) acc[u] = T::mfma(op[i & 1][u], w[st & 1], acc[u]);
            if (!last && p == kParts - 1) w[(st + 1) & 1] = decode(st + 1);
            __builtin_amdgcn_sched_barrier(kAnyAlu);
            if (p != kParts - 1 || (st + 1) % kStepsOfGroup) continue;
            // the group's end
            const int g = st / kStepsOfGroup;
#pragma unroll
            for (int u = 0; u < MT; ++u) {
                q4f4 xs[4];
                if constexpr (GS) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        xs[j] = *reinterpret_cast<const q4f4 *>(set_scales + (buf * kGroups + g) * kRows + u * 32 + 8 * j + 4 * half);
                }
                const float f = __builtin_bit_cast(float, now.sz[g] & ~15u);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    float v = (float)acc[u][j];
                    if constexpr (GS) v *= xs[j >> 2][j & 3];
                    total[u][j] = __builtin_fmaf(f, v, total[u][j]);
                }
                acc[u] = typename T::Acc{};
            }
            // (a second group's sums at the same time would not fit the registers)
#pragma unroll
            for (int u = 0; u < MT; ++u) asm volatile("" : "+v"(total[u]));
        }
        if (more) commit(buf ^ 1);
    }
    if constexpr (WK > 1) {                   // the sets' sums, in their order
        __syncthreads();
        q4f4 *const out = reinterpret_cast<q4f4 *>(lds);
        const int mine = in_set * 64 + lane;
        if (wk > 0)
#pragma unroll
            for (int e = 0; e < MT * 4; ++e) {
                const q4f16 &f = total[e / 4];
                out[((wk - 1) * MT * 4 + e) * kSet + mine] = q4f4{f[e % 4 * 4], f[e % 4 * 4 + 1], f[e % 4 * 4 + 2], f[e % 4 * 4 + 3]};
            }
        __syncthreads();
        if (wk == 0)
#pragma unroll
            for (int e = 0; e < MT * 4; ++e)
#pragma unroll
                for (int k = 0; k < WK - 1; ++k) {
                    const q4f4 f = out[(k * MT * 4 + e) * kSet + mine];
#pragma unroll
                    for (int i = 0; i < 4; ++i) total[e / 4][e % 4 * 4 + i] += f[i];
                }
    }
    if (gridDim.y > 1) {
        const int k = n0 + (lane & 31);
        if (wk == 0 && k < a.K)
#pragma unroll
            for (int u = 0; u < MT; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int m = m0 + u * 32 + 8 * (i >> 2) + 4 * half + (i & 3);
                    if (m >= a.M) continue;
                    float v = total[u][i];
                    if constexpr (kInt && !GS) v *= a.x_scale[m];
                    a.sums[((long long)blockIdx.y * a.M + m) * (a.tiles * 16LL) + k] = v;
                }
        return;
    }
    // 32 rows after the other by way of LDS, so that a lane stores 16 bytes of a row of y
    float *const area = reinterpret_cast<float *>(lds);
    const int cols0 = n0 - in_set * 32;
    const auto put = [&](int u) {
        float all[4] = {};
        if (kInt && !GS && threadIdx.x < 32 && m0 + u * 32 + (int)threadIdx.x < a.M) all[0] = fabsf(a.x_scale[m0 + u * 32 + threadIdx.x]);
        if (wk == 0)
#pragma unroll
            for (int i = 0; i < 16; ++i) all[i & 3] += fabsf(total[u][i]);
        if (!finite(all[0] + all[1] + (all[2] + all[3]))) odd = 1;   // one of them is not, or (no harm) their sum alone
        if (wk == 0)
#pragma unroll
            for (int i = 0; i < 16; ++i) area[(u & 1) * kArea + (8 * (i >> 2) + 4 * half + (i & 3)) * kPitch + in_set * 32 + (lane & 31)] = total[u][i];
    };
    const auto store = [&](int u, auto type) {
        using E = typename Elem<decltype(type)::value>::type;
        constexpr int kV = 16 / (int)sizeof(E), kRow = 32 * WN / kV;   // outputs of a thread; threads of a row
        for (int at = threadIdx.x; at < 32 * kRow; at += kSet * WK) {
            const int r = at / kRow, c = at % kRow * kV, m = m0 + u * 32 + r, k = cols0 + c;
            if (m >= a.M || k >= a.K) continue;
            const float *f = area + (u & 1) * kArea + r * kPitch + c;
            const float xs = kInt && !GS ? a.x_scale[m] : 1.0f;
            E e[kV];
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                float v = f[j];
                if (kInt && !GS) v *= xs;
                e[j] = (E)activated(v + (a.bias && k + j < a.K ? a.bias[k + j] : 0.0f), a.act);
            }
            E *y = static_cast<E *>(a.y) + (m * a.ldy + k);
            if (k + kV <= a.K) __builtin_memcpy(y, e, 16);
            else
#pragma unroll
                for (int j = 0; j < kV; ++j)
                    if (k + j < a.K) y[j] = e[j];
        }
    };
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MT; ++u) {            // (two areas: a barrier each)
        put(u);
        __syncthreads();
        if (a.y_type == FSCNN_F32) store(u, std::integral_constant<int, FSCNN_F32>{});
        else if (a.y_type == FSCNN_F16) store(u, std::integral_constant<int, FSCNN_F16>{});
        else store(u, std::integral_constant<int, FSCNN_BF16>{});
    }
    if (__builtin_expect(odd != 0, 0)) {      // (the same for all: written before the last barrier)
        __syncthreads();                      // what has been stored is in its place
        if (wk > 0) return;
        const int k = n0 + (lane & 31);
        unsigned long long bad = 0;           // which of the lane's
#pragma unroll
        for (int u = 0; u < MT; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) bad |= (unsigned long long)!finite(total[u][i]) << (u * 16 + i);
#pragma unroll 1
        for (int e = 0; e < MT * 16; ++e) {
            const int m = m0 + (e >> 4) * 32 + 8 * ((e & 15) >> 2) + (e & 3), mine = m + 4 * half;
            bool again = bad >> e & 1;
            if (kInt && !GS && mine < a.M) again |= !finite(a.x_scale[mine]);
            const unsigned long long lanes = __ballot(again && mine < a.M && k < a.K);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const uint32_t of_row = (uint32_t)(lanes >> (32 * h));
                if (!of_row) continue;
                const int r = m + 4 * h;
                const long long tile = n0 >> 4;
                const float v = row_again(of_row, a.x + r * a.ldx, XT, kInt ? a.x_scale + (long long)r * a.x_cols : nullptr, a.x_cols,
                                          reinterpret_cast<const uint32_t *>(a.codes) + tile * a.blocks * 256, a.scales + tile * a.blocks * (kGroups * 16),
                                          a.blocks, a.C, 32 * STEPS);
                if (half == h && (of_row >> (lane & 31) & 1)) store_output(a, r, k, v, a.bias ? a.bias[k] : 0.0f);
            }
        }
    }
}

template <int XT, int W> hipError_t launch_rows(const Q4Args &a, hipStream_t st)
{
    if (a.M > 16 || a.tiles * (W * 64LL) > 0xffffffffLL) return hipErrorInvalidValue;
    const dim3 grid(a.tiles), block(W * 64);
    if (a.steps == 1) hipLaunchKernelGGL((rows_kernel<XT, W, 1>), grid, block, 0, st, a);
    else if (a.steps == 2) hipLaunchKernelGGL((rows_kernel<XT, W, 2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rows_kernel<XT, W, 4>), grid, block, 0, st, a);
    return hipGetLastError();
}

constexpr int kMostStaged = 144 << 10;       // bytes of LDS

// (named by its template: kernels of one signature would share the static of a function that is handed one)
template <int XT, int W, int STEPS> hipError_t launch_staged_steps(const Q4Args &a, int cols, int bytes, hipStream_t st)
{
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(&staged_kernel<XT, W, STEPS>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, kMostStaged);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL((staged_kernel<XT, W, STEPS>), dim3(a.tiles), dim3(W * 64), bytes, st, a, cols);
    return hipGetLastError();
}

template <int XT, int W> hipError_t launch_staged(const Q4Args &a, hipStream_t st)
{
    constexpr int kBytes = XT == FSCNN_I8 ? 1 : 2, kMost = kMostStaged, kTurn = W * kQ4Block;
    const int rows = a.M * XOp<XT>::kParts;
    if (rows > 16 || a.tiles * (W * 64LL) > 0xffffffffLL) return hipErrorInvalidValue;
    // as many columns in LDS as leave room for a second work-group where there is one for a CU
    const int room = a.tiles > 256 ? kMost / 2 : kMost, fit = (room / rows - 16) / kBytes / kTurn * kTurn, all = a.blocks * kQ4Block;
    const int cols = all < fit ? all : fit, staged = rows * (cols * kBytes + 16), sums = W * 1024, bytes = staged > sums ? staged : sums;
    static_assert(16 * (kTurn * kBytes + 16) <= kMost / 2, "a turn of 16 rows fits");
    if (a.steps == 1) return launch_staged_steps<XT, W, 1>(a, cols, bytes, st);
    if (a.steps == 2) return launch_staged_steps<XT, W, 2>(a, cols, bytes, st);
    return launch_staged_steps<XT, W, 4>(a, cols, bytes, st);
}

template <int XT, int MT, int WN, int WK, bool DMA, bool GS> hipError_t launch_tiles(Q4Args a, int parts, hipStream_t st)
{
    constexpr int rows = 32 * MT, threads = WN * WK * 64;
    const long long mt = ((long long)a.M + rows - 1) / rows, nt = (a.K + 32LL * WN - 1) / (32 * WN);
    if (mt * nt * threads > 0xffffffffLL || 8 * nt > 0x7fffffffLL) return hipErrorInvalidValue;
    a.mt = (int)mt;
    a.nt = (int)nt;
    const dim3 grid((unsigned)(mt * nt), parts), block(threads);
    if (a.steps == 1) hipLaunchKernelGGL((tile_kernel<XT, MT, WN, WK, 1, DMA, GS>), grid, block, 0, st, a);
    else if (a.steps == 2) hipLaunchKernelGGL((tile_kernel<XT, MT, WN, WK, 2, DMA, GS>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((tile_kernel<XT, MT, WN, WK, 4, DMA, GS>), grid, block, 0, st, a);
    return hipGetLastError();
}

// x may go to LDS without registers: 16-byte loads, offsets of a tile's rows below 2^31
inline bool dma_serves(const Q4Args &a, int rows) { return !(((uintptr_t)a.x | (uintptr_t)a.ldx) & 15) && a.ldx * rows < 0x7fff0000LL; }

template <int XT, int MT, int WN, int WK, bool DMA> hipError_t launch_tiles(const Q4Args &a, int parts, hipStream_t st)
{
    if constexpr (XT == FSCNN_I8)
        if (a.x_cols > 1) return launch_tiles<XT, MT, WN, WK, DMA, true>(a, parts, st);
    return launch_tiles<XT, MT, WN, WK, DMA, false>(a, parts, st);
}

template <int XT> hipError_t launch_narrow(const Q4Args &a, int parts, hipStream_t st)
{
    constexpr bool kInt = XT == FSCNN_I8;
    const bool dma = dma_serves(a, 128);
    const Q4Choice c = narrow_choice(kInt, a.M, a.K, a.blocks, parts, dma);
    switch (c.kernel) {
        case Q4Choice::kRows: return c.waves == 16 ? launch_rows<XT, 16>(a, st) : launch_rows<XT, 8>(a, st);
        case Q4Choice::kStaged: return c.waves == 16 ? launch_staged<XT, 16>(a, st) : launch_staged<XT, 8>(a, st);
        default: break;
    }
    switch (c.shape) {
        case 0: return dma ? launch_tiles<XT, 1, 1, 8, true>(a, parts, st) : launch_tiles<XT, 1, 1, 8, false>(a, parts, st);
        case 1: return dma ? launch_tiles<XT, 1, 2, 4, true>(a, parts, st) : launch_tiles<XT, 1, 2, 4, false>(a, parts, st);
        case 2: return dma ? launch_tiles<XT, 2, 4, 2, true>(a, parts, st) : launch_tiles<XT, 2, 4, 2, false>(a, parts, st);
        case 3: return dma ? launch_tiles<XT, 2, 4, 1, true>(a, parts, st) : launch_tiles<XT, 2, 4, 1, false>(a, parts, st);
        case 5: if constexpr (!kInt) return launch_tiles<XT, 2, 2, 4, true>(a, parts, st);
        case 6: if constexpr (!kInt) return launch_tiles<XT, 3, 4, 2, true>(a, parts, st);
        default: return launch_tiles<XT, 4, 4, 1, true>(a, parts, st);
    }
}

}  // namespace

// parts: work-groups that divide the columns: q4_parts(), or 1 where a call has no room for their sums
template <int XT> hipError_t launch_q4_type(const Q4Args &a, int parts, hipStream_t st);
template <> hipError_t launch_q4_type<FSCNN_F32>(const Q4Args &a, int parts, hipStream_t st);
template <> hipError_t launch_q4_type<FSCNN_F16>(const Q4Args &a, int parts, hipStream_t st);
template <> hipError_t launch_q4_type<FSCNN_BF16>(const Q4Args &a, int parts, hipStream_t st);
template <> hipError_t launch_q4_type<FSCNN_I8>(const Q4Args &a, int parts, hipStream_t st);

}  // namespace fscnn
