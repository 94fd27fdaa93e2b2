// The kernels of y = act(x W^T + b) with 4-bit weights (internal.h has their order, q4_tile.h the operands), for one type of x a translation unit.
//
// rows_kernel (few rows of x): a work-group of W waves owns up to 16 MT rows of x and 16 NT rows of weights.  Both go straight from memory into the
// matrix cores' operands (16 bytes a lane hold the codes of 16 rows x 128 columns), the next block's loads on their way while one is computed.
// The waves divide the blocks of 128 columns, each keeps fp32 sums of its own, which are added at the end through LDS in the order of the
// waves.  Several work-groups may divide the blocks once more; then they leave their sums for join_kernel (q4_linear.hip).
//
// tile_kernel (many rows of x): WM x WN waves own 32 MT WM rows of x and 32 NT WN rows of weights.  A block of 128 columns of the rows
// of x is in LDS while the next one is on its way there (16 bytes a lane, without registers where x is aligned); codes come from memory into
// registers a block ahead.  What a wave does per block: 8 MT NT products of 32 x 32 x 16, codes to operands, and a multiply-add per output and
// group, since a group's sum is multiplied by its scale in fp32.  WK such sets of waves may divide the blocks; their sums are added through LDS.
#pragma once
#include <type_traits>

#include "internal.h"
#include "lds_dma.h"
#include "q4_tile.h"

namespace fscnn {

struct Q4Args {
    const u4v *codes;
    const uint32_t *scales;
    const char *x;
    const float *x_scale, *bias;
    void *y;
    float *sums;                              // rows_kernel: [gridDim.z][M][16 tiles], where the blocks are divided
    long long ldx, ldy;                       // ldx in bytes
    int K, C, M, blocks, tiles, steps, y_type, x_cols, act;   // steps: of 32 columns a group
    int mt, nt;                               // tile_kernel: tiles of the launch
};

namespace {

__device__ inline void store_output(const Q4Args &a, int m, int k, float v, float bias)
{
    store_float(a.y, m * a.ldy + k, a.y_type, act_apply(v + bias, a.act));
}

template <int XT, int NT, int MT, int W, int STEPS> __global__ void __launch_bounds__(W * 64) rows_kernel(const Q4Args a)
{
    using X = XOp<XT>;
    constexpr bool kInt = XT == FSCNN_I8;
    constexpr int kGroups = 4 / STEPS;        // of a block
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col16 = lane & 15, quarter = lane >> 4;
    const int tile0 = blockIdx.x * NT, m0 = blockIdx.y * (16 * MT);
    const u4v *codes[NT];
    const uint32_t *scales[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {            // (tiles past the last one repeat it, and so do rows of x: their outputs are not stored)
        const long long tile = tile0 + t < a.tiles ? tile0 + t : a.tiles - 1;
        codes[t] = a.codes + tile * a.blocks * 64 + lane;
        scales[t] = a.scales + tile * a.blocks * (kGroups * 16) + col16;
    }
    const char *rows[MT];
#pragma unroll
    for (int u = 0; u < MT; ++u) {
        const int m = m0 + 16 * u + col16;
        rows[u] = a.x + (m < a.M ? m : a.M - 1) * a.ldx;
    }
    q4f4 total[NT][MT] = {};
    struct Weights {
        u4v w[NT];
        uint32_t sz[NT][kGroups];
    };
    auto load_weights = [&](int b, Weights &v) {
#pragma unroll
        for (int t = 0; t < NT; ++t) v.w[t] = codes[t][(long long)b * 64];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int g = 0; g < kGroups; ++g) v.sz[t][g] = scales[t][((long long)b * kGroups + g) * 16];
    };
    typename X::Raw raw[4][MT];
    auto load_x = [&](int b, int s, auto tail) {
#pragma unroll
        for (int u = 0; u < MT; ++u) raw[s][u] = load_columns<XT, decltype(tail)::value>(rows[u], b * kQ4Block + s * 32 + quarter * 8, a.C);
    };
    // block b; its loads are done or on their way, those of block `then` are issued here (then < 0: none)
    auto block = [&](int b, int then, const Weights &v, Weights &next) {
        if (then >= 0) load_weights(then, next);
        typename X::Acc acc[NT][MT] = {}, sum[MT] = {};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            typename X::Op op[MT][X::kParts];
#pragma unroll
            for (int u = 0; u < MT; ++u) X::parts(raw[s][u], op[u]);
            if (then >= 0) load_x(then, s, std::false_type{});
#pragma unroll
            for (int u = 0; u < MT; ++u)
#pragma unroll
                for (int p = 0; p < X::kParts; ++p) sum[u] = X::mfma(op[u][p], X::ones(), sum[u]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const typename X::Op q = X::codes(v.w[t][s]);
#pragma unroll
                for (int u = 0; u < MT; ++u)
#pragma unroll
                    for (int p = 0; p < X::kParts; ++p) acc[t][u] = X::mfma(op[u][p], q, acc[t][u]);
            }
            if ((s + 1) % STEPS == 0) {       // the group's end
                const int g = b * kGroups + s / STEPS;
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
                    const uint32_t sz = v.sz[t][s / STEPS];
                    const float f = __builtin_bit_cast(float, sz & ~15u), z = -(float)(sz & 15);
#pragma unroll
                    for (int u = 0; u < MT; ++u) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float w;
                            if constexpr (kInt) w = (float)(acc[t][u][i] - (int)(sz & 15) * sum[u][i]) * xs[u][i];
                            else w = __builtin_fmaf(z, sum[u][i], acc[t][u][i]);
                            total[t][u][i] = __builtin_fmaf(f, w, total[t][u][i]);
                        }
                        acc[t][u] = {};
                    }
                }
#pragma unroll
                for (int u = 0; u < MT; ++u) sum[u] = {};
                // (a second group's sums at the same time would not fit the registers)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int u = 0; u < MT; ++u) asm volatile("" : "+v"(total[t][u]));
            }
        }
    };
    // this work-group's blocks: b0 up to b1, the last one of all perhaps a part of one
    const int b0 = (int)((long long)a.blocks * blockIdx.z / gridDim.z), b1 = (int)((long long)a.blocks * (blockIdx.z + 1) / gridDim.z);
    const int whole = a.C / kQ4Block < b1 ? a.C / kQ4Block : b1;
    Weights v[2];
    int b = b0 + wave;
    if (b < whole) {
        load_weights(b, v[0]);
#pragma unroll
        for (int s = 0; s < 4; ++s) load_x(b, s, std::false_type{});
        for (; b + 2 * W < whole; b += 2 * W) {
            block(b, b + W, v[0], v[1]);
            block(b + W, b + 2 * W, v[1], v[0]);
        }
        if (b + W < whole) {
            block(b, b + W, v[0], v[1]);
            block(b + W, -1, v[1], v[0]);
            b += 2 * W;
        } else {
            block(b, -1, v[0], v[1]);
            b += W;
        }
    }
    if (b < b1) {
        load_weights(b, v[0]);
#pragma unroll
        for (int s = 0; s < 4; ++s) load_x(b, s, std::true_type{});
        block(b, -1, v[0], v[1]);
    }

    __shared__ q4f4 sums[W][NT * MT][64];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int u = 0; u < MT; ++u) sums[wave][t * MT + u][lane] = total[t][u];
    __syncthreads();
    for (int e = wave; e < NT * MT; e += W) {
        q4f4 f = sums[0][e][lane];
#pragma unroll
        for (int i = 1; i < W; ++i) f += sums[i][e][lane];
        const int m = m0 + e % MT * 16 + 4 * quarter, k = (tile0 + e / MT) * 16 + col16;
        if (gridDim.z > 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (m + i < a.M && k < a.K) a.sums[((long long)blockIdx.z * a.M + m + i) * (a.tiles * 16LL) + k] = f[i];
            continue;
        }
        if (k >= a.K) continue;
        const float bias = a.bias ? a.bias[k] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (m + i < a.M) store_output(a, m + i, k, kInt && a.x_cols == 1 ? f[i] * a.x_scale[m + i] : f[i], bias);
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

// STEPS: of 32 columns a group.  DMA: rows of x are 16 bytes aligned, offsets in a tile below 2^31.  GS: x (8 bits) has a scale for each group.
// x in LDS: rows of kChunks 16-byte chunks a part, chunk c of row r at c ^ f(r), so that the 16 lanes that read a chunk of adjacent rows find
// it in all banks.
template <int XT, int MT, int NT, int WM, int WN, int WK, int STEPS, bool DMA, bool GS>
__global__ void __launch_bounds__(WM * WN * WK * 64, XT == FSCNN_F32 ? 1 : 2) tile_kernel(const Q4Args a)
{
    using X = XOp<XT>;
    using T = Tile<XT>;
    constexpr bool kInt = XT == FSCNN_I8;
    constexpr int kRows = 32 * MT * WM, kSet = WM * WN * 64, kParts = X::kParts, kCh = T::kChunks, kGroups = 4 / STEPS;
    constexpr int kAnyAlu = 6;                            // of sched_barrier: vector and scalar arithmetic may pass
    constexpr int kSteps = kInt ? 4 : 8, kStepsOfGroup = kSteps / kGroups;   // products of a block, of a group
    constexpr int kPer = kRows * kCh / kSet;              // chunks a thread brings
    constexpr int kBuf = kRows * kCh * kParts;            // chunks of a buffer
    constexpr int kScales = GS ? 2 * kGroups * kRows / 4 : 0;
    constexpr int kSums = (WK - 1) * kSet * MT * NT * 4;  // in 16 bytes, at the end
    constexpr int kChunksOfSet = 2 * kBuf + kScales;
    static_assert(kPer * kSet == kRows * kCh, "a whole number of chunks a thread");
    static_assert(!GS || kRows <= kSet, "a thread a row");
    constexpr int kPitch = 32 * NT * WN + 8, kArea = 32 * WM * kPitch;   // of outputs, in floats: rows 4 apart half of the banks apart
    constexpr int kNeed = kSums * 4 > 2 * kArea ? kSums : (2 * kArea + 3) / 4;
    __shared__ u4v lds[kChunksOfSet * WK > kNeed ? kChunksOfSet * WK : kNeed];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wk = wave / (WM * WN), in_set = wave % (WM * WN), half = lane >> 5, wm = in_set / WN, wn = in_set % WN;
    // panels of 8 tiles of x: work-groups that run together share both operands
    const int lid = xcd_neighbours(blockIdx.x, a.mt * a.nt), panel = lid / (8 * a.nt), in = lid % (8 * a.nt);
    const int tall = a.mt - panel * 8 < 8 ? a.mt - panel * 8 : 8;
    const int m0 = (panel * 8 + in % tall) * kRows, n0 = in / tall * (32 * NT * WN) + wn * (32 * NT);
    auto swizzle = [](int r) { return kCh == 16 ? r & 15 : r >> 1 & 7; };

    // codes and scales: a base for the wave, which moves from block to block, and what a lane is away from it
    const int first = (n0 >> 4) < a.tiles ? n0 >> 4 : a.tiles - 1;
    const char *codes = reinterpret_cast<const char *>(a.codes) + ((long long)first * a.blocks + wk) * 1024;
    const char *scales = reinterpret_cast<const char *>(a.scales) + ((long long)first * a.blocks + wk) * (kGroups * 64);
    uint32_t code_at[NT], scale_at[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {            // (tiles past the last one repeat it: their outputs are not stored)
        int tile = (n0 + 32 * t + (lane & 31)) >> 4;
        tile = (tile < a.tiles ? tile : a.tiles - 1) - first;
        code_at[t] = tile * a.blocks * 1024 + ((lane & 15) + 32 * half) * 16;
        scale_at[t] = tile * a.blocks * (kGroups * 64) + (lane & 15) * 4;
    }
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
    // a block of the rows of x by way of registers
    struct Chunk { typename X::Raw r[kInt ? 2 : 1]; };
    auto load_chunk = [&](int b, int i) {
        const int at = slot + i * 64, r = at / kCh, c = at % kCh ^ swizzle(r), col = b * kQ4Block + c * T::kChunk;
        Chunk v = {};
        if (r < live) {
            const char *row = x + r * a.ldx;
            v.r[0] = load_columns<XT, true>(row, col, a.C);
            if constexpr (kInt) v.r[1] = load_columns<XT, true>(row, col + 8, a.C);
        }
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
    u4v next[NT][2];
    uint32_t word[NT][kGroups];
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
                for (int i = 0; i < kPer; ++i) put_chunk(buf, i, load_chunk(b, i));
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) raw[i] = load_chunk(b, i);
        }
        if constexpr (GS) {
            const int r = in_set * 64 + lane;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int group = b * kGroups + g;
                xs_next[g] = r < live && group < a.x_cols ? a.x_scale[(long long)(m0 + r) * a.x_cols + group] : 0.0f;
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int e = 0; e < 2; ++e) next[t][e] = *reinterpret_cast<const u4v *>(codes + (code_at[t] + 256 * e));
#pragma unroll
            for (int g = 0; g < kGroups; ++g) word[t][g] = *reinterpret_cast<const uint32_t *>(scales + (scale_at[t] + 64 * g));
        }
        codes += WK * 1024;
        scales += WK * (kGroups * 64);
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
    q4f16 total[MT][NT] = {};
    const int row0 = wm * (32 * MT) + (lane & 31);
    const int turns = (a.blocks + WK - 1) / WK;

    if (wk < a.blocks) {
        fetch(wk, 0);
        commit(0);
    }
    for (int turn = 0; turn < turns; ++turn) {
        const int b = turn * WK + wk, buf = turn & 1;
        wait_vmcnt<0>();                      // the block is in LDS, its codes in registers
        u4v now[NT][2];
        uint32_t sz[NT][kGroups];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            now[t][0] = next[t][0];
            now[t][1] = next[t][1];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) sz[t][g] = word[t][g];
        }
        // step st of the block: the weights' operand
        auto decode = [&](int st, u4v *w) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const typename X::Zero z = X::zero(sz[t][st / kStepsOfGroup]);
                if constexpr (kInt) {
                    const u2v w0 = X::weights(now[t][0][st], z), w1 = X::weights(now[t][1][st], z);
                    w[t] = u4v{w0[0], w0[1], w1[0], w1[1]};
                } else {
                    w[t] = X::weights(now[t][st & 1][st >> 1], z);
                }
            }
        };
        const u4v *from_lds = set + buf * kBuf + row0 * kCh;
        // part p of the rows of x at that step
        auto read = [&](int st, int p, u4v *op) {
            const int chunk = kInt ? 2 * st + half : 4 * (st >> 1) + 2 * half + (st & 1);
#pragma unroll
            for (int u = 0; u < MT; ++u) op[u] = from_lds[p * kRows * kCh + u * 32 * kCh + (chunk ^ swizzle(row0))];
        };
        u4v op[2][MT], w[2][NT];
        decode(0, w[0]);
        __syncthreads();
        if (b >= a.blocks) continue;          // (the last turn of some sets)
        const bool more = b + WK < a.blocks;
        if (more) fetch(b + WK, buf ^ 1);
        read(0, 0, op[0]);
        typename T::Acc acc[MT][NT] = {};
        // one part of one step after the other; what the next one needs is read and made beside the products
#pragma unroll
        for (int i = 0; i < kSteps * kParts; ++i) {
            const int st = i / kParts, p = i % kParts;
            const bool last = i + 1 == kSteps * kParts;
            if (!last) read((i + 1) / kParts, (i + 1) % kParts, op[(i + 1) & 1]);
            __builtin_amdgcn_sched_barrier(kAnyAlu);   // (else the reads sink to their uses, to save registers)
#pragma unroll
            for (int u = 0; u < MT; ++u)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[u][t] = T::mfma(op[i & 1][u], w[st & 1][t], acc[u][t]);
            if (!last && p == kParts - 1) decode(st + 1, w[(st + 1) & 1]);
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
                        xs[j] = *reinterpret_cast<const q4f4 *>(set_scales + (buf * kGroups + g) * kRows + wm * (32 * MT) + u * 32 + 8 * j + 4 * half);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const float f = __builtin_bit_cast(float, sz[t][g] & ~15u);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float v = (float)acc[u][t][j];
                        if constexpr (GS) v *= xs[j >> 2][j & 3];
                        total[u][t][j] = __builtin_fmaf(f, v, total[u][t][j]);
                    }
                    acc[u][t] = typename T::Acc{};
                }
            }
            // (a second group's sums at the same time would not fit the registers)
#pragma unroll
            for (int u = 0; u < MT; ++u)
#pragma unroll
                for (int t = 0; t < NT; ++t) asm volatile("" : "+v"(total[u][t]));
        }
        if (more) commit(buf ^ 1);
    }
    if constexpr (WK > 1) {                   // the sets' sums, in their order
        __syncthreads();
        q4f4 *const out = reinterpret_cast<q4f4 *>(lds);
        const int mine = in_set * 64 + lane;
        if (wk > 0)
#pragma unroll
            for (int e = 0; e < MT * NT * 4; ++e) {
                const q4f16 &f = total[e / 4 / NT][e / 4 % NT];
                out[((wk - 1) * MT * NT * 4 + e) * kSet + mine] = q4f4{f[e % 4 * 4], f[e % 4 * 4 + 1], f[e % 4 * 4 + 2], f[e % 4 * 4 + 3]};
            }
        __syncthreads();
        if (wk == 0)
#pragma unroll
            for (int e = 0; e < MT * NT * 4; ++e)
#pragma unroll
                for (int k = 0; k < WK - 1; ++k) {
                    const q4f4 f = out[(k * MT * NT * 4 + e) * kSet + mine];
#pragma unroll
                    for (int i = 0; i < 4; ++i) total[e / 4 / NT][e / 4 % NT][e % 4 * 4 + i] += f[i];
                }
    }
    // 32 rows of every wave after the other by way of LDS, so that a lane stores 16 bytes of a row of y
    float *const area = reinterpret_cast<float *>(lds);
    const int cols0 = n0 - wn * (32 * NT);
    const auto put = [&](int u) {
        if (wk == 0)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    area[(u & 1) * kArea + (wm * 32 + 8 * (i >> 2) + 4 * half + (i & 3)) * kPitch + wn * (32 * NT) + t * 32 + (lane & 31)] = total[u][t][i];
    };
    const auto store = [&](int u, auto type) {
        using E = typename Elem<decltype(type)::value>::type;
        constexpr int kV = 16 / (int)sizeof(E), kRow = 32 * NT * WN / kV;   // outputs of a thread; threads of a row
        for (int at = threadIdx.x; at < 32 * WM * kRow; at += kSet * WK) {
            const int r = at / kRow, c = at % kRow * kV, m = m0 + (r >> 5) * (32 * MT) + u * 32 + (r & 31), k = cols0 + c;
            if (m >= a.M || k >= a.K) continue;
            const float *f = area + (u & 1) * kArea + r * kPitch + c;
            const float xs = kInt && !GS ? a.x_scale[m] : 1.0f;
            E e[kV];
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                float v = f[j];
                if (kInt && !GS) v *= xs;
                e[j] = (E)act_apply(v + (a.bias && k + j < a.K ? a.bias[k + j] : 0.0f), a.act);
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
}

template <int XT, int NT, int MT, int W> hipError_t launch_rows(const Q4Args &a, int parts, hipStream_t st)
{
    const long long gx = (a.tiles + NT - 1) / NT, gy = ((long long)a.M + 16 * MT - 1) / (16 * MT);
    if (gx * W * 64 > 0xffffffffLL || gy > 65535) return hipErrorInvalidValue;
    const dim3 grid((unsigned)gx, (unsigned)gy, parts), block(W * 64);
    if (a.steps == 1) hipLaunchKernelGGL((rows_kernel<XT, NT, MT, W, 1>), grid, block, 0, st, a);
    else if (a.steps == 2) hipLaunchKernelGGL((rows_kernel<XT, NT, MT, W, 2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rows_kernel<XT, NT, MT, W, 4>), grid, block, 0, st, a);
    return hipGetLastError();
}

template <int XT, int MT, int NT, int WM, int WN, int WK, bool DMA, bool GS> hipError_t launch_tiles(Q4Args a, hipStream_t st)
{
    constexpr int rows = 32 * MT * WM, threads = WM * WN * WK * 64;
    const long long mt = ((long long)a.M + rows - 1) / rows, nt = (a.K + 32LL * NT * WN - 1) / (32 * NT * WN);
    if (mt * nt * threads > 0xffffffffLL || 8 * nt > 0x7fffffffLL) return hipErrorInvalidValue;
    a.mt = (int)mt;
    a.nt = (int)nt;
    const dim3 grid((unsigned)(mt * nt)), block(threads);
    if (a.steps == 1) hipLaunchKernelGGL((tile_kernel<XT, MT, NT, WM, WN, WK, 1, DMA, GS>), grid, block, 0, st, a);
    else if (a.steps == 2) hipLaunchKernelGGL((tile_kernel<XT, MT, NT, WM, WN, WK, 2, DMA, GS>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((tile_kernel<XT, MT, NT, WM, WN, WK, 4, DMA, GS>), grid, block, 0, st, a);
    return hipGetLastError();
}

// x may go to LDS without registers: 16-byte loads, offsets of a tile's rows below 2^31
inline bool dma_serves(const Q4Args &a, int rows) { return !(((uintptr_t)a.x | (uintptr_t)a.ldx) & 15) && a.ldx * rows < 0x7fff0000LL; }

template <int XT, int MT, int NT, int WM, int WN, int WK> hipError_t launch_tiles(const Q4Args &a, hipStream_t st)
{
    constexpr int rows = 32 * MT * WM;
    if constexpr (XT == FSCNN_F32) return launch_tiles<XT, MT, NT, WM, WN, WK, false, false>(a, st);
    else if constexpr (XT == FSCNN_I8) {
        if (a.x_cols > 1)
            return dma_serves(a, rows) ? launch_tiles<XT, MT, NT, WM, WN, WK, true, true>(a, st) : launch_tiles<XT, MT, NT, WM, WN, WK, false, true>(a, st);
        return dma_serves(a, rows) ? launch_tiles<XT, MT, NT, WM, WN, WK, true, false>(a, st) : launch_tiles<XT, MT, NT, WM, WN, WK, false, false>(a, st);
    } else {
        return dma_serves(a, rows) ? launch_tiles<XT, MT, NT, WM, WN, WK, true, false>(a, st) : launch_tiles<XT, MT, NT, WM, WN, WK, false, false>(a, st);
    }
}

}  // namespace

// parts: as q4_parts() says, or 1
template <int XT> hipError_t launch_q4_type(const Q4Args &a, int parts, hipStream_t st);
template <> hipError_t launch_q4_type<FSCNN_F32>(const Q4Args &a, int parts, hipStream_t st);
template <> hipError_t launch_q4_type<FSCNN_F16>(const Q4Args &a, int parts, hipStream_t st);
template <> hipError_t launch_q4_type<FSCNN_BF16>(const Q4Args &a, int parts, hipStream_t st);
template <> hipError_t launch_q4_type<FSCNN_I8>(const Q4Args &a, int parts, hipStream_t st);

}  // namespace fscnn
