// Weights in 4 bits: from codes and scales that exist, or from dense weights, into the order that the matrix cores' operands have
// (internal.h), and back.  One pass each; done once per set of weights.
#include "internal.h"
#include "lowbits.h"

namespace fscnn {

namespace {

struct Shape {
    int K, C, group, blocks, groups;         // groups: of a padded row
    long long words;                         // of codes
};

Shape shape_of(const fscnn_q4 *q)
{
    const int blocks = (int)q4_blocks(q->C);
    return {q->K, q->C, q->group, blocks, blocks * (kQ4Block / q->group), (long long)(q4_code_bytes(q->K, q->C) / 4)};
}

// A thread's first item; the next ones are all_threads() apart
__device__ inline long long first_item() { return (long long)blockIdx.x * 256 + threadIdx.x; }
__device__ inline long long all_threads() { return (long long)gridDim.x * 256; }

// Row and first column of word i
__device__ inline void word_at(const Shape &p, long long i, long long *row, int *col)
{
    const int s = (int)(i & 3), lane = (int)(i >> 2) & 63;
    const long long b = i >> 8;
    *row = b / p.blocks * 16 + (lane & 15);
    *col = (int)(b % p.blocks) * kQ4Block + s * 32 + (lane >> 4) * 8;
}

__device__ inline uint32_t *scale_word(uint32_t *scales, const Shape &p, long long row, int g)
{
    return scales + ((row >> 4) * p.groups + g) * 16 + (row & 15);
}

__device__ inline uint32_t as_word(float v) { return __builtin_bit_cast(uint32_t, v); }

// One thread per word of codes; the one at a group's first column of a row writes the group's scale as well.
__global__ void __launch_bounds__(256) import_kernel(const Shape p, const unsigned char *codes, const void *scales_in, int scale_type,
                                                     const unsigned char *zeros, uint32_t *out, uint32_t *scales, int *flag)
{
    for (long long i = first_item(); i < p.words; i += all_threads()) {
        long long row;
        int col;
        word_at(p, i, &row, &col);
        const int g = col / p.group, ng = (p.C + p.group - 1) / p.group;
        const bool live = row < p.K && col < p.C;
        uint32_t zero = 8, w = 0;
        if (live && zeros) {
            zero = zeros[row * ng + g];
            if (zero > 15) *flag = 1;
            zero &= 15;
        }
        const long long pitch = ((long long)p.C + 1) / 2;
        if (live && col + 8 <= p.C) {
            uint32_t in;                          // column j in bits 4 j: the first four go to the low halves of the bytes, the others to the high ones
            __builtin_memcpy(&in, codes + (row * pitch + (col >> 1)), 4);
            const uint32_t lo = in & 0xffff, hi = in >> 16;
            const auto spread = [](uint32_t v) {
                v = (v | v << 8) & 0x00ff00ff;
                return (v | v << 4) & 0x0f0f0f0f;
            };
            w = spread(lo) | spread(hi) << 4;
        } else if (live) {
            for (int j = 0; j < 8; ++j)
                w |= (col + j < p.C ? codes[row * pitch + ((col + j) >> 1)] >> (4 * (j & 1)) & 15 : zero) << code_bit(j);
        }
        out[i] = w;
        if (col % p.group == 0) {
            const uint32_t s = live ? as_word(load_float(scales_in, row * ng + g, scale_type)) : 0;
            *scale_word(scales, p, row, g) = s | (live ? zero : 0);
        }
    }
}

__global__ void clear_kernel(int *flag) { *flag = 0; }

// One thread per group of a (padded) row: scale and zero point
__global__ void __launch_bounds__(256) group_kernel(const Shape p, const void *w, int type, long long ldw, int zeros, uint32_t *scales)
{
    const long long rows = ((long long)p.K + 15) / 16 * 16;
    for (long long i = first_item(); i < rows * p.groups; i += all_threads()) {
        const long long row = i / p.groups;
        const int g = (int)(i % p.groups), c0 = g * p.group, c1 = c0 + p.group < p.C ? c0 + p.group : p.C;
        uint32_t word = 0;
        if (row < p.K && c0 < p.C) {
            float lo = 0.0f, hi = 0.0f;
            bool finite = true;
            for (int c = c0; c < c1; ++c) {
                const float v = load_float(w, row * ldw + c, type);
                finite &= fabsf(v) < __builtin_inff();
                lo = fminf(lo, v);
                hi = fmaxf(hi, v);
            }
            // (in two halves: hi - lo may be past the largest float)
            float s = zeros ? hi / 15.0f - lo / 15.0f : fmaxf(-lo, hi) / 7.0f;
            if (!finite) s = __builtin_nanf("");
            s = type == FSCNN_F16 ? (float)(_Float16)s : (float)(__bf16)s;
            float z = 8.0f;
            if (zeros) z = s > 0.0f && finite ? fminf(rintf(-lo / s), 15.0f) : 0.0f;
            word = as_word(s) | (uint32_t)z;
        }
        *scale_word(scales, p, row, g) = word;
    }
}

__global__ void __launch_bounds__(256) compress_kernel(const Shape p, const void *w, int type, long long ldw, uint32_t *out, uint32_t *scales)
{
    for (long long i = first_item(); i < p.words; i += all_threads()) {
        long long row;
        int col;
        word_at(p, i, &row, &col);
        const uint32_t sz = *scale_word(scales, p, row, col / p.group), zero = sz & 15;
        const float s = __builtin_bit_cast(float, sz & ~15u), z = (float)zero;
        uint32_t word = 0;
        for (int j = 0; j < 8; ++j) {
            uint32_t code = zero;
            if (row < p.K && col + j < p.C && s > 0.0f)
                code = (uint32_t)fminf(fmaxf(rintf(load_float(w, row * ldw + col + j, type) / s) + z, 0.0f), 15.0f);
            word |= code << code_bit(j);
        }
        out[i] = word;
    }
}

// One thread per byte of codes
__global__ void __launch_bounds__(256) export_kernel(const Shape p, const uint32_t *in, const uint32_t *scales, int scale_type,
                                                     unsigned char *codes, void *scales_out, unsigned char *zeros)
{
    const long long pitch = ((long long)p.C + 1) / 2;
    for (long long i = first_item(); i < pitch * p.K; i += all_threads()) {
        const long long row = i / pitch;
        const int c = (int)(i % pitch) * 2, ng = (p.C + p.group - 1) / p.group, g = c / p.group;
        uint32_t byte = 0;
        for (int e = 0; e < 2 && c + e < p.C; ++e) {
            const int at = (c + e) % kQ4Block, lane = (at / 8 % 4) * 16 + (int)(row & 15);
            const long long b = (row >> 4) * p.blocks + (c + e) / kQ4Block;
            byte |= (in[(b * 64 + lane) * 4 + at / 32] >> code_bit(at % 8) & 15) << (4 * e);
        }
        codes[i] = (unsigned char)byte;
        if (c % p.group == 0) {
            const uint32_t sz = scales[((row >> 4) * p.groups + g) * 16 + (row & 15)];
            store_float(scales_out, row * ng + g, scale_type, __builtin_bit_cast(float, sz & ~15u));
            zeros[row * ng + g] = (unsigned char)(sz & 15);
        }
    }
}

// work-groups of 256 threads for n items: a thread each, or several where a launch does not hold as many
unsigned groups_for(long long n)
{
    constexpr long long kMost = 1 << 23;
    const long long b = (n + 255) / 256;
    return (unsigned)(b < kMost ? b : kMost);
}

}  // namespace

hipError_t launch_q4_import(const fscnn_q4 *q, const unsigned char *codes, const void *scales, const unsigned char *zeros, int *flag, hipStream_t st)
{
    const Shape p = shape_of(q);
    hipLaunchKernelGGL(clear_kernel, dim3(1), dim3(1), 0, st, flag);
    hipLaunchKernelGGL(import_kernel, dim3(groups_for(p.words)), dim3(256), 0, st, p, codes, scales, q->scale_type, zeros, q->codes, q->scales, flag);
    return hipGetLastError();
}

hipError_t launch_q4_compress(const fscnn_q4 *q, const void *w, int type, long long ldw, hipStream_t st)
{
    const Shape p = shape_of(q);
    hipLaunchKernelGGL(group_kernel, dim3(groups_for(q4_tiles(p.K) * 16 * p.groups)), dim3(256), 0, st, p, w, type, ldw, q->zeros, q->scales);
    hipLaunchKernelGGL(compress_kernel, dim3(groups_for(p.words)), dim3(256), 0, st, p, w, type, ldw, q->codes, q->scales);
    return hipGetLastError();
}

hipError_t launch_q4_export(const fscnn_q4 *q, unsigned char *codes, void *scales, unsigned char *zeros, hipStream_t st)
{
    const Shape p = shape_of(q);
    hipLaunchKernelGGL(export_kernel, dim3(groups_for(((long long)p.C + 1) / 2 * p.K)), dim3(256), 0, st, p, q->codes, q->scales, q->scale_type, codes, scales, zeros);
    return hipGetLastError();
}

}  // namespace fscnn
