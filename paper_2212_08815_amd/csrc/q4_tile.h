// Device helpers of the products with 4-bit weights: codes and rows of x as operands of the matrix cores (16 x 16 outputs, steps of 32 columns).
//
// A code 0..15 in a byte is, read as an 8-bit float with 4 exponent and 3 fraction bits, exactly code * 2^-9 (below 8 a denormal number, from
// 8 on the first binade), so that one conversion gives two codes as 16-bit floats: (3 masks and shifts + 4 conversions) / 8 instructions a
// code.  Codes go in as they are, without the zero point; a product with ones gives the sum of x over the group, and with it
//     sum (q - z) x = sum q x - z sum x,
// which costs one multiply-add per output and group, and in 32-bit floats at most (q + z) / |q - z| times the rounding of the plain sum.
// (codes.  weights, with the zero point subtracted, take 2.4 instructions a code and are for tiles of many rows, and for the products of three
// parts: where these meet in one sum, it and the one of x lose a digit, 2.4e-6 of the result instead of 1.3e-7 over 4096 columns that
// are not negative.  In sums of their own the parts' errors are alike and their difference has few of them: 2.5e-7.)
// Floats enter as three bfloat16 parts (8 bits of the significand each, by truncation: their sum is the float, but for bits below 2^-133, which
// bfloat16 does not have; the parts of an infinite x are infinite, NaN and NaN: mended() in q4_kernels.h), integers as they are.
#pragma once
#include "internal.h"
#include "lowbits.h"

namespace fscnn {

typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef float q4f4 __attribute__((ext_vector_type(4)));
typedef float q4f2 __attribute__((ext_vector_type(2)));
typedef float q4f16 __attribute__((ext_vector_type(16)));
typedef int q4i4 __attribute__((ext_vector_type(4)));
typedef int q4i16 __attribute__((ext_vector_type(16)));
typedef __bf16 q4b2 __attribute__((ext_vector_type(2)));
typedef __bf16 q4b8 __attribute__((ext_vector_type(8)));
typedef _Float16 q4h2 __attribute__((ext_vector_type(2)));
typedef _Float16 q4h8 __attribute__((ext_vector_type(8)));

// Eight columns of a row of x: as loaded (raw), and as the operands of kParts products
template <int XT> struct XOp;
template <> struct XOp<FSCNN_BF16> {
    static constexpr int kParts = 1;
    using Raw = u4v;
    using Op = u4v;
    using Acc = q4f4;
    __device__ static void parts(const Raw &r, Op *o) { o[0] = r; }
    __device__ static Op codes(uint32_t w)
    {
        const int lo = w & 0x0f0f0f0f, hi = w >> 4 & 0x0f0f0f0f;
        Op o;
        o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false));
        o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true));
        o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false));
        o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true));
        return o;
    }
    using Zero = float;
    __device__ static Zero zero(uint32_t word) { return (float)(word & 15); }
    __device__ static Op weights(uint32_t w, Zero z)
    {
        const int lo = w & 0x0f0f0f0f, hi = w >> 4 & 0x0f0f0f0f;
        const q4f2 f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, 512.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, 512.0f, true),
                           __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, 512.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, 512.0f, true)};
        Op o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_bit_cast(uint32_t, q4b2{(__bf16)(f[i][0] - z), (__bf16)(f[i][1] - z)});
        return o;
    }
    __device__ static Op ones() { return Op{0x3f803f80, 0x3f803f80, 0x3f803f80, 0x3f803f80}; }
    __device__ static Acc mfma(const Op &a, const Op &b, const Acc &c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q4b8, a), __builtin_bit_cast(q4b8, b), c, 0, 0, 0);
    }
};
template <> struct XOp<FSCNN_F16> {
    static constexpr int kParts = 1;
    using Raw = u4v;
    using Op = u4v;
    using Acc = q4f4;
    __device__ static void parts(const Raw &r, Op *o) { o[0] = r; }
    __device__ static Op codes(uint32_t w)
    {
        const int lo = w & 0x0f0f0f0f, hi = w >> 4 & 0x0f0f0f0f;
        Op o;
        o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false));
        o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true));
        o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false));
        o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true));
        return o;
    }
    using Zero = q4h2;
    __device__ static Zero zero(uint32_t word) { return Zero{(_Float16)(float)(word & 15), (_Float16)(float)(word & 15)}; }
    __device__ static Op weights(uint32_t w, Zero z)
    {
        const Op c = codes(w);
        Op o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pair = c[i];       // (a bit cast of a vector's element itself is read from the vector's start)
            o[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(q4h2, pair) - z);
        }
        return o;
    }
    __device__ static Op ones() { return Op{0x3c003c00, 0x3c003c00, 0x3c003c00, 0x3c003c00}; }
    __device__ static Acc mfma(const Op &a, const Op &b, const Acc &c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(q4h8, a), __builtin_bit_cast(q4h8, b), c, 0, 0, 0);
    }
};
template <> struct XOp<FSCNN_F32> {
    static constexpr int kParts = 3;
    struct Raw { u4v a, b; };
    using Op = u4v;
    using Acc = q4f4;
    __device__ static void parts(const Raw &r, Op *o)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w[2] = {i < 2 ? r.a[2 * i] : r.b[2 * i - 4], i < 2 ? r.a[2 * i + 1] : r.b[2 * i - 3]}, m[2], l[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float x = __builtin_bit_cast(float, w[e]), x1 = x - __builtin_bit_cast(float, w[e] & 0xffff0000u);
                m[e] = __builtin_bit_cast(uint32_t, x1);
                l[e] = __builtin_bit_cast(uint32_t, x1 - __builtin_bit_cast(float, m[e] & 0xffff0000u));
            }
            // the high halves of two words
            o[0][i] = __builtin_amdgcn_perm(w[1], w[0], 0x07060302);
            o[1][i] = __builtin_amdgcn_perm(m[1], m[0], 0x07060302);
            o[2][i] = __builtin_amdgcn_perm(l[1], l[0], 0x07060302);
        }
    }
    using Zero = float;
    __device__ static Zero zero(uint32_t word) { return XOp<FSCNN_BF16>::zero(word); }
    __device__ static Op weights(uint32_t w, Zero z) { return XOp<FSCNN_BF16>::weights(w, z); }
    __device__ static Acc mfma(const Op &a, const Op &b, const Acc &c) { return XOp<FSCNN_BF16>::mfma(a, b, c); }
};
template <> struct XOp<FSCNN_I8> {
    static constexpr int kParts = 1;
    using Raw = u2v;
    using Op = u2v;
    using Acc = q4i4;
    __device__ static void parts(const Raw &r, Op *o) { o[0] = r; }
    __device__ static Op codes(uint32_t w) { return Op{w & 0x0f0f0f0f, w >> 4 & 0x0f0f0f0f}; }
    using Zero = uint32_t;                    // (128 - z) in every byte: with a code's added, the high bit flipped is what signs it
    __device__ static Zero zero(uint32_t word) { return (128 - (word & 15)) * 0x01010101u; }
    __device__ static Op weights(uint32_t w, Zero z) { return Op{((w & 0x0f0f0f0f) + z) ^ 0x80808080u, ((w >> 4 & 0x0f0f0f0f) + z) ^ 0x80808080u}; }
    __device__ static Op ones() { return Op{0x01010101, 0x01010101}; }
    __device__ static Acc mfma(const Op &a, const Op &b, const Acc &c)
    {
        return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), c, 0, 0, 0);
    }
};

// Columns col .. col + 7 of a row (elements of any alignment that their type has), zeros from C on
template <int XT, bool TAIL> __device__ inline typename XOp<XT>::Raw load_columns(const char *row, int col, int C)
{
    using E = typename Elem<XT>::type;
    typename XOp<XT>::Raw r;
    const char *p = row + (long long)col * (int)sizeof(E);
    if (!TAIL || col + 8 <= C) {
        __builtin_memcpy(&r, p, sizeof(r));
    } else {
        E e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            e[j] = E{};
            if (col + j < C) e[j] = reinterpret_cast<const E *>(p)[j];
        }
        __builtin_memcpy(&r, e, sizeof(r));
    }
    return r;
}

}  // namespace fscnn
