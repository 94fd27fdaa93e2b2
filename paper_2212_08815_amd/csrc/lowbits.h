// Device helpers for tensors of 32, 16 and 8 bits: the types that fscnn_dtype_t names, conversions with one rounding to nearest even.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fscnn.h"

namespace fscnn {

template <int T> struct Elem;
template <> struct Elem<FSCNN_F32> { using type = float; };
template <> struct Elem<FSCNN_F16> { using type = _Float16; };
template <> struct Elem<FSCNN_BF16> { using type = __bf16; };
template <> struct Elem<FSCNN_I8> { using type = int8_t; };

__device__ inline float load_float(const void *p, long long i, int type)
{
    if (type == FSCNN_F32) return static_cast<const float *>(p)[i];
    if (type == FSCNN_F16) return (float)static_cast<const _Float16 *>(p)[i];
    return (float)static_cast<const __bf16 *>(p)[i];
}

__device__ inline void store_float(void *p, long long i, int type, float v)
{
    if (type == FSCNN_F32) static_cast<float *>(p)[i] = v;
    else if (type == FSCNN_F16) static_cast<_Float16 *>(p)[i] = (_Float16)v;
    else static_cast<__bf16 *>(p)[i] = (__bf16)v;
}

// f(std::integral_constant<int, type>) for a type known at run time only
template <class F> auto with_type(int type, F f)
{
    switch (type) {
        case FSCNN_F32: return f(std::integral_constant<int, FSCNN_F32>{});
        case FSCNN_F16: return f(std::integral_constant<int, FSCNN_F16>{});
        default: return f(std::integral_constant<int, FSCNN_BF16>{});
    }
}

}  // namespace fscnn
