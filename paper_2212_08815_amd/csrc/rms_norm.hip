// Root-mean-square norm with the residual's addition and, if wanted, an output in 8 bits with scales.  The simple form: a work-group of 1024
// threads per row, the row in registers.
#include <type_traits>

#include "internal.h"
#include "lowbits.h"

namespace fscnn {

namespace {

struct NormArgs {
    const void *x, *r, *w;
    void *ro, *y;
    float *scale;
    long long ldx, ldr, ldo, ldy;
    int type, w_type, y_type, M, D, group;
    float eps;
};

constexpr int kThreads = 1024;

// |v| as a number that orders as it does, NaN above all
__device__ inline uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

// Scale of a largest magnitude, and what y is multiplied by: first `up`, then `inv`.  (Below 2^-100, 127 / most would be past the largest float.)
__device__ inline float scale_of(uint32_t most, float *up, float *inv)
{
    const float a = __builtin_bit_cast(float, most);
    *up = a < 0x1p-100f ? 0x1p100f : 1.0f;
    *inv = a > 0.0f && a < __builtin_inff() ? 127.0f / (a * *up) : 0.0f;
    return a / 127.0f;
}

__device__ inline int8_t code_of(float y, float up, float inv)
{
    return inv > 0.0f ? (int8_t)(int)fminf(fmaxf(rintf(y * up * inv), -127.0f), 127.0f) : (int8_t)0;   // (y * 0 may be NaN)
}

template <int N> __global__ void __launch_bounds__(kThreads) rms_norm_kernel(const NormArgs a)
{
    __shared__ float sums[kThreads / 64];
    __shared__ uint32_t mags[kThreads / 64];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    for (int m = blockIdx.x; m < a.M; m += gridDim.x) {
        float h[N], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * kThreads + t;
            h[i] = 0.0f;
            if (c < a.D) {
                h[i] = load_float(a.x, m * a.ldx + c, a.type);
                if (a.r) h[i] += load_float(a.r, m * a.ldr + c, a.type);
                if (a.ro) store_float(a.ro, m * a.ldo + c, a.type, h[i]);
            }
            sum = __builtin_fmaf(h[i], h[i], sum);
        }
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        __syncthreads();
        if (lane == 0) sums[wave] = sum;
        __syncthreads();
        sum = 0.0f;
        for (int i = 0; i < kThreads / 64; ++i) sum += sums[i];
        const float f = 1.0f / sqrtf(sum / (float)a.D + a.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * kThreads + t;
            if (c < a.D) h[i] = h[i] * f * (a.w ? load_float(a.w, c, a.w_type) : 1.0f);
        }
        if (a.y_type != FSCNN_I8) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = i * kThreads + t;
                if (c < a.D) store_float(a.y, m * a.ldy + c, a.y_type, h[i]);
            }
            continue;
        }
        int8_t *y = static_cast<int8_t *>(a.y) + m * a.ldy;
        float up, inv;
        if (a.group == 0) {
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i * kThreads + t < a.D) most = max(most, magnitude(h[i]));
            for (int d = 1; d < 64; d *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, d));
            if (lane == 0) mags[wave] = most;
            __syncthreads();
            most = 0;
            for (int i = 0; i < kThreads / 64; ++i) most = max(most, mags[i]);
            const float s = scale_of(most, &up, &inv);
            if (t == 0) a.scale[m] = s;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = i * kThreads + t;
                if (c < a.D) y[c] = code_of(h[i], up, inv);
            }
            continue;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * kThreads + t;
            uint32_t most = c < a.D ? magnitude(h[i]) : 0;
            for (int d = 1; d < 32; d *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, d));
            if (a.group >= 64) most = max(most, (uint32_t)__shfl_xor((int)most, 32));
            if (a.group == 128) {          // two waves
                __syncthreads();
                if (lane == 0) mags[wave] = most;
                __syncthreads();
                most = max(mags[wave], mags[wave ^ 1]);
            }
            const float s = scale_of(most, &up, &inv);
            if (c < a.D) {
                y[c] = code_of(h[i], up, inv);
                if (c % a.group == 0) a.scale[m * (long long)((a.D + a.group - 1) / a.group) + c / a.group] = s;
            }
        }
    }
}

}  // namespace

hipError_t launch_rms_norm(const void *x, int type, long long ldx, const void *residual, long long ldr, void *residual_out, long long ldo,
                           const void *weight, int weight_type, int M, int D, float eps, void *y, int y_type, long long ldy, float *scale,
                           int group, hipStream_t st)
{
    const NormArgs a = {x, residual, weight, residual_out, y, scale, ldx, ldr, ldo, ldy, type, weight_type, y_type, M, D, group, eps};
    const dim3 grid(M < 65536 ? M : 65536), block(kThreads);
    if (D <= 4096) hipLaunchKernelGGL(rms_norm_kernel<4>, grid, block, 0, st, a);
    else if (D <= 16384) hipLaunchKernelGGL(rms_norm_kernel<16>, grid, block, 0, st, a);
    else if (D <= kNormMaxD) hipLaunchKernelGGL(rms_norm_kernel<64>, grid, block, 0, st, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace fscnn
