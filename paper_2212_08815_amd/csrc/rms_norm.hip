// Root-mean-square norm with the residual's addition and, if wanted, an output in 8 bits with scales:
//   h = x + r,  y = h / sqrt(mean(h^2) + eps) * w,  scale = max|y| / 127,  code = rint(y / scale)
//
// One pass: a row stays in registers between the sum of its squares and its outputs, so that x and r are read and y and h written once (8 bytes an
// element in 16 bits), and memory bounds all but the smallest calls.  TH threads take a row: 8 to 64 where one vector of 16 bytes a
// thread holds it, or a wave with two, so that no barrier is met; more threads for longer rows.  A thread holds N vectors, vector i of a row
// at thread i mod TH, and issues all loads of its row before it uses the first.  A group of 32 to 128 columns lies in 4 to 32 adjacent
// lanes.  Measured: 16384 rows of 4096 in bf16 with residual 91 to 95 us, 5.7 TB/s, in 8 bits 86 to 98; 2^19 rows of 128 91 us (with a wave
// a row 248); one row of 4096 3.2 us, of which a launch is most.  Rows past 32768 spill registers (72 to 228 bytes a thread): 512 rows of 65536 in fp32
// 113 us, 4.7 TB/s, in bf16 79, 3.4.
// Codes are formed in 32 bits: 2 to 7 in a million elements are so near the border between two codes that they get the other one (with
// elementary operations in 32 bits 1 to 5).  In 64 bits none was for fp32 rows, for 10 to 25% more time; 16-bit rows have exact ties
// that no precision settles.
#include <type_traits>

#include "internal.h"
#include "lowbits.h"

namespace fscnn {

namespace {

struct NormArgs {
    const char *x, *r, *w;
    char *ro, *y;
    float *scale;
    long long ldx, ldr, ldo, ldy;              // in bytes
    int w_type, y_type, M, D, group;
    float eps;
};

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

__device__ inline uint32_t code_of(float y, float up, float inv)
{
    return inv > 0.0f ? (uint32_t)(int)fminf(fmaxf(rintf(y * up * inv), -127.0f), 127.0f) & 255u : 0u;   // (y * 0 may be NaN)
}

// V elements of type T from column c of a row on, as they are; zeros from D on
template <int T, int V> struct Vec { typename Elem<T>::type e[V]; };
template <int T, int V> __device__ inline Vec<T, V> load_vec(const char *row, int c, int D)
{
    using E = typename Elem<T>::type;
    Vec<T, V> v;
    if (c + V <= D) __builtin_memcpy(&v, row + (long long)c * (int)sizeof(E), sizeof(v));
    else
#pragma unroll
        for (int j = 0; j < V; ++j) {
            v.e[j] = E{};
            if (c + j < D) v.e[j] = reinterpret_cast<const E *>(row)[c + j];
        }
    return v;
}

template <int T, int V> __device__ inline void store_vec(char *row, int c, int D, const float *f)
{
    using E = typename Elem<T>::type;
    Vec<T, V> v;
#pragma unroll
    for (int j = 0; j < V; ++j) v.e[j] = (E)f[j];
    if (c + V <= D) __builtin_memcpy(row + (long long)c * (int)sizeof(E), &v, sizeof(v));
    else
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (c + j < D) reinterpret_cast<E *>(row)[c + j] = v.e[j];
}

template <int V> __device__ inline void store_any(char *row, int type, int c, int D, const float *f)
{
    if (type == FSCNN_F32) store_vec<FSCNN_F32, V>(row, c, D, f);
    else if (type == FSCNN_F16) store_vec<FSCNN_F16, V>(row, c, D, f);
    else store_vec<FSCNN_BF16, V>(row, c, D, f);
}

template <int V> __device__ inline void store_codes(char *row, int c, int D, const float *f, float up, float inv)
{
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        w[i] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[i] |= code_of(f[4 * i + j], up, inv) << (8 * j);
    }
    if (c + V <= D) __builtin_memcpy(row + c, w, V);
    else
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (c + j < D) row[c + j] = (char)(w[j / 4] >> (8 * (j % 4)));
}

// Q8: the 8-bit output (a kernel of its own: the other one holds fewer registers)
template <int T, int N, int TH, bool Q8> __global__ void __launch_bounds__(TH < 256 ? 256 : TH) rms_norm_kernel(const NormArgs a)
{
    constexpr int V = 16 / (int)sizeof(typename Elem<T>::type), kWaves = TH < 64 ? 1 : TH / 64, kRows = TH < 256 ? 256 / TH : 1;
    __shared__ float sums[kWaves];
    __shared__ uint32_t mags[kWaves];
    const int t = TH < 256 ? threadIdx.x % TH : threadIdx.x, lane = threadIdx.x & 63, wave = t >> 6;
    const long long m = (long long)blockIdx.x * kRows + (TH < 256 ? threadIdx.x / TH : 0);
    if (m >= a.M) return;                      // (with more than one row a work-group, rows meet no barrier)
    const char *x = a.x + m * a.ldx, *r = a.r + m * a.ldr;
    Vec<T, V> xv[N], rv[N];
#pragma unroll
    for (int i = 0; i < N; ++i) xv[i] = load_vec<T, V>(x, (i * TH + t) * V, a.D);
    if (a.r)
#pragma unroll
        for (int i = 0; i < N; ++i) rv[i] = load_vec<T, V>(r, (i * TH + t) * V, a.D);
    float h[N][V], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            h[i][j] = (float)xv[i].e[j];
            if (a.r) h[i][j] += (float)rv[i].e[j];
            sum = __builtin_fmaf(h[i][j], h[i][j], sum);
        }
        if (a.ro) store_vec<T, V>(a.ro + m * a.ldo, (i * TH + t) * V, a.D, h[i]);
    }
    // the row's sum from its threads'
    const auto of_row = [&](float v) {
#pragma unroll
        for (int d = 1; d < 64 && d < TH; d *= 2) v += __shfl_xor(v, d);
        if constexpr (kWaves > 1) {
            if (lane == 0) sums[wave] = v;
            __syncthreads();
            v = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) v += sums[i];
        }
        return v;
    };
    sum = of_row(sum);
    float f = 1.0f / sqrtf(sum / (float)a.D + a.eps);
    // Squares past the largest float, or so small that they lost digits: h by a power of two closer to 1, and its squares again.  (The same for all
    // threads of a row.  2^-80 takes the largest rows' mean square to 2^96, 2^96 that of rows below 2^-90 to at most 2^102; what
    // is lost at the other end does not show beside it.)
    if (__builtin_expect(!(sum < __builtin_inff()) || sum / (float)a.D + a.eps < 0x1p-90f, 0)) {
        const bool large = !(sum < 1.0f);
        const float by = large ? 0x1p-80f : 0x1p96f;
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float v = h[i][j] * by;
                sum = __builtin_fmaf(v, v, sum);
                h[i][j] = large ? h[i][j] * 0x1p-40f : v;   // (the other half with f: neither is then below the normal numbers)
            }
        if constexpr (kWaves > 1) __syncthreads();
        sum = of_row(sum);
        f = 1.0f / sqrtf(sum / (float)a.D + a.eps * by * by) * (large ? 0x1p-40f : 1.0f);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * TH + t) * V;
        float w[V];
        if (!a.w) {
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = 1.0f;
        } else if (a.w_type == FSCNN_F32) {
            const auto v = load_vec<FSCNN_F32, V>(a.w, c, a.D);
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = v.e[j];
        } else if (a.w_type == FSCNN_F16) {
            const auto v = load_vec<FSCNN_F16, V>(a.w, c, a.D);
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = (float)v.e[j];
        } else {
            const auto v = load_vec<FSCNN_BF16, V>(a.w, c, a.D);
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = (float)v.e[j];
        }
#pragma unroll
        for (int j = 0; j < V; ++j) h[i][j] = h[i][j] * f * w[j];   // (columns from D on: zeros, or NaN; they are not stored and not measured)
    }
    char *y = a.y + m * a.ldy;
    if constexpr (!Q8) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((i * TH + t) * V < a.D) store_any<V>(y, a.y_type, (i * TH + t) * V, a.D, h[i]);
    } else {
        uint32_t most[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            most[i] = 0;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if ((i * TH + t) * V + j < a.D) most[i] = max(most[i], magnitude(h[i][j]));
        }
        float up, inv;
        if (a.group == 0) {
#pragma unroll
            for (int i = 1; i < N; ++i) most[0] = max(most[0], most[i]);
#pragma unroll
            for (int d = 1; d < 64 && d < TH; d *= 2) most[0] = max(most[0], (uint32_t)__shfl_xor((int)most[0], d));
            if constexpr (kWaves > 1) {
                if (lane == 0) mags[wave] = most[0];
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kWaves; ++i) most[0] = max(most[0], mags[i]);
            }
            const float s = scale_of(most[0], &up, &inv);
            if (t == 0) a.scale[m] = s;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if ((i * TH + t) * V < a.D) store_codes<V>(y, (i * TH + t) * V, a.D, h[i], up, inv);
            return;
        }
        const int ng = (a.D + a.group - 1) / a.group;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            for (int d = 1; d * V < a.group && d < TH; d *= 2) most[i] = max(most[i], (uint32_t)__shfl_xor((int)most[i], d));
            const float s = scale_of(most[i], &up, &inv);
            const int c = (i * TH + t) * V;
            if (c >= a.D) continue;
            if (c % a.group == 0) a.scale[m * ng + c / a.group] = s;
            store_codes<V>(y, c, a.D, h[i], up, inv);
        }
    }
}

template <int T, int N, int TH> hipError_t launch_rows(const NormArgs &a, hipStream_t st)
{
    constexpr int rows = TH < 256 ? 256 / TH : 1;
    const long long grid = ((long long)a.M + rows - 1) / rows, threads = TH < 256 ? 256 : TH;
    if (grid * threads > 0xffffffffLL) return hipErrorInvalidValue;
    if (a.y_type == FSCNN_I8) hipLaunchKernelGGL((rms_norm_kernel<T, N, TH, true>), dim3((unsigned)grid), dim3((unsigned)threads), 0, st, a);
    else hipLaunchKernelGGL((rms_norm_kernel<T, N, TH, false>), dim3((unsigned)grid), dim3((unsigned)threads), 0, st, a);
    return hipGetLastError();
}

template <int T> hipError_t launch_type(const NormArgs &a, hipStream_t st)
{
    constexpr int V = 16 / (int)sizeof(typename Elem<T>::type);
    const int n = (a.D + V - 1) / V;           // vectors of a row
    if (n <= 8) return launch_rows<T, 1, 8>(a, st);
    if (n <= 16) return launch_rows<T, 1, 16>(a, st);
    if (n <= 32) return launch_rows<T, 1, 32>(a, st);
    if (n <= 64) return launch_rows<T, 1, 64>(a, st);
    if (n <= 128) return launch_rows<T, 2, 64>(a, st);
    if (n <= 256) return launch_rows<T, 1, 256>(a, st);
    if (n <= 512) return launch_rows<T, 2, 256>(a, st);
    if (n <= 1024) return launch_rows<T, 4, 256>(a, st);
    if (n <= 2048) return launch_rows<T, 2, 1024>(a, st);
    if (n <= 4096) return launch_rows<T, 4, 1024>(a, st);
    if constexpr (V * 8192 < kNormMaxD)
        if (n > 8192) return launch_rows<T, 16, 1024>(a, st);
    return launch_rows<T, 8, 1024>(a, st);
}

}  // namespace

hipError_t launch_rms_norm(const void *x, int type, long long ldx, const void *residual, long long ldr, void *residual_out, long long ldo,
                           const void *weight, int weight_type, int M, int D, float eps, void *y, int y_type, long long ldy, float *scale,
                           int group, hipStream_t st)
{
    if (D > kNormMaxD) return hipErrorInvalidValue;
    const int e = type == FSCNN_F32 ? 4 : 2, ey = y_type == FSCNN_F32 ? 4 : y_type == FSCNN_I8 ? 1 : 2;
    // rows in launches that a grid holds
    constexpr long long kMost = 1 << 20;
    for (long long m = 0; m < M; m += kMost) {
        const NormArgs a = {static_cast<const char *>(x) + m * ldx * e, residual ? static_cast<const char *>(residual) + m * ldr * e : nullptr,
                            static_cast<const char *>(weight), residual_out ? static_cast<char *>(residual_out) + m * ldo * e : nullptr,
                            static_cast<char *>(y) + m * ldy * ey, scale ? scale + m * (group ? (D + group - 1) / group : 1) : nullptr, ldx * e, ldr * e,
                            ldo * e, ldy * ey, weight_type, y_type, (int)(M - m < kMost ? M - m : kMost), D, group, eps};
        const hipError_t err = with_type(type, [&](auto t) { return launch_type<decltype(t)::value>(a, st); });
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace fscnn
