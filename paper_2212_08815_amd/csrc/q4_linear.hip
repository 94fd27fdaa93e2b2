// y = act(x W^T + b) with 4-bit weights: which launch serves a call, and the sum of what divided launches leave (kernels: q4_kernels.h).
#include "q4_kernels.h"

namespace fscnn {

namespace {

// What the P work-groups that divide the columns have left, added in their order; four outputs a thread, all loads on their way together
template <int P> __global__ void __launch_bounds__(64) join_kernel(const Q4Args a)
{
    const int k = (blockIdx.x * 64 + threadIdx.x) * 4;
    const long long pitch = a.tiles * 16LL;
    for (int m = blockIdx.y; m < a.M; m += gridDim.y) {
        q4f4 v[P];
        v[0] = q4f4{};
        if (k < a.K) {
#pragma unroll
            for (int p = 0; p < P; ++p) __builtin_memcpy(&v[p], a.sums + (((long long)p * a.M + m) * pitch + k), 16);
#pragma unroll
            for (int p = 1; p < P; ++p) v[0] += v[p];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[0][i] = mended(a, k + i < a.K, m, k + i, v[0][i]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i < a.K) store_output(a, m, k + i, v[0][i], a.bias ? a.bias[k + i] : 0.0f);
    }
}

}  // namespace

int q4_parts(const fscnn_q4 *q, int x_type, int M) { return q4_parts(x_type, M, q->K, q->C); }

hipError_t launch_linear_q4(const fscnn_q4 *q, const void *x, int x_type, long long ldx, const float *x_scale, int x_scale_cols, int M,
                            const float *bias, int act, void *y, int y_type, long long ldy, float *sums, hipStream_t st)
{
    const int bytes = x_type == FSCNN_F32 ? 4 : x_type == FSCNN_I8 ? 1 : 2;
    const long long most = q4_launch_rows(q->K);   // rows of x in launches that a grid holds
    for (long long m = 0; m < M; m += most) {
        const Q4Args a = {reinterpret_cast<const u4v *>(q->codes), q->scales, static_cast<const char *>(x) + m * ldx * bytes,
                          x_scale ? x_scale + m * x_scale_cols : nullptr, bias, static_cast<char *>(y) + m * ldy * (y_type == FSCNN_F32 ? 4 : 2), sums,
                          ldx * bytes, ldy, q->K, q->C, (int)(M - m < most ? M - m : most), (int)q4_blocks(q->C), (int)q4_tiles(q->K),
                          q->group / 32, y_type, x_scale_cols, act, x_type, 0, 0};
        const int parts = sums ? q4_parts(q, x_type, M) : 1;
        hipError_t e;
        switch (x_type) {
            case FSCNN_F32: e = launch_q4_type<FSCNN_F32>(a, parts, st); break;
            case FSCNN_F16: e = launch_q4_type<FSCNN_F16>(a, parts, st); break;
            case FSCNN_BF16: e = launch_q4_type<FSCNN_BF16>(a, parts, st); break;
            default: e = launch_q4_type<FSCNN_I8>(a, parts, st);
        }
        if (e != hipSuccess) return e;
        if (parts > 1) {
            const dim3 grid((unsigned)((a.K + 255) / 256), a.M < 65535 ? a.M : 65535);
            if (parts == 2) hipLaunchKernelGGL(join_kernel<2>, grid, dim3(64), 0, st, a);
            else if (parts == 4) hipLaunchKernelGGL(join_kernel<4>, grid, dim3(64), 0, st, a);
            else if (parts == 8) hipLaunchKernelGGL(join_kernel<8>, grid, dim3(64), 0, st, a);
            else hipLaunchKernelGGL(join_kernel<16>, grid, dim3(64), 0, st, a);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace fscnn
