// som_norm_grad.hip -- layer norm backward: the threads a row takes, and the parts' sums.

#include "som_norm.h"

namespace som {
namespace {

using namespace layer;

template <class S> hipError_t grad(const NormArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)a.n_parts);
    if (a.D % S::V == 0) hipLaunchKernelGGL((k_norm_grad<S, true>), grid, dim3(S::NT), 0, st, a);
    else hipLaunchKernelGGL((k_norm_grad<S, false>), grid, dim3(S::NT), 0, st, a);
    return hipGetLastError();
}

template <typename X, typename Y> hipError_t by_width(const NormArgs &a, hipStream_t st)
{
    constexpr int V = 16 / (int)sizeof(X);
    const int vectors = (a.D + V - 1) / V;
    if (vectors <= 8) return grad<NormShape<X, Y, 8, 1, 512>>(a, st);
    if (vectors <= 16) return grad<NormShape<X, Y, 16, 1, 512>>(a, st);
    if (vectors <= 32) return grad<NormShape<X, Y, 32, 1, 512>>(a, st);
    if (vectors <= 64) return grad<NormShape<X, Y, 64, 1, 512>>(a, st);
    if (vectors <= 128) return grad<NormShape<X, Y, 64, 2, 512>>(a, st);
    if (vectors <= 256) return grad<NormShape<X, Y, 128, 2, 512>>(a, st);
    if (vectors <= 512) return grad<NormShape<X, Y, 256, 2, 512>>(a, st);
    if (vectors <= 1024) return grad<NormShape<X, Y, 512, 2, 512>>(a, st);
    if (vectors <= 2048) return grad<NormShape<X, Y, 512, 4, 512>>(a, st);
    if (a.dx) {
        hipLaunchKernelGGL((k_norm_means<X, Y>), dim3((unsigned)(a.N < 2048 ? a.N : 2048)), dim3(1024), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)a.n_parts, (unsigned)((vectors + 255) / 256));
    hipLaunchKernelGGL((k_norm_strips<X, Y>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

// 32 columns by 32 stretches of parts a workgroup; the stretches' sums are added in order.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_sums(const float *__restrict__ parts, int64_t n_parts, int D, T *dweight,
                                                    T *dbias)
{
    __shared__ float lds[32][33];
    const int col = (int)blockIdx.x * 32 + (int)threadIdx.x % 32, group = (int)threadIdx.x / 32, j = blockIdx.y;
    T *out = j ? dbias : dweight;
    if (!out) return;
    const int64_t per = (n_parts + 31) / 32, from = group * per, to = min(n_parts, from + per);
    float s = 0;
    if (col < D) {
#pragma unroll 8
        for (int64_t p = from; p < to; ++p) s += parts[(2 * p + j) * (int64_t)D + col];
    }
    lds[group][threadIdx.x % 32] = s;
    __syncthreads();
    if (group == 0 && col < D) {
        s = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += lds[i][threadIdx.x];
        out[col] = (T)s;
    }
}

template <typename T>
hipError_t sums(const float *parts, int64_t n_parts, int32_t D, void *dweight, void *dbias, hipStream_t st)
{
    hipLaunchKernelGGL(k_norm_sums<T>, dim3((unsigned)((D + 31) / 32), 2), dim3(1024), 0, st, parts, n_parts, D,
                       static_cast<T *>(dweight), static_cast<T *>(dbias));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_grad(int x_type, int y_type, const NormArgs &a, hipStream_t st)
{
    if (x_type == SOM_F16) return by_width<_Float16, _Float16>(a, st);
    if (x_type == SOM_BF16) return by_width<__bf16, __bf16>(a, st);
    if (y_type == SOM_F16) return by_width<float, _Float16>(a, st);
    if (y_type == SOM_BF16) return by_width<float, __bf16>(a, st);
    return by_width<float, float>(a, st);
}

hipError_t launch_norm_sums(const float *parts, int64_t n_parts, int32_t D, void *dweight, void *dbias, int type,
                            hipStream_t st)
{
    if (type == SOM_F16) return sums<_Float16>(parts, n_parts, D, dweight, dbias, st);
    if (type == SOM_BF16) return sums<__bf16>(parts, n_parts, D, dweight, dbias, st);
    return sums<float>(parts, n_parts, D, dweight, dbias, st);
}

}  // namespace som
