// som_norm_rows.hip -- layer norm forward: the threads a row takes, by its width.

#include "som_norm.h"

namespace som {
namespace {

using namespace layer;

// Workgroups a launch has at most: enough for every CU to hold what it can of them, so that a
// workgroup reads the weights once for all its rows.
constexpr int64_t kGroups = 2048;

template <class S> hipError_t rows(const NormArgs &a, hipStream_t st)
{
    const int64_t all = (a.N + S::ROWS - 1) / S::ROWS;
    const dim3 grid((unsigned)(all < kGroups ? all : kGroups));
    if (a.D % S::V == 0) hipLaunchKernelGGL((k_norm_rows<S, true>), grid, dim3(S::NT), 0, st, a);
    else hipLaunchKernelGGL((k_norm_rows<S, false>), grid, dim3(S::NT), 0, st, a);
    return hipGetLastError();
}

template <typename X, typename Y> hipError_t by_width(const NormArgs &a, hipStream_t st)
{
    const int vectors = (a.D + 16 / (int)sizeof(X) - 1) / (16 / (int)sizeof(X));
    if (vectors <= 8) return rows<NormShape<X, Y, 8, 1, 256>>(a, st);
    if (vectors <= 16) return rows<NormShape<X, Y, 16, 1, 256>>(a, st);
    if (vectors <= 32) return rows<NormShape<X, Y, 32, 1, 256>>(a, st);
    if (vectors <= 64) return rows<NormShape<X, Y, 64, 1, 256>>(a, st);
    if (a.N <= 256 && vectors <= 512) return rows<NormShape<X, Y, 256, 2, 256>>(a, st);  // a row a CU: latency counts
    if (vectors <= 128) return rows<NormShape<X, Y, 64, 2, 256>>(a, st);
    if (vectors <= 256) return rows<NormShape<X, Y, 64, 4, 256>>(a, st);
    if (vectors <= 512) return rows<NormShape<X, Y, 256, 2, 256>>(a, st);
    if (vectors <= 1024) return rows<NormShape<X, Y, 256, 4, 256>>(a, st);
    if (vectors <= 2048) return rows<NormShape<X, Y, 1024, 2, 1024>>(a, st);
    if (vectors <= 4096) return rows<NormShape<X, Y, 1024, 4, 1024>>(a, st);
    hipLaunchKernelGGL((k_norm_long<X, Y>), dim3((unsigned)(a.N < kGroups ? a.N : kGroups)), dim3(1024), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rows(int x_type, int y_type, const NormArgs &a, hipStream_t st)
{
    if (x_type == SOM_F16) return by_width<_Float16, _Float16>(a, st);
    if (x_type == SOM_BF16) return by_width<__bf16, __bf16>(a, st);
    if (y_type == SOM_F16) return by_width<float, _Float16>(a, st);
    if (y_type == SOM_BF16) return by_width<float, __bf16>(a, st);
    return by_width<float, float>(a, st);
}

}  // namespace som
