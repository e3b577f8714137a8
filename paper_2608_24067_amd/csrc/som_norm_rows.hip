// som_norm_rows.hip -- layer norm forward: the threads a row takes, by its width.

#include "som_norm.h"

namespace som {
namespace {

using namespace layer;

// Workgroups a launch has at most: as many as the CUs hold at once, so that each reads the weights once for
// all its rows and the rows in flight are neighbours (us with 256, 1024 and 2048 of them: 4000 x 8192 and
// 2000 x 16384 fp32, a row by 1024 threads, 48, 57, 62 and 39, 50, 51; 20011 x 1003 fp32, four vectors a
// thread, 37, 25.8, 28.1; 8192 x 4096 bf16, two, 1024 29.9, 2048 29.7).
// With four vectors of eight a thread (16-bit rows above 16,384 features) weights and biases, in fp32, do not all fit its
// registers: 165 are spilled of bf16's, and where rows end inside a vector 280, of fp16's 0 and 48 (2000 x 24576 bf16 66
// us, 24570 80, fp16 50, by the bytes 40).
template <class S> constexpr int64_t kGroups = S::NT == 1024 ? 256 : S::C == 4 ? 1024 : 2048;

template <class S> hipError_t rows(const NormArgs &a, hipStream_t st)
{
    const int64_t all = (a.N + S::ROWS - 1) / S::ROWS;
    const dim3 grid((unsigned)(all < kGroups<S> ? all : kGroups<S>));
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
    hipLaunchKernelGGL((k_norm_long<X, Y>), dim3((unsigned)(a.N < 2048 ? a.N : 2048)), dim3(1024), 0, st, a);
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
