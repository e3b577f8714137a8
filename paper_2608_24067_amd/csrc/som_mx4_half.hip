// som_mx4_half.hip -- products of many 16-bit rows with a 4-bit matrix.

#include "som_mx4_mm.h"

namespace som {
namespace {

using namespace four;

template <typename T, class S> hipError_t launch(const FourProduct &p, hipStream_t st)
{
    static std::atomic<uint64_t> done{0};
    const dim3 grid = grid_of((tiles<S>(p) + 7) / 8 * 8);
    if (grid.x == 0) return hipErrorInvalidValue;
    const hipError_t e = allow_lds(&k_mx4_half<T, S>, Half<S>::kBytes, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_mx4_half<T, S>), grid, dim3(S::NT), Half<S>::kBytes, st, p);
    return hipGetLastError();
}

template <typename T> hipError_t by_tile(FourTile t, const FourProduct &p, hipStream_t st)
{
    if (t == kFour64) return launch<T, Tile<64, 64, 2, 2, 2>>(p, st);
    if (t == kFour128) return launch<T, Tile<128, 128, 2, 2, 2>>(p, st);
    if (t == kFour192x256) return launch<T, Tile<192, 256, 2, 4, 1>>(p, st);
    return launch<T, Tile<256, 256, 2, 4, 1>>(p, st);
}

// 16-byte chunks of whole lines of a row, from rows of any alignment.
__global__ __launch_bounds__(256) void k_pad_rows(const uint16_t *x, int64_t ldx, int64_t rows, int32_t K, int32_t chunks, uint4 *to)
{
    typedef uint16_t eight __attribute__((ext_vector_type(8)));
    typedef eight any __attribute__((aligned(2)));
    const int64_t total = rows * chunks, step = (int64_t)gridDim.x * 256;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += step) {
        const int64_t row = at / chunks;
        const int k = (int)(at - row * chunks) * 8, n = K - k;
        const uint16_t *from = x + row * ldx + k;
        eight v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (n >= 8) {
            v = *reinterpret_cast<const any *>(from);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) v[i] = from[i];
        }
        to[at] = __builtin_bit_cast(uint4, v);
    }
}

}  // namespace

hipError_t launch_mx4_half(bool bf16, FourTile t, const FourProduct &p, hipStream_t st)
{
    return bf16 ? by_tile<__bf16>(t, p, st) : by_tile<_Float16>(t, p, st);
}

hipError_t launch_pad_rows(const void *x, int64_t ldx, int64_t rows, int64_t K, void *to, hipStream_t st)
{
    const int64_t chunks = four_width(K) / 8, groups = (rows * chunks + 255) / 256;
    hipLaunchKernelGGL(k_pad_rows, dim3((unsigned)(groups < 1 << 20 ? groups : 1 << 20)), dim3(256), 0, st,
                       static_cast<const uint16_t *>(x), ldx, rows, (int32_t)K, (int32_t)chunks, static_cast<uint4 *>(to));
    return hipGetLastError();
}

}  // namespace som
