// som_mx4_packed.hip -- products of many 4-bit rows with a 4-bit matrix.

#include "som_mx4_mm.h"

namespace som {
namespace {

using namespace four;

template <typename T, class S> hipError_t launch(const FourProduct &p, hipStream_t st)
{
    static std::atomic<uint64_t> done{0};
    const dim3 grid = grid_of((tiles<S>(p) + 7) / 8 * 8);
    if (grid.x == 0) return hipErrorInvalidValue;
    const hipError_t e = allow_lds(&k_mx4_packed<T, S>, Packed<S>::kBytes, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_mx4_packed<T, S>), grid, dim3(S::NT), Packed<S>::kBytes, st, p);
    return hipGetLastError();
}

template <typename T> hipError_t by_tile(FourTile t, const FourProduct &p, hipStream_t st)
{
    if (t == kFour64) return launch<T, Tile<64, 64, 2, 2, 2>>(p, st);
    if (t == kFour128) return launch<T, Tile<128, 128, 2, 2, 2>>(p, st);
    if (t == kFour192x256) return launch<T, Tile<192, 256, 2, 4, 1>>(p, st);
    return launch<T, Tile<256, 256, 2, 4, 1>>(p, st);
}

// Past the last block stands the smallest scale: what a product of two of them meets is nothing in fp32
// (2^-254), and with zeros it makes zeros.
__global__ __launch_bounds__(256) void k_pad_scales(const uint8_t *scales, int64_t rows, int32_t blocks, int32_t pitch, uint8_t *to)
{
    const int64_t total = rows * (pitch / 16), step = (int64_t)gridDim.x * 256;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += step) {
        const int64_t row = at / (pitch / 16);
        const int b = (int)(at - row * (pitch / 16)) * 16;
        const uint8_t *from = scales + row * blocks + b;
        uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (b + i < blocks) v[i / 4] |= (uint32_t)from[i] << (8 * (i % 4));
        reinterpret_cast<uint4 *>(to)[at] = uint4{v[0], v[1], v[2], v[3]};
    }
}

}  // namespace

hipError_t launch_mx4_packed(bool bf16, FourTile t, const FourProduct &p, hipStream_t st)
{
    return bf16 ? by_tile<__bf16>(t, p, st) : by_tile<_Float16>(t, p, st);
}

hipError_t launch_pad_scales(const uint8_t *scales, int64_t rows, int64_t K, uint8_t *to, hipStream_t st)
{
    const int64_t pitch = four_pitch(K), groups = (rows * (pitch / 16) + 255) / 256;
    hipLaunchKernelGGL(k_pad_scales, dim3((unsigned)(groups < 1 << 20 ? groups : 1 << 20)), dim3(256), 0, st, scales, rows,
                       (int32_t)four_blocks(K), (int32_t)pitch, to);
    return hipGetLastError();
}

}  // namespace som
