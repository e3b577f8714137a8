// som_mx4.hip -- values in 4 bits, blocks of 32 under a shared power of two, and back.
//
// A value is a sign and 0, 1/2, 1, 3/2, 2, 3, 4 or 6; a block's scale byte s stands for 2^(s - 127),
// chosen as s = exponent of the block's largest value + 127 - 2, not below 0, so that the largest
// lies in [4, 8) (and is held as 6 at most). Rounding is to nearest, ties to the even code. A block
// with an infinity or a NaN gets s = 255, and all of it stands for NaN. Block b of a row holds
// features 32 b to 32 b + 31, two to a byte, the first in the low half; past the last feature are zeros.
//
// Bound by the bytes read and written. Rows: four threads a block, eight values each.

#include "som_layer_device.h"

namespace som {
namespace {

using namespace layer;

constexpr int kThreads = 256;

// The scale's byte from the bits of the block's largest magnitude.
__device__ inline uint32_t scale_byte(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255 ? 255 : e > 2 ? e - 2 : 0;
}

// Eight values over the scale as codes.
__device__ inline uint32_t encode8(const float *v, float scale)
{
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
}

__device__ inline void decode8(uint32_t c, uint32_t s, float *v)
{
    typedef float two __attribute__((ext_vector_type(2)));
    const float scale = scale_value(s);
    const two a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
    const two d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
    v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = d[0], v[5] = d[1], v[6] = e[0], v[7] = e[1];
    if (s == 255) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_nanf("");
    }
}

__device__ inline uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFF; }

template <typename T> __global__ __launch_bounds__(kThreads) void k_quantise_rows(const FourArgs a, int64_t blocks, int32_t row_blocks)
{
    const int64_t step = (int64_t)gridDim.x * (kThreads / 4);
    for (int64_t block = (int64_t)blockIdx.x * (kThreads / 4) + threadIdx.x / 4; block < blocks; block += step) {
        const int64_t row = block / row_blocks;
        const int k = (int)(block - row * row_blocks) * kFourBlock + (int)threadIdx.x % 4 * 8;
        float v[8];
        load<8>(static_cast<const T *>(a.x) + row * a.ldx + k, (int)(a.K - k), v);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude(v[i]));
        top = max(top, swap32<0xB1>(top));
        top = max(top, swap32<0x4E>(top));
        const uint32_t s = scale_byte(top), c = encode8(v, scale_value(s));
        reinterpret_cast<uint32_t *>(a.codes)[block * 4 + threadIdx.x % 4] = c;
        if (threadIdx.x % 4 == 0) a.scales[block] = (uint8_t)s;
    }
}

// Feature-major matrices: a workgroup takes 128 features by 64 columns through LDS, rows by 16-byte
// vectors on the side of the matrix, one block of a column a thread on the side of the codes. 1003 x 5625
// fp32 takes 9.0 us and 8.1 back (22.6 MB); a thread for eight columns' blocks, without LDS, took as
// long there, but 12.6 us for a matrix in bf16 of any small size, its code being fetched (now 3.4).
constexpr int kCols = 64, kFeatures = kThreads / 64 * kFourBlock;

template <typename T> struct Vectors {
    static constexpr int V = 16 / sizeof(T), kAcross = kCols / V, kStep = kThreads / kAcross, kTurns = kFeatures / kStep;
};

__host__ __device__ inline int64_t column_tiles(int64_t N, int64_t row_blocks)
{
    return (N + kCols - 1) / kCols * ((row_blocks + kFeatures / kFourBlock - 1) / (kFeatures / kFourBlock));
}

template <typename T> __global__ __launch_bounds__(kThreads) void k_quantise_columns(const FourArgs a, int32_t row_blocks)
{
    typedef Vectors<T> S;
    typedef typename VecOf<T, S::V>::type vec;
    __shared__ __align__(16) T tile[kFeatures][kCols];
    const int64_t across = (a.N + kCols - 1) / kCols, total = column_tiles(a.N, row_blocks);
    const int c = (int)threadIdx.x % 64, own = (int)threadIdx.x / 64, v = (int)threadIdx.x % S::kAcross * S::V, r0 = (int)threadIdx.x / S::kAcross;
    for (int64_t i = blockIdx.x; i < total; i += gridDim.x) {
        const int64_t col = i % across * kCols, k = i / across * kFeatures;
        const T *x = static_cast<const T *>(a.x) + k * a.ldx + col;
        const int rows = (int)min((int64_t)kFeatures, a.K - k), cols = (int)min((int64_t)kCols, a.N - col);
        vec in[S::kTurns];
        if (cols == kCols) {
#pragma unroll
            for (int t = 0; t < S::kTurns; ++t)
                in[t] = *reinterpret_cast<const typename VecOf<T, S::V>::any *>(x + min(r0 + t * S::kStep, rows - 1) * a.ldx + v);
        } else {
#pragma unroll
            for (int t = 0; t < S::kTurns; ++t)
#pragma unroll
                for (int j = 0; j < S::V; ++j) in[t][j] = x[min(r0 + t * S::kStep, rows - 1) * a.ldx + min(v + j, cols - 1)];
        }
#pragma unroll
        for (int t = 0; t < S::kTurns; ++t) {
            const int r = r0 + t * S::kStep;
            *reinterpret_cast<vec *>(&tile[r][v]) = r < rows ? in[t] : vec(0);
        }
        __syncthreads();
        const int64_t block = k / kFourBlock + own;
        if (c < cols && block < row_blocks) {
            float f[kFourBlock];
            uint32_t top = 0, q[4];
#pragma unroll
            for (int e = 0; e < kFourBlock; ++e) f[e] = (float)tile[own * kFourBlock + e][c], top = max(top, magnitude(f[e]));
            const uint32_t s = scale_byte(top);
#pragma unroll
            for (int h = 0; h < 4; ++h) q[h] = encode8(f + 8 * h, scale_value(s));
            const int64_t at = (col + c) * row_blocks + block;
            reinterpret_cast<uint4 *>(a.codes)[at] = uint4{q[0], q[1], q[2], q[3]};
            a.scales[at] = (uint8_t)s;
        }
        __syncthreads();
    }
}

template <typename T> __global__ __launch_bounds__(kThreads) void k_values_rows(const FourArgs a, int64_t blocks, int32_t row_blocks, T *y, int64_t ldy)
{
    const int64_t step = (int64_t)gridDim.x * (kThreads / 4);
    for (int64_t block = (int64_t)blockIdx.x * (kThreads / 4) + threadIdx.x / 4; block < blocks; block += step) {
        const int64_t row = block / row_blocks;
        const int k = (int)(block - row * row_blocks) * kFourBlock + (int)threadIdx.x % 4 * 8;
        float v[8];
        decode8(reinterpret_cast<const uint32_t *>(a.codes)[block * 4 + threadIdx.x % 4], a.scales[block], v);
        if (k < a.K) store<8>(y + row * ldy + k, (int)(a.K - k), v);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_values_columns(const FourArgs a, int32_t row_blocks, T *y, int64_t ldy)
{
    typedef Vectors<T> S;
    typedef typename VecOf<T, S::V>::type vec;
    __shared__ __align__(16) T tile[kFeatures][kCols];
    const int64_t across = (a.N + kCols - 1) / kCols, total = column_tiles(a.N, row_blocks);
    const int c = (int)threadIdx.x % 64, own = (int)threadIdx.x / 64, v = (int)threadIdx.x % S::kAcross * S::V, r0 = (int)threadIdx.x / S::kAcross;
    for (int64_t i = blockIdx.x; i < total; i += gridDim.x) {
        const int64_t col = i % across * kCols, k = i / across * kFeatures;
        const int rows = (int)min((int64_t)kFeatures, a.K - k), cols = (int)min((int64_t)kCols, a.N - col);
        const int64_t at = (col + min(c, cols - 1)) * row_blocks + min(k / kFourBlock + own, (int64_t)row_blocks - 1);
        const uint4 q = reinterpret_cast<const uint4 *>(a.codes)[at];
        const uint32_t s = a.scales[at], words[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            float f[8];
            decode8(words[h], s, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[own * kFourBlock + 8 * h + e][c] = (T)f[e];
        }
        __syncthreads();
        T *out = y + k * ldy + col;
#pragma unroll
        for (int t = 0; t < S::kTurns; ++t) {
            const int r = r0 + t * S::kStep;
            if (r >= rows) continue;
            const vec w = *reinterpret_cast<const vec *>(&tile[r][v]);
            if (cols == kCols) {
                *reinterpret_cast<typename VecOf<T, S::V>::any *>(out + r * ldy + v) = w;
            } else {
#pragma unroll
                for (int j = 0; j < S::V; ++j)
                    if (v + j < cols) out[r * ldy + v + j] = w[j];
            }
        }
        __syncthreads();
    }
}

constexpr int64_t kGroups = 1 << 20;  // workgroups of a launch, which go on from there

dim3 column_grid(const FourArgs &a, int64_t row_blocks)
{
    const int64_t n = column_tiles(a.N, row_blocks);
    return dim3((unsigned)(n < kGroups ? n : kGroups));
}

template <typename T> hipError_t quantise(bool columns, const FourArgs &a, hipStream_t st)
{
    const int64_t row_blocks = four_blocks(a.K), blocks = a.N * row_blocks;
    if (columns) {
        hipLaunchKernelGGL(k_quantise_columns<T>, column_grid(a, row_blocks), dim3(kThreads), 0, st, a, (int32_t)row_blocks);
    } else {
        const int64_t n = (blocks + kThreads / 4 - 1) / (kThreads / 4);
        hipLaunchKernelGGL(k_quantise_rows<T>, dim3((unsigned)(n < kGroups ? n : kGroups)), dim3(kThreads), 0, st, a, blocks,
                           (int32_t)row_blocks);
    }
    return hipGetLastError();
}

template <typename T> hipError_t values(bool columns, const FourArgs &a, void *y, int64_t ldy, hipStream_t st)
{
    const int64_t row_blocks = four_blocks(a.K), blocks = a.N * row_blocks;
    if (columns) {
        hipLaunchKernelGGL(k_values_columns<T>, column_grid(a, row_blocks), dim3(kThreads), 0, st, a, (int32_t)row_blocks, static_cast<T *>(y), ldy);
    } else {
        const int64_t n = (blocks + kThreads / 4 - 1) / (kThreads / 4);
        hipLaunchKernelGGL(k_values_rows<T>, dim3((unsigned)(n < kGroups ? n : kGroups)), dim3(kThreads), 0, st, a, blocks,
                           (int32_t)row_blocks, static_cast<T *>(y), ldy);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_quantise(int type, bool columns, const FourArgs &a, hipStream_t st)
{
    if (type == SOM_F16) return quantise<_Float16>(columns, a, st);
    if (type == SOM_BF16) return quantise<__bf16>(columns, a, st);
    return quantise<float>(columns, a, st);
}

hipError_t launch_mx4_values(int type, bool columns, const FourArgs &a, void *y, int64_t ldy, hipStream_t st)
{
    if (type == SOM_F16) return values<_Float16>(columns, a, y, ldy, st);
    if (type == SOM_BF16) return values<__bf16>(columns, a, y, ldy, st);
    return values<float>(columns, a, y, ldy, st);
}

}  // namespace som
