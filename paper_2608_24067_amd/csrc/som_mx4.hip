// som_mx4.hip -- values in 4 bits, blocks of 32 under a shared power of two, and back.
//
// A value is a sign and 0, 1/2, 1, 3/2, 2, 3, 4 or 6; a block's scale byte s stands for 2^(s - 127),
// chosen as s = exponent of the block's largest value + 127 - 2, not below 0, so that the largest
// lies in [4, 8) (and is held as 6 at most). Rounding is to nearest, ties to the even code. A block
// with an infinity or a NaN gets s = 255, and all of it stands for NaN. Block b of a row holds
// features 32 b to 32 b + 31, two to a byte, the first in the low half; past the last feature are zeros.
//
// Bound by the bytes read and written. Rows: four threads a block, eight values each. Feature-major
// matrices: a thread takes one 16-byte vector of columns over a block's 32 features, 32 loads in
// flight, and needs no exchange.

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

// 2^(s - 127) as the conversions take it: 0 stands for 2^-127, a subnormal.
__device__ inline float scale_value(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x00400000u); }

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

// A thread: V columns by one block of features.
template <typename T> __device__ inline void quantise_columns(const FourArgs &a, int32_t row_blocks, int64_t col, int block)
{
    constexpr int V = 16 / sizeof(T);
    const int n = (int)min((int64_t)V, a.N - col), k = block * kFourBlock, left = (int)min((int64_t)kFourBlock, a.K - k);
    const T *x = static_cast<const T *>(a.x) + (int64_t)k * a.ldx + col;
    typename VecOf<T, V>::type v[kFourBlock];
#pragma unroll
    for (int i = 0; i < kFourBlock; ++i) {
        if (i < left && n == V) {
            v[i] = *reinterpret_cast<const typename VecOf<T, V>::any *>(x + i * a.ldx);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[i][j] = i < left && j < n ? x[i * a.ldx + j] : (T)0.0f;
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (j >= n) break;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kFourBlock; ++i) top = max(top, magnitude((float)v[i][j]));
        const uint32_t s = scale_byte(top);
        uint32_t c[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)v[8 * h + i][j];
            c[h] = encode8(f, scale_value(s));
        }
        const int64_t at = (col + j) * row_blocks + block;
        reinterpret_cast<uint4 *>(a.codes)[at] = uint4{c[0], c[1], c[2], c[3]};
        a.scales[at] = (uint8_t)s;
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
__device__ inline void values_columns(const FourArgs &a, int32_t row_blocks, T *y, int64_t ldy, int64_t col, int block)
{
    constexpr int V = 16 / sizeof(T);
    const int n = (int)min((int64_t)V, a.N - col), k = block * kFourBlock, left = (int)min((int64_t)kFourBlock, a.K - k);
    uint4 c[V];
    uint32_t s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int64_t at = (min(col + j, a.N - 1)) * row_blocks + block;
        c[j] = reinterpret_cast<const uint4 *>(a.codes)[at];
        s[j] = a.scales[at];
    }
    T *out = y + (int64_t)k * ldy + col;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        float v[V][8];
#pragma unroll
        for (int j = 0; j < V; ++j) decode8(h == 0 ? c[j].x : h == 1 ? c[j].y : h == 2 ? c[j].z : c[j].w, s[j], v[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (8 * h + i >= left) continue;
            float r[V];
#pragma unroll
            for (int j = 0; j < V; ++j) r[j] = v[j][i];
            store<V>(out + (int64_t)(8 * h + i) * ldy, n, r);
        }
    }
}

// A wave takes 16 vectors of columns by four blocks at a time; f(first column, block). Workgroups are single
// waves, which spread over the CUs (1,003 x 5,625 fp32 is 704 of them).
constexpr int kColumnBlocks = 4;

template <int V, typename F> __device__ inline void over_columns(const FourArgs &a, int32_t row_blocks, F f)
{
    const int64_t across = (a.N + 16 * V - 1) / (16 * V), total = across * ((row_blocks + kColumnBlocks - 1) / kColumnBlocks);
    for (int64_t i = blockIdx.x; i < total; i += gridDim.x) {
        const int64_t col = (i % across * 16 + threadIdx.x % 16) * V;
        const int block = (int)(i / across) * kColumnBlocks + (int)threadIdx.x / 16;
        if (col < a.N && block < row_blocks) f(col, block);
    }
}

template <typename T> __global__ __launch_bounds__(64) void k_quantise_columns(const FourArgs a, int32_t row_blocks)
{
    over_columns<16 / sizeof(T)>(a, row_blocks, [&](int64_t col, int block) { quantise_columns<T>(a, row_blocks, col, block); });
}

template <typename T>
__global__ __launch_bounds__(64) void k_values_columns(const FourArgs a, int32_t row_blocks, T *y, int64_t ldy)
{
    over_columns<16 / sizeof(T)>(a, row_blocks, [&](int64_t col, int block) { values_columns<T>(a, row_blocks, y, ldy, col, block); });
}

constexpr int64_t kGroups = 1 << 20;  // workgroups of a launch, which go on from there

template <typename T> dim3 column_grid(const FourArgs &a, int64_t row_blocks)
{
    constexpr int V = 16 / sizeof(T);
    const int64_t n = (a.N + 16 * V - 1) / (16 * V) * ((row_blocks + kColumnBlocks - 1) / kColumnBlocks);
    return dim3((unsigned)(n < kGroups ? n : kGroups));
}

template <typename T> hipError_t quantise(bool columns, const FourArgs &a, hipStream_t st)
{
    const int64_t row_blocks = four_blocks(a.K), blocks = a.N * row_blocks;
    if (columns) {
        hipLaunchKernelGGL(k_quantise_columns<T>, column_grid<T>(a, row_blocks), dim3(64), 0, st, a, (int32_t)row_blocks);
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
        hipLaunchKernelGGL(k_values_columns<T>, column_grid<T>(a, row_blocks), dim3(64), 0, st, a, (int32_t)row_blocks, static_cast<T *>(y), ldy);
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
