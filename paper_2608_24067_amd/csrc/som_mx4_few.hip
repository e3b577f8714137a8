// som_mx4_few.hip -- products with a 4-bit matrix, for few rows.
//
// A workgroup takes RT x 16 rows by CT x 16 columns, and its eight waves share out the features in
// units of 128 (four blocks), whose sums are joined in LDS. The matrix is read once, straight into
// registers: lane (q, i) of a wave holds block 4 u + q of column i, 16 bytes, of unit u.
//   Rows in 16 bits: the codes are widened to bf16 under their scale (exact: two significant bits and a
//   power of two), eight at a time, and meet the same features of the rows in four instructions of 32
//   features. fp16 rows go as two bf16 values each, x = hi + lo, which is exact and knows no scale
//   that fp16 could not hold.
//   Rows in 4 bits: one instruction takes both operands' 128 codes and applies the blocks' scales.
// The matrix is the instruction's first operand, so a lane owns four neighbouring columns of a row.

#include "som_layer_device.h"
#include "som_mm.h"

namespace som {
namespace {

using namespace layer;
using mm::bf16x8;
using mm::f16x8;
using mm::f32x4;

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8, kUnit = 128;

// 2^(s - 127), a subnormal for 0 and NaN for 255.
__device__ inline float scale_value(uint32_t s) { return __uint_as_float(max(s << 23, 0x00400000u) | (s + 1) >> 8 << 22); }

// Eight codes as bf16 values.
__device__ inline bf16x8 widen(uint32_t c, float scale)
{
    typedef __bf16 two __attribute__((ext_vector_type(2)));
    const two a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
    const two d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}

__device__ inline uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <typename T> struct Eight {
    typename mm::Vec8<T>::type v;
    __device__ void get(const T *p, int64_t n)
    {
        typedef typename mm::Vec8<T>::type any __attribute__((aligned(2)));
        if (n >= 8) {
            v = *reinterpret_cast<const any *>(p);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : (T)0.0f;
        }
    }
};

__device__ inline f32x4 multiply(bf16x8 w, bf16x8 x, f32x4 c) { return mm::mma(w, x, c); }
__device__ inline f32x4 multiply(bf16x8 w, f16x8 x, f32x4 c)
{
    bf16x8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float f = (float)x[i];
        hi[i] = (__bf16)f;
        const float rest = f - (float)hi[i];  // NaN where x is infinite: that is in hi already
        lo[i] = (__bf16)(rest == rest ? rest : 0.0f);
    }
    return mm::mma(w, lo, mm::mma(w, hi, c));
}

template <typename T, bool PACKED, int RT, int CT> __global__ __launch_bounds__(64 * kWaves) void k_mx4_few(const FourProduct p)
{
    __shared__ f32x4 joined[kWaves][RT * CT][64];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int q = lane >> 4, i = lane & 15;
    const int64_t across = (p.M + CT * 16 - 1) / (CT * 16), b = mm::block_number();
    const int64_t row0 = b / across * (RT * 16), col0 = b % across * (CT * 16);
    if (row0 >= p.N) return;
    const int64_t blocks = four_blocks(p.K);
    const int units = (int)((p.K + kUnit - 1) / kUnit);
    const uint4 *w[CT], *xc[RT];
    const uint8_t *ws[CT], *xs[RT];
    const T *x[RT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int64_t col = min(col0 + 16 * c + i, p.M - 1);
        w[c] = reinterpret_cast<const uint4 *>(p.w) + col * blocks;
        ws[c] = p.w_scales + col * blocks;
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int64_t row = min(row0 + 16 * r + i, p.N - 1);
        if (PACKED) {
            xc[r] = static_cast<const uint4 *>(p.x) + row * blocks;
            xs[r] = p.x_scales + row * blocks;
        } else {
            x[r] = static_cast<const T *>(p.x) + row * p.ldx;
        }
    }
    f32x4 acc[RT][CT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[r][c] = f32x4{0, 0, 0, 0};
    for (int u = wave; u < units; u += kWaves) {
        const int64_t block = 4 * (int64_t)u + q;
        const bool in = block < blocks;
        uint4 wc[CT];
        uint32_t sc[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            wc[c] = uint4{0, 0, 0, 0};
            sc[c] = 127;
            if (in) wc[c] = w[c][block], sc[c] = ws[c][block];
        }
        if (PACKED) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                uint4 v = uint4{0, 0, 0, 0};
                uint32_t s = 127;
                if (in) v = xc[r][block], s = xs[r][block];
                const i32x8 vx = {(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    const i32x8 vw = {(int)wc[c].x, (int)wc[c].y, (int)wc[c].z, (int)wc[c].w, 0, 0, 0, 0};
                    acc[r][c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vw, vx, acc[r][c], 4, 4, 0, (int)sc[c], 0, (int)s);
                }
            }
        } else {
            Eight<T> e[RT][4];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int s = 0; s < 4; ++s) e[r][s].get(x[r] + 32 * block + 8 * s, p.K - 32 * block - 8 * s);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const float scale = scale_value(sc[c]);
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const bf16x8 f = widen(word(wc[c], s), scale);
#pragma unroll
                    for (int r = 0; r < RT; ++r) acc[r][c] = multiply(f, e[r][s].v, acc[r][c]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) joined[wave][r * CT + c][lane] = acc[r][c];
    __syncthreads();
    for (int o = threadIdx.x; o < RT * CT * 64; o += 64 * kWaves) {
        const int tile = o / 64, l = o % 64;
        f32x4 s = joined[0][tile][l];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) s += joined[k][tile][l];
        const int64_t row = row0 + tile / CT * 16 + l % 16, col = col0 + tile % CT * 16 + l / 16 * 4;
        const int n = (int)min((int64_t)4, p.M - col);
        if (row >= p.N || n <= 0) continue;
        float v[4] = {s[0], s[1], s[2], s[3]}, t[4];
        if (p.bias) {
            if (p.bias_f32) mm::load4(static_cast<const float *>(p.bias) + col, n, t);
            else mm::load4(static_cast<const T *>(p.bias) + col, n, t);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += t[k];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = p.y_f32 ? mm::act_fine(p.act, v[k]) : mm::act_value(p.act, v[k]);
        if (p.res) {
            mm::load4(static_cast<const T *>(p.res) + row * p.ldr + col, n, t);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += t[k];
        }
        if (p.y_f32) mm::store4(static_cast<float *>(p.y) + row * p.ldy + col, n, v);
        else mm::store4(static_cast<T *>(p.y) + row * p.ldy + col, n, v);
    }
}

template <typename T, bool PACKED, int RT, int CT> hipError_t launch(const FourProduct &p, hipStream_t st)
{
    const dim3 grid = grid_of((p.N + RT * 16 - 1) / (RT * 16) * ((p.M + CT * 16 - 1) / (CT * 16)));
    if (grid.x == 0) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_mx4_few<T, PACKED, RT, CT>), grid, dim3(64 * kWaves), 0, st, p);
    return hipGetLastError();
}

template <typename T, bool PACKED> hipError_t by_rows(const FourProduct &p, hipStream_t st)
{
    if (p.N <= 16) return launch<T, PACKED, 1, 1>(p, st);
    if (p.N <= 32) return launch<T, PACKED, 2, 2>(p, st);
    return launch<T, PACKED, 4, 2>(p, st);
}

}  // namespace

hipError_t launch_mx4_few(bool bf16, const FourProduct &p, hipStream_t st)
{
    if (p.x_scales) return bf16 ? by_rows<__bf16, true>(p, st) : by_rows<_Float16, true>(p, st);
    return bf16 ? by_rows<__bf16, false>(p, st) : by_rows<_Float16, false>(p, st);
}

}  // namespace som
