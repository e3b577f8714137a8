// som_mx4_few.hip -- products with a 4-bit matrix, for few rows.
//
// A workgroup takes RT x 16 rows by CT x 16 columns, and its eight waves share out the features in
// units of 128 (four blocks), whose sums are joined in LDS. Both operands go straight into registers, a
// unit ahead of the one that is multiplied: a lane (q, i) of a wave loads block q of column i, 16 bytes.
//   Rows in 4 bits: it loads block q of row i likewise, and one instruction takes both operands' 128
//     codes and applies the blocks' scales.
//   Rows in 16 bits: they are read in the instruction's own order, eight features of block b by lane
//     (q, i), so that a row's 64 bytes are read side by side (the order of the codes, 16 bytes here and
//     there, took twice as long); the codes get into it by a 4 x 4 exchange of words between the lanes
//     of a column. They are widened to bf16 under their scale, or to fp16 without it: fp16 does not hold
//     all scales, and the instruction's sums over one block are then added under the scale in fp32.
// bf16 and 4 bits: the matrix is the instruction's first operand, so that a lane owns four neighbouring
// columns of a row; fp16: the rows are, so that it owns one column, under one scale.
// Bound by a CU's reads and, at the smallest sizes, by what a launch and the first loads take: 1 x 1024 x 4096
// takes 3.8 us (2.2 MB), 1 x 4096 x 4096 6.0 (8.9 MB), 64 x 4096 x 4096 in bf16 14.8 with 32 x 32 a workgroup,
// 33 x 2048 x 8192 11.4 with 32 x 64 (12.5 before the join took all threads and bias and residual came early).

#include "som_layer_device.h"
#include "som_mm.h"

namespace som {
namespace {

using namespace layer;
using mm::f32x4;

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8, kUnit = 128;

// Words w[s] of the four lanes (q, i) of each i: word s of lane q changes places with word q of lane s.
__device__ inline void exchange(uint32_t (&w)[4])
{
    auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    w[0] = c[0], w[1] = c[1], w[2] = d[0], w[3] = d[1];
}

template <typename T, bool PACKED, int RT, int CT> struct Operands {
    typedef typename mm::Vec8<T>::type Eight;
    uint4 w[CT], xc[PACKED ? RT : 1];
    uint32_t ws[CT], xs[PACKED ? RT : 1];  // rows in 16 bits: the bytes of the unit's four blocks
    Eight x[PACKED ? 1 : RT][4];
};

template <typename T, bool PACKED, int RT, int CT> __global__ __launch_bounds__(64 * kWaves) void k_mx4_few(const FourProduct p)
{
    typedef Operands<T, PACKED, RT, CT> Unit;
    constexpr bool kColumn = !PACKED && __is_same(T, _Float16);
    __shared__ f32x4 joined[kWaves][RT * CT][64];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int q = lane >> 4, i = lane & 15;
    const int64_t across = (p.M + CT * 16 - 1) / (CT * 16), b = mm::block_number();
    const int64_t row0 = b / across * (RT * 16), col0 = b % across * (CT * 16);
    if (row0 >= p.N) return;
    const int64_t blocks = four_blocks(p.K);
    const int units = (int)((p.K + kUnit - 1) / kUnit);
    int64_t wrow[CT], xrow[RT];  // the first block of a column, the first element (block) of a row
#pragma unroll
    for (int c = 0; c < CT; ++c) wrow[c] = min(col0 + 16 * c + i, p.M - 1) * blocks;
#pragma unroll
    for (int r = 0; r < RT; ++r) xrow[r] = min(row0 + 16 * r + i, p.N - 1) * (PACKED ? blocks : p.ldx);

    // Unit u; WHOLE: it lies within the features.
    auto load = [&](int u, Unit &o, auto whole) {
        constexpr bool W = decltype(whole)::value;
        const int64_t first = 4 * (int64_t)u, block = first + q;
        const bool in = W || block < blocks;
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            o.w[c] = uint4{0, 0, 0, 0};
            o.ws[c] = 127;
            if (in) o.w[c] = reinterpret_cast<const uint4 *>(p.w)[wrow[c] + block];
            const uint8_t *s = p.w_scales + wrow[c];
            if (PACKED) {
                if (in) o.ws[c] = s[block];
            } else if (W) {
                typedef uint32_t any __attribute__((aligned(1)));
                o.ws[c] = *reinterpret_cast<const any *>(s + first);
            } else {
                o.ws[c] = 0x7F7F7F7F;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (first + k < blocks) o.ws[c] = (o.ws[c] & ~(255u << (8 * k))) | (uint32_t)s[first + k] << (8 * k);
            }
        }
        if constexpr (PACKED) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                o.xc[r] = uint4{0, 0, 0, 0};
                o.xs[r] = 127;
                if (in) o.xc[r] = static_cast<const uint4 *>(p.x)[xrow[r] + block], o.xs[r] = p.x_scales[xrow[r] + block];
            }
        } else {
            typedef typename Unit::Eight any __attribute__((aligned(2)));
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const T *x = static_cast<const T *>(p.x) + xrow[r] + first * kFourBlock + 8 * q;
#pragma unroll
                for (int k = 0; k < 4; ++k, x += kFourBlock) {
                    const int64_t left = p.K - (first + k) * kFourBlock - 8 * q;
                    if (W || left >= 8) {
                        o.x[r][k] = *reinterpret_cast<const any *>(x);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) o.x[r][k][e] = e < left ? x[e] : (T)0.0f;
                    }
                }
            }
        }
    };
    f32x4 acc[RT][CT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[r][c] = f32x4{0, 0, 0, 0};
    auto multiply = [&](const Unit &o) {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            if constexpr (PACKED) {
                const i32x8 w = {(int)o.w[c].x, (int)o.w[c].y, (int)o.w[c].z, (int)o.w[c].w, 0, 0, 0, 0};
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const i32x8 x = {(int)o.xc[r].x, (int)o.xc[r].y, (int)o.xc[r].z, (int)o.xc[r].w, 0, 0, 0, 0};
                    acc[r][c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc[r][c], 4, 4, 0, (int)o.ws[c], 0, (int)o.xs[r]);
                }
            } else {
                uint32_t words[4] = {o.w[c].x, o.w[c].y, o.w[c].z, o.w[c].w};
                exchange(words);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t s = o.ws[c] >> (8 * k) & 255;
                    const typename Unit::Eight w = widen8<T>(words[k], s);
                    if constexpr (kColumn) {
                        const float scale = scale_value(s);
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            const f32x4 sum = mm::mma(o.x[r][k], w, f32x4{0, 0, 0, 0});
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[r][c][e] = fmaf(sum[e], scale, acc[r][c][e]);
                        }
                    } else {
#pragma unroll
                        for (int r = 0; r < RT; ++r) acc[r][c] = mm::mma(w, o.x[r][k], acc[r][c]);
                    }
                }
            }
        }
    };
    // A thread's four results after the join: four columns of a row, or (kColumn) four rows of a column.
    // Their bias and residual are loaded first, so that nothing waits for them at the end.
    static_assert(RT * CT <= kWaves, "four results a thread");
    const int64_t row = row0 + 16 * (wave / CT) + (kColumn ? q * 4 : i), col = col0 + 16 * (wave % CT) + (kColumn ? i : q * 4);
    const int n = wave < RT * CT && row < p.N && col < p.M ? (int)min((int64_t)4, kColumn ? p.N - row : p.M - col) : 0;
    float bias[4] = {0, 0, 0, 0}, res[4] = {0, 0, 0, 0};
    if (p.bias && n > 0) {
        if (p.bias_f32) mm::load4(static_cast<const float *>(p.bias) + col, kColumn ? 1 : n, bias);
        else mm::load4(static_cast<const T *>(p.bias) + col, kColumn ? 1 : n, bias);
    }
    if (p.res && n > 0) {
        const T *from = static_cast<const T *>(p.res) + row * p.ldr + col;
        if constexpr (kColumn) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < n) res[k] = (float)from[k * p.ldr];
        } else {
            mm::load4(from, n, res);
        }
    }
    // A wave's units are kWaves apart; the last unit of all may be a part of one.
    const int whole = (int)(p.K / kUnit);
    Unit even, odd;
    int u = wave;
    if (u < whole) load(u, even, mm::Inside<true>());
    for (; u + kWaves < whole; u += 2 * kWaves) {
        load(u + kWaves, odd, mm::Inside<true>());
        multiply(even);
        if (u + 2 * kWaves < whole) load(u + 2 * kWaves, even, mm::Inside<true>());
        multiply(odd);
    }
    if (u < whole) multiply(even), u += kWaves;
    if (u < units) {
        load(u, odd, mm::Inside<false>());
        multiply(odd);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) joined[wave][r * CT + c][lane] = acc[r][c];
    __syncthreads();
    if (n <= 0) return;
    f32x4 s = joined[0][wave][lane];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) s += joined[k][wave][lane];
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = s[k] + bias[kColumn ? 0 : k];
    if (p.act != SOM_ACT_NONE) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = p.y_f32 ? mm::act_fine(p.act, v[k]) : mm::act_value(p.act, v[k]);
    }
    if (p.res) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += res[k];
    }
    if constexpr (kColumn) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k >= n) continue;
            if (p.y_f32) static_cast<float *>(p.y)[(row + k) * p.ldy + col] = v[k];
            else static_cast<T *>(p.y)[(row + k) * p.ldy + col] = (T)v[k];
        }
    } else if (p.y_f32) {
        mm::store4(static_cast<float *>(p.y) + row * p.ldy + col, n, v);
    } else {
        mm::store4(static_cast<T *>(p.y) + row * p.ldy + col, n, v);
    }
}

template <typename T, bool PACKED, int RT, int CT> hipError_t launch(const FourProduct &p, hipStream_t st)
{
    const dim3 grid = grid_of((p.N + RT * 16 - 1) / (RT * 16) * ((p.M + CT * 16 - 1) / (CT * 16)));
    if (grid.x == 0) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_mx4_few<T, PACKED, RT, CT>), grid, dim3(64 * kWaves), 0, st, p);
    return hipGetLastError();
}

template <typename T, bool PACKED> hipError_t by_tile(FourTile t, const FourProduct &p, hipStream_t st)
{
    if (t == kFour16x16) return launch<T, PACKED, 1, 1>(p, st);
    if (t == kFour16x32) return launch<T, PACKED, 1, 2>(p, st);
    if constexpr (!PACKED && __is_same(T, __bf16))
        if (t == kFour32x64) return launch<T, PACKED, 2, 4>(p, st);
    return launch<T, PACKED, 2, 2>(p, st);
}

}  // namespace

hipError_t launch_mx4_few(bool bf16, FourTile t, const FourProduct &p, hipStream_t st)
{
    if (p.x_scales) return bf16 ? by_tile<__bf16, true>(t, p, st) : by_tile<_Float16, true>(t, p, st);
    return bf16 ? by_tile<__bf16, false>(t, p, st) : by_tile<_Float16, false>(t, p, st);
}

}  // namespace som
