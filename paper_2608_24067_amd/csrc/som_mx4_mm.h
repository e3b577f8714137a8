// som_mx4_mm.h -- products of many rows with a 4-bit matrix: rows in 4 bits too, or in 16.
//
// A workgroup computes a BM x BN tile of the result, each wave a part of it in 16 x 16 blocks. Operands
// go straight to LDS in 16-byte chunks, kStages tiles in a ring, in rows of 64 bytes: 128 codes (four
// blocks), or 32 values of 16 bits; the chunks' places are those of som_mm.h's "along" operands, so
// that a read of a fragment touches every bank once. The blocks' scales lie beside them, four steps' of
// a row at a time.
//   Rows in 4 bits: a step takes 128 features by v_mfma_scale_f32_16x16x128_f8f6f4, which applies
//     both blocks' scales: lane (q, i) holds block q of row i.
//   Rows in 16 bits: a step takes 32 features, one block of each column, by v_mfma_f32_16x16x32. The
//     codes come with every fourth step and are widened in registers, where a wave's rows share them: to
//     bf16 under their scale, which is exact; to fp16 without it, since fp16 does not hold all scales,
//     and the instruction's sums over the block are then added under the scale in fp32.
//
// Operands must be whole 16-byte chunks (the host copies others to the workspace). Chunks past the last
// feature are read as zeros, rows and columns past the last ones repeat it.
#pragma once

#include "som_layer.h"
#include "som_mm.h"

namespace som {
namespace four {

using mm::bf16x8;
using mm::f16x8;
using mm::f32x4;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

template <int BM_, int BN_, int WM_, int WN_, int PER_CU_> struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, PER_CU = PER_CU_, NT = 64 * WM_ * WN_;
    static constexpr int MI = BM_ / WM_ / 16, NI = BN_ / WN_ / 16;
};

constexpr int kStages = 4;
constexpr int kRowBytes = 64;

// BYTES-byte pieces (16 or 4) of a row's scales, one row a thread, straight to LDS.
template <int BYTES> __device__ inline void load_scales(const uint8_t *row, int64_t piece, int64_t pieces, uint32_t lds)
{
    const void *from = row + min(piece, pieces - 1) * BYTES;  // past the last one nothing is multiplied
    if (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(from) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds), "v"(from) : "memory");
}

// 2^(s - 127), a subnormal for 0 and NaN for 255; no branch, which a choice would become.
__device__ inline float scale_value(uint32_t s) { return __uint_as_float(max(s << 23, 0x00400000u) | (s + 1) >> 8 << 22); }

template <int V> struct Number {
    static constexpr int value = V;
};

__device__ inline uint32_t lds_byte(uint32_t at) { return *(const __attribute__((address_space(3))) uint8_t *)(uintptr_t)at; }
__device__ inline uint32_t lds_word(uint32_t at) { return *(const __attribute__((address_space(3))) uint32_t *)(uintptr_t)at; }
__device__ inline i32x4 lds_chunk(uint32_t at) { return *(const __attribute__((address_space(3))) i32x4 *)(uintptr_t)at; }

// Bias, activation, residual and the store, for a wave's MI x NI blocks. COLUMN: a lane holds rows 4g
// ... 4g + 3 of column i of each block, else row i and columns 4g ... 4g + 3. Sixteen rows at a time
// go through LDS, so that a row's columns are read and written side by side; the residual is loaded
// sixteen rows ahead.
template <typename T, int MI, int NI, bool COLUMN>
__device__ inline void finish(const FourProduct &p, const f32x4 (&acc)[MI][NI], int row0, int col0, float *own)
{
    constexpr int kCols = NI * 16, kRow = kCols + 4, kLanes = kCols / 4, kAtOnce = 64 / kLanes, kTurns = 16 / kAtOnce;
    const int lane = (int)threadIdx.x & 63, g = lane >> 4, li = lane & 15;
    const int sub = lane / kLanes, n = col0 + lane % kLanes * 4, cnt = min(4, (int)p.M - n);
    float bias[4] = {0, 0, 0, 0};
    if (p.bias && cnt > 0) {
        if (p.bias_f32) mm::load4(static_cast<const float *>(p.bias) + n, cnt, bias);
        else mm::load4(static_cast<const T *>(p.bias) + n, cnt, bias);
    }
    typedef T vec4 __attribute__((ext_vector_type(4)));
    typedef vec4 any4 __attribute__((aligned(sizeof(T))));
    const bool cols_in = col0 + kCols <= (int)p.M;
    vec4 ahead[kTurns];
    auto is_whole = [&](int i) { return cols_in && row0 + 16 * i + 16 <= (int)p.N; };
    auto fetch16 = [&](int i) {
        if (!p.res || i >= MI || !is_whole(i)) return;
#pragma unroll
        for (int r = 0; r < kTurns; ++r)
            ahead[r] = *reinterpret_cast<const any4 *>(static_cast<const T *>(p.res) +
                                                       (int64_t)(row0 + 16 * i + r * kAtOnce + sub) * p.ldr + n);
    };
    fetch16(0);
    auto rows16 = [&](int i, auto whole) {
        constexpr bool W = decltype(whole)::value;
        vec4 now[kTurns];
#pragma unroll
        for (int r = 0; r < kTurns; ++r) now[r] = ahead[r];
        fetch16(i + 1);
        float v[kTurns][4];
#pragma unroll
        for (int r = 0; r < kTurns; ++r) {
            const f32x4 c = *reinterpret_cast<const f32x4 *>(own + (r * kAtOnce + sub) * kRow + lane % kLanes * 4);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[r][q] = c[q] + bias[q];
        }
        auto activate = [&](auto f) {
#pragma unroll
            for (int r = 0; r < kTurns; ++r)
#pragma unroll
                for (int q = 0; q < 4; ++q) v[r][q] = f(v[r][q]);
        };
        if (p.act == SOM_ACT_RELU) activate([](float z) { return mm::act_value(SOM_ACT_RELU, z); });
        else if (p.act == SOM_ACT_GELU && p.y_f32) activate([](float z) { return mm::act_fine(SOM_ACT_GELU, z); });
        else if (p.act == SOM_ACT_GELU) activate([](float z) { return mm::act_value(SOM_ACT_GELU, z); });
        else if (p.act == SOM_ACT_SILU && p.y_f32) activate([](float z) { return mm::act_fine(SOM_ACT_SILU, z); });
        else if (p.act == SOM_ACT_SILU) activate([](float z) { return mm::act_value(SOM_ACT_SILU, z); });
#pragma unroll
        for (int r = 0; r < kTurns; ++r) {
            const int64_t m = row0 + 16 * i + r * kAtOnce + sub;
            if (!W && (m >= p.N || cnt <= 0)) continue;
            const int c4 = W ? 4 : cnt;
            if (p.res) {
                float t[4];
                if (W) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) t[q] = (float)now[r][q];
                } else {
                    mm::load4(static_cast<const T *>(p.res) + m * p.ldr + n, c4, t);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) v[r][q] += t[q];
            }
            if (p.y_f32) mm::store4(static_cast<float *>(p.y) + m * p.ldy + n, c4, v[r]);
            else mm::store4(static_cast<T *>(p.y) + m * p.ldy + n, c4, v[r]);
        }
    };
#pragma unroll 1
    for (int i = 0; i < MI; ++i) {  // rolled: the code of sixteen rows stands here once
#pragma unroll
        for (int at = 0; at < MI; ++at) {
            if (at != i) continue;
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                if (COLUMN) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) own[(4 * g + q) * kRow + j * 16 + li] = acc[at][j][q];
                } else {
                    *reinterpret_cast<f32x4 *>(own + li * kRow + j * 16 + 4 * g) = acc[at][j];
                }
            }
        }
        mm::wave_sync_lds();
        if (is_whole(i)) rows16(i, mm::Inside<true>());
        else rows16(i, mm::Inside<false>());
        mm::wave_sync_lds();
    }
}

// The tile of this workgroup; false where it has none.
template <class S> __device__ inline bool place(const FourProduct &p, int &m0, int &n0)
{
    const int nm = (int)((p.N + S::BM - 1) / S::BM), nn = (int)((p.M + S::BN - 1) / S::BN);
    const int64_t t = mm::tile_of(mm::block_number(), (int64_t)nm * nn);
    if (t < 0) return false;
    int mt, nt;
    mm::tile_place(t, nm, nn, mt, nt);
    m0 = mt * S::BM;
    n0 = nt * S::BN;
    return true;
}

// LDS: the rings of tiles, then two places for each operand's scales.
template <class S> struct Packed {
    static constexpr int kA = S::BM * kRowBytes, kB = S::BN * kRowBytes, kStage = kA + kB;
    static constexpr int kScales = kStages * kStage, kPlace = (S::BM + S::BN) * 16;
    static constexpr int kEnd = S::WM * S::WN * 16 * (S::NI * 16 + 4) * 4;
    static constexpr int kBytes = kScales + 2 * kPlace > kEnd ? kScales + 2 * kPlace : kEnd;
};

template <typename T, class S> __global__ __launch_bounds__(S::NT, S::PER_CU * S::NT / 256) void k_mx4_packed(const FourProduct p)
{
    typedef Packed<S> L;
    extern __shared__ __align__(1024) char lds[];
    int m0, n0;
    if (!place<S>(p, m0, n0)) return;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const int wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, li = lane & 15;
    const int64_t blocks = four_blocks(p.K);
    const int K = (int)blocks * 8, steps = (K + mm::kBK - 1) / mm::kBK, pieces = (int)((blocks + 15) / 16);  // K: pairs of bytes
    typedef mm::Loader<short, S::BM, false, false, S::NT> LoadA;
    typedef mm::Loader<short, S::BN, false, false, S::NT> LoadB;
    LoadA la;
    LoadB lb;
    la.template init<true>(static_cast<const short *>(p.x), K, nullptr, m0, (int)p.N, 0, K);
    lb.template init<true>(reinterpret_cast<const short *>(p.w), K, nullptr, n0, (int)p.M, 0, K);
    // A thread's row of scales: BM of x, then BN of w.
    static_assert(S::BM + S::BN == S::NT, "a row of scales a thread");
    const int sr = (int)threadIdx.x;
    const uint8_t *scale_row = sr < S::BM ? p.x_scales + (int64_t)min(m0 + sr, (int)p.N - 1) * p.x_pitch
                                          : p.w_scales + (int64_t)min(n0 + sr - S::BM, (int)p.M - 1) * p.w_pitch;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

    f32x4 acc[S::MI][S::NI];
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    // As in som_mm.h: step t multiplies tile t; its fragments of B and its first ones of A are in
    // registers when it starts, those of tile t + 1 are read meanwhile, and tiles up to t + kStages - 1
    // are on their way to LDS. A piece of scales goes ahead of the first tile it serves.
    struct Fragment {
        i32x4 v;
        uint32_t scale;
    };
    const uint32_t at_a = wm * S::MI * 16, at_b = wn * S::NI * 16, slot = (uint32_t)((q ^ mm::chunk_xor(li)) << 4);
    const uint32_t va = (at_a + li) * kRowBytes + slot, vb = L::kA + (at_b + li) * kRowBytes + slot;
    const uint32_t vsa = (at_a + li) * 16 + q, vsb = (S::BM + at_b + li) * 16 + q;
    static_assert(kStages == 4, "a ring of as many tiles as pieces of scales have steps");
    auto codes_at = [&](int t) { return base + (uint32_t)(t % kStages) * L::kStage; };
    auto scales_at = [&](int t) { return base + L::kScales + (uint32_t)(t / 4 % 2) * L::kPlace + (uint32_t)(t % 4) * 4; };
    auto read_a = [&](int t, int i) {
        return Fragment{lds_chunk(codes_at(t) + va + i * (16 * kRowBytes)), lds_byte(scales_at(t) + vsa + i * 256)};
    };
    auto read_b = [&](int t, int j) {
        return Fragment{lds_chunk(codes_at(t) + vb + j * (16 * kRowBytes)), lds_byte(scales_at(t) + vsb + j * 256)};
    };
    auto multiply = [&](const Fragment &b, const Fragment &a, f32x4 c) {
        const i32x8 w = {b.v[0], b.v[1], b.v[2], b.v[3], 0, 0, 0, 0}, x = {a.v[0], a.v[1], a.v[2], a.v[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 4, 4, 0, (int)b.scale, 0, (int)a.scale);
    };
    auto scales = [&](int t) {  // of the four steps from t on
        load_scales<16>(scale_row, t / 4, pieces, base + L::kScales + (uint32_t)(t / 4 % 2) * L::kPlace + wave * 1024);
    };
    constexpr int kLoads = LoadA::kPer + LoadB::kPer;
    static_assert(LoadA::kChunks % S::NT == 0 && LoadB::kChunks % S::NT == 0, "every thread loads");
#pragma unroll
    for (int t = 0; t < kStages - 1; ++t) {
        if (t == 0) scales(0);
#pragma unroll
        for (int i = 0; i < LoadA::kPer; ++i) la.template async<false>(i, base + t * L::kStage);
#pragma unroll
        for (int i = 0; i < LoadB::kPer; ++i) lb.template async<false>(i, base + t * L::kStage + L::kA);
        la.advance();
        lb.advance();
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 2) * kLoads) : "memory");
    constexpr int kWindow = S::MI < 4 ? S::MI : 4;
    Fragment even[S::NI], odd[S::NI], a[kWindow];
#pragma unroll
    for (int j = 0; j < S::NI; ++j) even[j] = read_b(0, j);
#pragma unroll
    for (int i = 0; i < kWindow; ++i) a[i] = read_a(0, i);
    // U: t % 4. No branch stands between a step's instructions: past one the compiler would move them.
    auto step = [&](int t, auto u, const Fragment (&now)[S::NI], Fragment (&then)[S::NI]) {
        constexpr int U = decltype(u)::value;
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 3) * kLoads) : "memory");
        const uint32_t to = base + (uint32_t)((U + kStages - 1) % kStages) * L::kStage;
        if ((U + kStages - 1) % 4 == 0) scales(t + kStages - 1);
        constexpr int kB = (2 * S::NI + S::MI - 1) / S::MI, kOf = (kLoads + S::MI - 1) / S::MI;
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
#pragma unroll
            for (int j = 0; j < S::NI; ++j) acc[i][j] = multiply(now[j], a[i % kWindow], acc[i][j]);
            a[i % kWindow] = i + kWindow < S::MI ? read_a(t, i + kWindow) : read_a(t + 1, i + kWindow - S::MI);
#pragma unroll
            for (int j = i * kB; j < (i + 1) * kB && j < S::NI; ++j) then[j] = read_b(t + 1, j);
#pragma unroll
            for (int c = i * kOf; c < (i + 1) * kOf && c < kLoads; ++c) {
                if (c < LoadA::kPer) la.template async<false>(c, to);
                else lb.template async<false>(c - LoadA::kPer, to + L::kA);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        la.advance();
        lb.advance();
    };
    int t = 0;
    for (; t + 4 <= steps; t += 4) {
        step(t, Number<0>(), even, odd);
        step(t + 1, Number<1>(), odd, even);
        step(t + 2, Number<2>(), even, odd);
        step(t + 3, Number<3>(), odd, even);
    }
    if (t < steps) step(t, Number<0>(), even, odd);
    if (t + 1 < steps) step(t + 1, Number<1>(), odd, even);
    if (t + 2 < steps) step(t + 2, Number<2>(), even, odd);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing lands in LDS after the workgroup left it
    __syncthreads();  // the tiles are no longer read
    finish<T, S::MI, S::NI, false>(p, acc, m0 + (int)at_a, n0 + (int)at_b,
                                   reinterpret_cast<float *>(lds) + wave * (16 * (S::NI * 16 + 4)));
}

// LDS: x's ring, two places for the codes and two for the scales, of four steps each.
template <class S> struct Half {
    static constexpr int kA = S::BM * kRowBytes, kB = S::BN * kRowBytes, kPlace = S::BN * 4;
    static constexpr int kCodes = kStages * kA, kScales = kCodes + 2 * kB;
    static constexpr int kEnd = S::WM * S::WN * 16 * (S::NI * 16 + 4) * 4;
    static constexpr int kBytes = kScales + 2 * kPlace > kEnd ? kScales + 2 * kPlace : kEnd;
};

template <typename T, class S> __global__ __launch_bounds__(S::NT, S::PER_CU * S::NT / 256) void k_mx4_half(const FourProduct p)
{
    typedef Half<S> L;
    constexpr bool kScaled = sizeof(T) == 2 && __is_same(T, __bf16);  // the widened codes hold their scale
    typedef typename mm::Vec8<T>::type Frag;
    extern __shared__ __align__(1024) char lds[];
    int m0, n0;
    if (!place<S>(p, m0, n0)) return;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const int wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, li = lane & 15;
    const int64_t blocks = four_blocks(p.K);
    const int K = (int)p.K, steps = (int)blocks, KB = (int)blocks * 8;
    typedef mm::Loader<T, S::BM, false, false, S::NT> LoadA;
    typedef mm::Loader<short, S::BN, false, false, S::NT> LoadB;
    LoadA la;
    LoadB lb;
    la.template init<true>(static_cast<const T *>(p.x), p.ldx, nullptr, m0, (int)p.N, 0, K);
    lb.template init<true>(reinterpret_cast<const short *>(p.w), KB, nullptr, n0, (int)p.M, 0, KB);
    // A thread's column of scales; the later waves repeat the earlier ones' loads.
    static_assert(S::NT % S::BN == 0, "whole columns");
    const uint8_t *scale_row = p.w_scales + (int64_t)min(n0 + (int)threadIdx.x % S::BN, (int)p.M - 1) * p.w_pitch;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const uint32_t at_a = wm * S::MI * 16, at_b = wn * S::NI * 16;
    mm::Reader<T, S::BM, false> ra;
    ra.init((int)at_a);

    f32x4 acc[S::MI][S::NI];
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    struct Raw {
        uint32_t codes, scale;
    };
    struct Wide {
        Frag v;
        float scale;
    };
    const uint32_t vb = L::kCodes + (at_b + li) * kRowBytes + 4 * q, vx = (uint32_t)mm::chunk_xor(li) << 4, vs = L::kScales + (at_b + li) * 4;
    auto read_b = [&](int t, int j) {
        return Raw{lds_word(base + (uint32_t)(t / 4 % 2) * L::kB + vb + (((uint32_t)(t % 4) << 4) ^ vx) + j * (16 * kRowBytes)),
                   lds_byte(base + (uint32_t)(t / 4 % 2) * L::kPlace + (uint32_t)(t % 4) + vs + j * 64)};
    };
    auto widen = [&](const Raw &r) {
        Wide w;
        w.scale = scale_value(r.scale);
        if constexpr (kScaled) {
            typedef __bf16 two __attribute__((ext_vector_type(2)));
            const two x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, w.scale, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, w.scale, 1);
            const two x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, w.scale, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.codes, w.scale, 3);
            w.v = Frag{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
        } else {
            typedef _Float16 two __attribute__((ext_vector_type(2)));
            const two x0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(r.codes, 1.0f, 0), x1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(r.codes, 1.0f, 1);
            const two x2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(r.codes, 1.0f, 2), x3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(r.codes, 1.0f, 3);
            w.v = Frag{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
        }
        return w;
    };
    auto multiply = [&](const Wide &b, const Frag &a, f32x4 c) {
        if constexpr (kScaled) return mm::mma(b.v, a, c);
        const f32x4 s = mm::mma(a, b.v, f32x4{0, 0, 0, 0});
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = fmaf(s[k], b.scale, c[k]);
        return c;
    };
    constexpr int kLoads = LoadA::kPer;
    static_assert(LoadA::kChunks % S::NT == 0 && LoadB::kChunks % S::NT == 0, "every thread loads");
    auto load_codes = [&](int t) {  // and scales, of the four steps from t on
        load_scales<4>(scale_row, t / 4, p.w_pitch / 4, base + L::kScales + (uint32_t)(t / 4 % 2) * L::kPlace + wave % (S::BN / 64) * 256);
        const uint32_t to = base + L::kCodes + (uint32_t)(t / 4 % 2) * L::kB;
#pragma unroll
        for (int i = 0; i < LoadB::kPer; ++i) lb.template async<false>(i, to);
        lb.advance();
    };
#pragma unroll
    for (int t = 0; t < kStages - 1; ++t) {
        if (t == 0) load_codes(0);
#pragma unroll
        for (int i = 0; i < LoadA::kPer; ++i) la.template async<false>(i, base + t * L::kA);
        la.advance();
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 2) * kLoads) : "memory");
    constexpr int kWindow = S::MI < 4 ? S::MI : 4;
    Wide even[S::NI], odd[S::NI];
    Frag a[kWindow];
#pragma unroll
    for (int j = 0; j < S::NI; ++j) even[j] = widen(read_b(0, j));
#pragma unroll
    for (int i = 0; i < kWindow; ++i) a[i] = ra.read(base, i);
    // U: t % 4; as above, no branches.
    auto step = [&](int t, auto u, const Wide (&now)[S::NI], Wide (&then)[S::NI]) {
        constexpr int U = decltype(u)::value;
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 3) * kLoads) : "memory");
        const uint32_t here = base + (uint32_t)(U % kStages) * L::kA, next = base + (uint32_t)((U + 1) % kStages) * L::kA;
        const uint32_t to = base + (uint32_t)((U + kStages - 1) % kStages) * L::kA;
        if ((U + kStages - 1) % 4 == 0) load_codes(t + kStages - 1);
        Raw raw[S::NI];
        // The next step's codes are read with the first row of blocks and widened with the later ones.
        constexpr int kFrom = S::MI / 2, kB = (S::NI + S::MI - kFrom - 1) / (S::MI - kFrom), kOf = (kLoads + S::MI - 1) / S::MI;
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
            if (i == 0) {
#pragma unroll
                for (int j = 0; j < S::NI; ++j) raw[j] = read_b(t + 1, j);
            }
#pragma unroll
            for (int j = 0; j < S::NI; ++j) acc[i][j] = multiply(now[j], a[i % kWindow], acc[i][j]);
            a[i % kWindow] = i + kWindow < S::MI ? ra.read(here, i + kWindow) : ra.read(next, i + kWindow - S::MI);
            if (i >= kFrom) {
#pragma unroll
                for (int j = (i - kFrom) * kB; j < (i - kFrom + 1) * kB && j < S::NI; ++j) then[j] = widen(raw[j]);
            }
#pragma unroll
            for (int c = i * kOf; c < (i + 1) * kOf && c < kLoads; ++c) la.template async<false>(c, to);
            __builtin_amdgcn_sched_barrier(0);
        }
        la.advance();
    };
    int t = 0;
    for (; t + 4 <= steps; t += 4) {
        step(t, Number<0>(), even, odd);
        step(t + 1, Number<1>(), odd, even);
        step(t + 2, Number<2>(), even, odd);
        step(t + 3, Number<3>(), odd, even);
    }
    if (t < steps) step(t, Number<0>(), even, odd);
    if (t + 1 < steps) step(t + 1, Number<1>(), odd, even);
    if (t + 2 < steps) step(t + 2, Number<2>(), even, odd);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing lands in LDS after the workgroup left it
    __syncthreads();  // the tiles are no longer read
    finish<T, S::MI, S::NI, !kScaled>(p, acc, m0 + (int)at_a, n0 + (int)at_b,
                                      reinterpret_cast<float *>(lds) + wave * (16 * (S::NI * 16 + 4)));
}

template <class S> int64_t tiles(const FourProduct &p) { return (p.N + S::BM - 1) / S::BM * ((p.M + S::BN - 1) / S::BN); }

// The attribute belongs to the function on each device; setting it again changes nothing.
template <typename F> hipError_t allow_lds(F *f, int bytes, std::atomic<uint64_t> &done)
{
    int dev = 0;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess || bytes <= 64 << 10 || (dev <= 63 && done.load() >> dev & 1)) return e;
    const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(f), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (err == hipSuccess && dev <= 63) done.fetch_or(1ull << dev);
    return err;
}

}  // namespace four
}  // namespace som
