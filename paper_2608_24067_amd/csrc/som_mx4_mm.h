// som_mx4_mm.h -- products of many rows with a 4-bit matrix: rows in 4 bits too, or in 16.
//
// A workgroup computes a BM x BN tile of the result, each wave a part of it in 16 x 16 blocks. Operands
// go straight to LDS in lines of 128 bytes a row (line_xor's places keep the reads free of bank
// conflicts), two tiles of them by turns; the blocks' scales lie beside them.
//   Rows in 4 bits: a step takes 128 features by v_mfma_scale_f32_16x16x128_f8f6f4, which applies
//     both blocks' scales: lane (q, i) holds block q of row i.
//   Rows in 16 bits: a step takes 32 features, one block of each column, by v_mfma_f32_16x16x32. The
//     codes come for eight steps at a time and are widened in registers, where a wave's rows share them,
//     under their scale, which is exact: to bf16, and to fp16 relative to the tile's largest scale. A tile
//     whose scales fp16 does not span widens without them; the instruction's sums over a block are then
//     added under the scale in fp32, four additions for each instruction.
// Measured, us and TFLOP/s: 8192 x 4096 x 4096 rows in 4 bits 77 and 3,560, in bf16 200 and 1,370, in fp16 212
// and 1,300 (316 and 870 without the scales; by 256 x 256 it spills six registers). Of 8192 x 2048 x 4096 in 4 bits, 54 us, some 30 go to the
// first loads and the results' stores, during which the matrix units wait: there is one workgroup a CU.
//
// Rows must be whole lines (the host copies others to the workspace). Rows and columns past the last
// ones repeat it; codes past the last feature meet zeros, or scales that make them nothing.
#pragma once

#include "som_layer_device.h"
#include "som_mm.h"

namespace som {
namespace four {

using mm::bf16x8;
using mm::f16x8;
using mm::f32x4;
using layer::scale_value;
using layer::widen8;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// PER_CU: workgroups of a CU.
template <int BM_, int BN_, int WM_, int WN_, int PER_CU_> struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, PER_CU = PER_CU_, NT = 64 * WM_ * WN_;
    static constexpr int MI = BM_ / WM_ / 16, NI = BN_ / WN_ / 16;
    static constexpr int WINDOW = MI % 4 || MI < 4 ? MI / 2 : 4;  // fragments of A in registers; they divide MI
};

// BYTES-byte pieces (16 or 4) of a row's scales, one row a thread, straight to LDS.
template <int BYTES> __device__ inline void load_scales(const uint8_t *row, int64_t piece, int64_t pieces, uint32_t lds)
{
    const void *from = row + min(piece, pieces - 1) * BYTES;  // past the last one nothing is multiplied
    if (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(from) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds), "v"(from) : "memory");
}

template <int V> struct Number {
    static constexpr int value = V;
};

__device__ inline uint32_t lds_byte(uint32_t at) { return *(const __attribute__((address_space(3))) uint8_t *)(uintptr_t)at; }
__device__ inline uint32_t lds_word(uint32_t at) { return *(const __attribute__((address_space(3))) uint32_t *)(uintptr_t)at; }
__device__ inline i32x4 lds_chunk(uint32_t at) { return *(const __attribute__((address_space(3))) i32x4 *)(uintptr_t)at; }

// An address that is formed where it stands: the places of a tile's fragments are constants of the loop,
// and the compiler would hold every one of them in a register; from here on they are offsets.
__device__ inline uint32_t formed(uint32_t at)
{
    asm volatile("" : "+v"(at));
    return at;
}

// The activation of 16-bit results, in the fewest instructions (a tile's epilogue is bound by them): as
// mm::act_value, but for silu's exponential, which may overflow here: z / infinity is 0.
__device__ inline float short_silu(float z) { return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }

template <typename F> __device__ inline void by_activation(const FourProduct &p, F f)
{
    if (p.act == SOM_ACT_RELU) f([](float z) { return z <= 0.0f ? 0.0f : z; });
    else if (p.act == SOM_ACT_GELU && p.y_f32) f([](float z) { return mm::act_fine(SOM_ACT_GELU, z); });
    else if (p.act == SOM_ACT_GELU) f([](float z) { return mm::act_value(SOM_ACT_GELU, z); });
    else if (p.act == SOM_ACT_SILU && p.y_f32) f([](float z) { return mm::act_fine(SOM_ACT_SILU, z); });
    else if (p.act == SOM_ACT_SILU) f([](float z) { return short_silu(z); });
}

// Sums start from the bias of their columns, which saves the epilogue an addition. COLUMN: a lane holds
// rows 4g ... 4g + 3 of column i of each block, else row i and columns 4g ... 4g + 3.
template <typename T, int MI, int NI, bool COLUMN> __device__ inline void start(const FourProduct &p, f32x4 (&acc)[MI][NI], int col0)
{
    const int lane = (int)threadIdx.x & 63, g = lane >> 4, li = lane & 15;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int n = col0 + 16 * j + (COLUMN ? li : 4 * g), cnt = min(COLUMN ? 1 : 4, (int)p.M - n);
        float b[4] = {0, 0, 0, 0};
        if (p.bias && cnt > 0) {
            if (p.bias_f32) mm::load4(static_cast<const float *>(p.bias) + n, cnt, b);
            else mm::load4(static_cast<const T *>(p.bias) + n, cnt, b);
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[i][j] = COLUMN ? f32x4{b[0], b[0], b[0], b[0]} : f32x4{b[0], b[1], b[2], b[3]};
    }
}

// Activation, residual and the store, for a wave's MI x NI blocks. Sixteen rows at a time go through
// LDS, so that a row's columns are read and written side by side; the residual is loaded sixteen rows
// ahead. Rows are addressed by a base that the wave shares and a lane's 32-bit offset in four rows.
template <typename T, int MI, int NI, bool COLUMN>
__device__ inline void finish(const FourProduct &p, const f32x4 (&acc)[MI][NI], int row0, int col0, float *own)
{
    constexpr int kCols = NI * 16, kRow = kCols + 4, kLanes = kCols / 4, kAtOnce = 64 / kLanes, kTurns = 16 / kAtOnce;
    const int lane = (int)threadIdx.x & 63, g = lane >> 4, li = lane & 15;
    const int sub = lane / kLanes, in_row = lane % kLanes * 4, n = col0 + in_row, cnt = min(4, (int)p.M - n);
    typedef T vec4 __attribute__((ext_vector_type(4)));
    typedef vec4 any4 __attribute__((aligned(sizeof(T))));
    typedef float fvec4 __attribute__((ext_vector_type(4)));
    typedef fvec4 fany4 __attribute__((aligned(4)));
    row0 = __builtin_amdgcn_readfirstlane(row0);
    col0 = __builtin_amdgcn_readfirstlane(col0);
    constexpr int64_t kMostLd = (int64_t)1 << 27;  // four rows of fp32 within 32 bits
    const bool cols_in = col0 + kCols <= (int)p.M && p.ldy < kMostLd && p.ldr < kMostLd;
    const uint32_t res_at = ((uint32_t)sub * (uint32_t)p.ldr + in_row) * 2, y_at = ((uint32_t)sub * (uint32_t)p.ldy + in_row) * (p.y_f32 ? 4 : 2);
    vec4 ahead[kTurns];
    auto is_whole = [&](int i) { return cols_in && row0 + 16 * i + 16 <= (int)p.N; };
    auto fetch16 = [&](int i) {
        if (!p.res || i >= MI || !is_whole(i)) return;
        const char *from = reinterpret_cast<const char *>(static_cast<const T *>(p.res) + (int64_t)(row0 + 16 * i) * p.ldr + col0);
#pragma unroll
        for (int r = 0; r < kTurns; ++r, from += kAtOnce * p.ldr * 2) ahead[r] = *reinterpret_cast<const any4 *>(from + res_at);
    };
    fetch16(0);
    auto whole16 = [&](int i) {
        vec4 now[kTurns];
#pragma unroll
        for (int r = 0; r < kTurns; ++r) now[r] = ahead[r];
        fetch16(i + 1);
        float v[kTurns][4];
#pragma unroll
        for (int r = 0; r < kTurns; ++r) {
            const f32x4 c = *reinterpret_cast<const f32x4 *>(own + (r * kAtOnce + sub) * kRow + in_row);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[r][q] = c[q];
        }
        by_activation(p, [&](auto f) {
#pragma unroll
            for (int r = 0; r < kTurns; ++r)
#pragma unroll
                for (int q = 0; q < 4; ++q) v[r][q] = f(v[r][q]);
        });
        if (p.res) {
#pragma unroll
            for (int r = 0; r < kTurns; ++r)
#pragma unroll
                for (int q = 0; q < 4; ++q) v[r][q] += (float)now[r][q];
        }
        if (p.y_f32) {
            char *to = reinterpret_cast<char *>(static_cast<float *>(p.y) + (int64_t)(row0 + 16 * i) * p.ldy + col0);
#pragma unroll
            for (int r = 0; r < kTurns; ++r, to += kAtOnce * p.ldy * 4)
                *reinterpret_cast<fany4 *>(to + y_at) = fvec4{v[r][0], v[r][1], v[r][2], v[r][3]};
        } else {
            char *to = reinterpret_cast<char *>(static_cast<T *>(p.y) + (int64_t)(row0 + 16 * i) * p.ldy + col0);
#pragma unroll
            for (int r = 0; r < kTurns; ++r, to += kAtOnce * p.ldy * 2)
                *reinterpret_cast<any4 *>(to + y_at) = vec4{(T)v[r][0], (T)v[r][1], (T)v[r][2], (T)v[r][3]};
        }
    };
    auto edge16 = [&](int i) {  // rows or columns past the last ones
#pragma unroll 1
        for (int r = 0; r < kTurns; ++r) {
            const int64_t m = row0 + 16 * i + r * kAtOnce + sub;
            if (m >= p.N || cnt <= 0) continue;
            const f32x4 c = *reinterpret_cast<const f32x4 *>(own + (r * kAtOnce + sub) * kRow + in_row);
            float v[4] = {c[0], c[1], c[2], c[3]}, t[4] = {0, 0, 0, 0};
            by_activation(p, [&](auto f) {
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = f(v[q]);
            });
            if (p.res) mm::load4(static_cast<const T *>(p.res) + m * p.ldr + n, cnt, t);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = p.res ? v[q] + t[q] : v[q];
            if (p.y_f32) mm::store4(static_cast<float *>(p.y) + m * p.ldy + n, cnt, v);
            else mm::store4(static_cast<T *>(p.y) + m * p.ldy + n, cnt, v);
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
        if (is_whole(i)) whole16(i);
        else edge16(i);
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

// Rows of 128 bytes in LDS (a whole line of the caches, which halves of one would be fetched twice for):
// chunk c of row r lies at c ^ f(r), so that the lanes that one read serves together touch every bank
// once: 16 rows, eight of either parity, at one or two neighbouring chunks.
__device__ inline int line_xor(int r) { return r >> 1 & 7; }

// A tile of ROWS lines of 128 bytes, loaded straight to LDS by NT threads. Addresses are a base that all
// threads share and 32-bit offsets: the rows of a tile lie within 2 GB.
template <int ROWS, int NT> struct LineLoader {
    static constexpr int kPer = ROWS * 8 / NT;
    static_assert(ROWS * 8 % NT == 0 && NT % 128 == 0, "every thread loads, the same chunk of each row");
    const char *base;
    uint32_t row[kPer], at, last;

    // Rows [r0, r1), `pitch` bytes apart, of `bytes` (whole chunks); those past the last repeat it.
    __device__ void init(const void *p, int64_t pitch, int r0, int r1, int64_t bytes)
    {
        const int t = (int)threadIdx.x;
        base = static_cast<const char *>(p) + (int64_t)r0 * pitch;
        at = (t % 8 ^ line_xor(t / 8)) * 16;
        last = (uint32_t)bytes - 16;
#pragma unroll
        for (int i = 0; i < kPer; ++i) row[i] = (uint32_t)min(i * (NT / 8) + t / 8, r1 - 1 - r0) * (uint32_t)pitch;
    }
    // Chunk i of line `line` of the rows. Past the end of a row its last chunk is read again: what meets
    // it must be zeros, or scales that make it nothing.
    __device__ void load(int i, int line, uint32_t lds) const
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        const uint32_t off = row[i] + min(at + (uint32_t)line * 128, last);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     :
                     : "s"(lds + (uint32_t)(i * NT + wave * 64) * 16), "v"(off), "s"(base)
                     : "memory");
    }
};

// LDS: two tiles of both operands, 256 features each, then two places for the scales of 512.
template <class S> struct Packed {
    static constexpr int kA = S::BM * 128, kB = S::BN * 128, kStage = kA + kB, kScales = 2 * kStage, kPlace = (S::BM + S::BN) * 16;
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
    const int64_t bytes = four_blocks(p.K) * 16;
    const int tiles = (int)((bytes + 127) / 128), pieces = (int)(four_pitch(p.K) / 16);
    typedef LineLoader<S::BM, S::NT> LoadA;
    typedef LineLoader<S::BN, S::NT> LoadB;
    LoadA la;
    LoadB lb;
    la.init(p.x, bytes, m0, (int)p.N, bytes);
    lb.init(p.w, bytes, n0, (int)p.M, bytes);
    // A thread's row of scales: BM of x, then BN of w; later waves repeat the earlier ones' loads.
    constexpr int kRows = S::BM + S::BN;
    static_assert(kRows % 64 == 0 && S::NT >= kRows, "whole waves");
    const int sr = wave % (kRows / 64) * 64 + lane;
    const uint8_t *scale_row = sr < S::BM ? p.x_scales + (int64_t)min(m0 + sr, (int)p.N - 1) * p.x_pitch
                                          : p.w_scales + (int64_t)min(n0 + sr - S::BM, (int)p.M - 1) * p.w_pitch;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

    f32x4 acc[S::MI][S::NI];
    start<T, S::MI, S::NI, false>(p, acc, n0 + wn * S::NI * 16);

    // Tile t lies at place t % 2 and is multiplied in two steps of 128 features. A step's fragments of B
    // and its first ones of A are in registers when it starts; the others of A are read kWindow rows
    // ahead, from the last rows on those of the next step. In the second step, when the tile's last
    // fragments are on their way, the waves meet: then tile t + 1 has arrived, and the loads of tile
    // t + 2 may take the place of tile t; they have the time of a whole tile.
    struct Fragment {
        i32x4 v;
        uint32_t scale;
    };
    const uint32_t at_a = wm * S::MI * 16, at_b = wn * S::NI * 16;
    const uint32_t va = base + (at_a + li) * 128, vb = base + L::kA + (at_b + li) * 128;
    const uint32_t slot[2] = {(uint32_t)(q ^ line_xor(li)) << 4, (uint32_t)((4 + q) ^ line_xor(li)) << 4};
    const uint32_t vsa = base + L::kScales + (at_a + li) * 16 + q, vsb = base + L::kScales + (S::BM + at_b + li) * 16 + q;
    // Where the fragments of a step and their scales start: D, which half of the features (128) of which
    // tile of two (P), at the place of its scales.
    struct Start {
        uint32_t a, b, sa, sb;
    };
    auto starts = [&](uint32_t scales, int P, int D) {
        const uint32_t at = slot[D] + P * L::kStage, s = scales + 8 * P + 4 * D;
        return Start{formed(va + at), formed(vb + at), formed(vsa + s), formed(vsb + s)};
    };
    auto read_a = [&](const Start &s, int i) { return Fragment{lds_chunk(s.a + i * 2048), lds_byte(s.sa + i * 256)}; };
    auto read_b = [&](const Start &s, int j) { return Fragment{lds_chunk(s.b + j * 2048), lds_byte(s.sb + j * 256)}; };
    auto multiply = [&](const Fragment &b, const Fragment &a, f32x4 c) {
        const i32x8 w = {b.v[0], b.v[1], b.v[2], b.v[3], 0, 0, 0, 0}, x = {a.v[0], a.v[1], a.v[2], a.v[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 4, 4, 0, (int)b.scale, 0, (int)a.scale);
    };
    constexpr int kLoads = LoadA::kPer + LoadB::kPer;
    auto load = [&](int c, int tile, int P) {
        if (c < LoadA::kPer) la.load(c, tile, base + P * L::kStage);
        else lb.load(c - LoadA::kPer, tile, base + P * L::kStage + L::kA);
    };
    auto load_piece = [&](int piece) {  // the scales of tiles 2 piece and 2 piece + 1
        load_scales<16>(scale_row, piece, pieces, base + L::kScales + (uint32_t)(piece % 2) * L::kPlace + wave % (kRows / 64) * 1024);
    };
    load_piece(0);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < kLoads; ++c) load(c, t, t);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLoads) : "memory");
    constexpr int kWindow = S::WINDOW, kMeet = S::MI - kWindow;
    Fragment even[S::NI], odd[S::NI], a[kWindow];
    Start first = starts(0, 0, 0);
#pragma unroll
    for (int j = 0; j < S::NI; ++j) even[j] = read_b(first, j);
#pragma unroll
    for (int i = 0; i < kWindow; ++i) a[i] = read_a(first, i);
    // Tile t at place P. No branch stands between its instructions: past one the compiler would move them.
    auto tile = [&](int t, auto place_of) {
        constexpr int P = decltype(place_of)::value;
        const uint32_t scales = (uint32_t)(t / 2 % 2) * L::kPlace;
        const Start second = starts(scales, P, 1), next = starts(P ? (uint32_t)((t / 2 + 1) % 2) * L::kPlace : scales, 1 - P, 0);
        constexpr int kB = (S::NI + S::MI / 2 - 1) / (S::MI / 2);
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
#pragma unroll
            for (int j = 0; j < S::NI; ++j) acc[i][j] = multiply(even[j], a[i % kWindow], acc[i][j]);
            a[i % kWindow] = i < kMeet ? read_a(first, i + kWindow) : read_a(second, i - kMeet);
#pragma unroll
            for (int j = i * kB; j < (i + 1) * kB && j < S::NI; ++j) odd[j] = read_b(second, j);
            __builtin_amdgcn_sched_barrier(0);
        }
        constexpr int kAfter = S::MI - kMeet, kOf = (kLoads + kAfter - 1) / kAfter, kBs = (S::NI + kAfter - 1) / kAfter;
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
            if (i == kMeet) {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                if (P == 0) load_piece(t / 2 + 1);
            }
#pragma unroll
            for (int j = 0; j < S::NI; ++j) acc[i][j] = multiply(odd[j], a[i % kWindow], acc[i][j]);
            a[i % kWindow] = i < kMeet ? read_a(second, i + kWindow) : read_a(next, i - kMeet);
            if (i >= kMeet) {
#pragma unroll
                for (int j = (i - kMeet) * kBs; j < (i - kMeet + 1) * kBs && j < S::NI; ++j) even[j] = read_b(next, j);
#pragma unroll
                for (int c = (i - kMeet) * kOf; c < (i - kMeet + 1) * kOf && c < kLoads; ++c) load(c, t + 2, P);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        first = next;
    };
    int t = 0;
    for (; t + 2 <= tiles; t += 2) {
        tile(t, Number<0>());
        tile(t + 1, Number<1>());
    }
    if (t < tiles) tile(t, Number<0>());
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing lands in LDS after the workgroup left it
    __syncthreads();  // the tiles are no longer read
    finish<T, S::MI, S::NI, false>(p, acc, m0 + (int)at_a, n0 + (int)at_b,
                                   reinterpret_cast<float *>(lds) + wave * (16 * (S::NI * 16 + 4)));
}

// LDS: two tiles of x, 64 features each, two places for the codes of 256 and two for their scales.
template <class S> struct Half {
    static constexpr int kA = S::BM * 128, kB = S::BN * 128, kCodes = 2 * kA, kScales = kCodes + 2 * kB, kPlace = S::BN * 8;
    // what the waves tell each other (fp16)
    static constexpr int kMarks = kScales + 2 * kPlace, kWaves = kMarks + S::NT / 64 * 8, kAll = kWaves + S::NT / 64 * 4;
    static constexpr int kEnd = S::WM * S::WN * 16 * (S::NI * 16 + 4) * 4;
    static constexpr int kBytes = kAll > kEnd ? kAll : kEnd;
    static_assert(kEnd <= kMarks, "the marks are read after the tiles");
};

// fp16 holds the codes of a tile under their scales, each over a power that the tile shares, where the scales
// span 2^26 at most: with the largest at 2^13 all are normal numbers, 6 x 2^13 and 2^-1 x 2^-13 and what is between.
// Then the sums run in the matrix instruction, as in bf16. `top`: the tile's largest byte. Two bytes count for
// nothing: 0, which blocks of zeros have (if others do, those below 2^-124, the answer is no), and 255, whose
// columns are marked in LDS and become NaN at the end.
template <class S> __device__ inline bool scales_fit(const FourProduct &p, const uint8_t *scale_row, int n0, char *lds, int &top)
{
    typedef uint16_t pair __attribute__((ext_vector_type(2)));
    constexpr int kParts = S::NT / S::BN;  // threads of a column
    const int64_t blocks = four_blocks(p.K);
    pair high = {0, 0}, low = {0xFFFF, 0xFFFF};  // of the bytes + 1: 255 becomes 0 and 0 becomes 1
    uint32_t others = 0, nans = 0;
    for (int64_t at = (int)threadIdx.x / S::BN; at < p.w_pitch / 16; at += kParts) {
        const uint4 piece = reinterpret_cast<const uint4 *>(scale_row)[at];
        const uint32_t w[4] = {piece.x, piece.y, piece.z, piece.w};
        uint32_t zeros = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const pair a = (__builtin_bit_cast(pair, w[i] & 0x00FF00FF) + (pair)1) & (pair)255, b = (__builtin_bit_cast(pair, w[i] >> 8 & 0x00FF00FF) + (pair)1) & (pair)255;
            high = __builtin_elementwise_max(high, __builtin_elementwise_max(a, b));
            low = __builtin_elementwise_min(low, __builtin_elementwise_min(a - (pair)2, b - (pair)2));  // 0 and 1 become the largest
            zeros |= (w[i] - 0x01010101u) & ~w[i] & 0x80808080u;
            nans |= (~w[i] - 0x01010101u) & w[i] & 0x80808080u;
        }
        if (zeros == 0) continue;
        const uint4 *codes = reinterpret_cast<const uint4 *>(p.w) + min(n0 + (int)threadIdx.x % S::BN, (int)p.M - 1) * blocks;
#pragma unroll 1
        for (int64_t b = at * 16; b < min(at * 16 + 16, blocks); ++b) {
            if (scale_row[b] != 0) continue;
            const uint4 c = codes[b];
            others |= (c.x | c.y | c.z | c.w) & 0x77777777u;
        }
    }
    uint32_t h = others ? 255 : max((uint32_t)max(high[0], high[1]), 1u) - 1, l = min((uint32_t)min(low[0], low[1]), 254u) + 1;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) h = max(h, (uint32_t)__shfl_xor((int)h, d)), l = min(l, (uint32_t)__shfl_xor((int)l, d));
    uint64_t *marks = reinterpret_cast<uint64_t *>(lds + Half<S>::kMarks);
    uint32_t *waves = reinterpret_cast<uint32_t *>(lds + Half<S>::kWaves);
    const uint64_t mark = __ballot(nans != 0);
    if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = h | l << 8, marks[threadIdx.x / 64] = mark;
    __syncthreads();
    h = 0, l = 255;
#pragma unroll
    for (int k = 0; k < S::NT / 64; ++k) h = max(h, waves[k] & 255), l = min(l, waves[k] >> 8);
    top = __builtin_amdgcn_readfirstlane((int)h);
    return top < 255 && top <= __builtin_amdgcn_readfirstlane((int)l) + 26;
}

// Whether scales_fit marked a column of the tile.
template <class S> __device__ inline bool marked(const char *lds, int column)
{
    const uint64_t *marks = reinterpret_cast<const uint64_t *>(lds + Half<S>::kMarks);
    uint64_t m = 0;
#pragma unroll
    for (int k = 0; k < S::NT / S::BN; ++k) m |= marks[k * (S::BN / 64) + column / 64];
    return m >> (column % 64) & 1;
}

template <typename T, class S> __global__ __launch_bounds__(S::NT, S::PER_CU * S::NT / 256) void k_mx4_half(const FourProduct p)
{
    typedef Half<S> L;
    constexpr bool kBf16 = __is_same(T, __bf16);
    typedef typename mm::Vec8<T>::type Frag;
    extern __shared__ __align__(1024) char lds[];
    int m0, n0;
    if (!place<S>(p, m0, n0)) return;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
    const int wm = wave / S::WN, wn = wave % S::WN, q = lane >> 4, li = lane & 15;
    const int64_t row_bytes = p.width * 2, code_bytes = four_blocks(p.K) * 16;
    const int tiles = (int)(row_bytes / 128);  // whole lines: the host sees to that
    LineLoader<S::BM, S::NT> la;
    LineLoader<S::BN, S::NT> lb;
    la.init(p.x, p.ldx * 2, m0, (int)p.N, row_bytes);
    lb.init(p.w, code_bytes, n0, (int)p.M, code_bytes);
    // A thread's column of scales; the later waves repeat the earlier ones' loads.
    static_assert(S::NT % S::BN == 0, "whole columns");
    const uint8_t *scale_row = p.w_scales + (int64_t)min(n0 + (int)threadIdx.x % S::BN, (int)p.M - 1) * p.w_pitch;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

    // As in the product of 4-bit rows, with tiles of 64 features in two steps of 32, a block of each
    // column. The codes come for four tiles at a time: when the waves meet in the last of four, those of
    // the four before are no longer read, and the ones after the next four take their place.
    struct Raw {
        uint32_t codes, scale;
    };
    struct Wide {
        Frag v;
        float scale;
    };
    const uint32_t at_a = wm * S::MI * 16, at_b = wn * S::NI * 16;
    const uint32_t va = base + (at_a + li) * 128, slot[2] = {(uint32_t)(q ^ line_xor(li)) << 4, (uint32_t)((4 + q) ^ line_xor(li)) << 4};
    const uint32_t vb = base + L::kCodes + (at_b + li) * 128 + 4 * q, vx = (uint32_t)line_xor(li) << 4;
    const uint32_t vs = base + L::kScales + (at_b + li) * 4;
    auto start_a = [&](int P, int D) { return formed(va + slot[D]) + P * L::kA; };
    auto read_a = [&](uint32_t at, int i) { return __builtin_bit_cast(Frag, lds_chunk(at + i * 2048)); };
    // Block B of the eight at a place (0 or 1): the scales of four blocks are a dword of a column.
    auto read_b = [&](uint32_t place, int B, Raw (&raw)[S::NI]) {
        const uint32_t at = formed(place * L::kB + vb + (((uint32_t)B << 4) ^ formed(vx)));
        const uint32_t s = formed(place * L::kPlace + vs) + (B / 4 * S::BN * 4 + B % 4);
#pragma unroll
        for (int j = 0; j < S::NI; ++j) raw[j] = Raw{lds_word(at + j * 2048), lds_byte(s + j * 64)};
    };
    constexpr int kA = LineLoader<S::BM, S::NT>::kPer, kB = LineLoader<S::BN, S::NT>::kPer;
    // Load c of the codes of four tiles: two of scales, the others of codes.
    auto load_codes = [&](int c, int four) {
        const uint32_t at = (uint32_t)(four % 2);
        if (c < 2)
            load_scales<4>(scale_row, 2 * four + c, p.w_pitch / 4, base + L::kScales + at * L::kPlace + (c * S::BN + wave % (S::BN / 64) * 64) * 4);
        else
            lb.load(c - 2, four, base + L::kCodes + at * L::kB);
    };
    auto load_first = [&] {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int c = 0; c < kB + 2; ++c) load_codes(c, t);
#pragma unroll
            for (int c = 0; c < kA; ++c) la.load(c, t, base + t * L::kA);
        }
    };
    // The product of the tile; scaled: the widened codes hold their scale, in fp16 over 2^(top - 13 - 127).
    auto run = [&](auto scaled, f32x4 (&acc)[S::MI][S::NI], int top) {
        constexpr bool kScaled = decltype(scaled)::value;
        const uint32_t over = (uint32_t)(140 - top) << 23;
        auto widen = [&](const Raw &r) {
            if constexpr (kBf16) return Wide{widen8<T>(r.codes, r.scale), 0.0f};
            // a block of zeros may end below 0 and is taken there
            else if constexpr (kScaled) return Wide{layer::widen8_by<T>(r.codes, __int_as_float(max((int)((r.scale << 23) + over), 0))), 0.0f};
            else return Wide{widen8<T>(r.codes, r.scale), scale_value(r.scale)};
        };
        auto multiply = [&](const Wide &b, const Frag &a, f32x4 c) {
            if constexpr (kScaled) return mm::mma(b.v, a, c);
            const f32x4 s = mm::mma(a, b.v, f32x4{0, 0, 0, 0});
#pragma unroll
            for (int k = 0; k < 4; ++k) c[k] = fmaf(s[k], b.scale, c[k]);
            return c;
        };
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kA + kB + 2) : "memory");
        constexpr int kWindow = S::WINDOW, kMeet = S::MI - kWindow;
        Wide even[S::NI], odd[S::NI];
        Frag a[kWindow];
        Raw raw[S::NI];
        read_b(0, 0, raw);
#pragma unroll
        for (int j = 0; j < S::NI; ++j) even[j] = widen(raw[j]);
        uint32_t first = start_a(0, 0);
#pragma unroll
        for (int i = 0; i < kWindow; ++i) a[i] = read_a(first, i);
        // Tile t, U: t % 4. No branch stands between its instructions: past one the compiler would move them.
        auto tile = [&](int t, auto u) {
            constexpr int U = decltype(u)::value, P = U % 2;
            const uint32_t codes = (uint32_t)(t / 4 % 2), next = U == 3 ? 1 - codes : codes;
            constexpr int kFrom = S::MI / 2, kWide = (S::NI + S::MI - kFrom - 1) / (S::MI - kFrom);
            const uint32_t second = start_a(P, 1), following = start_a(1 - P, 0);
#pragma unroll
            for (int i = 0; i < S::MI; ++i) {
                if (i == 0) read_b(codes, 2 * U + 1, raw);
#pragma unroll
                for (int j = 0; j < S::NI; ++j) acc[i][j] = multiply(even[j], a[i % kWindow], acc[i][j]);
                a[i % kWindow] = i < kMeet ? read_a(first, i + kWindow) : read_a(second, i - kMeet);
                if (i >= kFrom) {
#pragma unroll
                    for (int j = (i - kFrom) * kWide; j < (i - kFrom + 1) * kWide && j < S::NI; ++j) odd[j] = widen(raw[j]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            constexpr int kLoads = kA + (U == 3 ? kB + 2 : 0), kAfter = S::MI - kMeet, kOf = (kLoads + kAfter - 1) / kAfter;
#pragma unroll
            for (int i = 0; i < S::MI; ++i) {
                if (i == 0) read_b(next, (2 * U + 2) % 8, raw);
                if (i == kMeet) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
                for (int j = 0; j < S::NI; ++j) acc[i][j] = multiply(odd[j], a[i % kWindow], acc[i][j]);
                a[i % kWindow] = i < kMeet ? read_a(second, i + kWindow) : read_a(following, i - kMeet);
                if (i >= kFrom) {
#pragma unroll
                    for (int j = (i - kFrom) * kWide; j < (i - kFrom + 1) * kWide && j < S::NI; ++j) even[j] = widen(raw[j]);
                }
                if (i >= kMeet) {
#pragma unroll
                    for (int c = (i - kMeet) * kOf; c < (i - kMeet + 1) * kOf && c < kLoads; ++c) {
                        if (c < kA) la.load(c, t + 2, base + P * L::kA);
                        else load_codes(c - kA, t / 4 + 2);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            first = following;
        };
        int t = 0;
        for (; t + 4 <= tiles; t += 4) {
            tile(t, Number<0>());
            tile(t + 1, Number<1>());
            tile(t + 2, Number<2>());
            tile(t + 3, Number<3>());
        }
        if (t < tiles) tile(t, Number<0>());
        if (t + 1 < tiles) tile(t + 1, Number<1>());
        if (t + 2 < tiles) tile(t + 2, Number<2>());
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing lands in LDS after the workgroup left it
        __syncthreads();  // the tiles are no longer read
        if constexpr (!kBf16 && kScaled) {
            const int col0 = n0 + (int)at_b + 4 * q;
#pragma unroll
            for (int j = 0; j < S::NI; ++j) {
                float bias[4] = {0, 0, 0, 0};
                const int cnt = min(4, (int)p.M - col0 - 16 * j);
                if (p.bias && cnt > 0) {
                    if (p.bias_f32) mm::load4(static_cast<const float *>(p.bias) + col0 + 16 * j, cnt, bias);
                    else mm::load4(static_cast<const T *>(p.bias) + col0 + 16 * j, cnt, bias);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (marked<S>(lds, (int)at_b + 16 * j + 4 * q + k)) bias[k] = __builtin_nanf("");
#pragma unroll
                for (int i = 0; i < S::MI; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][j][k] = ldexpf(acc[i][j][k], top - 140) + bias[k];
            }
        }
        finish<T, S::MI, S::NI, !kScaled>(p, acc, m0 + (int)at_a, n0 + (int)at_b,
                                          reinterpret_cast<float *>(lds) + wave * (16 * (S::NI * 16 + 4)));
    };
    if constexpr (kBf16) {
        f32x4 acc[S::MI][S::NI];
        start<T, S::MI, S::NI, false>(p, acc, n0 + wn * S::NI * 16);
        load_first();
        run(Number<1>(), acc, 0);
    } else {
        load_first();
        int top;
        if (scales_fit<S>(p, scale_row, n0, lds, top)) {
            f32x4 acc[S::MI][S::NI];
#pragma unroll
            for (int i = 0; i < S::MI; ++i)
#pragma unroll
                for (int j = 0; j < S::NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
            run(Number<1>(), acc, top);
        } else {
            f32x4 acc[S::MI][S::NI];
            start<T, S::MI, S::NI, true>(p, acc, n0 + wn * S::NI * 16);
            run(Number<0>(), acc, 0);
        }
    }
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
