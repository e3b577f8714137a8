// som_mm.h -- matrix products on the matrix cores (gfx950), fp16 or bf16 operands, fp32 sums.
//
// A workgroup computes a BM x BN tile of the result, each wave a part of it in 16 x 16 blocks
// of v_mfma_f32_16x16x32. Operand tiles of 32 reduction steps go through LDS. An operand is
// stored either with the reduction running along its rows ("along": 8 steps are 16 bytes) or
// across them ("across": a row holds one step). The tile in LDS keeps the stored order, so
// both are loaded in 16-byte chunks; a fragment of an "across" operand is read with the LDS
// transpose read, which gives a lane four steps of one column.
//
// Chunks are placed in LDS so that the lanes of one read touch every bank once:
//   along:  64-byte rows of 4 chunks, chunk s of row r at s ^ f(r), f = -(r / 4) mod 4: sixteen
//           rows at one step octet cover sixteen different 16-byte slots, and so do rows 0-3 and
//           12-15 of one octet with rows 4-11 of the next, which is what LDS serves together;
//   across: rows of BR * 2 bytes, the 32-byte unit u (16 columns) of row k at u ^ f(k), f
//           from bits 0, 1 and 3 of k, so that the eight rows of a half wave's transpose read
//           lie in different units.
// The results are computed transposed (the B fragment is the instruction's first operand), so
// that a lane owns four consecutive columns of one row and the epilogue reads and writes
// 8 or 16 bytes at a time.
//
// What lies outside an operand is read as zero: from a page of zeros (loads straight to LDS)
// or element by element (loads through registers), so nothing outside the buffers is touched
// and no stray infinity meets a zero.
#pragma once

#include <atomic>

#include "som_dense.h"

namespace som {
namespace mm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

static __device__ __align__(64) const uint4 g_zero[1] = {{0, 0, 0, 0}};

// The workgroup's number in a launch by grid_of.
__device__ inline int64_t block_number() { return (int64_t)blockIdx.y * kBlocksAlongX + blockIdx.x; }

constexpr int kBK = 32;  // reduction steps of a tile

__device__ inline f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

template <typename T> struct Vec8;
template <> struct Vec8<_Float16> { typedef f16x8 type; };
template <> struct Vec8<__bf16> { typedef bf16x8 type; };

// exp(x): 2^t on the hardware with what t = x log2(e) lost in rounding put back, within 3 units in
// the last place; 0 below about -87, also at minus infinity.
__device__ inline float exp_f32(float x)
{
    x = fmaxf(x, -200.0f);
    const float t = x * 1.44269504f;
    const float lost = fmaf(x, 1.44269504f, -t) + x * 1.925963e-8f;
    return __builtin_amdgcn_exp2f(t) * fmaf(lost, 0.693147181f, 1.0f);
}

// exp(x) to |x| 2^-24 of it: enough where the result is rounded to 16 bits.
__device__ inline float exp_short(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// The normal distribution Phi(z) and exp(-z^2 / 2), by formula 7.1.26 of Abramowitz and Stegun's
// Handbook of Mathematical Functions for the error function: within 1.5e-7 of itself (of z Phi(z)
// for z below about -4 that is more than a 16-bit result's rounding, of values below 2e-4), for a
// third of erff's instructions. For 16-bit results; fp32 ones take act_fine.
__device__ inline float normal_f32(float z, float &bell)
{
    const float x = fabsf(z) * 0.707106781f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
    bell = exp_short(-0.5f * z * z);
    float q = fmaf(1.061405429f, t, -1.453152027f);
    q = fmaf(q, t, 1.421413741f);
    q = fmaf(q, t, -0.284496736f);
    q = fmaf(q, t, 0.254829592f);
    const float tail = 0.5f * q * t * bell;  // of Phi beyond |z|
    return z < 0.0f ? tail : 1.0f - tail;
}

// Activations and their derivatives at z, in fp32.
__device__ inline void act_both(int act, float z, float &value, float &slope)
{
    value = z;
    slope = 1.0f;
    if (act == SOM_ACT_RELU) {  // NaN stays NaN
        value = z <= 0.0f ? 0.0f : z;
        slope = z <= 0.0f ? 0.0f : z > 0.0f ? 1.0f : z;
    } else if (act == SOM_ACT_SILU) {
        const float q = __builtin_amdgcn_rcpf(1.0f + exp_short(fminf(-z, 88.0f)));
        value = z * q;
        slope = q * fmaf(z, 1.0f - q, 1.0f);
    } else if (act == SOM_ACT_GELU) {
        float bell;
        const float q = normal_f32(z, bell);
        value = z * q;
        slope = fmaf(0.39894228f * z, bell, q);
    }
}

__device__ inline float act_value(int act, float z)
{
    float value, slope;
    act_both(act, z, value, slope);
    return value;
}

// The activations where the result is fp32, to a few units in its last place (gelu far below zero:
// z^2 of them, from the rounding of erfc's argument). silu by exp(-|z|), which does not overflow.
__device__ inline float act_fine(int act, float z)
{
    if (act == SOM_ACT_GELU) return z * (0.5f * erfcf(z * -0.707106781f));
    if (act == SOM_ACT_SILU) {
        const float e = exp_f32(-fabsf(z));
        return z * ((z < 0.0f ? e : 1.0f) / (1.0f + e));
    }
    return act_value(act, z);
}

// n (1 to 4) consecutive values at p, whose alignment is that of one element.
template <typename T> __device__ inline void load4(const T *p, int n, float *v)
{
    typedef T vec __attribute__((ext_vector_type(4)));
    typedef vec any __attribute__((aligned(sizeof(T))));
    if (n == 4) {
        const vec t = *reinterpret_cast<const any *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
    }
}

// v[from ... n - 1] to p + from ...
template <typename T> __device__ inline void store4(T *p, int from, int n, const float *v)
{
    typedef T vec __attribute__((ext_vector_type(4)));
    typedef vec any __attribute__((aligned(sizeof(T))));
    if (from <= 0 && n == 4) {
        vec t;
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = (T)v[i];
        *reinterpret_cast<any *>(p) = t;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i >= from && i < n) p[i] = (T)v[i];
    }
}

template <typename T> __device__ inline void store4(T *p, int n, const float *v) { store4(p, 0, n, v); }

// The place of chunks in an "along" row.
__device__ inline int chunk_xor(int r) { return -(r >> 2) & 3; }

// The place of 32-byte units in an "across" row.
template <int BR> __device__ inline int unit_xor(int k)
{
    if (BR >= 128) return (k & 3) | ((k >> 3) & 1) << 2;
    return 0;
}

// Values whose last `left` (below 8) are wanted, moved to the front, zeros after them.
__device__ inline s16x8 shift_out(const s16x8 &v, int left)
{
    typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
    u64x2 x = __builtin_bit_cast(u64x2, v);
    const int s = 16 * min(8, 8 - left);  // bits, 16 to 128
    const unsigned long long lo = s < 64 ? x[0] >> s | x[1] << (64 - s) : s < 128 ? x[1] >> (s - 64) : 0;
    return __builtin_bit_cast(s16x8, u64x2{lo, s < 64 ? x[1] >> s : 0});
}

enum Fetch { kPlain, kClamped, kChecked };

// One operand's tile of kBK steps by BR rows (along) or columns (across), loaded by NT threads,
// tile after tile. A chunk past the last row (column) is read from inside the operand instead:
// it only reaches results that are not written. A chunk past the last step must be zero.
template <typename T, int BR, bool ACROSS, bool MAPPED, int NT> struct Loader {
    static constexpr int kChunks = BR * kBK / 8;
    static constexpr int kPer = (kChunks + NT - 1) / NT;
    static constexpr int kRowChunks = ACROSS ? BR / 8 : kBK / 8;
    static constexpr int kBytes = BR * kBK * 2;
    static constexpr int kWaveRows = 64 / kRowChunks;  // across: rows that a wave's chunks cover
    typedef const __attribute__((address_space(4))) int32_t *Scalar;

    const T *ptr[kPer];  // the chunk in the next tile (across with a map: its column in row 0)
    int k[kPer];         // its step in the tile
    int cnt[kPer];       // elements inside the operand, of loads through registers
    Scalar map;          // MAPPED (across): the rows' map, from the first row of the reduction
    int next[kPer][MAPPED ? kWaveRows : 1];  // and what it says for the wave's rows of the next tile
    int64_t ld;
    int K, t;            // reduction length; the next tile's first step

    // along: rows [r0, r1) of the operand (through `rows`); across: columns [r0, r1), reduction
    // rows from k0 on. CHUNKS: r1 - r0 and K are whole chunks where they run along a row.
    template <bool CHUNKS> __device__ void init(const T *p, int64_t ld_, const int32_t *rows, int r0, int r1, int64_t k0, int K_)
    {
        ld = ld_;
        K = K_;
        t = 0;
        if (MAPPED) map = (Scalar)(rows + k0);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int c = (i * NT + (int)threadIdx.x) % kChunks;  // threads without a chunk repeat others'
            const int row = c / kRowChunks, s = c % kRowChunks;
            if (ACROSS) {
                int col = r0 + 8 * (s ^ (unit_xor<BR>(row) << 1));
                k[i] = row;
                cnt[i] = min(8, r1 - col);
                if (CHUNKS) col = min(col, r1 - 8);
                ptr[i] = p + col + (MAPPED ? 0 : (k0 + row) * ld);
            } else {
                const int src = s ^ chunk_xor(row);
                const int r = min(r0 + row, r1 - 1);
                k[i] = 8 * src;
                cnt[i] = 8;
                ptr[i] = p + (rows ? (int64_t)rows[r] : (int64_t)r) * ld + k[i];
            }
        }
        look_up();
    }

    // The map's entries for the next tile, by scalar loads: they are not waited for with the
    // vector loads in flight.
    __device__ void look_up()
    {
        if (!MAPPED) return;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
#pragma unroll
            for (int q = 0; q < kWaveRows; ++q)
                next[i][q] = map[max(min(t + (i * NT + wave * 64) / kRowChunks + q, K - 1), 0)];
    }

    __device__ static bool mine(int i) { return kChunks % NT == 0 || i * NT + (int)threadIdx.x < kChunks; }

    // The chunk's address in the next tile.
    __device__ const T *source(int i) const
    {
        if (!MAPPED) return ptr[i];
        int row = 0;
#pragma unroll
        for (int q = 0; q < kWaveRows; ++q)
            row |= next[i][q] & -(int)(((int)threadIdx.x & 63) / kRowChunks == q);
        return ptr[i] + (int64_t)row * ld;
    }

    __device__ void advance()
    {
        t += kBK;
        if (!MAPPED) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) ptr[i] += ACROSS ? kBK * ld : (int64_t)kBK;
        }
        look_up();
    }

    // Whether every chunk can be loaded without a check (kClamped); the same for every thread.
    __device__ bool covers(int r0, int r1) const { return ACROSS ? r0 + BR <= r1 : K >= 8; }

    // Chunk i of the next tile, straight to LDS; INSIDE: the tile ends within the operand. The
    // instruction is written out because the compiler waits for every such load of its own before
    // any read of LDS; the kernel's loop waits as it needs. A wave's 64 chunks go to consecutive
    // 16-byte places from m0 on.
    template <bool INSIDE> __device__ void async(int i, uint32_t lds) const
    {
        if (!mine(i)) return;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        const void *from = source(i);
        if (!INSIDE) from = t + k[i] < K ? from : g_zero;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                     :
                     : "s"(lds + (uint32_t)(i * NT + wave * 64) * 16), "v"(from)
                     : "memory");
    }

    // The next tile, into registers. Where the loads are unconditional the compiler counts them and
    // waits for no more than it needs: kPlain for a tile within the operand; kClamped for any
    // tile, a chunk past the end is read from the last whole one before it (put sets that right);
    // kChecked reads value by value at the edges.
    template <Fetch HOW> __device__ void fetch(s16x8 *r)
    {
        typedef s16x8 any __attribute__((aligned(2)));
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const short *src = reinterpret_cast<const short *>(source(i));
            const int left = K - t - k[i];
            if (HOW == kPlain) {
                r[i] = *reinterpret_cast<const any *>(src);
            } else if (HOW == kClamped) {
                if (!ACROSS) src += min(0, left - 8);
                else if (!MAPPED) src += min(0, left - 1) * ld;
                r[i] = *reinterpret_cast<const any *>(src);
            } else {
                r[i] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
                if (!mine(i)) continue;
                const int n = ACROSS ? (left > 0 ? cnt[i] : 0) : min(8, left);
                if (n >= 8) {
                    r[i] = *reinterpret_cast<const any *>(src);
                } else if (n > 0) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < n) r[i][j] = src[j];
                }
            }
        }
        advance();
    }

    // Tile `tile` from registers to LDS. CLAMPED: the values past the end are shifted out.
    template <bool CLAMPED> __device__ void put(int tile, char *lds, const s16x8 *r) const
    {
        const bool ends = CLAMPED && (tile + 1) * kBK > K;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            s16x8 v = r[i];
            if (ends) {
                const int left = K - tile * kBK - k[i];
                if (ACROSS) {
                    if (left <= 0) v = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
                } else if (left < 8) {
                    v = shift_out(v, left);
                }
            }
            if (mine(i)) *reinterpret_cast<s16x8 *>(lds + (i * NT + (int)threadIdx.x) * 16) = v;
        }
    }
};

// A lane's fragments of 16 rows (columns) each, from row (column) `at` of a tile in LDS. `at` is a
// multiple of the wave's rows, so the unit of fragment j is an exclusive or away from the first's.
template <typename T, int BR, bool ACROSS> struct Reader {
    uint32_t base;

    __device__ void init(int at)
    {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4, i = lane & 15;
        if (ACROSS) {
            const int row = 8 * g + (i >> 2);
            base = row * (BR * 2) + ((((uint32_t)at >> 4) ^ unit_xor<BR>(row)) << 5) + (i & 3) * 8;
        } else {
            base = (at + i) * (kBK * 2) + ((g ^ chunk_xor(i)) << 4);
        }
    }

    // lds: the tile's address in LDS, a multiple of 1,024.
    __device__ typename Vec8<T>::type read(uint32_t lds, int j) const
    {
        s16x8 r;
        if (ACROSS) {
            const uint32_t p = (lds + base) ^ (uint32_t)(j << 5);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)p);
            const s16x4 hi =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)(p + 4 * BR * 2));
            r = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            r = *(const __attribute__((address_space(3))) s16x8 *)(uintptr_t)(lds + base + (uint32_t)j * (16 * kBK * 2));
        }
        return __builtin_bit_cast(typename Vec8<T>::type, r);
    }
};

// STAGES: tiles' places in LDS (loads straight there); AHEAD: tiles in registers (loads through them).
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int AHEAD_, int PER_CU_> struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, AHEAD = AHEAD_, PER_CU = PER_CU_;
    static constexpr int NT = 64 * WM * WN;
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;
};

// The value of another lane of the 16, by a pattern of data-parallel primitives.
template <int CTRL> __device__ inline float lane_swap(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}

// A wave's LDS accesses before this are done before those after it (LDS serves a wave in order;
// the wait is for the values, the clobber for the compiler). Nothing else is waited for.
__device__ inline void wave_sync_lds()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// Workgroup b of `total` tiles: consecutive tiles go to one XCD (workgroups are dealt to the
// eight XCDs in turn), so that its L2 serves the operands they share. The grid is a multiple
// of 8 at least as large as the tiles. Returns -1 for a workgroup without a tile.
__device__ inline int64_t tile_of(int64_t b, int64_t total)
{
    const int64_t per = (total + 7) / 8, t = (b & 7) * per + (b >> 3);
    return (b >> 3) < per && t < total ? t : -1;
}

// Tile t of nm x nn, in bands of 8 tile rows walked column by column.
__device__ inline void tile_place(int64_t t, int nm, int nn, int &m, int &n)
{
    const int band = 8;
    const int64_t per = (int64_t)band * nn;
    const int b = (int)(t / per), in = (int)(t % per);
    const int rows = min(band, nm - b * band);
    m = b * band + in % rows;
    n = in / rows;
}

enum Layout { kNN, kNT, kTN };

template <bool V> struct Inside {
    static constexpr bool value = V;
};

template <Fetch V> struct How {
    static constexpr Fetch value = V;
};

// Which operand of a product over rows (TN) goes through a map of its rows.
enum Mapped { kNoMap, kMapA, kMapB };

template <typename T, Layout L, Epilogue EPI, class S, bool ASYNC, Mapped MAP>
__global__ __launch_bounds__(S::NT, S::PER_CU * S::NT / 256) void k_product(const Product p)
{
    constexpr bool A_ACROSS = L == kTN, B_ACROSS = L != kNT;
    typedef Loader<T, S::BM, A_ACROSS, MAP == kMapA, S::NT> LoadA;
    typedef Loader<T, S::BN, B_ACROSS, MAP == kMapB, S::NT> LoadB;
    constexpr int kStage = LoadA::kBytes + LoadB::kBytes;
    constexpr int kStages = ASYNC ? S::STAGES : 2;
    extern __shared__ __align__(1024) char lds[];

    const int nn = (int)((p.N + S::BN - 1) / S::BN);
    int e = 0, mt, nt, m0, m1, K;
    int64_t k0 = 0;
    if (L == kTN) {
        const int nm = (int)((p.M + S::BM - 1) / S::BM);
        const int64_t per = (int64_t)nm * nn;
        // Experts take unequal numbers of rows: their tiles go round the XCDs, not each expert's to one.
        const int64_t total = per * max(1, p.groups);
        const int64_t b = block_number(), t = p.off ? (b < total ? b : -1) : tile_of(b, total);
        if (t < 0) return;
        e = (int)(t / per);
        tile_place(t % per, nm, nn, mt, nt);
        m0 = mt * S::BM;
        m1 = (int)p.M;
        K = (int)p.K;
        if (p.off) {
            k0 = p.off[e];
            K = p.off[e + 1] - (int)k0;
        } else if (p.groups) {  // a part of the rows, whole tiles of them
            const int len = ((K + p.groups - 1) / p.groups + kBK - 1) / kBK * kBK;
            k0 = min((int64_t)e * len, (int64_t)K);
            K = min(len, K - (int)k0);
        }
    } else {
        const int nm = p.groups ? *p.n_tiles * p.split : (int)((p.M + S::BM - 1) / S::BM);
        const int64_t t = tile_of(block_number(), (int64_t)nm * nn);
        if (t < 0) return;
        tile_place(t, nm, nn, mt, nt);
        m0 = mt * S::BM;
        m1 = (int)p.M;
        if (p.groups) {
            const TileRow r = p.tiles[mt / p.split];
            e = r.e;
            m0 = r.row + mt % p.split * S::BM;
            m1 = min(r.end, r.row + p.tile_height);
            if (m0 >= m1) return;
        }
        K = (int)p.K;
    }
    // Loads through registers: the last tile of columns (rows of a result by rows) is moved back to
    // end with the operand, so that its loads need no checks; what it repeats is not written twice.
    int n0 = nt * S::BN;
    const int n_from = n0, m_from = m0;
    if (!ASYNC && p.N >= S::BN) n0 = min(n0, (int)p.N - S::BN);
    if (!ASYNC && L == kTN && p.M >= S::BM) m0 = min(m0, (int)p.M - S::BM);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / S::WN, wn = wave % S::WN;

    LoadA la;
    LoadB lb;
    const T *A = static_cast<const T *>(p.A);
    const T *B = static_cast<const T *>(p.B) + (L == kTN ? 0 : (int64_t)e * p.strideB);
    la.template init<ASYNC>(A, p.lda, p.amap, m0, m1, k0, K);
    lb.template init<ASYNC>(B, p.ldb, L == kTN ? p.bmap : nullptr, n0, (int)p.N, k0, K);
    Reader<T, S::BM, A_ACROSS> ra;
    Reader<T, S::BN, B_ACROSS> rb;
    ra.init(wm * S::MI * 16);
    rb.init(wn * S::NI * 16);

    f32x4 acc[S::MI][S::NI];
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    // The column sums of B: one more block of rows for the tiles of the first tile row, each row
    // the weights (or ones); the WM waves that read the same columns share them out.
    const bool sums = L == kTN && p.db && mt == 0;
    constexpr int kSums = S::NI / S::WM;
    f32x4 col[kSums];
#pragma unroll
    for (int j = 0; j < kSums; ++j) col[j] = f32x4{0, 0, 0, 0};

    const int steps = (K + kBK - 1) / kBK;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    typedef typename Vec8<T>::type Frag;
    struct FragsB {
        Frag f[S::NI];
    };
    auto multiply_row = [&](int i, const Frag &a, const FragsB &b) {
#pragma unroll
        for (int j = 0; j < S::NI; ++j) acc[i][j] = mma(b.f[j], a, acc[i][j]);
    };
    // The fragment that stands for the row of ones, or of the reduction rows' weights: those of tile
    // t lie in LDS behind the tiles (ASYNC), or are read from memory. Rows of B past the end are
    // zero, so the ones need no end.
    constexpr int kWeights = kStages * kStage;  // [kStages][kBK] floats
    Frag ones;
    if (L == kTN) {
#pragma unroll
        for (int q = 0; q < 8; ++q) ones[q] = (T)1.0f;
    }
    auto add_sums = [&](int t, const FragsB &b) {
        if (p.w) {
            const int octet = ((int)threadIdx.x & 63) >> 4, left = K - t * kBK - 8 * octet;
            const float *own = reinterpret_cast<const float *>(lds + kWeights) + t % kStages * kBK + 8 * octet;
#pragma unroll
            for (int q = 0; q < 8; ++q)
                ones[q] = (T)(ASYNC ? own[q] : q < left ? p.w[k0 + t * kBK + 8 * octet + q] : 0.0f);
        }
#pragma unroll
        for (int w = 0; w < S::WM; ++w) {
            if (w != wm) continue;
#pragma unroll
            for (int j = 0; j < kSums; ++j) col[j] = mma(b.f[w * kSums + j], ones, col[j]);
        }
    };

    if (ASYNC) {
        // Step t multiplies tile t, MI rows of NI blocks. Its fragments of B and its first kWindow of
        // A are in registers when it starts; the others of A are read kWindow rows ahead, from the
        // last rows on those of tile t + 1, whose fragments of B are read as well; the loads of
        // tiles up to t + kStages - 1 are in flight. A wave waits for its own loads of tile t + 1 and
        // for its own reads of tile t - 1, the barrier makes that every wave's: tile t + 1 may be
        // read, and the place of tile t - 1 be loaded anew. Past the last tile the loads bring
        // zeros, so that the number in flight is the same in every step (a wave that has fewer
        // chunks than others counts on its own: kLoads is the least).
        constexpr int kLoads = LoadA::kChunks / S::NT + LoadB::kChunks / S::NT;
        static_assert(LoadA::kChunks % 64 == 0 && LoadB::kChunks % 64 == 0, "whole waves load");
        const bool weights = L == kTN && sums && p.w && threadIdx.x < kBK;  // half of the first wave
        auto load_weights = [&](int t) {
            const int k = t * kBK + (int)threadIdx.x;
            const void *from = k < K ? static_cast<const void *>(p.w + k0 + k) : static_cast<const void *>(g_zero);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                         :
                         : "s"(base + (uint32_t)(kWeights + t % kStages * kBK * 4)), "v"(from)
                         : "memory");
        };
#pragma unroll
        for (int t = 0; t < kStages - 1; ++t) {
            if (weights) load_weights(t);
#pragma unroll
            for (int i = 0; i < LoadA::kPer; ++i) la.template async<false>(i, base + t * kStage);
#pragma unroll
            for (int i = 0; i < LoadB::kPer; ++i) lb.template async<false>(i, base + t * kStage + LoadA::kBytes);
            la.advance();
            lb.advance();
        }
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 2) * kLoads) : "memory");
        constexpr int kWindow = S::MI < 4 ? S::MI : 4;
        FragsB even, odd;
        Frag a[kWindow];
#pragma unroll
        for (int j = 0; j < S::NI; ++j) even.f[j] = rb.read(base + LoadA::kBytes, j);
#pragma unroll
        for (int i = 0; i < kWindow; ++i) a[i] = ra.read(base, i);
        auto step = [&](int t, const FragsB &now, FragsB &then, auto inside) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 3) * kLoads) : "memory");
            const uint32_t here = base + (uint32_t)(t % kStages) * kStage;
            const uint32_t next = base + (uint32_t)((t + 1) % kStages) * kStage;
            const uint32_t to = base + (uint32_t)((t + kStages - 1) % kStages) * kStage;
            if (weights) load_weights(t + kStages - 1);
            constexpr int kB = (2 * S::NI + S::MI - 1) / S::MI;  // fragments of B a row: done in the first half
            constexpr int kAll = LoadA::kPer + LoadB::kPer, kOf = (kAll + S::MI - 1) / S::MI;
#pragma unroll
            for (int i = 0; i < S::MI; ++i) {
                multiply_row(i, a[i % kWindow], now);
                a[i % kWindow] = i + kWindow < S::MI ? ra.read(here, i + kWindow) : ra.read(next, i + kWindow - S::MI);
#pragma unroll
                for (int j = i * kB; j < (i + 1) * kB && j < S::NI; ++j)
                    then.f[j] = rb.read(next + LoadA::kBytes, j);
#pragma unroll
                for (int c = i * kOf; c < (i + 1) * kOf; ++c) {
                    if (c < LoadA::kPer) la.template async<decltype(inside)::value>(c, to);
                    else if (c < kAll) lb.template async<decltype(inside)::value>(c - LoadA::kPer, to + LoadA::kBytes);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            la.advance();
            lb.advance();
            if (L == kTN && sums) add_sums(t, now);
        };
        int t = 0;
        for (; (t + kStages + 1) * kBK <= K; t += 2) {
            step(t, even, odd, Inside<true>());
            step(t + 1, odd, even, Inside<true>());
        }
        for (; t < steps; t += 2) {
            step(t, even, odd, Inside<false>());
            if (t + 1 < steps) step(t + 1, odd, even, Inside<false>());
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing lands in LDS after the workgroup left it
    } else {
        // Tiles go through registers, kAhead of them in flight, into two places of LDS.
        constexpr int kAhead = S::AHEAD;
        s16x8 va[kAhead][LoadA::kPer], vb[kAhead][LoadB::kPer];
        auto fetch = [&](int i, auto how) {
            la.template fetch<decltype(how)::value>(va[i]);
            lb.template fetch<decltype(how)::value>(vb[i]);
        };
        auto step = [&](int t, int i, auto how, auto ends) {
            char *at = lds + (t % 2) * kStage;
            la.template put<decltype(ends)::value>(t, at, va[i]);
            lb.template put<decltype(ends)::value>(t, at + LoadA::kBytes, vb[i]);
            __syncthreads();
            fetch(i, how);
            FragsB b;
            const uint32_t from = base + (uint32_t)(t % 2) * kStage;
#pragma unroll
            for (int j = 0; j < S::NI; ++j) b.f[j] = rb.read(from + LoadA::kBytes, j);
#pragma unroll
            for (int m = 0; m < S::MI; ++m) multiply_row(m, ra.read(from, m), b);
            if (L == kTN && sums) add_sums(t, b);
        };
        int t = 0;
        if (steps > 0 && la.covers(m0, m1) && lb.covers(n0, (int)p.N)) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(i, How<kClamped>());
            for (; (t + 2 * kAhead) * kBK <= K; t += kAhead) {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) step(t + i, i, How<kPlain>(), Inside<false>());
            }
            for (; t < steps; t += kAhead) {  // past the last tile they multiply zeros
#pragma unroll
                for (int i = 0; i < kAhead; ++i) step(t + i, i, How<kClamped>(), Inside<true>());
            }
        } else if (steps > 0) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(i, How<kChecked>());
            for (; t < steps; t += kAhead) {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) step(t + i, i, How<kChecked>(), Inside<false>());
            }
        }
    }

    // Epilogue. Lane (g, i) of a wave has row i and columns 4g ... 4g + 3 of each 16 x 16 block; 16
    // rows at a time go through LDS, so that a row's columns are read and written side by side.
    // (Rows there are 16 bytes longer than the columns: the 64 writes of 16 bytes meet every
    // bank equally often.)
    constexpr int kCols = S::NI * 16, kRow = kCols + 4, kLanes = kCols / 4, kAtOnce = 64 / kLanes;
    const int lane = (int)threadIdx.x & 63, g = lane >> 4, li = lane & 15;
    const int row0 = m0 + wm * S::MI * 16, col0 = n0 + wn * kCols;
    const int64_t ob = L == kTN ? (int64_t)e * p.strideC : 0;
    const int sub = lane / kLanes, n = col0 + lane % kLanes * 4, cnt = min(4, (int)p.N - n);
    const int skip = ASYNC ? 0 : min(4, n_from - n);  // the first of the four that another tile writes
    float *own = reinterpret_cast<float *>(lds) + wave * (16 * kRow);
    float bias[4] = {0, 0, 0, 0};
    if ((EPI == kLinear || EPI == kInner || EPI == kPairs) && p.bias && cnt > 0) {
        if (p.bias_f32) load4(static_cast<const float *>(p.bias) + (int64_t)e * p.strideBias + n, cnt, bias);
        else load4(static_cast<const T *>(p.bias) + (int64_t)e * p.strideBias + n, cnt, bias);
    }
    __syncthreads();  // the tiles are no longer read
    constexpr int kTurns = 16 / kAtOnce;
    // 16 rows: a lane's four columns of every kAtOnce-th row. Each stage runs over all of them, so
    // that its loads are in flight together and its branches are taken once.
    // What it reads besides (residual; z and act(z)) is loaded sixteen rows ahead.
    typedef T vec4 __attribute__((ext_vector_type(4)));
    typedef vec4 any4 __attribute__((aligned(sizeof(T))));
    const bool cols_in = col0 + kCols <= (int)p.N && n0 == n_from && m0 == m_from;
    constexpr bool kReads = EPI == kLinear || EPI == kSlope;
    vec4 ahead[kReads ? kTurns : 1], ahead2[EPI == kSlope ? kTurns : 1];
    auto is_whole = [&](int i) { return cols_in && row0 + 16 * i + 16 <= m1; };
    auto fetch16 = [&](int i) {
        if (!kReads || i >= S::MI || !is_whole(i)) return;
#pragma unroll
        for (int r = 0; r < kTurns; ++r) {
            const int64_t row = row0 + 16 * i + r * kAtOnce + sub;
            if (EPI == kSlope) {
                ahead[r] = *reinterpret_cast<const any4 *>(static_cast<const T *>(p.pre) + row * p.ldp + n);
                ahead2[r] = *reinterpret_cast<const any4 *>(static_cast<const T *>(p.res) + row * p.ldr + n);
            } else if (p.res) {
                ahead[r] = *reinterpret_cast<const any4 *>(static_cast<const T *>(p.res) + row * p.ldr + n);
            }
        }
    };
    fetch16(0);
    auto rows16 = [&](int i, auto whole) {
        constexpr bool W = decltype(whole)::value;
        vec4 now[kReads ? kTurns : 1], now2[EPI == kSlope ? kTurns : 1];
        if (W && kReads) {
#pragma unroll
            for (int r = 0; r < kTurns; ++r) {
                now[r] = ahead[r];
                if (EPI == kSlope) now2[r] = ahead2[r];
            }
        }
        fetch16(i + 1);
        const int c4 = W ? 4 : cnt, c0 = W ? 0 : skip;
        float v[kTurns][4], wr[kTurns];
        int m[kTurns];
        bool in[kTurns];
#pragma unroll
        for (int r = 0; r < kTurns; ++r) {
            const f32x4 c = *reinterpret_cast<const f32x4 *>(own + (r * kAtOnce + sub) * kRow + lane % kLanes * 4);
            m[r] = row0 + 16 * i + r * kAtOnce + sub;
            in[r] = W || (m[r] < m1 && m[r] >= m_from && cnt > 0 && skip < 4);
            wr[r] = ((EPI == kInner && p.weighted) || EPI == kPairs || EPI == kSlope) && p.w && in[r] ? p.w[m[r]] : 1.0f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                v[r][q] = c[q];
                if (EPI == kLinear || EPI == kInner || EPI == kPairs) v[r][q] += bias[q];
                if (EPI == kPairs) v[r][q] *= wr[r];
            }
        }
        if (EPI == kLinear || EPI == kInner) {
            if (p.pre) {
#pragma unroll
                for (int r = 0; r < kTurns; ++r)
                    if (in[r]) store4(static_cast<T *>(p.pre) + (int64_t)m[r] * p.ldp + n, c0, c4, v[r]);
            }
            if (EPI == kLinear && p.out_f32 && (p.act == SOM_ACT_GELU || p.act == SOM_ACT_SILU)) {
#pragma unroll
                for (int r = 0; r < kTurns; ++r)
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[r][q] = act_fine(p.act, v[r][q]);
            } else if (p.act == SOM_ACT_GELU) {
#pragma unroll
                for (int r = 0; r < kTurns; ++r)
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[r][q] = act_value(SOM_ACT_GELU, v[r][q]);
            } else if (p.act == SOM_ACT_SILU) {
#pragma unroll
                for (int r = 0; r < kTurns; ++r)
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[r][q] = act_value(SOM_ACT_SILU, v[r][q]);
            } else if (p.act == SOM_ACT_RELU) {
#pragma unroll
                for (int r = 0; r < kTurns; ++r)
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[r][q] = act_value(SOM_ACT_RELU, v[r][q]);
            }
        }
        if (EPI == kInner && p.weighted) {
#pragma unroll
            for (int r = 0; r < kTurns; ++r) {
                if (!in[r]) continue;
                const float t[4] = {v[r][0] * wr[r], v[r][1] * wr[r], v[r][2] * wr[r], v[r][3] * wr[r]};
                store4(static_cast<T *>(p.weighted) + (int64_t)m[r] * p.ldo + n, c0, c4, t);
            }
        }
        if (EPI == kLinear && p.res) {
            float t[kTurns][4];
#pragma unroll
            for (int r = 0; r < kTurns; ++r) {
                if (W) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) t[r][q] = (float)now[r][q];
                } else if (in[r]) {
                    load4(static_cast<const T *>(p.res) + (int64_t)m[r] * p.ldr + n, c4, t[r]);
                }
            }
#pragma unroll
            for (int r = 0; r < kTurns; ++r)
#pragma unroll
                for (int q = 0; q < 4; ++q) v[r][q] += t[r][q];
        }
        if (EPI == kSlope) {
            float z[kTurns][4], h[kTurns][4];
#pragma unroll
            for (int r = 0; r < kTurns; ++r) {
                if (W) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) z[r][q] = (float)now[r][q], h[r][q] = (float)now2[r][q];
                } else if (in[r]) {
                    load4(static_cast<const T *>(p.pre) + (int64_t)m[r] * p.ldp + n, c4, z[r]);
                    load4(static_cast<const T *>(p.res) + (int64_t)m[r] * p.ldr + n, c4, h[r]);
                }
            }
            float part[kTurns];
            auto slopes = [&](int act) {
#pragma unroll
                for (int r = 0; r < kTurns; ++r) {
                    // act(z) as the forward pass rounded it: one rounding, where act of the rounded
                    // z adds what its slope makes of another
                    part[r] = 0.0f;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float value, slope;
                        act_both(act, z[r][q], value, slope);
                        part[r] += in[r] && q < c4 && q >= c0 ? h[r][q] * v[r][q] : 0.0f;
                        v[r][q] *= wr[r] * slope;
                    }
                }
            };
            if (p.act == SOM_ACT_GELU) slopes(SOM_ACT_GELU);
            else if (p.act == SOM_ACT_SILU) slopes(SOM_ACT_SILU);
            else if (p.act == SOM_ACT_RELU) slopes(SOM_ACT_RELU);
            else slopes(SOM_ACT_NONE);
#pragma unroll
            for (int r = 0; r < kTurns; ++r) {  // over the row's 8 or 16 lanes: pairs, quads, halves, rows of 16
                part[r] += lane_swap<0xB1>(part[r]);
                part[r] += lane_swap<0x4E>(part[r]);
                part[r] += lane_swap<0x141>(part[r]);
                if (kLanes == 16) part[r] += lane_swap<0x140>(part[r]);
            }
            static_assert(kLanes == 8 || kLanes == 16, "a row's lanes");
#pragma unroll
            for (int r = 0; r < kTurns; ++r)
                if (m[r] < m1 && lane % kLanes == 0) p.parts[(int64_t)m[r] * p.n_parts + nt * S::WN + wn] = part[r];
        }
        if (EPI == kPairs || ((EPI == kLinear || EPI == kGrad) && p.out_f32)) {
#pragma unroll
            for (int r = 0; r < kTurns; ++r)
                if (in[r]) store4(static_cast<float *>(p.out) + ob + (int64_t)m[r] * p.ldo + n, c0, c4, v[r]);
        } else {
#pragma unroll
            for (int r = 0; r < kTurns; ++r)
                if (in[r]) store4(static_cast<T *>(p.out) + ob + (int64_t)m[r] * p.ldo + n, c0, c4, v[r]);
        }
    };
#pragma unroll 1
    for (int i = 0; i < S::MI; ++i) {  // rolled: the code of sixteen rows stands here once
        if (L == kTN && !p.out) break;
#pragma unroll
        for (int at = 0; at < S::MI; ++at) {
            if (at != i) continue;
#pragma unroll
            for (int j = 0; j < S::NI; ++j) *reinterpret_cast<f32x4 *>(own + li * kRow + j * 16 + 4 * g) = acc[at][j];
        }
        wave_sync_lds();
        if (is_whole(i)) rows16(i, Inside<true>());
        else rows16(i, Inside<false>());
        wave_sync_lds();
    }
    if (L == kTN && sums && li == 0) {
#pragma unroll
        for (int j = 0; j < kSums; ++j) {
            const int c = col0 + 16 * (wm * kSums + j) + 4 * g, left = min(4, (int)p.N - c);
            if (left <= 0) continue;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = col[j][q];
            if (p.bias_f32) store4(static_cast<float *>(p.db) + (int64_t)e * p.strideDb + c, left, v);
            else store4(static_cast<T *>(p.db) + (int64_t)e * p.strideDb + c, left, v);
        }
    }
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Loads straight to LDS move whole 16-byte chunks: both operands' rows must start on them and
// the length that runs along a row must be whole chunks.
inline bool chunked(Layout l, const Product &p)
{
    if (!aligned16(p.A) || !aligned16(p.B) || p.lda % 8 || p.ldb % 8 || p.strideB % 8) return false;
    if (l != kTN && p.K % 8) return false;
    if (l != kNT && p.N % 8) return false;
    return l != kTN || p.M % 8 == 0;
}

template <typename T, Layout L, Epilogue EPI, class S, bool ASYNC, Mapped MAP = kNoMap>
hipError_t launch(const Product &p, int64_t tile_rows_total, hipStream_t st)
{
    constexpr int kStage = (S::BM + S::BN) * kBK * 2;
    constexpr int tiles = (kStage + (L == kTN ? kBK * 4 : 0)) * (ASYNC ? S::STAGES : 2), rows = S::WM * S::WN * 16 * (S::NI * 16 + 4) * 4;
    constexpr int bytes = tiles > rows ? tiles : rows;
    const int64_t nn = (p.N + S::BN - 1) / S::BN;
    const int64_t total = tile_rows_total * nn;
    if (total <= 0) return hipSuccess;
    const dim3 grid = grid_of((total + 7) / 8 * 8);
    if (grid.x == 0) return hipErrorInvalidValue;
    // The attribute belongs to the function on each device; setting it again changes nothing.
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    if (bytes > 64 << 10 && (hipGetDevice(&dev) != hipSuccess || dev > 63 || !(done.load() >> dev & 1))) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_product<T, L, EPI, S, ASYNC, MAP>),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (err != hipSuccess) return err;
        if (dev <= 63) done.fetch_or(1ull << dev);
    }
    hipLaunchKernelGGL((k_product<T, L, EPI, S, ASYNC, MAP>), grid, dim3(S::NT), bytes, st, p);
    return hipGetLastError();
}

// Small tiles are for few rows, of which there are seldom more than one a CU: they keep more
// tiles in flight.
typedef Shape<32, 128, 1, 4, 8, 6, 2> Small;
typedef Shape<128, 128, 2, 2, 4, 3, 2> Mid;
typedef Shape<256, 256, 2, 4, 4, 3, 1> Large;

}  // namespace mm
}  // namespace som
