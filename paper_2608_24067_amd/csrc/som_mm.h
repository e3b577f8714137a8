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
//   along:  64-byte rows of 4 chunks, chunk s of row r at s ^ (r / 4 % 4): sixteen rows at
//           one step octet cover sixteen different 16-byte slots;
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

#include "som_dense.h"

namespace som {
namespace mm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

static __device__ __align__(64) const uint4 g_zero[1] = {{0, 0, 0, 0}};

constexpr int kBK = 32;  // reduction steps of a tile

__device__ inline f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

template <typename T> struct Vec8;
template <> struct Vec8<_Float16> { typedef f16x8 type; };
template <> struct Vec8<__bf16> { typedef bf16x8 type; };

// Activations and their derivatives at z, in fp32.
__device__ inline float act_value(int act, float z)
{
    if (act == SOM_ACT_RELU) return z <= 0.0f ? 0.0f : z;  // NaN stays NaN
    if (act == SOM_ACT_SILU) return z / (1.0f + expf(-z));
    if (act == SOM_ACT_GELU) return z * (0.5f + 0.5f * erff(z * 0.70710678f));
    return z;
}

__device__ inline void act_both(int act, float z, float &value, float &slope)
{
    if (act == SOM_ACT_RELU) {
        value = act_value(act, z);
        slope = z <= 0.0f ? 0.0f : z > 0.0f ? 1.0f : z;
    } else if (act == SOM_ACT_SILU) {
        const float q = 1.0f / (1.0f + expf(-z));
        value = z * q;
        slope = q * (1.0f + z * (1.0f - q));
    } else if (act == SOM_ACT_GELU) {
        const float q = 0.5f + 0.5f * erff(z * 0.70710678f);
        value = z * q;
        slope = q + z * (0.39894228f * expf(-0.5f * z * z));
    } else {
        value = z;
        slope = 1.0f;
    }
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

template <typename T> __device__ inline void store4(T *p, int n, const float *v)
{
    typedef T vec __attribute__((ext_vector_type(4)));
    typedef vec any __attribute__((aligned(sizeof(T))));
    if (n == 4) {
        vec t;
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = (T)v[i];
        *reinterpret_cast<any *>(p) = t;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}

// The place of 32-byte units in an "across" row.
template <int BR> __device__ inline int unit_xor(int k)
{
    if (BR >= 128) return (k & 3) | ((k >> 3) & 1) << 2;
    return 0;
}

// One operand's tile of kBK steps by BR rows (along) or columns (across), loaded by NT threads,
// tile after tile. A chunk past the last row (column) is read from inside the operand instead:
// it only reaches results that are not written. A chunk past the last step must be zero.
template <typename T, int BR, bool ACROSS, int NT> struct Loader {
    static constexpr int kChunks = BR * kBK / 8;
    static constexpr int kPer = (kChunks + NT - 1) / NT;
    static constexpr int kRowChunks = ACROSS ? BR / 8 : kBK / 8;
    static constexpr int kBytes = BR * kBK * 2;
    static constexpr int kWaveRows = 64 / kRowChunks;  // across: rows that a wave's chunks cover
    typedef const __attribute__((address_space(4))) int32_t *Scalar;

    const T *ptr[kPer];  // the chunk in the next tile (across with a map: its column in row 0)
    int k[kPer];         // its step in the tile
    int cnt[kPer];       // elements inside the operand, of loads through registers
    Scalar map;          // across: the rows' map, from the first row of the reduction
    int next[kPer][ACROSS ? kWaveRows : 1];  // and what it says for the wave's rows of the next tile
    int64_t ld;
    int K, t;            // reduction length; the next tile's first step

    // along: rows [r0, r1) of the operand (through `rows`); across: columns [r0, r1), reduction
    // rows from k0 on. CHUNKS: r1 - r0 and K are whole chunks where they run along a row.
    template <bool CHUNKS> __device__ void init(const T *p, int64_t ld_, const int32_t *rows, int r0, int r1, int64_t k0, int K_)
    {
        ld = ld_;
        K = K_;
        t = 0;
        map = ACROSS && rows ? (Scalar)(rows + k0) : nullptr;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int c = i * NT + (int)threadIdx.x;
            const int row = c / kRowChunks, s = c % kRowChunks;
            if (ACROSS) {
                int col = r0 + 8 * (s ^ (unit_xor<BR>(row) << 1));
                k[i] = row;
                cnt[i] = min(8, r1 - col);
                if (CHUNKS) col = min(col, r1 - 8);
                ptr[i] = p + col + (map ? 0 : (k0 + row) * ld);
            } else {
                const int src = s ^ ((row >> 2) & 3);
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
        if (!ACROSS || !map) return;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
#pragma unroll
            for (int q = 0; q < kWaveRows; ++q)
                next[i][q] = t < K ? map[min(t + (i * NT + wave * 64) / kRowChunks + q, K - 1)] : 0;
    }

    __device__ static bool mine(int i) { return kChunks % NT == 0 || i * NT + (int)threadIdx.x < kChunks; }

    // The chunk's address in the next tile.
    __device__ const T *source(int i) const
    {
        if (!ACROSS || !map) return ptr[i];
        int row = next[i][0];
#pragma unroll
        for (int q = 1; q < kWaveRows; ++q)
            row = ((int)threadIdx.x & 63) / kRowChunks == q ? next[i][q] : row;
        return ptr[i] + (int64_t)row * ld;
    }

    __device__ void advance()
    {
        t += kBK;
        if (!ACROSS || !map) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) ptr[i] += ACROSS ? kBK * ld : (int64_t)kBK;
        }
        look_up();
    }

    // The next tile, straight to LDS. The instruction is written out because the compiler waits
    // for every such load of its own before any read of LDS; the kernel's loop waits as it needs.
    // A wave's 64 chunks go to consecutive 16-byte places from m0 on.
    __device__ void async(uint32_t lds)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!mine(i)) continue;
            const void *from = source(i);
            if (t + kBK > K && t + k[i] >= K) from = g_zero;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                         :
                         : "s"(lds + (uint32_t)(i * NT + wave * 64) * 16), "v"(from)
                         : "memory");
        }
        advance();
    }

    // The next tile, into registers.
    __device__ void fetch(s16x8 *r)
    {
        typedef s16x8 any __attribute__((aligned(2)));
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            r[i] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
            if (!mine(i)) continue;
            const int left = K - t - k[i], n = ACROSS ? (left > 0 ? cnt[i] : 0) : min(8, left);
            const short *src = reinterpret_cast<const short *>(source(i));
            if (n >= 8) {
                r[i] = *reinterpret_cast<const any *>(src);
            } else if (n > 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n) r[i][j] = src[j];
            }
        }
        advance();
    }

    __device__ static void put(char *lds, const s16x8 *r)
    {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (mine(i)) *reinterpret_cast<s16x8 *>(lds + (i * NT + (int)threadIdx.x) * 16) = r[i];
    }
};

// A lane's fragment of 16 rows (columns) from `at`, a multiple of 16, of a tile in LDS.
template <typename T, int BR, bool ACROSS> struct Reader {
    int base, f;

    __device__ void init(int at)
    {
        const int lane = (int)threadIdx.x & 63, g = lane >> 4, i = lane & 15;
        if (ACROSS) {
            const int row = 8 * g + (i >> 2);
            f = unit_xor<BR>(row);
            base = row * (BR * 2) + (i & 3) * 8;
            unit = at >> 4;
        } else {
            f = 0;
            unit = 0;
            base = (at + i) * (kBK * 2) + ((g ^ (i >> 2)) << 4);
        }
    }

    int unit;

    __device__ typename Vec8<T>::type read(const char *lds, int j) const
    {
        s16x8 r;
        if (ACROSS) {
            const char *p = lds + base + (((unit + j) ^ f) << 5);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4 *)(p + 4 * BR * 2));
            r = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            r = *reinterpret_cast<const s16x8 *>(lds + base + j * (16 * kBK * 2));
        }
        return __builtin_bit_cast(typename Vec8<T>::type, r);
    }
};

template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int PER_CU_> struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, PER_CU = PER_CU_;
    static constexpr int NT = 64 * WM * WN;
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;
};

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

template <typename T, Layout L, Epilogue EPI, class S, bool ASYNC>
__global__ __launch_bounds__(S::NT, S::PER_CU * S::NT / 256) void k_product(const Product p)
{
    constexpr bool A_ACROSS = L == kTN, B_ACROSS = L != kNT;
    typedef Loader<T, S::BM, A_ACROSS, S::NT> LoadA;
    typedef Loader<T, S::BN, B_ACROSS, S::NT> LoadB;
    constexpr int kStage = LoadA::kBytes + LoadB::kBytes;
    constexpr int kStages = ASYNC ? S::STAGES : 2;
    extern __shared__ __align__(1024) char lds[];

    const int nn = (int)((p.N + S::BN - 1) / S::BN);
    int e = 0, mt, nt, m0, m1, K;
    int64_t k0 = 0;
    if (L == kTN) {
        const int nm = (int)((p.M + S::BM - 1) / S::BM);
        const int64_t per = (int64_t)nm * nn;
        const int64_t t = tile_of(blockIdx.x, per * max(1, p.groups));
        if (t < 0) return;
        e = (int)(t / per);
        tile_place(t % per, nm, nn, mt, nt);
        m0 = mt * S::BM;
        m1 = (int)p.M;
        K = (int)p.K;
        if (p.groups) {
            k0 = p.off[e];
            K = p.off[e + 1] - (int)k0;
        }
    } else {
        const int nm = p.groups ? *p.n_tiles * p.split : (int)((p.M + S::BM - 1) / S::BM);
        const int64_t t = tile_of(blockIdx.x, (int64_t)nm * nn);
        if (t < 0) return;
        tile_place(t, nm, nn, mt, nt);
        m0 = mt * S::BM;
        m1 = (int)p.M;
        if (p.groups) {
            const TileRow r = p.tiles[mt / p.split];
            e = r.e;
            m0 = r.row + mt % p.split * S::BM;
            m1 = r.end;
            if (m0 >= m1) return;
        }
        K = (int)p.K;
    }
    const int n0 = nt * S::BN;
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

    // The column sums of B: one more block of rows for the waves of the first tile row, each
    // row the weights (or ones).
    const bool sums = L == kTN && p.db && mt == 0 && wm == 0;
    f32x4 col[S::NI];
#pragma unroll
    for (int j = 0; j < S::NI; ++j) col[j] = f32x4{0, 0, 0, 0};

    const int steps = (K + kBK - 1) / kBK;
    auto compute = [&](int t) {
        const char *at = lds + (t % kStages) * kStage;
        typename Vec8<T>::type b[S::NI];
#pragma unroll
        for (int j = 0; j < S::NI; ++j) b[j] = rb.read(at + LoadA::kBytes, j);
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
            const typename Vec8<T>::type a = ra.read(at, i);
#pragma unroll
            for (int j = 0; j < S::NI; ++j) acc[i][j] = mma(b[j], a, acc[i][j]);
        }
        if (L == kTN && sums) {
            typename Vec8<T>::type ones;
            const int k = t * kBK + 8 * (((int)threadIdx.x & 63) >> 4);
#pragma unroll
            for (int q = 0; q < 8; ++q) ones[q] = (T)(k + q < K ? (p.w ? p.w[k0 + k + q] : 1.0f) : 0.0f);
#pragma unroll
            for (int j = 0; j < S::NI; ++j) col[j] = mma(b[j], ones, col[j]);
        }
    };

    if (ASYNC) {
        // kStages - 1 tiles in flight. A wave waits for its own loads of the tile it needs,
        // the barrier makes that every wave's; it also says that the tile computed before is
        // no longer read, whose place the next loads take. Past the last tile the loads bring
        // zeros, so that the number in flight is the same in every step.
        // (a wave that has fewer chunks than others counts on its own: kLoads is the least).
        constexpr int kLoads = LoadA::kChunks / S::NT + LoadB::kChunks / S::NT;
        static_assert(LoadA::kChunks % 64 == 0 && LoadB::kChunks % 64 == 0, "whole waves load");
        const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
#pragma unroll
        for (int s = 0; s < kStages - 1; ++s) {
            la.async(base + s * kStage);
            lb.async(base + s * kStage + LoadA::kBytes);
        }
        for (int t = 0; t < steps; ++t) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 2) * kLoads) : "memory");
            const uint32_t next = base + (uint32_t)((t + kStages - 1) % kStages) * kStage;
            la.async(next);
            lb.async(next + LoadA::kBytes);
            compute(t);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing lands in LDS after the workgroup has left it
    } else {
        s16x8 va[LoadA::kPer], vb[LoadB::kPer];
        if (steps > 0) {
            la.fetch(va);
            lb.fetch(vb);
            LoadA::put(lds, va);
            LoadB::put(lds + LoadA::kBytes, vb);
            __syncthreads();
        }
        for (int t = 0; t < steps; ++t) {
            if (t + 1 < steps) {
                la.fetch(va);
                lb.fetch(vb);
            }
            compute(t);
            if (t + 1 < steps) {
                char *next = lds + ((t + 1) % 2) * kStage;
                LoadA::put(next, va);
                LoadB::put(next + LoadA::kBytes, vb);
            }
            __syncthreads();
        }
    }

    // Epilogue: lane (g, i) of the wave has the row i and the columns 4g ... 4g + 3 of each block.
    const int lane = (int)threadIdx.x & 63, g = lane >> 4, li = lane & 15;
    const int row0 = m0 + wm * S::MI * 16 + li, col0 = n0 + wn * S::NI * 16 + 4 * g;
    const int64_t ob = L == kTN ? (int64_t)e * p.strideC : 0;
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
        const int m = row0 + 16 * i;
        const bool row_in = m < m1 && (L != kTN || p.out);
        float wr = 1.0f, part = 0.0f;
        if (L != kTN && p.w && row_in) wr = p.w[m];
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            const int n = col0 + 16 * j, cnt = min(4, (int)p.N - n);
            if (!row_in || cnt <= 0) continue;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = acc[i][j][q];
            if (EPI == kLinear || EPI == kInner || EPI == kPairs) {
                if (p.bias) {
                    float b[4];
                    if (p.bias_f32) load4(static_cast<const float *>(p.bias) + (int64_t)e * p.strideBias + n, cnt, b);
                    else load4(static_cast<const T *>(p.bias) + (int64_t)e * p.strideBias + n, cnt, b);
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] += EPI == kPairs ? wr * b[q] : b[q];
                }
            }
            if (EPI == kLinear || EPI == kInner) {
                if (p.pre) store4(static_cast<T *>(p.pre) + (int64_t)m * p.ldp + n, cnt, v);
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = act_value(p.act, v[q]);
            }
            if (EPI == kInner) {
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] *= wr;
            }
            if (EPI == kLinear && p.res) {
                float r[4];
                load4(static_cast<const T *>(p.res) + (int64_t)m * p.ldr + n, cnt, r);
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] += r[q];
            }
            if (EPI == kSlope) {
                float z[4];
                load4(static_cast<const T *>(p.pre) + (int64_t)m * p.ldp + n, cnt, z);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float value, slope;
                    act_both(p.act, z[q], value, slope);
                    part += q < cnt ? value * v[q] : 0.0f;
                    v[q] *= wr * slope;
                }
            }
            if (EPI == kPairs || (EPI == kLinear && p.out_f32))
                store4(static_cast<float *>(p.out) + ob + (int64_t)m * p.ldo + n, cnt, v);
            else
                store4(static_cast<T *>(p.out) + ob + (int64_t)m * p.ldo + n, cnt, v);
        }
        if (EPI == kSlope) {
            part += __shfl_xor(part, 16);
            part += __shfl_xor(part, 32);
            if (row_in && g == 0 && col0 < p.N)
                p.parts[(int64_t)m * p.n_parts + (n0 / (16 * S::NI) + wn)] = part;
        }
    }
    if (L == kTN && sums && li == 0) {
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            const int n = col0 + 16 * j, cnt = min(4, (int)p.N - n);
            if (cnt <= 0) continue;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = col[j][q];
            if (p.bias_f32) store4(static_cast<float *>(p.db) + (int64_t)e * p.strideDb + n, cnt, v);
            else store4(static_cast<T *>(p.db) + (int64_t)e * p.strideDb + n, cnt, v);
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

template <typename T, Layout L, Epilogue EPI, class S, bool ASYNC>
hipError_t launch(const Product &p, int64_t tile_rows_total, hipStream_t st)
{
    constexpr int kStage = (S::BM + S::BN) * kBK * 2;
    constexpr int bytes = kStage * (ASYNC ? S::STAGES : 2);
    const int64_t nn = (p.N + S::BN - 1) / S::BN;
    const int64_t total = tile_rows_total * nn;
    if (total <= 0) return hipSuccess;
    const int64_t grid = (total + 7) / 8 * 8;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
    if (bytes > 64 << 10) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_product<T, L, EPI, S, ASYNC>),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL((k_product<T, L, EPI, S, ASYNC>), dim3((unsigned)grid), dim3(S::NT), bytes, st, p);
    return hipGetLastError();
}

typedef Shape<32, 128, 1, 4, 4, 4> Small;
typedef Shape<128, 128, 2, 2, 4, 2> Mid;
typedef Shape<256, 256, 2, 4, 4, 1> Large;

}  // namespace mm
}  // namespace som
