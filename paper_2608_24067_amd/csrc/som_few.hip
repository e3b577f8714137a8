// som_few.hip -- products of few rows with feature-major matrices: bound by reading the matrix once.
//
// A workgroup has a tile of up to 16 rows and 128 columns; its waves share out the reduction. A
// wave's step is 32 features: lane (c, g) reads, of features 8g ... 8g + 7, the eight columns
// from 8c on (16 bytes each; sixteen lanes read 256 bytes of a feature), and turns these 8 x 8
// values about in registers into eight operands of v_mfma_f32_16x16x32: operand j holds column
// 8c + j of every lane. The matrix goes from memory to registers with no LDS and no barrier in
// between, kDeep steps (32 KB a wave) in flight. The waves' sums meet in LDS, added in the waves'
// order. Rows past the tile repeat its last one; columns past the end are read again from inside
// (the last tile is moved back to end with the matrix, or the last lanes' columns are); features
// past the end count as zeros.
//
// Where the tiles are fewer than the CUs the reduction is also split over workgroups, whose
// results (kPairs only) are added by the kernel that combines a row's pairs.

#include "som_mm.h"

namespace som {
namespace {

using namespace mm;

constexpr int kDeep = 4, kCols = 128, kRows = tile_rows(kTileFew);

// An 8 x 8 block of 16-bit values turned about: out[j] element k = in[k] element j.
__device__ inline void turn(const s16x8 *in, s16x8 *out)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    u32x4 a[8], b[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) a[k] = __builtin_bit_cast(u32x4, in[k]);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)  // values j of rows 2k and 2k + 1
            b[j][k] = __builtin_amdgcn_perm(a[2 * k + 1][j / 2], a[2 * k][j / 2], j % 2 ? 0x07060302 : 0x05040100);
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = __builtin_bit_cast(s16x8, b[j]);
}

// n of 8 values at p, aligned to one; zeros for the others.
__device__ inline s16x8 load8(const short *p, int n)
{
    typedef s16x8 any __attribute__((aligned(2)));
    if (n >= 8) return *reinterpret_cast<const any *>(p);
    s16x8 r = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) r[j] = p[j];
    return r;
}

template <typename T, Epilogue EPI, int kWaves, bool Z = false>
__global__ __launch_bounds__(64 * kWaves, 2) void k_few(const Product p, int splits)
{
    typedef typename Vec8<T>::type Frag;
    __shared__ __align__(16) float lds[kWaves][kRows][kCols + 4];
    const int nn = (int)((p.N + kCols - 1) / kCols);
    const int nm = p.pairs ? (int)p.M : p.groups ? *p.n_tiles : (int)((p.M + kRows - 1) / kRows);
    const int64_t t = block_number();
    if (t >= (int64_t)nm * nn * splits) return;
    const int split = (int)(t % splits), nt = (int)(t / splits % nn), mt = (int)(t / splits / nn);
    int e = 0, m0 = mt * kRows, m1 = min((int)p.M, m0 + kRows);
    if (p.pairs) {
        e = p.pairs[mt];
        if ((unsigned)e >= (unsigned)p.groups) return;
        m0 = mt;
        m1 = mt + 1;
    } else if (p.groups) {
        const TileRow r = p.tiles[mt];
        e = r.e;
        m0 = r.row;
        m1 = min(r.end, m0 + kRows);
    }
    const int K = (int)p.K, N = (int)p.N;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int c = lane & 15, g = lane >> 4;
    // This wave's steps: an even share of the whole reduction's.
    const int parts = splits * kWaves, own = split * kWaves + wave, steps = (K + 31) / 32;
    const int s0 = (int)((int64_t)steps * own / parts), s1 = (int)((int64_t)steps * (own + 1) / parts);

    const int row = min(m0 + c, m1 - 1);
    const int64_t at = p.pairs ? row / p.pair_rows : p.amap ? p.amap[row] : row;
    const short *a = static_cast<const short *>(p.A) + (Z ? 0 : at * p.lda + 8 * g);
    const int n_from = nt * kCols, n0 = N >= kCols ? min(n_from, N - kCols) : 0;
    const int last = N - n0 - 8;  // where the last lane's eight columns start (negative: fewer than 8 in all)
    const int cols = last >= 0 ? 8 : min(8, N - n0 - 8 * c);  // of a lane's eight (moved back: all)
    const short *b = static_cast<const short *>(p.B) + (int64_t)e * p.strideB + 8 * (int64_t)g * p.ldb + n0 +
                     (last >= 0 ? min(8 * c, last) : cols > 0 ? 8 * c : 0);

    // Eight values of act(z + bias) from the parts of z (one pair: every lane's row is the same).
    auto inner8 = [&](int k0) {
        typedef T vec __attribute__((ext_vector_type(8)));
        vec r;
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            const int n = max(0, min(4, K - k0 - h));
            float z[4] = {0, 0, 0, 0}, b4[4] = {0, 0, 0, 0};
            if (n > 0) {
                for (int q = 0; q < p.z_parts; ++q) {
                    float v[4];
                    load4(static_cast<const float *>(p.A) + ((int64_t)q * p.M + m0) * p.lda + k0 + h, n, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] += v[i];
                }
                if (p.z_bias) load4(static_cast<const T *>(p.z_bias) + (int64_t)e * K + k0 + h, n, b4);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) r[h + i] = i < n ? (T)act_value(p.act, z[i] + b4[i]) : (T)0.0f;
        }
        return __builtin_bit_cast(s16x8, r);
    };

    f32x4 acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = f32x4{0, 0, 0, 0};
    auto multiply = [&](const s16x8 &va, const s16x8 *vb) {
        s16x8 f[8];
        turn(vb, f);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            acc[j] = mma(__builtin_bit_cast(Frag, f[j]), __builtin_bit_cast(Frag, va), acc[j]);
    };
    int s = s0;
    typedef s16x8 any __attribute__((aligned(2)));
    if (last >= 0 && K >= 8) {
        const int whole = min(s1, K / 32);  // steps with all their features
        for (; s + kDeep <= whole; s += kDeep) {
            s16x8 va[kDeep], vb[kDeep][8];
#pragma unroll
            for (int d = 0; d < kDeep; ++d) {
                const int64_t k = (int64_t)(s + d) * 32;
                if (!Z) va[d] = *reinterpret_cast<const any *>(a + k);
#pragma unroll
                for (int q = 0; q < 8; ++q) vb[d][q] = *reinterpret_cast<const any *>(b + (k + q) * p.ldb);
            }
#pragma unroll
            for (int d = 0; d < kDeep; ++d) {
                if (Z) va[d] = inner8((s + d) * 32 + 8 * g);
                multiply(va[d], vb[d]);
            }
        }
        for (; s < s1; ++s) {
            const int64_t k = (int64_t)s * 32;
            const int left = K - s * 32 - 8 * g;  // features of the lane's eight
            s16x8 va, vb[8];
            if (!Z) va = *reinterpret_cast<const any *>(a + k + min(0, left - 8));
#pragma unroll
            for (int q = 0; q < 8; ++q) vb[q] = *reinterpret_cast<const any *>(b + (k + min(q, left - 1)) * p.ldb);
            if (Z) va = inner8(s * 32 + 8 * g);
            if (left < 8) {
                if (!Z) va = shift_out(va, left);
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (q >= left) vb[q] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
            }
            multiply(va, vb);
        }
    }
    for (; s < s1; ++s) {  // fewer than eight columns or features
        const int64_t k = (int64_t)s * 32;
        const int left = K - s * 32 - 8 * g;
        s16x8 vb[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) vb[q] = load8(b + (k + q) * p.ldb, q < left ? cols : 0);
        multiply(Z ? inner8(s * 32 + 8 * g) : load8(a + k, left), vb);
    }

    // Lane (m, g) has columns (4g + i) 8 + j of row m in acc[j][i].
    if (n0 + kCols <= N) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<f32x4 *>(&lds[wave][c][(4 * g + i) * 8 + 4 * h]) =
                    f32x4{acc[4 * h][i], acc[4 * h + 1][i], acc[4 * h + 2][i], acc[4 * h + 3][i]};
    } else {  // lanes moved back leave the same sums in the same places
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                lds[wave][c][(last >= 0 ? min((4 * g + i) * 8, last) : (4 * g + i) * 8) + j] = acc[j][i];
    }
    __syncthreads();
    const int q4 = threadIdx.x % (kCols / 4) * 4, n = n0 + q4, cnt = min(4, N - n);
    const int skip = max(0, n_from - n);  // of the four, columns that the tile before writes
    for (int r = threadIdx.x / (kCols / 4); r < m1 - m0 && cnt > skip; r += 2 * kWaves) {
        const int m = m0 + r;
        f32x4 sum = *reinterpret_cast<const f32x4 *>(&lds[0][r][q4]);
#pragma unroll
        for (int w = 1; w < kWaves; ++w) sum += *reinterpret_cast<const f32x4 *>(&lds[w][r][q4]);
        float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        float wr = 1.0f;
        if (EPI == kPairs || (EPI == kInner && p.weighted))
            wr = p.pair_w ? (float)static_cast<const T *>(p.pair_w)[m] : p.w ? p.w[m] : 1.0f;
        if (p.bias && split == 0) {
            float bias[4];
            if (p.bias_f32) load4(static_cast<const float *>(p.bias) + (int64_t)e * p.strideBias + n, cnt, bias);
            else load4(static_cast<const T *>(p.bias) + (int64_t)e * p.strideBias + n, cnt, bias);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] += bias[q];
        }
        if (EPI == kPairs) {
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] *= wr;
            store4(static_cast<float *>(p.out) + ((int64_t)split * p.M + m) * p.ldo + n, skip, cnt, v);
            continue;
        }
        if (p.pre) store4(static_cast<T *>(p.pre) + (int64_t)m * p.ldp + n, skip, cnt, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = EPI == kLinear && p.out_f32 ? act_fine(p.act, v[q]) : act_value(p.act, v[q]);
        if (EPI == kInner && p.weighted) {
            const float t[4] = {v[0] * wr, v[1] * wr, v[2] * wr, v[3] * wr};
            store4(static_cast<T *>(p.weighted) + (int64_t)m * p.ldo + n, skip, cnt, t);
        }
        if (EPI == kLinear && p.res) {
            float t4[4];
            load4(static_cast<const T *>(p.res) + (int64_t)m * p.ldr + n, cnt, t4);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] += t4[q];
        }
        if (EPI == kLinear && p.out_f32) store4(static_cast<float *>(p.out) + (int64_t)m * p.ldo + n, skip, cnt, v);
        else store4(static_cast<T *>(p.out) + (int64_t)m * p.ldo + n, skip, cnt, v);
    }
}

template <typename T> hipError_t go(Epilogue e, const Product &p, int splits, hipStream_t st)
{
    const int64_t rows = p.pairs ? p.M : launch_tile_rows(p, kTileFew);
    const int64_t blocks = rows * ((p.N + kCols - 1) / kCols) * splits;
    const dim3 grid = grid_of(blocks);
    if (grid.x == 0) return hipErrorInvalidValue;
    auto with = [&](auto kernel, int waves) {
        hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), 0, st, p, splits);
        return hipGetLastError();
    };
    if (p.z_parts) return with(k_few<T, kPairs, 8, true>, 8);
    // Eight waves bring a tile's part of the matrix at once; from two tiles a CU on four do, so that
    // one workgroup's loads run while the other adds up.
    if (blocks >= 512)
        return e == kLinear ? with(k_few<T, kLinear, 4>, 4)
               : e == kInner ? with(k_few<T, kInner, 4>, 4)
                             : with(k_few<T, kPairs, 4>, 4);
    return e == kLinear ? with(k_few<T, kLinear, 8>, 8)
           : e == kInner ? with(k_few<T, kInner, 8>, 8)
                         : with(k_few<T, kPairs, 8>, 8);
}

}  // namespace

hipError_t launch_few(bool bf16, Epilogue e, const Product &p, int splits, hipStream_t st)
{
    if (p.M <= 0 || p.N <= 0) return hipSuccess;
    return bf16 ? go<__bf16>(e, p, splits, st) : go<_Float16>(e, p, splits, st);
}

}  // namespace som
