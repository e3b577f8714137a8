// som_experts.hip -- what the experts' products (som_mm*.hip) need around them: the pairs (row,
// place) in the order of their experts, the sum of a row's results, and the smaller gradients.

#include "som_mm.h"

namespace som {
namespace {

using mm::block_number;
using mm::load4;
using mm::store4;

// The pairs are ordered by counting: stretches of them, a wave each, are counted by expert; a
// scan over stretches and experts gives every stretch its first place in every expert; and each
// wave places its pairs 64 at a time, a pair after those of the same expert in lower lanes. The
// order is the pairs' own within an expert, so sums over it are the same on every run. Few pairs
// take one workgroup for all three (16 stretches at most); more take a kernel each.

// f(pair, expert or -1, weight) for a stretch, 64 pairs at a time; what is read of them is loaded
// eight times 64 at a time. w may be null.
template <typename T, typename F>
__device__ inline void chunks_of(const int32_t *idx, const T *w, int64_t first, int64_t last, int E, F f)
{
    const int lane = threadIdx.x % 64;
    for (int64_t i0 = first; i0 < last; i0 += 512) {
        int x[8];
        T v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const int64_t i = i0 + c * 64 + lane;
            x[c] = i < last ? idx[i] : -1;
            v[c] = w && i < last ? w[i] : (T)0.0f;
        }
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (i0 + c * 64 < last) f(i0 + c * 64 + lane, (unsigned)x[c] < (unsigned)E ? x[c] : -1, v[c]);
    }
}

// own: the expert's pairs (0 beyond E), a thread an expert. Writes the experts' starts and tile
// rows; scan: 2 * blockDim.x words of LDS. Returns the expert's start.
__device__ inline int lay_out(int own, int E, int rows, int *scan, const PairPlan &plan)
{
    const int e = threadIdx.x, tiles = (own + rows - 1) / rows;
    int *a = scan, *b = scan + blockDim.x;
    a[e] = own;
    b[e] = tiles;
    __syncthreads();
    for (int d = 1; d < (int)blockDim.x && d < E; d *= 2) {
        const int x = e >= d ? a[e - d] : 0, y = e >= d ? b[e - d] : 0;
        __syncthreads();
        a[e] += x;
        b[e] += y;
        __syncthreads();
    }
    const int at = a[e] - own;
    if (e < E) {
        plan.off[e] = at;
        if (e == E - 1) {
            plan.off[E] = a[e];
            *plan.n_tiles = b[e];
        }
        for (int t = 0; t < tiles; ++t) plan.tiles[b[e] - tiles + t] = TileRow{e, at + t * rows, at + own, 0};
    }
    return at;
}

// next[e]: the stretch's next place of expert e, in LDS, the wave's own.
template <typename T>
__device__ inline void place(const int32_t *idx, const T *w, int64_t first, int64_t last, int k, int E,
                             volatile int *next, const PairPlan &plan)
{
    const int lane = threadIdx.x % 64;
    chunks_of(idx, w, first, last, E, [&](int64_t i, int x, T weight) {
        const bool ok = x >= 0;
        unsigned long long same = __ballot(ok);
        for (int bit = 0; 1 << bit < E; ++bit) {
            const unsigned long long v = __ballot(x >> bit & 1);
            same &= (x >> bit & 1) ? v : ~v;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        const int base = ok ? next[x] : 0;
        __builtin_amdgcn_wave_barrier();
        if (ok && before == 0) next[x] = base + __popcll(same);  // reads before writes: one wave, in order
        __builtin_amdgcn_wave_barrier();
        if (i < last) {
            const int p = ok ? base + before : -1;
            plan.pos[i] = p;
            if (ok) {
                plan.row[p] = (int)i / k;  // fewer than 2^30 pairs
                plan.w[p] = (float)weight;
            }
        }
    });
}

__device__ inline int64_t stretch_of(int64_t P, int waves) { return ((P + waves - 1) / waves + 63) / 64 * 64; }

template <typename T>
__global__ __launch_bounds__(1024) void k_pairs(const int32_t *__restrict__ idx, const T *__restrict__ w, int64_t P,
                                                int k, int E, int rows, const PairPlan plan)
{
    extern __shared__ int lds[];
    const int waves = blockDim.x / 64, wave = threadIdx.x / 64;
    int *count = lds, *scan = lds + waves * E;  // [waves][E], [2][blockDim.x]
    for (int i = threadIdx.x; i < waves * E; i += blockDim.x) count[i] = 0;
    __syncthreads();
    const int64_t first = wave * stretch_of(P, waves), last = min(P, first + stretch_of(P, waves));
    chunks_of(idx, (const T *)nullptr, first, last, E, [&](int64_t, int x, T) {
        if (x >= 0) atomicAdd(&count[wave * E + x], 1);
    });
    __syncthreads();
    int own = 0;
    if ((int)threadIdx.x < E)
        for (int v = 0; v < waves; ++v) own += count[v * E + threadIdx.x];
    int at = lay_out(own, E, rows, scan, plan);
    if ((int)threadIdx.x < E)
        for (int v = 0; v < waves; ++v) {
            const int c = count[v * E + threadIdx.x];
            count[v * E + threadIdx.x] = at;
            at += c;
        }
    __syncthreads();
    place(idx, w, first, last, k, E, count + wave * E, plan);
}

// counts: [gridDim.x][E], one wave a workgroup.
__global__ __launch_bounds__(64) void k_pairs_count(const int32_t *__restrict__ idx, int64_t P, int E, int32_t *counts)
{
    extern __shared__ int lds[];
    for (int i = threadIdx.x; i < E; i += 64) lds[i] = 0;
    __syncthreads();
    const int64_t len = stretch_of(P, gridDim.x), first = blockIdx.x * len, last = min(P, first + len);
    chunks_of(idx, (const float *)nullptr, first, last, E, [&](int64_t, int x, float) {
        if (x >= 0) atomicAdd(&lds[x], 1);
    });
    __syncthreads();
    for (int i = threadIdx.x; i < E; i += 64) counts[(int64_t)blockIdx.x * E + i] = lds[i];
}

// The counts become each stretch's first places. A thread takes an expert's counts of a part of the
// stretches (parts * lanes = 1,024 threads, lanes a power of two of E at least).
__global__ __launch_bounds__(1024) void k_pairs_scan(int32_t *counts, int stretches, int E, int lanes, int rows,
                                                     const PairPlan plan)
{
    __shared__ int scan[2 * 1024], part[1024], start[1024];
    const int e = threadIdx.x & (lanes - 1), at_part = threadIdx.x / lanes, parts = 1024 / lanes;
    const int len = (stretches + parts - 1) / parts, v0 = min(stretches, at_part * len), v1 = min(stretches, v0 + len);
    int own = 0;
    if (e < E) {
#pragma unroll 8
        for (int v = v0; v < v1; ++v) own += counts[v * E + e];
    }
    part[threadIdx.x] = own;
    __syncthreads();
    int total = 0;
    if ((int)threadIdx.x < E)
        for (int q = 0; q < parts; ++q) total += part[q * lanes + threadIdx.x];
    const int first = lay_out(total, E, rows, scan, plan);
    if ((int)threadIdx.x < E) start[threadIdx.x] = first;
    __syncthreads();
    if (e < E) {
        int at = start[e];
        for (int q = 0; q < at_part; ++q) at += part[q * lanes + e];
#pragma unroll 8
        for (int v = v0; v < v1; ++v) {
            const int c = counts[v * E + e];
            counts[v * E + e] = at;
            at += c;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(64) void k_pairs_place(const int32_t *__restrict__ idx, const T *__restrict__ w, int64_t P,
                                                    int k, int E, const int32_t *__restrict__ counts, const PairPlan plan)
{
    extern __shared__ int lds[];
    for (int i = threadIdx.x; i < E; i += 64) lds[i] = counts[(int64_t)blockIdx.x * E + i];
    __syncthreads();
    const int64_t len = stretch_of(P, gridDim.x), first = blockIdx.x * len, last = min(P, first + len);
    place(idx, w, first, last, k, E, lds, plan);
}

template <typename T, bool SPLIT>
__global__ __launch_bounds__(256) void k_combine(const float *__restrict__ y, int splits,
                                                 const int32_t *__restrict__ pos, int no_plan_E, int64_t N, int k, int64_t D, const T *__restrict__ res, int64_t ldr,
                                                 T *out, int64_t ldo)
{
    const int64_t per = (D + 3) / 4, total = N * per;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t n = t / per, d = t % per * 4;
        const int cnt = (int)min((int64_t)4, D - d);
        float s[4] = {0, 0, 0, 0};
        if (res) load4(res + n * ldr + d, cnt, s);
        for (int j = 0; j < k; ++j) {
            int p = pos[n * k + j];
            if (no_plan_E) p = (unsigned)p < (unsigned)no_plan_E ? (int)(n * k + j) : -1;
            if (p < 0) continue;
            float v[4];
            load4(y + (int64_t)p * D + d, cnt, v);
            if (SPLIT) {
#pragma unroll 8
                for (int r = 1; r < splits; ++r) {
                    float u[4];
                    load4(y + (r * N * k + p) * D + d, cnt, u);
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] += u[q];
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] += v[q];
        }
        store4(out + n * ldo + d, cnt, s);
    }
}

// The same for few rows of many parts (k * splits): 64 columns a workgroup, each of its four waves
// a quarter of the parts, their sums added in order.
template <typename T>
__global__ __launch_bounds__(256) void k_combine_few(const float *__restrict__ y, int splits,
                                                     const int32_t *__restrict__ pos, int no_plan_E, int64_t N, int k,
                                                     int64_t D, const T *__restrict__ res, int64_t ldr, T *out,
                                                     int64_t ldo)
{
    __shared__ float part[4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t per = (D + 63) / 64, n = blockIdx.x / per, d = blockIdx.x % per * 64 + lane;
    const int all = k * splits, len = (all + 3) / 4, i1 = min(all, (wave + 1) * len);
    float s = 0;
    if (d < D) {
#pragma unroll 8
        for (int i = wave * len; i < i1; ++i) {
            int p = pos[n * k + i / splits];
            if (no_plan_E) p = (unsigned)p < (unsigned)no_plan_E ? (int)(n * k + i / splits) : -1;
            s += p >= 0 ? y[((int64_t)(i % splits) * N * k + p) * D + d] : 0.0f;
        }
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && d < D)
        out[n * ldo + d] = (T)((res ? (float)res[n * ldr + d] : 0.0f) + part[0][lane] + part[1][lane] + part[2][lane] +
                               part[3][lane]);
}

// A wave a row.
template <typename T>
__global__ __launch_bounds__(256) void k_weight_grad(const float *__restrict__ parts, int64_t n_parts,
                                                     const int32_t *__restrict__ pos, const int32_t *__restrict__ idx,
                                                     const T *__restrict__ b2, const T *__restrict__ dout, int64_t lddo,
                                                     int64_t N, int k, int64_t D, T *__restrict__ dw)
{
    const int lane = threadIdx.x % 64;
    const int64_t n = block_number() * 4 + threadIdx.x / 64;
    if (n >= N) return;
    for (int j = 0; j < k; ++j) {
        const int p = pos[n * k + j];
        float s = 0;
        if (p >= 0) {
            for (int64_t q = lane; q < n_parts; q += 64) s += parts[p * n_parts + q];
            if (b2) {
                const T *b = b2 + idx[n * k + j] * D;
                for (int64_t d = 4 * lane; d < D; d += 256) {
                    const int cnt = (int)min((int64_t)4, D - d);
                    float x[4], g[4];
                    load4(b + d, cnt, x);
                    load4(dout + n * lddo + d, cnt, g);
#pragma unroll
                    for (int q = 0; q < 4; ++q) s += x[q] * g[q];
                }
            }
        }
        for (int d = 32; d > 0; d /= 2) s += __shfl_xor(s, d);
        if (lane == 0) dw[n * k + j] = (T)s;
    }
}

// in: parts arrays of n values; four values a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_sum_parts(const float *__restrict__ in, int parts, int64_t n, int64_t M,
                                                   T *__restrict__ out, int64_t ldo)
{
    const int64_t per = (M + 3) / 4, total = n / M * per;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t row = t / per, m = t % per * 4;
        const int cnt = (int)min((int64_t)4, M - m);
        float s[4] = {0, 0, 0, 0};
#pragma unroll 8
        for (int r = 0; r < parts; ++r) {
            float v[4];
            load4(in + r * n + row * M + m, cnt, v);
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] += v[q];
        }
        store4(out + row * ldo + m, cnt, s);
    }
}

// Eight values of a row a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_slope(const T *__restrict__ dy, int64_t lddy, const T *__restrict__ pre,
                                               int64_t ldp, int act, int64_t N, int64_t M, T *__restrict__ dz)
{
    typedef T vec __attribute__((ext_vector_type(8)));
    typedef vec any __attribute__((aligned(2)));
    const int64_t per = (M + 7) / 8, total = N * per;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t n = t / per, m = t % per * 8;
        const T *g = dy + n * lddy + m, *z = pre + n * ldp + m;
        T *out = dz + n * M + m;
        float value, slope;
        if (m + 8 <= M) {
            const vec gv = *reinterpret_cast<const any *>(g), zv = *reinterpret_cast<const any *>(z);
            vec r;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                mm::act_both(act, (float)zv[q], value, slope);
                r[q] = (T)((float)gv[q] * slope);
            }
            *reinterpret_cast<any *>(out) = r;
        } else {
            for (int q = 0; m + q < M; ++q) {
                mm::act_both(act, (float)z[q], value, slope);
                out[q] = (T)((float)g[q] * slope);
            }
        }
    }
}

unsigned spread(int64_t items) { return (unsigned)(items < 1 ? 1 : items > 65536 ? 65536 : items); }

}  // namespace

hipError_t launch_pairs(bool bf16, const int32_t *idx, const void *w, int64_t P, int32_t k, int32_t E, int rows,
                        const PairPlan &plan, hipStream_t st)
{
    auto with = [&](auto one, auto many, auto *weights) {
        if (P <= kPairsOfOne) {
            const int waves = E <= 256 ? (P <= 512 ? 4 : 16) : E <= 512 ? 8 : 16;  // a thread an expert at least
            const size_t lds = ((size_t)waves * E + 2 * 64 * waves) * sizeof(int);  // at most 72 KB
            if (lds > 64 << 10) {
                const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(one),
                                                         hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
                if (e != hipSuccess) return e;
            }
            hipLaunchKernelGGL(one, dim3(1), dim3(64 * waves), lds, st, idx, weights, P, k, E, rows, plan);
            return hipGetLastError();
        }
        const int n = pair_stretches(P);
        hipLaunchKernelGGL(k_pairs_count, dim3(n), dim3(64), E * sizeof(int), st, idx, P, E, plan.counts);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        int lanes = 16;
        while (lanes < E) lanes *= 2;
        hipLaunchKernelGGL(k_pairs_scan, dim3(1), dim3(1024), 0, st, plan.counts, n, E, lanes, rows, plan);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL(many, dim3(n), dim3(64), E * sizeof(int), st, idx, weights, P, k, E, plan.counts, plan);
        return hipGetLastError();
    };
    return bf16 ? with(&k_pairs<__bf16>, &k_pairs_place<__bf16>, static_cast<const __bf16 *>(w))
                : with(&k_pairs<_Float16>, &k_pairs_place<_Float16>, static_cast<const _Float16 *>(w));
}

hipError_t launch_combine(bool bf16, const float *y, int splits, const int32_t *pos, int32_t no_plan_E, int64_t N, int32_t k, int64_t D,
                          const void *res, int64_t ldr, void *out, int64_t ldo, hipStream_t st)
{
    const unsigned grid = spread((N * ((D + 3) / 4) + 255) / 256);
    // From eight parts on, where four columns a thread do not fill the CUs (one row of 1,024 columns,
    // two places, 16 splits: 10.6 us).
    const bool few = k * splits >= 8 && N * D < 256 * 1024;
    auto with = [&](auto kernel, const auto *r, auto *o) {
        hipLaunchKernelGGL(kernel, dim3(few ? (unsigned)(N * ((D + 63) / 64)) : grid), dim3(256), 0, st, y, splits, pos,
                           no_plan_E, N, k, D, r, ldr, o, ldo);
        return hipGetLastError();
    };
    if (few && bf16) return with(&k_combine_few<__bf16>, static_cast<const __bf16 *>(res), static_cast<__bf16 *>(out));
    if (few) return with(&k_combine_few<_Float16>, static_cast<const _Float16 *>(res), static_cast<_Float16 *>(out));
    if (bf16) {
        const auto *r = static_cast<const __bf16 *>(res);
        auto *o = static_cast<__bf16 *>(out);
        return splits > 1 ? with(&k_combine<__bf16, true>, r, o) : with(&k_combine<__bf16, false>, r, o);
    }
    const auto *r = static_cast<const _Float16 *>(res);
    auto *o = static_cast<_Float16 *>(out);
    return splits > 1 ? with(&k_combine<_Float16, true>, r, o) : with(&k_combine<_Float16, false>, r, o);
}

hipError_t launch_weight_grad(bool bf16, const float *parts, int64_t n_parts, const int32_t *pos, const int32_t *idx,
                              const void *b2, const void *dout, int64_t lddo, int64_t N, int32_t k, int64_t D,
                              void *dw, hipStream_t st)
{
    const dim3 grid = grid_of((N + 3) / 4);  // fewer than 2^28
    if (bf16)
        hipLaunchKernelGGL(k_weight_grad<__bf16>, grid, dim3(256), 0, st, parts, n_parts, pos, idx,
                           static_cast<const __bf16 *>(b2), static_cast<const __bf16 *>(dout), lddo, N, k, D,
                           static_cast<__bf16 *>(dw));
    else
        hipLaunchKernelGGL(k_weight_grad<_Float16>, grid, dim3(256), 0, st, parts, n_parts, pos, idx,
                           static_cast<const _Float16 *>(b2), static_cast<const _Float16 *>(dout), lddo, N, k, D,
                           static_cast<_Float16 *>(dw));
    return hipGetLastError();
}

hipError_t launch_sum_parts(bool bf16, const float *in, int parts, int64_t n, int64_t M, void *out, int64_t ldo,
                            bool out_f32, hipStream_t st)
{
    const unsigned grid = spread((n / M * ((M + 3) / 4) + 255) / 256);
    auto with = [&](auto kernel, auto *to) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, st, in, parts, n, M, to, ldo);
        return hipGetLastError();
    };
    if (out_f32) return with(&k_sum_parts<float>, static_cast<float *>(out));
    return bf16 ? with(&k_sum_parts<__bf16>, static_cast<__bf16 *>(out))
                : with(&k_sum_parts<_Float16>, static_cast<_Float16 *>(out));
}

hipError_t launch_slope(bool bf16, const void *dy, int64_t lddy, const void *pre, int64_t ldp, int act, int64_t N,
                        int64_t M, void *dz, hipStream_t st)
{
    const unsigned grid = spread((N * ((M + 7) / 8) + 255) / 256);
    if (bf16)
        hipLaunchKernelGGL(k_slope<__bf16>, dim3(grid), dim3(256), 0, st, static_cast<const __bf16 *>(dy), lddy,
                           static_cast<const __bf16 *>(pre), ldp, act, N, M, static_cast<__bf16 *>(dz));
    else
        hipLaunchKernelGGL(k_slope<_Float16>, dim3(grid), dim3(256), 0, st, static_cast<const _Float16 *>(dy), lddy,
                           static_cast<const _Float16 *>(pre), ldp, act, N, M, static_cast<_Float16 *>(dz));
    return hipGetLastError();
}

}  // namespace som
