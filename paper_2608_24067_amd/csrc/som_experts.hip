// som_experts.hip -- what the experts' products (som_mm*.hip) need around them: the pairs (row,
// place) in the order of their experts, the sum of a row's results, and the smaller gradients.

#include "som_mm.h"

namespace som {
namespace {

using mm::load4;
using mm::store4;

// One workgroup orders all pairs: each wave counts its stretch of them by expert, a scan over
// waves and experts gives every wave its first place in every expert, and each wave places its
// pairs 64 at a time, a pair after those of the same expert in lower lanes. The order is the
// pairs' own within an expert, so sums over it are the same on every run.
template <typename T>
__global__ __launch_bounds__(1024) void k_pairs(const int32_t *__restrict__ idx, const T *__restrict__ w, int P,
                                                 int k, int E, int rows, const PairPlan plan)
{
    extern __shared__ int lds[];
    const int waves = blockDim.x / 64, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    int *count = lds;                // [waves][E]
    int *start = lds + waves * E;    // [E]
    int *scan = start + E;           // [2][blockDim.x]
    for (int i = threadIdx.x; i < waves * E; i += blockDim.x) count[i] = 0;
    __syncthreads();
    const int stretch = ((P + waves - 1) / waves + 63) / 64 * 64;
    const int64_t first = (int64_t)wave * stretch, last = min((int64_t)P, first + stretch);
    for (int64_t i = first + lane; i < last; i += 64) {
        const int e = idx[i];
        if (e >= 0 && e < E) atomicAdd(&count[wave * E + e], 1);
    }
    __syncthreads();
    // E <= blockDim.x: a thread an expert
    const int e = threadIdx.x;
    int own = 0;
    if (e < E)
        for (int v = 0; v < waves; ++v) {
            const int c = count[v * E + e];
            count[v * E + e] = own;
            own += c;
        }
    const int tiles = (own + rows - 1) / rows;
    int *a = scan, *b = scan + blockDim.x;
    a[e] = own;
    b[e] = tiles;
    __syncthreads();
    for (int d = 1; d < (int)blockDim.x; d *= 2) {
        const int x = e >= d ? a[e - d] : 0, y = e >= d ? b[e - d] : 0;
        __syncthreads();
        a[e] += x;
        b[e] += y;
        __syncthreads();
    }
    if (e < E) {
        const int at = a[e] - own;
        start[e] = at;
        plan.off[e] = at;
        if (e == E - 1) {
            plan.off[E] = a[e];
            *plan.n_tiles = b[e];
        }
        for (int t = 0; t < tiles; ++t) plan.tiles[b[e] - tiles + t] = TileRow{e, at + t * rows, at + own, 0};
    }
    __syncthreads();
    volatile int *mine = count + wave * E;  // read and then written by one wave, in order
    for (int64_t i0 = first; i0 < last; i0 += 64) {
        const int64_t i = i0 + lane;
        const int x = i < last ? idx[i] : -1;
        const bool ok = x >= 0 && x < E;
        unsigned long long same = __ballot(ok);
        for (int bit = 0; bit < 10; ++bit) {
            const unsigned long long v = __ballot(x >> bit & 1);
            same &= (x >> bit & 1) ? v : ~v;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        const int base = ok ? mine[x] : 0;
        __builtin_amdgcn_wave_barrier();
        if (ok && before == 0) mine[x] = base + __popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (i < last) {
            const int p = ok ? start[x] + base + before : -1;
            plan.pos[i] = p;
            if (ok) {
                plan.row[p] = (int)(i / k);
                plan.w[p] = (float)w[i];
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_combine(const float *__restrict__ y, const int32_t *__restrict__ pos,
                                                 int64_t N, int k, int64_t D, const T *__restrict__ res, int64_t ldr,
                                                 T *out, int64_t ldo)
{
    const int64_t per = (D + 3) / 4, total = N * per;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t n = t / per, d = t % per * 4;
        const int cnt = (int)min((int64_t)4, D - d);
        float s[4] = {0, 0, 0, 0};
        if (res) load4(res + n * ldr + d, cnt, s);
        for (int j = 0; j < k; ++j) {
            const int p = pos[n * k + j];
            if (p < 0) continue;
            float v[4];
            load4(y + (int64_t)p * D + d, cnt, v);
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] += v[q];
        }
        store4(out + n * ldo + d, cnt, s);
    }
}

// A wave a row.
template <typename T>
__global__ __launch_bounds__(256) void k_weight_grad(const float *__restrict__ parts, int64_t n_parts,
                                                     const int32_t *__restrict__ pos, const int32_t *__restrict__ idx,
                                                     const T *__restrict__ b2, const T *__restrict__ dout, int64_t lddo,
                                                     int64_t N, int k, int64_t D, T *__restrict__ dw)
{
    const int lane = threadIdx.x % 64;
    const int64_t n = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
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

template <typename T>
__global__ __launch_bounds__(256) void k_slope(const T *__restrict__ dy, int64_t lddy, const T *__restrict__ pre,
                                               int64_t ldp, int act, int64_t N, int64_t M, T *__restrict__ dz)
{
    const int64_t per = (M + 3) / 4, total = N * per;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t n = t / per, m = t % per * 4;
        const int cnt = (int)min((int64_t)4, M - m);
        float g[4], z[4];
        load4(dy + n * lddy + m, cnt, g);
        load4(pre + n * ldp + m, cnt, z);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float value, slope;
            mm::act_both(act, z[q], value, slope);
            g[q] *= slope;
        }
        store4(dz + n * M + m, cnt, g);
    }
}

unsigned spread(int64_t items) { return (unsigned)(items < 1 ? 1 : items > 65536 ? 65536 : items); }

}  // namespace

hipError_t launch_pairs(bool bf16, const int32_t *idx, const void *w, int64_t P, int32_t k, int32_t E, int rows,
                        const PairPlan &plan, hipStream_t st)
{
    int waves = P <= 512 && E <= 256 ? 4 : E <= 512 ? 8 : 16;  // a thread an expert at least
    if (P > 4096 && E <= 512) waves = 16;
    const size_t lds = ((size_t)waves * E + E + 2 * 64 * waves) * sizeof(int);  // at most 77 KB
    if (lds > 64 << 10) {
        const hipError_t e = hipFuncSetAttribute(
            bf16 ? reinterpret_cast<const void *>(&k_pairs<__bf16>) : reinterpret_cast<const void *>(&k_pairs<_Float16>),
            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    if (bf16)
        hipLaunchKernelGGL(k_pairs<__bf16>, dim3(1), dim3(64 * waves), lds, st, idx, static_cast<const __bf16 *>(w),
                           (int)P, k, E, rows, plan);
    else
        hipLaunchKernelGGL(k_pairs<_Float16>, dim3(1), dim3(64 * waves), lds, st, idx,
                           static_cast<const _Float16 *>(w), (int)P, k, E, rows, plan);
    return hipGetLastError();
}

hipError_t launch_combine(bool bf16, const float *y, const int32_t *pos, int64_t N, int32_t k, int64_t D,
                          const void *res, int64_t ldr, void *out, int64_t ldo, hipStream_t st)
{
    const unsigned grid = spread((N * ((D + 3) / 4) + 255) / 256);
    if (bf16)
        hipLaunchKernelGGL(k_combine<__bf16>, dim3(grid), dim3(256), 0, st, y, pos, N, k, D,
                           static_cast<const __bf16 *>(res), ldr, static_cast<__bf16 *>(out), ldo);
    else
        hipLaunchKernelGGL(k_combine<_Float16>, dim3(grid), dim3(256), 0, st, y, pos, N, k, D,
                           static_cast<const _Float16 *>(res), ldr, static_cast<_Float16 *>(out), ldo);
    return hipGetLastError();
}

hipError_t launch_weight_grad(bool bf16, const float *parts, int64_t n_parts, const int32_t *pos, const int32_t *idx,
                              const void *b2, const void *dout, int64_t lddo, int64_t N, int32_t k, int64_t D,
                              void *dw, hipStream_t st)
{
    const unsigned grid = (unsigned)((N + 3) / 4);
    if (bf16)
        hipLaunchKernelGGL(k_weight_grad<__bf16>, dim3(grid), dim3(256), 0, st, parts, n_parts, pos, idx,
                           static_cast<const __bf16 *>(b2), static_cast<const __bf16 *>(dout), lddo, N, k, D,
                           static_cast<__bf16 *>(dw));
    else
        hipLaunchKernelGGL(k_weight_grad<_Float16>, dim3(grid), dim3(256), 0, st, parts, n_parts, pos, idx,
                           static_cast<const _Float16 *>(b2), static_cast<const _Float16 *>(dout), lddo, N, k, D,
                           static_cast<_Float16 *>(dw));
    return hipGetLastError();
}

hipError_t launch_slope(bool bf16, const void *dy, int64_t lddy, const void *pre, int64_t ldp, int act, int64_t N,
                        int64_t M, void *dz, hipStream_t st)
{
    const unsigned grid = spread((N * ((M + 3) / 4) + 255) / 256);
    if (bf16)
        hipLaunchKernelGGL(k_slope<__bf16>, dim3(grid), dim3(256), 0, st, static_cast<const __bf16 *>(dy), lddy,
                           static_cast<const __bf16 *>(pre), ldp, act, N, M, static_cast<__bf16 *>(dz));
    else
        hipLaunchKernelGGL(k_slope<_Float16>, dim3(grid), dim3(256), 0, st, static_cast<const _Float16 *>(dy), lddy,
                           static_cast<const _Float16 *>(pre), ldp, act, N, M, static_cast<_Float16 *>(dz));
    return hipGetLastError();
}

}  // namespace som
