// som_route.hip -- each row's k best units by its logits, their weights, and the gradient.
//
// A row is held in the registers of 16 or 64 lanes (LPR), VPL logits a lane, four neighbours at
// a time. The choice is k rounds of a maximum over order-preserving 32-bit images of
// logit + bias, the lowest index among equals; each lane offers its best unit and knows its
// second, and looks at its units again only when both are taken (one pass of VPL units instead
// of one a round). Softmax statistics are fp32, shifted by the row's maximum.

#include "som_mm.h"

namespace som {
namespace {

using mm::exp_f32;
using mm::load4;
using mm::store4;

template <int CTRL> __device__ inline uint32_t lane_swap(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}

// Over the LPR lanes of a row, in every lane: pairs, quads, half rows, rows of 16, then the wave.
template <int LPR, typename F> __device__ inline uint32_t reduce(uint32_t v, F f)
{
    v = f(v, lane_swap<0xB1>(v));
    v = f(v, lane_swap<0x4E>(v));
    v = f(v, lane_swap<0x141>(v));
    v = f(v, lane_swap<0x140>(v));
    if (LPR == 64) {
        const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
        const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
        v = f(f(a, b), f(c, d));
    }
    return v;
}

template <int LPR> __device__ inline uint32_t max_u32(uint32_t v)
{
    return reduce<LPR>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int LPR> __device__ inline uint32_t min_u32(uint32_t v)
{
    return reduce<LPR>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
template <int LPR> __device__ inline float max_f32(float v)
{
    return __uint_as_float(reduce<LPR>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}
template <int LPR> __device__ inline float sum_f32(float v)
{
    return __uint_as_float(reduce<LPR>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}

// Order-preserving image of a float that is neither NaN nor -inf; 0 stands for a closed unit.
__device__ inline uint32_t image(float v)
{
    const uint32_t u = __float_as_uint(v);
    return (u >> 31) ? ~u : u | 0x80000000u;
}

constexpr float kMost = 3.402823466e38f;

// A logit as it is weighed (+inf counts as the largest value), its ranked key's image (0: closed).
__device__ inline void open_unit(float logit, float bias, float &l, uint32_t &key)
{
    const float s = logit + bias;  // -0 + 0 is 0: the two zeros rank alike
    const bool open = logit > -__builtin_inff() && s > -__builtin_inff();  // false for NaN
    l = open ? fminf(logit, kMost) : -__builtin_inff();
    key = open ? image(s) : 0;
}

__device__ inline float score_sigmoid(float l) { return 1.0f / (1.0f + exp_f32(fminf(-l, 88.0f))); }

__device__ inline void store_weight(int type, void *p, int64_t at, float v)
{
    if (type == SOM_F32) static_cast<float *>(p)[at] = v;
    else if (type == SOM_F16) static_cast<_Float16 *>(p)[at] = (_Float16)v;
    else static_cast<__bf16 *>(p)[at] = (__bf16)v;
}

__device__ inline float load_weight(int type, const void *p, int64_t at)
{
    if (type == SOM_F32) return static_cast<const float *>(p)[at];
    if (type == SOM_F16) return (float)static_cast<const _Float16 *>(p)[at];
    return (float)static_cast<const __bf16 *>(p)[at];
}

// A taken unit's share of the taken units' scores (l: -inf in lanes without one). The scores are
// scaled by exp(-top), top the largest logit (sigmoid: or 0), so that some score is not small:
// under softmax the other units cancel, sigmoid(l) exp(-top) = exp(l - top) / (1 + exp(l)).
template <int LPR> __device__ inline float share(bool softmax, float l)
{
    float top = max_f32<LPR>(l);
    if (!softmax) top = fminf(top, 0.0f);
    float s = 0;
    if (l > -__builtin_inff())
        s = softmax ? exp_f32(l - top) : top < 0.0f ? exp_f32(l - top) / (1.0f + exp_f32(l)) : score_sigmoid(l);
    const float total = sum_f32<LPR>(s);
    return total > 0.0f ? s / total : 0.0f;
}

template <int LPR, int VPL> struct Row {
    // Logit i of lane `sub` of a row: neighbours of four, the lanes' fours side by side.
    __device__ static int unit(int i, int sub) { return (i >> 2) * 4 * LPR + 4 * sub + (i & 3); }

    float l[VPL];
    uint32_t key[VPL];

    template <typename T> __device__ void load(const T *p, const float *bias, int E, int sub)
    {
#pragma unroll
        for (int i = 0; i < VPL; i += 4) {
            const int e = unit(i, sub), n = max(0, min(4, E - e));
            float v[4] = {0, 0, 0, 0}, b[4] = {0, 0, 0, 0};
            if (n > 0) load4(p + e, n, v);
            if (bias && n > 0) load4(bias + e, n, b);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                open_unit(v[q], b[q], l[i + q], key[i + q]);
                if (q >= n) l[i + q] = -__builtin_inff(), key[i + q] = 0;
            }
        }
    }

    // The maximum of the open logits (-inf where none is) and the sum of exp(l - maximum).
    __device__ float top() const
    {
        float m = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < VPL; ++i) m = fmaxf(m, l[i]);
        return max_f32<LPR>(m);
    }
    __device__ float total(float m)  // l becomes exp(l - m), 0 where closed
    {
        const float shift = m > -__builtin_inff() ? m : 0.0f;
        float z = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            l[i] = exp_f32(l[i] - shift);
            z += l[i];
        }
        return sum_f32<LPR>(z);
    }

    // The lane's two best units that rank after (key, e); 0 where there is none.
    uint32_t v1, v2;
    int i1, i2;
    __device__ void two_best(uint32_t after, int e, int sub)
    {
        v1 = v2 = 0;
        i1 = i2 = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const uint32_t x = key[i] < after || (key[i] == after && unit(i, sub) > e) ? key[i] : 0;
            const bool first = x > v1, second = x > v2;
            i2 = first ? i1 : second ? i : i2;
            v2 = first ? v1 : second ? x : v2;
            i1 = first ? i : i1;
            v1 = first ? x : v1;
        }
    }
};

constexpr int kThreads = 256;

template <typename T, int LPR, int VPL> __global__ __launch_bounds__(kThreads) void k_route(const RouteArgs a)
{
    constexpr int kRows = kThreads / LPR;
    __shared__ uint32_t best[kRows][SOM_ROUTE_MAX_GROUPS];
    __shared__ unsigned long long kept[kRows];
    const int sub = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + slot;
    const bool in = row < a.N;
    const T *p = static_cast<const T *>(a.logits) + (in ? row : 0) * a.ldl;

    Row<LPR, VPL> r;
    r.load(p, a.bias, a.E, sub);
    float m = 0, z = 1;
    const bool softmax = a.score == SOM_SCORE_SOFTMAX;
    if (softmax && !a.renorm) {
        m = r.top();
        z = r.total(m);
    }
    if (a.groups > 1) {
        // Groups by their best unit; one is kept if fewer than group_top are better (the lower
        // one first among equals).
        const float inv = 1.0f / (float)(a.E / a.groups);  // (e + 1/2) inv is never near a whole number
        for (int g = sub; g < a.groups; g += LPR) best[slot][g] = 0;
        if (sub == 0) kept[slot] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (r.key[i]) atomicMax(&best[slot][(int)((Row<LPR, VPL>::unit(i, sub) + 0.5f) * inv)], r.key[i]);
        __syncthreads();
        for (int g = sub; g < a.groups; g += LPR) {
            const uint32_t own = best[slot][g];
            int better = 0;
            for (int h = 0; h < a.groups; ++h) {
                const uint32_t other = best[slot][h];
                better += other > own || (other == own && h < g);
            }
            if (better < a.group_top) atomicOr(&kept[slot], 1ull << g);
        }
        __syncthreads();
        const unsigned long long keep = kept[slot];
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (!(keep >> (int)((Row<LPR, VPL>::unit(i, sub) + 0.5f) * inv) & 1)) r.key[i] = 0;
    }

    // Place j is held by lane j of the row.
    int unit = -1;
    r.two_best(~0u, 0, sub);
    int left = 2;  // units the lane offers before it must look again
    uint32_t last = ~0u;
    int last_e = 0;
    for (int j = 0; j < a.k; ++j) {
        const int own = Row<LPR, VPL>::unit(r.i1, sub);
        const uint32_t w = max_u32<LPR>(r.v1);
        const int e = (int)min_u32<LPR>(r.v1 == w ? (uint32_t)own : ~0u);
        if (sub == j) unit = w ? e : -1;
        if (w && own == e && r.v1 == w) {
            last = w;
            last_e = e;
            r.v1 = r.v2;
            r.i1 = r.i2;
            r.v2 = 0;
            --left;
        }
        if (__any(left == 0) && j + 1 < a.k) {
            if (left == 0) {
                r.two_best(last, last_e, sub);
                left = 2;
            }
        }
    }

    const bool took = unit >= 0;
    const float l = took ? fminf((float)p[unit], kMost) : -__builtin_inff();
    float s = 0;
    if (a.renorm) s = share<LPR>(softmax, l);
    else if (took) s = softmax ? exp_f32(l - m) / z : score_sigmoid(l);
    if (in && sub < a.k) {
        a.idx[row * a.k + sub] = unit;
        store_weight(a.weight_type, a.weights, row * a.k + sub, s);
    }
    // The counts: one workgroup counts its own rows; of more, the first clears them for k_counts.
    if (a.counts && blockIdx.x == 0) {
        for (int i = threadIdx.x; i < a.E; i += kThreads) a.counts[i] = 0;
        if (gridDim.x == 1) {
            __threadfence_block();
            __syncthreads();
            if (in && took) atomicAdd(&a.counts[unit], 1);
        }
    }
}

// How many rows took each unit: a workgroup counts its share of the choices in LDS and adds what
// it found. (Adding every choice in global memory took 80 of 89 us for 16,411 rows and 8 of 256
// units: neighbouring counts share a cache line, and a line takes about 90 additions a us.)
__global__ __launch_bounds__(1024) void k_counts(const int32_t *__restrict__ idx, int64_t n, int E, int32_t *counts)
{
    __shared__ int own[SOM_ROUTE_MAX_UNITS];
    for (int i = threadIdx.x; i < E; i += 1024) own[i] = 0;
    __syncthreads();
    const int64_t step = (int64_t)gridDim.x * 1024;
#pragma unroll 4
    for (int64_t i = (int64_t)blockIdx.x * 1024 + threadIdx.x; i < n; i += step) {
        const int e = idx[i];
        if (e >= 0) atomicAdd(&own[e], 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < E; i += 1024)
        if (own[i]) atomicAdd(&counts[i], own[i]);
}

// softmax: dl = p (dw - sum dw p) over all open units (dw is 0 where a unit was not taken);
// renormalised: dl = w (dw - sum dw w) over the taken ones; sigmoid: dl = dw s (1 - s);
// renormalised: dl = w (1 - s) (dw - sum dw w).
template <typename T, int LPR, int VPL> __global__ __launch_bounds__(kThreads) void k_route_bwd(const RouteArgs a)
{
    constexpr int kRows = kThreads / LPR;
    const int sub = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + slot;
    const bool in = row < a.N;
    const int64_t at = in ? row : 0;
    const T *p = static_cast<const T *>(a.logits) + at * a.ldl;
    T *d = static_cast<T *>(a.dlogits) + at * a.lddl;
    const bool softmax = a.score == SOM_SCORE_SOFTMAX, shares = softmax && !a.renorm;

    int unit = sub < a.k ? a.idx[at * a.k + sub] : -1;
    float l = -__builtin_inff();
    if (unit >= 0 && unit < a.E) {
        uint32_t key;
        open_unit((float)p[unit], a.bias ? a.bias[unit] : 0.0f, l, key);
        if (!key) unit = -1;
    } else {
        unit = -1;
    }
    const bool took = unit >= 0;
    const float dw = took ? load_weight(a.weight_type, a.weights, at * a.k + sub) : 0.0f;

    Row<LPR, VPL> r;
    float m = 0, z = 1;
    if (shares) {
        r.load(p, a.bias, a.E, sub);
        m = r.top();
        z = r.total(m);
    }
    const float over = z > 0.0f ? 1.0f / z : 0.0f;
    float g, sum = 0;  // g: the taken unit's gradient
    if (a.renorm) {
        const float w = share<LPR>(softmax, l);
        g = w * (dw - sum_f32<LPR>(dw * w));
        if (!softmax && took) g *= score_sigmoid(-l);
    } else if (softmax) {
        const float s = took ? exp_f32(l - m) * over : 0.0f;
        sum = sum_f32<LPR>(dw * s);
        g = s * (dw - sum);
    } else {
        g = took ? dw * score_sigmoid(l) * score_sigmoid(-l) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) r.l[i] = shares ? -sum * over * r.l[i] : 0.0f;
    for (int j = 0; j < a.k; ++j) {  // the taken units in their lanes
        if (LPR == 64) {
            const int u = __builtin_amdgcn_readlane(unit, j);
            const float gj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), j));
            if (u < 0) continue;
            const int at = (u / (4 * LPR)) * 4 + u % 4;  // the same register in every lane
            const bool mine = u / 4 % LPR == sub;
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (i == at) r.l[i] = mine ? gj : r.l[i];
        } else {
            const int u = __shfl(unit, j, LPR);
            const float gj = __shfl(g, j, LPR);
#pragma unroll
            for (int i = 0; i < VPL; ++i) r.l[i] = Row<LPR, VPL>::unit(i, sub) == u ? gj : r.l[i];
        }
    }
#pragma unroll
    for (int i = 0; i < VPL; i += 4) {
        const int e = Row<LPR, VPL>::unit(i, sub), n = max(0, min(4, a.E - e));
        if (in && n > 0) store4(d + e, n, &r.l[i]);
    }
}

__global__ void k_zero(int32_t *p, int n)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) p[i] = 0;
}

// Lanes that hold a row, and the rows of a workgroup.
int lanes_of(const RouteArgs &a) { return a.E <= 256 && a.k <= 16 ? 16 : 64; }
int rows_of_one(const RouteArgs &a) { return kThreads / lanes_of(a); }

template <typename T, bool BWD> hipError_t pick(const RouteArgs &a, hipStream_t st)
{
    auto go = [&](auto kernel, int lpr) {
        const int64_t rows = kThreads / lpr, grid = (a.N + rows - 1) / rows;
        if (grid > INT32_MAX) return hipErrorInvalidValue;
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kThreads), 0, st, a);
        return hipGetLastError();
    };
    const bool few = lanes_of(a) == 16;
    if (BWD) {
        if (few && a.E <= 64) return go(k_route_bwd<T, 16, 4>, 16);
        if (few) return go(k_route_bwd<T, 16, 16>, 16);
        if (a.E <= 1024) return go(k_route_bwd<T, 64, 16>, 64);
        return go(k_route_bwd<T, 64, 64>, 64);
    }
    if (few && a.E <= 64) return go(k_route<T, 16, 4>, 16);
    if (few) return go(k_route<T, 16, 16>, 16);
    if (a.E <= 1024) return go(k_route<T, 64, 16>, 64);
    return go(k_route<T, 64, 64>, 64);
}

template <bool BWD> hipError_t typed(int type, const RouteArgs &a, hipStream_t st)
{
    return type == SOM_F32   ? pick<float, BWD>(a, st)
           : type == SOM_F16 ? pick<_Float16, BWD>(a, st)
                             : pick<__bf16, BWD>(a, st);
}

}  // namespace

hipError_t launch_route(int logit_type, const RouteArgs &a, hipStream_t st)
{
    if (a.N == 0) {
        hipLaunchKernelGGL(k_zero, dim3((unsigned)((a.E + 255) / 256)), dim3(256), 0, st, a.counts, a.E);
        return hipGetLastError();
    }
    const hipError_t e = typed<false>(logit_type, a, st);
    if (e != hipSuccess || !a.counts || a.N <= rows_of_one(a)) return e;
    const int64_t n = a.N * a.k, blocks = (n + 8191) / 8192;
    hipLaunchKernelGGL(k_counts, dim3((unsigned)(blocks < 32 ? blocks : 32)), dim3(1024), 0, st, a.idx, n, a.E, a.counts);
    return hipGetLastError();
}

hipError_t launch_route_bwd(int logit_type, const RouteArgs &a, hipStream_t st)
{
    return typed<true>(logit_type, a, st);
}

}  // namespace som
