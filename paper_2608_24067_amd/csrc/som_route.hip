// som_route.hip -- each row's k best units by its logits, their weights, and the gradient.
//
// A row is held in the registers of 16 or 64 lanes (LPR), VPL logits a lane, four neighbours at
// a time. The choice is k rounds of a maximum over (closed units: minus infinity)
// logit + bias, the lowest index among equals; each lane offers its best unit and knows its
// second, and looks at its units again only when both are taken (one pass of VPL units instead
// of one a round). Softmax statistics are fp32, shifted by the row's maximum.

#include "som_mm.h"

namespace som {
namespace {

using mm::block_number;
using mm::exp_f32;
using mm::exp_short;
using mm::load4;
using mm::store4;

template <int CTRL> __device__ inline uint32_t lane_swap(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);  // every lane has a source
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

// The value of lane i of the row.
template <int LPR> __device__ inline float of_lane(float v, int i)
{
    return LPR == 64 ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), i)) : __shfl(v, i, LPR);
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

constexpr float kMost = 3.402823466e38f;

// What a unit is ranked by: logit + bias (fp32, one rounding; + 0 makes -0, which a logit and a bias
// of -0 add up to, the 0 that it equals), -inf for a closed one.
__device__ inline float rank_key(float logit, float bias)
{
    const float s = logit + bias + 0.0f;
    return logit > -__builtin_inff() && s > -__builtin_inff() ? s : -__builtin_inff();  // false for NaN
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

    float l[VPL];    // logits, at most the largest finite value; -inf for a closed unit
    float key[VPL];  // what they are ranked by

    template <bool BIAS, typename T> __device__ void load(const T *p, const float *bias, int E, int sub)
    {
#pragma unroll
        for (int i = 0; i < VPL; i += 4) {
            const int e = unit(i, sub), n = max(0, min(4, E - e));
            float v[4], b[4] = {0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = -__builtin_inff();
            if (n == 4) {
                load4(p + e, 4, v);
                if (BIAS) load4(bias + e, 4, b);
            } else if (n > 0) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < n) {
                        v[q] = (float)p[e + q];
                        if (BIAS) b[q] = bias[e + q];
                    }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                key[i + q] = BIAS ? rank_key(v[q], b[q]) : fmaxf(v[q] + 0.0f, -__builtin_inff());  // NaN: -inf; -0: 0
                l[i + q] = fminf(!BIAS ? key[i + q] : key[i + q] > -__builtin_inff() ? v[q] : key[i + q], kMost);
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
            l[i] = exp_short(l[i] - shift);
            z += l[i];
        }
        return sum_f32<LPR>(z);
    }

    // The lane's two best units, -inf where there is none; AGAIN: of those that rank after (after, e).
    float v1, v2;
    int i1, i2;
    template <bool AGAIN> __device__ void two_best(float after, int e, int sub)
    {
        v1 = v2 = -__builtin_inff();
        i1 = i2 = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const float x =
                !AGAIN || key[i] < after || (key[i] == after && unit(i, sub) > e) ? key[i] : -__builtin_inff();
            const bool first = x > v1, second = x > v2;
            i2 = first ? i1 : second ? i : i2;
            v2 = first ? v1 : second ? x : v2;
            i1 = first ? i : i1;
            v1 = first ? x : v1;
        }
    }
};

constexpr int kThreads = 256;

// An order-preserving image of a float that is no NaN (and no -0); 0 lies below all, kClosed is -inf's.
__device__ inline uint32_t image(float v)
{
    const uint32_t u = __float_as_uint(v);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
constexpr uint32_t kClosed = 0x007fffffu;

// The lowest unit of the row's lanes that are `in` (one at least): nearly always there is one.
template <int LPR> __device__ inline int lowest(bool in, int own)
{
    if (LPR == 64) {
        const unsigned long long lanes = __ballot(in);
        if ((lanes & (lanes - 1)) == 0) return __builtin_amdgcn_readlane(own, __builtin_ctzll(lanes));
    }
    return (int)min_u32<LPR>(in ? (uint32_t)own : ~0u);
}

template <typename T, int LPR, int VPL, bool BIAS>
__global__ __launch_bounds__(kThreads) void k_route(const RouteArgs a)
{
    constexpr int kRows = kThreads / LPR;
    __shared__ uint32_t best[kRows][SOM_ROUTE_MAX_GROUPS];
    __shared__ unsigned long long kept[kRows];
    const int sub = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    const int64_t row = block_number() * kRows + slot;
    const bool in = row < a.N;
    const T *p = static_cast<const T *>(a.logits) + (in ? row : 0) * a.ldl;

    Row<LPR, VPL> r;
    r.template load<BIAS>(p, a.bias, a.E, sub);
    float m = 0, z = 1;
    const bool softmax = a.score == SOM_SCORE_SOFTMAX;
    if (softmax && !a.renorm) {
        m = r.top();
        z = r.total(m);
    }
    if (a.groups > 1) {
        // Groups by their best unit; one is kept if fewer than group_top are better (the lower
        // one first among equals).
        const int width = a.E / a.groups;
        const float inv = 1.0f / (float)width;  // (e + 1/2) inv is never near a whole number
        const bool fours = width % 4 == 0;      // a lane's four neighbours are of one group
        for (int g = sub; g < a.groups; g += LPR) best[slot][g] = 0;
        if (sub == 0) kept[slot] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VPL; i += 4) {
            const int e = Row<LPR, VPL>::unit(i, sub);
            if (e >= a.E) continue;
            if (fours) {
                const float v = fmaxf(fmaxf(r.key[i], r.key[i + 1]), fmaxf(r.key[i + 2], r.key[i + 3]));
                if (v > -__builtin_inff()) atomicMax(&best[slot][(int)((e + 0.5f) * inv)], image(v));
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (r.key[i + q] > -__builtin_inff())
                        atomicMax(&best[slot][(int)((e + q + 0.5f) * inv)], image(r.key[i + q]));
            }
        }
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
        for (int i = 0; i < VPL; i += 4) {
            const int e = Row<LPR, VPL>::unit(i, sub);
            if (e >= a.E) continue;
            const bool in4 = keep >> (int)((e + 0.5f) * inv) & 1;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bool keep1 = fours ? in4 : keep >> (int)((e + q + 0.5f) * inv) & 1;
                r.key[i + q] = keep1 ? r.key[i + q] : -__builtin_inff();
            }
        }
    }

    // Place j is held by lane j of the row.
    int unit = -1;
    r.template two_best<false>(0.0f, 0, sub);
    int left = 2;  // units the lane offers before it must look again
    float last = 0.0f;
    int last_e = 0;
    for (int j = 0; j < a.k; ++j) {
        const int own = Row<LPR, VPL>::unit(r.i1, sub);
        const uint32_t offer = image(r.v1), w = max_u32<LPR>(offer);
        const bool some = w > kClosed;
        const int e = lowest<LPR>(offer == w, own);
        if (sub == j) unit = some ? e : -1;
        if (some && own == e && offer == w) {
            last = r.v1;
            last_e = e;
            r.v1 = r.v2;
            r.i1 = r.i2;
            r.v2 = -__builtin_inff();
            --left;
        }
        if (j + 1 < a.k && __any(left == 0)) {
            if (left == 0) {
                r.template two_best<true>(last, last_e, sub);
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
    if (a.counts && block_number() == 0) {
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
template <typename T, int LPR, int VPL, bool BIAS>
__global__ __launch_bounds__(kThreads) void k_route_bwd(const RouteArgs a)
{
    constexpr int kRows = kThreads / LPR;
    const int sub = threadIdx.x % LPR, slot = threadIdx.x / LPR;
    const int64_t row = block_number() * kRows + slot;
    const bool in = row < a.N;
    const int64_t at = in ? row : 0;
    const T *p = static_cast<const T *>(a.logits) + at * a.ldl;
    T *d = static_cast<T *>(a.dlogits) + at * a.lddl;
    const bool softmax = a.score == SOM_SCORE_SOFTMAX, shares = softmax && !a.renorm;

    int unit = sub < a.k ? a.idx[at * a.k + sub] : -1;
    float l = -__builtin_inff();
    if (unit >= 0 && unit < a.E) {
        l = fminf((float)p[unit], kMost);
        if (!(rank_key((float)p[unit], BIAS ? a.bias[unit] : 0.0f) > -__builtin_inff())) unit = -1, l = -__builtin_inff();
    } else {
        unit = -1;
    }
    const bool took = unit >= 0;
    const float dw = took ? load_weight(a.weight_type, a.weights, at * a.k + sub) : 0.0f;

    Row<LPR, VPL> r;
    float m = 0, z = 1;
    if (shares) {
        r.template load<BIAS>(p, a.bias, a.E, sub);
        m = r.top();
        z = r.total(m);
    }
    const float over = z > 0.0f ? 1.0f / z : 0.0f;
    float g, sum = 0;  // g: the taken unit's gradient
    if (a.renorm) {
        // the shares add up to 1: dw - sum dw w = sum over i of w_i (dw - dw_i), which loses nothing
        // where one share is nearly all
        const float w = share<LPR>(softmax, l);
        float left = 0;
        for (int i = 0; i < a.k; ++i) left = fmaf(of_lane<LPR>(w, i), dw - of_lane<LPR>(dw, i), left);
        g = w * left;
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
            const float gj = of_lane<LPR>(g, j);
            if (u < 0) continue;
            const int at = (u / (4 * LPR)) * 4 + u % 4;  // the same register in every lane
            const bool mine = u / 4 % LPR == sub;
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (i == at) r.l[i] = mine ? gj : r.l[i];
        } else {
            const int u = __shfl(unit, j, LPR);
            const float gj = of_lane<LPR>(g, j);
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

// Lanes that hold a row: 16 for up to 64 units (four rows a wave), else 64. (256 units and 8 taken:
// 16 lanes of 16 units look at them again in most rounds, 64 lanes of four hardly ever.)
int lanes_of(const RouteArgs &a) { return a.E <= 64 && a.k <= 16 ? 16 : 64; }
int rows_of_one(const RouteArgs &a) { return kThreads / lanes_of(a); }

template <typename T, bool BWD, bool BIAS> hipError_t pick(const RouteArgs &a, hipStream_t st)
{
    auto go = [&](auto kernel) {
        const int64_t rows = rows_of_one(a);
        hipLaunchKernelGGL(kernel, grid_of((a.N + rows - 1) / rows), dim3(kThreads), 0, st, a);
        return hipGetLastError();
    };
    if constexpr (BWD) {
        if (lanes_of(a) == 16) return go(k_route_bwd<T, 16, 4, BIAS>);
        if (a.E <= 256) return go(k_route_bwd<T, 64, 4, BIAS>);
        if (a.E <= 1024) return go(k_route_bwd<T, 64, 16, BIAS>);
        return go(k_route_bwd<T, 64, 64, BIAS>);
    } else {
        if (lanes_of(a) == 16) return go(k_route<T, 16, 4, BIAS>);
        if (a.E <= 256) return go(k_route<T, 64, 4, BIAS>);
        if (a.E <= 1024) return go(k_route<T, 64, 16, BIAS>);
        return go(k_route<T, 64, 64, BIAS>);
    }
}

template <bool BWD> hipError_t typed(int type, const RouteArgs &a, hipStream_t st)
{
    if (a.bias)
        return type == SOM_F32   ? pick<float, BWD, true>(a, st)
               : type == SOM_F16 ? pick<_Float16, BWD, true>(a, st)
                                 : pick<__bf16, BWD, true>(a, st);
    return type == SOM_F32   ? pick<float, BWD, false>(a, st)
           : type == SOM_F16 ? pick<_Float16, BWD, false>(a, st)
                             : pick<__bf16, BWD, false>(a, st);
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
    // as many workgroups as the choices fill, while those add at most 8,192 counts of a cache line's 16
    const int64_t n = a.N * a.k, most = a.E < 256 ? 8192 / a.E < 128 ? 8192 / a.E : 128 : 32;
    const int64_t blocks = (n + 8191) / 8192 < most ? (n + 8191) / 8192 : most;
    hipLaunchKernelGGL(k_counts, dim3((unsigned)blocks), dim3(1024), 0, st, a.idx, n, a.E, a.counts);
    return hipGetLastError();
}

hipError_t launch_route_bwd(int logit_type, const RouteArgs &a, hipStream_t st)
{
    return typed<true>(logit_type, a, st);
}

}  // namespace som
