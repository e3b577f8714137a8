// som_norm.h -- layer norm of rows, forward and backward.
//
// y = (x - mean) / sqrt(var + eps) * weight + bias, over a row's D features. Both directions are
// bound by the bytes they move, so a row is read once: TPR threads hold it in registers, C vectors
// of 16 bytes each. Mean and variance come from one pass: sums of d and d^2, d = x - x[0], in fp64,
// which neither a large mean (subtracted first) nor large or small values (fp64's range) spoil, and
// which takes one exchange between the threads instead of two. Workgroups walk over rows with the
// weights in registers, and load the next row before they finish one.
#pragma once

#include "som_layer_device.h"

namespace som {
namespace layer {

// A row's threads: TPR of them, in workgroups of NT, with C vectors of V values each.
template <typename X_, typename Y_, int TPR_, int C_, int NT_> struct NormShape {
    typedef X_ X;
    typedef Y_ Y;
    static constexpr int TPR = TPR_, C = C_, NT = NT_, V = 16 / sizeof(X_), ROWS = NT_ / TPR_;
};

// The sums of two values over a row's threads.
template <int TPR, typename T> __device__ inline void row_sums(T &a, T &b, T *lds)
{
    constexpr int L = TPR < 64 ? TPR : 64, W = TPR / L;
    a = lane_sum<L>(a);
    b = lane_sum<L>(b);
    if (W > 1) {
        const int wave = threadIdx.x / 64, first = wave / W * W;
        __syncthreads();  // the last row's sums have been read
        if (threadIdx.x % 64 == 0) lds[2 * wave] = a, lds[2 * wave + 1] = b;
        __syncthreads();
        a = b = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) a += lds[2 * (first + i)], b += lds[2 * (first + i) + 1];
    }
}

// Mean and 1 / std from the sums of d and d^2, d the distance from `from`.
__device__ inline void moments(double s, double q, double from, int D, double eps, double &mean, double &inv)
{
    const double m = s / D, var = q / D - m * m;
    mean = from + m;
    inv = 1.0 / sqrt((var < 0 ? 0.0 : var) + eps);
}

// (x - mean) / std in fp32: the mean in two parts, so that a mean much larger than the spread costs
// nothing. Rows that come near the end of fp32's range are scaled down first, which is exact and, in the
// fused product, free. The others are at most sqrt(D) < 2^10 times the spread, and so 2^126, from their mean.
struct Centre {
    float scale, hi, lo, inv, inv_std;
    __device__ Centre(double mean, double i) : inv_std((float)i)
    {
        const bool far = !(fabs(mean) < 0x1p125 && i > 0x1p-116);
        const double s = far ? 0x1p-32 : 1.0;
        scale = (float)s;
        hi = (float)(mean * s);
        lo = (float)(mean * s - (double)hi);
        inv = (float)(i * (far ? 0x1p32 : 1.0));
    }
    __device__ float of(float x) const { return (fmaf(x, scale, -hi) - lo) * inv; }
};

template <typename Y, int V> __device__ inline void load_weight(const void *p, bool f32, int at, int n, float *v, float none)
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = none;
    } else if (f32) {
        load<V>(static_cast<const float *>(p) + at, n, v);
    } else {
        load<V>(static_cast<const Y *>(p) + at, n, v);
    }
}

// Values of a row as they lie in memory, C vectors of this thread.
template <typename T, class S> struct Row {
    typename VecOf<T, S::V>::type v[S::C];

    template <bool WHOLE> __device__ void get(const T *p, int D)
    {
#pragma unroll
        for (int c = 0; c < S::C; ++c) {
            const int at = (c * S::TPR + (int)threadIdx.x % S::TPR) * S::V;
            if (at + S::V <= D) {
                v[c] = *reinterpret_cast<const typename VecOf<T, S::V>::any *>(p + at);
            } else {
#pragma unroll
                for (int i = 0; i < S::V; ++i) v[c][i] = !WHOLE && at + i < D ? p[at + i] : (T)0.0f;
            }
        }
    }
};

// WHOLE: D is a multiple of V.
template <class S, bool WHOLE> __global__ __launch_bounds__(S::NT) void k_norm_rows(const NormArgs a)
{
    typedef typename S::X X;
    typedef typename S::Y Y;
    constexpr int V = S::V, C = S::C;
    __shared__ double lds[2 * S::NT / 64];
    const int t = (int)threadIdx.x % S::TPR, D = a.D;
    float w[C][V], b[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * S::TPR + t) * V;
        load_weight<Y, V>(a.weight, a.weights_f32, at, D - at, w[c], 1.0f);
        load_weight<Y, V>(a.bias, a.weights_f32, at, D - at, b[c], 0.0f);
    }
    const int64_t step = (int64_t)gridDim.x * S::ROWS;
    const X *x = static_cast<const X *>(a.x);
    Row<X, S> now, next;
    int64_t n = (int64_t)blockIdx.x * S::ROWS, mine = n + threadIdx.x / S::TPR;
    X from = 0, from_next = 0;
    if (mine < a.N) {
        now.template get<WHOLE>(x + mine * a.ldx, D);
        from = x[mine * a.ldx];
    }
    for (; n < a.N; n += step, mine += step) {
        const int64_t row = mine;
        if (row + step < a.N) {
            next.template get<WHOLE>(x + (row + step) * a.ldx, D);
            from_next = x[(row + step) * a.ldx];
        }
        double s = 0, q = 0;
        const double f = (double)(float)from;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * S::TPR + t) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const double d = (double)(float)now.v[c][i] - f;
                if (WHOLE ? at < D : at + i < D) {
                    s += d;
                    q = fma(d, d, q);
                }
            }
        }
        row_sums<S::TPR>(s, q, lds);
        double mean, inv;
        moments(s, q, f, D, a.eps, mean, inv);
        if (row < a.N) {
            const Centre centre(mean, inv);
            if (a.stats && t == 0) a.stats[2 * row] = mean, a.stats[2 * row + 1] = inv;
            Y *y = static_cast<Y *>(a.y) + row * a.ldy;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = (c * S::TPR + t) * V;
                float v[V];
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = fmaf(centre.of((float)now.v[c][i]), w[c][i], b[c][i]);
                if (at < D) store<V>(y + at, WHOLE ? V : D - at, v);
            }
        }
        now = next;
        from = from_next;
    }
}

// Rows longer than a workgroup's registers: read twice, the second time from L2.
template <typename X, typename Y> __global__ __launch_bounds__(1024) void k_norm_long(const NormArgs a)
{
    constexpr int V = 16 / sizeof(X);
    __shared__ double lds[32];
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const X *x = static_cast<const X *>(a.x) + row * a.ldx;
        const double f = (double)(float)x[0];
        double s = 0, q = 0;
        for (int at = (int)threadIdx.x * V; at < a.D; at += 1024 * V) {
            float v[V];
            load<V>(x + at, a.D - at, v);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (at + i >= a.D) continue;
                const double d = (double)v[i] - f;
                s += d;
                q = fma(d, d, q);
            }
        }
        row_sums<1024>(s, q, lds);
        double mean, inv;
        moments(s, q, f, a.D, a.eps, mean, inv);
        const Centre centre(mean, inv);
        if (a.stats && threadIdx.x == 0) a.stats[2 * row] = mean, a.stats[2 * row + 1] = inv;
        Y *y = static_cast<Y *>(a.y) + row * a.ldy;
        for (int at = (int)threadIdx.x * V; at < a.D; at += 1024 * V) {
            float v[V], w[V], b[V];
            load<V>(x + at, a.D - at, v);
            load_weight<Y, V>(a.weight, a.weights_f32, at, a.D - at, w, 1.0f);
            load_weight<Y, V>(a.bias, a.weights_f32, at, a.D - at, b, 0.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = fmaf(centre.of(v[i]), w[i], b[i]);
            store<V>(y + at, a.D - at, v);
        }
    }
}

// The gradient. With h = (x - mean) / std and t = dy * weight:
//   dx = add + (t - mean(t) - h mean(t h)) / std,   dweight = sum over rows of dy h,   dbias = of dy.
// A workgroup holds its rows' sums of dweight and dbias in registers; they are joined over its waves in LDS
// and written as one part, and k_norm_sums adds the parts in order. Its rows are as far apart as there are
// workgroups, so that those in flight are neighbours (6000 x 4096 fp32: 44.5 us, 50.4 with its rows side by side).
// Two workgroups a CU, whose loads hide each other's exchanges, where a thread has two vectors at most; but one
// for rows of 512 threads that end inside a vector, whose code takes more registers (without add, on the same
// buffers in every pass: 5000 x 8190 bf16 101 us, with two 114; 8192 x 4095, 256 threads a row, 78 and with two
// 63, though 16-bit rows of that shape spill 70 registers). Such rows are further from their bytes than whole
// ones, every element being tested and the last ones loaded one by one: on buffers by turns 8192 x 4095 takes 77 us
// (with add 105), 8192 x 4096 51.5 (61.5).
template <class S, bool WHOLE> __global__ __launch_bounds__(S::NT, S::C <= 2 && (WHOLE || S::TPR < 512) ? 4 : 2) void k_norm_grad(const NormArgs a)
{
    typedef typename S::X X;
    typedef typename S::Y Y;
    constexpr int V = S::V, C = S::C;
    __shared__ float lds[2 * S::NT / 64];
    __shared__ float joined[S::ROWS > 1 ? S::NT * V : 1];
    const int t = (int)threadIdx.x % S::TPR, sub = (int)threadIdx.x / S::TPR, D = a.D;
    float w[C][V], dw[C][V], db[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * S::TPR + t) * V;
        load_weight<Y, V>(a.weight, a.weights_f32, at, D - at, w[c], 1.0f);
#pragma unroll
        for (int i = 0; i < V; ++i) dw[c][i] = db[c][i] = 0.0f;
    }
    const int64_t first = (int64_t)blockIdx.x * S::ROWS, end = a.N, step = (int64_t)gridDim.x * S::ROWS;
    const X *x = static_cast<const X *>(a.x);
    const Y *dy = static_cast<const Y *>(a.y);
    Row<X, S> xn, xl;
    Row<Y, S> gn, gl;
    double mean_n = 0, inv_n = 0, mean_l = 0, inv_l = 0;
    auto fetch = [&](int64_t row, Row<X, S> &xr, Row<Y, S> &gr, double &m, double &i) {
        if (row >= end) return;
        xr.template get<WHOLE>(x + row * a.ldx, D);
        gr.template get<WHOLE>(dy + row * a.ldy, D);
        m = a.stats[2 * row];
        i = a.stats[2 * row + 1];
    };
    fetch(first + sub, xn, gn, mean_n, inv_n);
    for (int64_t n = first; n < end; n += step) {
        const int64_t row = n + sub;
        fetch(row + step, xl, gl, mean_l, inv_l);
        const Centre centre(mean_n, inv_n);
        const bool in = row < end;
        float s = 0, q = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * S::TPR + t) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (!in || (WHOLE ? at >= D : at + i >= D)) continue;
                const float g = (float)gn.v[c][i], h = centre.of((float)xn.v[c][i]), u = g * w[c][i];
                s += u;
                q = fmaf(u, h, q);
                dw[c][i] = fmaf(g, h, dw[c][i]);
                db[c][i] += g;
            }
        }
        if (a.dx) {
            row_sums<S::TPR>(s, q, lds);
            s /= (float)D;
            q /= (float)D;
            if (in) {
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int at = (c * S::TPR + t) * V;
                    if (at >= D) continue;
                    float v[V], more[V];
                    if (a.add) load<V>(static_cast<const X *>(a.add) + row * a.lda + at, WHOLE ? V : D - at, more);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float h = centre.of((float)xn.v[c][i]), u = (float)gn.v[c][i] * w[c][i];
                        v[i] = (u - s - h * q) * centre.inv_std;
                        if (a.add) v[i] += more[i];
                    }
                    store<V>(static_cast<X *>(a.dx) + row * a.lddx + at, WHOLE ? V : D - at, v);
                }
            }
        }
        xn = xl;
        gn = gl;
        mean_n = mean_l;
        inv_n = inv_l;
    }
    if (!a.parts && !a.dweight && !a.dbias) return;
    float *out = a.parts + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * S::TPR + t) * V;
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = j ? db[c][i] : dw[c][i];
            if (S::ROWS > 1) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < V; ++i) joined[i * S::NT + threadIdx.x] = v[i];
                __syncthreads();
                if (sub == 0) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        v[i] = 0;
                        for (int r = 0; r < S::ROWS; ++r) v[i] += joined[i * S::NT + r * S::TPR + t];
                    }
                }
            }
            if (sub != 0 || at >= D) continue;
            if (a.parts) {
                store<V>(out + (int64_t)j * D + at, WHOLE ? V : D - at, v);
            } else if (void *to = j ? a.dbias : a.dweight) {  // of the only part
                if (a.weights_f32) store<V>(static_cast<float *>(to) + at, WHOLE ? V : D - at, v);
                else store<V>(static_cast<Y *>(to) + at, WHOLE ? V : D - at, v);
            }
        }
    }
}

// Rows longer than that (fp32 above 8,192 features, 16-bit above 16,384) are read twice: 2000 x 16384 fp32 takes 141 us,
// with add 166, 2000 x 24576 bf16 123 and 138, where the bytes of one pass take 80, 106, 60 and 80 at a copy's rate.
// First each row's mean(t) and mean(t h) ...
template <typename X, typename Y> __global__ __launch_bounds__(1024) void k_norm_means(const NormArgs a)
{
    constexpr int V = 16 / sizeof(X);
    __shared__ float lds[32];
    for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
        const X *x = static_cast<const X *>(a.x) + row * a.ldx;
        const Y *dy = static_cast<const Y *>(a.y) + row * a.ldy;
        const Centre centre(a.stats[2 * row], a.stats[2 * row + 1]);
        float s = 0, q = 0;
        for (int at = (int)threadIdx.x * V; at < a.D; at += 1024 * V) {
            float v[V], g[V], w[V];
            load<V>(x + at, a.D - at, v);
            load<V>(dy + at, a.D - at, g);
            load_weight<Y, V>(a.weight, a.weights_f32, at, a.D - at, w, 1.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (at + i >= a.D) continue;
                s += g[i] * w[i];
                q = fmaf(g[i] * w[i], centre.of(v[i]), q);
            }
        }
        row_sums<1024>(s, q, lds);
        if (threadIdx.x == 0) a.means[2 * row] = s / (float)a.D, a.means[2 * row + 1] = q / (float)a.D;
    }
}

// ... then strips of 256 threads' columns over a part's rows: dx, and the part's sums.
template <typename X, typename Y> __global__ __launch_bounds__(256) void k_norm_strips(const NormArgs a)
{
    constexpr int V = 16 / sizeof(X);
    const int at = ((int)blockIdx.y * 256 + (int)threadIdx.x) * V, n = a.D - at;
    if (n <= 0) return;
    float w[V], dw[V], db[V];
    load_weight<Y, V>(a.weight, a.weights_f32, at, n, w, 1.0f);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.0f;
    const int64_t first = (int64_t)blockIdx.x * a.part_rows, end = min(a.N, first + a.part_rows);
    for (int64_t row = first; row < end; ++row) {
        const Centre centre(a.stats[2 * row], a.stats[2 * row + 1]);
        float v[V], g[V], more[V];
        load<V>(static_cast<const X *>(a.x) + row * a.ldx + at, n, v);
        load<V>(static_cast<const Y *>(a.y) + row * a.ldy + at, n, g);
        if (a.add) load<V>(static_cast<const X *>(a.add) + row * a.lda + at, n, more);
        const float s = a.dx ? a.means[2 * row] : 0.0f, q = a.dx ? a.means[2 * row + 1] : 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float h = centre.of(v[i]);
            dw[i] = fmaf(g[i], h, dw[i]);
            db[i] += g[i];
            v[i] = (g[i] * w[i] - s - h * q) * centre.inv_std;
            if (a.add) v[i] += more[i];
        }
        if (a.dx) store<V>(static_cast<X *>(a.dx) + row * a.lddx + at, n, v);
    }
    if (!a.parts) return;
    float *out = a.parts + (int64_t)blockIdx.x * 2 * a.D + at;
    store<V>(out, n, dw);
    store<V>(out + a.D, n, db);
}

}  // namespace layer
}  // namespace som
