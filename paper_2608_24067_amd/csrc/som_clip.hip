// som_clip.hip -- the norm of many tensors together, and their scaling to a largest norm.
//
// Three passes: every workgroup sums the squares of one chunk of one tensor (fp64, so that no
// square of an fp32 value overflows or vanishes; the threads' sums joined in a fixed order), one
// workgroup adds the chunks' sums and forms the scale, and the chunks are scaled. Few chunks: the
// second pass is done by every workgroup of the third. Both large passes are bound by the bytes
// they move: 2.3 GB in three types are summed at 6.2 TB/s and read and written at 5.1 TB/s
// (375 + 919 us); the scale needs the norm, so the tensors are read twice.

#include "som_mm.h"

namespace som {
namespace {

constexpr int kThreads = 256;

__device__ inline double block_sum(double v, double *lds)
{
    for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
    const int waves = blockDim.x / 64;
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    double s = 0;
    for (int i = 0; i < waves; ++i) s += lds[i];
    return s;
}

// The tensor a chunk belongs to.
__device__ inline int tensor_of(const ClipTable &t, int chunk)
{
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// f(values, count) over a chunk, VEC values of a thread at a time; whole 16-byte vectors where
// the tensor starts on one.
template <typename T, typename F> __device__ inline void over(const T *p, int64_t from, int64_t to, F f)
{
    constexpr int V = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(V)));
    typedef vec any __attribute__((aligned(sizeof(T))));
#pragma unroll 4
    for (int64_t i = from + V * (int64_t)threadIdx.x; i < to; i += V * kThreads) {
        float v[V];
        if (i + V <= to) {
            const vec x = *reinterpret_cast<const any *>(p + i);
#pragma unroll
            for (int q = 0; q < V; ++q) v[q] = (float)x[q];
            f(i, V, v);
        } else {
#pragma unroll
            for (int q = 0; q < V; ++q) v[q] = i + q < to ? (float)p[i + q] : 0.0f;
            f(i, (int)(to - i), v);
        }
    }
}

template <typename T> __device__ inline double squares(const void *in, int64_t from, int64_t to)
{
    constexpr int V = 16 / sizeof(T);
    double s = 0;
    over(static_cast<const T *>(in), from, to, [&](int64_t, int, const float *v) {
#pragma unroll
        for (int q = 0; q < V; ++q) s = fma((double)v[q], (double)v[q], s);
    });
    return s;
}

__global__ __launch_bounds__(kThreads) void k_squares(const ClipTable t, double *__restrict__ partial)
{
    __shared__ double lds[kThreads / 64];
    const int chunk = blockIdx.x, i = tensor_of(t, chunk);
    const int64_t from = (int64_t)(chunk - t.first[i]) * t.chunk, to = min(t.size[i], from + t.chunk);
    double s;
    if (t.type[i] == SOM_F32) s = squares<float>(t.in[i], from, to);
    else if (t.type[i] == SOM_F16) s = squares<_Float16>(t.in[i], from, to);
    else s = squares<__bf16>(t.in[i], from, to);
    s = block_sum(s, lds);
    if (threadIdx.x == 0) partial[chunk] = s;
}

// The scale of a norm; an infinite or NaN norm, or one within the limit, scales nothing. Infinite is
// what the caller reads as such: the fp32 value of the fp64 norm. The scale is an fp32 value, unless
// that would be subnormal and lose bits (norms of 1e36 and more).
constexpr double kLeastNormal = 0x1p-126;

__device__ inline double scale_of(double r, float max_norm)
{
    if (!(r > (double)max_norm && (float)r < __builtin_inff())) return 1.0;
    const double c = (double)max_norm / r;
    return c < kLeastNormal ? c : (double)(float)c;
}

__global__ __launch_bounds__(1024) void k_norm(const double *__restrict__ partial, int64_t n, float max_norm,
                                               float *__restrict__ norm, double *__restrict__ scale)
{
    __shared__ double lds[16];
    double s = 0;
    for (int64_t i = threadIdx.x; i < n; i += blockDim.x) s += partial[i];
    s = block_sum(s, lds);
    if (threadIdx.x == 0) {
        const double r = sqrt(s);
        *norm = (float)r;
        *scale = scale_of(r, max_norm);
    }
}

// times: the value to write for one read.
template <typename T, typename F>
__device__ inline void scaled_by(const void *in, void *out, int64_t from, int64_t to, F times)
{
    constexpr int V = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(V)));
    typedef vec any __attribute__((aligned(sizeof(T))));
    T *o = static_cast<T *>(out);
    over(static_cast<const T *>(in), from, to, [&](int64_t i, int n, const float *v) {
        if (n == V) {
            vec x;
#pragma unroll
            for (int q = 0; q < V; ++q) x[q] = (T)times(v[q]);
            __builtin_nontemporal_store(x, reinterpret_cast<any *>(o + i));
        } else {
#pragma unroll
            for (int q = 0; q < V; ++q)
                if (q < n) o[i + q] = (T)times(v[q]);
        }
    });
}

template <typename T> __device__ inline void scaled(const void *in, void *out, int64_t from, int64_t to, double scale)
{
    const float c = (float)scale;
    if (scale < kLeastNormal) {
        scaled_by<T>(in, out, from, to, [&](float v) { return (float)((double)v * scale); });
    } else if (c != 1.0f || in != out) {
        scaled_by<T>(in, out, from, to, [&](float v) { return c == 1.0f ? v : v * c; });
    }
}

__global__ __launch_bounds__(kThreads) void k_scale(const ClipTable t, const double *__restrict__ scale,
                                                    const double *__restrict__ partial, int64_t n, float max_norm,
                                                    float *__restrict__ norm)
{
    __shared__ double lds[kThreads / 64];
    // From the last chunk to the first: the last ones summed are still in the 256 MB cache, which the
    // results pass by (372 million values in three types: 1,333 -> 1,315 us).
    const int chunk = (int)(gridDim.x - 1 - blockIdx.x), i = tensor_of(t, chunk);
    const int64_t from = (int64_t)(chunk - t.first[i]) * t.chunk, to = min(t.size[i], from + t.chunk);
    double c;
    if (scale) {
        c = *scale;
    } else {
        double s = 0;
        for (int64_t j = threadIdx.x; j < n; j += kThreads) s += partial[j];
        const double r = sqrt(block_sum(s, lds));
        c = scale_of(r, max_norm);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)r;
    }
    if (t.type[i] == SOM_F32) scaled<float>(t.in[i], t.out[i], from, to, c);
    else if (t.type[i] == SOM_F16) scaled<_Float16>(t.in[i], t.out[i], from, to, c);
    else scaled<__bf16>(t.in[i], t.out[i], from, to, c);
}

}  // namespace

hipError_t launch_squares(const ClipTable &t, double *partial, hipStream_t st)
{
    if (t.first[t.count] == 0) return hipSuccess;
    hipLaunchKernelGGL(k_squares, dim3((unsigned)t.first[t.count]), dim3(kThreads), 0, st, t, partial);
    return hipGetLastError();
}

hipError_t launch_norm(const double *partial, int64_t n, float max_norm, float *norm, double *scale, hipStream_t st)
{
    hipLaunchKernelGGL(k_norm, dim3(1), dim3(1024), 0, st, partial, n, max_norm, norm, scale);
    return hipGetLastError();
}

hipError_t launch_scale(const ClipTable &t, const double *scale, const double *partial, int64_t n, float max_norm,
                        float *norm, hipStream_t st)
{
    if (t.first[t.count] == 0) return hipSuccess;
    hipLaunchKernelGGL(k_scale, dim3((unsigned)t.first[t.count]), dim3(kThreads), 0, st, t, scale,
                       partial, n, max_norm, norm);
    return hipGetLastError();
}

}  // namespace som
