// som_adamw.hip -- a step of AdamW over many tensors, with the states in 32 bits or in 8.
//
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2
//   p' = p (1 - lr wd) - lr / (1 - b1^t) * m' / (sqrt(v') / sqrt(1 - b2^t) + eps)
//
// One launch takes the chunks of up to 44 tensors; a thread's four or eight elements are loaded in
// vectors. Bound by the bytes it moves: 28 an element in fp32 (168 million elements: 865 us, 5.5 TB/s), 10
// of a 16-bit parameter with 8-bit states (336 us, 5.0 TB/s), whose arithmetic, some 60 instructions an
// element, takes nearly as long. A block's bytes are loaded before its codes: asked for after them, their wait came on top.
//
// 8-bit states. A block of 256 values shares a power of two 2^e, the least at which its largest
// value is at most 1.875, held as e + 127 in a byte (255: the block held an infinity or NaN, and all
// of it stands for NaN; 0: all values below 2^-100, held as zeros). m is held with a sign, 4 bits
// of exponent and 3 behind the point, down to 2^-17 of the block's largest value; v, which has no
// sign and the square of m's range, with 5 bits of exponent, down to 2^-33. Rounding is to either
// neighbour, the nearer one more often, so that a value's mean is kept: with b2 = 0.999 a state moves
// by a thousandth of itself a step, and rounding to nearest, in steps of a sixteenth, would leave it
// where it is. The 16 bits that decide come from a hash of the seed, the step, the tensor's number in
// the call and the element's in the tensor: the same inputs give the same bits. A v above zero is
// never rounded to zero (but with its whole block), or a later step would divide what is left of m by eps alone.

#include "som_layer_device.h"

namespace som {
namespace {

using namespace layer;

constexpr int kThreads = 256;

// The bits of h spread over all of them: shifts, and multiplications by the fractional parts of the
// square roots of 3 and 2.
__device__ inline uint32_t mix_product(uint32_t h)  // all but the last step
{
    h ^= h >> 16;
    h *= 0xBB67AE85u;
    h ^= h >> 15;
    return h * 0x6A09E667u;
}
__device__ inline uint32_t mix(uint32_t h)
{
    h = mix_product(h);
    return h ^ h >> 16;
}

__device__ inline int tensor_of(const AdamwTable &t, int chunk)
{
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

struct Rates : AdamwRates {
    // As the host formed them, or with the step or the rate that lie on the device.
    __device__ explicit Rates(const AdamwArgs &a) : AdamwRates(a.rates)
    {
        if (a.step_at || a.lr_at) {
            const double lr = a.lr_at ? (double)*a.lr_at : a.lr;
            set(lr, a.beta1, a.beta2, a.weight_decay, a.step_at ? (uint32_t)max(*a.step_at, 1) : step);
        }
    }
    // by1, by2: b1 and b2, or what stands for them (an 8-bit block's). The products of m and v are
    // rounded one by one, as documented; the parameter's part takes the hardware's root and reciprocal,
    // good to a unit in the last place, for a third of an 8-bit step's instructions. The hardware takes a
    // subnormal root's argument as zero: such a v is taken times 2^64, and its root's factor over 2^32.
    __device__ void apply(float &p, float g, float &m, float &v, float by1, float by2) const
    {
        g *= grad;
        m = m * by1 + g * c1;
        v = v * by2 + g * g * c2;
        const bool small = v < 0x1p-126f;
        const float den = fmaf(__builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v), small ? root * 0x1p-32f : root, eps);
        p = fmaf(-rate, m * __builtin_amdgcn_rcpf(den), p * keep);
    }
};

// n values of any of the three types.
template <int V> __device__ inline void load_any(const void *p, int type, int64_t at, int n, float *v)
{
    if (type == SOM_F32) load<V>(static_cast<const float *>(p) + at, n, v);
    else if (type == SOM_F16) load<V>(static_cast<const _Float16 *>(p) + at, n, v);
    else load<V>(static_cast<const __bf16 *>(p) + at, n, v);
}
template <int V> __device__ inline void store_any(void *p, int type, int64_t at, int n, const float *v)
{
    if (type == SOM_F32) store<V>(static_cast<float *>(p) + at, n, v);
    else if (type == SOM_F16) store<V>(static_cast<_Float16 *>(p) + at, n, v);
    else store<V>(static_cast<__bf16 *>(p) + at, n, v);
}

// What codes stand for under a block's byte s: a code's bits (its sign at the front) are those of an
// fp32 value whose exponent is 127 - s + 112 (m) or 96 (v) too small; codes below the first exponent
// are subnormal there. `word` holds the code in its byte B.
template <bool SIGNED, int B> __device__ inline float decode(uint32_t word, int s)
{
    const uint32_t bits = SIGNED ? (uint32_t)((int32_t)(word << (24 - 8 * B)) >> 4) & 0x87F00000u : (word >> (8 * B) & 255) << 20;
    return ldexpf(__uint_as_float(bits), s - (SIGNED ? 15 : 31));
}

// What a block's old values are multiplied by: nothing where it is held as zeros, NaN where it holds none.
__device__ inline float block_factor(uint32_t s, float b) { return s == 255 ? __builtin_nanf("") : s ? b : 0.0f; }

// The exponent e of a block's power from the bits of its largest magnitude, as its byte.
__device__ inline uint32_t block_scale(uint32_t bits)
{
    const uint32_t f = ((bits & 0x7FFFFFFF) + 0xFFFFF) >> 23;  // a NaN may carry past 255
    return f < 27 ? 0 : min(f, 255u);
}

// The code of x by 16 random bits, which are added above the four that are dropped. Codes of a block whose
// byte is 0 are cleared afterwards; a block of NaN gets codes of no meaning.
template <bool SIGNED> __device__ inline uint32_t encode(float x, int s, uint32_t random)
{
    const uint32_t c = (__float_as_uint(ldexpf(fabsf(x), (SIGNED ? 15 : 31) - s)) + (random << 4)) >> 20;
    if (SIGNED) return min(c, 127u) | (x < 0.0f ? 128u : 0u);
    return min(max(c, x > 0.0f ? 1u : 0u), 255u);  // and 0 for 0, whose bits the random ones do not carry
}

// The largest over the 32 lanes of a block's half wave.
__device__ inline uint32_t half_wave_max(uint32_t v)
{
    v = max(v, swap32<0xB1>(v));
    v = max(v, swap32<0x4E>(v));
    v = max(v, swap32<0x141>(v));
    v = max(v, swap32<0x140>(v));
    return max(v, (uint32_t)__shfl_xor((int)v, 16));
}

// n codes (up to V, 4 or 8) as the bytes of words.
template <int V> __device__ inline void load_codes(const uint8_t *p, int n, uint32_t *w)
{
    typedef typename VecOf<uint32_t, V / 4>::type words;
    typedef words any __attribute__((aligned(1)));
    if (n >= V) {
        const words t = *reinterpret_cast<const any *>(p);
#pragma unroll
        for (int i = 0; i < V / 4; ++i) w[i] = t[i];
    } else {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) w[i] = 0;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) w[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
    }
}
template <int V> __device__ inline void store_codes(uint8_t *p, int n, const uint32_t *w)
{
    typedef typename VecOf<uint32_t, V / 4>::type words;
    typedef words any __attribute__((aligned(1)));
    if (n >= V) {
        words t;
#pragma unroll
        for (int i = 0; i < V / 4; ++i) t[i] = w[i];
        *reinterpret_cast<any *>(p) = t;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
    }
}

template <bool SIGNED> __device__ inline void decode4(uint32_t word, int s, float *v)
{
    v[0] = decode<SIGNED, 0>(word, s), v[1] = decode<SIGNED, 1>(word, s);
    v[2] = decode<SIGNED, 2>(word, s), v[3] = decode<SIGNED, 3>(word, s);
}

template <bool BITS8> __global__ __launch_bounds__(kThreads) void k_adamw(const AdamwTable t, const AdamwArgs a)
{
    if (a.norm && !(fabsf(*a.norm) < __builtin_inff())) return;
    const int chunk = blockIdx.x, i = tensor_of(t, chunk);
    const int64_t from = (int64_t)(chunk - t.first[i]) * t.chunk, to = min(t.size[i], from + t.chunk);
    const Rates r(a);
    const int type = t.type[i], grad_type = t.grad_type[i];
    float *master = t.master[i];
    const void *read = master ? static_cast<const void *>(master) : t.param[i];
    const int read_type = master ? SOM_F32 : type;
    if (!BITS8) {
        constexpr int V = 4;
        float *ms = static_cast<float *>(t.m[i]), *vs = static_cast<float *>(t.v[i]);
#pragma unroll 2
        for (int64_t at = from + V * (int64_t)threadIdx.x; at < to; at += V * kThreads) {
            const int n = (int)min((int64_t)V, to - at);
            float p[V], g[V], m[V], v[V];
            load_any<V>(read, read_type, at, n, p);
            load_any<V>(t.grad[i], grad_type, at, n, g);
            load<V>(ms + at, n, m);
            load<V>(vs + at, n, v);
#pragma unroll
            for (int q = 0; q < V; ++q) r.apply(p[q], g[q], m[q], v[q], r.b1, r.b2);
            store<V>(ms + at, n, m);
            store<V>(vs + at, n, v);
            if (master) store<V>(master + at, n, p);
            store_any<V>(t.param[i], type, at, n, p);
        }
    } else {
        constexpr int V = 8;
        uint8_t *mc = static_cast<uint8_t *>(t.m[i]), *vc = static_cast<uint8_t *>(t.v[i]);
        const uint32_t key = mix(a.seed + r.step * 0x9E3779B1u + (uint32_t)(t.number + i) * 0x1F83D9ABu);
        uint8_t *m_scales = t.m_scales[i], *v_scales = t.v_scales[i];
        // Whole blocks of 32 threads take part: past the end they hold zeros (NaN in a block of NaN).
        for (int64_t at = from + V * (int64_t)threadIdx.x; at < from + t.chunk; at += V * kThreads) {
            const int64_t block = at / kStateBlock;
            if (block * kStateBlock >= to) break;
            const int n = (int)max((int64_t)0, min((int64_t)V, to - at));
            float p[V], g[V], m[V], v[V];
            uint32_t cm[V / 4], cv[V / 4];
            const uint32_t old_m = m_scales[block], old_v = v_scales[block];
            load_any<V>(read, read_type, at, n, p);
            load_any<V>(t.grad[i], grad_type, at, n, g);
            load_codes<V>(mc + at, n, cm);
            load_codes<V>(vc + at, n, cv);
            const float by1 = block_factor(old_m, r.b1), by2 = block_factor(old_v, r.b2);
            uint32_t top_m = 0, top_v = 0;
#pragma unroll
            for (int h = 0; h < V / 4; ++h) decode4<true>(cm[h], (int)old_m, m + 4 * h), decode4<false>(cv[h], (int)old_v, v + 4 * h);
#pragma unroll
            for (int q = 0; q < V; ++q) {
                r.apply(p[q], g[q], m[q], v[q], by1, by2);
            }
#pragma unroll
            for (int q = 0; q < V; ++q) {
                top_m = max(top_m, __float_as_uint(m[q]) & 0x7FFFFFFF);
                top_v = max(top_v, __float_as_uint(v[q]));  // not negative, but for a NaN
            }
            const uint32_t new_m = block_scale(half_wave_max(top_m)), new_v = block_scale(half_wave_max(top_v));
            const uint32_t first = (uint32_t)at * 0x9E3779B1u + (uint32_t)((uint64_t)at >> 32) * 0xA54FF53Bu + key;
#pragma unroll
            for (int h = 0; h < V / 4; ++h) cm[h] = cv[h] = 0;
#pragma unroll
            for (int q = 0; q < V; ++q) {  // a thread's eight numbers share their upper half
                const uint32_t h = mix_product(first + (uint32_t)q * 0x9E3779B1u);
                cm[q / 4] |= encode<true>(m[q], (int)new_m, (h & 0xFFFF) ^ h >> 16) << (8 * (q % 4));
                cv[q / 4] |= encode<false>(v[q], (int)new_v, h >> 16) << (8 * (q % 4));
            }
#pragma unroll
            for (int h = 0; h < V / 4; ++h) cm[h] = new_m ? cm[h] : 0, cv[h] = new_v ? cv[h] : 0;
            store_codes<V>(mc + at, n, cm);
            store_codes<V>(vc + at, n, cv);
            if (threadIdx.x % 32 == 0) m_scales[block] = (uint8_t)new_m, v_scales[block] = (uint8_t)new_v;
            if (master) store<V>(master + at, n, p);
            store_any<V>(t.param[i], type, at, n, p);
        }
    }
}

__global__ __launch_bounds__(kThreads) void k_adamw_values(const AdamwTable t)
{
    constexpr int V = 4;
    const int chunk = blockIdx.x, i = tensor_of(t, chunk);
    const int64_t from = (int64_t)(chunk - t.first[i]) * t.chunk, to = min(t.size[i], from + t.chunk);
    const uint8_t *mc = static_cast<const uint8_t *>(t.m[i]), *vc = static_cast<const uint8_t *>(t.v[i]);
    float *om = static_cast<float *>(t.param[i]), *ov = t.master[i];
#pragma unroll 2
    for (int64_t at = from + V * (int64_t)threadIdx.x; at < to; at += V * kThreads) {
        const int n = (int)min((int64_t)V, to - at);
        const uint32_t sm = t.m_scales[i][at / kStateBlock], sv = t.v_scales[i][at / kStateBlock];
        const float by_m = block_factor(sm, 1.0f), by_v = block_factor(sv, 1.0f);
        uint32_t cm, cv;
        load_codes<V>(mc + at, n, &cm);
        load_codes<V>(vc + at, n, &cv);
        float m[V], v[V];
        decode4<true>(cm, (int)sm, m);
        decode4<false>(cv, (int)sv, v);
#pragma unroll
        for (int q = 0; q < V; ++q) m[q] *= by_m, v[q] *= by_v;
        store<V>(om + at, n, m);
        store<V>(ov + at, n, v);
    }
}

}  // namespace

hipError_t launch_adamw(const AdamwTable &t, bool bits8, const AdamwArgs &a, hipStream_t st)
{
    if (t.first[t.count] == 0) return hipSuccess;
    const dim3 grid((unsigned)t.first[t.count]);
    if (bits8) hipLaunchKernelGGL(k_adamw<true>, grid, dim3(kThreads), 0, st, t, a);
    else hipLaunchKernelGGL(k_adamw<false>, grid, dim3(kThreads), 0, st, t, a);
    return hipGetLastError();
}

hipError_t launch_adamw_values(const AdamwTable &t, hipStream_t st)
{
    if (t.first[t.count] == 0) return hipSuccess;
    hipLaunchKernelGGL(k_adamw_values, dim3((unsigned)t.first[t.count]), dim3(kThreads), 0, st, t);
    return hipGetLastError();
}

}  // namespace som
