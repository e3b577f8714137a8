// som_layer_device.h -- device helpers of layer norm, AdamW and the 4-bit operators: vectors of any
// alignment, and sums over lanes.
#pragma once

#include "som_layer.h"

namespace som {
namespace layer {

template <typename T, int V> struct VecOf {
    typedef T type __attribute__((ext_vector_type(V)));
    typedef type any __attribute__((aligned(sizeof(T))));
};

// v[0 ... n - 1] from p, zeros after them; whole vectors at any alignment of an element.
template <int V, typename T> __device__ inline void load(const T *p, int n, float *v)
{
    if (n >= V) {
        const typename VecOf<T, V>::type t = *reinterpret_cast<const typename VecOf<T, V>::any *>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
    }
}

template <int V, typename T> __device__ inline void store(T *p, int n, const float *v)
{
    if (n >= V) {
        typename VecOf<T, V>::type t;
#pragma unroll
        for (int i = 0; i < V; ++i) t[i] = (T)v[i];
        *reinterpret_cast<typename VecOf<T, V>::any *>(p) = t;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}

// The value of another lane of 16, by a pattern of data-parallel primitives.
template <int CTRL> __device__ inline uint32_t swap32(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL> __device__ inline float swapped(float v) { return __uint_as_float(swap32<CTRL>(__float_as_uint(v))); }
template <int CTRL> __device__ inline double swapped(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)swap32<CTRL>((uint32_t)(u >> 32)) << 32 | swap32<CTRL>((uint32_t)u));
}

// The sum over LANES neighbouring lanes (8 to 64), the same bits in every one: pairs, quads, halves
// and rows of 16 by data-parallel primitives, the last two steps by exchange.
template <int LANES, typename T> __device__ inline T lane_sum(T v)
{
    v += swapped<0xB1>(v);
    v += swapped<0x4E>(v);
    v += swapped<0x141>(v);
    if (LANES >= 16) v += swapped<0x140>(v);
    if (LANES >= 32) v += __shfl_xor(v, 16);
    if (LANES >= 64) v += __shfl_xor(v, 32);
    return v;
}

// ---------------------------------------------------------------- 4-bit values

// 2^(s - 127), a subnormal for 0 and NaN for 255; no branch, which a choice would become.
__device__ inline float scale_value(uint32_t s) { return __uint_as_float(max(s << 23, 0x00400000u) | (s + 1) >> 8 << 22); }

// Eight codes times a scale as 16-bit values. Of the scale the conversion reads the exponent's place alone
// (0 stands for 2^-127, 255 makes NaN).
template <typename T> __device__ inline T __attribute__((ext_vector_type(8))) widen8_by(uint32_t codes, float scale)
{
    typedef T two __attribute__((ext_vector_type(2)));
    typedef T eight __attribute__((ext_vector_type(8)));
    two a, b, c, d;
    if constexpr (__is_same(T, __bf16)) {
        a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    } else {
        a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3);
    }
    return eight{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The same, exactly: bf16 under the scale byte s, fp16 without it, since fp16 does not hold all scales.
template <typename T> __device__ inline T __attribute__((ext_vector_type(8))) widen8(uint32_t codes, uint32_t s)
{
    return widen8_by<T>(codes, __is_same(T, __bf16) ? __uint_as_float(s << 23) : 1.0f);
}

}  // namespace layer
}  // namespace som
