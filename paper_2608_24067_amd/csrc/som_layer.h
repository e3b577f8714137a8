// som_layer.h -- shared between the host layer of layer norm, AdamW and the 4-bit operators
// (include/som_dense.h) and their kernels.
#pragma once

#include <math.h>

#include "som_dense.h"

namespace som {

// ---------------------------------------------------------------- layer norm

struct NormArgs {
    const void *x;
    int64_t ldx;
    const void *weight, *bias;  // null: ones, zeros
    bool weights_f32;           // else of y's type
    double eps;
    void *y;                    // the gradient: dy
    int64_t ldy;
    double *stats;              // [N][2] mean, 1 / std; or null
    int64_t N;
    int32_t D;
    // the gradient
    const void *add;            // or null
    int64_t lda;
    void *dx;                   // or null
    int64_t lddx;
    float *parts;               // [n_parts][2][D]: dweight, dbias; or null
    void *dweight, *dbias;      // written by the only part itself; or null
    int64_t n_parts, part_rows; // of rows too long for registers: parts of part_rows rows each
    float *means;               // [N][2], of rows too long for registers
};

// Workgroups of the gradient, one part each: from 3,584 rows on as many as the CUs hold at once, two a CU or,
// where rows have more than 1,024 vectors, one (3000 x 16384 bf16: 78 us, with two 95); fewer for fewer
// rows (their parts cost as much as eight rows each), and so many that a part's fp32 sums run over 256
// rows at most before they are joined.
inline int64_t norm_parts(int64_t N, bool wide)
{
    int64_t n = 64 + N / 8;
    if (n > (wide ? 256 : 512)) n = wide ? 256 : 512;
    if (n < (N + 255) / 256) n = (N + 255) / 256;
    return n < N ? n : N < 1 ? 1 : N;
}

// Threads of a row of so many 16-byte vectors in the gradient, of a workgroup's 512. Where a workgroup is
// done with all rows in two turns, it writes dweight and dbias itself: 4 x 270 bf16 takes 4.6 us of a captured
// graph and 8.4 of a call with it, 6.8 and 11.4 with parts and their sums, but 12 x 4096, in six turns, 15 and 7.7.
inline int norm_grad_threads(int64_t vectors)
{
    return vectors <= 8 ? 8 : vectors <= 16 ? 16 : vectors <= 32 ? 32 : vectors <= 128 ? 64 : vectors <= 256 ? 128 : vectors <= 512 ? 256 : 512;
}

hipError_t launch_norm_rows(int x_type, int y_type, const NormArgs &a, hipStream_t st);
hipError_t launch_norm_grad(int x_type, int y_type, const NormArgs &a, hipStream_t st);
// out[j][d] = the sum of the parts' [j][d], j = 0, 1; an out that is null is left out.
hipError_t launch_norm_sums(const float *parts, int64_t n_parts, int32_t D, void *dweight, void *dbias, int type,
                            hipStream_t st);

// ---------------------------------------------------------------- AdamW

constexpr int kStateBlock = 256;   // 8-bit states: values of a block
constexpr int kAdamwTensors = 44;  // tensors of one launch: their table fits a kernel's arguments

// Elements of a workgroup. With states in 32 bits, and for the values of 8-bit states, one vector a thread:
// neighbouring workgroups then move neighbouring addresses (168 million elements, 1,024 against 32,768 a
// workgroup: 865 and 962 us in fp32, 658 and 753 in bf16; the values 280 and 361). A step with 8-bit states
// pays for its start, and takes eight times as many where there are enough (fp32 500 us with 2,048, 522 with 8,192,
// 554 with 32,768; bf16 367, 350 and 366). A tensor's workgroups stay below 2^23.
inline int64_t adamw_chunk(int64_t total, bool step8)
{
    const int64_t least = step8 ? 2048 : 1024, some = step8 ? total / 4096 < 8192 ? total / 4096 : 8192 : 0, most = total >> 22;
    const int64_t n = (some > most ? some : most) + least - 1;
    return n < 2 * least ? least : n / least * least;
}

struct AdamwTable {
    void *param[kAdamwTensors];
    const void *grad[kAdamwTensors];
    void *m[kAdamwTensors], *v[kAdamwTensors];
    uint8_t *m_scales[kAdamwTensors], *v_scales[kAdamwTensors];
    float *master[kAdamwTensors];
    int64_t size[kAdamwTensors];
    int32_t first[kAdamwTensors + 1];  // chunks before each tensor
    int8_t type[kAdamwTensors], grad_type[kAdamwTensors];
    int32_t count;
    int32_t number;  // of the first tensor in the call
    int64_t chunk;
};

// What a step multiplies by, in fp32 from fp64: the same bits on the host and on the device.
struct AdamwRates {
    float b1, c1, b2, c2, keep, rate, root, eps, grad;
    float down;  // 1; or, where eps is so large that a denominator's reciprocal is subnormal, 2^-8, which rate, root and eps hold
    uint32_t step;

    __host__ __device__ static double power(double b, uint32_t t)  // by squaring
    {
        double r = 1.0;
        for (; t; t >>= 1, b *= b)
            if (t & 1) r *= b;
        return r;
    }
    __host__ __device__ void set(double lr, double beta1, double beta2, double weight_decay, uint32_t t)
    {
        step = t;
        b1 = (float)beta1, c1 = (float)(1.0 - beta1);
        b2 = (float)beta2, c2 = (float)(1.0 - beta2);
        keep = (float)(1.0 - lr * weight_decay);
        rate = (float)(lr / (1.0 - power(beta1, t)) * down);
        root = (float)(1.0 / sqrt(1.0 - power(beta2, t)) * down);
    }
};

struct AdamwArgs {
    AdamwRates rates;
    double lr, beta1, beta2, weight_decay;
    uint32_t seed;
    const float *lr_at;      // device, or null: lr
    const int32_t *step_at;  // device, or null: the rates' step
    const float *norm;       // device, or null: where it is not finite nothing is written
};

hipError_t launch_adamw(const AdamwTable &t, bool bits8, const AdamwArgs &a, hipStream_t st);
// m and v of 8-bit states as fp32, to param and master (both fp32 here).
hipError_t launch_adamw_values(const AdamwTable &t, hipStream_t st);

// ---------------------------------------------------------------- 4-bit values

constexpr int kFourBlock = 32;  // values that share a power of two: 16 bytes of codes, one of scale
__host__ __device__ inline int64_t four_blocks(int64_t K) { return (K + kFourBlock - 1) / kFourBlock; }

struct FourArgs {
    const void *x;           // rows [N][K], or columns: [K][N]; the values' y is written instead
    int64_t ldx;
    uint8_t *codes, *scales; // [N][blocks * 16], [N][blocks]
    int64_t N, K;
};

hipError_t launch_mx4_quantise(int type, bool columns, const FourArgs &a, hipStream_t st);
hipError_t launch_mx4_values(int type, bool columns, const FourArgs &a, void *y, int64_t ldy, hipStream_t st);

// Y = residual + act(X W + bias), W in 4 bits by columns, X in 16 bits or in 4 bits by rows.
struct FourProduct {
    const void *x;            // [N][K] of the type, or codes
    int64_t ldx;              // elements; not read for codes
    const uint8_t *x_scales;  // null: x is of the type
    const uint8_t *w, *w_scales;
    int64_t x_pitch, w_pitch;  // bytes of a row's scales
    const void *bias;
    bool bias_f32;
    int32_t act;
    const void *res;
    int64_t ldr;
    void *y;
    int64_t ldy;
    bool y_f32;
    int64_t N, K, M;
    int64_t width;  // features of x's rows, K or more (zeros behind K)
};

// The tile of a workgroup; the first four are those of the kernel for few rows.
enum FourTile { kFour16x16, kFour16x32, kFour32x32, kFour32x64, kFour64, kFour128, kFour192x256, kFour256 };
hipError_t launch_mx4_few(bool bf16, FourTile t, const FourProduct &p, hipStream_t st);

// The same for many rows. Rows in 16 bits must be whole lines of 128 bytes (four_width), rows of scales
// whole 16-byte pieces (four_pitch).
hipError_t launch_mx4_half(bool bf16, FourTile t, const FourProduct &p, hipStream_t st);
hipError_t launch_mx4_packed(bool bf16, FourTile t, const FourProduct &p, hipStream_t st);

inline int64_t four_width(int64_t K) { return (K + 63) / 64 * 64; }
__host__ __device__ inline int64_t four_pitch(int64_t K) { return (four_blocks(K) + 15) / 16 * 16; }
// Rows' scales to rows of four_pitch bytes, and rows of K values to rows of four_width; zeros behind them.
hipError_t launch_pad_scales(const uint8_t *scales, int64_t rows, int64_t K, uint8_t *to, hipStream_t st);
hipError_t launch_pad_rows(const void *x, int64_t ldx, int64_t rows, int64_t K, void *to, hipStream_t st);

}  // namespace som
