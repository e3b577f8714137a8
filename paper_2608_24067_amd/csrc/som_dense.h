// som_dense.h -- shared between the host layer of the dense entry points (include/som_dense.h)
// and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/som.h"
#include "../../include/som_dense.h"

namespace som {

som_status set_error(som_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

// A launch of `blocks` workgroups, numbered by block_number. HIP takes fewer than 2^32 threads along x,
// so beyond 2^21 workgroups (of 1,024 threads at most) they go on along y; the last row of them
// reaches past `blocks`, which every kernel launched so checks. 0 blocks along x: more than a grid holds.
constexpr int64_t kBlocksAlongX = (int64_t)1 << 21;

inline dim3 grid_of(int64_t blocks)
{
    if (blocks <= kBlocksAlongX) return dim3((unsigned)blocks);
    const int64_t rows = (blocks + kBlocksAlongX - 1) / kBlocksAlongX;
    return rows < 65536 ? dim3((unsigned)kBlocksAlongX, (unsigned)rows) : dim3(0);
}

// ---------------------------------------------------------------- matrix products

// One tile row of a grouped product: the rows [row, end) of the ordered pairs belong to
// expert e; the tile starts at `row` and takes as many of them as it is high.
struct TileRow {
    int32_t e, row, end, pad;
};

// C = A B with an epilogue. `A` has the M rows of the result (the reduction runs along its
// columns) except in products over rows (TN), where the reduction runs over the rows of both
// operands and the result is K_cols(A) x K_cols(B).
struct Product {
    const void *A, *B;
    int64_t lda, ldb;       // elements
    const int32_t *amap;    // non-null: row r of A is row amap[r] of the array
    const int32_t *bmap;    // TN only: the same for B
    int64_t M, N, K;        // result rows and columns, reduction length (grouped: see below)
    // Grouped products. NN, NT: the tile rows; M is the number of pairs, B and the bias advance
    // by strideB and strideBias from expert to expert. TN: expert e reduces over the rows
    // [off[e], off[e + 1]) and the result advances by strideC; without `off` the groups are equal
    // parts of the K rows.
    const TileRow *tiles;
    const int32_t *n_tiles;
    int32_t split;          // workgroup tiles in the height of a tile row
    int32_t tile_height;    // rows of a tile row at most
    // Few pairs without a plan (launch_few): pair m is a tile of its own, for expert pairs[m], its
    // row of A is m / pair_rows and its weight pair_w[m] (null: 1).
    const int32_t *pairs;
    const void *pair_w;
    int32_t pair_rows;
    // Then A may be z in fp32, z_parts arrays of M rows to be added up: what is multiplied is
    // act(z + z_bias[e]), rounded to the rows' type.
    int32_t z_parts;
    const void *z_bias;
    const int32_t *off;
    int32_t groups;         // 0: not grouped
    int64_t strideB, strideBias, strideC;
    // Epilogue.
    const void *bias;
    int32_t bias_f32, act;
    const void *res;        // residual, rows' type (kSlope: act(pre) as the forward pass left it)
    int64_t ldr;
    void *out;
    int64_t ldo;
    int32_t out_f32;
    void *weighted;         // kInner: w act(...) too, as `out` is laid out; or null
    void *pre;              // value before the activation, rows' type: written by NN, read by kSlope
    int64_t ldp;
    const float *w;         // a weight for each row (kInner: with `weighted`; kPairs, kSlope; TN: of the
                            // reduction's rows)
    float *parts;           // kSlope: per row and column part, the sum of act(pre) * product
    int64_t n_parts;
    void *db;               // TN: the column sums of B (each row times w), as bias_f32 says
    int64_t strideDb;
};

// What the backward pass needs of z and dz is held in the rows' type. dz is an operand of the matrix
// instructions, which take 16 bits. z (`pre`) enters the slope only, which its rounding moves by at
// most 0.8 u |z|, u = 2^-8 or 2^-11 (bf16 gradients off by 0.24% of their size, 0.17% from an fp32
// z); in fp32 it would add 2 bytes to the 6 a value that kInner's and kSlope's epilogues move, which
// the products do not hide. w act(z) for dW2 is an operand too: in fp16, weights of 1e-5 make it
// subnormal, as they make dz; a caller who scales dout for dz's sake does not scale it.
enum Epilogue {
    kLinear,  // out = res + act(acc + bias), pre = acc + bias
    kInner,   // out = act(acc + bias), weighted = w * act(acc + bias), pre = acc + bias
    kPairs,   // out (fp32) = w * (acc + bias)
    kSlope,   // out = w * acc * act'(pre), parts = sum over columns of act(pre) * acc, act(pre) = res
    kGrad     // TN: out = acc, db = column sums of B
};

// Rows of a tile of the product the host picks, so that the plan can lay the tile rows out.
enum TileSize { kTileFew, kTileSmall, kTileMid, kTileLarge };  // kTileFew: som_few.hip, else som_mm*.hip
constexpr int tile_rows(TileSize t) { return t == kTileFew ? 16 : t == kTileSmall ? 32 : t == kTileMid ? 128 : 256; }
constexpr int tile_cols(TileSize t) { return t == kTileLarge ? 256 : 128; }

// Tile rows of a plan over P pairs of E experts, at most.
inline int64_t max_tile_rows(int64_t P, int64_t E, int rows) { return P / rows + (E < P ? E : P); }

// Tiles of t in the height of a tile row of a plan laid out for `plan`; a tile higher than that takes
// one tile row all the same.
inline int tiles_in_row(TileSize plan, TileSize t)
{
    return tile_rows(plan) > tile_rows(t) ? tile_rows(plan) / tile_rows(t) : 1;
}

// Rows of tiles a product (NN, NT) is launched with. A grouped one may meet any loads, so it needs
// as many as the plan has tile rows at the height the plan was laid out for: tiles higher than that
// are no fewer.
inline int64_t launch_tile_rows(const Product &p, TileSize t)
{
    return p.groups ? max_tile_rows(p.M, p.groups, p.tile_height) * p.split : (p.M + tile_rows(t) - 1) / tile_rows(t);
}

hipError_t launch_nn(bool bf16, Epilogue e, TileSize t, const Product &p, hipStream_t st);
// The same (kLinear, kInner, kPairs) for few rows. splits: workgroups that share out a tile's
// reduction (kPairs only, else 1); split s of row m is written to row s * M + m of the result.
hipError_t launch_few(bool bf16, Epilogue e, const Product &p, int splits, hipStream_t st);
hipError_t launch_nt(bool bf16, Epilogue e, TileSize t, const Product &p, hipStream_t st);
hipError_t launch_tn(bool bf16, TileSize t, const Product &p, hipStream_t st);  // kTileMid or kTileLarge

// Partial sums of a row that a kSlope product over N columns leaves (one for each wave's columns).
inline int64_t slope_parts(TileSize t, int64_t N)
{
    return (N + tile_cols(t) - 1) / tile_cols(t) * (tile_cols(t) / (t == kTileSmall ? 32 : 64));
}

// ---------------------------------------------------------------- routing

struct RouteArgs {
    const void *logits;
    int64_t ldl;
    const float *bias;
    int64_t N;
    int32_t E, k, score, renorm, groups, group_top;
    int32_t *idx;            // written by the choice, read by the gradient
    void *weights;           // the gradient's dweights
    int32_t weight_type;
    int32_t *counts;
    void *dlogits;
    int64_t lddl;
};

hipError_t launch_route(int logit_type, const RouteArgs &a, hipStream_t st);
hipError_t launch_route_bwd(int logit_type, const RouteArgs &a, hipStream_t st);

// ---------------------------------------------------------------- experts

// The pairs (row, place) ordered by expert, in the pairs' order within one.
struct PairPlan {
    int32_t *off;       // [E + 1] where each expert's pairs start
    int32_t *n_tiles;   // [1]
    TileRow *tiles;     // tile rows of `rows` pairs
    int32_t *row;       // [P] ordered pair -> row
    float *w;           // [P] ordered pair -> weight
    int32_t *pos;       // [P] pair -> its place in the order, -1 for a pair without an expert
    int32_t *counts;    // [pair_stretches(P)][E] scratch
};

// Up to this many pairs are ordered by one workgroup (2,048 pairs: one launch of about 8 us
// against three of 4); more in stretches of 256 pairs, at most 256 of them.
constexpr int64_t kPairsOfOne = 2048;
inline int pair_stretches(int64_t P)
{
    if (P <= kPairsOfOne) return 0;
    const int64_t n = (P + 255) / 256;
    return (int)(n < 256 ? n : 256);
}

hipError_t launch_pairs(bool bf16, const int32_t *idx, const void *w, int64_t P, int32_t k, int32_t E, int rows,
                        const PairPlan &plan, hipStream_t st);

// out[n] = res[n] + the rows y[pos[n, j]] (fp32, D wide) in the order of j, each the sum of
// `splits` rows N k apart. Without a plan `pos` are the pairs' experts and a pair's row is its own.
hipError_t launch_combine(bool bf16, const float *y, int splits, const int32_t *pos, int32_t no_plan_E, int64_t N, int32_t k, int64_t D,
                          const void *res, int64_t ldr, void *out, int64_t ldo, hipStream_t st);

// dw[n, j] = the sum of parts[pos] plus <b2[idx], dout[n]>; 0 for a pair without an expert.
hipError_t launch_weight_grad(bool bf16, const float *parts, int64_t n_parts, const int32_t *pos, const int32_t *idx,
                              const void *b2, const void *dout, int64_t lddo, int64_t N, int32_t k, int64_t D,
                              void *dw, hipStream_t st);

// out = the sum of `parts` fp32 arrays of n values, one after the other, in their order; out is
// fp32 or of the rows' type, in rows of M values ldo apart.
hipError_t launch_sum_parts(bool bf16, const float *in, int parts, int64_t n, int64_t M, void *out, int64_t ldo,
                            bool out_f32, hipStream_t st);

// dz = dy act'(pre), rows of M elements; dz is dense.
hipError_t launch_slope(bool bf16, const void *dy, int64_t lddy, const void *pre, int64_t ldp, int act, int64_t N,
                        int64_t M, void *dz, hipStream_t st);

// ---------------------------------------------------------------- clipping

constexpr int kClipTensors = 48;      // tensors of one launch

// Elements of a workgroup: 2,048 workgroups where the tensors hold that many, 64K elements at most.
inline int64_t clip_chunk(int64_t total)
{
    const int64_t n = (total / 2048 + 2047) / 2048 * 2048;
    return n < 2048 ? 2048 : n > 65536 ? 65536 : n;
}

struct ClipTable {
    const void *in[kClipTensors];
    void *out[kClipTensors];
    int64_t size[kClipTensors];
    int32_t first[kClipTensors + 1];  // chunks before each tensor
    int32_t type[kClipTensors];
    int32_t count;
    int64_t chunk;
};

hipError_t launch_squares(const ClipTable &t, double *partial, hipStream_t st);
hipError_t launch_norm(const double *partial, int64_t n, float max_norm, float *norm, double *scale, hipStream_t st);
// scale: what launch_norm wrote; or null and the n partial sums, which every workgroup then adds
// itself (the first also writes norm).
hipError_t launch_scale(const ClipTable &t, const double *scale, const double *partial, int64_t n, float max_norm,
                        float *norm, hipStream_t st);

}  // namespace som
