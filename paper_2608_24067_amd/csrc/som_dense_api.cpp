// som_dense_api.cpp -- host side of the dense entry points (include/som_dense.h): argument
// checks, workspace carving, the rules that choose tiles, launches on the caller's stream.

#include <hip/hip_runtime.h>

#include <cmath>

#include "som_dense.h"

namespace {

using som::Product;

som_status ok() { return som::set_error(SOM_OK, "%s", ""); }

som_status bad(const char *who, const char *what) { return som::set_error(SOM_ERR_INVALID_ARG, "%s: %s", who, what); }

som_status hip_fail(hipError_t e, const char *who)
{
    return som::set_error(SOM_ERR_HIP, "%s: %s (%d)", who, hipGetErrorString(e), (int)e);
}

bool half_type(int32_t t) { return t == SOM_F16 || t == SOM_BF16; }
bool any_type(int32_t t) { return t == SOM_F32 || half_type(t); }
bool act_ok(int32_t a) { return a >= SOM_ACT_NONE && a <= SOM_ACT_SILU; }
int64_t size_of(int32_t t) { return t == SOM_F32 ? 4 : 2; }
bool odd(const void *p, int32_t t) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size_t)(size_of(t) - 1)) != 0; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

som_status check_workspace(const char *who, const void *ws, size_t bytes, size_t need)
{
    if (need == 0) return SOM_OK;
    if (!ws) return som::set_error(SOM_ERR_WORKSPACE, "%s: workspace is NULL", who);
    if (reinterpret_cast<uintptr_t>(ws) & 255)
        return som::set_error(SOM_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", who);
    if (bytes < need)
        return som::set_error(SOM_ERR_WORKSPACE, "%s: workspace holds %zu bytes, the call needs %zu", who, bytes, need);
    return SOM_OK;
}

constexpr int64_t kMostDim = (int64_t)1 << 30;  // kernels number rows and columns in 32 bits, past the end too
bool dim_ok(int64_t v) { return v >= 1 && v < kMostDim; }

// Whether an operand's rows can be moved in whole 16-byte chunks.
bool chunks(const void *p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0; }

// Tiles of 16 rows and 128 columns, the height of the kernel for few rows.
int64_t few_tiles(int64_t rows, int64_t cols) { return (rows + 15) / 16 * ((cols + 127) / 128); }

// A product of few rows: all whose tiles are one a CU at most (bf16, us, few rows' kernel against the
// other: 96 rows 4096 x 4096 20.1 against 23.8, 512 rows 4096 x 1024 21.0 against 24.1; 48 rows
// 1024 x 16384, 384 tiles, 14.6 against 10.0), and every one of a single tile row.
bool few_rows(int64_t rows, int64_t cols) { return rows <= 16 || few_tiles(rows, cols) <= 256; }

// Experts go to the kernel for few rows from eight rows each on average down, where that can split
// the second reduction to fill the CUs (8 experts, D 1024, F 4096, 1 to 6 rows each: 34-48 us against
// 49-58 by Small tiles; 16 rows each 64 against 60) or rows are no whole chunks (13 experts of 1003 x
// 2001: 34-44 against 56-58). With a tile a CU without splits Small tiles, which keep six steps of
// loads in flight, read faster (32 experts, D 1024, F 2048, 1 to 6 rows: 43-68 us against 48-78).
constexpr int64_t kFewRows = 8;

// Pairs that are not ordered by expert first (a launch of 5 us): each reads its expert's weights for
// itself. While they are no more than the experts, few share one (64 experts, D 1024, F 2048: 16
// pairs 33 us against 39, 40 pairs 52 against 57; 16 experts, F 4096: 16 pairs 55 against 61, 24
// pairs 80 against 64; 4 experts: 16 pairs 40 against 29).
constexpr int64_t kFewPairs = 64;

// The tile of a product of `rows` rows a group and `cols` columns: the smallest of which two
// workgroups a CU hold all, since larger ones read each operand less often but take as long for one
// tile as for a CU's every (bf16, 4096 features, us by Small, Mid and Large tiles: 512 x 4096 38, 38,
// 80; 1024 x 4096 70, 43, 81; 2048 x 4096 134, 74, 84; 2304 x 4352 -, 102, 86; 2560 x 5120 209, 129,
// 95; 64 rows x 16384 25, 39, 78).
som::TileSize pick_tile(int64_t rows, int64_t groups, int64_t cols, bool whole)
{
    auto tiles = [&](som::TileSize t) {
        return (rows + tile_rows(t) - 1) / tile_rows(t) * groups * ((cols + tile_cols(t) - 1) / tile_cols(t));
    };
    if (whole && rows >= 192 && tiles(som::kTileMid) > 512) return som::kTileLarge;
    if (rows >= 64 && tiles(som::kTileSmall) > 512) return som::kTileMid;
    return som::kTileSmall;
}

// The tile of a product over rows (M x N a group), by the same rule (8192 rows, us by Mid and Large
// tiles: 2048 x 4096 145, 178; 2048 x 4352 184, 167; 4096 x 4096 253, 207; 10,007 rows of two among
// 32 experts, 2048 x 1000 each: 161, 122).
som::TileSize pick_tile_tn(int64_t M, int64_t N, int64_t groups)
{
    return (M + 127) / 128 * ((N + 127) / 128) * groups > 512 ? som::kTileLarge : som::kTileMid;
}

// Parts that a layer's weights' gradient (K x M from N rows) is computed in, where its tiles do not
// fill the CUs: of 512 rows at least, and of no more bytes (written and read again) than 32 MB and
// 7 KB a row (bf16, us in one part and in parts: 8192 rows 1024 x 1024 75, 32; 4096 rows 40, 24; 16384
// rows 256 x 256 144, 22, 2048 x 1024 146, 90; but 1024 rows 1024 x 1024 14, 16; 4096 rows 2048 x
// 2048 44, 48).
int grad_parts(int64_t N, int64_t K, int64_t M)
{
    const int64_t tiles = (K + 127) / 128 * ((M + 127) / 128), bytes = K * M * 4;
    int64_t n = 512 / tiles;
    if (n > N / 512) n = N / 512;
    const int64_t most = N * 7168 < (32 << 20) ? N * 7168 : 32 << 20;
    if (n > most / bytes) n = most / bytes;
    return n < 2 ? 1 : (int)n;
}

// ---------------------------------------------------------------- experts

struct ExpertsLayout {
    size_t off, n_tiles, tiles, row, w, pos, counts, inner, y, pre, weighted, dz, parts, total;
    som::TileSize tile;
    int splits;  // of the second product's reduction (few rows)
    bool plan;   // the pairs are ordered by expert
    int inner_splits;  // of the first product's reduction (without a plan)
    int64_t n_parts;
};

bool experts_dims(int64_t N, int32_t k, int64_t E, int64_t D, int64_t F)
{
    return N >= 0 && k >= 1 && k <= SOM_ROUTE_MAX_TAKEN && E >= 1 && E <= SOM_MAX_EXPERTS && N < (1 << 30) &&
           N * k < (1 << 30) && D >= 1 && D < (1 << 24) && F >= 1 && F < (1 << 24);
}

ExpertsLayout experts_layout(int64_t N, int32_t k, int64_t E, int64_t D, int64_t F, bool keep)
{
    ExpertsLayout L;
    const int64_t P = N * k, met = P < E ? (P < 1 ? 1 : P) : E;
    const bool whole = D % 8 == 0 && F % 8 == 0;
    L.tile = pick_tile(P / met, met, D < F ? D : F, whole);
    L.splits = 1;
    L.plan = true;
    L.inner_splits = 1;
    const int64_t tiles = met * ((D + 127) / 128);
    if (P / met <= kFewRows && (!whole || tiles < 256)) {
        // Few rows: fill the CUs by splitting the second reduction, a step of 32 a wave at least.
        L.tile = som::kTileFew;
        L.plan = keep || P > E || P > kFewPairs;
        const int64_t most = (F + 255) / 256;
        while (L.splits < 16 && tiles * L.splits < 256 && L.splits * 2 <= most) L.splits *= 2;
        if (!L.plan) {  // the first one too: its parts are added where the second reads them
            const int64_t inner_tiles = met * ((F + 127) / 128), inner_most = (D + 255) / 256;
            while (L.inner_splits < 8 && inner_tiles * L.inner_splits < 256 && L.inner_splits * 2 <= inner_most)
                L.inner_splits *= 2;
        }
    }
    L.n_parts = som::slope_parts(som::kTileSmall, F);  // the most of any tile
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t p = at;
        at += align256((size_t)bytes);
        return p;
    };
    L.off = take((E + 1) * 4);
    L.n_tiles = take(4);
    L.tiles = take(som::max_tile_rows(P, E, tile_rows(L.tile)) * (int64_t)sizeof(som::TileRow));
    L.row = take((P + 1) * 4);  // a product over no rows reads one entry past the last
    L.w = take(P * 4);
    L.pos = take(P * 4);
    L.counts = take(som::pair_stretches(P) * E * 4);
    L.inner = take(P * F * (L.inner_splits > 1 ? 4 * L.inner_splits : 2));
    L.y = take(L.splits * P * D * 4);
    L.pre = take(keep ? P * F * 2 : 0);
    L.weighted = take(keep ? P * F * 2 : 0);
    L.dz = take(keep ? P * F * 2 : 0);
    L.parts = take(keep ? P * L.n_parts * 4 : 0);
    L.total = at;
    return L;
}

struct Experts {
    som::PairPlan plan;
    void *inner, *pre, *weighted, *dz;
    float *y, *parts;
};

Experts carve(void *ws, const ExpertsLayout &L)
{
    char *b = static_cast<char *>(ws);
    Experts x;
    x.plan.off = reinterpret_cast<int32_t *>(b + L.off);
    x.plan.n_tiles = reinterpret_cast<int32_t *>(b + L.n_tiles);
    x.plan.tiles = reinterpret_cast<som::TileRow *>(b + L.tiles);
    x.plan.row = reinterpret_cast<int32_t *>(b + L.row);
    x.plan.w = reinterpret_cast<float *>(b + L.w);
    x.plan.pos = reinterpret_cast<int32_t *>(b + L.pos);
    x.plan.counts = reinterpret_cast<int32_t *>(b + L.counts);
    x.inner = b + L.inner;
    x.y = reinterpret_cast<float *>(b + L.y);
    x.pre = b + L.pre;
    x.weighted = b + L.weighted;
    x.dz = b + L.dz;
    x.parts = reinterpret_cast<float *>(b + L.parts);
    return x;
}

// The tile of a backward product: large ones need whole chunks, and few rows have no kernel of their own.
som::TileSize bwd_tile(som::TileSize t, bool whole)
{
    return t == som::kTileFew ? som::kTileSmall : t == som::kTileLarge && !whole ? som::kTileMid : t;
}

// A product over the plan's tile rows, by tiles of the plan's height or a part of it.
struct Grouped {
    const ExpertsLayout &L;
    const som::PairPlan &plan;
    int64_t P, E;
    Product product(som::TileSize t) const
    {
        Product p{};
        p.M = P;
        p.tiles = plan.tiles;
        p.n_tiles = plan.n_tiles;
        p.tile_height = tile_rows(L.tile);
        p.split = som::tiles_in_row(L.tile, t);
        p.groups = (int32_t)E;
        return p;
    }
};

}  // namespace

extern "C" {

som_status som_linear(int32_t type, const void *X, int64_t ldx, const void *W, int64_t ldw, const void *bias,
                      int32_t bias_type, int32_t act, const void *residual, int64_t ldr, void *Y, int64_t ldy,
                      int32_t y_type, void *pre, int64_t ldp, int64_t N, int64_t K, int64_t M, void *stream)
{
    const char *who = "som_linear";
    if (!half_type(type)) return bad(who, "type must be SOM_F16 or SOM_BF16");
    if (N < 0 || N >= kMostDim || !dim_ok(K) || !dim_ok(M)) return bad(who, "need 0 <= N, 1 <= K, M, all below 2^30");
    if (!act_ok(act)) return bad(who, "unknown activation");
    if (y_type != SOM_F32 && y_type != type) return bad(who, "y_type must be SOM_F32 or type");
    if (bias && bias_type != SOM_F32 && bias_type != type) return bad(who, "bias_type must be SOM_F32 or type");
    if (N == 0) return ok();
    if (!X || !W || !Y) return bad(who, "null pointer");
    if (ldx < K || ldw < M || ldy < M || (residual && ldr < M) || (pre && ldp < M))
        return bad(who, "a row stride is smaller than its row");
    if (odd(X, type) || odd(W, type) || odd(Y, y_type) || odd(pre, type) || odd(residual, type) ||
        (bias && odd(bias, bias_type)))
        return bad(who, "a pointer is not aligned to its elements");
    Product p{};
    p.A = X, p.lda = ldx, p.B = W, p.ldb = ldw;
    p.M = N, p.N = M, p.K = K, p.split = 1;
    p.bias = bias, p.bias_f32 = bias_type == SOM_F32, p.act = act;
    p.res = residual, p.ldr = ldr;
    p.out = Y, p.ldo = ldy, p.out_f32 = y_type == SOM_F32;
    p.pre = pre, p.ldp = ldp;
    const bool whole = chunks(X, ldx) && chunks(W, ldw) && K % 8 == 0 && M % 8 == 0;
    if (few_rows(N, M)) {
        const hipError_t e = som::launch_few(type == SOM_BF16, som::kLinear, p, 1, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? ok() : hip_fail(e, who);
    }
    const hipError_t e = som::launch_nn(type == SOM_BF16, som::kLinear, pick_tile(N, 1, M, whole), p,
                                        static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, who);
}

static size_t slope_bytes(int64_t N, int64_t M, int32_t act)
{
    return act == SOM_ACT_NONE ? 0 : align256((size_t)N * (size_t)M * 2);
}

size_t som_linear_bwd_workspace_bytes(int64_t N, int64_t K, int64_t M, int32_t act)
{
    if (N < 0 || N >= kMostDim || !dim_ok(K) || !dim_ok(M) || !act_ok(act)) return 0;
    const int parts = grad_parts(N, K, M);
    return slope_bytes(N, M, act) + (parts > 1 ? align256((size_t)parts * (size_t)(K + 1) * (size_t)M * 4) : 0);
}

som_status som_linear_bwd(int32_t type, const void *X, int64_t ldx, const void *W, int64_t ldw, const void *pre,
                          int64_t ldp, int32_t act, const void *dY, int64_t lddy, void *dX, int64_t lddx, void *dW,
                          int64_t lddw, void *dbias, int32_t bias_type, int64_t N, int64_t K, int64_t M,
                          void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "som_linear_bwd";
    if (!half_type(type)) return bad(who, "type must be SOM_F16 or SOM_BF16");
    if (N < 0 || N >= kMostDim || !dim_ok(K) || !dim_ok(M)) return bad(who, "need 0 <= N, 1 <= K, M, all below 2^30");
    if (!act_ok(act)) return bad(who, "unknown activation");
    if (dbias && bias_type != SOM_F32 && bias_type != type) return bad(who, "bias_type must be SOM_F32 or type");
    const bool slope = act != SOM_ACT_NONE;
    if (N > 0 && (!dY || (slope && !pre) || ((dW || dbias) && !X) || (dX && !W))) return bad(who, "null pointer");
    if ((N > 0 && (lddy < M || (slope && ldp < M) || ((dW || dbias) && ldx < K) || (dX && (ldw < M || lddx < K)))) ||
        (dW && lddw < M))
        return bad(who, "a row stride is smaller than its row");
    if (odd(X, type) || odd(W, type) || (slope && odd(pre, type)) || odd(dY, type) || odd(dX, type) || odd(dW, type) ||
        (dbias && odd(dbias, bias_type)))
        return bad(who, "a pointer is not aligned to its elements");
    const som_status st = check_workspace(who, workspace, workspace_bytes, som_linear_bwd_workspace_bytes(N, K, M, act));
    if (st != SOM_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf16 = type == SOM_BF16;
    hipError_t e = hipSuccess;
    const void *dz = dY;
    int64_t ldz = lddy;
    if (slope && N > 0) {
        e = som::launch_slope(bf16, dY, lddy, pre, ldp, act, N, M, workspace, s);
        if (e != hipSuccess) return hip_fail(e, who);
        dz = workspace, ldz = M;
    }
    if (dX && N > 0) {
        Product p{};
        p.A = dz, p.lda = ldz, p.B = W, p.ldb = ldw;
        p.M = N, p.N = K, p.K = M, p.split = 1;
        p.out = dX, p.ldo = lddx;
        const bool whole = chunks(dz, ldz) && chunks(W, ldw) && M % 8 == 0;
        e = som::launch_nt(bf16, som::kLinear, pick_tile(N, 1, K, whole), p, s);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    if (dW || dbias) {
        Product p{};
        p.A = X, p.lda = ldx, p.B = dz, p.ldb = ldz;
        p.M = K, p.N = M, p.K = N, p.split = 1;
        const int parts = grad_parts(N, K, M);
        if (parts == 1) {
            p.out = dW, p.ldo = lddw;
            p.db = dbias, p.bias_f32 = bias_type == SOM_F32;
            e = som::launch_tn(bf16, pick_tile_tn(K, M, 1), p, s);
            return e == hipSuccess ? ok() : hip_fail(e, who);
        }
        // each part's dW and column sums in fp32, then their sum
        float *sums = reinterpret_cast<float *>(static_cast<char *>(workspace) + slope_bytes(N, M, act));
        float *cols = sums + (size_t)parts * (size_t)K * (size_t)M;
        p.groups = parts;
        p.out = dW ? sums : nullptr, p.ldo = M, p.out_f32 = 1, p.strideC = K * M;
        p.db = dbias ? cols : nullptr, p.bias_f32 = 1, p.strideDb = M;
        e = som::launch_tn(bf16, pick_tile_tn(K, M, parts), p, s);
        if (e == hipSuccess && dW) e = som::launch_sum_parts(bf16, sums, parts, K * M, M, dW, lddw, false, s);
        if (e == hipSuccess && dbias)
            e = som::launch_sum_parts(bf16, cols, parts, M, M, dbias, M, bias_type == SOM_F32, s);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    return ok();
}

static som_status check_route(const char *who, int32_t logit_type, const void *logits, int64_t ldl, const float *bias,
                              int64_t N, int64_t E, int32_t k, const som_route_config *config, const void *idx,
                              int32_t weight_type, const void *weights, som::RouteArgs *a)
{
    if (!any_type(logit_type) || !any_type(weight_type)) return bad(who, "unknown type");
    if (N < 0 || N >= kMostDim) return bad(who, "need 0 <= N < 2^30");
    if (E < 1 || E > SOM_ROUTE_MAX_UNITS) return bad(who, "need 1 <= E <= SOM_ROUTE_MAX_UNITS");
    if (k < 1 || k > SOM_ROUTE_MAX_TAKEN || k > E) return bad(who, "need 1 <= k <= min(E, SOM_ROUTE_MAX_TAKEN)");
    som_route_config c{};
    if (config) c = *config;
    for (int32_t r : c.reserved)
        if (r != 0) return bad(who, "som_route_config.reserved must be zero");
    if (c.score != SOM_SCORE_SOFTMAX && c.score != SOM_SCORE_SIGMOID) return bad(who, "unknown score");
    if (c.renorm != 0 && c.renorm != 1) return bad(who, "renorm must be 0 or 1");
    if (c.groups == 0) c.groups = 1;
    if (c.groups < 1 || c.groups > SOM_ROUTE_MAX_GROUPS || E % c.groups != 0)
        return bad(who, "groups must divide E and be at most SOM_ROUTE_MAX_GROUPS");
    if (c.group_top == 0) c.group_top = c.groups;
    if (c.group_top < 1 || c.group_top > c.groups) return bad(who, "need 1 <= group_top <= groups");
    if (N > 0) {
        if (!logits || !idx || !weights) return bad(who, "null pointer");
        if (ldl < E) return bad(who, "a row stride is smaller than its row");
        if (odd(logits, logit_type) || odd(weights, weight_type) || odd(idx, SOM_F32) || odd(bias, SOM_F32))
            return bad(who, "a pointer is not aligned to its elements");
    }
    a->logits = logits, a->ldl = ldl, a->bias = bias, a->N = N, a->E = (int32_t)E, a->k = k;
    a->score = c.score, a->renorm = c.renorm, a->groups = c.groups, a->group_top = c.group_top;
    a->weight_type = weight_type;
    return SOM_OK;
}

som_status som_route(int32_t logit_type, const void *logits, int64_t ldl, const float *bias, int64_t N, int64_t E,
                     int32_t k, const som_route_config *config, int32_t *idx, int32_t weight_type, void *weights,
                     int32_t *counts, void *stream)
{
    const char *who = "som_route";
    som::RouteArgs a{};
    const som_status st = check_route(who, logit_type, logits, ldl, bias, N, E, k, config, idx, weight_type, weights, &a);
    if (st != SOM_OK) return st;
    if (odd(counts, SOM_F32)) return bad(who, "a pointer is not aligned to its elements");
    if (N == 0 && !counts) return ok();
    a.idx = idx, a.weights = weights, a.counts = counts;
    const hipError_t e = som::launch_route(logit_type, a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, who);
}

som_status som_route_bwd(int32_t logit_type, const void *logits, int64_t ldl, const float *bias, const int32_t *idx,
                         int32_t weight_type, const void *dweights, int64_t N, int64_t E, int32_t k,
                         const som_route_config *config, void *dlogits, int64_t lddl, void *stream)
{
    const char *who = "som_route_bwd";
    som::RouteArgs a{};
    const som_status st = check_route(who, logit_type, logits, ldl, bias, N, E, k, config, idx, weight_type, dweights, &a);
    if (st != SOM_OK) return st;
    if (N == 0) return ok();
    if (!dlogits) return bad(who, "null pointer");
    if (lddl < E) return bad(who, "a row stride is smaller than its row");
    if (odd(dlogits, logit_type)) return bad(who, "a pointer is not aligned to its elements");
    a.idx = const_cast<int32_t *>(idx), a.weights = const_cast<void *>(dweights);
    a.dlogits = dlogits, a.lddl = lddl;
    const hipError_t e = som::launch_route_bwd(logit_type, a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ok() : hip_fail(e, who);
}

size_t som_experts_workspace_bytes(int64_t N, int32_t k, int64_t E, int64_t D, int64_t F, int32_t keep)
{
    if (!experts_dims(N, k, E, D, F) || (keep != 0 && keep != 1)) return 0;
    return experts_layout(N, k, E, D, F, keep == 1).total;
}

static som_status check_experts(const char *who, int32_t type, int64_t N, int32_t k, int64_t E, int64_t D, int64_t F,
                                int32_t act)
{
    if (!half_type(type)) return bad(who, "type must be SOM_F16 or SOM_BF16");
    if (!experts_dims(N, k, E, D, F))
        return bad(who, "sizes out of range (1 <= k <= 32, 1 <= E <= 1024, N k < 2^30, 1 <= D, F < 2^24)");
    if (!act_ok(act)) return bad(who, "unknown activation");
    return SOM_OK;
}

som_status som_experts(int32_t type, const void *X, int64_t ldx, const int32_t *idx, const void *w, const void *W1,
                       const void *b1, const void *W2, const void *b2, int32_t act, const void *residual, int64_t ldr,
                       void *out, int64_t ldo, int64_t N, int32_t k, int64_t E, int64_t D, int64_t F, int32_t keep,
                       void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "som_experts";
    som_status st = check_experts(who, type, N, k, E, D, F, act);
    if (st != SOM_OK) return st;
    if (keep != 0 && keep != 1) return bad(who, "keep must be 0 or 1");
    if (N == 0) return ok();
    if (!X || !idx || !w || !W1 || !W2 || !out) return bad(who, "null pointer");
    if (ldx < D || ldo < D || (residual && ldr < D)) return bad(who, "a row stride is smaller than its row");
    if (odd(X, type) || odd(idx, SOM_F32) || odd(w, type) || odd(W1, type) || odd(b1, type) || odd(W2, type) ||
        odd(b2, type) || odd(residual, type) || odd(out, type))
        return bad(who, "a pointer is not aligned to its elements");
    const ExpertsLayout L = experts_layout(N, k, E, D, F, keep == 1);
    if ((st = check_workspace(who, workspace, workspace_bytes, L.total)) != SOM_OK) return st;
    const Experts x = carve(workspace, L);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf16 = type == SOM_BF16;
    const int64_t P = N * k;
    hipError_t e = hipSuccess;
    if (L.plan) e = som::launch_pairs(bf16, idx, w, P, k, (int32_t)E, tile_rows(L.tile), x.plan, s);
    if (e != hipSuccess) return hip_fail(e, who);
    const Grouped g{L, x.plan, P, E};
    {
        const bool whole = chunks(W1, F) && chunks(X, ldx);
        const som::TileSize t = L.tile == som::kTileLarge && !whole ? som::kTileMid : L.tile;
        Product p = g.product(t);
        p.A = X, p.lda = ldx, p.amap = x.plan.row;
        p.B = W1, p.ldb = F, p.strideB = D * F;
        p.N = F, p.K = D;
        p.bias = b1, p.strideBias = F, p.act = act;
        p.out = x.inner, p.ldo = F;
        if (!L.plan) p.pairs = idx, p.pair_rows = k;
        if (L.inner_splits > 1) {  // z in parts, without bias
            p.bias = nullptr;
            e = som::launch_few(bf16, som::kPairs, p, L.inner_splits, s);
            if (e != hipSuccess) return hip_fail(e, who);
        } else {
            if (keep) p.pre = x.pre, p.ldp = F, p.weighted = x.weighted, p.w = x.plan.w;
            e = t == som::kTileFew ? som::launch_few(bf16, som::kInner, p, 1, s) : som::launch_nn(bf16, som::kInner, t, p, s);
            if (e != hipSuccess) return hip_fail(e, who);
        }
    }
    {
        const som::TileSize t = L.tile == som::kTileLarge && !chunks(W2, D) ? som::kTileMid : L.tile;
        Product p = g.product(t);
        p.A = x.inner, p.lda = F;
        p.B = W2, p.ldb = D, p.strideB = D * F;
        p.N = D, p.K = F;
        p.bias = b2, p.strideBias = D;
        if (L.plan) p.w = x.plan.w;
        p.out = x.y, p.ldo = D;
        if (!L.plan) p.pairs = idx, p.pair_w = w, p.pair_rows = 1;
        if (L.inner_splits > 1) p.z_parts = L.inner_splits, p.z_bias = b1, p.act = act;
        e = t == som::kTileFew ? som::launch_few(bf16, som::kPairs, p, L.splits, s)
                               : som::launch_nn(bf16, som::kPairs, t, p, s);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    e = som::launch_combine(bf16, x.y, L.splits, L.plan ? x.plan.pos : idx, L.plan ? 0 : (int32_t)E, N, k, D, residual, ldr, out, ldo, s);
    return e == hipSuccess ? ok() : hip_fail(e, who);
}

som_status som_experts_bwd(int32_t type, const void *X, int64_t ldx, const int32_t *idx, const void *w, const void *W1,
                           const void *W2, const void *b2, int32_t act, const void *dout, int64_t lddo, void *dX,
                           int64_t lddx, void *dw, void *dW1, void *db1, void *dW2, void *db2, int64_t N, int32_t k,
                           int64_t E, int64_t D, int64_t F, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "som_experts_bwd";
    som_status st = check_experts(who, type, N, k, E, D, F, act);
    if (st != SOM_OK) return st;
    if (N > 0) {
        if (!X || !idx || !w || !W1 || !W2 || !dout) return bad(who, "null pointer");
        if (ldx < D || lddo < D || (dX && lddx < D)) return bad(who, "a row stride is smaller than its row");
    }
    if (odd(X, type) || odd(idx, SOM_F32) || odd(w, type) || odd(W1, type) || odd(W2, type) || odd(b2, type) ||
        odd(dout, type) || odd(dX, type) || odd(dw, type) || odd(dW1, type) || odd(db1, type) || odd(dW2, type) ||
        odd(db2, type))
        return bad(who, "a pointer is not aligned to its elements");
    const ExpertsLayout L = experts_layout(N, k, E, D, F, true);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf16 = type == SOM_BF16;
    if ((st = check_workspace(who, workspace, workspace_bytes, L.total)) != SOM_OK) return st;
    const Experts x = carve(workspace, L);
    const int64_t P = N * k;
    const Grouped g{L, x.plan, P, E};
    hipError_t e = hipSuccess;
    if (N == 0) {  // no rows: every expert's stretch is empty
        e = som::launch_pairs(bf16, idx, w, 0, k, (int32_t)E, tile_rows(L.tile), x.plan, s);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    if (N > 0 && (dX || dw || dW1 || db1)) {  // dz, and the weights' gradients in parts
        const bool whole = chunks(W2, D) && chunks(dout, lddo);
        const som::TileSize t = bwd_tile(L.tile, whole);
        Product p = g.product(t);
        p.A = dout, p.lda = lddo, p.amap = x.plan.row;
        p.B = W2, p.ldb = D, p.strideB = D * F;
        p.N = F, p.K = D;
        p.act = act, p.w = x.plan.w;
        p.pre = x.pre, p.ldp = F;
        p.res = x.inner, p.ldr = F;
        p.out = x.dz, p.ldo = F;
        p.parts = x.parts;
        p.n_parts = som::slope_parts(t, F);
        e = som::launch_nt(bf16, som::kSlope, t, p, s);
        if (e != hipSuccess) return hip_fail(e, who);
        if (dw) {
            e = som::launch_weight_grad(bf16, x.parts, p.n_parts, x.plan.pos, idx, b2, dout, lddo, N, k, D, dw, s);
            if (e != hipSuccess) return hip_fail(e, who);
        }
    }
    if (dX && N > 0) {
        const som::TileSize t = bwd_tile(L.tile, chunks(W1, F));
        Product p = g.product(t);
        p.A = x.dz, p.lda = F;
        p.B = W1, p.ldb = F, p.strideB = D * F;
        p.N = D, p.K = F;
        p.out = x.y, p.ldo = D;
        e = som::launch_nt(bf16, som::kPairs, t, p, s);
        if (e != hipSuccess) return hip_fail(e, who);
        e = som::launch_combine(bf16, x.y, 1, x.plan.pos, 0, N, k, D, nullptr, 0, dX, lddx, s);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    if (dW1 || db1) {
        Product p{};
        p.A = X, p.lda = ldx, p.amap = x.plan.row;
        p.B = x.dz, p.ldb = F;
        p.M = D, p.N = F, p.split = 1;
        p.off = x.plan.off, p.groups = (int32_t)E;
        p.out = dW1, p.ldo = F, p.strideC = D * F;
        p.db = db1, p.strideDb = F;
        e = som::launch_tn(bf16, pick_tile_tn(D, F, E), p, s);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    if (dW2 || db2) {
        Product p{};
        p.A = x.weighted, p.lda = F;
        p.B = dout, p.ldb = lddo, p.bmap = x.plan.row;
        p.M = F, p.N = D, p.split = 1;
        p.off = x.plan.off, p.groups = (int32_t)E;
        p.out = dW2, p.ldo = D, p.strideC = D * F;
        p.db = db2, p.strideDb = D, p.w = x.plan.w;
        e = som::launch_tn(bf16, pick_tile_tn(F, D, E), p, s);
        if (e != hipSuccess) return hip_fail(e, who);
    }
    return ok();
}

// Chunks of all tensors and their size; negative if a size is out of range.
static int64_t clip_chunks(const int64_t *sizes, int64_t count, int64_t *chunk)
{
    if (count < 0 || count > INT32_MAX || (count > 0 && !sizes)) return -1;
    int64_t total = 0, n = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] < 0 || sizes[i] > ((int64_t)1 << 40) || total > ((int64_t)1 << 45)) return -1;
        total += sizes[i];
    }
    *chunk = som::clip_chunk(total);
    for (int64_t i = 0; i < count; ++i) n += (sizes[i] + *chunk - 1) / *chunk;
    return n > INT32_MAX ? -1 : n;
}

size_t som_clip_workspace_bytes(const int64_t *sizes, int64_t count)
{
    int64_t chunk;
    const int64_t n = clip_chunks(sizes, count, &chunk);
    return n < 0 ? 0 : 256 + align256((size_t)n * 8);
}

som_status som_clip(const void *const *tensors, void *const *outs, const int64_t *sizes, const int32_t *types,
                    int64_t count, float max_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "som_clip";
    int64_t chunk;
    const int64_t chunks_total = clip_chunks(sizes, count, &chunk);
    if (chunks_total < 0) return bad(who, "count or a size is out of range");
    if (!norm || (count > 0 && (!tensors || !outs || !types))) return bad(who, "null pointer");
    if (!(max_norm > 0.0f) || std::isinf(max_norm)) return bad(who, "max_norm must be positive and finite");
    if (odd(norm, SOM_F32)) return bad(who, "a pointer is not aligned to its elements");
    for (int64_t i = 0; i < count; ++i) {
        if (!any_type(types[i])) return bad(who, "unknown type");
        if (sizes[i] > 0 && (!tensors[i] || !outs[i])) return bad(who, "null pointer");
        if (odd(tensors[i], types[i]) || odd(outs[i], types[i])) return bad(who, "a pointer is not aligned to its elements");
    }
    const som_status st = check_workspace(who, workspace, workspace_bytes, som_clip_workspace_bytes(sizes, count));
    if (st != SOM_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double *scale = static_cast<double *>(workspace);
    double *partial = reinterpret_cast<double *>(static_cast<char *>(workspace) + 256);
    // Few chunks: one launch less, each workgroup of the last pass adds them for itself.
    const bool few = chunks_total > 0 && chunks_total <= 4096 && count <= som::kClipTensors;
    for (int pass = 0; pass < 2; ++pass) {
        int64_t done = 0;
        for (int64_t i = 0; i < count; i += som::kClipTensors) {
            som::ClipTable t;
            t.count = (int32_t)(count - i < som::kClipTensors ? count - i : som::kClipTensors);
            t.chunk = chunk;
            t.first[0] = 0;
            for (int j = 0; j < t.count; ++j) {
                t.in[j] = tensors[i + j], t.out[j] = outs[i + j];
                t.size[j] = sizes[i + j], t.type[j] = types[i + j];
                t.first[j + 1] = t.first[j] + (int32_t)((t.size[j] + chunk - 1) / chunk);
            }
            const hipError_t e = pass == 0 ? som::launch_squares(t, partial + done, s)
                                 : few     ? som::launch_scale(t, nullptr, partial, chunks_total, max_norm, norm, s)
                                           : som::launch_scale(t, scale, nullptr, 0, max_norm, norm, s);
            if (e != hipSuccess) return hip_fail(e, who);
            done += t.first[t.count];
        }
        if (pass == 0 && !few) {
            const hipError_t e = som::launch_norm(partial, chunks_total, max_norm, norm, scale, s);
            if (e != hipSuccess) return hip_fail(e, who);
        }
    }
    return ok();
}

}  // extern "C"
