// som_layer_api.cpp -- host side of layer norm, AdamW and the 4-bit operators (include/som_dense.h):
// argument checks, workspace carving, launches on the caller's stream.

#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include "som_layer.h"

namespace {

som_status ok() { return som::set_error(SOM_OK, "%s", ""); }

som_status bad(const char *who, const char *what) { return som::set_error(SOM_ERR_INVALID_ARG, "%s: %s", who, what); }

som_status done(hipError_t e, const char *who)
{
    return e == hipSuccess ? ok() : som::set_error(SOM_ERR_HIP, "%s: %s (%d)", who, hipGetErrorString(e), (int)e);
}

bool half_type(int32_t t) { return t == SOM_F16 || t == SOM_BF16; }
bool any_type(int32_t t) { return t == SOM_F32 || half_type(t); }
int64_t size_of(int32_t t) { return t == SOM_F32 ? 4 : 2; }
bool off(const void *p, int64_t align) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(align - 1)) != 0; }
bool odd(const void *p, int32_t t) { return off(p, size_of(t)); }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

constexpr int64_t kMostDim = (int64_t)1 << 30;
bool dim_ok(int64_t v) { return v >= 1 && v < kMostDim; }
bool width_ok(int64_t v) { return v >= 1 && v < ((int64_t)1 << 20); }  // of normalised rows
bool rows_ok(int64_t v) { return v >= 0 && v < kMostDim; }

som_status check_workspace(const char *who, const void *ws, size_t bytes, size_t need)
{
    if (need == 0) return SOM_OK;
    if (!ws) return som::set_error(SOM_ERR_WORKSPACE, "%s: workspace is NULL", who);
    if (off(ws, 256)) return som::set_error(SOM_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", who);
    if (bytes < need)
        return som::set_error(SOM_ERR_WORKSPACE, "%s: workspace holds %zu bytes, the call needs %zu", who, bytes, need);
    return SOM_OK;
}

const char *const kNotAligned = "a pointer is not aligned to its elements";
const char *const kStride = "a row stride is smaller than its row";
const char *const kNull = "null pointer";

// What layer norm's two directions have in common.
const char *norm_types(int32_t type, int32_t y_type, int32_t weight_type)
{
    if (!any_type(type)) return "type must be SOM_F32, SOM_F16 or SOM_BF16";
    if (!any_type(y_type) || (y_type != type && type != SOM_F32)) return "y_type must be type, or any where that is SOM_F32";
    if (weight_type != SOM_F32 && weight_type != y_type) return "weight_type must be SOM_F32 or y_type";
    return nullptr;
}

som_status steps_ok(const char *who, const som_adamw_tensor *t, int64_t count, bool bits8, bool params)
{
    if (count < 0 || count > INT32_MAX) return bad(who, "count is out of range");
    if (count > 0 && !t) return bad(who, kNull);
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) {
        const som_adamw_tensor &x = t[i];
        if (x.size < 0 || x.size > ((int64_t)1 << 38) || total > ((int64_t)1 << 43)) return bad(who, "a size is out of range");
        total += x.size;
        if (params && (!any_type(x.type) || !any_type(x.grad_type))) return bad(who, "unknown type");
        if (x.size == 0) continue;
        if (!x.m || !x.v || (params && (!x.param || !x.grad)) || (bits8 && (!x.m_scales || !x.v_scales))) return bad(who, kNull);
        if (!bits8 && (odd(x.m, SOM_F32) || odd(x.v, SOM_F32))) return bad(who, kNotAligned);
        if (params && (odd(x.param, x.type) || odd(x.grad, x.grad_type) || odd(x.master, SOM_F32))) return bad(who, kNotAligned);
    }
    return SOM_OK;
}

// Tables of the tensors, as many as a launch takes at a time; f(table).
template <typename F> hipError_t over_tables(const som_adamw_tensor *tensors, int64_t count, bool step8, F f)
{
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) total += tensors[i].size;
    const int64_t chunk = som::adamw_chunk(total, step8);
    for (int64_t i = 0; i < count;) {
        som::AdamwTable t;
        t.count = 0;
        t.number = (int32_t)i;
        t.chunk = chunk;
        t.first[0] = 0;
        for (; i < count && t.count < som::kAdamwTensors; ++i) {
            const som_adamw_tensor &x = tensors[i];
            const int64_t chunks = (x.size + chunk - 1) / chunk;
            // a launch has fewer than 2^32 threads; a tensor has 2^22 chunks at most
            if (t.count > 0 && t.first[t.count] + chunks > (1 << 23)) break;
            const int j = t.count++;
            t.param[j] = x.param, t.grad[j] = x.grad, t.m[j] = x.m, t.v[j] = x.v;
            t.m_scales[j] = x.m_scales, t.v_scales[j] = x.v_scales, t.master[j] = x.master;
            t.size[j] = x.size, t.type[j] = (int8_t)x.type, t.grad_type[j] = (int8_t)x.grad_type;
            t.first[j + 1] = t.first[j] + (int32_t)chunks;
        }
        const hipError_t e = f(t, i);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

const char *product_sizes(int64_t N, int64_t K, int64_t M)
{
    return rows_ok(N) && dim_ok(K) && dim_ok(M) ? nullptr : "need 0 <= N, 1 <= K, M, all below 2^30";
}

// ---------------------------------------------------------------- products with a 4-bit matrix

// How a product is computed, and what of its workspace holds what.
struct FourLayout {
    som::FourTile tile;
    int64_t strip;            // rows in 16 bits that are copied and multiplied at a time
    size_t x, xs, ws, total;  // their copy, and padded rows of scales
};

// Bytes of the copied rows at most: strips of them stay in the cache.
constexpr int64_t kFourStrip = (int64_t)32 << 20;
// Rows of more than 65,536 features, 256 of which do not fit, are not copied: those off 16 bytes take the kernel for few
// rows, whatever their number (300 x 70001 x 200 in bf16 187 us; 65,600 features, which tiles read as they are, 68).
// Features up to which the rows of a tile lie within the 32-bit offsets that its loads use.
constexpr int64_t kFourMostWidth = (int64_t)1 << 22;

int64_t four_tiles(int64_t N, int64_t M, int64_t rows, int64_t cols) { return (N + rows - 1) / rows * ((M + cols - 1) / cols); }

// The tile of a product. The kernel for few rows reads the operands straight into registers and is bound
// by a CU's reads, about 28 KB a us: the smallest of its tiles whose workgroups are one a CU at most. In
// us, bf16 rows, by 16 x 16, 16 x 32, 32 x 32, 32 x 64 and by tiles of 64 through LDS:
//    64 x 4096 x 1024   8.4  10.2  14.4  18.3  21.5      128 x 4096 x 4096   45  32  27  19.0  22.2
//    64 x 4096 x 4096   25   17.6  14.7  18.5  21.9      128 x 2048 x 8192   46  33  29  20.9  13.8
// Of fp16 rows 32 x 64 does not fit the registers; up to 16 rows take 16 x 32 at any number of columns
// (1 x 1024 x 32768: 8.5, by 64 10.9). Rows in 4 bits go through LDS once 16 x 32 is too small (64 x
// 4096 x 4096: 17.5, 13.9, 10.9 by the first three, 8.7 by 64; 1 x 1024 x 32768 7.3, 7.6, 8.2, 6.0).
// Through LDS a tile is 64 while two a CU hold all (by 64, 128, 256 in bf16: 512 x 4096 x 4096 36, 42, 85;
// 1024 x 4096 x 4096 51, 46, 85; in 4 bits 12.8, 14.6, 28.7 and 22.1, 17.8, 30.8; fp16 512 x 2048 x 4096 21,
// 26, 56), and 256 where that fills three CUs in four (2048 x 2048 x 8192 104, 70, 60; 42.6, 31.9, 27.0),
// or 192 x 256 where that needs no more rounds of the CUs and fills them better (2011 x 1024 x 5625 by
// 128, 192, 256 36.9, 33.9, 37.5; 6000 x 1024 x 4096 56, 53, 59; 12000 x 1024 x 1024 32.7, 27.7, 30.7),
// unless a larger tile is too much padding (bf16 60000 x 1024 x 64 23, 24, 30; 100000 x 512 x 130 41, 48, 50;
// 100000 x 512 x 300 66, 62, 83; 130 x 1024 x 32768 25, 21, 29).
som::FourTile four_tile(int64_t N, int64_t K, int64_t M, bool packed, bool bf16)
{
    if (K > kFourMostWidth) return N <= 16 ? som::kFour16x32 : som::kFour32x32;
    if (four_tiles(N, M, 16, 16) <= 256) return som::kFour16x16;
    if (four_tiles(N, M, 16, 32) <= 256 || (!packed && N <= 16)) return som::kFour16x32;
    if (!packed && four_tiles(N, M, 32, 32) <= 256) return som::kFour32x32;
    if (!packed && bf16 && four_tiles(N, M, 32, 64) <= 256) return som::kFour32x64;
    const int64_t by64 = four_tiles(N, M, 64, 64), by128 = four_tiles(N, M, 128, 128), by256 = four_tiles(N, M, 256, 256);
    const int64_t by192 = four_tiles(N, M, 192, 256), rounds = (by256 + 255) / 256;
    if (by192 <= rounds * 256 && by192 >= rounds * 218 && by192 * 3 <= by128 + by128 / 8) return som::kFour192x256;
    if (by256 >= 192 && by256 * 4 <= by128 + by128 / 8) return som::kFour256;
    return by64 <= 512 || by128 * 3 > by64 ? som::kFour64 : som::kFour128;
}

bool few_rows(som::FourTile t) { return t <= som::kFour32x64; }

FourLayout four_layout(int64_t N, int64_t K, int64_t M, bool packed, bool bf16)
{
    FourLayout L{};
    L.tile = four_tile(N, K, M, packed, bf16);
    if (few_rows(L.tile)) return L;
    const int64_t row = som::four_width(K) * 2, most = kFourStrip / row / 256 * 256;
    L.strip = packed || N < most ? N : most;  // 0: rows that long are not copied
    const bool ragged = som::four_blocks(K) % 16 != 0;
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t p = at;
        at += align256((size_t)bytes);
        return p;
    };
    L.ws = take(ragged ? M * som::four_pitch(K) : 0);
    L.xs = take(ragged && packed ? N * som::four_pitch(K) : 0);
    L.x = take(packed ? 0 : L.strip * row);
    L.total = at;
    return L;
}

}  // namespace

extern "C" {

som_status som_layer_norm(int32_t type, const void *X, int64_t ldx, const void *weight, const void *bias,
                          int32_t weight_type, double eps, void *Y, int64_t ldy, int32_t y_type, double *stats,
                          int64_t N, int64_t D, void *stream)
{
    const char *who = "som_layer_norm";
    if (const char *what = norm_types(type, y_type, weight_type)) return bad(who, what);
    if (!rows_ok(N) || !width_ok(D)) return bad(who, "need 0 <= N < 2^30, 1 <= D < 2^20");
    if (!(eps >= (double)FLT_MIN) || std::isinf(eps)) return bad(who, "eps must be at least 2^-126 and finite");
    if (N == 0) return ok();
    if (!X || !Y) return bad(who, kNull);
    if (ldx < D || ldy < D) return bad(who, kStride);
    if (odd(X, type) || odd(Y, y_type) || odd(weight, weight_type) || odd(bias, weight_type) || off(stats, 8))
        return bad(who, kNotAligned);
    som::NormArgs a{};
    a.x = X, a.ldx = ldx, a.weight = weight, a.bias = bias, a.weights_f32 = weight_type == SOM_F32;
    a.eps = eps, a.y = Y, a.ldy = ldy, a.stats = stats, a.N = N, a.D = (int32_t)D;
    return done(som::launch_norm_rows(type, y_type, a, static_cast<hipStream_t>(stream)), who);
}

size_t som_layer_norm_bwd_workspace_bytes(int64_t N, int64_t D)
{
    if (!rows_ok(N) || !width_ok(D)) return 0;
    return align256((size_t)som::norm_parts(N, false) * 2 * (size_t)D * 4) + align256((size_t)N * 8);
}

som_status som_layer_norm_bwd(int32_t type, const void *X, int64_t ldx, const void *weight, int32_t weight_type,
                              const void *dY, int64_t lddy, int32_t y_type, const double *stats, const void *add,
                              int64_t ldadd, void *dX, int64_t lddx, void *dweight, void *dbias, int64_t N, int64_t D,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "som_layer_norm_bwd";
    if (const char *what = norm_types(type, y_type, weight_type)) return bad(who, what);
    if (!rows_ok(N) || !width_ok(D)) return bad(who, "need 0 <= N < 2^30, 1 <= D < 2^20");
    if (N > 0 && (!X || !dY || !stats)) return bad(who, kNull);
    if (ldx < D || lddy < D || (add && ldadd < D) || (dX && lddx < D)) return bad(who, kStride);
    if (odd(X, type) || odd(dY, y_type) || odd(weight, weight_type) || off(stats, 8) || odd(add, type) || odd(dX, type) ||
        odd(dweight, weight_type) || odd(dbias, weight_type))
        return bad(who, kNotAligned);
    const som_status st = check_workspace(who, workspace, workspace_bytes, som_layer_norm_bwd_workspace_bytes(N, D));
    if (st != SOM_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool sums = dweight || dbias;
    som::NormArgs a{};
    a.x = X, a.ldx = ldx, a.weight = weight, a.weights_f32 = weight_type == SOM_F32;
    a.y = const_cast<void *>(dY), a.ldy = lddy, a.stats = const_cast<double *>(stats), a.N = N, a.D = (int32_t)D;
    a.add = add, a.lda = ldadd, a.dx = dX, a.lddx = lddx;
    const int64_t vectors = (D * size_of(type) + 15) / 16;
    const bool whole = N > 0 && vectors <= 2048 && N * som::norm_grad_threads(vectors) <= 2 * 512;
    a.n_parts = whole ? 1 : som::norm_parts(N, vectors > 1024);
    a.part_rows = (N + a.n_parts - 1) / a.n_parts;
    if (whole) a.dweight = dweight, a.dbias = dbias;
    a.parts = sums && !whole ? static_cast<float *>(workspace) : nullptr;
    a.means = reinterpret_cast<float *>(static_cast<char *>(workspace) + align256((size_t)a.n_parts * 2 * (size_t)D * 4));
    if (N > 0 && (dX || sums)) {
        const hipError_t e = som::launch_norm_grad(type, y_type, a, s);
        if (e != hipSuccess) return done(e, who);
    }
    if (!sums || whole) return ok();
    return done(som::launch_norm_sums(a.parts, N > 0 ? a.n_parts : 0, a.D, dweight, dbias, weight_type, s), who);
}

som_status som_adamw(const som_adamw_tensor *tensors, int64_t count, const som_adamw_config *config, void *stream)
{
    const char *who = "som_adamw";
    if (!config) return bad(who, kNull);
    const som_adamw_config &c = *config;
    if (c.bits != 32 && c.bits != 8) return bad(who, "bits must be 32 or 8");
    if (!(c.lr >= 0) || std::isinf(c.lr) || !(c.weight_decay >= 0) || std::isinf(c.weight_decay))
        return bad(who, "lr and weight_decay must be finite and not negative");
    if (!(c.beta1 >= 0 && c.beta1 < 1) || !(c.beta2 >= 0 && c.beta2 < 1)) return bad(who, "beta1 and beta2 must be in [0, 1)");
    if (!(c.eps >= (double)FLT_MIN) || c.eps > (double)FLT_MAX) return bad(who, "eps must be at least 2^-126 and finite");
    if (!(std::fabs(c.grad_scale) <= (double)FLT_MAX)) return bad(who, "grad_scale must be finite");
    if (c.step < 1 || c.step > INT32_MAX) return bad(who, "step must be 1 ... 2^31 - 1");
    if (c.reserved[0] || c.reserved[1] || c.reserved[2] || c.reserved[3]) return bad(who, "reserved fields must be zero");
    if (off(c.lr_at, 4) || off(c.step_at, 4) || off(c.norm, 4)) return bad(who, kNotAligned);
    const bool bits8 = c.bits == 8;
    const som_status st = steps_ok(who, tensors, count, bits8, true);
    if (st != SOM_OK) return st;
    som::AdamwArgs a{};
    a.lr = c.lr, a.beta1 = c.beta1, a.beta2 = c.beta2, a.weight_decay = c.weight_decay;
    a.rates.down = c.eps > 0x1p100 ? 0x1p-8f : 1.0f;
    a.rates.set(c.lr, c.beta1, c.beta2, c.weight_decay, (uint32_t)c.step);
    a.rates.eps = (float)c.eps * a.rates.down, a.rates.grad = (float)c.grad_scale;
    a.seed = c.seed, a.lr_at = c.lr_at, a.step_at = c.step_at, a.norm = c.norm;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return done(over_tables(tensors, count, bits8, [&](som::AdamwTable &t, int64_t) { return som::launch_adamw(t, bits8, a, s); }), who);
}

som_status som_adamw_values(const som_adamw_tensor *tensors, int64_t count, float *const *m_out, float *const *v_out,
                            void *stream)
{
    const char *who = "som_adamw_values";
    const som_status st = steps_ok(who, tensors, count, true, false);
    if (st != SOM_OK) return st;
    if (count > 0 && (!m_out || !v_out)) return bad(who, kNull);
    for (int64_t i = 0; i < count; ++i) {
        if (tensors[i].size > 0 && (!m_out[i] || !v_out[i])) return bad(who, kNull);
        if (odd(m_out[i], SOM_F32) || odd(v_out[i], SOM_F32)) return bad(who, kNotAligned);
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const auto launch = [&](som::AdamwTable &t, int64_t end) {
        for (int j = 0; j < t.count; ++j) {
            const int64_t i = end - t.count + j;
            t.param[j] = m_out[i], t.master[j] = v_out[i];
        }
        return som::launch_adamw_values(t, s);
    };
    return done(over_tables(tensors, count, false, launch), who);
}

static const char *mx4_arguments(int32_t type, const void *x, int64_t ldx, int32_t columns, const void *codes,
                                 const void *scales, int64_t n, int64_t K)
{
    if (!any_type(type)) return "type must be SOM_F32, SOM_F16 or SOM_BF16";
    if (columns != 0 && columns != 1) return "columns must be 0 or 1";
    if (!rows_ok(n) || !dim_ok(K)) return "need 0 <= n, 1 <= K, both below 2^30";
    if (n == 0) return nullptr;
    if (!x || !codes || !scales) return kNull;
    if (ldx < (columns ? n : K)) return kStride;
    if (odd(x, type)) return kNotAligned;
    if (off(codes, 16)) return "codes must be 16-byte aligned";
    return nullptr;
}

som_status som_mx4_quantise(int32_t type, const void *X, int64_t ldx, int32_t columns, uint8_t *codes, uint8_t *scales,
                            int64_t n, int64_t K, void *stream)
{
    const char *who = "som_mx4_quantise";
    if (const char *what = mx4_arguments(type, X, ldx, columns, codes, scales, n, K)) return bad(who, what);
    if (n == 0) return ok();
    som::FourArgs a{X, ldx, codes, scales, n, K};
    return done(som::launch_mx4_quantise(type, columns != 0, a, static_cast<hipStream_t>(stream)), who);
}

som_status som_mx4_values(int32_t type, const uint8_t *codes, const uint8_t *scales, int32_t columns, void *Y,
                          int64_t ldy, int64_t n, int64_t K, void *stream)
{
    const char *who = "som_mx4_values";
    if (const char *what = mx4_arguments(type, Y, ldy, columns, codes, scales, n, K)) return bad(who, what);
    if (n == 0) return ok();
    som::FourArgs a{nullptr, 0, const_cast<uint8_t *>(codes), const_cast<uint8_t *>(scales), n, K};
    return done(som::launch_mx4_values(type, columns != 0, a, Y, ldy, static_cast<hipStream_t>(stream)), who);
}

size_t som_mx4_linear_workspace_bytes(int64_t N, int64_t K, int64_t M, int32_t packed)
{
    if (product_sizes(N, K, M) || (packed != 0 && packed != 1)) return 0;
    const size_t a = four_layout(N, K, M, packed == 1, true).total, b = four_layout(N, K, M, packed == 1, false).total;
    return a > b ? a : b;  // of either type
}

som_status som_mx4_linear(int32_t type, const void *X, int64_t ldx, const uint8_t *x_scales, const uint8_t *w_codes,
                          const uint8_t *w_scales, const void *bias, int32_t bias_type, int32_t act,
                          const void *residual, int64_t ldr, void *Y, int64_t ldy, int32_t y_type, int64_t N, int64_t K,
                          int64_t M, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "som_mx4_linear";
    if (!half_type(type)) return bad(who, "type must be SOM_F16 or SOM_BF16");
    if (const char *what = product_sizes(N, K, M)) return bad(who, what);
    if (act < SOM_ACT_NONE || act > SOM_ACT_SILU) return bad(who, "unknown activation");
    if (y_type != SOM_F32 && y_type != type) return bad(who, "y_type must be SOM_F32 or type");
    if (bias && bias_type != SOM_F32 && bias_type != type) return bad(who, "bias_type must be SOM_F32 or type");
    if (N == 0) return ok();
    if (!X || !w_codes || !w_scales || !Y) return bad(who, kNull);
    if ((!x_scales && ldx < K) || ldy < M || (residual && ldr < M)) return bad(who, kStride);
    if (off(w_codes, 16) || (x_scales && off(X, 16))) return bad(who, "codes must be 16-byte aligned");
    if ((!x_scales && odd(X, type)) || odd(Y, y_type) || odd(residual, type) || (bias && odd(bias, bias_type)))
        return bad(who, kNotAligned);
    const som_status st = check_workspace(who, workspace, workspace_bytes,
                                          som_mx4_linear_workspace_bytes(N, K, M, x_scales ? 1 : 0));
    if (st != SOM_OK) return st;
    som::FourProduct p{};
    p.x = X, p.ldx = ldx, p.x_scales = x_scales, p.w = w_codes, p.w_scales = w_scales;
    p.bias = bias, p.bias_f32 = bias_type == SOM_F32, p.act = act, p.res = residual, p.ldr = ldr;
    p.y = Y, p.ldy = ldy, p.y_f32 = y_type == SOM_F32, p.N = N, p.K = p.width = K, p.M = M;
    const bool bf16 = type == SOM_BF16, packed = x_scales != nullptr;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const FourLayout L = four_layout(N, K, M, packed, bf16);
    const bool ragged = som::four_blocks(K) % 16 != 0;
    const bool whole = packed || (!off(X, 16) && ldx % 8 == 0 && ldx <= kFourMostWidth && K % 64 == 0);
    // Tiles take rows of scales that start on 16 bytes, and whole lines of the rows, or a copy of them.
    if (few_rows(L.tile) || (!ragged && (off(w_scales, 16) || off(x_scales, 16))) || (!whole && L.strip == 0))
        return done(som::launch_mx4_few(bf16, few_rows(L.tile) ? L.tile : som::kFour32x32, p, s), who);
    char *b = static_cast<char *>(workspace);
    p.x_pitch = p.w_pitch = som::four_pitch(K);
    if (ragged) {  // in every call: 2048 x 768 x 4096 in 4 bits takes 17.7 us, of 1024 features, without these copies, 11.7
        uint8_t *ws = reinterpret_cast<uint8_t *>(b + L.ws), *xs = reinterpret_cast<uint8_t *>(b + L.xs);
        hipError_t e = som::launch_pad_scales(w_scales, M, K, ws, s);
        if (e == hipSuccess && packed) e = som::launch_pad_scales(x_scales, N, K, xs, s);
        if (e != hipSuccess) return done(e, who);
        p.w_scales = ws;
        if (packed) p.x_scales = xs;
    }
    if (packed) return done(som::launch_mx4_packed(bf16, L.tile, p, s), who);
    if (whole) return done(som::launch_mx4_half(bf16, L.tile, p, s), who);
    const int64_t width = som::four_width(K);
    for (int64_t n = 0; n < N; n += L.strip) {
        som::FourProduct q = p;
        q.N = N - n < L.strip ? N - n : L.strip;
        q.x = b + L.x, q.ldx = width, q.width = width;
        q.res = residual ? static_cast<const char *>(residual) + n * ldr * 2 : nullptr;
        q.y = static_cast<char *>(Y) + n * ldy * size_of(y_type);
        hipError_t e = som::launch_pad_rows(static_cast<const char *>(X) + n * ldx * 2, ldx, q.N, K, b + L.x, s);
        if (e == hipSuccess) e = som::launch_mx4_half(bf16, L.tile, q, s);
        if (e != hipSuccess) return done(e, who);
    }
    return ok();
}

}  // extern "C"
