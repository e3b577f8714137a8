// som_mm_tn.hip -- A's columns times B's columns, the reduction over the rows of both (weights'
// gradients), with the column sums of B (biases' gradients).

#include "som_mm.h"

namespace som {
namespace {

template <typename T, mm::Mapped MAP> hipError_t pick(TileSize t, const Product &p, hipStream_t st)
{
    using namespace mm;
    const int64_t g = p.groups ? p.groups : 1;
    auto rows = [&](int bm) { return (p.M + bm - 1) / bm * g; };
    if (!chunked(kTN, p)) return launch<T, kTN, kGrad, Mid, false, MAP>(p, rows(Mid::BM), st);
    return t == kTileLarge ? launch<T, kTN, kGrad, Large, true, MAP>(p, rows(Large::BM), st)
                           : launch<T, kTN, kGrad, Mid, true, MAP>(p, rows(Mid::BM), st);
}

template <typename T> hipError_t mapped(TileSize t, const Product &p, hipStream_t st)
{
    if (p.amap && p.bmap) return hipErrorInvalidValue;
    if (p.amap) return pick<T, mm::kMapA>(t, p, st);
    return p.bmap ? pick<T, mm::kMapB>(t, p, st) : pick<T, mm::kNoMap>(t, p, st);
}

}  // namespace

hipError_t launch_tn(bool bf16, TileSize t, const Product &p, hipStream_t st)
{
    if (p.M <= 0 || p.N <= 0) return hipSuccess;
    return bf16 ? mapped<__bf16>(t, p, st) : mapped<_Float16>(t, p, st);
}

}  // namespace som
