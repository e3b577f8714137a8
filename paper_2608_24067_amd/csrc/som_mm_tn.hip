// som_mm_tn.hip -- A's columns times B's columns, the reduction over the rows of both (weights'
// gradients), with the column sums of B (biases' gradients).

#include "som_mm.h"

namespace som {
namespace {

template <typename T, mm::Mapped MAP> hipError_t pick(const Product &p, hipStream_t st)
{
    using namespace mm;
    const int64_t g = p.groups ? p.groups : 1;
    auto rows = [&](int bm) { return (p.M + bm - 1) / bm * g; };
    if (!chunked(kTN, p)) return launch<T, kTN, kGrad, Mid, false, MAP>(p, rows(Mid::BM), st);
    const int64_t large = rows(Large::BM) * ((p.N + Large::BN - 1) / Large::BN);
    return large >= 200 ? launch<T, kTN, kGrad, Large, true, MAP>(p, rows(Large::BM), st)
                        : launch<T, kTN, kGrad, Mid, true, MAP>(p, rows(Mid::BM), st);
}

template <typename T> hipError_t mapped(const Product &p, hipStream_t st)
{
    if (p.amap && p.bmap) return hipErrorInvalidValue;
    if (p.amap) return pick<T, mm::kMapA>(p, st);
    return p.bmap ? pick<T, mm::kMapB>(p, st) : pick<T, mm::kNoMap>(p, st);
}

}  // namespace

hipError_t launch_tn(bool bf16, const Product &p, hipStream_t st)
{
    if (p.M <= 0 || p.N <= 0) return hipSuccess;
    return bf16 ? mapped<__bf16>(p, st) : mapped<_Float16>(p, st);
}

}  // namespace som
