// som_mm_tn.hip -- A's columns times B's columns, the reduction over the rows of both (weights'
// gradients), with the column sums of B (biases' gradients).

#include "som_mm.h"

namespace som {
namespace {

template <typename T> hipError_t pick(const Product &p, hipStream_t st)
{
    using namespace mm;
    const int64_t g = p.groups ? p.groups : 1;
    auto rows = [&](int bm) { return (p.M + bm - 1) / bm * g; };
    if (!chunked(kTN, p)) return launch<T, kTN, kGrad, Mid, false>(p, rows(Mid::BM), st);
    const int64_t large = rows(Large::BM) * ((p.N + Large::BN - 1) / Large::BN);
    return large >= 256 ? launch<T, kTN, kGrad, Large, true>(p, rows(Large::BM), st)
                        : launch<T, kTN, kGrad, Mid, true>(p, rows(Mid::BM), st);
}

}  // namespace

hipError_t launch_tn(bool bf16, const Product &p, hipStream_t st)
{
    if (p.M <= 0 || p.N <= 0) return hipSuccess;
    return bf16 ? pick<__bf16>(p, st) : pick<_Float16>(p, st);
}

}  // namespace som
