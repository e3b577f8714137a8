// som_mm_nn.hip -- A's rows times B, both as stored (weights feature-major: a row holds one feature).

#include "som_mm.h"

namespace som {
namespace {

template <typename T, Epilogue E> hipError_t pick(TileSize t, const Product &p, hipStream_t st)
{
    using namespace mm;
    const int64_t rows = launch_tile_rows(p, t);
    const bool async = chunked(kNN, p);
    if (t == kTileLarge) return async ? launch<T, kNN, E, Large, true>(p, rows, st) : hipErrorInvalidValue;
    if (t == kTileMid)
        return async ? launch<T, kNN, E, Mid, true>(p, rows, st) : launch<T, kNN, E, Mid, false>(p, rows, st);
    return async ? launch<T, kNN, E, Small, true>(p, rows, st) : launch<T, kNN, E, Small, false>(p, rows, st);
}

template <Epilogue E> hipError_t typed(bool bf16, TileSize t, const Product &p, hipStream_t st)
{
    return bf16 ? pick<__bf16, E>(t, p, st) : pick<_Float16, E>(t, p, st);
}

}  // namespace

hipError_t launch_nn(bool bf16, Epilogue e, TileSize t, const Product &p, hipStream_t st)
{
    if (p.M <= 0 || p.N <= 0) return hipSuccess;
    switch (e) {
    case kLinear: return typed<kLinear>(bf16, t, p, st);
    case kInner: return typed<kInner>(bf16, t, p, st);
    case kPairs: return typed<kPairs>(bf16, t, p, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace som
