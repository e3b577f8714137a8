// som_mm_nt.hip -- A's rows times B's rows: the reduction runs along both.

#include "som_mm.h"

namespace som {
namespace {

template <typename T, Epilogue E> hipError_t pick(TileSize t, const Product &p, hipStream_t st)
{
    using namespace mm;
    const int64_t rows = launch_tile_rows(p, t);
    const bool async = chunked(kNT, p);
    if (t == kTileLarge) return async ? launch<T, kNT, E, Large, true>(p, rows, st) : hipErrorInvalidValue;
    if (t == kTileMid)
        return async ? launch<T, kNT, E, Mid, true>(p, rows, st) : launch<T, kNT, E, Mid, false>(p, rows, st);
    return async ? launch<T, kNT, E, Small, true>(p, rows, st) : launch<T, kNT, E, Small, false>(p, rows, st);
}

template <Epilogue E> hipError_t typed(bool bf16, TileSize t, const Product &p, hipStream_t st)
{
    return bf16 ? pick<__bf16, E>(t, p, st) : pick<_Float16, E>(t, p, st);
}

}  // namespace

hipError_t launch_nt(bool bf16, Epilogue e, TileSize t, const Product &p, hipStream_t st)
{
    if (p.M <= 0 || p.N <= 0) return hipSuccess;
    switch (e) {
    case kLinear: return typed<kLinear>(bf16, t, p, st);
    case kPairs: return typed<kPairs>(bf16, t, p, st);
    case kSlope: return typed<kSlope>(bf16, t, p, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace som
