// dense_rules.cpp -- the host's rules on the grids of the dense products (som_dense.h), for the tests.
#include "../../paper_2608_24067_amd/csrc/som_dense.h"

extern "C" {
int32_t height(int32_t tile) { return som::tile_rows(static_cast<som::TileSize>(tile)); }

// Rows of tiles that a grouped product of P pairs and E experts by tiles of `tile` is launched with,
// the plan laid out for `plan`; split: tiles that cover one tile row.
int64_t launched(int64_t P, int32_t E, int32_t plan, int32_t tile, int32_t *split)
{
    som::Product p{};
    p.M = P;
    p.groups = E;
    p.tile_height = som::tile_rows(static_cast<som::TileSize>(plan));
    p.split = *split = som::tiles_in_row(static_cast<som::TileSize>(plan), static_cast<som::TileSize>(tile));
    return som::launch_tile_rows(p, static_cast<som::TileSize>(tile));
}

// The grid of a launch of `blocks` workgroups; returns the number of the last one in it.
int64_t grid(int64_t blocks, int64_t *x, int64_t *y)
{
    const dim3 g = som::grid_of(blocks);
    *x = g.x;
    *y = g.y;
    return (int64_t)(g.y - 1) * som::kBlocksAlongX + g.x - 1;  // block_number there
}
}
