// linear_tiles.h -- the tile shapes of the linear products and the dispatch
// over them.  Included by the linear_*.hip units.
#pragma once
#include "linear_kern.h"

namespace mxc {

// The shapes that linear.hip's plan chooses among (LIN_TILE_*).
template <int FA, int FB, int OP>
int linear_launch_op(const LinArgs& a, int tile, hipStream_t s) {
    if constexpr (OP != LIN_WGRAD) {
        if (tile == LIN_TILE_ROWS32) return linear_launch<FA, FB, OP, LinTile<1, 1, 1, 1, 8, 2, 4>>(a, s);
        if (tile == LIN_TILE_ROWS64) return linear_launch<FA, FB, OP, LinTile<1, 2, 1, 1, 8, 2, 3>>(a, s);
    }
    if (tile == LIN_TILE_64) return linear_launch<FA, FB, OP, LinTile<1, 1, 2, 2, 1, 4, 4>>(a, s);
    if (tile == LIN_TILE_128) return linear_launch<FA, FB, OP, LinTile<2, 2, 2, 2, 1, 4, 4>>(a, s);
    return MXC_ERR_SHAPE;
}

template <int FA, int FB>
int linear_launch_fmt(int op, const LinArgs& a, int tile, hipStream_t s) {
    if (op == LIN_FWD) return linear_launch_op<FA, FB, LIN_FWD>(a, tile, s);
    if (op == LIN_DGRAD) return linear_launch_op<FA, FB, LIN_DGRAD>(a, tile, s);
    return linear_launch_op<FA, FB, LIN_WGRAD>(a, tile, s);
}

}  // namespace mxc
