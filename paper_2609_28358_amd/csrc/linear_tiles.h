// linear_tiles.h -- the tile shapes of the linear products and the dispatch
// over them.  Included by the linear_*.hip units.
#pragma once
#include "linear_kern.h"

namespace mxc {

// Contraction blocks a wave takes from a stage: four for FP4 pairs, two for
// wider elements, whose blocks take 1 KB of LDS (so that the 128 x 128 and the
// 256 x 128 tile leave room for two workgroups on a CU: at four, MXFP8 16384 x
// 4096 x 4096 ran 1.4 times as long on 128 x 128 tiles).
template <int FA, int FB> constexpr int lin_ks() { return FA == MXC_E2M1 && FB == MXC_E2M1 ? 4 : 2; }

// The shapes that linear.hip's plan chooses among (LIN_TILE_*).
template <int FA, int FB, int OP>
int linear_launch_op(const LinArgs& a, int tile, hipStream_t s) {
    constexpr int KS = lin_ks<FA, FB>(), N64 = KS == 4 ? 4 : 3;
    if constexpr (OP != LIN_WGRAD) {
        if (tile == LIN_TILE_ROWS32) return linear_launch<FA, FB, OP, LinTile<1, 1, 1, 1, 8, 2, 4>>(a, s);
        if (tile == LIN_TILE_ROWS64) return linear_launch<FA, FB, OP, LinTile<1, 2, 1, 1, 8, 2, 3>>(a, s);
    }
    if (tile == LIN_TILE_64) return linear_launch<FA, FB, OP, LinTile<1, 1, 2, 2, 1, 4, N64>>(a, s);
    if (tile == LIN_TILE_128) return linear_launch<FA, FB, OP, LinTile<2, 2, 2, 2, 1, KS, 4>>(a, s);
    return linear_launch<FA, FB, OP, LinTile<4, 2, 2, 2, 1, KS, 3>>(a, s);
}

template <int FA, int FB>
int linear_launch_fmt(int op, const LinArgs& a, int tile, hipStream_t s) {
    if (op == LIN_FWD) return linear_launch_op<FA, FB, LIN_FWD>(a, tile, s);
    if (op == LIN_DGRAD) return linear_launch_op<FA, FB, LIN_DGRAD>(a, tile, s);
    return linear_launch_op<FA, FB, LIN_WGRAD>(a, tile, s);
}

}  // namespace mxc
