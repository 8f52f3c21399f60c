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

// The shapes that linear.hip's plan chooses among (LIN_TILE_*).  FP4 products
// leave time for more LDS reads, so eight waves with smaller parts share a 128 x
// 128 tile (4096 x 1024 x 4096 forward 20.3 -> 19.4, 2048 x 2048 x 1024 10.6 ->
// 9.6 us) and the weight gradient's 256 x 128 one (16384 x 4096 x 4096 180 ->
// 171 us, but forward 218 -> 262); MXFP8, which would decode each code twice as
// often, loses by that (4096 x 1024 x 4096 forward 40.6 -> 43.7).
template <int FA, int FB, int OP>
int linear_launch_op(const LinArgs& a, int tile, hipStream_t s) {
    constexpr int KS = lin_ks<FA, FB>();
    constexpr bool F4 = KS == 4;
    if constexpr (OP != LIN_WGRAD) {
        if (tile == LIN_TILE_ROWS32) return linear_launch<FA, FB, OP, LinTile<1, 1, 1, 1, 8, 2, 4>>(a, s);
        if (tile == LIN_TILE_ROWS64) return linear_launch<FA, FB, OP, LinTile<1, 2, 1, 1, 8, 2, 3>>(a, s);
    }
    using T64 = LinTile<1, 1, 2, 2, 1, 4, F4 ? 4 : 3>;
    using T64K = std::conditional_t<F4, LinTile<2, 1, 1, 2, 4, 2, 4>, LinTile<1, 2, 2, 1, 4, 2, 3>>;
    using T128 = std::conditional_t<F4, LinTile<1, 2, 4, 2, 1, KS, 4>, LinTile<2, 2, 2, 2, 1, KS, 4>>;
    using T256 = std::conditional_t<F4 && OP == LIN_WGRAD, LinTile<2, 2, 4, 2, 1, KS, 3>, LinTile<4, 2, 2, 2, 1, KS, 3>>;
    if (tile == LIN_TILE_64) return linear_launch<FA, FB, OP, T64>(a, s);
    if (tile == LIN_TILE_64K) return linear_launch<FA, FB, OP, T64K>(a, s);
    if (tile == LIN_TILE_128) return linear_launch<FA, FB, OP, T128>(a, s);
    return linear_launch<FA, FB, OP, T256>(a, s);
}

template <int FA, int FB>
int linear_launch_fmt(int op, const LinArgs& a, int tile, hipStream_t s) {
    if (op == LIN_FWD) return linear_launch_op<FA, FB, LIN_FWD>(a, tile, s);
    if (op == LIN_DGRAD) return linear_launch_op<FA, FB, LIN_DGRAD>(a, tile, s);
    return linear_launch_op<FA, FB, LIN_WGRAD>(a, tile, s);
}

}  // namespace mxc
