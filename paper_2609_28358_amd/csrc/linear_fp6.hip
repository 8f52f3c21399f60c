// linear_fp6.hip -- the linear products with FP6 operands: E2M3 alone, and FP4 with E3M2 activations (MicroQonv+).
// fa: the operand whose rows are the output's columns (forward W, input gradient W, weight gradient X).
#include "linear_tiles.h"

namespace mxc {

int launch_linear_fp6(int op, int fa, int fb, const LinArgs& a, int tile, hipStream_t s) {
    if (fa == MXC_E2M3) return linear_launch_fmt<MXC_E2M3, MXC_E2M3>(op, a, tile, s);
    // W in FP4, X or dZ in E3M2; the weight gradient has them the other way round
    if (op == LIN_FWD) return linear_launch_op<MXC_E2M1, MXC_E3M2, LIN_FWD>(a, tile, s);
    if (op == LIN_DGRAD) return linear_launch_op<MXC_E2M1, MXC_E3M2, LIN_DGRAD>(a, tile, s);
    return linear_launch_op<MXC_E3M2, MXC_E2M1, LIN_WGRAD>(a, tile, s);
}

}  // namespace mxc
