// linear_e2m1.hip -- the linear products on MXFP4 operands.
#include "linear_tiles.h"

namespace mxc {

int launch_linear_e2m1(int op, const LinArgs& a, int tile, hipStream_t s) {
    return linear_launch_fmt<MXC_E2M1, MXC_E2M1>(op, a, tile, s);
}

}  // namespace mxc
