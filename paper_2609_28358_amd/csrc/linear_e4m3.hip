// linear_e4m3.hip -- the linear products on MXFP8 operands (one translation unit per format group, so that the
// instantiations compile in parallel).
#include "linear_tiles.h"

namespace mxc {

int launch_linear_e4m3(int op, const LinArgs& a, int tile, hipStream_t s) {
    return linear_launch_fmt<MXC_E4M3, MXC_E4M3>(op, a, tile, s);
}

}  // namespace mxc
