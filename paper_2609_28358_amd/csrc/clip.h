// clip.h -- limits of the gradient-norm kernels (clip.hip), shared with the
// host-side checks of the C ABI.
#pragma once
#include "mx_internal.h"

namespace mxc {

constexpr int CLIP_TENSORS = 448;      // descriptors of a launch (12.4 KB of kernel arguments)
constexpr int CLIP_PARTS = 2048;       // partial sums of all launches

int launch_grad_clip(int count, const mxc_gtensor* t, bool scale, double max_norm, float* norm, void* ws,
                     hipStream_t s);

}  // namespace mxc
