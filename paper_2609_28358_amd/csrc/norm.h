// norm.h -- arguments of the residual-norm kernels (norm.hip), shared with the
// host-side checks of the C ABI.
#pragma once
#include "mx_internal.h"

namespace mxc {

constexpr int NORM_VALS = 16;          // values of a row a thread holds
constexpr int NORM_MAX_DIM = 8192;
constexpr int NORM_RUNS = 1024;        // backward: workgroups, so partial column sums
constexpr int NORM_FWD_RUNS = 4096;

// threads that share a row
inline int norm_tpr(int d) { return d <= 64 * NORM_VALS ? 64 : d <= 256 * NORM_VALS ? 256 : 512; }

struct NormArgs {
    const void* x;                     // forward X, backward dH
    const void* y;
    void* h;                           // forward written, backward read
    void* u;                           // forward U (written), backward dU (read)
    void* dx;
    void* dy;
    long long ldx, ldy, ldh, ldu, lddx, lddy;
    const float* w_post;
    const float* w_pre;
    const float* gate;                 // [gates][d], gate r / gate_rows for row r
    float* p_pre;                      // partial column sums [runs][d]
    float* p_post;
    float* p_gate;                     // [runs][d], or dgate itself
    long long rows, gates, gate_rows, run, runs, runs_per_gate, gates_per_run;
    int d;
    float scale, eps, inv_d;
};

int launch_norm_fwd(NormArgs a, bool bf16, bool vec, hipStream_t s);
size_t norm_bwd_workspace(long long rows, int d, long long gates, bool gate, bool post, bool pre);
int launch_norm_bwd(NormArgs a, bool bf16, bool vec, float* dw_pre, float* dw_post, float* dgate, void* ws,
                    hipStream_t s);

}  // namespace mxc
