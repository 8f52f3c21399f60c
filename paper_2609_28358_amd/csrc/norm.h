// norm.h -- arguments of the residual-norm kernels (norm.hip), shared with the
// host-side checks of the C ABI.
#pragma once
#include "mx_internal.h"

namespace mxc {

constexpr int NORM_MAX_DIM = 8192;

// Threads that share a row, and the values of it that each holds: 8, so that
// four waves a SIMD fit, but 16 for the longest rows (a row of 8192 on 1024
// threads of 8 ran at 3.3, on 512 of 16 at 3.8 TB/s forward).
inline int norm_vals(int d) { return d <= 4096 ? 8 : 16; }
inline int norm_tpr(int d) {
    int t = 64;
    while (t * norm_vals(d) < d) t *= 2;
    return t;
}
// rows a workgroup takes at a time: forward workgroups are a row's threads (at
// least 256), backward ones 512, for fewer partial sums
inline int norm_fwd_rows(int d) { return norm_tpr(d) == 64 ? 4 : 1; }
inline int norm_bwd_rows(int d) { return 512 / norm_tpr(d); }
// Workgroups, each with a run of rows: what the CUs hold at once (16 waves a CU,
// by registers), so that no part of the grid is left for a second round;
// backward it is also the number of partial column sums.
inline int norm_fwd_runs(int d) { return norm_tpr(d) == 64 ? 1024 : 256 * 16 / (norm_tpr(d) / 64); }
inline int norm_runs(int d) { return norm_vals(d) == 8 ? 512 : 256; }

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
    float* p_pre;                      // partial column sums [runs][d]: of du hh,
    float* p_c;                        // of dX yh, for runs inside one gate's rows;
    float* p_post;                     // else dw_post's, of whole gates,
    float* p_gate;                     // and dgate itself
    long long rows, gates, gate_rows, run, runs, runs_per_gate, gates_per_run;
    int d;
    bool nt;                           // non-temporal stores of the results (norm.hip, past())
    float scale, eps, inv_d;
};

int launch_norm_fwd(NormArgs a, bool bf16, hipStream_t s);
size_t norm_bwd_workspace(long long rows, int d, long long gates, bool gate, bool post, bool pre);
int launch_norm_bwd(NormArgs a, bool bf16, float* dw_pre, float* dw_post, float* dgate, void* ws, hipStream_t s);

}  // namespace mxc
