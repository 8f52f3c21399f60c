// linear.hip -- the plan of a linear product (tile shape, split of the
// contraction), its launch, and the kernel that joins split partial sums.
#include "linear_kern.h"

namespace mxc {
namespace {

struct LinPlan {
    int tile, ra, rb;             // tile shape, in 32-blocks
    int ta, tb, nsplit, span;     // tiles; splits of the contraction, blocks of each
    long long ldw;                // row length of the partial sums
};

// nra, nrb: 32-blocks along the output's columns and rows; ncb: along the
// contraction.  The formats play no part, so neither do they in the workspace.
LinPlan lin_plan(int op, int nra, int nrb, int ncb) {
    LinPlan q;
    auto tiles = [&](int a, int b) { return (long long)((nra + a - 1) / a) * ((nrb + b - 1) / b); };
    if (op != LIN_WGRAD && nrb == 1) { q.tile = LIN_TILE_ROWS32; q.ra = 1; q.rb = 1; }
    else if (op != LIN_WGRAD && nrb == 2) { q.tile = LIN_TILE_ROWS64; q.ra = 1; q.rb = 2; }
    else if (tiles(8, 4) >= 512) { q.tile = LIN_TILE_256; q.ra = 8; q.rb = 4; }
    else if (tiles(4, 4) >= 256) { q.tile = LIN_TILE_128; q.ra = 4; q.rb = 4; }
    else { q.tile = LIN_TILE_64; q.ra = 2; q.rb = 2; }
    q.ta = (nra + q.ra - 1) / q.ra;
    q.tb = (nrb + q.rb - 1) / q.rb;
    // a grid that leaves CUs idle is split along a long contraction, in units of
    // 16 blocks (a whole number of any shape's stages), four of them a split at
    // least.  The join is a launch of its own: 8 rows x 8192 x 1000 take 10.9 us
    // whole and 15.7 split, 8 x 16384 x 1000 16 either way; 100 x 8192 x 1000 take
    // 17 split and 18 whole.  (Splitting grids of one round in two did not pay:
    // 8192 x 4096 x 1024, both gradients, 84 us whole and 96 split.)
    const long long t = (long long)q.ta * q.tb;
    const int units = (ncb + 15) / 16;
    const bool rows = q.tile == LIN_TILE_ROWS32 || q.tile == LIN_TILE_ROWS64;
    const int n = t < 256 && units >= (rows ? 32 : 16) ? std::max(1, (int)std::min<long long>(256 / t, units / 4)) : 1;
    q.span = (units + n - 1) / n * 16;
    q.nsplit = (ncb + q.span - 1) / q.span;
    q.ldw = (long long)nra * 32;
    return q;
}

// out[r][c .. c + 3] = epilogue(sum over the splits, in order).
template <int OP>
__global__ __launch_bounds__(256) void lin_join_kernel(const LinEpi e, const float* __restrict__ part, int nsplit,
                                                       long long ldw, long long quads) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i < quads) {
        const int per = (e.ncols + 3) / 4;
        const int r = (int)(i / per), c = (int)(i - (long long)r * per) * 4;
        const float* p = part + (long long)r * ldw + c;
        const long long step = (long long)e.nrows * ldw;
        float4 v = *(const float4*)p;
        for (int k = 1; k < nsplit; k++) {
            const float4 u = *(const float4*)(p + k * step);
            v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
        lin_epilogue4<OP>(e, r, c, v);
    }
}

int lin_blocks(int n) { return (n + 31) / 32; }

}  // namespace

size_t linear_workspace(int op, int nrows, int ncols, int ncon) {
    const LinPlan q = lin_plan(op, lin_blocks(ncols), lin_blocks(nrows), lin_blocks(ncon));
    if (q.nsplit == 1) return 0;
    return (size_t)q.nsplit * (size_t)nrows * q.ldw * sizeof(float);
}

int launch_linear(int op, int fa, int fb, const LinMat& a, const LinMat& b, int ncon, const LinEpi& e, float* colsum,
                  void* ws, hipStream_t s) {
    const int nra = lin_blocks(e.ncols), nrb = lin_blocks(e.nrows), ncb = lin_blocks(ncon);
    const LinPlan q = lin_plan(op, nra, nrb, ncb);
    const long long tiles = (long long)q.ta * q.tb * q.nsplit;
    if (tiles > (1 << 22)) return MXC_ERR_SHAPE;
    LinArgs p;
    // blocks are stored [row block][column block] of the matrix: along the
    // product's rows where those are the matrix's rows, else along its columns
    const bool ta = op == LIN_FWD, tb = op != LIN_WGRAD;
    p.a = {a.codes, a.scales, nra, ncb, ta ? ncb : 1, ta ? 1 : nra};
    p.b = {b.codes, b.scales, nrb, ncb, tb ? ncb : 1, tb ? 1 : nrb};
    p.e = e;
    p.ta = q.ta; p.tb = q.tb; p.nsplit = q.nsplit; p.span = q.span;
    p.ldw = q.ldw;
    p.part = q.nsplit > 1 ? (float*)ws : nullptr;
    p.colsum = colsum;
    p.nsum = colsum ? (nrb + 7) / 8 * 8 : 0;
    int rc;
    if (fa == MXC_E4M3) rc = launch_linear_e4m3(op, p, q.tile, s);
    else if (fa == MXC_E2M1 && fb == MXC_E2M1) rc = launch_linear_e2m1(op, p, q.tile, s);
    else rc = launch_linear_fp6(op, fa, fb, p, q.tile, s);
    if (rc || q.nsplit == 1) return rc;
    const long long quads = (long long)e.nrows * ((e.ncols + 3) / 4);
    const unsigned grid = (unsigned)((quads + 255) / 256);
    if (op == LIN_FWD) lin_join_kernel<LIN_FWD><<<grid, 256, 0, s>>>(e, p.part, q.nsplit, q.ldw, quads);
    else if (op == LIN_DGRAD) lin_join_kernel<LIN_DGRAD><<<grid, 256, 0, s>>>(e, p.part, q.nsplit, q.ldw, quads);
    else lin_join_kernel<LIN_WGRAD><<<grid, 256, 0, s>>>(e, p.part, q.nsplit, q.ldw, quads);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_HIP;
}

}  // namespace mxc
