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
// Larger tiles read less, smaller ones fill more CUs.  Measured on both sides of
// each limit (forward, us, MXFP8 / MXFP4; rows x outs x ins):
//   32 rows or fewer, 64 or fewer: one tile takes them all and its waves share the
//     contraction.  32 x 4096 x 4096 7.9 / 5.9 against 18.7 / 10.6 by 64 x 64
//     tiles, 64 x 4096 x 4096 10.0 / 6.9 against 18.8 / 10.6;
//   two 256 x 128 tiles a CU: 4096 x 4096 x 1024 42.9 / 26.4 against 44.3 / 26.8
//     by 128 x 128 ones; with one a CU (2048 x 4096 x 1024) 27.2 / 18.6 against
//     24.3 / 13.9;
//   one 128 x 128 tile a CU: 2048 x 2048 x 1024 15.4 / 9.6 against 17.8 / 10.6 by
//     64 x 64 ones; half as many (1024 x 2048 x 1024) 13.9 / 9.6 against 10.7 / 7.2;
//   at most one 64 x 64 tile a CU and 40 blocks to contract: its waves share the
//     contraction, two to a SIMD.  128 x 8192 x 8192 27.5 / 14.6 against 40.3 /
//     18.5 by four waves with a quarter of the tile each, 1024 x 544 x 1504 8.9 /
//     6.8 against 9.7 / 6.7; 800 x 1120 x 1024 7.9 / 6.4 against 7.9 / 6.0.
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
    // least.  The join is a launch of its own, about 4 us of the host.  On the GPU
    // (forward, MXFP8 / MXFP4, rows x outs x ins): 100 x 1000 x 8192 whole 21.3 /
    // 12.4, split 11.9 / 9.4 us, x 4096 12.9 / 8.5 and 10.8 / 8.3; 8 x 1000 x 16384
    // 16.9 / 10.9 and 10.0 / 8.1, x 8192 10.4 / 7.3 and 8.0 / 6.9.  (Splitting
    // grids of one round in two did not pay: both gradients of 8192 x 4096 x 1024,
    // bf16 dX, MXFP4 57.7 us whole and 91.2 split, MXFP8 149 and 179.)
    const long long t = (long long)q.ta * q.tb;
    const int units = (ncb + 15) / 16;
    const bool rows = q.tile == LIN_TILE_ROWS32 || q.tile == LIN_TILE_ROWS64;
    const int n = t < 256 && units >= (rows ? 32 : 16) ? std::max(1, (int)std::min<long long>(256 / t, units / 4)) : 1;
    q.span = (units + n - 1) / n * 16;
    q.nsplit = (ncb + q.span - 1) / q.span;
    if (q.tile == LIN_TILE_64 && t * q.nsplit <= 256 && std::min(ncb, q.span) >= 40) q.tile = LIN_TILE_64K;
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

bool linear_fits(int op, int nrows, int ncols) {
    const long long tiles = (long long)((lin_blocks(ncols) + 7) / 8) * ((lin_blocks(nrows) + 3) / 4);
    return tiles <= (op == LIN_WGRAD ? 1 << 22 : 1 << 23);
}

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
    // column sums: up to four workgroups a column block, as many as there is room
    // for beside the tiles (one of the shared-contraction tiles a CU, two of the
    // others); where there is none, four short ones delay the tiles least (MXFP8
    // 8192 x 1024 x 1024 26 us, 39 with one), but past 64 blocks one (16384 x 4096 x
    // 1024 132 us, 188 with four)
    const long long room = (q.tile == LIN_TILE_64K ? 256 : 512) - tiles;
    p.sumsplit = room >= nrb ? (room >= 4 * nrb ? 2 : room >= 2 * nrb ? 1 : 0) : nrb <= 64 ? 2 : 0;
    p.nsum = colsum ? ((nrb << p.sumsplit) + 7) / 8 * 8 : 0;
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
