// linear_kern.h -- the products of a linear layer on MX matrices: the kernel
// template and its launch, instantiated per format pair in linear_*.hip.
// Included by .hip files only.
//
// An MX matrix of R rows and C columns is an array [ceil(R/32)][ceil(C/32)] of
// 32 x 32 blocks of codes, each block [column][row] (row fastest), with one
// E8M0 scale a block.  The square blocks serve both directions, so the three
// products of a layer (Y = X W^T, dX = dZ W, dW = dZ^T X) read the same stored
// blocks of X [rows][ins], W [outs][ins] and dZ [rows][outs]:
//   operand    product rows   contraction   stored order
//   fwd    W   outs           ins           row fastest: transposed reads
//   fwd    X   rows           ins           transposed reads
//   dgrad  W   ins            outs          contraction fastest: direct reads
//   dgrad  dZ  rows           outs          transposed reads
//   wgrad  X   ins            rows          direct reads
//   wgrad  dZ  outs           rows          direct reads
// The operand whose rows are the output's columns is the MFMA's first (A), so
// a lane's accumulator holds four consecutive output columns of one output
// row and the epilogue moves vectors.
//
// What bounds it (a pass among others on other inputs): large MXFP8 products the
// matrix units and their power (16384 x 4096 x 4096 436 to 446 us on different
// cards, 1.23 to 1.26 PFLOP/s, the matrix cores busy 48% of the cycles at 2.4 GHz; loops of
// the MFMAs alone reach 1.4 PFLOP/s); large MXFP4 ones the bytes of their results,
// stored behind the products (4096 x 4096 x 1024 with SiLU and the pre-activation
// kept 24.5 us, 71 MB at 2.9 TB/s, the matrix cores busy 13%); few rows the weights'
// bytes (24 x 8192 x 8192 MXFP8 13.7 us, 5.0 TB/s); small ones a chain of stages
// behind the launch (1 x 4096 x 1024 MXFP4 4.9 us of the GPU).
#pragma once
#include <atomic>

#include "mx_internal.h"

namespace mxc {

// One operand: blocks along the product's rows and along the contraction, and
// the block strides of both (in blocks).
struct LinOp {
    const uint8_t* codes;
    const uint8_t* scales;
    int nrb, ncb;
    int srow, scon;
};

// The epilogue: out[r][c] for output row r < nrows, column c < ncols.
//   fwd    z = v + bias[c]; pre[r][c] = z; out = fn(z) + res[r][c]
//   dgrad  out = v fn'(z[r][c]) + res[r][c]
// pre doubles as dgrad's z.  nt, ntp: out or pre is stored non-temporally, by its
// bytes and where its rows begin at cache lines (rows that begin elsewhere lose by
// it, 16384 x 300 x 8191 186 -> 241 us).  Measured with other inputs in between,
// plain stores -> non-temporal out, us, and in brackets with the quantization of
// the result behind it; rows x outs x ins, MXFP4 and MXFP8, bf16 results:
//                                  forward with residual         input gradient
//    4 MiB, fp4  2048 x 1024 x 1024  7.6 -> 7.4 (12.4 -> 12.7)     6.9 -> 6.8 (11.2 -> 11.3)
//    8,     fp8  4096 x 1024 x 1024  16.5 -> 16.0 (23.4 -> 23.2)   14.7 -> 13.7 (22.2 -> 21.7)
//   16,     fp4  8192 x 1024 x 1024  16.1 -> 15.9 (26.3 -> 27.1)   13.7 -> 11.5 (24.5 -> 23.2)
//   32,     fp4 16384 x 1024 x 1024  28.2 -> 27.7 (44.8 -> 47.2)   21.4 -> 18.5 (38.8 -> 38.4)
//   32,     fp8  4096 x 4096 x 1024  46.6 -> 45.1 (63.8 -> 66.5)   36.7 -> 34.8 (55.1 -> 57.2)
//   64,     fp4  8192 x 4096 x 1024  51.4 -> 50.6 (82.9 -> 86.2)   36.8 -> 34.8 (69.4 -> 72.1)
//  128,     fp8 16384 x 4096 x 1024  159 -> 157 (227 -> 224)       124 -> 122 (191 -> 198)
// From 32 MiB on the last-level cache still holds a plain result for what reads it
// next, so out is stored so from 4 to 32 MiB (fp32 weight gradients with an update
// behind them: 16 MiB, fp8 47.6 -> 46.9; 64 MiB, fp4 76.9 -> 82.9).  The
// pre-activation, which is read much later, is from 4 MiB on: MXFP4 with SiLU, both
// results at 8 MiB 11.7 -> 9.5 (18.4 -> 17.2), pre alone at 64 MiB 51.2 -> 49.9
// (83.5 -> 82.6) and at 128 MiB 98.2 -> 95.7 (171 -> 162).
struct LinEpi {
    void* out;
    const float* bias;
    const void* res;
    void* pre;
    long long ldo, ldr, ldp;
    int fn, bf16, nt, ntp;
    int nrows, ncols;
};

// A stored matrix.
struct LinMat {
    const uint8_t* codes;
    const uint8_t* scales;
};

struct LinArgs {
    LinOp a, b;
    LinEpi e;
    float* part;          // split contraction: partial sums [split][nrows][ldw], else NULL
    long long ldw;
    float* colsum;        // weight gradient: db, or NULL
    int nsum, sumsplit;   // workgroups in front of the tiles that form it, log2 of those of a column block
    int ta, tb;           // tiles along A's and B's rows
    int nsplit, span;     // splits of the contraction, blocks of each (whole stages)
};

enum { LIN_FWD = 0, LIN_DGRAD = 1, LIN_WGRAD = 2 };

// Tile shapes: blocks a wave holds (MB x NB), waves along A's rows, along B's
// rows and along the contraction, 32-blocks of the contraction a wave takes
// from a stage, and stages in the ring.
template <int MB_, int NB_, int WM_, int WN_, int WK_, int KS_, int NBUF_> struct LinTile {
    static constexpr int MB = MB_, NB = NB_, WM = WM_, WN = WN_, WK = WK_, KS = KS_, NBUF = NBUF_;
    static constexpr int RA = MB * WM, RB = NB * WN, KB = KS * WK, W = WM * WN * WK;
};

// LDS bytes of one block, blocks a 64-lane copy of 16 bytes a lane moves, and
// the source bytes a lane advances (FP6: 12 of a half row, in 16-byte slots)
template <int F> struct LinBlk {
    static constexpr int SRC = 32 * 32 * fmt_bits(F) / 8;
    static constexpr int LDS = fmt_bits(F) == 4 ? 512 : 1024;
    static constexpr int BPI = fmt_bits(F) == 4 ? 2 : 1;
    static constexpr int STEP = fmt_bits(F) == 6 ? 12 : 16;
};

template <int FA, int FB, class T> struct LinLds {
    static constexpr int ABYTES = T::RA * T::KB * LinBlk<FA>::LDS;
    static constexpr int BBYTES = T::RB * T::KB * LinBlk<FB>::LDS;
    static constexpr int NSI = ((T::RA + T::RB) * T::KB + 63) / 64;          // scale copies of a stage
    static constexpr int STAGE = ABYTES + BBYTES + NSI * 256;
    static constexpr int LD = 32 * T::MB + 4;                                // floats of an output row on its way out
    // joining the waves of the contraction, or the waves' output rows
    static constexpr int RED = T::WK > 1 ? T::W * T::MB * T::NB * 4096 : T::W * 32 * LD * 4;
    static constexpr int BYTES = T::NBUF * STAGE > RED ? T::NBUF * STAGE : RED;
};

// tile shapes a launch is asked for: outputs of at most 32 or 64 rows (the
// contraction is shared by a workgroup's waves), 64 x 64 without and with a
// shared contraction, 128 x 128, 256 columns x 128 rows
enum { LIN_TILE_ROWS32, LIN_TILE_ROWS64, LIN_TILE_64, LIN_TILE_64K, LIN_TILE_128, LIN_TILE_256 };

// linear.hip: whether a product's tiles fit a launch (half of a grid's 2^32
// threads: workgroups of 256, up to 512 for the weight gradient), its workspace
// bytes and its launch (nrows x ncols outputs over ncon, formats and matrices in
// the order A, B)
bool linear_fits(int op, int nrows, int ncols);
size_t linear_workspace(int op, int nrows, int ncols, int ncon);
int launch_linear(int op, int fa, int fb, const LinMat& a, const LinMat& b, int ncon, const LinEpi& e, float* colsum,
                  void* ws, hipStream_t s);
// linear_*.hip, by format
int launch_linear_e4m3(int op, const LinArgs& a, int tile, hipStream_t s);
int launch_linear_e2m1(int op, const LinArgs& a, int tile, hipStream_t s);
int launch_linear_fp6(int op, int fa, int fb, const LinArgs& a, int tile, hipStream_t s);

}  // namespace mxc

#if defined(__HIPCC__)
namespace mxc {

static __device__ __attribute__((aligned(16))) uint8_t g_lin_zero[1024];

// A 16-byte copy a lane to LDS from a uniform base and a lane offset: the
// base advances on the scalar unit.
__device__ __forceinline__ void dma16_base(const uint8_t* base, uint32_t off, uint32_t lds) {
    asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}

// ---------------------------------------------------------------- epilogue
// No contraction: every path (vectors, columns, joined splits) gives the same bits.
// ReLU keeps a NaN, and its gradient chooses instead of multiplying by 0 or 1: zero
// where z <= 0, whatever the product, and the product elsewhere.
template <int OP>
__device__ __forceinline__ float lin_value(int fn, float v, float b, float z, float r) {
#pragma clang fp contract(off)
    if constexpr (OP == LIN_FWD) {
        v += b;
        return (fn == MXC_FN_NONE ? v : fn == MXC_FN_RELU ? (v <= 0.0f ? 0.0f : v) : fn_apply_c<MXC_FN_SILU>(v)) + r;
    } else if constexpr (OP == LIN_DGRAD) {
        return (fn == MXC_FN_NONE ? v : fn == MXC_FN_RELU ? (z <= 0.0f ? 0.0f : v) : v * fn_grad_c<MXC_FN_SILU>(z)) + r;
    } else {
        return v;
    }
}

// N consecutive values of a full-precision row, of which `left` are before the
// row's end: one access of N elements at any element's address (global memory
// takes unaligned vectors), or element by element where the row ends inside.
template <int BYTES, int AL> struct __attribute__((packed, aligned(AL))) LinRaw {
    uint32_t w[BYTES / 4];
};
template <bool BF, int N> using LinVec = LinRaw<BF ? 2 * N : 4 * N, BF ? 2 : 4>;
template <bool BF, int N>
__device__ __forceinline__ LinVec<BF, N> lin_get(const void* base, long long i, int left) {
    LinVec<BF, N> u;
    if constexpr (BF) {
        const uint16_t* p = (const uint16_t*)base + i;
        if (left >= N) return *(const LinVec<BF, N>*)p;
#pragma unroll
        for (int k = 0; k < N / 2; k++)
            u.w[k] = (2 * k < left ? p[2 * k] : 0u) | (2 * k + 1 < left ? (uint32_t)p[2 * k + 1] : 0u) << 16;
    } else {
        const uint32_t* p = (const uint32_t*)base + i;
        if (left >= N) return *(const LinVec<BF, N>*)p;
#pragma unroll
        for (int k = 0; k < N; k++) u.w[k] = k < left ? p[k] : 0u;
    }
    return u;
}
template <bool BF, int N>
__device__ __forceinline__ void lin_unpack(const LinVec<BF, N>& u, float* o) {
    if constexpr (BF) {
#pragma unroll
        for (int k = 0; k < N / 2; k++) {
            o[2 * k] = __uint_as_float(u.w[k] << 16);
            o[2 * k + 1] = __uint_as_float(u.w[k] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; k++) o[k] = __uint_as_float(u.w[k]);
    }
}
template <bool BF, int N>
__device__ __forceinline__ void lin_load(const void* base, long long i, int left, float* o) {
    lin_unpack<BF, N>(lin_get<BF, N>(base, i, left), o);
}
// nt: the rows are whole cache lines (LinEpi).
template <bool BF, int N>
__device__ __forceinline__ void lin_store(void* base, long long i, int left, const float* v, bool nt) {
    if constexpr (BF) {
        uint16_t* p = (uint16_t*)base + i;
        if (left >= N) {
            LinRaw<2 * N, 2> u;
#pragma unroll
            for (int k = 0; k < N / 2; k++) u.w[k] = bf16_pack2(v[2 * k], v[2 * k + 1]);
            if (N == 8 && nt) store_nt(p, make_uint4(u.w[0], u.w[1], u.w[N / 2 - 2], u.w[N / 2 - 1]));
            else *(LinRaw<2 * N, 2>*)p = u;
        } else {
#pragma unroll
            for (int k = 0; k < N; k++)
                if (k < left) p[k] = (uint16_t)bf16_bits(v[k]);
        }
    } else {
        float* p = (float*)base + i;
        if (left >= N) {
            LinRaw<4 * N, 4> u;
#pragma unroll
            for (int k = 0; k < N; k++) u.w[k] = __float_as_uint(v[k]);
            if (nt) store_nt(p, make_uint4(u.w[0], u.w[1], u.w[2], u.w[3]));
            else *(LinRaw<4 * N, 4>*)p = u;
        } else {
#pragma unroll
            for (int k = 0; k < N; k++)
                if (k < left) p[k] = v[k];
        }
    }
}

// N consecutive columns c .. of output row r < nrows (those before ncols): the
// values v with what the epilogue reads (z: the pre-activation, s: the
// residual).  All arithmetic is fp32, rounded once where it is stored; the
// activation is applied to the unrounded pre-activation.
template <int OP, bool BF, int N, int FN>
__device__ __forceinline__ void lin_finish(const LinEpi& e, int r, int c, float* v, const float* b, float* z, const float* s) {
    const int left = e.ncols - c;
    if (OP == LIN_FWD && e.pre) {
#pragma unroll
        for (int q = 0; q < N; q++) z[q] = v[q] + b[q];
        lin_store<BF, N>(e.pre, r * e.ldp + c, left, z, e.ntp);
    }
#pragma unroll
    for (int q = 0; q < N; q++) v[q] = lin_value<OP>(FN, v[q], b[q], z[q], s[q]);
    lin_store<BF, N>(e.out, r * e.ldo + c, left, v, e.nt);
}

// body(FnTag) for the epilogue's activation, one uniform choice
template <int OP, class Body>
__device__ __forceinline__ void lin_fn(const LinEpi& e, Body&& body) {
    if (OP == LIN_WGRAD || e.fn == MXC_FN_NONE) body(FnTag<MXC_FN_NONE>{});
    else if (e.fn == MXC_FN_RELU) body(FnTag<MXC_FN_RELU>{});
    else body(FnTag<MXC_FN_SILU>{});
}

// Four columns, where they come one by one (split sums, joined waves).
template <int OP, bool BF>
__device__ __forceinline__ void lin_four(const LinEpi& e, int r, int c, float4 v) {
    const int left = e.ncols - c;
    if (left <= 0) return;
    float a[4] = {v.x, v.y, v.z, v.w}, b[4] = {0, 0, 0, 0}, z[4] = {0, 0, 0, 0}, s[4] = {0, 0, 0, 0};
    if (OP == LIN_FWD && e.bias) lin_load<false, 4>(e.bias, c, left, b);
    if (OP == LIN_DGRAD && e.fn != MXC_FN_NONE) lin_load<BF, 4>(e.pre, r * e.ldp + c, left, z);
    if (OP != LIN_WGRAD && e.res) lin_load<BF, 4>(e.res, r * e.ldr + c, left, s);
    lin_fn<OP>(e, [&](auto fn) { lin_finish<OP, BF, 4, decltype(fn)::fn>(e, r, c, a, b, z, s); });
}
template <int OP>
__device__ __forceinline__ void lin_epilogue4(const LinEpi& e, int r, int c, float4 v) {
    if (OP != LIN_WGRAD && e.bf16) lin_four<OP, true>(e, r, c, v);
    else lin_four<OP, false>(e, r, c, v);
}

// One 32-row block of a wave (rows r0 .. r0 + 31, columns c0 .. c0 + 32 MB -
// 1) on its way out through the wave's LDS rows: 16 bytes a lane, four rows'
// reads in flight (a round trip to memory a batch is what bounded this part).
// park() writes the block to LDS; the first batch's reads are issued before it.
template <int OP, bool BF, int MB, class Park>
__device__ __forceinline__ void lin_rows(const LinEpi& e, int r0, int c0, const float* mine, int lane, Park&& park) {
    constexpr int V = BF ? 8 : 4, LD = 32 * MB + 4;
    constexpr int LPR = 32 * MB / V, RS = 64 / LPR, CNT = 32 / RS, BN = CNT < 4 ? CNT : 4;
    const int row = lane / LPR, col = lane % LPR * V, c = c0 + col;
    // a lane past the last column reads the row's first ones and stores nothing
    const int cc = c < e.ncols ? c : 0, left = e.ncols - cc;
    const bool rd_z = OP == LIN_DGRAD && e.fn != MXC_FN_NONE, rd_s = OP != LIN_WGRAD && e.res;
    LinVec<BF, V> z[BN], s[BN];
    float b[V];
#pragma unroll
    for (int q = 0; q < V; q++) b[q] = 0.0f;
    auto read = [&](int n) {
#pragma unroll
        for (int k = 0; k < BN; k++) {
            const int r = min(r0 + row + (n + k) * RS, e.nrows - 1);
            if (rd_z) z[k] = lin_get<BF, V>(e.pre, r * e.ldp + cc, left);
            if (rd_s) s[k] = lin_get<BF, V>(e.res, r * e.ldr + cc, left);
        }
    };
    read(0);
    if (OP == LIN_FWD && e.bias) {
        lin_load<false, 4>(e.bias, cc, left, b);
        if constexpr (V == 8) lin_load<false, 4>(e.bias, left > 4 ? cc + 4 : cc, left - 4, b + 4);
    }
    park();
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int n = 0; n < CNT; n += BN) {
        if (n) read(n);
        lin_fn<OP>(e, [&](auto fn) {
#pragma unroll
            for (int k = 0; k < BN; k++) {
                const int r = r0 + row + (n + k) * RS;
                float v[V], zf[V], sf[V];
#pragma unroll
                for (int q = 0; q < V; q++) zf[q] = sf[q] = 0.0f;
                if (OP == LIN_DGRAD && decltype(fn)::fn != MXC_FN_NONE) lin_unpack<BF, V>(z[k], zf);
                if (rd_s) lin_unpack<BF, V>(s[k], sf);
#pragma unroll
                for (int q = 0; q < V; q += 4) {
                    const float4 u = *(const float4*)(mine + (row + (n + k) * RS) * LD + col + q);
                    v[q] = u.x; v[q + 1] = u.y; v[q + 2] = u.z; v[q + 3] = u.w;
                }
                if (r < e.nrows && c < e.ncols) lin_finish<OP, BF, V, decltype(fn)::fn>(e, r, c, v, b, zf, sf);
            }
        });
    }
    __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------- fragments
// The fragment (see mfma_mx) of a 32-row block for two contraction blocks at
// p and p + next (LDS).  TR: rows fastest in the block, read transposed;
// otherwise the contraction is fastest and a lane's row is contiguous.
template <int F, bool TR>
__device__ __forceinline__ v8i lin_frag(const uint8_t* p, int next, int lane) {
    v8i o;
    const int h = lane >> 5, i16 = lane & 15, cg = (lane >> 4) & 1;
    if constexpr (TR && F == MXC_E4M3) {
        const uint8_t* q = p + (16 * h + (i16 >> 1)) * 32 + 16 * cg + 8 * (i16 & 1);
#pragma unroll
        for (int kb = 0; kb < 2; kb++)
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                const v2i v = lds_tr8(q + kb * next + hf * 256);
                o[4 * kb + 2 * hf] = v[0];
                o[4 * kb + 2 * hf + 1] = v[1];
            }
    } else if constexpr (TR && F == MXC_E2M1) {
        const uint8_t* q = p + h * next + i16 * 16 + 8 * cg;
#pragma unroll
        for (int hf = 0; hf < 2; hf++) {
            const v2i v = lds_tr4(q + hf * 256);
            o[2 * hf] = v[0];
            o[2 * hf + 1] = v[1];
        }
        o[4] = o[5] = o[6] = o[7] = 0;
    } else if constexpr (TR) {
        const uint8_t* q = p + h * next + i16 * 32 + 16 * cg;
        const v3i lo = lds_tr6(q), hi = lds_tr6(q + 512);
        o[0] = lo[0]; o[1] = lo[1]; o[2] = lo[2];
        o[3] = hi[0]; o[4] = hi[1]; o[5] = hi[2];
        o[6] = o[7] = 0;
    } else if constexpr (F == MXC_E4M3) {
        const uint8_t* q = p + (lane & 31) * 32 + 16 * h;
        const v4i u = *(const v4i*)q, w = *(const v4i*)(q + next);
#pragma unroll
        for (int e = 0; e < 4; e++) { o[e] = u[e]; o[4 + e] = w[e]; }
    } else if constexpr (F == MXC_E2M1) {
        const v4i u = *(const v4i*)(p + h * next + (lane & 31) * 16);
#pragma unroll
        for (int e = 0; e < 4; e++) { o[e] = u[e]; o[4 + e] = 0; }
    } else {
        const uint8_t* q = p + h * next + (lane & 31) * 32;
        const v3i lo = *(const v3i*)q, hi = *(const v3i*)(q + 16);
        o[0] = lo[0]; o[1] = lo[1]; o[2] = lo[2];
        o[3] = hi[0]; o[4] = hi[1]; o[5] = hi[2];
        o[6] = o[7] = 0;
    }
    return o;
}

// Wait until the oldest of `later` + 1 <= MOST + 1 stages of PER copies each is
// complete.
template <int PER, int MOST>
__device__ __forceinline__ void lin_wait(int later) {
    static_assert(MOST * PER <= 63, "the stages in flight must fit the vmcnt counter");
    if constexpr (MOST == 0) {
        vm_wait<0>();
    } else {
        if (later >= MOST) vm_wait<MOST * PER>();
        else lin_wait<PER, MOST - 1>(later);
    }
}

// ---------------------------------------------------------------- column sums
// db: the sums of dZ over its rows, for 32, 16 or 8 of its columns (one, two or
// four workgroups a column block) -- a product with a row of ones, exact like
// the others, from fragments that are contiguous in memory.  The 32 rows of a
// fragment are those columns of one, two or four pairs of row blocks; the waves
// take such groups in turn, LIN_SUM_AHEAD of them in flight, and the parts are
// joined in order.  (Taken along by the tiles of the weight gradient, the sums
// cost every tile 16 or 32 registers: the 256 x 128 tile spilled and ran at a
// third.)
constexpr int LIN_SUM_AHEAD = 4;
template <int F, int W>
__device__ __forceinline__ void lin_colsum(const LinOp& o, float* out, int n, int part, int split, float* red) {
    constexpr int SRC = LinBlk<F>::SRC, ROW = SRC / 32, WORDS = ROW / 4;
    const int cols = 32 >> split, subs = 1 << split;          // columns; pairs of row blocks in a fragment
    const int rb = part >> split, first = (part & (subs - 1)) * cols;
    const int lane = threadIdx.x & 63, h = lane >> 5, col = first + (lane & (cols - 1)), sub = (lane & 31) >> (5 - split);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (rb >= o.nrb) return;
    v16f acc;
#pragma unroll
    for (int e = 0; e < 16; e++) acc[e] = 0.0f;
    const int pairs = (o.ncb + 1) / 2;
    for (int g = wave; g * subs < pairs; g += W * LIN_SUM_AHEAD) {
        uint32_t f[LIN_SUM_AHEAD][8];
        int s0[LIN_SUM_AHEAD], s1[LIN_SUM_AHEAD];
#pragma unroll
        for (int k = 0; k < LIN_SUM_AHEAD; k++) {
            // blocks past the end: the last one is read and counts as zeros
            const int c0 = 2 * (subs * (g + k * W) + sub), c1 = c0 + 1;
            const size_t b0 = (size_t)rb * o.srow + (size_t)min(c0, o.ncb - 1) * o.scon;
            const size_t b1 = (size_t)rb * o.srow + (size_t)min(c1, o.ncb - 1) * o.scon;
            s0[k] = o.scales[b0];
            s1[k] = o.scales[b1];
            if constexpr (F == MXC_E4M3) {
                const v4i u = *(const v4i*)(o.codes + b0 * SRC + col * ROW + 16 * h);
                const v4i w = *(const v4i*)(o.codes + b1 * SRC + col * ROW + 16 * h);
#pragma unroll
                for (int e = 0; e < 4; e++) { f[k][e] = c0 < o.ncb ? u[e] : 0; f[k][4 + e] = c1 < o.ncb ? w[e] : 0; }
            } else {
                const uint8_t* q = o.codes + (h ? b1 : b0) * SRC + col * ROW;
                const bool ok = (h ? c1 : c0) < o.ncb;
#pragma unroll
                for (int e = 0; e < 8; e++) f[k][e] = 0;
#pragma unroll
                for (int e = 0; e < WORDS; e += 2) {
                    const v2i u = *(const v2i*)(q + 4 * e);
                    f[k][e] = ok ? u[0] : 0;
                    f[k][e + 1] = ok ? u[1] : 0;
                }
            }
            s0[k] = c0 < o.ncb ? s0[k] : 0;
            s1[k] = c1 < o.ncb ? s1[k] : 0;
        }
#pragma unroll
        for (int k = 0; k < LIN_SUM_AHEAD; k++) {
            v8i v;
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = f[k][e];
            if constexpr (F == MXC_E4M3) {
                uint32_t one[16], d[16];
#pragma unroll
                for (int e = 0; e < 16; e++) one[e] = 0x3F803F80u;
                e4m3_decode32(v, s0[k], s1[k], d);
                acc = mfma_x8(one, d, acc);
            } else {
                v8i one;                          // E2M1 code 2 is 1.0
#pragma unroll
                for (int e = 0; e < 8; e++) one[e] = e < 4 ? 0x22222222 : 0;
                acc = mfma_mx<MXC_E2M1, F>(one, v, acc, 127, h ? s1[k] : s0[k]);
            }
        }
    }
    if (lane < 32) red[wave * 32 + lane] = acc[0];
    __syncthreads();
    const int c = rb * 32 + first + (int)threadIdx.x;
    if ((int)threadIdx.x < cols && c < n) {
        float v = 0.0f;
        for (int w = 0; w < W * subs; w++) v += red[w * cols + threadIdx.x];
        out[c] = v;
    }
}

// ---------------------------------------------------------------- the product
// A workgroup computes RA x RB blocks of 32 x 32 outputs.  A stage holds KB
// contraction blocks of both operands, copied to LDS by global -> LDS loads
// into a ring of NBUF stages: while one is multiplied the next is complete and
// the NBUF - 2 after it are in flight, issued between the products; one barrier
// a stage publishes the next and frees the one before.
// Row blocks past the end read the last one (their products are not stored);
// contraction blocks past the end read zero codes and scales.
template <int FA, int FB, int OP, class T>
__global__ __launch_bounds__(T::W * 64, 2) void linear_kernel(const LinArgs p) {
    constexpr int MB = T::MB, NB = T::NB, WM = T::WM, WN = T::WN, WK = T::WK, KS = T::KS, NBUF = T::NBUF;
    constexpr int RA = T::RA, RB = T::RB, KB = T::KB, W = T::W;
    constexpr bool TA = OP == LIN_FWD, TB = OP != LIN_WGRAD;      // transposed reads
    constexpr bool X8 = FA == MXC_E4M3;
    using BA = LinBlk<FA>;
    using BB = LinBlk<FB>;
    using L = LinLds<FA, FB, T>;
    constexpr int NA = RA * KB / BA::BPI, NSL = NA + RB * KB / BB::BPI;   // 1 KB copies of a stage
    constexpr int NQ = NSL / W, NSQ = (L::NSI + W - 1) / W, PER = NQ + NSQ;
    static_assert(NSL % W == 0 && RA * KB % BA::BPI == 0 && RB * KB % BB::BPI == 0 && KS % 2 == 0, "whole copies");
    static_assert(NBUF >= 3, "ring");
    static_assert(MB * NB <= 16, "accumulators");
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // workgroups are dealt round-robin to the 8 XCDs: each XCD takes a
    // contiguous run of tiles, so tiles that share an operand share its L2
    const int ntiles = p.ta * p.tb * p.nsplit;
    const int per = (ntiles + 7) / 8;
    int bid = blockIdx.x;
    if constexpr (OP == LIN_WGRAD) {
        if (bid < p.nsum) {
            lin_colsum<FB, W>(p.b, p.colsum, p.e.nrows, bid, p.sumsplit, (float*)smem);
            return;
        }
        bid -= p.nsum;
    }
    const int lin = (bid % 8) * per + bid / 8;
    if (lin >= ntiles) return;
    // runs of up to 8 tiles along B inside a column of A's tiles
    const int split = lin / (p.ta * p.tb), t2 = lin - split * (p.ta * p.tb);
    const int band = t2 / (8 * p.ta), in_band = t2 - band * 8 * p.ta;
    const int bw = min(8, p.tb - band * 8);
    const int ia = in_band / bw, ib = band * 8 + (in_band - ia * bw);
    const int ra0 = ia * RA, rb0 = ib * RB;

    const int kbeg = split * p.span;
    const int kend = min(p.a.ncb, kbeg + p.span);
    const int nst = (kend - kbeg + KB - 1) / KB;

    // ---- this lane's part of each copy: block (row block, contraction block)
    auto blk_of = [&](int q, int& rb, int& kb) {
        const int slice = q * W + wave;
        const bool isb = slice >= NA;
        const int n = isb ? (slice - NA) * BB::BPI + (BB::BPI == 2 ? lane >> 5 : 0)
                          : slice * BA::BPI + (BA::BPI == 2 ? lane >> 5 : 0);
        const bool tr = isb ? TB : TA;
        const int R = isb ? RB : RA;
        rb = tr ? n / KB : n % R;                 // transposed operands: the contraction is contiguous
        kb = tr ? n % KB : n / R;
        return isb;
    };
    uint32_t off[NQ];
#pragma unroll
    for (int q = 0; q < NQ; q++) {
        int rb, kb;
        const bool isb = blk_of(q, rb, kb);
        const LinOp& o = isb ? p.b : p.a;
        const int r0 = isb ? rb0 : ra0;
        const uint32_t in = isb ? (uint32_t)(BB::BPI == 2 ? lane & 31 : lane) * BB::STEP
                                : (uint32_t)(BA::BPI == 2 ? lane & 31 : lane) * BA::STEP;
        off[q] = (uint32_t)((min(r0 + rb, o.nrb - 1) - r0) * o.srow + kb * o.scon) * (uint32_t)(isb ? BB::SRC : BA::SRC) + in;
    }
    const uint8_t* abase = p.a.codes + ((size_t)ra0 * p.a.srow + (size_t)kbeg * p.a.scon) * BA::SRC;
    const uint8_t* bbase = p.b.codes + ((size_t)rb0 * p.b.srow + (size_t)kbeg * p.b.scon) * BB::SRC;
    const size_t astep = (size_t)KB * p.a.scon * BA::SRC, bstep = (size_t)KB * p.b.scon * BB::SRC;
    // scale entry e of a stage: [contraction block][row block] of A, then of B
    const uint8_t* sp[NSQ];
    uint32_t sstep[NSQ];
    int skb[NSQ];
#pragma unroll
    for (int q = 0; q < NSQ; q++) {
        const int e = ((q * W + wave) % L::NSI) * 64 + lane;
        const bool isb = e >= RA * KB;
        const int n = isb ? e - RA * KB : e, R = isb ? RB : RA;
        const LinOp& o = isb ? p.b : p.a;
        const int r0 = isb ? rb0 : ra0;
        const int kb = n / R, row = min(r0 + n % R, o.nrb - 1);
        const bool ok = e < (RA + RB) * KB;
        skb[q] = ok ? kb : 0x40000000;
        sp[q] = o.scales + (ok ? (size_t)row * o.srow + (size_t)(kbeg + kb) * o.scon : 0);
        sstep[q] = (uint32_t)(KB * o.scon);
    }

    // held in registers: the address would be loaded again for every stage
    const uint8_t* zero = g_lin_zero;
    asm("" : "+s"(zero));
    int kis = kbeg;                               // first contraction block of the next stage to copy
    // copy n of the stage's PER (codes, then scales) into the slot at lds; FULL:
    // every contraction block of the stage exists
    auto copy = [&](const uint8_t* lds, int n, auto full) {
        constexpr bool FULL = decltype(full)::value;
        if (n < NQ) {
            const int slice = n * W + wave;
            const bool isb = slice >= NA;
            if (FULL || kis + KB <= kend) {
                dma16_base(isb ? bbase : abase, off[n], lds_addr(lds + slice * 1024));
            } else {
                int rb, kb;
                blk_of(n, rb, kb);
                dma16_async(kis + kb < kend ? (isb ? bbase : abase) + off[n] : zero + lane * 16,
                            lds_addr(lds + slice * 1024));
            }
        } else {
            const int q = n - NQ;
            dma1_async((FULL && L::NSI * 64 == (RA + RB) * KB) || kis + skb[q] < kend ? sp[q] : zero,
                       lds_addr(lds + L::ABYTES + L::BBYTES + ((q * W + wave) % L::NSI) * 256));
            sp[q] += sstep[q];
        }
        if (n == PER - 1) {
            abase += astep;
            bbase += bstep;
            kis += KB;
        }
    };
    auto issue = [&](int buf) {
#pragma unroll
        for (int n = 0; n < PER; n++) copy(smem + buf * L::STAGE, n, std::false_type{});
    };

    const int wk = wave / (WM * WN), wmn = wave - wk * (WM * WN), wm = wmn % WM, wn = wmn / WM;
    v16f acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.0f;

    // ---- the fragments of a step (two contraction blocks of each operand) are
    // read from LDS one step ahead, each as soon as the registers of its
    // predecessor are free, so the products do not wait for LDS.  X8: the raw
    // codes are read ahead and decoded to bf16 in the step itself.
    constexpr int STEPS = KS / 2;
    v8i rawa[MB], rawb[NB];
    int sca[MB][X8 ? 2 : 1], scb[NB][X8 ? 2 : 1];
    auto scale = [&](const uint8_t* sc, int next, int* o) {
        if constexpr (X8) {                       // a lane holds both blocks' codes
            o[0] = *(const int*)sc;
            o[1] = *(const int*)(sc + next);
        } else {
            o[0] = *(const int*)(sc + (lane >> 5) * next);
        }
    };
    auto fetch_a = [&](const uint8_t* stage, int s, int i) {
        const int k0 = wk * KS + 2 * s, ra = wm * MB + i;
        rawa[i] = lin_frag<FA, TA>(stage + (TA ? ra * KB + k0 : k0 * RA + ra) * BA::LDS, (TA ? 1 : RA) * BA::LDS, lane);
        scale(stage + L::ABYTES + L::BBYTES + 4 * (k0 * RA + ra), 4 * RA, sca[i]);
    };
    auto fetch_b = [&](const uint8_t* stage, int s, int j, v8i& raw, int* sc) {
        const int k0 = wk * KS + 2 * s, rb = wn * NB + j;
        raw = lin_frag<FB, TB>(stage + L::ABYTES + (TB ? rb * KB + k0 : k0 * RB + rb) * BB::LDS,
                               (TB ? 1 : RB) * BB::LDS, lane);
        scale(stage + L::ABYTES + L::BBYTES + 4 * (RA * KB + k0 * RB + rb), 4 * RB, sc);
    };

    for (int j = 0; j < NBUF - 1 && j < nst; j++) issue(j);
    lin_wait<PER, NBUF - 2>(nst - 1);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NB; j++) fetch_b(smem, 0, j, rawb[j], scb[j]);
#pragma unroll
    for (int i = 0; i < MB; i++) fetch_a(smem, 0, i);
    int buf = 0;
    // One stage.  AHEAD: the copies of stage st + NBUF - 1, a full one, go out
    // between the products without a branch; else they go out first, where there
    // are any.
    auto stage = [&](int st, auto ahead) {
        constexpr bool AHEAD = decltype(ahead)::value;
        // stage st + 1 is complete for every wave, and stage st - 1's slot is free
        if (AHEAD) vm_wait<(NBUF - 3) * PER>();
        else if (st + 1 < nst) lin_wait<PER, NBUF - 3>(nst - 2 - st);
        __syncthreads();
        const uint8_t* const slot = smem + (buf == 0 ? NBUF - 1 : buf - 1) * L::STAGE;
        if (!AHEAD && st + NBUF - 1 < nst) issue(buf == 0 ? NBUF - 1 : buf - 1);
        auto next = [&](int product) {
            constexpr int PRODUCTS = STEPS * MB * NB, EACH = (PER + PRODUCTS - 1) / PRODUCTS;
            if constexpr (AHEAD) {
#pragma unroll
                for (int n = 0; n < EACH; n++)
                    if (product * EACH + n < PER) copy(slot, product * EACH + n, std::true_type{});
            }
        };
        const uint8_t* cur = smem + buf * L::STAGE;
        buf = buf + 1 == NBUF ? 0 : buf + 1;
        // past the last stage the ring's old bytes are read and not used
        const uint8_t* nxt = smem + buf * L::STAGE;
#pragma unroll
        for (int s = 0; s < STEPS; s++) {
            const uint8_t* ns = s + 1 < STEPS ? cur : nxt;
            const int n = s + 1 < STEPS ? s + 1 : 0;
            v8i fb[NB];
            int sb[NB];
            uint32_t db[X8 ? NB : 1][16];
#pragma unroll
            for (int j = 0; j < NB; j++) {
                if constexpr (X8) e4m3_decode32(rawb[j], scb[j][0], scb[j][1], db[j]);
                else { fb[j] = rawb[j]; sb[j] = scb[j][0]; }
                fetch_b(ns, n, j, rawb[j], scb[j]);
            }
#pragma unroll
            for (int i = 0; i < MB; i++) {
                if constexpr (X8) {
                    uint32_t da[16];
                    e4m3_decode32(rawa[i], sca[i][0], sca[i][1], da);
                    fetch_a(ns, n, i);
#pragma unroll
                    for (int j = 0; j < NB; j++) {
                        acc[i][j] = mfma_x8(da, db[j], acc[i][j]);
                        next((s * MB + i) * NB + j);
                    }
                } else {
                    const v8i fa = rawa[i];
                    const int sa = sca[i][0];
                    fetch_a(ns, n, i);
#pragma unroll
                    for (int j = 0; j < NB; j++) {
                        acc[i][j] = mfma_mx<FA, FB>(fa, fb[j], acc[i][j], sa, sb[j]);
                        next((s * MB + i) * NB + j);
                    }
                }
            }
        }
    };
    const int nahead = max(0, (kend - kbeg) / KB - (NBUF - 1));      // stages whose copies are of a full one
    int st0 = 0;
    for (; st0 < nahead; st0++) stage(st0, std::true_type{});
    for (; st0 < nst; st0++) stage(st0, std::false_type{});

    // ---- write: lane l holds output row l % 32 of B's block and, in quad q,
    // columns 8 q + 4 (l / 32) .. + 3 of A's block
    auto put = [&](int r, int c, float4 v) {
        if (r >= p.e.nrows) return;
        if (p.part) {
            if (c < p.ldw) *(float4*)(p.part + ((size_t)split * p.e.nrows + r) * p.ldw + c) = v;
        } else {
            lin_epilogue4<OP>(p.e, r, c, v);
        }
    };
    if constexpr (WK == 1) {
        // One block row of B at a time through LDS, each wave in a region of
        // its own, so that a row's MB blocks leave as one run: stored straight
        // from the accumulators, every instruction would touch 32 rows with
        // 16 (bf16) or 32 bytes each.  Rows are padded by four floats.
        constexpr int LD = L::LD;
        __syncthreads();                          // every wave is done with the ring
        float* const mine = (float*)smem + wave * 32 * LD;
#pragma unroll
        for (int j = 0; j < NB; j++) {
            auto park = [&]() {
#pragma unroll
                for (int i = 0; i < MB; i++)
#pragma unroll
                    for (int q = 0; q < 4; q++)
                        *(float4*)(mine + (lane & 31) * LD + 32 * i + 8 * q + 4 * (lane >> 5)) = make_float4(
                            acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
            };
            const int r0 = (rb0 + wn * NB + j) * 32, c0 = (ra0 + wm * MB) * 32;
            if (p.part) {
                park();
                __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                for (int n = 0; n < 4 * MB; n++) {
                    const int row = (n * 64 + lane) / (8 * MB), col = lane % (8 * MB) * 4;
                    put(r0 + row, c0 + col, *(const float4*)(mine + row * LD + col));
                }
                __builtin_amdgcn_wave_barrier();
            } else if (OP != LIN_WGRAD && p.e.bf16) {
                lin_rows<OP, true, MB>(p.e, r0, c0, mine, lane, park);
            } else {
                lin_rows<OP, false, MB>(p.e, r0, c0, mine, lane, park);
            }
        }
    } else {
        // the waves of one output block add their parts in order, through LDS
        __syncthreads();                          // every wave is done with the ring
        float4* red = (float4*)smem;              // [wk][wave of the tile][block][quad][lane]
        constexpr int BL = MB * NB * 256;         // float4s of a wave
#pragma unroll
        for (int i = 0; i < MB; i++)
#pragma unroll
            for (int j = 0; j < NB; j++)
#pragma unroll
                for (int q = 0; q < 4; q++)
                    red[(wk * WM * WN + wmn) * BL + (i * NB + j) * 256 + q * 64 + lane] =
                        make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
        __syncthreads();
        for (int n = tid; n < WM * WN * BL; n += W * 64) {
            float4 v = red[n];
#pragma unroll
            for (int k = 1; k < WK; k++) {
                const float4 u = red[k * WM * WN * BL + n];
                v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
            }
            const int l = n & 63, q = (n >> 6) & 3, b = (n >> 8) % (MB * NB), w = (n >> 8) / (MB * NB);
            put((rb0 + (w / WM) * NB + b % NB) * 32 + (l & 31), (ra0 + (w % WM) * MB + b / NB) * 32 + 8 * q + 4 * (l >> 5), v);
        }
    }
}

template <int FA, int FB, int OP, class T>
int linear_launch(const LinArgs& a, hipStream_t s) {
    // the plan counted tiles of this shape: one that begins past the last block would read out of range
    if (a.ta != (a.a.nrb + T::RA - 1) / T::RA || a.tb != (a.b.nrb + T::RB - 1) / T::RB || a.span % T::KB) return MXC_ERR_SHAPE;
    static std::atomic<uint64_t> devs{0};
    constexpr int lds = LinLds<FA, FB, T>::BYTES;
    static_assert(lds <= 163840, "LDS of a CU");
    auto kernel = linear_kernel<FA, FB, OP, T>;
    if (lds > 65536) {                            // above 64 KB the attribute is raised, once per device
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess) return MXC_ERR_HIP;
        const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
        if (!bit || !(devs.load(std::memory_order_acquire) & bit)) {
            if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
                return MXC_ERR_HIP;
            devs.fetch_or(bit, std::memory_order_release);
        }
    }
    const long long tiles = (long long)a.ta * a.tb * a.nsplit;
    kernel<<<(unsigned)((tiles + 7) / 8 * 8 + a.nsum), T::W * 64, lds, s>>>(a);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_HIP;
}

}  // namespace mxc
#endif
