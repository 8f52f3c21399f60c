// norm.hip -- the residual update of a block with its norms, fused:
//   H = X + s g . N(Y; w_post),   U = N(H; w_pre),   N(v; w) = w v r(v),   r(v) = (mean v^2 + eps)^(-1/2)
// and its gradients.  With hh = h r_h, t = du w_pre, yh = y r_y, p = yh w_post:
//   dX = dH + r_h (t - hh mean(t hh)),          dw_pre  = sum over rows of du hh
//   b  = s g dX,                                dg      = sum over the gate's rows of s dX p
//   dY = r_y (b w_post - yh mean(b w_post yh)), dw_post = sum over rows of b yh
// Without w_post, N(Y) is Y itself; without w_pre there is no U.  The backward
// pass takes H and Y and forms both norms' statistics again: the rows are in
// registers anyway, and nothing needs to be kept by the forward pass.
//
// What bounds both is memory: a row is read once and held in registers (8
// values of each tensor a thread, 16 of the longest rows), with two sums over the
// row forward (Y's square, then H's) and two rounds of sums backward (the second
// one needs dX).  bf16, other inputs in between: forward 8192 x 4096 57 us a pass
// among others (4.7 TB/s; 49 waited for alone, when the last results are still on
// their way out of the caches), backward 16384 x 1024 53 (3.8 TB/s; 43 alone and 6
// for the join); a copy of 2 GiB reaches 5.0 TB/s.
// Four waves a SIMD leave 128 registers, and some kernels spill a few: 2 to 4 in
// the backward pass of rows of 2049 to 4096, 8 in the bf16 forward of longer ones,
// and 6 to 18 (up to 76 bytes) where workgroups take whole gates, of bf16 rows up
// to 4096 and fp32 rows of 1025 to 4096.
// A workgroup takes a run of consecutive rows, so the weights and the gate are
// loaded once a run; backward, its column sums stay in registers until the
// run's end and are added over the workgroups by a second kernel, in order.
// All sums and statistics are fp32.
#include "mx_internal.h"
#include "norm.h"

namespace mxc {
namespace {

// A thread's vector of a row: 16 bytes (8 bf16 or 4 fp32), V values.  Rows of
// any length and stride are read and written with it: global memory takes
// 16-byte accesses at any element's address, so only the last, partial vector of
// a row goes element by element.  Values past the row's end are zeros, which no
// sum sees.
template <typename T> constexpr int VEC = 16 / (int)sizeof(T);
struct __attribute__((packed, aligned(2))) Raw16 {
    uint32_t w[4];
};
struct __attribute__((packed, aligned(4))) Raw16f {
    uint32_t w[4];
};
template <typename T> using Raw = std::conditional_t<sizeof(T) == 2, Raw16, Raw16f>;

template <typename T>
__device__ __forceinline__ void st1(T* p, float v) {
    if constexpr (sizeof(T) == 4) *p = v;
    else *(uint16_t*)p = (uint16_t)bf16_bits(v);
}
// n: values of the row left from here on.  get() reads a vector as it is stored,
// unpack() makes floats of it; the rows' loops read one row ahead.
template <typename T>
__device__ __forceinline__ Raw<T> get(const T* p, int n) {
    constexpr int V = VEC<T>;
    if (n >= V) return *(const Raw<T>*)p;
    Raw<T> u;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        if constexpr (V == 8) {
            const uint32_t lo = 2 * k < n ? *(const uint16_t*)(p + 2 * k) : 0u;
            const uint32_t hi = 2 * k + 1 < n ? *(const uint16_t*)(p + 2 * k + 1) : 0u;
            u.w[k] = lo | hi << 16;
        } else {
            u.w[k] = k < n ? __float_as_uint(p[k]) : 0u;
        }
    }
    return u;
}
template <typename T>
__device__ __forceinline__ void unpack(const Raw<T>& u, float* o) {
#pragma unroll
    for (int k = 0; k < 4; k++) {
        if constexpr (VEC<T> == 8) {
            o[2 * k] = __uint_as_float(u.w[k] << 16);
            o[2 * k + 1] = __uint_as_float(u.w[k] & 0xFFFF0000u);
        } else {
            o[k] = __uint_as_float(u.w[k]);
        }
    }
}
template <typename T>
__device__ __forceinline__ void ld(const T* p, int n, float* o) { unpack<T>(get(p, n), o); }
// nt: NormArgs
template <typename T>
__device__ __forceinline__ void st(T* p, int n, const float* v, bool nt = false) {
    constexpr int V = VEC<T>;
    if (n >= V) {
        Raw<T> u;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            if constexpr (V == 8) u.w[k] = bf16_pack2(v[2 * k], v[2 * k + 1]);
            else u.w[k] = __float_as_uint(v[k]);
        }
        if (nt) store_nt(p, make_uint4(u.w[0], u.w[1], u.w[2], u.w[3]));
        else *(Raw<T>*)p = u;
    } else {
#pragma unroll
        for (int e = 0; e < V; e++)
            if (e < n) st1(p + e, v[e]);
    }
}
// V consecutive fp32 parameters
template <int V>
__device__ __forceinline__ void ldp(const float* p, int n, float* o) {
    ld<float>(p, n, o);
    if constexpr (V == 8) ld<float>(n > 4 ? p + 4 : p, max(n - 4, 0), o + 4);
}

template <int V>
__device__ __forceinline__ void stp(float* p, int n, const float* v) {
    st<float>(p, n, v);
    if constexpr (V == 8) {
        if (n > 4) st<float>(p + 4, n - 4, v + 4);
    }
}

// Sums of K values over the TPR threads of a row, returned to all of them.
// red: LDS of two rounds, used in turn (par), so that a round's one barrier also
// separates its writes from the reads of the round before last.
template <int TPR, int K, int N>
__device__ __forceinline__ void row_sum(float* v, float (*both)[N], int& par) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
#pragma unroll
        for (int k = 0; k < K; k++) v[k] += __shfl_xor(v[k], m, 64);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float* red = both[par];
        par ^= 1;
        const int wave = threadIdx.x >> 6, first = wave / W * W;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; k++) red[wave * K + k] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; k++) v[k] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; w++)
#pragma unroll
            for (int k = 0; k < K; k++) v[k] += red[(first + w) * K + k];
    }
}

// The value q (of NV) of a thread is column (q / V) * TPR * V + t * V + q % V.
template <int V, int NV, int TPR, class F>
__device__ __forceinline__ void columns(int d, int t, F&& f) {
#pragma unroll
    for (int i = 0; i < NV / V; i++) {
        const int c = (i * TPR + t) * V;
        if (i * TPR * V < d && c < d) f(i * V, c, d - c);
    }
}

template <typename T, int NV, int TPR>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR, NV == 8 || sizeof(T) == 2 ? 4 : 2) void norm_fwd_kernel(const NormArgs a) {
    constexpr int V = VEC<T>;
    constexpr int RL = TPR == 64 ? 4 : 1;             // rows a workgroup takes at a time
    __shared__ float red[2][TPR / 64];
    int par = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR, d = a.d;
    const long long first = (long long)blockIdx.x * a.run, last = min(first + a.run, a.rows);
    float wp[NV], wq[NV], g[NV];
    columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
        if (a.w_post) ldp<V>(a.w_post + c, n, wp + q);
        if (a.w_pre) ldp<V>(a.w_pre + c, n, wq + q);
    });
    long long gate = -1;
    Raw<T> nx[NV / V], ny[NV / V];
    auto fetch = [&](long long r) {
        columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
            nx[q / V] = get((const T*)a.x + r * a.ldx + c, n);
            ny[q / V] = get((const T*)a.y + r * a.ldy + c, n);
        });
    };
    if (first + rl < last) fetch(first + rl);
    for (long long r = first + rl; r < last; r += RL) {
        const long long gr = a.gate ? r / a.gate_rows : 0;
        if (gr != gate) {                                     // s g, for this gate's rows
            gate = gr;
            columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
                float u[V];
                if (a.gate) ldp<V>(a.gate + gr * d + c, n, u);
#pragma unroll
                for (int e = 0; e < V; e++) g[q + e] = a.gate ? a.scale * u[e] : a.scale;
            });
        }
        float x[NV], y[NV], s[1] = {0.0f};
        columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
            unpack<T>(nx[q / V], x + q);
            unpack<T>(ny[q / V], y + q);
#pragma unroll
            for (int e = 0; e < V; e++) s[0] += y[q + e] * y[q + e];
        });
        if (r + RL < last) fetch(r + RL);
        float ry = 1.0f;
        if (a.w_post) {
            row_sum<TPR, 1>(s, red, par);
            ry = 1.0f / sqrtf(s[0] * a.inv_d + a.eps);
        }
        s[0] = 0.0f;
        columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float v = a.w_post ? y[q + e] * ry * wp[q + e] : y[q + e];
                x[q + e] += g[q + e] * v;
                s[0] += x[q + e] * x[q + e];
            }
            st<T>((T*)a.h + r * a.ldh + c, n, x + q, a.nt);
        });
        if (a.w_pre) {
            row_sum<TPR, 1>(s, red, par);
            const float rh = 1.0f / sqrtf(s[0] * a.inv_d + a.eps);
            columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
                float u[V];
#pragma unroll
                for (int e = 0; e < V; e++) u[e] = x[q + e] * rh * wq[q + e];
                st<T>((T*)a.u + r * a.ldu + c, n, u, a.nt);
            });
        }
    }
}

// The workgroups cover the rows in runs that do not cross a gate's rows
// (runs_per_gate of them a gate), or (WHOLE) take gates_per_run whole gates each.  Both
// column sums with dX come from one: with c = sum over a gate's rows of dX yh,
// dg = s w_post c and dw_post = s g c, added over the gates.
template <typename T, int NV, int TPR, bool WHOLE>
__global__ __launch_bounds__(512, NV == 8 ? 4 : 2) void norm_bwd_kernel(const NormArgs a) {
    constexpr int V = VEC<T>;
    constexpr int RL = 512 / TPR;
    __shared__ float red[2][512 / 64 * 3];
    __shared__ float col[RL > 1 ? RL * NV * TPR : 1];
    int par = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR, d = a.d;
    float wq[NV], gw[NV], s_pre[NV], s_c[NV];                 // w_pre, s g w_post, sums of du hh and dX yh
#pragma unroll
    for (int q = 0; q < NV; q++) wq[q] = gw[q] = s_pre[q] = s_c[q] = 0.0f;
    if (a.w_pre) columns<V, NV, TPR>(d, t, [&](int q, int c, int n) { ldp<V>(a.w_pre + c, n, wq + q); });
    // a thread's column sums, added over the workgroup's rows, as
    // out(column, values left, sums)
    auto flush = [&](const float* v, auto&& out) {
        if constexpr (RL > 1) {
            __syncthreads();
#pragma unroll
            for (int q = 0; q < NV; q++) col[(rl * NV + q) * TPR + t] = v[q];
            __syncthreads();
        }
        if (rl == 0) {
            columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
                float u[V];
#pragma unroll
                for (int e = 0; e < V; e++) {
                    u[e] = v[q + e];
                    if constexpr (RL > 1) {
                        u[e] = 0.0f;
#pragma unroll
                        for (int l = 0; l < RL; l++) u[e] += col[(l * NV + q + e) * TPR + t];
                    }
                }
                out(c, n, u);
            });
        }
    };
    const long long bid = blockIdx.x;
    // gates [g0, g1) of gate_rows rows each; a run inside one gate takes its
    // rows [o0, o1)
    const long long g0 = WHOLE ? bid * a.gates_per_run : bid / a.runs_per_gate;
    const long long g1 = WHOLE ? min(g0 + a.gates_per_run, a.gates) : g0 + 1;
    const long long o0 = WHOLE ? 0 : (bid - g0 * a.runs_per_gate) * a.run;
    const long long o1 = WHOLE ? a.gate_rows : min(o0 + a.run, a.gate_rows);
    for (long long gr = g0; gr < g1; gr++) {
        columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
            float u[V], w[V];
            if (a.gate) ldp<V>(a.gate + gr * d + c, n, u);
            if (a.w_post) ldp<V>(a.w_post + c, n, w);
#pragma unroll
            for (int e = 0; e < V; e++) gw[q + e] = (a.gate ? a.scale * u[e] : a.scale) * (a.w_post ? w[e] : 1.0f);
        });
        // the workgroup's rows in step, for the barriers of their sums: where the
        // last ones do not exist, the run's last row is computed and dropped
        // bf16 rows are read one ahead; fp32 ones leave no registers for that
        constexpr bool AHEAD = sizeof(T) == 2;
        constexpr int NR = AHEAD ? NV / V : 1;
        Raw<T> nx[NR], ny[NR], nh[NR], nu[NR];
        auto fetch = [&](long long rb) {
            const long long r = gr * a.gate_rows + min(rb + rl, o1 - 1);
            columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
                nx[q / V % NR] = get((const T*)a.x + r * a.ldx + c, n);  // dH
                ny[q / V % NR] = get((const T*)a.y + r * a.ldy + c, n);
                if (a.w_pre) {
                    nh[q / V % NR] = get((const T*)a.h + r * a.ldh + c, n);
                    nu[q / V % NR] = get((const T*)a.u + r * a.ldu + c, n);   // dU
                }
            });
        };
        if constexpr (AHEAD) fetch(o0);
        for (long long rb = o0; rb < o1; rb += RL) {
            const bool live = rb + rl < o1;
            const long long r = gr * a.gate_rows + (live ? rb + rl : o1 - 1);
            float x[NV], y[NV], h[NV], du[NV], s[3] = {0.0f, 0.0f, 0.0f};
            columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
                if constexpr (AHEAD) {
                    unpack<T>(nx[q / V], x + q);
                    unpack<T>(ny[q / V], y + q);
                    if (a.w_pre) {
                        unpack<T>(nh[q / V], h + q);
                        unpack<T>(nu[q / V], du + q);
                    }
                } else {
                    ld<T>((const T*)a.x + r * a.ldx + c, n, x + q);
                    ld<T>((const T*)a.y + r * a.ldy + c, n, y + q);
                    if (a.w_pre) {
                        ld<T>((const T*)a.h + r * a.ldh + c, n, h + q);
                        ld<T>((const T*)a.u + r * a.ldu + c, n, du + q);
                    }
                }
            });
            if constexpr (AHEAD) {
                if (rb + RL < o1) fetch(rb + RL);
            }
            columns<V, NV, TPR>(d, t, [&](int q, int, int) {
#pragma unroll
                for (int e = 0; e < V; e++) {
                    s[0] += y[q + e] * y[q + e];
                    if (a.w_pre) {
                        s[1] += h[q + e] * h[q + e];
                        s[2] += h[q + e] * (du[q + e] * wq[q + e]);
                    }
                }
            });
            row_sum<TPR, 3>(s, red, par);
            const float ry = a.w_post ? 1.0f / sqrtf(s[0] * a.inv_d + a.eps) : 1.0f;
            const float rh = 1.0f / sqrtf(s[1] * a.inv_d + a.eps);
            const float mh = s[2] * rh * a.inv_d;                        // mean(t hh)
            float m[1] = {0.0f};
            columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
#pragma unroll
                for (int e = 0; e < V; e++) {
                    if (a.w_pre) {
                        const float hh = h[q + e] * rh;
                        x[q + e] += rh * (du[q + e] * wq[q + e] - hh * mh);
                        s_pre[q + e] += live ? du[q + e] * hh : 0.0f;
                    }
                    const float yh = y[q + e] * ry;
                    s_c[q + e] += live ? x[q + e] * yh : 0.0f;
                    m[0] += gw[q + e] * x[q + e] * yh;                   // b w_post yh
                    y[q + e] = yh;
                }
                if (live) st<T>((T*)a.dx + r * a.lddx + c, n, x + q, a.nt);
            });
            float my = 0.0f;
            if (a.w_post) {
                row_sum<TPR, 1>(m, red, par);
                my = m[0] * a.inv_d;
            }
            columns<V, NV, TPR>(d, t, [&](int q, int c, int n) {
                float o[V];
#pragma unroll
                for (int e = 0; e < V; e++) o[e] = ry * (gw[q + e] * x[q + e] - y[q + e] * my);
                if (live) st<T>((T*)a.dy + r * a.lddy + c, n, o, a.nt);
            });
        }
        if constexpr (!WHOLE) {                               // the join makes both gradients of it
            if (a.p_c) flush(s_c, [&](int c, int n, const float* u) { stp<V>(a.p_c + bid * d + c, n, u); });
        } else if (a.gate || a.w_post) {
            float* const pg = a.gate ? a.p_gate + gr * d : nullptr;
            float* const pw = a.w_post ? a.p_post + bid * d : nullptr;
            flush(s_c, [&](int c, int n, const float* u) {
                float v[V], o[V];
                if (pg) {
                    if (pw) ldp<V>(a.w_post + c, n, v);
#pragma unroll
                    for (int e = 0; e < V; e++) o[e] = a.scale * u[e] * (pw ? v[e] : 1.0f);
                    stp<V>(pg + c, n, o);
                }
                if (pw) {
                    if (pg) ldp<V>(a.gate + gr * d + c, n, v);
#pragma unroll
                    for (int e = 0; e < V; e++) o[e] = a.scale * u[e] * (pg ? v[e] : 1.0f);
                    if (gr != g0) {                           // the gates before this one
                        ldp<V>(pw + c, n, v);
#pragma unroll
                        for (int e = 0; e < V; e++) o[e] += v[e];
                    }
                    stp<V>(pw + c, n, o);
                }
            });
        }
#pragma unroll
        for (int q = 0; q < NV; q++) s_c[q] = 0.0f;
    }
    if (a.w_pre) {
        float* const pq = a.p_pre + bid * d;
        flush(s_pre, [&](int c, int n, const float* u) { stp<V>(pq + c, n, u); });
    }
}

// dst[row][c] = f[c] (sum over n consecutive partial rows k, in a fixed order,
// of src[k][c], times mul[k / per][c] where there is one): 32 columns a
// workgroup, 32 threads a column, each taking every 32nd row, four loads at a
// time.
struct JoinJob {
    const float* src;
    const float* mul;
    const float* f;               // NULL: 1
    float* dst;
    float scale;
    int n, rows, per;             // partial rows of a result row, result rows
};
struct JoinArgs {
    JoinJob job[3];
    int d;
};
__global__ __launch_bounds__(1024) void norm_join_kernel(const JoinArgs a) {
    __shared__ float red[32][33];
    int j = 0, row = blockIdx.y;
    while (row >= a.job[j].rows) row -= a.job[j++].rows;
    const JoinJob& o = a.job[j];
    const int x = threadIdx.x & 31, l = threadIdx.x >> 5, c = blockIdx.x * 32 + x, cc = min(c, a.d - 1), n = o.n;
    const float* p = o.src + (size_t)row * n * a.d + cc;
    float s = 0.0f;
    for (int k = l; k < n; k += 128) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const int i = k + 32 * q;
            v[q] = i < n ? p[(size_t)i * a.d] : 0.0f;
            if (o.mul && i < n) v[q] *= o.mul[(size_t)(i / o.per) * a.d + cc];
        }
        s += (v[0] + v[1]) + (v[2] + v[3]);
    }
    red[l][x] = s;
    __syncthreads();
    if (l == 0) {
#pragma unroll
        for (int k = 1; k < 32; k++) s += red[k][x];
        if (c < a.d) o.dst[(size_t)row * a.d + c] = o.scale * s * (o.f ? o.f[c] : 1.0f);
    }
}

template <typename T>
void launch_rows(const NormArgs& a, bool bwd, int tpr, unsigned grid, hipStream_t s) {
    auto go = [&](auto vals, auto threads) {
        constexpr int NV = decltype(vals)::value, TPR = decltype(threads)::value;
        if (bwd && a.runs_per_gate > 1) norm_bwd_kernel<T, NV, TPR, false><<<grid, 512, 0, s>>>(a);
        else if (bwd) norm_bwd_kernel<T, NV, TPR, true><<<grid, 512, 0, s>>>(a);
        else norm_fwd_kernel<T, NV, TPR><<<grid, TPR == 64 ? 256 : TPR, 0, s>>>(a);
    };
    const std::integral_constant<int, 8> v8;
    if (norm_vals(a.d) == 16) go(std::integral_constant<int, 16>{}, std::integral_constant<int, 512>{});
    else if (tpr == 64) go(v8, std::integral_constant<int, 64>{});
    else if (tpr == 128) go(v8, std::integral_constant<int, 128>{});
    else if (tpr == 256) go(v8, std::integral_constant<int, 256>{});
    else go(v8, std::integral_constant<int, 512>{});
}

int launch(const NormArgs& a, bool bwd, bool bf16, unsigned grid, hipStream_t s) {
    if (bf16) launch_rows<__bf16>(a, bwd, norm_tpr(a.d), grid, s);
    else launch_rows<float>(a, bwd, norm_tpr(a.d), grid, s);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_HIP;
}

// Runs of the backward pass: about norm_runs() workgroups, none crossing a gate.
void plan_runs(NormArgs& a) {
    const long long rl = norm_bwd_rows(a.d);
    if (a.gates >= norm_runs(a.d)) {
        a.runs_per_gate = 1;
        a.gates_per_run = (a.gates + norm_runs(a.d) - 1) / norm_runs(a.d);
        a.run = a.gate_rows;
        a.runs = (a.gates + a.gates_per_run - 1) / a.gates_per_run;
    } else {
        const long long want = std::max<long long>(1, norm_runs(a.d) / a.gates);
        a.run = std::max<long long>(rl, (a.gate_rows + want - 1) / want);
        a.runs_per_gate = (a.gate_rows + a.run - 1) / a.run;
        a.gates_per_run = 1;
        a.runs = a.gates * a.runs_per_gate;
    }
}

}  // namespace

// Results whose rows begin at cache lines (ld: their row stride).
static bool lines(bool bf16, const void* p, long long ld) {
    const int es = bf16 ? 2 : 4;
    return !p || ((uintptr_t)p % 128 == 0 && ld * es % 128 == 0);
}
// Whether results are stored non-temporally, by the bytes of one.  Measured with
// other inputs in between, plain -> non-temporal stores, us, and in brackets with
// the quantization of U, or of dX and dY, behind them:
//                            forward                       backward
//   2 MiB (bf16 1024 rows)   6.0 -> 6.0 (9.7 -> 9.6)       13.5 -> 13.6 (20.7 -> 20.7)
//   4     (bf16 2048)        7.9 -> 7.1 (12.6 -> 12.1)     18.8 -> 17.7 (28.1 -> 27.8)
//   8     (bf16 4096)        11.9 -> 9.9 (18.3 -> 17.1)    24.8 -> 21.8 (37.9 -> 36.3)
//   16    (bf16 8192)        18.2 -> 18.4 (29.1 -> 29.5)   33.6 -> 32.7 (54.6 -> 55.5)
//   32    (bf16 16384)       31.1 -> 31.1 (47.8 -> 51.1)   53.0 -> 52.8 (86.2 -> 93.1)
//   64    (fp32 16384)       63.2 -> 62.8 (81.0 -> 85.5)   94.8 -> 91.3 (134.9 -> 136.8)
//   128   (fp32, d 4096)     112 -> 120 (154 -> 155)       188 -> 184 (272 -> 265)
// (d 1024): from 16 MiB on the last-level cache still holds plain results for
// what reads them next, until the backward pass's tensors no longer fit it
// together.  Rows that begin inside cache lines lose by them (backward, bf16 rows
// of 4095: 175 -> 187).
static bool past(const NormArgs& a, bool bf16, bool bwd) {
    const long long mib = (a.rows * a.d * (bf16 ? 2 : 4)) >> 20;
    return (mib >= 4 && mib < 16) || (bwd && mib >= 128);
}

int launch_norm_fwd(NormArgs a, bool bf16, hipStream_t s) {
    a.nt = past(a, bf16, false) && lines(bf16, a.h, a.ldh) && lines(bf16, a.u, a.ldu);
    const long long rl = norm_fwd_rows(a.d);
    a.run = std::max<long long>(rl, (a.rows + norm_fwd_runs(a.d) - 1) / norm_fwd_runs(a.d));
    return launch(a, false, bf16, (unsigned)((a.rows + a.run - 1) / a.run), s);
}

// Partial arrays of the backward pass: du hh's, and dX yh's or dw_post's.
static int norm_parts(const NormArgs& a, bool gate, bool post, bool pre) {
    const bool c = a.runs_per_gate > 1 ? gate || post : post;
    return (pre ? 1 : 0) + (c ? 1 : 0);
}

size_t norm_bwd_workspace(long long rows, int d, long long gates, bool gate, bool post, bool pre) {
    NormArgs a;
    a.d = d; a.rows = rows; a.gates = gates; a.gate_rows = rows / gates;
    plan_runs(a);
    return a.runs == 1 ? 0 : (size_t)norm_parts(a, gate, post, pre) * a.runs * d * sizeof(float);
}

int launch_norm_bwd(NormArgs a, bool bf16, float* dw_pre, float* dw_post, float* dgate, void* ws, hipStream_t s) {
    plan_runs(a);
    a.nt = past(a, bf16, true) && lines(bf16, a.dx, a.lddx) && lines(bf16, a.dy, a.lddy);
    const bool one = a.runs == 1;                 // a single workgroup writes the results itself
    float* p = (float*)ws;
    auto take = [&](float* dst) {
        if (one) return dst;
        float* q = p;
        p += (size_t)a.runs * a.d;
        return q;
    };
    a.p_pre = a.w_pre ? take(dw_pre) : nullptr;
    const bool c = a.runs_per_gate > 1 && (a.gate || a.w_post);
    a.p_c = c ? take(nullptr) : nullptr;
    a.p_post = !c && a.w_post ? take(dw_post) : nullptr;
    a.p_gate = !c ? dgate : nullptr;
    int rc = launch(a, true, bf16, (unsigned)a.runs, s);
    if (rc || one) return rc;
    JoinArgs j = {};
    int nj = 0;
    long long nrows = 0;
    auto add = [&](JoinJob job) {
        j.job[nj++] = job;
        nrows += job.rows;
    };
    const int runs = (int)a.runs, per = (int)a.runs_per_gate;
    if (a.w_pre) add({a.p_pre, nullptr, nullptr, dw_pre, 1.0f, runs, 1, 1});
    if (c && a.gate) add({a.p_c, nullptr, a.w_post, dgate, a.scale, per, (int)a.gates, 1});
    if (c && a.w_post) add({a.p_c, a.gate, nullptr, dw_post, a.scale, runs, 1, per});
    if (a.p_post) add({a.p_post, nullptr, nullptr, dw_post, 1.0f, runs, 1, 1});
    if (!nj) return MXC_OK;
    j.d = a.d;
    norm_join_kernel<<<dim3((a.d + 31) / 32, (unsigned)nrows), 1024, 0, s>>>(j);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_HIP;
}

}  // namespace mxc
