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
// What bounds both is memory: a row is read once and held in registers (16
// values of each tensor a thread), with two sums over the row forward (Y's
// square, then H's) and two rounds of sums backward (the second one needs dX).
// A workgroup takes a run of consecutive rows, so the weights and the gate are
// loaded once a run; backward, its column sums stay in registers until the
// run's end and are added over the workgroups by a second kernel, in order.
// All sums and statistics are fp32.
#include "mx_internal.h"
#include "norm.h"

namespace mxc {
namespace {

constexpr int NV = NORM_VALS;     // values of a row a thread holds

template <typename T, int V>
__device__ __forceinline__ void ld(const T* p, float* o) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (V == 4) {
            const float4 u = *(const float4*)p;
            o[0] = u.x; o[1] = u.y; o[2] = u.z; o[3] = u.w;
        } else {
            o[0] = *p;
        }
    } else if constexpr (V == 8) {
        const uint4 u = *(const uint4*)p;
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int k = 0; k < 4; k++) {
            o[2 * k] = __uint_as_float(w[k] << 16);
            o[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    } else {
        o[0] = __uint_as_float((uint32_t)*(const uint16_t*)p << 16);
    }
}
template <typename T, int V>
__device__ __forceinline__ void st(T* p, const float* v) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (V == 4) *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
        else *p = v[0];
    } else if constexpr (V == 8) {
        *(uint4*)p = make_uint4(bf16_pack2(v[0], v[1]), bf16_pack2(v[2], v[3]), bf16_pack2(v[4], v[5]),
                                bf16_pack2(v[6], v[7]));
    } else {
        *(uint16_t*)p = (uint16_t)bf16_bits(v[0]);
    }
}
// V consecutive fp32 parameters
template <int V>
__device__ __forceinline__ void ldp(const float* p, float* o) {
    if constexpr (V == 8) {
        ld<float, 4>(p, o);
        ld<float, 4>(p + 4, o + 4);
    } else {
        ld<float, V>(p, o);
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
        const int wave = threadIdx.x >> 6;
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
            for (int k = 0; k < K; k++) v[k] += red[w * K + k];
    }
}

// The value q of a thread is column (q / V) * TPR * V + t * V + q % V.
template <int V, int TPR, class F>
__device__ __forceinline__ void columns(int d, int t, F&& f) {
#pragma unroll
    for (int i = 0; i < NV / V; i++) {
        const int c = (i * TPR + t) * V;
        if (i * TPR * V < d && c < d) f(i * V, c);
    }
}

template <typename T, int V, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_fwd_kernel(const NormArgs a) {
    constexpr int RL = TPR < 256 ? 256 / TPR : 1;             // rows a workgroup takes at a time
    __shared__ float red[2][TPR / 64];
    int par = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR, d = a.d;
    const long long first = (long long)blockIdx.x * a.run, last = min(first + a.run, a.rows);
    float wp[NV], wq[NV], g[NV];
    columns<V, TPR>(d, t, [&](int q, int c) {
        if (a.w_post) ldp<V>(a.w_post + c, wp + q);
        if (a.w_pre) ldp<V>(a.w_pre + c, wq + q);
    });
    long long gate = -1;
    for (long long r = first + rl; r < last; r += RL) {
        const long long gr = a.gate ? r / a.gate_rows : 0;
        if (gr != gate) {                                     // the weights times s g, for this gate's rows
            gate = gr;
            columns<V, TPR>(d, t, [&](int q, int c) {
                float u[V];
                if (a.gate) ldp<V>(a.gate + gr * d + c, u);
#pragma unroll
                for (int e = 0; e < V; e++) g[q + e] = a.gate ? a.scale * u[e] : a.scale;
            });
        }
        float x[NV], y[NV], s[1] = {0.0f};
        columns<V, TPR>(d, t, [&](int q, int c) {
            ld<T, V>((const T*)a.x + r * a.ldx + c, x + q);
            ld<T, V>((const T*)a.y + r * a.ldy + c, y + q);
#pragma unroll
            for (int e = 0; e < V; e++) s[0] += y[q + e] * y[q + e];
        });
        float ry = 1.0f;
        if (a.w_post) {
            row_sum<TPR, 1>(s, red, par);
            ry = 1.0f / sqrtf(s[0] * a.inv_d + a.eps);
        }
        s[0] = 0.0f;
        columns<V, TPR>(d, t, [&](int q, int c) {
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float n = a.w_post ? y[q + e] * ry * wp[q + e] : y[q + e];
                x[q + e] += g[q + e] * n;
                s[0] += x[q + e] * x[q + e];
            }
            st<T, V>((T*)a.h + r * a.ldh + c, x + q);
        });
        if (a.w_pre) {
            row_sum<TPR, 1>(s, red, par);
            const float rh = 1.0f / sqrtf(s[0] * a.inv_d + a.eps);
            columns<V, TPR>(d, t, [&](int q, int c) {
                float u[V];
#pragma unroll
                for (int e = 0; e < V; e++) u[e] = x[q + e] * rh * wq[q + e];
                st<T, V>((T*)a.u + r * a.ldu + c, u);
            });
        }
    }
}

// The workgroups cover the rows in runs that do not cross a gate's rows
// (runs_per_gate of them a gate), or take gates_per_run whole gates each.
template <typename T, int V, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_bwd_kernel(const NormArgs a) {
    constexpr int RL = TPR < 256 ? 256 / TPR : 1;
    __shared__ float red[2][TPR / 64 * 3];
    int par = 0;
    __shared__ float col[RL > 1 ? RL * NV * TPR : 1];
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR, d = a.d;
    float wp[NV], wq[NV], g[NV], s_pre[NV], s_post[NV], s_gate[NV];
#pragma unroll
    for (int q = 0; q < NV; q++) wp[q] = 1.0f, wq[q] = 0.0f, g[q] = s_pre[q] = s_post[q] = s_gate[q] = 0.0f;
    columns<V, TPR>(d, t, [&](int q, int c) {
        if (a.w_post) ldp<V>(a.w_post + c, wp + q);
        if (a.w_pre) ldp<V>(a.w_pre + c, wq + q);
    });
    // a thread's column sums, added over the workgroup's rows, to dst[0 .. d)
    auto flush = [&](const float* v, float* dst) {
        if constexpr (RL > 1) {
            __syncthreads();
#pragma unroll
            for (int q = 0; q < NV; q++) col[(rl * NV + q) * TPR + t] = v[q];
            __syncthreads();
            if (rl == 0) {
                columns<V, TPR>(d, t, [&](int q, int c) {
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        float u = 0.0f;
#pragma unroll
                        for (int l = 0; l < RL; l++) u += col[(l * NV + q + e) * TPR + t];
                        dst[c + e] = u;
                    }
                });
            }
        } else {
            columns<V, TPR>(d, t, [&](int q, int c) {
#pragma unroll
                for (int e = 0; e < V; e++) dst[c + e] = v[q + e];
            });
        }
    };
    const long long bid = blockIdx.x;
    // gates [g0, g1) of gate_rows rows each; a run inside one gate takes its
    // rows [o0, o1)
    const long long g0 = a.runs_per_gate > 1 ? bid / a.runs_per_gate : bid * a.gates_per_run;
    const long long g1 = a.runs_per_gate > 1 ? g0 + 1 : min(g0 + a.gates_per_run, a.gates);
    const long long o0 = a.runs_per_gate > 1 ? (bid - g0 * a.runs_per_gate) * a.run : 0;
    const long long o1 = a.runs_per_gate > 1 ? min(o0 + a.run, a.gate_rows) : a.gate_rows;
    for (long long gr = g0; gr < g1; gr++) {
        columns<V, TPR>(d, t, [&](int q, int c) {
            float u[V];
            if (a.gate) ldp<V>(a.gate + gr * d + c, u);
#pragma unroll
            for (int e = 0; e < V; e++) g[q + e] = a.gate ? a.scale * u[e] : a.scale;
        });
        for (long long r = gr * a.gate_rows + o0 + rl; r < gr * a.gate_rows + o1; r += RL) {
            float x[NV], y[NV], h[NV], du[NV], s[3] = {0.0f, 0.0f, 0.0f};
            columns<V, TPR>(d, t, [&](int q, int c) {
                ld<T, V>((const T*)a.x + r * a.ldx + c, x + q);          // dH
                ld<T, V>((const T*)a.y + r * a.ldy + c, y + q);
                if (a.w_pre) {
                    ld<T, V>((const T*)a.h + r * a.ldh + c, h + q);
                    ld<T, V>((const T*)a.u + r * a.ldu + c, du + q);     // dU
                }
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
            columns<V, TPR>(d, t, [&](int q, int c) {
#pragma unroll
                for (int e = 0; e < V; e++) {
                    if (a.w_pre) {
                        const float hh = h[q + e] * rh;
                        x[q + e] += rh * (du[q + e] * wq[q + e] - hh * mh);
                        s_pre[q + e] += du[q + e] * hh;
                    }
                    const float yh = y[q + e] * ry, b = g[q + e] * x[q + e];
                    s_gate[q + e] += a.scale * x[q + e] * (yh * wp[q + e]);
                    s_post[q + e] += b * yh;
                    m[0] += b * wp[q + e] * yh;
                    y[q + e] = yh;
                }
                st<T, V>((T*)a.dx + r * a.lddx + c, x + q);
            });
            float my = 0.0f;
            if (a.w_post) {
                row_sum<TPR, 1>(m, red, par);
                my = m[0] * a.inv_d;
            }
            columns<V, TPR>(d, t, [&](int q, int c) {
                float o[V];
#pragma unroll
                for (int e = 0; e < V; e++) o[e] = ry * (g[q + e] * x[q + e] * wp[q + e] - y[q + e] * my);
                st<T, V>((T*)a.dy + r * a.lddy + c, o);
            });
        }
        if (a.gate) {
            flush(s_gate, a.p_gate + (a.runs_per_gate > 1 ? bid : gr) * d);
#pragma unroll
            for (int q = 0; q < NV; q++) s_gate[q] = 0.0f;
        }
    }
    if (a.w_pre) flush(s_pre, a.p_pre + bid * d);
    if (a.w_post) flush(s_post, a.p_post + bid * d);
}

// dst[k][c] = sum of n consecutive partial rows, in a fixed order: 32 columns a
// workgroup, 32 threads a column, each taking every 32nd row, four loads at a
// time.
struct JoinArgs {
    const float* src[3];
    float* dst[3];
    int n[3], rows[3];            // partial rows of a result row, result rows
    int d;
};
__global__ __launch_bounds__(1024) void norm_join_kernel(const JoinArgs a) {
    __shared__ float red[32][33];
    int job = 0, row = blockIdx.y;
    while (row >= a.rows[job]) row -= a.rows[job++];
    const int x = threadIdx.x & 31, l = threadIdx.x >> 5, c = blockIdx.x * 32 + x, n = a.n[job];
    const float* p = a.src[job] + (size_t)row * n * a.d + min(c, a.d - 1);
    float s = 0.0f;
    for (int k = l; k < n; k += 128) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; q++) v[q] = k + 32 * q < n ? p[(size_t)(k + 32 * q) * a.d] : 0.0f;
        s += (v[0] + v[1]) + (v[2] + v[3]);
    }
    red[l][x] = s;
    __syncthreads();
    if (l == 0) {
#pragma unroll
        for (int k = 1; k < 32; k++) s += red[k][x];
        if (c < a.d) a.dst[job][(size_t)row * a.d + c] = s;
    }
}

template <typename T, int V>
void launch_rows(const NormArgs& a, bool bwd, int tpr, unsigned grid, hipStream_t s) {
    const dim3 b(tpr < 256 ? 256 : tpr);
    if (bwd) {
        if (tpr == 64) norm_bwd_kernel<T, V, 64><<<grid, b, 0, s>>>(a);
        else if (tpr == 256) norm_bwd_kernel<T, V, 256><<<grid, b, 0, s>>>(a);
        else norm_bwd_kernel<T, V, 512><<<grid, b, 0, s>>>(a);
    } else {
        if (tpr == 64) norm_fwd_kernel<T, V, 64><<<grid, b, 0, s>>>(a);
        else if (tpr == 256) norm_fwd_kernel<T, V, 256><<<grid, b, 0, s>>>(a);
        else norm_fwd_kernel<T, V, 512><<<grid, b, 0, s>>>(a);
    }
}

int launch(const NormArgs& a, bool bwd, bool bf16, bool vec, unsigned grid, hipStream_t s) {
    const int tpr = norm_tpr(a.d);
    if (bf16) {
        if (vec) launch_rows<__bf16, 8>(a, bwd, tpr, grid, s);
        else launch_rows<__bf16, 1>(a, bwd, tpr, grid, s);
    } else {
        if (vec) launch_rows<float, 4>(a, bwd, tpr, grid, s);
        else launch_rows<float, 1>(a, bwd, tpr, grid, s);
    }
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_HIP;
}

// Runs of the backward pass: about NORM_RUNS workgroups, none crossing a gate.
void plan_runs(NormArgs& a) {
    const long long rl = norm_tpr(a.d) < 256 ? 256 / norm_tpr(a.d) : 1;
    if (a.gates >= NORM_RUNS) {
        a.runs_per_gate = 1;
        a.gates_per_run = (a.gates + NORM_RUNS - 1) / NORM_RUNS;
        a.run = a.gate_rows;
        a.runs = (a.gates + a.gates_per_run - 1) / a.gates_per_run;
    } else {
        const long long want = std::max<long long>(1, NORM_RUNS / a.gates);
        a.run = std::max<long long>(rl, (a.gate_rows + want - 1) / want);
        a.runs_per_gate = (a.gate_rows + a.run - 1) / a.run;
        a.gates_per_run = 1;
        a.runs = a.gates * a.runs_per_gate;
    }
}

}  // namespace

int launch_norm_fwd(NormArgs a, bool bf16, bool vec, hipStream_t s) {
    const long long rl = norm_tpr(a.d) < 256 ? 256 / norm_tpr(a.d) : 1;
    a.run = std::max<long long>(rl, (a.rows + NORM_FWD_RUNS - 1) / NORM_FWD_RUNS);
    return launch(a, false, bf16, vec, (unsigned)((a.rows + a.run - 1) / a.run), s);
}

size_t norm_bwd_workspace(long long rows, int d, long long gates, bool gate, bool post, bool pre) {
    NormArgs a;
    a.d = d; a.rows = rows; a.gates = gates; a.gate_rows = rows / gates;
    plan_runs(a);
    const long long n = (post ? a.runs : 0) + (pre ? a.runs : 0) + (gate && a.runs_per_gate > 1 ? a.runs : 0);
    return a.runs == 1 ? 0 : (size_t)n * d * sizeof(float);
}

int launch_norm_bwd(NormArgs a, bool bf16, bool vec, float* dw_pre, float* dw_post, float* dgate, void* ws,
                    hipStream_t s) {
    plan_runs(a);
    const bool one = a.runs == 1;                 // a single workgroup writes the results itself
    float* p = (float*)ws;
    auto take = [&](float* dst) {
        if (one) return dst;
        float* q = p;
        p += (size_t)a.runs * a.d;
        return q;
    };
    a.p_pre = a.w_pre ? take(dw_pre) : nullptr;
    a.p_post = a.w_post ? take(dw_post) : nullptr;
    a.p_gate = a.gate ? (a.runs_per_gate > 1 ? take(dgate) : dgate) : nullptr;
    int rc = launch(a, true, bf16, vec, (unsigned)a.runs, s);
    if (rc || one) return rc;
    JoinArgs j;
    int nj = 0, nrows = 0;
    auto add = [&](const float* src, float* dst, long long n, long long rows) {
        j.src[nj] = src; j.dst[nj] = dst; j.n[nj] = (int)n; j.rows[nj] = (int)rows;
        nj++;
        nrows += (int)rows;
    };
    if (a.w_pre) add(a.p_pre, dw_pre, a.runs, 1);
    if (a.w_post) add(a.p_post, dw_post, a.runs, 1);
    if (a.gate && a.runs_per_gate > 1) add(a.p_gate, dgate, a.runs_per_gate, a.gates);
    if (!nj) return MXC_OK;
    for (int k = nj; k < 3; k++) { j.src[k] = j.src[0]; j.dst[k] = j.dst[0]; j.n[k] = j.rows[k] = 0; }
    j.d = a.d;
    norm_join_kernel<<<dim3((a.d + 31) / 32, nrows), 1024, 0, s>>>(j);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_HIP;
}

}  // namespace mxc
