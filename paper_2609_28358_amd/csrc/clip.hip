// clip.hip -- the Euclidean norm of many tensors together and the tensors
// scaled to at most a given norm:
//   norm = sqrt(sum over all tensors of g^2),   out = g min(1, max_norm / (norm + 1e-6))
// One read of everything for the norm, one read and one write for the scaling;
// memory bounds both.  The squares are added in fp64 (neither overflow nor
// underflow of a finite gradient's square, and the order of the additions
// cannot be seen in an fp32 norm): at most 16 fp64 operations per 16 bytes,
// far from that unit's rate.  A launch takes the descriptors of up to
// CLIP_TENSORS tensors as kernel arguments; a workgroup finds the tensor of
// its chunk by counting, lane by lane, the tensors that begin no later.  Each workgroup of the norm
// leaves one partial sum; every workgroup of the scaling adds all of them, in
// the same order, so the result does not depend on timing and there is no
// third launch.  Other inputs in between, each pass waited for: 300 bf16 tensors of
// 1.15 GB together norm 196 us (5.9 TB/s; a copy of 2 GiB reaches 5.0), scaling 494
// (4.7 TB/s); 60 fp32 ones of 19 MB 8.0 and 11.1 us.  All launches
// together have CLIP_PARTS workgroups, one a partial sum: the more tensors, the
// fewer workgroups a launch (2000 tensors 409, 65536 13).
#include "mx_internal.h"
#include "clip.h"

namespace mxc {
namespace {

constexpr int CT = 256;
constexpr int STEP = 4 * 16 * CT;      // bytes a workgroup has in flight: four vectors a thread

struct ClipArgs {
    const void* src[CLIP_TENSORS];
    void* dst[CLIP_TENSORS];
    long long n[CLIP_TENSORS];         // elements; bit 62: bf16
    int first[CLIP_TENSORS + 1];       // first chunk of each tensor
    int count, nblk, chunk;            // chunk: bytes a workgroup takes at a time, a multiple of STEP
};
constexpr long long BF16_BIT = 1ll << 62;

// the tensor of chunk k: the last one whose first chunk is not past k (empty
// tensors have no chunk and are stepped over), counted by the wave's lanes
__device__ __forceinline__ int find_tensor(const ClipArgs& a, int k) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int b = 0; b < a.count; b += 64)
        n += __popcll(__ballot(b + lane < a.count && a.first[min(b + lane, a.count)] <= k));
    return __builtin_amdgcn_readfirstlane(n - 1);
}

// 16 bytes at any element's address: global memory takes unaligned vectors.
struct __attribute__((packed, aligned(2))) Vec16 {
    uint32_t w[4];
};

// body(16-byte offset in the chunk) for a workgroup's vectors, four at a time
// and independent of each other, then tail(first byte, last byte) for what is left
template <class Body, class Tail>
__device__ __forceinline__ void vectors(int len, Body&& body, Tail&& tail) {
    int o = threadIdx.x * 16;
    for (; o + STEP - 16 * CT + 16 <= len; o += STEP) body(o, std::integral_constant<int, 4>{});
    for (; o + 16 <= len; o += 16 * CT) body(o, std::integral_constant<int, 1>{});
    if (o < len) tail(o, min(o + 16, len));
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < CT / 64; w++) v += red[w];
    return v;
}

// 16 bytes: 4 fp32 or 8 bf16
__device__ __forceinline__ double squares(const Vec16& u, bool bf) {
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        if (bf) {
            const double lo = __uint_as_float(u.w[k] << 16), hi = __uint_as_float(u.w[k] & 0xFFFF0000u);
            s += lo * lo;
            s += hi * hi;
        } else {
            const double v = __uint_as_float(u.w[k]);
            s += v * v;
        }
    }
    return s;
}

__global__ __launch_bounds__(CT) void clip_norm_kernel(const ClipArgs a, double* __restrict__ part) {
    __shared__ double red[CT / 64];
    double s = 0.0;
    const int chunks = a.first[a.count];
    for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int t = find_tensor(a, k);
        const bool bf = (a.n[t] & BF16_BIT) != 0;
        const long long n = a.n[t] & ~BF16_BIT, bytes = bf ? 2 * n : 4 * n;
        const long long b0 = (long long)(k - a.first[t]) * a.chunk;
        const uint8_t* p = (const uint8_t*)a.src[t] + b0;
        const int len = (int)min((long long)a.chunk, bytes - b0);
        vectors(len, [&](int o, auto num) {
            constexpr int N = decltype(num)::value;
            Vec16 u[N];
#pragma unroll
            for (int i = 0; i < N; i++) u[i] = *(const Vec16*)(p + o + i * 16 * CT);
#pragma unroll
            for (int i = 0; i < N; i++) s += squares(u[i], bf);
        }, [&](int o, int e) {
            for (; o < e; o += bf ? 2 : 4) {
                const double v = bf ? __uint_as_float((uint32_t)*(const uint16_t*)(p + o) << 16) : *(const float*)(p + o);
                s += v * v;
            }
        });
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(CT) void clip_scale_kernel(const ClipArgs a, const double* __restrict__ part, int nparts,
                                                        double max_norm, float* __restrict__ norm_out) {
    __shared__ double red[CT / 64];
    double s = 0.0;
    for (int i = threadIdx.x; i < nparts; i += CT) s += part[i];
    const double norm = sqrt(block_sum(s, red));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const double ratio = max_norm / (norm + 1e-6);
    const float c = (float)(ratio >= 1.0 ? 1.0 : ratio);       // NaN stays NaN
    const int chunks = a.first[a.count];
    // from the back: what the norm read last is still in the last-level cache
    for (int k = chunks - 1 - (int)blockIdx.x; k >= 0; k -= gridDim.x) {
        const int t = find_tensor(a, k);
        const bool bf = (a.n[t] & BF16_BIT) != 0;
        if (a.src[t] == a.dst[t] && c == 1.0f) continue;       // already what it is scaled to
        const long long n = a.n[t] & ~BF16_BIT, bytes = bf ? 2 * n : 4 * n;
        const long long b0 = (long long)(k - a.first[t]) * a.chunk;
        const uint8_t* p = (const uint8_t*)a.src[t] + b0;
        uint8_t* d = (uint8_t*)a.dst[t] + b0;
        // non-temporal where the vectors are aligned: 60 tensors, other inputs in
        // between, both launches, plain stores -> these, and in brackets with an update
        // that reads the results behind them, us: fp32 2 MB 8.6 -> 8.7 (15.0 -> 15.1), 8 MB
        // 13.8 -> 12.6 (26.3 -> 25.4), 40 MB 31.6 -> 28.2 (62.2 -> 59.5), 160 MB 103 -> 89
        // (225 -> 221), 640 MB 376 -> 357 (808 -> 800); bf16 alike; in place no difference
        const bool nt = ((uintptr_t)d & 15) == 0;
        const int len = (int)min((long long)a.chunk, bytes - b0);
        vectors(len, [&](int o, auto num) {
            constexpr int N = decltype(num)::value;
            Vec16 u[N];
#pragma unroll
            for (int i = 0; i < N; i++) u[i] = *(const Vec16*)(p + o + i * 16 * CT);
#pragma unroll
            for (int i = 0; i < N; i++) {
                Vec16 r;
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const uint32_t w = u[i].w[q];
                    r.w[q] = bf ? bf16_pack2(__uint_as_float(w << 16) * c, __uint_as_float(w & 0xFFFF0000u) * c)
                                : __float_as_uint(__uint_as_float(w) * c);
                }
                if (nt) store_nt(d + o + i * 16 * CT, make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]));
                else *(Vec16*)(d + o + i * 16 * CT) = r;
            }
        }, [&](int o, int e) {
            for (; o < e; o += bf ? 2 : 4) {
                if (bf) *(uint16_t*)(d + o) =
                    (uint16_t)bf16_bits(__uint_as_float((uint32_t)*(const uint16_t*)(p + o) << 16) * c);
                else *(float*)(d + o) = *(const float*)(p + o) * c;
            }
        });
    }
}

}  // namespace

int launch_grad_clip(int count, const mxc_gtensor* t, bool scale, double max_norm, float* norm, void* ws,
                     hipStream_t s) {
    const int launches = std::max(1, (count + CLIP_TENSORS - 1) / CLIP_TENSORS);
    const int most = std::max(1, CLIP_PARTS / launches);
    // long chunks spread a workgroup's search over more bytes (200 tensors of 128
    // MB together 66 us by them, 69 by short ones), short ones fill the grid (60
    // tensors of 19 MB 15.8 us, 16.6 by long ones); either way a multiple of what
    // is in flight
    double total = 0.0;
    for (int i = 0; i < count; i++) total += (double)t[i].n * (t[i].dtype == MXC_BF16 ? 2 : 4);
    int at = 0;
    ClipArgs a;
    a.chunk = total > 64e6 ? 4 * STEP : STEP;
    auto table = [&](int l) {
        a.count = 0;
        a.first[0] = 0;
        for (int i = l * CLIP_TENSORS; i < count && i < (l + 1) * CLIP_TENSORS; i++) {
            const int bf = t[i].dtype == MXC_BF16;
            const int k = a.count++;
            a.src[k] = t[i].src;
            a.dst[k] = t[i].dst;
            a.n[k] = t[i].n | (bf ? BF16_BIT : 0);
            a.first[k + 1] = a.first[k] + (int)((t[i].n * (bf ? 2 : 4) + a.chunk - 1) / a.chunk);
        }
        if (a.count == 0) { a.count = 1; a.src[0] = a.dst[0] = nullptr; a.n[0] = 0; a.first[1] = 0; }
        a.nblk = std::max(1, std::min(most, a.first[a.count]));
    };
    for (int l = 0; l < launches; l++) {
        table(l);
        clip_norm_kernel<<<a.nblk, CT, 0, s>>>(a, (double*)ws + at);
        at += a.nblk;
        if (hipGetLastError() != hipSuccess) return MXC_ERR_HIP;
    }
    // without outputs, one workgroup writes the norm
    for (int l = scale ? launches - 1 : 0; l >= 0; l--) {
        table(l);
        if (!scale) a.count = 0, a.first[0] = 0;
        clip_scale_kernel<<<scale ? a.nblk : 1, CT, 0, s>>>(a, (const double*)ws, at, max_norm, l == 0 ? norm : nullptr);
        if (hipGetLastError() != hipSuccess) return MXC_ERR_HIP;
    }
    return MXC_OK;
}

}  // namespace mxc
