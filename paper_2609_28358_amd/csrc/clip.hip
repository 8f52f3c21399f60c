// clip.hip -- the Euclidean norm of many tensors together and the tensors
// scaled to at most a given norm:
//   norm = sqrt(sum over all tensors of g^2),   out = g min(1, max_norm / (norm + 1e-6))
// One read of everything for the norm, one read and one write for the scaling;
// memory bounds both.  The squares are added in fp64 (neither overflow nor
// underflow of a finite gradient's square, and the order of the additions
// cannot be seen in an fp32 norm): at most 16 fp64 operations per 16 bytes,
// far from that unit's rate.  A launch takes the descriptors of up to
// CLIP_TENSORS tensors as kernel arguments; a workgroup finds the tensor of
// its chunk by bisection over the chunk counts.  Each workgroup of the norm
// leaves one partial sum; every workgroup of the scaling adds all of them, in
// the same order, so the result does not depend on timing and there is no
// third launch.
#include "mx_internal.h"
#include "clip.h"

namespace mxc {
namespace {

constexpr int CHUNK = 16384;           // bytes a workgroup takes at a time
constexpr int CT = 256;

struct ClipArgs {
    const void* src[CLIP_TENSORS];
    void* dst[CLIP_TENSORS];
    long long n[CLIP_TENSORS];         // elements; bit 62: bf16
    int first[CLIP_TENSORS + 1];       // first chunk of each tensor
    int count, nblk;
};
constexpr long long BF16_BIT = 1ll << 62;

// the tensor of chunk k: the last one whose first chunk is not past k (empty
// tensors have no chunk and are stepped over)
__device__ __forceinline__ int find_tensor(const ClipArgs& a, int k) {
    int lo = 0, hi = a.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= k) lo = mid;
        else hi = mid;
    }
    return lo;
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
__device__ __forceinline__ double squares(uint4 u, bool bf) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        if (bf) {
            const double lo = __uint_as_float(w[k] << 16), hi = __uint_as_float(w[k] & 0xFFFF0000u);
            s += lo * lo;
            s += hi * hi;
        } else {
            const double v = __uint_as_float(w[k]);
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
        const long long b0 = (long long)(k - a.first[t]) * CHUNK;
        const uint8_t* p = (const uint8_t*)a.src[t] + b0;
        const int len = (int)min((long long)CHUNK, bytes - b0);
#pragma unroll
        for (int i = 0; i < CHUNK / (16 * CT); i++) {
            const int o = (i * CT + threadIdx.x) * 16;
            if (o + 16 <= len) {
                s += squares(*(const uint4*)(p + o), bf);
            } else {
                for (int q = o; q < len; q += bf ? 2 : 4) {
                    const double v = bf ? __uint_as_float((uint32_t)*(const uint16_t*)(p + q) << 16) : *(const float*)(p + q);
                    s += v * v;
                }
            }
        }
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
    for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int t = find_tensor(a, k);
        const bool bf = (a.n[t] & BF16_BIT) != 0;
        if (a.src[t] == a.dst[t] && c == 1.0f) continue;       // already what it is scaled to
        const long long n = a.n[t] & ~BF16_BIT, bytes = bf ? 2 * n : 4 * n;
        const long long b0 = (long long)(k - a.first[t]) * CHUNK;
        const uint8_t* p = (const uint8_t*)a.src[t] + b0;
        uint8_t* o = (uint8_t*)a.dst[t] + b0;
        const int len = (int)min((long long)CHUNK, bytes - b0);
#pragma unroll
        for (int i = 0; i < CHUNK / (16 * CT); i++) {
            const int at = (i * CT + threadIdx.x) * 16;
            if (at + 16 <= len) {
                const uint4 u = *(const uint4*)(p + at);
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
                uint32_t r[4];
#pragma unroll
                for (int q = 0; q < 4; q++)
                    r[q] = bf ? bf16_pack2(__uint_as_float(w[q] << 16) * c, __uint_as_float(w[q] & 0xFFFF0000u) * c)
                              : __float_as_uint(__uint_as_float(w[q]) * c);
                *(uint4*)(o + at) = make_uint4(r[0], r[1], r[2], r[3]);
            } else {
                for (int q = at; q < len; q += bf ? 2 : 4) {
                    if (bf) *(uint16_t*)(o + q) =
                        (uint16_t)bf16_bits(__uint_as_float((uint32_t)*(const uint16_t*)(p + q) << 16) * c);
                    else *(float*)(o + q) = *(const float*)(p + q) * c;
                }
            }
        }
    }
}

}  // namespace

int launch_grad_clip(int count, const mxc_gtensor* t, bool scale, double max_norm, float* norm, void* ws,
                     hipStream_t s) {
    const int launches = std::max(1, (count + CLIP_TENSORS - 1) / CLIP_TENSORS);
    const int most = std::max(1, CLIP_PARTS / launches);
    int at = 0;
    ClipArgs a;
    auto table = [&](int l) {
        a.count = 0;
        a.first[0] = 0;
        for (int i = l * CLIP_TENSORS; i < count && i < (l + 1) * CLIP_TENSORS; i++) {
            const int bf = t[i].dtype == MXC_BF16;
            const int k = a.count++;
            a.src[k] = t[i].src;
            a.dst[k] = t[i].dst;
            a.n[k] = t[i].n | (bf ? BF16_BIT : 0);
            a.first[k + 1] = a.first[k] + (int)((t[i].n * (bf ? 2 : 4) + CHUNK - 1) / CHUNK);
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
    for (int l = 0; l < (scale ? launches : 1); l++) {
        table(l);
        if (!scale) a.first[a.count] = 0;
        clip_scale_kernel<<<scale ? a.nblk : 1, CT, 0, s>>>(a, (const double*)ws, at, max_norm, l == 0 ? norm : nullptr);
        if (hipGetLastError() != hipSuccess) return MXC_ERR_HIP;
    }
    return MXC_OK;
}

}  // namespace mxc
