// Global norm over many arrays of gradients, gradients clipped to a norm, and the momentum step on clipped gradients.
//
//     n = sqrt(sum over all arrays and entries of g^2),   c = min(1, max_norm / n),   g <- c g  or  the momentum step with c g
//
// Two kernels: the first leaves one partial sum per work-group, each work-group of the second adds all of them up in the same
// fixed order, so that all get the same bits whatever the order in which the first ones ran, and nothing needs a
// counter that someone would have to clear.
// Squares are added up in 64 bits: the square of any fp32 number is exact there and in range (1e-90 ... 1e77), so the
// norm neither overflows nor loses small entries beside large ones.  At 4 bytes read per entry the memory leaves some 80
// cycles per wave and entry, which the conversion and the 64-bit multiply-add do not fill.
#include "device.h"
#include "experts.h"

namespace nerva {
namespace {

constexpr int kClipThreads = 256;
constexpr int kClipWaves = kClipThreads / kWave;
constexpr int kNormThreads = 1024;
constexpr int kListMax = 64;                       // arrays per launch: they travel in the kernel's arguments
constexpr int64_t kChunkMin = 4 * kNormThreads;    // entries per work-group, at least
constexpr int32_t kApplyBlocks = 4096;
constexpr int64_t kApplyChunkMin = 4 * kClipThreads;

struct NormList {
    const float *grads[kListMax];
    int64_t counts[kListMax];
    int32_t first[kListMax + 1];                   // work-group that an array starts with
    int32_t n;
    int64_t chunk;                                 // entries per work-group, a multiple of 4
    double *partial;                               // of this launch
};

struct ApplyList {
    float *a[kListMax];                            // weights, or scaled gradients
    float *v[kListMax];
    const float *grads[kListMax];
    int64_t counts[kListMax];
    int32_t first[kListMax + 1];
    int32_t n;
    int64_t chunk;
    const double *partial;
    int32_t n_partial;
    float lr, momentum, max_norm;
    int32_t nesterov;
    float *norm_out;
};

// array that a work-group works on: the last whose first work-group is not behind it
template <typename List>
__device__ __forceinline__ int array_of(const List &l, int block)
{
    int lo = 0, hi = l.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= block) lo = mid;
        else hi = mid;
    }
    return lo;
}

// sum over a work-group of `waves` waves in one fixed order; every thread gets it
__device__ __forceinline__ double block_sum(double x, double *lds, int waves)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d, kWave);
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0;
    for (int w = 0; w < waves; ++w) s += lds[w];
    return s;
}

__device__ __forceinline__ double add_squares(double s, float4 g)
{
    s = fma(static_cast<double>(g.x), static_cast<double>(g.x), s);
    s = fma(static_cast<double>(g.y), static_cast<double>(g.y), s);
    s = fma(static_cast<double>(g.z), static_cast<double>(g.z), s);
    return fma(static_cast<double>(g.w), static_cast<double>(g.w), s);
}

__global__ __launch_bounds__(kNormThreads) void norm_partial_kernel(const NormList l)
{
    __shared__ double lds[kNormThreads / kWave];
    const int t = array_of(l, blockIdx.x);
    const int64_t from = (blockIdx.x - l.first[t]) * l.chunk;
    const int64_t left = l.counts[t] - from;
    const int64_t n = left < l.chunk ? left : l.chunk;
    const float *g = l.grads[t] + from;
    double s0 = 0, s1 = 0;
    int64_t i = 4 * static_cast<int64_t>(threadIdx.x);
    constexpr int64_t kStep = 4 * kNormThreads;
    for (; i + 3 * kStep + 3 < n; i += 4 * kStep) {
        const float4 a = ld4(g + i), b = ld4(g + i + kStep), c = ld4(g + i + 2 * kStep), d = ld4(g + i + 3 * kStep);
        s0 = add_squares(s0, a);
        s1 = add_squares(s1, b);
        s0 = add_squares(s0, c);
        s1 = add_squares(s1, d);
    }
    for (; i + 3 < n; i += kStep) s0 = add_squares(s0, ld4(g + i));
    for (; i < n; ++i) s1 = fma(static_cast<double>(g[i]), static_cast<double>(g[i]), s1);   // (the array's last one to three entries: one thread has them)
    s0 = block_sum(s0 + s1, lds, kNormThreads / kWave);
    if (threadIdx.x == 0) l.partial[blockIdx.x] = s0;
}

// The norm from the partial sums, the same bits in every work-group.
__device__ __forceinline__ double norm_of(const double *partial, int n, double *lds)
{
    double s = 0;
    for (int i = threadIdx.x; i < n; i += kClipThreads) s += partial[i];
    return sqrt(block_sum(s, lds, kClipWaves));
}

__global__ __launch_bounds__(kClipThreads) void norm_finish_kernel(const double *partial, int n, float *norm_out)
{
    __shared__ double lds[kClipWaves];
    const double norm = norm_of(partial, n, lds);
    if (threadIdx.x == 0) *norm_out = static_cast<float>(norm);
}

template <bool kUpdate>
__global__ __launch_bounds__(kClipThreads) void clip_apply_kernel(const ApplyList l)
{
    __shared__ double lds[kClipWaves];
    const double norm = norm_of(l.partial, l.n_partial, lds);
    const float norm32 = static_cast<float>(norm);
    if (blockIdx.x == 0 && threadIdx.x == 0 && l.norm_out) *l.norm_out = norm32;
    if (!(norm32 <= 3.402823466e38f)) return;   // no factor makes such gradients finite: nothing is changed
    const float c = norm > l.max_norm ? static_cast<float>(l.max_norm / norm) : 1.f;

    const int t = array_of(l, blockIdx.x);
    const int64_t from = (blockIdx.x - l.first[t]) * l.chunk;
    const int64_t left = l.counts[t] - from;
    const int64_t n = left < l.chunk ? left : l.chunk;
    const float *g = l.grads[t] + from;
    float *a = l.a[t] + from;
    constexpr int64_t kStep = 4 * kClipThreads;
    int64_t i = 4 * static_cast<int64_t>(threadIdx.x);
    if constexpr (kUpdate) {
        float *v = l.v[t] + from;
        for (; i + 3 < n; i += kStep) {
            float4 ww = ld4(a + i), vv = ld4(v + i);
            const float4 gg = ld4(g + i);
            momentum_step(ww.x, vv.x, c * gg.x, l.lr, l.momentum, l.nesterov);
            momentum_step(ww.y, vv.y, c * gg.y, l.lr, l.momentum, l.nesterov);
            momentum_step(ww.z, vv.z, c * gg.z, l.lr, l.momentum, l.nesterov);
            momentum_step(ww.w, vv.w, c * gg.w, l.lr, l.momentum, l.nesterov);
            st4(v + i, vv);
            st4(a + i, ww);
        }
        for (; i < n; ++i) {
            float ww = a[i], vv = v[i];
            momentum_step(ww, vv, c * g[i], l.lr, l.momentum, l.nesterov);
            v[i] = vv;
            a[i] = ww;
        }
    } else {
        if (c == 1.f && a == g) return;
        for (; i + 3 < n; i += kStep) {
            float4 gg = ld4(g + i);
            gg.x *= c;
            gg.y *= c;
            gg.z *= c;
            gg.w *= c;
            st4(a + i, gg);
        }
        for (; i < n; ++i) a[i] = c * g[i];
    }
}

// entries per work-group: at most `blocks` of them and one more for each array
int64_t chunk_of(const ArrayList &l, int32_t blocks, int64_t least)
{
    int64_t total = 0;
    for (int32_t t = 0; t < l.n; ++t) total += l.counts[t];
    const int64_t even = (total + blocks - 1) / blocks;
    return even <= least ? least : (even + 3) / 4 * 4;
}

// whether arrays [a, a + n) and [b, b + m) share an entry
bool overlap(const float *a, int64_t n, const float *b, int64_t m) { return a < b + m && b < a + n; }

}  // namespace

// partial sums of all arrays; returns how many there are in *n_partial
static hipError_t launch_partial(const ArrayList &l, double *partial, int32_t *n_partial, hipStream_t s)
{
    const int64_t chunk = chunk_of(l, kNormBlocks, kChunkMin);
    int32_t done = 0;
    for (int32_t t = 0; t < l.n;) {
        NormList a;
        a.n = 0;
        int32_t blocks = 0;
        for (; t < l.n && a.n < kListMax; ++t) {
            if (l.counts[t] == 0) continue;
            a.grads[a.n] = l.grads[t];
            a.counts[a.n] = l.counts[t];
            a.first[a.n++] = blocks;
            blocks += static_cast<int32_t>((l.counts[t] + chunk - 1) / chunk);
        }
        if (blocks == 0) break;
        a.first[a.n] = blocks;
        a.chunk = chunk;
        a.partial = partial + done;
        hipLaunchKernelGGL(norm_partial_kernel, dim3(blocks), dim3(kNormThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        done += blocks;
    }
    *n_partial = done;
    return hipSuccess;
}

static hipError_t launch_finish(const double *partial, int32_t n, float *norm_out, hipStream_t s)
{
    if (!norm_out) return hipSuccess;
    hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kClipThreads), 0, s, partial, n, norm_out);
    return hipGetLastError();
}

hipError_t launch_norm(const ArrayList &l, double *partial, float *norm_out, hipStream_t s)
{
    int32_t n = 0;
    const hipError_t e = launch_partial(l, partial, &n, s);
    return e != hipSuccess ? e : launch_finish(partial, n, norm_out, s);
}

hipError_t launch_clipped(const ArrayList &l, const ClipArgs &c, hipStream_t s)
{
    int32_t n_partial = 0;
    hipError_t e = launch_partial(l, c.partial, &n_partial, s);
    if (e != hipSuccess) return e;
    if (n_partial == 0) return launch_finish(c.partial, 0, c.norm_out, s);
    float *const *out = l.values ? l.values : l.clipped;
    const int64_t chunk = chunk_of(l, kApplyBlocks, kApplyChunkMin);
    float *norm_out = c.norm_out;
    for (int32_t t = 0; t < l.n;) {
        ApplyList a;
        a.n = 0;
        int32_t blocks = 0;
        for (; t < l.n && a.n < kListMax; ++t) {
            const int64_t m = l.counts[t];
            if (m == 0) continue;
            // an array that is in the list twice is stepped twice, one launch after the other
            bool again = false;
            for (int32_t i = 0; i < a.n && !again; ++i)
                again = overlap(a.a[i], a.counts[i], out[t], m) || (l.values && overlap(a.v[i], a.counts[i], l.velocities[t], m));
            if (again) break;
            a.a[a.n] = out[t];
            a.v[a.n] = l.values ? l.velocities[t] : nullptr;
            a.grads[a.n] = l.grads[t];
            a.counts[a.n] = m;
            a.first[a.n++] = blocks;
            blocks += static_cast<int32_t>((m + chunk - 1) / chunk);
        }
        if (blocks == 0) break;
        a.first[a.n] = blocks;
        a.chunk = chunk;
        a.partial = c.partial;
        a.n_partial = n_partial;
        a.lr = c.lr;
        a.momentum = c.momentum;
        a.max_norm = c.max_norm;
        a.nesterov = c.nesterov;
        a.norm_out = norm_out;
        norm_out = nullptr;
        if (l.values) hipLaunchKernelGGL((clip_apply_kernel<true>), dim3(blocks), dim3(kClipThreads), 0, s, a);
        else hipLaunchKernelGGL((clip_apply_kernel<false>), dim3(blocks), dim3(kClipThreads), 0, s, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace nerva
