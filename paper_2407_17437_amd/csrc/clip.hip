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
#include <stdlib.h>
#include <string.h>
#include <type_traits>

#include "device.h"
#include "experts.h"

namespace nerva {
namespace {

// The arrays are cut into short chunks, and work-groups, as many as the GPU holds, take chunk after chunk, so that all of them together
// read one stretch of memory at a time.  (A long stretch for each work-group instead, all of the same length, keeps meeting in few
// memory channels: the norm and step of 135 M entries took 727 us that way, 600 so.)
constexpr int kClipThreads = 256;
constexpr int kClipWaves = kClipThreads / kWave;
constexpr int kNormThreads = 512;
constexpr int kNormLoads = 4;                      // 16-byte reads in flight per thread
constexpr int kNormChunk = 4 * kNormLoads * kNormThreads;
constexpr int kApplyLoads = 4;
constexpr int kPastLoads = 2;                      // of lists past the cache: four take more than 64 registers, and a wave of eight with them (535 us -> 566)
constexpr int kApplyBlocks = 2048;
constexpr int kFewEntries = 1 << 20;               // lists of so many and fewer are cut into chunks of a quarter
constexpr int kPartialMost = 2048;                 // more partial sums are first added up by a launch of their own
// Arrays per launch: they travel in the kernel's arguments, of which there may be 4 KiB.
constexpr int kApplyList = 104;

struct NormList {
    const float *grads[kNormList];
    int64_t counts[kNormList];
    int32_t first[kNormList + 1];                  // chunk that an array starts with, and one past the last
    int32_t n;
    double *partial;                               // of this launch
};

struct ApplyList {
    float *a[kApplyList];                          // weights, or scaled gradients
    float *v[kApplyList];
    const float *grads[kApplyList];
    int64_t counts[kApplyList];
    int32_t first[kApplyList + 1];
    int32_t n;
    const double *partial;
    int32_t n_partial;
    float lr, momentum, max_norm;
    int32_t nesterov;
    float *norm_out;
};
static_assert(sizeof(NormList) <= 4096 && sizeof(ApplyList) <= 4096, "kernel arguments");

// array of a chunk: the last that does not start behind it
template <typename List>
__device__ __forceinline__ int array_of(const List &l, int chunk)
{
    int lo = 0, hi = l.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= chunk) lo = mid;
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
    double s[2] = {0, 0};
    for (int back = blockIdx.x; back < l.first[l.n]; back += gridDim.x) {
        const int chunk = l.first[l.n] - 1 - back, t = array_of(l, chunk);   // (from the last one on: see kCacheBytes)
        const int64_t from = static_cast<int64_t>(chunk - l.first[t]) * kNormChunk;
        const int n = static_cast<int>(min(l.counts[t] - from, static_cast<int64_t>(kNormChunk)));
        const float *g = l.grads[t] + from;
        int i = 4 * threadIdx.x;
        if (n == kNormChunk) {
            float4 x[kNormLoads];
#pragma unroll
            for (int u = 0; u < kNormLoads; ++u) x[u] = ld4(g + i + u * 4 * kNormThreads);
#pragma unroll
            for (int u = 0; u < kNormLoads; ++u) s[u & 1] = add_squares(s[u & 1], x[u]);
        } else {
            for (; i + 3 < n; i += 4 * kNormThreads) s[0] = add_squares(s[0], ld4(g + i));
            for (; i < n; ++i) s[1] = fma(static_cast<double>(g[i]), static_cast<double>(g[i]), s[1]);   // (the array's last one to three: one thread has them)
        }
    }
    const double sum = block_sum(s[0] + s[1], lds, kNormThreads / kWave);
    if (threadIdx.x == 0) l.partial[blockIdx.x] = sum;
}

// the partial sums' sum, the same bits in every work-group (few of them: every wave adds up all, and none waits for another)
__device__ __forceinline__ double sum_of(const double *partial, int n, double *lds)
{
    if (n <= kWave) {
        const int lane = threadIdx.x & (kWave - 1);
        double s = lane < n ? partial[lane] : 0.0;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) s += __shfl_xor(s, d, kWave);
        return s;
    }
    double s = 0;
    for (int i = threadIdx.x; i < n; i += kClipThreads) s += partial[i];
    return block_sum(s, lds, kClipWaves);
}

__global__ __launch_bounds__(kClipThreads) void norm_finish_kernel(const double *partial, int n, double *sum_out, float *norm_out)
{
    __shared__ double lds[kClipWaves];
    const double sum = sum_of(partial, n, lds);
    if (threadIdx.x != 0) return;
    if (sum_out) *sum_out = sum;
    if (norm_out) *norm_out = static_cast<float>(sqrt(sum));
}

__device__ __forceinline__ void step4(float4 &w, float4 &v, float4 g, float c, const ApplyList &l)
{
    momentum_step(w.x, v.x, c * g.x, l.lr, l.momentum, l.nesterov);
    momentum_step(w.y, v.y, c * g.y, l.lr, l.momentum, l.nesterov);
    momentum_step(w.z, v.z, c * g.z, l.lr, l.momentum, l.nesterov);
    momentum_step(w.w, v.w, c * g.w, l.lr, l.momentum, l.nesterov);
}

// Of arrays that the 256 MiB of Infinity Cache cannot hold, weights and momentum buffers go past it, and the norm is taken from the last array to
// the first, so that the step, which goes forward, still finds the gradients there that were read last: 135 M entries 642 us -> 554
// (forward and past the cache 579, backward alone 639; now 535).  Smaller ones may still be there from the step before, and
// past the cache 4.6 M entries took 24.3 us instead of 22.5 (now 20.7).
constexpr int64_t kCacheBytes = 256ll << 20;
template <bool kPast>
__device__ __forceinline__ float4 load4(const float *p)
{
    if constexpr (!kPast) return ld4(p);
    const v4f_any x = __builtin_nontemporal_load(reinterpret_cast<const v4f_any *>(p));
    return make_float4(x.x, x.y, x.z, x.w);
}
template <bool kPast>
__device__ __forceinline__ void store4(float *p, float4 v)
{
    if constexpr (!kPast) return st4(p, v);
    const v4f_any x = {v.x, v.y, v.z, v.w};
    __builtin_nontemporal_store(x, reinterpret_cast<v4f_any *>(p));
}

template <bool kUpdate, bool kPast, int kLoads>
__global__ __launch_bounds__(kClipThreads) void clip_apply_kernel(const ApplyList l)
{
    __shared__ double lds[kClipWaves];
    constexpr int kStep = 4 * kClipThreads, kChunk = kLoads * kStep;
    const int i = 4 * threadIdx.x;
    const float *g = nullptr;
    float *a = nullptr, *v = nullptr;
    int n = 0;   // entries of the chunk
    float4 ww[kLoads], vv[kLoads], gg[kLoads];
    auto load = [&](int chunk) {
        const int t = array_of(l, chunk);
        const int64_t from = static_cast<int64_t>(chunk - l.first[t]) * kChunk;
        n = static_cast<int>(min(l.counts[t] - from, static_cast<int64_t>(kChunk)));
        g = l.grads[t] + from;
        a = l.a[t] + from;
        if constexpr (kUpdate) v = l.v[t] + from;
        auto all = [&](auto whole) {   // (a whole chunk without a look at its end)
#pragma unroll
            for (int u = 0; u < kLoads; ++u)
                if (whole.value || i + u * kStep + 3 < n) {
                    gg[u] = ld4(g + i + u * kStep);
                    if constexpr (kUpdate) {
                        ww[u] = load4<kPast>(a + i + u * kStep);
                        vv[u] = load4<kPast>(v + i + u * kStep);
                    }
                }
        };
        if (n == kChunk) all(std::true_type{});
        else all(std::false_type{});
    };
    load(blockIdx.x);   // (on its way while the norm is added up)

    const double norm = sqrt(sum_of(l.partial, l.n_partial, lds));
    const float norm32 = static_cast<float>(norm);
    if (blockIdx.x == 0 && threadIdx.x == 0 && l.norm_out) *l.norm_out = norm32;
    if (!(norm32 <= 3.402823466e38f)) return;   // no factor makes such gradients finite: nothing is changed
    const float c = norm > l.max_norm ? static_cast<float>(l.max_norm / norm) : 1.f;

    for (int chunk = blockIdx.x;;) {
        if (kUpdate || c != 1.f || a != g) {
            auto all = [&](auto whole) {
#pragma unroll
                for (int u = 0; u < kLoads; ++u)
                    if (whole.value || i + u * kStep + 3 < n) {
                        if constexpr (kUpdate) {
                            step4(ww[u], vv[u], gg[u], c, l);
                            store4<kPast>(v + i + u * kStep, vv[u]);
                            store4<kPast>(a + i + u * kStep, ww[u]);
                        } else {
                            st4(a + i + u * kStep, make_float4(c * gg[u].x, c * gg[u].y, c * gg[u].z, c * gg[u].w));
                        }
                    }
            };
            if (n == kChunk) all(std::true_type{});
            else all(std::false_type{});
            const int last = (n & ~3) + threadIdx.x;   // an array's last one to three
            if (last < n) {
                if constexpr (kUpdate) {
                    float w1 = a[last], v1 = v[last];
                    momentum_step(w1, v1, c * g[last], l.lr, l.momentum, l.nesterov);
                    v[last] = v1;
                    a[last] = w1;
                } else {
                    a[last] = c * g[last];
                }
            }
        }
        chunk += gridDim.x;
        if (chunk >= l.first[l.n]) break;
        load(chunk);
    }
}

// whether arrays [a, a + n) and [b, b + m) share an entry
bool overlap(const float *a, int64_t n, const float *b, int64_t m) { return a < b + m && b < a + n; }

// Arrays met so far, by their addresses: a table with room for twice as many as may come, searched from where an address's hash says.
struct Met {
    static constexpr int64_t kInline = 512;   // (lists of up to 256 arrays: no heap memory)
    const float *inline_[kInline], **table = inline_;
    int64_t size = kInline;
    Met() = default;
    Met(const Met &) = delete;
    ~Met() { if (table != inline_) free(table); }
    bool reserve(int64_t most)
    {
        while (size < 2 * most) size *= 2;
        if (size > kInline) table = static_cast<const float **>(malloc(static_cast<size_t>(size) * sizeof *table));
        if (table) memset(table, 0, static_cast<size_t>(size) * sizeof *table);
        else table = inline_;
        return size == kInline || table != inline_;
    }
    // p's place, which holds p if it came before, else null until p is put there
    const float **find(const float *p) const
    {
        int64_t i = static_cast<int64_t>(reinterpret_cast<uint64_t>(p) * UINT64_C(0x9E3779B97F4A7C15) >> 32) & (size - 1);
        while (table[i] && table[i] != p) i = (i + 1) & (size - 1);
        return table + i;
    }
};

}  // namespace

// Partial sums of all arrays; *n_partial receives how many there are, at most kPartialMost, from *partial on.
static hipError_t launch_partial(const ArrayList &l, double **partial, int32_t *n_partial, hipStream_t s)
{
    int32_t done = 0;
    for (int32_t end = l.n; end > 0;) {   // stretches of the list, the last one first
        const int32_t from = end > kNormList ? end - kNormList : 0;
        NormList a;
        a.n = 0;
        int64_t chunks = 0;
        for (int32_t t = from; t < end; ++t) {
            if (l.counts[t] == 0) continue;
            a.grads[a.n] = l.grads[t];
            a.counts[a.n] = l.counts[t];
            a.first[a.n++] = static_cast<int32_t>(chunks);
            chunks += (l.counts[t] + kNormChunk - 1) / kNormChunk;
        }
        end = from;
        if (chunks == 0) continue;
        a.first[a.n] = static_cast<int32_t>(chunks);
        a.partial = *partial + done;
        const int blocks = static_cast<int>(chunks < kNormBlocks ? chunks : kNormBlocks);
        hipLaunchKernelGGL(norm_partial_kernel, dim3(blocks), dim3(kNormThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        done += blocks;
    }
    if (done > kPartialMost) {
        hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kClipThreads), 0, s, *partial, done, *partial + done, static_cast<float *>(nullptr));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        *partial += done;
        done = 1;
    }
    *n_partial = done;
    return hipSuccess;
}

static hipError_t launch_finish(const double *partial, int32_t n, float *norm_out, hipStream_t s)
{
    if (!norm_out) return hipSuccess;
    hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kClipThreads), 0, s, partial, n, static_cast<double *>(nullptr), norm_out);
    return hipGetLastError();
}

hipError_t launch_norm(const ArrayList &l, double *partial, float *norm_out, hipStream_t s)
{
    int32_t n = 0;
    const hipError_t e = launch_partial(l, &partial, &n, s);
    return e != hipSuccess ? e : launch_finish(partial, n, norm_out, s);
}

hipError_t launch_clipped(const ArrayList &l, const ClipArgs &c, hipStream_t s)
{
    int32_t n_partial = 0;
    double *partial = c.partial;
    // Gradients that are clipped in place: where one comes again it is clipped already.
    int64_t in_place = 0;
    if (l.clipped)
        for (int32_t t = 0; t < l.n; ++t) in_place += l.clipped[t] == l.grads[t];
    Met met;
    if (in_place > 0 && !met.reserve(in_place)) return hipErrorOutOfMemory;
    hipError_t e = launch_partial(l, &partial, &n_partial, s);
    if (e != hipSuccess) return e;
    if (n_partial == 0) return launch_finish(partial, 0, c.norm_out, s);
    float *const *out = l.values ? l.values : l.clipped;
    float *norm_out = c.norm_out;
    int64_t entries = 0;
    for (int32_t t = 0; t < l.n; ++t) entries += l.counts[t];
    const bool past = 20 * entries > kCacheBytes, few = entries <= kFewEntries;
    const int64_t chunk = 4 * kClipThreads * (few ? 1 : l.values && past ? kPastLoads : kApplyLoads);
    for (int32_t t = 0; t < l.n;) {
        ApplyList a;
        a.n = 0;
        int64_t chunks = 0;
        for (; t < l.n && a.n < kApplyList; ++t) {
            const int64_t m = l.counts[t];
            if (m == 0) continue;
            const float **first_time = in_place > 0 && out[t] == l.grads[t] ? met.find(out[t]) : nullptr;
            if (first_time && *first_time) continue;
            // an array that is in the list twice is stepped twice, one launch after the other
            bool again = false;
            for (int32_t i = 0; i < a.n && !again; ++i)
                again = overlap(a.a[i], a.counts[i], out[t], m) || (l.values && overlap(a.v[i], a.counts[i], l.velocities[t], m));
            if (again) break;
            if (first_time) *first_time = out[t];
            a.a[a.n] = out[t];
            a.v[a.n] = l.values ? l.velocities[t] : nullptr;
            a.grads[a.n] = l.grads[t];
            a.counts[a.n] = m;
            a.first[a.n++] = static_cast<int32_t>(chunks);
            chunks += (m + chunk - 1) / chunk;
        }
        if (chunks == 0) break;
        a.first[a.n] = static_cast<int32_t>(chunks);
        a.partial = partial;
        a.n_partial = n_partial;
        a.lr = c.lr;
        a.momentum = c.momentum;
        a.max_norm = c.max_norm;
        a.nesterov = c.nesterov;
        a.norm_out = norm_out;
        norm_out = nullptr;
        const dim3 grid(static_cast<uint32_t>(chunks < kApplyBlocks ? chunks : kApplyBlocks));
        if (l.values && past) hipLaunchKernelGGL((clip_apply_kernel<true, true, kPastLoads>), grid, dim3(kClipThreads), 0, s, a);
        else if (l.values && !few) hipLaunchKernelGGL((clip_apply_kernel<true, false, kApplyLoads>), grid, dim3(kClipThreads), 0, s, a);
        else if (l.values) hipLaunchKernelGGL((clip_apply_kernel<true, false, 1>), grid, dim3(kClipThreads), 0, s, a);
        else if (!few) hipLaunchKernelGGL((clip_apply_kernel<false, false, kApplyLoads>), grid, dim3(kClipThreads), 0, s, a);
        else hipLaunchKernelGGL((clip_apply_kernel<false, false, 1>), grid, dim3(kClipThreads), 0, s, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace nerva
