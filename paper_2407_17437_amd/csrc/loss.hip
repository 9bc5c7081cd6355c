// Log-probabilities of labels under columns of logits, their sums over sequences of columns, the clipped policy loss with a KL term, and the
// loss of paired sequences; the losses with the gradient of the logits.
//
//     l = z_label - log sum exp z                              p = exp(z - log sum exp z)
//     policy:      r = exp(l - old),  q = exp(ref - l),  loss = sum_c w (-min(r A, clip(r, 1 - low, 1 + high) A) + beta (q - log q - 1))
//                  dl = w (-r A [not clipped] + beta (1 - q))
//     preference:  S = sum of l over a sequence,  x = beta ((S_c - R_c) - (S_r - R_r)),  loss = mean of (1 - t) log(1 + exp(-x)) + t log(1 + exp(x))
//                  dl = +-(sigmoid(x) - (1 - t)) beta / pairs
//     dz_i = dl ([i == label] - p_i)
//
// Bound by memory: the logits are read for the sum of exponentials and, where a work-group cannot hold a column, again for the gradient.  The first
// launch cuts the classes into chunks and leaves a maximum and a sum for each, from one pass with a running maximum; the second one, a thread per
// column, adds them up and does what a column needs (in 64 bits: log-probabilities are added up over sequences and compared with borders, and
// there are few of them); the last one writes the gradient.
#include <float.h>

#include <algorithm>

#include "columns.h"
#include "experts.h"
#include "loss.h"

namespace nerva {
namespace {

constexpr int kThreads = 256;
constexpr int kLanes = 6;              // log2 of the quads of a tile: 256 columns
constexpr int kLoads = 8;              // rows in flight per thread
constexpr int kColumns = 256;          // columns of a work-group that adds up chunks
constexpr int64_t kBlocks = 2048;      // work-groups that the classes are cut for

__device__ __forceinline__ float4 exp_of4(float4 x) { return make_float4(exp_of(x.x), exp_of(x.y), exp_of(x.z), exp_of(x.w)); }
__device__ __forceinline__ float4 max4(float4 a, float4 b) { return make_float4(fmaxf(a.x, b.x), fmaxf(a.y, b.y), fmaxf(a.z, b.z), fmaxf(a.w, b.w)); }

struct Shape {
    int lg, chunks, rows;              // rows of a chunk
    int32_t tiles;
};

// Running maximum and sum of a thread's rows of its four columns.  The maximum starts at the lowest number, not at -inf, so that no
// difference of two infinities arises where all logits are -inf; +inf and NaN make the sum NaN.
struct Running {
    float4 top, sum;
};
__device__ __forceinline__ void add_rows(Running &a, const float4 (&z)[kLoads])
{
    float4 top = a.top;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) top = max4(top, z[u]);
    float4 s = exp_of4(z[0] - top);
#pragma unroll
    for (int u = 1; u < kLoads; ++u) s = s + exp_of4(z[u] - top);
    a.sum = fma4(a.sum, exp_of4(a.top - top), s);
    a.top = top;
}
// over the threads with the same columns; the same in all of them
__device__ __forceinline__ Running join(Running a, int lg, float4 (*lds)[kThreads / kWave << kLanes])
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, q = threadIdx.x & ((1 << lg) - 1);
    for (int d = 1 << lg; d < kWave; d <<= 1) {
        const float4 top = max4(a.top, shfl_xor4(a.top, d));
        // (both lanes of a pair add the lower one's sum first)
        const float4 mine = a.sum * exp_of4(a.top - top), other = shfl_xor4(mine, d);
        a.sum = lane & d ? other + mine : mine + other;
        a.top = top;
    }
    if (lane < (1 << lg)) {
        lds[0][(wave << lg) + lane] = a.top;
        lds[1][(wave << lg) + lane] = a.sum;
    }
    __syncthreads();
    a.top = lds[0][q];
    for (int w = 1; w < kThreads / kWave; ++w) a.top = max4(a.top, lds[0][(w << lg) + q]);
    a.sum = splat(0.f);
    for (int w = 0; w < kThreads / kWave; ++w) a.sum = fma4(lds[1][(w << lg) + q], exp_of4(lds[0][(w << lg) + q] - a.top), a.sum);
    return a;
}

// One work-group: a chunk of the classes in a tile of columns.
__global__ __launch_bounds__(kThreads) void log_sum_kernel(const LossArgs a, const Shape z, float *partial)
{
    __shared__ float4 lds[2][kThreads / kWave << kLanes];
    const int chunk = blockIdx.x % z.chunks;
    const Spot p = spot_in(blockIdx.x / z.chunks, z.lg, a.batch);
    const int first = chunk * z.rows, end = min(a.classes, first + z.rows);
    Running r{splat(-FLT_MAX), splat(0.f)};
    for (int i = first + p.slot; i < end; i += kLoads * p.slots) {
        float4 x[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) x[u] = load_quad(a.Z + min(i + u * p.slots, end - 1) * a.ldz, p);
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            if (i + u * p.slots >= end) x[u] = splat(-INFINITY);
        add_rows(r, x);
    }
    r = join(r, z.lg, lds);
    if (p.slot) return;
    float *const at = partial + 2 * static_cast<int64_t>(chunk) * a.batch;
    store_quad(at, p, r.top);
    store_quad(at + a.batch, p, r.sum);
}

// A column's chunks added up: largest logit, sum of exponentials beyond it, and the label's log-probability (0 where the column does not count).
struct Column {
    float top;
    double sum, logp;
    int label;
    float at_label;
    bool counts;
};
__device__ __forceinline__ Column column_of(const LossArgs &a, const float *partial, int chunks, int col)
{
    Column c;
    c.label = a.labels[col];
    const bool inside = c.label >= 0 && c.label < a.classes;
    c.at_label = inside ? a.Z[c.label * a.ldz + col] : -INFINITY;
    c.counts = inside && c.at_label != -INFINITY;
    c.top = -FLT_MAX;
    for (int k = 0; k < chunks; ++k) c.top = fmaxf(c.top, partial[2 * static_cast<int64_t>(k) * a.batch + col]);
    c.sum = 0;
    for (int k = 0; k < chunks; ++k) {
        const float *const at = partial + 2 * static_cast<int64_t>(k) * a.batch + col;
        c.sum += at[a.batch] * exp(static_cast<double>(at[0]) - c.top);
    }
    c.logp = c.counts ? static_cast<double>(c.at_label) - c.top - log(c.sum) : 0.0;
    return c;
}
__device__ __forceinline__ ColumnState state_of(const Column &c, float slope)
{
    return {c.top, static_cast<float>(slope / c.sum), slope, c.label};
}

__device__ __forceinline__ double block_sum(double x, double *lds)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d, kWave);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0;
    for (int w = 0; w < static_cast<int>(blockDim.x >> 6); ++w) s += lds[w];
    return s;
}

// The clipped loss of a column.
struct Borders {
    double low, high;        // of l - old: log(1 - clip_low), log(1 + clip_high)
    float margin;            // how far l may be off
};
struct PolicyTerm {
    double surrogate, kl, slope;
    bool clipped, close;     // close: l does not tell on which side of its border the column lies
};
__device__ __forceinline__ PolicyTerm policy_term(const LossArgs &a, const Borders &b, double logp, int col)
{
    PolicyTerm t;
    const double A = a.advantages[col], d = logp - a.old_logp[col], r = exp(d);
    const double border = A > 0 ? b.high : b.low;
    t.clipped = A > 0 ? d > border : A < 0 && d < border;
    t.close = A != 0 && fabs(d - border) <= b.margin;
    t.surrogate = -A * (!t.clipped ? r : A > 0 ? 1.0 + a.clip_high : 1.0 - a.clip_low);
    t.slope = t.clipped ? 0.0 : -A * r;
    t.kl = 0;
    if (a.ref_logp) {
        const double g = a.ref_logp[col] - logp, q = exp(g);
        t.kl = q - g - 1;
        t.slope += a.beta * (1 - q);
    }
    return t;
}

// A thread per column.  The sums of exponentials come from 32 bits; where that does not tell whether a column is clipped, the work-group forms it again
// in 64 (some 1 column in 10^5 with ratios around 1).
__global__ __launch_bounds__(kColumns) void policy_columns_kernel(const LossArgs a, const Shape z, const LossSpace w, const Borders b)
{
    __shared__ double lds[kColumns / kWave];
    __shared__ int close[kColumns];
    __shared__ float tops[kColumns];
    const int col = blockIdx.x * kColumns + threadIdx.x;
    Column c{};
    double weight = 0;
    PolicyTerm t{};
    if (col < a.batch) {
        c = column_of(a, w.partial, z.chunks, col);
        weight = a.weights ? static_cast<double>(a.weights[col]) : 1.0 / a.batch;
        if (!c.counts) weight = 0;
        if (weight != 0) t = policy_term(a, b, c.logp, col);
    }
    close[threadIdx.x] = t.close;
    tops[threadIdx.x] = c.top;
    if (__syncthreads_or(t.close)) {
        for (int k = 0; k < kColumns; ++k) {
            if (!close[k]) continue;
            const float *const Z = a.Z + blockIdx.x * kColumns + k;
            const double top = tops[k];
            double s = 0;
            for (int i = threadIdx.x; i < a.classes; i += kColumns) s += exp(Z[i * a.ldz] - top);
            s = block_sum(s, lds);
            if (static_cast<int>(threadIdx.x) == k) {
                c.sum = s;
                c.logp = static_cast<double>(c.at_label) - top - log(s);
                t = policy_term(a, b, c.logp, col);
            }
        }
    }
    if (col < a.batch) {
        if (a.logp) a.logp[col] = static_cast<float>(c.logp);
        w.columns[col] = state_of(c, weight != 0 ? static_cast<float>(weight * t.slope) : 0.f);
    }
    const bool used = weight != 0;
    const double share[4] = {used ? weight * (t.surrogate + a.beta * t.kl) : 0, used ? weight * t.surrogate : 0, used ? weight * t.kl : 0,
                             used && t.clipped ? weight : 0};
    for (int k = 0; k < 4; ++k) {
        const double s = block_sum(share[k], lds);
        if (threadIdx.x == 0) w.shares[4 * blockIdx.x + k] = s;
    }
}

// first column and end of a sequence, whatever `starts` holds
__device__ __forceinline__ int2 columns_of(const LossArgs &a, int sequence)
{
    const int from = min(max(a.starts[sequence], 0), a.batch);
    return make_int2(from, min(max(a.starts[sequence + 1], from), a.batch));
}

// A thread per column: log-probabilities, and for the gradient of the preference loss what is not the pair's.
__global__ __launch_bounds__(kColumns) void log_prob_columns_kernel(const LossArgs a, const Shape z, const LossSpace w, const bool gradient)
{
    const int col = blockIdx.x * kColumns + threadIdx.x;
    if (col >= a.batch) return;
    const Column c = column_of(a, w.partial, z.chunks, col);
    w.logp[col] = c.logp;
    if (a.logp) a.logp[col] = static_cast<float>(c.logp);
    if (gradient) {
        const bool held = col >= a.starts[0] && col < a.starts[a.sequences];
        w.columns[col] = state_of(c, held && c.counts ? 1.f : 0.f);
    }
}

constexpr int kSequenceThreads = 1024;
__device__ __forceinline__ double sequence_sum(const LossArgs &a, const double *logp, int2 at, double *lds)
{
    double s = 0;
    for (int col = at.x + threadIdx.x; col < at.y; col += blockDim.x) s += logp[col];
    return block_sum(s, lds);
}
__global__ __launch_bounds__(kSequenceThreads) void sequence_sums_kernel(const LossArgs a, const LossSpace w)
{
    __shared__ double lds[kSequenceThreads / kWave];
    const double s = sequence_sum(a, w.logp, columns_of(a, blockIdx.x), lds);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = static_cast<float>(s);
}

// A work-group per pair.
__global__ __launch_bounds__(kSequenceThreads) void pairs_kernel(const LossArgs a, const LossSpace w)
{
    __shared__ double lds[kSequenceThreads / kWave];
    const int pair = blockIdx.x;
    int2 at[2];
    double s[2];
    for (int k = 0; k < 2; ++k) {
        at[k] = columns_of(a, 2 * pair + k);
        s[k] = sequence_sum(a, w.logp, at[k], lds);
    }
    double beyond = s[0] - s[1];
    if (a.ref_sums) beyond = (s[0] - a.ref_sums[2 * pair]) - (s[1] - a.ref_sums[2 * pair + 1]);
    const double x = a.beta * beyond, tail = log1p(exp(-fabs(x))), t = a.smoothing;
    // (the derivative from what is small, so that it does not vanish beside 1)
    const double e = exp(-fabs(x)), above = x > 0 ? 1 / (1 + e) : e / (1 + e), below = x > 0 ? e / (1 + e) : 1 / (1 + e);
    const double slope = (t * above - (1 - t) * below) * a.beta / gridDim.x;
    if (threadIdx.x == 0) {
        if (a.sums) a.sums[2 * pair] = static_cast<float>(s[0]), a.sums[2 * pair + 1] = static_cast<float>(s[1]);
        if (a.margins) a.margins[pair] = static_cast<float>(x);
        w.shares[pair] = (1 - t) * (tail + fmax(-x, 0.0)) + t * (tail + fmax(x, 0.0));
    }
    for (int k = 0; k < 2; ++k) {
        const float c = static_cast<float>(k ? -slope : slope);
        for (int col = at[k].x + threadIdx.x; col < at[k].y; col += blockDim.x) {
            ColumnState q = w.columns[col];
            if (q.c == 0.f) continue;
            q.share *= c;
            q.c = c;
            w.columns[col] = q;
        }
    }
}

// the shares of the loss, added up by one wave in one fixed order
__device__ void write_policy_stats(const LossArgs &a, const double *shares, int blocks)
{
    for (int k = 0; k < 4; ++k) {
        double s = 0;
        for (int b = threadIdx.x; b < blocks; b += kWave) s += shares[4 * static_cast<int64_t>(b) + k];
        for (int d = 1; d < kWave; d <<= 1) s += __shfl_xor(s, d, kWave);
        if (threadIdx.x == 0) a.stats[k] = static_cast<float>(s);
    }
}
__device__ void write_preference_loss(const LossArgs &a, const double *shares, int pairs)
{
    double s = 0;
    for (int b = threadIdx.x; b < pairs; b += kWave) s += shares[b];
    for (int d = 1; d < kWave; d <<= 1) s += __shfl_xor(s, d, kWave);
    if (threadIdx.x == 0 && a.loss) *a.loss = static_cast<float>(s / pairs);
}

__device__ __forceinline__ float gradient_of(float z, const ColumnState &c, int i)
{
    if (c.c == 0.f) return 0.f;
    return fmaf(-c.share, exp_of(z - c.top), i == c.label ? c.c : 0.f);
}

// One work-group: a chunk of the classes in a tile of columns.  `shares`: how many shares of the loss there are (policy: of four terms each).
__global__ __launch_bounds__(kThreads) void logits_gradient_kernel(const LossArgs a, const Shape z, const LossSpace w, const int shares)
{
    if (blockIdx.x == 0 && threadIdx.x < kWave) {
        if (a.stats) write_policy_stats(a, w.shares, shares);
        else write_preference_loss(a, w.shares, shares);
    }
    const int chunk = blockIdx.x % z.chunks;
    const Spot p = spot_in(blockIdx.x / z.chunks, z.lg, a.batch);
    if (p.n == 0) return;
    const int first = chunk * z.rows, end = min(a.classes, first + z.rows);
    ColumnState c[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = w.columns[p.col + min(k, p.n - 1)];
    for (int i = first + p.slot; i < end; i += kLoads * p.slots) {
        float4 x[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) x[u] = load_quad(a.Z + min(i + u * p.slots, end - 1) * a.ldz, p);
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int row = i + u * p.slots;
            if (row < end)
                store_quad(a.dZ + row * a.lddz, p, make_float4(gradient_of(x[u].x, c[0], row), gradient_of(x[u].y, c[1], row), gradient_of(x[u].z, c[2], row),
                                                               gradient_of(x[u].w, c[3], row)));
        }
    }
}

Shape shape_of(int32_t classes, int32_t batch)
{
    Shape z;
    z.lg = lanes_for(batch, kLanes);
    z.tiles = static_cast<int32_t>((batch + (INT64_C(4) << z.lg) - 1) >> (z.lg + 2));
    const int step = kLoads * (kThreads >> z.lg);
    const int64_t most = (static_cast<int64_t>(classes) + step - 1) / step, want = std::max<int64_t>(1, kBlocks / z.tiles);
    const int64_t steps = (most + std::min(most, want) - 1) / std::min(most, want);      // of kLoads rows a thread
    z.rows = static_cast<int>(std::min<int64_t>(steps * step, classes));
    z.chunks = static_cast<int>((static_cast<int64_t>(classes) + z.rows - 1) / z.rows);
    return z;
}
int column_blocks(int32_t batch) { return static_cast<int>((static_cast<int64_t>(batch) + kColumns - 1) / kColumns); }
void launch_log_sums(const LossArgs &a, const Shape &z, const LossSpace &w, hipStream_t s)
{
    log_sum_kernel<<<static_cast<uint32_t>(z.tiles) * z.chunks, kThreads, 0, s>>>(a, z, w.partial);
}
void launch_gradient(const LossArgs &a, const Shape &z, const LossSpace &w, int shares, hipStream_t s)
{
    logits_gradient_kernel<<<static_cast<uint32_t>(z.tiles) * z.chunks, kThreads, 0, s>>>(a, z, w, shares);
}

}  // namespace

LossSpace loss_space(void *memory, int32_t classes, int32_t batch, int32_t sequences)
{
    const Shape z = shape_of(classes, batch);
    LossSpace w;
    w.logp = static_cast<double *>(memory);
    w.shares = w.logp + batch;
    w.columns = reinterpret_cast<ColumnState *>(w.shares + std::max(4 * column_blocks(batch), sequences));
    w.partial = reinterpret_cast<float *>(w.columns + batch);
    w.bytes = reinterpret_cast<char *>(w.partial + 2 * static_cast<int64_t>(z.chunks) * batch) - static_cast<char *>(memory);
    return w;
}

hipError_t launch_log_probs(const LossArgs &a, hipStream_t s)
{
    const Shape z = shape_of(a.classes, a.batch);
    const LossSpace w = loss_space(a.workspace, a.classes, a.batch, a.sequences);
    if (!fits_launch(static_cast<int64_t>(z.tiles) * z.chunks, kThreads) || !fits_launch(a.sequences, kSequenceThreads)) return hipErrorInvalidConfiguration;
    launch_log_sums(a, z, w, s);
    log_prob_columns_kernel<<<column_blocks(a.batch), kColumns, 0, s>>>(a, z, w, false);
    if (a.sums) sequence_sums_kernel<<<a.sequences, kSequenceThreads, 0, s>>>(a, w);
    return hipGetLastError();
}

hipError_t launch_policy(const LossArgs &a, hipStream_t s)
{
    const Shape z = shape_of(a.classes, a.batch);
    const LossSpace w = loss_space(a.workspace, a.classes, a.batch, 0);
    if (!fits_launch(static_cast<int64_t>(z.tiles) * z.chunks, kThreads)) return hipErrorInvalidConfiguration;
    // An exponential is off by 2^-24 (2 |z - top| + 2), and the mean of |z - top| over p is at most log(classes) < 22; a thread adds up eight
    // rows, then their sum to the others'.
    const double adds = 2.0 * (z.rows / ((kThreads >> z.lg) * kLoads) + 1) + kLoads;
    const Borders b{a.clip_low < 1.f ? log1p(-static_cast<double>(a.clip_low)) : -INFINITY, log1p(static_cast<double>(a.clip_high)),
                    static_cast<float>((64 + adds) / (1 << 24))};
    launch_log_sums(a, z, w, s);
    policy_columns_kernel<<<column_blocks(a.batch), kColumns, 0, s>>>(a, z, w, b);
    launch_gradient(a, z, w, column_blocks(a.batch), s);
    return hipGetLastError();
}

hipError_t launch_preference(const LossArgs &a, hipStream_t s)
{
    const Shape z = shape_of(a.classes, a.batch);
    const LossSpace w = loss_space(a.workspace, a.classes, a.batch, a.sequences);
    if (!fits_launch(static_cast<int64_t>(z.tiles) * z.chunks, kThreads) || !fits_launch(a.sequences / 2, kSequenceThreads)) return hipErrorInvalidConfiguration;
    launch_log_sums(a, z, w, s);
    log_prob_columns_kernel<<<column_blocks(a.batch), kColumns, 0, s>>>(a, z, w, true);
    pairs_kernel<<<a.sequences / 2, kSequenceThreads, 0, s>>>(a, w);
    launch_gradient(a, z, w, a.sequences / 2, s);
    return hipGetLastError();
}

}  // namespace nerva
