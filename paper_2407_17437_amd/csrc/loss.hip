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
// Bound by memory.  Columns that a work-group can hold in registers are read once: maximum, sum, what a column needs, gradient.  Longer ones are cut into
// chunks of classes: the first launch leaves a maximum and a sum for each, from one pass with a running maximum; the second adds them up, 16 threads
// a column; the last one reads the logits again for the gradient.  What a column needs is done in 64 bits: log-probabilities are added up over
// sequences and compared with borders, and there are few of them.
#include <float.h>

#include <algorithm>

#include "columns.h"
#include "experts.h"
#include "loss.h"

namespace nerva {
namespace {

constexpr int kThreads = 256;          // of chunks
constexpr int kLanes = 6;              // log2 of the quads of their tiles: 256 columns
constexpr int kLoads = 8, kFewLoads = 2;   // rows in flight per thread
constexpr int64_t kBlocks = 8192;      // work-groups that the classes are cut for
constexpr int kColumns = 16, kParts = 16;   // columns of a work-group that adds up chunks, threads of a column
// Of a work-group that holds its columns.  (Eight rows a thread take all 128 registers that 1024 threads leave, and two more of the policy loss, five of the preference loss lie
// in scratch memory; with 16 rows 2048 classes x 8192 take 61.5 us instead of 48.5 in chunks.)
constexpr int kHeldThreads = 1024, kHeldRows = 8;

__device__ __forceinline__ float4 exp_of4(float4 x) { return make_float4(exp_of(x.x), exp_of(x.y), exp_of(x.z), exp_of(x.w)); }
__device__ __forceinline__ float4 max4(float4 a, float4 b) { return make_float4(fmaxf(a.x, b.x), fmaxf(a.y, b.y), fmaxf(a.z, b.z), fmaxf(a.w, b.w)); }

struct Shape {
    int lg, chunks, rows, loads;       // rows of a chunk; rows that a thread of the sums' launch reads at a time
    int32_t tiles;
    bool past;                         // results go past the caches
};

// Running maximum and sum of a thread's rows of its four columns.  The maximum starts at the lowest number, not at -inf, so that no
// difference of two infinities arises where all logits are -inf; +inf and NaN make the sum NaN.
struct Running {
    float4 top, sum;
};
template <int U>
__device__ __forceinline__ void add_rows(Running &a, const float4 (&z)[U])
{
    float4 top = a.top;
#pragma unroll
    for (int u = 0; u < U; ++u) top = max4(top, z[u]);
    float4 s = exp_of4(z[0] - top);
#pragma unroll
    for (int u = 1; u < U; ++u) s = s + exp_of4(z[u] - top);
    a.sum = fma4(a.sum, exp_of4(a.top - top), s);
    a.top = top;
}
// over the threads of a chunk with the same columns; the same in all of them.  lds: two float4 per wave and quad
__device__ __forceinline__ Running join(Running a, int lg, float4 *lds)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, q = threadIdx.x & ((1 << lg) - 1);
    constexpr int waves = kThreads / kWave;
    for (int d = 1 << lg; d < kWave; d <<= 1) {
        const float4 top = max4(a.top, shfl_xor4(a.top, d));
        // (both lanes of a pair add the lower one's sum first)
        const float4 mine = a.sum * exp_of4(a.top - top), other = shfl_xor4(mine, d);
        a.sum = lane & d ? other + mine : mine + other;
        a.top = top;
    }
    float4 *const sums = lds + (waves << lg);
    if (lane < (1 << lg)) {
        lds[(wave << lg) + lane] = a.top;
        sums[(wave << lg) + lane] = a.sum;
    }
    __syncthreads();
    a.top = lds[q];
    for (int w = 1; w < waves; ++w) a.top = max4(a.top, lds[(w << lg) + q]);
    a.sum = splat(0.f);
    for (int w = 0; w < waves; ++w) a.sum = fma4(sums[(w << lg) + q], exp_of4(lds[(w << lg) + q] - a.top), a.sum);
    return a;
}

template <int U, TileKind T>
__device__ __forceinline__ Running sum_rows(const LossArgs &a, const Spot &p, int first, int end)
{
    Running r{splat(-FLT_MAX), splat(0.f)};
    for (int i = first + p.slot; i < end; i += U * p.slots) {
        float4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load_of<T>(a.Z + min(i + u * p.slots, end - 1) * a.ldz, p);
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = i + u * p.slots < end ? own_of<T>(x[u], p) : splat(-INFINITY);
        add_rows(r, x);
    }
    return r;
}
// Chunk and tile of work-group b: all tiles of one chunk, then those of the next, so that those that run together read whole rows.  (All chunks of one tile first,
// rows a power of two apart meet in few memory channels: 4096 classes x 8192, sums 40.4 instead of 33.0 us, policy loss 86 instead of 79.)
struct Part {
    int chunk, tile;
};
__device__ __forceinline__ Part part_of(int b, const Shape &z) { return {b / z.tiles, b % z.tiles}; }
// One work-group: a chunk of the classes in a tile of columns.
template <int U>
__global__ __launch_bounds__(kThreads) void log_sum_kernel(const LossArgs a, const Shape z, float *partial)
{
    __shared__ float4 lds[2 * kThreads / kWave << kLanes];
    const Part part = part_of(blockIdx.x, z);
    const int chunk = part.chunk, first = chunk * z.rows, end = min(a.classes, first + z.rows);
    const Spot p = spot_in(part.tile, z.lg, a.batch);
    Running r;
    with_kind(p, [&](auto kind) { r = sum_rows<U, kind>(a, p, first, end); });
    r = join(r, z.lg, lds);
    if (p.slot) return;
    float *const at = partial + 2 * static_cast<int64_t>(chunk) * a.batch;
    store_quad(at, p, r.top);
    store_quad(at + a.batch, p, r.sum);
}

// ---- what a column needs ----
struct Column {
    float top, at_label;     // largest logit; the label's
    double sum, logp;        // of exp(z - top); 0 where the column does not count
    int label;
    bool counts;
};
__device__ __forceinline__ void read_label(const LossArgs &a, int col, Column &c)
{
    c.label = a.labels[col];
    const bool inside = c.label >= 0 && c.label < a.classes;
    c.at_label = inside ? a.Z[c.label * a.ldz + col] : -INFINITY;
    c.counts = inside && c.at_label != -INFINITY;
}
__device__ __forceinline__ void set_sum(Column &c, double sum)
{
    c.sum = sum;
    c.logp = c.counts ? static_cast<double>(c.at_label) - c.top - log(sum) : 0.0;
}
__device__ __forceinline__ ColumnState state_of(const Column &c, float slope) { return {c.top, static_cast<float>(slope / c.sum), slope, c.label}; }

// sum over a work-group in one fixed order; every thread gets it
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

// sum of exp(z - top) of a column in 64 bits, by the whole work-group
__device__ double exact_sum(const LossArgs &a, int col, double top, double *lds)
{
    double s = 0;
#pragma unroll 8
    for (int i = threadIdx.x; i < a.classes; i += blockDim.x) s += exp(a.Z[i * a.ldz + col] - top);
    return block_sum(s, lds);
}

// The clipped loss of a column.
struct Borders {
    double low, high;        // of l - old: log(1 - clip_low), log(1 + clip_high)
    float margin;            // how far l may be off
};
// what a column brings along, asked for beside the logits (1000 classes x 8192: 21.7 -> 20.9 us)
struct PolicyInputs {
    float weight, advantage, old_logp, ref_logp;
};
__device__ __forceinline__ PolicyInputs policy_inputs(const LossArgs &a, int col)
{
    return {a.weights ? a.weights[col] : 1.f, a.advantages[col], a.old_logp[col], a.ref_logp ? a.ref_logp[col] : 0.f};
}
struct PolicyTerm {
    double weight, surrogate, kl, slope;
    bool clipped, close;     // close: l does not tell on which side of its border the column lies
};
__device__ __forceinline__ PolicyTerm policy_term(const LossArgs &a, const Borders &b, const Column &c, const PolicyInputs &in)
{
    PolicyTerm t{};
    t.weight = !c.counts ? 0 : a.weights ? static_cast<double>(in.weight) : 1.0 / a.batch;
    if (t.weight == 0) return t;
    // (a ratio beyond 64 bits stays a number, of which an advantage of 0 makes 0; a NaN stays one)
    const double A = in.advantage, d = c.logp - in.old_logp, r = exp(d > 709.0 ? 709.0 : d);
    const double border = A > 0 ? b.high : b.low;
    t.clipped = A > 0 ? d > border : A < 0 && d < border;
    t.close = A != 0 && fabs(d - border) <= b.margin;
    t.surrogate = -A * (!t.clipped ? r : A > 0 ? 1.0 + a.clip_high : 1.0 - a.clip_low);
    t.slope = t.clipped ? 0.0 : -A * r;
    if (a.ref_logp) {
        const double g = in.ref_logp - c.logp, q = exp(g);
        t.kl = q > DBL_MAX ? q : q - g - 1;
        if (a.beta != 0.f) t.slope += a.beta * (1 - q);   // (q and the term may be infinite, of which a factor of 0 takes nothing)
    }
    return t;
}
// share k of a column in the loss and its terms
__device__ __forceinline__ double policy_share(const LossArgs &a, const PolicyTerm &t, int k)
{
    if (t.weight == 0) return 0;
    return t.weight * (k == 0 ? (a.beta != 0.f ? t.surrogate + a.beta * t.kl : t.surrogate) : k == 1 ? t.surrogate : k == 2 ? t.kl : t.clipped ? 1.0 : 0.0);
}

// The preference loss of a pair from its margin: the loss, and its derivative by the chosen sequence's sum times the number of pairs.
struct PairTerm {
    double loss, slope;
};
__device__ __forceinline__ PairTerm pair_term(const LossArgs &a, double x)
{
    // (the derivative from what is small, so that it does not vanish beside 1)
    const double e = exp(-fabs(x)), tail = log1p(e), t = a.smoothing;
    const double above = x > 0 ? 1 / (1 + e) : e / (1 + e), below = x > 0 ? e / (1 + e) : 1 / (1 + e);
    // (a side that has no share takes nothing, however large its loss is)
    const double chosen = t < 1 ? (1 - t) * (tail + fmax(-x, 0.0)) : 0.0, rejected = t > 0 ? t * (tail + fmax(x, 0.0)) : 0.0;
    return {chosen + rejected, (t * above - (1 - t) * below) * a.beta};
}
__device__ __forceinline__ double margin_of(const LossArgs &a, int pair, double chosen, double rejected)
{
    if (a.ref_sums) return a.beta * ((chosen - a.ref_sums[2 * pair]) - (rejected - a.ref_sums[2 * pair + 1]));
    return a.beta * (chosen - rejected);
}
// first column and end of a sequence, whatever `starts` holds
__device__ __forceinline__ int2 columns_of(const LossArgs &a, int sequence)
{
    const int from = min(max(a.starts[sequence], 0), a.batch);
    return make_int2(from, min(max(a.starts[sequence + 1], from), a.batch));
}
__device__ __forceinline__ bool in_sequences(const LossArgs &a, int col) { return col >= a.starts[0] && col < a.starts[a.sequences]; }

// e: exp(z - top)
__device__ __forceinline__ float gradient_of(float e, const ColumnState &c, int i)
{
    if (c.c == 0.f) return 0.f;
    return fmaf(-c.share, e, i == c.label ? c.c : 0.f);
}
__device__ __forceinline__ float4 gradient_of4(float4 e, const ColumnState (&c)[4], int i)
{
    return make_float4(gradient_of(e.x, c[0], i), gradient_of(e.y, c[1], i), gradient_of(e.z, c[2], i), gradient_of(e.w, c[3], i));
}

// ---- columns that a work-group holds ----
enum What { kLogProbs, kPolicy, kPreference };

// One work-group: all classes of a tile of columns, K rows a thread; at least as many threads as columns, of which each does what a column needs.
// kLogProbs: log-probabilities, and the sums of sequences where there is one tile.  kPolicy: all of it (the loss's shares are left for another launch
// where there are more tiles).  kPreference: all of it in one tile; in more, what the launches for pairs and for the gradient take.
template <int K, What W>
__global__ __launch_bounds__(kHeldThreads) void held_kernel(const LossArgs a, const Shape z, const LossSpace w, const Borders b)
{
    extern __shared__ float4 lds[];   // per wave and quad: maxima, then sums in 64 bits
    __shared__ double sums[kHeldThreads / kWave], parts[(4 << kLanes) / kWave][4];
    __shared__ float tops[4 << kLanes];
    __shared__ int close[4 << kLanes];
    __shared__ double logp[4 << kLanes];
    __shared__ ColumnState states[4 << kLanes];
    const Spot p = spot_in(near_tile(blockIdx.x, z.tiles, z.lg), z.lg, a.batch, z.past);
    const int width = 4 << z.lg, first = p.col - 4 * p.q, j = threadIdx.x, col = first + j;
    const bool mine = j < width && col < a.batch;
    Column c{};
    if (mine) read_label(a, col, c);
    PolicyInputs in{};
    if (W == kPolicy && mine) in = policy_inputs(a, col);
    float4 x[K];
    with_kind(p, [&](auto kind) {
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] = load_of<kind>(a.Z + min(p.slot + k * p.slots, a.classes - 1) * a.ldz, p);
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] = own_of<kind>(x[k], p);
    });
    const int lane = j & (kWave - 1), wave = j >> 6, waves = static_cast<int>(blockDim.x >> 6);
    float4 top = splat(-FLT_MAX);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (p.slot + k * p.slots >= a.classes) x[k] = splat(-INFINITY);
        top = max4(top, x[k]);
    }
    for (int d = 1 << z.lg; d < kWave; d <<= 1) top = max4(top, shfl_xor4(top, d));
    if (waves > 1) {
        if (lane < (1 << z.lg)) lds[(wave << z.lg) + lane] = top;
        __syncthreads();
        for (int u = 0; u < waves; ++u) top = max4(top, lds[(u << z.lg) + p.q]);
    }
    // x becomes the exponential, which the gradient takes as well; a thread's few are added up in 32 bits, the threads' sums in 64
    float4 few = splat(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        x[k] = exp_of4(x[k] - top);
        few = few + x[k];
    }
    double part[4] = {few.x, few.y, few.z, few.w};
    for (int d = 1 << z.lg; d < kWave; d <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) part[k] += __shfl_xor(part[k], d, kWave);
    double *const of_waves = reinterpret_cast<double *>(lds + (waves << z.lg));
    if (lane < (1 << z.lg))
#pragma unroll
        for (int k = 0; k < 4; ++k) of_waves[(wave << (z.lg + 2)) + 4 * lane + k] = part[k];
    if (p.slot == 0) *reinterpret_cast<float4 *>(tops + 4 * p.q) = top;
    __syncthreads();
    if (mine) {
        double sum = 0;
        for (int u = 0; u < waves; ++u) sum += of_waves[u * width + j];
        c.top = tops[j];
        set_sum(c, sum);
        if (a.logp && W != kPolicy) a.logp[col] = static_cast<float>(c.logp);
    }
    if constexpr (W == kPolicy) {
        PolicyTerm t{};
        if (mine) t = policy_term(a, b, c, in);
        if (j < width) close[j] = t.close;
        if (__syncthreads_or(t.close)) {
            // the sums of exponentials come from 32 bits; where that does not tell whether a column is clipped, it is formed again in 64
            for (int k = 0; k < width; ++k) {
                if (!close[k]) continue;
                const double again = exact_sum(a, first + k, tops[k], sums);
                if (j == k) {
                    set_sum(c, again);
                    t = policy_term(a, b, c, in);
                }
            }
        }
        if (mine && a.logp) a.logp[col] = static_cast<float>(c.logp);
        if (j < width) states[j] = state_of(c, t.weight != 0 ? static_cast<float>(t.weight * t.slope) : 0.f);
        // the four sums side by side: one after the other they take 6.7 us instead of 5.4 (10 classes x 100)
        double share[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) share[k] = policy_share(a, t, k);
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1)
#pragma unroll
            for (int k = 0; k < 4; ++k) share[k] += __shfl_xor(share[k], d, kWave);
        const int waves = static_cast<int>(blockDim.x >> 6), of = min(waves, (width + kWave - 1) >> 6);   // (waves that have columns)
        if ((j & (kWave - 1)) == 0 && j >> 6 < of)
#pragma unroll
            for (int k = 0; k < 4; ++k) parts[j >> 6][k] = share[k];
        __syncthreads();
        if (j < 4) {
            double s = 0;
            for (int u = 0; u < of; ++u) s += parts[u][j];
            if (z.tiles == 1) a.stats[j] = static_cast<float>(s);
            else w.shares[4 * static_cast<int64_t>(blockIdx.x) + j] = s;
        }
    } else {
        if (z.tiles > 1) {
            if (mine) {
                w.logp[col] = c.logp;
                if (W == kPreference) w.columns[col] = state_of(c, in_sequences(a, col) && c.counts ? 1.f : 0.f);
            }
            return;
        }
        if (j < width) logp[j] = c.logp;
        if constexpr (W == kPreference)
            if (j < width) states[j] = state_of(c, 0.f);
        __syncthreads();
        const auto sum_of = [&](int sequence) {
            const int2 at = columns_of(a, sequence);
            double s = 0;
            for (int k = at.x; k < at.y; ++k) s += logp[k];
            if (a.sums) a.sums[sequence] = static_cast<float>(s);
            return s;
        };
        if constexpr (W == kLogProbs) {
            if (a.sums)
                for (int k = j; k < a.sequences; k += blockDim.x) (void)sum_of(k);
            return;
        } else {
            const int pairs = a.sequences / 2;
            double loss = 0;
            for (int k = j; k < pairs; k += blockDim.x) {
                const double chosen = sum_of(2 * k), x = margin_of(a, k, chosen, sum_of(2 * k + 1));
                const PairTerm t = pair_term(a, x);
                loss += t.loss;
                if (a.margins) a.margins[k] = static_cast<float>(x);
                for (int side = 0; side < 2; ++side) {
                    const int2 at = columns_of(a, 2 * k + side);
                    for (int i = at.x; i < at.y; ++i) states[i].c = static_cast<float>((side ? -t.slope : t.slope) / pairs);
                }
            }
            loss = block_sum(loss, sums);   // (and a barrier)
            if (j == 0 && a.loss) *a.loss = static_cast<float>(loss / pairs);
            if (j < width) states[j] = state_of(c, c.counts ? states[j].c : 0.f);
        }
    }
    __syncthreads();
    ColumnState q[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) q[k] = states[4 * p.q + k];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int row = p.slot + k * p.slots;
        if (row < a.classes) store_quad(a.dZ + row * a.lddz, p, gradient_of4(x[k], q, row));   // (x: exponentials)
    }
}

// ---- columns in chunks ----
// The chunks of 16 columns added up; the columns' first threads get the result (col < batch), and all threads the largest logits in `tops`.
__device__ __forceinline__ Column column_of(const LossArgs &a, const float *partial, int chunks, int col, int part, float *tops, double (*lds)[kColumns])
{
    const int at_col = min(col, a.batch - 1), lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, j = threadIdx.x & (kColumns - 1);
    __shared__ float of_wave[kColumns * kParts / kWave][kColumns];
    Column c{};
    if (part == 0) read_label(a, at_col, c);
    float top = -FLT_MAX;
#pragma unroll 8
    for (int k = part; k < chunks; k += kParts) top = fmaxf(top, partial[2 * static_cast<int64_t>(k) * a.batch + at_col]);
    for (int d = kColumns; d < kWave; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, kWave));
    if (lane < kColumns) of_wave[wave][j] = top;
    __syncthreads();
    for (int w = 0; w < kColumns * kParts / kWave; ++w) top = fmaxf(top, of_wave[w][j]);
    double sum = 0;
#pragma unroll 8
    for (int k = part; k < chunks; k += kParts) {
        const float *const at = partial + 2 * static_cast<int64_t>(k) * a.batch + at_col;
        sum += at[a.batch] * exp(static_cast<double>(at[0]) - top);
    }
    for (int d = kColumns; d < kWave; d <<= 1) sum += __shfl_xor(sum, d, kWave);
    if (lane < kColumns) lds[wave][j] = sum;
    if (part == 0) tops[j] = top;
    __syncthreads();
    sum = 0;
    for (int w = 0; w < kColumns * kParts / kWave; ++w) sum += lds[w][j];
    c.top = top;
    if (part == 0) set_sum(c, sum);
    return c;
}

__global__ __launch_bounds__(kColumns *kParts) void policy_columns_kernel(const LossArgs a, const Shape z, const LossSpace w, const Borders b)
{
    __shared__ double lds[kColumns * kParts / kWave][kColumns], sums[kColumns * kParts / kWave];
    __shared__ float tops[kColumns];
    __shared__ int close[kColumns];
    const int j = threadIdx.x & (kColumns - 1), part = threadIdx.x / kColumns, col = blockIdx.x * kColumns + j;
    const bool mine = part == 0 && col < a.batch;
    PolicyInputs in{};
    if (mine) in = policy_inputs(a, col);
    Column c = column_of(a, w.partial, z.chunks, col, part, tops, lds);
    PolicyTerm t{};
    if (mine) t = policy_term(a, b, c, in);
    if (part == 0) close[j] = t.close;
    if (__syncthreads_or(t.close)) {
        // as above, in 64 bits (some 4 columns in 10^5 with ratios around 1; all of them where clip is 0 and the policy has not moved: 3000 classes x 8192 then take 493 us
        // instead of 57)
        for (int k = 0; k < kColumns; ++k) {
            if (!close[k]) continue;
            const double again = exact_sum(a, blockIdx.x * kColumns + k, tops[k], sums);
            if (part == 0 && j == k) {
                set_sum(c, again);
                t = policy_term(a, b, c, in);
            }
        }
    }
    if (mine) {
        if (a.logp) a.logp[col] = static_cast<float>(c.logp);
        w.columns[col] = state_of(c, t.weight != 0 ? static_cast<float>(t.weight * t.slope) : 0.f);
    }
    if (threadIdx.x >= kWave) return;
    for (int k = 0; k < 4; ++k) {
        double s = policy_share(a, t, k);
        for (int d = 1; d < kColumns; d <<= 1) s += __shfl_xor(s, d, kWave);
        if (threadIdx.x == 0) w.shares[4 * static_cast<int64_t>(blockIdx.x) + k] = s;
    }
}

// log-probabilities, and for the gradient of the preference loss what is not the pair's
__global__ __launch_bounds__(kColumns *kParts) void log_prob_columns_kernel(const LossArgs a, const Shape z, const LossSpace w, const bool gradient)
{
    __shared__ double lds[kColumns * kParts / kWave][kColumns], logp[kColumns];
    __shared__ float tops[kColumns];
    const int j = threadIdx.x & (kColumns - 1), part = threadIdx.x / kColumns, col = blockIdx.x * kColumns + j;
    const Column c = column_of(a, w.partial, z.chunks, col, part, tops, lds);
    if (part == 0) {
        logp[j] = c.logp;
        if (col < a.batch) {
            w.logp[col] = c.logp;
            if (a.logp) a.logp[col] = static_cast<float>(c.logp);
            if (gradient) w.columns[col] = state_of(c, in_sequences(a, col) && c.counts ? 1.f : 0.f);
        }
    }
    if (gradient || gridDim.x > 1 || !a.sums) return;
    __syncthreads();
    for (int k = threadIdx.x; k < a.sequences; k += blockDim.x) {
        const int2 at = columns_of(a, k);
        double s = 0;
        for (int i = at.x; i < at.y; ++i) s += logp[i];
        a.sums[k] = static_cast<float>(s);
    }
}

// ---- sequences ----
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
    __shared__ double lds[2][kSequenceThreads / kWave];
    const int pair = blockIdx.x, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, waves = static_cast<int>(blockDim.x >> 6);
    // (of a pair the sequences lie next to each other, if anything)
    const int2 at[2] = {columns_of(a, 2 * pair), columns_of(a, 2 * pair + 1)};
    double s[2] = {0, 0};
    for (int k = 0; k < 2; ++k)
#pragma unroll 4
        for (int col = at[k].x + static_cast<int>(threadIdx.x); col < at[k].y; col += blockDim.x) s[k] += w.logp[col];
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        s[0] += __shfl_xor(s[0], d, kWave);
        s[1] += __shfl_xor(s[1], d, kWave);
    }
    if (lane == 0) lds[0][wave] = s[0], lds[1][wave] = s[1];
    __syncthreads();
    s[0] = s[1] = 0;
    for (int u = 0; u < waves; ++u) s[0] += lds[0][u], s[1] += lds[1][u];
    const double x = margin_of(a, pair, s[0], s[1]);
    const PairTerm t = pair_term(a, x);
    if (threadIdx.x == 0) {
        if (a.sums) a.sums[2 * pair] = static_cast<float>(s[0]), a.sums[2 * pair + 1] = static_cast<float>(s[1]);
        if (a.margins) a.margins[pair] = static_cast<float>(x);
        w.shares[pair] = t.loss;
    }
    for (int k = 0; k < 2; ++k) {
        const float c = static_cast<float>((k ? -t.slope : t.slope) / gridDim.x);
        for (int col = at[k].x + static_cast<int>(threadIdx.x); col < at[k].y; col += blockDim.x) {
            ColumnState q = w.columns[col];
            if (q.c == 0.f) continue;
            q.share *= c;
            q.c = c;
            w.columns[col] = q;
        }
    }
}

// the shares of the loss, added up by one wave in one fixed order
__device__ __forceinline__ double wave_sum(const double *v, int n, int step)
{
    double s = 0;
#pragma unroll 4
    for (int b = threadIdx.x; b < n; b += kWave) s += v[static_cast<int64_t>(step) * b];
    for (int d = 1; d < kWave; d <<= 1) s += __shfl_xor(s, d, kWave);
    return s;
}
__device__ __forceinline__ void write_stats(const LossArgs &a, const double *shares, int n)
{
    for (int k = 0; k < 4; ++k) {
        const double s = wave_sum(shares + k, n, 4);
        if (threadIdx.x == 0) a.stats[k] = static_cast<float>(s);
    }
}
__global__ __launch_bounds__(kWave) void stats_kernel(const LossArgs a, const double *shares, const int n) { write_stats(a, shares, n); }

template <int U, TileKind T, bool PAST>
__device__ __forceinline__ void write_gradient(const LossArgs &a, const LossSpace &w, const Spot &p, int first, int end)
{
    ColumnState c[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = w.columns[p.col + (T == kWhole ? k : min(k, p.n - 1))];
    const float4 top = make_float4(c[0].top, c[1].top, c[2].top, c[3].top);
    for (int i = first + p.slot; i < end; i += U * p.slots) {
        float4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load_of<T>(a.Z + min(i + u * p.slots, end - 1) * a.ldz, p);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = i + u * p.slots;
            if (row < end) store_of<T, PAST>(a.dZ + row * a.lddz, p, gradient_of4(exp_of4(own_of<T>(x[u], p) - top), c, row));
        }
    }
}
// One work-group: a chunk of the classes in a tile of columns, from the last one read to the first.  `shares`: how many shares of the loss there are
// (policy: of four terms each).
template <int U>
__global__ __launch_bounds__(kThreads) void logits_gradient_kernel(const LossArgs a, const Shape z, const LossSpace w, const int shares)
{
    if (blockIdx.x == 0 && threadIdx.x < kWave) {
        if (a.stats) {
            write_stats(a, w.shares, shares);
        } else if (a.loss) {
            const double s = wave_sum(w.shares, shares, 1);
            if (threadIdx.x == 0) *a.loss = static_cast<float>(s / shares);
        }
    }
    const Part part = part_of(gridDim.x - 1 - blockIdx.x, z);
    const Spot p = spot_in(part.tile, z.lg, a.batch, z.past);
    if (p.n == 0) return;
    const int first = part.chunk * z.rows, end = min(a.classes, first + z.rows);
    // (few rows a thread: never past the caches, and little code, which small launches wait for)
    with_kind(p, [&](auto kind) {
        if (U == kLoads && z.past) write_gradient<U, kind, U == kLoads>(a, w, p, first, end);
        else write_gradient<U, kind, false>(a, w, p, first, end);
    });
}

// ---- launches ----
constexpr int64_t kFewTiles = 256;       // one per compute unit
// Chunks of eight rows a thread, in all tiles, below which they are of two rows a thread: where they are added up (4096 classes x 100: 19.1 -> 15.8 us; with 128 chunks
// already, 8192 x 100, more of them take 20.1 instead of 18.0), and where only the gradient is cut into them (1001 x 777, three launches: 15.8 -> 13.7).
constexpr int64_t kFewSums = 128, kFewGradients = 512;

// Of columns that are cut into chunks.
Shape chunks_of(int32_t classes, int32_t batch, bool sums)
{
    Shape z{};
    z.lg = lanes_for(batch, kLanes);
    z.tiles = static_cast<int32_t>((batch + (INT64_C(4) << z.lg) - 1) >> (z.lg + 2));
    const auto cut = [&](int loads) { return static_cast<int64_t>(loads) * (kThreads >> z.lg); };
    // a few rows a thread where that gives more compute units something to do
    z.loads = z.tiles * ((classes + cut(kLoads) - 1) / cut(kLoads)) < (sums ? kFewSums : kFewGradients) ? kFewLoads : kLoads;
    const int64_t step = cut(z.loads), most = (classes + step - 1) / step, want = std::max<int64_t>(1, kBlocks / z.tiles);
    const int64_t steps = (most + std::min(most, want) - 1) / std::min(most, want);
    z.rows = static_cast<int>(std::min<int64_t>(steps * step, classes));
    z.chunks = static_cast<int>((static_cast<int64_t>(classes) + z.rows - 1) / z.rows);
    z.past = 8 * static_cast<int64_t>(classes) * batch > kCacheBytes;
    return z;
}

// Of columns that a work-group holds.
struct Held {
    Shape z;
    int rows, threads;       // rows: of a thread; 0 where the columns are cut into chunks
};
Held held_of(int32_t classes, int32_t batch)
{
    Held h{};
    const auto tiles = [&](int lg) { return (batch + (INT64_C(4) << lg) - 1) >> (lg + 2); };
    const auto held = [&](int lg) { return static_cast<int64_t>(classes) << lg; };
    int lg = lanes_for(batch, kLanes);
    // The most that a work-group holds of columns that make few tiles, in quads.  Twice as many in one tile of 8 to 128 columns (policy loss, preference loss and
    // log-probabilities of 500 classes x 32, held and cut into chunks: 9.4, 9.4, 5.6 us and 11.6, 15.0, 11.4; 128 x 100: 11.0, 12.0, 5.5 and 12.6, 15.2, 11.3); not of fewer columns,
    // which keep few lanes busy (4096 x 3: 20.9, 20.1, 11.3 held, 13.1, 15.2, 8.5 in chunks), nor of 256, whose narrow tiles are as fast or
    // faster (64 x 256: 10.2, 14.1, 8.0 in one tile, 9.0, 11.1, 7.6 in 64).
    const auto most = [&](int lg) { return (tiles(lg) == 1 && lg > 0 && lg < kLanes ? 4 : 2) * kHeldThreads; };
    // one tile for all, with no launch for the sums behind it; or tiles of 32 columns, wider ones where they leave lanes idle, narrower ones where there
    // would be few
    if (tiles(lg) > 1 || held(lg) > most(lg)) {
        const int widest = lg;
        lg = lanes_for(batch, 3);
        while (lg < widest && held(lg) < kWave) ++lg;
        while (lg > 0 && tiles(lg) < kFewTiles && held(lg) > kWave) --lg;
    }
    h.z.lg = lg;
    h.z.tiles = static_cast<int32_t>(tiles(lg));
    h.z.past = 8 * static_cast<int64_t>(classes) * batch > kCacheBytes;
    if (held(lg) > kHeldRows * kHeldThreads || (h.z.tiles < kFewTiles && held(lg) > most(lg))) return h;
    h.rows = 1;
    while (h.rows < kHeldRows && held(lg) > (h.rows < 4 ? 256 : kHeldThreads) * h.rows) h.rows *= 2;
    const int64_t threads = std::max<int64_t>((held(lg) + h.rows - 1) / h.rows, 4 << lg);
    h.threads = static_cast<int>((threads + kWave - 1) / kWave * kWave);
    return h;
}
int column_blocks(int32_t batch) { return static_cast<int>((static_cast<int64_t>(batch) + kColumns - 1) / kColumns); }

template <What W, int Most = kHeldRows>
void launch_held(const LossArgs &a, const Held &h, const LossSpace &w, const Borders &b, hipStream_t s)
{
    if constexpr (Most > 1)
        if (h.rows < Most) return launch_held<W, Most / 2>(a, h, w, b, s);
    const int lds = static_cast<int>(sizeof(float4) + 4 * sizeof(double)) * (h.threads / kWave << h.z.lg);
    held_kernel<Most, W><<<static_cast<uint32_t>(h.z.tiles), h.threads, lds, s>>>(a, h.z, w, b);
}
void launch_log_sums(const LossArgs &a, const Shape &z, const LossSpace &w, hipStream_t s)
{
    const uint32_t grid = static_cast<uint32_t>(z.tiles) * z.chunks;
    if (z.loads == kLoads) log_sum_kernel<kLoads><<<grid, kThreads, 0, s>>>(a, z, w.partial);
    else log_sum_kernel<kFewLoads><<<grid, kThreads, 0, s>>>(a, z, w.partial);
}
void launch_gradient(const LossArgs &a, const Shape &z, const LossSpace &w, int shares, hipStream_t s)
{
    const uint32_t grid = static_cast<uint32_t>(z.tiles) * z.chunks;
    if (z.loads == kLoads) logits_gradient_kernel<kLoads><<<grid, kThreads, 0, s>>>(a, z, w, shares);
    else logits_gradient_kernel<kFewLoads><<<grid, kThreads, 0, s>>>(a, z, w, shares);
}
// Threads of a work-group that adds up a sequence: few for short ones (pairs of 62 columns on average: 14.2 -> 13.3 us with the launches around), not for longer ones (512: 17.6, with few
// 20.5).
int sequence_threads(const LossArgs &a) { return a.batch / a.sequences < 256 ? 256 : kSequenceThreads; }
bool too_large(const Held &h, const Shape &z, int32_t batch, int32_t sequences)
{
    return (h.rows && !fits_launch(h.z.tiles, h.threads)) || !fits_launch(static_cast<int64_t>(z.tiles) * z.chunks, kThreads) || (!h.rows && !fits_launch(column_blocks(batch), kColumns * kParts)) ||
           !fits_launch(sequences, kSequenceThreads);
}

}  // namespace

LossSpace loss_space(void *memory, int32_t classes, int32_t batch, int32_t sequences)
{
    const Held h = held_of(classes, batch);
    const int64_t chunks = h.rows ? 0 : chunks_of(classes, batch, true).chunks;
    LossSpace w;
    w.columns = static_cast<ColumnState *>(memory);
    w.logp = reinterpret_cast<double *>(w.columns + batch);
    w.shares = w.logp + batch;
    w.partial = reinterpret_cast<float *>(w.shares + std::max<int64_t>(4 * static_cast<int64_t>(h.rows ? h.z.tiles : column_blocks(batch)), sequences));
    w.bytes = reinterpret_cast<char *>(w.partial + 2 * chunks * batch) - static_cast<char *>(memory);
    return w;
}

hipError_t launch_log_probs(const LossArgs &a, hipStream_t s)
{
    const Held h = held_of(a.classes, a.batch);
    const Shape z = chunks_of(a.classes, a.batch, !h.rows);
    const LossSpace w = loss_space(a.workspace, a.classes, a.batch, a.sequences);
    if (too_large(h, z, a.batch, a.sequences)) return hipErrorInvalidConfiguration;
    bool summed;
    if (h.rows) {
        launch_held<kLogProbs>(a, h, w, Borders{}, s);
        summed = h.z.tiles == 1;
    } else {
        launch_log_sums(a, z, w, s);
        log_prob_columns_kernel<<<column_blocks(a.batch), kColumns * kParts, 0, s>>>(a, z, w, false);
        summed = column_blocks(a.batch) == 1;
    }
    if (a.sums && !summed) sequence_sums_kernel<<<a.sequences, sequence_threads(a), 0, s>>>(a, w);
    return hipGetLastError();
}

hipError_t launch_policy(const LossArgs &a, hipStream_t s)
{
    const Held h = held_of(a.classes, a.batch);
    const Shape z = chunks_of(a.classes, a.batch, !h.rows);
    const LossSpace w = loss_space(a.workspace, a.classes, a.batch, 0);
    if (too_large(h, z, a.batch, 0)) return hipErrorInvalidConfiguration;
    // In roundings of 2^-24: an exponential is off by |z - top| + 2, and the mean of |z - top| over p is at most log(classes) < 21 (z - top itself is
    // rounded as well, by as much).  A thread adds up its rows, in chunks eight at a time and then their sum to the others', which takes an exponential and
    // three roundings; ten levels of pairs and up to 16 waves follow with four each.
    const double adds = h.rows ? h.rows : 5.0 * (z.rows / ((kThreads >> z.lg) * z.loads) + 1) + z.loads;
    const Borders b{a.clip_low < 1.f ? log1p(-static_cast<double>(a.clip_low)) : -INFINITY, log1p(static_cast<double>(a.clip_high)),
                    static_cast<float>((2 * 21 + 2 + 10 * 4 + 16 * 4 + adds) / (1 << 24))};
    if (h.rows) {
        launch_held<kPolicy>(a, h, w, b, s);
        if (h.z.tiles > 1) stats_kernel<<<1, kWave, 0, s>>>(a, w.shares, h.z.tiles);
        return hipGetLastError();
    }
    launch_log_sums(a, z, w, s);
    policy_columns_kernel<<<column_blocks(a.batch), kColumns * kParts, 0, s>>>(a, z, w, b);
    launch_gradient(a, z, w, column_blocks(a.batch), s);
    return hipGetLastError();
}

hipError_t launch_preference(const LossArgs &a, hipStream_t s)
{
    const Held h = held_of(a.classes, a.batch);
    const Shape z = chunks_of(a.classes, a.batch, !h.rows);
    const LossSpace w = loss_space(a.workspace, a.classes, a.batch, a.sequences);
    if (too_large(h, z, a.batch, a.sequences / 2)) return hipErrorInvalidConfiguration;
    if (h.rows) {
        launch_held<kPreference>(a, h, w, Borders{}, s);
        if (h.z.tiles == 1) return hipGetLastError();
    } else {
        launch_log_sums(a, z, w, s);
        log_prob_columns_kernel<<<column_blocks(a.batch), kColumns * kParts, 0, s>>>(a, z, w, true);
    }
    pairs_kernel<<<a.sequences / 2, sequence_threads(a), 0, s>>>(a, w);
    launch_gradient(a, z, w, a.sequences / 2, s);
    return hipGetLastError();
}

}  // namespace nerva
