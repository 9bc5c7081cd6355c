// Group norm with an activation and dropout, forward and backward, and dropout by itself.
//
// Group g of column c holds m = features / groups rows:
//     mean = (1/m) sum x,   rstd = 1 / sqrt((1/m) sum (x - mean)^2 + eps),   xh = (x - mean) rstd,   u = gamma xh + beta,   y = D act(u)
// backward, with e = D dy act'(u) and h = gamma e:
//     dx = rstd (h - (1/m) sum h - xh (1/m) sum h xh),   dgamma = sum over columns of e xh,   dbeta = sum over columns of e
// D is 0 where an entry is dropped and 1/(1 - p) elsewhere; it is drawn from counters wherever it is needed and never stored.
//
// All of it is bound by memory: 8 bytes an entry forward, 12 backward, against some 30 operations.  A work-group owns a group of rows in a tile of
// columns and holds all of its entries in registers, so that statistics and results take one read.  Groups that are too long for that
// are cut into chunks: one launch leaves every chunk's statistics, a second one adds them up and reads the entries again.
#include <algorithm>
#include <type_traits>

#include "columns.h"
#include "experts.h"
#include "norm.h"

namespace nerva {
namespace {

constexpr int kLanes = 3;              // log2 of the quads of a tile: 32 columns, whose rows are 128-byte lines
constexpr int kThreadsMost = 1024;
constexpr int kChunkThreads = 256;     // of groups that are cut into chunks

// ---- the generator ----
// Philox4x32 of 10 rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011), key = seed.  Counter (column / 4, row / 2,
// layer, step) gives the bits of four columns in two rows: word column % 4, its low half for the even row and its high half for the odd one.  So
// an entry's bits depend on neither leading dimension nor batch nor launch.  16 bits an entry halve the generator's work, which
// is not small beside 8 bytes an entry (20 products of 32 bits for 8 entries: 67 M entries normalised and dropped issue 39 instructions an
// entry, which keep the vector units busy for some two thirds of the 105 us); the probability is a multiple of 2^-16 for it, and the scale is that of
// the multiple.
struct Bits {
    uint32_t x, y, z, w;
};
__device__ __forceinline__ Bits philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = static_cast<uint64_t>(0xD2511F53u) * c0, b = static_cast<uint64_t>(0xCD9E8D57u) * c2;
        c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
        c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
        c1 = static_cast<uint32_t>(b);
        c3 = static_cast<uint32_t>(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {c0, c1, c2, c3};
}
struct Drawn {
    uint32_t k0, k1, layer, step;
};
__device__ __forceinline__ Drawn drawn_from(const DropArgs &d)
{
    const uint64_t seed = static_cast<uint64_t>(d.state[0]), step = static_cast<uint64_t>(d.state[1]);
    return {static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32), d.layer, static_cast<uint32_t>(step)};
}
__device__ __forceinline__ Bits bits_of(const Drawn &d, int col, int pair)
{
    return philox(static_cast<uint32_t>(col) >> 2, static_cast<uint32_t>(pair), d.layer, d.step, d.k0, d.k1);
}
// row 0 or 1 of the pair: x * scale where it is kept, 0 (whatever x is) where it is dropped
__device__ __forceinline__ float4 drop(float4 x, const Bits &b, int row, const DropArgs &d)
{
    const uint32_t shift = row ? 16 : 0, low = 0xFFFFu;
    return make_float4((b.x >> shift & low) >= d.cut ? x.x * d.scale : 0.f, (b.y >> shift & low) >= d.cut ? x.y * d.scale : 0.f,
                       (b.z >> shift & low) >= d.cut ? x.z * d.scale : 0.f, (b.w >> shift & low) >= d.cut ? x.w * d.scale : 0.f);
}

// ---- activations ----
constexpr int kRelu = 1, kSilu = 2;
// (v_rcp_f32 is off by one unit in the last place, a division would take ten instructions.  The argument's rounding counts where exp(-u) does: below
// 1.2 roundings for u >= 0, 2 |u| for u < 0, where the result is small.)
__device__ __forceinline__ float sigmoid_of(float u) { return __builtin_amdgcn_rcpf(1.f + exp_of(-u)); }
// (act is the same for all threads; a NaN stays one)
__device__ __forceinline__ float4 activate4(float4 u, int act)
{
    if (act == kRelu) return make_float4(u.x < 0.f ? 0.f : u.x, u.y < 0.f ? 0.f : u.y, u.z < 0.f ? 0.f : u.z, u.w < 0.f ? 0.f : u.w);
    if (act == kSilu) return make_float4(u.x * sigmoid_of(u.x), u.y * sigmoid_of(u.y), u.z * sigmoid_of(u.z), u.w * sigmoid_of(u.w));
    return u;
}
__device__ __forceinline__ float silu_slope(float u)
{
    const float s = sigmoid_of(u);
    return s * fmaf(u, 1.f - s, 1.f);
}
// e act'(u)
__device__ __forceinline__ float4 activate_back4(float4 e, float4 u, int act)
{
    if (act == kRelu) return keep_where_positive(e, u);
    return make_float4(e.x * silu_slope(u.x), e.y * silu_slope(u.y), e.z * silu_slope(u.z), e.w * silu_slope(u.w));
}

// ---- sums down the columns ----
// Sum over the threads with the same columns, the same bits in all of them; lds: one float4 per wave and quad, not to be written again before
// the next barrier but one.
__device__ __forceinline__ float4 column_sum(float4 v, int lg, float4 *lds)
{
    for (int d = 1 << lg; d < kWave; d <<= 1) v = v + shfl_xor4(v, d);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    const int lane = threadIdx.x & (kWave - 1), q = threadIdx.x & ((1 << lg) - 1);
    if (lane < (1 << lg)) lds[(threadIdx.x >> 6 << lg) + lane] = v;
    __syncthreads();
    float4 s = lds[q];
    for (int w = 1; w < waves; ++w) s = s + lds[(w << lg) + q];
    return s;
}

// the memory of a second sum
__device__ __forceinline__ float4 *second(float4 *lds, int lg) { return lds + (blockDim.x >> 6 << lg); }

// A thread's rows: K pairs, `slots` pairs apart, of which those in [first, end) belong to its work-group's rows.  Pairs go by the rows' numbers in
// the whole operand, as the generator's do.
template <int K>
struct Rows {
    int pair, step, first, end;
    __device__ __forceinline__ int row(int i) const { return 2 * (pair + (i >> 1) * step) + (i & 1); }
    __device__ __forceinline__ bool in(int i) const { const int f = row(i); return f >= first && f < end; }
    // of rows outside some row is read, to be left out by whoever uses it
    __device__ __forceinline__ int readable(int i) const { return min(max(row(i), first), end - 1); }
    __device__ __forceinline__ void load(const float *X, int64_t ld, const Spot &p, float4 (&x)[2 * K]) const
    {
        load_quads([&](int i) { return X + readable(i) * ld; }, p, x);
    }
    // the same for the backward pass
    __device__ __forceinline__ void load_singly(const float *X, int64_t ld, const Spot &p, float4 (&x)[2 * K]) const
    {
        if (p.whole) {
#pragma unroll
            for (int i = 0; i < 2 * K; ++i) x[i] = ld4(X + readable(i) * ld + p.col);
        } else {
#pragma unroll
            for (int i = 0; i < 2 * K; ++i) x[i] = nerva::load_singly(X + readable(i) * ld, p);
        }
    }
};
// rows [first, end) of chunk `chunk` of a group: a chunk is as many pairs as a work-group holds
template <int K>
__device__ __forceinline__ Rows<K> rows_of(const NormArgs &a, int group, int chunk, const Spot &p)
{
    const int m = a.features / a.groups, first = group * m, pairs = K * p.slots;
    Rows<K> r;
    const int pair0 = (first >> 1) + chunk * pairs;
    r.pair = pair0 + p.slot;
    r.step = p.slots;
    r.first = max(first, 2 * pair0);
    r.end = min(first + m, 2 * (pair0 + pairs));
    return r;
}

struct Shape {
    int lg, chunks, slabs;
    bool past, joined;       // joined: the first chunk's place holds what all chunks come to
    int64_t tiles;
};
// A mean that its sum's roundings put off, from the differences of `n` entries to it: their mean is what it is off by, and
//     sum (x - mean)^2 = sum d^2 - (sum d)^2 / n.
// Without this step a group of equal numbers far from zero, whose differences are 0, comes out as the roundings of its mean over sqrt(eps) (273 times 1000.1: 0.019
// instead of 0).  With it the mean is off by the one rounding of its own 32 bits and what differences of their size leave.  Both passes go by that rounded mean, so that
// they see the same arguments of the activation.  A mean below the spread is as good as the differences' sum would make it, and a tile with no other is spared the sum (2048 rows
// in one group x 8192 columns, forward: 25.2 us, with it 26.3).
// differences(): this thread's share of it.
__device__ __forceinline__ bool far(float mean, float squares, float n) { return n * mean * mean > squares; }   // (not with an infinity or NaN)
template <typename F>
__device__ __forceinline__ void correct(float4 &mean, float4 &squares, float n, int lg, float4 *lds, F &&differences)
{
    const bool x = far(mean.x, squares.x, n), y = far(mean.y, squares.y, n), z = far(mean.z, squares.z, n), w = far(mean.w, squares.w, n);
    if (!__any(x || y || z || w)) return;   // (each wave holds all columns of the tile, with the same bits: all waves go the same way)
    const float4 d = column_sum(differences(), lg, lds), off = 1.f / n * d, s = squares - d * off;
    mean = make_float4(x ? mean.x + off.x : mean.x, y ? mean.y + off.y : mean.y, z ? mean.z + off.z : mean.z, w ? mean.w + off.w : mean.w);
    squares = make_float4(x ? fmaxf(s.x, 0.f) : squares.x, y ? fmaxf(s.y, 0.f) : squares.y, z ? fmaxf(s.z, 0.f) : squares.z, w ? fmaxf(s.w, 0.f) : squares.w);
}
// statistics of the entries that the work-group holds: mean and sum of squares about it; x becomes its difference from the mean
template <int K>
__device__ __forceinline__ void statistics(float4 (&x)[2 * K], const Rows<K> &r, int lg, float4 *lds, float4 &mean, float4 &squares)
{
    const int n = r.end - r.first;
    float4 s = splat(0.f);
#pragma unroll
    for (int i = 0; i < 2 * K; ++i)
        if (r.in(i)) s = s + x[i];
    mean = 1.f / static_cast<float>(n) * column_sum(s, lg, lds);
    float4 s2 = splat(0.f);
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        const float4 d = x[i] - mean;
        if (r.in(i)) s2 = fma4(d, d, s2);
    }
    squares = column_sum(s2, lg, second(lds, lg));
    correct(mean, squares, static_cast<float>(n), lg, lds, [&] {
        float4 s1 = splat(0.f);
#pragma unroll
        for (int i = 0; i < 2 * K; ++i)
            if (r.in(i)) s1 = s1 + (x[i] - mean);
        return s1;
    });
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) x[i] = x[i] - mean;
}
__device__ __forceinline__ float4 rstd_of(float4 squares, int m, float eps)
{
    const float4 v = 1.f / static_cast<float>(m) * squares + splat(eps);
    return make_float4(1.f / sqrtf(v.x), 1.f / sqrtf(v.y), 1.f / sqrtf(v.z), 1.f / sqrtf(v.w));
}

// the rows' gamma and beta
template <int K>
struct Affine {
    float gamma[2 * K], beta[2 * K];
    __device__ __forceinline__ void load(const NormArgs &a, const Rows<K> &r)
    {
#pragma unroll
        for (int i = 0; i < 2 * K; ++i) {
            gamma[i] = a.gamma ? a.gamma[r.readable(i)] : 1.f;
            beta[i] = a.beta ? a.beta[r.readable(i)] : 0.f;
        }
    }
};
// HELD: the rows' gamma and beta are in w
template <int K, bool HELD>
__device__ __forceinline__ void write_forward(const NormArgs &a, const float4 (&x)[2 * K], const Rows<K> &r, const Affine<K> &w, const Spot &p, float4 rstd)
{
    Drawn d{};
    if (a.drop.cut) d = drawn_from(a.drop);
    Bits bits{};
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        const int f = r.row(i);
        if (!(i & 1)) {
            __builtin_amdgcn_sched_barrier(0);   // (a pair after the other: all at once take more registers than there are)
            if (a.drop.cut) bits = bits_of(d, p.col, f >> 1);
        }
        if (!r.in(i)) continue;
        const float4 xh = x[i] * rstd;   // (x: less the mean)
        const float gamma = HELD ? w.gamma[i] : a.gamma ? a.gamma[f] : 1.f, beta = HELD ? w.beta[i] : a.beta ? a.beta[f] : 0.f;
        float4 y = activate4(fma4(splat(gamma), xh, splat(beta)), a.act);
        if (a.drop.cut) y = drop(y, bits, i & 1, a.drop);
        store_quad(a.Y + f * a.ldy, p, y);
    }
}

// One work-group: a chunk of a group in a tile of columns.  WHOLE: the chunk is the group.  Otherwise its statistics go to the workspace,
// {mean, sum of squares about it} (groups, chunks, batch).
template <int K, int T, bool WHOLE>
__global__ __launch_bounds__(T) void norm_forward_kernel(const NormArgs a, const Shape z)
{
    extern __shared__ float4 lds[];   // two per wave and quad
    const int64_t unit = blockIdx.x / z.chunks, tile = near_tile(unit % z.tiles, z.tiles, z.lg);
    const int chunk = static_cast<int>(blockIdx.x % z.chunks), group = static_cast<int>(unit / z.tiles);
    const Spot p = spot_in(tile, z.lg, a.batch, z.past);
    const Rows<K> r = rows_of<K>(a, group, chunk, p);
    float4 x[2 * K], mean, squares;
    r.load(a.X, a.ldx, p, x);
    constexpr bool kHeld = K <= 2;   // (asked for before the sums where there are registers for them)
    Affine<K> w;
    if constexpr (WHOLE && kHeld) w.load(a, r);
    statistics<K>(x, r, z.lg, lds, mean, squares);
    if constexpr (WHOLE) {
        const float4 rstd = rstd_of(squares, r.end - r.first, a.eps);
        if (p.slot == 0) {
            if (a.mean) store_quad(a.mean + group * a.lds, p, mean);
            if (a.rstd) store_quad(a.rstd + group * a.lds, p, rstd);
        }
        write_forward<K, kHeld>(a, x, r, w, p, rstd);
    } else if (p.slot == 0) {
        float *const at = a.workspace + 2 * (static_cast<int64_t>(group) * z.chunks + chunk) * a.batch;
        store_quad(at, p, mean);
        store_quad(at + a.batch, p, squares);
    }
}

// A group's statistics from those of its chunks: means weighed by their rows, then all squares about the mean of the group (Chan, Golub, LeVeque 1979), which is
// corrected as a chunk's is.  A thread adds up every slots-th chunk.
template <int K>
__device__ __forceinline__ void join_statistics(const NormArgs &a, const Shape &z, int group, const Spot &p, float4 *lds, float4 &mean, float4 &squares)
{
    const float *const stats = a.workspace + 2 * static_cast<int64_t>(group) * z.chunks * a.batch;
    if (z.joined) {
        mean = load_quad(stats, p);
        squares = load_quad(stats + a.batch, p);
        return;
    }
    mean = squares = splat(0.f);
    for (int c = p.slot; c < z.chunks; c += p.slots) {
        const Rows<K> of = rows_of<K>(a, group, c, p);
        mean = fma4(splat(static_cast<float>(of.end - of.first)), load_quad(stats + 2 * static_cast<int64_t>(c) * a.batch, p), mean);
    }
    mean = 1.f / static_cast<float>(a.features / a.groups) * column_sum(mean, z.lg, lds);
    for (int c = p.slot; c < z.chunks; c += p.slots) {
        const Rows<K> of = rows_of<K>(a, group, c, p);
        const float *const at = stats + 2 * static_cast<int64_t>(c) * a.batch;
        const float4 d = load_quad(at, p) - mean;
        squares = squares + fma4(static_cast<float>(of.end - of.first) * d, d, load_quad(at + a.batch, p));
    }
    squares = column_sum(squares, z.lg, second(lds, z.lg));
    correct(mean, squares, static_cast<float>(a.features / a.groups), z.lg, lds, [&] {
        float4 s1 = splat(0.f);
        for (int c = p.slot; c < z.chunks; c += p.slots) {
            const Rows<K> of = rows_of<K>(a, group, c, p);
            s1 = fma4(splat(static_cast<float>(of.end - of.first)), load_quad(stats + 2 * static_cast<int64_t>(c) * a.batch, p) - mean, s1);
        }
        return s1;
    });
}
// the sums of h and h xh over the chunks, in the same way
__device__ __forceinline__ void join_sums(const NormArgs &a, const Shape &z, int group, const Spot &p, float4 *lds, float4 &s, float4 &sx)
{
    const float *const sums = a.workspace + 2 * static_cast<int64_t>(group) * z.chunks * a.batch;
    if (z.joined) {
        s = load_singly(sums, p);
        sx = load_singly(sums + a.batch, p);
        return;
    }
    s = sx = splat(0.f);
    for (int c = p.slot; c < z.chunks; c += p.slots) {
        const float *const at = sums + 2 * static_cast<int64_t>(c) * a.batch;
        s = s + load_singly(at, p);
        sx = sx + load_singly(at + a.batch, p);
    }
    s = column_sum(s, z.lg, lds);
    sx = column_sum(sx, z.lg, second(lds, z.lg));
}
// Groups of very many chunks: one work-group per group and tile leaves what they come to in the first one's place, before all the work-groups of the second
// launch would add them up.
template <int K, bool BACKWARD>
__global__ __launch_bounds__(kChunkThreads) void norm_join_kernel(const NormArgs a, const Shape z)
{
    extern __shared__ float4 lds[];   // two per wave and quad
    const int group = static_cast<int>(blockIdx.x / z.tiles);
    const Spot p = spot_in(blockIdx.x % z.tiles, z.lg, a.batch);
    float4 one, two;
    if constexpr (BACKWARD) join_sums(a, z, group, p, lds, one, two);
    else join_statistics<K>(a, z, group, p, lds, one, two);
    if (p.slot) return;
    float *const at = a.workspace + 2 * static_cast<int64_t>(group) * z.chunks * a.batch;
    store_quad(at, p, one);
    store_quad(at + a.batch, p, two);
}

// the second launch of a group of several chunks
template <int K>
__global__ __launch_bounds__(kChunkThreads) void norm_apply_kernel(const NormArgs a, const Shape z)
{
    extern __shared__ float4 lds[];   // two per wave and quad
    const int64_t unit = blockIdx.x / z.chunks, tile = near_tile(unit % z.tiles, z.tiles, z.lg);
    const int chunk = static_cast<int>(blockIdx.x % z.chunks), group = static_cast<int>(unit / z.tiles);
    const Spot p = spot_in(tile, z.lg, a.batch, z.past);
    const Rows<K> r = rows_of<K>(a, group, chunk, p);
    float4 x[2 * K];
    r.load(a.X, a.ldx, p, x);
    Affine<K> w;
    w.load(a, r);
    const int m = a.features / a.groups;
    float4 mean, squares;
    join_statistics<K>(a, z, group, p, lds, mean, squares);
    const float4 rstd = rstd_of(squares, m, a.eps);
    if (p.slot == 0 && chunk == 0) {
        if (a.mean) store_quad(a.mean + group * a.lds, p, mean);
        if (a.rstd) store_quad(a.rstd + group * a.lds, p, rstd);
    }
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) x[i] = x[i] - mean;
    write_forward<K, true>(a, x, r, w, p, rstd);
}

// ---- backward ----
// x becomes xh, g becomes h; what the rows add to the gradients of gamma and beta from this thread's columns is added to `dg` and `db`
template <int K>
__device__ __forceinline__ void form_h(const NormArgs &a, float4 (&x)[2 * K], float4 (&g)[2 * K], const Rows<K> &r, const Affine<K> &w, const Spot &p, float4 mean, float4 rstd,
                                       float (&dg)[2 * K], float (&db)[2 * K])
{
    Drawn d{};
    if (a.drop.cut) d = drawn_from(a.drop);
    Bits bits{};
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        if (!(i & 1)) {
            __builtin_amdgcn_sched_barrier(0);
            if (a.drop.cut) bits = bits_of(d, p.col, r.row(i) >> 1);
        }
        x[i] = (x[i] - mean) * rstd;
        float4 e = g[i];
        if (a.drop.cut) e = drop(e, bits, i & 1, a.drop);
        if (a.act) e = activate_back4(e, fma4(splat(w.gamma[i]), x[i], splat(w.beta[i])), a.act);
        const float4 own = existing(e, p);
        if (r.in(i)) {
            dg[i] += sum4(existing(e * x[i], p));
            db[i] += sum4(own);
        }
        g[i] = w.gamma[i] * e;
    }
}
template <int K>
__device__ __forceinline__ void column_sums_of_h(const float4 (&x)[2 * K], const float4 (&g)[2 * K], const Rows<K> &r, int lg, float4 *lds,
                                                 float4 &s, float4 &sx)
{
    float4 t = splat(0.f), tx = splat(0.f);
#pragma unroll
    for (int i = 0; i < 2 * K; ++i)
        if (r.in(i)) {
            t = t + g[i];
            tx = fma4(g[i], x[i], tx);
        }
    s = column_sum(t, lg, lds);
    sx = column_sum(tx, lg, second(lds, lg));
}
template <int K>
__device__ __forceinline__ void write_backward(const NormArgs &a, const float4 (&x)[2 * K], const float4 (&g)[2 * K], const Rows<K> &r, const Spot &p, float4 rstd, float4 s,
                                               float4 sx)
{
    const float part = 1.f / static_cast<float>(a.features / a.groups);
    s = part * s;
    sx = part * sx;
#pragma unroll
    for (int i = 0; i < 2 * K; ++i)
        if (r.in(i)) store_quad(a.dX + r.row(i) * a.lddx, p, rstd * (fma4(make_float4(-x[i].x, -x[i].y, -x[i].z, -x[i].w), sx, g[i]) - s));
}
// Sums of the gradients of gamma and beta over the work-group's columns, to slab `slab` of (slabs, 2, features), or to the gradients themselves
// where there is one slab.
template <int K>
__device__ __forceinline__ void write_rows(const NormArgs &a, float *slabs, int n_slabs, int slab, const Rows<K> &r, int lg, float (&dg)[2 * K], float (&db)[2 * K])
{
    if (!a.dgamma && !a.dbeta) return;
    float *const g = n_slabs == 1 ? a.dgamma : slabs + 2 * static_cast<int64_t>(slab) * a.features;
    float *const b = n_slabs == 1 ? a.dbeta : slabs + (2 * static_cast<int64_t>(slab) + 1) * a.features;
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        if (lg == 3) {   // (without the local memory's crossbar: 47.3 -> 46.2 us for 8 x 1024 rows x 1024 columns, both ways)
            dg[i] = group_sum<8>(dg[i]);
            db[i] = group_sum<8>(db[i]);
        } else {
            for (int d = 1; d < 1 << lg; d <<= 1) {
                dg[i] += __shfl_xor(dg[i], d, kWave);
                db[i] += __shfl_xor(db[i], d, kWave);
            }
        }
        if (!(threadIdx.x & ((1 << lg) - 1)) && r.in(i)) {
            if (g) g[r.row(i)] = dg[i];
            if (b) b[r.row(i)] = db[i];
        }
    }
}

// A work-group takes the tiles slab, slab + slabs, ... of a chunk of a group.  WHOLE: the chunk is the group, and dX is written; otherwise the
// sums of h and h xh go to the workspace, (groups, chunks, 2, batch).
template <int K, int T, bool WHOLE>
__global__ __launch_bounds__(T) void norm_backward_kernel(const NormArgs a, const Shape z, float *slabs)
{
    extern __shared__ float4 lds[];   // two per wave and quad
    const int64_t unit = blockIdx.x / z.slabs;
    const int slab = static_cast<int>(near_tile(blockIdx.x % z.slabs, z.slabs, z.lg)), chunk = static_cast<int>(unit % z.chunks), group = static_cast<int>(unit / z.chunks);
    float dg[2 * K], db[2 * K];
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) dg[i] = db[i] = 0.f;
    Rows<K> r = rows_of<K>(a, group, chunk, spot_in(slab, z.lg, a.batch));
    Affine<K> w;
    w.load(a, r);
    for (int64_t tile = slab; tile < z.tiles; tile += z.slabs) {
        const Spot p = spot_in(tile, z.lg, a.batch, z.past);
        // (rows' addresses in three operands, kept from one tile to the next, would take more registers than the entries)
        asm volatile("" : "+v"(r.pair));
        float4 x[2 * K], g[2 * K], s, sx;
        r.load_singly(a.X, a.ldx, p, x);
        r.load_singly(a.dY, a.lddy, p, g);
        const float4 mean = load_singly(a.mean + group * a.lds, p), rstd = load_singly(a.rstd + group * a.lds, p);
        form_h<K>(a, x, g, r, w, p, mean, rstd, dg, db);
        column_sums_of_h<K>(x, g, r, z.lg, lds, s, sx);
        if constexpr (WHOLE) {
            write_backward<K>(a, x, g, r, p, rstd, s, sx);
        } else if (p.slot == 0) {
            float *const at = a.workspace + 2 * (static_cast<int64_t>(group) * z.chunks + chunk) * a.batch;
            store_quad(at, p, s);
            store_quad(at + a.batch, p, sx);
        }
        __syncthreads();   // (the sums of the next tile go to the same memory)
    }
    write_rows<K>(a, slabs, z.slabs, slab, r, z.lg, dg, db);
}

template <int K>
__global__ __launch_bounds__(kChunkThreads) void norm_apply_backward_kernel(const NormArgs a, const Shape z)
{
    extern __shared__ float4 lds[];   // two per wave and quad
    const int64_t unit = blockIdx.x / z.chunks, tile = near_tile(unit % z.tiles, z.tiles, z.lg);
    const int chunk = static_cast<int>(blockIdx.x % z.chunks), group = static_cast<int>(unit / z.tiles);
    const Spot p = spot_in(tile, z.lg, a.batch, z.past);
    const Rows<K> r = rows_of<K>(a, group, chunk, p);
    float4 x[2 * K], g[2 * K];
    r.load_singly(a.X, a.ldx, p, x);
    r.load_singly(a.dY, a.lddy, p, g);
    const float4 mean = load_singly(a.mean + group * a.lds, p), rstd = load_singly(a.rstd + group * a.lds, p);
    Affine<K> w;
    w.load(a, r);
    float dg[2 * K] = {}, db[2 * K] = {};   // (left to the first launch)
    form_h<K>(a, x, g, r, w, p, mean, rstd, dg, db);
    float4 s, sx;
    join_sums(a, z, group, p, lds, s, sx);
    write_backward<K>(a, x, g, r, p, rstd, s, sx);
}

// The slabs' sums: 64 features a work-group, 16 waves that take every 16th slab, four at a time.
constexpr int kSlabWaves = 16, kSlabLoads = 4;
__global__ __launch_bounds__(kSlabWaves *kWave) void norm_slabs_kernel(const float *slabs, int n_slabs, int features, float *dgamma, float *dbeta)
{
    __shared__ float lds[2][kSlabWaves][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    const int64_t f = static_cast<int64_t>(blockIdx.x) * kWave + lane;
    const float *const at = slabs + min(f, static_cast<int64_t>(features) - 1);
    float g = 0.f, b = 0.f;
    for (int s = wave; s < n_slabs; s += kSlabLoads * kSlabWaves) {
        float x[2][kSlabLoads];
#pragma unroll
        for (int u = 0; u < kSlabLoads; ++u) {
            const int64_t slab = 2 * static_cast<int64_t>(min(s + u * kSlabWaves, n_slabs - 1));
            x[0][u] = at[slab * features];
            x[1][u] = at[(slab + 1) * features];
        }
#pragma unroll
        for (int u = 0; u < kSlabLoads; ++u)
            if (s + u * kSlabWaves < n_slabs) {
                g += x[0][u];
                b += x[1][u];
            }
    }
    lds[0][wave][lane] = g;
    lds[1][wave][lane] = b;
    __syncthreads();
    if (wave > 0 || f >= features) return;
    for (int w = 1; w < kSlabWaves; ++w) {
        g += lds[0][w][lane];
        b += lds[1][w][lane];
    }
    if (dgamma) dgamma[f] = g;
    if (dbeta) dbeta[f] = b;
}

// ---- dropout by itself ----
constexpr int kDropThreads = 256;
constexpr int kDropPairs = 2;          // pairs of rows per thread
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(const DropoutArgs a, const int lg, const int64_t tiles, const bool past)
{
    const Spot p = spot_in(blockIdx.x % tiles, lg, a.batch, past);
    const int64_t pair0 = static_cast<int64_t>(blockIdx.x / tiles) * (kDropPairs * p.slots) + p.slot;
    if (p.n == 0) return;
    float4 x[2 * kDropPairs];
    // (of rows beyond the last some row is read)
    load_quads([&](int i) { return a.X + min(2 * (pair0 + (i >> 1) * p.slots) + (i & 1), static_cast<int64_t>(a.features) - 1) * a.ldx; }, p, x);
    Drawn d{};
    if (a.drop.cut) d = drawn_from(a.drop);
#pragma unroll
    for (int k = 0; k < kDropPairs; ++k) {
        const int64_t pair = pair0 + k * p.slots;
        Bits bits{};
        if (a.drop.cut) bits = bits_of(d, p.col, static_cast<int>(pair));
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (2 * pair + h < a.features) store_quad(a.Y + (2 * pair + h) * a.ldy, p, a.drop.cut ? drop(x[2 * k + h], bits, h, a.drop) : x[2 * k + h]);
    }
}

// ---- launches ----
struct Plan {
    Shape z;
    int threads, pairs;      // pairs: K
    int lds;                 // bytes
};
constexpr int64_t kFewGroups = 256;      // work-groups: one per compute unit
// Chunks that all work-groups of the second launch would add up together, beyond which a launch of its own does it before them (300000 rows x 300 columns,
// both ways: 1878 -> 737 us; 40000 x 300: 125 -> 112; but 100000 x 32, with 0.6 M of them: 50 -> 57).
constexpr int64_t kManyChunks = 3 << 18;
struct Limits {
    int most_pairs, most_threads;   // the most that a thread and a work-group hold of a group
    int chunk_pairs;                // of a thread at most, where the group is longer
    int bytes;                      // that an entry moves
    bool slabs;                     // tiles leave sums to be added up
};
constexpr Limits kForward{8, 1024, 4, 8, false}, kBackward{8, 512, 2, 12, true};
// Threads of a work-group, before a thread takes kGroupPairs pairs.  More of them where there are few work-groups: a compute unit has one, whose threads
// each have less to do in turn (both ways, 256 -> 512 threads: 1532 rows, 2 groups x 12 columns 20.1 -> 17.0 us, 2048 rows, 1 x 553 36.2 -> 32.2; 1024
// threads take 17.2 and 34.1).
constexpr int kGroupThreads = 256, kFewThreads = 512, kGroupPairs = 4;
Plan plan_norm(int32_t features, int32_t groups, int32_t batch, const Limits &l)
{
    Plan p{};
    const int64_t pairs = (static_cast<int64_t>(features / groups) + 1) / 2;
    const auto tiles = [&](int lg) { return (batch + (INT64_C(4) << lg) - 1) >> (lg + 2); };
    const int wide = lanes_for(batch, kLanes), widest = lanes_for(batch, 6);
    p.z.lg = wide;
    p.z.past = static_cast<int64_t>(features) * batch > kCacheBytes / l.bytes;
    // Wider tiles for groups that leave lanes idle (groups of 8 rows, 64 groups x 4096 columns, both ways: 23.3 -> 16.1 us).  Narrower ones where there would
    // be few work-groups, each with much to do (512 rows, 2 groups x 100 columns: 23.8 -> 13.6; 1024 rows, 1 x 1024: 30.6 -> 20.8).
    while (p.z.lg < widest && pairs << p.z.lg < kWave) ++p.z.lg;
    while (p.z.lg > 0 && groups * tiles(p.z.lg) < kFewGroups && pairs << p.z.lg > kWave) --p.z.lg;
    // One tile for all columns, where 256 threads hold it, leaves no slabs to add up (32 rows, 32 groups x 32 columns, both ways: 12.1 -> 8.7 us; with 512
    // threads 32 x 32 rows x 100 columns take 12.7 instead of 11.9).
    if (l.slabs && tiles(widest) == 1 && pairs << widest <= kGroupThreads) p.z.lg = widest;
    const bool few = groups * tiles(p.z.lg) < kFewGroups;
    p.z.tiles = tiles(p.z.lg);
    const int64_t held = pairs << p.z.lg;   // threads, of one pair each
    p.pairs = 1;
    while (p.pairs < kGroupPairs && held > (few ? kFewThreads : kGroupThreads) * p.pairs) p.pairs *= 2;
    while (p.pairs < l.most_pairs && held > l.most_threads * p.pairs) p.pairs *= 2;
    int64_t threads = (held + p.pairs - 1) / p.pairs;
    threads = (threads + kWave - 1) / kWave * kWave;
    p.z.chunks = 1;
    // In chunks what a work-group does not hold, and what few work-groups would take longer for than two launches do (8192 rows, 1 group x 32 columns,
    // both ways: 55.7 -> 22.5 us; 8192 rows, one column: 26.2 -> 11.2).  Held whole, 8 x 1024 rows x 8192 columns take 333 us, in chunks 446.
    if (threads > l.most_threads || (few && held > kThreadsMost)) {
        p.z.lg = wide;
        p.z.tiles = tiles(wide);
        threads = kChunkThreads;
        for (p.pairs = l.chunk_pairs;; p.pairs /= 2) {
            const int64_t of_chunk = static_cast<int64_t>(p.pairs) * (threads >> p.z.lg);
            p.z.chunks = static_cast<int>((pairs + of_chunk - 1) / of_chunk);
            if (p.pairs == 1 || groups * p.z.tiles * p.z.chunks >= 2 * kFewGroups) break;
        }
    }
    p.threads = static_cast<int>(threads);
    p.lds = 2 * static_cast<int>(sizeof(float4)) * (p.threads / kWave << p.z.lg);
    p.z.slabs = 1;
    return p;
}
constexpr int64_t kBackwardThreads = 2048 * 256;

Plan plan_forward(int32_t features, int32_t groups, int32_t batch) { return plan_norm(features, groups, batch, kForward); }
// Work-groups of the backward pass take tile after tile, and their sums for gamma and beta are a slab each: as many as the GPU holds about twice.
Plan plan_backward(int32_t features, int32_t groups, int32_t batch)
{
    Plan p = plan_norm(features, groups, batch, kBackward);
    const int64_t rows = static_cast<int64_t>(groups) * p.z.chunks;
    p.z.slabs = static_cast<int>(std::max<int64_t>(1, std::min(p.z.tiles, kBackwardThreads / p.threads / rows)));
    return p;
}
int64_t chunk_floats(const Plan &p, int32_t groups, int32_t batch) { return p.z.chunks > 1 ? 2 * static_cast<int64_t>(groups) * p.z.chunks * batch : 0; }

}  // namespace

int64_t norm_scratch_floats(int32_t features, int32_t groups, int32_t batch)
{
    const Plan f = plan_forward(features, groups, batch), b = plan_backward(features, groups, batch);
    const int64_t slabs = b.z.slabs > 1 ? 2 * static_cast<int64_t>(b.z.slabs) * features : 0;
    return std::max(chunk_floats(f, groups, batch), chunk_floats(b, groups, batch) + slabs);
}

template <int K>
using Pairs = std::integral_constant<int, K>;
// f of the pairs that a thread holds, `Most` at most
template <int Most, typename F>
void with_pairs(int pairs, F &&f)
{
    if constexpr (Most > 1)
        if (pairs < Most) return with_pairs<Most / 2>(pairs, f);
    f(Pairs<Most>());
}
// threads that the kernels of K pairs are compiled for
constexpr int most_threads(int pairs, const Limits &l) { return pairs < kGroupPairs ? kFewThreads : l.most_threads; }

hipError_t launch_norm_forward(const NormArgs &a, hipStream_t s)
{
    Plan p = plan_forward(a.features, a.groups, a.batch);
    const int64_t blocks = p.z.tiles * a.groups * p.z.chunks;
    if (!fits_launch(blocks, p.threads)) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<uint32_t>(blocks)), threads(p.threads), joins(static_cast<uint32_t>(p.z.tiles * a.groups));
    if (p.z.chunks == 1) {
        with_pairs<kForward.most_pairs>(p.pairs, [&](auto k) { norm_forward_kernel<k, most_threads(k, kForward), true><<<grid, threads, p.lds, s>>>(a, p.z); });
    } else {
        with_pairs<kForward.chunk_pairs>(p.pairs, [&](auto k) {
            norm_forward_kernel<k, kChunkThreads, false><<<grid, threads, p.lds, s>>>(a, p.z);
            if (blocks * p.z.chunks > kManyChunks) {
                norm_join_kernel<k, false><<<joins, threads, p.lds, s>>>(a, p.z);
                p.z.joined = true;
            }
            norm_apply_kernel<k><<<grid, threads, p.lds, s>>>(a, p.z);
        });
    }
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormArgs &a, hipStream_t s)
{
    Plan p = plan_backward(a.features, a.groups, a.batch);
    const int64_t rows = static_cast<int64_t>(a.groups) * p.z.chunks, blocks = rows * p.z.slabs;
    if (!fits_launch(blocks, p.threads) || (p.z.chunks > 1 && !fits_launch(rows * p.z.tiles, p.threads))) return hipErrorInvalidConfiguration;
    float *const slabs = a.workspace + chunk_floats(p, a.groups, a.batch);
    const dim3 grid(static_cast<uint32_t>(blocks)), threads(p.threads), joins(static_cast<uint32_t>(p.z.tiles * a.groups));
    if (p.z.chunks == 1) {
        with_pairs<kBackward.most_pairs>(p.pairs, [&](auto k) { norm_backward_kernel<k, most_threads(k, kBackward), true><<<grid, threads, p.lds, s>>>(a, p.z, slabs); });
    } else {
        const dim3 every(static_cast<uint32_t>(rows * p.z.tiles));
        with_pairs<kBackward.chunk_pairs>(p.pairs, [&](auto k) {
            norm_backward_kernel<k, kChunkThreads, false><<<grid, threads, p.lds, s>>>(a, p.z, slabs);
            if (rows * p.z.tiles * p.z.chunks > kManyChunks) {
                norm_join_kernel<1, true><<<joins, threads, p.lds, s>>>(a, p.z);
                p.z.joined = true;
            }
            norm_apply_backward_kernel<k><<<every, threads, p.lds, s>>>(a, p.z);
        });
    }
    if (p.z.slabs > 1 && (a.dgamma || a.dbeta))
        norm_slabs_kernel<<<(a.features + kWave - 1) / kWave, kSlabWaves * kWave, 0, s>>>(slabs, p.z.slabs, a.features, a.dgamma, a.dbeta);
    return hipGetLastError();
}

hipError_t launch_dropout(const DropoutArgs &a, hipStream_t s)
{
    const int lg = lanes_for(a.batch, 6);
    const int64_t tiles = (a.batch + (INT64_C(4) << lg) - 1) >> (lg + 2);
    const int64_t of_block = static_cast<int64_t>(kDropPairs) * (kDropThreads >> lg), pairs = (static_cast<int64_t>(a.features) + 1) / 2;
    const int64_t blocks = tiles * ((pairs + of_block - 1) / of_block);
    if (!fits_launch(blocks, kDropThreads)) return hipErrorInvalidConfiguration;
    dropout_kernel<<<static_cast<uint32_t>(blocks), kDropThreads, 0, s>>>(a, lg, tiles, 8 * static_cast<int64_t>(a.features) * a.batch > kCacheBytes);
    return hipGetLastError();
}

}  // namespace nerva
