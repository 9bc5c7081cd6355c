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

#include "columns.h"
#include "experts.h"
#include "norm.h"

namespace nerva {
namespace {

constexpr int kLanes = 3;              // log2 of the quads of a tile: 32 columns, whose rows are 128-byte lines
constexpr int kThreadsMost = 1024;

// ---- the generator ----
// Philox4x32 of 10 rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011), key = seed.  Counter (column / 4, row / 2,
// layer, step) gives the bits of four columns in two rows: word column % 4, its low half for the even row and its high half for the odd one.  So
// an entry's bits depend on neither leading dimension nor batch nor launch.  16 bits an entry halve the generator's work, which
// beside 8 bytes an entry is not small (some 130 cycles of a wave for 256 draws of 32 bits); the probability is a multiple of 2^-16
// for it, and the scale is that of the multiple.
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
__device__ __forceinline__ float sigmoid_of(float u) { return 1.f / (1.f + exp_of(-u)); }
__device__ __forceinline__ float activate(float u, int act)
{
    if (act == kRelu) return u < 0.f ? 0.f : u;
    if (act == kSilu) return u * sigmoid_of(u);
    return u;
}
// e act'(u)
__device__ __forceinline__ float activate_back(float e, float u, int act)
{
    if (act == kRelu) return u > 0.f ? e : 0.f;
    if (act == kSilu) {
        const float s = sigmoid_of(u);
        return e * (s * fmaf(u, 1.f - s, 1.f));
    }
    return e;
}
__device__ __forceinline__ float4 activate4(float4 u, int act) { return make_float4(activate(u.x, act), activate(u.y, act), activate(u.z, act), activate(u.w, act)); }
__device__ __forceinline__ float4 activate_back4(float4 e, float4 u, int act)
{
    return make_float4(activate_back(e.x, u.x, act), activate_back(e.y, u.y, act), activate_back(e.z, u.z, act), activate_back(e.w, u.w, act));
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
        if (p.whole) {
#pragma unroll
            for (int i = 0; i < 2 * K; ++i) x[i] = ld4(X + readable(i) * ld + p.col);
        } else {
#pragma unroll
            for (int i = 0; i < 2 * K; ++i) x[i] = load_quad(X + readable(i) * ld, p);
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
    int64_t tiles;
};

// statistics of the entries that the work-group holds: mean and sum of squares about it
template <int K>
__device__ __forceinline__ void statistics(const float4 (&x)[2 * K], const Rows<K> &r, int lg, float4 (*lds)[kThreadsMost / kWave << kLanes], float4 &mean, float4 &squares)
{
    const int n = r.end - r.first;
    float4 s = splat(0.f);
#pragma unroll
    for (int i = 0; i < 2 * K; ++i)
        if (r.in(i)) s = s + x[i];
    mean = 1.f / static_cast<float>(n) * column_sum(s, lg, lds[0]);
    float4 s2 = splat(0.f);
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        const float4 d = x[i] - mean;
        if (r.in(i)) s2 = fma4(d, d, s2);
    }
    squares = column_sum(s2, lg, lds[1]);
}
__device__ __forceinline__ float4 rstd_of(float4 squares, int m, float eps)
{
    const float4 v = 1.f / static_cast<float>(m) * squares + splat(eps);
    return make_float4(1.f / sqrtf(v.x), 1.f / sqrtf(v.y), 1.f / sqrtf(v.z), 1.f / sqrtf(v.w));
}

template <int K>
__device__ __forceinline__ void write_forward(const NormArgs &a, const float4 (&x)[2 * K], const Rows<K> &r, const Spot &p, float4 mean, float4 rstd)
{
    Drawn d{};
    if (a.drop.cut) d = drawn_from(a.drop);
    Bits bits{};
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        const int f = r.row(i);
        if (a.drop.cut && !(i & 1)) bits = bits_of(d, p.col, f >> 1);
        if (!r.in(i)) continue;
        const float4 xh = (x[i] - mean) * rstd;
        float4 y = activate4(fma4(splat(a.gamma ? a.gamma[f] : 1.f), xh, splat(a.beta ? a.beta[f] : 0.f)), a.act);
        if (a.drop.cut) y = drop(y, bits, i & 1, a.drop);
        store_quad(a.Y + f * a.ldy, p, y);
    }
}

// One work-group: a chunk of a group in a tile of columns.  WHOLE: the chunk is the group.  Otherwise its statistics go to the workspace,
// {mean, sum of squares about it} (groups, chunks, batch).
template <int K, bool WHOLE>
__global__ __launch_bounds__(kThreadsMost) void norm_forward_kernel(const NormArgs a, const Shape z)
{
    __shared__ float4 lds[2][kThreadsMost / kWave << kLanes];
    const int64_t unit = blockIdx.x / z.chunks, tile = unit % z.tiles;
    const int chunk = static_cast<int>(blockIdx.x % z.chunks), group = static_cast<int>(unit / z.tiles);
    const Spot p = spot_in(tile, z.lg, a.batch);
    const Rows<K> r = rows_of<K>(a, group, chunk, p);
    float4 x[2 * K], mean, squares;
    r.load(a.X, a.ldx, p, x);
    statistics<K>(x, r, z.lg, lds, mean, squares);
    if constexpr (WHOLE) {
        const float4 rstd = rstd_of(squares, r.end - r.first, a.eps);
        if (p.slot == 0) {
            if (a.mean) store_quad(a.mean + group * a.lds, p, mean);
            if (a.rstd) store_quad(a.rstd + group * a.lds, p, rstd);
        }
        write_forward<K>(a, x, r, p, mean, rstd);
    } else if (p.slot == 0) {
        float *const at = a.workspace + 2 * (static_cast<int64_t>(group) * z.chunks + chunk) * a.batch;
        store_quad(at, p, mean);
        store_quad(at + a.batch, p, squares);
    }
}

// the second launch of a group of several chunks
template <int K>
__global__ __launch_bounds__(kThreadsMost) void norm_apply_kernel(const NormArgs a, const Shape z)
{
    const int64_t unit = blockIdx.x / z.chunks, tile = unit % z.tiles;
    const int chunk = static_cast<int>(blockIdx.x % z.chunks), group = static_cast<int>(unit / z.tiles);
    const Spot p = spot_in(tile, z.lg, a.batch);
    const Rows<K> r = rows_of<K>(a, group, chunk, p);
    float4 x[2 * K];
    r.load(a.X, a.ldx, p, x);
    // the chunks' means weighed by their rows, then all squares about the mean of the group (Chan, Golub, LeVeque 1979)
    const int m = a.features / a.groups;
    const float *const stats = a.workspace + 2 * static_cast<int64_t>(group) * z.chunks * a.batch;
    float4 mean = splat(0.f), squares = splat(0.f);
    for (int c = 0; c < z.chunks; ++c) {
        const Rows<K> of = rows_of<K>(a, group, c, p);
        mean = fma4(splat(static_cast<float>(of.end - of.first)), load_quad(stats + 2 * static_cast<int64_t>(c) * a.batch, p), mean);
    }
    mean = 1.f / static_cast<float>(m) * mean;
    for (int c = 0; c < z.chunks; ++c) {
        const Rows<K> of = rows_of<K>(a, group, c, p);
        const float *const at = stats + 2 * static_cast<int64_t>(c) * a.batch;
        const float4 d = load_quad(at, p) - mean;
        squares = squares + fma4(static_cast<float>(of.end - of.first) * d, d, load_quad(at + a.batch, p));
    }
    const float4 rstd = rstd_of(squares, m, a.eps);
    if (p.slot == 0 && chunk == 0) {
        if (a.mean) store_quad(a.mean + group * a.lds, p, mean);
        if (a.rstd) store_quad(a.rstd + group * a.lds, p, rstd);
    }
    write_forward<K>(a, x, r, p, mean, rstd);
}

// ---- backward ----
// x becomes xh, g becomes h; what the rows add to the gradients of gamma and beta from this thread's columns is added to `dg` and `db`
template <int K>
__device__ __forceinline__ void form_h(const NormArgs &a, float4 (&x)[2 * K], float4 (&g)[2 * K], const Rows<K> &r, const Spot &p, float4 mean, float4 rstd,
                                       float (&dg)[2 * K], float (&db)[2 * K])
{
    Drawn d{};
    if (a.drop.cut) d = drawn_from(a.drop);
    Bits bits{};
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        const int f = r.readable(i);
        if (a.drop.cut && !(i & 1)) bits = bits_of(d, p.col, r.row(i) >> 1);
        x[i] = (x[i] - mean) * rstd;
        const float gamma = a.gamma ? a.gamma[f] : 1.f;
        float4 e = g[i];
        if (a.drop.cut) e = drop(e, bits, i & 1, a.drop);
        if (a.act) e = activate_back4(e, fma4(splat(gamma), x[i], splat(a.beta ? a.beta[f] : 0.f)), a.act);
        if (!r.in(i)) e = splat(0.f);
        const float4 ex = e * x[i];
        // (columns that do not exist hold zeros in e)
        dg[i] += r.in(i) ? sum4(ex) : 0.f;
        db[i] += sum4(e);
        g[i] = gamma * e;
    }
}
template <int K>
__device__ __forceinline__ void column_sums_of_h(const float4 (&x)[2 * K], const float4 (&g)[2 * K], const Rows<K> &r, int lg, float4 (*lds)[kThreadsMost / kWave << kLanes],
                                                 float4 &s, float4 &sx)
{
    float4 t = splat(0.f), tx = splat(0.f);
#pragma unroll
    for (int i = 0; i < 2 * K; ++i)
        if (r.in(i)) {
            t = t + g[i];
            tx = fma4(g[i], x[i], tx);
        }
    s = column_sum(t, lg, lds[0]);
    sx = column_sum(tx, lg, lds[1]);
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
__device__ __forceinline__ void write_rows(const NormArgs &a, float *slabs, int n_slabs, int slab, const Rows<K> &r, const Spot &p, int lg, float (&dg)[2 * K], float (&db)[2 * K])
{
    if (!a.dgamma && !a.dbeta) return;
    float *const g = n_slabs == 1 ? a.dgamma : slabs + 2 * static_cast<int64_t>(slab) * a.features;
    float *const b = n_slabs == 1 ? a.dbeta : slabs + (2 * static_cast<int64_t>(slab) + 1) * a.features;
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) {
        for (int d = 1; d < 1 << lg; d <<= 1) {
            dg[i] += __shfl_xor(dg[i], d, kWave);
            db[i] += __shfl_xor(db[i], d, kWave);
        }
        if (p.q == 0 && r.in(i)) {
            if (g) g[r.row(i)] = dg[i];
            if (b) b[r.row(i)] = db[i];
        }
    }
}

// A work-group takes the tiles slab, slab + slabs, ... of a chunk of a group.  WHOLE: the chunk is the group, and dX is written; otherwise the
// sums of h and h xh go to the workspace, (groups, chunks, 2, batch).
template <int K, bool WHOLE>
__global__ __launch_bounds__(kThreadsMost) void norm_backward_kernel(const NormArgs a, const Shape z, float *slabs)
{
    __shared__ float4 lds[2][kThreadsMost / kWave << kLanes];
    const int64_t unit = blockIdx.x / z.slabs;
    const int slab = static_cast<int>(blockIdx.x % z.slabs), chunk = static_cast<int>(unit % z.chunks), group = static_cast<int>(unit / z.chunks);
    float dg[2 * K], db[2 * K];
#pragma unroll
    for (int i = 0; i < 2 * K; ++i) dg[i] = db[i] = 0.f;
    for (int64_t tile = slab; tile < z.tiles; tile += z.slabs) {
        const Spot p = spot_in(tile, z.lg, a.batch);
        const Rows<K> r = rows_of<K>(a, group, chunk, p);
        float4 x[2 * K], g[2 * K], s, sx;
        r.load(a.X, a.ldx, p, x);
        r.load(a.dY, a.lddy, p, g);
        const float4 mean = load_quad(a.mean + group * a.lds, p), rstd = load_quad(a.rstd + group * a.lds, p);
        form_h<K>(a, x, g, r, p, mean, rstd, dg, db);
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
    const Spot p = spot_in(0, z.lg, a.batch);
    write_rows<K>(a, slabs, z.slabs, slab, rows_of<K>(a, group, chunk, p), p, z.lg, dg, db);
}

template <int K>
__global__ __launch_bounds__(kThreadsMost) void norm_apply_backward_kernel(const NormArgs a, const Shape z)
{
    const int64_t unit = blockIdx.x / z.chunks, tile = unit % z.tiles;
    const int chunk = static_cast<int>(blockIdx.x % z.chunks), group = static_cast<int>(unit / z.tiles);
    const Spot p = spot_in(tile, z.lg, a.batch);
    const Rows<K> r = rows_of<K>(a, group, chunk, p);
    float4 x[2 * K], g[2 * K];
    r.load(a.X, a.ldx, p, x);
    r.load(a.dY, a.lddy, p, g);
    const float4 mean = load_quad(a.mean + group * a.lds, p), rstd = load_quad(a.rstd + group * a.lds, p);
    float dg[2 * K] = {}, db[2 * K] = {};   // (left to the first launch)
    form_h<K>(a, x, g, r, p, mean, rstd, dg, db);
    float4 s = splat(0.f), sx = splat(0.f);
    const float *at = a.workspace + 2 * static_cast<int64_t>(group) * z.chunks * a.batch;
    for (int c = 0; c < z.chunks; ++c, at += 2 * static_cast<int64_t>(a.batch)) {
        s = s + load_quad(at, p);
        sx = sx + load_quad(at + a.batch, p);
    }
    write_backward<K>(a, x, g, r, p, rstd, s, sx);
}

// The slabs' sums: 64 features a work-group, 16 waves that take every 16th slab.
constexpr int kSlabWaves = 16;
__global__ __launch_bounds__(kSlabWaves *kWave) void norm_slabs_kernel(const float *slabs, int n_slabs, int features, float *dgamma, float *dbeta)
{
    __shared__ float lds[2][kSlabWaves][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
    const int64_t f = static_cast<int64_t>(blockIdx.x) * kWave + lane;
    float g = 0.f, b = 0.f;
    if (f < features)
        for (int s = wave; s < n_slabs; s += kSlabWaves) {
            g += slabs[2 * static_cast<int64_t>(s) * features + f];
            b += slabs[(2 * static_cast<int64_t>(s) + 1) * features + f];
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
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(const DropoutArgs a, const int lg, const int64_t tiles)
{
    const Spot p = spot_in(blockIdx.x % tiles, lg, a.batch);
    const int64_t pair0 = static_cast<int64_t>(blockIdx.x / tiles) * (kDropPairs * p.slots) + p.slot;
    if (p.n == 0) return;
    const float *const X = a.X;
    float4 x[2 * kDropPairs];
#pragma unroll
    for (int i = 0; i < 2 * kDropPairs; ++i) {
        const int64_t f = 2 * (pair0 + (i >> 1) * p.slots) + (i & 1);
        if (f < a.features) x[i] = load_quad(X + f * a.ldx, p);
    }
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
};
// `most`: pairs that a thread holds at most
Plan plan_norm(int32_t features, int32_t groups, int32_t batch, int most)
{
    Plan p{};
    p.z.lg = lanes_for(batch, kLanes);
    p.z.tiles = (batch + (INT64_C(4) << p.z.lg) - 1) >> (p.z.lg + 2);
    const int64_t pairs = (static_cast<int64_t>(features / groups) + 1) / 2, held = pairs << p.z.lg;   // threads, of one pair each
    p.pairs = 1;
    while (p.pairs < most && held > 256 * p.pairs) p.pairs *= 2;
    int64_t threads = (held + p.pairs - 1) / p.pairs;
    threads = (threads + kWave - 1) / kWave * kWave;
    p.z.chunks = 1;
    if (threads > kThreadsMost) {
        // (chunks of a work-group of 256 threads)
        p.pairs = most;
        threads = 256;
        const int64_t of_chunk = static_cast<int64_t>(most) * (threads >> p.z.lg);
        p.z.chunks = static_cast<int>((pairs + of_chunk - 1) / of_chunk);
    }
    p.threads = static_cast<int>(threads);
    p.z.slabs = 1;
    return p;
}
constexpr int kForwardPairs = 8, kBackwardPairs = 4;
constexpr int64_t kBackwardBlocks = 2048;

Plan plan_backward(int32_t features, int32_t groups, int32_t batch)
{
    Plan p = plan_norm(features, groups, batch, kBackwardPairs);
    const int64_t rows = static_cast<int64_t>(groups) * p.z.chunks;
    p.z.slabs = static_cast<int>(std::max<int64_t>(1, std::min(p.z.tiles, kBackwardBlocks * 256 / p.threads / rows)));
    return p;
}
int64_t chunk_floats(const Plan &p, int32_t groups, int32_t batch) { return p.z.chunks > 1 ? 2 * static_cast<int64_t>(groups) * p.z.chunks * batch : 0; }

}  // namespace

int64_t norm_scratch_floats(int32_t features, int32_t groups, int32_t batch)
{
    const Plan f = plan_norm(features, groups, batch, kForwardPairs), b = plan_backward(features, groups, batch);
    const int64_t slabs = b.z.slabs > 1 ? 2 * static_cast<int64_t>(b.z.slabs) * features : 0;
    return std::max(chunk_floats(f, groups, batch), chunk_floats(b, groups, batch) + slabs);
}

#define WITH_PAIRS(k, LAUNCH)                            \
    switch (k) {                                         \
    case 1: { constexpr int K = 1; LAUNCH; break; }      \
    case 2: { constexpr int K = 2; LAUNCH; break; }      \
    case 4: { constexpr int K = 4; LAUNCH; break; }      \
    default: { constexpr int K = 8; LAUNCH; break; }     \
    }

hipError_t launch_norm_forward(const NormArgs &a, hipStream_t s)
{
    const Plan p = plan_norm(a.features, a.groups, a.batch, kForwardPairs);
    const int64_t blocks = p.z.tiles * a.groups * p.z.chunks;
    if (!fits_launch(blocks, p.threads)) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<uint32_t>(blocks)), threads(p.threads);
    if (p.z.chunks == 1) {
        WITH_PAIRS(p.pairs, (norm_forward_kernel<K, true><<<grid, threads, 0, s>>>(a, p.z)))
    } else {
        norm_forward_kernel<kForwardPairs, false><<<grid, threads, 0, s>>>(a, p.z);
        norm_apply_kernel<kForwardPairs><<<grid, threads, 0, s>>>(a, p.z);
    }
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormArgs &a, hipStream_t s)
{
    const Plan p = plan_backward(a.features, a.groups, a.batch);
    const int64_t rows = static_cast<int64_t>(a.groups) * p.z.chunks, blocks = rows * p.z.slabs;
    if (!fits_launch(blocks, p.threads) || (p.z.chunks > 1 && !fits_launch(rows * p.z.tiles, p.threads))) return hipErrorInvalidConfiguration;
    float *const slabs = a.workspace + chunk_floats(p, a.groups, a.batch);
    const dim3 grid(static_cast<uint32_t>(blocks)), threads(p.threads);
    if (p.z.chunks == 1) {
        switch (p.pairs) {
        case 1: norm_backward_kernel<1, true><<<grid, threads, 0, s>>>(a, p.z, slabs); break;
        case 2: norm_backward_kernel<2, true><<<grid, threads, 0, s>>>(a, p.z, slabs); break;
        default: norm_backward_kernel<4, true><<<grid, threads, 0, s>>>(a, p.z, slabs); break;
        }
    } else {
        norm_backward_kernel<kBackwardPairs, false><<<grid, threads, 0, s>>>(a, p.z, slabs);
        norm_apply_backward_kernel<kBackwardPairs><<<static_cast<uint32_t>(rows * p.z.tiles), threads, 0, s>>>(a, p.z);
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
    dropout_kernel<<<static_cast<uint32_t>(blocks), kDropThreads, 0, s>>>(a, lg, tiles);
    return hipGetLastError();
}

}  // namespace nerva
