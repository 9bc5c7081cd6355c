// Device helpers of kernels whose work-groups own a tile of columns: the lanes that lie side by side hold four columns each, threads with the
// same columns differ in their rows (norm.hip, loss.hip).
#pragma once
#include <type_traits>

#include "device.h"

namespace nerva {
namespace {

// log2 of the lanes that a tile of columns takes: as many quads as the batch has, up to `most`
inline int lanes_for(int32_t batch, int most)
{
    int lg = 0;
    while (lg < most && (INT64_C(4) << lg) < batch) ++lg;
    return lg;
}

// Operands that together take more than half of the 256 MiB of memory-side cache: what is written would push out what is still to be read (norm of
// 3000 x 8192, forward: 53 -> 41 us, both ways 138 -> 135; policy loss of 3000 classes x 8192: 67 -> 60; 8192 x 8192, both ways: 314 -> 292).  Smaller ones stay
// in the cache for whoever reads them next (8190 x 777 past the cache, both ways: 76 instead of 64).
constexpr int64_t kCacheBytes = INT64_C(128) << 20;

// Where a thread stands: its four columns, of which n exist.
struct Spot {
    int q, slot, slots;      // quad in the tile; place among the threads of that quad
    int col, n, batch;
    bool whole;              // all columns of the tile exist (the same for all threads)
    bool past;               // results are written past the caches (the same for all threads)
};
__device__ __forceinline__ Spot spot_in(int64_t tile, int lg, int batch, bool past = false)
{
    Spot p;
    p.q = threadIdx.x & ((1 << lg) - 1);
    p.slot = threadIdx.x >> lg;
    p.slots = blockDim.x >> lg;
    const int64_t first = tile << (lg + 2);
    p.whole = first + (4 << lg) <= batch;
    p.col = static_cast<int>(first) + 4 * p.q;
    p.n = min(4, max(0, batch - p.col));
    p.batch = batch;
    p.past = past;
    return p;
}

// Tile of work-group b of n: those that share 128-byte lines (tiles of less than 32 columns) come to the same XCD, to which ids go in turn, so that its L2
// serves a line to all of them.
__device__ __forceinline__ int64_t near_tile(int64_t b, int64_t n, int lg)
{
    const int shift = 3 - lg;
    if (shift <= 0) return b;
    const int64_t set = b >> (3 + shift);
    if ((set + 1) << (3 + shift) > n) return b;
    const int in_set = static_cast<int>(b) & ((8 << shift) - 1);
    return (set << (3 + shift)) + ((in_set & 7) << shift) + (in_set >> 3);
}

// Four columns of a row, for loops that are compiled for each kind of tile.  An output may lie where the input does and nothing beyond the batch is touched: in a tile that is not
// whole the lane with the batch's last columns reads its last four, of which `own_of` keeps the lane's own once all reads of a loop are under way (in place of columns that do not exist:
// the batch's last one), and writes its own one by one.  A batch of one to three columns takes no more reads than columns.  (Read one by one by
// all lanes of such a tile, the preference loss of 5000 classes x 1000 takes 30.6 us instead of 26.4.)
enum TileKind { kWhole, kPart, kFewColumns };
template <TileKind T>
__device__ __forceinline__ float4 load_of(const float *row, const Spot &p)
{
    if constexpr (T == kWhole) return ld4(row + p.col);
    if constexpr (T == kPart) return ld4(row + min(p.col, p.batch - 4));
    float4 x = make_float4(row[min(p.col, p.batch - 1)], 0.f, 0.f, 0.f);
    if (p.batch > 1) x.y = row[min(p.col + 1, p.batch - 1)];
    if (p.batch > 2) x.z = row[min(p.col + 2, p.batch - 1)];
    return x;
}
template <TileKind T>
__device__ __forceinline__ float4 own_of(float4 x, const Spot &p)
{
    if constexpr (T != kPart) return x;
    const int shift = p.col - min(p.col, p.batch - 4);
    return make_float4(shift == 0 ? x.x : shift == 1 ? x.y : shift == 2 ? x.z : x.w, shift == 0 ? x.y : shift == 1 ? x.z : x.w, shift == 0 ? x.z : x.w, x.w);
}
// f of the tile's kind
template <typename F>
__device__ __forceinline__ void with_kind(const Spot &p, F &&f)
{
    if (p.whole) f(std::integral_constant<TileKind, kWhole>());
    else if (p.batch >= 4) f(std::integral_constant<TileKind, kPart>());
    else f(std::integral_constant<TileKind, kFewColumns>());
}
// (PAST: chosen before the loop as well; of two stores to one place, one of them past the caches, the compiler makes an ordinary one)
template <TileKind T, bool PAST>
__device__ __forceinline__ void store_of(float *row, const Spot &p, float4 x)
{
    if (T == kWhole || p.n == 4) {
        const v4f_any r = {x.x, x.y, x.z, x.w};
        if constexpr (PAST) __builtin_nontemporal_store(r, reinterpret_cast<v4f_any *>(row + p.col));
        else *reinterpret_cast<v4f_any *>(row + p.col) = r;
        return;
    }
    if (p.n > 0) row[p.col] = x.x;
    if (p.n > 1) row[p.col + 1] = x.y;
    if (p.n > 2) row[p.col + 2] = x.z;
}
// The quads of N rows, row(i), in one loop for whole tiles and others, which takes less code and time than one for each kind (dropout of two operands, 1024 x 100: 5.7 us instead
// of 6.1, 8191 x 9001: 242 instead of 251; with single reads in tiles that are not whole 6.6 and 248, 4096 x 1001 20.5 instead of 13.5, norm of 8190 rows x 777 forward
// 21.5 instead of 20.5).
template <int N, typename F>
__device__ __forceinline__ void load_quads(F &&row, const Spot &p, float4 (&x)[N])
{
    if (p.batch >= 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = load_of<kPart>(row(i), p);
        if (p.whole || !(p.batch & 3)) return;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = own_of<kPart>(x[i], p);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = load_of<kFewColumns>(row(i), p);
    }
}
__device__ __forceinline__ float4 load_quad(const float *row, const Spot &p)
{
    float4 x[1];
    load_quads([&](int) { return row; }, p, x);
    return x[0];
}
// A quad with single reads in a tile that is not whole: fewer registers, which norm's backward pass is short of (8192 rows in 32 groups x 8192 columns, both ways: 291 us
// instead of 296; 1024 rows in one group, whose kernel would keep 112 bytes a thread in scratch memory: 52 instead of 59).
__device__ __forceinline__ float4 load_singly(const float *row, const Spot &p)
{
    if (p.whole) return ld4(row + p.col);
    const int last = p.batch - 1;
    return make_float4(row[min(p.col, last)], row[min(p.col + 1, last)], row[min(p.col + 2, last)], row[min(p.col + 3, last)]);
}
__device__ __forceinline__ void store_quad(float *row, const Spot &p, float4 x)
{
    if (p.whole) {
        if (p.past) {
            const v4f_any r = {x.x, x.y, x.z, x.w};
            __builtin_nontemporal_store(r, reinterpret_cast<v4f_any *>(row + p.col));
        } else {
            st4(row + p.col, x);
        }
        return;
    }
    store_of<kPart, false>(row, p, x);
}
// 0 for columns that do not exist
__device__ __forceinline__ float4 existing(float4 x, const Spot &p)
{
    if (p.whole) return x;
    return make_float4(p.n > 0 ? x.x : 0.f, p.n > 1 ? x.y : 0.f, p.n > 2 ? x.z : 0.f, p.n > 3 ? x.w : 0.f);
}

__device__ __forceinline__ float4 splat(float x) { return make_float4(x, x, x, x); }
__device__ __forceinline__ float4 operator+(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ float4 operator-(float4 a, float4 b) { return make_float4(a.x - b.x, a.y - b.y, a.z - b.z, a.w - b.w); }
__device__ __forceinline__ float4 operator*(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
__device__ __forceinline__ float4 operator*(float a, float4 b) { return make_float4(a * b.x, a * b.y, a * b.z, a * b.w); }
__device__ __forceinline__ float4 fma4(float4 a, float4 b, float4 c) { return make_float4(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y), fmaf(a.z, b.z, c.z), fmaf(a.w, b.w, c.w)); }
__device__ __forceinline__ float4 shfl_xor4(float4 v, int d)
{
    return make_float4(__shfl_xor(v.x, d, kWave), __shfl_xor(v.y, d, kWave), __shfl_xor(v.z, d, kWave), __shfl_xor(v.w, d, kWave));
}
__device__ __forceinline__ float sum4(float4 v) { return (v.x + v.y) + (v.z + v.w); }

// exp(x) by one v_exp_f32: relative error 2^-24 (|x| + 2), of which the first part is the rounding of the argument.  (log2(e) in two parts, the smaller one first:
// rounded to one, it makes all results too large by 1.3e-8 |x|, which a sum over many columns shows.)
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(fmaf(x, 1.44269504f, x * 1.92596299e-8f)); }

}  // namespace
}  // namespace nerva
