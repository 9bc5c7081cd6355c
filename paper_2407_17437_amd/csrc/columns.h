// Device helpers of kernels whose work-groups own a tile of columns: the lanes that lie side by side hold four columns each, threads with the
// same columns differ in their rows (norm.hip, loss.hip).
#pragma once
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

// Where a thread stands: its four columns, of which n exist.
struct Spot {
    int q, slot, slots;      // quad in the tile; place among the threads of that quad
    int col, n;
    bool whole;              // all columns of the tile exist (the same for all threads)
};
__device__ __forceinline__ Spot spot_in(int64_t tile, int lg, int batch)
{
    Spot p;
    p.q = threadIdx.x & ((1 << lg) - 1);
    p.slot = threadIdx.x >> lg;
    p.slots = blockDim.x >> lg;
    const int64_t first = tile << (lg + 2);
    p.whole = first + (4 << lg) <= batch;
    p.col = static_cast<int>(first) + 4 * p.q;
    p.n = min(4, max(0, batch - p.col));
    return p;
}

// Four columns of a row.  Lanes that have fewer read and write one by one, so that an output may lie where the input does.
__device__ __forceinline__ float4 load_quad(const float *row, const Spot &p)
{
    if (p.whole || p.n == 4) return ld4(row + p.col);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p.n > 0) x.x = row[p.col];
    if (p.n > 1) x.y = row[p.col + 1];
    if (p.n > 2) x.z = row[p.col + 2];
    return x;
}
__device__ __forceinline__ void store_quad(float *row, const Spot &p, float4 x)
{
    if (p.whole || p.n == 4) {
        st4(row + p.col, x);
        return;
    }
    if (p.n > 0) row[p.col] = x.x;
    if (p.n > 1) row[p.col + 1] = x.y;
    if (p.n > 2) row[p.col + 2] = x.z;
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

// exp(x) with an error of about one unit in the last place: the product with log2(e) is formed in two parts, the second of which the exponential's
// own argument would lose.  (v_exp_f32 of the rounded product alone is off by 2^-24 |x| relative to the result.)
__device__ __forceinline__ float exp_of(float x)
{
    constexpr float hi = 1.44269504f, lo = 1.92596299e-8f;
    const float t = x * hi;
    const float rest = fmaf(x, lo, fmaf(x, hi, -t));
    const float e = __builtin_amdgcn_exp2f(t);
    // (an infinite x has no rest, and beside an e of 0 or infinity there is nothing to mend)
    return (e > 0.f && e < 3.0e38f) ? fmaf(e, rest * 0.693147181f, e) : e;
}

}  // namespace
}  // namespace nerva
