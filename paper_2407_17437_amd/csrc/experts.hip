// Mixtures of sparse layers: routing of columns to experts, places in the experts' blocks, and the exchange of columns
// with the blocks in both directions, forward and backward.
#include "../../include/nerva_sparse.h"
#include <type_traits>

#include "device.h"
#include "experts.h"

namespace nerva {
namespace {

constexpr float kInf = __builtin_huge_valf();

// Reductions over a wave in which lanes that a step leaves out keep what they have (dpp() of device.h gives them 0).
template <int CTRL, int ROW_MASK = 0xF>
__device__ __forceinline__ float dpp_keep(float x)
{
    const int v = __builtin_bit_cast(int, x);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(v, v, CTRL, ROW_MASK, 0xF, false));
}
template <int CTRL, int ROW_MASK = 0xF>
__device__ __forceinline__ double dpp_keep(double x)
{
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    const int lo = static_cast<int>(v), hi = static_cast<int>(v >> 32);
    const uint32_t l = __builtin_amdgcn_update_dpp(lo, lo, CTRL, ROW_MASK, 0xF, false);
    const uint32_t h = __builtin_amdgcn_update_dpp(hi, hi, CTRL, ROW_MASK, 0xF, false);
    return __builtin_bit_cast(double, static_cast<uint64_t>(h) << 32 | l);
}
__device__ __forceinline__ float read_lane(float x, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); }
__device__ __forceinline__ double read_lane(double x, int lane)
{
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), lane), hi = __builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane);
    return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}

// largest over the wave (no lane holds NaN), wave-uniform
template <typename T>
__device__ __forceinline__ T wave_max(T x)
{
    x = max(x, dpp_keep<0xB1>(x));        // quad_perm [1,0,3,2]
    x = max(x, dpp_keep<0x4E>(x));        // quad_perm [2,3,0,1]
    x = max(x, dpp_keep<0x141>(x));       // row_half_mirror
    x = max(x, dpp_keep<0x140>(x));       // row_mirror
    x = max(x, dpp_keep<0x142, 0xA>(x));  // row_bcast15 into rows 1 and 3
    x = max(x, dpp_keep<0x143, 0xC>(x));  // row_bcast31 into rows 2 and 3
    return read_lane(x, 63);
}
// sum over the wave in one fixed order
__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d, kWave);
    return x;
}
__device__ __forceinline__ float wave_sum(float x) { return group_sum<kWave>(x); }

// logarithm of the sigmoid, which does not run out of range where the sigmoid itself does
__device__ __forceinline__ float log_sigmoid(float z) { return fminf(z, 0.f) - log1pf(expf(-fabsf(z))); }

// ---- routing -----------------------------------------------------------------------------------
// Keys.  Softmax and sigmoid rise with the logit, so without a bias the logits themselves are the keys.  With a bias, or where
// a group's score is a sum, the scores are, in 64 bits: two biased scores that differ by less than 32 bits
// tell apart are common among a few hundred experts, and the choice must not depend on how a sum was rounded.
// The low 10 bits of a key's mantissa make way for the expert, so that the largest of several numbers says at once which expert is chosen and, among
// keys that agree in the other 42 bits (a logit has 23), that it is the lowest.
constexpr double kNone = -__builtin_huge_val();   // no expert
constexpr uint64_t kIndexBits = 1023;
static_assert(kExpertsMax <= static_cast<int>(kIndexBits) + 1, "experts in a key");
__device__ __forceinline__ double pack(double key, int index)
{
    if (!(key > kNone)) return kNone;             // (NaN too)
    key = fmin(key, 1.7976931348623157e308) + 0.0;   // (+inf has no mantissa to use, and -0 is 0)
    const uint64_t low = key < 0.0 ? index : kIndexBits - index;
    return __builtin_bit_cast(double, (__builtin_bit_cast(uint64_t, key) & ~kIndexBits) | low);
}
__device__ __forceinline__ int index_of(double packed)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, packed), low = b & kIndexBits;
    return static_cast<int>(b >> 63 ? low : kIndexBits - low);
}
__device__ __forceinline__ double key_of(double packed)
{
    return packed == kNone ? kNone : __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, packed) & ~kIndexBits);
}
// a group's score from its two best keys
__device__ __forceinline__ double group_score(double best, double second, bool pair, int group)
{
    return pair && second > kNone ? pack(key_of(best) + key_of(second), group) : pack(key_of(best), group);
}
// a logit that may not be chosen: NaN, or +inf where the softmax of its column is NaN (-inf is no key anyway)
__device__ __forceinline__ bool no_number(float z, bool sigmoid) { return !(z == z) || (!sigmoid && z == kInf); }

// What keys are made of: the logits, or the scores of either kind.
enum Keys { kLogits, kSigmoids, kSoftmaxes };
// Key of one expert.  top: the column's largest logit, part: 1 / the sum of exp(z - top), for softmax scores.
template <Keys kKeys>
__device__ __forceinline__ double key_from(float z, const float *bias, int e, float top, double part)
{
    if constexpr (kKeys == kLogits) return pack(z, e);   // (-inf is none)
    double q;
    if constexpr (kKeys == kSigmoids) {
        // 1 / (1 + exp(-z)), or exp(z) / (1 + exp(z)): nothing overflows.  The reciprocal from the hardware's first guess, good to 23 bits, and
        // two Newton steps.
        const double t = exp(-fabs(static_cast<double>(z))), d = 1.0 + t;
        q = __builtin_amdgcn_rcp(d);
#pragma unroll
        for (int i = 0; i < 2; ++i) q = fma(q, fma(-d, q, 1.0), q);
        if (z < 0.f) q *= t;
    } else {
        q = exp(static_cast<double>(z) - static_cast<double>(top)) * part;
    }
    if (bias) q += static_cast<double>(bias[e]);
    const double packed = pack(q, e);
    return z == -kInf ? kNone : packed;
}

// Few columns: a wave works on one column at a time, lane l holding the experts l, l + 64, ...; the k choices are k rounds of a maximum over the
// wave.  A work-group takes `cols` columns, whose logits come to LDS row by row.
// Work-groups of up to 1024 threads leave a thread 128 registers: from 513 experts on, R = 16, 27 more (logits as keys), 99 (sigmoids) or 123 (softmaxes) lie in scratch
// memory, with R = 8 none, 2 or 17.  One column and 8 choices, sigmoids: 16.5 us of 1024 experts, 8.5 of 512; 1024 columns 36.5 and 10.8.
template <int R, Keys kKeys>
__global__ __launch_bounds__(1024) void route_kernel(const RouteArgs a, const int cols)
{
    extern __shared__ __align__(16) char lds_raw[];
    const int E = a.experts, k = a.k;
    const int waves = blockDim.x / kWave, lane = threadIdx.x & (kWave - 1), wv = wave_in_block();
    const int pitch = cols + 1;                                         // (a column's logits fall on different banks)
    float *tile = reinterpret_cast<float *>(lds_raw);                   // [E][pitch]
    const int tile_floats = (E * pitch + 3) / 4 * 4;
    int32_t *out_e = reinterpret_cast<int32_t *>(tile + tile_floats);   // [cols][k]
    float *out_w = reinterpret_cast<float *>(out_e + cols * k);
    double *keys = reinterpret_cast<double *>(lds_raw + (tile_floats + 2 * cols * k + 3) / 4 * 16) + wv * E;   // [waves][E], with groups only

    const int c0 = blockIdx.x * cols, here = min(cols, a.batch - c0);
    for (int i = threadIdx.x; i < E * cols; i += blockDim.x) {
        const int e = i / cols, c = i - e * cols;
        if (c < here) tile[e * pitch + c] = a.Z[static_cast<int64_t>(e) * a.ldz + c0 + c];
    }
    __syncthreads();

    const bool sigmoid = a.flags & NERVA_EXPERT_SIGMOID, renormalise = a.flags & NERVA_EXPERT_RENORMALISE, pair = a.flags & NERVA_EXPERT_GROUP_PAIR;
    const int size = E / a.groups;
    for (int c = wv; c < here; c += waves) {
        float z[R];
        float top = -kInf;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int e = lane + i * kWave;
            z[i] = e < E ? tile[e * pitch + c] : -kInf;
            const bool off = no_number(z[i], sigmoid);
            bad |= off;
            if (off) z[i] = -kInf;
            top = fmaxf(top, z[i]);
        }
        bad = __ballot(bad) != 0;
        double total = 1.0;
        if (kKeys == kSoftmaxes || (!sigmoid && !renormalise)) {
            top = wave_max(top);
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                if constexpr (kKeys == kSoftmaxes) sum += z[i] == -kInf ? 0.0 : exp(static_cast<double>(z[i]) - static_cast<double>(top));
                else sum += z[i] == -kInf ? 0.f : expf(z[i] - top);
            }
            total = wave_sum(sum);
        }
        double key[R];
        const double part = 1.0 / total;
#pragma unroll
        for (int i = 0; i < R; ++i) key[i] = key_from<kKeys>(z[i], a.bias, min(lane + i * kWave, E - 1), top, part);

        if (a.groups > 1) {
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (lane + i * kWave < E) keys[lane + i * kWave] = key[i];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            // 2^n lanes a group, as many as there are
            int per_group = kWave;
            while (per_group * a.groups > kWave) per_group >>= 1;
            const int g = lane / per_group;
            double best = kNone, second = kNone;
            if (g < a.groups)
                for (int i = lane & (per_group - 1); i < size; i += per_group) {
                    const double q = keys[g * size + i];
                    second = fmax(second, fmin(best, q));
                    best = fmax(best, q);
                }
            for (int d = 1; d < per_group; d <<= 1) {
                const double b = __shfl_xor(best, d, kWave), q = __shfl_xor(second, d, kWave);
                second = fmax(fmin(best, b), fmax(second, q));
                best = fmax(best, b);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            double score = g < a.groups ? group_score(best, second, pair, g) : kNone;
            uint64_t open = 0;
            for (int t = 0; t < a.top_groups; ++t) {
                const double m = wave_max(score);
                if (!(m > kNone)) break;
                open |= 1ull << index_of(m);
                if (score == m) score = kNone;
            }
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (!(open >> (min(lane + i * kWave, E - 1) / size) & 1)) key[i] = kNone;
        }

        // lane j ends up with the j-th choice
        int mine = -1;
        for (int j = 0; j < k; ++j) {
            double m = key[0];
#pragma unroll
            for (int i = 1; i < R; ++i) m = fmax(m, key[i]);
            m = wave_max(m);
            if (!(m > kNone)) break;
            if (lane == j) mine = index_of(m);
#pragma unroll
            for (int i = 0; i < R; ++i) key[i] = key[i] == m ? kNone : key[i];
        }

        const float zm = mine >= 0 ? tile[mine * pitch + c] : -kInf;
        float w = 0.f;
        if (renormalise) {
            const float l = mine < 0 ? -kInf : sigmoid ? log_sigmoid(zm) : zm;
            const float high = wave_max(l);
            const float u = mine < 0 ? 0.f : expf(l - high);
            w = u / wave_sum(u);
        } else {
            w = sigmoid ? 1.f / (1.f + expf(-zm)) : expf(zm - top) / static_cast<float>(total);
        }
        w = mine >= 0 ? w * a.scale : 0.f;
        if (bad) w = __builtin_nanf("");
        if (lane < k) {
            out_e[c * k + lane] = mine;
            out_w[c * k + lane] = w;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < cols * k; i += blockDim.x) {
        const int j = i / cols, c = i - j * cols;
        if (c >= here) continue;
        a.chosen[j * a.ldk + c0 + c] = out_e[c * k + j];
        a.weights[j * a.ldk + c0 + c] = out_w[c * k + j];
    }
}

// the larger one to a
__device__ __forceinline__ void order(double &a, double &b)
{
    const double high = fmax(a, b);
    b = fmin(a, b);
    a = high;
}
// eight keys in falling order: pairs, then two sorted halves merged, twice
__device__ __forceinline__ void sort_down(double (&q)[8])
{
#pragma unroll
    for (int n = 1; n < 8; n *= 2)        // runs of n are sorted
#pragma unroll
        for (int d = n; d > 0; d /= 2)
#pragma unroll
            for (int j = d % n; j + d < 8; j += 2 * d)
#pragma unroll
                for (int i = 0; i < d; ++i)
                    if (j + i + d < 8 && (j + i) / (2 * n) == (j + i + d) / (2 * n)) order(q[j + i], q[j + i + d]);
}
// the K largest of two lists in falling order, x and y, in the same order
template <int K, typename Y>
__device__ __forceinline__ void keep_largest(double (&x)[K], Y y)
{
#pragma unroll
    for (int j = 0; j < K; ++j) x[j] = fmax(x[j], y(K - 1 - j));   // up and then down or the reverse
#pragma unroll
    for (int d = K / 2; d > 0; d /= 2)
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (!(j & d)) order(x[j], x[j + d]);
}

// Many columns: a lane owns a column, nothing crosses lanes.  The experts are cut into lists, of which a group has `parts`; a taker, which is kCols
// lanes, one for each of the work-group's columns, goes through the experts of a list and keeps its K best keys in order, in registers: two
// instructions for each key and rank, as the expert travels in the key, or, where K is as many as the keys at a time, a sort of
// those and one merge (128 instructions for eight keys -> 70; 256 experts in 8 groups, 16384 columns 20.1 us -> 19.3, 1024 experts 81.7 ->
// 79.4).  With the lists in LDS a group's score is read off their heads, lists of groups that are not taken are emptied, and pairs of
// lists are merged until one is left.
// Bound by the arithmetic on 64-bit keys, some 100 instructions each from the logit to its rank: the vector units are busy for 64 % of the 70 us of 65536
// columns of that kind in work-groups of 64, 78 % of the 65 in those of 32.  16384 columns take 19 us, where one column per wave takes 54.
constexpr int kRouteLists = 16;    // at most
template <int K, int kCols, Keys kKeys>
__global__ __launch_bounds__(kRouteLists * kCols) void route_columns_kernel(const RouteArgs a, const int lists, const int parts, const int size)
{
    static_assert((K & (K - 1)) == 0 && K >= 2, "lists are merged by halving");
    extern __shared__ double kept[];                                     // [lists][K][kCols]
    const int E = a.experts, k = a.k, takers = blockDim.x / kCols;
    const int lane = threadIdx.x & (kCols - 1), taker = kCols == kWave ? wave_in_block() : static_cast<int>(threadIdx.x / kCols);
    double *red = kept + lists * K * kCols;                              // [takers][kCols]
    float *logs = reinterpret_cast<float *>(red + takers * kCols);       // [K][kCols]
    int *bads = reinterpret_cast<int *>(logs + K * kCols);               // [takers][kCols]
    const int own = blockIdx.x * kCols + lane, c = min(own, a.batch - 1);
    const float *__restrict__ Z = a.Z + c;
    const int64_t ldz = a.ldz;
    const bool sigmoid = a.flags & NERVA_EXPERT_SIGMOID, renormalise = a.flags & NERVA_EXPERT_RENORMALISE, pair = a.flags & NERVA_EXPERT_GROUP_PAIR;
    constexpr int U = 8;   // logits in flight

    float top = -kInf;
    double total = 1.0;
    if (kKeys == kSoftmaxes || (!sigmoid && !renormalise)) {
        float z[U];
        for (int e = taker; e < E; e += U * takers) {
#pragma unroll
            for (int u = 0; u < U; ++u) z[u] = Z[min(e + u * takers, E - 1) * ldz];
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, no_number(z[u], false) ? -kInf : z[u]);
        }
        red[taker * kCols + lane] = top;
        __syncthreads();
        for (int w = 0; w < takers; ++w) top = fmaxf(top, static_cast<float>(red[w * kCols + lane]));
        __syncthreads();
        double sum = 0.0;
        for (int e = taker; e < E; e += U * takers) {
#pragma unroll
            for (int u = 0; u < U; ++u) z[u] = Z[min(e + u * takers, E - 1) * ldz];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (z[u] == -kInf || no_number(z[u], false) || e + u * takers >= E) continue;
                if constexpr (kKeys == kSoftmaxes) sum += exp(static_cast<double>(z[u]) - static_cast<double>(top));
                else sum += expf(z[u] - top);
            }
        }
        red[taker * kCols + lane] = sum;
        __syncthreads();
        total = 0.0;
        for (int w = 0; w < takers; ++w) total += red[w * kCols + lane];
    }

    const int group_size = E / a.groups;
    const double part = 1.0 / total;
    bool bad = false;
    for (int l = taker; l < lists; l += takers) {
        const int group = l / parts, start = group * group_size + (l - group * parts) * size, end = min(start + size, (group + 1) * group_size);
        double x[K];
#pragma unroll
        for (int j = 0; j < K; ++j) x[j] = kNone;
        float z[U], next[U];
        auto fetch = [&](int e0) {
            const float *p = Z + e0 * ldz;
            if (e0 + U <= end) {
#pragma unroll
                for (int u = 0; u < U; ++u, p += ldz) next[u] = *p;
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u, p += ldz) next[u] = e0 + u < end ? *p : -kInf;
            }
        };
        fetch(start);
        for (int e0 = start; e0 < end; e0 += U) {
#pragma unroll
            for (int u = 0; u < U; ++u) z[u] = next[u];
            fetch(e0 + U);
            double q[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool off = no_number(z[u], sigmoid);
                bad |= off;
                q[u] = key_from<kKeys>(off ? -kInf : z[u], a.bias, min(e0 + u, end - 1), top, part);
            }
            if constexpr (K == U) {
                sort_down(q);
                if (e0 == start) {
#pragma unroll
                    for (int j = 0; j < K; ++j) x[j] = q[j];
                } else {
                    keep_largest(x, [&](int j) { return q[j]; });
                }
                continue;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    const double high = fmax(x[j], q[u]);
                    q[u] = fmin(x[j], q[u]);
                    x[j] = high;
                }
        }
#pragma unroll
        for (int j = 0; j < K; ++j) kept[(l * K + j) * kCols + lane] = x[j];
    }
    bads[taker * kCols + lane] = bad;
    __syncthreads();

    if (a.groups > 1) {
        // scores to LDS, in the place of the sums that are done with
        for (int g = taker; g < a.groups; g += takers) {
            double best = kNone, second = kNone;
            for (int l = g * parts; l < (g + 1) * parts; ++l) {
                const double b = kept[l * K * kCols + lane], q = kept[(l * K + 1) * kCols + lane];
                second = fmax(fmin(best, b), fmax(second, q));
                best = fmax(best, b);
            }
            red[g * kCols + lane] = group_score(best, second, pair, g);
        }
        __syncthreads();
        for (int l = taker; l < lists; l += takers) {
            const double mine = red[l / parts * kCols + lane];
            int better = 0;
            for (int g = 0; g < a.groups; ++g) better += red[g * kCols + lane] > mine;
            if (better >= a.top_groups)
#pragma unroll
                for (int j = 0; j < K; ++j) kept[(l * K + j) * kCols + lane] = kNone;
        }
        __syncthreads();
    }
    for (int n = lists; n > 1;) {
        const int half = (n + 1) / 2;
        for (int l = taker; l < n - half; l += takers) {
            double *p = kept + l * K * kCols + lane, x[K];
            const double *q = p + half * K * kCols;
#pragma unroll
            for (int j = 0; j < K; ++j) x[j] = p[j * kCols];
            keep_largest(x, [&](int j) { return q[j * kCols]; });
#pragma unroll
            for (int j = 0; j < K; ++j) p[j * kCols] = x[j];
        }
        __syncthreads();
        n = half;
    }

    for (int j = taker; j < k; j += takers) {
        const double x = kept[j * kCols + lane];
        const float z = x > kNone ? Z[index_of(x) * ldz] : -kInf;
        logs[j * kCols + lane] = renormalise && sigmoid && z > -kInf ? log_sigmoid(z) : z;
    }
    __syncthreads();
    bad = false;
    for (int w = 0; w < takers; ++w) bad |= bads[w * kCols + lane];
    if (own >= a.batch) return;
    float high = -kInf, sum = 0.f;
    if (renormalise) {
        for (int j = 0; j < k; ++j) high = fmaxf(high, logs[j * kCols + lane]);
        for (int j = 0; j < k; ++j) {
            const float l = logs[j * kCols + lane];
            sum += l == -kInf ? 0.f : expf(l - high);
        }
    }
    for (int j = taker; j < k; j += takers) {
        const double x = kept[j * kCols + lane];
        const int e = x > kNone ? index_of(x) : -1;
        const float l = logs[j * kCols + lane];
        float w = renormalise ? expf(l - high) / sum : sigmoid ? 1.f / (1.f + expf(-l)) : expf(l - top) / static_cast<float>(total);
        w = e >= 0 ? w * a.scale : 0.f;
        a.chosen[j * a.ldk + own] = e;
        a.weights[j * a.ldk + own] = bad ? __builtin_nanf("") : w;
    }
}

// Gradient of the logits.  With u = weight / scale, d the gradients of the column's weights:
//     renormalised    dL_j = scale u_j (d_j - sum_i u_i d_i),  dz = dL for softmax, dL (1 - s) for sigmoid
//     softmax         dz_e = scale p_e ([e chosen] d_e - sum_i p_i d_i), over all experts
//     sigmoid         dz_e = scale s_e (1 - s_e) d_e
// A lane owns a column, the waves of a work-group share its choices and the experts, whose rows are written whole.  Where only the chosen
// experts have a gradient the zeros are under way before the choices are read, and the gradients follow one by one.
// (Over all experts with 9 to 16 choices 48 registers of a thread lie in scratch memory, in the other forms none.)
constexpr int kBackWaves = 16;   // at most
constexpr int kBackRows = 8;     // of dZ for a wave, where there may be fewer waves
template <int K, bool kFull>
__global__ __launch_bounds__(kBackWaves * kWave) void route_backward_kernel(const RouteBackwardArgs a)
{
    __shared__ float red[kFull ? 2 : 1][kBackWaves][kWave];
    __shared__ float logs[K][kWave], grads[K][kWave];   // of the scores (of the logits for a softmax), and the gradients of the weights
    __shared__ int chosen[K][kWave];
    const int lane = threadIdx.x & (kWave - 1), wv = wave_in_block(), waves = blockDim.x / kWave;
    const int own = blockIdx.x * kWave + lane, c = min(own, a.batch - 1);
    const int E = a.experts;
    const float *__restrict__ Z = a.Z + c;
    float *dZ = a.dZ + c;
    const bool on = own < a.batch, sigmoid = a.flags & NERVA_EXPERT_SIGMOID, renormalise = a.flags & NERVA_EXPERT_RENORMALISE;
    constexpr int U = 8;   // logits in flight
    float z[U];
    auto fetch = [&](int i) {
#pragma unroll
        for (int u = 0; u < U; ++u) z[u] = Z[min(i + u * waves, E - 1) * a.ldz];
    };
    const bool once = E <= U * waves;   // a wave's rows stay in registers
    if constexpr (kFull) fetch(wv);
    for (int j = wv; j < K; j += waves) {
        int e = j < a.k ? a.chosen[j * a.ldk + c] : -1;
        if (e < 0 || e >= E) e = -1;
        const float x = e >= 0 ? Z[e * a.ldz] : -kInf;
        chosen[j][lane] = e;
        grads[j][lane] = e >= 0 ? a.dweights[j * a.ldk + c] : 0.f;
        // (without renormalisation a sigmoid's own gradient is all: it takes the place of its logarithm)
        logs[j][lane] = e < 0 || !sigmoid ? x : renormalise ? log_sigmoid(x) : (1.f / (1.f + expf(-x))) * (1.f / (1.f + expf(x)));
    }
    if constexpr (kFull) {
        float top = -kInf, s = 0.f;
        for (int i = wv; i < E; i += U * waves) {
            if (i > wv) fetch(i);
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, z[u]);
        }
        red[0][wv][lane] = top;
        __syncthreads();
        for (int w = 0; w < waves; ++w) top = fmaxf(top, red[0][w][lane]);
        for (int i = wv; i < E; i += U * waves) {
            if (!once) fetch(i);
#pragma unroll
            for (int u = 0; u < U; ++u) s += z[u] == -kInf || i + u * waves >= E ? 0.f : expf(z[u] - top);
        }
        red[1][wv][lane] = s;
        __syncthreads();
        s = 0.f;
        for (int w = 0; w < waves; ++w) s += red[1][w][lane];
        const float inv = 1.f / s;
        int e[K];
        float g[K], all = 0.f;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            e[j] = chosen[j][lane];
            g[j] = e[j] >= 0 ? a.scale * grads[j][lane] * (expf(logs[j][lane] - top) * inv) : 0.f;
            all += g[j];
        }
        if (!on) return;
        for (int i = wv; i < E; i += U * waves) {
            if (!once) fetch(i);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = i + u * waves;
                if (x >= E) break;
                float d = 0.f;
#pragma unroll
                for (int j = 0; j < K; ++j) d += e[j] == x ? g[j] : 0.f;
                if (!(z[u] == -kInf)) d -= expf(z[u] - top) * inv * all;
                dZ[x * a.lddz] = d;
            }
        }
    } else {
        if (on)
            for (int i = wv; i < E; i += waves) dZ[i * a.lddz] = 0.f;
        // the zeros come before what another wave writes in their places: they are waited for (vmcnt 0), and the barrier orders the work-group's
        // writes.  (A fence for the whole device would write the L2 back: 96 us where this takes 6.6, for 256 experts, 16384 columns and 8 choices.)
        __builtin_amdgcn_s_waitcnt(0x0F70);
        __syncthreads();
        if (!on || wv >= a.k) return;
        float high = -kInf, s = 0.f, mean = 0.f;
        if (renormalise) {
#pragma unroll
            for (int j = 0; j < K; ++j) high = fmaxf(high, logs[j][lane]);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const float u = chosen[j][lane] >= 0 ? expf(logs[j][lane] - high) : 0.f;
                s += u;
                mean = fmaf(u, grads[j][lane], mean);
            }
            s = 1.f / s;
            mean *= s;
        }
        auto gradient = [&](int j) {
            const float l = logs[j][lane], d = grads[j][lane];
            if (!renormalise) return a.scale * d * l;
            const float g = a.scale * (expf(l - high) * s) * (d - mean);
            return sigmoid ? g * -expm1f(l) : g;   // (times 1 - score)
        };
        for (int j = wv; j < a.k; j += waves) {
            const int e = chosen[j][lane];
            bool first = e >= 0;
            float d = 0.f;
            if (first) d = gradient(j);
            for (int i = 0; i < a.k; ++i) {   // an expert that a column has several times gets their sum, from the first of them
                if (i == j || chosen[i][lane] != e || e < 0) continue;
                if (i < j) first = false;
                else d += gradient(i);
            }
            if (first) dZ[e * a.lddz] = d;
        }
    }
}

template <int R>
hipError_t route_go(const RouteArgs &a, Keys keys, int cols, int waves, size_t lds, hipStream_t s)
{
    const dim3 grid((a.batch + cols - 1) / cols), block(waves * kWave);
    if (!fits_launch(grid.x, block.x)) return hipErrorInvalidConfiguration;
    if (keys == kLogits) hipLaunchKernelGGL((route_kernel<R, kLogits>), grid, block, lds, s, a, cols);
    else if (keys == kSigmoids) hipLaunchKernelGGL((route_kernel<R, kSigmoids>), grid, block, lds, s, a, cols);
    else hipLaunchKernelGGL((route_kernel<R, kSoftmaxes>), grid, block, lds, s, a, cols);
    return hipGetLastError();
}

constexpr int kRouteListSize = 8;  // experts in one, at least, where there may be fewer lists
template <int K, int kCols>
hipError_t route_columns_of(const RouteArgs &a, Keys keys, hipStream_t s)
{
    const int group_size = a.experts / a.groups;
    int parts = kRouteLists / a.groups;
    if (parts > group_size / kRouteListSize) parts = group_size / kRouteListSize;
    if (parts < 1) parts = 1;
    const int size = (group_size + parts - 1) / parts, lists = a.groups * parts, takers = lists < 4 ? 4 : lists;
    const size_t lds = (static_cast<size_t>(lists) * K + takers) * kCols * 8 + (K + takers) * kCols * 4;
    const dim3 grid((a.batch + kCols - 1) / kCols), block(takers * kCols);
    if (!fits_launch(grid.x, block.x)) return hipErrorInvalidConfiguration;
    if (keys == kLogits) hipLaunchKernelGGL((route_columns_kernel<K, kCols, kLogits>), grid, block, lds, s, a, lists, parts, size);
    else if (keys == kSigmoids) hipLaunchKernelGGL((route_columns_kernel<K, kCols, kSigmoids>), grid, block, lds, s, a, lists, parts, size);
    else hipLaunchKernelGGL((route_columns_kernel<K, kCols, kSoftmaxes>), grid, block, lds, s, a, lists, parts, size);
    return hipGetLastError();
}

// Work-groups of 64 columns where each of them finds a compute unit of its own and those of 32 would not; else of 32, which share one by two: 8192
// columns, 256 experts in 8 groups 18.3 us -> 14.0, 20000 columns 34.2 -> 27.7, 65536 70.5 -> 65; 16384 19.1 against 19.9, without groups
// 11.1 against 12.8.  Logits as keys and few choices leave registers for two of 64 at a time: 65536 columns of 96 experts 16.8, in 32s 19.8.
constexpr int kComputeUnits = 256;
template <int K>
hipError_t route_columns_go(const RouteArgs &a, Keys keys, hipStream_t s)
{
    const bool wide = a.batch > 32 * kComputeUnits && (a.batch <= 64 * kComputeUnits || (keys == kLogits && K <= 4));
    return wide ? route_columns_of<K, 64>(a, keys, s) : route_columns_of<K, 32>(a, keys, s);
}

// ---- places --------------------------------------------------------------------------------------
constexpr int kPlaceThreads = 512;
constexpr int kPlaceWaves = kPlaceThreads / kWave;

__device__ __forceinline__ int expert_at(const PlaceArgs &a, int c, int j)
{
    const int e = a.chosen[j * a.ldk + c];
    return e >= 0 && e < a.experts ? e : a.experts;   // (one more for "no expert")
}

constexpr int kPlaceCounts = 4096;
// Whether every work-group counts the choices of the whole batch for itself, in the place of a launch before: 777 columns with 4 choices
// 8.4 us against 2.4 + 6.4 and the gap between two launches, 1024 with 8 choices 15.8 against 4.7 + 10.3.
__host__ __device__ inline bool counts_itself(const PlaceArgs &a) { return a.batch * a.k <= kPlaceCounts; }

constexpr int kPlaceSums = 8192;
// Whether the counts of all runs are added up once, by a launch of its own, and not by every work-group for those before its own. That launch takes 2
// to 3 us (8192 columns and 2 choices of 8 experts 10.2 us against 7.0, 4 of 64 13.8 against 11.6), and adding up in every work-group takes time
// by the square of the columns: 8192 columns and 8 choices of 256 experts 19.8 us -> 18.8, 32768 and 4 of 64 15.1 -> 14.4, 65536 and 8 of 256 55 -> 23,
// 2^20 and one of 256 1300 -> 75.
__host__ __device__ inline bool sums_ahead(const PlaceArgs &a) { return !counts_itself(a) && static_cast<int64_t>(a.p.subs) * a.experts >= kPlaceSums; }

// choices of every expert in one run of kPlaceSub columns
__global__ __launch_bounds__(kPlaceThreads) void place_count_kernel(const PlaceArgs a)
{
    __shared__ int32_t n[kExpertsMax + 1];
    for (int e = threadIdx.x; e <= a.experts; e += kPlaceThreads) n[e] = 0;
    __syncthreads();
    const int c0 = blockIdx.x * kPlaceSub, here = min(kPlaceSub, a.batch - c0);
    for (int i = threadIdx.x; i < here * a.k; i += kPlaceThreads) {
        const int j = i / here;
        atomicAdd(&n[expert_at(a, c0 + i - j * here, j)], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += kPlaceThreads) a.p.before[static_cast<int64_t>(blockIdx.x) * a.experts + e] = n[e];
}

// Those counts to the numbers of choices in the runs before, with the totals behind the last run: a work-group has 64 experts, its waves one
// stretch of runs each, which they read for its sum and again for the numbers themselves.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(kSumWaves * kWave) void place_sum_kernel(const PlaceArgs a)
{
    __shared__ int32_t sums[kSumWaves][kWave];
    const int lane = threadIdx.x & (kWave - 1), wv = wave_in_block();
    const int e = blockIdx.x * kWave + lane, own = min(e, a.experts - 1);
    const int per = (a.p.subs + kSumWaves - 1) / kSumWaves;
    const int from = min(wv * per, a.p.subs), to = min(from + per, a.p.subs);
    int32_t *n = a.p.before + own;
    const int64_t E = a.experts;
    constexpr int U = 16;   // counts in flight
    int sum = 0;
    for (int q = from; q < to; q += U) {
        int32_t x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = n[min(q + u, to - 1) * E];
#pragma unroll
        for (int u = 0; u < U; ++u) sum += q + u < to ? x[u] : 0;
    }
    sums[wv][lane] = sum;
    __syncthreads();
    sum = 0;
    for (int w = 0; w < wv; ++w) sum += sums[w][lane];
    if (e >= a.experts) return;
    for (int q = from; q < to; q += U) {
        int32_t x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = n[min(q + u, to - 1) * E];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (q + u >= to) break;
            n[(q + u) * E] = sum;
            sum += x[u];
        }
    }
    if (wv == kSumWaves - 1) n[a.p.subs * E] = sum;   // (a stretch may be empty: the last wave's sum is that of all)
}

// exclusive scans of N numbers over the work-group's threads; total: their sums
template <int N>
__device__ __forceinline__ void block_scan(int (&x)[N], int (*lds)[N], int (&total)[N])
{
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x >> 6;
    int s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = x[i];
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int y = __shfl_up(s[i], d, kWave);
            if (lane >= d) s[i] += y;
        }
        if (lane == kWave - 1) lds[wv][i] = s[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        int off = 0;
        total[i] = 0;
#pragma unroll
        for (int w = 0; w < kPlaceWaves; ++w) {
            const int n = lds[w][i];
            off += w < wv ? n : 0;
            total[i] += n;
        }
        x[i] = off + s[i] - x[i];
    }
}

// Turns of the 64 entries from i on (one wave): how many of the lanes before hold the same column, from one ballot per bit of it.
__device__ __forceinline__ void set_turns(int2 *list, int i, int kept)
{
    const int lane = threadIdx.x & (kWave - 1);
    const bool on = i + lane < kept;
    const int word = on ? list[i + lane].y : 0;
    uint64_t same = __ballot(on);
    for (int b = 0; b < 10; ++b) {
        const uint64_t has = __ballot(word >> b & 1);
        same &= word >> b & 1 ? has : ~has;
    }
    const int turn = __popcll(same & ((1ull << lane) - 1));
    if (on && turn > 0) list[i + lane].y = static_cast<int>(static_cast<uint32_t>(word) | static_cast<uint32_t>(turn) << 26);
}

// Places of one run of kPlaceSub columns.  A choice's place is the number of choices of its expert before it, in the order of columns
// and, in a column, of choices: those of the runs before (added up before this launch or here), of the run's earlier rounds of one choice per
// thread, of the waves before in the round, and of the lanes before in the wave (the lanes that hold the same expert, from one
// ballot per bit of its number).
__global__ __launch_bounds__(kPlaceThreads) void place_kernel(const PlaceArgs a)
{
    __shared__ int32_t next[kExpertsMax + 1];     // the expert's next place
    __shared__ int32_t kept_at[kExpertsMax + 1];  // list position of a place: kept_at + place, or ...
    __shared__ int32_t lost_at[kExpertsMax + 1];  // ... lost_at + place, of places beyond the capacity
    __shared__ int scan[kPlaceWaves][3];
    extern __shared__ int32_t by_wave[];          // [kPlaceWaves][E + 1] choices in one turn of the loop; at first before | inside | mine, [E + 1] each
    const int E = a.experts, E1 = E + 1;
    const int lane = threadIdx.x & (kWave - 1), wv = wave_in_block();
    const int subs_per_tile = a.p.tile / kPlaceSub, sub = blockIdx.x, tile = sub / subs_per_tile;
    const int tile_sub = tile * subs_per_tile, tile_end = min(tile_sub + subs_per_tile, a.p.subs);
    const int c0 = sub * kPlaceSub, here = min(kPlaceSub, a.batch - c0);

    // choices per expert: before the tile, in the tile, and in its runs before this one
    int32_t *before = by_wave, *inside = by_wave + E1, *mine = by_wave + 2 * E1;
    static_assert(kPlaceWaves >= 3, "room for them");
    if (!sums_ahead(a)) {
        for (int i = threadIdx.x; i < 3 * E1; i += kPlaceThreads) by_wave[i] = 0;
        __syncthreads();
        auto add = [&](int q, int e, int n) {   // n choices of expert e in run q
            if (q < tile_sub) {
                atomicAdd(&before[e], n);
            } else if (q < tile_end) {
                atomicAdd(&inside[e], n);
                if (q < sub) atomicAdd(&mine[e], n);
            }
        };
        if (counts_itself(a)) {
            for (int i = threadIdx.x; i < a.batch * a.k; i += kPlaceThreads) {
                const int j = i / a.batch, c = i - j * a.batch;
                add(c / kPlaceSub, expert_at(a, c, j), 1);
            }
        } else {
            const int n = tile_end * E;   // (at most kPlaceSums)
#pragma unroll 4
            for (int i = threadIdx.x; i < n; i += kPlaceThreads) {
                const int q = i / E;
                add(q, i - q * E, a.p.before[i]);
            }
        }
    } else {
        for (int e = threadIdx.x; e < E; e += kPlaceThreads) {
            const int32_t *n = a.p.before + e;
            const int at_tile = n[static_cast<int64_t>(tile_sub) * E];
            before[e] = at_tile;
            inside[e] = n[static_cast<int64_t>(tile_end) * E] - at_tile;
            mine[e] = n[static_cast<int64_t>(sub) * E] - at_tile;
        }
    }
    __syncthreads();
    int sums[3] = {0, 0, 0};   // choices with a place in this tile, without one, and of any expert in its runs before this one
    const int per = (E1 + kPlaceThreads - 1) / kPlaceThreads;   // consecutive experts per thread
    int kept[(kExpertsMax + 1 + kPlaceThreads - 1) / kPlaceThreads], lost[sizeof kept / sizeof *kept], at[sizeof kept / sizeof *kept], now[sizeof kept / sizeof *kept];
    const int first = threadIdx.x * per;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof kept / sizeof *kept); ++i) {
        kept[i] = lost[i] = at[i] = now[i] = 0;
        const int e = first + i;
        if (i >= per || e >= E) continue;
        at[i] = before[e];
        now[i] = at[i] + mine[e];
        kept[i] = min(a.capacity, at[i] + inside[e]) - min(a.capacity, at[i]);
        lost[i] = inside[e] - kept[i];
        sums[0] += kept[i];
        sums[1] += lost[i];
        sums[2] += mine[e];
        if (tile == a.p.tiles - 1 && sub == tile_sub) {   // one work-group knows the whole batch
            if (a.counts) a.counts[e] = at[i] + inside[e];
            a.p.filled[e] = min(a.capacity, at[i] + inside[e]);
        }
    }
    int totals[3];
    block_scan(sums, scan, totals);   // (its barrier: the counts are read)
    int kept_off = sums[0], lost_off = sums[1];
    const int kept_all = totals[0], lost_all = totals[1], mine_all = totals[2];
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof kept / sizeof *kept); ++i) {
        const int e = first + i;
        if (i >= per || e >= E) continue;
        next[e] = now[i];
        kept_at[e] = kept_off - min(a.capacity, at[i]);
        lost_at[e] = kept_all + lost_off - max(a.capacity, at[i]);
        kept_off += kept[i];
        lost_off += lost[i];
    }
    // choices of no expert come last, counted from the tile's start
    if (threadIdx.x == 0) {
        next[E] = (sub - tile_sub) * kPlaceSub * a.k - mine_all;
        lost_at[E] = kept_all + lost_all;
        if (sub == tile_sub) a.p.listed[tile] = kept_all;
    }
    for (int i = threadIdx.x; i < kPlaceWaves * E1; i += kPlaceThreads) by_wave[i] = 0;
    __syncthreads();

    int bits = 0;
    while (E >> bits) ++bits;
    int2 *list = a.p.lists + static_cast<int64_t>(tile) * a.p.tile * a.k;
    const int wave_columns = kWave / a.k;   // whole columns per wave, a lane for each of their choices
    const int lane_column = lane / a.k, j = lane - lane_column * a.k;
    for (int r = 0; r < here; r += kPlaceWaves * wave_columns) {
        const int cl = r + wv * wave_columns + lane_column;
        const bool on = lane_column < wave_columns && cl < here;
        const int e = on ? expert_at(a, c0 + cl, j) : 0;
        uint64_t same = __ballot(on);
        for (int b = 0; b < bits; ++b) {
            const uint64_t has = __ballot(e >> b & 1);
            same &= e >> b & 1 ? has : ~has;
        }
        const uint64_t below = (1ull << lane) - 1;
        const int rank = __popcll(same & below);
        if (on && rank == 0) by_wave[wv * E1 + e] = __popcll(same);
        __syncthreads();
        for (int x = threadIdx.x; x < E1; x += kPlaceThreads) {
            int p = next[x];
            for (int w = 0; w < kPlaceWaves; ++w) {
                const int n = by_wave[w * E1 + x];
                by_wave[w * E1 + x] = p;
                p += n;
            }
            next[x] = p;
        }
        __syncthreads();
        int place = 0;
        if (on) place = by_wave[wv * E1 + e] + rank;
        __syncthreads();
        for (int x = threadIdx.x; x < kPlaceWaves * E1; x += kPlaceThreads) by_wave[x] = 0;
        __syncthreads();
        if (!on) continue;
        const bool has = e < E && place < a.capacity;
        if (a.slots) a.slots[j * a.ldk + c0 + cl] = has ? place : -1;
        const int column = c0 + cl - tile * a.p.tile;
        list[(has ? kept_at[e] : lost_at[e]) + place] = make_int2(has ? place : -1, column | j << 10 | e << 15);
    }
    if (subs_per_tile > 1) return;   // (place_turns_kernel follows)
    __syncthreads();
    for (int i = wv * kWave; i < kept_all; i += kPlaceThreads) set_turns(list, i, kept_all);
}

// the same for tiles that several work-groups have listed
__global__ __launch_bounds__(kPlaceThreads) void place_turns_kernel(const PlaceArgs a, const int blocks_per_tile)
{
    const int tile = blockIdx.x / blocks_per_tile, i = (blockIdx.x - tile * blocks_per_tile) * kPlaceThreads + wave_in_block() * kWave;
    const int kept = a.p.listed[tile];
    if (i < kept) set_turns(a.p.lists + static_cast<int64_t>(tile) * a.p.tile * a.k, i, kept);
}

// ---- exchange --------------------------------------------------------------------------------------
struct Entry {
    int place, column, choice, expert, turn;
};
__device__ __forceinline__ Entry entry_of(int2 x)
{
    return Entry{x.x, x.y & 1023, x.y >> 10 & 31, x.y >> 15 & 2047, static_cast<int>(static_cast<uint32_t>(x.y) >> 26)};
}
// whether an entry lies in this call's operands: a placement made for other sizes must not lead outside
__device__ __forceinline__ bool inside(const Entry &t, const ExchangeArgs &a, int here)
{
    return static_cast<uint32_t>(t.place) < static_cast<uint32_t>(a.capacity) && t.column < here && t.choice < a.k && t.expert < a.experts;
}

// Work-groups are numbered tile by tile and then by rows, and every XCD gets one run of consecutive ones: the runs of one row that
// neighbouring tiles read or write share cache lines, which then meet in one L2.
__device__ __forceinline__ int xcd_run(int block, int blocks) { return (block & 7) * (blocks >> 3) + (block >> 3); }   // (blocks: a multiple of 8)

// Rows of a matrix to LDS, `pitch` (a multiple of 4) apart: all of a thread's reads are in flight before the first is written.
__device__ __forceinline__ void stage_rows(float *lds, int pitch, const float *in, int64_t ld, int n, int columns)
{
    const int threads = blockDim.x;
    if (columns < 4) {
        for (int i = threadIdx.x; i < n * columns; i += threads) lds[i / columns * pitch + i % columns] = in[i / columns * ld + i % columns];
        return;
    }
    const int per_row = (columns + 3) >> 2, total = n * per_row;
    for (int i = threadIdx.x; i < total; i += 4 * threads) {
        float4 x[4];
        int at[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = min(i + u * threads, total - 1), r = j / per_row, c = four_columns(4 * (j - r * per_row), columns);
            x[u] = ld4(in + r * ld + c);
            at[u] = r * pitch + c;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float *p = lds + at[u];
            if ((at[u] & 3) == 0) {
                *reinterpret_cast<float4 *>(p) = x[u];
            } else {   // (a row's last four, where its length is no multiple of 4)
                p[0] = x[u].x;
                p[1] = x[u].y;
                p[2] = x[u].z;
                p[3] = x[u].w;
            }
        }
    }
}
__device__ __host__ __forceinline__ int pitch_of(int batch, int tile) { return ((batch < tile ? batch : tile) + 3) / 4 * 4; }

// Columns to blocks: dispatch (kGrad false), or the combine's backward pass (kGrad true), which weighs the columns and takes their products
// with the blocks' results.  A work-group keeps kRows rows of one tile's columns in LDS and walks through the tile's list, whose
// neighbours lie next to each other in a block.  The empty places are cleared on the way, a share of the experts by each tile's work-groups.
constexpr int kMoveThreads = 1024;   // at most; one per entry of the list where that is fewer
template <int kRows, bool kGrad>
__global__ __launch_bounds__(kMoveThreads) void dispatch_kernel(const ExchangeArgs a, const int staged)
{
    extern __shared__ __align__(16) float rows[];   // [kRows][width], then with `staged` the weights [k][width]
    const int tiles = a.p.tiles, at_block = xcd_run(blockIdx.x, gridDim.x), threads = blockDim.x;
    const int group = at_block / tiles, tile = at_block - group * tiles;
    const int f0 = group * kRows, nf = min(kRows, a.features - f0);
    if (nf <= 0) return;
    const int c0 = tile * a.p.tile, here = min(a.p.tile, a.batch - c0), width = pitch_of(a.batch, a.p.tile);
    stage_rows(rows, width, a.columns + static_cast<int64_t>(f0) * a.ldc + c0, a.ldc, nf, here);
    if (kGrad && staged) stage_rows(rows + kRows * width, width, a.weights + c0, a.ldk, a.k, here);
    __syncthreads();
    const int total = here * a.k, kept = min(max(a.p.listed[tile], 0), total);
    const int2 *list = a.p.lists + static_cast<int64_t>(tile) * a.p.tile * a.k;
    float *partial = kGrad ? a.partial + static_cast<int64_t>(group) * a.batch * a.k + static_cast<int64_t>(tile) * a.p.tile * a.k : nullptr;
    auto move = [&](auto whole) {
        const int n = whole.value ? kRows : nf;   // (without a bound inside, a whole group's loads are all in flight at once)
        for (int i = threadIdx.x; i < kept; i += threads) {
            const Entry t = entry_of(list[i]);
            if (!inside(t, a, here)) continue;
            const int64_t at = (static_cast<int64_t>(t.expert) * a.features + f0) * a.ldb + t.place;
            float *out = a.out_blocks + at;
            if constexpr (kGrad) {
                const float w = staged ? rows[(kRows + t.choice) * width + t.column] : a.weights ? a.weights[t.choice * a.ldk + c0 + t.column] : 1.f;
                if (a.dweights) {
                    const float *y = a.blocks + at;
                    float dot = 0.f;
#pragma unroll
                    for (int r = 0; r < n; ++r) dot = fmaf(y[r * a.ldb], rows[r * width + t.column], dot);
                    partial[i] = dot;
                }
                if (!a.out_blocks) continue;
#pragma unroll
                for (int r = 0; r < n; ++r) out[r * a.ldb] = w * rows[r * width + t.column];
            } else {
#pragma unroll
                for (int r = 0; r < n; ++r) out[r * a.ldb] = rows[r * width + t.column];
            }
        }
    };
    if (nf == kRows) move(std::true_type{});
    else move(std::false_type{});
    if (!a.out_blocks) return;
    const int lane = threadIdx.x & (kWave - 1), waves = threads / kWave;
    const int share = (a.experts + tiles - 1) / tiles, end = min(a.experts, (tile + 1) * share);
    for (int e0 = tile * share + wave_in_block(); e0 < end; e0 += waves * kWave) {
        // lane l knows how full block e0 + l * waves is
        const int filled = min(max(a.p.filled[min(e0 + lane * waves, a.experts - 1)], 0), a.capacity);
        for (int l = 0; l < kWave && e0 + l * waves < end; ++l) {
            float *block = a.out_blocks + (static_cast<int64_t>(e0 + l * waves) * a.features + f0) * a.ldb;
            for (int p = __builtin_amdgcn_readlane(filled, l) + lane; p < a.capacity; p += kWave)
                for (int r = 0; r < nf; ++r) block[r * a.ldb + p] = 0.f;
        }
    }
}

// Gradients of the weights from the products of every group of rows: a wave adds up every eighth group for 64 entries, and
// the waves' sums are added in their order.
__global__ __launch_bounds__(kGradThreads) void weight_gradient_kernel(const ExchangeArgs a, const int groups)
{
    constexpr int kGradWaves = kGradThreads / kWave;
    __shared__ double sums[kGradWaves][kWave];
    const int lane = threadIdx.x & (kWave - 1), wv = wave_in_block();
    const int64_t total = static_cast<int64_t>(a.batch) * a.k, i = static_cast<int64_t>(blockIdx.x) * kWave + lane;
    const int tile = static_cast<int>(min(i, total - 1) / (static_cast<int64_t>(a.p.tile) * a.k));
    const int64_t from = static_cast<int64_t>(tile) * a.p.tile * a.k;
    double sum = 0.0;   // (hundreds of sums, each read once: 64 bits cost nothing)
    if (i < total && i - from < a.p.listed[tile]) {
        const float *p = a.partial + i;
        int g = wv;
        for (; g + 3 * kGradWaves < groups; g += 4 * kGradWaves) {
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = p[(g + u * kGradWaves) * total];
#pragma unroll
            for (int u = 0; u < 4; ++u) sum += v[u];
        }
        for (; g < groups; g += kGradWaves) sum += p[g * total];
    }
    sums[wv][lane] = sum;
    __syncthreads();
    if (wv > 0 || i >= total) return;
#pragma unroll
    for (int w = 1; w < kGradWaves; ++w) sum += sums[w][lane];
    const int c0 = tile * a.p.tile, here = min(a.p.tile, a.batch - c0);
    const Entry t = entry_of(a.p.lists[i]);
    if (t.column >= here || t.choice >= a.k) return;
    a.dweights[t.choice * a.ldk + c0 + t.column] = static_cast<float>(sum);
}

// Blocks to columns, Y = sum of the kept choices' results times their weights, in the order of the list.  A wave keeps the sums of
// kCombineRows rows and one tile's columns in LDS, for itself alone, so that nothing waits for other waves, and adds 64 entries of the
// list to them at a time: read, add, write, for the first entry of every column, then for the second ones, as the turns say.
// (LDS additions as atomics would need no turns, but take about 176 cycles for 64 lanes: 600 us for 4096 features, 8192 columns and four
// choices of 64 experts, where this takes 158, 5.1 TB/s, and 171 with weights.)
constexpr size_t kCombineLds = 160 * 1024;
constexpr int64_t kCombineWavesWanted = 1536;
constexpr int kCombineUnroll = 4;    // list entries per lane and iteration; those of the next one are on their way
enum Weights { kAllOne, kGathered, kStaged };
template <int kRows, int kWaves, Weights kWeights>
__global__ __launch_bounds__(kWaves * kWave) void combine_kernel(const ExchangeArgs a)
{
    constexpr int U = kCombineUnroll;
    extern __shared__ __align__(16) float rows[];   // [waves][kRows][width], then with kStaged the weights [k][width]
    const int lane = threadIdx.x & (kWave - 1), wv = wave_in_block();
    const int tiles = a.p.tiles, at_block = xcd_run(blockIdx.x, gridDim.x);
    const int group = at_block / tiles, tile = at_block - group * tiles;
    if (group * kWaves * kRows >= a.features) return;
    const int f0 = (group * kWaves + wv) * kRows, nf = min(kRows, a.features - f0);
    const int c0 = tile * a.p.tile, here = min(a.p.tile, a.batch - c0), width = pitch_of(a.batch, a.p.tile);
    const int total = here * a.k, kept = min(max(a.p.listed[tile], 0), total);
    const int2 *__restrict__ list = a.p.lists + static_cast<int64_t>(tile) * a.p.tile * a.k;
    const float *__restrict__ weights = a.weights + c0;
    float *staged = rows + kWaves * kRows * width;
    float *sum = rows + wv * kRows * width;
    for (int i = lane; i < kRows * width; i += kWave) sum[i] = 0.f;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int64_t block = a.features * a.ldb, last_row = (max(nf, 1) - 1) * a.ldb;
    const float *__restrict__ first = a.blocks + min(f0, a.features - 1) * a.ldb;
    // Entries are read one iteration before their values, and those one before they are added.  All reads are made, at a place of their own or
    // a valid one, so that none waits for a branch.  Weights are staged between the first of these reads, and taken from LDS where they are
    // used: 1501 rows of 777 columns 13.4 us -> 12.1, 512 of 4096 with 16 experts 12.2 -> 11.4, 4096 of 8192 174 -> 171.
    struct Values {
        float w[U], v[U][kRows];
        int column[U], turn[U], weight[U];   // (turn -1: no entry; weight: where it is in `staged`)
    };
    int2 entry[U];
    auto fetch_entries = [&](int i) {
#pragma unroll
        for (int u = 0; u < U; ++u) entry[u] = list[min(i + u * kWave + lane, total - 1)];
    };
    auto fetch_values = [&](int i) {
        Values x;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Entry t = entry_of(entry[u]);
            const bool on = i + u * kWave + lane < kept && inside(t, a, here);
            x.column[u] = t.column;
            x.turn[u] = on ? t.turn : -1;
            const float *y = first + (on ? t.expert * block + t.place : 0);
#pragma unroll
            for (int r = 0; r < kRows; ++r) x.v[u][r] = y[min(r * a.ldb, last_row)];
            if constexpr (kWeights == kGathered) x.w[u] = weights[on ? t.choice * a.ldk + t.column : 0];
            else if constexpr (kWeights == kStaged) x.weight[u] = on ? t.choice * width + t.column : 0;
            else x.w[u] = 1.f;
        }
        return x;
    };
    fetch_entries(0);
    if constexpr (kWeights == kStaged) stage_rows(staged, width, weights, a.ldk, a.k, here);
    Values now = fetch_values(0);
    fetch_entries(U * kWave);
    if constexpr (kWeights == kStaged) __syncthreads();
    if (nf <= 0) return;              // (no barrier from here on: waves share nothing that is written)
    for (int i = 0; i < kept; i += U * kWave) {
        const Values next = fetch_values(i + U * kWave);
        fetch_entries(i + 2 * U * kWave);
        if constexpr (kWeights == kStaged) {
#pragma unroll
            for (int u = 0; u < U; ++u) now.w[u] = staged[now.weight[u]];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            int m = 0;
            do {
                if (now.turn[u] == m) {
                    float *s = sum + now.column[u];
                    float x[kRows];
#pragma unroll
                    for (int r = 0; r < kRows; ++r) x[r] = s[r * width];
#pragma unroll
                    for (int r = 0; r < kRows; ++r) s[r * width] = x[r] + __fmul_rn(now.w[u], now.v[u][r]);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                ++m;
            } while (__ballot(now.turn[u] >= m));
        }
        now = next;
    }
    float *out = a.out_columns + f0 * a.ldc + c0;
    for (int r = 0; r < nf; ++r, out += a.ldc)
        for (int c = lane; c < here; c += kWave) out[c] = sum[r * width + c];
}

uint32_t whole_eights(int64_t blocks) { return static_cast<uint32_t>((blocks + 7) / 8 * 8); }

constexpr size_t kMoveLds = 160 * 1024;
template <int kRows, bool kGrad>
hipError_t dispatch_go(const ExchangeArgs &a, hipStream_t s)
{
    const int groups = (a.features + kRows - 1) / kRows, width = pitch_of(a.batch, a.p.tile);
    const int share = (a.experts + a.p.tiles - 1) / a.p.tiles;   // of the experts, cleared one per wave
    int threads = (width * a.k > 16 * share ? width * a.k : 16 * share);
    // (with few work-groups rather twice as many at a time on a compute unit: 1501 rows of 777 columns 15.0 us -> 12.8, 512 of 4096 12.6 -> 10.6;
    // with many it is the other way round: 4096 rows of 8192 columns, one choice, 77 us -> 91)
    if (static_cast<int64_t>(groups) * a.p.tiles < 2048) threads /= 2;
    threads = (threads + kWave - 1) / kWave * kWave;
    threads = threads < 512 ? 512 : threads > kMoveThreads ? kMoveThreads : threads;
    // Weights from LDS, if only one work-group fits a compute unit with them: 64 experts and 4 choices 337 us -> 315, 256 and 8 (96 KiB) 413 -> 371; from the
    // caches 64 lanes read 64 lines.
    const size_t lds = kRows * width * sizeof(float), with_weights = lds + static_cast<size_t>(width) * a.k * sizeof(float);
    const bool staged = kGrad && a.weights && a.out_blocks && with_weights <= kMoveLds;
    const uint32_t blocks = whole_eights(static_cast<int64_t>(groups) * a.p.tiles);
    if (!fits_launch(blocks, threads)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((dispatch_kernel<kRows, kGrad>), dim3(blocks), dim3(threads), staged ? with_weights : lds, s, a, staged ? 1 : 0);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_route(const RouteArgs &a, hipStream_t s)
{
    const Keys keys = !a.bias && !(a.flags & NERVA_EXPERT_GROUP_PAIR) ? kLogits : a.flags & NERVA_EXPERT_SIGMOID ? kSigmoids : kSoftmaxes;
    // A lane per column from where work-groups of a wave per column, which take 16, no longer find a compute unit each (5000 columns, 256 experts, 8
    // choices 25.0 us -> 13.9, 96 experts and 4 choices 9.8 -> 6.3), a little later for one or two choices, which a wave finds in as many
    // rounds (4100 columns, 60 experts, one choice 4.3 against 6.0; 5000 5.8 and 6.0, 128 experts in groups 15 and 9), and with half of
    // that already for many choices from many experts (4096 columns 14.4 -> 11.5 with 256 experts, 11.9 -> 8.9 with 128, 30 -> 14 with
    // 1024; 512 experts and 2048 columns 15.0 against 15.8, 64 and four choices 5.8 against 6.3).
    if (a.k <= 8 && a.groups <= kRouteLists) {
        if (a.batch > (a.k > 2 ? 16 : 18) * kComputeUnits)
            return a.k <= 2 ? route_columns_go<2>(a, keys, s) : a.k <= 4 ? route_columns_go<4>(a, keys, s) : route_columns_go<8>(a, keys, s);
        if (a.batch >= 8 * kComputeUnits && a.experts >= 128 && a.k > 4) return route_columns_of<8, 16>(a, keys, s);
    }
    int cols = a.batch >= 8192 ? 32 : a.batch >= 2048 ? 16 : a.batch >= 512 ? 8 : 4;
    auto bytes = [&](int c) {
        const int waves = c < 16 ? c : 16;
        const size_t tile = static_cast<size_t>((a.experts * (c + 1) + 3) / 4 * 4 + 2 * c * a.k + 3) / 4 * 16;
        return tile + (a.groups > 1 ? static_cast<size_t>(waves) * a.experts * 8 : 0);
    };
    while (cols > 4 && bytes(cols) > 64 * 1024) cols /= 2;
    const int waves = cols < 16 ? cols : 16;
    const size_t lds = bytes(cols);
    if (a.experts <= 64) return route_go<1>(a, keys, cols, waves, lds, s);
    if (a.experts <= 128) return route_go<2>(a, keys, cols, waves, lds, s);
    if (a.experts <= 256) return route_go<4>(a, keys, cols, waves, lds, s);
    if (a.experts <= 512) return route_go<8>(a, keys, cols, waves, lds, s);
    return route_go<16>(a, keys, cols, waves, lds, s);
}

template <int K>
static hipError_t route_backward_go(const RouteBackwardArgs &a, hipStream_t s)
{
    int waves = a.experts / kBackRows;
    waves = waves < 4 ? 4 : waves > kBackWaves ? kBackWaves : waves;
    const dim3 grid((a.batch + kWave - 1) / kWave), block(waves * kWave);
    if (!fits_launch(grid.x, block.x)) return hipErrorInvalidConfiguration;
    if (a.flags & (NERVA_EXPERT_SIGMOID | NERVA_EXPERT_RENORMALISE)) hipLaunchKernelGGL((route_backward_kernel<K, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((route_backward_kernel<K, true>), grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_route_backward(const RouteBackwardArgs &a, hipStream_t s)
{
    if (a.k <= 1) return route_backward_go<1>(a, s);
    if (a.k <= 2) return route_backward_go<2>(a, s);
    if (a.k <= 4) return route_backward_go<4>(a, s);
    if (a.k <= 8) return route_backward_go<8>(a, s);
    if (a.k <= 16) return route_backward_go<16>(a, s);
    return route_backward_go<32>(a, s);
}

hipError_t launch_place(const PlaceArgs &a, hipStream_t s)
{
    if (!counts_itself(a)) {
        hipLaunchKernelGGL(place_count_kernel, dim3(a.p.subs), dim3(kPlaceThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (sums_ahead(a)) {
        hipLaunchKernelGGL(place_sum_kernel, dim3((a.experts + kWave - 1) / kWave), dim3(kSumWaves * kWave), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(place_kernel, dim3(a.p.subs), dim3(kPlaceThreads), kPlaceWaves * (a.experts + 1) * sizeof(int32_t), s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.p.tile == kPlaceSub) return e;
    const int blocks = (a.p.tile * a.k + kPlaceThreads - 1) / kPlaceThreads;
    hipLaunchKernelGGL(place_turns_kernel, dim3(static_cast<uint32_t>(a.p.tiles) * blocks), dim3(kPlaceThreads), 0, s, a, blocks);
    return hipGetLastError();
}

hipError_t launch_dispatch(const ExchangeArgs &a, hipStream_t s)
{
    // All that the work-groups of one XCD write at a time should stay in its L2 until the neighbouring tile has filled the lines up.
    int most = 16;
    while (most > 4 && most * a.p.tile * a.k > 8192) most /= 2;
    int rows = move_rows(a.features, a.p.tiles, most);
    while (rows < 16 && !fits_launch(static_cast<int64_t>((a.features + rows - 1) / rows) * a.p.tiles + 7, kMoveThreads)) rows *= 2;   // (2^32 entries and more)
    return rows == 16 ? dispatch_go<16, false>(a, s) : rows == 8 ? dispatch_go<8, false>(a, s) : dispatch_go<4, false>(a, s);
}

template <int kRows, int kWaves>
static hipError_t combine_go(const ExchangeArgs &a, hipStream_t s)
{
    constexpr int per_block = kRows * kWaves;
    const int groups = (a.features + per_block - 1) / per_block, width = pitch_of(a.batch, a.p.tile);
    const dim3 grid(whole_eights(static_cast<int64_t>(groups) * a.p.tiles)), block(kWaves * kWave);
    const size_t lds = per_block * width * sizeof(float), with_weights = lds + static_cast<size_t>(width) * a.k * sizeof(float);
    if (!fits_launch(grid.x, block.x)) return hipErrorInvalidConfiguration;
    if (!a.weights) hipLaunchKernelGGL((combine_kernel<kRows, kWaves, kAllOne>), grid, block, lds, s, a);
    else if (with_weights <= kCombineLds) hipLaunchKernelGGL((combine_kernel<kRows, kWaves, kStaged>), grid, block, with_weights, s, a);
    else hipLaunchKernelGGL((combine_kernel<kRows, kWaves, kGathered>), grid, block, lds, s, a);
    return hipGetLastError();
}

hipError_t launch_combine(const ExchangeArgs &a, hipStream_t s)
{
    auto waves = [&](int rows) { return static_cast<int64_t>((a.features + rows - 1) / rows) * a.p.tiles; };
    if (waves(4) < kCombineWavesWanted) return waves(2) < kCombineWavesWanted ? combine_go<1, 4>(a, s) : combine_go<2, 4>(a, s);
    return a.p.tile * a.k > 4096 ? combine_go<4, 8>(a, s) : combine_go<4, 4>(a, s);
}

hipError_t launch_combine_backward(const ExchangeArgs &a, hipStream_t s)
{
    const int rows = move_rows(a.features, a.p.tiles, 16);   // (at least partial_rows, which the workspace has room for)
    const int64_t sums = weight_gradient_blocks(a.batch, a.k);
    if (a.dweights && !fits_launch(sums, kGradThreads)) return hipErrorInvalidConfiguration;
    const hipError_t e = rows == 16 ? dispatch_go<16, true>(a, s) : rows == 8 ? dispatch_go<8, true>(a, s) : dispatch_go<4, true>(a, s);
    if (e != hipSuccess || !a.dweights) return e;
    hipLaunchKernelGGL(weight_gradient_kernel, dim3(static_cast<uint32_t>(sums)), dim3(kGradThreads), 0, s, a, (a.features + rows - 1) / rows);
    return hipGetLastError();
}

}  // namespace nerva
