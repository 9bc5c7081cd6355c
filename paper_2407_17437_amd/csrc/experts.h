// Internal launch interface between the C ABI (api.hip) and the kernels of mixtures (experts.hip) and of clipped
// gradients (clip.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nerva {

// ---- routing (experts.hip) ----------------------------------------------------------------
// A launch holds fewer than 2^32 threads.  Those of mixtures return hipErrorInvalidConfiguration, with nothing launched, where one of them would
// take more.
inline bool fits_launch(int64_t blocks, int64_t threads) { return blocks * threads < (INT64_C(1) << 32); }

struct RouteArgs {
    const float *Z;
    int64_t ldz;
    const float *bias;     // [experts] or nullptr
    int32_t experts, batch, k, groups, top_groups, flags;
    float scale;
    int32_t *chosen;       // (k, ldk)
    float *weights;        // (k, ldk)
    int64_t ldk;
};
struct RouteBackwardArgs {
    const float *Z;
    int64_t ldz;
    const int32_t *chosen;
    const float *dweights;
    int64_t ldk;
    int32_t experts, batch, k, flags;
    float scale;
    float *dZ;
    int64_t lddz;
};
hipError_t launch_route(const RouteArgs &a, hipStream_t s);
hipError_t launch_route_backward(const RouteBackwardArgs &a, hipStream_t s);

// ---- places of columns in the experts' blocks -----------------------------------------------
// The batch is cut into tiles of columns.  Every tile has a list of its choices: those that have a place, by expert and then by place,
// followed by those that have none.  An entry is {place or -1, column in the tile | choice << 10 | expert << 15 | turn << 26}.
// Entries that 64 lanes take at a time and that belong to one column get turns 0, 1, ... in their order; an expert's entries lie
// next to each other in its block.
// Tiles: as many columns as give an expert some kPlaceRun consecutive entries, a multiple of kPlaceSub.  Longer tiles would only
// take local memory and parallelism from the kernels that hold a tile's columns.
constexpr int32_t kPlaceTileMax = 1024;
constexpr int32_t kPlaceSub = 256;           // columns per work-group that assigns places
constexpr int32_t kPlaceRun = 64;
constexpr int32_t kExpertsMax = 1024;        // 11 bits, with "no expert"
constexpr int32_t kChoicesMax = 32;          // 5 bits
constexpr int32_t kGroupsMax = 64;           // one per lane

struct Placement {
    int32_t *filled;       // [experts] places that hold a column
    int32_t *listed;       // [tiles] entries with a place
    int32_t *before;       // [(subs + 1) * experts] choices of an expert in a run of kPlaceSub columns, then in all runs before it
    int2 *lists;           // [batch * k]: tile t's from t * tile * k on
    int32_t tile, tiles, subs;
    int64_t bytes;
};
// the parts of a caller's buffer (which may be nullptr, for its size)
inline Placement placement_of(void *memory, int32_t experts, int32_t batch, int32_t k)
{
    Placement p{};
    p.tile = kPlaceSub;
    while (p.tile < kPlaceTileMax && p.tile * k < kPlaceRun * experts && p.tile <= batch / 4) p.tile *= 2;
    p.tiles = (batch + p.tile - 1) / p.tile;
    p.subs = (batch + kPlaceSub - 1) / kPlaceSub;
    char *m = static_cast<char *>(memory);
    const int64_t lists = static_cast<int64_t>(batch) * k;
    p.lists = reinterpret_cast<int2 *>(m);
    p.filled = reinterpret_cast<int32_t *>(p.lists + lists);
    p.listed = p.filled + experts;
    p.before = p.listed + p.tiles;
    p.bytes = (8 * lists + 4 * (experts + p.tiles + (static_cast<int64_t>(p.subs) + 1) * experts) + 15) / 16 * 16;
    return p;
}

struct PlaceArgs {
    const int32_t *chosen;
    int64_t ldk;
    int32_t experts, batch, k, capacity;
    int32_t *slots;        // (k, ldk) or nullptr
    int32_t *counts;       // [experts] or nullptr
    Placement p;
};
hipError_t launch_place(const PlaceArgs &a, hipStream_t s);

// Columns to blocks and back.  Block e of an operand (experts, features, ld) starts at e * features * ld.
struct ExchangeArgs {
    const float *columns;  // (features, ldc): X of the dispatch, dY of the combine's backward pass
    float *out_columns;    // (features, ldc): Y of the combine
    int64_t ldc;
    const float *blocks;   // Ye
    float *out_blocks;     // Xe, dYe
    int64_t ldb;
    const float *weights;  // (k, ldk) or nullptr: all 1
    float *dweights;       // (k, ldk) or nullptr
    int64_t ldk;
    float *partial;        // [row groups * batch * k]
    int32_t features, experts, batch, k, capacity;
    Placement p;
};
// Rows of the operands that one work-group moves: as many as leave the GPU two work-groups per compute unit.
inline int32_t move_rows(int32_t features, int64_t tiles, int32_t most)
{
    int32_t rows = most;
    while (rows > 4 && (features + rows - 1) / rows * tiles < 512) rows /= 2;
    return rows;
}
// The fewest that the combine's backward pass takes, whose products over so many rows make one entry of `partial`: the workspace is asked for without
// the experts, and with them there may be more tiles.
inline int32_t partial_rows(int32_t features, int32_t batch) { return move_rows(features, (batch + kPlaceTileMax - 1) / kPlaceTileMax, 16); }
// work-groups that form the gradients of the weights, one for 64 choices
constexpr int32_t kGradThreads = 512;
inline int64_t weight_gradient_blocks(int32_t batch, int32_t k) { return (static_cast<int64_t>(batch) * k + 63) / 64; }
hipError_t launch_dispatch(const ExchangeArgs &a, hipStream_t s);
hipError_t launch_combine(const ExchangeArgs &a, hipStream_t s);
hipError_t launch_combine_backward(const ExchangeArgs &a, hipStream_t s);

// ---- norm over many arrays (clip.hip) -------------------------------------------------------
constexpr int32_t kNormList = 192;           // arrays per launch that adds up squares
constexpr int32_t kNormBlocks = 1024;        // its work-groups, at most, each of which leaves a sum
inline int64_t norm_workspace_bytes(int64_t arrays) { return (8 * (kNormBlocks * ((arrays + kNormList - 1) / kNormList + 1) + 1) + 255) / 256 * 256; }

struct ArrayList {
    int32_t n;
    float *const *values;            // updated arrays, or nullptr
    float *const *velocities;
    const float *const *grads;
    float *const *clipped;           // scaled gradients, or nullptr
    const int64_t *counts;
};
struct ClipArgs {
    float lr, momentum, max_norm;
    int32_t nesterov;
    double *partial;
    float *norm_out;                 // or nullptr
};
hipError_t launch_norm(const ArrayList &l, double *partial, float *norm_out, hipStream_t s);
// the norm, then the momentum step (l.values) or the scaled gradients (l.clipped)
hipError_t launch_clipped(const ArrayList &l, const ClipArgs &c, hipStream_t s);

}  // namespace nerva
