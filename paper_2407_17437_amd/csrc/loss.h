// Internal launch interface between the C ABI (api.hip) and the kernels of label log-probabilities and of the losses on them (loss.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nerva {

// What a column of logits leaves for the gradient: dZ[i] = c [i == label] - share * exp(Z[i] - top), share = c / (sum of exp(Z - top)); 0 where c is 0.
struct ColumnState {
    float top, share, c;
    int32_t label;
};

struct LossArgs {
    const float *Z;
    int64_t ldz;
    const int32_t *labels;
    int32_t classes, batch, sequences;   // sequences: of which starts holds the first columns and the end of the last
    const int32_t *starts;               // [sequences + 1] or nullptr
    float *logp;                         // [batch] or nullptr
    float *sums;                         // [sequences] or nullptr
    // policy
    const float *old_logp, *ref_logp, *advantages, *weights;
    float clip_low, clip_high;
    float *stats;                        // [4]
    // preference
    const float *ref_sums;               // [sequences] or nullptr
    float smoothing;
    float *margins;                      // [sequences / 2] or nullptr
    float *loss;                         // [1] or nullptr
    float beta;                          // of the KL term, or of the margin
    float *dZ;
    int64_t lddz;
    void *workspace;
};
// parts of a workspace (which may be nullptr, for its size)
struct LossSpace {
    double *logp;            // [batch]
    double *shares;          // [4 * blocks]: of the loss, per work-group of columns or per pair
    ColumnState *columns;    // [batch]
    float *partial;          // [chunks][top, sum][batch]
    int64_t bytes;
};
LossSpace loss_space(void *memory, int32_t classes, int32_t batch, int32_t sequences);

hipError_t launch_log_probs(const LossArgs &a, hipStream_t s);
hipError_t launch_policy(const LossArgs &a, hipStream_t s);
hipError_t launch_preference(const LossArgs &a, hipStream_t s);

}  // namespace nerva
