// What the files of qless_token_loss share.
#pragma once
#include "common.h"

namespace qless {

// near 0 the loss keeps its digits
__device__ inline float loss_of(float top, float sum, float hit) { return logf(sum) + (top - hit); }
// Maximum and sum (relative to it) joined with another such pair.
__device__ inline void join_pair(float &top, float &sum, float top2, float sum2) {
    const float next = fmaxf(top, top2);
    if (next == -INFINITY) sum += sum2;                     // 0, or NaN of logits that are not numbers
    else sum = sum * __expf(top - next) + sum2 * __expf(top2 - next);
    top = next;
}

// token_loss_single.hip: the loss (and dH) of at most four tokens, in one pass over W, whose rows are whole 16-byte chunks.
bool single_serves(int64_t T, int32_t D, int32_t V, bool want_dH);
size_t single_workspace(int64_t T, int32_t D, int32_t V, bool want_dH);
qless_status launch_single(const uint16_t *H, int64_t ldH, const uint16_t *W, int64_t ldW, int T, int32_t D, int32_t V, const int64_t *target,
                           const float *weight, float *nll, float *lse, uint16_t *dH, int64_t ldDH, void *ws, hipStream_t st);

}  // namespace qless
