// What the files of qless_token_loss share.
#pragma once
#include "common.h"

namespace qless {

// What follows from a token's greatest logit, the sum of exp(z - top) over the entries other than its target, and the target's logit.  With
// the target's 1 in the sum, a loss would be rounded to steps of 2^-23, and 1 - p_target with it; apart from it, both keep their digits.
struct TokenResult { float nll, lse, scale, pull; };        // scale, pull: of the others' sum of exp(z - top) W, and of W_target, in dH
__device__ inline TokenResult token_result(float top, float others, float hit, float weight) {
    const float mine = __expf(hit - top), total = others + mine, scale = weight / total;
    return TokenResult{others < mine ? log1pf(others / mine) : logf(total) + (top - hit), top + logf(total), scale, -scale * others};
}
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
