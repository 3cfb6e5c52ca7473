// Log probabilities of tokens: what the host glue hands to the kernel.
#pragma once
#include "essa_internal.h"

namespace essa_k {

constexpr int kLogprobSegment = 128;       // values whose largest is kept for finding the largest ones of a row
constexpr int kLogprobMostTop = ESSA_LOGPROB_MAX_TOP;
constexpr int kLogprobSplitRows = 512;     // calls of fewer rows share a row among workgroups; as many counts
// Each in memory of its own: counts next to one another are one place to the memory that all XCDs' atomics go to, and 64 parts of 64 rows took 39 us
// instead of 11.
constexpr int kLogprobCountStep = 64;

struct logprob_args {
    const void* logits;
    long long stride;          // in values
    int V, n_tokens, n_top;
    float scale, k;            // k = scale log2(e)
    const int32_t* tokens;     // [R, n_tokens]
    float *logp, *entropy;     // [R, n_tokens], [R] or null
    int32_t* top_ids;          // [R, n_top]
    float* top_logp;
    // set by the launcher
    int parts;                 // workgroups a row
    int row_segments;
    int32_t* done;             // [kLogprobSplitRows, kLogprobCountStep] the first of each: finished parts of a row; 0 between calls
    float *sums, *segments;    // [R, parts, 4] and [R, row_segments]
};
size_t token_logprobs_bytes(int R, int V, int x_dtype, int n_top);
hipError_t token_logprobs(hipStream_t st, logprob_args a, int x_dtype, int R, int32_t* done, void* ws);

}  // namespace essa_k
