// What the lists of the largest words (toplogits.cu) and the log probabilities of tokens (logprobs.cu) share.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace lda {

struct TopArgs {
    const void* logits;
    int64_t stride;
    int32_t V, top;
    float scale;     // log2(e) / temperature
    double inv_tau;
    int32_t* ids;
    void* values;
    float* lse;
    int ring;  // bytes of the walk's ring, or of the lists that take its place
    // log probabilities and entropies (logprobs.cu): then instead of values and lse
    const int32_t* tokens;
    float *logprobs, *entropy, *stats, *alternatives;
};

// Rows' lists with log probabilities in the values' place, and what logprobs.cu says of rows without lists.
cudaError_t top_logprobs(const TopArgs& a, int dtype, int64_t rows, cudaStream_t st);

}  // namespace lda
