// Device state of a scorer handle and its launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rheo {

struct ScoreDev {
    int V, dtype;
    int64_t stride;
    char* work;                    // partial results of split rows (score_workspace() bytes)
};

struct LogprobArgs {
    const char* logits;
    int B, n, m, top;
    const int32_t *path, *token;
    float kT, T;                   // log2(e) / T, T
    float *logprob, *entropy;
    int32_t *rank, *top_token;
    float* top_logprob;
};

size_t score_workspace();
hipError_t launch_token_logprobs(const ScoreDev& c, const LogprobArgs& a, hipStream_t s);

}  // namespace rheo
