// Internal declarations of the 8-bit proposal path: codes, logits, sampling.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "logits_fp8_geo.h"
#include "route.h"

namespace dcd {

struct QuantProblem {
    long long rows;
    int cols, groups;  // groups = ceil(cols / kGroup)
    int dtype, block_rows;
    const void *x;
    uint8_t *q;
    float *scale;
};

hipError_t launch_quantize(const QuantProblem &p, hipStream_t st);

struct Fp8Problem {
    int M, N, K, groups;  // rows, vocabulary, hidden size, ceil(K / kGroup)
    int dtype;            // of the logits
    long long stride;     // elements from one row of logits to the next
    const uint8_t *h, *w;
    const float *hs, *ws, *bias;
    void *out;
};

hipError_t launch_logits_fp8(const Fp8Problem &p, hipStream_t st);
hipError_t launch_logits_tile(const Fp8Problem &p, hipStream_t st);  // more than 64 rows

struct SampleProblem {
    int R, V, dtype;
    long long stride;
    const void *logits;
    const float *u, *temperature, *top_p, *min_p;  // the rules may be null: off
    const int32_t *top_k;
    int32_t *tokens, *kept;
    float *probs, *logprob;
};

size_t sample_workspace(const SampleProblem &p);
hipError_t launch_sample(const SampleProblem &p, void *ws, hipStream_t st);

}  // namespace dcd
