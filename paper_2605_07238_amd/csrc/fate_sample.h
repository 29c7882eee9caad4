// Launch arguments of the sampling kernel.
#pragma once

#include <stdint.h>

#include "fate.h"

namespace fate {

struct SampleLaunch {
    const char *logits;
    const float *u, *temperature, *top_p, *min_p;  // per row; null: the value for all
    const int32_t *top_k;
    int32_t *token, *status;
    float *logprob;
    int64_t stride;  // elements
    int32_t rows, vocab, dtype;
    int32_t top_k_all;
    float temperature_all, top_p_all, min_p_all;
};
int launch_sample(const SampleLaunch &a, void *stream);

}  // namespace fate
