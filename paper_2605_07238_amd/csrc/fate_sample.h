// Launch arguments of the sampling kernel.
#pragma once

#include <stddef.h>
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
    // calls of few rows, by slices of each: of each slice the largest entry, the complement of the threads' least key,
    // the sums by bins or by waves, those over the cut by waves and in all, what is listed, the threads' largest logits;
    // of each row the sum of all, the bin of the cut and the lowest logit in question
    int32_t slices;
    unsigned long long *tops, *lows, *hist, *lists;
    double *parts, *kept, *over, *wholes;
    float *best, *bottoms;
    int32_t *counts, *cuts;
};
size_t sample_ws(int64_t rows, int64_t vocab);  // bytes
int launch_sample(const SampleLaunch &a, void *ws, void *stream);

}  // namespace fate
