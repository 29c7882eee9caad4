// Launch arguments of the page table kernels.
#pragma once

#include <stdint.h>

#include "fate.h"

namespace fate {

struct PagesLaunch {
    const int32_t *counts;  // reserve: new tokens, trim: keys that stay
    const int32_t *kv_len, *n_free;
    int32_t *pages, *free;
    int32_t *off, *kv_out, *n_free_out, *moved;  // moved: pages taken or given, summed
    int64_t *slots;
    int32_t *positions, *status;
    int64_t T, pages_stride, max_keys;
    int32_t B, n_pages, shift;
};
int launch_reserve(const PagesLaunch &a, void *stream);
int launch_trim(const PagesLaunch &a, void *stream);

constexpr int64_t kReserveSmall = 4096;
constexpr int32_t kTrimSmall = 512;

}  // namespace fate
