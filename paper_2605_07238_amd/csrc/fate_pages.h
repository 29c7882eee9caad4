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

// Calls of one workgroup and one launch: rows of a reserve, sequences of a trim.
// A launch more costs the host 2 us; one workgroup needs 6.9 us for 512 rows and
// 9.9 for 4096, of 64 sequences (8192 rows in two launches 10.3), and for trims of
// 256, 512 and 1024 sequences 9, 14 and 26 us, where three launches take 7.5 to 8
// and their host 15 (of one launch 10).
constexpr int64_t kReserveSmall = 4096;
constexpr int32_t kTrimSmall = 512;

}  // namespace fate
