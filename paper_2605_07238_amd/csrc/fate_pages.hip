// Page tables of the key-value cache on the device: pages for new tokens off
// the stack of free ones, and back on it when a sequence is cut.
//
//   reserve  need_b = ceil((kv_b + new_b) / P) - ceil(kv_b / P); x_b, y_b = the
//            sums of need and new up to b.  b is served if it needs no page or
//            x_b <= n_free, and y_b <= T.  Both sums grow, so that of two
//            sequences that need pages the earlier is served if the later is:
//            the pages of those served lie on the stack without gaps.
//   trim     the pages past ceil(min(keep, kv) / P) go on the stack, in order.
//
// Latency bounds both: an answer's step moves a few kilobytes.  One workgroup
// adds the lengths up, 1024 sequences a step, and in small calls does the rest
// too, in the same launch; in others a second launch spreads what is left over
// the chip.  Nothing is kept between the launches but the call's results, so
// that lengths and counts may be updated in place, which a grid that reads
// them in every workgroup could not.
#include "fate_attn.h"
#include "fate_pages.h"

namespace fate {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kStaged = 2048;  // sequences that fit LDS

struct Scans {
    int64_t a[kWaves], b[kWaves];
};

// Inclusive sums over the workgroup's threads, of two values in the same steps.
__device__ __forceinline__ void block_scan2(int64_t &x, int64_t &y, Scans &s, int64_t &all_x, int64_t &all_y) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    x = wave_scan_add(x);
    y = wave_scan_add(y);
    if (lane == 63) s.a[w] = x, s.b[w] = y;
    __syncthreads();
    int64_t before_x = 0, before_y = 0;
    all_x = all_y = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i < w) before_x += s.a[i], before_y += s.b[i];
        all_x += s.a[i], all_y += s.b[i];
    }
    x += before_x;
    y += before_y;
    __syncthreads();
}

// Inclusive sums over the workgroup's threads; `before` holds kWaves entries.
template <class I>
__device__ __forceinline__ I block_scan(I x, I *before, I &total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const I in_wave = wave_scan_add(x);
    if (lane == 63) before[w] = in_wave;
    __syncthreads();
    I sum = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i < w) sum += before[i];
        total += before[i];
    }
    __syncthreads();
    return sum + in_wave;
}

// Of each sequence, where rows are placed: its first row, its keys before the
// call, and the pages taken before it.
struct Staged {
    int off[kStaged + 1], old[kStaged], taken[kStaged];
};

__device__ __forceinline__ int pages_for(int64_t keys, int shift) {
    return (int)((keys + (1 << shift) - 1) >> shift);
}

// A count of free pages that no stack can hold counts as none.
__device__ __forceinline__ int free_pages(const PagesLaunch &a) {
    const int n = *a.n_free;
    return n >= 0 && n <= a.n_pages ? n : 0;
}

// Lengths of all sequences: off, kv_out, taken, status and n_free_out; in LDS too
// if `staged` is given.  Returns the rows of the call.
__device__ __forceinline__ int reserve_lengths(const PagesLaunch &a, Scans &lds, Staged *staged) {
    const int tid = threadIdx.x, stack = *a.n_free, n_free = free_pages(a);
    int64_t asked = 0, rows = 0, done = 0;  // before this step; done: rows and pages given, in the halves of a word
    for (int64_t at = 0; at < a.B; at += kThreads) {
        const int64_t b = at + tid;
        int64_t fresh_tokens = 0, kv = 0;
        bool good = false;
        if (b < a.B) {
            fresh_tokens = a.counts[b];
            kv = a.kv_len[b];
            good = fresh_tokens >= 0 && kv >= 0 && kv + fresh_tokens <= a.max_keys;
            if (!good) fresh_tokens = 0;
        }
        const int need = good ? pages_for(kv + fresh_tokens, a.shift) - pages_for(kv, a.shift) : 0;
        int64_t all_pages, all_rows, all_done;
        int64_t x = need, y = fresh_tokens;
        block_scan2(x, y, lds, all_pages, all_rows);
        const bool fits = (need == 0 || asked + x <= n_free) && rows + y <= a.T;
        const int64_t mine = fits ? fresh_tokens << 32 | need : 0;  // rows are at most T, pages at most n_free
        const int64_t upto = done + block_scan(mine, lds.a, all_done);
        if (b < a.B) {
            if (staged) {
                staged->off[b + 1] = (int)(upto >> 32);
                staged->old[b] = (int)kv;
                staged->taken[b] = (int)upto - (fits ? need : 0);
            }
            a.off[b + 1] = (int)(upto >> 32);
            a.moved[b + 1] = (int)upto;
            a.kv_out[b] = (int)(fits ? kv + fresh_tokens : kv);
            if (a.status && !(good && fits)) a.status[b] = good ? FATE_ESIZE : FATE_EINVAL;
        }
        asked += all_pages;
        rows += all_rows;
        done += all_done;
    }
    if (tid == 0) {
        if (staged) staged->off[0] = 0;
        a.off[0] = a.moved[0] = 0;
        *a.n_free_out = stack - (int)done;
    }
    return (int)(done >> 32);
}

// Rows [from, to): their positions, slots, and the pages that start with them;
// `end` rows are in the call, and `stack` pages were free before it.
template <class Old, class Taken>
__device__ __forceinline__ void reserve_rows(const PagesLaunch &a, const int *off, Old old_of, Taken taken_of, int stack,
                                             int64_t end, int64_t from, int64_t to) {
    for (int64_t t = from + threadIdx.x; t < to; t += blockDim.x) {
        int64_t slot = -1;
        int pos = -1;
        if (t < end) {
            int lo = 0, hi = a.B - 1;  // the last sequence that starts at t or before, which has rows: its end is past t
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (off[mid + 1] <= t) lo = mid + 1;
                else hi = mid;
            }
            const int start = off[lo], old = old_of(lo);
            pos = old + (int)(t - start);
            const int j = pos >> a.shift, have = pages_for(old, a.shift), in_page = pos & ((1 << a.shift) - 1);
            int32_t *const entry = a.pages + lo * a.pages_stride + j;
            int page;
            if (j >= have) {
                page = a.free[stack - 1 - taken_of(lo) - (j - have)];
                if (in_page == 0) *entry = page;
            } else {
                page = *entry;
            }
            if ((uint32_t)page < (uint32_t)a.n_pages) slot = ((int64_t)page << a.shift) + in_page;
            else if (a.status) a.status[lo] = FATE_EINVAL;
        }
        if (a.slots) a.slots[t] = slot;
        if (a.positions) a.positions[t] = pos;
    }
}

__global__ __launch_bounds__(kThreads) void k_kv_reserve(PagesLaunch a) {
    __shared__ Scans lds;
    reserve_lengths(a, lds, nullptr);
}

// Small calls: with the rows, from LDS.  (Read back from memory, what the scan
// has written costs two round trips more: 8.0 against 7.0 us for 64 sequences.)
__global__ __launch_bounds__(kThreads) void k_kv_reserve_small(PagesLaunch a) {
    __shared__ Scans lds;
    __shared__ Staged s;
    const int stack = *a.n_free;
    const int end = reserve_lengths(a, lds, &s);
    __syncthreads();
    reserve_rows(a, s.off, [&](int b) { return s.old[b]; }, [&](int b) { return s.taken[b]; }, stack, end, 0, a.T);
}

constexpr int kRowsPer = 1024;  // rows of a workgroup of the second launch

template <bool STAGED>
__global__ __launch_bounds__(256) void k_kv_rows(PagesLaunch a) {
    __shared__ int in_lds[STAGED ? kStaged + 1 : 1];
    const int64_t from = (int64_t)blockIdx.x * kRowsPer, to = min(from + kRowsPer, a.T);
    const int *off = a.off;
    const int end = a.B ? a.off[a.B] : 0, stack = *a.n_free_out + a.moved[a.B];
    if (STAGED) {
        for (int i = threadIdx.x; i <= a.B; i += 256) in_lds[i] = a.off[i];
        __syncthreads();
        off = in_lds;
    }
    reserve_rows(a, off, [&](int b) { return a.kv_out[b] - (off[b + 1] - off[b]); }, [&](int b) { return a.moved[b]; }, stack,
                 end, from, to);
}

// Pages `left` to `have` of a sequence, which it gives back: none of them if
// lengths are in error (have < 0) or, where a wave has looked, a page.
struct Given {
    int left, have;
};
__device__ __forceinline__ Given given_by(const PagesLaunch &a, int64_t b) {
    const int kv = a.kv_len[b], keep = a.counts[b];
    if (kv < 0 || keep < 0 || kv > a.max_keys) return {0, -1};
    return {pages_for(min(kv, keep), a.shift), pages_for(kv, a.shift)};
}
// f(j, page j) for the pages, by LANES neighbouring threads, LOADS of each asked for at once.
template <int LANES, int LOADS, class F>
__device__ __forceinline__ void each_page(const PagesLaunch &a, int64_t b, Given x, F f) {
    const int32_t *const row = a.pages + b * a.pages_stride;
    for (int j = x.left + (int)(threadIdx.x & (LANES - 1)); j < x.have; j += LANES * LOADS) {
        int page[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) page[i] = j + LANES * i < x.have ? row[j + LANES * i] : 0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if (j + LANES * i < x.have) f(j + LANES * i, page[i]);
    }
}
// How many pages a sequence gives back, -1 if it is in error.  (All lanes of the wave come here.)
template <int LANES, int LOADS>
__device__ __forceinline__ int gone_of(const PagesLaunch &a, int64_t b, Given x) {
    bool bad = x.have < 0;
    each_page<LANES, LOADS>(a, b, x, [&](int, int page) { bad = bad || (uint32_t)page >= (uint32_t)a.n_pages; });
    const uint64_t who = __ballot(bad) >> (threadIdx.x & 63 & -LANES);
    return (LANES < 64 ? who & ((1ull << LANES % 64) - 1) : who) ? -1 : x.have - x.left;
}

// Of the sequences of a small call: what each gives back, and the sum up to it.
struct Trimmed {
    Given given[kTrimSmall];
    int gone[kTrimSmall], upto[kTrimSmall];
};

// Sums over gone(b), what the sequences give back: moved, kv_out, status, n_free_out; in LDS
// too if `staged` is given.
template <class Gone>
__device__ __forceinline__ void trim_lengths(const PagesLaunch &a, Scans &lds, Gone gone_by, Trimmed *staged) {
    const int tid = threadIdx.x, stack = *a.n_free;
    const bool known = stack >= 0 && stack <= a.n_pages;
    int64_t asked = 0, done = 0;
    for (int64_t at = 0; at < a.B; at += kThreads) {
        const int64_t b = at + tid;
        const int gone = b < a.B ? gone_by(b) : 0;
        int64_t all, all_done;
        const int64_t x = asked + block_scan((int64_t)max(gone, 0), lds.a, all);
        const bool fits = gone == 0 || (gone > 0 && known && stack + x <= a.n_pages);
        const int64_t upto = done + block_scan((int64_t)(fits ? gone : 0), lds.b, all_done);
        if (b < a.B) {
            a.moved[b + 1] = (int)upto;
            if (staged) staged->upto[b] = (int)upto, staged->gone[b] = fits ? gone : 0;
            const int kv = a.kv_len[b];
            a.kv_out[b] = fits ? min(kv, a.counts[b]) : kv;
            if (a.status && !fits) a.status[b] = FATE_EINVAL;
        }
        asked += all;
        done += all_done;
    }
    if (tid == 0) {
        a.moved[0] = 0;
        *a.n_free_out = stack + (int)done;
    }
}

// A call of one workgroup, sixteen lanes a sequence.  The lengths are read once, by
// threads, and pages eight loads at a time: 200 sequences with up to 512 pages
// took 14.4 us by a wave each with a lane's loads one behind the other, 11.3 with
// four at a time, 8.2 so.
__global__ __launch_bounds__(kThreads) void k_kv_trim(PagesLaunch a) {
    constexpr int kLanes = 16, kLoads = 8;
    __shared__ Scans lds;
    __shared__ Trimmed s;
    const int mine = threadIdx.x / kLanes, stack = *a.n_free;
    if ((int)threadIdx.x < a.B) s.given[threadIdx.x] = given_by(a, threadIdx.x);
    __syncthreads();
    for (int at = 0; at < a.B; at += kThreads / kLanes) {
        const int b = at + mine;
        const int gone = gone_of<kLanes, kLoads>(a, b, b < a.B ? s.given[b] : Given{0, 0});
        if (b < a.B && threadIdx.x % kLanes == 0) s.gone[b] = gone;
    }
    __syncthreads();
    trim_lengths(a, lds, [&](int64_t b) { return s.gone[b]; }, &s);
    __syncthreads();
    for (int b = mine; b < a.B; b += kThreads / kLanes) {
        if (s.gone[b] <= 0) continue;
        int32_t *const to = a.free + stack + s.upto[b] - s.gone[b] - s.given[b].left;
        each_page<kLanes, kLoads>(a, b, s.given[b], [&](int j, int page) { to[j] = page; });
    }
}

// The three steps of a large call.
__global__ __launch_bounds__(256) void k_kv_trim_counts(PagesLaunch a) {
    for (int64_t b = blockIdx.x * 4 + (threadIdx.x >> 6); b < a.B; b += gridDim.x * 4) {
        const int gone = gone_of<64, 4>(a, b, given_by(a, b));
        if ((threadIdx.x & 63) == 0) a.moved[b + 1] = gone;
    }
}
__global__ __launch_bounds__(kThreads) void k_kv_trim_lengths(PagesLaunch a) {
    __shared__ Scans lds;
    trim_lengths(a, lds, [&](int64_t b) { return a.moved[b + 1]; }, nullptr);
}
__global__ __launch_bounds__(256) void k_kv_trim_pages(PagesLaunch a) {
    const int stack = *a.n_free_out - a.moved[a.B];
    for (int64_t b = blockIdx.x * 4 + (threadIdx.x >> 6); b < a.B; b += gridDim.x * 4) {
        const int from = a.moved[b], n = a.moved[b + 1] - from, left = pages_for(a.kv_out[b], a.shift);
        int32_t *const to = a.free + stack + from - left;
        if (n) each_page<64, 4>(a, b, {left, left + n}, [&](int j, int page) { to[j] = page; });
    }
}

}  // namespace

int launch_reserve(const PagesLaunch &a, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (a.B <= kStaged && a.T <= kReserveSmall) {
        hipLaunchKernelGGL(k_kv_reserve_small, dim3(1), dim3(kThreads), 0, s, a);
        return (int)hipGetLastError();
    }
    hipLaunchKernelGGL(k_kv_reserve, dim3(1), dim3(kThreads), 0, s, a);
    const dim3 grid((unsigned)((a.T + kRowsPer - 1) / kRowsPer));
    if (grid.x > 0 && a.B <= kStaged) hipLaunchKernelGGL((k_kv_rows<true>), grid, dim3(256), 0, s, a);
    else if (grid.x > 0) hipLaunchKernelGGL((k_kv_rows<false>), grid, dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

int launch_trim(const PagesLaunch &a, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (a.B <= kTrimSmall) {
        hipLaunchKernelGGL(k_kv_trim, dim3(1), dim3(kThreads), 0, s, a);
        return (int)hipGetLastError();
    }
    const unsigned groups = (unsigned)((a.B + 3) / 4 < 1024 ? (a.B + 3) / 4 : 1024);
    hipLaunchKernelGGL(k_kv_trim_counts, dim3(groups), dim3(256), 0, s, a);
    hipLaunchKernelGGL(k_kv_trim_lengths, dim3(1), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(k_kv_trim_pages, dim3(groups), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

}  // namespace fate
