// One token of each row of logits, from a given random number.
//
//   w_i = exp((l_i - max l) / temperature); of the tokens by falling logit (equal
//   ones by rising index), the first top_k; of these those before which less than
//   top_p of their sum lies; of these those with w_i >= min_p.  The token is the
//   lowest i with sum of w_j over the kept j <= i greater than u W, W the sum of
//   all kept.  What is kept is a stretch of that order from its start, so one
//   place in it, a key and an index, says which tokens are kept.
//
// Everything that a token hangs on is computed in 64 bits: between two
// neighbours of 100000 tokens lies 1e-5 of W, and a sum that is off by 2^-24
// would pick another one in every hundredth row.  Sums have a fixed order, and
// where atomics add they add whole numbers: two calls give the same token.
//
// k_sample: one workgroup per row.  It reads the row once for its largest
// logit.  Where few tokens can be kept (few tokens at all, a small top_k, a min_p
// without top_p) a second reading gathers them into LDS, where they are
// ranked, cut, put back in order and summed.  The bound for top_k is the k-th
// largest of the threads' own largest logits: at least k tokens reach it, and
// hardly more do.  Where the gathered do not fit, and for top_p over all tokens,
// the place of the cut is found by its digits (11, 11 and 10 bits of the key),
// each by a histogram, of counts or of weights as whole numbers; then two
// readings find the token, of which the second is of a sixteenth of the row.
#include <hip/hip_runtime.h>

#include "fate_sample.h"

namespace fate {
namespace {

typedef unsigned long long u64;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kList = 4096;   // tokens that are ranked in LDS
constexpr int kSmallK = 1024; // largest top_k that the threads' largest logits bound
constexpr int kBins = 2048;

struct Lds {
    u64 list[kList];
    u64 hist[kBins];
    u64 whole[kWaves];
    double real[kWaves];
    uint32_t word[kWaves];
    int count, found, sub;
    u64 above, in_bin;
    double rest, weight;
};

// Keys: whole numbers in the order of the logits.  0 is no token: NaN, -infinity
// and places outside the row.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (!(x > -INFINITY)) return 0;
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);  // -0 is 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

struct F32 {
    static constexpr int kPer = 4;
    static __device__ __forceinline__ float get(const u32x4 &x, int e) {
        const uint32_t w = x[e];  // (a cast of the vector's element itself takes the first one's bits)
        return __builtin_bit_cast(float, w);
    }
    static __device__ __forceinline__ float at(const char *p, int64_t i) { return ((const float *)p)[i]; }
    static constexpr int kBytes = 4;
};
struct B16 {
    static constexpr int kPer = 8;
    static __device__ __forceinline__ float get(const u32x4 &x, int e) {
        const uint32_t w = x[e / 2];
        return __builtin_bit_cast(float, e & 1 ? w & 0xffff0000u : w << 16);
    }
    static __device__ __forceinline__ float at(const char *p, int64_t i) {
        return __builtin_bit_cast(float, (uint32_t)((const uint16_t *)p)[i] << 16);
    }
    static constexpr int kBytes = 2;
};
struct H16 {
    static constexpr int kPer = 8;
    static __device__ __forceinline__ float get(const u32x4 &x, int e) {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(x[e / 2] >> (e & 1) * 16));
    }
    static __device__ __forceinline__ float at(const char *p, int64_t i) { return (float)((const _Float16 *)p)[i]; }
    static constexpr int kBytes = 2;
};

// A row in pieces of 16 aligned bytes, numbered from that of its first element;
// the first and last may reach over its ends, and are read element by element.
template <class T>
struct Row {
    const char *data;
    int V, lead, pieces;  // lead: places of the first piece before the row

    __device__ __forceinline__ Row(const SampleLaunch &a, int row) {
        data = a.logits + (int64_t)row * a.stride * T::kBytes;
        V = a.vocab;
        lead = (int)((uintptr_t)data % 16) / T::kBytes;
        pieces = (int)(((int64_t)V + lead + T::kPer - 1) / T::kPer);
    }
    // Index of the piece's first element, and its keys.
    __device__ __forceinline__ int keys(int piece, uint32_t (&k)[T::kPer]) const {
        const int i0 = piece * T::kPer - lead;
        if (i0 >= 0 && i0 + T::kPer <= V) {
            const u32x4 x = *(const u32x4 *)(data + (int64_t)i0 * T::kBytes);
#pragma unroll
            for (int e = 0; e < T::kPer; ++e) k[e] = key_of(T::get(x, e));
        } else {
#pragma unroll
            for (int e = 0; e < T::kPer; ++e) {
                const int i = i0 + e;
                k[e] = i >= 0 && i < V ? key_of(T::at(data, i)) : 0;
            }
        }
        return i0;
    }
};

// f(key, index) for the tokens of pieces from + lane, from + lane + step ..
template <class T, class F>
__device__ __forceinline__ void each(const Row<T> &row, int from, int to, int step, F f) {
    for (int p = from; p < to; p += step) {
        uint32_t k[T::kPer];
        const int i0 = row.keys(p, k);
#pragma unroll
        for (int e = 0; e < T::kPer; ++e)
            if (k[e]) f(k[e], i0 + e);
    }
}

// e^z for z <= 0 to some 2^-52: z = n ln 2 + x with |x| <= ln 2 / 2, and the
// series of e^x to x^13 / 13! (the next term is 2^-57 of it).
__device__ __forceinline__ double exp_of(double z) {
    z = fmax(z, -800.0);  // 0 from -745 on
    const double n = __builtin_rint(z * 1.4426950408889634074);
    const double x = __builtin_fma(n, -0.69314718055994530942, z);
    double f = 1.0 / 6227020800.0;
    f = __builtin_fma(f, x, 1.0 / 479001600.0);
    f = __builtin_fma(f, x, 1.0 / 39916800.0);
    f = __builtin_fma(f, x, 1.0 / 3628800.0);
    f = __builtin_fma(f, x, 1.0 / 362880.0);
    f = __builtin_fma(f, x, 1.0 / 40320.0);
    f = __builtin_fma(f, x, 1.0 / 5040.0);
    f = __builtin_fma(f, x, 1.0 / 720.0);
    f = __builtin_fma(f, x, 1.0 / 120.0);
    f = __builtin_fma(f, x, 1.0 / 24.0);
    f = __builtin_fma(f, x, 1.0 / 6.0);
    f = __builtin_fma(f, x, 0.5);
    f = __builtin_fma(f, x, 1.0);
    f = __builtin_fma(f, x, 1.0);
    return __builtin_ldexp(f, (int)n);
}

// Weight of a key below the largest one.
struct Weight {
    uint32_t top;
    double max, per;  // 1 / temperature
    __device__ __forceinline__ double operator()(uint32_t key) const {
        return key == top ? 1.0 : exp_of(((double)value_of(key) - max) * per);
    }
};

// The least whole number that is p * n or more, p in (0, 1], 1 <= n < 2^63.
__device__ __forceinline__ u64 share_of(float p, u64 n) {
    const uint32_t b = __builtin_bit_cast(uint32_t, p), e = b >> 23;
    const unsigned __int128 x = (unsigned __int128)n * (e ? (b & 0x7fffffu) | 0x800000u : b);
    const int shift = 150 - (int)(e ? e : 1);  // p = mantissa / 2^shift
    if (shift > 90) return 1;
    return (u64)((x + (((unsigned __int128)1 << shift) - 1)) >> shift);
}

// The kept tokens: those over a place in the order.
struct Place {
    uint32_t key;
    int index;
    __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= index); }
};
constexpr int kAll = 0x7fffffff;

__device__ __forceinline__ double wave_add(double x) {
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) x += __shfl_xor(x, i);
    return x;
}
template <class I>
__device__ __forceinline__ I wave_upto(I x) {  // sums up to and with this lane
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const I y = __shfl_up(x, i);
        if (lane >= i) x += y;
    }
    return x;
}
// Sums up to and with this thread, and of all.
template <class I>
__device__ __forceinline__ I block_upto(I x, I (&part)[kWaves], I &total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    x = wave_upto(x);
    if (lane == 63) part[w] = x;
    __syncthreads();
    I before = 0;
    total = 0;
    for (int i = 0; i < kWaves; ++i) {
        if (i < w) before += part[i];
        total += part[i];
    }
    __syncthreads();
    return before + x;
}

__device__ __forceinline__ u64 block_max(u64 x, Lds &s) {
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const u64 y = __shfl_xor(x, i);
        x = y > x ? y : x;
    }
    if ((threadIdx.x & 63) == 0) s.whole[threadIdx.x >> 6] = x;
    __syncthreads();
    for (int i = 0; i < kWaves; ++i) x = s.whole[i] > x ? s.whole[i] : x;
    __syncthreads();
    return x;
}

// The list's first n entries (n at most kList) by falling value, pair by pair
// in a bitonic network: up to 64 in one wave's registers, more in LDS.
__device__ void sort_list(Lds &s, int n) {
    const int tid = threadIdx.x;
    if (n <= 64) {
        if (tid < 64) {
            u64 x = tid < n ? s.list[tid] : 0;
#pragma unroll
            for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
                for (int d = size >> 1; d > 0; d >>= 1) {
                    const u64 y = __shfl_xor(x, d);
                    const bool larger = ((tid & size) == 0) == ((tid & d) == 0);  // this lane keeps the larger one
                    x = (y > x) == larger ? y : x;
                }
            if (tid < n) s.list[tid] = x;
        }
        __syncthreads();
        return;
    }
    int all = 128;
    while (all < n) all <<= 1;
    for (int i = n + tid; i < all; i += kThreads) s.list[i] = 0;
    __syncthreads();
    for (int size = 2; size <= all; size <<= 1)
        for (int d = size >> 1; d > 0; d >>= 1) {
            for (int x = tid; x < all / 2; x += kThreads) {
                const int i = 2 * x - (x & (d - 1)), j = i + d;
                const u64 a = s.list[i], b = s.list[j];
                if ((a < b) == ((i & size) == 0)) {
                    s.list[i] = b;
                    s.list[j] = a;
                }
            }
            __syncthreads();
        }
}

// The k-th largest of the threads' words (1 <= k <= kThreads), by digits of eight bits.
__device__ uint32_t kth_word(Lds &s, uint32_t mine, int k) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    int left = k;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) s.hist[tid] = 0;
        __syncthreads();
        if (shift == 24 || mine >> (shift + 8) == prefix) atomicAdd(&s.hist[mine >> shift & 255u], 1ull);
        __syncthreads();
        u64 total;
        const u64 has = tid < 256 ? s.hist[255 - tid] : 0;
        const u64 upto = block_upto(has, s.whole, total);
        if (has && upto >= (u64)left && upto - has < (u64)left) {
            s.found = 255 - tid;
            s.above = upto - has;
        }
        __syncthreads();
        prefix = prefix << 8 | (uint32_t)s.found;
        left -= (int)s.above;
        __syncthreads();
    }
    return prefix;
}

// Of the tokens that `kept` keeps, each of `size(key)`: the key at which the
// sizes of the tokens with this key or a larger one reach aim(sum of all); how
// many of this key that takes, and how many there are.
template <class T, class Size, class Aim>
__device__ uint32_t key_at(Lds &s, const Row<T> &row, const Place &kept, Size size, Aim aim, u64 &need, u64 &have) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    u64 above = 0, in_bin = 0, target = 0;
    for (int level = 0; level < 3; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
        for (int i = tid; i < kBins; i += kThreads) s.hist[i] = 0;
        __syncthreads();
        each(row, tid, row.pieces, kThreads, [&](uint32_t k, int i) {
            if ((level == 0 || k >> (shift + bits) == prefix) && kept.keeps(k, i)) {
                const u64 x = size(k);
                if (x) atomicAdd(&s.hist[k >> shift & (uint32_t)((1 << bits) - 1)], x);
            }
        });
        __syncthreads();
        const u64 hi = s.hist[kBins - 1 - 2 * tid], lo = s.hist[kBins - 2 - 2 * tid];
        u64 total;
        const u64 upto = above + block_upto(hi + lo, s.whole, total);
        if (level == 0) target = aim(total);
        const u64 before = upto - hi - lo;
        if (before < target && upto >= target) {
            const bool first = before + hi >= target;
            s.found = kBins - (first ? 1 : 2) - 2 * tid;
            s.above = first ? before : before + hi;
            s.in_bin = first ? hi : lo;
        }
        __syncthreads();
        prefix = prefix << bits | (uint32_t)s.found;
        above = s.above;
        in_bin = s.in_bin;
        __syncthreads();
    }
    const u64 one = size(prefix);
    need = (target - above + one - 1) / one;
    have = in_bin / one;
    return prefix;
}

// The lowest index at which the sums of size(key, index) exceed target(sum of
// all), or the last of some size if rounding leaves none.
template <class T, class Size, class Target>
__device__ int index_at(Lds &s, const Row<T> &row, Size size, Target target, double &total) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int from = 0, to = row.pieces;
    double t = 0.0;
    for (int level = 0; level < 2; ++level) {  // a sixteenth of the row, a sixteenth of that
        const int n = (to - from + kWaves - 1) / kWaves;
        double sum = 0.0;
        each(row, from + w * n + lane, min(to, from + (w + 1) * n), 64, [&](uint32_t k, int i) { sum += size(k, i); });
        sum = wave_add(sum);
        if (lane == 0) s.real[w] = sum;
        __syncthreads();
        if (level == 0) {
            total = 0.0;
            for (int i = 0; i < kWaves; ++i) total += s.real[i];
            t = target(total);
        }
        double upto = 0.0, rest = t;
        int part = 0;
        for (int i = 0; i < kWaves; ++i) {
            if (s.real[i] > 0.0) {
                part = i;
                rest = t - upto;
            }
            upto += s.real[i];
            if (upto > t) break;
        }
        t = rest;
        from += part * n;
        to = min(to, from + n);
        __syncthreads();
    }
    if (w == 0) {
        const int n = (to - from + 63) / 64;
        double sum = 0.0;
        const int mine = from + lane * n, end = min(to, mine + n);
        each(row, mine, end, 1, [&](uint32_t k, int i) { sum += size(k, i); });
        const double upto = wave_upto(sum);
        const u64 past = __ballot(sum > 0.0 && upto > t), some = __ballot(sum > 0.0);
        const int who = past ? __ffsll(past) - 1 : some ? 63 - __clzll(some) : 0;
        if (lane == who) {
            double at = upto - sum;
            int index = -1;
            bool done = false;
            each(row, mine, end, 1, [&](uint32_t k, int i) {
                const double x = size(k, i);
                if (!done && x > 0.0) {
                    index = i;
                    at += x;
                    done = at > t;
                }
            });
            s.found = index;
        }
    }
    __syncthreads();
    const int index = s.found;
    __syncthreads();
    return index;
}

struct Settings {
    double temperature, top_p, min_p, u;
    int top_k;  // 0: all
};

// The list's n tokens, which are all that may be kept and all that count for
// top_p: ranked, cut, put in order of their indices and summed.
__device__ void from_list(Lds &s, const Settings &set, const Weight &weight, int n, int &token, double &share) {
    constexpr int kPer = kList / kThreads;
    const int tid = threadIdx.x;
    sort_list(s, n);  // by falling key, then rising index
    const int most = set.top_k ? min(set.top_k, n) : n;
    double w[kPer], sum = 0.0, total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int j = tid * kPer + e;
        w[e] = j < most ? weight((uint32_t)(s.list[j] >> 32)) : 0.0;
        sum += w[e];
    }
    double before = block_upto(sum, s.real, total) - sum;
    if (tid == 0) s.count = 0;
    __syncthreads();
    int kept = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int j = tid * kPer + e;
        if (j < most && (j == 0 || ((set.top_p >= 1.0 || before < set.top_p * total) && w[e] >= set.min_p))) ++kept;
        before += w[e];
    }
    if (kept) atomicAdd(&s.count, kept);
    __syncthreads();
    const int keep = s.count;
    __syncthreads();
    // by rising index, with the key
    for (int j = tid; j < keep; j += kThreads) {
        const u64 x = s.list[j];
        s.list[j] = x << 32 | x >> 32;  // index complemented: falling is rising
    }
    sort_list(s, keep);
    sum = 0.0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int j = tid * kPer + e;
        w[e] = j < keep ? weight((uint32_t)s.list[j]) : 0.0;
        sum += w[e];
    }
    const double upto = block_upto(sum, s.real, total);
    double at = upto - sum;
    const double t = set.u * total;
    if (tid == 0) s.found = keep - 1;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int j = tid * kPer + e;
        at += w[e];
        if (j < keep && w[e] > 0.0 && at > t) {
            atomicMin(&s.found, j);
            break;
        }
    }
    __syncthreads();
    const u64 x = s.list[s.found];
    token = (int)~(uint32_t)(x >> 32);
    share = weight((uint32_t)x) / total;
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_sample(SampleLaunch a) {
    __shared__ Lds s;
    const int tid = threadIdx.x, r = blockIdx.x;
    Settings set;
    const float temperature = a.temperature ? a.temperature[r] : a.temperature_all;
    const float top_p = a.top_p ? a.top_p[r] : a.top_p_all, min_p = a.min_p ? a.min_p[r] : a.min_p_all, u = a.u[r];
    set.temperature = temperature, set.top_p = top_p, set.min_p = min_p, set.u = u;
    set.top_k = a.top_k ? a.top_k[r] : a.top_k_all;
    auto answer = [&](int token, double logprob) {
        if (tid == 0) {
            a.token[r] = token;
            if (a.logprob) a.logprob[r] = (float)logprob;
        }
    };
    if (!(temperature >= 0.0f && temperature < INFINITY && set.top_k >= 0 && top_p > 0.0f && top_p <= 1.0f &&
          min_p >= 0.0f && min_p <= 1.0f && u >= 0.0f && u < 1.0f)) {
        if (tid == 0 && a.status) a.status[r] = FATE_EINVAL;
        answer(-1, -INFINITY);
        return;
    }
    const Row<T> row(a, r);

    // the largest logit, of equal ones the lowest index
    uint32_t mine = 0;
    int mine_at = 0;
    each(row, tid, row.pieces, kThreads, [&](uint32_t k, int i) {
        if (k > mine) {
            mine = k;
            mine_at = i;
        }
    });
    const u64 best = block_max((u64)mine << 32 | (mine ? (uint32_t)~mine_at : 0u), s);
    Weight weight;
    weight.top = (uint32_t)(best >> 32);
    if (weight.top == 0) {  // nothing to choose from
        answer(-1, -INFINITY);
        return;
    }
    if (temperature == 0.0f || set.top_k == 1) {
        answer((int)~(uint32_t)best, 0.0);
        return;
    }
    weight.max = value_of(weight.top);
    weight.per = 1.0 / set.temperature;

    int token;
    double share;
    const bool small_k = set.top_k > 0 && set.top_k <= kSmallK, least = set.top_p >= 1.0 && set.min_p > 0.0;
    if (row.V <= kList || small_k || least) {
        uint32_t bound = 1;
        if (row.V > kList) {
            if (small_k) bound = max(bound, kth_word(s, mine, set.top_k));
            if (least) {  // a little below the logit of weight min_p; weights decide
                const double x = weight.max + set.temperature * log(set.min_p);
                bound = max(bound, key_of((float)(x - 1e-6 * (fabs(x) + fabs(weight.max)))));
            }
        }
        if (tid == 0) s.count = 0;
        __syncthreads();
        each(row, tid, row.pieces, kThreads, [&](uint32_t k, int i) {
            if (k >= bound) {
                const int at = atomicAdd(&s.count, 1);
                if (at < kList) s.list[at] = (u64)k << 32 | (uint32_t)~i;
            }
        });
        __syncthreads();
        const int n = s.count;
        __syncthreads();
        if (n <= kList) {
            from_list(s, set, weight, n, token, share);
            answer(token, log(share));
            return;
        }
    }

    Place kept = {0, kAll};
    auto cut = [&](uint32_t key, u64 need, u64 have) {  // the first `need` of the key's `have` tokens are kept
        int index = kAll;
        if (need < have) {
            double all;
            const Place was = kept;
            index = index_at(s, row, [&](uint32_t k, int i) { return k == key && was.keeps(k, i) ? 1.0 : 0.0; },
                             [&](double) { return (double)need - 1.0; }, all);
        } else if (kept.key == key) {
            index = kept.index;
        }
        kept = {key, index};
    };
    if (set.top_k > 0 && set.top_k < row.V) {
        u64 need, have;
        const u64 k = (u64)set.top_k;
        const uint32_t key = key_at(s, row, kept, [](uint32_t) { return 1ull; },
                                    [&](u64 all) { return k < all ? k : all; }, need, have);
        cut(key, need, have);
    }
    if (set.top_p < 1.0) {
        double sum = 0.0;
        each(row, tid, row.pieces, kThreads, [&](uint32_t k, int i) {
            if (kept.keeps(k, i)) sum += weight(k);
        });
        double total;
        block_upto(sum, s.real, total);
        // weights as whole numbers, 2^61 to 2^62 for all together: each is off by less than 2^-61 of the sum, equal
        // ones alike
        const int unit = 61 - (int)((__builtin_bit_cast(u64, total) >> 52) - 1023);
        u64 need, have;
        const uint32_t key = key_at(s, row, kept, [&](uint32_t k) { return (u64)(__builtin_ldexp(weight(k), unit) + 0.5); },
                                    [&](u64 all) { return share_of(top_p, all); }, need, have);
        cut(key, need, have);
    }
    double total;
    token = index_at(s, row, [&](uint32_t k, int i) {
        if (!kept.keeps(k, i)) return 0.0;
        const double w = weight(k);
        return w >= set.min_p ? w : 0.0;
    }, [&](double all) { return set.u * all; }, total);
    if (a.logprob) share = weight(key_of(T::at(row.data, max(token, 0)))) / total;
    answer(token, a.logprob ? log(share) : 0.0);
}

}  // namespace

int launch_sample(const SampleLaunch &a, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)a.rows), block(kThreads);
    if (a.dtype == FATE_BF16) hipLaunchKernelGGL((k_sample<B16>), grid, block, 0, s, a);
    else if (a.dtype == FATE_F16) hipLaunchKernelGGL((k_sample<H16>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_sample<F32>), grid, block, 0, s, a);
    return (int)hipGetLastError();
}

}  // namespace fate
