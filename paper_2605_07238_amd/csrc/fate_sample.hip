// One token of each row of logits, from a given random number.
//
//   w_i = exp((l_i - max l) / temperature); of the tokens by falling logit (equal
//   ones by rising index), the first top_k; of these those before which less than
//   top_p of their sum lies; of these those with w_i >= min_p.  The token is the
//   lowest i with sum of w_j over the kept j <= i greater than u W, W the sum of
//   all kept.  What is kept is a stretch of that order from its start, so one
//   place in it, a logit and an index, says which tokens are kept.
//
// Everything that a token hangs on is computed in 64 bits: between two
// neighbours of 100000 tokens lies 1e-5 of W, and a sum that is off by 2^-24
// would pick another one in every hundredth row.  Sums have a fixed order, and
// where atomics add they add whole numbers: two calls give the same token.
//
// k_sample: one workgroup per row.  It reads the row for its largest logit and,
// for top_p, once more for the sum of all weights.  Where few tokens can be kept
// the next reading gathers them into LDS in the order of their indices, where
// the place of the cut is found by ranking those in question against each other,
// and the token by sums up to each.  What can be kept is known from bins of the
// logits: of the threads' largest ones for top_k (at least k tokens reach the k-th
// of these, and hardly more do), of all that matter, by weights as whole numbers,
// for top_p.  Where the gathered do not fit, the place of the cut is found by its
// digits (11, 11 and 10 bits of the key), each by a histogram, of counts or of
// weights; then two readings find the token, of which the second is of a
// sixteenth of the row.  Instructions bind it, of a weight some 22; code that is
// run once costs what its fetching costs, so that loops are kept short.  Rows of
// 16-bit logits can go by their values instead (by_values): 512 rows of 131072 in
// bfloat16 with top_p 0.9, inputs in turn, 91 us where weights of each token took 218.
#include <hip/hip_runtime.h>

#include "fate_sample.h"

namespace fate {
namespace {

typedef unsigned long long u64;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kOwn = 512;      // tokens that a wave gathers in LDS, at most
constexpr int kMany = kWaves * kOwn + 1;  // more than the list holds
constexpr int kRanked = 512;   // of these, most that are ranked
constexpr int kSmallK = 1024;  // largest top_k that the threads' largest logits bound
constexpr int kBins = 2048;

struct Ranked {
    u64 entry;
    double weight;
};

// Rows of 16-bit logits by their values (see by_values): how many tokens have each
// of the 65536, two counts to a word, and then the weights of the kept ones; of the
// stretches of 64 values that occur, the value that starts them, their tokens, and
// the sum of their weights.
constexpr int kValues = 65536, kStretch = 64, kStretches = kValues / kStretch;
constexpr int kWeights = 16384;
struct Values {
    union {
        uint32_t counts[kValues / 2];
        double weights[kWeights];
    };
    double sum[kStretches];
    int num[kStretches], first[kStretches];
};

struct Lds {
    double table[256];
    union {
        struct {
            u64 list[kWaves * kOwn];
            u64 hist[kBins];
            Ranked ranked[kRanked];
        };
        Values values;
    };
    u64 whole[kWaves], least[kWaves];
    double real[kWaves];
    float ends[2][8];  // the values of the row's first and last piece
    u64 above, in_bin;
    double share;
    int found, counts[kWaves];
};

// The workgroup's, of the kernel and of what it calls.
__device__ __forceinline__ Lds &lds() {
    __shared__ Lds s;
    return s;
}

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
// A token of the list: key and index, larger ones earlier in the order.
__device__ __forceinline__ u64 entry_of(uint32_t key, int index) { return (u64)key << 32 | (uint32_t)~index; }
__device__ __forceinline__ float logit_of(u64 entry) { return value_of((uint32_t)(entry >> 32)); }
__device__ __forceinline__ int index_of(u64 entry) { return (int)~(uint32_t)entry; }

struct F32 {
    static constexpr int kPer = 4;
    static __device__ __forceinline__ float get(const u32x4 &x, int e) {
        const uint32_t w = x[e];  // (a cast of the vector's element itself takes the first one's bits)
        return __builtin_bit_cast(float, w);
    }
    static __device__ __forceinline__ float at(const char *p, int64_t i) { return ((const float *)p)[i]; }
    static constexpr int kBytes = 4, kValuesFrom = 0;
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
    static constexpr int kInfinity = 0x7f80, kValuesFrom = 8192;
    static __device__ __forceinline__ float of_bits(int b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }
    static __device__ __forceinline__ uint32_t bits(float v) { return __builtin_bit_cast(uint32_t, v) >> 16; }
};
struct H16 {
    static constexpr int kPer = 8;
    static __device__ __forceinline__ float get(const u32x4 &x, int e) {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(x[e / 2] >> (e & 1) * 16));
    }
    static __device__ __forceinline__ float at(const char *p, int64_t i) { return (float)((const _Float16 *)p)[i]; }
    static constexpr int kBytes = 2;
    static constexpr int kInfinity = 0x7c00, kValuesFrom = 16384;
    static __device__ __forceinline__ float of_bits(int b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }
    static __device__ __forceinline__ uint32_t bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

// A row in pieces of 16 aligned bytes, numbered from that of its first element;
// the first and the last may reach over its ends.
template <class T>
struct Row {
    const char *data;
    int V, lead, pieces;  // lead: places of the first piece before the row
    int whole0, whole1;   // the first and the last piece within the row; none if the last is before the first

    __device__ __forceinline__ Row(const SampleLaunch &a, int row) {
        data = a.logits + (int64_t)row * a.stride * T::kBytes;
        V = a.vocab;
        lead = (int)((uintptr_t)data % 16) / T::kBytes;
        pieces = (int)(((int64_t)V + lead + T::kPer - 1) / T::kPer);
        whole0 = lead ? 1 : 0;
        whole1 = (int)(((int64_t)V + lead) / T::kPer) - 1;
    }
    // (a barrier before the first `each`)
    __device__ __forceinline__ void read_ends() const {
        const int tid = threadIdx.x;
        if (tid < 16) {
            const int i = index(tid < 8 ? 0 : pieces - 1) + (tid & 7);
            lds().ends[tid >> 3][tid & 7] = i >= 0 && i < V && (tid & 7) < T::kPer ? T::at(data, i) : __builtin_nanf("");
        }
    }
    __device__ __forceinline__ int index(int piece) const { return piece * T::kPer - lead; }
    __device__ __forceinline__ u32x4 load(int piece) const {
        return *(const u32x4 *)(data + (int64_t)index(piece) * T::kBytes);
    }
};

// f(values, index of the first) for pieces from, from + step .., in this order;
// what lies outside the row is NaN, which compares as nothing.  Pieces within
// the row go four (of 16-bit logits two) at a time, their loads together and
// without checks of each.  All lanes of a wave call f as often, those without a
// piece on NaN.
template <class T, class F>
__device__ __forceinline__ void each(const Row<T> &row, int from, int to, int step, F f) {
    constexpr int kAhead = 16 / T::kPer;
    const int last = min(to - 1, row.whole1);
    for (int p = from; __any(p < to);) {
        if (__all(p >= row.whole0 && p + (kAhead - 1) * step <= last)) {
            u32x4 x[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) x[u] = row.load(p + u * step);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                float v[T::kPer];
#pragma unroll
                for (int e = 0; e < T::kPer; ++e) v[e] = T::get(x[u], e);
                f(v, row.index(p + u * step));
            }
            p += kAhead * step;
        } else {
            float v[T::kPer];
#pragma unroll
            for (int e = 0; e < T::kPer; ++e) v[e] = __builtin_nanf("");
            if (p < to && (p < row.whole0 || p > row.whole1)) {
#pragma unroll
                for (int e = 0; e < T::kPer; ++e) v[e] = lds().ends[p > 0][e];
            } else if (p < to) {
                const u32x4 x = row.load(p);
#pragma unroll
                for (int e = 0; e < T::kPer; ++e) v[e] = T::get(x, e);
            }
            f(v, row.index(p));
            p += step;
        }
    }
}

// Weight of a logit, e^z with z = (l - max) / temperature <= 0; 0 of NaN and -infinity.
// With y = z 256 / ln 2 = 256 n + j + x, |x| <= 1/2, it is 2^n 2^(j / 256) and
// the series of e^(x ln 2 / 256) to its fourth power (the next term is 2^-54):
// half the steps of a series without the table, 2^(j / 256) by j in LDS.
constexpr int kTable = 256;
struct Weight {
    double max, per;  // per = 256 / (ln 2 temperature)
    __device__ __forceinline__ double operator()(float v) const {
        constexpr double c = 0.69314718055994530942 / kTable;
        const double y = fmax(((double)v - max) * per, -4e5);  // 0 from there on
        const double n = __builtin_rint(y), x = y - n;
        double f = __builtin_fma(x, c * c * c * c / 24.0, c * c * c / 6.0);
        f = __builtin_fma(f, x, c * c / 2.0);
        f = __builtin_fma(f, x, c);
        f = __builtin_fma(f, x, 1.0);
        const int i = (int)n;
        return __builtin_ldexp(f * lds().table[i & (kTable - 1)], i >> 8);
    }
    __device__ __forceinline__ double of_key(uint32_t key) const { return (*this)(value_of(key)); }
};

// The kept tokens: those over a place in the order.
struct Place {
    float value;
    int index;
    __device__ __forceinline__ bool keeps(float v, int i) const { return (v > value) | ((v == value) & (i <= index)); }
};
constexpr int kAll = 0x7fffffff;

// The least whole number that is p * n or more, p in (0, 1], 1 <= n < 2^63.
__device__ __forceinline__ u64 share_of(float p, u64 n) {
    const uint32_t b = __builtin_bit_cast(uint32_t, p), e = b >> 23;
    const unsigned __int128 x = (unsigned __int128)n * (e ? (b & 0x7fffffu) | 0x800000u : b);
    const int shift = 150 - (int)(e ? e : 1);  // p = mantissa / 2^shift
    if (shift > 90) return 1;
    return (u64)((x + (((unsigned __int128)1 << shift) - 1)) >> shift);
}

// Another lane's value, by a move within rows of 16 lanes or from one to the
// next (0 where there is none), and lane i's value, the same in all lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved32(int x) {
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS, class I>
__device__ __forceinline__ I moved(I x) {
    static_assert(sizeof(I) == 8, "eight bytes");
    const u64 y = __builtin_bit_cast(u64, x);
    return __builtin_bit_cast(I, (u64)(uint32_t)moved32<CTRL, ROWS>((int)(y >> 32)) << 32 |
                                     (uint32_t)moved32<CTRL, ROWS>((int)y));
}
template <class I>
__device__ __forceinline__ I of_lane(I x, int i) {
    const u64 y = __builtin_bit_cast(u64, x);
    return __builtin_bit_cast(I, (u64)(uint32_t)__builtin_amdgcn_readlane((int)(y >> 32), i) << 32 |
                                     (uint32_t)__builtin_amdgcn_readlane((int)y, i));
}
template <class I>
__device__ __forceinline__ I wave_upto(I x) {  // sums up to and with this lane
    x += moved<0x111, 0xF>(x);
    x += moved<0x112, 0xF>(x);
    x += moved<0x114, 0xF>(x);
    x += moved<0x118, 0xF>(x);
    x += moved<0x142, 0xA>(x);
    x += moved<0x143, 0xC>(x);
    return x;
}
template <class I>
__device__ __forceinline__ I wave_add(I x) { return of_lane(wave_upto(x), 63); }
__device__ __forceinline__ u64 larger(u64 x, u64 y) { return x > y ? x : y; }
__device__ __forceinline__ u64 wave_max(u64 x) {
    x = larger(x, moved<0x111, 0xF>(x));
    x = larger(x, moved<0x112, 0xF>(x));
    x = larger(x, moved<0x114, 0xF>(x));
    x = larger(x, moved<0x118, 0xF>(x));
    x = larger(x, moved<0x142, 0xA>(x));
    x = larger(x, moved<0x143, 0xC>(x));
    return of_lane(x, 63);
}

// Sums up to and with this thread, and of all.  (The waves' sums go through lanes:
// added one after the other by every wave they took 2 us.)
template <class I>
__device__ __forceinline__ I block_upto(I x, I (&part)[kWaves], I &total) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    x = wave_upto(x);
    if (lane == 63) part[w] = x;
    __syncthreads();
    const I upto = wave_upto(lane < kWaves ? part[lane] : I(0));
    __syncthreads();
    total = of_lane(upto, kWaves - 1);
    return w ? of_lane(upto, w - 1) + x : x;
}

__device__ __forceinline__ u64 block_max(u64 x, Lds &s) {
    x = wave_max(x);
    if ((threadIdx.x & 63) == 0) s.whole[threadIdx.x >> 6] = x;
    __syncthreads();
    x = wave_max((threadIdx.x & 63) < kWaves ? s.whole[threadIdx.x & 63] : 0);
    __syncthreads();
    return x;
}

// Bins of logits from `top` down to `bottom`, which falls into the last.
struct Bins {
    float top, per;
    __device__ __forceinline__ Bins(float t, float bottom) : top(t), per((kBins - 1) / (t - bottom)) {}
    __device__ __forceinline__ bool good() const { return per > 0.0f && per < INFINITY; }
    __device__ __forceinline__ int of(float v) const {
        return (int)fminf(__fmul_rn(__fsub_rn(top, v), per), kBins - 1);
    }
    // a logit below all of the bin's
    __device__ __forceinline__ float under(int bin) const {
        const float edge = top - (float)(bin + 1) / per;
        return edge - 1e-6f * (__builtin_fabsf(top) + __builtin_fabsf(edge));
    }
};

__device__ __forceinline__ void clear_bins(Lds &s) {
    for (int i = threadIdx.x; i < kBins; i += kThreads) s.hist[i] = 0;
}

// What top_p keeps of a sum, as a whole number of 2^-bits: 1 at least, since the first token always is kept, and no bin
// reaches 0.
__device__ __forceinline__ u64 aim_of(double top_p, double whole, int bits) {
    const u64 aim = (u64)__builtin_ldexp(top_p * whole, bits);
    return aim ? aim : 1;
}

// The bin in which the sums of s.hist reach `target`, or -1.
__device__ __forceinline__ int bin_at(Lds &s, u64 target) {
    const int tid = threadIdx.x;
    if (tid == 0) s.found = -1;
    const u64 hi = s.hist[2 * tid], lo = s.hist[2 * tid + 1];
    u64 all;
    const u64 upto = block_upto(hi + lo, s.whole, all), before = upto - hi - lo;
    if (before < target && upto >= target) s.found = 2 * tid + (before + hi >= target ? 0 : 1);
    __syncthreads();
    const int bin = s.found;
    __syncthreads();
    return bin;
}

// A row's pieces are the waves' by sixteenths, of so many pieces each.
template <class T>
__device__ __forceinline__ int sixteenth(const Row<T> &row) {
    return (row.pieces + kWaves - 1) / kWaves;
}

// Of the tokens that `kept` keeps, each of `size(key)`: the key at which the
// sizes of the tokens with this key or a larger one reach aim(sum of all); how
// many of this key that takes, and how many there are.
template <class T, class Size, class Aim>
__device__ __forceinline__ uint32_t key_at(Lds &s, const Row<T> &row, const Place &kept, Size size, Aim aim, u64 &need,
                                           u64 &have) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    u64 above = 0, in_bin = 0, target = 0;
#pragma nounroll
    for (int level = 0; level < 3; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
        for (int i = tid; i < kBins; i += kThreads) s.hist[i] = 0;
        __syncthreads();
        each(row, tid, row.pieces, kThreads, [&](const float (&v)[T::kPer], int i0) {
#pragma unroll
            for (int e = 0; e < T::kPer; ++e) {
                const uint32_t k = key_of(v[e]);
                if (k && (level == 0 || k >> (shift + bits) == prefix) && kept.keeps(v[e], i0 + e)) {
                    const u64 x = size(k);
                    if (x) atomicAdd(&s.hist[k >> shift & (uint32_t)((1 << bits) - 1)], x);
                }
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

// A stretch of a row's pieces, and where in its sums a token is sought.
struct Part {
    int from, to;
    double t;
};

// The lowest index at which the sums of size(logit, index) exceed target(sum of
// all), or the last of some size if rounding leaves none; its size in s.share.  `known`: s.real has
// the sums of the sixteenths; `part`: of these or other parts of the row, the one
// that it lies in, found already.
template <class T, class Size, class Target>
__device__ __forceinline__ int index_at(Lds &s, const Row<T> &row, bool known, const Part *part, Size size, Target target,
                                        double &total) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int from = part ? part->from : 0, to = part ? part->to : row.pieces;
    double t = part ? part->t : 0.0;
#pragma nounroll
    for (int level = part ? 1 : 0; level < 2; ++level) {  // a sixteenth of the row, a sixteenth of that
        const int n = level == 0 ? sixteenth(row) : (to - from + kWaves - 1) / kWaves;
        if (level > 0 || !known) {
            double sum = 0.0;
            each(row, from + w * n + lane, min(to, from + (w + 1) * n), 64, [&](const float (&v)[T::kPer], int i0) {
#pragma unroll
                for (int e = 0; e < T::kPer; ++e) sum += size(v[e], i0 + e);
            });
            sum = wave_add(sum);
            if (lane == 0) s.real[w] = sum;
            __syncthreads();
        }
        const double sum = lane < kWaves ? s.real[lane] : 0.0, upto = wave_upto(sum);
        if (level == 0) {
            total = of_lane(upto, 63);
            t = target(total);
        }
        const u64 past = __ballot(sum > 0.0 && upto > t), some = __ballot(sum > 0.0);
        const int at = __builtin_amdgcn_readfirstlane(past ? __ffsll(past) - 1 : some ? 63 - __clzll(some) : 0);
        t -= of_lane(upto - sum, at);
        from += at * n;
        to = min(to, from + n);
        __syncthreads();
    }
    if (w == 0) {
        const int n = (to - from + 63) / 64, mine = from + lane * n, end = min(to, mine + n);
        double sum = 0.0, x[T::kPer] = {};  // x: sizes of the lane's last piece, its only one where there are few
        int x0 = 0;
        each(row, mine, end, 1, [&](const float (&v)[T::kPer], int i0) {
            x0 = i0;
#pragma unroll
            for (int e = 0; e < T::kPer; ++e) sum += x[e] = size(v[e], i0 + e);
        });
        const double upto = wave_upto(sum);
        const u64 past = __ballot(sum > 0.0 && upto > t), some = __ballot(sum > 0.0);
        const int who = past ? __ffsll(past) - 1 : some ? 63 - __clzll(some) : 0;
        if (lane == who) {
            double at = upto - sum, its = 0.0;
            int index = 0;
            bool done = false;
            auto look = [&](double y, int i) __attribute__((always_inline)) {
                if (!done && y > 0.0) {
                    index = i;
                    its = y;
                    at += y;
                    done = at > t;
                }
            };
            if (n == 1) {
#pragma unroll
                for (int e = 0; e < T::kPer; ++e) look(x[e], x0 + e);
            } else {
                each(row, mine, end, 1, [&](const float (&v)[T::kPer], int i0) {
                    for (int e = 0; e < T::kPer; ++e) look(size(v[e], i0 + e), i0 + e);
                });
            }
            s.found = index;
            s.share = its;
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
struct Answer {
    int token;
    double share;
};

// The tokens that want(logit) takes, to the list; returns how many, or kMany if
// they do not fit: of the pieces from .. to.  Each wave counts its own places, and
// they are moved together behind it; a wave whose places run out stops.  In order
// of the indices each wave goes through n16 pieces of its own, otherwise all go
// through the same stretches, which for a whole row of 131072 takes 6 us less.
template <class T, class Want>
__device__ __forceinline__ int gather(const Row<T> &row, int from, int to, int n16, bool in_order, Want want) {
    Lds &s = lds();
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    u64 *const own = s.list + w * kOwn;
    int count = 0;  // the same in all lanes
    each(row, from + (in_order ? w * n16 + lane : tid), in_order ? min(to, from + (w + 1) * n16) : to, in_order ? 64 : kThreads,
         [&](const float (&v)[T::kPer], int i0) {
        bool mine[T::kPer], any = false;
#pragma unroll
        for (int e = 0; e < T::kPer; ++e) any |= mine[e] = want(v[e]);
        if (__any(any) && count <= kOwn) {
            int at = count;  // places of lower lanes' tokens
#pragma unroll
            for (int e = 0; e < T::kPer; ++e) {
                const u64 who = __ballot(mine[e]);
                at += __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                count += __popcll(who);
            }
#pragma unroll
            for (int e = 0; e < T::kPer; ++e)
                if (mine[e]) {
                    if (at < kOwn) own[at] = entry_of(key_of(v[e]), i0 + e);
                    ++at;
                }
        }
    });
    if (lane == 0) s.counts[w] = count;
    __syncthreads();
    int n = 0, before = 0;
    bool fits = true;
    for (int i = 0; i < kWaves; ++i) {
        before += i < w ? s.counts[i] : 0;
        n += s.counts[i];
        fits = fits && s.counts[i] <= kOwn;
    }
    u64 x[kOwn / 64];
#pragma unroll
    for (int i = 0; i < kOwn / 64; ++i) x[i] = i * 64 + lane < count ? own[i * 64 + lane] : 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOwn / 64; ++i)
        if (fits && i * 64 + lane < count) s.list[before + i * 64 + lane] = x[i];
    __syncthreads();
    return fits ? n : kMany;
}

// Of this thread's one of the n <= kRanked entries of s.ranked: how many are
// before it, the sum of their weights, and how many have lower indices.  Where n
// is small several neighbouring threads share an entry, `owns` in the first.
struct Rank {
    int entry, rank, place;
    bool owns;
    double before;
};
template <int CTRL>
__device__ __forceinline__ void add_moved(Rank &x) {
    x.rank += moved32<CTRL, 0xF>(x.rank);
    x.place += moved32<CTRL, 0xF>(x.place);
    x.before += moved<CTRL, 0xF>(x.before);
}
__device__ __forceinline__ Rank rank_of(const Lds &s, int n) {
    const int share = n > 256 ? 1 : n > 128 ? 2 : n > 64 ? 3 : 4;  // 2 to 16 threads
    const int tid = threadIdx.x, part = tid & ((1 << share) - 1);
    Rank x = {tid >> share, 0, 0, part == 0 && tid >> share < n, 0.0};
    const u64 mine = x.entry < n ? s.ranked[x.entry].entry : 0;
#pragma unroll 4
    for (int i = part; i < n; i += 1 << share) {
        const u64 y = s.ranked[i].entry;
        const double z = s.ranked[i].weight;
        x.rank += y > mine;
        x.place += (uint32_t)y > (uint32_t)mine;
        x.before += y > mine ? z : 0.0;
    }
    add_moved<0xB1>(x);  // neighbours, pairs of them, then the mirror images of quads and of eights
    if (share > 1) add_moved<0x4E>(x);
    if (share > 2) add_moved<0x141>(x);
    if (share > 3) add_moved<0x140>(x);
    return x;
}

// The token among the list's n <= kRanked, in any order, which hold all that may
// be kept: each is ranked, by the order of the cuts and by its index, against all.
// top_p is of `whole`, or, if that is 0, of what top_k leaves.
__device__ __noinline__ Answer from_short(Settings set, Weight weight, int n, double whole) {
    Lds &s = lds();
    const int tid = threadIdx.x;
    if (tid < n) s.ranked[tid].entry = s.list[tid], s.ranked[tid].weight = weight(logit_of(s.list[tid]));
    __syncthreads();
    const Rank at = rank_of(s, n);
    const u64 x = at.owns ? s.ranked[at.entry].entry : 0;
    const double w = at.owns ? s.ranked[at.entry].weight : 0.0;
    double sum, total;
    const bool of_k = at.owns && (!set.top_k || at.rank < set.top_k);
    block_upto(of_k ? w : 0.0, s.real, sum);  // (its barriers: the entries have been read)
    const double aim = set.top_p * (whole > 0.0 ? whole : sum);
    const bool kept = of_k && (set.top_p >= 1.0 || at.before < aim || at.rank == 0) && w >= set.min_p;
    if (at.owns) s.ranked[at.place].entry = x, s.ranked[at.place].weight = kept ? w : 0.0;
    __syncthreads();
    // by rising index, sums up to each
    const double mine = tid < n ? s.ranked[tid].weight : 0.0, upto = block_upto(mine, s.real, total);
    if (tid == 0) s.found = n - 1;
    __syncthreads();
    if (mine > 0.0 && upto > set.u * total) atomicMin(&s.found, tid);
    __syncthreads();
    return {index_of(s.ranked[s.found].entry), s.ranked[s.found].weight / total};
}

// Of the list's n tokens from `floor` up (as entries), the last that is kept:
// those of a bin before `cut` are, those in it are ranked, and the first `most`
// of all are kept, or, where that is 0, those before which less than `aim` of the
// weights lies.  0 if too many are to be ranked, or the cut is not in the bin,
// where the rounding of the bins' sums has put it.
__device__ __noinline__ u64 last_of_list(Weight weight, int n, Bins bins, int cut, u64 floor, int most, double aim) {
    Lds &s = lds();
    const int tid = threadIdx.x, per = (n + kThreads - 1) / kThreads, lo = tid * per, hi = min(n, lo + per);
    u64 mine = 0, all;  // tokens to be ranked, and kept for sure, in the halves
    double over = 0.0, above;
    for (int j = lo; j < hi; ++j) {
        const u64 x = s.list[j];
        const int b = x >= floor ? bins.of(logit_of(x)) : kBins;
        mine += b == cut ? 1 : b < cut ? 1ull << 32 : 0;
        over += b < cut ? weight(logit_of(x)) : 0.0;
    }
    int at = (int)(uint32_t)(block_upto(mine, s.whole, all) - mine);
    const int m = (int)(uint32_t)all, sure = (int)(all >> 32);
    block_upto(over, s.real, above);
    if (m > kRanked) return 0;
    for (int j = lo; j < hi; ++j) {
        const u64 x = s.list[j];
        if (x >= floor && bins.of(logit_of(x)) == cut) {
            s.ranked[at].entry = x;
            s.ranked[at].weight = weight(logit_of(x));
            ++at;
        }
    }
    __syncthreads();
    const Rank its = rank_of(s, m);
    const u64 x = its.owns ? s.ranked[its.entry].entry : 0;
    const double before = above + its.before;
    double sum;
    block_upto(its.owns ? s.ranked[its.entry].weight : 0.0, s.real, sum);
    const bool kept = its.owns && (most ? sure + its.rank < most : before < aim || sure + its.rank == 0);
    u64 n_kept;
    block_upto((u64)kept, s.whole, n_kept);
    if (n_kept == 0 || (!most && (int)n_kept == m && above + sum < aim)) return 0;
    return ~block_max(kept ? ~x : 0, s);
}

// The token among those of the list's n that are kept, from `last` up; the list
// is in order of the indices.
__device__ __noinline__ Answer from_list(Settings set, Weight weight, int n, u64 last) {
    Lds &s = lds();
    const int tid = threadIdx.x, per = (n + kThreads - 1) / kThreads, lo = tid * per, hi = min(n, lo + per);
    double part = 0.0, total;
    for (int j = lo; j < hi; ++j) {
        const double x = s.list[j] >= last ? weight(logit_of(s.list[j])) : 0.0;
        part += x >= set.min_p ? x : 0.0;
    }
    const double upto = block_upto(part, s.real, total), t = set.u * total;
    if (tid == 0) s.found = kThreads;
    __syncthreads();
    if (part > 0.0 && upto > t) atomicMin(&s.found, tid);
    __syncthreads();
    if (tid == s.found) {
        double sofar = upto - part;
        bool done = false;
        for (int j = lo; j < hi && !done; ++j) {
            const double x = s.list[j] >= last ? weight(logit_of(s.list[j])) : 0.0;
            if (x > 0.0 && x >= set.min_p) {
                sofar += x;
                done = sofar > t;
                s.counts[0] = index_of(s.list[j]);
                s.share = x / total;
            }
        }
    }
    __syncthreads();
    return {s.counts[0], s.share};
}

// The last that top_k, and then top_p, keep of the list's n tokens, which hold
// all that they may keep; 0 as above.  Bins of the list's own logits tell where.
__device__ __noinline__ u64 last_of_k(Settings set, Weight weight, int n, Bins bins) {
    Lds &s = lds();
    constexpr double magic = 256.0;  // + w: w as a whole number of 2^-44 in the last places
    u64 last = 1;
    double whole = 0.0;
#pragma nounroll
    for (int by_weight = 0; by_weight < (set.top_p < 1.0 ? 2 : 1); ++by_weight) {
        clear_bins(s);
        __syncthreads();
        double sum = 0.0;
        for (int j = threadIdx.x; j < n; j += kThreads) {
            const u64 x = s.list[j];
            if (x < last) continue;
            const double w = weight(logit_of(x));
            sum += w;
            atomicAdd(&s.hist[bins.of(logit_of(x))],
                      by_weight ? __builtin_bit_cast(u64, w + magic) - __builtin_bit_cast(u64, magic) : 1ull);
        }
        block_upto(sum, s.real, whole);
        const int cut = bin_at(s, by_weight ? aim_of(set.top_p, whole, 44) : (u64)set.top_k);
        if (cut < 0) return 0;
        last = last_of_list(weight, n, bins, cut, last, by_weight ? 0 : set.top_k, set.top_p * whole);
        if (last == 0) return 0;
    }
    return last;
}

// The token of the list's n, in order of their indices, and all that top_k may
// keep; false where their number or their ties are too many.
__device__ __forceinline__ bool from_list_of_k(const Settings &set, const Weight &weight, int n, const Bins &bins, Answer &x) {
    const u64 last = last_of_k(set, weight, n, bins);
    if (last) x = from_list(set, weight, n, last);
    return last != 0;
}

// The place of top_k's and top_p's cuts by its digits.
template <class T>
__device__ __noinline__ Place by_digits(Row<T> row, Settings set, Weight weight, float top_p) {
    Lds &s = lds();
    const int tid = threadIdx.x;
    Place kept = {-INFINITY, kAll};
#pragma nounroll
    for (int by_weight = 0; by_weight < 2; ++by_weight) {
        if (by_weight ? !(set.top_p < 1.0) : !(set.top_k > 0 && set.top_k < row.V)) continue;
        // weights as whole numbers, 2^61 to 2^62 for all together: each is off by less than 2^-61 of the sum, equal
        // ones alike
        int unit = 0;
        if (by_weight) {
            double sum = 0.0, total;
            each(row, tid, row.pieces, kThreads, [&](const float (&v)[T::kPer], int i0) {
#pragma unroll
                for (int e = 0; e < T::kPer; ++e) sum += weight(kept.keeps(v[e], i0 + e) ? v[e] : __builtin_nanf(""));
            });
            block_upto(sum, s.real, total);
            unit = 61 - (int)((__builtin_bit_cast(u64, total) >> 52) - 1023);
        }
        const u64 k = (u64)set.top_k;
        u64 need, have;
        const uint32_t key = key_at(s, row, kept, [&](uint32_t x) {
            return by_weight ? (u64)(__builtin_ldexp(weight.of_key(x), unit) + 0.5) : 1ull;
        }, [&](u64 all) { return by_weight ? share_of(top_p, all) : k < all ? k : all; }, need, have);
        // the first `need` of the key's `have` tokens are kept
        const float value = value_of(key);
        int index = kept.value == value ? kept.index : kAll;
        if (need < have) {
            double all;
            const Place was = kept;
            index = index_at(s, row, false, nullptr, [&](float v, int i) { return ((v == value) & was.keeps(v, i)) ? 1.0 : 0.0; },
                             [&](double) { return (double)need - 1.0; }, all);
        }
        kept = {value, index};
    }
    return kept;
}

// The token among those kept.  `known`, `part` (within `total`): as above.
template <class T>
__device__ __noinline__ Answer token_at(Row<T> row, Settings set, Weight weight, Place kept, bool known, bool parted,
                                        Part part, double total) {
    Lds &s = lds();
    const int token = index_at(s, row, known, parted ? &part : nullptr, [&](float v, int i) {
        const double x = weight(kept.keeps(v, i) ? v : __builtin_nanf(""));
        return x < set.min_p ? 0.0 : x;
    }, [&](double all) { return set.u * all; }, total);
    return {token, s.share / total};
}

// The tokens at +infinity share the row, and nothing else counts.
template <class T>
__device__ __noinline__ Answer token_at_infinity(Row<T> row, Settings set, float top_p) {
    double n = 0.0, all;
    const int token = index_at(lds(), row, false, nullptr, [&](float v, int) { return v == INFINITY ? 1.0 : 0.0; }, [&](double x) {
        n = set.top_k && set.top_k < x ? set.top_k : x;
        if (top_p < 1.0f) n = (double)share_of(top_p, (u64)n);
        return floor(set.u * n);
    }, all);
    return {token, 1.0 / n};
}

// Weights of the pieces of this wave's part of from .. to, `n16` pieces a wave,
// that lie over the bin `cut`: `over`, and of these, those that min_p leaves; the
// tokens of the bin to the list, in order of their indices.
template <class T>
__device__ __forceinline__ int sums_over_bin(const Row<T> &row, int from, int to, int n16, const Settings &set,
                                             const Weight &weight, const Bins &bins, float bottom, int cut, double &over,
                                             double &part) {
    over = part = 0.0;
    return gather(row, from, to, n16, true, [&](float v) {
        const int bin = v >= bottom ? bins.of(v) : kBins + 1;
        const double x = weight(bin < cut ? v : __builtin_nanf(""));
        over += x;
        part += x >= set.min_p ? x : 0.0;
        return bin == cut;
    });
}

// The last that top_p keeps of the list's n tokens, those of the bin of the cut,
// with `above` before them and `whole` in all; 0 if they are too many, or the cut
// is not in the bin, where the rounding of the bins' sums has put it.
__device__ __noinline__ u64 last_in_bin(Settings set, Weight weight, int n, double above, double whole) {
    Lds &s = lds();
    const int tid = threadIdx.x;
    if (n > kRanked) return 0;
    if (tid < n) s.ranked[tid].entry = s.list[tid], s.ranked[tid].weight = weight(logit_of(s.list[tid]));
    __syncthreads();
    const Rank at = rank_of(s, n);
    const u64 x = at.owns ? s.ranked[at.entry].entry : 0;
    const double before = above + at.before;
    double in_bin;
    block_upto(at.owns ? s.ranked[at.entry].weight : 0.0, s.real, in_bin);
    const double aim = set.top_p * whole;
    const bool keeps = x && before < aim;
    const u64 last = ~block_max(keeps ? ~x : 0, s), none = ~0ull;
    if (last == none || (above + in_bin < aim && last == ~block_max(x ? ~x : 0, s))) return 0;
    return last;
}

// Where the bins' sums do not reach top_p's cut (kBins), whether it lies behind all tokens in question, so that min_p
// cuts before it: weights decide, `over` their sum, since sums of whole numbers fall short of the cut also by what
// small weights lose in them.
__device__ __forceinline__ bool min_p_cuts(const Settings &set, double over, double whole) { return over < set.top_p * whole; }

// The place of top_p's cut over all of a row, and the sums of what is kept of
// each sixteenth in s.real, where what it keeps does not fit the list; false as
// above.
template <class T>
__device__ __noinline__ bool cut_in_bin(Row<T> row, Settings set, Weight weight, Bins bins, float bottom, int cut,
                                        double whole, Place &kept) {
    Lds &s = lds();
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n16 = sixteenth(row);
    double over, part, above;
    const int n = sums_over_bin(row, 0, row.pieces, n16, set, weight, bins, bottom, cut, over, part);
    block_upto(over, s.real, above);
    const u64 last = cut == kBins ? (u64)min_p_cuts(set, above, whole) : last_in_bin(set, weight, n, above, whole);
    if (last == 0) return false;
    if (cut < kBins) kept = {logit_of(last), index_of(last)};
    for (int j = lane; j < n; j += 64) {  // of the bin's tokens, those kept count for their sixteenths
        const u64 y = s.list[j];
        const int first = row.index(w * n16), end = row.index((w + 1) * n16);
        if (y >= last && index_of(y) >= first && index_of(y) < end) {
            const double z = weight(logit_of(y));
            part += z >= set.min_p ? z : 0.0;
        }
    }
    part = wave_add(part);
    if (lane == 0) s.real[w] = part;
    __syncthreads();
    return true;
}

// What a call asks of a row.
__device__ __forceinline__ Settings settings_of(const SampleLaunch &a, int r) {
    Settings set;
    set.temperature = a.temperature ? a.temperature[r] : a.temperature_all;
    set.top_p = a.top_p ? a.top_p[r] : a.top_p_all;
    set.min_p = a.min_p ? a.min_p[r] : a.min_p_all;
    set.u = a.u[r];
    set.top_k = a.top_k ? a.top_k[r] : a.top_k_all;
    return set;
}
__device__ __forceinline__ bool good(const Settings &x) {
    return x.temperature >= 0.0 && x.temperature < INFINITY && x.top_k >= 0 && x.top_p > 0.0 && x.top_p <= 1.0 &&
           x.min_p >= 0.0 && x.min_p <= 1.0 && x.u >= 0.0 && x.u < 1.0;
}
// top_p over all of a row of V tokens; no cuts at all.
__device__ __forceinline__ bool by_nucleus(const Settings &x, int V) { return x.top_p < 1.0 && !(x.top_k > 0 && x.top_k < V); }
__device__ __forceinline__ bool uncut(const Settings &x, int V) {
    return x.top_p >= 1.0 && !(x.top_k > 0 && x.top_k < V) && x.min_p == 0.0;
}

// Rows that go by their values: 16-bit logits whose nucleus, or many largest, are
// asked for.  512 rows of 131072 in bfloat16 take 74 us so for any cut, otherwise
// 210 for top-p 0.9 and 73 to 147 for top-k 200 to 1000, but 57 for 50; 64 rows of
// 8192 15 for top-p, otherwise 23, and of 4096 15 either way; in float16, of which
// more values occur, of 16384 26 against 39, and of 8192 24 against 23.  Past 2^19
// the slices of a row's other way win: 100 against 105 us for one of 524288.
template <class T>
__device__ __host__ __forceinline__ bool by_values_pays(double temperature, int top_k, double top_p, int V) {
    if (T::kBytes > 2 || V < T::kValuesFrom || V > 1 << 19 || !(temperature > 0.0)) return false;
    return top_k > 0 && top_k < V ? top_k > 256 : top_p < 1.0;
}
template <class T>
__device__ __forceinline__ bool goes_by_values(const Settings &x, int V) {
    return by_values_pays<T>(x.temperature, x.top_k, x.top_p, V);
}

__device__ __forceinline__ Weight weight_of(const Settings &set, float top) {
    return {top, 369.32993046757463 / set.temperature};
}

// A little below the logit of weight w; weights decide.
__device__ __forceinline__ float logit_below(const Settings &set, float top, double w) {
    const double x = (double)top + set.temperature * log(w);
    return fmaxf((float)(x - 1e-6 * (fabs(x) + fabs((double)top))), -3.402823466e38f);
}

// A thread's largest logits of each of a row's slices; -infinity past them.
constexpr int kSlices = 8;
template <int N>
struct Mine {
    float best[N];
};

// The lowest logit that top_p over all of a row may keep: tokens of weight
// (1 - top_p) S / V or less sum to (1 - top_p) S at most and are cut, and the
// threads' largest logits give a bound of S from below (in 32 bits, less what
// these may be off by).
template <int N>
__device__ __forceinline__ float nucleus_bottom(Lds &s, const Settings &set, const Weight &weight, float top, int V,
                                                const Mine<N> &mine) {
    const float per = (float)(weight.per / kTable);
    float low = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float z = mine.best[i] - top;
        if (mine.best[i] > -INFINITY) low += z < 0.0f ? __builtin_amdgcn_exp2f(z * per) : 1.0f;
    }
    double all;
    block_upto((double)low, s.real, all);
    return logit_below(set, top, fmax((1.0 - set.top_p) * 0.999 * all / V, set.min_p));
}

// Weights of the pieces from .. to: their sum, by thread, and those at `bottom` and
// over it in the bins, as whole numbers of 2^-bits: w + 2^(52 - bits) has them in
// its last places, and a sum of V of them stays under 2^63.
__device__ __forceinline__ int bits_of(int V) { return min(52, 30 + __builtin_clz((uint32_t)V)); }
template <class T>
__device__ __forceinline__ double sum_by_bins(Lds &s, const Row<T> &row, int from, int to, const Weight &weight,
                                              const Bins &bins, float bottom) {
    const bool good = bins.good();
    const double magic = __builtin_ldexp(1.0, 52 - bits_of(row.V));
    double sum = 0.0;
    each(row, from + (int)threadIdx.x, to, kThreads, [&](const float (&v)[T::kPer], int) {
#pragma unroll
        for (int e = 0; e < T::kPer; ++e) {
            const double y = weight(v[e]);
            sum += y;
            if (good & (v[e] >= bottom))
                atomicAdd(&s.hist[bins.of(v[e])], __builtin_bit_cast(u64, y + magic) - __builtin_bit_cast(u64, magic));
        }
    });
    return sum;
}

// The largest logit of pieces from .. to and, of equal ones, the lowest index:
// this thread's.
template <class T>
__device__ __forceinline__ u64 best_of(const Row<T> &row, int from, int to, float &best) {
    int at = 0;
    best = -INFINITY;
    each(row, from + (int)threadIdx.x, to, kThreads, [&](const float (&v)[T::kPer], int i0) {
#pragma unroll
        for (int e = 0; e < T::kPer; ++e)
            if (v[e] > best) {
                best = v[e];
                at = i0 + e;
            }
    });
    return key_of(best) ? entry_of(key_of(best), at) : 0;
}

// The largest entry of the workgroup, and the complement of its least key.
__device__ __forceinline__ void block_range(Lds &s, u64 mine, u64 &top, u64 &low) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const u64 first = wave_max(mine), least = wave_max(mine ? ~(mine >> 32) : 0);
    if (lane == 0) s.whole[w] = first, s.least[w] = least;
    __syncthreads();
    top = wave_max(lane < kWaves ? s.whole[lane] : 0);
    low = wave_max(lane < kWaves ? s.least[lane] : 0);
    __syncthreads();
}

// Calls of few rows: each row's readings by `slices` workgroups, so that the chip
// is filled, in a launch each; k_sample then takes what they found.  64 rows of
// 131072 with top_p 0.9: 100 us by one workgroup a row, 59 so.
template <class T>
__device__ __forceinline__ int slice_of(const Row<T> &row, int slices) { return (row.pieces + slices - 1) / slices; }

template <class T>
__global__ __launch_bounds__(kThreads) void k_sample_tops(SampleLaunch a) {
    Lds &s = lds();
    const int r = blockIdx.x / a.slices, g = blockIdx.x - r * a.slices;
    if (T::kBytes == 2 && goes_by_values<T>(settings_of(a, r), a.vocab)) return;
    const Row<T> row(a, r);
    row.read_ends();
    __syncthreads();
    const int n = slice_of(row, a.slices);
    float best;
    u64 top, low;
    const u64 mine = best_of(row, g * n, min(row.pieces, (g + 1) * n), best);
    block_range(s, mine, top, low);
    a.best[(int64_t)blockIdx.x * kThreads + threadIdx.x] = best;
    if (threadIdx.x == 0) a.tops[blockIdx.x] = top, a.lows[blockIdx.x] = low;
}

// What the slices have found, all of it asked for at once: a round trip to what
// another chiplet has written takes a microsecond.
__device__ __forceinline__ void tops_of(const SampleLaunch &a, int r, u64 &top, u64 &low, Mine<kSlices> &mine) {
    const int lane = threadIdx.x & 63;
    const bool has = lane < a.slices;
    const u64 its_top = has ? a.tops[r * a.slices + lane] : 0, its_low = has ? a.lows[r * a.slices + lane] : 0;
    const float *const best = a.best + (int64_t)r * a.slices * kThreads + threadIdx.x;
#pragma unroll
    for (int g = 0; g < kSlices; ++g) mine.best[g] = g < a.slices ? best[g * kThreads] : -INFINITY;
    top = wave_max(its_top);
    low = wave_max(its_low);
}

// Sums of the rows that need all weights: by bins for top_p, of each wave's part
// without cuts.
template <class T>
__global__ __launch_bounds__(kThreads) void k_sample_sums(SampleLaunch a) {
    Lds &s = lds();
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, r = blockIdx.x / a.slices, g = blockIdx.x - r * a.slices;
    const Settings set = settings_of(a, r);
    if (T::kBytes == 2 && goes_by_values<T>(set, a.vocab)) return;
    u64 first, low;
    Mine<kSlices> mine;
    tops_of(a, r, first, low, mine);
    const bool nucleus = by_nucleus(set, a.vocab);
    if (!good(set) || set.temperature == 0.0 || set.top_k == 1 || first == 0 || !(nucleus || uncut(set, a.vocab))) return;
    const float top = logit_of(first);
    if (__builtin_isinf(top)) return;
    const Row<T> row(a, r);
    row.read_ends();
    if (tid < kTable) s.table[tid] = exp2(tid * (1.0 / kTable));
    clear_bins(s);
    __syncthreads();
    const Weight weight = weight_of(set, top);
    const int n = slice_of(row, a.slices), from = g * n, to = min(row.pieces, from + n);
    if (nucleus) {
        const float bottom = nucleus_bottom(s, set, weight, top, row.V, mine);
        if (g == 0 && tid == 0) a.bottoms[r] = bottom;
        double whole;
        block_upto(sum_by_bins(s, row, from, to, weight, Bins(top, bottom), bottom), s.real, whole);
        if (tid == 0) a.parts[(int64_t)blockIdx.x * kWaves] = whole;
        for (int i = tid; i < kBins; i += kThreads) a.hist[(int64_t)blockIdx.x * kBins + i] = s.hist[i];
    } else {
        const int n16 = (n + kWaves - 1) / kWaves;
        double sum = 0.0;
        each(row, from + w * n16 + lane, min(to, from + (w + 1) * n16), 64, [&](const float (&v)[T::kPer], int) {
#pragma unroll
            for (int e = 0; e < T::kPer; ++e) sum += weight(v[e]);
        });
        sum = wave_add(sum);
        if (lane == 0) a.parts[(int64_t)blockIdx.x * kWaves + w] = sum;
    }
}

// The lowest logit that may be kept by rows whose tokens are listed: small top_k,
// or min_p alone.  At least top_k tokens reach the top_k-th largest of the threads'
// largest logits.
template <int N>
__device__ __forceinline__ float list_bottom(Lds &s, const Settings &set, float top, u64 low, bool small_k, const Mine<N> &mine) {
    float bottom = -3.402823466e38f;
    if (set.min_p > 0.0 && set.top_p >= 1.0) bottom = logit_below(set, top, set.min_p);
    if (small_k) {
        const Bins of_threads(top, value_of(~(uint32_t)low));
        if (of_threads.good()) {
            for (float best : mine.best)
                if (best > -INFINITY) atomicAdd(&s.hist[of_threads.of(best)], 1ull);
            __syncthreads();
            const int bin = bin_at(s, (u64)set.top_k);
            if (bin >= 0) bottom = fmaxf(bottom, of_threads.under(bin));
        }
    }
    return bottom;
}
__device__ __forceinline__ bool has_small_k(const Settings &x, int V) { return x.top_k > 0 && x.top_k < V && x.top_k <= kSmallK; }
// What is gathered over its bottom is kept, as far as min_p leaves it.
__device__ __forceinline__ bool only_min_p(const Settings &x, int V) {
    return x.top_p >= 1.0 && x.min_p > 0.0 && !(x.top_k > 0 && x.top_k < V);
}

// The slices' sums by bins, this thread's two, and of all.  (Asked for ahead of
// what the launch does first.)
struct SlicesSums {
    u64 bin[kSlices][2];
    double its[kSlices];
};
__device__ __forceinline__ SlicesSums sums_of_slices(const SampleLaunch &a, int r) {
    SlicesSums x;
    const int tid = threadIdx.x;
    const int64_t at = (int64_t)r * a.slices;
#pragma unroll
    for (int g = 0; g < kSlices; ++g) {
        x.its[g] = g < a.slices ? a.parts[(at + g) * kWaves] : 0.0;
        x.bin[g][0] = g < a.slices ? a.hist[(at + g) * kBins + tid] : 0;
        x.bin[g][1] = g < a.slices ? a.hist[(at + g) * kBins + kThreads + tid] : 0;
    }
    return x;
}

// The bin of top_p's cut, from these; -1 if none, kBins if they do not reach it, as where min_p cuts before it.
// `whole`: the sum of all weights.
__device__ __forceinline__ int cut_of_slices(Lds &s, const SlicesSums &x, const Settings &set, int V, const Bins &bins,
                                             double &whole) {
    const int tid = threadIdx.x;
    u64 sum0 = 0, sum1 = 0;
    whole = 0.0;
#pragma unroll
    for (int g = 0; g < kSlices; ++g) whole += x.its[g], sum0 += x.bin[g][0], sum1 += x.bin[g][1];
    s.hist[tid] = sum0, s.hist[kThreads + tid] = sum1;
    __syncthreads();
    int cut = -1;
    if (bins.good()) cut = bin_at(s, aim_of(set.top_p, whole, bits_of(V)));
    return bins.good() && cut < 0 && set.min_p > 0.0 ? kBins : cut;
}

// Each slice's tokens that may be kept, or, for top_p over all, those of the bin of
// the cut, and the sums over it of each wave's part.
template <class T>
__global__ __launch_bounds__(kThreads) void k_sample_lists(SampleLaunch a) {
    Lds &s = lds();
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, r = blockIdx.x / a.slices, g = blockIdx.x - r * a.slices;
    const Settings set = settings_of(a, r);
    if (T::kBytes == 2 && goes_by_values<T>(set, a.vocab)) return;
    SlicesSums sums = {};
    float bottom_of_row = 0.0f;
    if (by_nucleus(set, a.vocab)) {
        sums = sums_of_slices(a, r);
        bottom_of_row = a.bottoms[r];
    }
    u64 first, low;
    Mine<kSlices> mine;
    tops_of(a, r, first, low, mine);
    const bool nucleus = by_nucleus(set, a.vocab), small_k = has_small_k(set, a.vocab);
    if (!good(set) || set.temperature == 0.0 || set.top_k == 1 || first == 0) return;
    if (!nucleus && !small_k && !only_min_p(set, a.vocab)) return;
    const float top = logit_of(first);
    if (__builtin_isinf(top)) return;
    const Row<T> row(a, r);
    row.read_ends();
    if (tid < kTable) s.table[tid] = exp2(tid * (1.0 / kTable));
    clear_bins(s);
    __syncthreads();
    const Weight weight = weight_of(set, top);
    const int n = slice_of(row, a.slices), from = g * n, to = min(row.pieces, from + n), n16 = (n + kWaves - 1) / kWaves;
    int count;
    if (nucleus) {
        const float bottom = bottom_of_row;
        const Bins bins(top, bottom);
        double whole, over = 0.0, part = 0.0, all;
        const int cut = cut_of_slices(s, sums, set, a.vocab, bins, whole);
        if (g == 0 && tid == 0) a.cuts[r] = cut, a.wholes[r] = whole;
        if (cut < 0) return;
        count = sums_over_bin(row, from, to, n16, set, weight, bins, bottom, cut, over, part);
        block_upto(over, s.real, all);
        part = wave_add(part);
        if (lane == 0) a.kept[(int64_t)blockIdx.x * kWaves + w] = part;
        if (tid == 0) a.over[blockIdx.x] = all;
    } else {
        const float bottom = list_bottom(s, set, top, low, small_k, mine);
        count = gather(row, from, to, n16, true, [&](float v) { return v >= bottom; });
    }
    if (tid == 0) a.counts[blockIdx.x] = count;
    if (count < kMany)
        for (int i = tid; i < count; i += kThreads) a.lists[(int64_t)blockIdx.x * (kMany - 1) + i] = s.list[i];
}

// The least entry of the list's n.
__device__ __forceinline__ u64 block_bottom(Lds &s, int n) {
    u64 x = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) x = larger(x, ~s.list[i]);
    return ~block_max(x, s);
}

// The slices' lists, one behind the other; returns how many tokens they are, kMany
// if they do not fit.
__device__ __forceinline__ int lists_of(Lds &s, const SampleLaunch &a, int r) {
    const int lane = threadIdx.x & 63;
    const int its = lane < a.slices ? a.counts[r * a.slices + lane] : 0;
    int n = 0;
    for (int g = 0; g < a.slices; ++g) {
        const int count = __builtin_amdgcn_readlane(its, g);
        if (n + count >= kMany) return kMany;
        const u64 *const list = a.lists + (int64_t)(r * a.slices + g) * (kMany - 1);
        for (int i = threadIdx.x; i < count; i += kThreads) s.list[n + i] = list[i];
        n += count;
    }
    __syncthreads();
    return n;
}

// The part of the row in which the sums of `sum` (this thread's part of the
// slices' waves) pass u of their whole.
template <class T>
__device__ __forceinline__ Part part_of(Lds &s, const Row<T> &row, int slices, double sum, double u, double &whole) {
    const int tid = threadIdx.x, n = slice_of(row, slices), n16 = (n + kWaves - 1) / kWaves;
    const double upto = block_upto(sum, s.real, whole), t = u * whole;
    if (tid == 0) s.found = kThreads;
    __syncthreads();
    if (sum > 0.0 && upto > t) atomicMin(&s.found, tid);
    __syncthreads();
    if (tid == s.found) s.share = t - (upto - sum);
    __syncthreads();
    const int g = s.found / kWaves, from = g * n + s.found % kWaves * n16;
    return {from, min(min(row.pieces, (g + 1) * n), from + n16), s.share};
}

// 16-bit logits are few values, and what is kept is a stretch of these: of its
// last value the first `need` tokens.  One reading counts each value's tokens, the
// cuts are found among the values, and a second reading adds up weights from a
// table.  Values by falling order: 0 is the bits 0x7fff, 32767 is 0, and from there
// on they are the bits themselves.
__device__ __forceinline__ int turned(int x) { return x < 0x8000 ? 0x7fff - x : x; }  // bits to order, and back
template <class T>
__device__ __forceinline__ int order_of(float v) { return turned((int)T::bits(v + 0.0f)); }  // -0 is 0

struct Kept {
    int upto, need;  // the values before `upto`, and so many tokens of it
};

// The first of n stretches with which the sums of size(stretch) reach the target,
// n - 1 if none; `before`: the sum of those before it.  (One wave's work.)
template <class I, class Size>
__device__ __forceinline__ int stretch_at(int n, I target, Size size, I &before) {
    const int lane = threadIdx.x & 63;
    I sum = 0;
    for (int base = 0;; base += 64) {
        const int i = base + lane;
        const I upto = sum + wave_upto(i < n ? size(i) : I(0));
        const u64 reach = __ballot(i < n && upto >= target);
        if (reach || base + 64 >= n) {
            const int at = reach ? __builtin_amdgcn_readfirstlane(__ffsll(reach) - 1) : n - 1 - base;
            before = at ? of_lane(upto, at - 1) : sum;
            return base + at;
        }
        sum = of_lane(upto, 63);
    }
}

// This lane's value of a stretch: its place in the order, its tokens, its weight.
template <class T>
__device__ __forceinline__ int value_in(const Values &s, const Weight &weight, int stretch, int &count, double &w) {
    const int order = s.first[stretch] + (int)(threadIdx.x & 63);
    count = ((const uint16_t *)s.counts)[turned(order)];
    w = count ? weight(T::of_bits(turned(order))) : 0.0;
    return order;
}

// What the settings keep of a row with n stretches.
template <class T>
__device__ __forceinline__ Kept cuts_of(const Values &s, const Settings &set, const Weight &weight, int V, int n) {
    int count, last = n - 1;
    double w, before, whole;
    int order = value_in<T>(s, weight, last, count, w);
    const int end = 63 - __clzll(__ballot(count > 0));  // (a stretch has a token)
    Kept kept = {__builtin_amdgcn_readlane(order, end) + 1, 0};
    if (set.top_k > 0 && set.top_k < V) {
        u64 tokens;
        const int at = stretch_at<u64>(n, (u64)set.top_k, [&](int i) { return (u64)s.num[i]; }, tokens);
        order = value_in<T>(s, weight, at, count, w);
        const u64 upto = tokens + wave_upto((u64)count), reach = __ballot(upto >= (u64)set.top_k);
        if (reach) {
            const int i = __builtin_amdgcn_readfirstlane(__ffsll(reach) - 1);
            last = at;
            kept = {__builtin_amdgcn_readlane(order, i),
                    (int)((u64)set.top_k - of_lane(upto, i)) + __builtin_amdgcn_readlane(count, i)};
        }
    }
    // of the last stretch, what is kept so far
    order = value_in<T>(s, weight, last, count, w);
    const double rest = wave_add((order < kept.upto ? count : order == kept.upto ? kept.need : 0) * w);
    auto sum = [&](int i) { return i == last ? rest : s.sum[i]; };
    if (set.top_p < 1.0) {
        stretch_at<double>(last + 1, INFINITY, sum, whole);
        const double aim = set.top_p * (whole + rest);
        const int at = stretch_at<double>(last + 1, aim, sum, before);
        order = value_in<T>(s, weight, at, count, w);
        count = order < kept.upto ? count : order == kept.upto ? kept.need : 0;
        before += wave_upto(count * w) - count * w;
        const u64 some = __ballot(count > 0), less = __ballot(count > 0 && before < aim);
        const int i = __builtin_amdgcn_readfirstlane(less ? 63 - __clzll(less) : __ffsll(some) - 1);
        const double need = __builtin_ceil((aim - before) / w);  // tokens of the value before which less than top_p lies
        kept = {__builtin_amdgcn_readlane(order, i),
                __builtin_amdgcn_readlane(need >= count ? count : need > 1.0 ? (int)need : 1, i)};
    }
    if (set.min_p > 0.0)
        for (int i = 0; i < n && s.first[i] <= kept.upto; ++i) {
            order = value_in<T>(s, weight, i, count, w);
            const u64 less = __ballot(count > 0 && w < set.min_p);
            if (less) {
                order = __builtin_amdgcn_readlane(order, __builtin_amdgcn_readfirstlane(__ffsll(less) - 1));
                if (order <= kept.upto) kept = {order, 0};
                break;
            }
        }
    return kept;
}

// Weights of the values first .. upto - 1, and 0 behind them; of more than fit,
// all but `gap` from `hole` on, next to zero, which are worked out where they occur.
template <class T>
struct Table {
    Weight weight;
    int first, upto, hole, gap;
    __device__ __forceinline__ Table(const Weight &w, int f, int u) : weight(w), first(f), upto(u) {
        gap = max(0, upto - first - (kWeights - 1));
        hole = min(max(0x8000 - gap / 2, first), upto - gap);
    }
    __device__ __forceinline__ void fill(Values &s) const {
        const int n = upto - first - gap;
        for (int i = threadIdx.x; i <= n; i += kThreads) {
            const int order = first + i + (first + i < hole ? 0 : gap);
            s.weights[i] = i < n ? weight(T::of_bits(turned(order))) : 0.0;
        }
    }
    // (NaN comes before `first` or behind `upto`, -infinity behind it or at it, where nothing is kept then)
    template <bool GAP>
    __device__ __forceinline__ double of(const Values &s, int order, float v) const {
        const uint32_t i = min((uint32_t)(order - first), (uint32_t)(upto - first));
        if (!GAP) return s.weights[i];
        if (order >= hole && order < hole + gap) return weight(v);
        return s.weights[order < hole && order >= first ? i : i - gap];
    }
};

// Of some tokens, the sum of the weights of values that are kept, and how many have
// the last of them.
struct Sums {
    double sum;
    int ties;
};
template <bool GAP, class T>
__device__ __forceinline__ Sums sums_of(const Values &s, const Row<T> &row, const Table<T> &table, int from, int to, int step) {
    Sums x = {0.0, 0};
    each(row, from, to, step, [&](const float (&v)[T::kPer], int) {
#pragma unroll
        for (int e = 0; e < T::kPer; ++e) {
            const int order = order_of<T>(v[e]);
            x.sum += table.template of<GAP>(s, order, v[e]);
            x.ties += order == table.upto;
        }
    });
    return x;
}

// The token, from the table and `need` ties: a sixteenth of the row, a sixteenth of
// that, and there a lane's pieces.
template <bool GAP, class T>
__device__ __forceinline__ void token_by_table(Lds &all_of, const Row<T> &row, const Table<T> &table, double tie, int need, double u) {
    const Values &s = all_of.values;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int from = 0, to = row.pieces, left = need;  // left: ties that are still to be kept
    double t = 0.0, total = 0.0;
#pragma nounroll
    for (int level = 0; level < 2; ++level) {
        const int per = (to - from + kWaves - 1) / kWaves;
        const Sums x = sums_of<GAP>(s, row, table, from + wave * per + lane, min(to, from + (wave + 1) * per), 64);
        const double its = wave_add(x.sum);
        const u64 ties = wave_add((u64)x.ties);
        if (lane == 0) all_of.real[wave] = its, all_of.counts[wave] = (int)ties;
        __syncthreads();
        const int mine = lane < kWaves ? all_of.counts[lane] : 0;
        const int my_left = max(0, left - (int)(wave_upto((u64)mine) - (u64)mine));
        const double sum = lane < kWaves ? all_of.real[lane] + min(my_left, mine) * tie : 0.0, upto = wave_upto(sum);
        if (level == 0) {
            total = of_lane(upto, 63);
            t = u * total;
        }
        const u64 past = __ballot(sum > 0.0 && upto > t), some = __ballot(sum > 0.0);
        const int part = __builtin_amdgcn_readfirstlane(past ? __ffsll(past) - 1 : some ? 63 - __clzll(some) : 0);
        t -= of_lane(upto - sum, part);
        left = __builtin_amdgcn_readlane(my_left, part);
        from += part * per;
        to = min(to, from + per);
        __syncthreads();
    }
    if (wave == 0) {
        const int its = (to - from + 63) / 64, mine = from + lane * its, end = min(to, mine + its);
        const Sums x = sums_of<GAP>(s, row, table, mine, end, 1);
        const int my_left = max(0, left - (int)(wave_upto((u64)x.ties) - (u64)x.ties));
        const double sum = x.sum + min(my_left, x.ties) * tie, upto = wave_upto(sum);
        const u64 past = __ballot(sum > 0.0 && upto > t), some = __ballot(sum > 0.0);
        const int who = past ? __ffsll(past) - 1 : some ? 63 - __clzll(some) : 0;
        if (lane == who) {
            double at = upto - sum, share = 0.0;
            int index = 0, ties = 0;
            bool done = false;
            each(row, mine, end, 1, [&](const float (&v)[T::kPer], int i0) {
                for (int e = 0; e < T::kPer; ++e) {
                    const int order = order_of<T>(v[e]);
                    const bool tied = order == table.upto && ties < my_left;
                    const double w = tied ? tie : table.template of<GAP>(s, order, v[e]);
                    ties += tied;
                    if (!done && w > 0.0) {
                        index = i0 + e;
                        share = w;
                        at += w;
                        done = at > t;
                    }
                }
            });
            all_of.found = index;
            all_of.share = share / total;
        }
    }
    __syncthreads();
}

// The token and its share, by values; false where a count does not fit 16 bits, or
// infinities or no tokens are there.
template <class T>
__device__ __noinline__ bool by_values(Row<T> row, Settings set, Answer &answer) {
    Lds &all_of = lds();
    Values &s = all_of.values;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int i = tid; i < kValues / 8; i += kThreads) ((u32x4 *)s.counts)[i] = u32x4{0, 0, 0, 0};
    if (tid == 0) all_of.found = 0;
    __syncthreads();
    int tokens = 0;
    each(row, tid, row.pieces, kThreads, [&](const float (&v)[T::kPer], int) {
#pragma unroll
        for (int e = 0; e < T::kPer; ++e)
            if (v[e] > -INFINITY) {
                const uint32_t bits = T::bits(v[e] + 0.0f);  // -0 is 0
                atomicAdd(&s.counts[bits >> 1], bits & 1 ? 0x10000u : 1u);
                ++tokens;
            }
    });
    tokens = (int)wave_add((u64)tokens);
    if (lane == 0) atomicAdd(&all_of.found, tokens);
    __syncthreads();
    // a thread's stretch: its tokens.  (A count that has passed 65535 makes the sum of all less than it should be.)
    const int start = (tid < kStretches / 2 ? kStretches / 2 - 1 - tid : tid) * (kStretch / 8);
    int count = 0;
    for (int i = 0; i < kStretch / 8; ++i) {
        const u32x4 x = ((const u32x4 *)s.counts)[start + (i + tid) % (kStretch / 8)];
#pragma unroll
        for (int e = 0; e < 4; ++e) count += (int)(x[e] & 0xffff) + (int)(x[e] >> 16);
    }
    u64 found;
    const int at = (int)(block_upto((u64)(count > 0) << 32 | (uint32_t)count, all_of.whole, found) >> 32);
    const int n = (int)(found >> 32);
    if (count > 0) s.num[at - 1] = count, s.first[at - 1] = tid * kStretch;
    __syncthreads();
    if (n == 0 || (int)(uint32_t)found != all_of.found || ((const uint16_t *)s.counts)[T::kInfinity] > 0) return false;
    const int top = s.first[0] + __ffsll(__ballot(((const uint16_t *)s.counts)[turned(s.first[0] + lane)] > 0)) - 1;
    const Weight weight = weight_of(set, T::of_bits(turned(top)));
    for (int i = wave; i < n; i += kWaves) {
        double w;
        value_in<T>(s, weight, i, count, w);
        const double sum = wave_add(count * w);
        if (lane == 0) s.sum[i] = sum;
    }
    __syncthreads();
    if (wave == 0) {
        const Kept x = cuts_of<T>(s, set, weight, row.V, n);
        if (lane == 0) all_of.counts[0] = x.upto, all_of.counts[1] = x.need;
    }
    __syncthreads();
    const Kept kept = {all_of.counts[0], all_of.counts[1]};
    const Table<T> table(weight, top, kept.upto);
    table.fill(s);
    const double tie = weight(T::of_bits(turned(kept.upto)));
    __syncthreads();
    if (table.gap) token_by_table<true>(all_of, row, table, tie, kept.need, set.u);
    else token_by_table<false>(all_of, row, table, tie, kept.need, set.u);
    answer = {all_of.found, all_of.share};
    return true;
}

// SLICED: the launches above have gone before.
template <class T, bool SLICED>
__global__ __launch_bounds__(kThreads) void k_sample(SampleLaunch a) {
    Lds &s = lds();
    const int tid = threadIdx.x, r = blockIdx.x;
    const Settings set = settings_of(a, r);
    auto answer = [&](int token, double share) {
        if (tid == 0) {
            a.token[r] = token;
            if (a.logprob) a.logprob[r] = (float)log(share);
        }
    };
    if (!good(set)) {
        if (tid == 0 && a.status) a.status[r] = FATE_EINVAL;
        answer(-1, 0.0);
        return;
    }
    // (of the slices, asked for ahead of what comes first; used where they have left it)
    int cut_of_row = -1;
    double whole_of_row = 0.0, its_over = 0.0, its_kept = 0.0;
    if constexpr (SLICED)
        if (by_nucleus(set, a.vocab)) {
            cut_of_row = a.cuts[r];
            whole_of_row = a.wholes[r];
            its_over = (tid & 63) < a.slices ? a.over[r * a.slices + (tid & 63)] : 0.0;
            its_kept = tid < a.slices * kWaves ? a.kept[(int64_t)r * a.slices * kWaves + tid] : 0.0;
        }
    const Row<T> row(a, r);
    row.read_ends();
    if (tid < kTable) s.table[tid] = exp2(tid * (1.0 / kTable));
    clear_bins(s);
    __syncthreads();

    Answer x;
    bool sliced = SLICED;  // not where by_values has not been the way after all
    if constexpr (T::kBytes == 2)
        if (goes_by_values<T>(set, row.V)) {
            if (by_values(row, set, x)) {
                answer(x.token, x.share);
                return;
            }
            sliced = false;
            __syncthreads();
            clear_bins(s);
            __syncthreads();
        }

    u64 first = 0, low = 0;
    Mine<SLICED ? kSlices : 1> mine;
    if constexpr (SLICED)
        if (sliced) tops_of(a, r, first, low, mine);
    if (!sliced) block_range(s, best_of(row, 0, row.pieces, mine.best[0]), first, low);
    if (first == 0) {  // nothing to choose from
        answer(-1, 0.0);
        return;
    }
    if (set.temperature == 0.0 || set.top_k == 1) {
        answer(index_of(first), 1.0);
        return;
    }
    const float top = logit_of(first);
    const Weight weight = weight_of(set, top);
    if (__builtin_isinf(top)) {
        const Answer x = token_at_infinity(row, set, (float)set.top_p);
        answer(x.token, x.share);
        return;
    }

    const bool cuts_k = set.top_k > 0 && set.top_k < row.V, small_k = has_small_k(set, row.V);
    const bool nucleus = by_nucleus(set, row.V);
    Place kept = {-INFINITY, kAll};
    bool known = false;        // s.real has the sums of the sixteenths
    Part part = {0, 0, 0.0};   // or the part that the token lies in is known
    double whole = 0.0;
    if (nucleus) {
        if constexpr (SLICED) {
            const int cut = sliced ? cut_of_row : -1;
            if (sliced) whole = whole_of_row;
            if (cut >= 0) {
                double sum = its_kept;
                const int n = lists_of(s, a, r);
                const double above = wave_add(its_over);
                const u64 last = cut == kBins ? (u64)min_p_cuts(set, above, whole) : n < kMany ? last_in_bin(set, weight, n, above, whole) : 0;
                if (last) {
                    if (cut < kBins) kept = {logit_of(last), index_of(last)};
                    // of the bin's tokens, those kept count for their parts
                    if (tid < n) {
                        const int its = slice_of(row, a.slices), n16 = (its + kWaves - 1) / kWaves;
                        const u64 y = s.list[tid];
                        const int piece = (index_of(y) + row.lead) / T::kPer, g = piece / its;
                        const double z = y >= last ? weight(logit_of(y)) : 0.0;
                        s.ranked[tid].entry = g * kWaves + (piece - g * its) / n16;
                        s.ranked[tid].weight = z >= set.min_p ? z : 0.0;
                    }
                    __syncthreads();
                    if (tid < a.slices * kWaves)
                        for (int j = 0; j < n; ++j) sum += s.ranked[j].entry == (u64)tid ? s.ranked[j].weight : 0.0;
                    part = part_of(s, row, a.slices, sum, set.u, whole);
                }
            }
        } else {
            const float bottom = nucleus_bottom(s, set, weight, top, row.V, mine);
            const Bins bins(top, bottom);
            block_upto(sum_by_bins(s, row, 0, row.pieces, weight, bins, bottom), s.real, whole);
            const int bits = bits_of(row.V);
            int cut = bins.good() ? bin_at(s, aim_of(set.top_p, whole, bits)) : -1;
            if (bins.good() && cut < 0 && set.min_p > 0.0) cut = kBins;  // min_p may cut before top_p does
            if (cut >= 0) {  // how many it keeps, about: a bin's sum by the weight in its middle
                double n = 0.0, all;
                for (int b = 2 * tid; b < 2 * tid + 2 && b <= cut; ++b)
                    if (s.hist[b]) n += __builtin_ldexp((double)s.hist[b], -bits) / weight(top - ((float)b + 0.5f) / bins.per);
                block_upto(n, s.real, all);
                if (all <= kRanked) {
                    const int listed = gather(row, 0, row.pieces, sixteenth(row), false, [&](float v) {
                        return (v >= bottom) & (bins.of(v) <= cut);
                    });
                    if (listed <= kRanked) {
                        x = from_short(set, weight, listed, whole);
                        answer(x.token, x.share);
                        return;
                    }
                }
                known = cut_in_bin(row, set, weight, bins, bottom, cut, whole, kept);
            }
        }
    } else if (small_k || only_min_p(set, row.V)) {
        int n = 0;
        float bottom = -3.402823466e38f;
        const bool in_order = SLICED || (small_k && set.top_k > kRanked);  // as many at least are listed, too many to be ranked
        if constexpr (SLICED) {
            n = sliced ? lists_of(s, a, r) : kMany;
            if (n < kMany && n > 0) bottom = logit_of(block_bottom(s, n));
        } else {
            bottom = list_bottom(s, set, top, low, small_k, mine);
            n = gather(row, 0, row.pieces, sixteenth(row), in_order, [&](float v) { return v >= bottom; });
        }
        if (n <= kRanked) {
            x = from_short(set, weight, n, 0.0);
            answer(x.token, x.share);
            return;
        }
        if (!in_order && n < kMany) n = gather(row, 0, row.pieces, sixteenth(row), true, [&](float v) { return v >= bottom; });
        // (of few threads' largest logits no bound follows: the bins go by the least that is listed)
        if (!SLICED && n < kMany && small_k && bottom == -3.402823466e38f) bottom = logit_of(block_bottom(s, n));
        const Bins bins(top, bottom);
        if (n < kMany && (small_k ? bins.good() && from_list_of_k(set, weight, n, bins, x) : (x = from_list(set, weight, n, 1), true))) {
            answer(x.token, x.share);
            return;
        }
    } else if (SLICED && uncut(set, row.V)) {
        part = part_of(s, row, a.slices, tid < a.slices * kWaves ? a.parts[(int64_t)r * a.slices * kWaves + tid] : 0.0, set.u, whole);
    }
    const bool parted = part.to > 0;
    if (!known && !parted && (cuts_k || set.top_p < 1.0)) kept = by_digits(row, set, weight, (float)set.top_p);
    x = token_at(row, set, weight, kept, known, parted, part, whole);
    answer(x.token, x.share);
}

}  // namespace

// Workgroups of a row's slices: calls of up to 128 rows by as many as the chip
// runs at once, of 32768 logits each at least.  The three launches more cost some
// 10 us.  By one workgroup a row and by slices of 32768, us, 1 and 64 rows:
//   131072  top-p 0.9 93 and 51, 100 and 59; no cut 41 and 23, 44 and 30; top-k 1000 42 and 32, 45 and 36; top-k 50 21 and 23,
//           23 and 28; min-p 18 and 21, 21 and 26
//   64 rows of 32768 by one and by two  top-p 0.9 42 and 43, no cut 17 and 22, top-k 50 14 and 24
// Where the host knows that a call's rows list few tokens at once, it is one, for rows of up to 131072, the longest
// measured so.
int sample_slices(int64_t rows, int64_t vocab) {
    const int64_t fill = rows > 0 ? 256 / rows : 1, most = vocab / 32768;
    const int64_t n = fill < most ? fill : most;
    return n < 2 ? 1 : n > kSlices ? kSlices : (int)n;
}

size_t sample_ws(int64_t rows, int64_t vocab) {
    const int n = sample_slices(rows, vocab);
    if (n == 1) return 0;
    return (size_t)rows * n * ((2 + kMany - 1 + kBins) * sizeof(u64) + (2 * kWaves + 1) * sizeof(double) +
                               kThreads * sizeof(float) + sizeof(int32_t)) +
           (size_t)rows * (sizeof(double) + sizeof(int32_t) + sizeof(float));
}

namespace {

template <class T>
void go(SampleLaunch a, void *ws, hipStream_t s) {
    const dim3 block(kThreads);
    const bool by_values = !a.temperature && !a.top_k && !a.top_p &&
                           by_values_pays<T>(a.temperature_all, a.top_k_all, a.top_p_all, a.vocab);
    const bool largest = !a.temperature && a.temperature_all == 0.0f;
    const bool small_k = !a.top_k && a.top_k_all > 0 && a.top_k_all <= 256;
    const bool only_min_p = !a.top_k && !a.top_p && !a.min_p && a.top_k_all == 0 && a.top_p_all >= 1.0f && a.min_p_all > 0.0f;
    const bool listed = a.vocab <= 1 << 17 && (largest || small_k || only_min_p);
    a.slices = by_values || listed ? 1 : sample_slices(a.rows, a.vocab);
    if (a.slices == 1) {
        hipLaunchKernelGGL((k_sample<T, false>), dim3((unsigned)a.rows), block, 0, s, a);
        return;
    }
    const int64_t n = (int64_t)a.rows * a.slices;
    a.tops = static_cast<unsigned long long *>(ws);
    a.lows = a.tops + n;
    a.hist = a.lows + n;
    a.parts = reinterpret_cast<double *>(a.hist + n * kBins);
    a.kept = a.parts + n * kWaves;
    a.over = a.kept + n * kWaves;
    a.wholes = a.over + n;
    a.lists = reinterpret_cast<unsigned long long *>(a.wholes + a.rows);
    a.best = reinterpret_cast<float *>(a.lists + n * (kMany - 1));
    a.counts = reinterpret_cast<int32_t *>(a.best + n * kThreads);
    a.cuts = a.counts + n;
    a.bottoms = reinterpret_cast<float *>(a.cuts + a.rows);
    hipLaunchKernelGGL((k_sample_tops<T>), dim3((unsigned)n), block, 0, s, a);
    hipLaunchKernelGGL((k_sample_sums<T>), dim3((unsigned)n), block, 0, s, a);
    hipLaunchKernelGGL((k_sample_lists<T>), dim3((unsigned)n), block, 0, s, a);
    hipLaunchKernelGGL((k_sample<T, true>), dim3((unsigned)a.rows), block, 0, s, a);
}

}  // namespace

int launch_sample(const SampleLaunch &a, void *ws, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (a.dtype == FATE_BF16) go<B16>(a, ws, s);
    else if (a.dtype == FATE_F16) go<H16>(a, ws, s);
    else go<F32>(a, ws, s);
    return (int)hipGetLastError();
}

}  // namespace fate
