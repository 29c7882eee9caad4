// Shared by the attention kernels of a planned wave: launch arguments, types
// of the matrix instructions, and the search of a workgroup's piece of work.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fate.h"

namespace fate {

struct RowsArg {
    char *data;
    int64_t token, head;  // elements
};

struct SeqsArg {
    const int32_t *off, *kv_len, *pages;
    int64_t T, pages_stride, max_keys;  // max_keys = max_pages * page_size
    int32_t B;
};

struct CacheArg {
    const char *k, *v;
    int64_t page, head, token;  // elements
    int32_t n_pages, page_shift;
};

struct AppendLaunch {
    SeqsArg s;
    RowsArg q, k, v, qo;
    char *ck, *cv;
    CacheArg c;
    const float *table;
    int32_t *status;
    int64_t table_rows;
    int32_t hq, hkv, d, rot, interleaved, dtype;
    int32_t past_cache;  // the call moves more than the last-level cache holds
};
int launch_append(const AppendLaunch &a, void *stream);

// Tokens of an append's workgroup in large calls: its first wave finds them all
// at once.  Four: 82 us for 18261 tokens (48 heads of 128), 30.5 for 5579; two 80
// and 32.5, eight 96 and 41, one 83 and 31.  One in calls of up to 1024, where
// four leave compute units idle: 5.4 against 9.1 us for 64 tokens, 9.1 against
// 12.2 for 1024 (for 2048 one would take 12.9 against four's 14.1, for 4096 20.6
// against 24.4).
constexpr int kAppendTokens = 4;
inline int append_tokens(int64_t T) { return T <= 1024 ? 1 : kAppendTokens; }
inline int64_t append_grid(int64_t T) { return (T + append_tokens(T) - 1) / append_tokens(T); }

// Attention over pages (kv in CacheArg) or over packed rows (k, v).  Rows of
// one key head are packed for the matrix tiles: packed row r of a sequence is
// token r / G, query head hk * G + r % G, G = heads_q / heads_kv.
struct AttnLaunch {
    SeqsArg s;
    RowsArg q, k, v, out;
    CacheArg c;
    float *lse;       // [T][hq] or null
    int32_t *status;  // [B] or null
    float *part;      // partial outputs [2 pieces][hkv][rows][d], then (max, sum) pairs [2 pieces][hkv][rows][2]
    float scale_log2; // scale * log2(e)
    int32_t hq, hkv, G, d, dtype;
    int32_t pieces;   // paged calls: shares of the work axis (few rows), or parts aimed at (row tiles), per key head
    int32_t grid;     // workgroups per key head
};
int launch_attn_tile(const AttnLaunch &a, bool paged, void *stream);
int launch_attn_few(const AttnLaunch &a, int rows, void *stream);
int launch_attn_join(const AttnLaunch &a, int rows, int tiles, int groups, void *stream);

constexpr int kKeyTile = 64;    // keys per tile: the unit in which the key axis is split
constexpr int kTileRows = 128;  // packed rows of a workgroup of the tile kernel
// Fewest key tiles of a share: one block of 32 keys for each wave of the
// few-row kernel; enough work to pay for the join in the tile kernel.
constexpr int kFewLeast = 2, kTileLeast = 4;
// What a row tile costs in the few-row kernel beside its keys (finding it, its
// queries, the waves' join, its results), in key tiles.
constexpr int kUnitTiles = 2;

#if defined(__HIPCC__)

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The running maximum m that a row's weights 2^(S - m) refer to (S in units of
// log2) stands kLift below its largest score, or up to kLag above that: the
// largest weight is 2^kLift to 2^(kLift + kLag).  Float16 gives up bits of
// weights under 2^-14 and all of them under 2^-25, which many keys behind one
// large score add up to: 100000 of 2^-25.6 are 0.2% of the result.  Lifted,
// they lose at most 2^-32 of the largest weight each.  The range allows no
// more (2^16); bfloat16 reaches as far down as float32.
constexpr float kLag = 8.0f;

struct BF16 {
    static constexpr float kLift = 0.0f;
    typedef __bf16 el;
    typedef __bf16 x4 __attribute__((ext_vector_type(4)));
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kExp = 0x7f807f80u, kOne = 0x00800080u;  // exponent bits of a pair; their lowest
    static __device__ __forceinline__ f32x16 mfma32(x8 a, x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 mfma16(x8 a, x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ x4 read_tr(const el *p) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) x4 *)p);
    }
    static __device__ __forceinline__ x4 read_tr_at(uint32_t at) {  // LDS byte address
        return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) x4 *)at);
    }
};

struct F16 {
    static constexpr float kLift = 7.0f;
    typedef _Float16 el;
    typedef _Float16 x4 __attribute__((ext_vector_type(4)));
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kExp = 0x7c007c00u, kOne = 0x04000400u;
    static __device__ __forceinline__ f32x16 mfma32(x8 a, x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 mfma16(x8 a, x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ x4 read_tr(const el *p) {
        typedef __fp16 h4 __attribute__((ext_vector_type(4)));
        return __builtin_bit_cast(
            x4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) h4 *)p));
    }
    static __device__ __forceinline__ x4 read_tr_at(uint32_t at) {
        typedef __fp16 h4 __attribute__((ext_vector_type(4)));
        return __builtin_bit_cast(
            x4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) h4 *)at));
    }
};

// Lowest finite value: the running maximum of rows that have seen no key yet.
// Differences from it are finite or -infinity, never NaN.
constexpr float kLowest = -3.402823466e38f;
constexpr float kLn2 = 0.6931471805599453f;

// Nonzero if one of the pair's halves is an infinity or a NaN: the exponent
// bits, plus their lowest bit, carry into the sign's place.
template <class T>
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {
    return ((x & T::kExp) + T::kOne) & 0x80008000u;
}

// The pair with halves that are infinite or NaN set to zero.
template <class T>
__device__ __forceinline__ uint32_t only_finite(uint32_t x) {
    const uint32_t bad = not_finite<T>(x);
    return x & ~((bad & 0x8000u ? 0xffffu : 0u) | (bad & 0x80000000u ? 0xffff0000u : 0u));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
    return (int64_t)(((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32) | (uint32_t)uniform((int)x));
}

// Inclusive sums over the 64 lanes (all active): shifts right by 1, 2, 4 and 8
// within each row of 16 lanes, then the last lanes of rows 0 and 2, and of row
// 1, to the rows after them, in DPP moves as wave_exscan_u32.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int x) {
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t moved(int64_t x) {
    return (int64_t)(((uint64_t)(uint32_t)moved<CTRL, ROWS>((int)(x >> 32)) << 32) |
                     (uint32_t)moved<CTRL, ROWS>((int)x));
}
template <class I>
__device__ __forceinline__ I wave_scan_add(I x) {
    x += moved<0x111, 0xF>(x);
    x += moved<0x112, 0xF>(x);
    x += moved<0x114, 0xF>(x);
    x += moved<0x118, 0xF>(x);
    x += moved<0x142, 0xA>(x);
    x += moved<0x143, 0xC>(x);
    return x;
}

__device__ __forceinline__ int wave_scan_max(int x) {  // of values of at least 0, as which others count
    x = max(x, moved<0x111, 0xF>(x));
    x = max(x, moved<0x112, 0xF>(x));
    x = max(x, moved<0x114, 0xF>(x));
    x = max(x, moved<0x118, 0xF>(x));
    x = max(x, moved<0x142, 0xA>(x));
    x = max(x, moved<0x143, 0xC>(x));
    return x;
}

// Lane i's value, i the same in all lanes.
__device__ __forceinline__ int lane_of(int x, int i) { return __builtin_amdgcn_readlane(x, i); }
__device__ __forceinline__ int64_t lane_of(int64_t x, int i) {
    return (int64_t)(((uint64_t)(uint32_t)lane_of((int)(x >> 32), i) << 32) | (uint32_t)lane_of((int)x, i));
}

template <class I>
__device__ __forceinline__ I wave_sum(I x) { return lane_of(wave_scan_add(x), 63); }

// One sequence as the kernels see it: its first row, tokens and keys; no
// tokens and no keys past the last sequence and where the device arrays are
// out of range (`report`: say so in the status).
struct Lens {
    int lo, n, L;
};

// Lane i: sequence at + i.  `reach`: the largest offset before the group, 0
// for the first; on return, before the next one.  A sequence that starts below
// an earlier offset is out of range: those that are not hold different rows,
// in order, so that the tiles that the host counts from T and B are enough.
template <bool PAGED, class A>
__device__ __forceinline__ Lens read_lens(const A &a, int at, int lane, int &reach, bool report) {
    Lens s = {0, 0, 0};
    const int b = at + lane;
    int hi = 0;
    if (b < a.s.B) {
        s.lo = a.s.off[b];
        hi = a.s.off[b + 1];
        if (PAGED) s.L = a.s.kv_len[b];
    }
    const int before = max(reach, wave_scan_max(s.lo));  // its own offset among them
    reach = lane_of(before, 63);
    s.n = hi - s.lo;
    bool bad = s.lo < before || hi < s.lo || (int64_t)hi > a.s.T;
    if (PAGED) bad = bad || s.L < 0 || (int64_t)s.L > a.s.max_keys;
    else s.L = s.n;
    if (bad || b >= a.s.B) {
        s.lo = s.n = s.L = 0;
        if (report && a.status && b < a.s.B) a.status[b] = FATE_EINVAL;
    }
    return s;
}

// The launch arguments where the kernel finds them.  A workgroup that walks
// through several pieces of work reads them again for each (and its thread
// number goes through fresh()), or the compiler would keep everything that
// does not change between pieces in registers, which the piece itself needs.
typedef const __attribute__((address_space(4))) AttnLaunch Args;

__device__ __forceinline__ const Args &launch_args() {
    const Args *p = (const Args *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *p;
}

__device__ __forceinline__ int fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// The first 64 sequences, and the largest offset before the next.
struct Group {
    Lens lens;
    int reach;
};

template <bool PAGED, class A>
__device__ __forceinline__ Group first_group(const A &a, int lane, bool report) {
    Group g;
    g.reach = 0;
    g.lens = read_lens<PAGED>(a, 0, lane, g.reach, report);
    return g;
}

// The group from sequence `at` on: `first`, or read; `reach` as in read_lens.
template <bool PAGED, class A>
__device__ __forceinline__ Lens group_at(const A &a, int at, int lane, const Group &first, int &reach) {
    if (at > 0) return read_lens<PAGED>(a, at, lane, reach, false);
    reach = first.reach;
    return first.lens;
}

__device__ __forceinline__ int tiles_of(int n, int tile) { return (int)(((int64_t)n + tile - 1) / tile); }

// A row tile: packed rows [tile * M, ...) of sequence b, which has n tokens in
// rows from lo_row and L keys.
struct Unit {
    int b, n, lo_row, L, tile;
    int64_t start, cost;  // its place on the work axis (paged calls)
    bool ok;
};

// ---- calls of few rows: an axis of work, equal shares -----------------------
// The work axis of a paged call.  Its row tiles lie on it one after the other,
// each as long as its cost: G times the keys that its last row sees, about
// G A + (tile + 1) M for a sequence with A keys cached before the call, and
// kUnitTiles more (without these, 37 sequences of six keys were one workgroup's,
// one after the other: 100 us).  The axis is cut into equal shares, one workgroup each, whatever the
// mix of lengths; a tile that a cut goes through is done in parts and joined.
// The lengths are read on the device, where a serving step has them (and a
// captured step finds the current ones), so that every workgroup adds them up
// for itself: B / 64 steps of a wave.
struct Axis {
    int64_t total, share;
};

__device__ __forceinline__ int64_t tile_start(int t, int64_t GA, int M) {
    return t * GA + (int64_t)M * t * (t + 1) / 2;
}

__device__ __forceinline__ int64_t axis_keys(int n, int L, int G) {
    return (int64_t)G * (max(0, L - n) + kUnitTiles * kKeyTile);
}

__device__ __forceinline__ int64_t seq_cost(const Lens &s, int G, int M) {
    return tile_start(tiles_of(s.n * G, M), axis_keys(s.n, s.L, G), M);
}

// `first`: the first 64 sequences, which most calls end with.
template <class A>
__device__ __forceinline__ Axis axis_of(const A &a, int M, const Group &first, int lane, bool report) {
    int64_t sum = seq_cost(first.lens, a.G, M);
    int reach = first.reach;
    for (int at = 64; at < a.s.B; at += 64) sum += seq_cost(read_lens<true>(a, at, lane, reach, report), a.G, M);
    Axis x;
    x.total = wave_sum(sum);
    const int64_t least_share = (int64_t)kFewLeast * kKeyTile * a.G;
    x.share = (x.total + a.pieces - 1) / a.pieces;
    if (x.share < least_share) x.share = least_share;
    return x;
}

// Where the search for a place of the axis stands: a group of 64 sequences,
// the largest offset and the cost before it.  Places only grow, so it never goes back.
struct Search {
    int at, reach;
    int64_t before;
};

// The row tile at place x < total of the axis.
template <class A>
__device__ __forceinline__ Unit unit_at(const A &a, int M, const Group &first, int64_t x, int lane, Search &from) {
    Unit u;
    u.ok = false;
    int64_t before = from.before;
    int reach = from.reach;
    for (int at = from.at; at < a.s.B; at += 64) {
        const int reach0 = reach;
        const Lens s = group_at<true>(a, at, lane, first, reach);
        const int64_t mine = seq_cost(s, a.G, M);
        const int64_t end = before + wave_scan_add(mine);
        const uint64_t has = __ballot(x < end);
        if (has) {
            from = {at, reach0, before};
            const int src = uniform(__ffsll((unsigned long long)has) - 1);
            u.b = at + src;
            u.n = lane_of(s.n, src);
            u.lo_row = lane_of(s.lo, src);
            u.L = lane_of(s.L, src);
            const int64_t base = lane_of(end - mine, src), y = x - base;
            const int64_t GA = axis_keys(u.n, u.L, a.G);
            const int tiles = tiles_of(u.n * a.G, M);
            int t = 0;
            if (tiles > 1) {
                // largest t with tile_start(t) <= y: the root of M t^2 / 2 + (GA + M / 2) t - y, then by one steps
                const double h = (double)GA + 0.5 * M;
                t = min(max((int)((__builtin_sqrt(h * h + 2.0 * M * (double)y) - h) / M), 0), tiles - 1);
                while (t > 0 && tile_start(t, GA, M) > y) --t;
                while (t + 1 < tiles && tile_start(t + 1, GA, M) <= y) ++t;
            }
            u.tile = uniform(t);
            u.start = base + tile_start(u.tile, GA, M);
            u.cost = GA + (int64_t)(u.tile + 1) * M;
            u.ok = true;
            return u;
        }
        before = lane_of(end, 63);
    }
    return u;
}

// The key tile at which a cut at place x of the axis, inside the unit, parts
// its `tiles` key tiles: both sides compute the same number.
__device__ __forceinline__ int cut_at(const Unit &u, int64_t x, int tiles) {
    return min(tiles, (int)((double)(x - u.start) / (double)u.cost * tiles));
}

// ---- calls of many rows: row tiles in order of length -----------------------
// A row tile is one workgroup's, or several workgroups' where the call has too
// few for the chip or one is much longer than the others: its keys are then
// done in parts of at most `chunk` key tiles.  Longest sequences go first and
// neighbours walk the same keys at the same time, which their shared L2 sees;
// an equal cut of all the work, as for few rows, lost that (737 against 884
// TFLOP/s on 16384 new tokens).

// A part of a row tile.
struct Piece {
    Unit u;
    int split, splits, slot;  // which part of how many; its slot for partial results
};

__device__ __forceinline__ int wave_max(int x) { return lane_of(wave_scan_max(x), 63); }

// Sequences of a group of 64 by decreasing keys, to half an octave: what
// belongs in this lane's place.  Few steps for the few classes that a batch
// has (a full sort of 64 took 13 of 68 us of a call of 64 short prompts).
__device__ __forceinline__ void sort_longest(int group, int lane, int &b, Lens &s) {
    constexpr int kTop = 0xff << 1;  // over every class of a 31-bit length
    const int cls = (int)(__builtin_bit_cast(uint32_t, (float)max(s.L, 1)) >> 22);  // 254 to 314
    const bool in = lane < group;
    const int hi = wave_max(in ? cls : 0), lo = kTop - wave_max(in ? kTop - cls : 0);
    int rank = lane, before = 0;
    for (int c = hi; c >= lo; --c) {
        const uint64_t mine = __ballot(in && cls == c);
        if (in && cls == c) rank = before + __popcll(mine & ((1ull << lane) - 1));
        before += __popcll(mine);
    }
    s.n = __builtin_amdgcn_ds_permute(rank << 2, s.n);
    s.L = __builtin_amdgcn_ds_permute(rank << 2, s.L);
    s.lo = __builtin_amdgcn_ds_permute(rank << 2, s.lo);
    b = __builtin_amdgcn_ds_permute(rank << 2, b);
}

__device__ __forceinline__ int parts_of(int L, int chunk) {
    const int tiles = tiles_of(L, kKeyTile);
    return tiles > chunk ? (tiles + chunk - 1) / chunk : 1;
}

// Key tiles of a part: an even share of the call's work over `pieces` parts.
// So no row tile outlasts the others' work (52 chunks of 42 to 162 tokens over
// up to 14430: 396 us when only tiles over two shares were cut, 310 so).  With
// fewer row tiles than parts it is raised by eighths, up to twice, until there
// are no more than `pieces` parts (where the sequences fit the wave's lanes):
// one part over what runs at once costs a whole round.
template <class A>
__device__ __forceinline__ int chunk_of(const A &a, int M, const Group &first, int lane, bool report) {
    const int nt = tiles_of(first.lens.n * a.G, M), kt = tiles_of(first.lens.L, kKeyTile);
    int64_t sum = (int64_t)nt * kt;
    int units = nt, reach = first.reach;
    for (int at = 64; at < a.s.B; at += 64) {
        const Lens s = read_lens<true>(a, at, lane, reach, report);
        const int t = tiles_of(s.n * a.G, M);
        units += t;
        sum += (int64_t)t * tiles_of(s.L, kKeyTile);
    }
    const int64_t least = max((wave_sum(sum) + a.pieces - 1) / a.pieces, (int64_t)kTileLeast);
    int chunk = (int)min(least, (int64_t)0x7ffffffe);
    if (a.s.B <= 64 && wave_sum(units) < a.pieces) {
        for (int k = 1; k <= 8; ++k) {
            if (wave_sum(nt * (kt > chunk ? (kt + chunk - 1) / chunk : 1)) <= a.pieces) break;
            chunk = (int)min(least + (least * k + 7) / 8, (int64_t)0x7ffffffe);
        }
    }
    return chunk;
}

// The part with number `item`; JOIN: the row tile with number `item` among
// those done in parts.  Row tiles of a sequence go from the last, which sees
// the most keys, to the first.
template <bool PAGED, bool JOIN, class A>
__device__ __forceinline__ Piece find_piece(const A &a, int M, const Group &first, int chunk, int item, int lane) {
    Piece p;
    p.u.ok = false;
    int items = 0, slots = 0, reach = 0;  // before this group of 64 sequences
    for (int at = 0; at < a.s.B; at += 64) {
        int b = at + lane;
        Lens s = group_at<PAGED>(a, at, lane, first, reach);
        int nt = tiles_of(s.n * a.G, M), sp = PAGED ? parts_of(s.L, chunk) : 1;
        int mine = JOIN ? (sp > 1 ? nt : 0) : nt * sp, my_slots = sp > 1 ? nt * sp : 0;
        const int group = min(64, a.s.B - at);
        if (at + 64 < a.s.B) {  // not in this group: its sums alone
            const int all = wave_sum(mine);
            if (item >= items + all) {
                items += all;
                if (PAGED) slots += wave_sum(my_slots);
                continue;
            }
        }
        if (group > 1) {
            sort_longest(group, lane, b, s);
            nt = tiles_of(s.n * a.G, M);
            sp = PAGED ? parts_of(s.L, chunk) : 1;
            mine = JOIN ? (sp > 1 ? nt : 0) : nt * sp;
            my_slots = sp > 1 ? nt * sp : 0;
        }
        const int end = items + wave_scan_add(mine);
        const int slot_end = PAGED ? slots + wave_scan_add(my_slots) : 0;
        const uint64_t has = __ballot(item < end);
        if (has) {
            const int src = uniform(__ffsll((unsigned long long)has) - 1);
            const int local = item - lane_of(end - mine, src);
            p.u.b = lane_of(b, src);
            p.u.n = lane_of(s.n, src);
            p.u.L = lane_of(s.L, src);
            p.u.lo_row = lane_of(s.lo, src);
            p.splits = PAGED ? lane_of(sp, src) : 1;
            const int from_last = JOIN || p.splits == 1 ? local : local / p.splits;
            p.split = JOIN ? 0 : local - from_last * p.splits;
            p.u.tile = lane_of(nt, src) - 1 - from_last;
            p.slot = (PAGED ? lane_of(slot_end - my_slots, src) : 0) + from_last * p.splits + p.split;
            p.u.ok = true;
            return p;
        }
        return p;  // past the last
    }
    return p;
}

#endif  // __HIPCC__

}  // namespace fate
