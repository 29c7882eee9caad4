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
};
int launch_append(const AppendLaunch &a, void *stream);

// Attention over pages (kv in CacheArg) or over packed rows (k, v).  Rows of
// one key head are packed for the matrix tiles: packed row r of a sequence is
// token r / G, query head hk * G + r % G, G = heads_q / heads_kv.
struct AttnLaunch {
    SeqsArg s;
    RowsArg q, k, v, out;
    CacheArg c;
    float *lse;       // [T][hq] or null
    int32_t *status;  // [B] or null
    float *part;      // partial outputs [slots][hkv][rows][d], then (max, sum) pairs [slots][hkv][rows][2]
    float scale_log2; // scale * log2(e)
    int32_t hq, hkv, G, d, dtype;
    int32_t pieces;   // target pieces of work per key head (splitting); 0 = never split
    int32_t slots;    // partial slots per key head
    int32_t grid;     // pieces launched per key head
};
int launch_attn_tile(const AttnLaunch &a, bool paged, void *stream);
int launch_attn_few(const AttnLaunch &a, int rows, void *stream);
int launch_attn_join(const AttnLaunch &a, int rows, int tiles, void *stream);

constexpr int kKeyTile = 64;    // keys per tile: the unit in which the key axis is split
constexpr int kTileRows = 128;  // packed rows of a workgroup of the tile kernel
// Fewest key tiles of a part: one block of 32 keys for each wave of the
// few-row kernel; enough work to pay for the join in the tile kernel.
constexpr int kFewLeast = 2, kTileLeast = 4;

#if defined(__HIPCC__)

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct BF16 {
    typedef __bf16 el;
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
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
};

struct F16 {
    typedef _Float16 el;
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
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
        return __builtin_bit_cast(x4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) h4 *)p));
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

// A workgroup's piece of work: packed rows [tile * M, ...) of sequence b over
// key tiles [lo, hi) of its keys.
struct Piece {
    int b, n, lo_row;  // sequence, its tokens, first token row (off[b])
    int L;             // its keys
    int tile;          // row tile
    int split, splits; // which part of the key axis, of how many
    int slot;          // partial slot (splits > 1)
    int chunk;         // key tiles per split
    bool ok;
};

// One sequence as the kernels see it: token count and keys, both zero where
// the device arrays are out of range.
template <bool PAGED>
__device__ __forceinline__ void read_seq(const AttnLaunch &a, int b, int &lo, int &n, int &L, bool &bad) {
    lo = a.s.off[b];
    const int hi = a.s.off[b + 1];
    bad = lo < 0 || hi < lo || (int64_t)hi > a.s.T;
    n = bad ? 0 : hi - lo;
    L = n;
    if (PAGED) {
        L = a.s.kv_len[b];
        if (L < 0 || (int64_t)L > a.s.max_keys) bad = true;
        if (bad) L = n = 0;
    }
}

__device__ __forceinline__ int wave_scan_add(int x, int lane) {  // inclusive
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    return x;
}

__device__ __forceinline__ int tiles_of(int n, int tile) { return (int)(((int64_t)n + tile - 1) / tile); }

// Key tiles per piece: the call's key tiles over all row tiles of M packed
// rows, shared out over the target number of pieces.  The lengths are read on
// the device (a serving step's lengths live there), so every workgroup adds
// them up for itself: B / 64 loads per lane, which a small batch barely feels.
template <bool PAGED>
__device__ __forceinline__ int chunk_of(const AttnLaunch &a, int M, int least, int lane) {
    if (!PAGED || a.pieces == 0) return 0x7fffffff;
    int64_t sum = 0;
    for (int b = lane; b < a.s.B; b += 64) {
        int lo, n, L;
        bool bad;
        read_seq<PAGED>(a, b, lo, n, L, bad);
        sum += (int64_t)tiles_of(n * a.G, M) * tiles_of(L, kKeyTile);
    }
    sum = wave_sum(sum);
    const int64_t c = (sum + a.pieces - 1) / a.pieces;
    return c < least ? least : (int)(c > 0x7fffffff ? 0x7fffffff : c);
}

// The piece with number `item`: sequences in order, each with its row tiles
// from the last (which sees the most keys) to the first, each of these split
// over its keys.  JOIN: number only the row tiles of split sequences.
template <bool PAGED, bool JOIN>
__device__ __forceinline__ Piece find_piece(const AttnLaunch &a, int M, int chunk, int item, int lane, bool report) {
    Piece p;
    p.ok = false;
    p.chunk = chunk;
    int items = 0, slots = 0;  // before this group of 64 sequences
    for (int at = 0; at < a.s.B; at += 64) {
        const int b = at + lane;
        int lo = 0, n = 0, L = 0;
        if (b < a.s.B) {
            bool bad;
            read_seq<PAGED>(a, b, lo, n, L, bad);
            if (bad && report && a.status) a.status[b] = FATE_EINVAL;
        }
        const int nt = tiles_of(n * a.G, M);
        int sp = 1;
        if (PAGED && chunk != 0x7fffffff) {
            sp = (tiles_of(L, kKeyTile) + chunk - 1) / chunk;
            if (sp < 1) sp = 1;
        }
        const int mine = JOIN ? (sp > 1 ? nt : 0) : nt * sp;
        const int my_slots = sp > 1 ? nt * sp : 0;
        const int end = wave_scan_add(mine, lane) + items;
        const int slot_end = wave_scan_add(my_slots, lane) + slots;
        const uint64_t has = __ballot(item < end);
        if (has) {
            const int src = __ffsll((unsigned long long)has) - 1;
            const int local = item - __shfl(end - mine, src);
            p.b = uniform(at + src);
            p.n = uniform(__shfl(n, src));
            p.lo_row = uniform(__shfl(lo, src));
            p.L = uniform(__shfl(L, src));
            p.splits = uniform(__shfl(sp, src));
            const int tiles = uniform(__shfl(nt, src));
            const int first_slot = uniform(__shfl(slot_end - my_slots, src));
            const int from_last = uniform(JOIN ? local : local / p.splits);
            p.split = uniform(JOIN ? 0 : local - from_last * p.splits);
            p.tile = tiles - 1 - from_last;
            p.slot = first_slot + from_last * p.splits + p.split;
            p.ok = true;
            return p;
        }
        items = __shfl(end, 63);
        slots = __shfl(slot_end, 63);
    }
    return p;
}

#endif  // __HIPCC__

}  // namespace fate
