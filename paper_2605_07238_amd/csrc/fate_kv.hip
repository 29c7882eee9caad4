// Appending keys and values to a paged cache, with the position rotation
// applied on the way (and to the queries).
//
//   (x, y) -> (x cos - y sin, y cos + x sin) per rotated pair, in float32,
//   rounded once to the operands' type; values and the dimensions past `rot`
//   are copied.
//
// k_kv_append: memory bounds it (each element is read once and written once).
// A workgroup takes one token, or four in large calls; its first wave finds
// their sequences, positions and pages (a scan of `off`, 64 entries a step for
// all of them).  Then a thread is one unit of sixteen elements in every HS-th
// (token, head) pair: two chunks of eight that the rotation pairs (j and
// j + rot / 2), or two neighbouring chunks.  The unit's place is worked out
// once, and its elements belong to one thread, which lets queries be rotated
// in place.  18261 tokens of 48 heads of 128, 451 MB: 82 us, 5480 GB/s, in calls
// on the same few inputs, 97 on inputs and caches that were not near (a copy of
// as many bytes: 84); with a division per unit and a token per wave, 154 us.
//
// A call that moves more than the last-level cache holds reads past it: 82
// against 96 us there.  For a third of the bytes, 29 against 31 us on inputs in
// turn, but 29 against 25 where the cache still has the rows from the projection
// that wrote them.
#include "fate_attn.h"

namespace fate {
namespace {

struct Place {
    int64_t cache;  // element of the token's slot, head 0; negative: no place
    int pos;        // position; negative: no place
};

// With several axes: the token's position on each.
struct Turns {
    int on[FATE_MAX_AXES];
};

// VEC: chunks are 16-byte loads (rot / 2 a multiple of 8, or pairs
// interleaved with rot a multiple of 8); otherwise element by element.
// PAST: rows are read past the last-level cache.  AXES: a pair turns by its
// axis's position instead of the token's own.  The workgroup gathers each
// token's cosines and sines into LDS once, for all heads: with axes in turn, 16
// loads of a unit's own took 133 us for 18261 tokens of 48 heads of 128, 99 us so.
template <class T, bool VEC, bool PAST, bool AXES>
__global__ __launch_bounds__(256) void k_kv_append(AppendLaunch a, int per_wg, int units, int heads,
                                                   uint32_t heads_inv) {
    typedef typename T::el el;
    typedef typename T::x8 x8;
    __shared__ Place place[kAppendTokens];
    __shared__ Turns turns[AXES ? kAppendTokens : 1];
    __shared__ __align__(16) float angles[AXES ? kAppendTokens : 1][FATE_MAX_HEAD_DIM];  // cosines, then sines
    const int tid = threadIdx.x;
    const int64_t t0 = (int64_t)blockIdx.x * per_wg;
    const int toks = (int)min((int64_t)per_wg, a.s.T - t0);
    if (tid < 64) {
        // Lane i: the sequence that holds token t0 + i.  The first workgroup goes through all sequences, which reports
        // those that are out of range; the others stop at their last token's.
        int b = 0, n = 0, L = -1, row = 0, found = 0, reach = 0;
        for (int at = 0; at < a.s.B && (found < toks || blockIdx.x == 0); at += 64) {
            const Lens s = read_lens<true>(a, at, tid, reach, blockIdx.x == 0);
            for (int i = 0; i < toks; ++i) {
                const uint64_t has = __ballot(t0 + i >= s.lo && t0 + i - s.lo < s.n);
                if (!has) continue;
                const int src = uniform(__ffsll((unsigned long long)has) - 1);
                const int its_n = lane_of(s.n, src), its_L = lane_of(s.L, src), its_lo = lane_of(s.lo, src);
                if (tid == i) {
                    b = at + src;
                    n = its_n;
                    L = its_L;
                    row = (int)(t0 + i - its_lo);
                }
                ++found;
            }
        }
        if (tid < toks) {
            Place p = {-1, -2};  // in no sequence: not touched
            if (L >= 0) {
                const int64_t pos = (int64_t)L - n + row;
                p.pos = -1;
                if (pos >= 0) {
                    const int page = a.s.pages[b * a.s.pages_stride + (pos >> a.c.page_shift)];
                    bool turned = AXES || !a.rot || pos < a.table_rows;
                    if (AXES) {
                        for (int x = 0; x < a.n_axes; ++x) {
                            const int on = a.positions[x * a.positions_stride + t0 + tid];
                            turned = turned && on >= 0 && on < a.table_rows;
                            turns[tid].on[x] = on;
                        }
                    }
                    if (page < 0 || page >= a.c.n_pages || !turned) {
                        if (a.status) a.status[b] = FATE_EINVAL;
                    } else {
                        p.pos = (int)pos;
                        p.cache = page * a.c.page + (pos & ((1 << a.c.page_shift) - 1)) * a.c.token;
                    }
                }
            }
            place[tid] = p;
        }
    }
    __syncthreads();

    const int half = a.rot / 2;
    if (AXES) {
        for (int x = tid; x < toks * half; x += 256) {
            const int tk = x / half, j = x - tk * half;
            if (place[tk].pos < 0) continue;
            const int axis = a.axis[j / 16] >> j % 16 * 2 & 3u;
            const float *at = a.table + (int64_t)turns[tk].on[axis] * a.rot + j;
            angles[tk][j] = at[0];
            angles[tk][half + j] = at[half];
        }
        __syncthreads();
    }
    const int pair_units = a.interleaved ? 0 : (half + 7) / 8;
    const int hs = tid / units, u = tid - hs * units, HS = 256 / units;
    if (hs >= HS) return;
    // the unit's two chunks: those that the rotation pairs, or neighbours
    const bool pair = u < pair_units;
    int e0, e1, len0, len1;
    if (pair) {
        e0 = u * 8;
        e1 = e0 + half;
        len0 = len1 = min(8, half - e0);
    } else {
        e0 = (a.interleaved ? 0 : a.rot) + (u - pair_units) * 16;
        e1 = e0 + 8;
        len0 = max(0, min(8, a.d - e0));
        len1 = max(0, min(8, a.d - e1));
    }
    const bool rotated = pair || (a.interleaved && e0 < a.rot);
    const int j0 = pair ? e0 : e0 / 2;  // the unit's first pair: a multiple of 8

    for (int x = hs; x < toks * heads; x += HS) {
        const int tk = heads == 1 ? x : (int)__umulhi((uint32_t)x, heads_inv), h = x - tk * heads;
        const Place p = place[tk];
        const bool is_q = h < a.hq, is_k = !is_q && h < a.hq + a.hkv;
        if (p.pos == -2 || (p.pos < 0 && !is_q)) continue;
        const int64_t t = t0 + tk;
        const int kh = is_q ? h : is_k ? h - a.hq : h - a.hq - a.hkv;
        const RowsArg &rows = is_q ? a.q : is_k ? a.k : a.v;
        const el *src = (const el *)rows.data + t * rows.token + (int64_t)kh * rows.head;
        el *dst = is_q ? (el *)a.qo.data + t * a.qo.token + (int64_t)h * a.qo.head
                       : (el *)(is_k ? a.ck : a.cv) + p.cache + (int64_t)kh * a.c.head;
        x8 x0 = {}, x1 = {};
        if (p.pos >= 0) {  // a query without a place comes out zero
            if (VEC && PAST) {
                if (len0 > 0) x0 = __builtin_nontemporal_load((const x8 *)(src + e0));
                if (len1 > 0) x1 = __builtin_nontemporal_load((const x8 *)(src + e1));
            } else if (VEC) {
                if (len0 > 0) x0 = *(const x8 *)(src + e0);
                if (len1 > 0) x1 = *(const x8 *)(src + e1);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (e < len0) x0[e] = src[e0 + e];
                    if (e < len1) x1[e] = src[e1 + e];
                }
            }
            if (rotated && (is_q || is_k)) {
                const float *row = AXES ? &angles[tk][j0] : a.table + (int64_t)p.pos * a.rot + j0;
                float cs[8] = {}, sn[8] = {};
                if (AXES && VEC && j0 + 8 <= half) {  // half is a multiple of four
#pragma unroll
                    for (int e = 0; e < 8; e += 4) {
                        *(f32x4 *)&cs[e] = *(const f32x4 *)(row + e);
                        *(f32x4 *)&sn[e] = *(const f32x4 *)(row + half + e);
                    }
                } else if (VEC && j0 + 8 <= half) {
                    __builtin_memcpy(cs, row, 32);
                    __builtin_memcpy(sn, row + half, 32);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (j0 + e < half) {
                            cs[e] = row[e];
                            sn[e] = row[half + e];
                        }
                }
                if (pair) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float v = (float)x0[e], w = (float)x1[e];
                        x0[e] = (el)(v * cs[e] - w * sn[e]);
                        x1[e] = (el)(w * cs[e] + v * sn[e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = (float)x0[2 * e], w = (float)x0[2 * e + 1];
                        const float y = (float)x1[2 * e], z = (float)x1[2 * e + 1];
                        if (e0 + 2 * e < a.rot) {
                            x0[2 * e] = (el)(v * cs[e] - w * sn[e]);
                            x0[2 * e + 1] = (el)(w * cs[e] + v * sn[e]);
                        }
                        if (e1 + 2 * e < a.rot) {
                            x1[2 * e] = (el)(y * cs[4 + e] - z * sn[4 + e]);
                            x1[2 * e + 1] = (el)(z * cs[4 + e] + y * sn[4 + e]);
                        }
                    }
                }
            }
        }
        if (VEC) {
            if (len0 > 0) *(x8 *)(dst + e0) = x0;
            if (len1 > 0) *(x8 *)(dst + e1) = x1;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e < len0) dst[e0 + e] = x0[e];
                if (e < len1) dst[e1 + e] = x1[e];
            }
        }
    }
}

template <class T>
int go(const AppendLaunch &a, hipStream_t s) {
    const int half = a.rot / 2;
    const int heads = a.hq + 2 * a.hkv;
    // units of a head: rotated pairs of chunks, then the rest in sixteens
    const int units = a.interleaved ? (a.d + 15) / 16 : (half + 7) / 8 + (a.d - a.rot + 15) / 16;
    const bool vec = a.interleaved ? a.rot % 8 == 0 : half % 8 == 0;
    const int per_wg = append_tokens(a.s.T);
    const unsigned grid = (unsigned)append_grid(a.s.T);
    // multiplier of __umulhi for x / heads: ceil(2^32 / heads), exact while x * heads < 2^32 (x < kAppendTokens * heads)
    const uint32_t inv = heads > 1 ? (uint32_t)((0x100000000ull + heads - 1) / heads) : 0u;
    const dim3 g(grid), b(256);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, g, b, 0, s, a, per_wg, units, heads, inv); };
    if (a.positions) {
        if (vec && a.past_cache) launch(k_kv_append<T, true, true, true>);
        else if (vec) launch(k_kv_append<T, true, false, true>);
        else launch(k_kv_append<T, false, false, true>);
    } else {
        if (vec && a.past_cache) launch(k_kv_append<T, true, true, false>);
        else if (vec) launch(k_kv_append<T, true, false, false>);
        else launch(k_kv_append<T, false, false, false>);
    }
    return (int)hipGetLastError();
}

}  // namespace

int launch_append(const AppendLaunch &a, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return a.dtype == FATE_BF16 ? go<BF16>(a, s) : go<F16>(a, s);
}

}  // namespace fate
