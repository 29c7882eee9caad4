// Appending keys and values to a paged cache, with the position rotation
// applied on the way (and to the queries).
//
//   (x, y) -> (x cos - y sin, y cos + x sin) per rotated pair, in float32,
//   rounded once to the operands' type; values and the dimensions past `rot`
//   are copied.
//
// k_kv_append: memory bounds it (each element is read once and written once).
// A workgroup takes one or four tokens; first each of its waves finds one
// token's sequence, position and page (a scan of `off`, 64 entries a step),
// then the threads walk the tokens' (head, unit) pairs, a unit being sixteen
// elements: two chunks of eight that the rotation pairs (j and j + rot/2), or
// two neighbouring chunks.  A unit's elements belong to one thread, so queries
// can be rotated in place.
#include "fate_attn.h"

namespace fate {
namespace {

struct Place {
    int64_t cache;  // element of the token's slot, head 0; negative: no place
    int pos;        // position; negative: no place
};

// VEC: chunks are 16-byte loads (rot / 2 a multiple of 8, or pairs
// interleaved with rot a multiple of 8); otherwise element by element.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void k_kv_append(AppendLaunch a, int per_wg, int units, uint32_t units_inv,
                                                   int heads, uint32_t items_inv) {
    typedef typename T::el el;
    typedef typename T::x8 x8;
    __shared__ Place place[4];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t t0 = (int64_t)blockIdx.x * per_wg;
    const int toks = (int)min((int64_t)per_wg, a.s.T - t0);
    if (w < toks) {
        const int64_t t = t0 + w;
        int b = 0;  // sequences that end at or before t
        for (int at = 0; at < a.s.B; at += 64) {
            const int i = at + lane;
            b += __popcll(__ballot(i < a.s.B && (int64_t)a.s.off[i + 1] <= t));
        }
        if (lane == 0) {
            Place p = {-1, -2};  // in no sequence: not touched
            if (b < a.s.B) {
                const int lo = a.s.off[b], hi = a.s.off[b + 1], n = a.s.kv_len[b];
                if (lo >= 0 && (int64_t)lo <= t && t < (int64_t)hi && (int64_t)hi <= a.s.T) {
                    bool bad = n < 0 || (int64_t)n > a.s.max_keys;
                    const int64_t pos = (int64_t)n - (hi - lo) + (t - lo);
                    p.pos = -1;
                    if (!bad && pos >= 0) {
                        const int page = a.s.pages[b * a.s.pages_stride + (pos >> a.c.page_shift)];
                        bad = page < 0 || page >= a.c.n_pages || (a.rot && pos >= a.table_rows);
                        if (!bad) {
                            p.pos = (int)pos;
                            p.cache = page * a.c.page + (pos & ((1 << a.c.page_shift) - 1)) * a.c.token;
                        }
                    }
                    if (bad && a.status) a.status[b] = FATE_EINVAL;
                } else if (a.status) {
                    a.status[b] = FATE_EINVAL;
                }
            }
            place[w] = p;
        }
    }
    __syncthreads();

    const int items = heads * units, half = a.rot / 2;
    const int pair_units = a.interleaved ? 0 : (half + 7) / 8;
    for (int x = tid; x < toks * items; x += 256) {
        const int tk = per_wg == 1 ? 0 : (int)__umulhi((uint32_t)x, items_inv);
        const int y = x - tk * items;
        const int h = units == 1 ? y : (int)__umulhi((uint32_t)y, units_inv), u = y - h * units;
        const Place p = place[tk];
        if (p.pos == -2) continue;
        const int64_t t = t0 + tk;
        const bool is_q = h < a.hq, is_k = !is_q && h < a.hq + a.hkv;
        if (!is_q && p.pos < 0) continue;
        const int kh = is_k ? h - a.hq : h - a.hq - a.hkv;
        const RowsArg &src_rows = is_q ? a.q : is_k ? a.k : a.v;
        const el *src = (const el *)src_rows.data + t * src_rows.token + (int64_t)(is_q ? h : kh) * src_rows.head;
        el *dst = is_q ? (el *)a.qo.data + t * a.qo.token + (int64_t)h * a.qo.head
                       : (el *)(is_k ? a.ck : a.cv) + p.cache + (int64_t)kh * a.c.head;
        const bool turn = (is_q || is_k) && p.pos >= 0;
        const bool pair = u < pair_units;  // chunks that the rotation pairs: e0 and e0 + half
        int e0, e1, len0, len1;            // the unit's two chunks
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
        const float *row = a.table + (int64_t)max(p.pos, 0) * a.rot;
        float c0[8], c1[8];
        if (VEC) {
            x8 i0 = {}, i1 = {};
            if (len0 > 0) i0 = *(const x8 *)(src + e0);
            if (len1 > 0) i1 = *(const x8 *)(src + e1);
            if (!(turn && (pair || (a.interleaved && e0 < a.rot))) && !(is_q && p.pos < 0)) {
                if (len0 > 0) *(x8 *)(dst + e0) = i0;
                if (len1 > 0) *(x8 *)(dst + e1) = i1;
                continue;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                c0[e] = (float)i0[e];
                c1[e] = (float)i1[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                c0[e] = e < len0 ? (float)src[e0 + e] : 0.0f;
                c1[e] = e < len1 ? (float)src[e1 + e] : 0.0f;
            }
        }
        if (is_q && p.pos < 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) c0[e] = c1[e] = 0.0f;
        } else if (turn && pair) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < len0) {
                    const float cs = row[e0 + e], sn = row[half + e0 + e];
                    const float x0 = c0[e], y0 = c1[e];
                    c0[e] = x0 * cs - y0 * sn;
                    c1[e] = y0 * cs + x0 * sn;
                }
        } else if (turn && a.interleaved) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                if (e0 + e < a.rot) {
                    const float cs = row[(e0 + e) / 2], sn = row[half + (e0 + e) / 2];
                    const float x0 = c0[e], y0 = c0[e + 1];
                    c0[e] = x0 * cs - y0 * sn;
                    c0[e + 1] = y0 * cs + x0 * sn;
                }
                if (e1 + e < a.rot) {
                    const float cs = row[(e1 + e) / 2], sn = row[half + (e1 + e) / 2];
                    const float x0 = c1[e], y0 = c1[e + 1];
                    c1[e] = x0 * cs - y0 * sn;
                    c1[e + 1] = y0 * cs + x0 * sn;
                }
            }
        }
        if (VEC) {
            x8 o0, o1;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                o0[e] = (el)c0[e];
                o1[e] = (el)c1[e];
            }
            if (len0 > 0) *(x8 *)(dst + e0) = o0;
            if (len1 > 0) *(x8 *)(dst + e1) = o1;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e < len0) dst[e0 + e] = (el)c0[e];
                if (e < len1) dst[e1 + e] = (el)c1[e];
            }
        }
    }
}

// Multiplier m = ceil(2^32 / n) of __umulhi for x / n: exact while x (m n - 2^32)
// < 2^32.  Here x < 4 n, m n - 2^32 < n and n <= 3 * 256 heads * 17 units, so
// x n < 7e8.  n = 1 has no 32-bit multiplier and is left to the kernel.
uint32_t inverse(uint32_t n) { return n <= 1 ? 0u : (uint32_t)((0x100000000ull + n - 1) / n); }

template <class T>
int go(const AppendLaunch &a, hipStream_t s) {
    const int half = a.rot / 2;
    const int heads = a.hq + 2 * a.hkv;
    // units of a head: rotated pairs of chunks, then the rest in sixteens
    const int units = a.interleaved ? (a.d + 15) / 16 : (half + 7) / 8 + (a.d - a.rot + 15) / 16;
    const bool vec = a.interleaved ? a.rot % 8 == 0 : half % 8 == 0;
    const int per_wg = a.s.T <= 1024 ? 1 : 4;
    const unsigned grid = (unsigned)((a.s.T + per_wg - 1) / per_wg);
    if (vec) hipLaunchKernelGGL((k_kv_append<T, true>), dim3(grid), dim3(256), 0, s, a, per_wg, units, inverse(units), heads, inverse(heads * units));
    else hipLaunchKernelGGL((k_kv_append<T, false>), dim3(grid), dim3(256), 0, s, a, per_wg, units, inverse(units), heads, inverse(heads * units));
    return (int)hipGetLastError();
}

}  // namespace

int launch_append(const AppendLaunch &a, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return a.dtype == FATE_BF16 ? go<BF16>(a, s) : go<F16>(a, s);
}

}  // namespace fate
