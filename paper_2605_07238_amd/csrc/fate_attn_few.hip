// Attention of few new tokens per sequence over a paged cache (one token of
// an answer, some drafted tokens), and the joining of parts of the key axis.
//
// With few rows the call reads each key and value once and computes little:
// memory bounds it.  k_attn_few: all row tiles of a key head (16 or 32 packed
// rows of one sequence) lie on one axis of work, worked out from the lengths on
// the device, and a workgroup of four waves walks an equal share of it: several
// tiles, one, or parts at either end, which k_attn_join puts together.  There
// are about as many shares as the chip runs workgroups, whatever the mix of
// lengths.  In a tile, a wave takes every fourth block of 32 keys by itself:
// keys go from memory to registers as the first product's operand (16-byte
// loads, 64 bytes of each of 16 rows at a time), values through the wave's own
// LDS rows, because the second product needs them transposed.  The products are transposed as in
// the tile kernel (S^T = k q^T, O^T = v^T p^T), on 16 x 16 x 32 matrix
// instructions: 16 packed rows are one column block.  The four waves'
// statistics and outputs meet in LDS at the end.  A step of 64 answers over 128
// to 8192 keys: 101 us and 6.4 for the join, 4.7 TB/s; two answers over 65536
// and 131072: 144 and 8.3 us, 5.2 TB/s.  One block a wave at a time is enough:
// two workgroups a compute unit hold 128 KB of loads under way (head size 128;
// the shares' number: plan_paged).
//
// k_attn_join: the parts of a row tile, o = sum 2^(m_i - M) o_i / sum 2^(m_i - M) l_i.
#include "fate_attn.h"

namespace fate {
namespace {

template <class T, int D, int RT>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void k_attn_few(AttnLaunch) {
    typedef typename T::el el;
    typedef typename T::x4 x4;
    typedef typename T::x8 x8;
    constexpr int M = 16 * RT, KS = D / 32, DT = D / 16;
    constexpr int VS = D + 8;   // row of a wave's value rows in LDS: eight elements of padding against bank conflicts
    constexpr int OS = D + 4;   // row of the waves' outputs in LDS
    constexpr int kBytes = 4 * 32 * VS * 2 > 4 * 16 * OS * 4 ? 4 * 32 * VS * 2 : 4 * 16 * OS * 4;
    __shared__ __align__(16) char raw[kBytes];
    __shared__ float sm[4][M], sl[4][M];

    int hk, piece;
    int64_t from, to;
    Group lens;
    {
        const Args &a = launch_args();
        const bool report = blockIdx.x == 0 && threadIdx.x < 64;
        hk = blockIdx.x % a.hkv, piece = blockIdx.x / a.hkv;
        lens = first_group<true>(a, threadIdx.x & 63, report);
        const Axis axis = axis_of(a, M, lens, threadIdx.x & 63, report);
        from = piece * axis.share;
        to = min(from + axis.share, axis.total);
    }
    Search search = {0, 0, 0};
    for (int64_t x = from; x < to;) {  // the row tiles of this share
        const Args &a = launch_args();
        const int tid = fresh(threadIdx.x), lane = tid & 63, w = uniform(tid >> 6);
        const Unit p = unit_at(a, M, lens, x, lane, search);
        if (!p.ok) return;
        x = p.start + p.cost;

        const int rows = p.n * a.G, row0 = p.tile * M;
        const int first = p.L - p.n + 1;
        const int last_row = min(row0 + M, rows) - 1;
        const int most = min(p.L, max(0, last_row / a.G + first));
        const int least = max(0, min(p.L, row0 / a.G + first));
        const int blocks = (most + 31) / 32;
        const bool part = p.start < from || p.start + p.cost > to;
        const int k_lo = p.start < from ? 32 * cut_at(p, from, blocks) : 0;
        const int k_hi = p.start + p.cost > to ? min(most, 32 * cut_at(p, to, blocks)) : most;

        const int c = lane & 15, g = lane >> 4;
        x8 q[RT][KS];
        int ends[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int row = row0 + rt * 16 + c;
            const bool live = row < rows;
            const int tok = live ? row / a.G : 0;
            ends[rt] = live ? max(0, min(p.L, tok + first)) : 0;
            const el *src = (const el *)a.q.data + (p.lo_row + (int64_t)tok) * a.q.token +
                            (int64_t)(hk * a.G + row - tok * a.G) * a.q.head + g * 8;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                u32x4 x = {0, 0, 0, 0};
                if (live && s * 32 + g * 8 < a.d) x = *(const u32x4 *)(src + s * 32);
                q[rt][s] = __builtin_bit_cast(x8, x);
            }
        }
        f32x4 o[RT][DT];
        float m[RT], l[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = kLowest;
            l[rt] = 0.0f;
#pragma unroll
            for (int i = 0; i < DT; ++i) o[rt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        el *const vrow = (el *)raw + w * 32 * VS;
        const int32_t *const table = a.s.pages + p.b * a.s.pages_stride;
        const int mask = (1 << a.c.page_shift) - 1;
        int pg[2];
        auto find_pages = [&](int kb) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int key = kb + 16 * i + c;
                pg[i] = key < k_hi ? table[key >> a.c.page_shift] : 0;
            }
        };
        find_pages(k_lo + 32 * w);
        bool odd = false;  // a value on some row's edge is infinite or NaN
        for (int kb = k_lo + 32 * w; kb < k_hi; kb += 128) {
            u32x4 rk[2][KS], rv[2][KS];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int key = kb + 16 * i + c;
                bool in = key < k_hi;
                if (in && (uint32_t)pg[i] >= (uint32_t)a.c.n_pages) {
                    in = false;
                    if (a.status) a.status[p.b] = FATE_EINVAL;
                }
                const int64_t at = pg[i] * a.c.page + (int64_t)hk * a.c.head + (key & mask) * a.c.token + g * 8;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const bool ld = in && s * 32 + g * 8 < a.d;
                    rk[i][s] = u32x4{0, 0, 0, 0};
                    rv[i][s] = u32x4{0, 0, 0, 0};
                    if (ld) {
                        rk[i][s] = *(const u32x4 *)((const el *)a.c.k + at + s * 32);
                        rv[i][s] = *(const u32x4 *)((const el *)a.c.v + at + s * 32);
                    }
                }
            }
            find_pages(kb + 128);
            const bool edge = kb + 32 > least;  // uniform
            if (edge) {
                uint32_t bad = 0;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        bad |= not_finite<T>(rv[i][s][0]) | not_finite<T>(rv[i][s][1]) | not_finite<T>(rv[i][s][2]) |
                               not_finite<T>(rv[i][s][3]);
                if (__any(bad != 0)) {  // left out here, added at the end to the rows that see them
                    odd = true;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int s = 0; s < KS; ++s)
#pragma unroll
                            for (int e = 0; e < 4; ++e) rv[i][s][e] = only_finite<T>(rv[i][s][e]);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int s = 0; s < KS; ++s) *(u32x4 *)&vrow[(16 * i + c) * VS + s * 32 + g * 8] = rv[i][s];

            x8 pr[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                f32x4 s2[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    s2[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int s = 0; s < KS; ++s) s2[i] = T::mfma16(__builtin_bit_cast(x8, rk[i][s]), q[rt][s], s2[i]);
                }
                // s2[i][j]: key 16 i + 4 g + j of the block, packed row c
                if (edge || kb + 32 > k_hi) {
                    const int left = min(ends[rt], k_hi) - kb - 4 * g;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (16 * i + j >= left) s2[i][j] = -INFINITY;
                }
                float top = fmaxf(fmaxf(fmaxf(s2[0][0], s2[0][1]), fmaxf(s2[0][2], s2[0][3])),
                                  fmaxf(fmaxf(s2[1][0], s2[1][1]), fmaxf(s2[1][2], s2[1][3])));
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                top = fmaxf(top * a.scale_log2, kLowest);
                if (__any(top > m[rt] + (kLag + T::kLift))) {
                    const float next = fmaxf(m[rt], top - T::kLift), f = exp2_fast(m[rt] - next);
                    m[rt] = next;
                    l[rt] *= f;
#pragma unroll
                    for (int i = 0; i < DT; ++i) o[rt][i] *= f;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float x = exp2_fast(__builtin_fmaf(s2[i][j], a.scale_log2, -m[rt]));
                        l[rt] += x;
                        pr[rt][4 * i + j] = (el)x;
                    }
            }
            __builtin_amdgcn_wave_barrier();
            const int vr = 4 * g + c / 4, vc = 4 * (c & 3);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const x4 v1 = T::read_tr(&vrow[vr * VS + dt * 16 + vc]);
                const x4 v2 = T::read_tr(&vrow[(vr + 16) * VS + dt * 16 + vc]);
                const x8 vf = __builtin_shufflevector(v1, v2, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) o[rt][dt] = T::mfma16(vf, pr[rt], o[rt][dt]);
            }
            __builtin_amdgcn_wave_barrier();
        }

        if (odd) {  // uniform in the wave
            for (int kb = k_lo + 32 * w; kb < k_hi; kb += 128)
                for (int key = max(kb, least / 32 * 32); key < min(kb + 32, k_hi); ++key) {
                    const int page = table[key >> a.c.page_shift];
                    if ((uint32_t)page >= (uint32_t)a.c.n_pages) continue;
                    const el *src = (const el *)a.c.v + page * a.c.page + (int64_t)hk * a.c.head + (key & mask) * a.c.token;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        asm volatile("" ::: "memory");  // one load at a time: a rare path is to cost no registers
                        const int d0 = dt * 16 + 4 * g;
                        x4 x = {};
                        if (d0 < a.d) x = *(const x4 *)(src + d0);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                o[rt][dt][e] += key < ends[rt] && !__builtin_isfinite((float)x[e]) ? (float)x[e] : 0.0f;
                    }
                }
        }

        // the four waves' rows: common maximum, sums
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] += __shfl_xor(l[rt], 16);
            l[rt] += __shfl_xor(l[rt], 32);
            if (g == 0) {
                sm[w][rt * 16 + c] = m[rt];
                sl[w][rt * 16 + c] = l[rt];
            }
        }
        float *const so = (float *)raw;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            __syncthreads();  // the value rows (rt = 0), or the last block's outputs, are done with
            const int r = rt * 16 + c;
            const float mm = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r]));
            const float f = exp2_fast(m[rt] - mm);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) *(f32x4 *)&so[(w * 16 + c) * OS + dt * 16 + 4 * g] = o[rt][dt] * f;
            __syncthreads();
            for (int x = tid; x < 16 * (D / 8); x += 256) {
                const int cc = x / (D / 8), d0 = x % (D / 8) * 8, rr = rt * 16 + cc, row = row0 + rr;
                if (row >= rows || d0 >= a.d) continue;
                const float top = fmaxf(fmaxf(sm[0][rr], sm[1][rr]), fmaxf(sm[2][rr], sm[3][rr]));
                float sum = 0.0f;
                f32x4 y0 = {0.0f, 0.0f, 0.0f, 0.0f}, y1 = y0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    sum += sl[k][rr] * exp2_fast(sm[k][rr] - top);
                    y0 += *(const f32x4 *)&so[(k * 16 + cc) * OS + d0];
                    y1 += *(const f32x4 *)&so[(k * 16 + cc) * OS + d0 + 4];
                }
                const int tok = row / a.G, qh = hk * a.G + row - tok * a.G;
                const int64_t out_row = p.lo_row + (int64_t)tok;
                if (part) {  // unscaled sums, joined by k_attn_join
                    const int64_t at = ((int64_t)(2 * piece + (p.start > from)) * a.hkv + hk) * M + rr;
                    *(f32x4 *)(a.part + at * a.d + d0) = y0;
                    *(f32x4 *)(a.part + at * a.d + d0 + 4) = y1;
                    if (d0 == 0) {
                        float *ml = a.part + 2 * (int64_t)a.pieces * a.hkv * M * a.d + at * 2;
                        ml[0] = top;
                        ml[1] = sum;
                    }
                    continue;
                }
                const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
                x8 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = (el)(y0[e] * inv);
                    y[4 + e] = (el)(y1[e] * inv);
                }
                *(x8 *)((el *)a.out.data + out_row * a.out.token + (int64_t)qh * a.out.head + d0) = y;
                if (d0 == 0 && a.lse)
                    a.lse[out_row * a.hq + qh] = sum != 0.0f ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
            }
        }
        __syncthreads();  // the outputs' and statistics' rows serve the next row tile
    }
}

// One wave per row of a row tile done in parts (a workgroup takes four rows and
// every `groups`-th four after them): its lanes are sixteen chunks of eight
// dimensions times four parts at a time, so that a row's parts are read side
// by side and the chain of reads stays short however many parts there are.
template <class T, bool TILE>
__global__ __launch_bounds__(256) void k_attn_join(AttnLaunch a, int M, int items, int groups) {
    typedef typename T::el el;
    typedef typename T::x8 x8;
    const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
    const int hk = blockIdx.x % a.hkv;
    const Group lens = first_group<true>(a, lane, false);
    Axis axis = {0, 0};
    int chunk = 0;
    if (TILE) chunk = chunk_of(a, M, lens, lane, false);
    else axis = axis_of(a, M, lens, lane, false);
    for (int at = blockIdx.x / a.hkv; at < items * groups; at += gridDim.x / a.hkv) {
        const int item = at / groups, group = at - item * groups;
        // part i lies in slot first_slot (i = 0), next_slot + step * i (others)
        Unit p;
        int splits, first_slot, next_slot, step;
        if (TILE) {
            const Piece piece = find_piece<true, true>(a, M, lens, chunk, item, lane);
            p = piece.u;
            if (!p.ok) return;
            splits = piece.splits;
            first_slot = next_slot = piece.slot;
            step = 1;
        } else {
            Search search = {0, 0, 0};
            const int64_t cut = (item + 1) * axis.share;
            if (cut >= axis.total) return;
            p = unit_at(a, M, lens, cut, lane, search);
            if (!p.ok || p.start >= cut || p.start < cut - axis.share) return;  // this row tile's first cut alone
            splits = uniform((int)((p.start + p.cost - 1) / axis.share)) - item + 1;
            first_slot = 2 * item + (p.start > cut - axis.share);  // behind the share's first where the tile begins within
            next_slot = 2 * item;
            step = 2;
        }
        const int rows = p.n * a.G, row0 = p.tile * M;
        const float *ml0 = a.part + 2 * (int64_t)a.pieces * a.hkv * M * a.d;
        auto place = [&](int i, int rr) {
            return ((int64_t)(i == 0 ? first_slot : next_slot + step * i) * a.hkv + hk) * M + rr;
        };
        for (int rr = group * 4 + w; rr < min(M, rows - row0); rr += groups * 4) {
            float top = kLowest, sum = 0.0f;
            for (int i = lane; i < splits; i += 64) top = fmaxf(top, ml0[place(i, rr) * 2]);
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
            for (int i = lane; i < splits; i += 64) {
                const float *ml = ml0 + place(i, rr) * 2;
                sum += ml[1] * exp2_fast(ml[0] - top);
            }
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
            const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
            const int row = row0 + rr, tok = row / a.G, qh = hk * a.G + row - tok * a.G;
            const int64_t out_row = p.lo_row + (int64_t)tok;
            el *dst = (el *)a.out.data + out_row * a.out.token + (int64_t)qh * a.out.head;
            for (int c0 = 0; c0 < a.d; c0 += 128) {
                const int d0 = c0 + (lane & 15) * 8;
                f32x4 y0 = {0.0f, 0.0f, 0.0f, 0.0f}, y1 = y0;
                if (d0 < a.d) {
#pragma unroll 4
                    for (int i = lane >> 4; i < splits; i += 4) {
                        const int64_t at = place(i, rr);
                        const float f = exp2_fast(ml0[at * 2] - top);
                        y0 += *(const f32x4 *)(a.part + at * a.d + d0) * f;
                        y1 += *(const f32x4 *)(a.part + at * a.d + d0 + 4) * f;
                    }
                }
                x8 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y0[e] += __shfl_xor(y0[e], 16);
                    y1[e] += __shfl_xor(y1[e], 16);
                    y0[e] += __shfl_xor(y0[e], 32);
                    y1[e] += __shfl_xor(y1[e], 32);
                    y[e] = (el)(y0[e] * inv);
                    y[4 + e] = (el)(y1[e] * inv);
                }
                if (lane < 16 && d0 < a.d) *(x8 *)(dst + d0) = y;
            }
            if (lane == 0 && a.lse)
                a.lse[out_row * a.hq + qh] = sum != 0.0f ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
        }
        if (!TILE) return;
    }
}

template <class T, int D>
int go(const AttnLaunch &a, int rows, hipStream_t s) {
    const dim3 grid((unsigned)a.grid * (unsigned)a.hkv);
    if (rows == 16) hipLaunchKernelGGL((k_attn_few<T, D, 1>), grid, dim3(256), 0, s, a);
    else if constexpr (D <= 128) hipLaunchKernelGGL((k_attn_few<T, D, 2>), grid, dim3(256), 0, s, a);
    else return (int)hipErrorInvalidValue;
    return (int)hipGetLastError();
}

template <class T>
int go(const AttnLaunch &a, int rows, hipStream_t s) {
    return a.d <= 64 ? go<T, 64>(a, rows, s) : a.d <= 128 ? go<T, 128>(a, rows, s) : go<T, 256>(a, rows, s);
}

}  // namespace

int launch_attn_few(const AttnLaunch &a, int rows, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return a.dtype == FATE_BF16 ? go<BF16>(a, rows, s) : go<F16>(a, rows, s);
}

int launch_attn_join(const AttnLaunch &a, int rows, int tiles, int groups, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    // row tiles: at most about 1024 workgroups, each of which goes on a grid's length further; most calls cut few
    const bool bf = a.dtype == FATE_BF16, tile = rows == kTileRows;
    const int most = 1024 / a.hkv > 0 ? 1024 / a.hkv : 1, all = tiles * groups;
    const dim3 grid((unsigned)(tile && all > most ? most : all) * (unsigned)a.hkv);
    if (bf && tile) hipLaunchKernelGGL((k_attn_join<BF16, true>), grid, dim3(256), 0, s, a, rows, tiles, groups);
    else if (bf) hipLaunchKernelGGL((k_attn_join<BF16, false>), grid, dim3(256), 0, s, a, rows, tiles, groups);
    else if (tile) hipLaunchKernelGGL((k_attn_join<F16, true>), grid, dim3(256), 0, s, a, rows, tiles, groups);
    else hipLaunchKernelGGL((k_attn_join<F16, false>), grid, dim3(256), 0, s, a, rows, tiles, groups);
    return (int)hipGetLastError();
}

}  // namespace fate
