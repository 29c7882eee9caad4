// Causal attention with matrix tiles: whole prompts over packed keys, and
// chunks of new tokens over a paged cache.
//
//   S = scale q k^T over the keys a row sees, O = softmax(S) v
// One pass over the keys with the running maximum m and sum l of each row:
// per key tile, m' = max(m, max S), O = O 2^(m - m') + 2^(S - m') v (S in
// units of log2), l likewise; at the end O / l.  m moves only when a tile
// exceeds it by more than 8, so O is rescaled rarely and the weights stay under
// 2^8 (in float16 under 2^15: kLift).
//
// k_attn_tile: one workgroup of four 64-lane waves per (sequence, key head,
// 128 packed rows, part of the key axis).  The G query heads of a key head are
// packed with the tokens into rows (row r: token r / G, head r % G), so that a
// key tile read once serves all of them and a tile's causal edge spans 128 / G
// tokens only.  Each wave owns 32 rows.  Both products are computed
// transposed: S^T = k q^T leaves one row's scores in the two lanes of its
// column, so the statistics need one exchange between lane halves, and the
// weights are the second product's operand where they lie, with no shuffle:
// the order of the keys in that product's sum is free, and v is read from LDS
// in the order that the first product's result has (transposing reads).
//
// Keys and values come from memory straight into LDS (no registers hold them
// on the way), values one tile ahead and keys two, so that a step works out the
// next tile's scores on the matrix cores beside the softmax of this one's in
// the vector units.  With tiles that passed through registers, one ahead, and
// each tile's scores in its own step: 2346 us for 16384 tokens against 2034.
// Now 1978 us, 1112 TFLOP/s (a large library product reaches 1418): the matrix
// cores are busy 58% of the cycles and the clock stands at 1.8 GHz for it.
//
// Key tiles go from the last to the first: the tiles on a row's causal edge
// come first.  Values that a row must not see cannot be left out of a matrix
// product by a zero weight when they are infinite or NaN (0 * inf): in the
// tiles on an edge such values are made zeros, and added at the end to the
// rows that do see them.
#include <type_traits>

#include "fate_attn.h"

namespace fate {
namespace {

// Sixteen bytes a lane from memory straight to LDS: lane i's land at dst + 16 i
// bytes.  Lane addresses are base + off bytes (base the same in all lanes), or
// p.  Nothing arrives in a register, so nothing that the compiler placed can be
// overwritten on the way; the wave waits for them with dma_wait before the
// barrier behind which the tile is read, and the waits that the compiler counts
// for its own loads can only wait for more.  m0 holds the place in LDS; nothing else here uses m0 (on
// this architecture only such loads and a few global-data instructions do).
__device__ __forceinline__ void dma16(const void *base, uint32_t off, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(uniform((int)dst)),
                 "v"(off), "s"(uniform64((int64_t)base))
                 : "memory");
}
__device__ __forceinline__ void dma16(const void *p, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(uniform((int)dst)), "v"(p)
                 : "memory");
}
__device__ __forceinline__ void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The larger of this lane's value and that of the lane 32 away.
__device__ __forceinline__ float both_halves_max(float x) {
    const uint32_t y = __builtin_bit_cast(uint32_t, x);
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(y, y, false, false));
    const uint32_t a = r[0], b = r[1];  // the lower half's values in both, the upper half's in both
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// Where keys and values are: packed rows, pages of at least the rows of one
// load, smaller pages.
enum Source { kRows, kPages, kSmallPages };

template <class T, int D, Source FROM>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void k_attn_tile(AttnLaunch) {
    const Args &a = launch_args();  // read where they lie: copied, they go to scratch and what uses them after them
    typedef typename T::el el;
    typedef typename T::x4 x4;
    typedef typename T::x8 x8;
    constexpr int BK = kKeyTile, CH = D / 8;   // keys per tile, 16-byte chunks per row
    constexpr int RI = 64 / CH, NI = 16 / RI;  // rows of one load of a wave; loads of its 16 rows of a tile
    constexpr uint32_t kTile = BK * D * 2;     // bytes
    constexpr bool PAGED = FROM != kRows;
    __shared__ __align__(1024) char smem[4 * kTile];  // keys of two tiles, values of two
    __shared__ int odd;  // a value on the edge is infinite or NaN

    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
    const int hk = blockIdx.x % a.hkv, item = blockIdx.x / a.hkv;
    const bool report = blockIdx.x == 0 && tid < 64;
    const Group lens = first_group<PAGED>(a, lane, report);
    if (!PAGED && report) {
        int reach = lens.reach;
        for (int at = 64; at < a.s.B; at += 64) read_lens<false>(a, at, lane, reach, true);
    }
    const int chunk = PAGED ? chunk_of(a, kTileRows, lens, lane, report) : 0x7fffffff;
    const Piece piece = find_piece<PAGED, false>(a, kTileRows, lens, chunk, item, lane);
    const Unit &p = piece.u;
    if (!p.ok) return;

    // rows of this workgroup and wave: keys that a row sees are [0, token + first)
    const int rows = p.n * a.G, row0 = p.tile * kTileRows;
    const int first = p.L - p.n + 1;
    const int wg_last = min(row0 + kTileRows, rows) - 1;
    const int wg_most = min(p.L, max(0, wg_last / a.G + first));  // most keys a row of the workgroup sees
    int t_lo = 0, t_hi = (wg_most + BK - 1) / BK;
    if (PAGED && piece.splits > 1) {
        t_lo = piece.split * chunk;
        t_hi = min(t_hi, t_lo + chunk);
    }

    const int wrow0 = row0 + w * 32;
    const int row = wrow0 + (lane & 31), half = lane >> 5;
    const bool live = row < rows;
    const int tok = live ? row / a.G : 0;
    const int qh = hk * a.G + (row - tok * a.G);
    const int ends = live ? max(0, min(p.L, tok + first)) : 0;  // keys this lane's row sees
    const int w_most = wrow0 < rows ? min(p.L, max(0, (min(wrow0 + 32, rows) - 1) / a.G + first)) : 0;
    const int w_least = wrow0 < rows ? max(0, min(p.L, wrow0 / a.G + first)) : 0;

    // queries: the first product's second operand, column = row of the tile
    x8 q[D / 16];
    {
        const el *src =
            (const el *)a.q.data + (p.lo_row + (int64_t)tok) * a.q.token + (int64_t)qh * a.q.head + half * 8;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            const bool in = live && s * 16 + half * 8 < a.d;
            u32x4 x = {0, 0, 0, 0};
            if (in) x = *(const u32x4 *)(src + s * 16);
            q[s] = __builtin_bit_cast(x8, x);
        }
    }

    f32x16 o[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    float m = kLowest, l = 0.0f;

    int ids1 = 0, ids2 = 0;
    // Loads of a tile: wave w brings rows [16 w, 16 w + 16), RI rows a load.  A
    // row's chunks are xored in LDS against bank conflicts: keys, read by many
    // rows at once, by the row; values, read four rows times 64 bytes at once,
    // in groups of four chunks.  Lane i's chunk is the one that belongs at its place.
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int lr = lane / CH, lc = lane % CH;
    const int64_t tok_k = PAGED ? a.c.token : a.k.token, tok_v = PAGED ? a.c.token : a.v.token;
    const char *base_k = PAGED ? a.c.k + (int64_t)hk * a.c.head * 2
                               : a.k.data + (p.lo_row * a.k.token + (int64_t)hk * a.k.head) * 2;
    const char *base_v = PAGED ? a.c.v + (int64_t)hk * a.c.head * 2
                               : a.v.data + (p.lo_row * a.v.token + (int64_t)hk * a.v.head) * 2;
    auto chunk_k = [&](int i) { return lc ^ ((i * RI + lr) & (CH < 16 ? CH - 1 : 15)); };
    auto chunk_v = [&](int i) {
        const int r = i * RI + lr;
        return CH < 16 ? lc ^ (((r >> 1) & 1) << 2) : lc ^ ((r & 3) << 2);
    };
    // lanes past a head's last dimension load nothing: their places in LDS are zero from the start
    const bool whole = a.d == D;
    const int page_mask = (1 << a.c.page_shift) - 1;
    // Rows of one page a load: addresses are a scalar and a lane's constant (token strides are under 2^24).  Lane i's
    // entry is the page of load i, or one that may be read where none belongs.
    auto pages_of = [&](int t) {
        int id = 0;
        if (FROM == kPages && lane < NI && t >= t_lo) {
            const int key = t * BK + w * 16 + lane * RI;
            if (key < wg_most) {
                id = a.s.pages[p.b * a.s.pages_stride + (key >> a.c.page_shift)];
                if ((uint32_t)id >= (uint32_t)a.c.n_pages) {
                    id = 0;
                    if (a.status) a.status[p.b] = FATE_EINVAL;
                }
            }
        }
        return id;
    };
    auto load_rows = [&](bool keys, int t, int ids, uint32_t dst) __attribute__((always_inline)) {
        dst += w * 16 * D * 2;
        const int key0 = t * BK + w * 16;
        const int64_t tok = keys ? tok_k : tok_v;
        const char *base = keys ? base_k : base_v;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int key = key0 + i * RI, c = keys ? chunk_k(i) : chunk_v(i);
            const char *src = PAGED ? base + (lane_of(ids, i) * a.c.page + (key & page_mask) * tok) * 2
                                    : base + (int64_t)key * tok * 2;
            if (whole || c * 8 < a.d) dma16(src, (uint32_t)(lr * (int)tok * 2 + c * 16), dst + i * 1024);
        }
    };
    // Row by row: pages of fewer rows than a load, and the last tile of a prompt (rows past its end: the last one
    // again; a cached sequence's are of their page's own slots).  Both tiles' pages are looked up before either's rows.
    auto load_by_row = [&](int tv, uint32_t dst_v, int tk, uint32_t dst_k) __attribute__((always_inline)) {
        int id[2][NI];
        if (PAGED) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int t = x ? tk : tv, key = max(0, min(t * BK + w * 16 + i * RI + lr, wg_most - 1));
                    id[x][i] = a.s.pages[p.b * a.s.pages_stride + (key >> a.c.page_shift)];
                }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int t = x ? tk : tv;
            if (t < t_lo) continue;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int key = min(t * BK + w * 16 + i * RI + lr, wg_most - 1), c = x ? chunk_k(i) : chunk_v(i);
                const char *src = (x ? base_k : base_v) + c * 16;
                bool in = c * 8 < a.d;
                if (PAGED) {
                    if ((uint32_t)id[x][i] >= (uint32_t)a.c.n_pages) {
                        in = false;
                        if (a.status) a.status[p.b] = FATE_EINVAL;
                    }
                    src += (id[x][i] * a.c.page + (key & page_mask) * (x ? tok_k : tok_v)) * 2;
                } else {
                    src += (int64_t)key * (x ? tok_k : tok_v) * 2;
                }
                if (in) dma16(src, (x ? dst_k : dst_v) + w * 16 * D * 2 + i * 1024);
            }
        }
    };
    // values of tile tv and keys of tile tk (those there are); last: the last tile is one of them
    auto load_tiles = [&](bool last, int tv, int ids_v, uint32_t dst_v, int tk, int ids_k,
                          uint32_t dst_k) __attribute__((always_inline)) {
        if (FROM == kPages || (FROM == kRows && !last)) {
            if (tv >= t_lo) load_rows(false, tv, ids_v, dst_v);
            if (tk >= t_lo) load_rows(true, tk, ids_k, dst_k);
        } else {
            load_by_row(tv, dst_v, tk, dst_k);
        }
    };
    const int wg_least = max(0, min(p.L, row0 / a.G + first));  // fewest keys a row of the workgroup sees

    // LDS addresses of the products' operands (the xors as above)
    const int r32 = lane & 31;
    const uint32_t k0 = lds0 + r32 * D * 2 + ((half ^ (r32 & (CH < 16 ? CH - 1 : 15))) * 16);
    const int vr = 4 * half + (lane & 15) / 4;
    const int vx = CH < 16 ? (vr >> 1) & 1 : vr & 3;
    const uint32_t v0 = lds0 + 2 * kTile + vr * D * 2 + vx * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    auto scores = [&](f32x16 (&s)[2], uint32_t buf) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int j = 0; j < 16; ++j) s[kt][j] = 0.0f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const uint32_t at = (k0 ^ (i * 32)) + (kt * 32 * D * 2 + buf);
                const x8 kf = *(__attribute__((address_space(3))) const x8 *)(uintptr_t)at;
                s[kt] = T::mfma32(kf, q[i], s[kt]);
            }
        }
    };

    // Tile t is in buffer B: its scores are in `cur` when its turn comes, and
    // the next tile's are worked out beside its softmax.
    auto step = [&](auto which, int t, f32x16 (&cur)[2], f32x16 (&nxt)[2]) {
        constexpr uint32_t B = decltype(which)::value;
        load_tiles(false, t - 1, ids1, lds0 + (2 + (B ^ 1)) * kTile, t - 2, ids2, lds0 + B * kTile);
        ids1 = ids2;
        ids2 = pages_of(t - 3);
        if ((t + 1) * BK > wg_least) {  // uniform: on the edge of some row
            bool any = false;
#pragma unroll
            for (int j = 0; j < BK * CH / 256; ++j) {
                const int c = tid + 256 * j;
                u32x4 *at = (u32x4 *)(smem + (2 + B) * kTile + c * 16);
                u32x4 x = *at;
                if (not_finite<T>(x[0]) | not_finite<T>(x[1]) | not_finite<T>(x[2]) | not_finite<T>(x[3])) {
                    any = any || t * BK + c / CH < wg_most;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = only_finite<T>(x[e]);
                    *at = x;
                }
            }
            if (any) odd = 1;
            __syncthreads();
        }
        if (t * BK < w_most) {  // uniform in the wave
            // cur[kt][j]: key kt * 32 + 8 (j / 4) + 4 half + j % 4 of the tile, row lane % 32
            if ((t + 1) * BK > w_least) {
                asm volatile("");  // a branch, not selects in every tile
                const int left = ends - t * BK - 4 * half;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (kt * 32 + 8 * (j / 4) + j % 4 >= left) cur[kt][j] = -INFINITY;
            }
            float top = cur[0][0];
#pragma unroll
            for (int j = 1; j < 16; ++j) top = fmaxf(top, cur[0][j]);
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, cur[1][j]);
            top = fmaxf(both_halves_max(top) * a.scale_log2, kLowest);
            if (__any(top > m + (kLag + T::kLift))) {
                const float next = fmaxf(m, top - T::kLift), f = exp2_fast(m - next);
                m = next;
                l *= f;
#pragma unroll
                for (int i = 0; i < D / 32; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][j] *= f;
            }
            scores(nxt, (B ^ 1) * kTile);  // past the last tile: of nothing, and not used
            x8 pr[4];                      // weights of keys 16 i + 8 (e / 4) + 4 half + e % 4
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = exp2_fast(__builtin_fmaf(cur[i / 2][8 * (i % 2) + e], a.scale_log2, -m));
                    l += x;
                    pr[i][e] = (el)x;
                }
            // second product: v transposed, four keys at a time, in the weights' order
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) {
                    const uint32_t at = (v0 ^ (dt * 64)) + (i * 16 * D * 2 + B * kTile);
                    const x4 v1 = T::read_tr_at(at);
                    const x4 v2 = T::read_tr_at(at + 8 * D * 2);
                    const x8 vf = __builtin_shufflevector(v1, v2, 0, 1, 2, 3, 4, 5, 6, 7);
                    o[dt] = T::mfma32(vf, pr[i], o[dt]);
                }
            // the order of issue: the next scores' products, each behind its read, with the softmax
            // between them (2067 us where the scheduler's own order took 2097), then the second product
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
            for (int g = 0; g < 2 * (D / 16); ++g) {
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // matrix
                __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);  // vector
                __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);  // exponential
            }
#pragma unroll
            for (int g = 0; g < 4 * (D / 32); ++g) {
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
        } else if (t - 1 >= t_lo && (t - 1) * BK < w_most) {
            scores(nxt, (B ^ 1) * kTile);
        }
        dma_wait();
        __syncthreads();
    };

    if (tid == 0) odd = 0;
    if (!whole) {
#pragma unroll
        for (int i = 0; i < (int)(4 * kTile / 4096); ++i) *(u32x4 *)(smem + (i * 256 + tid) * 16) = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
    if (t_hi > t_lo) {
        const int ids0 = pages_of(t_hi - 1);
        load_tiles(true, t_hi - 1, ids0, lds0 + 2 * kTile, t_hi - 1, ids0, lds0);
        ids1 = pages_of(t_hi - 2);
        load_tiles(false, t_lo - 1, 0, 0, t_hi - 2, ids1, lds0 + kTile);
        ids2 = pages_of(t_hi - 3);
    }
    dma_wait();
    __syncthreads();
    f32x16 sa[2], sb[2];
    scores(sa, 0);
    __syncthreads();  // the first step loads over these keys
    for (int t = t_hi - 1; t >= t_lo; t -= 2) {
        step(std::integral_constant<uint32_t, 0>(), t, sa, sb);
        if (t - 1 >= t_lo) step(std::integral_constant<uint32_t, 1>(), t - 1, sb, sa);
    }

    if (odd) {  // values that the tiles left out, for the rows that see them (any weight makes them what they are)
        for (int key = max(t_lo, wg_least / BK) * BK; key < min(ends, t_hi * BK); ++key) {
            const el *src;
            if (PAGED) {
                const int page = a.s.pages[p.b * a.s.pages_stride + (key >> a.c.page_shift)];
                if ((uint32_t)page >= (uint32_t)a.c.n_pages) continue;
                src = (const el *)a.c.v + page * a.c.page + (int64_t)hk * a.c.head +
                      (key & ((1 << a.c.page_shift) - 1)) * a.c.token;
            } else {
                src = (const el *)a.v.data + (p.lo_row + (int64_t)key) * a.v.token + (int64_t)hk * a.v.head;
            }
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = dt * 32 + 8 * j + 4 * half;
                    x4 x = {};
                    if (c < a.d) x = *(const x4 *)(src + c);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[dt][4 * j + e] += __builtin_isfinite((float)x[e]) ? 0.0f : (float)x[e];
                }
        }
    }
    l += __shfl_xor(l, 32);
    const int64_t out_row = p.lo_row + (int64_t)tok;
    if (PAGED && piece.splits > 1) {  // a part of the keys: unscaled sums, joined by k_attn_join
        const int64_t at = ((int64_t)piece.slot * a.hkv + hk) * kTileRows + (row - row0);
        float *dst = a.part + at * a.d;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = dt * 32 + 8 * j + 4 * half;
                if (live && c < a.d)
                    *(f32x4 *)(dst + c) = f32x4{o[dt][4 * j], o[dt][4 * j + 1], o[dt][4 * j + 2], o[dt][4 * j + 3]};
            }
        if (live && half == 0) {
            float *ml = a.part + 2 * (int64_t)a.pieces * a.hkv * kTileRows * a.d + at * 2;
            ml[0] = m;
            ml[1] = l;
        }
        return;
    }
    // results to their rows: through the wave's 32 rows of LDS (chunks xored as
    // above), so that whole rows are written, not sixteen bytes of each of 32
    // rows at a time (373 against 340 us without the stores on a wave of prompts)
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
    char *const mine = smem + w * 32 * D * 2;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (el)(o[dt][4 * j + e] * inv);
            *(x4 *)(mine + r32 * D * 2 + ((dt * 4 + j) ^ (r32 & (CH < 16 ? CH - 1 : 15))) * 16 + half * 8) = x;
        }
    if (half == 0 && live && a.lse)
        a.lse[out_row * a.hq + qh] = l != 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    const int64_t at = live ? out_row * a.out.token + (int64_t)qh * a.out.head : -1;
#pragma unroll
    for (int i = 0; i < 32 / RI; ++i) {
        const int r = i * RI + lr;
        const int64_t to =
            (int64_t)(((uint64_t)(uint32_t)__shfl((int)(at >> 32), r) << 32) | (uint32_t)__shfl((int)at, r));
        const x8 x = *(const x8 *)(mine + r * D * 2 + (lc ^ (r & (CH < 16 ? CH - 1 : 15))) * 16);
        if (to >= 0 && lc * 8 < a.d) *(x8 *)((el *)a.out.data + to + lc * 8) = x;
    }
}

template <class T, Source FROM>
int go(const AttnLaunch &a, hipStream_t s) {
    const dim3 grid((unsigned)a.grid * (unsigned)a.hkv);
    if (a.d <= 64) hipLaunchKernelGGL((k_attn_tile<T, 64, FROM>), grid, dim3(256), 0, s, a);
    else if (a.d <= 128) hipLaunchKernelGGL((k_attn_tile<T, 128, FROM>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_attn_tile<T, 256, FROM>), grid, dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

template <class T>
int go(const AttnLaunch &a, bool paged, hipStream_t s) {
    if (!paged) return go<T, kRows>(a, s);
    const int rows = a.d <= 64 ? 8 : a.d <= 128 ? 4 : 2;  // of a load: 1024 bytes
    return (1 << a.c.page_shift) >= rows ? go<T, kPages>(a, s) : go<T, kSmallPages>(a, s);
}

}  // namespace

int launch_attn_tile(const AttnLaunch &a, bool paged, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return a.dtype == FATE_BF16 ? go<BF16>(a, paged, s) : go<F16>(a, paged, s);
}

}  // namespace fate
