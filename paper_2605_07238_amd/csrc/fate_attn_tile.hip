// Causal attention with matrix tiles: whole prompts over packed keys, and
// chunks of new tokens over a paged cache.
//
//   S = scale q k^T over the keys a row sees, O = softmax(S) v
// One pass over the keys with the running maximum m and sum l of each row:
// per key tile, m' = max(m, max S), O = O 2^(m - m') + 2^(S - m') v (S in
// units of log2), l likewise; at the end O / l.  m moves only when a tile
// exceeds it by more than 8, so the weights stay under 2^8 and O is rescaled
// rarely.
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
// Key tiles go from the last to the first: the tiles on a row's causal edge
// come first.  Values that a row must not see cannot be left out of a matrix
// product by a zero weight when they are infinite or NaN (0 * inf): in the
// tiles on an edge such values are stored as zeros, and added at the end to
// the rows that do see them.
#include "fate_attn.h"

namespace fate {
namespace {

// Rows of a tile in LDS are padded against bank conflicts: keys are read by
// eight rows at once, 16 bytes each (rows 16 bytes apart in the banks), values
// four rows at once, 64 bytes each (rows 64 bytes apart).  Padding, unlike
// xored chunks, leaves every address one register plus a constant.
constexpr int kKeyPad = 8, kValPad = 32;

template <class T, int D, bool PAGED>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void k_attn_tile(AttnLaunch a) {
    typedef typename T::el el;
    typedef typename T::x4 x4;
    typedef typename T::x8 x8;
    constexpr int BK = kKeyTile, CH = D / 8;  // keys per tile, 16-byte chunks per row
    constexpr int NL = BK * CH / 256;         // chunks each thread loads of a key (and of a value) tile
    constexpr int KS = D + kKeyPad, VS = D + kValPad;
    __shared__ __align__(16) el sk[2][BK * KS];
    __shared__ __align__(16) el sv[2][BK * VS];
    __shared__ int odd;  // a value on the edge is infinite or NaN

    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
    const int hk = blockIdx.x % a.hkv, item = blockIdx.x / a.hkv;
    const bool report = blockIdx.x == 0 && tid < 64;
    const Lens lens = read_lens<PAGED>(a, lane, report);
    const int chunk = PAGED ? chunk_of(a, kTileRows, lens, lane, report) : 0x7fffffff;
    const Piece piece = find_piece<PAGED, false>(a, kTileRows, lens, chunk, item, lane, !PAGED && report);
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
        const el *src = (const el *)a.q.data + (p.lo_row + (int64_t)tok) * a.q.token + (int64_t)qh * a.q.head + half * 8;
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

    // key and value chunks of this thread: rows ld_row + i * (256 / CH), chunk ld_col
    const int ld_row = tid / CH, ld_col = tid % CH;
    const bool ld_in = ld_col * 8 < a.d;
    u32x4 rk[NL], rv[NL];
    int pg[NL];  // pages of the tile to load next
    auto find_pages = [&](int t) {
        if (PAGED) {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int key = t * BK + ld_row + i * (256 / CH);
                pg[i] = key < wg_most ? a.s.pages[p.b * a.s.pages_stride + (key >> a.c.page_shift)] : 0;
            }
        }
    };
    auto load_tile = [&](int t) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int key = t * BK + ld_row + i * (256 / CH);
            bool in = ld_in && key < wg_most;
            rk[i] = u32x4{0, 0, 0, 0};
            rv[i] = u32x4{0, 0, 0, 0};
            if (PAGED) {
                if (in && (uint32_t)pg[i] >= (uint32_t)a.c.n_pages) {
                    in = false;
                    if (a.status) a.status[p.b] = FATE_EINVAL;
                }
                const int64_t at = pg[i] * a.c.page + (int64_t)hk * a.c.head +
                                   (key & ((1 << a.c.page_shift) - 1)) * a.c.token + ld_col * 8;
                if (in) {
                    rk[i] = *(const u32x4 *)((const el *)a.c.k + at);
                    rv[i] = *(const u32x4 *)((const el *)a.c.v + at);
                }
            } else {
                const int64_t r = p.lo_row + (int64_t)key;
                if (in) {
                    rk[i] = *(const u32x4 *)((const el *)a.k.data + r * a.k.token + (int64_t)hk * a.k.head + ld_col * 8);
                    rv[i] = *(const u32x4 *)((const el *)a.v.data + r * a.v.token + (int64_t)hk * a.v.head + ld_col * 8);
                }
            }
        }
    };
    const int wg_least = max(0, min(p.L, row0 / a.G + first));  // fewest keys a row of the workgroup sees
    auto store_tile = [&](int t, int buf) {
        if ((t + 1) * BK > wg_least) {  // uniform: on the edge of some row
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < NL; ++i)
                bad |= not_finite<T>(rv[i][0]) | not_finite<T>(rv[i][1]) | not_finite<T>(rv[i][2]) | not_finite<T>(rv[i][3]);
            if (bad) {
                odd = 1;
#pragma unroll
                for (int i = 0; i < NL; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) rv[i][e] = only_finite<T>(rv[i][e]);
            }
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int r = ld_row + i * (256 / CH);
            *(u32x4 *)&sk[buf][r * KS + ld_col * 8] = rk[i];
            *(u32x4 *)&sv[buf][r * VS + ld_col * 8] = rv[i];
        }
    };

    int buf = 0;
    if (tid == 0) odd = 0;
    if (t_hi > t_lo) {
        find_pages(t_hi - 1);
        load_tile(t_hi - 1);
        if (t_hi - 1 > t_lo) find_pages(t_hi - 2);
    }
    __syncthreads();
    if (t_hi > t_lo) store_tile(t_hi - 1, 0);
    __syncthreads();

    for (int t = t_hi - 1; t >= t_lo; --t) {
        if (t > t_lo) {
            load_tile(t - 1);
            if (t - 1 > t_lo) find_pages(t - 2);
        }
        if (t * BK < w_most) {  // uniform in the wave
            f32x16 s[2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int j = 0; j < 16; ++j) s[kt][j] = 0.0f;
                const int r = kt * 32 + (lane & 31);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const x8 kf = *(const x8 *)&sk[buf][r * KS + i * 16 + half * 8];
                    s[kt] = T::mfma32(kf, q[i], s[kt]);
                }
            }
            // s[kt][j]: key kt * 32 + 8 (j / 4) + 4 half + j % 4 of the tile, row lane % 32
            const bool edge = (t + 1) * BK > w_least;
            if (edge) {
                asm volatile("");  // a branch, not selects in every tile
                const int left = ends - t * BK - 4 * half;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (kt * 32 + 8 * (j / 4) + j % 4 >= left) s[kt][j] = -INFINITY;
            }
            float top = s[0][0];
#pragma unroll
            for (int j = 1; j < 16; ++j) top = fmaxf(top, s[0][j]);
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[1][j]);
            top = fmaxf(top, __shfl_xor(top, 32));
            top = fmaxf(top * a.scale_log2, kLowest);
            if (__any(top > m + 8.0f)) {
                const float next = fmaxf(m, top), f = exp2_fast(m - next);
                m = next;
                l *= f;
#pragma unroll
                for (int i = 0; i < D / 32; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][j] *= f;
            }
            x8 pr[4];  // weights of keys 16 i + 8 (e / 4) + 4 half + e % 4
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = exp2_fast(__builtin_fmaf(s[i / 2][8 * (i % 2) + e], a.scale_log2, -m));
                    l += x;
                    pr[i][e] = (el)x;
                }
            // second product: v transposed, four keys at a time, in the weights' order
            const int vr = 4 * half + (lane & 15) / 4, vc = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) {
                    const int r1 = 16 * i + vr, r2 = r1 + 8, c = dt * 32 + vc;
                    const x4 v1 = T::read_tr(&sv[buf][r1 * VS + c]);
                    const x4 v2 = T::read_tr(&sv[buf][r2 * VS + c]);
                    const x8 vf = __builtin_shufflevector(v1, v2, 0, 1, 2, 3, 4, 5, 6, 7);
                    o[dt] = T::mfma32(vf, pr[i], o[dt]);
                }
        }
        if (t > t_lo) store_tile(t - 1, buf ^ 1);
        __syncthreads();
        buf ^= 1;
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
                    for (int e = 0; e < 4; ++e) o[dt][4 * j + e] += __builtin_isfinite((float)x[e]) ? 0.0f : (float)x[e];
                }
        }
    }
    l += __shfl_xor(l, 32);
    if (!live) return;
    const int64_t out_row = p.lo_row + (int64_t)tok;
    if (PAGED && piece.splits > 1) {  // a part of the keys: unscaled sums, joined by k_attn_join
        const int64_t at = ((int64_t)piece.slot * a.hkv + hk) * kTileRows + (row - row0);
        float *dst = a.part + at * a.d;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = dt * 32 + 8 * j + 4 * half;
                if (c < a.d) *(f32x4 *)(dst + c) = f32x4{o[dt][4 * j], o[dt][4 * j + 1], o[dt][4 * j + 2], o[dt][4 * j + 3]};
            }
        if (half == 0) {
            float *ml = a.part + 2 * (int64_t)a.pieces * a.hkv * kTileRows * a.d + at * 2;
            ml[0] = m;
            ml[1] = l;
        }
        return;
    }
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
    el *dst = (el *)a.out.data + out_row * a.out.token + (int64_t)qh * a.out.head;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = dt * 32 + 8 * j + 4 * half;
            x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (el)(o[dt][4 * j + e] * inv);
            if (c < a.d) *(x4 *)(dst + c) = x;
        }
    if (half == 0 && a.lse)
        a.lse[out_row * a.hq + qh] = l != 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

template <class T, bool PAGED>
int go(const AttnLaunch &a, hipStream_t s) {
    const dim3 grid((unsigned)a.grid * (unsigned)a.hkv);
    if (a.d <= 64) hipLaunchKernelGGL((k_attn_tile<T, 64, PAGED>), grid, dim3(256), 0, s, a);
    else if (a.d <= 128) hipLaunchKernelGGL((k_attn_tile<T, 128, PAGED>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_attn_tile<T, 256, PAGED>), grid, dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_attn_tile(const AttnLaunch &a, bool paged, void *stream) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (a.dtype == FATE_BF16) return paged ? go<BF16, true>(a, s) : go<BF16, false>(a, s);
    return paged ? go<F16, true>(a, s) : go<F16, false>(a, s);
}

}  // namespace fate
