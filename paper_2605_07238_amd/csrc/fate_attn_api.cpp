// C entries of the attention calls of a planned wave: checks of what the host
// can see, choice of the kernels, launches.  Nothing here allocates or throws.
#include <cmath>
#include <cstdint>

#include "fate.h"
#include "fate_attn.h"

namespace {

using fate::AppendLaunch;
using fate::AttnLaunch;

// Token strides of keys and values: offsets of neighbouring rows are 32-bit in the kernels.
constexpr int64_t kMaxToken = int64_t(1) << 24;
// A launch takes fewer than 2^32 threads: workgroups of 256.
constexpr int64_t kMaxGrid = (int64_t(1) << 24) - 1;

bool good_rows(const fate_rows_t *r) {
    return r && r->data && reinterpret_cast<uintptr_t>(r->data) % 16 == 0 && r->token >= 0 && r->head >= 0 &&
           r->token % 8 == 0 && r->head % 8 == 0;
}

bool good_out(const fate_rows_t *r, const fate_heads_t *h) {
    return good_rows(r) && r->token >= h->head_dim && r->head >= h->head_dim;
}

fate_status_t check_heads(const fate_heads_t *h) {
    if (!h) return FATE_EINVAL;
    if (h->dtype != FATE_BF16 && h->dtype != FATE_F16) return FATE_EINVAL;
    if (h->heads_q < 1 || h->heads_kv < 1 || h->head_dim < 1) return FATE_EINVAL;
    if (h->heads_q > FATE_MAX_HEADS || h->heads_kv > FATE_MAX_HEADS || h->head_dim > FATE_MAX_HEAD_DIM)
        return FATE_ERANGE;
    if (h->heads_q % h->heads_kv || h->head_dim % 8) return FATE_EINVAL;
    return FATE_OK;
}

fate_status_t check_sizes(const fate_heads_t *h, const fate_seqs_t *s) {
    if (!s || s->B < 0 || s->T < 0) return FATE_EINVAL;
    // packed rows and piece numbers are 32-bit in the kernels (T first: the product is then within 64 bits)
    if (s->T >= (int64_t(1) << 31) || s->T * (int64_t)(h->heads_q + 2 * h->heads_kv) >= (int64_t(1) << 31) ||
        s->B > (1 << 24))
        return FATE_ERANGE;
    return FATE_OK;
}

fate_status_t check_cache(const fate_heads_t *h, const fate_seqs_t *s, const fate_kv_cache_t *c) {
    if (!c || s->max_pages < 0 || s->pages_stride < 0 || c->n_pages < 0) return FATE_EINVAL;
    if (c->page_size < 1 || (c->page_size & (c->page_size - 1))) return FATE_EINVAL;
    if (c->page_size > 1024 || (int64_t)s->max_pages * c->page_size > (int64_t(1) << 30) || c->token >= kMaxToken)
        return FATE_ERANGE;
    const fate_rows_t k = {c->k, c->token, c->head}, v = {c->v, c->token, c->head};
    if (c->n_pages > 0 && (!good_out(&k, h) || !good_out(&v, h) || c->page < h->head_dim || c->page % 8))
        return FATE_EINVAL;
    return FATE_OK;
}

fate::RowsArg rows(const fate_rows_t *r) { return {static_cast<char *>(r->data), r->token, r->head}; }

int log2_of(int x) {
    int n = 0;
    while ((1 << n) < x) ++n;
    return n;
}

void set_seqs(fate::SeqsArg &out, const fate_seqs_t *s, const fate_kv_cache_t *c) {
    out = {s->off, s->kv_len, s->pages, s->T, s->pages_stride, c ? (int64_t)s->max_pages * c->page_size : 0, s->B};
}

void set_cache(fate::CacheArg &out, const fate_kv_cache_t *c) {
    out = {static_cast<const char *>(c->k), static_cast<const char *>(c->v), c->page, c->head, c->token, c->n_pages,
           log2_of(c->page_size)};
}

// Which kernel a paged call takes, and how its key axis is shared out.
struct PagedPlan {
    int rows;    // packed rows per workgroup: 16 or 32 (few-row kernel) or kTileRows
    int pieces;  // shares of the work axis, or parts aimed at, per key head; twice as many slots hold all partials
    int tiles;   // most row tiles of the call
    int grid;    // workgroups per key head
};

// Most row tiles of T tokens in B sequences.
int tiles_of(const fate_seqs_t *s, int64_t G, int rows) {
    return (int)(s->T * G / rows + (s->B < s->T ? s->B : s->T));
}

PagedPlan plan_paged(const fate_heads_t *h, const fate_seqs_t *s, int64_t max_new) {
    // a token's rows at least: the work axis of the few-row kernel is within 64 bits where they are 32 or fewer
    const int64_t G = h->heads_q / h->heads_kv, packed = (max_new > 1 ? max_new : 1) * G, few = h->head_dim <= 128 ? 32 : 16;
    PagedPlan p;
    p.rows = packed <= 16 ? 16 : packed <= few ? 32 : fate::kTileRows;
    // two workgroups a compute unit, one of head sizes over 128.  More shares cost more in joins and in the shares'
    // starts than they bring in loads under way, also at head size 64 where four would fit: 768 and 1024 for a step
    // of 64 answers over 128 to 8192 keys 61 and 61 against 57 us (at 128 113 and 111 against 108; at 256, for 256,
    // 81 and 88 against 68), for two over 65536 and 131072 85 and 85 against 81, for 16 chunks 74 and 78 against 56
    const int target = h->head_dim <= 128 ? 512 : 256;
    p.pieces = target / h->heads_kv > 0 ? target / h->heads_kv : 1;
    p.tiles = tiles_of(s, G, p.rows);
    p.grid = p.rows == fate::kTileRows ? p.pieces + p.tiles : p.pieces;
    return p;
}

size_t ws_of(const fate_heads_t *h, const PagedPlan &p) {
    return 2 * (size_t)p.pieces * h->heads_kv * p.rows * (h->head_dim + 2) * sizeof(float);
}

fate_status_t fill(AttnLaunch &a, const fate_heads_t *h, const fate_rows_t *q, const fate_rows_t *out, float scale,
                   float *d_lse, int32_t *d_status) {
    if (!std::isfinite(scale) || !(scale > 0.0f)) return FATE_EINVAL;
    if (!good_rows(q) || !good_out(out, h)) return FATE_EINVAL;
    a.q = rows(q);
    a.out = rows(out);
    a.lse = d_lse;
    a.status = d_status;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    if (!std::isfinite(a.scale_log2)) return FATE_EINVAL;
    a.hq = h->heads_q;
    a.hkv = h->heads_kv;
    a.G = h->heads_q / h->heads_kv;
    a.d = h->head_dim;
    a.dtype = h->dtype;
    return FATE_OK;
}

// `axes`: rotation by several axes, or null.
fate_status_t append(const fate_heads_t *heads, const fate_seqs_t *seqs, const fate_rows_t *q, const fate_rows_t *k,
                     const fate_rows_t *v, const float *table, int64_t table_rows, int32_t rot, int32_t interleaved,
                     const fate_axes_t *axes, const fate_kv_cache_t *cache, const fate_rows_t *q_out, int32_t *d_status,
                     void *stream) {
    fate_status_t st = check_heads(heads);
    if (st != FATE_OK || (st = check_sizes(heads, seqs)) != FATE_OK ||
        (st = check_cache(heads, seqs, cache)) != FATE_OK)
        return st;
    if (rot < 0 || rot > heads->head_dim || rot % 2 || table_rows < 0 || (interleaved != 0 && interleaved != 1))
        return FATE_EINVAL;
    if (rot && (!table || reinterpret_cast<uintptr_t>(table) % 4)) return FATE_EINVAL;
    if (axes) {
        if (rot < 2 || axes->n_axes < 1 || !axes->pair_axis || axes->stride < 0) return FATE_EINVAL;
        if (axes->n_axes > FATE_MAX_AXES) return FATE_ERANGE;
        for (int j = 0; j < rot / 2; ++j)
            if (axes->pair_axis[j] >= axes->n_axes) return FATE_EINVAL;
    }
    if (!q != !q_out) return FATE_EINVAL;
    if (seqs->T == 0 || seqs->B == 0) return FATE_OK;
    if (fate::append_grid(seqs->T) > kMaxGrid) return FATE_ERANGE;
    if (cache->n_pages < 1 || !seqs->off || !seqs->kv_len || !seqs->pages || !good_rows(k) || !good_rows(v))
        return FATE_EINVAL;
    if (q && (!good_rows(q) || !good_out(q_out, heads))) return FATE_EINVAL;
    if (q && q->data == q_out->data && (q->token != q_out->token || q->head != q_out->head)) return FATE_EINVAL;
    if (axes && (!axes->positions || reinterpret_cast<uintptr_t>(axes->positions) % 4)) return FATE_EINVAL;
    AppendLaunch a = {};
    set_seqs(a.s, seqs, cache);
    set_cache(a.c, cache);
    a.ck = static_cast<char *>(cache->k);
    a.cv = static_cast<char *>(cache->v);
    if (q) {
        a.q = rows(q);
        a.qo = rows(q_out);
    }
    a.k = rows(k);
    a.v = rows(v);
    a.table = table;
    a.table_rows = table_rows;
    a.status = d_status;
    a.hq = q ? heads->heads_q : 0;
    a.hkv = heads->heads_kv;
    a.d = heads->head_dim;
    a.rot = rot;
    a.interleaved = interleaved;
    a.dtype = heads->dtype;
    if (axes) {
        a.positions = axes->positions;
        a.positions_stride = axes->stride;
        a.n_axes = axes->n_axes;
        for (int j = 0; j < rot / 2; ++j) a.axis[j / 16] |= (uint32_t)axes->pair_axis[j] << j % 16 * 2;
    }
    const int64_t bytes = seqs->T * (2 * (int64_t)a.hq + 4 * (int64_t)a.hkv) * a.d * 2;
    a.past_cache = bytes > (int64_t(256) << 20);
    return fate::launch_append(a, stream) == 0 ? FATE_OK : FATE_EHIP;
}

// Caps over 100 in log2 units: see capped_wide.
constexpr float kWideCap = 100.0f;

fate_status_t fill_scores(AttnLaunch &a, const fate_scores_t *s, float scale) {
    if (!std::isfinite(s->cap) || s->cap < 0.0f) return FATE_EINVAL;
    for (const void *p : {(const void *)s->slopes, (const void *)s->prefix, (const void *)s->start})
        if (reinterpret_cast<uintptr_t>(p) % 4) return FATE_EINVAL;
    a.shaped = 1;
    if (s->cap > 0.0f) {
        a.cap_log2 = (float)((double)s->cap * 1.4426950408889634);
        a.cap_in = (float)(2.0 * (double)scale * 1.4426950408889634 / (double)s->cap);
        if (!std::isnormal(a.cap_log2) || !std::isnormal(a.cap_in)) return FATE_EINVAL;
        a.cap_wide = a.cap_log2 > kWideCap;
    }
    a.slopes = s->slopes;
    a.prefix = s->prefix;
    a.start = s->start;
    return FATE_OK;
}

// `scores`: how the scores are shaped, or null for causal ones as they are.
fate_status_t paged(const fate_heads_t *heads, const fate_seqs_t *seqs, const fate_rows_t *q,
                    const fate_kv_cache_t *cache, int64_t max_new, float scale, const fate_scores_t *scores,
                    const fate_rows_t *out, float *d_lse, int32_t *d_status, void *d_ws, size_t ws_bytes,
                    void *stream) {
    fate_status_t st = check_heads(heads);
    if (st != FATE_OK || (st = check_sizes(heads, seqs)) != FATE_OK ||
        (st = check_cache(heads, seqs, cache)) != FATE_OK)
        return st;
    if (max_new < 0 || max_new > seqs->T) return FATE_EINVAL;
    if (seqs->T == 0 || seqs->B == 0) return FATE_OK;
    if (cache->n_pages < 1 || !seqs->off || !seqs->kv_len || !seqs->pages) return FATE_EINVAL;
    const PagedPlan p = plan_paged(heads, seqs, max_new);
    if ((int64_t)p.grid * heads->heads_kv > kMaxGrid) return FATE_ERANGE;
    AttnLaunch a = {};
    if ((st = fill(a, heads, q, out, scale, d_lse, d_status)) != FATE_OK) return st;
    if (scores && (st = fill_scores(a, scores, scale)) != FATE_OK) return st;
    if (!d_ws || reinterpret_cast<uintptr_t>(d_ws) % 16) return FATE_EINVAL;
    if (ws_bytes < ws_of(heads, p)) return FATE_ESIZE;
    set_seqs(a.s, seqs, cache);
    set_cache(a.c, cache);
    a.part = static_cast<float *>(d_ws);
    a.pieces = p.pieces;
    const bool tile = p.rows == fate::kTileRows;
    a.grid = p.grid;
    const int rc = tile ? fate::launch_attn_tile(a, true, stream) : fate::launch_attn_few(a, p.rows, stream);
    if (rc) return FATE_EHIP;
    // row tiles done in parts: each has a part more than it has cuts, so fewer than there are shares; of those in
    // order of length (each with over `chunk` key tiles of the sum) fewer than pieces, and no more than there are
    const int tiles = !tile ? p.pieces - 1 : p.tiles < p.pieces ? p.tiles : p.pieces;
    // (the tile kernel makes no part of fewer than kTileLeast key tiles)
    if (tiles < 1 || (tile && a.s.max_keys <= (int64_t)fate::kTileLeast * fate::kKeyTile)) return FATE_OK;
    // four rows a workgroup at a time, sixteen at most: as many workgroups as max_new tokens have rows for
    const int64_t most = max_new * a.G < p.rows ? max_new * a.G : p.rows;
    const int groups = most > 64 ? 8 : most > 4 ? (int)((most + 3) / 4) : 1;
    return fate::launch_attn_join(a, p.rows, tiles, groups, stream) == 0 ? FATE_OK : FATE_EHIP;
}

fate_status_t prompt(const fate_heads_t *heads, const fate_seqs_t *seqs, const fate_rows_t *q, const fate_rows_t *k,
                     const fate_rows_t *v, float scale, const fate_scores_t *scores, const fate_rows_t *out,
                     float *d_lse, int32_t *d_status, void *stream) {
    fate_status_t st = check_heads(heads);
    if (st != FATE_OK || (st = check_sizes(heads, seqs)) != FATE_OK) return st;
    if (seqs->T == 0 || seqs->B == 0) return FATE_OK;
    const int64_t G = heads->heads_q / heads->heads_kv;
    const int grid = tiles_of(seqs, G, fate::kTileRows);
    if ((int64_t)grid * heads->heads_kv > kMaxGrid) return FATE_ERANGE;
    if (!seqs->off || !good_rows(k) || !good_rows(v)) return FATE_EINVAL;
    if (k->token >= kMaxToken || v->token >= kMaxToken) return FATE_ERANGE;
    AttnLaunch a = {};
    if ((st = fill(a, heads, q, out, scale, d_lse, d_status)) != FATE_OK) return st;
    if (scores && (st = fill_scores(a, scores, scale)) != FATE_OK) return st;
    set_seqs(a.s, seqs, nullptr);
    a.k = rows(k);
    a.v = rows(v);
    a.grid = grid;
    return fate::launch_attn_tile(a, false, stream) == 0 ? FATE_OK : FATE_EHIP;
}

}  // namespace

extern "C" {

fate_status_t fate_kv_append(const fate_heads_t *heads, const fate_seqs_t *seqs, const fate_rows_t *q,
                             const fate_rows_t *k, const fate_rows_t *v, const float *table, int64_t table_rows,
                             int32_t rot, int32_t interleaved, const fate_kv_cache_t *cache,
                             const fate_rows_t *q_out, int32_t *d_status, void *stream) {
    return append(heads, seqs, q, k, v, table, table_rows, rot, interleaved, nullptr, cache, q_out, d_status, stream);
}

fate_status_t fate_kv_append_axes(const fate_heads_t *heads, const fate_seqs_t *seqs, const fate_rows_t *q,
                                  const fate_rows_t *k, const fate_rows_t *v, const float *table, int64_t table_rows,
                                  int32_t rot, int32_t interleaved, const fate_axes_t *axes,
                                  const fate_kv_cache_t *cache, const fate_rows_t *q_out, int32_t *d_status,
                                  void *stream) {
    if (!axes) return FATE_EINVAL;
    return append(heads, seqs, q, k, v, table, table_rows, rot, interleaved, axes, cache, q_out, d_status, stream);
}

fate_status_t fate_attn_paged_ws_size(const fate_heads_t *heads, const fate_seqs_t *seqs,
                                      const fate_kv_cache_t *cache, int64_t max_new, size_t *bytes) {
    fate_status_t st = check_heads(heads);
    if (st != FATE_OK || (st = check_sizes(heads, seqs)) != FATE_OK ||
        (st = check_cache(heads, seqs, cache)) != FATE_OK)
        return st;
    if (!bytes || max_new < 0 || max_new > seqs->T) return FATE_EINVAL;
    if (seqs->T == 0 || seqs->B == 0) {
        *bytes = 0;
        return FATE_OK;
    }
    const PagedPlan p = plan_paged(heads, seqs, max_new);
    if ((int64_t)p.grid * heads->heads_kv > kMaxGrid) return FATE_ERANGE;
    *bytes = ws_of(heads, p);
    return FATE_OK;
}

fate_status_t fate_attn_paged(const fate_heads_t *heads, const fate_seqs_t *seqs, const fate_rows_t *q,
                              const fate_kv_cache_t *cache, int64_t max_new, float scale, const fate_rows_t *out,
                              float *d_lse, int32_t *d_status, void *d_ws, size_t ws_bytes, void *stream) {
    return paged(heads, seqs, q, cache, max_new, scale, nullptr, out, d_lse, d_status, d_ws, ws_bytes, stream);
}

fate_status_t fate_attn_prompt(const fate_heads_t *heads, const fate_seqs_t *seqs, const fate_rows_t *q,
                               const fate_rows_t *k, const fate_rows_t *v, float scale, const fate_rows_t *out,
                               float *d_lse, int32_t *d_status, void *stream) {
    return prompt(heads, seqs, q, k, v, scale, nullptr, out, d_lse, d_status, stream);
}

fate_status_t fate_attn_paged_shaped(const fate_heads_t *heads, const fate_seqs_t *seqs, const fate_rows_t *q,
                                     const fate_kv_cache_t *cache, int64_t max_new, float scale,
                                     const fate_scores_t *scores, const fate_rows_t *out, float *d_lse,
                                     int32_t *d_status, void *d_ws, size_t ws_bytes, void *stream) {
    if (!scores) return FATE_EINVAL;
    return paged(heads, seqs, q, cache, max_new, scale, scores, out, d_lse, d_status, d_ws, ws_bytes, stream);
}

fate_status_t fate_attn_prompt_shaped(const fate_heads_t *heads, const fate_seqs_t *seqs, const fate_rows_t *q,
                                      const fate_rows_t *k, const fate_rows_t *v, float scale,
                                      const fate_scores_t *scores, const fate_rows_t *out, float *d_lse,
                                      int32_t *d_status, void *stream) {
    if (!scores) return FATE_EINVAL;
    return prompt(heads, seqs, q, k, v, scale, scores, out, d_lse, d_status, stream);
}

}  // extern "C"
