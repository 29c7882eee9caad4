// C entries of the calls around the attention of a planned wave: page tables, sampling.
// Checks of what the host can see, launches.  Nothing here allocates or throws.
#include <cmath>
#include <cstdint>

#include "fate.h"
#include "fate_pages.h"
#include "fate_sample.h"

namespace {

using fate::PagesLaunch;

bool aligned(const void *p, uintptr_t n) { return p && reinterpret_cast<uintptr_t>(p) % n == 0; }

fate_status_t check_tables(const fate_kv_tables_t *t) {
    if (!t || t->B < 0 || t->max_pages < 0 || t->n_pages < 0 || t->pages_stride < 0) return FATE_EINVAL;
    if (t->page_size < 1 || (t->page_size & (t->page_size - 1))) return FATE_EINVAL;
    if (t->page_size > 1024 || (int64_t)t->max_pages * t->page_size > (int64_t(1) << 30) || t->B > (1 << 24))
        return FATE_ERANGE;
    if (t->B > 1 && t->pages_stride < t->max_pages) return FATE_EINVAL;  // rows are written
    if (!aligned(t->n_free, 4)) return FATE_EINVAL;
    if (t->B > 0 && (!aligned(t->kv_len, 4) || (t->max_pages > 0 && !aligned(t->pages, 4)))) return FATE_EINVAL;
    if (t->n_pages > 0 && !aligned(t->free, 4)) return FATE_EINVAL;
    return FATE_OK;
}

PagesLaunch launch_of(const fate_kv_tables_t *t) {
    PagesLaunch a = {};
    a.kv_len = t->kv_len;
    a.n_free = t->n_free;
    a.pages = t->pages;
    a.free = t->free;
    a.pages_stride = t->pages_stride;
    a.max_keys = (int64_t)t->max_pages * t->page_size;
    a.B = t->B;
    a.n_pages = t->n_pages;
    a.shift = __builtin_ctz((unsigned)t->page_size);
    return a;
}

// A launch takes fewer than 2^32 threads, and a row has a workgroup of 1024; places in a row are 32-bit.
constexpr int32_t kMaxRows = (1 << 22) - 1, kMaxVocab = 1 << 30;

fate_status_t check_sampling(const fate_sampling_t *s) {
    if (!s || s->rows < 0 || s->vocab < 1 || s->stride < 0) return FATE_EINVAL;
    if (s->dtype != FATE_BF16 && s->dtype != FATE_F16 && s->dtype != FATE_F32) return FATE_EINVAL;
    if (s->rows > kMaxRows || s->vocab > kMaxVocab) return FATE_ERANGE;
    if (!s->temperature && !(std::isfinite(s->temperature_all) && s->temperature_all >= 0.0f)) return FATE_EINVAL;
    if (!s->top_k && s->top_k_all < 0) return FATE_EINVAL;
    if (!s->top_p && !(s->top_p_all > 0.0f && s->top_p_all <= 1.0f)) return FATE_EINVAL;
    if (!s->min_p && !(s->min_p_all >= 0.0f && s->min_p_all <= 1.0f)) return FATE_EINVAL;
    return FATE_OK;
}

}  // namespace

extern "C" {

fate_status_t fate_kv_reserve(const fate_kv_tables_t *tables, const int32_t *new_tokens, int64_t T, int32_t *off,
                              int32_t *kv_len_out, int32_t *n_free_out, int32_t *taken, int64_t *slots,
                              int32_t *positions, int32_t *d_status, void *stream) {
    const fate_status_t st = check_tables(tables);
    if (st != FATE_OK) return st;
    if (T < 0) return FATE_EINVAL;
    if (T >= (int64_t(1) << 31)) return FATE_ERANGE;
    if (!aligned(off, 4) || !aligned(taken, 4) || !aligned(n_free_out, 4)) return FATE_EINVAL;
    if (tables->B > 0 && (!aligned(new_tokens, 4) || !aligned(kv_len_out, 4))) return FATE_EINVAL;
    if ((slots && !aligned(slots, 8)) || (positions && !aligned(positions, 4))) return FATE_EINVAL;
    PagesLaunch a = launch_of(tables);
    a.counts = new_tokens;
    a.T = T;
    a.off = off;
    a.kv_out = kv_len_out;
    a.n_free_out = n_free_out;
    a.moved = taken;
    a.slots = slots;
    a.positions = positions;
    a.status = d_status;
    return fate::launch_reserve(a, stream) == 0 ? FATE_OK : FATE_EHIP;
}

fate_status_t fate_kv_trim(const fate_kv_tables_t *tables, const int32_t *keep, int32_t *kv_len_out,
                           int32_t *n_free_out, int32_t *given, int32_t *d_status, void *stream) {
    const fate_status_t st = check_tables(tables);
    if (st != FATE_OK) return st;
    if (!aligned(given, 4) || !aligned(n_free_out, 4)) return FATE_EINVAL;
    if (tables->B > 0 && (!aligned(keep, 4) || !aligned(kv_len_out, 4))) return FATE_EINVAL;
    PagesLaunch a = launch_of(tables);
    a.counts = keep;
    a.kv_out = kv_len_out;
    a.n_free_out = n_free_out;
    a.moved = given;
    a.status = d_status;
    return fate::launch_trim(a, stream) == 0 ? FATE_OK : FATE_EHIP;
}

fate_status_t fate_sample_ws_size(const fate_sampling_t *s, size_t *bytes) {
    const fate_status_t st = check_sampling(s);
    if (st != FATE_OK) return st;
    if (!bytes) return FATE_EINVAL;
    *bytes = fate::sample_ws(s->rows, s->vocab);
    return FATE_OK;
}

fate_status_t fate_sample(const fate_sampling_t *s, int32_t *d_token, float *d_logprob, int32_t *d_status, void *d_ws,
                          size_t ws_bytes, void *stream) {
    size_t need = 0;
    const fate_status_t st = fate_sample_ws_size(s, &need);
    if (st != FATE_OK) return st;
    if (s->rows == 0) return FATE_OK;
    if (!aligned(s->logits, s->dtype == FATE_F32 ? 4 : 2) || !aligned(s->u, 4) || !aligned(d_token, 4)) return FATE_EINVAL;
    for (const void *p : {(const void *)s->temperature, (const void *)s->top_k, (const void *)s->top_p,
                          (const void *)s->min_p, (const void *)d_logprob, (const void *)d_status})
        if (p && !aligned(p, 4)) return FATE_EINVAL;
    if (need && !aligned(d_ws, 16)) return FATE_EINVAL;
    if (ws_bytes < need) return FATE_ESIZE;
    fate::SampleLaunch a = {};
    a.logits = static_cast<const char *>(s->logits);
    a.u = s->u;
    a.temperature = s->temperature;
    a.top_k = s->top_k;
    a.top_p = s->top_p;
    a.min_p = s->min_p;
    a.token = d_token;
    a.logprob = d_logprob;
    a.status = d_status;
    a.stride = s->stride;
    a.rows = s->rows;
    a.vocab = s->vocab;
    a.dtype = s->dtype;
    a.temperature_all = s->temperature_all;
    a.top_k_all = s->top_k_all;
    a.top_p_all = s->top_p_all;
    a.min_p_all = s->min_p_all;
    return fate::launch_sample(a, d_ws, stream) == 0 ? FATE_OK : FATE_EHIP;
}

}  // extern "C"
