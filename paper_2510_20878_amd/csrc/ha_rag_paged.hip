// Entry points of include/ha_rag.h for new tokens in a paged cache: checks of arguments, the layout of a step's plan, launches.
#include "ha_rag_internal.h"
#include "ha_rag_paged.h"

#include <algorithm>

using namespace ha_rag_host;

namespace {

constexpr uint64_t kMaxQueryRows = 1ull << 27;
constexpr uint64_t kMaxWorkgroups = 1ull << 23;  // of 256 threads: a grid's threads are counted in 32 bits

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1u)) == 0; }

// Where the rows that the step has room for come to no more than 16 query rows of a KV head per request, all tiles are of
// 16 (a request with more has several); else requests of more than 16 have tiles of kStepTileRows.
StepLayout step_layout(const ha_rag_ctx *c, uint32_t n_requests, uint32_t n_rows, uint32_t n_q_heads)
{
    const uint32_t H = c->cfg.n_kv_heads, share = n_q_heads / H;
    StepLayout l{};
    l.rows_only = (uint64_t)n_rows * share <= 16ull * n_requests;
    l.target = std::max(1u, 2u * kChipCUs / H);
    l.part_rows = l.rows_only ? 16u : kStepTileRows;
    const uint32_t tiles = std::min(n_requests, n_rows) + (uint32_t)((uint64_t)n_rows * share / l.part_rows);
    l.cap_wgs = std::max(l.target, tiles);
    uint64_t at = 0;
    auto section = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += (bytes + 255u) / 256u * 256u;
        return here;
    };
    section(sizeof(StepHdr));
    l.req = section((uint64_t)n_requests * sizeof(StepReq));
    l.freed_ex = section((n_requests + 1ull) * 4u);
    l.line_ex = section((n_requests + 1ull) * 4u);
    l.work = section((uint64_t)n_requests * sizeof(StepWork));
    l.starts = section((uint64_t)l.cap_wgs * sizeof(StepStart));
    l.counters = section((uint64_t)l.target * H * 4u);
    // a run has two tiles at most that others have a part of, too: its first and its last
    l.parts = section(2ull * l.target * H * step_part_floats(c->cfg.head_dim, l.part_rows) * 4u);
    l.total = at;
    return l;
}

bool step_counts_ok(const ha_rag_ctx *c, uint32_t n_requests, uint32_t n_rows, uint32_t n_q_heads)
{
    const uint32_t H = c->cfg.n_kv_heads;
    return n_requests != 0 && n_requests <= HA_RAG_MAX_PAGED_REQUESTS && n_rows != 0 && n_rows <= 0x7FFFFFFFu &&
           n_q_heads != 0 && n_q_heads % H == 0 && n_q_heads / H <= 64u && H <= 65535u &&
           (uint64_t)n_rows * (n_q_heads / H) <= kMaxQueryRows &&
           (uint64_t)step_layout(c, n_requests, n_rows, n_q_heads).cap_wgs * H <= kMaxWorkgroups;
}

int check_step(const ha_rag_ctx *c, const ha_rag_paged_step *s, StepLayout *lay)
{
    if (!s || !s->row_start || !s->slots || !s->plan || !step_counts_ok(c, s->n_requests, s->n_rows, s->n_q_heads))
        return HA_RAG_EINVAL;
    if (!aligned(s->row_start, 4) || !aligned(s->slots, 4) || !aligned(s->positions, 4) || !aligned(s->refused, 4) ||
        !aligned(s->plan, 256))
        return HA_RAG_EINVAL;
    *lay = step_layout(c, s->n_requests, s->n_rows, s->n_q_heads);
    return s->plan_bytes < lay->total ? HA_RAG_ENOSPC : HA_RAG_OK;
}

int check_pool(const ha_rag_paged_cache *pg)
{
    if (!pg || !pg->base || pg->page_tokens == 0 || pg->n_pages == 0) return HA_RAG_EINVAL;
    if (!aligned(pg->base, 16) || !aligned(pg->bad_pages, 4)) return HA_RAG_EINVAL;
    if ((pg->page_stride & 15u) || (pg->tile_stride & 15u)) return HA_RAG_EINVAL;
    if ((uint64_t)pg->n_pages * pg->page_tokens > 0x7FFFFFFFull) return HA_RAG_EINVAL;
    return HA_RAG_OK;
}

bool rows_ok(const ha_rag_rows *r)
{
    return r && r->base && aligned(r->base, 16) && (r->row_stride & 15u) == 0 && (r->head_stride & 15u) == 0;
}

}  // namespace

extern "C" {

int ha_rag_step_plan_bytes(ha_rag_ctx *c, uint32_t n_requests, uint32_t n_rows, uint32_t n_q_heads, size_t *bytes)
{
    if (!c || !bytes || !step_counts_ok(c, n_requests, n_rows, n_q_heads)) return HA_RAG_EINVAL;
    *bytes = (size_t)step_layout(c, n_requests, n_rows, n_q_heads).total;
    return HA_RAG_OK;
}

int ha_rag_page_step(ha_rag_ctx *c, const ha_rag_page_tables *t, const int32_t *n_new, const ha_rag_paged_step *s,
                     void *stream)
{
    if (!c || !t || !n_new) return HA_RAG_EINVAL;
    StepLayout lay;
    const int rc = check_step(c, s, &lay);
    if (rc) return rc;
    if (!t->table || !t->n_tokens || !t->n_tokens_after || !t->free_pages || !t->n_free || !t->n_free_after)
        return HA_RAG_EINVAL;
    for (const void *x : {(const void *)t->table, (const void *)t->n_tokens, (const void *)t->n_tokens_after,
                          (const void *)t->free_pages, (const void *)t->n_free, (const void *)t->n_free_after,
                          (const void *)n_new})
        if (!aligned(x, 4)) return HA_RAG_EINVAL;
    if (t->n_requests != s->n_requests || t->n_table == 0 || t->n_pages == 0 || t->page_tokens == 0) return HA_RAG_EINVAL;
    if ((uint64_t)t->n_pages * t->page_tokens > 0x7FFFFFFFull || (uint64_t)t->n_table * t->page_tokens > 0x7FFFFFFFull ||
        (uint64_t)t->n_requests * t->n_table > 0x7FFFFFFFull)
        return HA_RAG_EINVAL;
    if (c->dry()) return HA_RAG_OK;
    K9Params p{};
    p.table = t->table;
    p.n_tokens = t->n_tokens;
    p.n_tokens_after = t->n_tokens_after;
    p.free_pages = t->free_pages;
    p.n_free = t->n_free;
    p.n_free_after = t->n_free_after;
    p.n_new = n_new;
    p.row_start = s->row_start;
    p.slots = s->slots;
    p.positions = s->positions;
    p.refused = s->refused;
    p.plan = static_cast<uint8_t *>(s->plan);
    p.lay = lay;
    p.n_requests = s->n_requests;
    p.n_table = t->n_table;
    p.n_pages = t->n_pages;
    p.page_tokens = t->page_tokens;
    p.n_rows = s->n_rows;
    p.n_q_heads = s->n_q_heads;
    p.n_kv_heads = c->cfg.n_kv_heads;
    p.head_dim = c->cfg.head_dim;
    p.n_layers = c->cfg.n_layers;
    p.unit = step_unit(t->n_table, t->page_tokens);
    std::lock_guard<std::mutex> g(c->mu);
    HIPCHK(c, launch_k9(p, (hipStream_t)stream));
    return HA_RAG_OK;
}

int ha_rag_append_paged(ha_rag_ctx *c, const ha_rag_rows *k, const ha_rag_rows *v, const ha_rag_paged_step *s,
                        const ha_rag_paged_cache *cache, uint32_t layer, void *stream)
{
    if (!c || !s || !s->slots || !aligned(s->slots, 4) || s->n_rows == 0 || s->n_rows > 0x7FFFFFFFu) return HA_RAG_EINVAL;
    if (!rows_ok(k) || !rows_ok(v) || layer >= c->cfg.n_layers) return HA_RAG_EINVAL;
    const int rc = check_pool(cache);
    if (rc) return rc;
    if (c->dry()) return HA_RAG_OK;
    K10Params p{};
    p.k = static_cast<const uint8_t *>(k->base);
    p.v = static_cast<const uint8_t *>(v->base);
    p.k_row = k->row_stride;
    p.k_head = k->head_stride;
    p.v_row = v->row_stride;
    p.v_head = v->head_stride;
    p.slots = s->slots;
    p.base = static_cast<uint8_t *>(cache->base);
    p.bad_pages = cache->bad_pages;
    p.page_stride = cache->page_stride;
    p.tile_stride = cache->tile_stride;
    p.n_rows = s->n_rows;
    p.n_kv_heads = c->cfg.n_kv_heads;
    p.head_dim = c->cfg.head_dim;
    p.page_tokens = cache->page_tokens;
    p.n_pages = cache->n_pages;
    p.layer = layer;
    std::lock_guard<std::mutex> g(c->mu);
    HIPCHK(c, launch_k10(p, (hipStream_t)stream));
    return HA_RAG_OK;
}

int ha_rag_attend_paged(ha_rag_ctx *c, const ha_rag_rows *q, const ha_rag_paged_step *s, const ha_rag_paged_cache *cache,
                        uint32_t layer, float sm_scale, const ha_rag_rows *out, float *lse, const float *prior_out,
                        const float *prior_lse, void *stream)
{
    if (!c) return HA_RAG_EINVAL;
    if (!step_head_dim(c->cfg.head_dim)) return HA_RAG_EFORMAT;
    StepLayout lay;
    int rc = check_step(c, s, &lay);
    if (rc) return rc;
    if (!rows_ok(q) || !rows_ok(out) || layer >= c->cfg.n_layers || !(sm_scale > 0.0f) || !(sm_scale < 1e30f)) return HA_RAG_EINVAL;
    if (!aligned(lse, 4) || !aligned(prior_out, 16) || !aligned(prior_lse, 4) || !prior_out != !prior_lse) return HA_RAG_EINVAL;
    if ((rc = check_pool(cache)) != HA_RAG_OK) return rc;
    if (!cache->page_table || !aligned(cache->page_table, 4) || cache->n_table == 0) return HA_RAG_EINVAL;
    if (c->dry()) return HA_RAG_OK;
    K11Params p{};
    p.q = static_cast<const uint8_t *>(q->base);
    p.q_row = q->row_stride;
    p.q_head = q->head_stride;
    p.out = static_cast<uint8_t *>(out->base);
    p.out_row = out->row_stride;
    p.out_head = out->head_stride;
    p.lse = lse;
    p.prior_out = prior_out;
    p.prior_lse = prior_lse;
    p.base = static_cast<const uint8_t *>(cache->base);
    p.table = cache->page_table;
    p.bad_pages = cache->bad_pages;
    p.page_stride = cache->page_stride;
    p.tile_stride = cache->tile_stride;
    p.plan = static_cast<uint8_t *>(s->plan);
    p.lay = lay;
    p.scale_log2 = sm_scale * 1.44269504088896340736f;
    p.n_requests = s->n_requests;
    p.n_rows = s->n_rows;
    p.n_table = cache->n_table;
    p.n_pages = cache->n_pages;
    p.page_tokens = cache->page_tokens;
    p.n_kv_heads = c->cfg.n_kv_heads;
    p.n_q_heads = s->n_q_heads;
    p.layer = layer;
    std::lock_guard<std::mutex> g(c->mu);
    HIPCHK(c, launch_k11(p, c->cfg.head_dim, (hipStream_t)stream));
    return HA_RAG_OK;
}

}  // extern "C"
