// C entry points of the 8-bit paged cache (include/lookat_q8.h): argument checks and dispatch.
#include <cstring>

#include "pages.cuh"
#include "q8_checks.cuh"

namespace lookat {

namespace {

lookat_status state_of(Ctx *ctx, const lookat_page_state *s, PageState *out)
{
    if (!s) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "state is NULL");
    Q8_TRY(need(ctx, s->tables, "state.tables", 4));
    Q8_TRY(need(ctx, s->seq_lens, "state.seq_lens", 4));
    Q8_TRY(need(ctx, s->refs, "state.refs", 4));
    Q8_TRY(need(ctx, s->free_list, "state.free_list", 4));
    Q8_TRY(need(ctx, s->n_free, "state.n_free", 4));
    if (s->B < 1 || s->B > kPageMaxRows)
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "B=%d out of range 1..%d", (int)s->B, kPageMaxRows);
    if (s->n_pages < 1 || s->n_pages > kPageMaxPages)
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "n_pages=%d out of range 1..2^20", (int)s->n_pages);
    if (page_shift(s->page) < 0)
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "page=%d is not 16, 32, 64 or 128 tokens", (int)s->page);
    if (s->max_pages < 1 || (long long)s->max_pages * s->page > (1ll << 30))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "max_pages=%d out of range (at most 2^30 tokens per row)", (int)s->max_pages);
    out->tables = s->tables;
    out->seq_lens = s->seq_lens;
    out->refs = s->refs;
    out->free_list = s->free_list;
    out->n_free = s->n_free;
    out->B = s->B;
    out->max_pages = s->max_pages;
    out->n_pages = s->n_pages;
    out->page_shift = page_shift(s->page);
    out->status = ctx->status_word;
    return LOOKAT_OK;
}

lookat_status pools_of(Ctx *ctx, const lookat_page_pool *pools, int32_t n_pools, PagePools *out)
{
    if (n_pools < 0 || n_pools > LOOKAT_MAX_POOLS || (n_pools && !pools))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "n_pools=%d out of range 0..%d, or pools is NULL", (int)n_pools, (int)LOOKAT_MAX_POOLS);
    out->n = n_pools;
    out->items = 0;
    for (int i = 0; i < n_pools; ++i) {
        Q8_TRY(need(ctx, pools[i].base, "pool base"));
        if (pools[i].page_bytes < 4 || pools[i].page_bytes % 4 || pools[i].page_bytes > (1ll << 30))
            return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "pool %d: page_bytes=%lld is not a multiple of 4 in 4..2^30", i, (long long)pools[i].page_bytes);
        out->base[i] = static_cast<unsigned char *>(pools[i].base);
        out->page_bytes[i] = pools[i].page_bytes;
        out->first[i] = out->items;
        out->items += (int)((pools[i].page_bytes + kPageCopyChunk - 1) / kPageCopyChunk);
    }
    return LOOKAT_OK;
}

}  // namespace
}  // namespace lookat

using namespace lookat;

extern "C" {

lookat_status lookat_q8_append(lookat_ctx *handle, const lookat_q8_cache *cache, const void *k_new, const void *v_new, int32_t B,
                               int32_t n, const int32_t *tables, int32_t max_pages, const int32_t *seq_lens, const int32_t *n_new)
{
    if (!handle) return LOOKAT_ERR_INVALID_ARG;
    Ctx *ctx = reinterpret_cast<Ctx *>(handle);
    Q8AppendArgs a;
    memset(&a, 0, sizeof(a));
    Q8_TRY(view_of(ctx, cache, B, tables, max_pages, seq_lens, &a.c));
    if (n < 1 || n > (1 << 20)) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "n=%d out of range 1..2^20", (int)n);
    Q8_TRY(need(ctx, k_new, "k_new"));
    Q8_TRY(need(ctx, v_new, "v_new"));
    if (n_new) Q8_TRY(need(ctx, n_new, "n_new", 4));
    Q8DeviceGuard guard(ctx->device);
    if (!guard.ok) return set_error(ctx, LOOKAT_ERR_CUDA, "cannot select device %d", ctx->device);
    a.k_new = static_cast<const __half *>(k_new);
    a.v_new = static_cast<const __half *>(v_new);
    a.n_new = n_new;
    a.B = B;
    a.n = n;
    a.format = cache->format;
    return launch_q8_append(ctx, a);
}

lookat_status lookat_attend_q8(lookat_ctx *handle, const lookat_q8_cache *cache, const void *q, int32_t B, int32_t L_q,
                               const int32_t *tables, int32_t max_pages, const int32_t *seq_lens, void *out, int32_t out_fp16)
{
    if (!handle) return LOOKAT_ERR_INVALID_ARG;
    Ctx *ctx = reinterpret_cast<Ctx *>(handle);
    Q8AttendArgs a;
    memset(&a, 0, sizeof(a));
    Q8_TRY(view_of(ctx, cache, B, tables, max_pages, seq_lens, &a.c));
    if (ctx->timeout_flag && *(volatile int *)ctx->timeout_flag) {
        *(volatile int *)ctx->timeout_flag = 0;
        return set_error(ctx, LOOKAT_ERR_TIMEOUT, "an earlier attention kernel gave up a bounded barrier wait; its output is not valid");
    }
    if (L_q < 1 || L_q > (1 << 20)) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "L_q=%d out of range 1..2^20", (int)L_q);
    if (out_fp16 != 0 && out_fp16 != 1) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "out_fp16=%d is not 0 or 1", (int)out_fp16);
    Q8_TRY(need(ctx, q, "q"));
    Q8_TRY(need(ctx, out, "out"));
    Q8DeviceGuard guard(ctx->device);
    if (!guard.ok) return set_error(ctx, LOOKAT_ERR_CUDA, "cannot select device %d", ctx->device);
    a.q = static_cast<const __half *>(q);
    a.out = out;
    a.out_fp16 = out_fp16;
    a.B = B;
    a.H_q = ctx->cfg.n_q_heads;
    a.g = ctx->cfg.n_q_heads / ctx->cfg.n_kv_heads;
    a.L_q = L_q;
    a.format = cache->format;
    a.scale_log2 = ctx->scale * 1.4426950408889634f;
    return launch_attend_q8(ctx, a);
}

lookat_status lookat_pages_extend(lookat_ctx *handle, const lookat_page_state *state, int32_t *n_new, const lookat_page_pool *pools,
                                  int32_t n_pools)
{
    if (!handle) return LOOKAT_ERR_INVALID_ARG;
    Ctx *ctx = reinterpret_cast<Ctx *>(handle);
    PageState s;
    PagePools p;
    Q8_TRY(state_of(ctx, state, &s));
    Q8_TRY(need(ctx, n_new, "n_new", 4));
    Q8_TRY(pools_of(ctx, pools, n_pools, &p));
    Q8DeviceGuard guard(ctx->device);
    if (!guard.ok) return set_error(ctx, LOOKAT_ERR_CUDA, "cannot select device %d", ctx->device);
    return launch_pages_extend(ctx, s, n_new, p);
}

lookat_status lookat_pages_fork(lookat_ctx *handle, const lookat_page_state *state, const int32_t *parents)
{
    if (!handle) return LOOKAT_ERR_INVALID_ARG;
    Ctx *ctx = reinterpret_cast<Ctx *>(handle);
    PageState s;
    Q8_TRY(state_of(ctx, state, &s));
    Q8_TRY(need(ctx, parents, "parents", 4));
    Q8DeviceGuard guard(ctx->device);
    if (!guard.ok) return set_error(ctx, LOOKAT_ERR_CUDA, "cannot select device %d", ctx->device);
    return launch_pages_fork(ctx, s, parents);
}

lookat_status lookat_pages_compact(lookat_ctx *handle, const lookat_page_state *state, const lookat_page_pool *pools, int32_t n_pools,
                                   int32_t *remap)
{
    if (!handle) return LOOKAT_ERR_INVALID_ARG;
    Ctx *ctx = reinterpret_cast<Ctx *>(handle);
    PageState s;
    PagePools p;
    Q8_TRY(state_of(ctx, state, &s));
    Q8_TRY(pools_of(ctx, pools, n_pools, &p));
    if (remap) Q8_TRY(need(ctx, remap, "remap", 4));
    Q8DeviceGuard guard(ctx->device);
    if (!guard.ok) return set_error(ctx, LOOKAT_ERR_CUDA, "cannot select device %d", ctx->device);
    return launch_pages_compact(ctx, s, p, remap);
}

}  // extern "C"
