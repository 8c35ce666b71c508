// Checks of arguments that the entry points of the 8-bit paged cache and of what runs around it share.
#pragma once

#include "q8.cuh"

namespace lookat {

struct Q8DeviceGuard {
    int prev = -1;
    bool ok = false, moved = false;
    explicit Q8DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) return;
        moved = prev != dev;
        ok = !moved || cudaSetDevice(dev) == cudaSuccess;
    }
    ~Q8DeviceGuard()
    {
        if (ok && moved) cudaSetDevice(prev);
    }
};

#define Q8_TRY(expr)                            \
    do {                                        \
        lookat_status st__ = (expr);            \
        if (st__ != LOOKAT_OK) return st__;     \
    } while (0)

inline lookat_status need(Ctx *ctx, const void *p, const char *name, unsigned align = 16)
{
    if (!p) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) & (align - 1))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "%s is not %u-byte aligned", name, align);
    return LOOKAT_OK;
}

inline int page_shift(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : -1; }

inline lookat_status view_of(Ctx *ctx, const lookat_q8_cache *cache, int32_t B, const int32_t *tables, int32_t max_pages,
                      const int32_t *seq_lens, Q8View *v)
{
    const lookat_config &c = ctx->cfg;
    if (!cache) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "cache is NULL");
    Q8_TRY(need(ctx, cache->k, "cache.k"));
    Q8_TRY(need(ctx, cache->v, "cache.v"));
    Q8_TRY(need(ctx, cache->k_amax, "cache.k_amax"));
    Q8_TRY(need(ctx, cache->v_amax, "cache.v_amax"));
    if (cache->format != LOOKAT_Q8_INT8 && cache->format != LOOKAT_Q8_E4M3)
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "unknown 8-bit format %d", (int)cache->format);
    if (page_shift(cache->page) < 0)
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "page=%d is not 16, 32, 64 or 128 tokens", (int)cache->page);
    if (cache->n_pages < 1) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "n_pages=%d is less than 1", (int)cache->n_pages);
    if (B < 1 || B > 65535) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "B=%d out of range 1..65535", (int)B);
    if (max_pages < 1 || (long long)max_pages * cache->page > (1ll << 30))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "max_pages=%d out of range (at most 2^30 tokens per row)", (int)max_pages);
    Q8_TRY(need(ctx, tables, "tables", 4));
    Q8_TRY(need(ctx, seq_lens, "seq_lens", 4));
    if (c.d_k % 16 || c.d_v % 16 || c.d_k > 256 || c.d_v > 256)
        return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "the 8-bit cache wants d_k and d_v as multiples of 16 up to 256 (%d, %d)", c.d_k, c.d_v);
    if (c.n_q_heads > 65535) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "more than 65535 query heads");
    v->k = static_cast<uint8_t *>(cache->k);
    v->v = static_cast<uint8_t *>(cache->v);
    v->k_amax = cache->k_amax;
    v->v_amax = cache->v_amax;
    v->tables = tables;
    v->seq_lens = seq_lens;
    v->n_pages = cache->n_pages;
    v->max_pages = max_pages;
    v->page_shift = page_shift(cache->page);
    v->H_kv = c.n_kv_heads;
    v->d_k = c.d_k;
    v->d_v = c.d_v;
    v->status = ctx->status_word;
    return LOOKAT_OK;
}

}  // namespace lookat
