// Internal declarations of the page upkeep (pages.cu).
#pragma once

#include "q8.cuh"

namespace lookat {

constexpr int kPageMaxRows = 4096, kPageMaxPages = 1 << 20;
constexpr int kPageCopyChunk = 4096;            // bytes of a page that one warp copies

struct PageState {
    int32_t *tables, *seq_lens, *refs, *free_list, *n_free;
    int B, max_pages, n_pages, page_shift;
    int *status;
};

struct PagePools {
    unsigned char *base[LOOKAT_MAX_POOLS];
    long long page_bytes[LOOKAT_MAX_POOLS];
    int first[LOOKAT_MAX_POOLS];                // chunks of the pools before this one
    int n, items;                               // items: chunks of one page in all pools
};

lookat_status launch_pages_extend(Ctx *ctx, const PageState &s, int32_t *n_new, const PagePools &pools);
lookat_status launch_pages_fork(Ctx *ctx, const PageState &s, const int32_t *parents);
lookat_status launch_pages_compact(Ctx *ctx, const PageState &s, const PagePools &pools, int32_t *remap);

}  // namespace lookat
