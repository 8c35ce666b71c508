// Page upkeep of the 8-bit paged cache (include/lookat_q8.h): lookat_pages_extend, lookat_pages_fork,
// lookat_pages_compact.
//
// Each call is a plan over the page lists, whose results have to be the same whatever the scheduling (the order of the
// free list is part of the state), and a move of page contents.  The plans of extend and compact are one CTA's block scans
// over rows or pages: the lists are a few KB to a few MB, and one launch of one CTA costs less than the launches that a
// grid-wide scan takes.  fork counts references by integer atomics over all table entries (their order does not show in
// the sums).  The move is a grid of warps, each taking 4 KB of one (page, pool) pair at a time with eight 16-byte loads in
// flight per lane: bound by HBM, 2 bytes of traffic per byte moved.
#include "pages.cuh"

namespace lookat {

namespace {

constexpr int kPgThreads = 1024;

// exclusive prefix sum over the CTA's threads; *total gets the sum (every thread)
__device__ __forceinline__ long long pg_scan(long long x, long long *warp_sums, long long *total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        long long s = warp_sums[lane];                          // 32 warps
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        warp_sums[lane] = s;
    }
    __syncthreads();
    const long long before = warp ? warp_sums[warp - 1] : 0;
    *total = warp_sums[31];
    __syncthreads();                                            // warp_sums may be written again
    return before + incl - x;
}

__device__ __forceinline__ bool pg_valid(int page, const PageState &s) { return page >= 0 && page < s.n_pages; }
__device__ __forceinline__ int pg_blocks(long long len, int shift) { return (int)((len + (1ll << shift) - 1) >> shift); }

// ---- extend: who needs which pages ----
// Rows in order.  Row b's place on the stack is the sum of what the rows before it take; whether it takes a copy of its
// begun last page depends on how many rows before it (of this call) left that page: refs - rank > 1.
// taken: per row what pages_extend_apply_kernel does, {first page off the stack, pages, table place of the first, the page that
// a copy replaces or -1}.
__global__ void __launch_bounds__(kPgThreads) pages_extend_plan_kernel(PageState s, int32_t *__restrict__ n_new, int2 *__restrict__ pairs,
                                                                       int *__restrict__ n_pairs, int4 *__restrict__ taken)
{
    extern __shared__ int rows_s[];                             // per row:
    int *const last_s = rows_s;                                 // the begun page it appends to, -1 if it has none
    int *const start_s = last_s + s.B;                          // pages taken by the rows before; low bit: takes a copy
    int *const len_s = start_s + s.B, *const n_s = len_s + s.B; // tokens held and coming
    __shared__ long long sums[32];
    __shared__ int pair_count;
    pdl_release();
    const int tid = threadIdx.x, page = 1 << s.page_shift;
    const long long cap = (long long)s.max_pages << s.page_shift;
    const int nf = *s.n_free;
    bool bad = nf < 0 || nf > s.n_pages;
    if (tid == 0) pair_count = 0;

    for (int b = tid; b < s.B; b += kPgThreads) {
        const int n = max(n_new[b], 0), L = s.seq_lens[b];
        int last = -1;
        if (L < 0 || L > cap || L + (long long)n > cap) bad = true;
        else if (n > 0 && (L & (page - 1))) {
            last = s.tables[(size_t)b * s.max_pages + (L >> s.page_shift)];
            if (!pg_valid(last, s)) {
                bad = true;
                last = -1;
            }
        }
        last_s[b] = last;
        len_s[b] = L;
        n_s[b] = n;
    }
    bad = __syncthreads_or(bad);
    long long base = 0;
    if (!bad) {
        for (int b0 = 0; b0 < s.B; b0 += kPgThreads) {
            const int b = b0 + tid;
            int take = 0, copy = 0;
            if (b < s.B) {
                const int n = n_s[b], L = len_s[b], last = last_s[b];
                take = pg_blocks((long long)L + n, s.page_shift) - pg_blocks(L, s.page_shift);
                if (last >= 0) {
                    int holders = s.refs[last];
                    for (int e = 0; e < b && holders > 1; ++e) holders -= last_s[e] == last;
                    copy = holders > 1;
                }
            }
            long long total;
            const long long at = base + pg_scan(take + copy, sums, &total);
            base += total;
            if (b < s.B) start_s[b] = (int)min(at, (long long)nf) * 2 + copy;
        }
        bad = base > nf;
    }
    __syncthreads();
    if (bad) {                                                  // (the same for every thread)
        for (int b = tid; b < s.B; b += kPgThreads) {
            n_new[b] = 0;
            taken[b] = make_int4(0, 0, 0, -1);
        }
        if (tid == 0) {
            *n_pairs = 0;
            q8_report(s.status, kStatusNoPages);
        }
        return;
    }
    for (int b = tid; b < s.B; b += kPgThreads) {
        const int n = n_s[b], L = len_s[b];
        const int copy = start_s[b] & 1, start = start_s[b] >> 1, have = pg_blocks(L, s.page_shift);
        taken[b] = make_int4(nf - 1 - start, pg_blocks((long long)L + n, s.page_shift) - have + copy, have - copy, copy ? last_s[b] : -1);
        if (copy) pairs[atomicAdd(&pair_count, 1)] = make_int2(last_s[b], s.free_list[nf - 1 - start]);
        if (n > 0) s.seq_lens[b] = L + n;
    }
    __syncthreads();
    if (tid == 0) {
        *n_pairs = pair_count;
        *s.n_free = nf - (int)base;
    }
}

// ---- the move: page pairs[i].x to page pairs[i].y in every pool ----
// A warp takes 4 KB of one page of one pool at a time.
__device__ __forceinline__ void pg_move(const PagePools &pools, const int2 *pairs, int n_pairs, int n_pages)
{
    const int lane = threadIdx.x & 31;
    const long long n_items = (long long)n_pairs * pools.items;
    const long long step = (long long)gridDim.x * (blockDim.x >> 5);
    for (long long it = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); it < n_items; it += step) {
        const int2 pr = pairs[it / pools.items];
        const int r = (int)(it % pools.items);
        if (pr.x < 0 || pr.x >= n_pages || pr.y < 0 || pr.y >= n_pages) continue;
        int lo = 0, hi = pools.n - 1;                           // the pool whose chunks hold r
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (pools.first[mid] <= r) lo = mid;
            else hi = mid - 1;
        }
        const long long bytes = pools.page_bytes[lo], off = (long long)(r - pools.first[lo]) * kPageCopyChunk;
        const unsigned char *src = pools.base[lo] + pr.x * bytes + off;
        unsigned char *dst = pools.base[lo] + pr.y * bytes + off;
        const int here = (int)min((long long)kPageCopyChunk, bytes - off);
        if ((bytes & 15) == 0) {
            uint4 u[kPageCopyChunk / 512];
#pragma unroll
            for (int i = 0; i < kPageCopyChunk / 512; ++i)
                if ((i * 32 + lane) * 16 < here) u[i] = __ldcs(reinterpret_cast<const uint4 *>(src) + i * 32 + lane);
#pragma unroll
            for (int i = 0; i < kPageCopyChunk / 512; ++i)
                if ((i * 32 + lane) * 16 < here) __stcs(reinterpret_cast<uint4 *>(dst) + i * 32 + lane, u[i]);
        } else {                                                // pages of an odd number of words: 4 bytes at a time
            for (int i = lane; i * 4 < here; i += 32) reinterpret_cast<uint32_t *>(dst)[i] = reinterpret_cast<const uint32_t *>(src)[i];
        }
    }
}

// the plan of an extend: tables and refs, 8 threads per row (one CTA's stores for 11,000 pages took 6 us), and the copies
__global__ void __launch_bounds__(256) pages_extend_apply_kernel(const __grid_constant__ PagePools pools, PageState s, const int2 *__restrict__ pairs,
                                                                 const int *__restrict__ n_pairs, const int4 *__restrict__ taken)
{
    pdl_wait();
    for (int b = blockIdx.x * 32 + (threadIdx.x >> 3); b < s.B; b += gridDim.x * 32) {
        const int4 t = taken[b];
        int32_t *row = s.tables + (size_t)b * s.max_pages + t.z;
#pragma unroll 4
        for (int k = threadIdx.x & 7; k < t.y; k += 8) {
            const int p = s.free_list[t.x - k];
            if (pg_valid(p, s)) s.refs[p] = 1;
            else q8_report(s.status, kStatusBadPage);           // (the row's tokens there are left out by whoever reads the table)
            row[k] = p;
        }
        if ((threadIdx.x & 7) == 0 && t.w >= 0) atomicSub(s.refs + t.w, 1);
    }
    pg_move(pools, pairs, *n_pairs, s.n_pages);
}

// ---- fork: references and the new rows ----
// One CTA per row.  marks: one bit per page that lost a reference here.
__global__ void __launch_bounds__(256) pages_fork_count_kernel(PageState s, const int32_t *__restrict__ parents, int32_t *__restrict__ rows,
                                                               int32_t *__restrict__ lens, unsigned *__restrict__ marks)
{
    pdl_release();
    const int b = blockIdx.x, p = parents[b];
    const bool alive = p >= 0 && p < s.B;
    const int cap = s.max_pages << s.page_shift;
    const int len_b = s.seq_lens[b], len_p = alive ? s.seq_lens[p] : 0;
    const int old_len = min(max(len_b, 0), cap), new_len = min(max(len_p, 0), cap);
    if (threadIdx.x == 0) {
        lens[b] = new_len;
        if (old_len != len_b || new_len != len_p) q8_report(s.status, kStatusBadPage);
    }
    if (p == b) return;                                         // the row stays as it is
    const int n_old = pg_blocks(old_len, s.page_shift), n_now = pg_blocks(new_len, s.page_shift);
    const int32_t *mine = s.tables + (size_t)b * s.max_pages, *theirs = s.tables + (size_t)(alive ? p : 0) * s.max_pages;
    for (int i = threadIdx.x; i < max(n_old, n_now); i += blockDim.x) {
        const int was = i < n_old ? mine[i] : -1, now = i < n_now ? theirs[i] : -1;
        if (i < n_now) rows[(size_t)b * s.max_pages + i] = now;
        if ((i < n_old && !pg_valid(was, s)) || (i < n_now && !pg_valid(now, s))) q8_report(s.status, kStatusBadPage);
        if (was == now) continue;                               // a page that both share: one reference goes, one comes
        if (pg_valid(now, s)) atomicAdd(s.refs + now, 1);
        if (pg_valid(was, s)) {
            atomicSub(s.refs + was, 1);
            atomicOr(marks + (was >> 5), 1u << (was & 31));
        }
    }
}

// The first cluster: the pages that lost their last reference go onto the free list, ascending; each of its CTAs looks at
// an eighth of the marks and learns from the others how many pages come before its own.  (One CTA over 110,000 pages took
// 52 us, the cluster 13.)  The other CTAs: the rows' new tables.
constexpr int kPgCluster = 8;
__global__ void __cluster_dims__(kPgCluster, 1, 1) __launch_bounds__(kPgThreads)
pages_fork_write_kernel(PageState s, const int32_t *__restrict__ parents, const int32_t *__restrict__ rows, const int32_t *__restrict__ lens,
                        unsigned *__restrict__ marks)
{
    const int tid = threadIdx.x, rank = blockIdx.x % kPgCluster;
    pdl_wait();
    if (blockIdx.x >= kPgCluster) {
        for (int b = blockIdx.x - kPgCluster; b < s.B; b += gridDim.x - kPgCluster) {
            if (parents[b] == b) continue;
            const int len = lens[b], n = pg_blocks(len, s.page_shift);
            for (int i = tid; i < n; i += kPgThreads) s.tables[(size_t)b * s.max_pages + i] = rows[(size_t)b * s.max_pages + i];
            if (tid == 0) s.seq_lens[b] = len;
        }
        return;                                                 // (clusters of these CTAs never synchronise)
    }
    __shared__ unsigned dead_s[kPageMaxPages / 32 / kPgCluster];
    __shared__ long long sums[32];
    __shared__ int count_s;
    const int words = (s.n_pages + 31) / 32, per = (words + kPgCluster - 1) / kPgCluster, w0 = min(rank * per, words), mine = min(per, words - w0);
    const int lane = tid & 31, warp = tid >> 5, nf = *s.n_free;
    // a word per warp: lane i looks at page i of it
    constexpr int kAtOnce = 16;
    for (int k0 = warp; k0 < mine; k0 += 32 * kAtOnce) {
        unsigned bits[kAtOnce];
        bool dead[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) bits[j] = k0 + 32 * j < mine ? marks[w0 + k0 + 32 * j] : 0u;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) dead[j] = (bits[j] >> lane & 1) && s.refs[(w0 + k0 + 32 * j) * 32 + lane] == 0;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const unsigned m = __ballot_sync(0xffffffffu, dead[j]);
            if (k0 + 32 * j < mine && lane == 0) {
                dead_s[k0 + 32 * j] = m;
                if (bits[j]) marks[w0 + k0 + 32 * j] = 0u;      // all zero again for the next call
            }
        }
    }
    __syncthreads();
    int at = 0;                                                 // dead pages of this CTA below the thread's words
    {
        const int each = (mine + kPgThreads - 1) / kPgThreads, k0 = min(tid * each, mine), k1 = min(k0 + each, mine);
        int n = 0;
        for (int k = k0; k < k1; ++k) n += __popc(dead_s[k]);
        long long total;
        at = (int)pg_scan(n, sums, &total);
        if (tid == 0) count_s = (int)total;
        asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
        int before = 0, all = 0;
#pragma unroll
        for (int r = 0; r < kPgCluster; ++r) {
            uint32_t addr, c;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"((uint32_t)__cvta_generic_to_shared(&count_s)), "r"(r));
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(addr) : "memory");
            if (r < rank) before += (int)c;
            all += (int)c;
        }
        at += nf + before;
        for (int k = k0; k < k1; ++k)
            for (unsigned d = dead_s[k]; d; d &= d - 1, ++at)
                if (at >= 0 && at < s.n_pages) s.free_list[at] = (w0 + k) * 32 + __ffs(d) - 1;
        // everyone has read the counts (and n_free) before a CTA ends or writes
        asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
        if (rank == 0 && tid == 0 && all) *s.n_free = nf + all;
    }
}

// ---- compact: where every page goes ----
// live bits of all pages and, per two words of them, the number of live pages below, in shared memory
__global__ void __launch_bounds__(kPgThreads) pages_compact_plan_kernel(PageState s, int2 *__restrict__ pairs, int *__restrict__ n_pairs,
                                                                        int32_t *__restrict__ map, int32_t *__restrict__ remap)
{
    extern __shared__ unsigned bits[];                          // [2 * duos], then int below[duos]
    pdl_release();
    __shared__ long long sums[32];
    const int tid = threadIdx.x, lane = tid & 31, duos = (s.n_pages + 63) / 64;
    int *below = reinterpret_cast<int *>(bits + 2 * duos);
    for (int p0 = 0; p0 < duos * 64; p0 += kPgThreads) {
        const int p = p0 + tid;
        const unsigned w = __ballot_sync(0xffffffffu, p < s.n_pages && s.refs[p] > 0);
        if (lane == 0 && p < duos * 64) bits[p >> 5] = w;
    }
    __syncthreads();
    int live = 0;
    for (int d0 = 0; d0 < duos; d0 += kPgThreads) {
        const int d = d0 + tid;
        long long total;
        const long long at = pg_scan(d < duos ? __popc(bits[2 * d]) + __popc(bits[2 * d + 1]) : 0, sums, &total);
        if (d < duos) below[d] = live + (int)at;
        live += (int)total;
    }
    __syncthreads();
    auto live_below = [&](int p) {                              // p < n_pages
        const int w = p >> 5;
        return below[w >> 1] + ((w & 1) ? __popc(bits[w - 1]) : 0) + __popc(bits[w] & ((1u << (p & 31)) - 1u));
    };
    const int front = live < s.n_pages ? live_below(live) : live;       // live pages that stay
    const int moves = live - front;
    for (int p = tid; p < s.n_pages; p += kPgThreads) {
        const bool on = bits[p >> 5] >> (p & 31) & 1;
        const int r = live_below(p);
        if (p < live) {
            if (!on) pairs[p - r].y = p;
        } else if (on) {
            pairs[r - front].x = p;
        }
        map[p] = on ? p : -1;
    }
    __syncthreads();
    for (int i = tid; i < moves; i += kPgThreads) {
        const int2 pr = pairs[i];
        map[pr.x] = pr.y;
        s.refs[pr.y] = s.refs[pr.x];
        s.refs[pr.x] = 0;
    }
    __syncthreads();
    if (remap)
        for (int p = tid; p < s.n_pages; p += kPgThreads) remap[p] = map[p];
    for (int i = tid; i < s.n_pages - live; i += kPgThreads) s.free_list[i] = s.n_pages - 1 - i;
    if (tid == 0) {
        *n_pairs = moves;
        *s.n_free = s.n_pages - live;
    }
}

__global__ void __launch_bounds__(256) pages_compact_move_kernel(const __grid_constant__ PagePools pools, PageState s,
                                                                 const int2 *__restrict__ pairs, const int *__restrict__ n_pairs,
                                                                 const int32_t *__restrict__ map)
{
    const int cap = s.max_pages << s.page_shift;
    pdl_wait();
    for (int b = blockIdx.x; b < s.B; b += gridDim.x) {
        const int len_in = s.seq_lens[b], len = min(max(len_in, 0), cap), n = pg_blocks(len, s.page_shift);
        if (threadIdx.x == 0 && len != len_in) q8_report(s.status, kStatusBadPage);
        int32_t *row = s.tables + (size_t)b * s.max_pages;
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int p = row[i];
            const int to = pg_valid(p, s) ? map[p] : -1;
            if (to >= 0) row[i] = to;
            else q8_report(s.status, kStatusBadPage);           // an entry that names no live page stays as it is
        }
    }
    pg_move(pools, pairs, *n_pairs, s.n_pages);
}

// the lists a plan hands to its move: a count (16 bytes), pairs, a page map
lookat_status lists(Ctx *ctx, size_t n_pairs, size_t n_map, int **count, int2 **pairs, int32_t **map, const char *what)
{
    const size_t at_map = 16 + n_pairs * sizeof(int2);
    lookat_status st = workspace(ctx, ctx->page_lists, at_map + n_map * sizeof(int32_t), false, what);
    if (st != LOOKAT_OK) return st;
    char *p = static_cast<char *>(ctx->page_lists.ptr);
    *count = reinterpret_cast<int *>(p);
    *pairs = reinterpret_cast<int2 *>(p + 16);
    *map = reinterpret_cast<int32_t *>(p + at_map);
    return LOOKAT_OK;
}

unsigned move_grid(const Ctx *ctx, long long most_items)
{
    const long long want = (most_items + 7) / 8, most = (long long)ctx->sm_count * 8;
    return (unsigned)(want < 1 ? 1 : want < most ? want : most);
}

}  // namespace

lookat_status launch_pages_extend(Ctx *ctx, const PageState &s, int32_t *n_new, const PagePools &pools)
{
    int *count;
    int2 *pairs;
    int32_t *map;
    const int even = (s.B + 1) / 2 * 2;                         // (what follows the pairs is 16-byte aligned)
    lookat_status st = lists(ctx, even, (size_t)s.B * 4, &count, &pairs, &map, "pages_extend");
    if (st != LOOKAT_OK) return st;
    int4 *taken = reinterpret_cast<int4 *>(map);
    const int smem = s.B * 16;                                  // 64 KB at most
    if (smem > 40 * 1024 && cudaFuncSetAttribute(pages_extend_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
        return check_launch(ctx, "pages_extend: shared-memory opt-in");
    pages_extend_plan_kernel<<<1, kPgThreads, smem, ctx->stream>>>(s, n_new, pairs, count, taken);
    st = check_launch(ctx, "pages_extend_plan_kernel");
    if (st != LOOKAT_OK) return st;
    const unsigned movers = move_grid(ctx, (long long)s.B * pools.items), rows = (unsigned)(s.B + 31) / 32;
    launch_after(ctx, pages_extend_apply_kernel, movers > rows ? movers : rows, 256, 0, pools, s, pairs, count, taken);
    return check_launch(ctx, "pages_extend_apply_kernel");
}

lookat_status launch_pages_fork(Ctx *ctx, const PageState &s, const int32_t *parents)
{
    int *count;
    int2 *pairs;
    int32_t *rows;
    lookat_status st = lists(ctx, 0, (size_t)s.B * s.max_pages + s.B, &count, &pairs, &rows, "pages_fork");
    if (st == LOOKAT_OK) st = workspace(ctx, ctx->page_marks, ((size_t)s.n_pages + 31) / 32 * 4, true, "pages_fork");
    if (st != LOOKAT_OK) return st;
    int32_t *lens = rows + (size_t)s.B * s.max_pages;
    unsigned *marks = static_cast<unsigned *>(ctx->page_marks.ptr);
    pages_fork_count_kernel<<<s.B, 256, 0, ctx->stream>>>(s, parents, rows, lens, marks);
    st = check_launch(ctx, "pages_fork_count_kernel");
    if (st != LOOKAT_OK) return st;
    const int writers = ((s.B < 512 ? s.B : 512) + kPgCluster - 1) / kPgCluster * kPgCluster;
    launch_after(ctx, pages_fork_write_kernel, kPgCluster + writers, kPgThreads, 0, s, parents, rows, lens, marks);
    return check_launch(ctx, "pages_fork_write_kernel");
}

lookat_status launch_pages_compact(Ctx *ctx, const PageState &s, const PagePools &pools, int32_t *remap)
{
    int *count;
    int2 *pairs;
    int32_t *map;
    lookat_status st = lists(ctx, s.n_pages, s.n_pages, &count, &pairs, &map, "pages_compact");
    if (st != LOOKAT_OK) return st;
    const int smem = (s.n_pages + 63) / 64 * 12;                // two words and a count per 64 pages: 192 KB at 2^20 pages
    if (smem > 40 * 1024 &&
        cudaFuncSetAttribute(pages_compact_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
        return check_launch(ctx, "pages_compact: shared-memory opt-in");
    pages_compact_plan_kernel<<<1, kPgThreads, smem, ctx->stream>>>(s, pairs, count, map, remap);
    st = check_launch(ctx, "pages_compact_plan_kernel");
    if (st != LOOKAT_OK) return st;
    launch_after(ctx, pages_compact_move_kernel, move_grid(ctx, (long long)s.n_pages * pools.items), 256, 0, pools, s, pairs, count, map);
    return check_launch(ctx, "pages_compact_move_kernel");
}

}  // namespace lookat
