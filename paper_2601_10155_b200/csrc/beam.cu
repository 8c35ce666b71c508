// lookat_beam_select: one step of beam search.
//
// Bound by HBM: the logits are read once.  A row is cut into `splits` parts, a CTA each; in one pass a warp keeps
//   - sum exp(x - M) against a reference M that follows its largest logit at a distance of at most 1: fp32 exponentials, sixteen
//     of a lane added in fp32 before they go into fp64 sums.  A term at distance d is off by 2^-22 (ex2.approx), 5 * 2^-24 (the
//     additions) and d * 1.25 * 2^-24 (its exponent, and log2(e) as an fp32 number) of itself: a row with one likely token by
//     less than 2^-20, one of very many tokens 20 below the largest by less than 2^-18;
//   - its best 32 logits (a beam's candidates rank as its logits do), sorted over the lanes.  What reaches a bar is collected in
//     shared memory and sorted in 32 at a time (a bitonic sort and a merge).  The bar comes from the lanes' largest logits so far
//     and is renewed at the batches 1, 2, 4, ...: few logits reach it.
// Rows are read in the same order whatever their alignment (16-byte loads where all rows lie on such borders, else 4-byte ones):
// beams with equal logits and scores get equal ranks, and the lower one goes first.
// A CTA's candidates find their places by counting those before them.  The last CTA of a group to finish (a counter, no waiting)
// joins the parts, ranks in fp64, and moves the beams.
//   32 x 16 beams over 131072 tokens: 68 us (3.9 TB/s: 24 of the 32 warps that an SM has room for, on average; 205 instructions per
// warp and batch; a batch more on its way changes nothing), histories of 512 tokens 5 us more; 64 x 8 over 50257, an odd number, whose
// rows come by 4-byte copies, 39 us (2.6 TB/s); 8 x 4 13.6 us, most of it the chain of dependent steps of a part and of the join.
#include "serve.cuh"

namespace lookat {

namespace {

constexpr int kBsThreads = 256, kBsWarps = kBsThreads / 32, kBsVecs = 4, kBsMost = 32;
constexpr int kBsBatch = kBsThreads * kBsVecs * 4;            // logits that a CTA has in flight
constexpr int kBsRing = 2 * kBsBatch * 4;                      // bytes of the batches in shared memory
constexpr int kBsSplits = 64;                                  // most parts of a row
constexpr int kBsHold = 32;                                    // candidates that a warp collects before it sorts them in

struct BsPart {                     // of a row: its best logits, sum exp(x - M) and M
    float best[kBsMost];
    int at[kBsMost];
    double sum, m;
    int bad;                        // a NaN or +inf among them
};

// 32 candidates of a warp, one per lane
template <class Key>
struct BsBlock {
    Key key;
    int at;
    __device__ bool before(Key k, int i) const { return key > k || (key == k && at < i); }      // this one goes first
    __device__ void exchange(int mask, bool first)             // with the lane at that distance; first: this lane keeps what goes first
    {
        const Key k = __shfl_xor_sync(0xffffffffu, key, mask);
        const int i = __shfl_xor_sync(0xffffffffu, at, mask);
        if (before(k, i) != first) key = k, at = i;
    }
    // first to last over the lanes, or with `up` last to first
    __device__ void sort(int lane, bool up)
    {
#pragma unroll
        for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
            for (int j = k >> 1; j; j >>= 1) exchange(j, (((lane & k) == 0) == ((lane & j) == 0)) != up);
    }
    // the first 32 of this block (first to last) and of another's candidates, last to first: first to last
    __device__ void join(Key k, int i, int lane)
    {
        if (!before(k, i)) key = k, at = i;
#pragma unroll
        for (int j = 16; j; j >>= 1) exchange(j, (lane & j) == 0);
    }
};

__device__ __forceinline__ float bs_max_nan(float a, float b, float c)          // NaN if one of them is
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
constexpr float kBsLog2e = 1.4426950408889634f;
// exp(x - M), exp(y - M), added to sum, for M = -c / log2(e): the exponents two at a time, rounded once
__device__ __forceinline__ void bs_add_exp2(float2 &sum, float x, float y, float c)
{
    float u, v;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %4};\nmov.b64 d, {%5, %5};\nfma.rn.f32x2 a, a, b, d;\nmov.b64 {%0, %1}, a;\n}"
        : "=f"(u), "=f"(v) : "f"(x), "f"(y), "f"(kBsLog2e), "f"(c));
    u = ex2_approx(u), v = ex2_approx(v);
    asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %3};\nadd.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}" : "+f"(sum.x), "+f"(sum.y) : "f"(u), "f"(v));
}
// the lanes' numbers in falling order
__device__ __forceinline__ float bs_sorted(float v, int lane)
{
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j; j >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, v, j);
            v = ((lane & k) == 0) == ((lane & j) == 0) ? fmaxf(v, o) : fminf(v, o);
        }
    return v;
}

// the 32 largest of the lanes' numbers, in falling order, and of others in rising order: in falling order
__device__ __forceinline__ float bs_merged(float v, float others, int lane)
{
    v = fmaxf(v, others);
#pragma unroll
    for (int j = 16; j; j >>= 1) {
        const float o = __shfl_xor_sync(0xffffffffu, v, j);
        v = (lane & j) == 0 ? fmaxf(v, o) : fminf(v, o);
    }
    return v;
}
// Ranks as whole numbers that go in the same order (as which they are compared faster; -0 and 0 are one)
constexpr long long kBsNone = (long long)0x800fffffffffffffull;         // -inf
__device__ __forceinline__ double bs_rank(long long key) { return __longlong_as_double(key ^ ((key >> 63) & 0x7fffffffffffffffll)); }
__device__ __forceinline__ long long bs_key(double rank)
{
    const long long bits = __double_as_longlong(rank + 0.0);
    return bits ^ ((bits >> 63) & 0x7fffffffffffffffll);
}

// What a group's beams were before the call, and where its rows' candidates stand.
struct BsGroup {
    float score[kBsMost];
    int len[kBsMost], fin[kBsMost];
    double base[kBsMost], norm[kBsMost], m[kBsMost];           // rank = (base + (x - m)) / norm
    int parent[kBsMost], slot[kBsMost], token[kBsMost];
};
struct BsBest {                     // the warps' best of it, and the parts to look through
    long long key[kBsWarps][kBsMost];
    int at[kBsWarps][kBsMost];
    float firsts[kBsWarps][kBsMost];
    int count, list[kBsMost * kBsSplits];
};
static_assert(kBsThreads * 8 + sizeof(BsBest) <= kBsRing, "what lies over the batches once they are read");

// Columns of the histories, of up to MOST beams each: all are read before the first is written.
template <int MOST, class T>
__device__ __forceinline__ void beam_move(T *rows, int columns, int beams, const int *parent)
{
    for (int c = threadIdx.x; c < columns; c += kBsThreads) {
        T y[MOST];
#pragma unroll
        for (int w = 0; w < MOST; ++w)
            if (w < beams) y[w] = rows[(size_t)parent[w] * columns + c];
#pragma unroll
        for (int w = 0; w < MOST; ++w)
            if (w < beams) rows[(size_t)w * columns + c] = y[w];
    }
}

// The group's parts joined and ranked, its beams moved.
__device__ __noinline__ void beam_finish(const BeamArgs &a, int splits, const BsPart *__restrict__ parts, int group, BsGroup &g, BsBest &warps)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, W = a.beams;
    const int g0 = group * W;
    const BsPart *const p0 = parts + (size_t)g0 * splits;
    // A group of many parts looks through those only whose first is not behind the W-th of the threads' best firsts: about W of them,
    // which takes as long to find as a warp takes for three more parts (8 x 4 beams over 50257 tokens, 52 parts a group, 12.9 us, 16.6
    // through all of them; one group of 32 beams over 131072, 512 parts, 29 and 60; with 13 parts for one beam 13.8 and 11).
    const int items = W * splits;
    const bool chosen = items > W + 24;
    const float head = chosen && tid < items ? __ldcg(&p0[tid].best[0]) : -INFINITY;
    // ---- the rows' sums, as many lanes per row as there are ----
    {
        const int lanes = W <= 8 ? 32 : W <= 16 ? 16 : 8, w = tid / lanes, sub = tid % lanes;
        const bool row = w < W;
        const float sc = row ? g.score[w] : -INFINITY;
        const bool counts = sc > -INFINITY && sc < INFINITY, goes_on = counts && !g.fin[w];
        const BsPart *const p = p0 + (size_t)(row ? w : 0) * splits;
        double top = -INFINITY, total = 0.0;                   // a lane's parts: sum exp(x - top)
        bool bad = false;
        if (goes_on && sub < splits) {
            top = __ldcg(&p[sub].m);
            total = __ldcg(&p[sub].sum);
            bad = __ldcg(&p[sub].bad) != 0;
        }
#pragma unroll 1
        for (int i = sub + lanes; goes_on && i < splits; i += lanes) {
            const double m = __ldcg(&p[i].m), sum = __ldcg(&p[i].sum);
            bad |= __ldcg(&p[i].bad) != 0;
            if (!(m > -INFINITY)) continue;
            const double k = exp(-fabs(m - top));              // (0 where there was none)
            total = m > top ? fma(total, k, sum) : fma(sum, k, total);
            top = fmax(top, m);
        }
        double most = top;
        for (int o = lanes / 2; o; o >>= 1) most = fmax(most, __shfl_xor_sync(0xffffffffu, most, o));
        total = top > -INFINITY ? total * exp(top - most) : 0.0;
        for (int o = lanes / 2; o; o >>= 1) {
            total += __shfl_xor_sync(0xffffffffu, total, o);
            bad |= __shfl_xor_sync(0xffffffffu, (int)bad, o) != 0;
        }
        if (row && sub == 0) {
            const int grown = max(g.len[w] + (g.fin[w] ? 0 : 1), 1);
            g.base[w] = !counts || (goes_on && (bad || most == -INFINITY)) ? -INFINITY : goes_on ? (double)sc - log(total) : (double)sc;
            g.norm[w] = a.penalty == 0.0 ? 1.0 : pow((double)grown, a.penalty);
            g.m[w] = goes_on ? most : 0.0;
        }
    }
    __syncthreads();
    // ---- the best of all parts' candidates, which stand first to last there: read last to first ----
    auto rank_of = [&](int item, float x, bool first) {        // of a part's candidate
        const int w = item / splits;
        const double base = g.base[w], norm = g.norm[w];
        if (!(base > -INFINITY) || (g.fin[w] ? item != w * splits || !first : !(x > -INFINITY))) return (double)-INFINITY;    // (finished: itself, once)
        const double score = g.fin[w] ? base : base + ((double)x - g.m[w]);
        return norm == 1.0 ? score : score / norm;
    };
    int count = items;
    if (chosen) {
        // (fp32, rounded up: in the same order)
        const float mine = tid < items ? __double2float_ru(rank_of(tid, head, true)) : -INFINITY;
        float top = mine;
        for (int item = tid + kBsThreads; item < items; item += kBsThreads) top = fmaxf(top, __double2float_ru(rank_of(item, __ldcg(&p0[item].best[0]), true)));
        if (tid == 0) warps.count = 0;
        top = bs_sorted(top, lane);
        warps.firsts[warp][lane] = top;
#pragma unroll 1
        for (int half = kBsWarps / 2; half; half >>= 1) {
            __syncthreads();
            if (warp < half) warps.firsts[warp][lane] = top = bs_merged(top, warps.firsts[warp + half][31 - lane], lane);
        }
        __syncthreads();
        const float bar = warps.firsts[0][W - 1];
        if (mine > -INFINITY && mine >= bar) warps.list[atomicAdd(&warps.count, 1)] = tid;
        for (int item = tid + kBsThreads; item < items; item += kBsThreads) {
            const float first = __double2float_ru(rank_of(item, __ldcg(&p0[item].best[0]), true));
            if (first > -INFINITY && first >= bar) warps.list[atomicAdd(&warps.count, 1)] = item;
        }
        __syncthreads();
        count = warps.count;
    }
    BsBlock<long long> best = {kBsNone, 0x7fffffff};
    constexpr int kAhead = 4;
#pragma unroll 1
    for (int i0 = warp; i0 < count; i0 += kBsWarps * kAhead) {
        float x[kAhead];
        int at[kAhead], item[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = min(i0 + i * kBsWarps, count - 1);
            item[i] = chosen ? warps.list[k] : k;
            x[i] = __ldcg(&p0[item[i]].best[31 - lane]);
            at[i] = __ldcg(&p0[item[i]].at[31 - lane]);
        }
#pragma unroll 1
        for (int i = 0; i < kAhead && i0 + i * kBsWarps < count; ++i) {
            const float xi = i == 0 ? x[0] : i == 1 ? x[1] : i == 2 ? x[2] : x[3];
            const int ai = i == 0 ? at[0] : i == 1 ? at[1] : i == 2 ? at[2] : at[3], it = i == 0 ? item[0] : i == 1 ? item[1] : i == 2 ? item[2] : item[3];
            const int w = it / splits;
            const long long key = bs_key(rank_of(it, xi, lane == 31)), bar = __shfl_sync(0xffffffffu, best.key, W - 1);
            const bool on = key > kBsNone;
            if (__any_sync(0xffffffffu, on && key >= bar)) best.join(key, on ? w * a.vocab + (g.fin[w] ? max(a.eos, 0) : ai) : 0x7fffffff, lane);
        }
    }
    warps.key[warp][lane] = best.key;
    warps.at[warp][lane] = best.at;
#pragma unroll 1
    for (int half = kBsWarps / 2; half; half >>= 1) {
        __syncthreads();
        if (warp < half) {
            best.join(warps.key[warp + half][31 - lane], warps.at[warp + half][31 - lane], lane);
            warps.key[warp][lane] = best.key;
            warps.at[warp][lane] = best.at;
        }
    }
    if (warp == 0 && lane < W) {
        const bool there = best.key > kBsNone;
        const int parent = there ? best.at / a.vocab : lane, token = there ? best.at % a.vocab : max(a.eos, 0);
        const bool grows = there && !g.fin[parent];
        const int was = g.len[parent];
        a.scores[g0 + lane] = !there ? -INFINITY : g.fin[parent] ? g.score[parent] : (float)(bs_rank(best.key) * g.norm[parent]);
        a.lengths[g0 + lane] = was + (grows ? 1 : 0);
        a.finished[g0 + lane] = g.fin[parent] || (grows && token == a.eos);
        a.next_ids[g0 + lane] = token;
        a.parents[g0 + lane] = g0 + parent;
        g.parent[lane] = parent;
        g.slot[lane] = grows && was >= 0 && was < a.max_len ? was : -1;
        g.token[lane] = token;
    }
    if (!a.max_len) return;
    __syncthreads();
    // ---- the histories ----
    int32_t *const tokens = a.tokens + (size_t)g0 * a.max_len;
    // (as wide as 32 registers allow)
    const bool wide = a.max_len % 4 == 0 && (reinterpret_cast<uintptr_t>(a.tokens) & 15) == 0;
    if (W <= 8 && wide) beam_move<8>(reinterpret_cast<int4 *>(tokens), a.max_len / 4, W, g.parent);
    else if (W <= 16 && wide) beam_move<16>(reinterpret_cast<int2 *>(tokens), a.max_len / 2, W, g.parent);
    else beam_move<kBsMost>(tokens, a.max_len, W, g.parent);
    __syncthreads();
    if (tid < W && g.slot[tid] >= 0) tokens[(size_t)tid * a.max_len + g.slot[tid]] = g.token[tid];
}

// the candidates that a warp holds among its best (out of line: it is called from several places and would fill the
// instruction cache)
__device__ __noinline__ BsBlock<float> beam_sort_in(BsBlock<float> best, const float *hold, const int *hold_at, int held)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll 1
    for (int i = 0; i < held; i += 32) {
        const bool on = i + lane < held;
        BsBlock<float> more = {on ? hold[i + lane] : -INFINITY, on ? hold_at[i + lane] : 0x7fffffff};
        more.sort(lane, true);
        best.join(more.key, more.at, lane);
    }
    __syncwarp();
    return best;
}

template <bool WIDE>
__global__ void __launch_bounds__(kBsThreads, 4)
beam_select_kernel(const __grid_constant__ BeamArgs a, int splits, int part, BsPart *__restrict__ parts, unsigned *__restrict__ tickets)
{
    extern __shared__ float4 beam_smem[];
    __shared__ float s_hold[kBsWarps][kBsHold + 32];           // a warp's candidates
    __shared__ int s_hold_at[kBsWarps][kBsHold + 32];
    __shared__ int s_count[kBsWarps];
    __shared__ BsGroup s_group;
    __shared__ double s_sum[kBsWarps], s_m[kBsWarps];
    __shared__ int s_bad[kBsWarps], s_last;
    __shared__ float s_bars[2][4 * kBsWarps];                  // the largest of the lanes' largest logits, four of each warp
    // once the batches are read: all warps' last candidates (logit, element), the group's best
    float2 *const s_all = reinterpret_cast<float2 *>(beam_smem);
    BsBest &s_best = *reinterpret_cast<BsBest *>(s_all + kBsThreads);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, W = a.beams;
    const int row = blockIdx.x / splits, split = blockIdx.x % splits, group = row / W;
    const float score = a.scores[row];
    const bool live = a.finished[row] == 0 && score > -INFINITY && score < INFINITY;

    if (tid < W) {                                             // (for the last CTA)
        s_group.score[tid] = a.scores[group * W + tid];
        s_group.len[tid] = a.lengths[group * W + tid];
        s_group.fin[tid] = a.finished[group * W + tid] != 0;
    }
    if (live) {                                                // (the same for the whole CTA)
        const float *x0 = a.logits + (long long)row * a.stride;
        const int e1 = min((split + 1) * part, a.vocab);
        BsBlock<float> best = {-INFINITY, 0x7fffffff};
        float bar = -INFINITY, m = -INFINITY, limit = -INFINITY;     // limit: what to look at closer
        // The reference M: -c / log2(e), c a whole number (a new one moves the sum by a power of 2, exactly); or where that would
        // leave too few bits, the logit m itself (`far`), from which those that count differ by exact numbers.
        float c = 0.f;
        bool far = false;
        auto reference = [&]() { return far ? (double)m : -(double)c * (1.0 / (double)kBsLog2e); };
        int held = 0;
        double sum = 0.0;
        float lane_top = -INFINITY;
        int batch = 0;
        bool bad = false, sorted = false;
        auto sort_in = [&]() {
            sorted = true;
            best = beam_sort_in(best, s_hold[warp], s_hold_at[warp], held);
            held = 0;
            bar = fmaxf(bar, __shfl_sync(0xffffffffu, best.key, W - 1));
            limit = fminf(bar, m + 1.f);
        };
        // A batch's logits by way of the thread's own places in shared memory, one batch ahead.  Element of a batch: e0 + 4 tid +
        // 1024 i + j (wide), or e0 + tid + 256 (4 i + j); places hold 16 bytes: [buffer][i][thread].
        auto element = [&](int e0, int i, int j) { return WIDE ? e0 + 4 * (i * kBsThreads + tid) + j : e0 + (4 * i + j) * kBsThreads + tid; };
        float4 *const place = beam_smem + tid;
        auto fetch = [&](int e0, int buf) {
            const unsigned dst = (unsigned)__cvta_generic_to_shared(place + buf * kBsVecs * kBsThreads);
            const float *const src = x0 + element(e0, 0, 0);
            if (e0 + kBsBatch <= e1) {
#pragma unroll
                for (int i = 0; i < kBsVecs; ++i) {
                    if constexpr (WIDE) {
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + i * kBsThreads * 16), "l"(src + i * kBsThreads * 4) : "memory");
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + i * kBsThreads * 16 + 4 * j), "l"(src + (4 * i + j) * kBsThreads) : "memory");
                    }
                }
            } else {
#pragma unroll 1
                for (int k = 0; k < 4 * kBsVecs; ++k)
                    if (element(e0, k >> 2, k & 3) < e1)
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + (k >> 2) * kBsThreads * 16 + 4 * (k & 3)),
                                     "l"(x0 + element(e0, k >> 2, k & 3)) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        fetch(split * part, 0);
#pragma unroll 1
        for (int e0 = split * part; e0 < e1; e0 += kBsBatch) {
            if (e0 + kBsBatch < e1) {
                fetch(e0 + kBsBatch, (batch + 1) & 1);
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            } else {
                asm volatile("cp.async.wait_group 0;" ::: "memory");
            }
            float x[kBsVecs][4];
#pragma unroll
            for (int i = 0; i < kBsVecs; ++i) {
                const float4 y = place[((batch & 1) * kBsVecs + i) * kBsThreads];
                x[i][0] = y.x, x[i][1] = y.y, x[i][2] = y.z, x[i][3] = y.w;
            }
            if (e0 + kBsBatch > e1) {
#pragma unroll
                for (int i = 0; i < kBsVecs; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (element(e0, i, j) >= e1) x[i][j] = -INFINITY;
            }
            float tops[kBsVecs];
#pragma unroll
            for (int i = 0; i < kBsVecs; ++i) tops[i] = bs_max_nan(x[i][0], x[i][1], bs_max_nan(x[i][2], x[i][3], x[i][3]));
            const float top = bs_max_nan(tops[0], tops[1], bs_max_nan(tops[2], tops[3], tops[3]));
            const bool hit = __any_sync(0xffffffffu, !(top < limit));
            lane_top = fmaxf(lane_top, top);
            ++batch;
            float to = -INFINITY;                              // where the reference goes
            if (hit) {
                bad |= __any_sync(0xffffffffu, !(top < INFINITY));             // nothing of the row counts any more
                if (__any_sync(0xffffffffu, top > m + 1.f)) {
                    to = top;
#pragma unroll
                    for (int o = 16; o; o >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, o));
                }
            }
            if ((batch & (batch - 1)) == 0) {
                // the bar, renewed at batches 1, 2, 4, ...: the `beams`-th of 32 of the part's logits, the largest four lanes' of every
                // warp.  All warps come here (they have the same batches), and the next renewal writes to the other half: a warp's four
                // are seen as it wrote them, so that no logit counts twice.  The largest of all is the reference.
                float *const bars = s_bars[__popc(batch - 1) & 1];
                const float in_order = bs_sorted(lane_top, lane);
                if (lane < 4) bars[warp * 4 + lane] = in_order;
                __syncthreads();
                const float of_all = bs_sorted(bars[lane], lane);
                bar = fmaxf(bar, __shfl_sync(0xffffffffu, of_all, W - 1));
                to = __shfl_sync(0xffffffffu, of_all, 0);
            }
            if (to > m) {
                const double was = reference();
                const float c1 = -ceilf(to * kBsLog2e);
                if (!far && fabsf(to) <= 0x1p20f) {
                    const int k = min(max((int)(c1 - c), -1023), 0);           // (above 0 only before the first, with nothing summed)
                    sum *= __hiloint2double((1023 + k) << 20, 0);
                    c = c1, m = to;
                } else {
                    far = !(fabsf(to) <= 0x1p20f);
                    c = c1, m = to;
                    sum = sum > 0.0 ? sum * exp(was - reference()) : 0.0;
                }
            }
            limit = fminf(bar, m + 1.f);
            if (!far) {
                float2 add[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int i = 0; i < kBsVecs; ++i) {
                    bs_add_exp2(add[0], x[i][0], x[i][1], c);
                    bs_add_exp2(add[1], x[i][2], x[i][3], c);
                }
                sum += (double)((add[0].x + add[0].y) + (add[1].x + add[1].y));
            } else {
#pragma unroll 1
                for (int k = 0; k < 4 * kBsVecs; ++k)
                    if (element(e0, k >> 2, k & 3) < e1)
                        sum += (double)ex2_approx((reinterpret_cast<const float *>(place + ((~batch & 1) * kBsVecs + (k >> 2)) * kBsThreads)[k & 3] - m) * kBsLog2e);
            }
            if (!hit) continue;
#pragma unroll
            for (int i = 0; i < kBsVecs; ++i) {
                if (!__any_sync(0xffffffffu, tops[i] >= bar)) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool on = x[i][j] >= bar && x[i][j] > -INFINITY;
                    const unsigned who = __ballot_sync(0xffffffffu, on);
                    if (!who) continue;
                    const int at = held + __popc(who & ((1u << lane) - 1));
                    if (on) s_hold[warp][at] = x[i][j], s_hold_at[warp][at] = element(e0, i, j);
                    held += __popc(who);
                    if (held > kBsHold) sort_in();
                }
            }
        }
        // ---- the part's best: a warp brings what it holds, or its best if it has sorted, and each finds its place by counting ----
        if (sorted || held > 32) {
            sort_in();
            held = W;
        } else {
            __syncwarp();
            if (lane < held) best.key = s_hold[warp][lane], best.at = s_hold_at[warp][lane];
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) s_sum[warp] = sum, s_m[warp] = m > -INFINITY ? reference() : -INFINITY, s_bad[warp] = bad, s_count[warp] = held;
        __syncthreads();
        int first = 0, n = 0;
#pragma unroll
        for (int w = 0; w < kBsWarps; ++w) {
            if (w == warp) first = n;
            n += s_count[w];
        }
        if (lane < held) s_all[first + lane] = make_float2(best.key, __int_as_float(best.at));
        __syncthreads();
        BsPart &p = parts[(size_t)row * splits + split];
        if (tid < n) {
            const float2 mine = s_all[tid];
            const int at = __float_as_int(mine.y);
            int place = 0;
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                const float2 o = s_all[i];
                place += o.x > mine.x || (o.x == mine.x && __float_as_int(o.y) < at);
            }
            // (a warp's list that is not full ends with places that hold nothing)
            if (place < kBsMost && mine.x > -INFINITY) p.best[place] = mine.x, p.at[place] = at;
        }
        const int real = __syncthreads_count(tid < n && s_all[min(tid, n - 1)].x > -INFINITY);
        if (tid >= real && tid < kBsMost) p.best[tid] = -INFINITY, p.at[tid] = 0x7fffffff;
        if (warp == 0) {
            double top = -INFINITY, mine = 0.0;
            bool any_bad = false;
            for (int w = 0; w < kBsWarps; ++w) top = fmax(top, s_m[w]), any_bad |= s_bad[w] != 0;
            if (lane < kBsWarps && s_m[lane] > -INFINITY) mine = s_sum[lane] * exp(s_m[lane] - top);
#pragma unroll
            for (int o = kBsWarps / 2; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
            if (lane == 0) p.sum = mine, p.m = top, p.bad = any_bad;
        }
        __threadfence();
    }

    // ---- the group's last CTA goes on ----
    __syncthreads();
    if (tid == 0) {
        const unsigned last = (unsigned)(W * splits - 1);
        s_last = atomicAdd(tickets + group, 1u) == last;
        if (s_last) tickets[group] = 0;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    beam_finish(a, splits, parts, group, s_group, s_best);
}

}  // namespace

lookat_status launch_beam_select(Ctx *ctx, const BeamArgs &a)
{
    const long long rows = (long long)a.groups * a.beams;
    // Parts of a row, whole batches each: as many as make the least of (waves of CTAs) x (batches of a part + 6), what a CTA does
    // besides its batches taking about as long as 6 of them.
    const int batches = (a.vocab + kBsBatch - 1) / kBsBatch;
    const long long slots = 4ll * ctx->sm_count;
    long long splits = 1, least = 0;
    int per = batches;
    for (int s = 1; s <= batches && s <= kBsSplits; ++s) {
        const int each = (batches + s - 1) / s;
        const long long cost = (rows * s + slots - 1) / slots * (each + 6);
        if (s == 1 || cost < least) least = cost, per = each;
    }
    splits = (batches + per - 1) / per;
    lookat_status st = workspace(ctx, ctx->beam_parts, (size_t)(rows * splits) * sizeof(BsPart), false, "beam_select");
    if (st != LOOKAT_OK) return st;
    st = workspace(ctx, ctx->beam_tickets, (size_t)a.groups * sizeof(unsigned), true, "beam_select");
    if (st != LOOKAT_OK) return st;
    const bool wide = (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0 && a.stride % 4 == 0;
    auto kern = wide ? beam_select_kernel<true> : beam_select_kernel<false>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kBsRing) != cudaSuccess)
        return check_launch(ctx, "beam_select: shared-memory opt-in");
    kern<<<(unsigned)(rows * splits), kBsThreads, kBsRing, ctx->stream>>>(a, (int)splits, per * kBsBatch, static_cast<BsPart *>(ctx->beam_parts.ptr),
                                                                    static_cast<unsigned *>(ctx->beam_tickets.ptr));
    return check_launch(ctx, "beam_select_kernel");
}

}  // namespace lookat
