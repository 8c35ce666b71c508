// lookat_beam_select: one step of beam search.
//
// Bound by HBM: the logits are read once.  A row is cut into `splits` parts, a CTA each; in one pass a warp keeps
//   - sum exp(x - m) against a reference m that it takes from its first logits and seldom moves: fp32 exponentials, their sums
//     fp64, so that the ranks of different beams are compared to 1e-8;
//   - its `beams` best logits (a beam's candidates rank as its logits do), sorted over the lanes: lane i holds the i-th.  A logit
//     enters if it beats the last of them, which soon is rare; the first 512 logits' lane maxima give the bar to begin with.
// Rows are read in the same order whatever their alignment (16-byte loads where all rows lie on such borders, else 4-byte ones):
// beams with equal logits and scores get equal ranks, and the lower one goes first.
// The CTA's warps join in shared memory.  The last CTA of a group to finish (a counter, no waiting) joins the parts, ranks
// in fp64, and moves the beams.
#include "serve.cuh"

namespace lookat {

namespace {

constexpr int kBsThreads = 256, kBsWarps = kBsThreads / 32, kBsVecs = 4, kBsMost = 32;
constexpr int kBsBatch = kBsThreads * kBsVecs * 4;            // logits that a CTA has in flight

struct BsPart {                     // of a row: its best logits, sum exp(x - m) and m
    float best[kBsMost];
    int at[kBsMost];
    double sum;
    float m;
    int bad;                        // a NaN or +inf among them
};

// A warp's best so far, lane i the i-th; equal keys in rising order of `at`.
template <class Key>
struct BsList {
    Key key, bar;                   // bar, bar_at: what a candidate has to beat (all lanes the same)
    int at, bar_at;
    __device__ void clear()
    {
        key = bar = -INFINITY;
        at = bar_at = 0x7fffffff;
    }
    __device__ bool beats(Key k, int i) const { return k > bar || (k == bar && k > -INFINITY && i < bar_at); }
    // one candidate (the same in all lanes); returns its place
    __device__ int insert(Key k, int i, int lane, int beams)
    {
        const int place = __popc(__ballot_sync(0xffffffffu, key > k || (key == k && at < i)));
        const Key up = __shfl_up_sync(0xffffffffu, key, 1);
        const int up_at = __shfl_up_sync(0xffffffffu, at, 1);
        if (lane > place) key = up, at = up_at;
        if (lane == place) key = k, at = i;
        const Key last = __shfl_sync(0xffffffffu, key, beams - 1);
        const int last_at = __shfl_sync(0xffffffffu, at, beams - 1);
        if (beats(last, last_at)) bar = last, bar_at = last_at;
        return place;
    }
};

__device__ __forceinline__ float bs_max_nan(float a, float b)   // NaN if either is
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// whole numbers in the order of floats
__device__ __forceinline__ int bs_ordered(float x)
{
    const int i = __float_as_int(x);
    return i < 0 ? i ^ 0x7fffffff : i;
}
__device__ __forceinline__ float bs_number(int i) { return __int_as_float(i < 0 ? i ^ 0x7fffffff : i); }
// the (n + 1)-th largest of the lanes' numbers
__device__ __forceinline__ float bs_nth(float v, int n, int lane)
{
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j; j >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, v, j);
            const bool larger = ((lane & k) == 0) == ((lane & j) == 0);     // descending blocks, then ascending ones
            v = larger ? fmaxf(v, o) : fminf(v, o);
        }
    return __shfl_sync(0xffffffffu, v, n);
}

// The group's parts joined and ranked, its beams moved.
__device__ __noinline__ void beam_finish(const BeamArgs &a, int splits, const BsPart *__restrict__ parts, int group, double (*s_rank)[kBsMost],
                                         int (*s_at)[kBsMost])
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, W = a.beams;
    __shared__ double s_base[kBsMost];                         // score = base + (x - m)
    __shared__ float s_top[kBsMost], s_score[kBsMost];
    __shared__ int s_len[kBsMost], s_fin[kBsMost], s_parent[kBsMost];
    const int g0 = group * W;
    if (tid < W) {
        s_score[tid] = a.scores[g0 + tid];
        s_len[tid] = a.lengths[g0 + tid];
        s_fin[tid] = a.finished[g0 + tid] != 0;
    }
    __syncthreads();
    BsList<double> list;
    list.clear();
    auto offer = [&](double k, int at, bool on) {              // a candidate per lane
        unsigned who = __ballot_sync(0xffffffffu, on && list.beats(k, at));
        while (who) {
            const int src = __ffs(who) - 1;
            who &= who - 1;
            const double kk = __shfl_sync(0xffffffffu, k, src);
            const int aa = __shfl_sync(0xffffffffu, at, src);
            if (list.beats(kk, aa)) list.insert(kk, aa, lane, W);
        }
    };
    for (int w = warp; w < W; w += kBsWarps) {
        const float sc = s_score[w];
        const bool counts = sc > -INFINITY && sc < INFINITY;
        const int grown = max(s_len[w] + (s_fin[w] ? 0 : 1), 1);
        const double norm = a.penalty == 0.0 ? 1.0 : pow((double)grown, a.penalty);
        double base = sc;
        float top = 0.f;
        if (counts && !s_fin[w]) {
            const BsPart *p = parts + (size_t)(g0 + w) * splits;
            top = -INFINITY;
            bool bad = false;
            for (int i = lane; i < splits; i += 32) top = fmaxf(top, __ldcg(&p[i].m)), bad |= __ldcg(&p[i].bad) != 0;
#pragma unroll
            for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            bad = __any_sync(0xffffffffu, bad) || top == -INFINITY;
            if (!bad) {
                double total = 0.0;
                for (int i = lane; i < splits; i += 32)
                    if (__ldcg(&p[i].m) > -INFINITY) total += __ldcg(&p[i].sum) * exp((double)__ldcg(&p[i].m) - (double)top);
#pragma unroll
                for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
                base = (double)sc - log(total);
                for (int i = 0; i < splits; ++i) {
                    const float x = __ldcg(&p[i].best[lane]);
                    const int at = __ldcg(&p[i].at[lane]);
                    offer((base + ((double)x - (double)top)) / norm, w * a.vocab + at, lane < W && x > -INFINITY);
                }
            }
        } else if (counts) {
            offer((double)sc / norm, w * a.vocab + max(a.eos, 0), lane == 0);
        }
        if (lane == 0) s_base[w] = base, s_top[w] = top;
    }
    s_rank[warp][lane] = list.key;
    s_at[warp][lane] = list.at;
    __syncthreads();
    if (warp == 0) {
        for (int w = 1; w < kBsWarps; ++w) offer(s_rank[w][lane], s_at[w][lane], lane < W && s_rank[w][lane] > -INFINITY);
        if (lane < W) {
            const bool there = list.key > -INFINITY;
            const int parent = there ? list.at / a.vocab : lane, token = there ? list.at % a.vocab : max(a.eos, 0);
            const bool grows = there && !s_fin[parent];
            float now = -INFINITY;
            if (there) now = s_fin[parent] ? s_score[parent] : (float)(s_base[parent] + ((double)a.logits[(long long)(g0 + parent) * a.stride + token] - (double)s_top[parent]));
            const int was = s_len[parent];
            a.scores[g0 + lane] = now;
            a.lengths[g0 + lane] = was + (grows ? 1 : 0);
            a.finished[g0 + lane] = s_fin[parent] || (grows && token == a.eos);
            a.next_ids[g0 + lane] = token;
            a.parents[g0 + lane] = g0 + parent;
            s_parent[lane] = parent;
            s_at[0][lane] = grows ? was : -1;                  // where its token goes
            s_at[1][lane] = token;
        }
    }
    if (!a.max_len) return;
    __syncthreads();
    // ---- the histories, a column per thread: all beams' numbers are read before the first is written ----
    int32_t *const tokens = a.tokens + (size_t)g0 * a.max_len;
    for (int c = tid; c < a.max_len; c += kBsThreads) {
        int32_t y[kBsMost];
#pragma unroll
        for (int w = 0; w < kBsMost; ++w)
            if (w < W) y[w] = s_at[0][w] == c ? s_at[1][w] : tokens[(size_t)s_parent[w] * a.max_len + c];
#pragma unroll
        for (int w = 0; w < kBsMost; ++w)
            if (w < W) tokens[(size_t)w * a.max_len + c] = y[w];
    }
}

template <bool WIDE>
__global__ void __launch_bounds__(kBsThreads, 3)
beam_select_kernel(const __grid_constant__ BeamArgs a, int splits, int part, BsPart *__restrict__ parts, unsigned *__restrict__ tickets)
{
    __shared__ float s_key[kBsWarps][kBsMost];
    __shared__ double s_rank[kBsWarps][kBsMost];
    __shared__ int s_at[kBsWarps][kBsMost];
    __shared__ double s_sum[kBsWarps];
    __shared__ float s_m[kBsWarps];
    __shared__ int s_bad[kBsWarps];
    __shared__ int s_last, s_bar;                              // s_bar: a logit that `beams` of the part reach, as bs_ordered
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, W = a.beams;
    const int row = blockIdx.x / splits, split = blockIdx.x % splits, group = row / W;
    const float score = a.scores[row];
    const bool live = a.finished[row] == 0 && score > -INFINITY && score < INFINITY;

    if (live) {                                                // (the same for the whole CTA)
        if (tid == 0) s_bar = bs_ordered(-INFINITY);
        __syncthreads();
        const float *x0 = a.logits + (long long)row * a.stride;
        const int e1 = min((split + 1) * part, a.vocab);
        BsList<float> list;
        list.clear();
        float m = -INFINITY;
        double sum = 0.0;
        bool bad = false;
        for (int e0 = split * part; e0 < e1; e0 += kBsBatch) {
            // element e0 + 4 tid + 1024 i + j (wide), or e0 + tid + 256 (4 i + j)
            float x[kBsVecs][4];
            auto element = [&](int i, int j) { return WIDE ? e0 + 4 * (i * kBsThreads + tid) + j : e0 + (4 * i + j) * kBsThreads + tid; };
#pragma unroll
            for (int i = 0; i < kBsVecs; ++i) {
                if (WIDE && element(i, 3) < e1) {
                    const float4 y = __ldcs(reinterpret_cast<const float4 *>(x0 + element(i, 0)));
                    x[i][0] = y.x, x[i][1] = y.y, x[i][2] = y.z, x[i][3] = y.w;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[i][j] = element(i, j) < e1 ? __ldcs(x0 + element(i, j)) : -INFINITY;
                }
            }
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < kBsVecs; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) top = bs_max_nan(top, x[i][j]);
            if (__any_sync(0xffffffffu, !(top < INFINITY))) {  // nothing of the row counts any more
                bad = true;
                break;
            }
            if (m == -INFINITY || __any_sync(0xffffffffu, top > m + 20.f)) {
                float t = top;
#pragma unroll
                for (int o = 16; o; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
                if (m > -INFINITY) sum *= exp((double)m - (double)t);
                else if (t > -INFINITY) list.bar = bs_nth(top, W - 1, lane);
                m = t;
                if (m == -INFINITY) continue;
            }
            float add = 0.f;
#pragma unroll
            for (int i = 0; i < kBsVecs; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) add += ex2_approx((x[i][j] - m) * 1.4426950408889634f);
            sum += (double)add;
            const float shared_bar = bs_number(*(volatile int *)&s_bar);
            if (shared_bar > list.bar) list.bar = shared_bar, list.bar_at = 0x7fffffff;
            if (!__any_sync(0xffffffffu, top >= list.bar)) continue;
#pragma unroll
            for (int i = 0; i < kBsVecs; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int e = element(i, j);
                    unsigned who = __ballot_sync(0xffffffffu, list.beats(x[i][j], e));
                    while (who) {
                        const int src = __ffs(who) - 1;
                        who &= who - 1;
                        const float k = __shfl_sync(0xffffffffu, x[i][j], src);
                        const int at = e + (WIDE ? 4 : 1) * (src - lane);
                        if (list.beats(k, at)) list.insert(k, at, lane, W);
                    }
                }
            if (lane == 0) atomicMax(&s_bar, bs_ordered(list.bar));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        s_key[warp][lane] = list.key;
        s_at[warp][lane] = list.at;
        if (lane == 0) s_sum[warp] = sum, s_m[warp] = m, s_bad[warp] = bad;
        __syncthreads();
        if (warp == 0) {
            BsPart &p = parts[(size_t)row * splits + split];
            for (int w = 1; w < kBsWarps; ++w) {
                const float k = s_key[w][lane];
                const int at = s_at[w][lane];
                unsigned who = __ballot_sync(0xffffffffu, lane < W && list.beats(k, at));
                while (who) {
                    const int src = __ffs(who) - 1;
                    who &= who - 1;
                    const float kk = __shfl_sync(0xffffffffu, k, src);
                    const int aa = __shfl_sync(0xffffffffu, at, src);
                    if (list.beats(kk, aa)) list.insert(kk, aa, lane, W);
                }
            }
            p.best[lane] = list.key;
            p.at[lane] = list.at;
            float top = -INFINITY;
            bool any_bad = false;
            for (int w = 0; w < kBsWarps; ++w) top = fmaxf(top, s_m[w]), any_bad |= s_bad[w] != 0;
            double total = 0.0;                                // (the same in every lane)
            for (int w = 0; w < kBsWarps; ++w)
                if (s_m[w] > -INFINITY) total += s_sum[w] * exp((double)s_m[w] - (double)top);
            if (lane == 0) p.sum = total, p.m = top, p.bad = any_bad;
            __threadfence();
        }
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

    beam_finish(a, splits, parts, group, s_rank, s_at);
}

}  // namespace

lookat_status launch_beam_select(Ctx *ctx, const BeamArgs &a)
{
    const long long rows = (long long)a.groups * a.beams;
    // parts of a row: enough CTAs to fill the GPU a few times over, whole batches each
    const int batches = (a.vocab + kBsBatch - 1) / kBsBatch;
    long long splits = (4ll * 4 * ctx->sm_count + rows - 1) / rows;
    if (splits > batches) splits = batches;
    const int per = (int)((batches + splits - 1) / splits);
    splits = (batches + per - 1) / per;
    lookat_status st = workspace(ctx, ctx->beam_parts, (size_t)(rows * splits) * sizeof(BsPart), false, "beam_select");
    if (st != LOOKAT_OK) return st;
    st = workspace(ctx, ctx->beam_tickets, (size_t)a.groups * sizeof(unsigned), true, "beam_select");
    if (st != LOOKAT_OK) return st;
    const bool wide = (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0 && a.stride % 4 == 0;
    auto kern = wide ? beam_select_kernel<true> : beam_select_kernel<false>;
    kern<<<(unsigned)(rows * splits), kBsThreads, 0, ctx->stream>>>(a, (int)splits, per * kBsBatch, static_cast<BsPart *>(ctx->beam_parts.ptr),
                                                                    static_cast<unsigned *>(ctx->beam_tickets.ptr));
    return check_launch(ctx, "beam_select_kernel");
}

}  // namespace lookat
