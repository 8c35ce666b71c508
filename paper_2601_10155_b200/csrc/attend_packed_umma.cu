// lookat_attend_packed for head dims of 64 and 128: exact causal attention of packed prompts on the 5th-generation tensor cores.
//
//     S = Q K^T (fp16 operands, fp32)      w = 2^(S scale log2(e) - M)      O += w V,  l += w      out = O / l
// M lies kPackedLift below a line's largest score and moves only when the scores run ahead of it by more than kPuSlack: the
// weights, fp16 numbers, use fp16's range (up to 2^15), and O in tensor memory is seldom rescaled.
//
// A line is one (token, query head) pair of a KV head, line = token * g + head.  An item is two tiles of 128 lines of one row (`per`
// lines: one tile where there are few items), against chunks of 128 tokens; a persistent CTA per SM goes through every gridDim.x-th item of the list, which begins with those
// that see the most tokens (packed_tile).  Tensor memory is full: per tile 128 columns of scores, over whose first half the
// weights are written, and up to 128 of O.  So a tile's products alternate, S, O, S, O, and while the softmax threads work on
// one tile the tensor pipe works on the other.  With values of 64 dims there is room for the weights of their own (kApart), and a
// chunk's scores are made while the softmax threads work on the one before.  The roles run ahead of each other from item to item, so that an item's queries,
// keys and first scores are there when the one before is written out (12 warps, one CTA per SM by tensor memory):
//   warps 0-3 / 4-7  softmax of tile 0 / 1: thread r owns line r of its tile = tensor-memory lane r;
//   warp 8      fetches keys and values by tiled bulk copies, 128 tokens x 64 dims with the 128-byte swizzle, through maps over
//               the caller's strides; in the row's last chunk it zeroes the values behind the last token (a copy brings the next
//               row's tokens along, whose infinities the weights of zero would not take away);
//   warps 9, 10 one thread each issues the MMAs of tile 0 / 1 and commits them to mbarriers;
//   warp 11     fetches the query lines: by tiled bulk copies where a tile's lines are whole tokens of [tokens][heads][dims], else
//               by cp.async (any strides and groups).
//   4 x 4096 tokens, 32 and 8 heads of 128: 500 to 530 us, 1.04 to 1.1 PFLOP/s; one row of 16384 1.8 ms (1.2), 2.0 under the power cap.
// Softmax alone (the MMAs cut to one each) and MMAs alone (no exponentials, maxima, sums) take about three quarters of that each:
// the rest is that a tile's scores wait for its weights.  Short rows pay 3 to 4 us per item for its first scores and its way out.
// Every mbarrier wait gives up after a bounded number of polls, raises the context's time-out flag and lets the CTA drain and
// free its tensor memory.
#include <cuda.h>           // CUtensorMap only

#include <atomic>

#include "serve.cuh"
#include "umma.cuh"

namespace lookat {

namespace {

constexpr int kPuRows = 128, kPuChunk = 128, kPuTiles = 2, kPuBoth = kPuTiles * kPuRows;
constexpr int kPuSoftmax = kPuBoth, kPuThreads = kPuSoftmax + 128;
constexpr float kPuSlack = 8.f;
// Registers: the softmax threads hold 128 scores each.  The launch's 168 of each thread are split anew (2 x 128 x 208 + 128 x 88 is what
// 384 x 168 is): 4 x 4096 tokens, 32 and 8 heads of 128, 524 -> 500 us, 23 ragged rows 215 -> 198.
constexpr int kPuLaunchRegs = 168, kPuSoftmaxRegs = 208, kPuOtherRegs = 88;
static_assert(kPuSoftmax * kPuSoftmaxRegs + (kPuThreads - kPuSoftmax) * kPuOtherRegs <= kPuThreads * kPuLaunchRegs, "register split");
constexpr int kPuListed = 128;                  // items that a CTA finds at its start, with all its warps; later ones every role finds by itself

template <int DK, int DV>
struct PuLayout {
    static constexpr int kStages = DK == 64 && DV == 64 ? 4 : 2;
    static constexpr int kKb = DK / 64, kVb = DV / 64, kBox = kPuChunk * 128;        // 64 dims of a chunk: 16 KB
    static constexpr int kK = kKb * kBox, kV = kVb * kBox, kQ = kPuRows * 2 * DK;
    static constexpr int kOffK = 0, kOffV = kStages * kK, kOffQ = kOffV + kStages * kV;
    static constexpr int kTurn = 4096, kOffTurn = kOffQ + kPuTiles * kQ, kOffBars = kOffTurn + kPuSoftmax / 32 * kTurn;     // turn: a warp's results on their way out
    static constexpr int kOffItems = kOffBars + 512, kBytes = kOffItems + kPuListed * 16;
    // tensor memory: scores of both tiles, O of both, and where that leaves room (kApart) the weights of both beside the scores
    static constexpr bool kApart = DV == 64;
    static constexpr int kColO = kPuTiles * kPuChunk, kColP = kColO + kPuTiles * DV;
    // instruction descriptors: fp32 accumulate, fp16 operands, N >> 3 at bit 17, M >> 4 at bit 24; bit 16: B is MN-major
    static constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)(kPuChunk >> 3) << 17) | ((uint32_t)(kPuRows >> 4) << 24);
    static constexpr uint32_t kIdescO = (1u << 4) | (1u << 16) | ((uint32_t)(DV >> 3) << 17) | ((uint32_t)(kPuRows >> 4) << 24);
};

__device__ __forceinline__ float2 pu_fma2(float2 a, float b, float c)           // a * b + c, both halves in one instruction
{
    float2 d;
    asm("{\n.reg .b64 u, v, w, r;\nmov.b64 u, {%2, %3};\nmov.b64 v, {%4, %4};\nmov.b64 w, {%5, %5};\nfma.rn.f32x2 r, u, v, w;\nmov.b64 {%0, %1}, r;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float2 pu_add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n.reg .b64 u, v, r;\nmov.b64 u, {%2, %3};\nmov.b64 v, {%4, %5};\nadd.rn.f32x2 r, u, v;\nmov.b64 {%0, %1}, r;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float pu_max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// one box of a map over [tokens][heads][dims]; heads_last: over [heads][tokens][dims] (the map's dims go by their strides)
__device__ __forceinline__ void pu_copy(uint32_t dst, const CUtensorMap *map, int c, int h, int t, bool heads_last, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(c), "r"(heads_last ? t : h), "r"(heads_last ? h : t), "r"(bar)
                 : "memory");
}

template <int DK, int DV>
__global__ void __launch_bounds__(kPuThreads, 1)
attend_packed_umma_kernel(const __grid_constant__ PackedAttendArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                          const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap out_map,
                          int q_boxes, int out_boxes /* 0: none, 2: map over [heads][tokens] */, int per, int k_order, int v_order, int *__restrict__ timeout_flag)
{
    using Lay = PuLayout<DK, DV>;
    constexpr int kStages = Lay::kStages;
    extern __shared__ __align__(1024) unsigned char pu_smem[];
    unsigned char *const sm = pu_smem;
    const uint32_t sm0 = um_smem(sm);
    uint64_t *const bars = reinterpret_cast<uint64_t *>(sm + Lay::kOffBars);
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(bars + 30);
    // per stage: keys there, keys free, values there, values free; per tile: scores done and weights stored (of each of its
    // chunks; with kApart also scores read, value MMAs done), queries there, queries free, O done, O read (of each of its items); copies of a row's last values there.  A phase of each
    // ends only after every waiter of the one before has moved on.
    const uint32_t bar0 = um_smem(bars), bar_k = bar0, bar_kf = bar0 + 32, bar_v = bar0 + 64, bar_vf = bar0 + 96;
    const uint32_t bar_s = bar0 + 128, bar_p = bar0 + 144, bar_q = bar0 + 160, bar_qf = bar0 + 176, bar_o = bar0 + 192, bar_of = bar0 + 208;
    const uint32_t bar_t = bar0 + 224, bar_sf = bar0 + 256, bar_pv = bar0 + 272;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (blockIdx.x == 0) packed_check(a.rows, tid, kPuThreads);
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            um_bar_init(bar_k + 8 * i, 1);
            um_bar_init(bar_v + 8 * i, 1);
            um_bar_init(bar_kf + 8 * i, kPuTiles);
            um_bar_init(bar_vf + 8 * i, kPuTiles);
        }
        for (int t = 0; t < kPuTiles; ++t) {
            um_bar_init(bar_s + 8 * t, 1);
            um_bar_init(bar_p + 8 * t, kPuRows / 32);
            um_bar_init(bar_q + 8 * t, 1);
            um_bar_init(bar_sf + 8 * t, kPuRows / 32);
            um_bar_init(bar_pv + 8 * t, 1);
            um_bar_init(bar_qf + 8 * t, 1);
            um_bar_init(bar_o + 8 * t, 1);
            um_bar_init(bar_of + 8 * t, kPuRows / 32);
        }
        um_bar_init(bar_t, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(um_smem(tmem_slot)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // ---- the CTA's items: up to two tiles of a row and KV head each: {first token, tokens of the row, place of the tiles, what packed_tile said} ----
    int4 *const listed = reinterpret_cast<int4 *>(sm + Lay::kOffItems);
    for (int k = warp; k < kPuListed; k += kPuThreads / 32) {
        int4 item = make_int4(0, 0, 0, 0);
        item.w = packed_tile(a.rows, a.g, per, (blockIdx.x + k * gridDim.x) / a.H_kv, lane, item.z, item.x, item.y);
        if (lane == 0) listed[k] = item;
        if (item.w == kNoMore) break;                          // (a warp of an earlier place has met the end, too, or will)
    }
    um_fence_before();
    __syncthreads();
    um_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool dead = (sm0 & 1023u) != 0;                            // a wait ran out (or the base is misaligned): leave, free, return

    // every role goes through the items by itself
    int k = -1, h = 0, first = 0, n = 0, line0 = 0, lines = 0, n_chunks = 0;
    auto next = [&]() {
        int4 item;
        do {
            ++k;
            if (k < kPuListed) item = listed[k];
            else item.w = packed_tile(a.rows, a.g, per, (blockIdx.x + k * gridDim.x) / a.H_kv, lane, item.z, item.x, item.y);
            if (item.w == kNoMore) return false;
        } while (item.w == kNoTile);
        first = item.x, n = item.y;
        h = (blockIdx.x + k * gridDim.x) % a.H_kv;
        line0 = item.z * per;
        lines = n * a.g;
        n_chunks = (min(line0 + per, lines) - 1) / a.g / kPuChunk + 1;
        return true;
    };
    auto chunks_of = [&](int t) { return t * kPuRows < per && line0 + t * kPuRows < lines ? (min(line0 + (t + 1) * kPuRows, lines) - 1) / a.g / kPuChunk + 1 : 0; };

    if (dead) {
        // misaligned shared-memory base: nothing runs
    } else if (warp >= kPuSoftmax / 32) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPuOtherRegs));
        if (warp == kPuSoftmax / 32) {
            // =================== the fetcher ===================
            // A row's last values, where it ends inside a chunk, come by a barrier of their own; with zeros behind them they are handed
            // on.
            int sent = 0, v_sent = 0, tails = 0;                   // chunks of keys, of values, of those with an end
            while (!dead && next()) {
                const int tail = n - (n_chunks - 1) * kPuChunk;
                if (um_elect()) {
                    for (int ch = 0; ch < n_chunks; ++ch) {
                        const int st = sent % kStages, t0 = first + ch * kPuChunk;
                        const uint32_t done = (sent / kStages - 1) & 1, v_bar = ch == n_chunks - 1 && tail < kPuChunk ? bar_t : bar_v + 8 * st;
                        if (sent >= kStages && !um_bar_wait(bar_kf + 8 * st, done)) { dead = true; break; }
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar_k + 8 * st), "r"(Lay::kK) : "memory");
#pragma unroll
                        for (int i = 0; i < Lay::kKb; ++i) pu_copy(sm0 + Lay::kOffK + st * Lay::kK + i * Lay::kBox, &k_map, i * 64, h, t0, k_order, bar_k + 8 * st);
                        ++sent;
                        if (sent > kStages && !um_bar_wait(bar_vf + 8 * st, done)) { dead = true; break; }
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(v_bar), "r"(Lay::kV) : "memory");
#pragma unroll
                        for (int i = 0; i < Lay::kVb; ++i) pu_copy(sm0 + Lay::kOffV + st * Lay::kV + i * Lay::kBox, &v_map, i * 64, h, t0, v_order, v_bar);
                        ++v_sent;
                    }
                    if (dead) {                                    // copies in flight end before the CTA does
                        for (int i = max(0, sent - kStages); i < sent; ++i) um_bar_wait(bar_k + 8 * (i % kStages), (i / kStages) & 1);
                        for (int i = max(0, v_sent - kStages); i < v_sent; ++i) um_bar_wait(bar_v + 8 * (i % kStages), (i / kStages) & 1);
                    }
                }
                dead = __any_sync(0xffffffffu, dead);
                sent = __reduce_max_sync(0xffffffffu, sent);
                v_sent = __reduce_max_sync(0xffffffffu, v_sent);
                if (!dead && tail < kPuChunk) {
                    const int st = (v_sent - 1) % kStages;
                    if (!__all_sync(0xffffffffu, um_bar_wait(bar_t, tails & 1))) { dead = true; break; }
                    ++tails;
                    unsigned char *const rows = sm + Lay::kOffV + st * Lay::kV;
                    for (int i = tail * 8 + lane; i < kPuChunk * 8; i += 32)
#pragma unroll
                        for (int j = 0; j < Lay::kVb; ++j) *reinterpret_cast<uint4 *>(rows + j * Lay::kBox + i * 16) = make_uint4(0u, 0u, 0u, 0u);
                    um_fence_async_smem();
                    __syncwarp();
                    if (lane == 0) um_bar_arrive(bar_v + 8 * st);
                }
            }
        } else if (warp == kPuThreads / 32 - 1) {
            // =================== the queries: A operand of the scores, 64 dims each, 128-byte swizzle ===================
            constexpr int kPieces = DK / 8;
            int seen[kPuTiles] = {0, 0}, chunks = 0;               // chunks: of the item before, all of whose scores this waits for
            bool started = false;
            while (!dead && next()) {
                const int tiles = chunks_of(1) ? 2 : 1;
                for (int t = 0; t < tiles; ++t) {
                    bool there = seen[t] == 0;
                    for (int i = 0; i <= chunks && !there; ++i) there = __all_sync(0xffffffffu, um_bar_wait(bar_qf + 8 * t, (seen[t] - 1) & 1));
                    if (!there) { dead = true; break; }
                    if (q_boxes) {                                 // (tokens behind the row's end are lines that are not written)
                        if (um_elect()) {
                            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar_q + 8 * t), "r"(Lay::kQ) : "memory");
#pragma unroll
                            for (int i = 0; i < Lay::kKb; ++i)
                                pu_copy(sm0 + Lay::kOffQ + t * Lay::kQ + i * (kPuRows * 128), &q_map, i * 64, h * a.g, first + (line0 + t * kPuRows) / a.g, q_boxes == 2, bar_q + 8 * t);
                        }
                        __syncwarp();
                        ++seen[t];
                        continue;
                    }
#pragma unroll 1
                    for (int part = 0; part < kPuRows / 32; ++part) {
                        const int line = min(line0 + t * kPuRows + part * 32 + lane, lines - 1);       // lines beyond the last repeat it
                        const unsigned long long src = reinterpret_cast<unsigned long long>(a.q.p + (first + line / a.g) * a.q.ts + (h * a.g + line % a.g) * a.q.hs);
#pragma unroll
                        for (int i = 0; i < kPieces; ++i) {
                            const int idx = i * 32 + lane, row = part * 32 + idx / kPieces, piece = idx % kPieces;
                            const unsigned long long from = __shfl_sync(0xffffffffu, src, idx / kPieces);
                            um_cp_async16(sm0 + Lay::kOffQ + t * Lay::kQ + (piece >> 3) * (kPuRows * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4),
                                          reinterpret_cast<const uint4 *>(from) + piece);
                        }
                    }
                    asm volatile("cp.async.commit_group;" ::: "memory");
                    if (!started && tiles == 2) {                  // (both tiles of the first item at once)
                        if (t == 0) continue;
                        asm volatile("cp.async.wait_group 1;" ::: "memory");
                        um_fence_async_smem();
                        __syncwarp();
                        if (lane == 0) um_bar_arrive(bar_q);
                        ++seen[0];
                    }
                    asm volatile("cp.async.wait_group 0;" ::: "memory");
                    um_fence_async_smem();
                    __syncwarp();
                    if (lane == 0) um_bar_arrive(bar_q + 8 * t);
                    ++seen[t];
                }
                started = true;
                chunks = n_chunks;
            }
            // copies in flight end before the CTA does
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (q_boxes && dead)
                for (int t = 0; t < kPuTiles; ++t)
                    if (seen[t]) um_bar_wait(bar_q + 8 * t, (seen[t] - 1) & 1);
        } else if (warp > kPuSoftmax / 32) {
            // =================== the MMA thread of a tile ===================
            const int t = warp - kPuSoftmax / 32 - 1;
            // descriptors: stride 1024 B, version 1, 128-byte swizzle in the high word; start address and leading offset in
            // the low word
            const uint32_t desc_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
            const uint32_t k_lo = ((sm0 + Lay::kOffK) >> 4) | (1u << 16);                              // leading offset unused (16 B)
            const uint32_t q_lo = ((sm0 + Lay::kOffQ + t * Lay::kQ) >> 4) | (1u << 16);
            const uint32_t v_lo = ((sm0 + Lay::kOffV) >> 4) | ((uint32_t)(Lay::kBox / 16) << 16);      // between 64-column blocks
            const uint32_t tm_s = tmem + t * kPuChunk, tm_o = tmem + Lay::kColO + t * DV, tm_p = Lay::kApart ? tmem + Lay::kColP + t * (kPuChunk / 2) : tm_s;
            int chunk0 = 0, mine0 = 0, items = 0;                  // chunks of all items so far, the tile's own, its items
            while (!dead && next()) {
                const int mine = chunks_of(t);
                if (um_elect()) {
                    // (waits that are over already go first: between a tile's weights and its next scores there is nothing but the MMAs)
                    auto keys_there = [&](int ch) { return um_bar_wait(bar_k + 8 * ((chunk0 + ch) % kStages), ((chunk0 + ch) / kStages) & 1); };
                    auto values_there = [&](int ch) { return um_bar_wait(bar_v + 8 * ((chunk0 + ch) % kStages), ((chunk0 + ch) / kStages) & 1); };
                    auto score_mma = [&](int ch) {
                        const int st = (chunk0 + ch) % kStages;
                        const uint32_t lo = k_lo + st * (Lay::kK >> 4);
#pragma unroll
                        for (int ks = 0; ks < DK / 16; ++ks) {
                            const uint32_t off = ((ks >> 2) * Lay::kBox + (ks & 3) * 32) >> 4;
                            if (ks == 0) um_mma_ss<false>(tm_s, q_lo + off, desc_hi, lo + off, desc_hi, Lay::kIdescS);
                            else um_mma_ss<true>(tm_s, q_lo + off, desc_hi, lo + off, desc_hi, Lay::kIdescS);
                        }
                        um_commit(bar_s + 8 * t);
                        um_commit(bar_kf + 8 * st);
                        if (ch == mine - 1) um_commit(bar_qf + 8 * t);
                    };
                    auto value_mma = [&](int ch) {
                        const int st = (chunk0 + ch) % kStages;
                        const uint32_t lo = v_lo + st * (Lay::kV >> 4);
#pragma unroll
                        for (int kt = 0; kt < kPuChunk / 16; ++kt) {
                            if (kt == 0 && ch == 0) um_mma_ts<false>(tm_o, tm_p, lo, desc_hi, Lay::kIdescO);
                            else um_mma_ts<true>(tm_o, tm_p + kt * 8, lo + kt * (2048 >> 4), desc_hi, Lay::kIdescO);
                        }
                        if (Lay::kApart) um_commit(bar_pv + 8 * t);
                        um_commit(bar_vf + 8 * st);
                    };
                    bool ok = true;
                    if (mine) {
                        ok = keys_there(0) && um_bar_wait(bar_q + 8 * t, items & 1) && (!Lay::kApart || !mine0 || um_bar_wait(bar_sf + 8 * t, (mine0 - 1) & 1));
                        if (ok) {
                            um_fence_after();
                            score_mma(0);
                        }
                        ok = ok && (!items || um_bar_wait(bar_of + 8 * t, (items - 1) & 1));
                        for (int ch = 0; ok && ch < mine; ++ch) {
                            const bool last = ch + 1 >= mine;
                            if (Lay::kApart && !last) {            // the next scores while the softmax threads work on these
                                ok = keys_there(ch + 1) && um_bar_wait(bar_sf + 8 * t, (mine0 + ch) & 1);
                                if (!ok) break;
                                um_fence_after();
                                score_mma(ch + 1);
                            }
                            ok = values_there(ch) && (Lay::kApart || last || keys_there(ch + 1)) && um_bar_wait(bar_p + 8 * t, (mine0 + ch) & 1);
                            if (!ok) break;
                            um_fence_after();
                            value_mma(ch);
                            if (!Lay::kApart && !last) score_mma(ch + 1);
                        }
                        if (ok) um_commit(bar_o + 8 * t);
                    }
                    for (int ch = mine; ok && ch < n_chunks; ++ch) {               // chunks that only the other tile sees
                        const int st = (chunk0 + ch) % kStages;
                        ok = um_bar_wait(bar_k + 8 * st, ((chunk0 + ch) / kStages) & 1);
                        if (ok) um_bar_arrive(bar_kf + 8 * st);
                        ok = ok && um_bar_wait(bar_v + 8 * st, ((chunk0 + ch) / kStages) & 1);
                        if (ok) um_bar_arrive(bar_vf + 8 * st);
                    }
                    dead = !ok;
                }
                dead = __any_sync(0xffffffffu, dead);
                chunk0 += n_chunks;
                mine0 += mine;
                items += mine > 0;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPuSoftmaxRegs));
        // =================== softmax: thread r owns line r of its tile ===================
        const int tile = warp >> 2;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tm_s = tmem + tile * kPuChunk + lane_base, tm_o = tmem + Lay::kColO + tile * DV + lane_base;
        const uint32_t tm_p = Lay::kApart ? tmem + Lay::kColP + tile * (kPuChunk / 2) + lane_base : tm_s;
        unsigned char *const turn = sm + Lay::kOffTurn + warp * Lay::kTurn;
        int mine0 = 0, items = 0;                              // the tile's chunks and items so far
        bool more = next();
        while (!dead && more) {
            const int mine = chunks_of(tile), line = line0 + tile * kPuRows + (warp & 3) * 32 + lane, line_c = min(line, lines - 1);
            if (!mine) {
                more = next();
                continue;
            }
            const int tok = line_c / a.g;                      // (lines beyond the last repeat it)
            const unsigned long long out = line < lines ? reinterpret_cast<unsigned long long>(a.out.p + (first + tok) * a.out.ts + (h * a.g + line_c % a.g) * a.out.hs) : 0;
            // (all of the warp's lines are the row's, and in one box)
            const int line_w = line0 + tile * kPuRows + (warp & 3) * 32, box_head = h * a.g, box_token = first + line_w / a.g;
            const bool boxed = out_boxes && line_w + 32 <= lines;
            float m_run = 0.f, l_run = 0.f;
            for (int ch = 0; ch < mine; ++ch) {
                if (!__all_sync(0xffffffffu, um_bar_wait(bar_s + 8 * tile, (mine0 + ch) & 1))) { dead = true; break; }     // warp-uniform
                um_fence_after();
                float2 y[kPuChunk / 2];
                {
                    uint32_t s[kPuChunk / 32][32];
#pragma unroll
                    for (int p = 0; p < kPuChunk / 32; ++p) um_ld32(s[p], tm_s + p * 32);
                    um_wait_ld();
#pragma unroll
                    for (int i = 0; i < kPuChunk / 2; ++i) y[i] = make_float2(__uint_as_float(s[i / 16][2 * i % 32]), __uint_as_float(s[i / 16][2 * i % 32 + 1]));
                }
                if (Lay::kApart) {
                    um_fence_before();
                    __syncwarp();
                    if (lane == 0) um_bar_arrive(bar_sf + 8 * tile);
                }
                const int sees = tok + 1 - ch * kPuChunk;      // tokens of the chunk that this line sees
                if (__any_sync(0xffffffffu, sees < kPuChunk)) {
#pragma unroll
                    for (int i = 0; i < kPuChunk / 2; ++i) {
                        if (2 * i >= sees) y[i].x = -INFINITY;
                        if (2 * i + 1 >= sees) y[i].y = -INFINITY;
                    }
                }
                float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < kPuChunk / 2; ++i) tops[i & 3] = pu_max3(tops[i & 3], y[i].x, y[i].y);
                const float top = fmaxf(pu_max3(tops[0], tops[1], tops[2]), tops[3]) * a.scale_log2;
                // M moves only when the scores run ahead by more than kPuSlack (token 0 is in every line's first chunk)
                float alpha = 1.f;
                if (ch == 0) {
                    m_run = top - kPackedLift;
                } else if (top > m_run + (kPackedLift + kPuSlack)) {
                    alpha = ex2_approx(m_run - (top - kPackedLift));
                    m_run = top - kPackedLift;
                }
                // the value MMAs of the chunk before are over: with kApart asked for here, else known by these scores, which the same
                // thread issued after them
                if (Lay::kApart && mine0 + ch && !__all_sync(0xffffffffu, um_bar_wait(bar_pv + 8 * tile, (mine0 + ch - 1) & 1))) { dead = true; break; }
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t pk[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const float2 e = pu_fma2(y[half * 32 + i], a.scale_log2, -m_run);
                        const float2 w = make_float2(ex2_approx(e.x), ex2_approx(e.y));
                        sum[i & 1] = pu_add2(sum[i & 1], w);
                        const __half2 x = __floats2half2_rn(w.x, w.y);
                        pk[i] = *reinterpret_cast<const uint32_t *>(&x);
                    }
                    um_st32(tm_p + half * 32, pk);
                }
                l_run = fmaf(l_run, alpha, (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
                if (__any_sync(0xffffffffu, alpha != 1.f)) {
                    um_fence_after();
#pragma unroll 1
                    for (int p = 0; p < DV / 32; ++p) {
                        uint32_t o[32];
                        um_ld32(o, tm_o + p * 32);
                        um_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                        um_st32(tm_o + p * 32, o);
                    }
                }
                um_wait_st();
                um_fence_before();
                __syncwarp();
                if (lane == 0) um_bar_arrive(bar_p + 8 * tile);         // (one of a warp: 128 arrivals at a barrier take their time)
            }
            mine0 += mine;
            const int parity = items++ & 1;
            more = next();                                     // (found while the last products run)
            if (dead || !__all_sync(0xffffffffu, um_bar_wait(bar_o + 8 * tile, parity))) { dead = true; break; }
            // ---- results, 64 dims at a time by way of the warp's shared memory: whole lines of global memory ----
            um_fence_after();
            const float inv = 1.f / l_run;
#pragma unroll
            for (int part = 0; part < DV / 64; ++part) {
                uint32_t o[2][32];
                um_ld32(o[0], tm_o + part * 64);
                um_ld32(o[1], tm_o + part * 64 + 32);
                um_wait_ld();
                if (part == DV / 64 - 1) {
                    um_fence_before();
                    __syncwarp();
                    if (lane == 0) um_bar_arrive(bar_of + 8 * tile);
                }
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");         // the copy before has read them
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t *const w = &o[i >> 2][(i & 3) * 8];
                    uint4 x;
                    x.x = q8_half2(__uint_as_float(w[0]) * inv, __uint_as_float(w[1]) * inv);
                    x.y = q8_half2(__uint_as_float(w[2]) * inv, __uint_as_float(w[3]) * inv);
                    x.z = q8_half2(__uint_as_float(w[4]) * inv, __uint_as_float(w[5]) * inv);
                    x.w = q8_half2(__uint_as_float(w[6]) * inv, __uint_as_float(w[7]) * inv);
                    *reinterpret_cast<uint4 *>(turn + lane * 128 + ((i ^ (lane & 7)) << 4)) = x;
                }
                if (boxed) {
                    um_fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(&out_map), "r"(part * 64),
                                     "r"(out_boxes == 2 ? box_token : box_head), "r"(out_boxes == 2 ? box_head : box_token), "r"(um_smem(turn))
                                     : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                    continue;
                }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int row = i * 4 + (lane >> 3), piece = lane & 7;
                    const uint4 x = *reinterpret_cast<const uint4 *>(turn + row * 128 + ((piece ^ (row & 7)) << 4));
                    const unsigned long long dst = __shfl_sync(0xffffffffu, out, row);
                    if (dst) *(reinterpret_cast<uint4 *>(dst) + part * 8 + piece) = x;
                }
                __syncwarp();
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");      // (results on their way out)
    }

    if (dead) atomicExch(timeout_flag, 1);
    um_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

template <int DK, int DV>
lookat_status launch_pu(Ctx *ctx, const PackedAttendArgs &a)
{
    using Lay = PuLayout<DK, DV>;
    auto kern = attend_packed_umma_kernel<DK, DV>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay::kBytes) != cudaSuccess)
        return check_launch(ctx, "attend_packed (tcgen05 form): shared-memory opt-in");
    // (with fewer registers than it was written for, the split would wait for ever; an answer is kept, a failure to get one is not)
    static std::atomic<int> regs{0};
    if (!regs) {
        cudaFuncAttributes attributes;
        if (cudaFuncGetAttributes(&attributes, kern) == cudaSuccess) regs = attributes.numRegs;
        else cudaGetLastError();
    }
    if (regs < kPuLaunchRegs) return launch_attend_packed_any(ctx, a);
    CUtensorMap k_map, v_map, q_map, out_map;
    int k_order, v_order, q_order = 0, out_order = 0;
    if (!make_rows_map_f16(&k_map, a.k.p, DK, a.H_kv, a.rows.n, a.k.hs, a.k.ts, 1, kPuChunk, &k_order) ||
        !make_rows_map_f16(&v_map, a.v.p, DV, a.H_kv, a.rows.n, a.v.hs, a.v.ts, 1, kPuChunk, &v_order))
        return launch_attend_packed_any(ctx, a);               // (strides that the driver makes no map of)
    // a tile's lines in one box: g heads of 128 / g tokens, heads innermost
    const bool whole = kPuRows % a.g == 0 &&
                       make_rows_map_f16(&q_map, a.q.p, DK, a.H_q, a.rows.n, a.q.hs, a.q.ts, a.g, kPuRows / a.g, &q_order);
    const int q_boxes = whole && (!q_order || a.g == 1);
    if (!q_boxes) q_map = k_map;                               // (not used)
    // a warp's lines of results, 64 dims, likewise
    const bool out_whole = 32 % a.g == 0 &&
                           make_rows_map_f16(&out_map, a.out.p, DV, a.H_q, a.rows.n, a.out.hs, a.out.ts, a.g, 32 / a.g, &out_order);
    const int out_boxes = out_whole && (!out_order || a.g == 1);
    if (!out_boxes) out_map = k_map;
    // (no more than this, whatever the rows' lengths)
    auto items = [&](int per) { return packed_tiles(a.rows, a.g, per) * a.H_kv; };
    // items of one tile where there is an SM for each (2048 tokens, 8 and 2 heads of 128: 38 us, and 46 with two; 1000 tokens, 32 and 8
    // heads, where there is not, 34 and 32)
    const int per = items(kPuRows) <= ctx->sm_count ? kPuRows : kPuBoth;
    const long long ctas = items(per);
    if (ctas > 0x3fffffffll) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "attend_packed: too many tokens for one call");
    kern<<<(unsigned)(ctas < ctx->sm_count ? ctas : ctx->sm_count), kPuThreads, Lay::kBytes, ctx->stream>>>(a, k_map, v_map, q_map, out_map, q_boxes ? 1 + q_order : 0,
                                                                                                   out_boxes ? 1 + out_order : 0, per, k_order, v_order, ctx->timeout_flag);
    return check_launch(ctx, "attend_packed_umma_kernel");
}

}  // namespace

bool attend_packed_umma_covers(const Ctx *ctx, const PackedAttendArgs &a)
{
    // Rows of more than 64 lines (one tile of attend_packed_kernel) on average, as far as the host knows: shorter ones leave most of
    // two tiles of 128 empty.  16384 tokens, 12 heads of 64: rows of 32 tokens 202 us here and 97 there, of 64 109 and 69, of 128 62
    // and 77; 32 and 8 heads of 128: rows of 16 306 and 259, of 32 160 and 249.  The average is over all B rows: one of 4096 tokens,
    // 32 and 8 heads of 128, takes 142 us alone, 149 with 254 empty rows and 654, on the other form, with 255.
    const bool dims = (a.d_k == 64 || a.d_k == 128) && (a.d_v == 64 || a.d_v == 128);
    return dims && (long long)a.rows.n * a.g > 64ll * a.rows.B && ctx->timeout_flag && tile_maps_available();
}

lookat_status launch_attend_packed_umma(Ctx *ctx, const PackedAttendArgs &a)
{
    if (a.d_k == 128) return a.d_v == 128 ? launch_pu<128, 128>(ctx, a) : launch_pu<128, 64>(ctx, a);
    return a.d_v == 128 ? launch_pu<64, 128>(ctx, a) : launch_pu<64, 64>(ctx, a);
}

}  // namespace lookat
