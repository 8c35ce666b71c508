// lookat_attend_q8 for prompts and pieces of them: many queries meet every token, so the products run on the
// 5th-generation tensor cores and the 8-bit numbers are widened once per 256 query rows.
//
//     S = Q n^K^T   (fp16 operands, exact)            y = S amax^K / R scale log2(e) + log2(amax^V) - M
//     w = 2^y       O += w n^V       l += w / amax^V       o = O / (R l)
// Scale and offset of y belong to a block of tokens (a page), so blocks of any size share one running exponent M per row;
// M follows the largest score lazily, kPqLift below it: the weights use fp16's whole range.  A row is one (query, query head) pair of a KV head: row = query * g + head, so a
// CTA's rows stand at neighbouring positions and share the tokens they see.
//   fp16 results take the weights in fp16 (2^-12 of each).  fp32 results take them as two fp16 numbers, whose second halves
// lie in the scores' second half of tensor memory, and move O out of tensor memory every 8 chunks: the tensor pipe cuts
// its sums off: over a prompt of 4096 tokens one chain's largest error was 2.3e-6, that of chains of 8 chunks 1.0e-6.
// (The fp32 variants spill 76 to 112 bytes at 128 registers, the fp16 ones nothing at 122.)
//
// A CTA works on two tiles of 128 rows against the same chunks of 64 tokens.  The scores of a tile have two buffers in
// tensor memory, so the tensor pipe makes the next chunk's while the softmax threads work on this one's.  Roles (16 warps,
// one CTA per SM by tensor memory):
//   warps 0-3 / 4-7  softmax of tile 0 / 1: thread r owns row r of its tile = tensor-memory lane r;
//   warps 8, 9 / 10, 11  producers of the keys / values: from 8-bit rows to fp16 operand rows (128-byte swizzle), both in
//               shared memory;
//   warps 12, 13  one thread each issues the MMAs of tile 0 / 1 and commits them to mbarriers;
//   warp 14     fetches 8-bit rows: a bulk copy per 16 tokens (a page holds whole ones) of K and of V, kPqRaw chunks ahead;
//   warp 15     the scales of each chunk's blocks.
// Tensor memory (512 columns): per tile S (2 x 64; the weights overwrite it) and O (d_v).  Q lies in shared memory.
// Measured (B200, e4m3, one row of 4096 queries over its 4096 tokens, 8 KV heads of 4 query heads, 128 dims): fp16
// results 180 us = 762 TFLOP/s, 46 % of a large bf16 matrix product; fp32 results 326 us.  What bounds it is the chain
// of a chunk: 256 rows of 64 tokens take about 2800 cycles, of which the tensor pipe works a third, the exponentials
// a third and the widening of the 8-bit rows the rest of the issue slots; see the counters' shares: tensor 36 %, issue
// 38 %.  A second CTA per SM has no tensor memory left.
//   Few rows over a long cache are cut along the tokens (blockIdx), every piece leaves O, M and l in the workspace and
// attend_q8_join_kernel joins them in order.
// Every mbarrier wait gives up after a bounded number of polls, raises the context's time-out flag and lets the CTA drain
// and free its tensor memory.
#include <type_traits>

#include "q8.cuh"
#include "umma.cuh"

namespace lookat {

namespace {

constexpr int kPqRows = 128, kPqChunk = 64, kPqTiles = 2, kPqBoth = kPqTiles * kPqRows;
constexpr int kPqSoftmax = kPqBoth, kPqProducers = 128, kPqOperand = kPqProducers / 2, kPqThreads = kPqSoftmax + kPqProducers + 32 * kPqTiles + 64;
constexpr int kPqGroups = kPqChunk / 16;        // groups of 16 tokens: a page holds whole ones
constexpr int kPqRaw = 3;                       // chunks of 8-bit rows in shared memory
constexpr int kPqFlush = 8;                     // chunks that O stays in tensor memory for fp32 results
// Least chunks of a piece of a row as long as its table.  The host knows the table's width alone: a shorter row has as many
// pieces of fewer chunks, down to one.  (Holding those to 8 chunks too, in the kernel, was slower: 40 queries over 256 tokens in
// a table for 32768, fp32 results, 19.3 us cut into single chunks and 23.8 as one piece, 17.9 in a table that fits; 200 queries
// over 1000 tokens 24.0 and 30.2.  The join is there in any case.)
constexpr int kPqMinPiece = 8;
// How far M lies below the largest score (base-2 units), and how far scores may run ahead of that before M moves: weights
// stay up to 2^(lift + slack) = 2^15.  With fp32 results the ones down to 2^-14 of the largest have 22 bits and what is dropped
// is 2^-36 of it; with fp16 results those down to 2^-21 have 11.  (The lift cancels in O / (R l).)  Moving M costs a pass
// over O in tensor memory: a prompt of 4096 tokens, fp16 results: slack 8 180 us, 6 or 4 183, 2 188 to 200; fp32 results: 321,
// 325, 326, 330.  The bits are worth that to fp32 results alone: a row of 4096 tokens whose first takes 96 % of the weight and
// has values near zero is 4e-4 off without a lift, 5e-6 with 7 and 1e-6 with 11.
template <bool FULL>
constexpr float kPqSlack = FULL ? 4.f : 8.f;
template <bool FULL>
constexpr float kPqLift = 15.f - kPqSlack<FULL>;

struct PqMeta {                                 // of 16 tokens: y = s * ks + le - M, l += w * inv
    float ks, le, inv, pad;
};

template <int DK, int DV>
struct PqLayout {
    static constexpr int kKb = DK / 64, kNb = DV / 64;
    static constexpr int kKeys = kKb * kPqChunk * 128, kV = kNb * kPqChunk * 128, kQ = kKb * kPqRows * 128;     // [64 dims each][row][128 B]
    static constexpr int kOffKeys = 0, kOffV = 2 * kKeys, kOffQ = kOffV + 2 * kV, kOffMeta = kOffQ + kPqTiles * kQ;
    static constexpr int kOffRaw = kOffMeta + 2 * kPqGroups * (int)sizeof(PqMeta);
    static constexpr int kRawK = kPqChunk * DK, kRaw = kRawK + kPqChunk * DV;
    static constexpr int kOffTurn = (kOffRaw + kPqRaw * kRaw + 127) / 128 * 128;     // 32 rows x 32 columns per softmax warp
    static constexpr int kOffThere = kOffTurn + kPqSoftmax / 32 * 4096;                        // int [stage][group]: the group's page is there
    static constexpr int kOffBars = kOffThere + 64;
    static constexpr int kBytes = kOffBars + 256;
    static constexpr int kColO = kPqTiles * 2 * kPqChunk;
    static_assert(kColO + kPqTiles * DV <= 512, "tensor memory");
    // instruction descriptors: fp32 accumulate, fp16 operands, N >> 3 at bit 17, M >> 4 at bit 24; bit 16: B is MN-major
    static constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)(kPqChunk >> 3) << 17) | ((uint32_t)(kPqRows >> 4) << 24);
    static constexpr uint32_t kIdescO = (1u << 4) | (1u << 16) | ((uint32_t)(DV >> 3) << 17) | ((uint32_t)(kPqRows >> 4) << 24);
    static constexpr int kPart = kPqBoth * (DV + 2);            // floats of a piece: O [row][DV], then M [row], l [row]
};

__device__ __forceinline__ float2 pq_fma2(float2 a, float b, float c)           // a * b + c, both halves in one instruction
{
    float2 d;
    asm("{\n.reg .b64 u, v, w, r;\nmov.b64 u, {%2, %3};\nmov.b64 v, {%4, %4};\nmov.b64 w, {%5, %5};\nfma.rn.f32x2 r, u, v, w;\nmov.b64 {%0, %1}, r;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float2 pq_add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n.reg .b64 u, v, r;\nmov.b64 u, {%2, %3};\nmov.b64 v, {%4, %5};\nadd.rn.f32x2 r, u, v;\nmov.b64 {%0, %1}, r;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float pq_max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Where row `row` of KV head h of batch row b stands in q and in the result.
__device__ __forceinline__ size_t pq_out_row(const Q8AttendArgs &a, int b, int h, int row)
{
    return ((size_t)b * a.H_q + h * a.g + row % a.g) * a.L_q + row / a.g;
}

template <int FORMAT, int DK, int DV, bool FULL>      // FULL: fp32 results
__global__ void __launch_bounds__(kPqThreads, 1)
attend_q8_umma_kernel(Q8AttendArgs a, int *__restrict__ timeout_flag, int n_super, int pieces, float *__restrict__ parts)
{
    using Lay = PqLayout<DK, DV>;
    extern __shared__ __align__(1024) unsigned char pq_raw[];
    unsigned char *const sm = pq_raw;
    const uint32_t sm0 = um_smem(sm);
    PqMeta *const meta = reinterpret_cast<PqMeta *>(sm + Lay::kOffMeta);             // [buf][group]
    uint64_t *const bars = reinterpret_cast<uint64_t *>(sm + Lay::kOffBars);
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(bars + 30);
    // k_ready[buf], v_ready[buf]; per tile s_full[t][buf] (scores done), pv_done[t][buf] (value MMA done), p_ready[t][buf]
    // (weights stored); meta_ready[buf]; k_free[buf], v_free[buf] (both tiles' MMAs are done with it);
    // raw_full[stage], raw_free[stage].  A phase of each can only end after every waiter of the one before has
    // moved on, so waits by parity are safe.
    const uint32_t bar0 = um_smem(bars);
    const uint32_t bar_k = bar0, bar_v = bar0 + 16, bar_s = bar0 + 32, bar_pv = bar0 + 64, bar_p = bar0 + 96, bar_m = bar0 + 128;
    const uint32_t bar_kf = bar0 + 144, bar_vf = bar0 + 160, bar_raw = bar0 + 176, bar_rawf = bar0 + 200;
    int *const there_s = reinterpret_cast<int *>(sm + Lay::kOffThere);

    if (pieces > 1) pdl_release();
    const Q8View &c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n_rows = a.g * a.L_q;
    // heads and batch rows first, then the pieces, then the row tiles, longest first: the last CTAs to start are short ones
    const int h = blockIdx.x % c.H_kv, b = blockIdx.x / c.H_kv % a.B, piece = blockIdx.x / (c.H_kv * a.B) % pieces;
    const int super = n_super - 1 - blockIdx.x / (c.H_kv * a.B * pieces), row0 = super * kPqBoth;
    const int tiles = n_rows - row0 > kPqRows ? 2 : 1;         // a second tile without rows has no work
    const int page = 1 << c.page_shift, cap = c.max_pages << c.page_shift;
    const int len_in = c.seq_lens[b], len = min(max(len_in, 0), cap);
    if (tid == 0 && len != len_in && h == 0) q8_report(c.status, kStatusBadPage);
    const int t_end = len - a.L_q + (min(row0 + kPqBoth, n_rows) - 1) / a.g + 1;     // tokens the CTA's last row sees
    const int all_chunks = max(0, (t_end + kPqChunk - 1) / kPqChunk), per_piece = (all_chunks + pieces - 1) / pieces;
    const int chunk0 = piece * per_piece, n_chunks = max(0, min(per_piece, all_chunks - chunk0));
    float *const part = parts + (pieces > 1 ? (((size_t)super * a.B + b) * c.H_kv + h) * pieces + piece : 0) * Lay::kPart;

    if (n_chunks == 0) {                                       // nothing to see for any row here
        if (pieces > 1) {
            for (int i = tid; i < kPqBoth; i += kPqThreads) part[kPqBoth * (DV + 1) + i] = 0.f;
            return;
        }
        const int quads = DV * (a.out_fp16 ? 2 : 4) / 16;
        for (int i = tid; i < min(kPqBoth, n_rows - row0) * quads; i += kPqThreads)
            *reinterpret_cast<uint4 *>(static_cast<char *>(a.out) + (pq_out_row(a, b, h, row0 + i / quads) * quads + i % quads) * 16) =
                make_uint4(0u, 0u, 0u, 0u);
        return;
    }

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            um_bar_init(bar_k + 8 * i, kPqOperand);
            um_bar_init(bar_v + 8 * i, kPqOperand);
            um_bar_init(bar_kf + 8 * i, tiles);
            um_bar_init(bar_vf + 8 * i, tiles);
            for (int t = 0; t < kPqTiles; ++t) {
                um_bar_init(bar_s + 16 * t + 8 * i, 1);
                um_bar_init(bar_pv + 16 * t + 8 * i, 1);
                um_bar_init(bar_p + 16 * t + 8 * i, kPqRows);
            }
        }
        for (int i = 0; i < 2; ++i) um_bar_init(bar_m + 8 * i, kPqGroups);
        for (int i = 0; i < kPqRaw; ++i) {
            um_bar_init(bar_raw + 8 * i, kPqGroups);
            um_bar_init(bar_rawf + 8 * i, kPqProducers / 32);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(um_smem(tmem_slot)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // ---- the query rows, A operand of the scores: row r of a tile, 64 dims each, 128-byte swizzle ----
    if (warp < kPqSoftmax / 32) {
        const int t = warp >> 2, r = (warp & 3) * 32 + lane, row = min(row0 + t * kPqRows + r, n_rows - 1);  // rows beyond the last repeat it
        const uint4 *src = reinterpret_cast<const uint4 *>(a.q + pq_out_row(a, b, h, row) * DK);
#pragma unroll
        for (int i = 0; i < DK / 8; ++i)
            *reinterpret_cast<uint4 *>(sm + Lay::kOffQ + t * Lay::kQ + (i >> 3) * (kPqRows * 128) + r * 128 + (((i & 7) ^ (r & 7)) << 4)) = __ldg(src + i);
        um_fence_async_smem();
    }
    um_fence_before();
    __syncthreads();
    um_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool dead = (sm0 & 1023u) != 0;                            // a wait ran out (or the base is misaligned): leave, free, return

    if (dead) {
        // misaligned shared-memory base: nothing runs
    } else if (warp == kPqThreads / 32 - 2) {
        // =================== the fetcher: a thread per group of 16 tokens ===================
        if (lane < kPqGroups) {
            const int32_t *table = c.tables + (size_t)b * c.max_pages;
            auto entry_of = [&](int ch) {
                const int tok = (chunk0 + ch) * kPqChunk + lane * 16;
                return ch < n_chunks && tok < len ? __ldg(table + (tok >> c.page_shift)) : -1;
            };
            int entry = entry_of(0), ch = 0;
            for (; ch < n_chunks; ++ch) {
                const int stage = ch % kPqRaw, tok = (chunk0 + ch) * kPqChunk + lane * 16;
                const bool there = entry >= 0 && entry < c.n_pages;
                if (tok < len && !there) q8_report(c.status, kStatusBadPage);
                const size_t row = there ? ((size_t)entry * c.H_kv + h) * page + (tok & (page - 1)) : 0;
                entry = entry_of(ch + 1);
                if (ch >= kPqRaw && !um_bar_wait(bar_rawf + 8 * stage, (ch / kPqRaw - 1) & 1)) { dead = true; break; }
                there_s[stage * kPqGroups + lane] = there;
                const uint32_t bar = bar_raw + 8 * stage, dst = sm0 + Lay::kOffRaw + stage * Lay::kRaw + lane * 16 * DK;
                if (!there) {
                    um_bar_arrive(bar);
                    continue;
                }
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(16 * (DK + DV)) : "memory");
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                             "l"(c.k + row * DK), "r"(16 * DK), "r"(bar)
                             : "memory");
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                                 sm0 + Lay::kOffRaw + stage * Lay::kRaw + Lay::kRawK + lane * 16 * DV),
                             "l"(c.v + row * DV), "r"(16 * DV), "r"(bar)
                             : "memory");
            }
            for (int i = max(0, ch - kPqRaw); i < ch; ++i) um_bar_wait(bar_raw + 8 * (i % kPqRaw), (i / kPqRaw) & 1);     // copies in flight end first
        }
    } else if (warp == kPqThreads / 32 - 1) {
        // =================== the scales: a thread per group of 16 tokens ===================
        if (lane < kPqGroups) {
            const int32_t *table = c.tables + (size_t)b * c.max_pages;
            auto entry_of = [&](int ch) {
                const int tok = (chunk0 + ch) * kPqChunk + lane * 16;
                return ch < n_chunks && tok < len ? __ldg(table + (tok >> c.page_shift)) : -1;
            };
            int entry = entry_of(0);
            for (int ch = 0; ch < n_chunks; ++ch) {
                const bool there = entry >= 0 && entry < c.n_pages;
                const size_t block = there ? (size_t)entry * c.H_kv + h : 0;
                const float ak = there ? __ldg(c.k_amax + block) : 0.f, av = there ? __ldg(c.v_amax + block) : 0.f;
                entry = entry_of(ch + 1);
                PqMeta m;
                m.ks = ak * (kQ8Unit<FORMAT> * a.scale_log2);
                m.le = !there ? -INFINITY : av > 0.f ? log2f(av) : kQ8ZeroExponent;
                m.inv = av > 0.f ? 1.f / av : kQ8ZeroInverse;
                m.pad = 0.f;
                // the slot's last reader was the softmax of chunk ch - 2, over when the value MMAs of that chunk are done (and
                // those of chunk ch, the barrier's next phase, wait for these scales)
                if (ch >= 2 && !um_bar_wait(bar_vf + 8 * (ch & 1), ((ch - 2) >> 1) & 1)) { dead = true; break; }
                meta[(ch & 1) * kPqGroups + lane] = m;
                um_bar_arrive(bar_m + 8 * (ch & 1));
            }
        }
    } else if (warp >= (kPqSoftmax + kPqProducers) / 32) {
        // =================== the MMA thread of a tile ===================
        const int t = warp - (kPqSoftmax + kPqProducers) / 32;
        if (t < tiles && um_elect()) {
            // descriptors: stride 1024 B, version 1, 128-byte swizzle in the high word; start address and leading offset in
            // the low word
            const uint32_t desc_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
            const uint32_t keys_lo = ((sm0 + Lay::kOffKeys) >> 4) | (1u << 16);                    // leading offset unused (16 B)
            const uint32_t q_lo = ((sm0 + Lay::kOffQ + t * Lay::kQ) >> 4) | (1u << 16);
            const uint32_t v_lo = ((sm0 + Lay::kOffV) >> 4) | ((uint32_t)(kPqChunk * 128 / 16) << 16);   // between 64-column blocks
            const uint32_t tm_s = tmem + t * 2 * kPqChunk, tm_o = tmem + Lay::kColO + t * DV;
            auto score_mma = [&](int ch) {                     // into the buffer that the weights of chunk ch - 2 lay in
                const int buf = ch & 1;
                if (!um_bar_wait(bar_k + 8 * buf, (ch >> 1) & 1)) return false;
                um_fence_after();
                const uint32_t lo = keys_lo + buf * (Lay::kKeys >> 4), d = tm_s + buf * kPqChunk;
#pragma unroll
                for (int ks = 0; ks < DK / 16; ++ks) {
                    const uint32_t qo = ((ks >> 2) * (kPqRows * 128) + (ks & 3) * 32) >> 4, ko = ((ks >> 2) * (kPqChunk * 128) + (ks & 3) * 32) >> 4;
                    if (ks == 0) um_mma_ss<false>(d, q_lo + qo, desc_hi, lo + ko, desc_hi, Lay::kIdescS);
                    else um_mma_ss<true>(d, q_lo + qo, desc_hi, lo + ko, desc_hi, Lay::kIdescS);
                }
                um_commit(bar_s + 16 * t + 8 * buf);
                um_commit(bar_kf + 8 * buf);
                return true;
            };
            auto value_mma = [&](int ch) {                     // weights over the scores: first halves, then (FULL) second ones
                const int buf = ch & 1;
                if (!um_bar_wait(bar_p + 16 * t + 8 * buf, (ch >> 1) & 1) || !um_bar_wait(bar_v + 8 * buf, (ch >> 1) & 1)) return false;
                um_fence_after();
                const uint32_t lo = v_lo + buf * (Lay::kV >> 4), pa = tm_s + buf * kPqChunk;
                const bool first = FULL ? ch % kPqFlush == 0 : ch == 0;
#pragma unroll
                for (int half = 0; half < (FULL ? 2 : 1); ++half)
#pragma unroll
                    for (int kt = 0; kt < kPqChunk / 16; ++kt) {
                        if (half == 0 && kt == 0 && first) um_mma_ts<false>(tm_o, pa, lo, desc_hi, Lay::kIdescO);
                        else um_mma_ts<true>(tm_o, pa + half * 32 + kt * 8, lo + kt * (2048 >> 4), desc_hi, Lay::kIdescO);
                    }
                um_commit(bar_pv + 16 * t + 8 * buf);
                um_commit(bar_vf + 8 * buf);
                return true;
            };
            bool ok = score_mma(0);
            if (n_chunks > 1) ok = ok && score_mma(1);
            for (int ch = 0; ok && ch < n_chunks; ++ch) ok = value_mma(ch) && (ch + 2 >= n_chunks || score_mma(ch + 2));
            dead = !ok;
        }
    } else if (warp >= kPqSoftmax / 32) {
        // =================== producers: two warps for the keys, two for the values ===================
        // An item: 8 tokens by 64 dims; lane: token lane >> 2, 16 dims lane & 3.  Odd tokens take the other 64 dims than even
        // ones, so that 8 lanes read 128 different bytes (of two rows) and store to 8 different columns of the swizzle.
        auto produce = [&](auto values) {
            constexpr bool V = decltype(values)::value;
            constexpr int D = V ? DV : DK, kBlocks = D / 64, kItems = 4 * kBlocks;   // per warp and chunk
            const int pw = (warp - kPqSoftmax / 32) & 1, tl = lane >> 2, pl = lane & 3;
            const uint32_t bar_full = V ? bar_v : bar_k, bar_free = V ? bar_vf : bar_kf;
            const unsigned char *const raw0 = sm + Lay::kOffRaw + (V ? Lay::kRawK : 0) + (pw * 32 + tl) * D + pl * 16;
            unsigned char *const rows0 = sm + (V ? Lay::kOffV : Lay::kOffKeys) + (pw * 32 + tl) * 128;
            for (int ch = 0; ch < n_chunks; ++ch) {
                const int buf = ch & 1, stage = ch % kPqRaw, tok = (chunk0 + ch) * kPqChunk + pw * 32 + tl;
                if (!__all_sync(0xffffffffu, um_bar_wait(bar_raw + 8 * stage, (ch / kPqRaw) & 1))) return false;
                const unsigned char *const raw = raw0 + stage * Lay::kRaw;
                uint4 u[kItems];
#pragma unroll
                for (int i = 0; i < kItems; ++i) {             // zeros behind the row's last token and for bad entries
                    const int octet = i / kBlocks, block = kBlocks == 2 ? (i & 1) ^ (tl & 1) : 0;
                    u[i] = *reinterpret_cast<const uint4 *>(raw + octet * 8 * D + block * 64);
                    if (tok + octet * 8 >= len || !there_s[stage * kPqGroups + pw * 2 + (octet >> 1)]) u[i] = make_uint4(0u, 0u, 0u, 0u);
                }
                __syncwarp();
                if (lane == 0) um_bar_arrive(bar_rawf + 8 * stage);
                if (ch >= 2 && !__all_sync(0xffffffffu, um_bar_wait(bar_free + 8 * buf, ((ch - 2) >> 1) & 1))) return false;
                unsigned char *const rows = rows0 + buf * (V ? Lay::kV : Lay::kKeys);
#pragma unroll
                for (int i = 0; i < kItems; ++i) {             // 16 numbers as two 16-byte pieces of a row
                    const int octet = i / kBlocks, block = kBlocks == 2 ? (i & 1) ^ (tl & 1) : 0;
                    unsigned char *const row = rows + block * (kPqChunk * 128) + octet * (8 * 128);
                    uint4 x, y;
                    q8_pairs<FORMAT>(u[i].x, x.x, x.y);
                    q8_pairs<FORMAT>(u[i].y, x.z, x.w);
                    q8_pairs<FORMAT>(u[i].z, y.x, y.y);
                    q8_pairs<FORMAT>(u[i].w, y.z, y.w);
                    *reinterpret_cast<uint4 *>(row + (((2 * pl) ^ tl) << 4)) = x;
                    *reinterpret_cast<uint4 *>(row + (((2 * pl + 1) ^ tl) << 4)) = y;
                }
                um_fence_async_smem();                         // generic-proxy writes before the MMA's reads
                um_bar_arrive(bar_full + 8 * buf);
            }
            return true;
        };
        const bool ok = warp < kPqSoftmax / 32 + 2 ? produce(std::false_type{}) : produce(std::true_type{});
        dead = !ok;
    } else if (warp >> 2 < tiles) {
        // =================== softmax: thread r owns row r of tile t ===================
        const int t = warp >> 2, rq = warp & 3, r = t * kPqRows + rq * 32 + lane, row = row0 + r;
        const bool on = row < n_rows;
        const int vis_end = len - a.L_q + (on ? row : n_rows - 1) / a.g + 1;       // tokens this row sees (may be <= 0)
        const uint32_t lane_base = (uint32_t)(rq * 32) << 16;
        const uint32_t tm_s = tmem + t * 2 * kPqChunk + lane_base, tm_o = tmem + Lay::kColO + t * DV + lane_base;
        float m_run = 0.f, l_run = 0.f, m_out = 0.f;           // M; m_out: M at the time of what was moved out of tensor memory
        bool set = false;                                      // the row has seen a token
        // O in tensor memory (a thread's row) times the row's `mul`, plus `old` times what is there if `again`, to rows in
        // global memory; 32 columns at a time through the warp's own shared memory, so that 8 lanes write 128 bytes of a row
        // (a lane writing its own row costs a line per 16 bytes: moving O out every 8 chunks took a third of the time)
        float4 *const turn = reinterpret_cast<float4 *>(sm + Lay::kOffTurn + warp * 4096);
        const size_t out_at = on ? pq_out_row(a, b, h, row) * DV : 0;
        float *const acc = pieces > 1 ? part + (size_t)r * DV : static_cast<float *>(a.out) + (FULL ? out_at : 0);
        auto move = [&](float mul, float old, bool again, bool halves) {
            const unsigned rows_on = __ballot_sync(0xffffffffu, on);
#pragma unroll 1
            for (int p = 0; p < DV / 32; ++p) {
                uint32_t o[32];
                um_ld32(o, tm_o + p * 32);
                um_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    turn[lane * 8 + (i ^ (lane & 7))] = make_float4(__uint_as_float(o[4 * i]) * mul, __uint_as_float(o[4 * i + 1]) * mul,
                                                                    __uint_as_float(o[4 * i + 2]) * mul, __uint_as_float(o[4 * i + 3]) * mul);
                __syncwarp();
                float4 y[8];                                   // all loads before the first store
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int rr = i * 4 + (lane >> 3);
                    const unsigned long long at = __shfl_sync(0xffffffffu, (unsigned long long)acc, rr);
                    y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (again && (rows_on >> rr & 1)) y[i] = *(reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(at) + p * 32) + (lane & 7));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int rr = i * 4 + (lane >> 3), quad = lane & 7;
                    float4 x = turn[rr * 8 + (quad ^ (rr & 7))];
                    const float k = __shfl_sync(0xffffffffu, old, rr);
                    const unsigned long long at = __shfl_sync(0xffffffffu, (unsigned long long)(halves ? out_at : (size_t)acc), rr);
                    if (!(rows_on >> rr & 1)) continue;
                    if (halves) {
                        *reinterpret_cast<uint2 *>(static_cast<__half *>(a.out) + at + p * 32 + quad * 4) = make_uint2(q8_half2(x.x, x.y), q8_half2(x.z, x.w));
                    } else {
                        if (again) x = make_float4(fmaf(y[i].x, k, x.x), fmaf(y[i].y, k, x.y), fmaf(y[i].z, k, x.z), fmaf(y[i].w, k, x.w));
                        *(reinterpret_cast<float4 *>(reinterpret_cast<float *>(at) + p * 32) + quad) = x;
                    }
                }
                __syncwarp();
            }
        };
        // ... together with what was moved out before
        auto move_out = [&](float mul, bool again) {
            move(mul, ex2_approx(m_out - m_run) * mul, again, false);
            m_out = set ? m_run : -1e30f;
        };
        auto values_done = [&](int ch) {                       // the tile's value MMAs up to chunk ch (warp-uniform)
            const bool ok = __all_sync(0xffffffffu, um_bar_wait(bar_pv + 16 * t + 8 * (ch & 1), (ch >> 1) & 1));
            um_fence_after();
            return ok;
        };
        for (int ch = 0; ch < n_chunks; ++ch) {
            const int buf = ch & 1, tok0 = (chunk0 + ch) * kPqChunk;
            const uint32_t tm_sb = tm_s + buf * kPqChunk;
            const bool ok = um_bar_wait(bar_s + 16 * t + 8 * buf, (ch >> 1) & 1) && um_bar_wait(bar_m + 8 * buf, (ch >> 1) & 1);
            if (!__all_sync(0xffffffffu, ok)) { dead = true; break; }              // warp-uniform
            um_fence_after();
            float2 y[kPqChunk / 2];
            {
                uint32_t s0[32], s1[32];
                um_ld32(s0, tm_sb);
                um_ld32(s1, tm_sb + 32);
                um_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    y[i] = make_float2(__uint_as_float(s0[2 * i]), __uint_as_float(s0[2 * i + 1]));
                    y[16 + i] = make_float2(__uint_as_float(s1[2 * i]), __uint_as_float(s1[2 * i + 1]));
                }
            }
            if (FULL && ch > 0 && ch % kPqFlush == 0) {        // the next value MMA starts from zero
                if (!values_done(ch - 1)) { dead = true; break; }
                move_out(1.f, ch > kPqFlush);
            }
            float inv[kPqGroups];
#pragma unroll
            for (int gr = 0; gr < kPqGroups; ++gr) {
                const PqMeta m = meta[buf * kPqGroups + gr];
                const float off = m.le - m_run;
                inv[gr] = m.inv;
#pragma unroll
                for (int i = gr * 8; i < gr * 8 + 8; ++i) y[i] = pq_fma2(y[i], m.ks, off);
            }
            if (tok0 + kPqChunk > vis_end) {                   // the chunk crosses (or lies beyond) this row's causal limit
#pragma unroll
                for (int i = 0; i < kPqChunk / 2; ++i) {
                    if (tok0 + 2 * i >= vis_end) y[i].x = -INFINITY;
                    if (tok0 + 2 * i + 1 >= vis_end) y[i].y = -INFINITY;
                }
            }
            float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < kPqChunk / 2; ++i) tops[i & 3] = pq_max3(tops[i & 3], y[i].x, y[i].y);
            const float top = fmaxf(pq_max3(tops[0], tops[1], tops[2]), tops[3]);
            // M moves only when the scores run ahead by more than kPqSlack, or to the first score
            const bool move = top > kPqLift<FULL> + kPqSlack<FULL> || (!set && top > -INFINITY);
            float alpha = 1.f;
            if (__any_sync(0xffffffffu, move)) {
                const float d = move ? top - kPqLift<FULL> : 0.f;
                alpha = set ? ex2_approx(-d) : 1.f;            // (no score so far: O and l are zero)
                set |= move;
                m_run += d;
                const float2 nd = make_float2(-d, -d);
#pragma unroll
                for (int i = 0; i < kPqChunk / 2; ++i) y[i] = pq_add2(y[i], nd);
            }
            uint32_t pk[32], pl[FULL ? 32 : 1];
            float l = 0.f;
#pragma unroll
            for (int gr = 0; gr < kPqGroups; ++gr) {
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int i = gr * 8; i < gr * 8 + 8; ++i) {
                    const float2 w = make_float2(ex2_approx(y[i].x), ex2_approx(y[i].y));
                    sum[i & 1] = pq_add2(sum[i & 1], w);
                    const __half2 hi = __floats2half2_rn(w.x, w.y);
                    pk[i] = *reinterpret_cast<const uint32_t *>(&hi);
                    if constexpr (FULL) {
                        const float2 hf = __half22float2(hi);
                        const __half2 lo = __floats2half2_rn(w.x - hf.x, w.y - hf.y);
                        pl[i] = *reinterpret_cast<const uint32_t *>(&lo);
                    }
                }
                l = fmaf((sum[0].x + sum[0].y) + (sum[1].x + sum[1].y), inv[gr], l);
            }
            l_run = fmaf(l_run, alpha, l);
            um_st32(tm_sb, pk);
            if constexpr (FULL) um_st32(tm_sb + 32, pl);
            if (ch >= 1 && !(FULL && ch % kPqFlush == 0) && __any_sync(0xffffffffu, alpha != 1.f)) {
                if (!values_done(ch - 1)) { dead = true; break; }
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
            um_bar_arrive(bar_p + 16 * t + 8 * buf);
        }
        if (!dead && values_done(n_chunks - 1)) {
            const float mul = pieces > 1 ? 1.f : l_run != 0.f ? kQ8Unit<FORMAT> / l_run : 0.f;
            if (FULL || pieces > 1) {
                move_out(mul, FULL && n_chunks > kPqFlush);
                if (pieces > 1) {
                    part[kPqBoth * DV + r] = m_run;
                    part[kPqBoth * (DV + 1) + r] = l_run;
                }
            } else {
                move(mul, 0.f, false, true);
            }
        } else {
            dead = true;
        }
    }

    if (dead) atomicExch(timeout_flag, 1);
    um_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

// The pieces of rows that were cut along the tokens, one warp per row; a piece without a token for the row has l = 0.
template <int FORMAT, int DV>
__global__ void __launch_bounds__(256) attend_q8_join_kernel(Q8AttendArgs a, int n_super, int pieces, const float *__restrict__ parts)
{
    constexpr int kPart = kPqBoth * (DV + 2), kEach = DV / 32;
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);           // [super][b][h][row of the tiles]
    const int r = (int)(item % kPqBoth), h = (int)(item / kPqBoth % a.c.H_kv), b = (int)(item / kPqBoth / a.c.H_kv % a.B);
    const int super = (int)(item / kPqBoth / a.c.H_kv / a.B), row = super * kPqBoth + r;
    if (super >= n_super || row >= a.g * a.L_q) return;
    const float *p0 = parts + (((size_t)super * a.B + b) * a.c.H_kv + h) * pieces * kPart;
    float top = -INFINITY, l = 0.f, o[kEach] = {};
    for (int p = 0; p < pieces; ++p) {
        const float lp = p0[(size_t)p * kPart + kPqBoth * (DV + 1) + r];
        if (lp != 0.f) top = fmaxf(top, p0[(size_t)p * kPart + kPqBoth * DV + r]);
    }
    for (int p = 0; p < pieces; ++p) {
        const float *q = p0 + (size_t)p * kPart;
        const float lp = q[kPqBoth * (DV + 1) + r];
        if (lp == 0.f) continue;                               // (nothing was written for it)
        const float k = ex2_approx(q[kPqBoth * DV + r] - top);
        l = fmaf(k, lp, l);
        if constexpr (kEach == 4) {
            const float4 x = *reinterpret_cast<const float4 *>(q + (size_t)r * DV + lane * 4);
            o[0] = fmaf(k, x.x, o[0]), o[1] = fmaf(k, x.y, o[1]), o[2] = fmaf(k, x.z, o[2]), o[3] = fmaf(k, x.w, o[3]);
        } else {
            const float2 x = *reinterpret_cast<const float2 *>(q + (size_t)r * DV + lane * 2);
            o[0] = fmaf(k, x.x, o[0]), o[1] = fmaf(k, x.y, o[1]);
        }
    }
    const float mul = l != 0.f ? kQ8Unit<FORMAT> / l : 0.f;
    const size_t at = pq_out_row(a, b, h, row) * DV + lane * kEach;
#pragma unroll
    for (int i = 0; i < kEach; i += 2) {
        if (a.out_fp16) *reinterpret_cast<uint32_t *>(static_cast<__half *>(a.out) + at + i) = q8_half2(o[i] * mul, o[i + 1] * mul);
        else *reinterpret_cast<float2 *>(static_cast<float *>(a.out) + at + i) = make_float2(o[i] * mul, o[i + 1] * mul);
    }
}

template <int FORMAT, int DK, int DV, bool FULL>
lookat_status launch_pq(Ctx *ctx, const Q8AttendArgs &a)
{
    using Lay = PqLayout<DK, DV>;
    auto kern = attend_q8_umma_kernel<FORMAT, DK, DV, FULL>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay::kBytes) != cudaSuccess)
        return check_launch(ctx, "attend_q8 (tcgen05 form): shared-memory opt-in");
    const int n_super = (a.g * a.L_q + kPqBoth - 1) / kPqBoth;
    const long long ctas = (long long)n_super * a.c.H_kv * a.B;
    // Few row tiles: cut the tokens so that one wave of CTAs fills the GPU (the host knows the longest length only)
    const long long chunks = (((long long)a.c.max_pages << a.c.page_shift) + kPqChunk - 1) / kPqChunk;
    int pieces = 1;
    if (ctas * 2 <= ctx->sm_count) {
        const long long fill = ctx->sm_count / ctas, most = chunks / kPqMinPiece;
        pieces = (int)(fill < most ? fill : most);
        if (pieces < 1) pieces = 1;
    }
    if (ctas > 0x7fffffffll / kPqBoth) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "attend_q8: too many queries for one call");
    float *parts = nullptr;
    if (pieces > 1) {
        lookat_status st = workspace(ctx, ctx->q8_pieces, (size_t)ctas * pieces * Lay::kPart * sizeof(float), false, "attend_q8");
        if (st != LOOKAT_OK) return st;
        parts = static_cast<float *>(ctx->q8_pieces.ptr);
    }
    kern<<<(unsigned)(ctas * pieces), kPqThreads, Lay::kBytes, ctx->stream>>>(a, ctx->timeout_flag, n_super, pieces, parts);
    lookat_status st = check_launch(ctx, "attend_q8_umma_kernel");
    if (st != LOOKAT_OK || pieces == 1) return st;
    launch_after(ctx, attend_q8_join_kernel<FORMAT, DV>, (unsigned)(ctas * kPqBoth / 8), 256, 0, a, n_super, pieces, parts);
    return check_launch(ctx, "attend_q8_join_kernel");
}

template <int FORMAT, bool FULL>
lookat_status launch_pq_dims(Ctx *ctx, const Q8AttendArgs &a)
{
    if (a.c.d_k == 128) return a.c.d_v == 128 ? launch_pq<FORMAT, 128, 128, FULL>(ctx, a) : launch_pq<FORMAT, 128, 64, FULL>(ctx, a);
    return a.c.d_v == 128 ? launch_pq<FORMAT, 64, 128, FULL>(ctx, a) : launch_pq<FORMAT, 64, 64, FULL>(ctx, a);
}

}  // namespace

bool attend_q8_umma_covers(const Ctx *ctx, const Q8AttendArgs &a)
{
    // Rows of a KV head (queries times heads of its group) from which on this form is the faster one; the streaming kernel
    // reads the cache once per 16 rows.  16 sequences of 4096 tokens, 32 rows per head: fp16 results 88 us there, 65 here, fp32
    // results 88 and 124; 48 rows per head: fp16 126 and 66, fp32 126 and 126; 64 rows: fp32 158 and 126.
    const bool dims = (a.c.d_k == 64 || a.c.d_k == 128) && (a.c.d_v == 64 || a.c.d_v == 128);
    return dims && (long long)a.g * a.L_q > (a.out_fp16 ? 16 : 32) && ctx->timeout_flag;
}

lookat_status launch_attend_q8_umma(Ctx *ctx, const Q8AttendArgs &a)
{
    if (a.format == LOOKAT_Q8_INT8) return a.out_fp16 ? launch_pq_dims<LOOKAT_Q8_INT8, false>(ctx, a) : launch_pq_dims<LOOKAT_Q8_INT8, true>(ctx, a);
    return a.out_fp16 ? launch_pq_dims<LOOKAT_Q8_E4M3, false>(ctx, a) : launch_pq_dims<LOOKAT_Q8_E4M3, true>(ctx, a);
}

}  // namespace lookat
