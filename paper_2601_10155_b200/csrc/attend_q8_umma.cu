// lookat_attend_q8 for prompts and pieces of them: many queries meet every token, so the products run on the
// 5th-generation tensor cores and the 8-bit numbers are widened once per 256 query rows.
//
//     S = Q n^K^T   (fp16 operands, exact)            y = S amax^K / R scale log2(e) + log2(amax^V) - M
//     w = 2^y       O += w n^V       l += w / amax^V       o = O / (R l)
// Scale and offset of y belong to a block of tokens (a page), so blocks of any size share one running exponent M per row;
// M follows the largest score lazily.  A row is one (query, query head) pair of a KV head: row = query * g + head, so a
// CTA's rows stand at neighbouring positions and share the tokens they see.
//   fp16 results take the weights in fp16 (2^-12 of each).  fp32 results take them as two fp16 numbers, whose second halves
// lie in the scores' second half of tensor memory, and move O out of tensor memory every 16 chunks: the tensor pipe cuts
// its sums off, and a chain of 16 chunks stays below 2^-20.
//
// A CTA works on two tiles of 128 rows against the same chunks of 64 tokens: while the softmax threads of one tile work,
// the tensor pipe has the other tile's products.  Roles (13 warps, one CTA per SM by tensor memory):
//   warps 0-3 / 4-7  softmax of tile 0 / 1: thread r owns row r of its tile = tensor-memory lane r;
//   warps 8-11  producers: the next chunk's keys and values from the pages to fp16 operand rows in shared memory (128-byte
//               swizzle), a chunk's loads issued before the wait for its buffer;
//   warp 12     one thread issues every MMA and commits them to mbarriers.
// Tensor memory (512 columns): per tile S (64; the weights overwrite it), O (d_v), Q (d_k / 2).
// Every mbarrier wait gives up after a bounded number of polls, raises the context's time-out flag and lets the CTA drain
// and free its tensor memory.
#include "q8.cuh"
#include "umma.cuh"

namespace lookat {

namespace {

constexpr int kPqRows = 128, kPqChunk = 64, kPqTiles = 2;
constexpr int kPqSoftmax = kPqTiles * kPqRows, kPqProducers = 128, kPqThreads = kPqSoftmax + kPqProducers + 32;
constexpr int kPqGroups = kPqChunk / 16;        // groups of 16 tokens: a page holds whole ones
constexpr int kPqFlush = 16;                    // chunks that O stays in tensor memory for fp32 results
constexpr float kPqSlack = 8.f;

struct PqMeta {                                 // of 16 tokens: y = s * ks + le - M, l += w * inv
    float ks, le, inv, pad;
};

template <int DK, int DV>
struct PqLayout {
    static constexpr int kKb = DK / 64, kNb = DV / 64;
    static constexpr int kKeys = kKb * kPqChunk * 128, kV = kNb * kPqChunk * 128;   // [64 dims each][token][128 B]
    static constexpr int kOffKeys = 0, kOffV = 2 * kKeys, kOffMeta = kOffV + 2 * kV;
    static constexpr int kOffBars = kOffMeta + 4 * kPqGroups * (int)sizeof(PqMeta);
    static constexpr int kBytes = kOffBars + 256;
    static constexpr int kColO = kPqTiles * kPqChunk, kColQ = kColO + kPqTiles * DV;
    static constexpr int kTmemCols = kColQ + kPqTiles * (DK / 2) <= 256 ? 256 : 512;
    static_assert(kColQ + kPqTiles * (DK / 2) <= 512, "tensor memory");
    // instruction descriptors: fp32 accumulate, fp16 operands, N >> 3 at bit 17, M >> 4 at bit 24; bit 16: B is MN-major
    static constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)(kPqChunk >> 3) << 17) | ((uint32_t)(kPqRows >> 4) << 24);
    static constexpr uint32_t kIdescO = (1u << 4) | (1u << 16) | ((uint32_t)(DV >> 3) << 17) | ((uint32_t)(kPqRows >> 4) << 24);
};

template <int FORMAT, int DK, int DV, bool FULL>      // FULL: fp32 results
__global__ void __launch_bounds__(kPqThreads, 1) attend_q8_umma_kernel(Q8AttendArgs a, int *__restrict__ timeout_flag)
{
    using Lay = PqLayout<DK, DV>;
    extern __shared__ __align__(1024) unsigned char pq_raw[];
    unsigned char *const sm = pq_raw;
    const uint32_t sm0 = um_smem(sm);
    PqMeta *const meta = reinterpret_cast<PqMeta *>(sm + Lay::kOffMeta);             // [chunk & 3][group]
    uint64_t *const bars = reinterpret_cast<uint64_t *>(sm + Lay::kOffBars);
    uint32_t *const tmem_slot = reinterpret_cast<uint32_t *>(bars + 24);
    // k_ready[buf], v_ready[buf]; per tile s_full[t][buf] (scores done), pv_done[t][buf] (value MMA done), p_ready[t];
    // meta_ready[chunk & 3]
    const uint32_t bar0 = um_smem(bars);
    const uint32_t bar_k = bar0, bar_v = bar0 + 16, bar_s = bar0 + 32, bar_pv = bar0 + 64, bar_p = bar0 + 96, bar_m = bar0 + 112;

    const Q8View &c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n_rows = a.g * a.L_q, h = blockIdx.y, b = blockIdx.z;
    const int row0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * (kPqTiles * kPqRows);  // longest first
    const int page = 1 << c.page_shift, cap = c.max_pages << c.page_shift;
    const int len_in = c.seq_lens[b], len = min(max(len_in, 0), cap);
    if (tid == 0 && len != len_in && h == 0) q8_report(c.status, kStatusBadPage);
    const int t_end = len - a.L_q + (min(row0 + kPqTiles * kPqRows, n_rows) - 1) / a.g + 1;      // tokens the CTA's last row sees
    const int n_chunks = (t_end + kPqChunk - 1) / kPqChunk;
    auto out_row = [&](int row) { return (((size_t)b * a.H_q + h * a.g + row % a.g) * a.L_q + row / a.g); };

    if (t_end <= 0) {                                          // nothing to see for any row here
        const int quads = DV * (a.out_fp16 ? 2 : 4) / 16;
        for (int i = tid; i < min(kPqTiles * kPqRows, n_rows - row0) * quads; i += kPqThreads)
            *reinterpret_cast<uint4 *>(static_cast<char *>(a.out) + (out_row(row0 + i / quads) * quads + i % quads) * 16) = make_uint4(0u, 0u, 0u, 0u);
        return;
    }

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            um_bar_init(bar_k + 8 * i, kPqProducers);
            um_bar_init(bar_v + 8 * i, kPqProducers);
            for (int t = 0; t < kPqTiles; ++t) {
                um_bar_init(bar_s + 16 * t + 8 * i, 1);
                um_bar_init(bar_pv + 16 * t + 8 * i, 1);
            }
            um_bar_init(bar_p + 8 * i, kPqRows);               // i as the tile index here
        }
        for (int i = 0; i < 4; ++i) um_bar_init(bar_m + 8 * i, kPqGroups);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(um_smem(tmem_slot)), "n"(Lay::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    um_fence_before();
    __syncthreads();
    um_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool dead = (sm0 & 1023u) != 0;                            // a wait ran out (or the base is misaligned): leave, free, return

    // ---- the query rows to tensor memory, the A operand of the scores: lane r = row r, two halves per column ----
    if (warp < kPqSoftmax / 32) {
        const int t = warp >> 2, row = min(row0 + t * kPqRows + (warp & 3) * 32 + lane, n_rows - 1);     // rows beyond the last repeat it
        const uint4 *src = reinterpret_cast<const uint4 *>(a.q + out_row(row) * DK);
#pragma unroll
        for (int part = 0; part < DK / 64; ++part) {
            uint32_t w[32];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint4 x = __ldg(src + part * 8 + i);
                w[4 * i] = x.x;
                w[4 * i + 1] = x.y;
                w[4 * i + 2] = x.z;
                w[4 * i + 3] = x.w;
            }
            um_st32(tmem + Lay::kColQ + t * (DK / 2) + part * 32 + ((uint32_t)((warp & 3) * 32) << 16), w);
        }
        um_wait_st();
    }
    um_fence_before();
    __syncthreads();
    um_fence_after();

    if (dead) {
        // misaligned shared-memory base: nothing runs
    } else if (warp == (kPqSoftmax + kPqProducers) / 32) {
        // =================== the MMA thread ===================
        if (lane == 0) {
            // descriptors: stride 1024 B, version 1, 128-byte swizzle in the high word; start address and leading offset in
            // the low word
            const uint32_t desc_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
            const uint32_t keys_lo = ((sm0 + Lay::kOffKeys) >> 4) | (1u << 16);                    // leading offset unused (16 B)
            const uint32_t v_lo = ((sm0 + Lay::kOffV) >> 4) | ((uint32_t)(kPqChunk * 128 / 16) << 16);   // between 64-column blocks
            auto score_mma = [&](int t, int ch) {
                const int buf = ch & 1;
                const uint32_t lo = keys_lo + buf * (Lay::kKeys >> 4), d = tmem + t * kPqChunk, q = tmem + Lay::kColQ + t * (DK / 2);
#pragma unroll
                for (int ks = 0; ks < DK / 16; ++ks) {
                    const uint32_t off = ((ks >> 2) * (kPqChunk * 128) + (ks & 3) * 32) >> 4;
                    if (ks == 0) um_mma_ts<false>(d, q + ks * 8, lo + off, desc_hi, Lay::kIdescS);
                    else um_mma_ts<true>(d, q + ks * 8, lo + off, desc_hi, Lay::kIdescS);
                }
                um_commit(bar_s + 16 * t + 8 * buf);
            };
            auto value_mma = [&](int t, int ch) {              // the weights lie over S(t): first halves, then (FULL) second ones
                const int buf = ch & 1;
                const uint32_t lo = v_lo + buf * (Lay::kV >> 4), pa = tmem + t * kPqChunk, d = tmem + Lay::kColO + t * DV;
                const bool first = FULL ? ch % kPqFlush == 0 : ch == 0;
#pragma unroll
                for (int part = 0; part < (FULL ? 2 : 1); ++part)
#pragma unroll
                    for (int kt = 0; kt < kPqChunk / 16; ++kt) {
                        if (part == 0 && kt == 0 && first) um_mma_ts<false>(d, pa, lo, desc_hi, Lay::kIdescO);
                        else um_mma_ts<true>(d, pa + part * 32 + kt * 8, lo + kt * (2048 >> 4), desc_hi, Lay::kIdescO);
                    }
                um_commit(bar_pv + 16 * t + 8 * buf);
            };
            // Per tile strictly scores(c) -> [softmax] -> value(c) -> scores(c + 1); the two tiles take turns.
            int next_qk[kPqTiles] = {0, 0}, next_pv[kPqTiles] = {0, 0};
            int polls = 0;
            while (next_pv[0] < n_chunks || next_pv[1] < n_chunks) {
                bool progress = false;
#pragma unroll
                for (int t = 0; t < kPqTiles; ++t) {
                    const int cp = next_pv[t];
                    if (cp < next_qk[t] && um_bar_test(bar_p + 8 * t, cp & 1) && um_bar_test(bar_v + 8 * (cp & 1), (cp >> 1) & 1)) {
                        um_fence_after();
                        value_mma(t, cp);
                        next_pv[t] = cp + 1;
                        progress = true;
                    }
                    const int cq = next_qk[t];
                    if (cq < n_chunks && next_pv[t] == cq && um_bar_test(bar_k + 8 * (cq & 1), (cq >> 1) & 1)) {
                        um_fence_after();
                        score_mma(t, cq);
                        next_qk[t] = cq + 1;
                        progress = true;
                    }
                }
                if (progress) polls = 0;
                else if (++polls > kUmPolls) { dead = true; break; }
            }
        }
    } else if (warp >= kPqSoftmax / 32) {
        // =================== producers ===================
        // A warp's item: 8 tokens (an octet; it lies in one page) by 64 dims; lane: token lane & 7, 16 dims lane >> 3.  The
        // stores of 8 lanes then go to 8 different columns of the swizzle.
        const int ptid = tid - kPqSoftmax, pw = ptid >> 5, tl = lane & 7, pl = lane >> 3;
        constexpr int kItemsK = 8 * Lay::kKb / 4, kItemsV = 8 * Lay::kNb / 4;       // per warp and chunk
        const int32_t *table = c.tables + (size_t)b * c.max_pages;
        auto entry_of = [&](int tok) { return tok < len ? __ldg(table + (tok >> c.page_shift)) : -1; };
        auto held = [&](int tok, int p) {                      // reports a bad entry
            const bool ok = p >= 0 && p < c.n_pages;
            if (tok < len && !ok) q8_report(c.status, kStatusBadPage);
            return ok;
        };
        // warp w takes the octets w and w + 4 (for every 64 dims): two table entries a chunk
        uint4 rk[kItemsK], rv[kItemsV];
        int ent[2], ent_meta;
        float am_k = 0.f, am_v = 0.f;
        bool meta_there = false;
        auto ask_entries = [&](int ch) {
#pragma unroll
            for (int i = 0; i < 2; ++i) ent[i] = entry_of(ch * kPqChunk + (pw + 4 * i) * 8);
            ent_meta = entry_of(ch * kPqChunk + (ptid & 3) * 16);
        };
        auto ask_rows = [&](int ch) {                          // zeros behind the row's last token and for bad entries
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int oct = pw + 4 * i, tok = ch * kPqChunk + oct * 8;
                const bool ok = held(tok, ent[i]) && tok + tl < len;
                const size_t row = ok ? ((size_t)ent[i] * c.H_kv + h) * page + ((tok + tl) & (page - 1)) : 0;
#pragma unroll
                for (int kb = 0; kb < Lay::kKb; ++kb)
                    rk[i * Lay::kKb + kb] = ok ? __ldg(reinterpret_cast<const uint4 *>(c.k + row * DK + kb * 64 + pl * 16)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int nb = 0; nb < Lay::kNb; ++nb)
                    rv[i * Lay::kNb + nb] = ok ? __ldg(reinterpret_cast<const uint4 *>(c.v + row * DV + nb * 64 + pl * 16)) : make_uint4(0u, 0u, 0u, 0u);
            }
            if (ptid < kPqGroups) {
                meta_there = ch * kPqChunk + ptid * 16 < len && ent_meta >= 0 && ent_meta < c.n_pages;
                const size_t block = meta_there ? (size_t)ent_meta * c.H_kv + h : 0;
                am_k = meta_there ? __ldg(c.k_amax + block) : 0.f;
                am_v = meta_there ? __ldg(c.v_amax + block) : 0.f;
            }
        };
        auto widen = [&](unsigned char *block, int oct, const uint4 &u) {          // 16 numbers as two 16-byte pieces of a row
            const int r = oct * 8 + tl;
            uint4 x, y;
            q8_pairs<FORMAT>(u.x, x.x, x.y);
            q8_pairs<FORMAT>(u.y, x.z, x.w);
            q8_pairs<FORMAT>(u.z, y.x, y.y);
            q8_pairs<FORMAT>(u.w, y.z, y.w);
            *reinterpret_cast<uint4 *>(block + r * 128 + (((2 * pl) ^ tl) << 4)) = x;
            *reinterpret_cast<uint4 *>(block + r * 128 + (((2 * pl + 1) ^ tl) << 4)) = y;
        };
        ask_entries(0);
        ask_rows(0);
        ask_entries(1);
        for (int ch = 0; ch < n_chunks; ++ch) {
            const int buf = ch & 1;
            bool ok = true;
            if (ch >= 2) {                                     // both tiles' scores of chunk ch - 2 are done with the buffer
#pragma unroll
                for (int t = 0; t < kPqTiles; ++t)
                    ok = um_group_wait<1, kPqProducers>(ptid == 0, bar_s + 16 * t + 8 * buf, ((ch - 2) >> 1) & 1) && ok;
                if (!ok) { dead = true; break; }
            }
            // (the softmax of chunk ch - 2 may still run, that of ch - 4 is over: its slot is free)
            if (ptid < kPqGroups) {
                PqMeta m;
                m.ks = am_k * (kQ8Unit<FORMAT> * a.scale_log2);
                m.le = !meta_there ? -INFINITY : am_v > 0.f ? log2f(am_v) : 0.f;   // (amax 0: the numbers are 0, the weights count)
                m.inv = am_v > 0.f ? 1.f / am_v : 1.f;
                m.pad = 0.f;
                meta[(ch & 3) * kPqGroups + ptid] = m;
                um_bar_arrive(bar_m + 8 * (ch & 3));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int kb = 0; kb < Lay::kKb; ++kb)
                    widen(sm + Lay::kOffKeys + buf * Lay::kKeys + kb * (kPqChunk * 128), pw + 4 * i, rk[i * Lay::kKb + kb]);
            um_fence_async_smem();                             // generic-proxy writes before the MMA's reads
            um_bar_arrive(bar_k + 8 * buf);
            if (ch >= 2) {                                     // ... and their value MMAs with the V buffer
#pragma unroll
                for (int t = 0; t < kPqTiles; ++t)
                    ok = um_group_wait<1, kPqProducers>(ptid == 0, bar_pv + 16 * t + 8 * buf, ((ch - 2) >> 1) & 1) && ok;
                if (!ok) { dead = true; break; }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int nb = 0; nb < Lay::kNb; ++nb)
                    widen(sm + Lay::kOffV + buf * Lay::kV + nb * (kPqChunk * 128), pw + 4 * i, rv[i * Lay::kNb + nb]);
            um_fence_async_smem();
            um_bar_arrive(bar_v + 8 * buf);
            ask_rows(ch + 1);                                  // in flight while the next buffer is waited for
            ask_entries(ch + 2);
        }
    } else {
        // =================== softmax: thread r owns row r of tile t ===================
        const int t = warp >> 2, rq = warp & 3, row = row0 + t * kPqRows + rq * 32 + lane;
        const bool on = row < n_rows;
        const int vis_end = len - a.L_q + (on ? row : n_rows - 1) / a.g + 1;       // tokens this row sees (may be <= 0)
        const uint32_t lane_base = (uint32_t)(rq * 32) << 16;
        const uint32_t tm_s = tmem + t * kPqChunk + lane_base, tm_o = tmem + Lay::kColO + t * DV + lane_base;
        float m_run = 0.f, l_run = 0.f, m_out = 0.f;           // M; m_out: M at the time of what lies in `out`
        bool set = false;                                      // the row has seen a token
        // O in tensor memory, and what was moved out before, times `mul`, to the result's row
        auto move_out = [&](float mul, bool again) {
            const float old = ex2_approx(m_out - m_run) * mul;
#pragma unroll 1
            for (int part = 0; part < DV / 32; ++part) {
                uint32_t o[32];
                um_ld32(o, tm_o + part * 32);
                um_wait_ld();
                float4 *dst = reinterpret_cast<float4 *>(static_cast<float *>(a.out) + (on ? out_row(row) * DV : 0) + part * 32);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (!on) break;
                    float4 x = make_float4(__uint_as_float(o[4 * i]) * mul, __uint_as_float(o[4 * i + 1]) * mul, __uint_as_float(o[4 * i + 2]) * mul,
                                           __uint_as_float(o[4 * i + 3]) * mul);
                    if (again) {
                        const float4 y = dst[i];
                        x = make_float4(fmaf(y.x, old, x.x), fmaf(y.y, old, x.y), fmaf(y.z, old, x.z), fmaf(y.w, old, x.w));
                    }
                    dst[i] = x;
                }
                __syncwarp();
            }
            m_out = set ? m_run : -1e30f;
        };
        for (int ch = 0; ch < n_chunks; ++ch) {
            const int buf = ch & 1, tok0 = ch * kPqChunk;
            const bool ok = um_bar_wait(bar_s + 16 * t + 8 * buf, (ch >> 1) & 1) && um_bar_wait(bar_m + 8 * (ch & 3), (ch >> 2) & 1);
            if (!__all_sync(0xffffffffu, ok)) { dead = true; break; }              // warp-uniform
            um_fence_after();
            // The tile's previous value MMA is complete: the commit behind s_full covers every MMA its thread issued before.
            if (FULL && ch > 0 && ch % kPqFlush == 0) move_out(1.f, ch > kPqFlush);     // the next value MMA starts from zero
            float y[kPqChunk];
            {
                uint32_t s0[32], s1[32];
                um_ld32(s0, tm_s);
                um_ld32(s1, tm_s + 32);
                um_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    y[i] = __uint_as_float(s0[i]);
                    y[32 + i] = __uint_as_float(s1[i]);
                }
            }
            float inv[kPqGroups], top = -INFINITY;
#pragma unroll
            for (int gr = 0; gr < kPqGroups; ++gr) {
                const PqMeta m = meta[(ch & 3) * kPqGroups + gr];
                const float off = m.le - m_run;
                inv[gr] = m.inv;
#pragma unroll
                for (int i = 0; i < 16; ++i) y[gr * 16 + i] = fmaf(y[gr * 16 + i], m.ks, off);
            }
            if (tok0 + kPqChunk > vis_end) {                   // the chunk crosses (or lies beyond) this row's causal limit
#pragma unroll
                for (int i = 0; i < kPqChunk; ++i)
                    if (tok0 + i >= vis_end) y[i] = -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < kPqChunk; ++i) top = fmaxf(top, y[i]);
            // M moves only when the scores run ahead of it by more than kPqSlack (base-2 units), or to the first score
            const bool move = top > kPqSlack || (!set && top > -INFINITY);
            float alpha = 1.f;
            if (__any_sync(0xffffffffu, move)) {
                const float d = move ? top : 0.f;
                alpha = set ? ex2_approx(-d) : 1.f;            // (no score so far: O and l are zero)
                set |= move;
                m_run += d;
#pragma unroll
                for (int i = 0; i < kPqChunk; ++i) y[i] -= d;
            }
            uint32_t pk[32], pl[FULL ? 32 : 1];
            float l = 0.f;
#pragma unroll
            for (int gr = 0; gr < kPqGroups; ++gr) {
                float sum = 0.f;
#pragma unroll
                for (int i = gr * 8; i < gr * 8 + 8; ++i) {
                    const float w0 = ex2_approx(y[2 * i]), w1 = ex2_approx(y[2 * i + 1]);
                    sum += w0 + w1;
                    const __half2 hi = __floats2half2_rn(w0, w1);
                    pk[i] = *reinterpret_cast<const uint32_t *>(&hi);
                    if constexpr (FULL) {
                        const float2 hf = __half22float2(hi);
                        const __half2 lo = __floats2half2_rn(w0 - hf.x, w1 - hf.y);
                        pl[i] = *reinterpret_cast<const uint32_t *>(&lo);
                    }
                }
                l = fmaf(sum, inv[gr], l);
            }
            l_run = fmaf(l_run, alpha, l);
            if (ch >= 1 && !(FULL && ch % kPqFlush == 0) && __any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
                for (int part = 0; part < DV / 32; ++part) {
                    uint32_t o[32];
                    um_ld32(o, tm_o + part * 32);
                    um_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                    um_st32(tm_o + part * 32, o);
                }
            }
            um_st32(tm_s, pk);
            if constexpr (FULL) um_st32(tm_s + 32, pl);
            um_wait_st();
            um_fence_before();
            um_bar_arrive(bar_p + 8 * t);
        }
        if (!dead && __all_sync(0xffffffffu, um_bar_wait(bar_pv + 16 * t + 8 * ((n_chunks - 1) & 1), ((n_chunks - 1) >> 1) & 1))) {
            um_fence_after();
            const float mul = l_run != 0.f ? kQ8Unit<FORMAT> / l_run : 0.f;
            if constexpr (FULL) {
                move_out(mul, n_chunks > kPqFlush);
            } else {
#pragma unroll 1
                for (int part = 0; part < DV / 32; ++part) {
                    uint32_t o[32];
                    um_ld32(o, tm_o + part * 32);
                    um_wait_ld();
                    uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__half *>(a.out) + (on ? out_row(row) * DV : 0) + part * 32);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (!on) break;
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const __half2 x = __floats2half2_rn(__uint_as_float(o[8 * i + 2 * j]) * mul, __uint_as_float(o[8 * i + 2 * j + 1]) * mul);
                            w[j] = *reinterpret_cast<const uint32_t *>(&x);
                        }
                        dst[i] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    __syncwarp();
                }
            }
        } else {
            dead = true;
        }
    }

    if (dead) atomicExch(timeout_flag, 1);
    um_fence_before();
    __syncthreads();
    if (warp == 0)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Lay::kTmemCols) : "memory");
}

template <int FORMAT, int DK, int DV, bool FULL>
lookat_status launch_pq(Ctx *ctx, const Q8AttendArgs &a)
{
    auto kern = attend_q8_umma_kernel<FORMAT, DK, DV, FULL>;
    constexpr int smem = PqLayout<DK, DV>::kBytes;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
        return check_launch(ctx, "attend_q8 (tcgen05 form): shared-memory opt-in");
    const int rows = a.g * a.L_q, per = kPqTiles * kPqRows;
    dim3 grid((unsigned)((rows + per - 1) / per), (unsigned)a.c.H_kv, (unsigned)a.B);
    kern<<<grid, kPqThreads, smem, ctx->stream>>>(a, ctx->timeout_flag);
    return check_launch(ctx, "attend_q8_umma_kernel");
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
    const bool dims = (a.c.d_k == 64 || a.c.d_k == 128) && (a.c.d_v == 64 || a.c.d_v == 128);
    return dims && (long long)a.g * a.L_q >= 64 && ctx->timeout_flag;
}

lookat_status launch_attend_q8_umma(Ctx *ctx, const Q8AttendArgs &a)
{
    if (a.format == LOOKAT_Q8_INT8) return a.out_fp16 ? launch_pq_dims<LOOKAT_Q8_INT8, false>(ctx, a) : launch_pq_dims<LOOKAT_Q8_INT8, true>(ctx, a);
    return a.out_fp16 ? launch_pq_dims<LOOKAT_Q8_E4M3, false>(ctx, a) : launch_pq_dims<LOOKAT_Q8_E4M3, true>(ctx, a);
}

}  // namespace lookat
