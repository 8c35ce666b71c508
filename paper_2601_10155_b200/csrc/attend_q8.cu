// lookat_attend_q8 for one token or a few per row: a kernel that streams the cache once.
//
// A column is one (query, query head) pair of a KV head; a unit is 8 or 16 columns of one (row, KV head).  Per unit the
// kernel takes, 16 tokens at a time,
//     s = (n^K . q) amax^K / R * scale             x = s log2(e)
//     w = 2^(x + e - M),   amax^V = 2^e f          (f in [1, 2); M follows the largest x + e, lazily)
//     O += (w f) n^V,   l += w 2^-e,               o = O / (R l)
// so that one running exponent M serves blocks of any size: w f is at most 2^9 where it matters and is a sum of two fp16
// numbers (22 bits), the 8-bit numbers are fp16 numbers as they are, and every sum is fp32.
//
// It is bound by HBM: (d_k + d_v) bytes per token and KV head against 4 d flops per column, so the products run on
// mma.sync.m16n8k16 (tokens or value dims are the rows, columns the 8 columns; the tensor pipe is under half used) and the
// design serves the loads.  Every lane copies by cp.async exactly the bytes that its own fragments are made of, into
// slots of its own: no barrier, no bank conflict and no shuffle between the copy and the product, and the ring
// (kAqStages tiles per warp) holds the bytes in flight without registers.
//   Scores: rows = 16 tokens, k = dims.  Lane (g, t) supplies rows g, g + 8; which dims stand behind its k indices is free
//     as long as q agrees: it takes the 16-byte pieces t, t + 4, .. of a token row, a product step per 4 bytes.
//   Values: rows = dims, k = 16 tokens.  Lane (g, t) supplies tokens 2t, 2t+1, 2t+8, 2t+9 and, with the dims permuted the
//     same way, the g-th piece of each row.
//   The weights go from the first product's accumulators to the second one's operand by movmatrix (8x8 transposes).
// Work: rows, units and 64-token tiles form one flat sequence, cut evenly among the resident CTAs on the device (the host
// does not know the lengths).  A unit cut between CTAs is joined by the CTA that finishes it last, in the order of the
// pieces, so the result does not depend on timing.
#include "q8.cuh"

namespace lookat {

namespace {

constexpr int kAqWarps = 4, kAqThreads = kAqWarps * 32;
constexpr int kAqTile = 16 * kAqWarps;          // tokens of a CTA's step
constexpr int kAqStages = 4;
constexpr int kAqMinChunk = 4;                  // steps per CTA below which a row is not cut
constexpr int kAqMaxParts = 128;                // pieces that a unit is cut into at most (one CTA joins them)
constexpr float kAqSlack = 8.f;                 // how far scores may run ahead of M (base-2 units)

__device__ __forceinline__ uint32_t aq_smem(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int BYTES>
__device__ __forceinline__ void aq_copy(uint32_t dst, const void *src)
{
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void aq_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t aq_transpose(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Four stored numbers as two pairs of fp16 numbers.  int8: with the sign bit flipped a byte u stands for u - 128, and the
// half 0x6400 + u is 1024 + u, so one exact subtraction gives n.  e4m3: the bits moved into an fp16's places (2^8 too
// small; kAqUnit makes up for it).
template <int FORMAT>
__device__ __forceinline__ void aq_pairs(uint32_t w, uint32_t &lo, uint32_t &hi)       // bytes 0,1 and 2,3
{
    if constexpr (FORMAT == LOOKAT_Q8_INT8) {
        const uint32_t u = w ^ 0x80808080u;
        const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
        const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), off), y = __hsub2(*reinterpret_cast<const __half2 *>(&b), off);
        lo = *reinterpret_cast<const uint32_t *>(&x);
        hi = *reinterpret_cast<const uint32_t *>(&y);
    } else {
        const uint32_t a = __byte_perm(w, 0u, 0x1404), b = __byte_perm(w, 0u, 0x3424);
        lo = ((a >> 1) & 0x3f803f80u) | (a & 0x80008000u);
        hi = ((b >> 1) & 0x3f803f80u) | (b & 0x80008000u);
    }
}
template <int FORMAT>
constexpr float kAqUnit = FORMAT == LOOKAT_Q8_INT8 ? 1.f / kQ8RangeInt8 : 256.f / kQ8RangeE4m3;   // value of a fp16 number per amax

template <int DP, int NT>
struct AqLayout {
    static constexpr int kJ = DP / 64;                          // 16-byte pieces per lane and token row of K
    static constexpr int kVBytes = DP == 64 ? 8 : 16;           // a lane's piece of a V row
    static constexpr int kVPieces = DP / 8 / kVBytes;           // ... and how many of them
    static constexpr int kTile = 32 * (2 * kJ * 16 + 4 * kVPieces * kVBytes);      // bytes of 16 tokens (padded to DP dims)
    static constexpr int kStage = kTile + 16;                   // + amax^K, amax^V
    static constexpr int kRing = kAqWarps * kAqStages * kStage;
    // the warps' results of a unit lie over the drained ring: O [warp][col][DP + 4], M and l [warp][col]
    static constexpr int kCols = 8 * NT, kPitch = DP + 4;
    static constexpr int kJoin = kAqWarps * kCols * (kPitch + 2) * 4;
    static constexpr int kBytes = kRing > kJoin ? kRing : kJoin;
    // a piece of a unit in global memory: M [col], l [col], O [col][DP]
    static constexpr int kPart = kCols * (DP + 2);              // floats
};

template <int FORMAT, int DP, int NT>
__global__ void __launch_bounds__(kAqThreads, DP == 256 ? 2 : 3)
attend_q8_kernel(Q8AttendArgs a, float *__restrict__ parts, unsigned *__restrict__ tickets)
{
    using Lay = AqLayout<DP, NT>;
    constexpr int KJ = Lay::kJ, VP = Lay::kVPieces, VB = Lay::kVBytes, MT = DP / 16;
    extern __shared__ __align__(16) unsigned char aq_raw[];
    __shared__ long long s_ll[kAqWarps + 2];
    __shared__ int s_i[kAqWarps + 2];
    const Q8View &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int page = 1 << c.page_shift, cap = c.max_pages << c.page_shift;
    const int n_cols = a.g * a.L_q, groups = (n_cols + Lay::kCols - 1) / Lay::kCols, units = c.H_kv * groups;

    // ---- this CTA's part of the flat sequence ----
    auto steps_of = [&](int b) {                                // an empty row has one step, which writes its zeros
        const int n = min(max(c.seq_lens[b], 0), cap);
        return max(1, (n + kAqTile - 1) / kAqTile);
    };
    long long chunk, pos, end, base;
    int b;
    {
        const int per = (a.B + kAqThreads - 1) / kAqThreads, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
        long long mine = 0;
        int longest = 0;
        for (int i = b0; i < b1; ++i) {
            const int len = c.seq_lens[i], n = steps_of(i);
            if (blockIdx.x == 0 && (len < 0 || len > cap)) q8_report(c.status, kStatusBadPage);
            mine += n;
            longest = max(longest, n);
        }
        long long incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
            longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
        }
        if (lane == 31) {
            s_ll[warp] = incl;
            s_i[warp] = longest;
        }
        __syncthreads();
        long long before = incl - mine, total = 0;
#pragma unroll
        for (int i = 0; i < kAqWarps; ++i) {
            if (i < warp) before += s_ll[i];
            total += s_ll[i];
            longest = max(longest, s_i[i]);
        }
        total *= units;
        chunk = (total + gridDim.x - 1) / gridDim.x;
        chunk = max(chunk, (long long)max(min(kAqMinChunk, longest), (longest + kAqMaxParts - 1) / kAqMaxParts));
        pos = chunk * blockIdx.x;
        end = min(pos + chunk, total);
        if (pos >= end) return;                                 // (the whole CTA)
        if (pos >= before * units && pos < (before + mine) * units) {
            int i = b0;
            for (; pos >= (before + steps_of(i)) * units; ++i) before += steps_of(i);
            s_i[kAqWarps] = i;
            s_ll[kAqWarps] = before * units;
        }
        __syncthreads();
        b = s_i[kAqWarps];
        base = s_ll[kAqWarps];
    }

    unsigned char *const ring = aq_raw + warp * (kAqStages * Lay::kStage);
    const uint32_t ring0 = aq_smem(ring);
    float *const sO = reinterpret_cast<float *>(aq_raw);                            // [warp][col][kPitch]
    float *const sM = sO + kAqWarps * Lay::kCols * Lay::kPitch, *const sL = sM + kAqWarps * Lay::kCols;
    const float k_unit = kAqUnit<FORMAT> * a.scale_log2;

    while (pos < end) {
        const int len = min(max(c.seq_lens[b], 0), cap), steps = max(1, (len + kAqTile - 1) / kAqTile);
        const int unit = (int)((pos - base) / steps), step0 = (int)((pos - base) % steps);
        const int n_steps = (int)min((long long)(steps - step0), end - pos);
        const int h = unit / groups, col0 = unit % groups * Lay::kCols;
        const int32_t *table = c.tables + (size_t)b * c.max_pages;

        // ---- q as the scores' second operand; the last token each of this lane's result columns sees ----
        uint32_t qf[NT][KJ * 4][2];
        int last[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int col = col0 + nt * 8 + g;
            const bool on = col < n_cols;
            const __half *qr = a.q + (((size_t)b * a.H_q + h * a.g + (on ? col % a.g : 0)) * a.L_q + (on ? col / a.g : 0)) * c.d_k;
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
                if (on && 64 * j + 16 * t < c.d_k) {
                    x = __ldg(reinterpret_cast<const uint4 *>(qr + 64 * j + 16 * t));
                    y = __ldg(reinterpret_cast<const uint4 *>(qr + 64 * j + 16 * t + 8));
                }
                qf[nt][4 * j][0] = x.x, qf[nt][4 * j][1] = x.y;
                qf[nt][4 * j + 1][0] = x.z, qf[nt][4 * j + 1][1] = x.w;
                qf[nt][4 * j + 2][0] = y.x, qf[nt][4 * j + 2][1] = y.y;
                qf[nt][4 * j + 3][0] = y.z, qf[nt][4 * j + 3][1] = y.w;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int cc = col0 + nt * 8 + 2 * t + k;
                last[nt][k] = cc < n_cols ? len - a.L_q + cc / a.g : -1;
            }
        }

        // ---- the ring: tile n of this warp holds tokens (step0 + n) * 64 + warp * 16 .. + 15 ----
        auto token_of = [&](int n) { return (step0 + n) * kAqTile + warp * 16; };
        auto page_of = [&](int n) {                             // -1: nothing there (beyond the row, or a bad entry)
            const int tok = token_of(n);
            if (n >= n_steps || tok >= len) return -1;
            const int p = __ldg(table + (tok >> c.page_shift));
            if (p < 0 || p >= c.n_pages) {
                q8_report(c.status, kStatusBadPage);
                return -1;
            }
            return p;
        };
        auto fetch = [&](int n, int pid) {
            const uint32_t s = ring0 + (n % kAqStages) * Lay::kStage;
            if (pid >= 0) {
                const size_t block = (size_t)pid * c.H_kv + h, row = block * page + (token_of(n) & (page - 1));
                const uint8_t *k = c.k + (row + g) * c.d_k + 16 * t;
#pragma unroll
                for (int j = 0; j < KJ; ++j)
                    if (DP == 64 ? 16 * t < c.d_k : 64 * j + 16 * t < c.d_k) {
                        aq_copy<16>(s + (2 * j) * 512 + lane * 16, k + 64 * j);
                        aq_copy<16>(s + (2 * j + 1) * 512 + lane * 16, k + 8 * c.d_k + 64 * j);
                    }
                const uint8_t *v = c.v + (row + 2 * t) * c.d_v + VB * g;
#pragma unroll
                for (int j = 0; j < VP; ++j)
                    if (VB * g + 128 * j < c.d_v) {
                        const uint32_t sv = s + 2 * KJ * 512 + j * 4 * (32 * VB) + lane * VB;
                        aq_copy<VB>(sv, v + 128 * j);
                        aq_copy<VB>(sv + 32 * VB, v + c.d_v + 128 * j);
                        aq_copy<VB>(sv + 2 * 32 * VB, v + 8 * c.d_v + 128 * j);
                        aq_copy<VB>(sv + 3 * 32 * VB, v + 9 * c.d_v + 128 * j);
                    }
                if (lane == 0) {
                    aq_copy<4>(s + Lay::kTile, c.k_amax + block);
                    aq_copy<4>(s + Lay::kTile + 4, c.v_amax + block);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        int pids[kAqStages];                                    // pages of the tiles in flight and of the next one
#pragma unroll
        for (int n = 0; n < kAqStages; ++n) pids[n] = page_of(n);
#pragma unroll
        for (int n = 0; n < kAqStages - 1; ++n) fetch(n, pids[n]);

        float o[NT][MT][4], m_ref[NT][2], l_sum[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
            m_ref[nt][0] = m_ref[nt][1] = -1e30f;
            l_sum[nt][0] = l_sum[nt][1] = 0.f;
        }

        for (int n = 0; n < n_steps; ++n) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kAqStages - 2) : "memory");
            __syncwarp();                                       // lane 0's amax is there; everyone is done with tile n - 1
            const int pid = pids[0];
            fetch(n + kAqStages - 1, pids[kAqStages - 1]);
#pragma unroll
            for (int i = 0; i < kAqStages - 1; ++i) pids[i] = pids[i + 1];
            pids[kAqStages - 1] = page_of(n + kAqStages);
            if (pid < 0) continue;
            const unsigned char *s = ring + (n % kAqStages) * Lay::kStage;
            const float2 amax = *reinterpret_cast<const float2 *>(s + Lay::kTile);
            const float ks = amax.x * k_unit;

            // scores of tokens g, g + 8 for columns 2t, 2t + 1; two chains of products per column group
            float sc[NT][4], sd[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
                sd[nt][0] = sd[nt][1] = sd[nt][2] = sd[nt][3] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
                if (64 * j + 16 * t < c.d_k) {
                    x = *reinterpret_cast<const uint4 *>(s + (2 * j) * 512 + lane * 16);
                    y = *reinterpret_cast<const uint4 *>(s + (2 * j + 1) * 512 + lane * 16);
                }
                const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t a0, a1, a2, a3;
                    aq_pairs<FORMAT>(xw[w], a0, a2);
                    aq_pairs<FORMAT>(yw[w], a1, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        aq_mma((w & 1) ? sd[nt] : sc[nt], a0, a1, a2, a3, qf[nt][4 * j + w][0], qf[nt][4 * j + w][1]);
                }
            }

            // weights; amax^V = 2^e f
            const int vb = __float_as_int(amax.y) >> 23;
            const float e = vb > 0 ? (float)(vb - 127) : 0.f;
            const float f = vb > 0 ? __int_as_float((__float_as_int(amax.y) & 0x7fffff) | 0x3f800000) : amax.y;
            const float inv_e = vb > 0 ? __int_as_float((254 - vb) << 23) : 1.f;
            const int tok = token_of(n) + g;
            uint32_t ph[NT][2], pl[NT][2];
            bool ahead = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = fmaf(sc[nt][i] + sd[nt][i], ks, e);
                    sc[nt][i] = tok + 8 * (i >> 1) <= last[nt][i & 1] ? x : -INFINITY;
                    ahead |= sc[nt][i] > m_ref[nt][i & 1] + kAqSlack;
                }
            if (__any_sync(0xffffffffu, ahead)) {               // M moves (seldom): the largest of the tile, per column
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float top = fmaxf(sc[nt][k], sc[nt][k + 2]);
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                        top = fmaxf(top, m_ref[nt][k]);
                        const float keep = ex2_approx(m_ref[nt][k] - top);
                        m_ref[nt][k] = top;
                        l_sum[nt][k] *= keep;
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            o[nt][i][k] *= keep;
                            o[nt][i][k + 2] *= keep;
                        }
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = ex2_approx(sc[nt][i] - m_ref[nt][i & 1]);
                    l_sum[nt][i & 1] = fmaf(w[i], inv_e, l_sum[nt][i & 1]);
                    w[i] *= f;
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {                   // tokens g and g + 8
                    const __half2 hi = __floats2half2_rn(w[2 * r], w[2 * r + 1]);
                    const float2 hf = __half22float2(hi);
                    const __half2 lo = __floats2half2_rn(w[2 * r] - hf.x, w[2 * r + 1] - hf.y);
                    ph[nt][r] = aq_transpose(*reinterpret_cast<const uint32_t *>(&hi));
                    pl[nt][r] = aq_transpose(*reinterpret_cast<const uint32_t *>(&lo));
                }
            }

            // values: product steps of two dims per lane
#pragma unroll
            for (int j = 0; j < VP; ++j) {
                uint32_t r[4][VB / 4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const unsigned char *sv = s + 2 * KJ * 512 + (j * 4 + k) * (32 * VB) + lane * VB;
                    if constexpr (VB == 16) {
                        uint4 u = make_uint4(0u, 0u, 0u, 0u);
                        if (VB * g + 128 * j < c.d_v) u = *reinterpret_cast<const uint4 *>(sv);
                        r[k][0] = u.x, r[k][1] = u.y, r[k][2] = u.z, r[k][3] = u.w;
                    } else {
                        uint2 u = make_uint2(0u, 0u);
                        if (VB * g + 128 * j < c.d_v) u = *reinterpret_cast<const uint2 *>(sv);
                        r[k][0] = u.x, r[k][1] = u.y;
                    }
                }
#pragma unroll
                for (int w = 0; w < VB / 4; ++w) {
                    // bytes of two tokens side by side: dims 4w, 4w + 1 and dims 4w + 2, 4w + 3
                    uint32_t x0, x1, x2, x3, y0, y1, y2, y3;
                    aq_pairs<FORMAT>(__byte_perm(r[0][w], r[1][w], 0x5140), x0, x1);        // tokens 2t, 2t + 1
                    aq_pairs<FORMAT>(__byte_perm(r[0][w], r[1][w], 0x7362), x2, x3);
                    aq_pairs<FORMAT>(__byte_perm(r[2][w], r[3][w], 0x5140), y0, y1);        // tokens 2t + 8, 2t + 9
                    aq_pairs<FORMAT>(__byte_perm(r[2][w], r[3][w], 0x7362), y2, y3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            // the tile's own sum first, from zero, then onto O: the tensor pipe cuts its sums off
                            float acc[4] = {0.f, 0.f, 0.f, 0.f};
                            const uint32_t a0 = half ? x2 : x0, a1 = half ? x3 : x1, a2 = half ? y2 : y0, a3 = half ? y3 : y1;
                            aq_mma(acc, a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
                            aq_mma(acc, a0, a1, a2, a3, ph[nt][0], ph[nt][1]);
                            float (&dst)[4] = o[nt][(j * (VB / 4) + w) * 2 + half];
#pragma unroll
                            for (int i = 0; i < 4; ++i) dst[i] += acc[i];
                        }
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");

        // ---- the four warps' results, then the pieces of the unit ----
        __syncthreads();                                        // the ring is drained
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float l = l_sum[nt][k];
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
                const int col = nt * 8 + 2 * t + k;
                if (g == 0) {
                    sM[warp * Lay::kCols + col] = m_ref[nt][k];
                    sL[warp * Lay::kCols + col] = l;
                }
                if (col0 + col < n_cols)
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        // step i of piece j: dims 128 j + VB g + 2 (i % (VB / 2)), + 1
                        const int dim = i / (VB / 2) * 128 + VB * g + 2 * (i % (VB / 2));
                        *reinterpret_cast<float2 *>(sO + (warp * Lay::kCols + col) * Lay::kPitch + dim) = make_float2(o[nt][i][k], o[nt][i][k + 2]);
                    }
            }
        __syncthreads();
        const long long u0 = base + (long long)unit * steps;
        const int first = (int)(u0 / chunk), pieces = (int)((u0 + steps - 1) / chunk) - first + 1, me = blockIdx.x;
        const int n_here = min(Lay::kCols, n_cols - col0);
        float *const part = parts + (size_t)(2 * me + (me == first)) * Lay::kPart;
        auto store = [&](int col, int dim, float x) {           // o = O / (R l)
            const int cc = col0 + col;
            const size_t at = (((size_t)b * a.H_q + h * a.g + cc % a.g) * a.L_q + cc / a.g) * c.d_v + dim;
            if (a.out_fp16) static_cast<__half *>(a.out)[at] = __float2half_rn(x);
            else static_cast<float *>(a.out)[at] = x;
        };
        for (int i = tid; i < n_here * c.d_v; i += kAqThreads) {
            const int col = i / c.d_v, dim = i % c.d_v;
            float top = sM[col], l = 0.f, x = 0.f;
#pragma unroll
            for (int w = 1; w < kAqWarps; ++w) top = fmaxf(top, sM[w * Lay::kCols + col]);
#pragma unroll
            for (int w = 0; w < kAqWarps; ++w) {
                const float k = ex2_approx(sM[w * Lay::kCols + col] - top);
                l = fmaf(k, sL[w * Lay::kCols + col], l);
                x = fmaf(k, sO[(w * Lay::kCols + col) * Lay::kPitch + dim], x);
            }
            if (pieces == 1) {
                store(col, dim, l != 0.f ? x * kAqUnit<FORMAT> / l : 0.f);
            } else {
                if (dim == 0) {
                    __stcg(part + col, top);
                    __stcg(part + Lay::kCols + col, l);
                }
                __stcg(part + 2 * Lay::kCols + col * DP + dim, x);
            }
        }
        if (pieces > 1) {
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const unsigned seen = atomicAdd(tickets + first, 1u);
                s_i[kAqWarps + 1] = seen == (unsigned)pieces - 1;
                if (seen == (unsigned)pieces - 1) tickets[first] = 0u;      // all pieces are in: ready for the next launch
            }
            __syncthreads();
            if (s_i[kAqWarps + 1]) {
                __threadfence();
                for (int i = tid; i < n_here * c.d_v; i += kAqThreads) {
                    const int col = i / c.d_v, dim = i % c.d_v;
                    float top = -1e30f, l = 0.f, x = 0.f;
                    for (int p = 0; p < pieces; ++p) {
                        const float *q = parts + (size_t)(p == 0 ? 2 * first + 1 : 2 * (first + p)) * Lay::kPart;
                        const float m = __ldcg(q + col), lp = __ldcg(q + Lay::kCols + col), xp = __ldcg(q + 2 * Lay::kCols + col * DP + dim);
                        const float now = fmaxf(top, m), k0 = ex2_approx(top - now), k1 = ex2_approx(m - now);
                        top = now;
                        l = l * k0 + lp * k1;
                        x = x * k0 + xp * k1;
                    }
                    store(col, dim, l != 0.f ? x * kAqUnit<FORMAT> / l : 0.f);
                }
            }
        }
        __syncthreads();                                        // the ring's memory may be written again

        pos += n_steps;
        if (pos == base + (long long)units * steps) {
            base = pos;
            ++b;
        }
    }
}

template <int FORMAT, int DP, int NT>
lookat_status launch_aq(Ctx *ctx, const Q8AttendArgs &a)
{
    using Lay = AqLayout<DP, NT>;
    auto kern = attend_q8_kernel<FORMAT, DP, NT>;
    static int resident[64];                                    // CTAs per SM, by device (0: not asked yet)
    int &per_sm = resident[ctx->device & 63];
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay::kBytes) != cudaSuccess)
        return check_launch(ctx, "attend_q8: shared-memory opt-in");
    if (!per_sm) {
        int n = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, kAqThreads, Lay::kBytes) != cudaSuccess || n < 1)
            return check_launch(ctx, "attend_q8: occupancy");
        per_sm = n;
    }
    const long long n_cols = (long long)a.g * a.L_q;
    const long long most = (long long)a.B * a.c.H_kv * ((n_cols + Lay::kCols - 1) / Lay::kCols) *
                           ((((long long)a.c.max_pages << a.c.page_shift) + kAqTile - 1) / kAqTile);
    const long long full = (long long)ctx->sm_count * per_sm;
    const unsigned grid = (unsigned)(most < full ? most : full);
    lookat_status st = workspace(ctx, ctx->q8_partials, (size_t)full * 2 * Lay::kPart * sizeof(float), false, "attend_q8");
    if (st == LOOKAT_OK) st = workspace(ctx, ctx->q8_tickets, (size_t)ctx->sm_count * 16 * sizeof(unsigned), true, "attend_q8");
    if (st != LOOKAT_OK) return st;
    kern<<<grid, kAqThreads, Lay::kBytes, ctx->stream>>>(a, static_cast<float *>(ctx->q8_partials.ptr), static_cast<unsigned *>(ctx->q8_tickets.ptr));
    return check_launch(ctx, "attend_q8_kernel");
}

template <int FORMAT>
lookat_status launch_aq_dims(Ctx *ctx, const Q8AttendArgs &a)
{
    const int d = a.c.d_k > a.c.d_v ? a.c.d_k : a.c.d_v;
    const bool wide = (long long)a.g * a.L_q > 8;
    if (d <= 64) return wide ? launch_aq<FORMAT, 64, 2>(ctx, a) : launch_aq<FORMAT, 64, 1>(ctx, a);
    if (d <= 128) return wide ? launch_aq<FORMAT, 128, 2>(ctx, a) : launch_aq<FORMAT, 128, 1>(ctx, a);
    return launch_aq<FORMAT, 256, 1>(ctx, a);
}

}  // namespace

lookat_status launch_attend_q8(Ctx *ctx, const Q8AttendArgs &a)
{
    if ((long long)a.H_q * a.L_q > (1ll << 30)) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "attend_q8: more than 2^30 queries per row");
    return a.format == LOOKAT_Q8_INT8 ? launch_aq_dims<LOOKAT_Q8_INT8>(ctx, a) : launch_aq_dims<LOOKAT_Q8_E4M3>(ctx, a);
}

}  // namespace lookat
