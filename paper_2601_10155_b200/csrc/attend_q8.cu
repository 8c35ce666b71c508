// lookat_attend_q8 for one token or a few per row: a kernel that streams the cache once.
//
// A column is one (query, query head) pair of a KV head; a unit is 8 or 16 columns of one (row, KV head).  Per unit the
// kernel takes, 16 tokens at a time,
//     s = (n^K . q) amax^K / R * scale             x = s log2(e)
//     w = 2^(x + e - M),   amax^V = 2^e f          (f in [1, 2); M follows the largest x + e, lazily)
//     O += (w f) n^V,   l += w 2^-e,               o = O / (R l)
// so that one running exponent M serves blocks of any size.  The 8-bit numbers are fp16 numbers as they are, and every sum is
// fp32.  w f is a sum of two fp16 numbers and uses their whole range: M lies kAqLift below the largest x + e, so the
// largest weight is 2^10 to 2^14, those down to 2^-13 of it have 22 bits, and what is dropped is 2^-35 of it.  (The lift
// cancels in O / (R l).  Without it, a row of 4096 tokens whose first takes 96 % of the weight and has values near zero was
// 1.5e-4 off.)
//
// It is bound by HBM: (d_k + d_v) bytes per token and KV head against 4 d flops per column, so the products run on
// mma.sync.m16n8k16 (tokens or value dims are the rows, columns the 8 columns; the tensor pipe is under half used) and the
// design serves the loads.  Every warp has a ring of its own (kAqStages tiles), which holds the bytes in flight without
// registers: its lanes copy linearly by cp.async into a permuted order (aq_piece), so that the reads of the fragments meet no
// bank conflict and need no shuffle.  A lane reads pieces that other lanes of its warp copied: every lane waits for its own
// copies (wait_group) and the __syncwarp behind that makes them visible to the others; no barrier of the CTA is needed.
//   Scores: rows = 16 tokens, k = dims.  Lane (g, t) supplies rows g, g + 8; which dims stand behind its k indices is free
//     as long as q agrees: it takes the 16-byte pieces t, t + 4, .. of a token row, a product step per 4 bytes.
//   Values: rows = dims, k = 16 tokens.  Lane (g, t) supplies tokens 2t, 2t+1, 2t+8, 2t+9 and, with the dims permuted the
//     same way, the g-th piece of each row.
//   The weights go from the first product's accumulators to the second one's operand by movmatrix (8x8 transposes).
// Measured (B200): 16 rows of 32768 int8 tokens, 8 KV heads of 4 query heads, 128 + 128 dims, 1.07 GB of cache: 190 us =
// 5.65 TB/s, 88 % of a large copy's rate (a kernel of the copies alone: 180 us); 226-234 us in a long run under the power
// cap, where the 512 warp instructions per 16 tokens (issue slots 59 % full) bound it.  One row of GPT-2's 12 heads over
// 128 tokens: 5.4 us.
// Work: rows, units and 64-token tiles form one flat sequence, cut evenly among the resident CTAs on the device (the host
// does not know the lengths).  A unit cut between CTAs is joined by the CTA that finishes it last, in the order of the
// pieces, so the result does not depend on timing.
#include "q8.cuh"

namespace lookat {

namespace {

constexpr int kAqWarps = 4, kAqThreads = kAqWarps * 32;
constexpr int kAqTile = 16 * kAqWarps;          // tokens of a CTA's step
constexpr int kAqStages = 3;                    // tiles in a warp's ring
// Cutting a unit costs about 5 us (pieces through global memory, a counter, the join), a step of a lone CTA 0.7 us: where no unit
// has more than kAqWhole steps, a CTA's part is at least the longest unit, so that units of one length stay whole and others
// are cut once at most (rows of 200 to 900 tokens, 8 KV heads: 16.3 us, 24.1 with the rule at 16 steps; rows of 500
// tokens, 16 columns: 19 us whole, 23 cut); else a part has at least kAqMinChunk steps and a cell (one row of
// 1024 tokens, 12 heads: 9.5 us with 3, 10.0 with 4, 11.3 with 6, 14.4 whole).  What joining a unit costs weighs as much as
// kAqJoinCells steps when the work is cut (23 rows of up to 8189 tokens, 16 columns: 78.5 us with 1, 65 with 3, 64 with 4,
// 63 with 6; rows of 32768 tokens, 4 columns: 173, 171, 169, 169; rows of up to 4000 tokens, 8 columns of 64 dims: 15.9,
// 15.5, 14.8, 16.2).
constexpr int kAqWhole = 10, kAqMinChunk = 3;
constexpr int kAqJoinCells = 4;
constexpr int kAqMaxParts = 128;                // pieces that a unit is cut into at most (one CTA joins them)
// How far M lies below the largest score (base-2 units), and how far scores may run ahead of that before M moves: f is below
// 2, so w f stays below 2^(lift + slack + 1) = 2^15.  A smaller slack leaves more bits to small weights and moves M more
// often: 23 ragged rows with 4 drafts 65.5 us with a slack of 4, 6 or 8, 66.8 with 2; one column: no difference.
constexpr float kAqLift = 10.f, kAqSlack = 4.f;

__device__ __forceinline__ uint32_t aq_smem(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int BYTES>
__device__ __forceinline__ void aq_copy(uint32_t dst, const void *src)
{
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
// the same, or zeros
template <int BYTES>
__device__ __forceinline__ void aq_copy_if(uint32_t dst, const void *src, bool there)
{
    const int n = there ? BYTES : 0;
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(n) : "memory");
}
__device__ __forceinline__ void aq_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void aq_mma_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t aq_transpose(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Where the 16-byte pieces of a tile's rows lie: a row of 64, 128 or 256 bytes after the other as in the cache, the pieces
// of row r permuted by XOR with aq_turn(r) within their 128 bytes.  The copies are then linear (512 consecutive bytes per
// warp instruction: reading every other row instead cost a quarter of the bandwidth), and each quarter-warp's reads below
// touch eight different 16-byte columns: rows r, r + 1 with pieces 0..3 (scores) since the turns of 2i and 2i + 1 differ in
// bit 2; rows 0, 2, 4, 6 (or 1, 3, 5, 7) with pieces 2i, 2i + 1 (values) since their turns differ above bit 0.
__device__ __forceinline__ constexpr int aq_turn(int r) { return (r & 6) ^ ((r & 1) << 2); }
template <int DP>
__device__ __forceinline__ int aq_piece(int r, int p)           // byte offset of piece p of row r
{
    if constexpr (DP == 64) return ((r >> 1) * 8 + (p ^ aq_turn(r))) * 16;
    else return (r * (DP / 16) + (p & ~7) + ((p ^ aq_turn(r)) & 7)) * 16;
}

template <int DP, int NT, bool PACK>
struct AqLayout {
    static constexpr int kJ = DP / 64;                          // 16-byte pieces of a K row per lane
    static constexpr int kVBytes = DP == 64 ? 8 : 16;           // a lane's piece of a V row
    static constexpr int kVPieces = DP / 8 / kVBytes;           // ... and how many of them
    static constexpr int kOffV = 16 * DP, kTile = 2 * kOffV;    // bytes of 16 tokens (padded to DP dims): K, V
    static constexpr int kStage = kTile + 16;                   // + amax^K, amax^V, whether the tile is there
    static constexpr int kRing = kAqWarps * kAqStages * kStage;
    // the warps' results of 8 (or 4) columns at a time: O [col][DP] of each warp in the stage of its last tile, whose next
    // copy comes after the join; M, l and the factor of M [warp][col], then M and l of the CTA
    static constexpr int kCols = PACK ? 4 : 8 * NT, kJoinCols = PACK ? 4 : 8;
    static_assert(kJoinCols * DP * 4 <= kTile, "O of a warp lies in a stage of the ring");
    static constexpr int kJoin = (kAqWarps * kJoinCols * 3 + 2 * kCols) * 4;
    // when a CTA joins the pieces of a unit, their factors [col][kAqMaxParts] lie over the drained ring
    static_assert(kRing >= kCols * kAqMaxParts * 4, "factors of the pieces");
    static constexpr int kBytes = kRing + kJoin;
    // a piece of a unit in global memory: M [col], l [col], O [col][DP]
    static constexpr int kPart = kCols * (DP + 2);              // floats
};

// A place in the flat sequence of rows, units and steps.  A unit takes steps + kAqJoinCells cells of it (what precedes its
// first step stands for the join); an empty row takes none.
struct AqCursor {
    int b, unit, step, steps, len;
    int at;                                                     // cells from the start of the CTA's part
    __device__ __forceinline__ void row(const Q8View &c, int cap)
    {
        len = min(max(__ldg(c.seq_lens + b), 0), cap);
        steps = (len + kAqTile - 1) / kAqTile;
    }
    __device__ __forceinline__ void advance(const Q8View &c, int B, int cap, int units, int end)
    {
        ++at;
        if (++step < steps) return;
        step = 0;
        at += kAqJoinCells;
        if (at < end && ++unit == units) {
            unit = 0;
            do {
                ++b;
                row(c, cap);
            } while (steps == 0);                               // (a later row has steps: at < end)
        }
    }
};

// EXACT: d_k = d_v = DP
template <int FORMAT, int DP, int NT, bool PACK, bool EXACT>
__global__ void __launch_bounds__(kAqThreads, DP == 256 ? 2 : NT == 2 ? 3 : 4)
attend_q8_kernel(Q8AttendArgs a, float *__restrict__ parts, unsigned *__restrict__ tickets)
{
    using Lay = AqLayout<DP, NT, PACK>;
    constexpr int KJ = Lay::kJ, VP = Lay::kVPieces, VB = Lay::kVBytes, MT = DP / 16;
    extern __shared__ __align__(16) unsigned char aq_raw[];
    __shared__ long long s_ll[kAqWarps + 2];
    __shared__ int s_i[kAqWarps + 2];
    const Q8View &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int page = 1 << c.page_shift, cap = c.max_pages << c.page_shift;
    const int n_cols = a.g * a.L_q, groups = (n_cols + Lay::kCols - 1) / Lay::kCols, units = c.H_kv * groups;

    // ---- rows without a token: zeros ----
    for (int b = blockIdx.x; b < a.B; b += gridDim.x)
        if (c.seq_lens[b] <= 0) {
            const size_t n = (size_t)a.H_q * a.L_q * c.d_v * (a.out_fp16 ? 2 : 4) / 16;
            uint4 *row = static_cast<uint4 *>(a.out) + n * b;
            for (size_t i = tid; i < n; i += kAqThreads) row[i] = make_uint4(0u, 0u, 0u, 0u);
        }

    // ---- this CTA's part of the flat sequence: cells pos .. pos + end - 1 ----
    long long chunk, pos;
    int end;
    AqCursor at;                                                // where the products are
    {
        const int per = (a.B + kAqThreads - 1) / kAqThreads, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
        long long mine = 0;
        int longest = 0;
        AqCursor r;
        for (r.b = b0; r.b < b1; ++r.b) {
            r.row(c, cap);
            if (blockIdx.x == 0 && r.len != c.seq_lens[r.b]) q8_report(c.status, kStatusBadPage);
            mine += r.steps ? r.steps + kAqJoinCells : 0;
            longest = max(longest, r.steps);
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
        chunk = max(chunk, (long long)max(longest <= kAqWhole ? kAqJoinCells + longest : 1 + kAqMinChunk, 1 + (longest + kAqMaxParts - 2) / (kAqMaxParts - 1)));
        pos = chunk * blockIdx.x;
        if (pos >= total) return;                               // (the whole CTA)
        end = (int)min(chunk, total - pos);
        if (pos >= before * units && pos < (before + mine) * units) {
            r.b = b0;
            for (;; ++r.b) {
                r.row(c, cap);
                const int cells = r.steps ? r.steps + kAqJoinCells : 0;
                if (pos < (before + cells) * units) break;
                before += cells;
            }
            s_i[kAqWarps] = r.b;
            s_ll[kAqWarps] = pos - before * units;
        }
        __syncthreads();
        at.b = s_i[kAqWarps];
        at.row(c, cap);
        const int cells = at.steps + kAqJoinCells, cell = (int)(s_ll[kAqWarps] % cells);
        at.unit = (int)(s_ll[kAqWarps] / cells);
        at.step = max(cell - kAqJoinCells, 0);
        at.at = max(kAqJoinCells - cell, 0);
        if (at.at >= end) return;                               // nothing but a unit's join cells: no step of it is here
    }

    unsigned char *const ring = aq_raw + warp * (kAqStages * Lay::kStage);
    constexpr int JC = Lay::kJoinCols;
    float *const sM = reinterpret_cast<float *>(aq_raw + Lay::kRing), *const sL = sM + kAqWarps * JC, *const sK = sL + kAqWarps * JC;
    float *const sTop = sK + kAqWarps * JC, *const sSum = sTop + Lay::kCols;
    const int d_k = EXACT ? DP : c.d_k, d_v = EXACT ? DP : c.d_v;
    // O of warp w [col][DP], during a join after step n
    auto results = [&](int w, int n) { return reinterpret_cast<float *>(aq_raw + (w * kAqStages + n % kAqStages) * Lay::kStage); };
    const float k_unit = kQ8Unit<FORMAT> * a.scale_log2;

    // ---- the ring runs ahead of the products, over the borders of units; this warp's tile of a step holds tokens
    //      step * 64 + warp * 16 .. + 15 of the row ----
    AqCursor ahead = at;
    auto entry_of = [&](const AqCursor &x) {                    // the table's entry, not looked at yet
        const int tok = x.step * kAqTile + warp * 16;
        return x.at < end && tok < x.len ? __ldg(c.tables + (size_t)x.b * c.max_pages + (tok >> c.page_shift)) : -1;
    };
    auto fetch = [&](int n, int pid) {                          // the tile at `ahead` into stage n % kAqStages
        unsigned char *const stage = ring + (n % kAqStages) * Lay::kStage;
        const uint32_t s = aq_smem(stage);
        if (ahead.at < end) {
            const int tok = ahead.step * kAqTile + warp * 16;
            const bool there = tok < ahead.len && pid >= 0 && pid < c.n_pages;
            if (lane == 0) {
                *reinterpret_cast<int *>(stage + Lay::kTile + 8) = there;
                if (!there && tok < ahead.len) q8_report(c.status, kStatusBadPage);
            }
            if (there) {
                const size_t block = (size_t)pid * c.H_kv + (groups == 1 ? ahead.unit : ahead.unit / groups), row = block * page + (tok & (page - 1));
                // lanes over the pieces of a row, then the rows; behind the row's last token zeros for V: a weight of 0
                // does not mend a NaN that was left there
                constexpr int kLanes = DP / 16 < 32 ? DP / 16 : 32, kRows = 32 / kLanes;
                const int r0 = lane / kLanes, p = lane % kLanes;
                const uint8_t *k = c.k + (row + r0) * d_k + 16 * p, *v = c.v + (row + r0) * d_v + 16 * p;
                if (EXACT || 16 * p < d_k)
#pragma unroll
                    for (int i = 0; i < 16 / kRows; ++i) aq_copy<16>(s + aq_piece<DP>(r0 + i * kRows, p), k + i * kRows * d_k);
                if (EXACT || 16 * p < d_v)
#pragma unroll
                    for (int i = 0; i < 16 / kRows; ++i)
                        aq_copy_if<16>(s + Lay::kOffV + aq_piece<DP>(r0 + i * kRows, p), v + i * kRows * d_v, tok + r0 + i * kRows < ahead.len);
                if (lane == 0) {
                    aq_copy<4>(s + Lay::kTile, c.k_amax + block);
                    aq_copy<4>(s + Lay::kTile + 4, c.v_amax + block);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int entry;
    {
        AqCursor x = at;
        int entries[kAqStages];                                 // asked for together
#pragma unroll
        for (int n = 0; n < kAqStages; ++n) {
            entries[n] = entry_of(x);
            if (x.at < end) x.advance(c, a.B, cap, units, end);
        }
#pragma unroll
        for (int n = 0; n < kAqStages - 1; ++n) {
            fetch(n, entries[n]);
            if (ahead.at < end) ahead.advance(c, a.B, cap, units, end);
        }
        entry = entries[kAqStages - 1];
    }

    // pieces of units that other CTAs hold pieces of: the first and the last unit of this CTA's part
    int split_first[2] = {-1, -1}, split_pieces[2] = {0, 0}, split_b[2] = {0, 0}, split_unit[2] = {0, 0}, n_split = 0;
    uint32_t qf[NT][KJ * 4][2];
    int last[NT][2];
    float o[NT][MT][4], m_ref[NT][2], l_sum[NT][2];
    const int quads = d_v / 4;
    auto store = [&](int b, int unit, int col, int quad, float4 x, float l) {       // o = O / (R l); nothing seen: zeros
        const int cc = unit % groups * Lay::kCols + col;
        const float r = l != 0.f ? kQ8Unit<FORMAT> / l : 0.f;
        const size_t to = (((size_t)b * a.H_q + unit / groups * a.g + cc % a.g) * a.L_q + cc / a.g) * d_v + quad * 4;
        x = make_float4(x.x * r, x.y * r, x.z * r, x.w * r);
        if (a.out_fp16) {
            *reinterpret_cast<uint2 *>(static_cast<__half *>(a.out) + to) = make_uint2(q8_half2(x.x, x.y), q8_half2(x.z, x.w));
        } else {
            *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + to) = x;
        }
    };
    auto add = [](float4 &x, float k, const float4 &y) {
        x = make_float4(fmaf(k, y.x, x.x), fmaf(k, y.y, x.y), fmaf(k, y.z, x.z), fmaf(k, y.w, x.w));
    };

    bool fresh = true;                                          // a unit begins
    for (int n = 0;; ++n) {
        if (fresh) {
            // ---- q as the scores' second operand; the last token each of this lane's result columns sees ----
            fresh = false;
            const int h = at.unit / groups, col0 = at.unit % groups * Lay::kCols;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int col = col0 + (PACK ? g & 3 : nt * 8 + g);
                const bool on = col < n_cols;
                const __half *qr = a.q + (((size_t)at.b * a.H_q + h * a.g + (on ? col % a.g : 0)) * a.L_q + (on ? col / a.g : 0)) * d_k;
#pragma unroll
                for (int j = 0; j < KJ; ++j) {
                    uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
                    if (on && 64 * j + 16 * t < d_k) {
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
                    const int cc = col0 + (PACK ? 2 * (t & 1) : nt * 8 + 2 * t) + k;
                    last[nt][k] = cc < n_cols ? at.len - a.L_q + cc / a.g : -1;
                    m_ref[nt][k] = -1e30f;
                    l_sum[nt][k] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
            }
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kAqStages - 2) : "memory");
        __syncwarp();                                           // lane 0's words are there; everyone is done with step n - 1
        fetch(n + kAqStages - 1, entry);
        if (ahead.at < end) ahead.advance(c, a.B, cap, units, end);
        entry = entry_of(ahead);
        const unsigned char *s = ring + (n % kAqStages) * Lay::kStage;
        const float4 meta = *reinterpret_cast<const float4 *>(s + Lay::kTile);
        if (__float_as_int(meta.z)) {
            const float ks = meta.x * k_unit;

            // scores of tokens g, g + 8 for columns 2t, 2t + 1; two chains of products per column group
            float sc[NT][4], sd[NT][4];
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
                if (EXACT || 64 * j + 16 * t < d_k) {
                    x = *reinterpret_cast<const uint4 *>(s + aq_piece<DP>(g, t + 4 * j));
                    y = *reinterpret_cast<const uint4 *>(s + aq_piece<DP>(g + 8, t + 4 * j));
                }
                const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t a0, a1, a2, a3;
                    q8_pairs<FORMAT>(xw[w], a0, a2);
                    q8_pairs<FORMAT>(yw[w], a1, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float (&dst)[4] = (w & 1) ? sd[nt] : sc[nt];
                        if (j == 0 && w < 2) aq_mma_zero(dst, a0, a1, a2, a3, qf[nt][w][0], qf[nt][w][1]);
                        else aq_mma(dst, a0, a1, a2, a3, qf[nt][4 * j + w][0], qf[nt][4 * j + w][1]);
                    }
                }
            }

            // weights; amax^V = 2^e f.  A block of zeros adds to l alone, and l has fp32's range: its e keeps it from leading M
            const int vb = __float_as_int(meta.y) >> 23;
            const float e = vb > 0 ? (float)(vb - 127) : kQ8ZeroExponent;
            const float f = vb > 0 ? __int_as_float((__float_as_int(meta.y) & 0x7fffff) | 0x3f800000) : meta.y;
            const float inv_e = vb > 0 ? __int_as_float((254 - vb) << 23) : kQ8ZeroInverse;
            const int tok = at.step * kAqTile + warp * 16 + g;
            uint32_t ph[NT][2], pl[NT][2];
            bool beyond = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = fmaf(sc[nt][i] + sd[nt][i], ks, e);
                    sc[nt][i] = tok + 8 * (i >> 1) <= last[nt][i & 1] ? x : -INFINITY;
                    beyond |= sc[nt][i] > m_ref[nt][i & 1] + (kAqLift + kAqSlack);
                }
            if (__any_sync(0xffffffffu, beyond)) {              // M moves (seldom): to the largest of the tile, per column, less the lift
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float top = fmaxf(sc[nt][k], sc[nt][k + 2]);
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                        top = fmaxf(top - kAqLift, m_ref[nt][k]);
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
                    const uint32_t hw = *reinterpret_cast<const uint32_t *>(&hi), lw = *reinterpret_cast<const uint32_t *>(&lo);
                    ph[nt][r] = aq_transpose(PACK && t >= 2 ? lw : hw);
                    if constexpr (!PACK) pl[nt][r] = aq_transpose(lw);
                }
            }

            // values: product steps of two dims per lane
#pragma unroll
            for (int j = 0; j < VP; ++j) {
                uint32_t r[4][VB / 4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int row = 2 * t + (k & 1) + 8 * (k >> 1);
                    if constexpr (VB == 16) {
                        uint4 u = make_uint4(0u, 0u, 0u, 0u);
                        if (EXACT || 16 * g + 128 * j < d_v) u = *reinterpret_cast<const uint4 *>(s + Lay::kOffV + aq_piece<DP>(row, g + 8 * j));
                        r[k][0] = u.x, r[k][1] = u.y, r[k][2] = u.z, r[k][3] = u.w;
                    } else {
                        const uint2 u = *reinterpret_cast<const uint2 *>(s + Lay::kOffV + aq_piece<DP>(row, g >> 1) + (g & 1) * 8);
                        r[k][0] = u.x, r[k][1] = u.y;
                    }
                }
#pragma unroll
                for (int w = 0; w < VB / 4; ++w) {
                    // bytes of two tokens side by side: dims 4w, 4w + 1 and dims 4w + 2, 4w + 3
                    uint32_t x0, x1, x2, x3, y0, y1, y2, y3;
                    q8_pairs<FORMAT>(__byte_perm(r[0][w], r[1][w], 0x5140), x0, x1);        // tokens 2t, 2t + 1
                    q8_pairs<FORMAT>(__byte_perm(r[0][w], r[1][w], 0x7362), x2, x3);
                    q8_pairs<FORMAT>(__byte_perm(r[2][w], r[3][w], 0x5140), y0, y1);        // tokens 2t + 8, 2t + 9
                    q8_pairs<FORMAT>(__byte_perm(r[2][w], r[3][w], 0x7362), y2, y3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const uint32_t a0 = half ? x2 : x0, a1 = half ? x3 : x1, a2 = half ? y2 : y0, a3 = half ? y3 : y1;
                            float (&dst)[4] = o[nt][(j * (VB / 4) + w) * 2 + half];
                            // the tile's own sum from zero, then onto O: the tensor pipe cuts its sums off, and a chain
                            // of a hundred tiles through its accumulator tripled the error of the result
                            float acc[4];
                            if constexpr (PACK) {
                                aq_mma_zero(acc, a0, a1, a2, a3, ph[nt][0], ph[nt][1]);
                            } else {
                                aq_mma_zero(acc, a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
                                aq_mma(acc, a0, a1, a2, a3, ph[nt][0], ph[nt][1]);
                            }
#pragma unroll
                            for (int i = 0; i < 4; ++i) dst[i] += acc[i];
                        }
                }
            }
        }
        const bool done = at.step + 1 == at.steps || at.at + 1 == end;
        if (!done) {
            ++at.step;
            ++at.at;
            continue;
        }

        // ---- the unit, or this CTA's piece of it, is done: join the warps (the ring stays full meanwhile) ----
        fresh = true;
        const long long u0 = pos + at.at - at.step;             // the unit's first step
        const int first = (int)(u0 / chunk), pieces = (int)((u0 + at.steps - 1) / chunk) - first + 1, me = blockIdx.x;
        const int left = n_cols - at.unit % groups * Lay::kCols;                    // columns of the unit and beyond
        float *const part = parts + (size_t)(2 * me + (me == first)) * Lay::kPart;
        float *const mine = results(warp, n);
        __syncwarp();                                           // everyone is done with the tile
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt > 0 && nt * 8 >= left) break;
            if (nt > 0) __syncthreads();                        // the results of the columns before have been read
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float l = l_sum[nt][k];
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
                const int col = 2 * t + k;
                if (g == 0 && (!PACK || t < 2)) {
                    sM[warp * JC + col] = m_ref[nt][k];
                    sL[warp * JC + col] = l;
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    // step i % (VB / 2) of piece j: dims 128 j + VB g + 2 (i % (VB / 2)), + 1
                    const int dim = i / (VB / 2) * 128 + VB * g + 2 * (i % (VB / 2));
                    float2 x = make_float2(o[nt][i][k], o[nt][i][k + 2]);
                    if constexpr (PACK) {                       // columns 4..7 hold the products of the weights' lower halves
                        x.x += __shfl_xor_sync(0xffffffffu, x.x, 2);
                        x.y += __shfl_xor_sync(0xffffffffu, x.y, 2);
                    }
                    if (!PACK || t < 2) *reinterpret_cast<float2 *>(mine + col * DP + dim) = x;
                }
            }
            __syncthreads();
            if (tid < JC) {
                float top = sM[tid], l = 0.f;
#pragma unroll
                for (int w = 1; w < kAqWarps; ++w) top = fmaxf(top, sM[w * JC + tid]);
#pragma unroll
                for (int w = 0; w < kAqWarps; ++w) {
                    const float k = ex2_approx(sM[w * JC + tid] - top);
                    sK[w * JC + tid] = k;
                    l = fmaf(k, sL[w * JC + tid], l);
                }
                sTop[nt * 8 + tid] = top;
                sSum[nt * 8 + tid] = l;
            }
            __syncthreads();
            const int n_here = min(JC, left - nt * 8) * quads;  // groups of 4 dims, of all columns
            for (int i = tid; i < n_here; i += kAqThreads) {
                const int col = i / quads, quad = i % quads;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kAqWarps; ++w)
                    add(x, sK[w * JC + col], *reinterpret_cast<const float4 *>(results(w, n) + col * DP + quad * 4));
                if (pieces == 1) store(at.b, at.unit, nt * 8 + col, quad, x, sSum[nt * 8 + col]);
                else __stcg(reinterpret_cast<float4 *>(part + 2 * Lay::kCols + (nt * 8 + col) * DP + quad * 4), x);
            }
        }
        if (pieces > 1) {
            if (tid < min(Lay::kCols, left)) {
                __stcg(part + tid, sTop[tid]);
                __stcg(part + Lay::kCols + tid, sSum[tid]);
            }
            split_first[n_split] = first;
            split_pieces[n_split] = pieces;
            split_b[n_split] = at.b;
            split_unit[n_split] = at.unit;
            ++n_split;
        }
        at.advance(c, a.B, cap, units, end);
        if (at.at >= end) break;
        __syncthreads();                                        // the results have been read
    }
    if (n_split == 0) return;

    // ---- units of several CTAs: whoever brings the last piece joins them, in the order of the pieces ----
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    float *const sF = reinterpret_cast<float *>(aq_raw);        // [col][kAqMaxParts]
    __syncthreads();
    if (tid < n_split) {
        const int first = tid ? split_first[1] : split_first[0], pieces = tid ? split_pieces[1] : split_pieces[0];
        __threadfence();                                        // the CTA's pieces (ordered before by the barrier), then the count
        const unsigned seen = atomicAdd(tickets + first, 1u);
        __threadfence();                                        // the count, then what the others wrote
        s_i[tid] = seen == (unsigned)pieces - 1;
        if (seen == (unsigned)pieces - 1) tickets[first] = 0u;  // all pieces are in: ready for the next launch
    }
    __syncthreads();
    for (int u = 0; u < n_split; ++u) {
        if (!s_i[u]) continue;
        const int first = u ? split_first[1] : split_first[0], pieces = u ? split_pieces[1] : split_pieces[0];
        const int b = u ? split_b[1] : split_b[0], unit = u ? split_unit[1] : split_unit[0];
        const float *const head = parts + (size_t)(2 * first + 1) * Lay::kPart, *const rest = parts + (size_t)2 * first * Lay::kPart;
        auto piece = [&](int p) { return p == 0 ? head : rest + (size_t)2 * p * Lay::kPart; };
        const int n_here = min(Lay::kCols, n_cols - unit % groups * Lay::kCols) * quads;
        __syncthreads();
        for (int col = warp; col < min(Lay::kCols, n_cols - unit % groups * Lay::kCols); col += kAqWarps) {    // a warp's lanes over the pieces
            float m[kAqMaxParts / 32], lp[kAqMaxParts / 32], l = 0.f, top = -1e30f;
#pragma unroll
            for (int i = 0; i < kAqMaxParts / 32; ++i) {
                const bool on = lane + 32 * i < pieces;
                m[i] = on ? __ldcg(piece(lane + 32 * i) + col) : -1e30f;
                lp[i] = on ? __ldcg(piece(lane + 32 * i) + Lay::kCols + col) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < kAqMaxParts / 32; ++i) top = fmaxf(top, m[i]);
#pragma unroll
            for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
#pragma unroll
            for (int i = 0; i < kAqMaxParts / 32; ++i) {
                const float k = ex2_approx(m[i] - top);
                if (lane + 32 * i < pieces) sF[col * kAqMaxParts + lane + 32 * i] = k;
                l = fmaf(k, lp[i], l);
            }
#pragma unroll
            for (int s = 16; s; s >>= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
            if (lane == 0) sSum[col] = l;
        }
        __syncthreads();
        for (int i = tid; i < n_here; i += kAqThreads) {
            const int col = i / quads, quad = i % quads;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            const int off = 2 * Lay::kCols + col * DP + quad * 4;
            for (int p0 = 0; p0 < pieces; p0 += 16) {           // 16 loads in flight
                float4 y[16];
#pragma unroll
                for (int p = 0; p < 16; ++p)
                    y[p] = p0 + p < pieces ? __ldcg(reinterpret_cast<const float4 *>(piece(p0 + p) + off)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int p = 0; p < 16; ++p) add(x, p0 + p < pieces ? sF[col * kAqMaxParts + p0 + p] : 0.f, y[p]);
            }
            store(b, unit, col, quad, x, sSum[col]);
        }
    }
}

template <int FORMAT, int DP, int NT, bool PACK, bool EXACT>
lookat_status launch_aq(Ctx *ctx, const Q8AttendArgs &a)
{
    using Lay = AqLayout<DP, NT, PACK>;
    auto kern = attend_q8_kernel<FORMAT, DP, NT, PACK, EXACT>;
    static int resident[64];                                    // CTAs per SM, by device (0: not asked yet)
    int &per_sm = resident[ctx->device & 63];
    if (!per_sm) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay::kBytes) != cudaSuccess)
            return check_launch(ctx, "attend_q8: shared-memory opt-in");
        int n = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, kAqThreads, Lay::kBytes) != cudaSuccess || n < 1)
            return check_launch(ctx, "attend_q8: occupancy");
        per_sm = n;
    }
    const long long n_cols = (long long)a.g * a.L_q;
    const long long most = (long long)a.B * a.c.H_kv * ((n_cols + Lay::kCols - 1) / Lay::kCols) *
                           ((((long long)a.c.max_pages << a.c.page_shift) + kAqTile - 1) / kAqTile);
    const long long full = (long long)ctx->sm_count * per_sm;
    if (most / full > (1ll << 29)) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "attend_q8: too many tokens for one call");
    const unsigned grid = (unsigned)(most < full ? most : full);
    lookat_status st = workspace(ctx, ctx->q8_partials, (size_t)full * 2 * Lay::kPart * sizeof(float), false, "attend_q8");
    if (st == LOOKAT_OK) st = workspace(ctx, ctx->q8_tickets, (size_t)ctx->sm_count * 16 * sizeof(unsigned), true, "attend_q8");
    if (st != LOOKAT_OK) return st;
    kern<<<grid, kAqThreads, Lay::kBytes, ctx->stream>>>(a, static_cast<float *>(ctx->q8_partials.ptr), static_cast<unsigned *>(ctx->q8_tickets.ptr));
    return check_launch(ctx, "attend_q8_kernel");
}

// columns of a unit: 4 where that is all there are (the two halves of the weights then share the 8 columns of a product),
// 8, or 16
template <int FORMAT, int DP, bool EXACT>
lookat_status launch_aq_cols(Ctx *ctx, const Q8AttendArgs &a)
{
    const long long n = (long long)a.g * a.L_q;
    if (n <= 4) return launch_aq<FORMAT, DP, 1, true, EXACT>(ctx, a);
    if constexpr (DP <= 128)
        if (n > 8) return launch_aq<FORMAT, DP, 2, false, EXACT>(ctx, a);
    return launch_aq<FORMAT, DP, 1, false, EXACT>(ctx, a);
}

// head dims: 64 and 128 as they are, others padded to 128 or 256
template <int FORMAT>
lookat_status launch_aq_dims(Ctx *ctx, const Q8AttendArgs &a)
{
    const int dk = a.c.d_k, dv = a.c.d_v;
    if (dk == 64 && dv == 64) return launch_aq_cols<FORMAT, 64, true>(ctx, a);
    if (dk == 128 && dv == 128) return launch_aq_cols<FORMAT, 128, true>(ctx, a);
    return dk <= 128 && dv <= 128 ? launch_aq_cols<FORMAT, 128, false>(ctx, a) : launch_aq_cols<FORMAT, 256, false>(ctx, a);
}

}  // namespace

lookat_status launch_attend_q8(Ctx *ctx, const Q8AttendArgs &a)
{
    if ((long long)a.H_q * a.L_q > (1ll << 30)) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "attend_q8: more than 2^30 queries per row");
    if (attend_q8_umma_covers(ctx, a)) return launch_attend_q8_umma(ctx, a);
    return a.format == LOOKAT_Q8_INT8 ? launch_aq_dims<LOOKAT_Q8_INT8>(ctx, a) : launch_aq_dims<LOOKAT_Q8_E4M3>(ctx, a);
}

}  // namespace lookat
