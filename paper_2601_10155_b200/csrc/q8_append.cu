// lookat_q8_append: new keys and values into the blocks of the 8-bit paged cache.
//
// Per block (one page of one KV head), with x its new tokens:  amax' = max(amax if the block holds earlier tokens, |x|),
// n = round(R x / amax'), and where amax has grown the earlier numbers become round(n amax / amax').  x and amax are fp16
// values and n has at most 8 bits, so R x and n amax are exact in fp32 (at most 19 bits) and the quotient of two such
// numbers lies on a rounding border only if the real quotient does, or at least 2^-21 of itself away from it: the
// correctly rounded fp32 quotient rounds to the same 8-bit number as the real one.
//
// One group of threads per (row, KV head, K or V, block): it reads the block's new tokens once (kept in registers between
// the maximum and the rounding), so nothing is read from HBM twice and no two groups share a block.
#include "q8.cuh"

namespace lookat {

namespace {

constexpr int kApKeep = 4;                      // 16-element units a thread keeps in registers between the two passes

__device__ __forceinline__ float ap_finite(float x)
{
    return x == x ? fminf(fmaxf(x, -65504.f), 65504.f) : 0.f;
}

__device__ __forceinline__ float ap_max16(const uint4 (&u)[2])
{
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t w = j == 0 ? u[i].x : j == 1 ? u[i].y : j == 2 ? u[i].z : u[i].w;
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
            m = fmaxf(m, fmaxf(fabsf(ap_finite(f.x)), fabsf(ap_finite(f.y))));
        }
    return m;
}

// 16 new elements to 16 bytes; amax > 0
template <int FORMAT>
__device__ __forceinline__ uint4 ap_round16(const uint4 (&u)[2], float amax)
{
    const float R = FORMAT == LOOKAT_Q8_INT8 ? kQ8RangeInt8 : kQ8RangeE4m3;
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w0 = (i & 1) ? u[i >> 1].z : u[i >> 1].x, w1 = (i & 1) ? u[i >> 1].w : u[i >> 1].y;
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&w0));
        const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&w1));
        o[i] = q8_round<FORMAT>(__fdiv_rn(R * ap_finite(a.x), amax)) | q8_round<FORMAT>(__fdiv_rn(R * ap_finite(a.y), amax)) << 8 |
               q8_round<FORMAT>(__fdiv_rn(R * ap_finite(b.x), amax)) << 16 | q8_round<FORMAT>(__fdiv_rn(R * ap_finite(b.y), amax)) << 24;
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// 16 earlier numbers of a block whose amax grows from `was` to `now`
template <int FORMAT>
__device__ __forceinline__ uint4 ap_shrink16(uint4 u, float was, float now)
{
    uint32_t in[4] = {u.x, u.y, u.z, u.w}, o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o[i] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            o[i] |= q8_round<FORMAT>(__fdiv_rn(q8_value<FORMAT>((in[i] >> (8 * j)) & 0xffu) * was, now)) << (8 * j);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// THREADS per group: a warp where a row brings a few tokens, else a whole CTA
template <int FORMAT, int THREADS>
__global__ void __launch_bounds__(THREADS == 32 ? 128 : THREADS) q8_append_kernel(Q8AppendArgs a, int blocks_per_row)
{
    constexpr int kGroups = THREADS == 32 ? 4 : 1;
    const int lane = THREADS == 32 ? (threadIdx.x & 31) : threadIdx.x;
    const long long item = (long long)blockIdx.x * kGroups + (THREADS == 32 ? threadIdx.x >> 5 : 0);
    const Q8View &c = a.c;
    const int j = (int)(item % blocks_per_row), which = (int)(item / blocks_per_row & 1);
    const long long bh = item / blocks_per_row >> 1;
    const int b = (int)(bh / c.H_kv), h = (int)(bh % c.H_kv);
    if (b >= a.B) return;                                       // (whole groups leave)

    const int page = 1 << c.page_shift, cap = c.max_pages << c.page_shift;
    const int len_in = c.seq_lens[b], count_in = a.n_new ? a.n_new[b] : a.n;
    const int len = min(max(len_in, 0), cap), count = min(max(count_in, 0), a.n);
    const int first = len_in - count;                           // position of the row's token 0 (may be out of range)
    if (lane == 0 && (len_in != len || count_in != count || first < 0)) q8_report(c.status, kStatusBadPage);
    if (count == 0) return;
    const int blk = (max(first, 0) >> c.page_shift) + j;
    const int lo = max(max(first, 0), blk << c.page_shift), hi = min(len, (blk + 1) << c.page_shift);
    if (lo >= hi) return;
    const int pid = c.tables[(size_t)b * c.max_pages + blk];
    if (pid < 0 || pid >= c.n_pages) {
        if (lane == 0) q8_report(c.status, kStatusBadPage);
        return;
    }
    const int d = which ? c.d_v : c.d_k, old = lo - (blk << c.page_shift);
    const size_t block = (size_t)pid * c.H_kv + h;
    const uint4 *src = reinterpret_cast<const uint4 *>((which ? a.v_new : a.k_new) + ((size_t)bh * a.n + (lo - first)) * d);
    uint8_t *base = (which ? c.v : c.k) + block * page * d;
    float *amax_at = (which ? c.v_amax : c.k_amax) + block;
    const int units = (hi - lo) * d / 16;

    uint4 keep[kApKeep][2];
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kApKeep; ++i) {
        const int u = lane + i * THREADS;
        if (u < units) {
            keep[i][0] = __ldg(src + 2 * u);
            keep[i][1] = __ldg(src + 2 * u + 1);
            top = fmaxf(top, ap_max16(keep[i]));
        }
    }
    for (int u = lane + kApKeep * THREADS; u < units; u += THREADS) {
        const uint4 x[2] = {__ldg(src + 2 * u), __ldg(src + 2 * u + 1)};
        top = fmaxf(top, ap_max16(x));
    }
    float was = 0.f;
    if (old > 0) was = fmaxf(*amax_at, 0.f);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if constexpr (THREADS > 32) {
        __shared__ float tops[THREADS / 32];
        if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
        __syncthreads();                                        // (also: everyone has read *amax_at)
#pragma unroll
        for (int i = 0; i < THREADS / 32; ++i) top = fmaxf(top, tops[i]);
    }
    const float now = fmaxf(was, top);

    if (now > was && old > 0 && was > 0.f) {                    // (with was = 0 the earlier numbers are all 0)
        uint4 *o = reinterpret_cast<uint4 *>(base);
        for (int u = lane; u < old * d / 16; u += THREADS) o[u] = ap_shrink16<FORMAT>(o[u], was, now);
    }
    uint4 *dst = reinterpret_cast<uint4 *>(base + (size_t)old * d);
#pragma unroll
    for (int i = 0; i < kApKeep; ++i) {
        const int u = lane + i * THREADS;
        if (u < units) dst[u] = now > 0.f ? ap_round16<FORMAT>(keep[i], now) : make_uint4(0u, 0u, 0u, 0u);
    }
    for (int u = lane + kApKeep * THREADS; u < units; u += THREADS) {
        const uint4 x[2] = {__ldg(src + 2 * u), __ldg(src + 2 * u + 1)};
        dst[u] = now > 0.f ? ap_round16<FORMAT>(x, now) : make_uint4(0u, 0u, 0u, 0u);
    }
    if constexpr (THREADS == 32) __syncwarp();
    if (lane == 0) *amax_at = now;
}

}  // namespace

lookat_status launch_q8_append(Ctx *ctx, const Q8AppendArgs &a)
{
    const int page = 1 << a.c.page_shift;
    const int blocks = (a.n + page - 2) / page + 1;             // blocks that n consecutive tokens can touch
    const long long items = (long long)a.B * a.c.H_kv * 2 * blocks;
    const bool few = a.n <= 8;
    const long long ctas = few ? (items + 3) / 4 : items;
    if (ctas > 0x7fffffffll) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "q8_append: too many blocks for one call");
    if (a.format == LOOKAT_Q8_INT8) {
        if (few) q8_append_kernel<LOOKAT_Q8_INT8, 32><<<(unsigned)ctas, 128, 0, ctx->stream>>>(a, blocks);
        else q8_append_kernel<LOOKAT_Q8_INT8, 256><<<(unsigned)ctas, 256, 0, ctx->stream>>>(a, blocks);
    } else {
        if (few) q8_append_kernel<LOOKAT_Q8_E4M3, 32><<<(unsigned)ctas, 128, 0, ctx->stream>>>(a, blocks);
        else q8_append_kernel<LOOKAT_Q8_E4M3, 256><<<(unsigned)ctas, 256, 0, ctx->stream>>>(a, blocks);
    }
    return check_launch(ctx, "q8_append_kernel");
}

}  // namespace lookat
