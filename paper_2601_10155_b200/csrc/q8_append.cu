// lookat_q8_append: new keys and values into the blocks of the 8-bit paged cache.
//
// Per block (one page of one KV head), with x its new tokens:  amax' = max(amax if the block holds earlier tokens, |x|),
// n = round(R x / amax'), and where amax has grown the earlier numbers become round(n amax / amax').  x and amax are fp16
// values and n has at most 8 bits, so R x and n amax are exact in fp32.  A rounding border of n has at most 8 significant
// bits and amax 11: a quotient that is not on a border is at least 2^-19 of itself away from it.  So x times the rounded
// R / amax' (within 2^-22 of the quotient) rounds as the quotient does unless that is a tie; a unit of 16 elements that holds
// one is done again by division, whose correctly rounded fp32 quotient is the tie itself.
//
// One group of threads per (row, KV head, K or V, block): it reads the block's new tokens once (kept in registers between
// the maximum and the rounding), so nothing is read from HBM twice and no two groups share a block.
#include "q8.cuh"

namespace lookat {

namespace {

constexpr int kApKeep = 4;                      // 16-element units a thread keeps in registers between the two passes

// two halves with NaN taken as 0 and infinities as the largest finite number
__device__ __forceinline__ uint32_t ap_finite2(uint32_t w)
{
    const __half2 x = *reinterpret_cast<const __half2 *>(&w), top = __halves2half2(__ushort_as_half(0x7bff), __ushort_as_half(0x7bff));
    const uint32_t number = w & __heq2_mask(x, x);
    const __half2 y = __hmax2(__hmin2(*reinterpret_cast<const __half2 *>(&number), top), __hneg2(top));
    return *reinterpret_cast<const uint32_t *>(&y);
}
struct ApUnit {                                 // 16 new elements
    uint32_t w[8];
};
__device__ __forceinline__ ApUnit ap_load(const uint4 *src)
{
    const uint4 a = __ldg(src), b = __ldg(src + 1);
    return {{ap_finite2(a.x), ap_finite2(a.y), ap_finite2(a.z), ap_finite2(a.w), ap_finite2(b.x), ap_finite2(b.y), ap_finite2(b.z), ap_finite2(b.w)}};
}
__device__ __forceinline__ void ap_max(__half2 &top, const ApUnit &u)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) top = __hmax2(top, __habs2(*reinterpret_cast<const __half2 *>(&u.w[i])));
}

// 16 new elements to 16 bytes; amax > 0, scale = R / amax rounded
template <int FORMAT>
__device__ __forceinline__ uint4 ap_round16(const ApUnit &u, float amax, float scale)
{
    constexpr float R = FORMAT == LOOKAT_Q8_INT8 ? kQ8RangeInt8 : kQ8RangeE4m3;
    uint32_t o[4];
    bool tie = false;
    if constexpr (FORMAT == LOOKAT_Q8_INT8) {
        constexpr float kMagic = 12582912.f;    // 1.5 * 2^23: the sum's low bits are the rounded number
        const float half = 0.5f * amax;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t t[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&u.w[2 * i + j]));
                const float a = fmaf(x.x, scale, kMagic), b = fmaf(x.y, scale, kMagic);
                // what is left of R x, exactly: half of amax or more only at a tie
                tie |= fabsf(fmaf(kMagic - a, amax, R * x.x)) >= half || fabsf(fmaf(kMagic - b, amax, R * x.y)) >= half;
                t[2 * j] = __float_as_uint(a);
                t[2 * j + 1] = __float_as_uint(b);
            }
            o[i] = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
        }
    } else {
        constexpr float kUp = 1.f + 0x1p-21f, kDown = 1.f - 0x1p-21f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t t[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&u.w[2 * i + j]));
                const float2 r = make_float2(x.x * scale, x.y * scale);
                t[j] = __nv_cvt_float2_to_fp8x2(make_float2(r.x * kUp, r.y * kUp), __NV_SATFINITE, __NV_E4M3);
                tie |= t[j] != __nv_cvt_float2_to_fp8x2(make_float2(r.x * kDown, r.y * kDown), __NV_SATFINITE, __NV_E4M3);
            }
            o[i] = t[0] | t[1] << 16;
        }
    }
    if (tie) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[i] = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&u.w[2 * i + j]));
                o[i] |= (q8_round<FORMAT>(__fdiv_rn(R * x.x, amax)) | q8_round<FORMAT>(__fdiv_rn(R * x.y, amax)) << 8) << (16 * j);
            }
        }
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

// THREADS per group: as many as hold a block's new tokens in kApKeep units each, since what bounds the kernel is how many
// groups wait for their loads at a time (4 rows of up to 4096 tokens, 8 heads of 128 dims, pages of 64: 24 us with 128
// threads, 25 with 256, 35 with 512; pages of 16: 39, 51 and 97)
template <int FORMAT, int THREADS>
__global__ void __launch_bounds__(THREADS == 32 ? 128 : THREADS, THREADS == 256 ? 4 : 8) q8_append_kernel(Q8AppendArgs a, int blocks_per_row)
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
    const int len_in = c.seq_lens[b], count_in = a.n_new ? max(a.n_new[b], 0) : a.n;
    const int len = min(max(len_in, 0), cap), count = min(count_in, a.n);
    const int first = len_in - count;                           // position of the row's token 0 (may be out of range)
    if (lane == 0 && (len_in != len || count_in != count || first < 0)) q8_report(c.status, kStatusBadPage);
    if (count == 0) return;
    const int blk = (max(first, 0) >> c.page_shift) + j;
    const int lo = max(max(first, 0), blk << c.page_shift), hi = min(len, (blk + 1) << c.page_shift);
    if (lo >= hi) return;
    const int pid = c.tables[(size_t)b * c.max_pages + blk];   // (looked at once the new tokens are on their way too)
    const int d = which ? c.d_v : c.d_k, old = lo - (blk << c.page_shift);
    const uint4 *src = reinterpret_cast<const uint4 *>((which ? a.v_new : a.k_new) + ((size_t)bh * a.n + (lo - first)) * d);
    const int units = (hi - lo) * d / 16;

    ApUnit keep[kApKeep];
    __half2 tops2 = __halves2half2(__ushort_as_half(0), __ushort_as_half(0));
#pragma unroll
    for (int i = 0; i < kApKeep; ++i) {
        const int u = lane + i * THREADS;
        if (u < units) {
            keep[i] = ap_load(src + 2 * u);
            ap_max(tops2, keep[i]);
        }
    }
    for (int u = lane + kApKeep * THREADS; u < units; u += THREADS) ap_max(tops2, ap_load(src + 2 * u));
    float top = fmaxf(__low2float(tops2), __high2float(tops2));
    if (pid < 0 || pid >= c.n_pages) {                          // (the same for the whole group)
        if (lane == 0) q8_report(c.status, kStatusBadPage);
        return;
    }
    const size_t block = (size_t)pid * c.H_kv + h;
    uint8_t *base = (which ? c.v : c.k) + block * page * d;
    float *amax_at = (which ? c.v_amax : c.k_amax) + block;
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
    const float scale = now > 0.f ? __fdiv_rn(FORMAT == LOOKAT_Q8_INT8 ? kQ8RangeInt8 : kQ8RangeE4m3, now) : 0.f;
#pragma unroll
    for (int i = 0; i < kApKeep; ++i) {
        const int u = lane + i * THREADS;
        if (u < units) dst[u] = now > 0.f ? ap_round16<FORMAT>(keep[i], now, scale) : make_uint4(0u, 0u, 0u, 0u);
    }
    for (int u = lane + kApKeep * THREADS; u < units; u += THREADS)
        dst[u] = now > 0.f ? ap_round16<FORMAT>(ap_load(src + 2 * u), now, scale) : make_uint4(0u, 0u, 0u, 0u);
    if constexpr (THREADS == 32) __syncwarp();
    if (lane == 0) *amax_at = now;
}

}  // namespace

lookat_status launch_q8_append(Ctx *ctx, const Q8AppendArgs &a)
{
    const int page = 1 << a.c.page_shift;
    const int blocks = (a.n + page - 2) / page + 1;             // blocks that n consecutive tokens can touch
    const long long items = (long long)a.B * a.c.H_kv * 2 * blocks;
    const int d = a.c.d_k > a.c.d_v ? a.c.d_k : a.c.d_v, units = (a.n < page ? a.n : page) * d / 16;     // of the largest group
    const int threads = units <= 32 * kApKeep ? 32 : units <= 128 * kApKeep ? 128 : 256;
    const long long ctas = threads == 32 ? (items + 3) / 4 : items;
    if (ctas > 0x7fffffffll) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "q8_append: too many blocks for one call");
    auto launch = [&](auto kern) { kern<<<(unsigned)ctas, threads == 32 ? 128 : threads, 0, ctx->stream>>>(a, blocks); };
    if (a.format == LOOKAT_Q8_INT8)
        threads == 32 ? launch(q8_append_kernel<LOOKAT_Q8_INT8, 32>) : threads == 128 ? launch(q8_append_kernel<LOOKAT_Q8_INT8, 128>)
                                                                                      : launch(q8_append_kernel<LOOKAT_Q8_INT8, 256>);
    else
        threads == 32 ? launch(q8_append_kernel<LOOKAT_Q8_E4M3, 32>) : threads == 128 ? launch(q8_append_kernel<LOOKAT_Q8_E4M3, 128>)
                                                                                      : launch(q8_append_kernel<LOOKAT_Q8_E4M3, 256>);
    return check_launch(ctx, "q8_append_kernel");
}

}  // namespace lookat
