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
// the maximum and the rounding), so nothing is read from HBM twice and no two groups share a block.  Magnitudes are compared as
// the whole numbers that their bits are; only where one is an infinity or a NaN are the numbers made finite.
#include <type_traits>

#include "serve.cuh"

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
    return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ void ap_finite(ApUnit &u)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) u.w[i] = ap_finite2(u.w[i]);
}
// magnitudes as whole numbers, which go in the same order; infinities are 0x7c00, NaN more
__device__ __forceinline__ void ap_max(uint32_t &top, const ApUnit &u)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) top = __vmaxu2(top, u.w[i] & 0x7fff7fffu);
}
__device__ __forceinline__ uint32_t ap_higher(uint32_t top) { return max(top & 0xffffu, top >> 16); }

__device__ __forceinline__ unsigned long long ap_two(float x, float y)
{
    unsigned long long p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(x), "f"(y));
    return p;
}
__device__ __forceinline__ float2 ap_each(unsigned long long p)
{
    float2 x;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x.x), "=f"(x.y) : "l"(p));
    return x;
}
__device__ __forceinline__ unsigned long long ap_mul(unsigned long long a, unsigned long long b)
{
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(a) : "l"(b));
    return a;
}
__device__ __forceinline__ unsigned long long ap_fma(unsigned long long a, unsigned long long b, unsigned long long c)
{
    asm("fma.rn.f32x2 %0, %0, %1, %2;" : "+l"(a) : "l"(b), "l"(c));
    return a;
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
        const unsigned long long scale2 = ap_two(scale, scale), magic2 = ap_two(kMagic, kMagic), minus2 = ap_two(-1.f, -1.f),
                                 amax2 = ap_two(amax, amax), R2 = ap_two(R, R);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t t[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 xf = __half22float2(*reinterpret_cast<const __half2 *>(&u.w[2 * i + j]));
                const unsigned long long x = ap_two(xf.x, xf.y), a = ap_fma(x, scale2, magic2);
                // what is left of R x, exactly: half of amax or more only at a tie
                const float2 left = ap_each(ap_fma(ap_fma(a, minus2, magic2), amax2, ap_mul(x, R2))), n = ap_each(a);
                tie |= fmaxf(fabsf(left.x), fabsf(left.y)) >= half;
                t[2 * j] = __float_as_uint(n.x);
                t[2 * j + 1] = __float_as_uint(n.y);
            }
            o[i] = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
        }
    } else {
        const float up = scale * (1.f + 0x1p-21f), down = scale * (1.f - 0x1p-21f);
        const unsigned long long up2 = ap_two(up, up), down2 = ap_two(down, down);
        uint32_t differ = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t t[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 xf = __half22float2(*reinterpret_cast<const __half2 *>(&u.w[2 * i + j]));
                const unsigned long long x = ap_two(xf.x, xf.y);
                t[j] = __nv_cvt_float2_to_fp8x2(ap_each(ap_mul(x, up2)), __NV_SATFINITE, __NV_E4M3);
                differ |= t[j] ^ __nv_cvt_float2_to_fp8x2(ap_each(ap_mul(x, down2)), __NV_SATFINITE, __NV_E4M3);
            }
            o[i] = t[0] | t[1] << 16;
        }
        tie = differ != 0;
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
// groups wait for their loads at a time (4 rows of up to 4096 tokens, 8 heads of 128 dims, pages of 64: 28 us with 32 threads, 19
// with 128, 25 with 256; pages of 16: 25, 34 and 61.  As packed rows of 4096 tokens, pages of 64: 32, 31 and 34 us)
//
// PACKED: the rows' tokens stand one behind the other (a.starts), and the host does not know the rows' lengths.  A row of c
// tokens touches at most c / page + 2 blocks (rounded down), so row b has the slots from starts[b] / page + 2 b on: those of
// different rows lie apart, a bisection over the rows finds a slot's, and n / page + 2 B slots do for any lengths.
template <int FORMAT, int THREADS, bool PACKED>
__global__ void __launch_bounds__(THREADS == 32 ? 128 : THREADS, THREADS == 256 ? 4 : 8) q8_append_kernel(Q8AppendArgs a, int blocks_per_row)
{
    constexpr int kGroups = THREADS == 32 ? 4 : 1;
    const int lane = THREADS == 32 ? (threadIdx.x & 31) : threadIdx.x;
    const long long item = (long long)blockIdx.x * kGroups + (THREADS == 32 ? threadIdx.x >> 5 : 0);
    const Q8View &c = a.c;
    [[maybe_unused]] const Packed rows = {a.starts, a.B, a.n, c.status};
    int j, which, b, h, start = 0;
    long long bh = 0;
    if constexpr (PACKED) {                                     // [slot][head][K or V]
        if (item == 0) packed_check(rows, lane, THREADS);       // (slot 0 may be no row's)
        const unsigned pair = (unsigned)item >> 1;              // (fewer than 2^31 items)
        which = (int)(item & 1);
        h = (int)(pair % (unsigned)c.H_kv);
        const int slot = (int)(pair / (unsigned)c.H_kv);
        if (slot >= blocks_per_row) return;                     // (here the number of slots; whole groups leave)
        auto slot0 = [&](int row) { return (min(max(__ldg(a.starts + row), 0), a.n) >> c.page_shift) + 2 * row; };
        int lo = 0, hi = a.B;                                   // the last row whose first slot is not behind this one
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            (slot0(mid) <= slot ? lo : hi) = mid;
        }
        b = lo;
        j = slot - slot0(b);
        if (j < 0) return;
    } else {
        j = (int)(item % blocks_per_row), which = (int)(item / blocks_per_row & 1);
        bh = item / blocks_per_row >> 1;
        b = (int)(bh / c.H_kv), h = (int)(bh % c.H_kv);
        if (b >= a.B) return;                                   // (whole groups leave)
    }

    const int page = 1 << c.page_shift, cap = c.max_pages << c.page_shift;
    const int len_in = c.seq_lens[b];
    int count_in;
    if constexpr (PACKED) {
        count_in = packed_row(rows, b, start);
        if (count_in == 0) return;
    } else {
        count_in = a.n_new ? max(a.n_new[b], 0) : a.n;
    }
    const int len = min(max(len_in, 0), cap), count = min(count_in, a.n);
    const int first = len_in - count;                           // position of the row's token 0 (may be out of range)
    if (lane == 0 && (len_in != len || count_in != count || first < 0)) q8_report(c.status, kStatusBadPage);
    if (count == 0) return;
    const int blk = (max(first, 0) >> c.page_shift) + j;
    const int lo = max(max(first, 0), blk << c.page_shift), hi = min(len, (blk + 1) << c.page_shift);
    if (lo >= hi) return;
    const int pid = c.tables[(size_t)b * c.max_pages + blk];   // (looked at once the new tokens are on their way too)
    const int d = which ? c.d_v : c.d_k, old = lo - (blk << c.page_shift);
    const int units = (hi - lo) * d / 16;
    // unit u: 16 elements of token u / (d / 16) of the block's new ones (below 2^11: the product with 2^20 / (d / 16) rounded up
    // gives the quotient)
    const unsigned per = (unsigned)d / 16, inverse = PACKED ? ((1u << 20) + per - 1) / per : 0;
    const __half *src = which ? a.v_new : a.k_new;
    const long long ts = which ? a.v_ts : a.k_ts;
    if constexpr (PACKED) src += (start + (lo - first)) * ts + h * (which ? a.v_hs : a.k_hs);
    else src += ((size_t)bh * a.n + (lo - first)) * d;
    auto load = [&](int u) {
        if constexpr (PACKED) {
            const unsigned t = (unsigned)u * inverse >> 20;
            return ap_load(reinterpret_cast<const uint4 *>(src + t * ts + (u - t * per) * 16));
        } else {
            return ap_load(reinterpret_cast<const uint4 *>(src) + 2 * u);
        }
    };

    ApUnit keep[kApKeep];
    uint32_t tops2 = 0;
#pragma unroll
    for (int i = 0; i < kApKeep; ++i) {
        const int u = lane + i * THREADS;
        if (u < units) {
            keep[i] = load(u);
            ap_max(tops2, keep[i]);
        }
    }
    for (int u = lane + kApKeep * THREADS; u < units; u += THREADS) ap_max(tops2, load(u));
    uint32_t top = ap_higher(tops2);
    if (pid < 0 || pid >= c.n_pages) {                          // (the same for the whole group)
        if (lane == 0) q8_report(c.status, kStatusBadPage);
        return;
    }
    const size_t block = (size_t)pid * c.H_kv + h;
    uint8_t *base = (which ? c.v : c.k) + block * page * d;
    float *amax_at = (which ? c.v_amax : c.k_amax) + block;
    float was = 0.f;
    if (old > 0) was = fmaxf(*amax_at, 0.f);
    // the group's largest; where that is an infinity or a NaN, the numbers are made finite and it is taken again
    __shared__ uint32_t tops[2][THREADS / 32];
    auto of_group = [&](uint32_t mine, int round) {
        mine = __reduce_max_sync(0xffffffffu, mine);
        if constexpr (THREADS > 32) {
            if ((threadIdx.x & 31) == 0) tops[round][threadIdx.x >> 5] = mine;
            __syncthreads();                                    // (also: everyone has read *amax_at)
#pragma unroll
            for (int i = 0; i < THREADS / 32; ++i) mine = max(mine, tops[round][i]);
        }
        return mine;
    };
    top = of_group(top, 0);
    const bool odd = top >= 0x7c00u;                            // (the same for the whole group)
    if (odd) {
        tops2 = 0;
#pragma unroll
        for (int i = 0; i < kApKeep; ++i)
            if (lane + i * THREADS < units) {
                ap_finite(keep[i]);
                ap_max(tops2, keep[i]);
            }
        for (int u = lane + kApKeep * THREADS; u < units; u += THREADS) {
            ApUnit more = load(u);
            ap_finite(more);
            ap_max(tops2, more);
        }
        top = of_group(ap_higher(tops2), 1);
    }
    const float now = fmaxf(was, __half2float(__ushort_as_half((unsigned short)top)));

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
    for (int u = lane + kApKeep * THREADS; u < units; u += THREADS) {
        ApUnit more = load(u);
        if (odd) ap_finite(more);
        dst[u] = now > 0.f ? ap_round16<FORMAT>(more, now, scale) : make_uint4(0u, 0u, 0u, 0u);
    }
    if constexpr (THREADS == 32) __syncwarp();
    if (lane == 0) *amax_at = now;
}

}  // namespace

lookat_status launch_q8_append(Ctx *ctx, const Q8AppendArgs &a)
{
    const int page = 1 << a.c.page_shift;
    // blocks that n consecutive tokens can touch; packed rows: slots for all rows' blocks
    const int blocks = a.starts ? (a.n >> a.c.page_shift) + 2 * a.B : (a.n + page - 2) / page + 1;
    const long long items = (long long)(a.starts ? 1 : a.B) * a.c.H_kv * 2 * blocks;
    const int d = a.c.d_k > a.c.d_v ? a.c.d_k : a.c.d_v, units = (a.n < page ? a.n : page) * d / 16;     // of the largest group
    const int threads = units <= 32 * kApKeep ? 32 : units <= 128 * kApKeep ? 128 : 256;
    const long long ctas = threads == 32 ? (items + 3) / 4 : items;
    if (ctas > 0x7fffffffll || (a.starts && items > 0x7fffffffll)) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "q8_append: too many blocks for one call");
    auto launch = [&](auto kern) { kern<<<(unsigned)ctas, threads == 32 ? 128 : threads, 0, ctx->stream>>>(a, blocks); };
    auto sized = [&](auto format, auto packed) {
        constexpr int F = decltype(format)::value;
        constexpr bool P = decltype(packed)::value;
        threads == 32 ? launch(q8_append_kernel<F, 32, P>) : threads == 128 ? launch(q8_append_kernel<F, 128, P>) : launch(q8_append_kernel<F, 256, P>);
    };
    using Int8 = std::integral_constant<int, LOOKAT_Q8_INT8>;
    using E4m3 = std::integral_constant<int, LOOKAT_Q8_E4M3>;
    if (a.format == LOOKAT_Q8_INT8) a.starts ? sized(Int8{}, std::true_type{}) : sized(Int8{}, std::false_type{});
    else a.starts ? sized(E4m3{}, std::true_type{}) : sized(E4m3{}, std::false_type{});
    return check_launch(ctx, "q8_append_kernel");
}

}  // namespace lookat
