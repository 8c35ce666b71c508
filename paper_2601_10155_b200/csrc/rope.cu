// lookat_rope: rotary positions of queries and keys.
//
// Pair i of token t turns by the fraction positions[t] * turns[i] mod 2^64 of 2^64: an integer product that wraps where the
// angle does, so a position of 10^6 is as good as one of 10 (an fp32 angle of 10^6 radians is off by 0.03).  The top 32 bits
// go to sincospif as a number of half turns in -1..1.
//
// Bound by HBM: every element is read and written once.  A thread forms the cosines and sines of its pairs once and turns
// those of several heads with them; `each` heads per thread are as many as still leave the GPU full of threads.
#include "serve.cuh"

namespace lookat {

namespace {

enum { kRopeHalves, kRopePairs, kRopeAny };     // 16-byte pieces of both halves, of neighbouring pairs, or single pairs

struct RopePlan {
    int slots, turning;         // pieces of a head that a thread each takes, those of them that turn (the others are copied)
    int each, splits;           // heads per thread, threads per piece
    int inplace[2];
    long long threads;
};

__device__ __forceinline__ float2 rope_turn(unsigned long long turns, int position)
{
    const unsigned long long at = turns * (unsigned long long)(long long)position;
    float2 cs;
    sincospif((float)(int)(at >> 32) * 0x1p-31f, &cs.y, &cs.x);
    return cs;
}
__device__ __forceinline__ void rope_pair(float &x, float &y, float2 cs)
{
    const float a = x, b = y;
    x = a * cs.x - b * cs.y;
    y = b * cs.x + a * cs.y;
}
__device__ __forceinline__ uint32_t rope_half2(float x, float y)
{
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 rope_float2(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

template <int FORM>
__global__ void __launch_bounds__(256) rope_kernel(RopeArgs a, RopePlan p)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    if (id >= p.threads) return;
    long long t;
    int slot, split;
    if (p.threads < 0x7fffffffll) {
        const unsigned u = (unsigned)id, rest = u / (unsigned)p.slots;
        slot = (int)(u % (unsigned)p.slots);
        split = (int)(rest % (unsigned)p.splits);
        t = rest / (unsigned)p.splits;
    } else {
        const long long rest = id / p.slots;
        slot = (int)(id % p.slots);
        split = (int)(rest % p.splits);
        t = rest / p.splits;
    }
    const int head0 = split * p.each, heads = a.heads[0] + a.heads[1], head1 = min(head0 + p.each, heads), c = a.r / 2;
    const bool turns = slot < p.turning;
    auto at = [&](const Rows *rows, int h) {
        const int i = h >= a.heads[0];
        return rows[i].p + t * rows[i].ts + (h - (i ? a.heads[0] : 0)) * rows[i].hs;
    };

    if constexpr (FORM == kRopeAny) {
        const int i = turns ? (a.interleaved ? 2 * slot : slot) : a.r + 2 * (slot - p.turning), j = turns && !a.interleaved ? i + c : i + 1;
        float2 cs = make_float2(1.f, 0.f);
        if (turns) {
            cs = rope_turn(a.turns[slot], a.positions[t]);
            cs.x *= a.amplitude, cs.y *= a.amplitude;
        }
        for (int h = head0; h < head1; ++h) {
            if (!turns && p.inplace[h >= a.heads[0]]) continue;
            const __half *src = at(a.in, h);
            __half *dst = at(a.out, h);
            const __half u = src[i], v = src[j];
            if (!turns) {
                dst[i] = u, dst[j] = v;
                continue;
            }
            float x = __half2float(u), y = __half2float(v);
            rope_pair(x, y, cs);
            dst[i] = __float2half_rn(x), dst[j] = __float2half_rn(y);
        }
        return;
    }
    if (!turns) {
        const int i = a.r + 8 * (slot - p.turning);
        for (int h = head0; h < head1; ++h)
            if (!p.inplace[h >= a.heads[0]]) *reinterpret_cast<uint4 *>(at(a.out, h) + i) = *reinterpret_cast<const uint4 *>(at(a.in, h) + i);
        return;
    }
    constexpr int kPairs = FORM == kRopeHalves ? 8 : 4, kBatch = 4;
    float2 cs[kPairs];
    const int pos = a.positions[t];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        cs[i] = rope_turn(a.turns[slot * kPairs + i], pos);
        cs[i].x *= a.amplitude, cs[i].y *= a.amplitude;
    }
    for (int h0 = head0; h0 < head1; h0 += kBatch) {
        uint4 x[kBatch], y[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (h0 + k >= head1) continue;
            const __half *src = at(a.in, h0 + k) + slot * 8;
            x[k] = *reinterpret_cast<const uint4 *>(src);
            if (FORM == kRopeHalves) y[k] = *reinterpret_cast<const uint4 *>(src + c);
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (h0 + k >= head1) continue;
            uint32_t u[4] = {x[k].x, x[k].y, x[k].z, x[k].w}, v[4] = {y[k].x, y[k].y, y[k].z, y[k].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 m = rope_float2(u[i]);
                if constexpr (FORM == kRopeHalves) {
                    float2 n = rope_float2(v[i]);
                    rope_pair(m.x, n.x, cs[2 * i]);
                    rope_pair(m.y, n.y, cs[2 * i + 1]);
                    v[i] = rope_half2(n.x, n.y);
                } else {
                    rope_pair(m.x, m.y, cs[i]);
                }
                u[i] = rope_half2(m.x, m.y);
            }
            __half *dst = at(a.out, h0 + k) + slot * 8;
            *reinterpret_cast<uint4 *>(dst) = make_uint4(u[0], u[1], u[2], u[3]);
            if (FORM == kRopeHalves) *reinterpret_cast<uint4 *>(dst + c) = make_uint4(v[0], v[1], v[2], v[3]);
        }
    }
}

}  // namespace

lookat_status launch_rope(Ctx *ctx, const RopeArgs &a)
{
    // whole 16-byte pieces where the halves (or the pairs) and what follows them begin on such borders
    const int form = a.interleaved ? (a.r % 8 == 0 ? kRopePairs : kRopeAny) : (a.r % 16 == 0 ? kRopeHalves : kRopeAny);
    RopePlan p;
    bool copies = false;
    for (int i = 0; i < 2; ++i) {
        p.inplace[i] = a.in[i].p == a.out[i].p && a.in[i].ts == a.out[i].ts && a.in[i].hs == a.out[i].hs;
        copies |= a.heads[i] > 0 && !p.inplace[i];
    }
    p.turning = form == kRopeHalves ? a.r / 16 : form == kRopePairs ? a.r / 8 : a.r / 2;
    p.slots = p.turning + (copies ? (a.d - a.r) / (form == kRopeAny ? 2 : 8) : 0);
    const int heads = a.heads[0] + a.heads[1];
    const long long full = (long long)ctx->sm_count * 2048;    // resident threads
    for (p.each = 16; p.each > 1 && a.n * p.slots * ((heads + p.each - 1) / p.each) < 2 * full;) p.each /= 2;
    p.splits = (heads + p.each - 1) / p.each;
    p.threads = a.n * p.slots * p.splits;
    const long long ctas = (p.threads + 255) / 256;
    if (ctas > 0x7fffffffll) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "rope: too many tokens for one call");
    if (form == kRopeHalves) rope_kernel<kRopeHalves><<<(unsigned)ctas, 256, 0, ctx->stream>>>(a, p);
    else if (form == kRopePairs) rope_kernel<kRopePairs><<<(unsigned)ctas, 256, 0, ctx->stream>>>(a, p);
    else rope_kernel<kRopeAny><<<(unsigned)ctas, 256, 0, ctx->stream>>>(a, p);
    return check_launch(ctx, "rope_kernel");
}

}  // namespace lookat
