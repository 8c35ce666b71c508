// lookat_rope: rotary positions of queries and keys.
//
// Pair i of token t turns by the fraction positions[t] * turns[i] mod 2^64 of 2^64: an integer product that wraps where the
// angle does, so a position of 10^6 is as good as one of 10 (an fp32 angle of 10^6 radians is off by 0.03).  The top 32 bits
// go to sincospif as a number of half turns in -1..1.
//
// Bound by HBM: every element is read and written once.  A lane takes one 16-byte piece of several heads of a token: it forms
// the cosines and sines of its pairs once, and has the other half of a pair from the lane that holds it (a lane that took both
// halves itself left the lanes of a partial rotary part apart: 16384 tokens, 32 and 8 heads of 128, 64 dims rotated, 95 us; 64 so).
// `each` heads per lane are as many as still leave the GPU a quarter full of threads: the same tokens with all 128 dims rotated
// 61 us (5.5 TB/s) with 20 of the 40 heads, 66 with 8; 4096 tokens 17 us.
#include "serve.cuh"

namespace lookat {

namespace {

// pieces with pairs half a rotary part apart, pieces of neighbouring pairs; halves that do not begin on pieces' borders, or of more than
// a warp's pieces, two elements at a time
enum { kRopeHalves, kRopePairs, kRopeAny };

struct RopePlan {
    int lanes;                  // per token and split: pieces of a head (kRopeHalves: up to a power of two; kRopeAny: two elements each)
    int each, splits;           // heads per lane, lanes per piece
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
__device__ __forceinline__ uint32_t rope_half2(float x, float y)
{
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 rope_float2(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

template <int FORM>
__global__ void __launch_bounds__(256) rope_kernel(RopeArgs a, RopePlan p)
{
    const long long id_in = (long long)blockIdx.x * 256 + threadIdx.x, id = id_in < p.threads ? id_in : p.threads - 1;
    long long t;
    int at, split;
    if (p.threads < 0x7fffffffll) {
        const unsigned rest = (unsigned)id / (unsigned)p.lanes;
        at = (int)((unsigned)id % (unsigned)p.lanes);
        split = (int)(rest % (unsigned)p.splits);
        t = rest / (unsigned)p.splits;
    } else {
        const long long rest = id / p.lanes;
        at = (int)(id % p.lanes);
        split = (int)(rest % p.splits);
        t = rest / p.splits;
    }
    const int head0 = split * p.each, heads = a.heads[0] + a.heads[1], head1 = min(head0 + p.each, heads), c = a.r / 2;
    auto vector = [&](const Rows *rows, int h) {
        const int i = h >= a.heads[0];
        return rows[i].p + t * rows[i].ts + (h - (i ? a.heads[0] : 0)) * rows[i].hs;
    };
    auto pair = [&](int i) {                                   // amplitude times cosine and sine
        float2 cs = rope_turn(a.turns[i], a.positions[t]);
        cs.x *= a.amplitude, cs.y *= a.amplitude;
        return cs;
    };

    if constexpr (FORM == kRopeAny) {
        if (id != id_in) return;
        const bool turns = at < c;
        const float2 cs = turns ? pair(at) : make_float2(1.f, 0.f);
        constexpr int kBatch = 4;
        for (int h0 = head0; h0 < head1; h0 += kBatch) {
            __half u[kBatch], v[kBatch];
            uint32_t w[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (h0 + k >= head1) continue;
                const __half *src = vector(a.in, h0 + k);
                if (turns) u[k] = src[at], v[k] = src[at + c];
                else w[k] = *reinterpret_cast<const uint32_t *>(src + 2 * at);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (h0 + k >= head1) continue;
                __half *dst = vector(a.out, h0 + k);
                if (turns) {
                    const float x = __half2float(u[k]), y = __half2float(v[k]);
                    dst[at] = __float2half_rn(x * cs.x - y * cs.y), dst[at + c] = __float2half_rn(y * cs.x + x * cs.y);
                } else if (!p.inplace[h0 + k >= a.heads[0]]) {
                    *reinterpret_cast<uint32_t *>(dst + 2 * at) = w[k];
                }
            }
        }
    } else {
        constexpr int kPairs = FORM == kRopeHalves ? 8 : 4, kBatch = 4;         // kBatch: heads whose loads are in flight together
        // the lane's piece: in the first half, in the second, or behind the rotary part
        const bool on = id == id_in && at < a.d / 8, turns = at * 8 < a.r, second = FORM == kRopeHalves && at >= c / 8;
        const int lane = threadIdx.x & 31, other = FORM == kRopeHalves && turns ? (second ? lane - c / 8 : lane + c / 8) : lane;
        float cosine[kPairs], sine[kPairs];                    // sine: with the sign that it has in this half
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (FORM == kRopeHalves) {               // the two lanes of the same pairs form four each
                const float2 own = turns ? pair((second ? at - c / 8 : at) * 8 + (second ? 4 : 0) + i) : make_float2(1.f, 0.f);
                const float2 had = make_float2(__shfl_sync(0xffffffffu, own.x, other), __shfl_sync(0xffffffffu, own.y, other));
                cosine[i] = second ? had.x : own.x, sine[i] = second ? had.y : -own.y;
                cosine[4 + i] = second ? own.x : had.x, sine[4 + i] = second ? own.y : -had.y;
            } else {
                const float2 own = at * 8 + 2 * i < a.r ? pair(at * 4 + i) : make_float2(1.f, 0.f);
                cosine[i] = own.x, sine[i] = own.y;
            }
        }
        for (int k0 = 0; k0 < p.each; k0 += kBatch) {          // (the same for all lanes: they exchange)
            uint4 x[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                x[k] = make_uint4(0u, 0u, 0u, 0u);
                if (on && head0 + k0 + k < head1) x[k] = *reinterpret_cast<const uint4 *>(vector(a.in, head0 + k0 + k) + at * 8);
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int h = head0 + k0 + k;
                uint32_t u[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 m = rope_float2(u[i]);
                    if constexpr (FORM == kRopeHalves) {
                        const float2 n = rope_float2(__shfl_sync(0xffffffffu, u[i], other));
                        if (turns) u[i] = rope_half2(fmaf(m.x, cosine[2 * i], n.x * sine[2 * i]), fmaf(m.y, cosine[2 * i + 1], n.y * sine[2 * i + 1]));
                    } else {
                        if (at * 8 + 2 * i < a.r) u[i] = rope_half2(fmaf(m.x, cosine[i], -m.y * sine[i]), fmaf(m.y, cosine[i], m.x * sine[i]));
                    }
                }
                if (on && h < head1 && (turns || !p.inplace[h >= a.heads[0]]))
                    *reinterpret_cast<uint4 *>(vector(a.out, h) + at * 8) = make_uint4(u[0], u[1], u[2], u[3]);
            }
        }
    }
}

}  // namespace

lookat_status launch_rope(Ctx *ctx, const RopeArgs &a)
{
    const int form = a.interleaved ? kRopePairs : a.d <= 256 && a.r % 16 == 0 ? kRopeHalves : kRopeAny;
    RopePlan p;
    for (int i = 0; i < 2; ++i) p.inplace[i] = a.in[i].p == a.out[i].p && a.in[i].ts == a.out[i].ts && a.in[i].hs == a.out[i].hs;
    p.lanes = a.d / 8;
    if (form == kRopeHalves) for (p.lanes = 1; p.lanes < a.d / 8;) p.lanes *= 2;
    if (form == kRopeAny) p.lanes = a.d / 2;
    const int heads = a.heads[0] + a.heads[1];
    const long long full = (long long)ctx->sm_count * 2048;    // resident threads
    for (p.each = 32; p.each > 1 && 4 * a.n * p.lanes * ((heads + p.each - 1) / p.each) < full;) p.each /= 2;
    p.splits = (heads + p.each - 1) / p.each;
    p.each = (heads + p.splits - 1) / p.splits;
    p.threads = a.n * p.lanes * p.splits;
    const long long ctas = (p.threads + 255) / 256;
    if (ctas > 0x7fffffffll) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "rope: too many tokens for one call");
    if (form == kRopeHalves) rope_kernel<kRopeHalves><<<(unsigned)ctas, 256, 0, ctx->stream>>>(a, p);
    else if (form == kRopePairs) rope_kernel<kRopePairs><<<(unsigned)ctas, 256, 0, ctx->stream>>>(a, p);
    else rope_kernel<kRopeAny><<<(unsigned)ctas, 256, 0, ctx->stream>>>(a, p);
    return check_launch(ctx, "rope_kernel");
}

}  // namespace lookat
