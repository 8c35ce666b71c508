// lookat_attend_packed for any head dims (multiples of 16 up to 256): exact causal attention of packed prompts.
//
// A line is one (token, query head) pair of a KV head, line = token * g + head, so that a tile's lines share the keys they see.
// A CTA has 64 lines of one row and KV head, 16 per warp, against blocks of 64 tokens in shared memory; both products on
// mma.sync.m16n8k16 (fp16 in, fp32 accumulate), the softmax with a running exponent in between.  Dims are padded with zeros to
// DIM in shared memory.  The sum is over the weights as they are rounded for the second product, so that what the values have in
// common is not touched by their rounding (96 dims, 4 x 1024 tokens: 91 us, as over the unrounded ones; by conversions back from
// fp16 104).  Head dims of 64 and 128 go to attend_packed_umma.cu, but for short rows: 4 x 4096 tokens, 32 and 8 heads of
// 128, take 2.5 ms here and 0.53 there.  Bound by the issue of the products: one barrier pair, one softmax and 16 to 64 products of
// 16 x 8 x 16 per warp and 16 dims of a block, with nothing in flight meanwhile: 4 x 1024 tokens, 16 and 4 heads of 16 to 48 dims 54 us,
// of 80 to 112 91, of 144 to 256 186 to 205 (of 64 and 128 on the other form 32 and 35).
#include "serve.cuh"

namespace lookat {

namespace {

constexpr int kPaLines = 64, kPaBlock = 64, kPaThreads = 128;

__device__ __forceinline__ void pa_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int DIM>
__global__ void __launch_bounds__(kPaThreads) attend_packed_kernel(PackedAttendArgs a)
{
    constexpr int kPitch = DIM + 8;                            // halfs per row: fragment reads without bank conflicts
    extern __shared__ __align__(16) __half pa_smem[];
    __half *const qs = pa_smem, *const ks = qs + kPaLines * kPitch, *const vs = ks + kPaBlock * kPitch;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, t = lane & 3;
    const int h = blockIdx.x % a.H_kv;
    int place, first, n;
    if (blockIdx.x == 0) packed_check(a.rows, tid, kPaThreads);
    if (packed_tile(a.rows, a.g, kPaLines, blockIdx.x / a.H_kv, lane, place, first, n) != kTile) return;
    const int line0 = place * kPaLines, lines = n * a.g;       // (the host sees to it that lines fit 31 bits)
    const __half *const kg = a.k.p + first * a.k.ts + h * a.k.hs, *const vg = a.v.p + first * a.v.ts + h * a.v.hs;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);

    for (int i = tid; i < kPaLines * (DIM / 8); i += kPaThreads) {
        const int l = i / (DIM / 8), c = i % (DIM / 8) * 8, line = min(line0 + l, lines - 1);
        const __half *src = a.q.p + (first + line / a.g) * a.q.ts + (h * a.g + line % a.g) * a.q.hs + c;
        *reinterpret_cast<uint4 *>(qs + l * kPitch + c) = c < a.d_k ? *reinterpret_cast<const uint4 *>(src) : zero;
    }
    float o[DIM / 8][4];
#pragma unroll
    for (int i = 0; i < DIM / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    const int mine = line0 + warp * 16 + r;                    // this thread's lines: mine and mine + 8
    const int last0 = min(mine, lines - 1) / a.g, last1 = min(mine + 8, lines - 1) / a.g;      // the tokens they see last
    float m0 = 0.f, m1 = 0.f, l0 = 0.f, l1 = 0.f;
    bool set = false;
    const int tokens = (min(line0 + kPaLines, lines) - 1) / a.g + 1;

    for (int t0 = 0; t0 < tokens; t0 += kPaBlock) {
        __syncthreads();
        for (int i = tid; i < kPaBlock * (DIM / 8); i += kPaThreads) {
            const int row = i / (DIM / 8), c = i % (DIM / 8) * 8, tok = t0 + row;
            *reinterpret_cast<uint4 *>(ks + row * kPitch + c) = tok < n && c < a.d_k ? *reinterpret_cast<const uint4 *>(kg + tok * a.k.ts + c) : zero;
            *reinterpret_cast<uint4 *>(vs + row * kPitch + c) = tok < n && c < a.d_v ? *reinterpret_cast<const uint4 *>(vg + tok * a.v.ts + c) : zero;
        }
        __syncthreads();
        float s[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll 4
        for (int kk = 0; kk < DIM / 16; ++kk) {
            const __half *qr = qs + (warp * 16 + r) * kPitch + kk * 16 + 2 * t;
            const uint32_t qa[4] = {*reinterpret_cast<const uint32_t *>(qr), *reinterpret_cast<const uint32_t *>(qr + 8 * kPitch),
                                    *reinterpret_cast<const uint32_t *>(qr + 8), *reinterpret_cast<const uint32_t *>(qr + 8 * kPitch + 8)};
#pragma unroll
            for (int nt = 0; nt < 8; ++nt) {
                const __half *kr = ks + (nt * 8 + r) * kPitch + kk * 16 + 2 * t;
                pa_mma(s[nt], qa, *reinterpret_cast<const uint32_t *>(kr), *reinterpret_cast<const uint32_t *>(kr + 8));
            }
        }
        float top0 = -INFINITY, top1 = -INFINITY;
#pragma unroll
        for (int nt = 0; nt < 8; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int tok = t0 + nt * 8 + 2 * t + (i & 1);
                const float x = tok <= (i < 2 ? last0 : last1) ? s[nt][i] * a.scale_log2 : -INFINITY;
                s[nt][i] = x;
                if (i < 2) top0 = fmaxf(top0, x); else top1 = fmaxf(top1, x);
            }
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
            top0 = fmaxf(top0, __shfl_xor_sync(0xffffffffu, top0, d));
            top1 = fmaxf(top1, __shfl_xor_sync(0xffffffffu, top1, d));
        }
        // (the first block has every line's first token: M is set there)
        const float n0 = set ? fmaxf(m0, top0 - kPackedLift) : top0 - kPackedLift, n1 = set ? fmaxf(m1, top1 - kPackedLift) : top1 - kPackedLift;
        const float f0 = set ? ex2_approx(m0 - n0) : 0.f, f1 = set ? ex2_approx(m1 - n1) : 0.f;
        m0 = n0, m1 = n1, set = true;
        uint32_t w[4][4];
        float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = ex2_approx(s[nt][i] - (i < 2 ? n0 : n1));
                e[i] = fmaf(x, -8192.f, fmaf(x, 8192.f, x));   // to 11 bits: the first sum is rounded 13 bits above x's last
            }
            sum0 += e[0] + e[1];
            sum1 += e[2] + e[3];
            const __half2 h01 = __floats2half2_rn(e[0], e[1]), h23 = __floats2half2_rn(e[2], e[3]);
            w[nt >> 1][(nt & 1) * 2] = *reinterpret_cast<const uint32_t *>(&h01);
            w[nt >> 1][(nt & 1) * 2 + 1] = *reinterpret_cast<const uint32_t *>(&h23);
        }
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
            sum0 += __shfl_xor_sync(0xffffffffu, sum0, d);
            sum1 += __shfl_xor_sync(0xffffffffu, sum1, d);
        }
        l0 = l0 * f0 + sum0;
        l1 = l1 * f1 + sum1;
#pragma unroll
        for (int i = 0; i < DIM / 8; ++i) { o[i][0] *= f0; o[i][1] *= f0; o[i][2] *= f1; o[i][3] *= f1; }
#pragma unroll
        for (int kt = 0; kt < kPaBlock / 16; ++kt)
#pragma unroll
            for (int dt = 0; dt < DIM / 8; ++dt) {
                uint32_t b0, b1;
                const unsigned at = (unsigned)__cvta_generic_to_shared(vs + (kt * 16 + (lane & 15)) * kPitch + dt * 8);
                asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(b0), "=r"(b1) : "r"(at) : "memory");
                pa_mma(o[dt], w[kt], b0, b1);
            }
    }
    const float i0 = 1.f / l0, i1 = 1.f / l1;                  // (every line has seen its own token)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int line = mine + 8 * half;
        if (line >= lines) continue;
        __half *dst = a.out.p + (first + line / a.g) * a.out.ts + (h * a.g + line % a.g) * a.out.hs + 2 * t;
        const float inv = half ? i1 : i0;
#pragma unroll
        for (int dt = 0; dt < DIM / 8; ++dt)
            if (dt * 8 < a.d_v) *reinterpret_cast<uint32_t *>(dst + dt * 8) = q8_half2(o[dt][2 * half] * inv, o[dt][2 * half + 1] * inv);
    }
}

template <int DIM>
lookat_status launch_pa(Ctx *ctx, const PackedAttendArgs &a)
{
    constexpr int kBytes = (kPaLines + 2 * kPaBlock) * (DIM + 8) * 2;
    auto kern = attend_packed_kernel<DIM>;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes) != cudaSuccess)
        return check_launch(ctx, "attend_packed: shared-memory opt-in");
    const long long ctas = packed_tiles(a.rows, a.g, kPaLines) * a.H_kv;
    if (ctas > 0x7fffffffll) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "attend_packed: too many tokens for one call");
    kern<<<(unsigned)ctas, kPaThreads, kBytes, ctx->stream>>>(a);
    return check_launch(ctx, "attend_packed_kernel");
}

}  // namespace

lookat_status launch_attend_packed_any(Ctx *ctx, const PackedAttendArgs &a)
{
    const int dim = a.d_k > a.d_v ? a.d_k : a.d_v;
    return dim <= 64 ? launch_pa<64>(ctx, a) : dim <= 128 ? launch_pa<128>(ctx, a) : launch_pa<256>(ctx, a);
}

lookat_status launch_attend_packed(Ctx *ctx, const PackedAttendArgs &a)
{
    if ((long long)a.rows.n * a.g >= (1ll << 31) - 1024) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "attend_packed: too many tokens for one call");
    return attend_packed_umma_covers(ctx, a) ? launch_attend_packed_umma(ctx, a) : launch_attend_packed_any(ctx, a);
}

}  // namespace lookat
