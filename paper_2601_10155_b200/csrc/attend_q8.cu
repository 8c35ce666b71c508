// lookat_attend_q8: softmax attention over the 8-bit paged cache.
//
// s_t = (q . n^K_t) amax^K / R * scale, o = sum_t alpha_t n^V_t amax^V / R, alpha = softmax over the tokens a query sees.
// One CTA per (row, query head, query): tiles of 128 tokens, one thread per token for the scores, one per value dim for
// the sum.
#include "q8.cuh"

namespace lookat {

namespace {

constexpr int kAqThreads = 128;

__device__ __forceinline__ float aq_block_max(float x, float *s)
{
    for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    x = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    __syncthreads();
    return x;
}
__device__ __forceinline__ float aq_block_sum(float x, float *s)
{
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    x = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    return x;
}

template <int FORMAT>
__global__ void __launch_bounds__(kAqThreads) attend_q8_simple_kernel(Q8AttendArgs a)
{
    __shared__ float qs[256], ws[kAqThreads], red[4];
    __shared__ int pages_s[kAqThreads];
    const Q8View &c = a.c;
    const int i = blockIdx.x % a.L_q, hq = blockIdx.x / a.L_q, b = blockIdx.y, h = hq / a.g, tid = threadIdx.x;
    const int page = 1 << c.page_shift;
    const int len_in = c.seq_lens[b], len = min(max(len_in, 0), c.max_pages << c.page_shift);
    if (tid == 0 && len != len_in) q8_report(c.status, kStatusBadPage);
    const int seen = len - a.L_q + i + 1;
    const size_t row = ((size_t)b * a.H_q + hq) * a.L_q + i;
    for (int k = tid; k < c.d_k; k += kAqThreads) qs[k] = __half2float(a.q[row * c.d_k + k]);
    constexpr float kInvR = 1.f / (FORMAT == LOOKAT_Q8_INT8 ? kQ8RangeInt8 : kQ8RangeE4m3);
    float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
    __syncthreads();
    for (int t0 = 0; t0 < seen; t0 += kAqThreads) {
        const int t = t0 + tid;
        float s = -INFINITY;
        int pid = -1;
        if (t < seen) {
            pid = c.tables[(size_t)b * c.max_pages + (t >> c.page_shift)];
            if (pid < 0 || pid >= c.n_pages) {
                q8_report(c.status, kStatusBadPage);
                pid = -1;
            }
        }
        if (pid >= 0) {
            const size_t block = (size_t)pid * c.H_kv + h;
            const uint4 *k = reinterpret_cast<const uint4 *>(c.k + (block * page + (t & (page - 1))) * c.d_k);
            float dot = 0.f;
            for (int x = 0; x < c.d_k / 16; ++x) {
                const uint4 u = k[x];
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int y = 0; y < 16; ++y) dot = fmaf(qs[x * 16 + y], q8_value<FORMAT>((w[y >> 2] >> (8 * (y & 3))) & 0xffu), dot);
            }
            s = dot * (c.k_amax[block] * kInvR * a.scale_log2);
        }
        const float top = fmaxf(m, aq_block_max(s, red));
        const float keep = top == -INFINITY ? 1.f : exp2f(m - top);
        const float w = s == -INFINITY ? 0.f : exp2f(s - top);
        l = l * keep + aq_block_sum(w, red);
        m = top;
        pages_s[tid] = pid;
        ws[tid] = pid < 0 ? 0.f : w * (c.v_amax[(size_t)pid * c.H_kv + h] * kInvR);
        __syncthreads();
        o[0] *= keep;
        o[1] *= keep;
        for (int y = 0; y < min(kAqThreads, seen - t0); ++y) {
            if (pages_s[y] < 0) continue;
            const uint8_t *v = c.v + (((size_t)pages_s[y] * c.H_kv + h) * page + ((t0 + y) & (page - 1))) * c.d_v;
            if (tid < c.d_v) o[0] = fmaf(ws[y], q8_value<FORMAT>(v[tid]), o[0]);
            if (tid + kAqThreads < c.d_v) o[1] = fmaf(ws[y], q8_value<FORMAT>(v[tid + kAqThreads]), o[1]);
        }
        __syncthreads();
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    for (int k = 0; k < 2; ++k) {
        const int dim = tid + k * kAqThreads;
        if (dim >= c.d_v) break;
        if (a.out_fp16) static_cast<__half *>(a.out)[row * c.d_v + dim] = __float2half_rn(o[k] * inv);
        else static_cast<float *>(a.out)[row * c.d_v + dim] = o[k] * inv;
    }
}

}  // namespace

lookat_status launch_attend_q8(Ctx *ctx, const Q8AttendArgs &a)
{
    const long long x = (long long)a.H_q * a.L_q;
    if (x > 0x7fffffffll) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "attend_q8: too many queries for one call");
    dim3 grid((unsigned)x, (unsigned)a.B);
    if (a.format == LOOKAT_Q8_INT8) attend_q8_simple_kernel<LOOKAT_Q8_INT8><<<grid, kAqThreads, 0, ctx->stream>>>(a);
    else attend_q8_simple_kernel<LOOKAT_Q8_E4M3><<<grid, kAqThreads, 0, ctx->stream>>>(a);
    return check_launch(ctx, "attend_q8_simple_kernel");
}

}  // namespace lookat
