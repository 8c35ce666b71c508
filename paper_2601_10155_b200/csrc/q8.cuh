// Internal declarations of the 8-bit paged cache (include/lookat_q8.h): argument blocks, workspaces, the arithmetic of
// the stored numbers.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "lookat_q8.h"

namespace lookat {

constexpr int kStatusBadPage = 4;           // a page id, a length or a count outside its range was met and left out
constexpr int kStatusNoPages = 8;           // lookat_pages_extend found too few pages and changed nothing

constexpr float kQ8RangeInt8 = 127.f, kQ8RangeE4m3 = 448.f;

// The attention's running exponent M follows the largest score + log2 amax^V, so that the fp16 weights serve blocks of any
// size.  A block of zero values (amax 0) counts in the softmax's denominator l but adds nothing to the sum: with an exponent
// far below every real one (fp16 amax: -24 to 16) it does not push the other blocks' weights out of fp16's range.  Its weights
// are lost to l only where they are below 2^-46 of the largest (2^-126 is the least fp32 weight), and l stays below 2^110.
// With an exponent of 0, one such block among values of 1e-4 made the result 1.5e-4 wrong, among values of 1e-5 1.6e-3.
constexpr float kQ8ZeroExponent = -64.f, kQ8ZeroInverse = 0x1p64f;

// Where the tokens of the cache are, as the kernels take it.
struct Q8View {
    uint8_t *k, *v;
    float *k_amax, *v_amax;
    const int32_t *tables;      // [B][max_pages]
    const int32_t *seq_lens;    // [B]
    int n_pages, max_pages, page_shift, H_kv, d_k, d_v;
    int *status;
};

__device__ __forceinline__ void q8_report(int *status, int bit)
{
    if (status) atomicOr(status, bit);
}

struct Q8AppendArgs {
    Q8View c;
    const __half *k_new, *v_new;    // [B][H_kv][n][d]
    const int32_t *n_new;           // [B] or null
    int B, n, format;
    // packed rows (lookat_q8_append_packed): row b's new tokens are starts[b] .. starts[b + 1] - 1 of n, their vectors
    // ts elements apart by tokens and hs by heads
    const int32_t *starts;          // [B + 1], or null
    long long k_ts, k_hs, v_ts, v_hs;
};
lookat_status launch_q8_append(Ctx *ctx, const Q8AppendArgs &a);

struct Q8AttendArgs {
    Q8View c;
    const __half *q;                // [B][H_q][L_q][d_k]
    void *out;                      // [B][H_q][L_q][d_v], fp32 or fp16
    int out_fp16, B, H_q, g, L_q, format;
    float scale_log2;               // softmax scale * log2(e)
};
lookat_status launch_attend_q8(Ctx *ctx, const Q8AttendArgs &a);
// prompts and pieces of them, on tcgen05 (attend_q8_umma.cu)
bool attend_q8_umma_covers(const Ctx *ctx, const Q8AttendArgs &a);
lookat_status launch_attend_q8_umma(Ctx *ctx, const Q8AttendArgs &a);

// Scratch of at least `bytes` (zeroed when it is new, if asked).  Grows by allocating anew; the old buffer stays until the
// context is destroyed, because a captured graph may still name it.  Refuses to allocate while the stream is captured.
lookat_status workspace(Ctx *ctx, Workspace &w, size_t bytes, bool zeroed, const char *what);

// Launches a kernel that may start while the one before it on the stream still runs: that one has called pdl_release() and
// this one calls pdl_wait() before it touches anything the other writes.  Saves the launch latency between the two halves
// of a call (1 to 2 us).
template <class... P, class... A>
cudaError_t launch_after(Ctx *ctx, void (*kernel)(P...), unsigned grid, unsigned block, size_t smem, A &&...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// one 8-bit number nearest to x (ties to even; |x| <= R up to rounding), as its byte
template <int FORMAT>
__device__ __forceinline__ uint32_t q8_round(float x)
{
    if constexpr (FORMAT == LOOKAT_Q8_INT8) {
        return (uint32_t)__float2int_rn(fminf(fmaxf(x, -127.f), 127.f)) & 0xffu;
    } else {
        return (uint32_t)__nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3);
    }
}
// the number a byte holds
template <int FORMAT>
__device__ __forceinline__ float q8_value(uint32_t byte)
{
    if constexpr (FORMAT == LOOKAT_Q8_INT8) {
        return (float)(int)(int8_t)(uint8_t)byte;
    } else {
        // sign, 4 exponent and 3 fraction bits moved to the same places of an fp16: the value comes out 2^8 too small
        // (exponent biases 7 and 15), for subnormals as well
        const uint32_t h = ((byte & 0x80u) << 8) | ((byte & 0x7fu) << 7);
        return __half2float(__ushort_as_half((unsigned short)h)) * 256.f;
    }
}

// Four stored numbers as two pairs of fp16 numbers, in order.  int8: with the sign bit flipped a byte u stands for u - 128,
// and the half 0x6400 + u is 1024 + u, so one exact subtraction gives n (5 instructions per 4 numbers).  e4m3: the
// conversion instruction (moving the bits into an fp16's places by hand takes 8 instructions per 4 numbers; 32768-token
// rows took 277 us with it and 242 with the conversion, in the kernel of that day).  A NaN stays one.
template <int FORMAT>
__device__ __forceinline__ void q8_pairs(uint32_t w, uint32_t &lo, uint32_t &hi)       // bytes 0, 1 and 2, 3
{
    if constexpr (FORMAT == LOOKAT_Q8_INT8) {
        const uint32_t u = w ^ 0x80808080u;
        const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
        const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), off), y = __hsub2(*reinterpret_cast<const __half2 *>(&b), off);
        lo = *reinterpret_cast<const uint32_t *>(&x);
        hi = *reinterpret_cast<const uint32_t *>(&y);
    } else {
        asm("{\n.reg .b16 x, y;\nmov.b32 {x, y}, %2;\ncvt.rn.f16x2.e4m3x2 %0, x;\ncvt.rn.f16x2.e4m3x2 %1, y;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
    }
}
// Two fp16 results.  A weighted mean of values lies among them, within fp16's range, but the rounded weights of a prompt can
// put it up to 2^-11 above: what passes 65504 is 65504, not infinity (a NaN stays one).
__device__ __forceinline__ uint32_t q8_half2(float x, float y)
{
    uint32_t d;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %2, %1;" : "=r"(d) : "f"(x), "f"(y));
    return d;
}
template <int FORMAT>
constexpr float kQ8Unit = 1.f / (FORMAT == LOOKAT_Q8_INT8 ? kQ8RangeInt8 : kQ8RangeE4m3);      // value of a number per amax

}  // namespace lookat
