// C entry points of what a server runs around the 8-bit paged cache (include/lookat_serve.h): argument checks and dispatch.
#include <cmath>
#include <cstring>

#include "q8_checks.cuh"
#include "serve.cuh"

namespace lookat {

namespace {

constexpr int64_t kMaxTokens = 1ll << 30;
// With lengths below 2^31 a norm is at most 2^868, so that the rank of the smallest fp32 score, 2^-149, is still a normal fp64
// number, and the score is what the rank times the norm is, to 2^-52.
constexpr double kMaxPenalty = 28.0;

// fp16 vectors of n tokens and `heads` heads
lookat_status rows_of(Ctx *ctx, const lookat_rows *r, int64_t n, int heads, const char *name, Rows *out)
{
    if (!r) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "%s is NULL", name);
    out->p = static_cast<__half *>(r->data);
    out->ts = n > 1 ? r->token_stride : 0;
    out->hs = heads > 1 ? r->head_stride : 0;
    if (n > 0) Q8_TRY(need(ctx, r->data, name));
    const int64_t top = 1ll << 31;
    if (n > 1 && (out->ts <= 0 || out->ts % 8 || out->ts >= top))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "%s: token_stride=%lld is not a positive multiple of 8 below 2^31", name, (long long)out->ts);
    if (heads > 1 && (out->hs <= 0 || out->hs % 8 || out->hs >= top))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "%s: head_stride=%lld is not a positive multiple of 8 below 2^31", name, (long long)out->hs);
    return LOOKAT_OK;
}

// rows that are written do not overlap themselves: heads lie within tokens, or tokens within heads
lookat_status apart(Ctx *ctx, const Rows &r, int64_t n, int heads, int d, const char *name)
{
    const int64_t ts = r.ts, hs = r.hs;
    const bool tokens_outside = (heads < 2 || hs >= d) && (n < 2 || ts >= (heads < 2 ? d : (heads - 1) * hs + d));
    const bool heads_outside = (n < 2 || ts >= d) && (heads < 2 || hs >= (n < 2 ? d : (n - 1) * ts + d));
    if (tokens_outside || heads_outside) return LOOKAT_OK;
    return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "%s: vectors of %d elements at strides %lld and %lld: tokens lie neither within heads nor around them", name, d, (long long)ts, (long long)hs);
}

lookat_status packed_of(Ctx *ctx, int64_t n_tokens, int32_t B, const int32_t *starts, Packed *out)
{
    if (n_tokens < 0 || n_tokens >= kMaxTokens) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "n_tokens=%lld out of range 0..2^30-1", (long long)n_tokens);
    if (B < 1 || B > 65535) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "B=%d out of range 1..65535", (int)B);
    Q8_TRY(need(ctx, starts, "starts", 4));
    out->starts = starts;
    out->B = B;
    out->n = (int)n_tokens;
    out->status = ctx->status_word;
    return LOOKAT_OK;
}

}  // namespace
}  // namespace lookat

using namespace lookat;

extern "C" {

lookat_status lookat_rope_table(const lookat_rope_config *cfg, uint64_t *turns, float *amplitude)
{
    if (!cfg || !turns || !amplitude) return LOOKAT_ERR_INVALID_ARG;
    const lookat_rope_config &c = *cfg;
    const int r = c.rotary_dim;
    const bool spread = c.scaling == LOOKAT_ROPE_BANDS || c.scaling == LOOKAT_ROPE_RAMP;
    if (r < 2 || r > 1024 || r % 2 || c.scaling < LOOKAT_ROPE_NONE || c.scaling > LOOKAT_ROPE_RAMP) return LOOKAT_ERR_INVALID_ARG;
    if (!(c.base > 1.0) || !std::isfinite(c.base)) return LOOKAT_ERR_INVALID_ARG;
    if (c.scaling != LOOKAT_ROPE_NONE && (!(c.factor >= 1.0) || !std::isfinite(c.factor))) return LOOKAT_ERR_INVALID_ARG;
    if (c.scaling == LOOKAT_ROPE_BASE && r < 4) return LOOKAT_ERR_INVALID_ARG;
    if (spread && (!(c.original_len > 0) || !(c.low > 0) || !(c.high > c.low) || !std::isfinite(c.high) || !std::isfinite(c.original_len)))
        return LOOKAT_ERR_INVALID_ARG;
    const long double pi = 3.14159265358979323846264338327950288L, base = c.base, factor = c.factor, len = c.original_len;
    const long double b = c.scaling == LOOKAT_ROPE_BASE ? base * powl(factor, (long double)r / (r - 2)) : base;
    long double i0 = 0, i1 = 0;
    if (c.scaling == LOOKAT_ROPE_RAMP) {
        i0 = fmaxl(floorl(r * logl(len / (2 * pi * c.high)) / (2 * logl(base))), 0);
        i1 = fminl(ceill(r * logl(len / (2 * pi * c.low)) / (2 * logl(base))), r - 1);
    }
    for (int i = 0; i < r / 2; ++i) {
        long double f = powl(b, -2.0L * i / r);
        if (c.scaling == LOOKAT_ROPE_LINEAR) f /= factor;
        if (spread) {
            const long double along = c.scaling == LOOKAT_ROPE_BANDS ? (len * f / (2 * pi) - c.low) / ((long double)c.high - c.low)
                                                                     : 1 - (i - i0) / fmaxl(i1 - i0, 0.001L);
            const long double keep = fminl(fmaxl(along, 0), 1);
            f *= keep + (1 - keep) / factor;
        }
        turns[i] = (uint64_t)rintl(ldexpl(f / (2 * pi), 64));  // f <= 1: below 2^62
    }
    *amplitude = c.scaling == LOOKAT_ROPE_RAMP ? (float)(0.1L * logl(factor) + 1) : 1.f;
    return LOOKAT_OK;
}

lookat_status lookat_rope(lookat_ctx *handle, const lookat_rows *q, const lookat_rows *k, int64_t n_tokens, const int32_t *positions,
                          const uint64_t *turns, int32_t rotary_dim, int32_t interleaved, float amplitude, const lookat_rows *q_out,
                          const lookat_rows *k_out)
{
    if (!handle) return LOOKAT_ERR_INVALID_ARG;
    Ctx *ctx = reinterpret_cast<Ctx *>(handle);
    const lookat_config &c = ctx->cfg;
    RopeArgs a;
    memset(&a, 0, sizeof(a));
    if (!q && !k) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "q and k are both NULL");
    if ((!q && q_out) || (!k && k_out)) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "a result without its input");
    if (n_tokens < 0 || n_tokens >= kMaxTokens) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "n_tokens=%lld out of range 0..2^30-1", (long long)n_tokens);
    if (c.d_k % 8) return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "rope wants d_k as a multiple of 8 (%d)", c.d_k);
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > c.d_k)
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "rotary_dim=%d is not an even number in 2..d_k", (int)rotary_dim);
    if (interleaved != 0 && interleaved != 1) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "interleaved=%d is not 0 or 1", (int)interleaved);
    if (!std::isfinite(amplitude)) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "amplitude is not a finite number");
    const lookat_rows *in[2] = {q, k}, *out[2] = {q_out, k_out};
    for (int i = 0; i < 2; ++i) {
        if (!in[i]) continue;
        a.heads[i] = i ? c.n_kv_heads : c.n_q_heads;
        Q8_TRY(rows_of(ctx, in[i], n_tokens, a.heads[i], i ? "k" : "q", &a.in[i]));
        a.out[i] = a.in[i];
        if (out[i]) Q8_TRY(rows_of(ctx, out[i], n_tokens, a.heads[i], i ? "k_out" : "q_out", &a.out[i]));
        Q8_TRY(apart(ctx, a.out[i], n_tokens, a.heads[i], c.d_k, i ? "k_out" : "q_out"));
    }
    if (n_tokens == 0) return LOOKAT_OK;
    Q8_TRY(need(ctx, positions, "positions", 4));
    Q8_TRY(need(ctx, turns, "turns", 8));
    Q8DeviceGuard guard(ctx->device);
    if (!guard.ok) return set_error(ctx, LOOKAT_ERR_CUDA, "cannot select device %d", ctx->device);
    a.positions = positions;
    a.turns = reinterpret_cast<const unsigned long long *>(turns);
    a.n = n_tokens;
    a.d = c.d_k;
    a.r = rotary_dim;
    a.interleaved = interleaved;
    a.amplitude = amplitude;
    return launch_rope(ctx, a);
}

lookat_status lookat_attend_packed(lookat_ctx *handle, const lookat_rows *q, const lookat_rows *k, const lookat_rows *v, int64_t n_tokens,
                                   int32_t B, const int32_t *starts, const lookat_rows *out)
{
    if (!handle) return LOOKAT_ERR_INVALID_ARG;
    Ctx *ctx = reinterpret_cast<Ctx *>(handle);
    const lookat_config &c = ctx->cfg;
    PackedAttendArgs a;
    memset(&a, 0, sizeof(a));
    if (ctx->timeout_flag && *(volatile int *)ctx->timeout_flag) {
        *(volatile int *)ctx->timeout_flag = 0;
        return set_error(ctx, LOOKAT_ERR_TIMEOUT, "an earlier attention kernel gave up a bounded barrier wait; its output is not valid");
    }
    Q8_TRY(packed_of(ctx, n_tokens, B, starts, &a.rows));
    if (c.d_k % 16 || c.d_v % 16 || c.d_k > 256 || c.d_v > 256)
        return set_error(ctx, LOOKAT_ERR_UNSUPPORTED, "packed attention wants d_k and d_v as multiples of 16 up to 256 (%d, %d)", c.d_k, c.d_v);
    Q8_TRY(rows_of(ctx, q, n_tokens, c.n_q_heads, "q", &a.q));
    Q8_TRY(rows_of(ctx, k, n_tokens, c.n_kv_heads, "k", &a.k));
    Q8_TRY(rows_of(ctx, v, n_tokens, c.n_kv_heads, "v", &a.v));
    Q8_TRY(rows_of(ctx, out, n_tokens, c.n_q_heads, "out", &a.out));
    Q8_TRY(apart(ctx, a.out, n_tokens, c.n_q_heads, c.d_v, "out"));
    if (n_tokens == 0) return LOOKAT_OK;
    Q8DeviceGuard guard(ctx->device);
    if (!guard.ok) return set_error(ctx, LOOKAT_ERR_CUDA, "cannot select device %d", ctx->device);
    a.H_q = c.n_q_heads;
    a.H_kv = c.n_kv_heads;
    a.g = c.n_q_heads / c.n_kv_heads;
    a.d_k = c.d_k;
    a.d_v = c.d_v;
    a.scale_log2 = ctx->scale * 1.4426950408889634f;
    return launch_attend_packed(ctx, a);
}

lookat_status lookat_q8_append_packed(lookat_ctx *handle, const lookat_q8_cache *cache, const lookat_rows *k, const lookat_rows *v,
                                      int64_t n_tokens, int32_t B, const int32_t *starts, const int32_t *tables, int32_t max_pages,
                                      const int32_t *seq_lens)
{
    if (!handle) return LOOKAT_ERR_INVALID_ARG;
    Ctx *ctx = reinterpret_cast<Ctx *>(handle);
    const lookat_config &c = ctx->cfg;
    Q8AppendArgs a;
    memset(&a, 0, sizeof(a));
    Packed p;
    Rows rk, rv;
    Q8_TRY(view_of(ctx, cache, B, tables, max_pages, seq_lens, &a.c));
    Q8_TRY(packed_of(ctx, n_tokens, B, starts, &p));
    Q8_TRY(rows_of(ctx, k, n_tokens, c.n_kv_heads, "k", &rk));
    Q8_TRY(rows_of(ctx, v, n_tokens, c.n_kv_heads, "v", &rv));
    if (n_tokens == 0) return LOOKAT_OK;
    Q8DeviceGuard guard(ctx->device);
    if (!guard.ok) return set_error(ctx, LOOKAT_ERR_CUDA, "cannot select device %d", ctx->device);
    a.k_new = rk.p;
    a.v_new = rv.p;
    a.k_ts = rk.ts, a.k_hs = rk.hs;
    a.v_ts = rv.ts, a.v_hs = rv.hs;
    a.starts = starts;
    a.B = B;
    a.n = (int)n_tokens;
    a.format = cache->format;
    return launch_q8_append(ctx, a);
}

lookat_status lookat_beam_select(lookat_ctx *handle, const lookat_beam_state *state, const float *logits, int64_t logits_stride,
                                 int32_t vocab, int32_t eos, double length_penalty, int32_t *next_ids, int32_t *parents)
{
    if (!handle) return LOOKAT_ERR_INVALID_ARG;
    Ctx *ctx = reinterpret_cast<Ctx *>(handle);
    BeamArgs a;
    memset(&a, 0, sizeof(a));
    if (!state) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "state is NULL");
    const lookat_beam_state &s = *state;
    if (s.beams < 1 || s.beams > 32) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "beams=%d out of range 1..32", (int)s.beams);
    if (s.groups < 1 || (int64_t)s.groups * s.beams > 65535)
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "groups=%d: groups * beams out of range 1..65535", (int)s.groups);
    if (vocab < 1 || (int64_t)vocab * s.beams > (1ll << 30))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "vocab=%d: vocab * beams out of range 1..2^30", (int)vocab);
    if (logits_stride < vocab || logits_stride >= (1ll << 31))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "logits_stride=%lld is less than vocab, or 2^31 or more", (long long)logits_stride);
    if (eos < -1 || eos >= vocab) return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "eos=%d is not -1 or a token", (int)eos);
    if (!(length_penalty >= 0 && length_penalty <= kMaxPenalty))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "length_penalty is not a number in 0..%g", kMaxPenalty);
    if (s.max_len < 0 || s.max_len > (1 << 24) || (s.max_len > 0) != (s.tokens != nullptr))
        return set_error(ctx, LOOKAT_ERR_INVALID_ARG, "max_len=%d out of range 0..2^24, or not 0 without tokens", (int)s.max_len);
    Q8_TRY(need(ctx, s.scores, "state.scores", 4));
    Q8_TRY(need(ctx, s.lengths, "state.lengths", 4));
    Q8_TRY(need(ctx, s.finished, "state.finished", 4));
    if (s.tokens) Q8_TRY(need(ctx, s.tokens, "state.tokens", 4));
    Q8_TRY(need(ctx, logits, "logits", 4));
    Q8_TRY(need(ctx, next_ids, "next_ids", 4));
    Q8_TRY(need(ctx, parents, "parents", 4));
    Q8DeviceGuard guard(ctx->device);
    if (!guard.ok) return set_error(ctx, LOOKAT_ERR_CUDA, "cannot select device %d", ctx->device);
    a.scores = s.scores;
    a.lengths = s.lengths;
    a.finished = s.finished;
    a.tokens = s.tokens;
    a.logits = logits;
    a.stride = logits_stride;
    a.groups = s.groups;
    a.beams = s.beams;
    a.max_len = s.max_len;
    a.vocab = vocab;
    a.eos = eos;
    a.penalty = length_penalty;
    a.next_ids = next_ids;
    a.parents = parents;
    return launch_beam_select(ctx, a);
}

}  // extern "C"
