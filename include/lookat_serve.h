/*
 * lookat_serve.h - C ABI of what a server runs around the 8-bit paged cache (part of liblookat.so): rotary positions, exact
 * attention of packed prompts, their keys and values into the cache, and beam search's selection.
 *
 * PACKED ROWS.  The tokens of a batch's rows stand one behind the other: row b is the tokens starts[b] .. starts[b + 1] - 1 of
 * n_tokens (starts: device int32 [B + 1]; starts[0] need not be 0, and tokens of no row are neither read nor written).  Rows may
 * be empty and of any lengths.  A lookat_rows names fp16 vectors of such tokens: element i of head h of token t lies at
 *     data + t * token_stride + h * head_stride + i,
 * so the thirds of a fused projection's output are used where they lie, and [heads][tokens][d] as well as [tokens][heads][d].
 * data is 16-byte aligned device memory; the strides are positive multiples of 8 elements below 2^31 (that of a single head or a
 * single token is not used).  Rows that are written may not overlap themselves.
 *   A context serves one attention shape: its n_q_heads, n_kv_heads, d_k, d_v and scale.
 *
 * DEVICE-SIDE FINDINGS.  The host does not see starts: a row for which 0 <= starts[b] <= starts[b + 1] <= n_tokens does not hold is
 * taken as empty, and lookat_last_error reports it as lookat_q8.h describes.  A row's tokens are found by bisection, for which starts
 * must not fall: with an entry below an earlier one (rows that overlap, a list that ends in zeros) tokens of other rows may keep
 * their former results.  A batch of fewer rows than B ends in repeats of its last entry, which are empty rows.
 *
 * Work is enqueued on the context's stream; scratch and captures are as in lookat_q8.h.
 */
#ifndef LOOKAT_SERVE_H
#define LOOKAT_SERVE_H

#include "lookat.h"
#include "lookat_q8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lookat_rows {
    void *data;              /* fp16, device */
    int64_t token_stride;    /* in elements */
    int64_t head_stride;
} lookat_rows;

/*
 * The speeds of rotary positions.  Pair i of the rotary_dim / 2 turns by f_i radians per position,
 *     f_i = base^(-2 i / rotary_dim),
 * changed for contexts longer than the original ones by one of:
 *   LOOKAT_ROPE_NONE     f_i
 *   LOOKAT_ROPE_LINEAR   f_i / factor
 *   LOOKAT_ROPE_BASE     base * factor^(rotary_dim / (rotary_dim - 2)) in place of base
 *   LOOKAT_ROPE_BANDS    f_i (c + (1 - c) / factor),  c = (u_i - low) / (high - low) cut to 0..1, with u_i = original_len f_i / 2 pi the
 *                        turns over the original context: fast pairs stay, slow ones are stretched
 *   LOOKAT_ROPE_RAMP     the same with c falling linearly in i from 1 at i0 to 0 at i1, the indexes where u is `high` and `low`:
 *                        i(u) = rotary_dim ln(original_len / (2 pi u)) / (2 ln base), i0 = max(floor(i(high)), 0),
 *                        i1 = min(ceil(i(low)), rotary_dim - 1), over a distance of at least 0.001; cosines and sines are multiplied by
 *                        0.1 ln(factor) + 1
 */
enum {
    LOOKAT_ROPE_NONE = 0,
    LOOKAT_ROPE_LINEAR = 1,
    LOOKAT_ROPE_BASE = 2,
    LOOKAT_ROPE_BANDS = 3,
    LOOKAT_ROPE_RAMP = 4
};
typedef struct lookat_rope_config {
    int32_t rotary_dim;      /* even, 2..1024 (at least 4 with LOOKAT_ROPE_BASE) */
    int32_t scaling;         /* LOOKAT_ROPE_* */
    double base;             /* > 1 */
    double factor;           /* >= 1 (not used by LOOKAT_ROPE_NONE) */
    double original_len;     /* > 0 (BANDS, RAMP) */
    double low, high;        /* 0 < low < high (BANDS, RAMP) */
} lookat_rope_config;

/* Host only, no context: turns[i] (rotary_dim / 2 of them) = f_i / 2 pi as a fraction of 2^64, so that position p stands at the
 * turn p * turns[i] mod 2^64, exactly; *amplitude the factor on cosines and sines.  Returns LOOKAT_ERR_INVALID_ARG for settings out
 * of range. */
lookat_status lookat_rope_table(const lookat_rope_config *cfg, uint64_t *turns, float *amplitude);

/*
 * Rotary positions: of every query and key head of token t, with angle_i = 2 pi (positions[t] * turns[i] mod 2^64) / 2^64,
 *     y_a = amplitude (x_a cos angle_i - x_b sin angle_i),   y_b = amplitude (x_b cos angle_i + x_a sin angle_i)
 * for the pairs (a, b) = (2 i, 2 i + 1) with interleaved = 1, (i, i + rotary_dim / 2) with 0; elements from rotary_dim on are
 * copied.  The angles are good to 2^-22 radians at any position, negative ones too; sums are fp32, rounded once to fp16.
 *
 *   q, k           lookat_rows of n_q_heads and n_kv_heads heads of d_k; either may be NULL
 *   q_out, k_out   where the results go; NULL or the same rows: in place.  Rows that overlap their input in any other way are the
 *                  caller's error
 *   positions      device int32 [n_tokens]
 *   turns          device uint64 [rotary_dim / 2]
 * Requires 0 <= n_tokens < 2^30, d_k a multiple of 8 and rotary_dim <= d_k.
 */
lookat_status lookat_rope(lookat_ctx *ctx, const lookat_rows *q, const lookat_rows *k, int64_t n_tokens, const int32_t *positions,
                          const uint64_t *turns, int32_t rotary_dim, int32_t interleaved, float amplitude, const lookat_rows *q_out,
                          const lookat_rows *k_out);

/*
 * Exact causal attention of packed prompts: token t of a row attends the row's tokens up to itself,
 *     s_u = q_t . k_u * scale (u <= t),   out_t = sum_u softmax(s)_u v_u,
 * query head h with KV head h / (n_q_heads / n_kv_heads).  What lookat_causal_attention does for equal lengths and one KV head per
 * query head, and, as it does, before the keys are quantised.
 *
 *   q, k    lookat_rows of n_q_heads and n_kv_heads heads of d_k;  v  n_kv_heads heads of d_v;  out  n_q_heads heads of d_v
 * Scores, softmax statistics and sums are fp32; the weights are fp16 numbers, 11 bits down to 2^-21 of a row's largest.  A NaN or an
 * infinity among a row's values may reach every query of that row (of other rows never), one among its keys every query that
 * attends it.  out may not overlap q, k or v.
 * Requires 0 <= n_tokens < 2^30 and 1 <= B <= 65535; d_k and d_v multiples of 16 up to 256, else LOOKAT_ERR_UNSUPPORTED.
 * The kernel is chosen by the mean length n_tokens / B, empty rows counted: a long row among so many empty ones that a row has no more
 * than 64 tokens times query heads per KV head on average runs on the kernel for short rows, several times slower.
 * Returns LOOKAT_ERR_TIMEOUT once if an earlier attention kernel of the context gave up a bounded wait (its output is not valid);
 * until a call has returned it, lookat_last_error reports it too, behind the findings above.
 */
lookat_status lookat_attend_packed(lookat_ctx *ctx, const lookat_rows *q, const lookat_rows *k, const lookat_rows *v, int64_t n_tokens,
                                   int32_t B, const int32_t *starts, const lookat_rows *out);

/*
 * lookat_q8_append for packed rows: the tokens starts[b] .. starts[b + 1] - 1 are the newest of row b, going to its positions
 * seq_lens[b] - (starts[b + 1] - starts[b]) ...; no padding is read.  Same numbers and scales.
 *   k, v  lookat_rows of n_kv_heads heads of d_k and d_v
 * Requires 0 <= n_tokens < 2^30.
 */
lookat_status lookat_q8_append_packed(lookat_ctx *ctx, const lookat_q8_cache *cache, const lookat_rows *k, const lookat_rows *v,
                                      int64_t n_tokens, int32_t B, const int32_t *starts, const int32_t *tables, int32_t max_pages,
                                      const int32_t *seq_lens);

/* The beams of a batch (device arrays): `groups` searches of `beams` rows each, row = group * beams + beam. */
typedef struct lookat_beam_state {
    float *scores;           /* [groups][beams] sum of the chosen tokens' log-probabilities; -inf: the beam does not count (all but the
                                first of a group before its first step) */
    int32_t *lengths;        /* [groups][beams] tokens chosen so far */
    int32_t *finished;       /* [groups][beams] 0, or 1 once eos was chosen */
    int32_t *tokens;         /* [groups][beams][max_len] the tokens chosen, or NULL (max_len 0) */
    int32_t groups;
    int32_t beams;           /* 1..32 */
    int32_t max_len;
} lookat_beam_state;

/*
 * One step of beam search: of every group the best `beams` candidates, in falling order of rank, become its beams.
 * The candidates of beam w: each token c, with
 *     score = scores[w] + logits[w][c] - log sum_c' exp logits[w][c'],   rank = score / (lengths[w] + 1)^length_penalty,
 * or, once it is finished, itself alone with its score and length, standing at c = eos (0 with eos = -1).  Equal ranks go to the lowest w * vocab + c.
 * A score of -inf is no candidate (a masked token), and a row with a NaN or +inf among its logits, or with a score of NaN or
 * +inf, has none.
 * A place for which there is no candidate keeps its row as it is, with a score of -inf.
 * Scores, lengths, flags and the first max_len tokens follow the beams in place; next_ids[row] is the token to feed next (eos for
 * finished beams and for places without a candidate, or 0 with eos = -1), parents[row] the row it continues from, as lookat_pages_fork
 * and lookat_gpt2_fork take it.  Ranks are fp64 over sums of fp32 exponentials; scores are rounded once.
 *
 *   logits          fp32 [groups * beams] rows of `vocab`, logits_stride elements apart (any alignment of 4 bytes)
 *   eos             the token that ends a beam, or -1
 *   length_penalty  0 compares plain sums; 0 to 28 (beyond, the norm of a long beam would leave no fp64 rank)
 * Requires groups * beams <= 65535, vocab * beams <= 2^30, 0 <= max_len <= 2^24.
 */
lookat_status lookat_beam_select(lookat_ctx *ctx, const lookat_beam_state *state, const float *logits, int64_t logits_stride,
                                 int32_t vocab, int32_t eos, double length_penalty, int32_t *next_ids, int32_t *parents);

#ifdef __cplusplus
}
#endif
#endif /* LOOKAT_SERVE_H */
