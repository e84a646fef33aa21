/*
 * mikv_layer.h -- the operators of one attention layer around the
 * mixed-precision cache of mikv.h: rotary positions of a projection's rows,
 * attention of whole prompts, its importance scores and decode attention,
 * the last three under score rules (a tanh cap, a bias by distance, masks of
 * documents, prefixes, windows and padding).  Exported by libmikv.so.
 *
 * The conventions of mikv.h hold: device pointers unless stated otherwise,
 * the caller allocates everything, every call is asynchronous on `stream`
 * (which belongs to the current device), arguments are validated on the host
 * before any launch, nothing throws, aborts or prints, and head_dim is 128.
 */
#ifndef MIKV_LAYER_H
#define MIKV_LAYER_H

#include "mikv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions ------------------------------------------------------- */

enum mikv_type { MIKV_F16 = 0, MIKV_BF16 = 1, MIKV_F32 = 2 };

/* Frequencies for contexts longer than the trained one. */
enum mikv_rotary_scaling {
  MIKV_ROTARY_PLAIN = 0,  /* w_p = base^(-2 p / rot_dim) */
  MIKV_ROTARY_LINEAR = 1, /* w_p / factor: positions interpolated */
  MIKV_ROTARY_NTK = 2,    /* base * factor^(rot_dim / (rot_dim - 2)) in place of base */
  /* by the turns n = original_length * w_p / (2 pi) a pair makes over the
   * trained context: w_p from `high` turns on, w_p / factor up to `low`, and
   * in between w_p (t + (1 - t) / factor), t = (n - low) / (high - low) */
  MIKV_ROTARY_BANDS = 3,
  /* YaRN (arXiv 2309.00071): the same blend with t falling linearly over the
   * pair index, from 1 at floor(p(high)) to 0 at ceil(p(low)), p(n) = rot_dim ln(
   * original_length / (2 pi n)) / (2 ln base) the pair that makes n turns;
   * rotated channels are multiplied by 0.1 ln(factor) + 1 */
  MIKV_ROTARY_YARN = 4
};

typedef struct mikv_rotary_scheme {
  int32_t rot_dim;        /* channels that rotate, the first of the head: even, 2 .. 128 */
  int32_t scaling;        /* mikv_rotary_scaling */
  double base;            /* > 1 */
  double factor;          /* >= 1 (ignored by PLAIN) */
  double original_length; /* > 0; BANDS and YARN */
  double low, high;       /* turns, 0 < low < high; BANDS and YARN */
} mikv_rotary_scheme;

/*
 * Frequencies of a scheme, as the fraction of a turn per position in units of
 * 2^-64 (so that a position's phase is exact to 2^-32 turns at any int32
 * position), and the factor on rotated channels.  A host function: `freq`
 * (rot_dim / 2 values) and `magnitude` are HOST pointers; the caller copies
 * `freq` to the device once.
 * Errors: INVALID_ARG (NULL, a field outside the ranges above, NTK with rot_dim 2).
 */
int mikv_rotary_frequencies(const mikv_rotary_scheme *scheme, uint64_t *freq, float *magnitude);

/* One tensor of mikv_rotary: x -> y, both [batch, heads, tokens, 128] through
 * their strides (batch, head, token; in elements; channels are contiguous). */
typedef struct mikv_heads {
  const void *x;
  void *y;
  int64_t x_stride[3], y_stride[3];
  int32_t heads;
  int32_t rotate; /* 0: converted and laid out only (values) */
} mikv_heads;

/*
 * Rotary positions of up to three tensors (queries, keys, values) of the same
 * tokens in one launch: for every rotated row at position pos and every pair p
 * of its channels (p, p + rot_dim / 2), or with `interleaved` (2 p, 2 p + 1),
 *   (a, b) -> magnitude (a cos - b sin, b cos + a sin) at angle pos * w_p,
 * in fp32, rounded once to y's type; channels from rot_dim on are converted.
 *   tensors    HOST array of n (1 .. 3) tensors;
 *   x_type, y_type  mikv_type of every x and every y: y_type is x_type or MIKV_F16;
 *   positions  int32 [batch, tokens], or NULL: pos0 + t for token t.  Any int32
 *              value: a negative position turns backwards, which undoes (up to
 *              the square of the magnitude) and is the transpose of the turn by
 *              its absolute value;
 *   freq       uint64 [rot_dim / 2] on the device (mikv_rotary_frequencies).
 * y may be x (same pointer, strides and type); other overlaps are not allowed.
 * Rows that are 16-byte aligned, with rot_dim a multiple of 16, are read
 * and written 16 bytes at a time; others work, more slowly.
 * Errors: INVALID_ARG (NULL, counts < 1, rot_dim odd or outside 2 .. 128, x or y not
 * aligned to its type, unknown types or pairs of types, in place between two types or
 * strides, rows of y that share memory: a stride of 0);
 * UNSUPPORTED (head_dim != 128, over 2^24 tokens in all, over 2^16 heads).
 */
int mikv_rotary(const mikv_heads *tensors, int32_t n, int32_t batch, int32_t tokens, int32_t head_dim, int32_t x_type,
                int32_t y_type, const int32_t *positions, int32_t pos0, const uint64_t *freq, int32_t rot_dim,
                int32_t interleaved, float magnitude, void *stream);

/* ---- attention under score rules -------------------------------------------------- */

/*
 * The score of query i and key j (positions) in query head h, and which keys
 * a query sees:
 *   s = scale q . k;  s = cap tanh(s / cap) if cap > 0;  s -= slopes[h] |i - j|;
 *   begin <= j < end, and j > i - window if window > 0.
 * begin and end may hold any values (they are clamped to the sequence); where
 * begin >= end the query sees nothing: its output is 0, its log-sum-exp -inf.
 * K and V rows that a query does not see add nothing to it, whatever
 * they hold, NaN and infinities included.
 */
typedef struct mikv_score_rules {
  float cap;            /* 0: none; finite, and scale / cap within fp32's normal range */
  const float *slopes;  /* fp32 [q_heads], finite; NULL: no bias */
  const int32_t *begin; /* prompt: [batch, tokens], decode: [batch]; NULL: 0 */
  const int32_t *end;   /* prompt: [batch, tokens], NULL: i + 1 (causal); decode: must be NULL */
  int32_t window;       /* 0: none */
} mikv_score_rules;

/*
 * begin and end of every query of a prompt, from documents, a prefix and a
 * window.  Query i sees the keys j of its document with (j <= i or j <
 * prefix[b]) and (j > i - window, window > 0):
 *   documents int32 [batch, tokens] or NULL (one document): a document is a
 *             run of equal ids; tokens with a negative id are padding, which
 *             sees nothing and is seen by none;
 *   prefix    int32 [batch] or NULL: leading positions that every query of the same document sees;
 *   window    0: none;
 *   begin, end int32 [batch, tokens] (outputs).
 * Errors: INVALID_ARG (NULL outputs, counts < 1, window < 0); UNSUPPORTED (over 2^30 tokens).
 */
int mikv_mask_spans(const int32_t *documents, const int32_t *prefix, int32_t batch, int32_t tokens, int32_t window,
                    int32_t *begin, int32_t *end, void *stream);

/* The prompt of one layer: fp16 rows of 128 channels through their strides
 * (batch, head, token; in elements, multiples of 8; rows 16-byte aligned). */
typedef struct mikv_prompt {
  int32_t batch, q_heads, kv_heads; /* q_heads / kv_heads in {1, 2, 4, 8} */
  int32_t tokens, head_dim;
  float scale;                      /* > 0 */
  const uint16_t *q, *k, *v;        /* v: NULL for mikv_prompt_importance */
  int64_t q_stride[3], k_stride[3], v_stride[3];
} mikv_prompt;

/*
 * Attention of whole prompts:  out = softmax over the keys seen (s) v.
 * Products are fp16 with fp32 sums on the matrix cores; scores, maxima, sums and
 * the output's accumulation are fp32, the weights of the value product fp16.
 *   rules  HOST pointer, or NULL: causal, no cap, no bias;
 *   out    fp16 [batch, q_heads, tokens, 128] through out_stride (as q's, no stride 0);
 *   lse    fp32 [batch, q_heads, tokens] or NULL: natural log of the sum of exp(s).
 * Errors: INVALID_ARG (NULL, counts < 1, q_heads % kv_heads, alignment, strides, scale, cap, window);
 * UNSUPPORTED (head_dim, query heads per KV head, a token stride over 2^22, grids over 2^31).
 */
int mikv_prompt_attention(const mikv_prompt *prompt, const mikv_score_rules *rules, uint16_t *out,
                          const int64_t out_stride[3], float *lse, void *stream);

/*
 * H2O importance of the prompt's tokens under the same rules (mikv_prefill_importance
 * is the causal case without rules, from q and k alone):
 *   scores[b, h, j] = sum_{g in group(h)} sum_{i sees j} exp(s_ij - lse[b, g, i]),
 * in fp32, in an order that the sizes fix.
 *   lse       as mikv_prompt_attention wrote it for the same prompt and rules;
 *   scores    fp32 [batch, kv_heads, tokens] (output);
 *   workspace at least mikv_prompt_importance_workspace_size(...) bytes.
 * Errors: those of mikv_prompt_attention; CAPACITY for a too-small workspace.
 */
size_t mikv_prompt_importance_workspace_size(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t tokens);
int mikv_prompt_importance(const mikv_prompt *prompt, const mikv_score_rules *rules, const float *lse, float *scores,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * mikv_decode_attention and mikv_decode_step under score rules: the query is
 * the token at position length - 1, a cached token's position is the one it
 * was placed at, and `begin` (per sequence) hides earlier ones (left padding,
 * an earlier document).  Hidden tokens have probability 0; a sequence that
 * sees nothing gets an output of 0.
 *   rules  HOST pointer; NULL: the unscored call.
 * Other arguments, results, workspaces and errors as there; INVALID_ARG also for a
 * negative or NaN cap, a negative window and for rules->end.
 */
int mikv_decode_attention_scored(const mikv_cache *c, int32_t length, const uint16_t *q, const float *balance,
                                 float scale, const mikv_score_rules *rules, float *out, float *probs_hi,
                                 float *probs_lo, int32_t flags, void *workspace, size_t workspace_bytes,
                                 void *stream);
int mikv_decode_step_scored(const mikv_cache *c, int32_t length, const uint16_t *q, const uint16_t *k_new,
                            const uint16_t *v_new, const float *balance, float scale, const mikv_score_rules *rules,
                            float *out, float *probs_hi, float *probs_lo, int32_t k_heavy, int32_t window,
                            int32_t flags, void *workspace, size_t workspace_bytes, void *const *phase_events,
                            void *stream);

#ifdef __cplusplus
}
#endif

#endif /* MIKV_LAYER_H */
