/*
 * rac_tokens.h - C ABI of what a round of drafted tokens does around the
 * attention of rac_cache.h (MI355X, gfx950): turning queries and keys by their
 * positions, and scoring the drafted tokens with the logits of the tail.
 *
 * The conventions of rac.h hold: device pointers on the current device,
 * caller-owned memory, work enqueued on `stream`, nothing allocated, kept or
 * synchronized, argument errors before any launch.  Every call can be recorded in
 * a HIP graph.  Positions, tokens and row numbers that lie in device memory are
 * checked by the kernels: whatever they hold, no access leaves the buffers.  A
 * call gives the same bits every time.
 */
#ifndef RAC_TOKENS_H
#define RAC_TOKENS_H

#include "rac.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    RAC_TYPE_BF16 = 0,
    RAC_TYPE_FP16 = 1,
    RAC_TYPE_FP32 = 2
};

/* ---- Rotary positions -----------------------------------------------------
 * Channel pair i of a head in row r turns by pos[r] * freq[i] turns (a turn is
 * 2 pi): with c and s the cosine and sine of that angle times `amplitude`,
 *   (x, y) -> (x c - y s, y c + x s).
 * The pairs are channels (2 i, 2 i + 1), as the predictor's, or with
 * RAC_ROTARY_HALF channels (i, i + rotary_dim / 2), i < rotary_dim / 2; the
 * channels from rotary_dim on are kept.  `transpose` turns the other way, which is
 * the gradient: given those of the results it leaves those of the inputs.
 *
 * The fraction of a turn is taken in binary64, so far positions lose nothing;
 * sines and products are fp32, rounded once to the type. */
enum {
    RAC_ROTARY_INTERLEAVED = 0,
    RAC_ROTARY_HALF = 1
};

typedef struct {
    int32_t rows;       /* 0..2^24                                                  */
    int32_t q_heads;    /* 1..4096                                                  */
    int32_t k_heads;    /* 0..4096; 0: queries only                                 */
    int32_t head_dim;   /* multiple of 16, 16..256                                  */
    int32_t rotary_dim; /* multiple of 16, 16..head_dim                             */
    int32_t type;       /* RAC_TYPE_*                                               */
    int32_t layout;     /* RAC_ROTARY_*                                             */
    int32_t transpose;  /* 0, 1                                                     */
    float amplitude;    /* finite; 1 but for some scaled contexts                   */
} rac_rotary_config;

/* Host-only, pure.  turns[i] (host memory, rotary_dim / 2) for
 *   f_i = base^(-2 i / rotary_dim) / (2 pi),
 *   turns[i] = f_i (g + (1 - g) / factor),  g = (trained f_i - slow) / (fast - slow)
 * with g kept within 0..1: a context `factor` times the `trained` one, in which the
 * pairs that turn less than `slow` times over the trained length are stretched,
 * those that turn more than `fast` times are kept, and those between are blended.
 * factor 1: plain rotary positions; trained 0: every pair is stretched (linear
 * scaling).  RAC_ERR_INVALID unless rotary_dim is as above, base > 1, factor > 0,
 * trained >= 0, 0 <= slow < fast, all finite. */
rac_status rac_rotary_frequencies(int32_t rotary_dim, double base, double factor, int32_t trained, double slow,
                                  double fast, double* turns);

typedef struct {
    const void* q; /* [rows][q_heads][head_dim], rows q_stride elements apart           */
    const void* k; /* [rows][k_heads][head_dim], k_stride; NULL without keys            */
    void* q_out;   /* as q and k, with strides of their own; each may be its input      */
    void* k_out;   /* (with its stride), and overlaps nothing else                      */
    int64_t q_stride, k_stride, q_out_stride, k_out_stride; /* multiples of 8           */
} rac_rotary_tensors;

/* pos: int32 [rows], freq: binary64 [rotary_dim / 2], finite, in device memory.  A
 * row with a negative position (padding) is left as it is, its outputs unwritten.
 * q, k and outputs 16-byte aligned, pos 4-byte, freq 8-byte.  One kernel launch.
 * RAC_ERR_INVALID and _ALIGN. */
rac_status rac_rotary(const rac_rotary_config* cfg, const int32_t* pos, const double* freq,
                      const rac_rotary_tensors* t, rac_stream_t stream);

/* ---- Log probabilities of tokens --------------------------------------------
 * Of row r of the logits x, with c = scale (an inverse temperature):
 *   lse[r]     = ln(sum_v exp(c x[r][v]))
 *   entropy[r] = lse[r] - sum_v p_v c x[r][v],  p_v = exp(c x[r][v] - lse[r])
 *   the `top` largest logits, ties to the lower v, as top_ids[r][i] and
 *   top_logprobs[r][i] = c x[r][v] - lse[r]
 * and for scored token j
 *   logprob[j] = c x[row][tokens[j]] - lse[row],  row = token_rows[j], or j.
 * A drafted tree is scored with token_rows[j] the row of j's parent.
 *
 * A logit of -infinity (a masked word) has no part in the sums and is no
 * alternative: where a row has fewer, the rest have id -1 and -infinity.  A row of
 * such logits only has an lse of -infinity, entropy 0, and log probabilities of
 * -infinity; so does one whose lse lies below the range of fp32, but for its entropy.  A
 * token outside the vocabulary, or a row outside the rows, scores 0 (padding).  A NaN or
 * +infinity makes its row's lse, entropy and log probabilities NaN; a NaN is no alternative.
 * An lse above the range of fp32 (finite logits, a scale above 1) is NaN, and so are
 * the row's log probabilities.
 *
 * Sums are fp32, whatever the type. */
typedef struct {
    int32_t rows;   /* 0..2^24                                                      */
    int32_t vocab;  /* 1..2^24                                                      */
    int32_t tokens; /* scored tokens, 0..2^24; rows or 0 without token_rows         */
    int32_t top;    /* 0..64                                                        */
    int32_t type;   /* RAC_TYPE_* of the logits                                     */
    float scale;    /* 2^-40..2^40; 0: 1                                            */
} rac_logprob_config;

typedef struct {
    const void* logits;        /* [rows][vocab], rows `stride` elements apart, at any  */
    int64_t stride;            /* multiple of an element's size                        */
    const int32_t* tokens;     /* [tokens]                                             */
    const int32_t* token_rows; /* [tokens], or NULL                                    */
    float* logprob;            /* [tokens]                                             */
    float* lse;                /* [rows]                                               */
    float* entropy;            /* [rows], or NULL                                      */
    int32_t* top_ids;          /* [rows][top]   (both NULL with top = 0)               */
    float* top_logprobs;       /* [rows][top]                                          */
} rac_logprob_tensors;

/* Host-only, pure.  Bytes of the call's device scratch, or 0 for a configuration
 * outside the ranges above. */
size_t rac_logprobs_workspace(const rac_logprob_config* cfg);

/* int32 and fp32 arrays 4-byte aligned, workspace 256-byte.  One kernel launch, one
 * more where rows are cut into parts and one with token_rows.  RAC_ERR_INVALID,
 * _ALIGN and _CAPACITY (workspace). */
rac_status rac_logprobs(const rac_logprob_config* cfg, const rac_logprob_tensors* t, void* workspace,
                        size_t workspace_bytes, rac_stream_t stream);

/* Gradients of the logits for one scored token a row (token_rows NULL, cfg->tokens
 * = rows; cfg->top is not looked at), from those of logprob and entropy and what
 * the forward pass left:
 *   grad_logits[r][v] = c (g_l (v == tokens[r]) - p_v (g_l + g_e (ln p_v + entropy[r])))
 * with g_l = grad_logprob[r] (0 for a token outside the vocabulary) and g_e =
 * grad_entropy[r]; either array may be NULL (zeros), not both.  A masked word gets
 * g_l's part alone, a row whose lse is -infinity zeros, one whose lse is NaN NaN. */
typedef struct {
    const void* logits; /* as above                                                    */
    int64_t stride;
    const int32_t* tokens;
    const float* lse;          /* [rows]                                               */
    const float* entropy;      /* [rows]; needed with grad_entropy                     */
    const float* grad_logprob; /* [rows], or NULL                                      */
    const float* grad_entropy; /* [rows], or NULL                                      */
    void* grad_logits;         /* [rows][vocab] of the logits' type, rows grad_stride  */
    int64_t grad_stride;       /* elements apart; may be the logits (with their stride)*/
} rac_logprob_gradients;

/* One kernel launch.  Fastest where logits and gradients lie alike within 16 bytes. */
rac_status rac_logprobs_backward(const rac_logprob_config* cfg, const rac_logprob_gradients* g, rac_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* RAC_TOKENS_H */
