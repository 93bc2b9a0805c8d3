/*
 * spex_prompt.h -- causal attention over whole prompts, from the tensors a model's projections leave.
 *
 * A new user query enters the search as a root that holds its prompt (spex_tree.h, spex_tree_fork).  Its
 * tokens are all new: queries, keys and values of every position lie in the projections' own tensors, and
 * nothing of the prompt is in the cache yet that the attention could share.  This call computes their
 * attention from there -- packed prompts of any lengths, none padded -- while spex_tree_append_rotated
 * writes the same keys and values into the page pool for the decoding that follows.  Against
 * spex_tree_decode_attention over the appended prompt it needs no plan, reads keys and values as the
 * model made them (an fp8 cache holds them rounded to e4m3) and returns the model's own type.  Its form
 * for single new tokens over a cache is spex_tree_decode_attention.
 *
 * The call keeps no state: it has no handle and no workspace, allocates nothing, and its lists travel in the
 * kernel arguments.  It may be called from any thread, on any stream of the current device, several at a
 * time, and may be recorded in a HIP graph (the recorded launches keep the lengths and addresses of the call).
 * Status codes are spex_status_t (spex_tree.h); nothing is launched when an error other than SPEX_ERR_DEVICE
 * is returned.
 */
#ifndef SPEX_PROMPT_H_
#define SPEX_PROMPT_H_

#include <stdint.h>

#include "spex_tree.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t num_q_heads;  /* multiple of num_kv_heads; query head h uses kv head h / (Hq/Hkv) */
  int32_t num_kv_heads; /* 1..255 */
  int32_t head_dim;     /* 1..256 */
  int32_t dtype;        /* SPEX_F32 or SPEX_BF16, of q, k, v and out */
  /* Elements between consecutive tokens; 0 = dense (heads * head_dim).  The heads of a token are always
   * dense, so a stride is at least heads * head_dim; q, k and v may be parts of one tensor. */
  int64_t q_stride, k_stride, v_stride, out_stride;
} spex_prompt_config_t;

/*
 * n_prompts prompts of lens[i] >= 0 tokens (HOST), packed one behind the other: prompt i's tokens are
 * rows lens[0] + .. + lens[i-1] onwards of q, k, v, out and lse.  Token t of a prompt sees its tokens 0 .. t.
 *   q    : DEVICE [sum(lens)][num_q_heads][head_dim]
 *   k, v : DEVICE [sum(lens)][num_kv_heads][head_dim]
 *   out  : DEVICE, shape of q:  sum_s softmax_s(sm_scale * <q_t, k_s>) v_s, rounded to nearest
 *   lse  : DEVICE fp32 [sum(lens)][num_q_heads] or NULL:  ln sum_s exp(sm_scale * <q_t, k_s>)
 * q, k and v must be finite (a value of v that is not may spoil rows of tokens before its own, too), and so must the scores <q_t, k_s> in fp32 and, times sm_scale, stay within +-1e30; sm_scale in
 * 1e-38 .. 1e37 (else SPEX_ERR_INVALID_ARG).  out must not overlap q, k or v.  Nothing outside
 * the prompts' rows is read or written.  Scores, softmax statistics and sums are fp32 (a weight's exponent is a difference of
 * scores, also where the scores are so large that fp32 rounds their scaled values to many units); for bf16 the
 * softmax weights are rounded to bf16 (to nearest) for their product with v, so that an output is within
 * 2^-8 of the weighted mean of |v| besides its own rounding.
 * Rows whose address, stride or head_dim is no multiple of 16 bytes take a slower kernel.
 * A prompt may have up to 2^24 tokens, and up to 2^31 - 65 sets of 32 tokens of one of a kv head's query heads, and all prompts INT32_MAX
 * tokens (else SPEX_ERR_UNSUPPORTED).  SPEX_ERR_CAPACITY: no host memory
 * for the list of the prompts.
 */
spex_status_t spex_prompt_attention(const spex_prompt_config_t *cfg, const int32_t *lens, int32_t n_prompts,
                                    const void *q, const void *k, const void *v, void *out, float *lse,
                                    float sm_scale, void *hip_stream);

/* The kernel that a call with these arguments launches, for tests: -1 = none (no tokens); 0 = element by element; 1 = workgroups that
 * share tiles between their wavefronts, of 64 keys (fp32: 32); 2 = the same with tiles of 32 keys; 3, 4 = workgroups of four, eight
 * wavefronts that split the keys of their rows.  The tensors are not touched. */
spex_status_t spex_prompt_form(const spex_prompt_config_t *cfg, const int32_t *lens, int32_t n_prompts, const void *q,
                               const void *k, const void *v, const void *out, int32_t *form);

#ifdef __cplusplus
}
#endif
#endif /* SPEX_PROMPT_H_ */
