/*
 * vmonarch_sequence.h -- token sequences around Monarch attention, in the same library (libvmonarch):
 * rotary positions, attention over packed sequences of different lengths (forward and backward), and a
 * cache of keys and values in pages with the attention that reads it.
 *
 * What include/vmonarch.h says of streams, errors, workspaces and concurrency holds here too.  What differs:
 *   - A token tensor is described by a vmonarch_tokens: element (t, h, c) lies at data[t * token_stride +
 *     h * head_stride + c], strides in elements, channels adjacent.  Both [tokens][heads][d] and this library's
 *     [heads][tokens][d] are such tensors, and so is a slice of a fused projection.  Descriptors are read during
 *     the call only.
 *   - Calls without suffix take bfloat16 token tensors, `_f32` twins float32; statistics are float32.
 *   - The current device is the one that holds the tensors.
 *   - 1 <= d <= 256, heads_q a multiple of heads_kv; query head h reads key head h / (heads_q / heads_kv).  Tokens, tokens times
 *     heads_q / heads_kv, and the tokens a row of a table has room for are at most 2^31 - 65536 each, sequences at most 2^30 - 1.
 *   - Sequences: sequence s of n_seqs holds the packed tokens starts[s] .. starts[s + 1] - 1 (int32, DEVICE memory,
 *     n_seqs + 1 entries, non-decreasing).  A sequence may be empty.  The host cannot see these: entries are clamped to
 *     [0, tokens] on the device, and rows of a tensor that belong to no sequence are neither read nor written.
 *   - causal != 0: query i of a sequence's nq sees its keys 0 .. nk - nq + i; causal == 0: all nk.  A row that sees no
 *     key, or whose logits are all -inf, gives zeros and a log-sum-exp of -inf.  Keys and values that a row does not see do not
 *     reach it, infinities and NaN among them (forward passes; gradients are defined for finite tensors).
 *   - bf16 with d <= 128, d a multiple of 8, rows on 16-byte boundaries (and packed keys less than 2^24 elements apart)
 *     runs on the bf16 matrix units; everything else on the fp32 matrix units, with the same results to the tensors'
 *     precision.  Values beyond 2^98 may overflow in sums that would not overflow as weights of at most 1.
 *   - Logits are formed in fp32, so a weight is off by 2^-24 of its logit's magnitude, relatively; in gradients twice, the log-sum-exp is one too.  The
 *     bf16 matrix units take finite logits of up to 2^28 in magnitude (beyond, the rounding of a row's reference alone can carry its weights out of
 *     fp32's range: the row may come out as zeros or not finite), the fp32 ones any that fp32 holds.
 *   - Results do not depend on the order in which workgroups run: nothing is accumulated across them by atomics.
 */
#ifndef VMONARCH_SEQUENCE_H_
#define VMONARCH_SEQUENCE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct vmonarch_tokens {
  void* data;
  long long token_stride;
  long long head_stride;
} vmonarch_tokens;

/* ---- rotary positions ------------------------------------------------------------------------------ */

#define VMONARCH_ROTARY_HALF 0        /* pair i is channels i and i + n of the n pairs' 2 n channels */
#define VMONARCH_ROTARY_INTERLEAVED 1 /* pair i is channels 2 i and 2 i + 1 */
#define VMONARCH_ROTARY_MAX_PAIRS 128

/*
 * Which pairs turn how fast.  The first axis_pairs[0] pairs turn with a token's position on axis 0, the next
 * axis_pairs[1] with axis 1, and so on; channels past the pairs pass through.  A pair's angle is position *
 * frequency[pair] radians.  Filled by vmonarch_rotary_init; frequency and amplitude may be changed afterwards.
 */
typedef struct vmonarch_rotary_plan {
  uint32_t struct_bytes; /* sizeof(vmonarch_rotary_plan) */
  int layout;            /* VMONARCH_ROTARY_* */
  int axes;              /* 1 .. 3 */
  int axis_pairs[3];
  double amplitude;      /* multiplies the turned channels (1 by default) */
  double frequency[VMONARCH_ROTARY_MAX_PAIRS];
} vmonarch_rotary_plan;

/* frequency of pair i of an axis with n pairs: base^(-i / n), the usual choice for one axis of 2 n channels.  HOST. */
int vmonarch_rotary_init(vmonarch_rotary_plan* plan, int layout, double base, int axes, const int* axis_pairs_host);

/*
 * Frequencies for contexts `factor` times as long as trained.  context == 0: all divided by factor (positions are
 * interpolated).  Otherwise by band: with turns = context * frequency / 2 pi, a pair's full turns over the trained context,
 *   keep = clamp((turns - low_turns) / (high_turns - low_turns), 0, 1)
 *   frequency <- frequency * (keep + (1 - keep) / factor).
 * factor > 0; low_turns < high_turns.  HOST.
 */
int vmonarch_rotary_scale(vmonarch_rotary_plan* plan, double factor, double context, double low_turns, double high_turns);

/*
 * Turns every pair (x0, x1) of every head: y0 = A (x0 cos a - x1 sin a), y1 = A (x0 sin a + x1 cos a), a and A
 * the pair's angle and the plan's amplitude; backward != 0: the transpose (sin a negated), which takes the gradient
 * of y to that of x.  k may be NULL (heads_k 0).  positions: DEVICE int32 [axes][tokens], row a at
 * positions + a * axis_stride.  Angles are formed and reduced in 64 bits, to
 * 2^-52 of themselves: below fp32's rounding up to 2^28 radians, 5e-7 at 2^31.
 * Outputs may be their inputs (same pointer and strides); otherwise no output may overlap a tensor of the call (the same address is refused).
 * tokens == 0 is a no-op.
 */
int vmonarch_rotary(const vmonarch_tokens* q, const vmonarch_tokens* q_out, int heads_q, const vmonarch_tokens* k,
                    const vmonarch_tokens* k_out, int heads_k, long long tokens, int d, const int32_t* positions,
                    long long axis_stride, const vmonarch_rotary_plan* plan, int backward, void* stream);
int vmonarch_rotary_f32(const vmonarch_tokens* q, const vmonarch_tokens* q_out, int heads_q, const vmonarch_tokens* k,
                        const vmonarch_tokens* k_out, int heads_k, long long tokens, int d, const int32_t* positions,
                        long long axis_stride, const vmonarch_rotary_plan* plan, int backward, void* stream);

/* ---- attention over packed sequences --------------------------------------------------------------- */

/*
 * out[i] = sum_j softmax_j(scale * q[i] . k[j]) v[j] over the keys j of the query's own sequence that it sees.
 * q, out: heads_q heads, tokens_q tokens; k, v: heads_kv heads, tokens_k tokens.  q_starts and k_starts cut both into the
 * same n_seqs sequences (they may be the same array).  scale > 0 and finite.  lse (float32 [heads_q][tokens_q], may be
 * NULL): the natural log-sum-exp of each row's logits, for the backward pass.  No workspace.
 */
int vmonarch_packed_attention(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v,
                              const vmonarch_tokens* out, float* lse, const int32_t* q_starts, const int32_t* k_starts,
                              int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d,
                              float scale, int causal, void* stream);
int vmonarch_packed_attention_f32(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v,
                                  const vmonarch_tokens* out, float* lse, const int32_t* q_starts, const int32_t* k_starts,
                                  int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d,
                                  float scale, int causal, void* stream);

/*
 * Its backward pass: with P[i,j] = exp(scale q[i] . k[j] - lse[i]) and dS[i,j] = P (d_out[i] . v[j] - d_out[i] . out[i]),
 *   dq[i] = scale sum_j dS[i,j] k[j]     dk[j] = scale sum_i dS[i,j] q[i]     dv[j] = sum_i P[i,j] d_out[i],
 * dk and dv summed over the query heads that share a key head.  out and lse as the forward pass left them.  Rows of dk and dv that
 * no query sees are set to zero.  workspace: DEVICE, 256-byte aligned, at least
 * vmonarch_packed_attention_bwd_workspace_bytes(...) bytes for the call's type and sizes (0 on invalid ones, and without queries), or NULL for the
 * process-wide one.  (bf16: partial gradients of keys that many rows see are among them; float32, and bf16 that the bf16 matrix units do not take, need two
 * floats a row.)
 */
size_t vmonarch_packed_attention_bwd_workspace_bytes(int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d);
size_t vmonarch_packed_attention_bwd_workspace_bytes_f32(int n_seqs, long long tokens_q, long long tokens_k, int heads_q, int heads_kv, int d);
int vmonarch_packed_attention_bwd(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v,
                                  const vmonarch_tokens* out, const vmonarch_tokens* d_out, const float* lse,
                                  const vmonarch_tokens* dq, const vmonarch_tokens* dk, const vmonarch_tokens* dv,
                                  const int32_t* q_starts, const int32_t* k_starts, int n_seqs, long long tokens_q,
                                  long long tokens_k, int heads_q, int heads_kv, int d, float scale, int causal,
                                  void* workspace, size_t workspace_bytes, void* stream);
int vmonarch_packed_attention_bwd_f32(const vmonarch_tokens* q, const vmonarch_tokens* k, const vmonarch_tokens* v,
                                      const vmonarch_tokens* out, const vmonarch_tokens* d_out, const float* lse,
                                      const vmonarch_tokens* dq, const vmonarch_tokens* dk, const vmonarch_tokens* dv,
                                      const int32_t* q_starts, const int32_t* k_starts, int n_seqs, long long tokens_q,
                                      long long tokens_k, int heads_q, int heads_kv, int d, float scale, int causal,
                                      void* workspace, size_t workspace_bytes, void* stream);

/* ---- keys and values in pages ---------------------------------------------------------------------- */

/*
 * A cache of n_pages pages of page_size tokens each: element (page, slot, head, c) of the keys lies at
 * k[page * k_page_stride + slot * k_token_stride + head * k_head_stride + c], of the values likewise.  Token p of sequence s is
 * slot p % page_size of page table[s * table_stride + p / page_size] (DEVICE int32); lengths[s] (DEVICE int32) tokens of it are
 * there, the chunk of new ones last.  On the device lengths are clamped to [0, table_width * page_size]; an entry outside
 * [0, n_pages) is never followed: the writer skips its tokens, the reader takes page 0 in its place.
 */
typedef struct vmonarch_cache {
  void* k;
  void* v;
  long long k_page_stride, k_token_stride, k_head_stride;
  long long v_page_stride, v_token_stride, v_head_stride;
  int n_pages;
  int page_size;
  const int32_t* table;
  long long table_stride;
  int table_width;
  const int32_t* lengths;
} vmonarch_cache;

/*
 * Writes each sequence's chunk of new tokens, its packed tokens q_starts[s] .. q_starts[s + 1] - 1 of k and v, into the last slots
 * of its lengths[s]: chunk token i goes to position lengths[s] - chunk + i (below zero: skipped).  plan may be NULL; otherwise
 * keys are turned on the way as vmonarch_rotary does, at `positions` ([axes][tokens] as there) or, where that is NULL and the plan
 * has one axis, at the tokens' positions in the sequence.  No slot may be named twice.
 */
int vmonarch_paged_append(const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_cache* cache,
                          const int32_t* q_starts, int n_seqs, long long tokens, int heads_kv, int d,
                          const vmonarch_rotary_plan* plan, const int32_t* positions, long long axis_stride, void* stream);
int vmonarch_paged_append_f32(const vmonarch_tokens* k, const vmonarch_tokens* v, const vmonarch_cache* cache,
                              const int32_t* q_starts, int n_seqs, long long tokens, int heads_kv, int d,
                              const vmonarch_rotary_plan* plan, const int32_t* positions, long long axis_stride, void* stream);

/*
 * Attention of each sequence's chunk of new tokens (or its single one) over its lengths[s] cached tokens, the chunk's own
 * included: vmonarch_packed_attention with the keys and values of sequence s taken from its pages.  Few rows over long caches are
 * cut into ranges of keys and joined by a second launch; the cut, and with it the workspace, follows what the host knows (tokens, n_seqs, heads, the
 * mask, the longest sequence the table has room for), so the same sizes give the same bits.  Of a table with room for far more than is there give
 * the columns that the longest sequence needs (a smaller table_width at the same table_stride): its prompts are not cut then (8 of up to 2000 tokens, 12
 * heads, d = 128: 144 us with room for 2000 to 8192 tokens, 324 for 32,768).  workspace: DEVICE, 256-byte aligned, at least
 * vmonarch_paged_attention_workspace_bytes(...) bytes (0: none needed), or NULL for the process-wide one.
 */
size_t vmonarch_paged_attention_workspace_bytes(const vmonarch_cache* cache, int n_seqs, long long tokens, int heads_q,
                                                int heads_kv, int d);
int vmonarch_paged_attention(const vmonarch_tokens* q, const vmonarch_cache* cache, const vmonarch_tokens* out,
                             const int32_t* q_starts, int n_seqs, long long tokens, int heads_q, int heads_kv, int d,
                             float scale, int causal, void* workspace, size_t workspace_bytes, void* stream);
int vmonarch_paged_attention_f32(const vmonarch_tokens* q, const vmonarch_cache* cache, const vmonarch_tokens* out,
                                 const int32_t* q_starts, int n_seqs, long long tokens, int heads_q, int heads_kv, int d,
                                 float scale, int causal, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* VMONARCH_SEQUENCE_H_ */
