/*
 * per_seq.h -- C-ABI of the sequence operators: what a learner of replayed sequences, and the actors beside it, run on
 * the rows that per.h samples.
 *
 * A row of the replay buffer may hold a stretch of an episode, its length and the state the agent had at its start.  The
 * operators here turn such rows into outputs and gradients, and advance the states of many actors by one token:
 *
 *   rotary positions         per_rotate
 *   norms of queries and     per_norm_rotate, per_norm_rotate_backward
 *   keys with the rotation
 *   linear attention with a  per_linear_attention (sequences), per_linear_attention_backward (their gradient),
 *   decay for each head      per_linear_attention_step (one token)
 *
 * Conventions (where they are not those of per.h)
 *  - No handle: every call stands for itself.  It only enqueues work on `stream`; errors are the PER_E* codes of per.h,
 *    found on the host before anything is enqueued.  The library allocates nothing: the caller provides the workspace
 *    where one is needed (sized by the *_workspace function, 256-byte aligned; its contents need not be kept).  Calls hold
 *    no state between them and may be captured into a HIP graph and replayed.
 *  - Element type of rows: PER_SEQ_BF16 or PER_SEQ_F32.  Sums, norms, states and weights are fp32.  A result is rounded to
 *    its type once, at the end; only sequences of linear attention and their gradients in bfloat16 round inside as well,
 *    where it says so.
 *  - Outputs must not overlap inputs or each other, except where a call says so.
 *  - A batch, a length or a number of heads of 0 is valid: nothing is written but states (which are then copied), and zeros
 *    for gradients of keys and values that no head reads.
 */
#ifndef PER_SEQ_H_
#define PER_SEQ_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PER_SEQ_BF16 1u
#define PER_SEQ_F32  2u

#define PER_SEQ_HALF        0u   /* pair p of a head: elements p and p + rot/2 */
#define PER_SEQ_INTERLEAVED 1u   /* pair p of a head: elements 2p and 2p + 1   */

/* Rows [batch][token][head][width] in device memory: strides in elements, the innermost dimension contiguous.  A stride of
 * 0 repeats an input.  Any alignment that the element type allows works; rows whose address and strides are multiples of 16
 * bytes are the fast ones. */
typedef struct per_seq_rows {
  void* d;
  int64_t batch, token, head;
} per_seq_rows;

/* States [batch][head][dk][dv] in fp32, the innermost two dimensions contiguous. */
typedef struct per_seq_states {
  float* d;
  int64_t batch, head;
} per_seq_states;

/* Positions [batch][token]; d == NULL: token t is at position t. */
typedef struct per_seq_positions {
  const int32_t* d;
  int64_t batch, token;
} per_seq_positions;

/* ---------------------------------------------------------------------------------------------- rotary positions */
typedef struct per_rotary_config {
  uint32_t struct_size;   /* sizeof(per_rotary_config)                                                           */
  uint32_t dtype;
  uint32_t batch, length;
  uint32_t heads;         /* of x, or of the queries                                                              */
  uint32_t kv_heads;      /* of the keys (ignored by per_rotate)                                                  */
  uint32_t dim;           /* width of a head, 1..256                                                              */
  uint32_t rot;           /* the first rot elements of a head are rotated: even, 0..dim                           */
  uint32_t layout;        /* PER_SEQ_HALF or PER_SEQ_INTERLEAVED                                                  */
  uint32_t inverse;       /* per_rotate: != 0 turns the other way (also the gradient of the rotation)             */
  float    magnitude;     /* the rotated elements are multiplied with it (scaled positions use values above 1)    */
  float    eps;           /* added to the mean square of a head (ignored by per_rotate)                           */
} per_rotary_config;

/* out = x with pair p of every head turned by position * d_freqs[p].  d_freqs: rot/2 values; the angle is formed and
 * reduced in 64 bits, so positions of any size keep their precision.  out may be x. */
int per_rotate(const per_rotary_config* c, const per_seq_rows* x, const per_seq_positions* at, const float* d_freqs,
               const per_seq_rows* out, void* stream);

/* q_out = rotation of (q / sqrt(mean over the head of q^2 + eps) * d_q_weight), and the same for the keys, in one pass.
 * d_*_weight: dim values, or NULL for ones.  q_out may be q, k_out may be k. */
int per_norm_rotate(const per_rotary_config* c, const per_seq_rows* q, const per_seq_rows* k, const float* d_q_weight,
                    const float* d_k_weight, const per_seq_positions* at, const float* d_freqs, const per_seq_rows* q_out,
                    const per_seq_rows* k_out, void* stream);

/* Its gradient: from dq_out, dk_out (those of its results) and its inputs to dq, dk and the weights' d_dq_weight,
 * d_dk_weight (dim values each, sums over all tokens and heads in a fixed order; NULL where not wanted).  dq may be dq_out,
 * dk may be dk_out. */
int per_norm_rotate_workspace(const per_rotary_config* c, size_t* bytes);
int per_norm_rotate_backward(const per_rotary_config* c, const per_seq_rows* dq_out, const per_seq_rows* dk_out,
                             const per_seq_rows* q, const per_seq_rows* k, const float* d_q_weight, const float* d_k_weight,
                             const per_seq_positions* at, const float* d_freqs, const per_seq_rows* dq, const per_seq_rows* dk,
                             float* d_dq_weight, float* d_dk_weight, void* d_work, size_t work_bytes, void* stream);

/* ---------------------------------------------------------------------- linear attention with a decay for each head */
typedef struct per_attention_config {
  uint32_t struct_size;   /* sizeof(per_attention_config)                                                         */
  uint32_t dtype;
  uint32_t batch, length;
  uint32_t heads;         /* of queries, outputs, states and decays                                               */
  uint32_t kv_heads;      /* of keys and values: divides heads, head h reads kv head h / (heads / kv_heads)       */
  uint32_t dk, dv;        /* widths, 1..128                                                                       */
  float    scale;         /* of the queries                                                                       */
} per_attention_config;

/* S[t] = exp(d_log_decay[h]) S[t-1] + k[t] v[t]^T,  out[t] = scale * q[t]^T S[t],  for t = 0 .. d_lengths[b]-1 of each
 * sequence and head, from S[-1] = state (NULL: zeros).
 *   d_log_decay : [heads] natural logarithms of the decays: at most 0; -infinity keeps nothing of the state
 *   d_lengths   : [batch] valid tokens of each sequence (values outside 0..length are taken as the nearest of these), or
 *                 NULL: all.  Tokens behind them are not read; their outputs are zeros.
 *   out_state   : S behind the last valid token, or NULL.  It may be state.
 * Rows in fp32 are computed to fp32's accuracy throughout.  Rows in bfloat16 are multiplied in bfloat16: the state that a
 * chunk of 32 tokens starts from and the decayed products of pairs of its tokens are rounded to it where they are factors
 * (each held, and summed, in fp32), so that an output carries up to three roundings of 2^-8, of its parts and of itself:
 * 2.3e-3 of the outputs by the 2-norm, where one rounding is 1.7e-3.  What a token adds to a state is rounded to 16 bits
 * where the state itself is no result, and to 24 where it is; outputs may differ by that much with out_state.
 * A value among the valid tokens, or of the state, that is not finite makes all outputs and states that depend on it not
 * finite (those of tokens before it do not). */
int per_linear_attention_workspace(const per_attention_config* c, int backward, size_t* bytes);
int per_linear_attention(const per_attention_config* c, const per_seq_rows* q, const per_seq_rows* k, const per_seq_rows* v,
                         const float* d_log_decay, const int32_t* d_lengths, const per_seq_states* state,
                         const per_seq_rows* out, const per_seq_states* out_state, void* d_work, size_t work_bytes, void* stream);

/* Its gradient, the decays being constants: from dout (of out) and dstate (of out_state; NULL: zeros) to dq, dk, dv and
 * dstate0 (of state; NULL where not wanted).  Gradients of keys and values that several heads share are sums in a fixed
 * order.  dstate0 may be dstate, and not state.  Of roundings, and of values that are not
 * finite, the same holds as above. */
int per_linear_attention_backward(const per_attention_config* c, const per_seq_rows* dout, const per_seq_rows* q,
                                  const per_seq_rows* k, const per_seq_rows* v, const float* d_log_decay,
                                  const int32_t* d_lengths, const per_seq_states* state, const per_seq_states* dstate,
                                  const per_seq_rows* dq, const per_seq_rows* dk, const per_seq_rows* dv,
                                  const per_seq_states* dstate0, void* d_work, size_t work_bytes, void* stream);

/* One token for every sequence (length must be 1), the states updated in place.  d_lengths[b] < 1: sequence b stands still
 * (its state is not touched, its output is zero). */
int per_linear_attention_step(const per_attention_config* c, const per_seq_rows* q, const per_seq_rows* k,
                              const per_seq_rows* v, const float* d_log_decay, const int32_t* d_lengths,
                              const per_seq_states* state, const per_seq_rows* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif  /* PER_SEQ_H_ */
