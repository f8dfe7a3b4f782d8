// Arguments of the sequence operators' kernels and their launchers (host side of seq_attention.hip and seq_rotate.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/per_seq.h"

namespace per {

// Rows of a pass over heads: head h of the pass reads head h / share.
struct SeqRows {
  void* d;
  int64_t batch, token, head;
  uint32_t share;
  uint32_t wide;   // address and strides are multiples of 16 bytes (and near)
  uint32_t near;   // the tokens of a chunk lie within 2^31 bytes of the first
};

// Rows as a caller gives them.
inline SeqRows rows(const per_seq_rows& r, uint32_t dtype, uint32_t share) {
  const int64_t per16 = dtype == PER_SEQ_BF16 ? 8 : 4;
  const bool near = r.token >= 0 && r.token < (1 << 24);
  const bool wide = near && (reinterpret_cast<uintptr_t>(r.d) & 15) == 0 && r.batch % per16 == 0 && r.token % per16 == 0 && r.head % per16 == 0;
  return SeqRows{r.d, r.batch, r.token, r.head, share, wide ? 1u : 0u, near ? 1u : 0u};
}
// Packed rows [B][L][heads][d] in fp32.
inline SeqRows packed(float* d, uint32_t L, uint32_t heads, uint32_t width, uint32_t share) {
  const bool near = (uint64_t)heads * width < (1 << 24);
  return SeqRows{d, (int64_t)L * heads * width, (int64_t)heads * width, (int64_t)width, share, near && width % 4 == 0, near};
}

struct SeqStates {
  float* d;
  int64_t batch, head;
};

// How states larger than the last cache are read and written (see k_attend_step.h).
enum Past { KEPT, STORES_PAST, ALL_PAST };
inline Past past(uint64_t state_bytes) { return state_bytes <= 256ull << 20 ? KEPT : state_bytes <= 768ull << 20 ? STORES_PAST : ALL_PAST; }

// Sizes of a linear attention.
struct AttentionSizes {
  uint32_t dtype, B, L, H, G, dk, dv;
  float scale;
  const float* log_decay;
  const int32_t* lengths;
};

size_t attention_work_bytes(const AttentionSizes& a, bool backward);
hipError_t launch_attention(const AttentionSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                            const per_seq_states* state, const per_seq_rows& out, const per_seq_states* out_state, void* work,
                            hipStream_t s);
hipError_t launch_attention_backward(const AttentionSizes& a, const per_seq_rows& dout, const per_seq_rows& q,
                                     const per_seq_rows& k, const per_seq_rows& v, const per_seq_states* state,
                                     const per_seq_states* dstate, const per_seq_rows& dq, const per_seq_rows& dk,
                                     const per_seq_rows& dv, const per_seq_states* dstate0, void* work, hipStream_t s);
hipError_t launch_attention_step(const AttentionSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                                 const per_seq_states& state, const per_seq_rows& out, hipStream_t s);

// Sizes of a gated delta rule; its gates [batch][token][head].
struct DeltaSizes {
  uint32_t dtype, B, L, H, Q, K, V, dk, dv;
  float scale;
  per_seq_gates log_decay, beta;
  const int32_t* lengths;
};

size_t delta_work_bytes(const DeltaSizes& a, bool backward);
hipError_t launch_delta(const DeltaSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v, const per_seq_states* state,
                        const per_seq_rows& out, const per_seq_states* out_state, void* work, hipStream_t s);
hipError_t launch_delta_backward(const DeltaSizes& a, const per_seq_rows& dout, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                                 const per_seq_states* state, const per_seq_states* dstate, const per_seq_rows& dq, const per_seq_rows& dk,
                                 const per_seq_rows& dv, const per_seq_gates& dlog_decay, const per_seq_gates& dbeta,
                                 const per_seq_states* dstate0, void* work, hipStream_t s);
hipError_t launch_delta_step(const DeltaSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                             const per_seq_states& state, const per_seq_rows& out, hipStream_t s);

// One tensor of a rotation: its rows, where they go, the norm's weight.
struct RotarySide {
  SeqRows x, out, dout;   // dout: gradients only
  const float* weight;
  uint32_t heads;
};
struct RotaryArgs {
  RotarySide side[2];     // queries, keys
  uint32_t B, L, dim, rot, layout;
  const int32_t* at;
  int64_t at_batch, at_token;
  const float* freqs;
  float magnitude, sign;  // sign: -1 turns the other way
  float eps;
  float* partial;         // gradients only: the workgroups' sums for the weights
  // heads in vectors: tokens that a workgroup takes at a time, how often there are so many; of a gradient by queries and keys, and
  // the workgroups of either
  uint32_t tokens[2], tiles[2], blocks[2];
};

// Rows of a block: layer norm and dropout.
struct BlockArgs {
  SeqRows x, more, out;   // more: dout, or the residual
  const float *weight, *bias;
  float *dweight, *dbias, *partial;
  uint32_t B, L, H, dim;
  float eps;
  uint32_t border;        // of 65536: dropped below
  uint64_t seed, offset;
  const int64_t* d_offset;
};
size_t norm_work_bytes(uint32_t dtype, const BlockArgs& a);
hipError_t launch_layer_norm(uint32_t dtype, const BlockArgs& a, hipStream_t s);
hipError_t launch_layer_norm_backward(uint32_t dtype, const BlockArgs& a, hipStream_t s);
hipError_t launch_dropout(uint32_t dtype, const BlockArgs& a, hipStream_t s);

enum RotaryKind { ROTATE, NORM_ROTATE, NORM_ROTATE_BACK };
size_t rotary_work_bytes(uint64_t tokens, uint32_t heads, uint32_t dim);
hipError_t launch_rotary(RotaryKind kind, uint32_t dtype, RotaryArgs a, float* dqw, float* dkw, hipStream_t s);

}  // namespace per
