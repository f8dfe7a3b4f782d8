// C-ABI of the sequence operators: argument checks.  The kernels are in seq_attention.hip, seq_rotate.hip, seq_delta.hip and seq_block.hip.
#include <math.h>

#include "../../include/per.h"
#include "seq_geom.h"

using namespace per;

namespace {

int hip_rc(hipError_t e) { return e == hipSuccess ? PER_OK : PER_EHIP; }

uint32_t element(uint32_t dtype) { return dtype == PER_SEQ_BF16 ? 2u : 4u; }

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

struct Extent {
  uint32_t batch, token, head;
  bool empty() const { return !batch || !token || !head; }
};

bool readable(const per_seq_rows* r, const Extent& n, uint32_t dtype) {
  if (n.empty()) return true;
  return r && r->d && !misaligned(r->d, element(dtype));
}
// As readable, and no two rows at the same place.
bool writable(const per_seq_rows* r, const Extent& n, uint32_t dtype) {
  if (!readable(r, n, dtype)) return false;
  if (n.empty()) return true;
  return (n.batch == 1 || r->batch != 0) && (n.token == 1 || r->token != 0) && (n.head == 1 || r->head != 0);
}
bool state_ok(const per_seq_states* s, const per_attention_config* c, bool written) {
  if (!c->batch || !c->heads) return true;
  if (!s->d || misaligned(s->d, 4)) return false;
  return !written || ((c->batch == 1 || s->batch != 0) && (c->heads == 1 || s->head != 0));
}
bool same(const per_seq_rows* a, const per_seq_rows* b) { return a && b && a->d && a->d == b->d; }
per_seq_rows none() { return per_seq_rows{nullptr, 0, 0, 0}; }
const per_seq_rows& or_none(const per_seq_rows* r) {
  static const per_seq_rows empty = none();
  return r ? *r : empty;
}

// most: sequences times heads, so that a launch stays within 2^32 threads
int check_attention(const per_attention_config* c, uint32_t most = 1u << 21) {
  if (!c || c->struct_size != sizeof(per_attention_config)) return PER_EINVAL;
  if (c->dtype != PER_SEQ_BF16 && c->dtype != PER_SEQ_F32) return PER_EINVAL;
  if (c->dk < 1 || c->dk > 128 || c->dv < 1 || c->dv > 128) return PER_ERANGE;
  if (c->heads && (!c->kv_heads || c->heads % c->kv_heads)) return PER_EINVAL;
  if (c->length > (1u << 30) || (uint64_t)c->batch * c->heads > most) return PER_ERANGE;
  if (!isfinite(c->scale)) return PER_EINVAL;
  return PER_OK;
}

AttentionSizes sizes(const per_attention_config* c, const float* log_decay, const int32_t* lengths) {
  return AttentionSizes{c->dtype, c->batch, c->length, c->heads, c->kv_heads, c->dk, c->dv, c->scale, log_decay, lengths};
}

int check_rotary(const per_rotary_config* c, bool pair) {
  if (!c || c->struct_size != sizeof(per_rotary_config)) return PER_EINVAL;
  if (c->dtype != PER_SEQ_BF16 && c->dtype != PER_SEQ_F32) return PER_EINVAL;
  if (c->dim < 1 || c->dim > 256) return PER_ERANGE;
  if (c->rot > c->dim || (c->rot & 1) || c->layout > PER_SEQ_INTERLEAVED) return PER_EINVAL;
  if (!isfinite(c->magnitude)) return PER_EINVAL;
  if (pair && !(c->eps >= 0.0f && isfinite(c->eps))) return PER_EINVAL;
  const uint64_t heads = (uint64_t)c->heads + (pair ? c->kv_heads : 0);
  if (heads > (1u << 16) || (uint64_t)c->batch * c->length > (1ull << 31)) return PER_ERANGE;
  return PER_OK;
}

RotarySide side(const per_rotary_config* c, uint32_t heads, const per_seq_rows* x, const per_seq_rows* out, const per_seq_rows* dout,
                const float* weight) {
  auto rows = [&](const per_seq_rows* r) {
    const per_seq_rows& q = or_none(r);
    const uint32_t per16 = 16 / element(c->dtype);
    const bool wide = !misaligned(q.d, 16) && q.batch % per16 == 0 && q.token % per16 == 0 && q.head % per16 == 0;
    return SeqRows{q.d, q.batch, q.token, q.head, 1, wide ? 1u : 0u, 0};
  };
  return RotarySide{rows(x), rows(out), rows(dout), weight, heads};
}

RotaryArgs rotary(const per_rotary_config* c, const per_seq_positions* at, const float* freqs) {
  RotaryArgs a{};
  a.B = c->batch;
  a.L = c->length;
  a.dim = c->dim;
  a.rot = c->rot;
  a.layout = c->layout;
  if (at) { a.at = at->d; a.at_batch = at->batch; a.at_token = at->token; }
  a.freqs = freqs;
  a.magnitude = c->magnitude;
  a.sign = c->inverse ? -1.0f : 1.0f;
  a.eps = c->eps;
  return a;
}

bool tables_ok(const per_rotary_config* c, const per_seq_positions* at, const float* freqs) {
  if (c->rot && (!freqs || misaligned(freqs, 4))) return false;
  return !at || !at->d || !misaligned(at->d, 4);
}

// Launches stay within 2^32 threads: a workgroup for each sequence and head and up to 64 columns, or for each 32 tokens of it.
int check_delta(const per_delta_config* c, bool step = false) {
  if (!c || c->struct_size != sizeof(per_delta_config)) return PER_EINVAL;
  if (c->dtype != PER_SEQ_BF16 && c->dtype != PER_SEQ_F32) return PER_EINVAL;
  if (c->dk < 1 || c->dk > 128 || c->dv < 1 || c->dv > 128) return PER_ERANGE;
  for (uint32_t n : {c->q_heads, c->k_heads, c->v_heads})
    if (c->heads ? !n || c->heads % n : n != 0) return PER_EINVAL;
  const uint64_t rows = (uint64_t)c->batch * c->heads;
  if (rows > (step ? 1u << 23 : 1u << 22) || c->length > (1u << 29)) return PER_ERANGE;
  if (!step && rows * ((c->length + 31) / 32) >= (1u << 24)) return PER_ERANGE;
  if (!isfinite(c->scale)) return PER_EINVAL;
  return PER_OK;
}
bool gates_ok(const per_seq_gates* g, const Extent& n, bool written) {
  if (n.empty()) return true;
  if (!g || !g->d || misaligned(g->d, 4)) return false;
  return !written || ((n.batch == 1 || g->batch != 0) && (n.token == 1 || g->token != 0) && (n.head == 1 || g->head != 0));
}
bool states_ok(const per_seq_states* s, const per_delta_config* c, bool written) {
  if (!s->d || misaligned(s->d, 4)) return false;
  return !written || ((c->batch == 1 || s->batch != 0) && (c->heads == 1 || s->head != 0));
}
DeltaSizes sizes(const per_delta_config* c, const per_seq_gates* log_decay, const per_seq_gates* beta, const int32_t* lengths) {
  const per_seq_gates none{nullptr, 0, 0, 0};
  return DeltaSizes{c->dtype, c->batch, c->length, c->heads, c->q_heads, c->k_heads, c->v_heads, c->dk, c->dv, c->scale,
                    log_decay ? *log_decay : none, beta ? *beta : none, lengths};
}

int check_block(const per_block_config* c, uint32_t widest = 65536) {
  if (!c || c->struct_size != sizeof(per_block_config)) return PER_EINVAL;
  if (c->dtype != PER_SEQ_BF16 && c->dtype != PER_SEQ_F32) return PER_EINVAL;
  if (c->dim < 1 || c->dim > widest) return PER_ERANGE;
  const uint64_t tokens = (uint64_t)c->batch * c->length;
  if (tokens > (1ull << 31) || tokens * c->heads > (1ull << 31)) return PER_ERANGE;
  return PER_OK;
}
BlockArgs block(const per_block_config* c) {
  BlockArgs a{};
  a.B = c->batch;
  a.L = c->length;
  a.H = c->heads;
  a.dim = c->dim;
  a.eps = c->eps;
  return a;
}
SeqRows block_rows(const per_seq_rows* r) {
  const per_seq_rows& q = or_none(r);
  return SeqRows{q.d, q.batch, q.token, q.head, 1, 0, 0};
}

}  // namespace

extern "C" {

int per_rotate(const per_rotary_config* c, const per_seq_rows* x, const per_seq_positions* at, const float* d_freqs,
               const per_seq_rows* out, void* stream) {
  int rc = check_rotary(c, false);
  if (rc != PER_OK) return rc;
  const Extent n{c->batch, c->length, c->heads};
  if (n.empty()) return PER_OK;
  if (!readable(x, n, c->dtype) || !writable(out, n, c->dtype) || !tables_ok(c, at, d_freqs)) return PER_EINVAL;
  RotaryArgs a = rotary(c, at, d_freqs);
  a.side[0] = side(c, c->heads, x, out, nullptr, nullptr);
  return hip_rc(launch_rotary(ROTATE, c->dtype, a, nullptr, nullptr, static_cast<hipStream_t>(stream)));
}

int per_norm_rotate(const per_rotary_config* c, const per_seq_rows* q, const per_seq_rows* k, const float* d_q_weight,
                    const float* d_k_weight, const per_seq_positions* at, const float* d_freqs, const per_seq_rows* q_out,
                    const per_seq_rows* k_out, void* stream) {
  int rc = check_rotary(c, true);
  if (rc != PER_OK) return rc;
  const Extent nq{c->batch, c->length, c->heads}, nk{c->batch, c->length, c->kv_heads};
  if (nq.empty() && nk.empty()) return PER_OK;
  if (!readable(q, nq, c->dtype) || !readable(k, nk, c->dtype) || !writable(q_out, nq, c->dtype) || !writable(k_out, nk, c->dtype) ||
      !tables_ok(c, at, d_freqs) || misaligned(d_q_weight, 4) || misaligned(d_k_weight, 4))
    return PER_EINVAL;
  RotaryArgs a = rotary(c, at, d_freqs);
  a.side[0] = side(c, c->heads, q, q_out, nullptr, d_q_weight);
  a.side[1] = side(c, c->kv_heads, k, k_out, nullptr, d_k_weight);
  return hip_rc(launch_rotary(NORM_ROTATE, c->dtype, a, nullptr, nullptr, static_cast<hipStream_t>(stream)));
}

int per_norm_rotate_workspace(const per_rotary_config* c, size_t* bytes) {
  int rc = check_rotary(c, true);
  if (rc != PER_OK) return rc;
  if (!bytes) return PER_EINVAL;
  *bytes = rotary_work_bytes((uint64_t)c->batch * c->length, c->heads + c->kv_heads, c->dim);
  return PER_OK;
}

int per_norm_rotate_backward(const per_rotary_config* c, const per_seq_rows* dq_out, const per_seq_rows* dk_out,
                             const per_seq_rows* q, const per_seq_rows* k, const float* d_q_weight, const float* d_k_weight,
                             const per_seq_positions* at, const float* d_freqs, const per_seq_rows* dq, const per_seq_rows* dk,
                             float* d_dq_weight, float* d_dk_weight, void* d_work, size_t work_bytes, void* stream) {
  int rc = check_rotary(c, true);
  if (rc != PER_OK) return rc;
  const Extent nq{c->batch, c->length, c->heads}, nk{c->batch, c->length, c->kv_heads};
  if (!readable(q, nq, c->dtype) || !readable(k, nk, c->dtype) || !readable(dq_out, nq, c->dtype) || !readable(dk_out, nk, c->dtype) ||
      !writable(dq, nq, c->dtype) || !writable(dk, nk, c->dtype) || !tables_ok(c, at, d_freqs) || misaligned(d_q_weight, 4) ||
      misaligned(d_k_weight, 4) || misaligned(d_dq_weight, 4) || misaligned(d_dk_weight, 4))
    return PER_EINVAL;
  const size_t need = rotary_work_bytes((uint64_t)c->batch * c->length, c->heads + c->kv_heads, c->dim);
  if (need && (!d_work || misaligned(d_work, 256))) return PER_EINVAL;
  if (work_bytes < need) return PER_ENOMEM;
  if (nq.empty() && nk.empty() && !d_dq_weight && !d_dk_weight) return PER_OK;
  RotaryArgs a = rotary(c, at, d_freqs);
  a.side[0] = side(c, c->heads, q, dq, dq_out, d_q_weight);
  a.side[1] = side(c, c->kv_heads, k, dk, dk_out, d_k_weight);
  a.partial = static_cast<float*>(d_work);
  return hip_rc(launch_rotary(NORM_ROTATE_BACK, c->dtype, a, d_dq_weight, d_dk_weight, static_cast<hipStream_t>(stream)));
}

int per_linear_attention_workspace(const per_attention_config* c, int backward, size_t* bytes) {
  int rc = check_attention(c);
  if (rc != PER_OK) return rc;
  if (!bytes) return PER_EINVAL;
  *bytes = attention_work_bytes(sizes(c, nullptr, nullptr), backward != 0);
  return PER_OK;
}

int per_linear_attention(const per_attention_config* c, const per_seq_rows* q, const per_seq_rows* k, const per_seq_rows* v,
                         const float* d_log_decay, const int32_t* d_lengths, const per_seq_states* state,
                         const per_seq_rows* out, const per_seq_states* out_state, void* d_work, size_t work_bytes, void* stream) {
  int rc = check_attention(c);
  if (rc != PER_OK) return rc;
  const Extent nq{c->batch, c->length, c->heads}, nk{c->batch, c->length, c->kv_heads};
  if (!c->batch || !c->heads) return PER_OK;
  if (!readable(q, nq, c->dtype) || !readable(k, nk, c->dtype) || !readable(v, nk, c->dtype) || !writable(out, nq, c->dtype)) return PER_EINVAL;
  if (!d_log_decay || misaligned(d_log_decay, 4) || misaligned(d_lengths, 4)) return PER_EINVAL;
  if ((state && !state_ok(state, c, false)) || (out_state && !state_ok(out_state, c, true))) return PER_EINVAL;
  if (same(out, q) || same(out, k) || same(out, v)) return PER_EINVAL;
  const AttentionSizes a = sizes(c, d_log_decay, d_lengths);
  const size_t need = attention_work_bytes(a, false);
  if (need && (!d_work || misaligned(d_work, 256))) return PER_EINVAL;
  if (work_bytes < need) return PER_ENOMEM;
  return hip_rc(launch_attention(a, or_none(q), or_none(k), or_none(v), state, or_none(out), out_state, d_work, static_cast<hipStream_t>(stream)));
}

int per_linear_attention_backward(const per_attention_config* c, const per_seq_rows* dout, const per_seq_rows* q,
                                  const per_seq_rows* k, const per_seq_rows* v, const float* d_log_decay,
                                  const int32_t* d_lengths, const per_seq_states* state, const per_seq_states* dstate,
                                  const per_seq_rows* dq, const per_seq_rows* dk, const per_seq_rows* dv,
                                  const per_seq_states* dstate0, void* d_work, size_t work_bytes, void* stream) {
  int rc = check_attention(c);
  if (rc != PER_OK) return rc;
  const Extent nq{c->batch, c->length, c->heads}, nk{c->batch, c->length, c->kv_heads};
  if (!c->batch || (!c->heads && nk.empty())) return PER_OK;
  if (!readable(dout, nq, c->dtype) || !readable(q, nq, c->dtype) || !readable(k, nk, c->dtype) || !readable(v, nk, c->dtype)) return PER_EINVAL;
  if (!writable(dq, nq, c->dtype) || !writable(dk, nk, c->dtype) || !writable(dv, nk, c->dtype)) return PER_EINVAL;
  if ((c->heads && !d_log_decay) || misaligned(d_log_decay, 4) || misaligned(d_lengths, 4)) return PER_EINVAL;
  if ((state && !state_ok(state, c, false)) || (dstate && !state_ok(dstate, c, false)) || (dstate0 && !state_ok(dstate0, c, true))) return PER_EINVAL;
  if (c->heads && state && dstate0 && state->d == dstate0->d) return PER_EINVAL;
  for (const per_seq_rows* o : {dq, dk, dv})
    for (const per_seq_rows* i : {dout, q, k, v})
      if (same(o, i)) return PER_EINVAL;
  if (same(dq, dk) || same(dq, dv) || same(dk, dv)) return PER_EINVAL;
  const AttentionSizes a = sizes(c, d_log_decay, d_lengths);
  const size_t need = attention_work_bytes(a, true);
  if (need && (!d_work || misaligned(d_work, 256))) return PER_EINVAL;
  if (work_bytes < need) return PER_ENOMEM;
  return hip_rc(launch_attention_backward(a, or_none(dout), or_none(q), or_none(k), or_none(v), state, dstate, or_none(dq), or_none(dk),
                                          or_none(dv), dstate0, d_work, static_cast<hipStream_t>(stream)));
}

int per_linear_attention_step(const per_attention_config* c, const per_seq_rows* q, const per_seq_rows* k,
                              const per_seq_rows* v, const float* d_log_decay, const int32_t* d_lengths,
                              const per_seq_states* state, const per_seq_rows* out, void* stream) {
  int rc = check_attention(c, 1u << 23);
  if (rc != PER_OK) return rc;
  if (c->length != 1) return PER_ERANGE;
  const Extent nq{c->batch, 1, c->heads}, nk{c->batch, 1, c->kv_heads};
  if (!c->batch || !c->heads) return PER_OK;
  if (!readable(q, nq, c->dtype) || !readable(k, nk, c->dtype) || !readable(v, nk, c->dtype) || !writable(out, nq, c->dtype)) return PER_EINVAL;
  if (!d_log_decay || misaligned(d_log_decay, 4) || misaligned(d_lengths, 4) || !state || !state_ok(state, c, true)) return PER_EINVAL;
  if (same(out, q) || same(out, k) || same(out, v)) return PER_EINVAL;
  return hip_rc(launch_attention_step(sizes(c, d_log_decay, d_lengths), *q, *k, *v, *state, *out, static_cast<hipStream_t>(stream)));
}

int per_gated_delta_workspace(const per_delta_config* c, int backward, size_t* bytes) {
  int rc = check_delta(c);
  if (rc != PER_OK) return rc;
  if (!bytes) return PER_EINVAL;
  *bytes = delta_work_bytes(sizes(c, nullptr, nullptr, nullptr), backward != 0);
  return PER_OK;
}

int per_gated_delta(const per_delta_config* c, const per_seq_rows* q, const per_seq_rows* k, const per_seq_rows* v,
                    const per_seq_gates* log_decay, const per_seq_gates* beta, const int32_t* d_lengths, const per_seq_states* state,
                    const per_seq_rows* out, const per_seq_states* out_state, void* d_work, size_t work_bytes, void* stream) {
  int rc = check_delta(c);
  if (rc != PER_OK) return rc;
  if (!c->batch || !c->heads) return PER_OK;
  const Extent n{c->batch, c->length, c->heads}, nq{c->batch, c->length, c->q_heads}, nk{c->batch, c->length, c->k_heads}, nv{c->batch, c->length, c->v_heads};
  if (!readable(q, nq, c->dtype) || !readable(k, nk, c->dtype) || !readable(v, nv, c->dtype) || !writable(out, n, c->dtype)) return PER_EINVAL;
  if (!gates_ok(log_decay, n, false) || !gates_ok(beta, n, false) || misaligned(d_lengths, 4)) return PER_EINVAL;
  if ((state && !states_ok(state, c, false)) || (out_state && !states_ok(out_state, c, true))) return PER_EINVAL;
  if (same(out, q) || same(out, k) || same(out, v)) return PER_EINVAL;
  const DeltaSizes a = sizes(c, log_decay, beta, d_lengths);
  const size_t need = delta_work_bytes(a, false);
  if (need && (!d_work || misaligned(d_work, 256))) return PER_EINVAL;
  if (work_bytes < need) return PER_ENOMEM;
  return hip_rc(launch_delta(a, or_none(q), or_none(k), or_none(v), state, or_none(out), out_state, d_work, static_cast<hipStream_t>(stream)));
}

int per_gated_delta_backward(const per_delta_config* c, const per_seq_rows* dout, const per_seq_rows* q, const per_seq_rows* k,
                             const per_seq_rows* v, const per_seq_gates* log_decay, const per_seq_gates* beta,
                             const int32_t* d_lengths, const per_seq_states* state, const per_seq_states* dstate,
                             const per_seq_rows* dq, const per_seq_rows* dk, const per_seq_rows* dv,
                             const per_seq_gates* dlog_decay, const per_seq_gates* dbeta, const per_seq_states* dstate0,
                             void* d_work, size_t work_bytes, void* stream) {
  int rc = check_delta(c);
  if (rc != PER_OK) return rc;
  if (!c->batch || !c->heads) return PER_OK;
  const Extent n{c->batch, c->length, c->heads}, nq{c->batch, c->length, c->q_heads}, nk{c->batch, c->length, c->k_heads}, nv{c->batch, c->length, c->v_heads};
  if (!readable(dout, n, c->dtype) || !readable(q, nq, c->dtype) || !readable(k, nk, c->dtype) || !readable(v, nv, c->dtype)) return PER_EINVAL;
  if (!writable(dq, nq, c->dtype) || !writable(dk, nk, c->dtype) || !writable(dv, nv, c->dtype)) return PER_EINVAL;
  if (!gates_ok(log_decay, n, false) || !gates_ok(beta, n, false) || !gates_ok(dlog_decay, n, true) || !gates_ok(dbeta, n, true) ||
      misaligned(d_lengths, 4))
    return PER_EINVAL;
  if ((state && !states_ok(state, c, false)) || (dstate && !states_ok(dstate, c, false)) || (dstate0 && !states_ok(dstate0, c, true))) return PER_EINVAL;
  if (state && dstate0 && state->d == dstate0->d) return PER_EINVAL;
  if (!n.empty()) {
    for (const per_seq_rows* o : {dq, dk, dv})
      for (const per_seq_rows* i : {dout, q, k, v})
        if (same(o, i)) return PER_EINVAL;
    if (same(dq, dk) || same(dq, dv) || same(dk, dv)) return PER_EINVAL;
    const float* gate[4] = {dlog_decay->d, dbeta->d, log_decay->d, beta->d};
    if (gate[0] == gate[1] || gate[0] == gate[2] || gate[0] == gate[3] || gate[1] == gate[2] || gate[1] == gate[3]) return PER_EINVAL;
  }
  const DeltaSizes a = sizes(c, log_decay, beta, d_lengths);
  const size_t need = delta_work_bytes(a, true);
  if (need && (!d_work || misaligned(d_work, 256))) return PER_EINVAL;
  if (work_bytes < need) return PER_ENOMEM;
  const per_seq_gates none_g{nullptr, 0, 0, 0};
  return hip_rc(launch_delta_backward(a, or_none(dout), or_none(q), or_none(k), or_none(v), state, dstate, or_none(dq), or_none(dk), or_none(dv),
                                      dlog_decay ? *dlog_decay : none_g, dbeta ? *dbeta : none_g, dstate0, d_work, static_cast<hipStream_t>(stream)));
}

int per_gated_delta_step(const per_delta_config* c, const per_seq_rows* q, const per_seq_rows* k, const per_seq_rows* v,
                         const per_seq_gates* log_decay, const per_seq_gates* beta, const int32_t* d_lengths,
                         const per_seq_states* state, const per_seq_rows* out, void* stream) {
  int rc = check_delta(c, true);
  if (rc != PER_OK) return rc;
  if (c->length != 1) return PER_ERANGE;
  if (!c->batch || !c->heads) return PER_OK;
  const Extent n{c->batch, 1, c->heads}, nq{c->batch, 1, c->q_heads}, nk{c->batch, 1, c->k_heads}, nv{c->batch, 1, c->v_heads};
  if (!readable(q, nq, c->dtype) || !readable(k, nk, c->dtype) || !readable(v, nv, c->dtype) || !writable(out, n, c->dtype)) return PER_EINVAL;
  if (!gates_ok(log_decay, n, false) || !gates_ok(beta, n, false) || misaligned(d_lengths, 4) || !state || !states_ok(state, c, true)) return PER_EINVAL;
  if (same(out, q) || same(out, k) || same(out, v)) return PER_EINVAL;
  return hip_rc(launch_delta_step(sizes(c, log_decay, beta, d_lengths), *q, *k, *v, *state, *out, static_cast<hipStream_t>(stream)));
}

int per_layer_norm(const per_block_config* c, const per_seq_rows* x, const float* d_weight, const float* d_bias,
                   const per_seq_rows* out, void* stream) {
  int rc = check_block(c);
  if (rc != PER_OK) return rc;
  if (!(c->eps >= 0.0f && isfinite(c->eps))) return PER_EINVAL;
  const Extent n{c->batch, c->length, c->heads};
  if (n.empty()) return PER_OK;
  if (!readable(x, n, c->dtype) || !writable(out, n, c->dtype) || misaligned(d_weight, 4) || misaligned(d_bias, 4)) return PER_EINVAL;
  BlockArgs a = block(c);
  a.x = block_rows(x);
  a.out = block_rows(out);
  a.weight = d_weight;
  a.bias = d_bias;
  return hip_rc(launch_layer_norm(c->dtype, a, static_cast<hipStream_t>(stream)));
}

int per_layer_norm_workspace(const per_block_config* c, size_t* bytes) {
  int rc = check_block(c);
  if (rc != PER_OK) return rc;
  if (!bytes) return PER_EINVAL;
  *bytes = norm_work_bytes(c->dtype, block(c));
  return PER_OK;
}

int per_layer_norm_backward(const per_block_config* c, const per_seq_rows* dout, const per_seq_rows* x, const float* d_weight,
                            const per_seq_rows* dx, float* d_dweight, float* d_dbias, void* d_work, size_t work_bytes, void* stream) {
  int rc = check_block(c);
  if (rc != PER_OK) return rc;
  if (!(c->eps >= 0.0f && isfinite(c->eps))) return PER_EINVAL;
  const Extent n{c->batch, c->length, c->heads};
  if (!readable(x, n, c->dtype) || !readable(dout, n, c->dtype) || !writable(dx, n, c->dtype) || misaligned(d_weight, 4) ||
      misaligned(d_dweight, 4) || misaligned(d_dbias, 4))
    return PER_EINVAL;
  if (!n.empty() && same(dx, x)) return PER_EINVAL;
  if (d_dweight && d_dweight == d_dbias) return PER_EINVAL;
  BlockArgs a = block(c);
  const size_t need = norm_work_bytes(c->dtype, a);
  if (need && (!d_work || misaligned(d_work, 256))) return PER_EINVAL;
  if (work_bytes < need) return PER_ENOMEM;
  if (n.empty() && !d_dweight && !d_dbias) return PER_OK;
  a.x = block_rows(x);
  a.more = block_rows(dout);
  a.out = block_rows(dx);
  a.weight = d_weight;
  a.dweight = d_dweight;
  a.dbias = d_dbias;
  a.partial = static_cast<float*>(d_work);
  return hip_rc(launch_layer_norm_backward(c->dtype, a, static_cast<hipStream_t>(stream)));
}

int per_dropout(const per_block_config* c, const per_seq_rows* x, const per_seq_rows* residual, const int64_t* d_offset,
                const per_seq_rows* out, void* stream) {
  int rc = check_block(c, ~0u);
  if (rc != PER_OK) return rc;
  if (!(c->p >= 0.0f && c->p < 1.0f)) return PER_EINVAL;
  const Extent n{c->batch, c->length, c->heads};
  if (n.empty()) return PER_OK;
  if (!readable(x, n, c->dtype) || !writable(out, n, c->dtype) || (residual && !readable(residual, n, c->dtype)) || misaligned(d_offset, 8)) return PER_EINVAL;
  BlockArgs a = block(c);
  a.x = block_rows(x);
  a.out = block_rows(out);
  if (residual) a.more = block_rows(residual);
  const double border = floor((double)c->p * 65536.0 + 0.5);
  a.border = border > 65535.0 ? 65535u : (uint32_t)border;
  a.seed = c->seed;
  a.offset = c->offset;
  a.d_offset = d_offset;
  return hip_rc(launch_dropout(c->dtype, a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
