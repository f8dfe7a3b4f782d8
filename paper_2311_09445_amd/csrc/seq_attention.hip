// Linear attention with a decay for each head.
//
// Every direction is the same pass.  With rows x, y, z of a head taken in order i = 0, 1, ...
//   out[i] = c_in  sum over j <= i of decay^(i-j) (x[i].y[j]) z[j]  +  c_out decay^(i+1-lag) x[i]^T S
//   S      = decay^n S + c_state sum over j of decay^(n-1-j+lag) y[j] z[j]^T
//     out          : x, y, z = q, k, v;     S the state;                          lag 0
//     gradient of q:           dout, v, k;  S the state, transposed;              lag 0
//     gradient of v:           k, q, dout;  S the state's gradient; against time, lag 1
//     gradient of k:           v, dout, q;  the same, transposed;   against time, lag 1
#include "dev_seq.h"

namespace per {

namespace {

struct AttentionPass {
  SeqRows x, y, z, out;
  uint32_t L, H, dx, dz;
  uint32_t back;                 // against time (and lag 1)
  float c_in, c_state, c_out;
  const float* log_decay;
  const int32_t* lengths;
  // states [b][h], element (i of dx, j of dz) at i * in_x + j * in_z
  const float* in;
  int64_t in_batch, in_head;
  uint32_t in_x, in_z;
  float* to;
  int64_t to_batch, to_head;
};

template <typename T, typename O>
__global__ __launch_bounds__(128) void k_attend_tokens(AttentionPass p) {
  __shared__ float xs[128], ys[128];
  const uint32_t h = blockIdx.x % p.H, b = blockIdx.x / p.H, j = threadIdx.x;
  const uint32_t n = valid_tokens(p.lengths, b, p.L);
  const float decay = expf(p.log_decay[h]);
  float S[128];
#pragma unroll
  for (uint32_t i = 0; i < 128; ++i) {
    S[i] = 0.0f;
    if (p.in && i < p.dx && j < p.dz) S[i] = p.in[(int64_t)b * p.in_batch + (int64_t)h * p.in_head + (int64_t)i * p.in_x + (int64_t)j * p.in_z];
  }
  for (uint32_t i = 0; i < p.L; ++i) {
    const uint32_t t = i < n && p.back ? n - 1 - i : i;
    float sum = 0.0f;
    if (i < n) {
      __syncthreads();
      xs[j] = j < p.dx ? as_float(row_of<T>(p.x, b, t, h)[j]) : 0.0f;
      ys[j] = j < p.dx ? as_float(row_of<T>(p.y, b, t, h)[j]) : 0.0f;
      __syncthreads();
      const float z = j < p.dz ? as_float(row_of<T>(p.z, b, t, h)[j]) : 0.0f;
      float dot = 0.0f;
#pragma unroll
      for (uint32_t m = 0; m < 128; ++m) {
        if (!p.back) S[m] *= decay;
        sum = fmaf(xs[m], S[m], sum);
        dot = fmaf(xs[m], ys[m], dot);
        S[m] = fmaf(ys[m], z * p.c_state, S[m]);
        if (p.back) S[m] *= decay;
      }
      sum = p.c_out * sum + p.c_in * dot * z;
    }
    if (j < p.dz) row_to<O>(p.out, b, t, h)[j] = (O)sum;
  }
  if (p.to && j < p.dz)
#pragma unroll
    for (uint32_t i = 0; i < 128; ++i)
      if (i < p.dx) p.to[(int64_t)b * p.to_batch + (int64_t)h * p.to_head + (int64_t)i * p.dz + j] = S[i];
}

// Rows of heads that share one, added up: from [B][L][H][d] in fp32 to [B][L][G][d].
template <typename T>
__global__ __launch_bounds__(256) void k_fold_heads(const float* from, SeqRows to, uint32_t L, uint32_t G, uint32_t share, uint32_t d, uint64_t n) {
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const uint32_t e = (uint32_t)(i % d);
  const uint64_t row = i / d;
  const uint32_t g = (uint32_t)(row % G), t = (uint32_t)(row / G % L), b = (uint32_t)(row / G / L);
  float sum = 0.0f;
  for (uint32_t m = 0; m < share; ++m) sum += from[((row / G * G + g) * share + m) * d + e];
  row_to<T>(to, b, t, g)[e] = (T)sum;
}

template <typename T>
__global__ __launch_bounds__(128) void k_attend_step(SeqRows q, SeqRows k, SeqRows v, SeqStates st, SeqRows out, uint32_t H, uint32_t dk, uint32_t dv,
                                                     float scale, const float* log_decay, const int32_t* lengths) {
  const uint32_t h = blockIdx.x % H, b = blockIdx.x / H, j = threadIdx.x;
  if (j >= dv) return;
  T* o = row_to<T>(out, b, 0, h);
  if (lengths && lengths[b] < 1) {
    o[j] = (T)0.0f;
    return;
  }
  const T *x = row_of<T>(q, b, 0, h), *y = row_of<T>(k, b, 0, h);
  const float z = as_float(row_of<T>(v, b, 0, h)[j]), decay = expf(log_decay[h]);
  float* S = st.d + (int64_t)b * st.batch + (int64_t)h * st.head + j;
  float sum = 0.0f;
  for (uint32_t i = 0; i < dk; ++i) {
    const float s = fmaf(as_float(y[i]), z, S[(size_t)i * dv] * decay);
    S[(size_t)i * dv] = s;
    sum = fmaf(as_float(x[i]), s, sum);
  }
  o[j] = (T)(scale * sum);
}

SeqRows rows(const per_seq_rows& r, uint32_t dtype, uint32_t share) {
  const int64_t per16 = dtype == PER_SEQ_BF16 ? 8 : 4;
  const bool wide = (reinterpret_cast<uintptr_t>(r.d) & 15) == 0 && r.batch % per16 == 0 && r.token % per16 == 0 && r.head % per16 == 0;
  return SeqRows{r.d, r.batch, r.token, r.head, share, wide ? 1u : 0u};
}
// Packed rows [B][L][H][d] in fp32.
SeqRows packed(float* d, const AttentionSizes& a, uint32_t width) {
  return SeqRows{d, (int64_t)a.L * a.H * width, (int64_t)a.H * width, (int64_t)width, 1, 0};
}

AttentionPass make_pass(const AttentionSizes& a, bool back, uint32_t dx, uint32_t dz) {
  AttentionPass p{};
  p.L = a.L;
  p.H = a.H;
  p.dx = dx;
  p.dz = dz;
  p.back = back;
  p.c_in = a.scale;
  p.c_state = back ? a.scale : 1.0f;
  p.c_out = back ? 1.0f : a.scale;
  p.log_decay = a.log_decay;
  p.lengths = a.lengths;
  return p;
}
void from_states(AttentionPass* p, const per_seq_states* s, uint32_t dv, bool transposed) {
  if (!s) return;
  p->in = s->d;
  p->in_batch = s->batch;
  p->in_head = s->head;
  p->in_x = transposed ? 1 : dv;
  p->in_z = transposed ? dv : 1;
}
void to_states(AttentionPass* p, const per_seq_states* s) {
  if (!s) return;
  p->to = s->d;
  p->to_batch = s->batch;
  p->to_head = s->head;
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T, typename O>
hipError_t run_pass(const AttentionSizes& a, const AttentionPass& p, hipStream_t s) {
  k_attend_tokens<T, O><<<a.B * a.H, 128, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T>
hipError_t forward(const AttentionSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                   const per_seq_states* state, const per_seq_rows& out, const per_seq_states* out_state, void*, hipStream_t s) {
  const uint32_t share = a.H / a.G;
  AttentionPass p = make_pass(a, false, a.dk, a.dv);
  p.x = rows(q, a.dtype, 1);
  p.y = rows(k, a.dtype, share);
  p.z = rows(v, a.dtype, share);
  p.out = rows(out, a.dtype, 1);
  from_states(&p, state, a.dv, false);
  to_states(&p, out_state);
  return run_pass<T, T>(a, p, s);
}

template <typename T>
hipError_t backward(const AttentionSizes& a, const per_seq_rows& dout, const per_seq_rows& q, const per_seq_rows& k,
                    const per_seq_rows& v, const per_seq_states* state, const per_seq_states* dstate, const per_seq_rows& dq,
                    const per_seq_rows& dk, const per_seq_rows& dv, const per_seq_states* dstate0, void* work, hipStream_t s) {
  const uint32_t share = a.H / a.G;
  const SeqRows Q = rows(q, a.dtype, 1), K = rows(k, a.dtype, share), V = rows(v, a.dtype, share), D = rows(dout, a.dtype, 1);
  float* fold = static_cast<float*>(work);
  AttentionPass p = make_pass(a, false, a.dv, a.dk);
  p.x = D; p.y = V; p.z = K;
  p.out = rows(dq, a.dtype, 1);
  from_states(&p, state, a.dv, true);
  hipError_t e = run_pass<T, T>(a, p, s);
  for (int which = 0; which < 2 && e == hipSuccess; ++which) {
    const bool of_v = which == 1;   // (last: it may write over dstate)
    const uint32_t width = of_v ? a.dv : a.dk;
    p = make_pass(a, true, of_v ? a.dk : a.dv, width);
    p.x = of_v ? K : V;
    p.y = of_v ? Q : D;
    p.z = of_v ? D : Q;
    from_states(&p, dstate, a.dv, !of_v);
    if (of_v) to_states(&p, dstate0);
    const SeqRows to = rows(of_v ? dv : dk, a.dtype, 1);
    if (share == 1) {
      p.out = to;
      e = run_pass<T, T>(a, p, s);
      continue;
    }
    p.out = packed(fold, a, width);
    e = run_pass<T, float>(a, p, s);
    const uint64_t n = (uint64_t)a.B * a.L * a.G * width;
    if (e != hipSuccess || !n) continue;
    k_fold_heads<T><<<(uint32_t)((n + 255) / 256), 256, 0, s>>>(fold, to, a.L, a.G, share, width, n);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

size_t attention_work_bytes(const AttentionSizes& a, bool backward) {
  if (!backward || a.H == a.G) return 0;
  return align256((size_t)a.B * a.L * a.H * (a.dk > a.dv ? a.dk : a.dv) * sizeof(float));
}

hipError_t launch_attention(const AttentionSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                            const per_seq_states* state, const per_seq_rows& out, const per_seq_states* out_state, void* work,
                            hipStream_t s) {
  return a.dtype == PER_SEQ_BF16 ? forward<bf16>(a, q, k, v, state, out, out_state, work, s)
                                 : forward<float>(a, q, k, v, state, out, out_state, work, s);
}

hipError_t launch_attention_backward(const AttentionSizes& a, const per_seq_rows& dout, const per_seq_rows& q,
                                     const per_seq_rows& k, const per_seq_rows& v, const per_seq_states* state,
                                     const per_seq_states* dstate, const per_seq_rows& dq, const per_seq_rows& dk,
                                     const per_seq_rows& dv, const per_seq_states* dstate0, void* work, hipStream_t s) {
  return a.dtype == PER_SEQ_BF16 ? backward<bf16>(a, dout, q, k, v, state, dstate, dq, dk, dv, dstate0, work, s)
                                 : backward<float>(a, dout, q, k, v, state, dstate, dq, dk, dv, dstate0, work, s);
}

hipError_t launch_attention_step(const AttentionSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                                 const per_seq_states& state, const per_seq_rows& out, hipStream_t s) {
  const uint32_t share = a.H / a.G;
  const SeqRows Q = rows(q, a.dtype, 1), K = rows(k, a.dtype, share), V = rows(v, a.dtype, share), O = rows(out, a.dtype, 1);
  const SeqStates st{state.d, state.batch, state.head};
  if (a.dtype == PER_SEQ_BF16)
    k_attend_step<bf16><<<a.B * a.H, 128, 0, s>>>(Q, K, V, st, O, a.H, a.dk, a.dv, a.scale, a.log_decay, a.lengths);
  else
    k_attend_step<float><<<a.B * a.H, 128, 0, s>>>(Q, K, V, st, O, a.H, a.dk, a.dv, a.scale, a.log_decay, a.lengths);
  return hipGetLastError();
}

}  // namespace per
