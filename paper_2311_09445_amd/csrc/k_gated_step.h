// One token of the gated delta rule.  Part of seq_delta.hip (included inside namespace per).
//
// With a = e^g: r = S^T k, w = S^T q, u = beta (v - a r), S <- a S + k u^T, out = scale (a w + (q.k) u).  Nothing but the state's bytes
// counts, so it is read once and held: a workgroup takes the state of one head, VEC columns to a thread, `groups` threads of rows side by
// side, R rows of each.  Both products with the state are formed while it comes in and added up over the groups in their order; what is
// written follows one barrier.  512 MiB of states (512 sequences of 16 heads of 128 x 128) take 219 us, 4.9 TB/s, as fast as a copy (171 where
// the last cache holds part of them from the call before); 64 sequences of 4 heads of 64 x 64 5.2, a launch.  How states pass the last cache: see k_attend_step.h.
struct DeltaStep {
  SeqRows q, k, v, out;
  Gates log_decay, beta;
  SeqStates state;
  uint32_t H, dk, dv, groups;
  float scale;
  const int32_t* active;
};

template <typename T, int VEC, int R, Past PAST>
__global__ __launch_bounds__(256) void k_delta_step(DeltaStep p) {
  typedef float Vec __attribute__((ext_vector_type(VEC)));
  __shared__ float qs[128], ks[128];
  __shared__ __attribute__((aligned(16))) float reads[256 * VEC], asks[256 * VEC];
  __shared__ float meets[2];
  const uint32_t h = blockIdx.x % p.H, b = blockIdx.x / p.H, tid = threadIdx.x;
  T* const out = row_to<T>(p.out, b, 0, h);
  if (p.active && p.active[b] < 1) {
    if (tid < p.dv) out[tid] = (T)0.0f;
    return;
  }
  const uint32_t columns = (p.dv + VEC - 1) / VEC, group = tid / columns, col = tid % columns * VEC;
  const bool on = group < p.groups;
  float* const S = p.state.d + (int64_t)b * p.state.batch + (int64_t)h * p.state.head + col;
  Vec s[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t row = group + r * p.groups;
    s[r] = Vec(0.0f);
    if (!on || row >= p.dk) continue;
    const Vec* from = reinterpret_cast<const Vec*>(S + (size_t)row * p.dv);
    s[r] = PAST == ALL_PAST ? __builtin_nontemporal_load(from) : *from;
  }
  float q = 0.0f, k = 0.0f;
  if (tid < p.dk) {
    q = as_float(row_of<T>(p.q, b, 0, h)[tid]);
    k = as_float(row_of<T>(p.k, b, 0, h)[tid]);
    qs[tid] = q;
    ks[tid] = k;
  }
  if (tid < 128) {
    float meet = sum16(q * k);
    meet += __shfl_xor(meet, 16);
    meet += __shfl_xor(meet, 32);
    if ((tid & 63) == 0) meets[tid >> 6] = meet;
  }
  Vec v = Vec(0.0f), read = Vec(0.0f), ask = Vec(0.0f);
  if (on) {
    const T* vr = row_of<T>(p.v, b, 0, h) + col;
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = as_float(vr[i]);
  }
  const float g = p.log_decay.at(b, 0, h), beta = p.beta.at(b, 0, h), a = expf(g);
  const Keep keep = keeps(g);
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t row = group + r * p.groups;
    if (!on || row >= p.dk) continue;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      read[i] = fmaf(ks[row], s[r][i], read[i]);
      ask[i] = fmaf(qs[row], s[r][i], ask[i]);
    }
  }
  if (on) {
    *reinterpret_cast<Vec*>(reads + group * columns * VEC + col) = read;
    *reinterpret_cast<Vec*>(asks + group * columns * VEC + col) = ask;
  }
  __syncthreads();
  if (!on) return;
  read = Vec(0.0f);
  for (uint32_t i = 0; i < p.groups; ++i) read += *reinterpret_cast<const Vec*>(reads + i * columns * VEC + col);
  const Vec u = beta * (v - a * read);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t row = group + r * p.groups;
    if (row >= p.dk) continue;
#pragma unroll
    for (int i = 0; i < VEC; ++i) s[r][i] = fmaf(ks[row], u[i], kept(s[r][i], keep));
    Vec* to = reinterpret_cast<Vec*>(S + (size_t)row * p.dv);
    if (PAST != KEPT) __builtin_nontemporal_store(s[r], to);
    else *to = s[r];
  }
  if (group == 0) {
    ask = Vec(0.0f);
    for (uint32_t i = 0; i < p.groups; ++i) ask += *reinterpret_cast<const Vec*>(asks + i * columns * VEC + col);
    const Vec o = p.scale * (a * ask + (meets[0] + meets[1]) * u);
#pragma unroll
    for (int i = 0; i < VEC; ++i) out[col + i] = (T)o[i];
  }
}
