// One token of linear attention: the state is read, decayed, added to and written, and the query's product with it formed on the
// way.  Part of seq_attention.hip (included inside namespace per).
//
// Nothing but the state's bytes counts (8 dk dv per head, against 4 dk dv operations).  A workgroup takes the state of one head: VEC
// columns to a thread, `groups` threads of rows side by side, R rows of each in flight.  The rows of query and key are put into LDS
// meanwhile; the parts of the product are added up over the groups in their order.  1 GiB of states (1024 sequences of 16 heads of
// 128 x 128) takes 415 us, 5.2 TB/s, as fast as a copy.
// What is left of a state is formed as over the chunks of a sequence (keeps, kept): with the rounded power itself an actor's state
// would be off by the same 2^-25 at every one of thousands of tokens.
//
// PAST: states that do not fit the last cache (256 MB) would only push each other out of it: the stores go past it, of more than
// three times as much the loads too.  Us by size, kept / stores past / both: 128 MB 40 / 43 / 49, 256 MB 82 / 81 / 100, 512 MB
// 219 / 171 / 205, 1 GB 434 / 433 / 415.
enum Past { KEPT, STORES_PAST, ALL_PAST };

template <typename T, int VEC, int R, Past PAST>
__global__ __launch_bounds__(256) void k_attend_step(AttentionStep p) {
  typedef float Vec __attribute__((ext_vector_type(VEC)));
  __shared__ float qs[128], ks[128];
  __shared__ __attribute__((aligned(16))) float parts[256 * VEC];
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
  auto fetch = [&](uint32_t row0) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint32_t row = row0 + r * p.groups;
      if (!on || row >= p.dk) continue;
      const Vec* from = reinterpret_cast<const Vec*>(S + (size_t)row * p.dv);
      s[r] = PAST == ALL_PAST ? __builtin_nontemporal_load(from) : *from;
    }
  };
  fetch(group);
  if (tid < p.dk) {
    qs[tid] = as_float(row_of<T>(p.q, b, 0, h)[tid]);
    ks[tid] = as_float(row_of<T>(p.k, b, 0, h)[tid]);
  }
  Vec v = Vec(0.0f), sum = Vec(0.0f);
  if (on) {
    const T* vr = row_of<T>(p.v, b, 0, h) + col;
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = as_float(vr[i]);
  }
  const Keep keep = keeps(p.log_decay[h]);
  __syncthreads();
  for (uint32_t row0 = group; row0 < p.dk; row0 += R * p.groups) {
    if (row0 != group) fetch(row0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint32_t row = row0 + r * p.groups;
      if (on && row < p.dk) {
        const float k = ks[row], q = qs[row];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          s[r][i] = fmaf(k, v[i], kept(s[r][i], keep));
          sum[i] = fmaf(q, s[r][i], sum[i]);
        }
        Vec* to = reinterpret_cast<Vec*>(S + (size_t)row * p.dv);
        if (PAST != KEPT) __builtin_nontemporal_store(s[r], to);
        else *to = s[r];
      }
    }
  }
  if (on) *reinterpret_cast<Vec*>(parts + group * columns * VEC + col) = sum;
  __syncthreads();
  if (tid < p.dv) {
    float all = 0.0f;
    for (uint32_t i = 0; i < p.groups; ++i) all += parts[i * columns * VEC + tid];
    out[tid] = (T)(p.scale * all);
  }
}
