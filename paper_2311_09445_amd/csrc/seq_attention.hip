// Linear attention with a decay for each head.
//
// Every direction is the same pass.  With rows x, y, z of a head taken in order i = 0, 1, ...
//   out[i] = c_in  sum over j <= i of decay^(i-j) (x[i].y[j]) z[j]  +  c_out decay^(i+1-lag) x[i]^T S
//   S      = decay^n S + c_state sum over j of decay^(n-1-j+lag) y[j] z[j]^T
//     out          : x, y, z = q, k, v;     S the state;                          lag 0
//     gradient of q:           dout, v, k;  S the state, transposed;              lag 0
//     gradient of v:           k, q, dout;  S the state's gradient; against time, lag 1
//     gradient of k:           v, dout, q;  the same, transposed;   against time, lag 1
#include "dev_tiles.h"
#include "seq_launch.h"

namespace per {

namespace {

struct AttentionPass {
  SeqRows x, y, z, out;
  uint32_t L, H, dx, dz;
  uint32_t back;                 // against time (and lag 1)
  uint32_t out_f32;              // out is fp32 whatever the rows' type
  uint32_t summed;               // out is the sum over a workgroup's heads
  uint32_t exact;                // the state itself is an output (of this pass or behind it)
  float c_in, c_state, c_out;
  const float* log_decay;
  const int32_t* lengths;
  // states [b][h] (and [segment]), element (i of dx, j of dz) at i * in_x + j * in_z
  const float* in;
  int64_t in_batch, in_head, in_segment;
  uint32_t in_x, in_z;
  float* to;
  int64_t to_batch, to_head;
  float* part;                   // [b][h][segment][dx][dz]: what each segment brings
};
struct AttentionPasses {
  AttentionPass pass[3];
  uint32_t count, teams, items, slices, segments, run, segment;   // items: workgroups of a pass; run: segments taken; segment: tokens
};

struct JoinPass {
  float* part;
  const float* in;
  int64_t in_batch, in_head;
  uint32_t dx, dz;
};
struct JoinPasses {
  JoinPass pass[2];
  uint32_t BH, H, L, segments, segment;
  const float* log_decay;
  const int32_t* lengths;
};

#include "k_attend.h"

// Rows of heads that share one, added up in the heads' order: from [B][L][H][d] in fp32 to [B][L][G][d].
struct Fold {
  const float* from;
  SeqRows to;
  uint32_t d;
};
struct Folds {
  Fold fold[2];
  uint32_t L, G, share;
  uint64_t rows;   // B L G
};
// VEC elements to a lane.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void k_fold_heads(Folds all) {
  typedef float Vec __attribute__((ext_vector_type(VEC)));
  typedef T Out __attribute__((ext_vector_type(VEC)));
  const Fold& f = all.fold[blockIdx.y];
  const uint32_t lanes = (f.d + VEC - 1) / VEC, per = 256 / lanes, lane = threadIdx.x % lanes;
  if (threadIdx.x / lanes >= per) return;
  for (uint64_t row = (uint64_t)blockIdx.x * per + threadIdx.x / lanes; row < all.rows; row += (uint64_t)gridDim.x * per) {
    const uint32_t g = (uint32_t)(row % all.G);
    const uint64_t tok = row / all.G;
    const float* from = f.from + row * all.share * f.d + lane * VEC;
    Vec sum = Vec(0.0f);
    for (uint32_t m = 0; m < all.share; ++m) sum += *reinterpret_cast<const Vec*>(from + (size_t)m * f.d);
    Out o;
#pragma unroll
    for (int i = 0; i < VEC; ++i) o[i] = (T)sum[i];
    *reinterpret_cast<Out*>(row_to<T>(f.to, (uint32_t)(tok / all.L), (uint32_t)(tok % all.L), g) + lane * VEC) = o;
  }
}

struct AttentionStep {
  SeqRows q, k, v, out;
  SeqStates state;
  uint32_t H, dk, dv, groups;
  float scale;
  const float* log_decay;
  const int32_t* active;
};

#include "k_attend_step.h"

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

// Rows in fp32 of the heads of workgroups, where several of these share one.
size_t fold_bytes(const AttentionSizes& a, uint32_t teams, uint32_t width) {
  const uint32_t from = a.H / teams;
  return from == a.G ? 0 : align256((size_t)a.B * a.L * from * width * sizeof(float));
}

// How a sequence is cut.  A workgroup takes its tokens one chunk behind the other, so what cuts the time of few sequences is
// workgroups: the sequence in segments, each from the state that those before it bring.  That costs another pass over keys and values
// for those states (the last segment's is not needed), a state in memory per segment, and two launches.  A gradient of unlike
// widths is two launches, or one as wide as the widest.  The fewest microseconds by these measured figures are taken:
//   a chunk of 64 x 64 takes 0.85 (fp32: 1.9), of 128 x 64 1.2 (2.8), of 128 x 128 1.9; two workgroups on a compute unit 1.45 times
//   that, more take turns; the pass for the states 0.55 of that for outputs (0.42 where it serves a gradient's); states move at 4 TB/s.
// Heads that share a key and value bring gradients of their own, in fp32, which are added up behind; in bfloat16, up to 64 wide, a
// gradient's workgroup may take two or four of them, a team of waves each, and add up in LDS.  That spares most of this memory, but
// keeps a compute unit busy longer: a chunk takes 1.6 with two teams (2.4 for two workgroups on a compute unit, 1.2 for each of more)
// and 2.6 with four (each; 3.1 where none waits for another, since then sequences of unlike lengths do not even out), and their starts
// are one and two chunks longer.  The memory moves at 8 TB/s up to 128 MB, at 4 above.
// Measured, teams of 1, 2, 4 (64 x 64, 8 heads): that share 2, 32 x 512 tokens 50, 52, 49 us, 64 x 512 102, 82, 91, 256 x 512 445, 315,
// 278, 48 x 80 26, 30, 33; that share 4 64 x 512 110, 67, 16 x 80 16, 13, 8 x 512 27, 33.
// Measured, whole against cut: 64 rows of 1024 tokens (64 x 64) 33 us and 26 in four; 4 rows of 1024 32 and 17 in sixteen; 4 rows of
// 512 18 and 16; the gradient of 64 rows of 1024 33 and 37 in four; of 32 rows of 16384 (128 x 128) 429 in 5, 456 in 8, 462 in 10.
struct Cut {
  uint32_t segments, segment;
  bool one;   // a gradient's passes in one launch
  uint32_t teams;
};
uint32_t kernel_width(uint32_t d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }
// Half of the columns to a workgroup: see launch_dz.
bool halved(uint32_t dtype, uint32_t dz, uint64_t workgroups) { return dz > 64 && (dtype == PER_SEQ_F32 || workgroups <= 256); }
float launch_us(uint32_t dtype, uint64_t workgroups, uint32_t dx, uint32_t dz, uint32_t chunks, uint32_t teams = 1) {
  if (teams > 1) {
    const float area = (float)(dx * dz) / 4096.0f, each = (float)((workgroups / teams + 255) / 256);
    return teams == 2 ? (0.8f + 0.8f * area) * (float)(chunks + 1) * (each <= 1 ? 1.0f : each <= 2 ? 1.5f : 0.75f * each)
                      : (0.7f + 1.9f * area) * (float)(chunks + 2) * (each <= 1 ? 1.2f : each);
  }
  const bool half = halved(dtype, dz, workgroups);
  const float area = (float)(dx * (half ? dz / 2 : dz)) / 4096.0f, each = (float)((workgroups * (half ? 2 : 1) + 255) / 256);
  return (dtype == PER_SEQ_F32 ? 0.97f + 0.93f * area : 0.5f + 0.35f * area) * (float)chunks * (each <= 1 ? 1.0f : each <= 2 ? 1.45f : 0.25f + 0.8f * each);
}
Cut cut(const AttentionSizes& a, bool backward) {
  const uint64_t rows = (uint64_t)a.B * a.H;
  const uint32_t wk = kernel_width(a.dk), wv = kernel_width(a.dv), widest = wk > wv ? wk : wv, most = a.L / 64 < 64 ? a.L / 64 : 64;
  const uint32_t share = a.G ? a.H / a.G : 1;
  const uint32_t teams = !backward || a.dtype != PER_SEQ_BF16 || widest > 64 ? 1 : share % 4 == 0 ? 4 : share % 2 == 0 ? 2 : 1;
  float best = 0.0f;
  Cut c{1, a.L ? a.L : 1, true, 1};
  for (uint32_t s = 1; rows && a.L && (s == 1 || s <= most); ++s) {
    const uint64_t n = rows * s;
    const uint32_t segment = ((a.L + s - 1) / s + kChunk - 1) / kChunk * kChunk, chunks = segment / kChunk;
    for (uint32_t t = 1; t <= teams; t *= 2) {
      bool one = true;
      float us = backward ? launch_us(a.dtype, 3 * n, widest, widest, chunks, t) : launch_us(a.dtype, n, wk, wv, chunks);
      if (backward && wk != wv) {
        const float apart = launch_us(a.dtype, 2 * n, wv, wk, chunks, t) + launch_us(a.dtype, n, wk, wv, chunks, t) + 3.0f;
        one = us <= apart;
        if (!one) us = apart;
      }
      if (s > 1)
        us += (backward ? 0.42f : 0.55f) * launch_us(a.dtype, (backward ? 2 : 1) * (n - rows), wk, wv, chunks) + 10.0f +
              4.0f * a.dk * a.dv * (float)(n * (backward ? 8 : 4)) / 4e6f;
      if (backward && share > t) {
        const float bytes = (float)(fold_bytes(a, t, a.dk) + fold_bytes(a, t, a.dv));
        us += 4.0f + bytes / (bytes <= 128e6f ? 8e6f : 4e6f);
      }
      if ((s == 1 && t == 1) || us < best) {
        best = us;
        c = s == 1 ? Cut{1, a.L, one, t} : Cut{(a.L + segment - 1) / segment, segment, one, t};
      }
    }
  }
  return c;
}
size_t part_bytes(const AttentionSizes& a, const Cut& c) {
  return c.segments < 2 ? 0 : align256((size_t)a.B * a.H * c.segments * a.dk * a.dv * sizeof(float));
}

template <typename T, int DX, int NT, int WAVES, bool OUT, Way WAY, int TEAMS = 1>
hipError_t launch_as(const AttentionPasses& p, hipStream_t s) {
  constexpr uint32_t lds = lds_bytes<T, DX, NT, WAVES, OUT, WAY, TEAMS>();
  auto* kernel = k_attend<T, DX, NT, WAVES, OUT, WAY, TEAMS>;
  static std::atomic<uint64_t> granted{0};
  const hipError_t e = grant_lds(reinterpret_cast<const void*>(kernel), &granted, lds);
  if (e != hipSuccess) return e;
  kernel<<<(p.items + 7) / 8 * 8 * p.count, dim3(64 * WAVES, TEAMS), lds, s>>>(p);
  return hipGetLastError();
}
// In bfloat16 straight into LDS where rows are made up of pieces of 16 bytes; through registers in pieces where they hold one.
template <typename T, int DX, int NT, int WAVES, bool OUT>
hipError_t launch_way(const AttentionPasses& p, hipStream_t s) {
  constexpr uint32_t W = 16 / sizeof(T);
  bool direct = sizeof(T) == 2, pieces = true;
  for (uint32_t i = 0; i < p.count; ++i) {
    const AttentionPass& a = p.pass[i];
    direct = direct && (!OUT || (a.x.wide && a.out.wide)) && a.y.wide && a.z.wide && a.dx % W == 0 && a.dz % W == 0;
    pieces = pieces && (!OUT || a.out.near) && a.dx >= W && a.dz >= W;
  }
  if constexpr (sizeof(T) == 2) {
    if (direct) return launch_as<T, DX, NT, WAVES, OUT, DIRECT>(p, s);
  }
  return pieces ? launch_as<T, DX, NT, WAVES, OUT, PIECES>(p, s) : launch_as<T, DX, NT, WAVES, OUT, ELEMENTS>(p, s);
}
// Teams of two waves: more columns to a wave, so that the waves read less LDS (of four waves each, 64 x 64, 128 x 512 tokens with 8
// heads that share 2: 166 us, of two 142).
template <int DX, int NT>
hipError_t launch_teams(const AttentionPasses& p, hipStream_t s) {
  bool pieces = true;
  for (uint32_t i = 0; i < p.count; ++i) pieces = pieces && p.pass[i].out.near && p.pass[i].dx >= 8 && p.pass[i].dz >= 8;
  if (p.teams == 4) return pieces ? launch_as<bf16, DX, NT, 2, true, PIECES, 4>(p, s) : launch_as<bf16, DX, NT, 2, true, ELEMENTS, 4>(p, s);
  return pieces ? launch_as<bf16, DX, NT, 2, true, PIECES, 2>(p, s) : launch_as<bf16, DX, NT, 2, true, ELEMENTS, 2>(p, s);
}
template <typename T, int DX, bool OUT>
hipError_t launch_dz(AttentionPasses& p, uint32_t rows, hipStream_t s) {
  uint32_t dz = 0;
  for (uint32_t i = 0; i < p.count; ++i) dz = dz < p.pass[i].dz ? p.pass[i].dz : dz;
  p.slices = 1;
  p.items = rows / p.teams * p.run;
  if constexpr (sizeof(T) == 2 && DX <= 64 && OUT) {
    if (p.teams > 1) return dz <= 32 ? launch_teams<DX, 1>(p, s) : launch_teams<DX, 2>(p, s);
  }
  if (dz <= 32) return launch_way<T, DX, 1, 2, OUT>(p, s);
  if (dz <= 64) return launch_way<T, DX, 1, 4, OUT>(p, s);
  // Wider states: two tiles of columns to a wave, or half of the columns to a workgroup where there are few (each then reads x and y:
  // 16 rows of 1024 tokens of 128 x 128 61 us and 44, 128 rows of 512 37 and 29, but 16 of 65536 in 32 segments 371 and 434) and in
  // fp32, where two tiles do not fit the registers (16 rows of 1024 333 us and 170).
  if (halved(sizeof(T) == 4 ? PER_SEQ_F32 : PER_SEQ_BF16, dz, (uint64_t)p.items * p.count)) {
    p.slices = 2;
    p.items *= 2;
    return launch_way<T, DX, 1, 4, OUT>(p, s);
  }
  if constexpr (sizeof(T) == 2) return launch_way<T, DX, 2, 4, OUT>(p, s);
  return hipErrorInvalidValue;
}
// Passes in one launch, as wide as the widest.
template <typename T, bool OUT>
hipError_t launch_passes(AttentionPasses p, uint32_t rows, hipStream_t s) {
  uint32_t dx = 0;
  for (uint32_t i = 0; i < p.count; ++i) dx = dx < p.pass[i].dx ? p.pass[i].dx : dx;
  if (dx <= 32) return launch_dz<T, 32, OUT>(p, rows, s);
  if (dx <= 64) return launch_dz<T, 64, OUT>(p, rows, s);
  return launch_dz<T, 128, OUT>(p, rows, s);
}

void join_from(JoinPass* j, const per_seq_states* s) {
  if (s) { j->in = s->d; j->in_batch = s->batch; j->in_head = s->head; }
}
// A pass whose segments start from the joined states.
void from_parts(AttentionPass* p, float* part, const AttentionSizes& a, const Cut& c, bool transposed) {
  const int64_t per = (int64_t)a.dk * a.dv;
  p->in = part;
  p->in_segment = per;
  p->in_head = per * c.segments;
  p->in_batch = p->in_head * a.H;
  p->in_x = transposed ? 1 : a.dv;
  p->in_z = transposed ? a.dv : 1;
}
hipError_t launch_join(JoinPasses j, const AttentionSizes& a, const Cut& c, uint32_t count, hipStream_t s) {
  j.BH = a.B * a.H;
  j.H = a.H;
  j.L = a.L;
  j.segments = c.segments;
  j.segment = c.segment;
  j.log_decay = a.log_decay;
  j.lengths = a.lengths;
  const uint64_t n = (uint64_t)j.BH * a.dk * a.dv;
  k_join<<<dim3((uint32_t)((n + 255) / 256), count), 256, 0, s>>>(j);
  return hipGetLastError();
}

template <typename T>
hipError_t forward(const AttentionSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                   const per_seq_states* state, const per_seq_rows& out, const per_seq_states* out_state, void* work, hipStream_t s) {
  const uint32_t share = a.H / a.G, bh = a.B * a.H;
  const Cut c = cut(a, false);
  AttentionPasses all{};
  all.count = all.teams = 1;
  all.segments = c.segments;
  all.segment = c.segment;
  AttentionPass& p = all.pass[0];
  p = make_pass(a, false, a.dk, a.dv);
  p.x = rows(q, a.dtype, 1);
  p.y = rows(k, a.dtype, share);
  p.z = rows(v, a.dtype, share);
  p.out = rows(out, a.dtype, 1);
  to_states(&p, out_state);
  p.exact = out_state != nullptr;
  if (c.segments == 1) {
    all.run = 1;
    from_states(&p, state, a.dv, false);
    return launch_passes<T, true>(all, bh, s);
  }
  float* const part = static_cast<float*>(work);
  all.run = c.segments - 1;
  p.part = part;
  hipError_t e = launch_passes<T, false>(all, bh, s);
  if (e != hipSuccess) return e;
  all.run = c.segments;
  JoinPasses j{};
  j.pass[0] = JoinPass{part, nullptr, 0, 0, a.dk, a.dv};
  join_from(&j.pass[0], state);
  e = launch_join(j, a, c, 1, s);
  if (e != hipSuccess) return e;
  from_parts(&p, part, a, c, false);
  return launch_passes<T, true>(all, bh, s);
}

template <typename T>
hipError_t launch_fold(const Folds& f, hipStream_t s) {
  if (!f.rows) return hipSuccess;
  const uint32_t dk = f.fold[0].d, dv = f.fold[1].d;
  const bool wide = dk % 4 == 0 && dv % 4 == 0 && f.fold[0].to.wide && f.fold[1].to.wide;
  const uint32_t widest = dk > dv ? dk : dv, per = 256 / (wide ? (widest + 3) / 4 : widest);   // rows of a workgroup
  const uint64_t blocks = (f.rows + per - 1) / per;
  const dim3 grid((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20), 2);
  if (wide) k_fold_heads<T, 4><<<grid, 256, 0, s>>>(f);
  else k_fold_heads<T, 1><<<grid, 256, 0, s>>>(f);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const AttentionSizes& a, const per_seq_rows& dout, const per_seq_rows& q, const per_seq_rows& k,
                    const per_seq_rows& v, const per_seq_states* state, const per_seq_states* dstate, const per_seq_rows& dq,
                    const per_seq_rows& dk, const per_seq_rows& dv, const per_seq_states* dstate0, void* work, hipStream_t s) {
  Folds f{};
  f.fold[0] = Fold{nullptr, rows(dk, a.dtype, 1), a.dk};
  f.fold[1] = Fold{nullptr, rows(dv, a.dtype, 1), a.dv};
  f.L = a.L;
  f.G = a.G;
  f.rows = (uint64_t)a.B * a.L * a.G;
  if (!a.H) return launch_fold<T>(f, s);   // (sums over no heads)
  const uint32_t share = a.H / a.G, bh = a.B * a.H;
  const Cut c = cut(a, true);
  const uint32_t team = c.teams, left = share / team;   // left: to be added up behind
  const SeqRows Q = rows(q, a.dtype, 1), K = rows(k, a.dtype, share), V = rows(v, a.dtype, share), D = rows(dout, a.dtype, 1);
  uint8_t* at = static_cast<uint8_t*>(work);
  float* part[2];   // of the states, of their gradients
  for (int i = 0; i < 2; ++i, at += part_bytes(a, c)) part[i] = reinterpret_cast<float*>(at);
  float* const fold_k = reinterpret_cast<float*>(at);
  float* const fold_v = reinterpret_cast<float*>(at + fold_bytes(a, team, a.dk));

  AttentionPass of_q = make_pass(a, false, a.dv, a.dk), of_k = make_pass(a, true, a.dv, a.dk), of_v = make_pass(a, true, a.dk, a.dv);
  of_q.x = D; of_q.y = V; of_q.z = K;
  of_k.x = V; of_k.y = D; of_k.z = Q;
  of_v.x = K; of_v.y = Q; of_v.z = D;
  of_q.out = rows(dq, a.dtype, 1);
  of_k.out = left == 1 ? rows(dk, a.dtype, team) : packed(fold_k, a.L, a.H / team, a.dk, team);
  of_v.out = left == 1 ? rows(dv, a.dtype, team) : packed(fold_v, a.L, a.H / team, a.dv, team);
  of_k.out_f32 = of_v.out_f32 = left > 1;
  of_k.summed = of_v.summed = team > 1;
  AttentionPasses all{};
  all.segments = c.segments;
  all.segment = c.segment;
  to_states(&of_v, dstate0);
  of_v.exact = dstate0 != nullptr;
  hipError_t e;
  if (c.segments == 1) {
    from_states(&of_q, state, a.dv, true);
    from_states(&of_k, dstate, a.dv, true);
    from_states(&of_v, dstate, a.dv, false);
  } else {
    all.run = c.segments - 1;
    all.teams = 1;
    all.count = 2;
    all.pass[0] = make_pass(a, false, a.dk, a.dv);
    all.pass[0].y = K;
    all.pass[0].z = V;
    all.pass[1] = of_v;
    for (int i = 0; i < 2; ++i) all.pass[i].part = part[i];
    e = launch_passes<T, false>(all, bh, s);
    if (e != hipSuccess) return e;
    JoinPasses j{};
    for (int i = 0; i < 2; ++i) j.pass[i] = JoinPass{part[i], nullptr, 0, 0, a.dk, a.dv};
    join_from(&j.pass[0], state);
    join_from(&j.pass[1], dstate);
    e = launch_join(j, a, c, 2, s);
    if (e != hipSuccess) return e;
    from_parts(&of_q, part[0], a, c, true);
    from_parts(&of_k, part[1], a, c, true);
    from_parts(&of_v, part[1], a, c, false);
  }
  all.run = c.segments;
  all.teams = team;
  // All three in one launch, if that is best; but the gradient of k reads dstate, which that of v may write over.
  all.pass[0] = of_q;
  all.pass[1] = of_k;
  all.pass[2] = of_v;
  const bool over = c.segments == 1 && dstate && dstate0 && dstate->d == dstate0->d;
  all.count = c.one && !over ? 3 : 2;
  e = launch_passes<T, true>(all, bh, s);
  if (e == hipSuccess && all.count == 2) {
    all.count = 1;
    all.pass[0] = of_v;
    e = launch_passes<T, true>(all, bh, s);
  }
  if (e != hipSuccess || left == 1) return e;
  f.fold[0].from = fold_k;
  f.fold[1].from = fold_v;
  f.share = left;
  return launch_fold<T>(f, s);
}

}  // namespace

size_t attention_work_bytes(const AttentionSizes& a, bool backward) {
  const Cut c = cut(a, backward);
  if (!backward) return part_bytes(a, c);
  const size_t need = 2 * part_bytes(a, c) + fold_bytes(a, c.teams, a.dk) + fold_bytes(a, c.teams, a.dv);
  // (a gradient of shared heads always has a workspace: what a caller passes does not depend on who adds up)
  return need || !a.H || a.H == a.G || !a.B || !a.L ? need : 256;
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

template <typename T, int VEC, int R>
static hipError_t step(const AttentionStep& p, uint32_t rows, hipStream_t s) {
  const Past way = past((uint64_t)rows * p.dk * p.dv * 4);
  if (way == KEPT) k_attend_step<T, VEC, R, KEPT><<<rows, 256, 0, s>>>(p);
  else if (way == STORES_PAST) k_attend_step<T, VEC, R, STORES_PAST><<<rows, 256, 0, s>>>(p);
  else k_attend_step<T, VEC, R, ALL_PAST><<<rows, 256, 0, s>>>(p);
  return hipGetLastError();
}
template <typename T>
static hipError_t step(AttentionStep p, uint32_t rows, hipStream_t s) {
  const bool wide = p.dv % 4 == 0 && (reinterpret_cast<uintptr_t>(p.state.d) & 15) == 0 && p.state.batch % 4 == 0 && p.state.head % 4 == 0;
  const uint32_t columns = wide ? p.dv / 4 : p.dv;
  p.groups = 256 / columns < p.dk ? 256 / columns : p.dk;
  const bool few = (p.dk + p.groups - 1) / p.groups <= 4;   // rows of a thread
  return !wide ? step<T, 1, 16>(p, rows, s) : few ? step<T, 4, 4>(p, rows, s) : step<T, 4, 16>(p, rows, s);
}

hipError_t launch_attention_step(const AttentionSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                                 const per_seq_states& state, const per_seq_rows& out, hipStream_t s) {
  const uint32_t share = a.H / a.G;
  const AttentionStep p{rows(q, a.dtype, 1), rows(k, a.dtype, share), rows(v, a.dtype, share), rows(out, a.dtype, 1),
                        SeqStates{state.d, state.batch, state.head}, a.H, a.dk, a.dv, 0, a.scale, a.log_decay, a.lengths};
  return a.dtype == PER_SEQ_BF16 ? step<bf16>(p, a.B * a.H, s) : step<float>(p, a.B * a.H, s);
}

}  // namespace per
