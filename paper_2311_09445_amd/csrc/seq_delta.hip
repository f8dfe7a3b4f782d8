// The gated delta rule: a state that is decayed, corrected and read.
//
//   D = exp(g_t) S[t-1],  u_t = beta_t (v_t - D^T k_t),  S[t] = D + k_t u_t^T,  out_t = scale S[t]^T q_t.
//
// Sequences are taken in chunks of 32 tokens (k_gated_pairs.h: what a chunk's tokens make of each other, all chunks at once; k_gated_run.h: the
// states one chunk behind the other; k_gated_back.h: the gradient, against time and then all chunks at once), single tokens in k_gated_step.h.
#include <math.h>

#include "dev_parts.h"
#include "seq_launch.h"

namespace per {

namespace {

#include "k_gated_pairs.h"
#include "k_gated_run.h"
#include "k_gated_back.h"
#include "k_gated_step.h"

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
Gates gates(const per_seq_gates& g) { return Gates{g.d, g.batch, g.token, g.head}; }
uint32_t chunks_of(uint32_t L) { return (L + kChunk - 1) / kChunk; }
// (256 divides every chunk's part of a workspace, so that the parts stay aligned)
uint32_t padded(uint32_t dk) { return dk <= 64 ? 64 : 128; }

// How a sequence is cut: in segments of whole chunks, each from the state that those before it bring.  A workgroup takes its chunks one behind
// the other, so what cuts the time of few sequences is workgroups.  That costs another pass over all segments but the last, over dk
// columns more (what a segment makes of a state is a product, k_delta_join), and two launches (a gradient: as much again but for the
// product).  The fewest microseconds by these measured figures are taken, for widths up to 64 and above:
//   a chunk's outputs 1.8, 2.45 (fp32 3.4, 5.5), what it carries 1.1, 1.65 (2.6, 4.0), its gradient's two passes 5.2, 8.3 (9, 15), what that carries 1.8,
//   2.95 (4, 6); two workgroups on a compute unit take 1.75 times as long, more take turns; a gradient's, which move the states, take 1.4 times
//   as long where every compute unit has one, 2.5 with two; to join 3.2, 4.5 a segment.
// Measured, in 1, 4, 8, 16 segments, us: 65536 tokens of 16 heads of 128 x 128 5453, 2363, 1513, 1351; 2 x 8192 of them 690, 411, 380, 433, their gradient
// 2673, 1577, 1502, 1611; 4 x 4096 of 8 of 64 x 64 256, 136, 102, 110 and 836, 466, 370, 388; 32 x 512 of them, in 1 and 4, 58, 90 and 267, 368.
struct Cut { uint32_t segments, segment; };
Cut cut(const DeltaSizes& a, bool backward) {
  const uint32_t chunks = chunks_of(a.L), wide = a.dk > 64, f32 = a.dtype == PER_SEQ_F32, slices = (a.dv + 63) / 64, more = slices + (a.dk + 63) / 64;
  static const float forward_us[2][2] = {{1.8f, 2.45f}, {3.4f, 5.5f}}, carry_us[2][2] = {{1.1f, 1.65f}, {2.6f, 4.0f}};
  static const float back_us[2][2] = {{5.2f, 8.3f}, {9.0f, 15.0f}}, carry_back_us[2][2] = {{1.8f, 2.95f}, {4.0f, 6.0f}};
  const uint64_t rows = (uint64_t)a.B * a.H;
  // (in fp32 above 64 the rows of one workgroup fill a compute unit's LDS)
  auto crowd = [&](uint64_t workgroups) {
    const float w = (float)workgroups / 256.0f;
    return w <= 1.0f ? 1.0f : f32 && wide ? ceilf(w) : w <= 2.0f ? 1.75f : 0.15f + 0.8f * w;
  };
  auto crowd_back = [&](uint64_t workgroups) {
    const float w = (float)workgroups / 256.0f;
    return w <= 0.5f ? 1.0f : w <= 1.0f ? 1.4f : f32 && wide ? 1.4f * ceilf(w) : w <= 2.0f ? 2.5f : 1.25f * w;
  };
  const uint32_t most = chunks / 2 < 64 ? chunks / 2 : 64;
  float best = 0.0f;
  Cut c{1, chunks ? chunks : 1};
  for (uint32_t s = 1; rows && chunks && (s == 1 || s <= most); ++s) {
    const uint32_t segment = (chunks + s - 1) / s;
    float us = (float)segment * (backward ? back_us[f32][wide] * crowd_back(rows * s * slices) : forward_us[f32][wide] * crowd(rows * s * slices));
    if (s > 1) {
      us += (float)segment * carry_us[f32][wide] * crowd(rows * (backward ? s : s - 1) * more) + 12.0f + (wide ? 4.5f : 3.2f) * (float)s * crowd(rows * slices);
      if (backward) us += (float)segment * carry_back_us[f32][wide] * crowd(rows * (s - 1) * slices) + 12.0f + (wide ? 4.5f : 3.2f) * (float)s * crowd(rows * slices);
    }
    if (s == 1 || us < best) {
      best = us;
      c = Cut{(chunks + segment - 1) / segment, segment};
    }
  }
  return c;
}
uint32_t carried_floats(const DeltaSizes& a, bool turned) { return a.dk * (a.dk * (turned ? 2 : 1) + a.dv); }   // of a segment
size_t carried_bytes(const DeltaSizes& a, const Cut& c, bool turned) {
  return c.segments < 2 ? 0 : align256((size_t)a.B * a.H * c.segments * carried_floats(a, turned) * sizeof(float));
}

size_t record_bytes(const DeltaSizes& a) { return (size_t)a.B * a.H * chunks_of(a.L) * sizeof(DeltaRecord); }

// Where a gradient's intermediate results lie in the workspace.
struct BackWork {
  size_t records, states, dstates, y, x, dz, read, along, strength, write, stay, past, fold_q, fold_k, carried, carried_back, bytes;
};
BackWork back_work(const DeltaSizes& a) {
  const uint64_t bh = (uint64_t)a.B * a.H, chunks = bh * chunks_of(a.L), tokens = chunks * kChunk;
  const uint64_t blocks = (a.dv + 31) / 32, parts = blocks * 2;
  const bool f32 = a.dtype == PER_SEQ_F32;
  BackWork w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  const uint64_t state = blocks * 32 * padded(a.dk) * sizeof(bf16);
  w.records = take(chunks * sizeof(DeltaRecordBack));
  w.states = take(chunks * state * (f32 ? kStateParts<float> : kStateParts<bf16>));
  w.dstates = take(chunks * state * (f32 ? kGradParts<float> : kGradParts<bf16>));
  w.y = take(tokens * blocks * 32 * sizeof(float));
  w.x = take(tokens * blocks * 32 * sizeof(float));
  w.dz = take(tokens * blocks * 32 * sizeof(float));
  w.read = take(tokens * parts * sizeof(float));
  w.along = take(tokens * parts * sizeof(float));
  w.strength = take(tokens * parts * sizeof(float));
  w.write = take(tokens * parts * sizeof(float));
  w.stay = take(tokens * parts * sizeof(float));
  w.past = take(tokens * sizeof(float));
  w.fold_q = take(a.Q == a.H ? 0 : tokens * a.dk * sizeof(float));
  w.fold_k = take(a.K == a.H ? 0 : tokens * a.dk * sizeof(float));
  const Cut c = cut(a, true);
  w.carried = take(carried_bytes(a, c, true));
  w.carried_back = take(c.segments < 2 ? 0 : bh * c.segments * a.dk * a.dv * sizeof(float));
  w.bytes = at;
  return w;
}

template <typename Args>
hipError_t launch(void (*kernel)(Args), std::atomic<uint64_t>* granted, uint32_t grid, uint32_t lds, const Args& args, hipStream_t s) {
  const hipError_t e = grant_lds(reinterpret_cast<const void*>(kernel), granted, lds);
  if (e != hipSuccess) return e;
  kernel<<<grid, 256, lds, s>>>(args);
  return hipGetLastError();
}
// In bfloat16 straight into LDS where rows are made up of pieces of 16 bytes.
template <typename T, int DK, DeltaMode MODE, bool OWN = false>
hipError_t launch_run(const DeltaRun& p, uint32_t bh, hipStream_t s) {
  static std::atomic<uint64_t> granted[2] = {};
  constexpr int NP = kPairParts<T, MODE>;
  const uint32_t grid = bh * p.run * (p.slices + (MODE == CARRYING ? (p.dk + 63) / 64 : 0));
  auto lds = [](uint32_t bytes) { return OWN && bytes < 4 * sizeof(PairLds) ? (uint32_t)(4 * sizeof(PairLds)) : bytes; };
  if constexpr (sizeof(T) == 2) {
    if (p.q.wide && p.k.wide && p.v.wide && p.dk % 8 == 0 && p.dv % 8 == 0)
      return launch(k_delta_run<T, DK, MODE, true, OWN>, &granted[1], grid, lds(RunLds<T, DK, NP, true, MODE>::BYTES), p, s);
  }
  return launch(k_delta_run<T, DK, MODE, false, OWN>, &granted[0], grid, lds(RunLds<T, DK, NP, false, MODE>::BYTES), p, s);
}
template <typename T, int DK, bool CARRY>
hipError_t launch_back(const DeltaBack& p, uint32_t bh, hipStream_t s) {
  static std::atomic<uint64_t> granted[2] = {};
  const uint32_t grid = bh * p.run * p.slices;
  if constexpr (sizeof(T) == 2) {
    if (p.q.wide && p.k.wide && p.dout.wide && p.dk % 8 == 0 && p.dv % 8 == 0)
      return launch(k_delta_back<T, DK, CARRY, true>, &granted[1], grid, BackLds<T, DK, true>::BYTES, p, s);
  }
  return launch(k_delta_back<T, DK, CARRY, false>, &granted[0], grid, BackLds<T, DK, false>::BYTES, p, s);
}
template <typename T, int DK>
hipError_t launch_grads(const DeltaGrads& p, uint32_t bh, hipStream_t s) {
  static std::atomic<uint64_t> granted{0};
  return launch(k_delta_grads<T, DK>, &granted, bh * p.chunks, grads_lds<T, DK>(), p, s);
}
DeltaPairs make_pairs(const DeltaSizes& a, const per_seq_rows& q, const per_seq_rows& k, void* records) {
  return DeltaPairs{rows(q, a.dtype, a.H / a.Q), rows(k, a.dtype, a.H / a.K), gates(a.log_decay), gates(a.beta), a.lengths, records,
                    a.L, a.H, a.dk, chunks_of(a.L), a.B * a.H * chunks_of(a.L), a.scale};
}
template <typename T, int DK, bool BACK>
hipError_t launch_pairs(const DeltaSizes& a, const per_seq_rows& q, const per_seq_rows& k, void* records, hipStream_t s) {
  const DeltaPairs p = make_pairs(a, q, k, records);
  if (!p.items) return hipSuccess;
  if (p.q.wide && p.k.wide && p.dk % (16 / sizeof(T)) == 0) k_delta_pairs<T, DK, BACK, true><<<(p.items + 3) / 4, 256, 0, s>>>(p);
  else k_delta_pairs<T, DK, BACK, false><<<(p.items + 3) / 4, 256, 0, s>>>(p);
  return hipGetLastError();
}

DeltaRun make_run(const DeltaSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v, const per_seq_states* state, const void* records,
                  size_t record) {
  DeltaRun p{};
  p.q = rows(q, a.dtype, a.H / a.Q);
  p.k = rows(k, a.dtype, a.H / a.K);
  p.v = rows(v, a.dtype, a.H / a.V);
  p.records = records;
  p.record_bytes = (uint32_t)record;
  p.lengths = a.lengths;
  if (state) { p.in = state->d; p.in_batch = state->batch; p.in_head = state->head; }
  p.L = a.L;
  p.H = a.H;
  p.dk = a.dk;
  p.dv = a.dv;
  p.chunks = chunks_of(a.L);
  p.slices = (a.dv + 63) / 64;
  p.scale = a.scale;
  p.segments = p.segment = p.run = 1;
  if (p.chunks) p.segment = p.chunks;
  return p;
}
// The states that segments start from: what each carries (all but the last; with `all`, for a gradient, the last's too, and products
// transposed), then one behind the other.
template <typename T, int DK>
hipError_t launch_carry(DeltaRun* p, const DeltaSizes& a, const Cut& c, const per_seq_states* state, float* carried, bool all, hipStream_t s) {
  p->segments = p->run = c.segments;
  p->segment = c.segment;
  if (c.segments < 2) return hipSuccess;
  p->carried = carried;
  p->each = carried_floats(a, all);
  p->turned = all;
  p->run = all ? c.segments : c.segments - 1;
  hipError_t e = launch_run<T, DK, CARRYING>(*p, a.B * a.H, s);
  if (e != hipSuccess) return e;
  const size_t each = p->each;
  DeltaJoin j{carried, carried + (size_t)a.dk * a.dv, nullptr, 0, 0, each, each, a.lengths, a.L, a.H, a.dk, a.dv, p->slices, c.segments, c.segment};
  if (state) { j.in = state->d; j.in_batch = state->batch; j.in_head = state->head; }
  k_delta_join<DK, false><<<a.B * a.H * p->slices, 4 * DK, 0, s>>>(j);
  e = hipGetLastError();
  p->run = c.segments;
  p->in = carried;
  p->in_segment = (int64_t)each;
  p->in_head = p->in_segment * c.segments;
  p->in_batch = p->in_head * a.H;
  return e;
}

// Whether the workgroups over the sequences form their chunks' records themselves: a launch less, but a wave for a chunk, so that waves stand idle where
// there are fewer than four chunks, and no other workgroup's passes beside them where the chip is full.  64 x 64, 4 heads, us, as a launch of
// their own and by the workgroups: 64 x 32 tokens 15.6, 13.4; 128 x 64 24.2, 19.3; 256 x 64 36.2, 35.2; 512 x 64 60.8, 63.4; 4096 x 32 322, 413;
// of three or four chunks 64 x 80 21.2, 17.7; 512 x 128 98.8, 96.3; 1024 x 128 208, 196; 4096 x 80 601, 607.  In fp32, where a workgroup has a compute unit,
// 64 x 64 23.1, 19.9; 128 x 64 34.5, 37.4.  A gradient, whose records are twice as much work: 128 x 32 54.9, 53.3; 256 x 32 91.6, 93.2.
bool makes_own(const DeltaSizes& a, const Cut& c, bool backward) {
  const uint32_t chunks = chunks_of(a.L);
  if (!a.L || chunks > 4 || c.segments > 1 || a.dv > 64) return false;
  const uint64_t rows = (uint64_t)a.B * a.H;
  if (a.dtype == PER_SEQ_F32) return rows <= 256;
  return rows <= (backward ? 512 : chunks > 2 ? ~0ull : 1024);
}

template <typename T, int DK>
hipError_t forward(const DeltaSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v, const per_seq_states* state,
                   const per_seq_rows& out, const per_seq_states* out_state, void* work, hipStream_t s) {
  DeltaRun p = make_run(a, q, k, v, state, work, sizeof(DeltaRecord));
  const Cut c = cut(a, false);
  const bool own = makes_own(a, c, false);
  hipError_t e = own ? hipSuccess : launch_pairs<T, DK, false>(a, q, k, work, s);
  if (e != hipSuccess) return e;
  e = launch_carry<T, DK>(&p, a, c, state, reinterpret_cast<float*>(static_cast<uint8_t*>(work) + record_bytes(a)), false, s);
  if (e != hipSuccess) return e;
  p.out = rows(out, a.dtype, 1);
  if (out_state) { p.to = out_state->d; p.to_batch = out_state->batch; p.to_head = out_state->head; }
  if (!own) return launch_run<T, DK, FORWARD>(p, a.B * a.H, s);
  p.pairs = make_pairs(a, q, k, work);
  return launch_run<T, DK, FORWARD, true>(p, a.B * a.H, s);
}

DeltaFold fold(const DeltaSizes& a, const float* from, const per_seq_rows& to, uint32_t n, uint32_t width, uint32_t stride) {
  DeltaFold f{from, rows(to, a.dtype, 1), n, width, stride, 0};
  if (n == a.H) return f;
  const uint32_t per = 256 / ((width + 3) / 4);
  const uint64_t blocks = ((uint64_t)a.B * a.L * n + per - 1) / per;
  f.blocks = (uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20);
  return f;
}

template <typename T, int DK>
hipError_t backward(const DeltaSizes& a, const per_seq_rows& dout, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                    const per_seq_states* state, const per_seq_states* dstate, const per_seq_rows& dq, const per_seq_rows& dk,
                    const per_seq_rows& dv, const per_seq_gates& dlog_decay, const per_seq_gates& dbeta, const per_seq_states* dstate0,
                    void* work, hipStream_t s) {
  const BackWork w = back_work(a);
  uint8_t* const at = static_cast<uint8_t*>(work);
  auto floats = [&](size_t o) { return reinterpret_cast<float*>(at + o); };
  const uint32_t bh = a.B * a.H;
  const Cut c = cut(a, true);
  const bool own = makes_own(a, c, true);
  hipError_t e = own ? hipSuccess : launch_pairs<T, DK, true>(a, q, k, at + w.records, s);
  if (e != hipSuccess) return e;
  DeltaRun run = make_run(a, q, k, v, state, at + w.records, sizeof(DeltaRecordBack));
  run.dout = rows(dout, a.dtype, 1);
  run.states = reinterpret_cast<bf16x8*>(at + w.states);
  run.y = floats(w.y);
  run.x = floats(w.x);
  run.read = floats(w.read);
  e = launch_carry<T, DK>(&run, a, c, state, floats(w.carried), true, s);
  if (own) run.pairs = make_pairs(a, q, k, at + w.records);
  if (e == hipSuccess && run.chunks) e = own ? launch_run<T, DK, KEEPING, true>(run, bh, s) : launch_run<T, DK, KEEPING>(run, bh, s);
  if (e != hipSuccess) return e;
  DeltaBack b{};
  b.q = run.q;
  b.k = run.k;
  b.dout = run.dout;
  b.records = run.records;
  b.lengths = a.lengths;
  if (dstate) { b.in = dstate->d; b.in_batch = dstate->batch; b.in_head = dstate->head; }
  b.L = a.L;
  b.H = a.H;
  b.dk = a.dk;
  b.dv = a.dv;
  b.chunks = run.chunks;
  b.slices = run.slices;
  b.segments = c.segments;
  b.segment = c.segment;
  b.scale = a.scale;
  b.states = run.states;
  b.y = run.y;
  b.x = run.x;
  b.dstates = reinterpret_cast<bf16x8*>(at + w.dstates);
  b.dz = floats(w.dz);
  b.along = floats(w.along);
  b.strength = floats(w.strength);
  b.write = floats(w.write);
  b.stay = floats(w.stay);
  if (c.segments > 1) {   // what each segment but the first adds, then the gradients behind the segments
    b.carried = floats(w.carried_back);
    b.first_segment = 1;
    b.run = c.segments - 1;
    e = launch_back<T, DK, true>(b, bh, s);
    if (e != hipSuccess) return e;
    const size_t each = (size_t)a.dk * a.dv;
    const DeltaJoin j{b.carried, floats(w.carried) + (size_t)a.dk * (a.dv + a.dk), b.in, b.in_batch, b.in_head, each, carried_floats(a, true),
                      a.lengths, a.L, a.H, a.dk, a.dv, b.slices, c.segments, c.segment};
    k_delta_join<DK, true><<<bh * b.slices, 4 * DK, 0, s>>>(j);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    b.in = b.carried;
    b.in_segment = (int64_t)each;
    b.in_head = b.in_segment * c.segments;
    b.in_batch = b.in_head * a.H;
  }
  b.first_segment = 0;
  b.run = c.segments;
  if (dstate0) { b.to = dstate0->d; b.to_batch = dstate0->batch; b.to_head = dstate0->head; }
  e = launch_back<T, DK, false>(b, bh, s);
  if (e != hipSuccess || !run.chunks) return e;
  DeltaGrads g{};
  g.q = run.q;
  g.k = run.k;
  g.dout = run.dout;
  g.dq = rows(dq, a.dtype, 1);
  g.dk = rows(dk, a.dtype, 1);
  g.dvr = rows(dv, a.dtype, 1);
  g.log_decay = gates(a.log_decay);
  g.beta = gates(a.beta);
  g.lengths = a.lengths;
  g.L = a.L;
  g.H = a.H;
  g.dkw = a.dk;
  g.dv = a.dv;
  g.chunks = run.chunks;
  g.scale = a.scale;
  g.direct_q = a.Q == a.H;
  g.direct_k = a.K == a.H;
  g.direct_v = a.V == a.H;
  g.fold_q = floats(w.fold_q);
  g.fold_k = floats(w.fold_k);
  g.states = run.states;
  g.dstates = b.dstates;
  g.y = run.y;
  g.dz = b.dz;
  g.past = floats(w.past);
  e = launch_grads<T, DK>(g, bh, s);
  if (e != hipSuccess) return e;
  DeltaFinish f{};
  f.gates = DeltaGates{gates(dlog_decay), gates(dbeta), a.lengths, bh, a.L, a.H, run.chunks, (a.dv + 31) / 32 * 2, run.read, b.along, b.strength, b.write, b.stay, g.past};
  f.gate_blocks = (bh * run.chunks + 256 / kChunk - 1) / (256 / kChunk);
  f.fold[0] = fold(a, g.fold_q, dq, a.Q, a.dk, a.dk);
  f.fold[1] = fold(a, g.fold_k, dk, a.K, a.dk, a.dk);
  f.fold[2] = fold(a, b.dz, dv, a.V, a.dv, (a.dv + 31) / 32 * 32);
  k_delta_finish<T><<<f.gate_blocks + f.fold[0].blocks + f.fold[1].blocks + f.fold[2].blocks, 256, 0, s>>>(f);
  e = hipGetLastError();
  return e;
}

template <typename T, int VEC, int R>
hipError_t step(const DeltaStep& p, uint32_t rows, hipStream_t s) {
  const Past way = past((uint64_t)rows * p.dk * p.dv * 4);
  if (way == KEPT) k_delta_step<T, VEC, R, KEPT><<<rows, 256, 0, s>>>(p);
  else if (way == STORES_PAST) k_delta_step<T, VEC, R, STORES_PAST><<<rows, 256, 0, s>>>(p);
  else k_delta_step<T, VEC, R, ALL_PAST><<<rows, 256, 0, s>>>(p);
  return hipGetLastError();
}
template <typename T>
hipError_t step(DeltaStep p, uint32_t rows, hipStream_t s) {
  const bool wide = p.dv % 4 == 0 && (reinterpret_cast<uintptr_t>(p.state.d) & 15) == 0 && p.state.batch % 4 == 0 && p.state.head % 4 == 0;
  const uint32_t columns = wide ? p.dv / 4 : p.dv;
  p.groups = 256 / columns < p.dk ? 256 / columns : p.dk;
  const uint32_t held = (p.dk + p.groups - 1) / p.groups;   // rows of a thread
  if (!wide) return held <= 16 ? step<T, 1, 16>(p, rows, s) : step<T, 1, 64>(p, rows, s);
  return held <= 4 ? step<T, 4, 4>(p, rows, s) : step<T, 4, 16>(p, rows, s);
}

}  // namespace

size_t delta_work_bytes(const DeltaSizes& a, bool backward) {
  if (!a.B || !a.H || !a.L) return 0;
  return backward ? back_work(a).bytes : record_bytes(a) + carried_bytes(a, cut(a, false), false);
}

hipError_t launch_delta(const DeltaSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v, const per_seq_states* state,
                        const per_seq_rows& out, const per_seq_states* out_state, void* work, hipStream_t s) {
  auto* call = a.dtype == PER_SEQ_BF16 ? (a.dk <= 64 ? forward<bf16, 64> : forward<bf16, 128>) : (a.dk <= 64 ? forward<float, 64> : forward<float, 128>);
  return call(a, q, k, v, state, out, out_state, work, s);
}

hipError_t launch_delta_backward(const DeltaSizes& a, const per_seq_rows& dout, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                                 const per_seq_states* state, const per_seq_states* dstate, const per_seq_rows& dq, const per_seq_rows& dk,
                                 const per_seq_rows& dv, const per_seq_gates& dlog_decay, const per_seq_gates& dbeta,
                                 const per_seq_states* dstate0, void* work, hipStream_t s) {
  auto* call = a.dtype == PER_SEQ_BF16 ? (a.dk <= 64 ? backward<bf16, 64> : backward<bf16, 128>) : (a.dk <= 64 ? backward<float, 64> : backward<float, 128>);
  return call(a, dout, q, k, v, state, dstate, dq, dk, dv, dlog_decay, dbeta, dstate0, work, s);
}

hipError_t launch_delta_step(const DeltaSizes& a, const per_seq_rows& q, const per_seq_rows& k, const per_seq_rows& v,
                             const per_seq_states& state, const per_seq_rows& out, hipStream_t s) {
  const DeltaStep p{rows(q, a.dtype, a.H / a.Q), rows(k, a.dtype, a.H / a.K), rows(v, a.dtype, a.H / a.V), rows(out, a.dtype, 1),
                    gates(a.log_decay), gates(a.beta), SeqStates{state.d, state.batch, state.head}, a.H, a.dk, a.dv, 0, a.scale, a.lengths};
  return a.dtype == PER_SEQ_BF16 ? step<bf16>(p, a.B * a.H, s) : step<float>(p, a.B * a.H, s);
}

}  // namespace per
