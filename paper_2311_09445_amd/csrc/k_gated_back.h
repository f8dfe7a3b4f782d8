// The gradient of the gated delta rule.  Part of seq_delta.hip (included inside namespace per).
//
// Against time, with R the gradient of the state behind a chunk,
//   dU = pairs^T dO + left K R,  du = (1 + diag(beta) N)^-T dU,  dV = dZ = beta du,  dbeta = Y . du,
//   R <- e^Gn R + Q^T (scale e^G dO) - K^T (e^G dZ),
// in columns that do not meet, as over time (k_delta_back).  What is left does not depend on the order of the chunks (k_delta_grads):
//   dQ = scale e^G dO S^T + dM K,   dK = -e^G dZ S^T + left U R^T + dM^T Q + (dN + dN^T) K,
//   dM = scale e_ij dO U^T (i >= j),   dN = -e_ij dZ U^T (i > j).
//
// What bounds them, in bfloat16: k_delta_back, which asks for everything a chunk ahead, takes 3.9 us for a chunk of 64 x 64 (32 sequences of 512 tokens of 8
// heads 62 us); of 2 x 8192 tokens of 16 heads of 128 x 128 it moves 2.1 GB in 369 us, memory's rate.  k_delta_grads takes 426 us for 1.8 GB of
// the latter, waiting for memory with two workgroups to a compute unit (three spilled: 710 where two took 447).
//
// The gradient of a decay's logarithm is the sum of all that goes past its token t, each term with the decays between as a factor.  Of a chunk that is
//   sum (i >= t > j) dM_ij q_i.k_j + dN_ij k_i.k_j   (what tokens of the chunk read of each other's writes; k_delta_grads)
//   + sum (i >= t) scale e^G_i dO_i . S^T q_i - dZ_i . e^G_i S^T k_i   (what they read of the state before the chunk; rows of both passes)
//   + sum (j < t) left_j u_j . R^T k_j   (what they write to the state behind it)   + e^Gn <R, S>   (what stays).
// So what a fast decay leaves is exact to 2^-24 of itself.  (As a border's <R, S> less a sum of out . dO - dZ . V over the tokens before t, it was what is
// left of large numbers: noise of 2^-24 of theirs, also behind a decay that keeps nothing.)

struct DeltaBack {
  SeqRows q, k, dout;
  const void* records;
  const int32_t* lengths;
  const float* in;
  float* to;
  int64_t in_batch, in_head, in_segment, to_batch, to_head;
  uint32_t L, H, dk, dv, chunks, slices, segments, segment;   // segment: chunks of one
  uint32_t first_segment, run;   // the segments that are taken
  float scale;
  float* carried;                // [sequence, head][segment][dk][dv]: what a segment adds to the gradient of the state before it
  const bf16x8* states;
  const float *y, *x;
  bf16x8* dstates;                 // the gradients of the states behind the chunks
  float *dz, *along, *strength, *write, *stay;   // along: rows of dZ . what keys read; write: of left u . R^T k; stay: 32 terms of e^Gn <R, S>
};

// Parts of states and their gradients in the products for rows.  (In bfloat16 with one, rounded, gradients of keys were off by 1.9 to 2.6e-3 in 2-norm, of
// queries by up to 2.1e-3, where their own rounding, all that is left with two, is 1.7e-3.  It took 204 us for 217 of 32 ragged sequences of 512 tokens of 8 heads of
// 64 x 64, 951 for 995 of 128 of them, 1367 for 1480 of 2 x 8192 of 16 heads of 128 x 128.)
template <typename T>
constexpr int kGradParts = sizeof(T) == 2 ? 2 : 3;

template <typename T, int DK, bool DIRECT_ROWS>
struct BackLds {
  static constexpr uint32_t Q = 0, K = kParts<T> * Tile<DK>::SIZE, D = 2 * K,
                            SOLVE = D + (DIRECT_ROWS ? Tile<64>::SIZE : 0), SIZE = SOLVE + (DIRECT_ROWS ? 3 * 1024 : 0), BYTES = 2 * SIZE * sizeof(bf16);
};

// CARRY: only what a segment adds; two workgroups to a compute unit where rows go straight to LDS.  The whole pass has one: with two, registers for 64 x 64
// spill (32 ragged sequences of 512 tokens of 8 heads, the whole gradient, 204 us and 254; 128 of them 951 and 1084).
template <typename T, int DK, bool CARRY, bool DIRECT_ROWS>
__global__ __launch_bounds__(256, DIRECT_ROWS && CARRY ? 2 : 1) void k_delta_back(DeltaBack p) {
  constexpr int PT = kParts<T>, TX = DK / 16, KX = DK / 32, TURN = PT == 1 ? TX : 4;
  constexpr bool AHEAD = DIRECT_ROWS && !CARRY;   // the state before a chunk is asked for a chunk ahead too
  typedef BackLds<T, DK, DIRECT_ROWS> Lds;
  static_assert(!DIRECT_ROWS || Lds::BYTES <= 65536, "loads to LDS have 16 bits of address");
  extern __shared__ __attribute__((aligned(256))) uint8_t lds_raw[];
  bf16* const lds = reinterpret_cast<bf16*>(lds_raw);
  const uint32_t slice = blockIdx.x % p.slices, item = blockIdx.x / p.slices, seg = p.first_segment + item % p.run, bh = item / p.run, h = bh % p.H, b = bh / p.H;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const uint32_t L = p.L, dk = p.dk, dv = p.dv, blocks = (dv + 31) / 32, col0 = 64 * slice + 16 * wave, col = col0 + m;
  const bool on = col < dv, works = col0 < blocks * 32;
  const uint32_t valid = __builtin_amdgcn_readfirstlane(valid_tokens(p.lengths, b, L)), all_chunks = (valid + kChunk - 1) / kChunk, width = blocks * 32;
  const uint32_t chunk0 = seg * p.segment, chunks = all_chunks < chunk0 ? chunk0 : all_chunks - chunk0 < p.segment ? all_chunks : chunk0 + p.segment;   // its end
  const DeltaRecordBack* const records = static_cast<const DeltaRecordBack*>(p.records) + (size_t)bh * p.chunks;
  const bool pieces = p.q.near && p.k.near && dk >= 16 / sizeof(T);
  const size_t row0 = (size_t)bh * p.chunks * kChunk, part0 = ((size_t)bh * (blocks * 2) + col0 / 16) * p.chunks;

  f32x4 s[TX];
#pragma unroll
  for (int a = 0; a < TX; ++a)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t row = state_row(a, 4 * g + r);
      s[a][r] = !CARRY && p.in && on && row < dk ? p.in[(int64_t)b * p.in_batch + (int64_t)h * p.in_head + seg * p.in_segment + (size_t)row * dv + col] : 0.0f;
    }
  const T *const q0 = row_of<T>(p.q, b, 0, h), *const k0 = row_of<T>(p.k, b, 0, h), *const d0 = row_of<T>(p.dout, b, 0, h);
  TwoRows<T, DK> rows;
  DirectRows<DK> direct_q, direct_k;
  DirectRows<64> direct_d;
  Walk walk_q, walk_k, walk_d;
  struct Next {
    bf16x8 pairs[3][2], solve[3][2];
    f32x4 y[2], x[2];
    bf16x8 before[KX][kStateParts<T>];   // the state before the chunk
    Column<T> d;
  } next, now;
  RecordNumbers num, next_num;
  const uint32_t lds0 = lds_address(lds);
  auto ask_state = [&](uint32_t c, Next& to) {
    if (CARRY || !works) return;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) to.x[i][r] = p.x[(row0 + c * kChunk + 16 * i + 4 * g + r) * width + col];
#pragma unroll
    for (int k = 0; k < KX; ++k)
#pragma unroll
      for (int t = 0; t < kStateParts<T>; ++t) to.before[k][t] = p.states[state_at<DK>(bh, p.chunks, c, blocks, kStateParts<T>, t, col0 / 16) + k * 64 + lane];
  };
  auto fetch = [&](uint32_t c) {
    const DeltaRecordBack* const record = records + c;
    if constexpr (DIRECT_ROWS) {
      const uint32_t n = valid - c * kChunk, to = lds0 + (c & 1) * Lds::SIZE * 2;
      direct_q.ask(to + Lds::Q * 2, walk_q.next(), wave, n);
      direct_k.ask(to + Lds::K * 2, walk_k.next(), wave, n);
      direct_d.ask(to + Lds::D * 2, walk_d.next(), wave, n);
      ask_rows<6>(to + Lds::SOLVE * 2, record->solve_t, wave, lane);
    } else {
      rows.store(lds + (c & 1) * Lds::SIZE, valid - c * kChunk, dk, pieces);
      if (c > chunk0) rows.load(p.q, p.k, q0, k0, (c - 1) * kChunk, valid, dk, pieces);
      next.d.ask(p.dout, d0, c * kChunk, valid, on, col, g);
#pragma unroll
      for (int t = 0; t < 3; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) next.solve[t][i] = record->solve_t[t][i][lane];
    }
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) next.pairs[t][i] = record->of.pairs[t][i][lane];
    if (!CARRY && works)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) next.y[i][r] = p.y[(row0 + c * kChunk + 16 * i + 4 * g + r) * width + col];
    if (AHEAD) ask_state(c, next);
    next_num.load(&record->of, m, g);
  };
  if constexpr (DIRECT_ROWS) {
    const uint32_t last = chunks > chunk0 ? chunks - 1 : chunk0;
    walk_q.set(p.q, q0, last, true);
    walk_k.set(p.k, k0, last, true);
    walk_d.set(p.dout, d0 + 64 * slice, last, true);
    direct_q.set(p.q, dk, wave, lane);
    direct_k.set(p.k, dk, wave, lane);
    direct_d.set(p.dout, dv - 64 * slice, wave, lane);
    if (dk < DK || dv - 64 * slice < 64) {
      for (uint32_t i = 0; i < 2; ++i) {
        DirectRows<DK>::clear(lds + i * Lds::SIZE + Lds::Q, 0, threadIdx.x);
        DirectRows<DK>::clear(lds + i * Lds::SIZE + Lds::K, 0, threadIdx.x);
        DirectRows<64>::clear(lds + i * Lds::SIZE + Lds::D, 0, threadIdx.x);
      }
      __syncthreads();
    }
  } else if (chunk0 < chunks) {
    rows.load(p.q, p.k, q0, k0, (chunks - 1) * kChunk, valid, dk, pieces);
  }
  if (chunk0 < chunks) fetch(chunks - 1);
  f32x4 dz[2] = {};
  float sums = 0.0f, more = 0.0f;
  auto flush = [&](uint32_t c) {   // (behind the next barrier, as over time)
    if (CARRY || !works) return;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) p.dz[(row0 + c * kChunk + 16 * i + 4 * g + r) * width + col] = dz[i][r];
    const size_t at = part0 * kChunk + c * kChunk + 4 * (m & 4) + 4 * g + (m & 3);
    (m & 8 ? p.strength : p.along)[at] = sums;
    (m & 8 ? p.stay : p.write)[at] = more;
  };
  for (uint32_t end = chunks; end > chunk0; --end) {
    const uint32_t c = end - 1, first = c * kChunk;
    bf16 *const buffer = lds + (c & 1) * Lds::SIZE, *const Q = buffer + Lds::Q, *const K = buffer + Lds::K;
    if constexpr (DIRECT_ROWS) {
      // (what is stored behind the loads: the gradient's planes, and from the second chunk dZ)
      if (!CARRY && works && end + 1 < chunks) arrive<kGradParts<T> * KX + 8>();
      else arrive<0>();
      if (valid - first < kChunk) {
        DirectRows<DK>::clear(Q, valid - first, threadIdx.x);
        DirectRows<DK>::clear(K, valid - first, threadIdx.x);
        DirectRows<64>::clear(buffer + Lds::D, valid - first, threadIdx.x);
        __syncthreads();
      }
    } else {
      __syncthreads();
    }
    next_num.there();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!CARRY) asm volatile("" : "+v"(next.y[i]));
      if (AHEAD) asm volatile("" : "+v"(next.x[i]));
#pragma unroll
      for (int t = 0; t < 3; ++t) asm volatile("" : "+v"(next.pairs[t][i]));
    }
    num = next_num;
    if constexpr (AHEAD) {
#pragma unroll
      for (int k = 0; k < KX; ++k)
#pragma unroll
        for (int t = 0; t < kStateParts<T>; ++t) asm volatile("" : "+v"(next.before[k][t]));
    }
    now = next;
    if (!AHEAD) ask_state(c, now);
    if (c > chunk0) fetch(c - 1);
    if (end < chunks) flush(c + 1);
    if (!CARRY && works) {
#pragma unroll
      for (int k = 0; k < KX; ++k) {
        const Parts<kGradParts<T>> parts = Parts<kGradParts<T>>::of(s[2 * k], s[2 * k + 1]);
#pragma unroll
        for (int t = 0; t < kGradParts<T>; ++t) p.dstates[state_at<DK>(bh, p.chunks, c, blocks, kGradParts<T>, t, col0 / 16) + k * 64 + lane] = parts.v[t];
      }
    }
    if (works) {
      f32x4 w4[4] = {};   // (of even and odd k)
#pragma unroll
      for (int k = 0; k < KX; k += 2) {
        Operand<T> rows_k[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) rows_k[j] = Operand<T>::template along<DK>(K, 16 * (j & 1) + m, k + j / 2, g);
        const Parts<3> sp[2] = {Parts<3>::of(s[2 * k], s[2 * k + 1]), Parts<3>::of(s[2 * k + 2], s[2 * k + 3])};
        mma_turns<4, 2, PT, 3>([&](int j) -> const bf16x8 (&)[PT] { return rows_k[j].v; }, [&](int j) -> const bf16x8 (&)[3] { return sp[j / 2].v; }, w4);
      }
      f32x4 d[2];
      bf16x8 solve[2][3], pairs[2][3];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < 3; ++t) {
          solve[i][t] = DIRECT_ROWS ? reinterpret_cast<const bf16x8*>(buffer + Lds::SOLVE)[(2 * t + i) * 64 + lane] : now.solve[t][i];
          pairs[i][t] = now.pairs[t][i];
        }
      if constexpr (DIRECT_ROWS) {
        auto column = [&](uint32_t i) { return 16 * wave + i; };
        Operand<bf16>::across<64>(buffer + Lds::D, column, m, g).widen(&d[0], &d[1]);
      } else {
        now.d.widen(first, valid, on, g, d);
      }
      const Operand<T> dp = operand_of<T>(d);
      f32x4 w[2], du[2] = {};
#pragma unroll
      for (int i = 0; i < 2; ++i) w[i] = num.left[i] * (w4[i] + w4[i + 2]);
      if constexpr (!CARRY) {
        float products[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          products[i] = w[i / 4][i % 4] * (num.beta[i / 4][i % 4] * now.y[i / 4][i % 4]);
          products[i + 8] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < KX; ++k) {
          f32x4 S[2] = {};
          if constexpr (sizeof(T) == 2) {
            of_halves(now.before[k], &S[0], &S[1]);
          } else {
#pragma unroll
            for (int t = 2; t >= 0; --t)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                S[0][e] += (float)now.before[k][t][e];
                S[1][e] += (float)now.before[k][t][e + 4];
              }
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) products[i + 8] = fmaf(S[i / 4][i % 4], s[2 * k + i / 4][i % 4], products[i + 8]);
        }
        more = sums16(products, m);
        if (m & 8) more = fmaf(more, num.kept[0], more * num.kept[1]);
      }
      mma_turns<2, 2, 3, PT>([&](int i) -> const bf16x8 (&)[3] { return pairs[i]; }, [&](int) -> const bf16x8 (&)[PT] { return dp.v; }, w);
      const Parts<3> wp = Parts<3>::of(w[0], w[1]);
      mma_turns<2, 2, 3, 3>([&](int i) -> const bf16x8 (&)[3] { return solve[i]; }, [&](int) -> const bf16x8 (&)[3] { return wp.v; }, du);
#pragma unroll
      for (int i = 0; i < 2; ++i) dz[i] = num.beta[i] * du[i];
      const Parts<3> ip = Parts<3>::of(p.scale * num.gamma[0] * d[0], p.scale * num.gamma[1] * d[1]), op = Parts<3>::of(-num.gamma[0] * dz[0], -num.gamma[1] * dz[1]);
#pragma unroll
      for (int a0 = 0; a0 < TX; a0 += TURN) {
        Operand<T> cols[TURN];
        f32x4 part[TURN];
#pragma unroll
        for (int a = 0; a < TURN; ++a) {
          cols[a] = Operand<T>::template across<DK>(Q, [&](uint32_t i) { return state_row(a0 + a, i); }, m, g);
          part[a] = num.keep(s[a0 + a]);
        }
        mma_turns<TURN, 2, PT, 3>([&](int a) -> const bf16x8 (&)[PT] { return cols[a].v; }, [&](int) -> const bf16x8 (&)[3] { return ip.v; }, part);
#pragma unroll
        for (int a = 0; a < TURN; ++a) cols[a] = Operand<T>::template across<DK>(K, [&](uint32_t i) { return state_row(a0 + a, i); }, m, g);
        mma_turns<TURN, 2, PT, 3>([&](int a) -> const bf16x8 (&)[PT] { return cols[a].v; }, [&](int) -> const bf16x8 (&)[3] { return op.v; }, part);
#pragma unroll
        for (int a = 0; a < TURN; ++a) s[a0 + a] = part[a];
      }
      if constexpr (!CARRY) {
        float products[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          products[i] = dz[i / 4][i % 4] * now.x[i / 4][i % 4];
          products[i + 8] = now.y[i / 4][i % 4] * du[i / 4][i % 4];
        }
        sums = sums16(products, m);
      }
    }
  }
  if (chunk0 < chunks) flush(chunk0);
  float* to = seg == 0 && p.to ? p.to + (int64_t)b * p.to_batch + (int64_t)h * p.to_head : nullptr;
  if (CARRY) to = p.carried + ((size_t)bh * p.segments + seg) * dk * dv;
  if (to && on)
#pragma unroll
    for (int a = 0; a < TX; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t row = state_row(a, 4 * g + r);
        if (row < dk) to[(size_t)row * dv + col] = s[a][r];
      }
}

struct DeltaGrads {
  SeqRows q, k, dout, dq, dk, dvr;
  Gates log_decay, beta;
  const int32_t* lengths;
  uint32_t L, H, dkw, dv, chunks;
  float scale;
  uint32_t direct_q, direct_k, direct_v;   // to their rows; else to fold_q, fold_k, [sequence and head][token][dk] in fp32, and left in dz
  float *fold_q, *fold_k;
  const bf16x8 *states, *dstates;
  const float *y, *dz;
  float* past;   // [sequence and head][token]: what goes past it within its chunk
};
struct DeltaGates {
  Gates dlog_decay, dbeta;
  const int32_t* lengths;
  uint32_t rows, L, H, chunks, parts;   // rows: sequences and heads; parts: slices of 16 columns, which sums come in
  const float *read, *along, *strength, *write, *stay, *past;
};
// Eight neighbours of a row.
template <typename T>
__device__ __forceinline__ void store_eight(T* row, bool wide, uint32_t col, uint32_t width, f32x4 a, f32x4 c) {
  typedef T Vec __attribute__((ext_vector_type(8)));
  if (sizeof(T) == 2 && wide && col + 8 <= width) {
    Vec o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i] = (T)a[i];
      o[i + 4] = (T)c[i];
    }
    *reinterpret_cast<Vec*>(row + col) = o;
  } else {
    store_four<T>(row, wide, col, width, a);
    store_four<T>(row, wide, col + 4, width, c);
  }
}

template <typename T, int DK>
constexpr uint32_t grads_lds() { return (2 * kParts<T> + 2 * kGradParts<T>) * Tile<DK>::SIZE * sizeof(bf16) + 3 * 32 * kPairRow * sizeof(float); }

// A workgroup takes a chunk; its waves share the chunk's columns of dk, and the four 16 x 16 tiles of its pairs.  Everything that comes from memory is
// asked for before anything is waited for.  Columns of dv go to LDS mixed, column 8 g + 4 s + e of a block to row 16 s + 4 g + e, and so are rows of
// results, so that what a lane reads and writes of a token are eight elements in a row.
template <typename T, int DK>
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : DK == 64 ? 3 : 2) void k_delta_grads(DeltaGrads p) {
  constexpr int NC = DK / 64, PT = kParts<T>, PS = kGradParts<T>, PU = PS, LESS = PU - 1;
  static_assert(kStateParts<T> == PS, "planes are read as parts, or halves of as many");
  extern __shared__ __attribute__((aligned(256))) uint8_t lds_raw[];
  bf16* const Q = reinterpret_cast<bf16*>(lds_raw);
  bf16* const K = Q + PT * Tile<DK>::SIZE;
  bf16* const S = K + PT * Tile<DK>::SIZE;
  bf16* const R = S + PS * Tile<DK>::SIZE;
  float* const dM = reinterpret_cast<float*>(R + PS * Tile<DK>::SIZE);
  float* const dN = dM + 32 * kPairRow;
  float* const pasts = dN + 32 * kPairRow;
  __shared__ double G[32];
  __shared__ __attribute__((aligned(16))) float gamma[32], left[32], beta[32];
  const uint32_t chunk = blockIdx.x % p.chunks, bh = blockIdx.x / p.chunks, h = bh % p.H, b = bh / p.H;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const uint32_t L = p.L, dk = p.dkw, dv = p.dv, blocks = (dv + 31) / 32, width = blocks * 32;
  const uint32_t valid = __builtin_amdgcn_readfirstlane(valid_tokens(p.lengths, b, L)), first = chunk * kChunk, end = L - first < kChunk ? L - first : kChunk;
  const size_t row0 = (size_t)bh * p.chunks * kChunk + first;
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  if (first >= valid) {
    for (uint32_t i = threadIdx.x; i < end * ((dk + 3) / 4); i += 256) {
      const uint32_t t = first + i / ((dk + 3) / 4), col = i % ((dk + 3) / 4) * 4;
      if (p.direct_q) store_four<T>(row_to<T>(p.dq, b, t, h), p.dq.wide, col, dk, zero);
      if (p.direct_k) store_four<T>(row_to<T>(p.dk, b, t, h), p.dk.wide, col, dk, zero);
    }
    for (uint32_t i = threadIdx.x; p.direct_v && i < end * ((dv + 3) / 4); i += 256)
      store_four<T>(row_to<T>(p.dvr, b, first + i / ((dv + 3) / 4), h), p.dvr.wide, i % ((dv + 3) / 4) * 4, dv, zero);
    return;
  }
  const uint32_t n = valid - first;   // (and more)
  constexpr uint32_t HELD = 2 * (DK / 32) * 64 / 256;   // pieces of a thread in 32 columns of a plane
  bf16x8 next_s[PS][HELD], next_r[PS][HELD];
  Four<T> next_d[2][2];
  f32x4 next_z[2][2], next_y[2][2];
  auto ask = [&](uint32_t block) {
#pragma unroll
    for (int t = 0; t < PS; ++t)
#pragma unroll
      for (uint32_t i = 0; i < HELD; ++i) {
        next_s[t][i] = p.states[state_at<DK>(bh, p.chunks, chunk, blocks, kStateParts<T>, t, 2 * block) + threadIdx.x + 256 * i];
        next_r[t][i] = p.dstates[state_at<DK>(bh, p.chunks, chunk, blocks, PS, t, 2 * block) + threadIdx.x + 256 * i];
      }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t t = 16 * i + m;
      const T* row = row_of<T>(p.dout, b, t < n ? first + t : first, h);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t col = 32 * block + 8 * g + 4 * e;
        ask_four<T>(row, p.dout.wide, col, dv, &next_d[i][e]);
        next_z[i][e] = *reinterpret_cast<const f32x4*>(p.dz + (row0 + t) * width + col);
        next_y[i][e] = *reinterpret_cast<const f32x4*>(p.y + (row0 + t) * width + col);
      }
    }
  };
  TwoRows<T, DK> rows;
  const bool pieces = p.q.near && p.k.near && dk >= 16 / sizeof(T);
  rows.load(p.q, p.k, row_of<T>(p.q, b, 0, h), row_of<T>(p.k, b, 0, h), first, valid, dk, pieces);
  ask(0);
  if (wave == 0) {
    const uint32_t column = lane & 31;
    const bool here = column < n;
    const float strength = here ? p.beta.at(b, first + column, h) : 0.0f;
    const double sum = decay_sums(p.log_decay, b, h, here ? first + column : first, here, lane);
    const double total = __shfl(sum, 31);
    if (lane < 32) {
      G[lane] = sum;
      gamma[lane] = expf((float)sum);
      left[lane] = expf((float)(total - sum));
      beta[lane] = strength;
    }
  }
  rows.store(Q, n, dk, pieces);
  // of queries; of keys by the state, and by its gradient, whose rows are scaled at the end
  f32x4 aq[2][NC] = {}, as[2][NC] = {}, ar[2][NC] = {}, dm = zero, dn = zero;
  const uint32_t ti = wave >> 1, tj = wave & 1;
  auto column = [&](uint32_t a, uint32_t i) { return NC == 2 ? 32 * wave + 8 * (i >> 2) + 4 * a + (i & 3) : 16 * wave + i; };   // of the wave's
  for (uint32_t block = 0; block < blocks; ++block) {
    if (block) __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < HELD; ++i) {   // lane 16 g + m of tile and k: column 16 tile + m, places 32 k + 8 g ..
      const uint32_t at = threadIdx.x + 256 * i, c = 16 * (at / (64 * (DK / 32))) + (at & 15);
      const uint32_t place = Tile<DK>::at(16 * (c >> 2 & 1) + 4 * (c >> 3) + (c & 3), 4 * (at / 64 % (DK / 32)) + (at >> 4 & 3));
      Parts<PS> s;
      if constexpr (sizeof(T) == 2) {
        const bf16x8 both[2] = {next_s[0][i], next_s[1][i]};
        f32x4 a, b;
        of_halves(both, &a, &b);
        s = Parts<PS>::of(a, b);
      } else {
#pragma unroll
        for (int t = 0; t < PS; ++t) s.v[t] = next_s[t][i];
      }
#pragma unroll
      for (int t = 0; t < PS; ++t) {
        *reinterpret_cast<bf16x8*>(S + t * Tile<DK>::SIZE + place) = s.v[t];
        *reinterpret_cast<bf16x8*>(R + t * Tile<DK>::SIZE + place) = next_r[t][i];
      }
    }
    __syncthreads();
    Operand<T> d[2];
    Parts<3> z[2], u[2];   // (whole for the pairs, which the gradients of decays are made of too; rows take PU of them)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t t = 16 * i + m;
      d[i] = Operand<T>::of(four_of<T>(next_d[i][0], t < n, 32 * block + 8 * g, dv), four_of<T>(next_d[i][1], t < n, 32 * block + 8 * g + 4, dv));
      z[i] = Parts<3>::of(next_z[i][0], next_z[i][1]);
      u[i] = Parts<3>::of(beta[t] * next_y[i][0], beta[t] * next_y[i][1]);
      if (p.direct_v && wave == (block & 3) && t < end) {
        T* const to = row_to<T>(p.dvr, b, first + t, h);
        store_eight<T>(to, p.dvr.wide, 32 * block + 8 * g, dv, t < n ? next_z[i][0] : zero, t < n ? next_z[i][1] : zero);
      }
    }
    // (branches: operands that are chosen by a number would lie in memory)
    auto pair = [&](int i, int j) {
      dm = mma(d[i].v, u[j].v, dm);
      dn = mma(z[i].v, u[j].v, dn);
    };
    if (wave == 0) pair(0, 0);
    else if (wave == 2) pair(1, 0);
    else if (wave == 3) pair(1, 1);
    if (block + 1 < blocks) ask(block + 1);
#pragma unroll
    for (int a = 0; a < NC; ++a) {
      bf16x8 s[PS], r[PS];
#pragma unroll
      for (int t = 0; t < PS; ++t) {
        s[t] = Operand<bf16>::template across<DK>(S + t * Tile<DK>::SIZE, [&](uint32_t i) { return column(a, i); }, m, g).v[0];
        r[t] = Operand<bf16>::template across<DK>(R + t * Tile<DK>::SIZE, [&](uint32_t i) { return column(a, i); }, m, g).v[0];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        aq[i][a] = mma<LESS>(s, d[i].v, aq[i][a]);
        as[i][a] = mma<LESS>(s, z[i].v, as[i][a]);
        ar[i][a] = mma<LESS>(r, u[i].v, ar[i][a]);
      }
    }
  }
  f32x4 qk = zero, kk = zero;
#pragma unroll
  for (int s = 0; s < DK / 32; ++s) {
    const Operand<T> k = Operand<T>::template along<DK>(K, 16 * tj + m, s, g);
    qk = mma(Operand<T>::template along<DK>(Q, 16 * ti + m, s, g).v, k.v, qk);
    kk = mma(Operand<T>::template along<DK>(K, 16 * ti + m, s, g).v, k.v, kk);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t i = 16 * ti + 4 * g + e, j = 16 * tj + m;
    const float x = expf((float)(G[i] - G[j])), by_q = i >= j ? p.scale * x * dm[e] : 0.0f, by_k = i > j ? -x * dn[e] : 0.0f;
    dM[i * kPairRow + j] = by_q;
    dN[i * kPairRow + j] = by_k;
    pasts[i * kPairRow + j] = i > j ? fmaf(by_q, qk[e], by_k * kk[e]) : 0.0f;
  }
  __syncthreads();
  if (wave == 1) {   // (which has no pairs) the sums of rows i >= t, columns j < t: up each column, then along each row, 16 to a half of the wave
    const uint32_t at = lane & 31, half = lane & 32 ? 0 : 16;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = pasts[(half + i) * kPairRow + at];
#pragma unroll
    for (int i = 14; i >= 0; --i) x[i] += x[i + 1];
    const float upper = __shfl(x[0], at), below = half ? 0.0f : upper;   // (of rows 16 .. 31)
#pragma unroll
    for (int i = 0; i < 16; ++i) pasts[(half + i) * kPairRow + at] = x[i] + below;
    wave_sync();
    float sum = 0.0f;
#pragma unroll
    for (uint32_t j = 0; j < 16; j += 4) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(pasts + at * kPairRow + half + j);
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) sum += half + j + e < at ? v[e] : 0.0f;
    }
    sum += __shfl_xor(sum, 32);
    if (lane < 32) p.past[row0 + at] = sum;
  }
  Operand<T> qs[NC], ks[NC];
#pragma unroll
  for (int a = 0; a < NC; ++a) {
    qs[a] = Operand<T>::template across<DK>(Q, [&](uint32_t i) { return column(a, i); }, m, g);
    ks[a] = Operand<T>::template across<DK>(K, [&](uint32_t i) { return column(a, i); }, m, g);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t t = 16 * i + m;
    f32x4 x, y, na, nc;
    const float *rm = dM + t * kPairRow + 4 * g, *rn = dN + t * kPairRow + 4 * g, *cm = dM + 4 * g * kPairRow + t, *cn = dN + 4 * g * kPairRow + t;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x[r] = cm[r * kPairRow];
      y[r] = cm[(16 + r) * kPairRow];
      na[r] = rn[r] + cn[r * kPairRow];
      nc[r] = rn[16 + r] + cn[(16 + r) * kPairRow];
    }
    const Parts<PU> rows_m = Parts<PU>::of(*reinterpret_cast<const f32x4*>(rm), *reinterpret_cast<const f32x4*>(rm + 16));
    const Parts<PU> cols_m = Parts<PU>::of(x, y), both_n = Parts<PU>::of(na, nc);
    f32x4 oq[2], ok[2];
#pragma unroll
    for (int a = 0; a < NC; ++a) {
      oq[a] = mma<LESS>(ks[a].v, rows_m.v, p.scale * gamma[t] * aq[i][a]);
      ok[a] = mma<LESS>(qs[a].v, cols_m.v, left[t] * ar[i][a] - gamma[t] * as[i][a]);
      ok[a] = mma<LESS>(ks[a].v, both_n.v, ok[a]);
      if (t >= n) oq[a] = ok[a] = zero;
    }
    if (t >= end) continue;
    auto put = [&](const SeqRows& to, bool direct, float* fold, const f32x4 (&o)[2]) {
      T* const row = direct ? row_to<T>(to, b, first + t, h) : nullptr;
      float* const apart = fold + (row0 + t) * dk;
      if constexpr (NC == 2) {
        if (direct) store_eight<T>(row, to.wide, 32 * wave + 8 * g, dk, o[0], o[1]);
        else store_eight<float>(apart, dk % 4 == 0, 32 * wave + 8 * g, dk, o[0], o[1]);
      } else {
        if (direct) store_four<T>(row, to.wide, 16 * wave + 4 * g, dk, o[0]);
        else store_four<float>(apart, dk % 4 == 0, 16 * wave + 4 * g, dk, o[0]);
      }
    };
    put(p.dq, p.direct_q, p.fold_q, oq);
    put(p.dk, p.direct_k, p.fold_k, ok);
  }
}

// The gates' gradients: a thread takes a token, 32 of them a chunk.
__device__ __forceinline__ void gates_of(const DeltaGates& p, uint32_t block) {
  const uint32_t at = threadIdx.x & 31, all = p.rows * p.chunks, place = block * (256 / kChunk) + threadIdx.x / kChunk;
  const uint32_t item = place < all ? place : all - 1, chunk = item % p.chunks, bh = item / p.chunks, h = bh % p.H, b = bh / p.H;
  const uint32_t t = chunk * kChunk + at, valid = valid_tokens(p.lengths, b, p.L), tokens = p.chunks * kChunk;
  float strengths[8], reads[8], writes[8], stays[8];
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {   // (all at once: a loop that adds as it loads takes a memory's latency for each)
    const size_t part = (size_t)bh * p.parts + (i < p.parts ? i : p.parts - 1);
    strengths[i] = p.strength[part * tokens + t];
    reads[i] = p.read[part * tokens + t] - p.along[part * tokens + t];
    writes[i] = p.write[part * tokens + t];
    stays[i] = p.stay[part * tokens + t];
  }
  const float past = p.past[(size_t)bh * tokens + t];
  float strength = 0.0f, read = 0.0f, write = 0.0f, stay = 0.0f;
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    if (i >= p.parts) break;
    strength += strengths[i];
    read += reads[i];
    write += writes[i];
    stay += stays[i];
  }
  // (a chunk is written whole or, behind the sequence's end, not at all)
  float written = __shfl_up(write, 1, 32);   // of the tokens before
  if (at == 0) written = 0.0f;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const float later = __shfl_down(read, d, 32), before = __shfl_up(written, d, 32);
    if (at + d < 32) read += later;
    if (at >= (uint32_t)d) written += before;
    stay += __shfl_xor(stay, d, 32);
  }
  if (t >= p.L || place >= all) return;
  float* const dg = const_cast<float*>(p.dlog_decay.d) + (int64_t)b * p.dlog_decay.batch + (int64_t)t * p.dlog_decay.token + (int64_t)h * p.dlog_decay.head;
  float* const db = const_cast<float*>(p.dbeta.d) + (int64_t)b * p.dbeta.batch + (int64_t)t * p.dbeta.token + (int64_t)h * p.dbeta.head;
  *dg = t < valid ? (past + read) + (written + stay) : 0.0f;
  *db = t < valid ? strength : 0.0f;
}

// Rows of heads that share one, added up in the heads' order: from [sequence and head][token][stride] in fp32.
struct DeltaFold {
  const float* from;
  SeqRows to;
  uint32_t n, width, stride, blocks;
};
template <typename T>
__device__ __forceinline__ void fold_of(const DeltaFold& f, const DeltaGates& p, uint32_t block) {
  const uint32_t lanes = (f.width + 3) / 4, per = 256 / lanes, at = threadIdx.x / lanes, col = threadIdx.x % lanes * 4, share = p.H / f.n;
  if (at >= per) return;
  const uint64_t rows = (uint64_t)(p.rows / p.H) * p.L * f.n;
  for (uint64_t row = (uint64_t)block * per + at; row < rows; row += (uint64_t)f.blocks * per) {
    const uint32_t i = (uint32_t)(row % f.n);
    const uint64_t tok = row / f.n;
    const uint32_t b = (uint32_t)(tok / p.L), t = (uint32_t)(tok % p.L);
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (t < valid_tokens(p.lengths, b, p.L))
      for (uint32_t s = 0; s < share; ++s)
        sum += load_four<float>(f.from + (((size_t)b * p.H + i * share + s) * p.chunks * kChunk + t) * f.stride, f.stride % 4 == 0, col, f.width);
    store_four<T>(row_to<T>(f.to, b, t, i), f.to.wide, col, f.width, sum);
  }
}

// What is left of a gradient when its rows are there, in one launch (each by itself took 6 us of 32 sequences of 512 tokens, 3 of them a launch's).
struct DeltaFinish {
  DeltaGates gates;
  uint32_t gate_blocks;
  DeltaFold fold[3];   // of queries, keys and values; blocks 0: there is nothing to add up
};
template <typename T>
__global__ __launch_bounds__(256) void k_delta_finish(DeltaFinish p) {
  uint32_t block = blockIdx.x;
  if (block < p.gate_blocks) return gates_of(p.gates, block);
  block -= p.gate_blocks;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (block < p.fold[i].blocks) return fold_of<T>(p.fold[i], p.gates, block);
    block -= p.fold[i].blocks;
  }
}
