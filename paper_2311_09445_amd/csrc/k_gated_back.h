// The gradient of the gated delta rule.  Part of seq_delta.hip (included inside namespace per).
//
// Against time, with R the gradient of the state behind a chunk,
//   dU = pairs^T dO + left K R,  du = (1 + diag(beta) N)^-T dU,  dV = dZ = beta du,  dbeta = Y . du,
//   R <- e^Gn R + Q^T (scale e^G dO) - K^T (e^G dZ),
// in columns that do not meet, as over time (k_delta_back).  What is left does not depend on the order of the chunks (k_delta_grads):
//   dQ = scale e^G dO S^T + dM K,   dK = -e^G dZ S^T + left U R^T + dM^T Q + (dN + dN^T) K,
//   dM = scale e_ij dO U^T (i >= j),   dN = -e_ij dZ U^T (i > j).
// The gradient of a decay's logarithm is that of the state before the token times the state itself.  At the first token of a chunk that is
// <R, S>; from one token to the next it falls by out . dO - dZ . V, which is added up within a chunk only.

struct DeltaBack {
  SeqRows q, k, v, dout, dv;
  const void* records;
  const int32_t* lengths;
  const float* in;
  float* to;
  int64_t in_batch, in_head, to_batch, to_head;
  uint32_t L, H, dk, dvw, chunks, slices;
  float scale;
  uint32_t direct;               // dV goes to its rows (no heads share them)
  const bf16* states;
  const float* y;
  bf16* dstates;                 // the gradients of the states behind the chunks
  float *dz, *along, *strength, *border;
};

template <typename T>
constexpr int kGradParts = sizeof(T) == 2 ? 1 : 3;   // of states in the products for rows

template <typename T, int DK>
__global__ __launch_bounds__(256) void k_delta_back(DeltaBack p) {
  constexpr int TX = DK / 16, KX = DK / 32, PT = kParts<T>;
  constexpr uint32_t BUFFER = RunLds<T, DK, 3, false>::SIZE;
  extern __shared__ __attribute__((aligned(256))) uint8_t lds_raw[];
  bf16* const lds = reinterpret_cast<bf16*>(lds_raw);
  const uint32_t slice = blockIdx.x % p.slices, bh = blockIdx.x / p.slices, h = bh % p.H, b = bh / p.H;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const uint32_t L = p.L, dk = p.dk, dv = p.dvw, blocks = (dv + 31) / 32, col0 = 64 * slice + 16 * wave, col = col0 + m;
  const bool on = col < dv, works = col0 < blocks * 32;
  const uint32_t valid = valid_tokens(p.lengths, b, L), chunks = (valid + kChunk - 1) / kChunk, width = blocks * 32;
  const DeltaRecordBack* const records = static_cast<const DeltaRecordBack*>(p.records) + (size_t)bh * p.chunks;
  const bool pieces = p.q.near && p.k.near && dk >= 16 / sizeof(T);
  const size_t row0 = (size_t)bh * p.chunks * kChunk, part0 = ((size_t)bh * (blocks * 2) + col0 / 16) * p.chunks;

  f32x4 s[TX];
#pragma unroll
  for (int a = 0; a < TX; ++a)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t row = state_row(a, 4 * g + r);
      s[a][r] = p.in && on && row < dk ? p.in[(int64_t)b * p.in_batch + (int64_t)h * p.in_head + (size_t)row * dv + col] : 0.0f;
    }
  const T *const q0 = row_of<T>(p.q, b, 0, h), *const k0 = row_of<T>(p.k, b, 0, h), *const v0 = row_of<T>(p.v, b, 0, h), *const d0 = row_of<T>(p.dout, b, 0, h);
  TwoRows<T, DK> rows;
  if (chunks) {
    rows.load(p.q, p.k, q0, k0, (chunks - 1) * kChunk, valid, dk, pieces);
    rows.store(lds + ((chunks - 1) & 1) * BUFFER, valid - (chunks - 1) * kChunk, dk, pieces);
    if (chunks > 1) rows.load(p.q, p.k, q0, k0, (chunks - 2) * kChunk, valid, dk, pieces);
    __syncthreads();
  }
  for (uint32_t left_chunks = chunks; left_chunks; --left_chunks) {
    const uint32_t c = left_chunks - 1, first = c * kChunk;
    bf16 *const Q = lds + (c & 1) * BUFFER, *const K = Q + PT * Tile<DK>::SIZE;
    if (c) {
      rows.store(lds + ((c - 1) & 1) * BUFFER, kChunk, dk, pieces);
      if (c > 1) rows.load(p.q, p.k, q0, k0, first - 2 * kChunk, valid, dk, pieces);
    }
    if (works) {
      RecordRows<3> rec;
      RecordNumbers num;
      rec.load(&records[c].solve_t[0][0][0], &records[c].pairs_t[0][0][0], lane);
      num.load(&records[c].of, m, g);
      f32x4 v[2], d[2], y[2], w[2] = {};
      load_column<T>(p.v, v0, first, valid, on, col, g, v);
      load_column<T>(p.dout, d0, first, valid, on, col, g, d);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) y[i][r] = p.y[(row0 + first + 16 * i + 4 * g + r) * width + col];
#pragma unroll
      for (int k = 0; k < KX; ++k) {
        const Parts<3> sp = Parts<3>::of(s[2 * k], s[2 * k + 1]);
        bf16* to = p.dstates + state_at<DK>(bh, p.chunks, c, dv, kGradParts<T>) + (size_t)(col0 / 32) * Tile<DK>::SIZE + Tile<DK>::at(col0 % 32 + m, 4 * k + g);
#pragma unroll
        for (int t = 0; t < kGradParts<T>; ++t) *reinterpret_cast<bf16x8*>(to + (size_t)t * blocks * Tile<DK>::SIZE) = sp.v[t];
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = mma(Operand<T>::template along<DK>(K, 16 * i + m, k, g).v, sp.v, w[i]);
      }
      const Operand<T> dp = operand_of<T>(d);
      f32x4 du[2], dz[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) w[i] = mma(rec.pairs[i], dp.v, num.left[i] * w[i]);
      const Parts<3> wp = Parts<3>::of(w[0], w[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        du[i] = mma(rec.solve[i], wp.v, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
        dz[i] = num.beta[i] * du[i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t t = first + 16 * i + 4 * g + r;
          p.dz[(row0 + t) * width + col] = dz[i][r];
          if (p.direct && on && t < L) row_to<T>(p.dv, b, t, h)[col] = (T)(t < valid ? dz[i][r] : 0.0f);
          const float along = sum16(dz[i][r] * v[i][r]), strength = sum16(y[i][r] * du[i][r]);
          if (m == 0) {
            p.along[part0 * kChunk + t] -= along;
            p.strength[part0 * kChunk + t] = strength;
          }
        }
      f32x4 into[2], outof[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        into[i] = p.scale * num.gamma[i] * d[i];
        outof[i] = -num.gamma[i] * dz[i];
      }
      const Parts<3> ip = Parts<3>::of(into[0], into[1]), op = Parts<3>::of(outof[0], outof[1]);
      float border = 0.0f;
#pragma unroll
      for (int k = 0; k < KX; ++k) {
#pragma unroll
        for (int a = 2 * k; a < 2 * k + 2; ++a) {
          s[a] = num.keep(s[a]);
          auto column = [&](uint32_t i) { return state_row(a, i); };
          s[a] = mma(Operand<T>::template across<DK>(Q, column, m, g).v, ip.v, s[a]);
          s[a] = mma(Operand<T>::template across<DK>(K, column, m, g).v, op.v, s[a]);
        }
        const bf16* from = p.states + state_at<DK>(bh, p.chunks, c, dv, kStateParts<T>) + (size_t)(col0 / 32) * Tile<DK>::SIZE + Tile<DK>::at(col0 % 32 + m, 4 * k + g);
        f32x4 before[2] = {};
        bf16x8 x[kStateParts<T>];
#pragma unroll
        for (int t = 0; t < kStateParts<T>; ++t) x[t] = *reinterpret_cast<const bf16x8*>(from + (size_t)t * blocks * Tile<DK>::SIZE);
        if constexpr (sizeof(T) == 2) {
          of_halves(x, &before[0], &before[1]);
        } else {
#pragma unroll
          for (int t = 2; t >= 0; --t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              before[0][e] += (float)x[t][e];
              before[1][e] += (float)x[t][e + 4];
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) border = fmaf(before[0][e], s[2 * k][e], fmaf(before[1][e], s[2 * k + 1][e], border));
      }
      border = sum16(border);
      border += __shfl_xor(border, 16);
      border += __shfl_xor(border, 32);
      if (lane == 0) p.border[part0 + c] = border;
    }
    __syncthreads();
  }
  if (p.direct && works)
    for (uint32_t t = chunks * kChunk + m; t < L; t += 16) store_four<T>(row_to<T>(p.dv, b, t, h), p.dv.wide, col0 + 4 * g, dv, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
  if (p.to && on)
#pragma unroll
    for (int a = 0; a < TX; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t row = state_row(a, 4 * g + r);
        if (row < dk) p.to[(int64_t)b * p.to_batch + (int64_t)h * p.to_head + (size_t)row * dv + col] = s[a][r];
      }
}

struct DeltaGrads {
  SeqRows q, k, dout, dq, dk;
  Gates log_decay, beta, dlog_decay, dbeta;
  const int32_t* lengths;
  uint32_t L, H, dkw, dv, chunks;
  float scale;
  uint32_t direct_q, direct_k;   // to their rows; else to fold_q, fold_k, [sequence and head][token][dk] in fp32
  float *fold_q, *fold_k;
  const bf16 *states, *dstates;
  const float *y, *dz, *along, *strength, *border;
};

template <typename T, int DK>
constexpr uint32_t grads_lds() { return (2 * kParts<T> + 2 * kGradParts<T>) * Tile<DK>::SIZE * sizeof(bf16) + 2 * 32 * kPairRow * sizeof(float); }

// Places {4 g .., 16 + 4 g ..} of a row's 32 from column `col`.
template <typename T>
__device__ __forceinline__ Operand<T> row_places(const T* row, bool on, bool wide, uint32_t col, uint32_t g, uint32_t width) {
  f32x4 a = {}, c = {};
  if (on) {
    a = load_four<T>(row, wide, col + 4 * g, width);
    c = load_four<T>(row, wide, col + 16 + 4 * g, width);
  }
  return Operand<T>::of(a, c);
}

// A workgroup takes a chunk; its waves share the chunk's columns of dk, and the four 16 x 16 tiles of its pairs.
template <typename T, int DK>
__global__ __launch_bounds__(256) void k_delta_grads(DeltaGrads p) {
  constexpr int NC = DK / 64, PT = kParts<T>, PS = kGradParts<T>, PU = sizeof(T) == 2 ? 2 : 3, LESS = PU - 1;
  extern __shared__ __attribute__((aligned(256))) uint8_t lds_raw[];
  bf16* const Q = reinterpret_cast<bf16*>(lds_raw);
  bf16* const K = Q + PT * Tile<DK>::SIZE;
  bf16* const S = K + PT * Tile<DK>::SIZE;
  bf16* const R = S + PS * Tile<DK>::SIZE;
  float* const dM = reinterpret_cast<float*>(R + PS * Tile<DK>::SIZE);
  float* const dN = dM + 32 * kPairRow;
  __shared__ double G[32];
  __shared__ __attribute__((aligned(16))) float gamma[32], left[32], beta[32];
  const uint32_t chunk = blockIdx.x % p.chunks, bh = blockIdx.x / p.chunks, h = bh % p.H, b = bh / p.H;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const uint32_t L = p.L, dk = p.dkw, dv = p.dv, blocks = (dv + 31) / 32, width = blocks * 32, parts = blocks * 2;
  const uint32_t valid = valid_tokens(p.lengths, b, L), first = chunk * kChunk, end = L - first < kChunk ? L - first : kChunk;
  const size_t row0 = (size_t)bh * p.chunks * kChunk + first;
  auto to_gate = [&](const Gates& x, uint32_t t) { return const_cast<float*>(x.d) + (int64_t)b * x.batch + (int64_t)t * x.token + (int64_t)h * x.head; };
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  if (first >= valid) {
    for (uint32_t i = threadIdx.x; i < end * ((dk + 3) / 4); i += 256) {
      const uint32_t t = first + i / ((dk + 3) / 4), col = i % ((dk + 3) / 4) * 4;
      if (p.direct_q) store_four<T>(row_to<T>(p.dq, b, t, h), p.dq.wide, col, dk, zero);
      if (p.direct_k) store_four<T>(row_to<T>(p.dk, b, t, h), p.dk.wide, col, dk, zero);
    }
    if (threadIdx.x < end) {
      *to_gate(p.dlog_decay, first + threadIdx.x) = 0.0f;
      *to_gate(p.dbeta, first + threadIdx.x) = 0.0f;
    }
    return;
  }
  const uint32_t n = valid - first;   // (and more)
  {
    TwoRows<T, DK> rows;
    const bool pieces = p.q.near && p.k.near && dk >= 16 / sizeof(T);
    rows.load(p.q, p.k, row_of<T>(p.q, b, 0, h), row_of<T>(p.k, b, 0, h), first, valid, dk, pieces);
    rows.store(Q, n, dk, pieces);
  }
  if (wave == 0) {
    const uint32_t column = lane & 31;
    const bool here = column < n;
    const double sum = decay_sums(p.log_decay, b, h, here ? first + column : first, here, lane);
    const double total = __shfl(sum, 31);
    if (lane < 32) {
      G[lane] = sum;
      gamma[lane] = expf((float)sum);
      left[lane] = expf((float)(total - sum));
      beta[lane] = here ? p.beta.at(b, first + lane, h) : 0.0f;
    }
  } else if (wave == 1) {
    const uint32_t column = lane & 31;
    float strength = 0.0f, along = 0.0f, border = 0.0f;
    for (uint32_t i = 0; i < parts; ++i) {
      const size_t at = (size_t)bh * parts + i;
      strength += p.strength[at * p.chunks * kChunk + first + column];
      along += p.along[at * p.chunks * kChunk + first + column];
      border += p.border[at * p.chunks + chunk];
    }
    float before = along;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const float x = __shfl_up(before, d);
      if (column >= (uint32_t)d) before += x;
    }
    before = __shfl_up(before, 1);
    if (lane < end) {
      *to_gate(p.dlog_decay, first + lane) = lane >= n ? 0.0f : lane ? border - before : border;
      *to_gate(p.dbeta, first + lane) = lane < n ? strength : 0.0f;
    }
  }
  __syncthreads();
  f32x4 aq[2][NC] = {}, ak[2][NC] = {}, dm = zero, dn = zero;
  const uint32_t ti = wave >> 1, tj = wave & 1;
  const size_t from_s = state_at<DK>(bh, p.chunks, chunk, dv, kStateParts<T>), from_r = state_at<DK>(bh, p.chunks, chunk, dv, PS);
  for (uint32_t block = 0; block < blocks; ++block) {
    if (block) __syncthreads();
#pragma unroll
    for (int t = 0; t < PS; ++t)
      for (uint32_t i = threadIdx.x; i < Tile<DK>::SIZE / 8; i += 256) {
        *reinterpret_cast<bf16x8*>(S + t * Tile<DK>::SIZE + 8 * i) = *reinterpret_cast<const bf16x8*>(p.states + from_s + ((size_t)t * blocks + block) * Tile<DK>::SIZE + 8 * i);
        *reinterpret_cast<bf16x8*>(R + t * Tile<DK>::SIZE + 8 * i) = *reinterpret_cast<const bf16x8*>(p.dstates + from_r + ((size_t)t * blocks + block) * Tile<DK>::SIZE + 8 * i);
      }
    Operand<T> d[2];
    Parts<PU> z[2], zs[2], u[2], ul[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t t = 16 * i + m;
      d[i] = row_places<T>(row_of<T>(p.dout, b, t < n ? first + t : first, h), t < n, p.dout.wide, 32 * block, g, dv);
      const float *zr = p.dz + (row0 + t) * width + 32 * block + 4 * g, *yr = p.y + (row0 + t) * width + 32 * block + 4 * g;
      const f32x4 z0 = *reinterpret_cast<const f32x4*>(zr), z1 = *reinterpret_cast<const f32x4*>(zr + 16);
      const f32x4 u0 = beta[t] * *reinterpret_cast<const f32x4*>(yr), u1 = beta[t] * *reinterpret_cast<const f32x4*>(yr + 16);
      z[i] = Parts<PU>::of(z0, z1);
      u[i] = Parts<PU>::of(u0, u1);
      zs[i] = Parts<PU>::of(-gamma[t] * z0, -gamma[t] * z1);
      ul[i] = Parts<PU>::of(left[t] * u0, left[t] * u1);
    }
    if (tj <= ti) {
      dm = mma<LESS>(ti ? d[1].v : d[0].v, tj ? u[1].v : u[0].v, dm);
      dn = mma<LESS>(ti ? z[1].v : z[0].v, tj ? u[1].v : u[0].v, dn);
    }
    __syncthreads();
#pragma unroll
    for (int a = 0; a < NC; ++a) {
      auto column = [&](uint32_t i) { return 16 * (wave * NC + a) + i; };
      bf16x8 s[PS], r[PS];
#pragma unroll
      for (int t = 0; t < PS; ++t) {
        s[t] = Operand<bf16>::template across<DK>(S + t * Tile<DK>::SIZE, column, m, g).v[0];
        r[t] = Operand<bf16>::template across<DK>(R + t * Tile<DK>::SIZE, column, m, g).v[0];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        aq[i][a] = mma<LESS>(s, d[i].v, aq[i][a]);
        ak[i][a] = mma<LESS>(s, zs[i].v, ak[i][a]);
        ak[i][a] = mma<LESS>(r, ul[i].v, ak[i][a]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t i = 16 * ti + 4 * g + e, j = 16 * tj + m;
    const float x = expf((float)(G[i] - G[j]));
    dM[i * kPairRow + j] = i >= j ? p.scale * x * dm[e] : 0.0f;
    dN[i * kPairRow + j] = i > j ? -x * dn[e] : 0.0f;
  }
  __syncthreads();
  Parts<PU> rows_m[2], cols_m[2], both_n[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t t = 16 * i + m;
    f32x4 a, c, e, f;
    const f32x4 na = *reinterpret_cast<const f32x4*>(dN + t * kPairRow + 4 * g), nc = *reinterpret_cast<const f32x4*>(dN + t * kPairRow + 16 + 4 * g);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      a[r] = dM[(4 * g + r) * kPairRow + t];
      c[r] = dM[(16 + 4 * g + r) * kPairRow + t];
      e[r] = dN[(4 * g + r) * kPairRow + t];
      f[r] = dN[(16 + 4 * g + r) * kPairRow + t];
    }
    rows_m[i] = Parts<PU>::of(*reinterpret_cast<const f32x4*>(dM + t * kPairRow + 4 * g), *reinterpret_cast<const f32x4*>(dM + t * kPairRow + 16 + 4 * g));
    cols_m[i] = Parts<PU>::of(a, c);
    both_n[i] = Parts<PU>::of(na + e, nc + f);
  }
#pragma unroll
  for (int a = 0; a < NC; ++a) {
    const uint32_t tile = wave * NC + a;
    auto column = [&](uint32_t i) { return 16 * tile + i; };
    const Operand<T> q = Operand<T>::template across<DK>(Q, column, m, g), k = Operand<T>::template across<DK>(K, column, m, g);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t t = 16 * i + m, col = 16 * tile + 4 * g;
      aq[i][a] *= p.scale * gamma[t];
      aq[i][a] = mma<LESS>(k.v, rows_m[i].v, aq[i][a]);
      ak[i][a] = mma<LESS>(q.v, cols_m[i].v, ak[i][a]);
      ak[i][a] = mma<LESS>(k.v, both_n[i].v, ak[i][a]);
      if (t >= end) continue;
      if (t >= n) aq[i][a] = ak[i][a] = zero;
      if (p.direct_q) store_four<T>(row_to<T>(p.dq, b, first + t, h), p.dq.wide, col, dk, aq[i][a]);
      else store_four<float>(p.fold_q + (row0 + t) * dk, dk % 4 == 0, col, dk, aq[i][a]);
      if (p.direct_k) store_four<T>(row_to<T>(p.dk, b, first + t, h), p.dk.wide, col, dk, ak[i][a]);
      else store_four<float>(p.fold_k + (row0 + t) * dk, dk % 4 == 0, col, dk, ak[i][a]);
    }
  }
}

// Rows of heads that share one, added up in the heads' order: from [sequence and head][token][stride] in fp32.
struct DeltaFold {
  const float* from;
  SeqRows to;
  const int32_t* lengths;
  uint64_t rows;   // B L n
  uint32_t L, H, n, width, stride, tokens;
};
template <typename T>
__global__ __launch_bounds__(256) void k_delta_fold(DeltaFold f) {
  const uint32_t lanes = (f.width + 3) / 4, per = 256 / lanes, at = threadIdx.x / lanes, col = threadIdx.x % lanes * 4, share = f.H / f.n;
  if (at >= per) return;
  for (uint64_t row = (uint64_t)blockIdx.x * per + at; row < f.rows; row += (uint64_t)gridDim.x * per) {
    const uint32_t i = (uint32_t)(row % f.n);
    const uint64_t tok = row / f.n;
    const uint32_t b = (uint32_t)(tok / f.L), t = (uint32_t)(tok % f.L);
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (t < valid_tokens(f.lengths, b, f.L))
      for (uint32_t s = 0; s < share; ++s)
        sum += load_four<float>(f.from + (((size_t)b * f.H + i * share + s) * f.tokens + t) * f.stride, f.stride % 4 == 0, col, f.width);
    store_four<T>(row_to<T>(f.to, b, t, i), f.to.wide, col, f.width, sum);
  }
}
