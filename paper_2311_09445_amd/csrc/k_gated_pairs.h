// The gated delta rule within a chunk: what its tokens make of each other.  Part of seq_delta.hip (included inside namespace per).
//
// With G the sums of the decays' logarithms up to each of the 32 tokens, e_ij = exp(G_i - G_j) and
//   N_ij = e_ij k_i.k_j (i > j),   M_ij = scale e_ij q_i.k_j (i >= j),
// the tokens write U = diag(beta) Y with Y = (1 + N diag(beta))^-1 (V - e^G K S), and read  scale e^G Q S + M U.  The inverse is what
// makes the tokens of a chunk independent of each other.  It does not depend on the state, so it is formed for all chunks at once: a wave
// takes one chunk, the products on the matrix cores straight from memory, the inverse by substitution, a column to a lane (the upper
// half of the wave forms (1 + diag(beta) N)^-1, which a gradient runs backwards through).
//
// What bounds it: 9 us for 768 chunks of 64 x 64 are loads' and LDS's latency and the substitution's chain (of 32 rows in one piece, with the
// rows asked for behind the sums of decays, 11); 32768 chunks of 128 take 167 us for 350 MB written and 670 read (rows that two heads share by both).  Registers for
// four waves to a SIMD would spill (300 us).
//
// What goes into the record of a chunk is laid out as the operands that the passes over the sequence take: places {4 g .. 4 g + 3, 16 + 4 g ..} of
// the inner dimension in lane 16 g + m, in three parts.

struct Gates {
  const float* d;
  int64_t batch, token, head;
  __device__ __forceinline__ float at(uint32_t b, uint32_t t, uint32_t h) const { return d[(int64_t)b * batch + (int64_t)t * token + (int64_t)h * head]; }
};

struct DeltaRecord {
  bf16x8 solve[3][2][64], pairs[3][2][64];   // (of a gradient, which has no outputs: the pairs transposed)
  float gamma[32], left[32], beta[32];   // e^G, e^(G at the end - G), strengths
  float kept[2];                         // what is left of a state over the chunk, as a number and what rounding it left
  float pad[30];
};
struct DeltaRecordBack {
  DeltaRecord of;
  bf16x8 solve_t[3][2][64];
};
template <bool BACK>
struct RecordOf { typedef DeltaRecord type; };
template <>
struct RecordOf<true> { typedef DeltaRecordBack type; };

struct DeltaPairs {
  SeqRows q, k;
  Gates log_decay, beta;
  const int32_t* lengths;
  void* records;
  uint32_t L, H, dk, chunks, items;
  float scale;
};

// Elements col .. col + 7 of a row as it has them; the operand that they are, zeros behind `width` and where the row is not `on`.  FAST: rows are
// made of pieces of 16 bytes.
template <typename T>
struct EightOf {
  typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T))));
  Vec v[sizeof(T) / 2];
};
template <typename T, bool FAST>
__device__ __forceinline__ void ask_eight(const T* row, uint32_t col, uint32_t width, EightOf<T>* o) {
  constexpr uint32_t W = 16 / sizeof(T);
#pragma unroll
  for (uint32_t i = 0; i < 8 / W; ++i) {
    if constexpr (FAST) {
      o->v[i] = *reinterpret_cast<const typename EightOf<T>::Vec*>(row + (col + W * i < width ? col + W * i : 0));
    } else {
#pragma unroll
      for (uint32_t e = 0; e < W; ++e) o->v[i][e] = row[col + W * i + e < width ? col + W * i + e : 0];
    }
  }
}
template <typename T>
__device__ __forceinline__ Operand<T> operand_of_eight(const EightOf<T>& x, bool on, uint32_t col, uint32_t width) {
  constexpr uint32_t W = 16 / sizeof(T);
  T y[8];
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e) y[e] = on && col + e < width ? x.v[e / W][e % W] : T(0.0f);
  if constexpr (sizeof(T) == 2) {
    Operand<T> o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o.v[0][e] = y[e];
    return o;
  } else {
    return Operand<T>::of(f32x4{y[0], y[1], y[2], y[3]}, f32x4{y[4], y[5], y[6], y[7]});
  }
}

// Sums of the logarithms up to each token of a chunk, in 64 bits: differences of far sums keep what a slow decay adds.  A decay that keeps
// nothing in fp32 anyway (e^-104) counts as e^-10000, so that differences stay numbers.
__device__ __forceinline__ double decay_sums(const Gates& log_decay, uint32_t b, uint32_t h, uint32_t t, bool on, uint32_t lane) {
  float x = on ? log_decay.at(b, t, h) : 0.0f;
  x = x < -1e4f ? -1e4f : x;
  double G = x;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const double before = __shfl_up(G, d);
    if ((lane & 31) >= (uint32_t)d) G += before;
  }
  return G;
}

constexpr uint32_t kPairRow = 36;   // floats of a row of 32 in LDS

// c + a b of 16 x 16 x 16 in fp32: four of the inner dimension's places 4 g .. to a lane.
__device__ __forceinline__ f32x4 mma_f32(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
  return c;
}

// LDS of a wave that takes a chunk.
struct PairLds {
  float a[32 * kPairRow], b[32 * kPairRow], beta[32];
  double g[32];
};
template <typename T, int DK, bool BACK, bool FAST>
__device__ __forceinline__ void pairs_of(const DeltaPairs& p, uint32_t item, uint32_t lane, PairLds* lds) {
  const uint32_t m = lane & 15, g = lane >> 4;
  const uint32_t chunk = item % p.chunks, bh = item / p.chunks, h = bh % p.H, b = bh / p.H;
  const uint32_t valid = valid_tokens(p.lengths, b, p.L), first = chunk * kChunk;
  if (first >= valid) return;
  typename RecordOf<BACK>::type* const whole = static_cast<typename RecordOf<BACK>::type*>(p.records) + item;
  DeltaRecord* const record = reinterpret_cast<DeltaRecord*>(whole);
  float *const A = lds->a, *const B = lds->b, *const beta = lds->beta;
  double* const G = lds->g;

  // all that comes from memory, before anything is waited for
  EightOf<T> qx[DK / 32][2], kx[DK / 32][2];
  bool on[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t t = first + 16 * i + m;
    on[i] = t < valid;
    const uint32_t at = on[i] ? t : valid - 1;
    const T *const qr = row_of<T>(p.q, b, at, h), *const kr = row_of<T>(p.k, b, at, h);
#pragma unroll
    for (int s = 0; s < DK / 32; ++s) {
      ask_eight<T, FAST>(kr, 32 * s + 8 * g, p.dk, &kx[s][i]);
      ask_eight<T, FAST>(qr, 32 * s + 8 * g, p.dk, &qx[s][i]);
    }
  }
  const uint32_t column = lane & 31;
  const bool here = first + column < valid;
  const float strength = here ? p.beta.at(b, first + column, h) : 0.0f;
  const double sum = decay_sums(p.log_decay, b, h, here ? first + column : first, here, lane);
  if (lane < 32) {
    G[lane] = sum;
    beta[lane] = strength;
  }
  f32x4 kk[3] = {}, qk[3] = {};
#pragma unroll
  for (int s = 0; s < DK / 32; ++s) {
    Operand<T> q[2], k[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      q[i] = operand_of_eight<T>(qx[s][i], on[i], 32 * s + 8 * g, p.dk);
      k[i] = operand_of_eight<T>(kx[s][i], on[i], 32 * s + 8 * g, p.dk);
    }
#pragma unroll
    for (int x = 0; x < 3; ++x) {   // tiles (0, 0), (1, 0), (1, 1)
      kk[x] = mma(k[x > 0].v, k[x > 1].v, kk[x]);
      qk[x] = mma(q[x > 0].v, k[x > 1].v, qk[x]);
    }
  }
  wave_sync();
  const double total = G[31];
  if (lane < 32) {
    record->gamma[lane] = expf((float)sum);
    record->left[lane] = expf((float)(total - sum));
    record->beta[lane] = strength;
  }
  if (lane == 0) {
    const double all = exp(total);
    record->kept[0] = (float)all;
    record->kept[1] = (float)(all - (double)(float)all);
  }
#pragma unroll
  for (int x = 0; x < 3; ++x) {
    const uint32_t row = 16 * (x > 0) + 4 * g, col = 16 * (x > 1) + m;
    const double Gj = G[col];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t i = row + r;
      const float e = expf((float)(G[i] - Gj));
      kk[x][r] = i > col ? e * kk[x][r] : 0.0f;
      qk[x][r] = i >= col ? p.scale * e * qk[x][r] : 0.0f;
      A[i * kPairRow + col] = kk[x][r];
      B[i * kPairRow + col] = qk[x][r];
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) B[(4 * g + r) * kPairRow + 16 + m] = 0.0f;
  wave_sync();
  constexpr int PAIR_PARTS = sizeof(T) == 2 ? 2 : 3;   // (as many as outputs in bfloat16 take)
  auto put = [&](bf16x8 (&to)[3][2][64], int tile, f32x4 a, f32x4 c, int parts = 3) {
    const Parts<3> o = Parts<3>::of(a, c);
#pragma unroll
    for (int t = 0; t < parts; ++t) to[t][tile][lane] = o.v[t];
  };
  auto put_rows = [&](bf16x8 (&to)[3][2][64], const float* from, int parts = 3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float* row = from + (16 * i + m) * kPairRow + 4 * g;
      put(to, i, *reinterpret_cast<const f32x4*>(row), *reinterpret_cast<const f32x4*>(row + 16), parts);
    }
  };
  if constexpr (BACK) {
    put(record->pairs, 0, qk[0], qk[1]);
    put(record->pairs, 1, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, qk[2]);
  } else {
    put_rows(record->pairs, B, PAIR_PARTS);
  }
  // The inverse of  1 + N diag(beta)  (upper half: 1 + diag(beta) N) by halves: of the two blocks on the diagonal by substitution, a column to a lane,
  // 16 lanes to a block; then the one below, -X11 A10 X00, by two products in fp32.
  const bool other = BACK && lane >= 32;
  const uint32_t corner = 16 * (g & 1);
  float x[16], w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int l = 0; l + 3 < i + 3; l += 4) {
      const f32x4 n = *reinterpret_cast<const f32x4*>(A + (corner + i) * kPairRow + corner + l);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (l + e < i) {
          if (e & 1) s1 = fmaf(n[e], w[l + e], s1);
          else s0 = fmaf(n[e], w[l + e], s0);
        }
    }
    const float all = s0 + s1, bi = beta[corner + i];
    x[i] = ((uint32_t)i == m ? 1.0f : 0.0f) - (other ? bi * all : all);
    w[i] = other ? x[i] : bi * x[i];
  }
  // N10 as an operand, before its place is written over
  const f32x4 below = *reinterpret_cast<const f32x4*>(A + (16 + m) * kPairRow + 4 * g);
  const f32x4 beta0 = *reinterpret_cast<const f32x4*>(beta + 4 * g);
  const float beta1 = beta[16 + m];
  wave_sync();
  float* const X = other ? B : A;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    X[(corner + i) * kPairRow + corner + m] = x[i];
    if (corner) X[i * kPairRow + 16 + m] = 0.0f;
  }
  wave_sync();
#pragma unroll
  for (int way = 0; way < (BACK ? 2 : 1); ++way) {
    float* const Y = way ? B : A;
    f32x4 upper, lower = *reinterpret_cast<const f32x4*>(Y + (16 + m) * kPairRow + 16 + 4 * g);
#pragma unroll
    for (int r = 0; r < 4; ++r) upper[r] = Y[(4 * g + r) * kPairRow + m];
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 inner = mma_f32(way ? beta1 * below : below * beta0, upper, zero);
    // (outputs: a row that is not finite would reach the rows before it, of which it is taken 0 times)
    if constexpr (!BACK)
#pragma unroll
      for (int r = 0; r < 4; ++r) inner[r] = inner[r] * 0.0f == 0.0f ? inner[r] : 0.0f;
    const f32x4 under = mma_f32(lower, inner, zero);
#pragma unroll
    for (int r = 0; r < 4; ++r) Y[(16 + 4 * g + r) * kPairRow + m] = -under[r];
  }
  wave_sync();
  put_rows(record->solve, A);
  if constexpr (BACK) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f32x4 a, c;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        a[r] = B[(4 * g + r) * kPairRow + 16 * j + m];
        c[r] = B[(16 + 4 * g + r) * kPairRow + 16 * j + m];
      }
      put(whole->solve_t, j, a, c);
    }
  }
}
template <typename T, int DK, bool BACK, bool FAST>
__global__ __launch_bounds__(256, 2) void k_delta_pairs(DeltaPairs p) {
  __shared__ __attribute__((aligned(16))) PairLds lds[4];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), item = blockIdx.x * 4 + wave;
  if (item < p.items) pairs_of<T, DK, BACK, FAST>(p, item, threadIdx.x & 63, &lds[wave]);
}
