// The gated delta rule over sequences.  Part of seq_delta.hip (included inside namespace per).
//
// With the record of a chunk (k_gated_pairs.h) and S the state before it,
//   Z = V - e^G K S,  Y = solve Z,  U = diag(beta) Y,  out = scale e^G Q S + pairs U,  S <- e^Gn S + K^T (left U).
// The columns of the state do not meet, so a wave holds 16 of them for all of dk in registers and goes over the whole sequence; four
// waves share the rows of queries and keys in LDS.  The result of one product is the operand of the next: rows of Z, Y and U are
// tokens, which the next product runs over.  The outputs are formed transposed, so that a lane has four neighbours of a token.
//
// Whatever is computed is taken apart into three parts in bfloat16 where it becomes an operand, since the state is fp32 and what is
// written to it comes out of the state: 24 bits.  What only the outputs see keeps 16 bits of itself where these are bfloat16.

struct DeltaRun {
  SeqRows q, k, v, out, dout;
  const void* records;
  const int32_t* lengths;
  const float* in;
  float* to;
  int64_t in_batch, in_head, to_batch, to_head;
  uint32_t L, H, dk, dv, chunks, slices;
  float scale;
  // kept for a gradient: the states before the chunks, Y, rows of out . dout
  bf16* states;
  float *y, *along;
};

enum DeltaMode { FORWARD, KEEPING };

// Planes of 16 bits that states are kept in for a gradient: where rows are bfloat16 the rounded state, which the products for bfloat16 gradients
// take, and the lower half of the sum that rounded it, so that both together are the 32 bits (two rounded parts held 17, and the decays'
// gradient was off by 2e-6 of itself); else the three parts that an operand takes.
template <typename T>
constexpr int kStateParts = sizeof(T) == 2 ? 2 : 3;

// Where the states kept for chunk c of a sequence and head start: [part][32 columns of dv][Tile of dk], columns as rows.
template <int DK>
__device__ __forceinline__ size_t state_at(uint32_t bh, uint32_t chunks, uint32_t c, uint32_t dv, uint32_t parts) {
  return ((size_t)bh * chunks + c) * parts * ((dv + 31) / 32) * Tile<DK>::SIZE;
}

template <int N>
struct RecordRows {   // what a pass takes of a record, in registers
  bf16x8 solve[2][3], pairs[2][N];
  f32x4 gamma[2], left[2], beta[2];
  Keep keep;
  __device__ __forceinline__ void load(const DeltaRecord* r, const bf16x8 (&s)[3][2][64], const bf16x8 (&p)[3][2][64], uint32_t lane, uint32_t g) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int t = 0; t < 3; ++t) solve[i][t] = s[t][i][lane];
#pragma unroll
      for (int t = 0; t < N; ++t) pairs[i][t] = p[t][i][lane];
      gamma[i] = *reinterpret_cast<const f32x4*>(r->gamma + 16 * i + 4 * g);
      left[i] = *reinterpret_cast<const f32x4*>(r->left + 16 * i + 4 * g);
      beta[i] = *reinterpret_cast<const f32x4*>(r->beta + 16 * i + 4 * g);
    }
    keep = r->keep;
  }
};

struct Halves { bf16x8 v[2]; };
__device__ __forceinline__ Halves halves_of(f32x4 a, f32x4 b) {
  u32x4 upper, lower;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t x[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float f = i < 2 ? a[2 * i + e] : b[2 * i + e - 4];
      x[e] = (f != f ? 0x7FC00000u : __builtin_bit_cast(uint32_t, f)) + 0x8000u;   // (any other NaN could become a number)
    }
    upper[i] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);
    lower[i] = __builtin_amdgcn_perm(x[1], x[0], 0x05040100u);
  }
  return Halves{{__builtin_bit_cast(bf16x8, upper), __builtin_bit_cast(bf16x8, lower)}};
}
__device__ __forceinline__ void of_halves(const bf16x8 (&h)[2], f32x4* a, f32x4* b) {
  const u32x4 upper = __builtin_bit_cast(u32x4, h[0]), lower = __builtin_bit_cast(u32x4, h[1]);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t x = __builtin_amdgcn_perm(upper[i], lower[i], e ? 0x07060302u : 0x05040100u) - 0x8000u;
      if (i < 2) (*a)[2 * i + e] = __builtin_bit_cast(float, x);
      else (*b)[2 * i + e - 4] = __builtin_bit_cast(float, x);
    }
}

// Rows 16 i + 4 g + r of a chunk, column col, as fp32.
template <typename T>
__device__ __forceinline__ void load_column(const SeqRows& rows, const T* head, uint32_t first, uint32_t valid, bool on, uint32_t col, uint32_t g, f32x4 (&v)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t t = first + 16 * i + 4 * g + r;
      const T x = head[(int64_t)(t < valid ? t : valid - 1) * rows.token + (on ? col : 0)];
      v[i][r] = on && t < valid ? as_float(x) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ Operand<T> operand_of(const f32x4 (&v)[2]) { return Operand<T>::of(v[0], v[1]); }

// Four neighbours of a row, from column col of `width`.
template <typename T>
__device__ __forceinline__ f32x4 load_four(const T* row, bool wide, uint32_t col, uint32_t width) {
  typedef T Vec __attribute__((ext_vector_type(4)));
  f32x4 o = {};
  if (wide && col + 4 <= width) {
    const Vec v = *reinterpret_cast<const Vec*>(row + col);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = as_float(v[i]);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      if (col + i < width) o[i] = as_float(row[col + i]);
  }
  return o;
}
template <typename T>
__device__ __forceinline__ void store_four(T* row, bool wide, uint32_t col, uint32_t width, f32x4 v) {
  typedef T Vec __attribute__((ext_vector_type(4)));
  if (wide && col + 4 <= width) {
    Vec o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (T)v[i];
    *reinterpret_cast<Vec*>(row + col) = o;
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      if (col + i < width) row[col + i] = (T)v[i];
  }
}

// Rows of queries and keys on their way to LDS.
template <typename T, int DK>
struct TwoRows {
  Staged<T, DK, 256> q, k;
  __device__ __forceinline__ void load(const SeqRows& rq, const SeqRows& rk, const T* q0, const T* k0, uint32_t first, uint32_t valid, uint32_t dk, bool pieces) {
    if (pieces) {
      q.load_pieces(rq, q0, first, valid, valid, false, 0, dk);
      k.load_pieces(rk, k0, first, valid, valid, false, 0, dk);
    } else {
      q.load(rq, q0, first, valid - first, valid, false, 0, dk);
      k.load(rk, k0, first, valid - first, valid, false, 0, dk);
    }
  }
  __device__ __forceinline__ void store(bf16* lds, uint32_t n, uint32_t dk, bool pieces) {
    constexpr uint32_t W = 16 / sizeof(T);
    bf16 *const to_q = lds, *const to_k = lds + kParts<T> * Tile<DK>::SIZE;
    if (pieces) {
      q.clear(n, 0, dk);
      k.clear(n, 0, dk);
    }
    q.store(to_q);
    k.store(to_k);
    if (pieces && dk % W) {
      q.store_ends(to_q, dk);
      k.store_ends(to_k, dk);
    }
  }
};

template <typename T, int DK>
constexpr uint32_t run_lds() { return 2 * 2 * kParts<T> * Tile<DK>::SIZE * sizeof(bf16); }

template <typename T, int DK, DeltaMode MODE>
__global__ __launch_bounds__(256) void k_delta_run(DeltaRun p) {
  constexpr int TX = DK / 16, KX = DK / 32, PT = kParts<T>, LESS = sizeof(T) == 2 && MODE == FORWARD ? 1 : 2, NP = LESS + 1;
  constexpr uint32_t BUFFER = 2 * PT * Tile<DK>::SIZE;
  extern __shared__ __attribute__((aligned(256))) uint8_t lds_raw[];
  bf16* const lds = reinterpret_cast<bf16*>(lds_raw);
  const uint32_t slice = blockIdx.x % p.slices, bh = blockIdx.x / p.slices, h = bh % p.H, b = bh / p.H;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const uint32_t L = p.L, dk = p.dk, dv = p.dv, col0 = 64 * slice + 16 * wave, col = col0 + m;
  const bool on = col < dv, works = col0 < (dv + 31) / 32 * 32;
  const uint32_t valid = valid_tokens(p.lengths, b, L), chunks = (valid + kChunk - 1) / kChunk;
  typedef typename RecordOf<MODE == KEEPING>::type Record;
  const Record* const records = static_cast<const Record*>(p.records) + (size_t)bh * p.chunks;
  const bool pieces = p.q.near && p.k.near && dk >= 16 / sizeof(T);

  f32x4 s[TX];
#pragma unroll
  for (int a = 0; a < TX; ++a)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t row = state_row(a, 4 * g + r);
      s[a][r] = p.in && on && row < dk ? p.in[(int64_t)b * p.in_batch + (int64_t)h * p.in_head + (size_t)row * dv + col] : 0.0f;
    }
  const T *const q0 = row_of<T>(p.q, b, 0, h), *const k0 = row_of<T>(p.k, b, 0, h), *const v0 = row_of<T>(p.v, b, 0, h);
  TwoRows<T, DK> rows;
  RecordRows<NP> rec, next;
  f32x4 v[2], next_v[2];
  auto load_record = [&](uint32_t c, RecordRows<NP>* to) {
    const DeltaRecord* r = reinterpret_cast<const DeltaRecord*>(records + c);
    to->load(r, r->solve, r->pairs, lane, g);
  };
  if (chunks) {
    rows.load(p.q, p.k, q0, k0, 0, valid, dk, pieces);
    load_record(0, &next);
    load_column<T>(p.v, v0, 0, valid, on, col, g, next_v);
    rows.store(lds, valid, dk, pieces);
    if (chunks > 1) rows.load(p.q, p.k, q0, k0, kChunk, valid, dk, pieces);
    __syncthreads();
  }
  for (uint32_t c = 0; c < chunks; ++c) {
    const uint32_t first = c * kChunk;
    bf16 *const Q = lds + (c & 1) * BUFFER, *const K = Q + PT * Tile<DK>::SIZE;
    rec = next;
    v[0] = next_v[0];
    v[1] = next_v[1];
    if (c + 1 < chunks) {
      rows.store(lds + ((c + 1) & 1) * BUFFER, valid - first - kChunk, dk, pieces);
      if (c + 2 < chunks) rows.load(p.q, p.k, q0, k0, first + 2 * kChunk, valid, dk, pieces);
      load_record(c + 1, &next);
      load_column<T>(p.v, v0, first + kChunk, valid, on, col, g, next_v);
    }
    if (works) {
      f32x4 x[2] = {}, o[2] = {};
#pragma unroll
      for (int k = 0; k < KX; ++k) {
        const Parts<3> sp = Parts<3>::of(s[2 * k], s[2 * k + 1]);
        if constexpr (MODE == KEEPING) {
          bf16* to = p.states + state_at<DK>(bh, p.chunks, c, dv, kStateParts<T>) + (size_t)(col0 / 32) * Tile<DK>::SIZE + Tile<DK>::at(col0 % 32 + m, 4 * k + g);
          if constexpr (sizeof(T) == 2) {
            const Halves both = halves_of(s[2 * k], s[2 * k + 1]);
#pragma unroll
            for (int t = 0; t < 2; ++t) *reinterpret_cast<bf16x8*>(to + (size_t)t * ((dv + 31) / 32) * Tile<DK>::SIZE) = both.v[t];
          } else {
#pragma unroll
            for (int t = 0; t < 3; ++t) *reinterpret_cast<bf16x8*>(to + (size_t)t * ((dv + 31) / 32) * Tile<DK>::SIZE) = sp.v[t];
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          x[i] = mma(Operand<T>::template along<DK>(K, 16 * i + m, k, g).v, sp.v, x[i]);
          o[i] = mma<LESS>(sp.v, Operand<T>::template along<DK>(Q, 16 * i + m, k, g).v, o[i]);
        }
      }
      const Parts<3> z = Parts<3>::of(v[0] - rec.gamma[0] * x[0], v[1] - rec.gamma[1] * x[1]);
      f32x4 y[2], u[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        y[i] = mma(rec.solve[i], z.v, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
        u[i] = rec.beta[i] * y[i];
      }
      const Parts<NP> up = Parts<NP>::of(u[0], u[1]);
      const DeltaRecord* r = reinterpret_cast<const DeltaRecord*>(records + c);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        o[i] *= p.scale * r->gamma[16 * i + m];
        o[i] = mma<LESS>(up.v, rec.pairs[i], o[i]);
      }
      if constexpr (MODE == KEEPING) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float* to = p.y + ((size_t)bh * p.chunks * kChunk + first + 16 * i + 4 * g) * ((dv + 31) / 32 * 32) + col;
#pragma unroll
          for (int e = 0; e < 4; ++e) to[(size_t)e * ((dv + 31) / 32 * 32)] = y[i][e];
          const uint32_t t = first + 16 * i + m;
          float dot = 0.0f;
          if (t < valid) {
            const f32x4 d = load_four<T>(row_of<T>(p.dout, b, t, h), p.dout.wide, col0 + 4 * g, dv);
#pragma unroll
            for (int e = 0; e < 4; ++e) dot = fmaf(d[e], o[i][e], dot);
          }
          dot += __shfl_xor(dot, 16);
          dot += __shfl_xor(dot, 32);
          if (g == 0) p.along[((size_t)bh * ((dv + 31) / 32 * 2) + col0 / 16) * p.chunks * kChunk + t] = dot;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t t = first + 16 * i + m;
          if (t < L) store_four<T>(row_to<T>(p.out, b, t, h), p.out.wide, col0 + 4 * g, dv, t < valid ? o[i] : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
        }
      }
      const Parts<3> w = Parts<3>::of(rec.left[0] * u[0], rec.left[1] * u[1]);
#pragma unroll
      for (int a = 0; a < TX; ++a) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[a][e] = kept(s[a][e], rec.keep);
        s[a] = mma(Operand<T>::template across<DK>(K, [&](uint32_t i) { return state_row(a, i); }, m, g).v, w.v, s[a]);
      }
    }
    __syncthreads();
  }
  if (MODE == FORWARD && works)
    for (uint32_t t = chunks * kChunk + m; t < L; t += 16) store_four<T>(row_to<T>(p.out, b, t, h), p.out.wide, col0 + 4 * g, dv, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
  if (p.to && on)
#pragma unroll
    for (int a = 0; a < TX; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t row = state_row(a, 4 * g + r);
        if (row < dk) p.to[(int64_t)b * p.to_batch + (int64_t)h * p.to_head + (size_t)row * dv + col] = s[a][r];
      }
}
