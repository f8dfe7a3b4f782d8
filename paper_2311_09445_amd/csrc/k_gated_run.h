// The gated delta rule over sequences.  Part of seq_delta.hip (included inside namespace per).
//
// With the record of a chunk (k_gated_pairs.h) and S the state before it,
//   Z = V - e^G K S,  Y = solve Z,  U = diag(beta) Y,  out = scale e^G Q S + pairs U,  S <- e^Gn S + K^T (left U).
// The columns of the state do not meet, so a wave holds 16 of them for all of dk in registers and goes over the whole sequence; four
// waves share the rows of queries and keys in LDS.  The result of one product is the operand of the next: rows of Z, Y and U are
// tokens, which the next product runs over.  The outputs are formed transposed, so that a lane has four neighbours of a token.
//
// What bounds it, in bfloat16 at 128 x 128: a workgroup by itself takes 2.45 us for a chunk (1.8 of its products alone, 1.5 of its loads alone; at
// 64 x 64 1.8 in all); with the chip full a SIMD's two waves take 3600 cycles each, of which 500 vector instructions are 2000 and 82 matrix
// instructions 1300: 65536 tokens of 16 heads 504 us, and what their segments carry, over twice the columns, 666.  A third of the vector
// instructions take the state apart.  Keeping states for a gradient is bound by memory: 1.4 GB in 260 us of 2 x 8192 tokens of 16 heads.  Rows are asked for a chunk ahead, straight to LDS where they are whole pieces (by way of registers a
// chunk took 6.6 us), and results are stored behind the next barrier, so that nothing waits for a store.
//
// Whatever is computed is taken apart into three parts in bfloat16 where it becomes an operand, since the state is fp32 and what is
// written to it comes out of the state: 24 bits.  What only the outputs see keeps 16 bits of itself where these are bfloat16.

struct DeltaRun {
  SeqRows q, k, v, out, dout;
  const void* records;
  uint32_t record_bytes;
  const int32_t* lengths;
  const float* in;
  float* to;
  int64_t in_batch, in_head, in_segment, to_batch, to_head;
  uint32_t L, H, dk, dv, chunks, slices, segments, segment, run;   // segment: chunks of one; run: segments that are taken
  float scale;
  float* carried;                // [sequence, head][segment], `each` floats: what a segment adds [dk][dv], what it makes of a state [dk][dk], and
  uint32_t each, turned;         // (turned) that transposed
  // kept for a gradient: the states before the chunks, Y, what keys read of them (e^G K S), and rows of what queries read . dout
  bf16x8* states;
  float *y, *x, *read;
  DeltaPairs pairs;              // for a workgroup that makes its records itself
};

// CARRYING: no outputs; what a segment adds to a state, and (in slices of their own) what it makes of one: its product with the state before it.
enum DeltaMode { FORWARD, KEEPING, CARRYING };

// Planes of 16 bits that the states before the chunks are kept in for a gradient: where rows are bfloat16 the two halves of the 32 bits (the
// gradients of decays take the state whole), else the three parts that an operand takes.
template <typename T>
constexpr int kStateParts = sizeof(T) == 2 ? 2 : 3;

// Where plane `part` of the states kept for chunk c of a sequence and head lies: [part][16 columns of dv][32 places of dk][lane], eight places a lane
// as registers hold them, so that a wave's instruction writes and reads 1 KiB in a row.  (As tiles of columns, pieces of 16 bytes in lines of
// their own, the pass that keeps them took 6.5 us for a chunk of 128 x 128, and the one that reads them 6.)
template <int DK>
__device__ __forceinline__ size_t state_at(uint32_t bh, uint32_t chunks, uint32_t c, uint32_t blocks, uint32_t parts, uint32_t part, uint32_t tile) {
  return ((((size_t)bh * chunks + c) * parts + part) * blocks * 2 + tile) * (DK / 32) * 64;
}

// What a pass takes of a record: rows of products, and numbers for the tokens 16 i + 4 g + r (and 16 i + m).
template <int N>
struct RecordRows {
  bf16x8 solve[2][3], pairs[2][N];
  template <bool PAIRS = true>
  __device__ __forceinline__ void load(const bf16x8* solves, const bf16x8* pairings, uint32_t lane) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int t = 0; t < 3; ++t) solve[i][t] = solves[(2 * t + i) * 64 + lane];
#pragma unroll
      for (int t = 0; t < (PAIRS ? N : 0); ++t) pairs[i][t] = pairings[(2 * t + i) * 64 + lane];
    }
  }
};
struct RecordNumbers {
  f32x4 gamma[2], left[2], beta[2];
  float gamma_m[2], kept[2];
  __device__ __forceinline__ void load(const DeltaRecord* r, uint32_t m, uint32_t g) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      gamma[i] = *reinterpret_cast<const f32x4*>(r->gamma + 16 * i + 4 * g);
      left[i] = *reinterpret_cast<const f32x4*>(r->left + 16 * i + 4 * g);
      beta[i] = *reinterpret_cast<const f32x4*>(r->beta + 16 * i + 4 * g);
      gamma_m[i] = r->gamma[16 * i + m];
      kept[i] = r->kept[i];
    }
  }
  // They are there: the compiler waits for its loads here, not where they are used, behind loads to LDS that it does not know of.
  __device__ __forceinline__ void there() {
#pragma unroll
    for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(gamma[i]), "+v"(left[i]), "+v"(beta[i]), "+v"(gamma_m[i]), "+v"(kept[i]));
  }
  // What is left of a state: one rounding, of the sum (a rounded decay alone would be off by the same 2^-25 in each chunk).
  __device__ __forceinline__ f32x4 keep(f32x4 s) const {
    f32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(s[e], kept[0], s[e] * kept[1]);
    return o;
  }
};

// Rows of D columns straight into a tile in LDS, by four waves: each instruction of a wave fills 1 KiB, 64 pieces, and asks memory for those that
// belong there.  Pieces behind the width are never asked for (they are cleared once); rows behind the last valid one are asked for as that
// one, and cleared when they are there.
template <int D>
struct DirectRows {
  static constexpr uint32_t N = Tile<D>::SIZE / 512 / 4;   // of a wave
  uint32_t offset[N], row[N];
  bool on[N];
  uint32_t bytes;
  __device__ __forceinline__ void set(const SeqRows& r, uint32_t width, uint32_t wave, uint32_t lane) {
    bytes = (uint32_t)r.token * 2;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      const uint32_t place = (wave + 4 * i) * 64 + lane;
      row[i] = place / Tile<D>::PIECES;
      const uint32_t piece = place % Tile<D>::PIECES ^ Tile<D>::turn(row[i]);
      on[i] = piece * 8 < width;
      offset[i] = row[i] * bytes + piece * 16;
    }
  }
  // n: rows that there are, of 32
  __device__ __forceinline__ void ask(uint32_t to, const uint8_t* base, uint32_t wave, uint32_t n) const {
    if (n >= kChunk) {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i)
        if (on[i]) load_to_lds(to + (wave + 4 * i) * 1024, base, offset[i]);
      return;
    }
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      const uint32_t back = row[i] < n ? 0 : row[i] - (n - 1);
      if (on[i]) load_to_lds(to + (wave + 4 * i) * 1024, base, offset[i] - back * bytes);
    }
  }
  __device__ __forceinline__ static void clear(bf16* tile, uint32_t n, uint32_t thread) {
    const bf16x8 zero = {};
    for (uint32_t i = n * Tile<D>::PIECES + thread; i < Tile<D>::SIZE / 8; i += 256) *reinterpret_cast<bf16x8*>(tile + 8 * i) = zero;
  }
};
// The first n KiB of a record's rows of products.
template <uint32_t N>
__device__ __forceinline__ void ask_rows(uint32_t to, const void* from, uint32_t wave, uint32_t lane) {
#pragma unroll
  for (uint32_t i = 0; i < N; i += 4)   // (the last wave's twice where four waves do not share N)
    load_to_lds(to + (i + wave < N ? i + wave : N - 1) * 1024, static_cast<const uint8_t*>(from), (i + wave < N ? i + wave : N - 1) * 1024 + lane * 16);
}
// Rows of a head from chunk to chunk.
struct Walk {
  const uint8_t* at;
  int64_t step;
  __device__ __forceinline__ void set(const SeqRows& r, const void* head, uint32_t chunk, bool back) {
    const int64_t bytes = (int64_t)kChunk * r.token * 2;
    at = static_cast<const uint8_t*>(head) + chunk * bytes;
    step = back ? -bytes : bytes;
  }
  __device__ __forceinline__ const uint8_t* next() {
    const uint8_t* here = at;
    at += step;
    return here;
  }
};
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}

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

// Rows 16 i + 4 g + r of a chunk, column col, as the rows have them (a conversion, or clearing one, would be waited for where it is asked for),
// and as fp32.
template <typename T>
struct Column {
  T v[2][4];
  __device__ __forceinline__ void ask(const SeqRows& rows, const T* head, uint32_t first, uint32_t valid, bool on, uint32_t col, uint32_t g) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t t = first + 16 * i + 4 * g + r;
        v[i][r] = head[(int64_t)(t < valid ? t : valid - 1) * rows.token + (on ? col : 0)];
      }
  }
  __device__ __forceinline__ void widen(uint32_t first, uint32_t valid, bool on, uint32_t g, f32x4 (&x)[2]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[i][r] = on && first + 16 * i + 4 * g + r < valid ? as_float(v[i][r]) : 0.0f;
  }
};
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

// The same as the row has them.
template <typename T>
struct Four {
  typedef T Vec __attribute__((ext_vector_type(4)));
  Vec v;
};
template <typename T>
__device__ __forceinline__ void ask_four(const T* row, bool wide, uint32_t col, uint32_t width, Four<T>* o) {
  if (wide && width % 4 == 0) {
    o->v = *reinterpret_cast<const typename Four<T>::Vec*>(row + (col < width ? col : 0));
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) o->v[i] = row[col + i < width ? col + i : 0];
  }
}
template <typename T>
__device__ __forceinline__ f32x4 four_of(const Four<T>& f, bool on, uint32_t col, uint32_t width) {
  f32x4 o;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) o[i] = on && col + i < width ? as_float(f.v[i]) : 0.0f;
  return o;
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

// Values that are not finite and the tokens before them.  Products over a chunk take every token with every other, those behind it 0 times, and 0 times such
// a value is one too.  So where a column (rows 16 i + 4 g + r of it in a lane) has one, it is cleared from there, and what depends on it is made NaN behind
// the product.
__device__ __forceinline__ bool all_finite(const f32x4 (&x)[2]) {   // of the wave
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = fmaf(x[i / 4][i % 4], 0.0f, sum);
  return __ballot(!(sum == 0.0f)) == 0;
}
__device__ __forceinline__ uint32_t clear_from_first(f32x4 (&x)[2], uint32_t g) {   // the column's first such row, or 32
  uint32_t first = kChunk;
#pragma unroll
  for (int i = 7; i >= 0; --i)
    if (!(x[i / 4][i % 4] * 0.0f == 0.0f)) first = 16 * (i / 4) + 4 * g + i % 4;
  for (int d = 16; d < 64; d *= 2) {
    const uint32_t other = __shfl_xor(first, d);
    first = other < first ? other : first;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (16 * (i / 4) + 4 * g + i % 4 >= first) x[i / 4][i % 4] = 0.0f;
  return first;
}

// LDS of a chunk: rows of queries and keys, and where they come straight from memory those of 64 values and the record's products too (twice 32 KiB:
// as far as such loads reach).
// (Only outputs take pairs; a pass that only carries has no queries either.)
template <typename T, int DK, int NP, bool DIRECT_ROWS, DeltaMode MODE>
struct RunLds {
  static constexpr uint32_t ROWS = kParts<T> * Tile<DK>::SIZE, Q = 0, K = MODE != CARRYING || !DIRECT_ROWS ? ROWS : 0, V = K + ROWS,
                            SOLVE = V + (DIRECT_ROWS ? Tile<64>::SIZE : 0), PAIRS = SOLVE + (DIRECT_ROWS ? 3 * 1024 : 0),
                            SIZE = PAIRS + (DIRECT_ROWS && MODE == FORWARD ? NP * 1024 : 0), BYTES = 2 * SIZE * sizeof(bf16);
};
template <typename T, DeltaMode MODE>
constexpr int kPairParts = MODE != FORWARD ? 1 : sizeof(T) == 2 ? 2 : 3;

// OWN: a workgroup forms its chunks' records itself, a wave a chunk: one launch less where sequences have no more than four (64 stretches of up to 80
// tokens of 4 heads of 64 x 64: 20.0 us and 17.6).  It has all columns then, so that nobody else needs them.
template <typename T, int DK, DeltaMode MODE, bool DIRECT_ROWS, bool OWN = false>
__global__ __launch_bounds__(256, !DIRECT_ROWS ? 1 : MODE == CARRYING && DK == 64 ? 3 : 2) void k_delta_run(DeltaRun p) {
  constexpr int PT = kParts<T>, TX = DK / 16, KX = DK / 32, NP = kPairParts<T, MODE>, LESS = MODE == FORWARD ? NP - 1 : 2;
  typedef RunLds<T, DK, NP, DIRECT_ROWS, MODE> Lds;
  static_assert(!DIRECT_ROWS || Lds::BYTES <= 65536, "loads to LDS have 16 bits of address");
  extern __shared__ __attribute__((aligned(256))) uint8_t lds_raw[];
  bf16* const lds = reinterpret_cast<bf16*>(lds_raw);
  const uint32_t dk = p.dk, all_slices = MODE == CARRYING ? p.slices + (dk + 63) / 64 : p.slices;
  const uint32_t item = blockIdx.x / all_slices, slice_of_all = blockIdx.x % all_slices, seg = item % p.run, bh = item / p.run, h = bh % p.H, b = bh / p.H;
  const bool product = MODE == CARRYING && slice_of_all >= p.slices;
  const uint32_t slice = product ? slice_of_all - p.slices : slice_of_all;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const uint32_t L = p.L, dv = product ? dk : p.dv, blocks = (dv + 31) / 32, col0 = 64 * slice + 16 * wave, col = col0 + m;
  const bool on = col < dv, works = col0 < blocks * 32, takes = on && !product;   // takes: values
  const uint32_t valid = __builtin_amdgcn_readfirstlane(valid_tokens(p.lengths, b, L)), all_chunks = (valid + kChunk - 1) / kChunk;
  const uint32_t chunk0 = seg * p.segment, chunks = all_chunks < chunk0 ? chunk0 : all_chunks - chunk0 < p.segment ? all_chunks : chunk0 + p.segment;   // its end
  const uint8_t* const records = static_cast<const uint8_t*>(p.records) + (size_t)bh * p.chunks * p.record_bytes;
  const bool pieces = p.q.near && p.k.near && dk >= 16 / sizeof(T);
  auto record = [&](uint32_t c) { return reinterpret_cast<const DeltaRecord*>(records + (size_t)c * p.record_bytes); };
  if constexpr (OWN) {
    const bool fast = DIRECT_ROWS || (p.q.wide && p.k.wide && dk % (16 / sizeof(T)) == 0);
    PairLds* const own_lds = reinterpret_cast<PairLds*>(lds_raw) + wave;
    for (uint32_t c = wave; c < chunks; c += 4) {
      if (fast) pairs_of<T, DK, MODE == KEEPING, true>(p.pairs, bh * p.chunks + c, lane, own_lds);
      else pairs_of<T, DK, MODE == KEEPING, false>(p.pairs, bh * p.chunks + c, lane, own_lds);
    }
    arrive<0>();   // (what the waves have stored is in L2, from where it is read)
  }

  f32x4 s[TX];
#pragma unroll
  for (int a = 0; a < TX; ++a)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t row = state_row(a, 4 * g + r);
      if (MODE == CARRYING) s[a][r] = product && row == col && on ? 1.0f : 0.0f;
      else s[a][r] = p.in && on && row < dk ? p.in[(int64_t)b * p.in_batch + (int64_t)h * p.in_head + seg * p.in_segment + (size_t)row * dv + col] : 0.0f;
    }
  const T *const q0 = row_of<T>(p.q, b, 0, h), *const k0 = row_of<T>(p.k, b, 0, h), *const v0 = row_of<T>(p.v, b, 0, h);
  TwoRows<T, DK> rows;
  DirectRows<DK> direct_q, direct_k;
  DirectRows<64> direct_v;
  Walk walk_q, walk_k, walk_v, walk_out;
  RecordRows<NP> next;
  RecordNumbers num, next_num;
  Column<T> next_v, now_v;
  Four<T> next_d[2], now_d[2];
  const uint32_t lds0 = lds_address(lds);
  auto fetch = [&](uint32_t c) {   // chunk c, to LDS or (rows by way of registers: the one behind it) to registers
    if constexpr (DIRECT_ROWS) {
      const uint32_t n = valid - c * kChunk, to = lds0 + (c & 1) * Lds::SIZE * 2;
      if (MODE != CARRYING) direct_q.ask(to + Lds::Q * 2, walk_q.next(), wave, n);
      direct_k.ask(to + Lds::K * 2, walk_k.next(), wave, n);
      if (!product) direct_v.ask(to + Lds::V * 2, walk_v.next(), wave, n);
      ask_rows<6>(to + Lds::SOLVE * 2, record(c)->solve, wave, lane);
      if (MODE == FORWARD) ask_rows<2 * NP>(to + Lds::PAIRS * 2, record(c)->pairs, wave, lane);
    } else {
      rows.store(lds + (c & 1) * Lds::SIZE, valid - c * kChunk, dk, pieces);
      if (c + 1 < chunks) rows.load(p.q, p.k, q0, k0, (c + 1) * kChunk, valid, dk, pieces);
      next.template load<MODE == FORWARD>(&record(c)->solve[0][0][0], &record(c)->pairs[0][0][0], lane);
      next_v.ask(p.v, v0, c * kChunk, valid, takes, col, g);
    }
    if constexpr (MODE == KEEPING) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t t = c * kChunk + 16 * i + m;
        ask_four<T>(row_of<T>(p.dout, b, t < valid ? t : valid - 1, h), p.dout.wide, col0 + 4 * g, dv, &next_d[i]);
      }
    }
    next_num.load(record(c), m, g);
  };
  if constexpr (DIRECT_ROWS) {
    walk_q.set(p.q, q0, chunk0, false);
    walk_k.set(p.k, k0, chunk0, false);
    walk_v.set(p.v, v0 + 64 * slice, chunk0, false);
    if (MODE == FORWARD) walk_out.set(p.out, row_to<T>(p.out, b, 0, h) + 64 * slice, chunk0, false);
    direct_q.set(p.q, dk, wave, lane);
    direct_k.set(p.k, dk, wave, lane);
    direct_v.set(p.v, product ? 0 : dv - 64 * slice, wave, lane);
    if (dk < DK || dv - 64 * slice < 64 || product) {
      for (uint32_t i = 0; i < 2; ++i) {
        if (MODE != CARRYING) DirectRows<DK>::clear(lds + i * Lds::SIZE + Lds::Q, 0, threadIdx.x);
        DirectRows<DK>::clear(lds + i * Lds::SIZE + Lds::K, 0, threadIdx.x);
        DirectRows<64>::clear(lds + i * Lds::SIZE + Lds::V, 0, threadIdx.x);
      }
      __syncthreads();
    }
  } else if (chunk0 < chunks) {
    rows.load(p.q, p.k, q0, k0, chunk0 * kChunk, valid, dk, pieces);
  }
  if (chunk0 < chunks) fetch(chunk0);
  f32x4 o[2] = {}, y[2] = {};
  const uint32_t out_at[2] = {m * (uint32_t)p.out.token * 2 + (16 * wave + 4 * g) * 2, (16 + m) * (uint32_t)p.out.token * 2 + (16 * wave + 4 * g) * 2};
  // What chunk c leaves in memory is stored behind the next barrier: stores are older then than the loads that are waited for.
  auto flush = [&](uint32_t c) {
    if (!works || MODE == CARRYING) return;
    const uint32_t first = c * kChunk;
    if constexpr (MODE == KEEPING) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float* const to = p.y + ((size_t)bh * p.chunks * kChunk + first + 16 * i + 4 * g) * (blocks * 32) + col;
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e * blocks * 32] = y[i][e];
        const uint32_t t = first + 16 * i + m;
        if (g == 0) p.read[((size_t)bh * (blocks * 2) + col0 / 16) * p.chunks * kChunk + t] = o[i][0];
      }
    } else if (DIRECT_ROWS && p.out.wide && valid - first >= kChunk) {
      uint8_t* const to = const_cast<uint8_t*>(walk_out.next());
      if (col0 + 4 * g < dv) {
#pragma unroll
        for (int i = 0; i < 2; ++i) store_four<T>(reinterpret_cast<T*>(to + out_at[i]), true, 0, ~0u, o[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t t = first + 16 * i + m;
        if (t < L) store_four<T>(row_to<T>(p.out, b, t, h), p.out.wide, col0 + 4 * g, dv, t < valid ? o[i] : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
      }
    }
  };
  for (uint32_t c = chunk0; c < chunks; ++c) {
    const uint32_t first = c * kChunk;
    bf16 *const buffer = lds + (c & 1) * Lds::SIZE, *const Q = buffer + Lds::Q, *const K = buffer + Lds::K;
    if constexpr (DIRECT_ROWS) {
      // (what a pass that keeps states stores behind the loads: the state's planes, what keys read, and from the second chunk Y)
      if (MODE == KEEPING && works && c > chunk0 + 1) arrive<2 * KX + 16>();
      else arrive<0>();
      if (valid - first < kChunk) {
        if (MODE != CARRYING) DirectRows<DK>::clear(Q, valid - first, threadIdx.x);
        DirectRows<DK>::clear(K, valid - first, threadIdx.x);
        DirectRows<64>::clear(buffer + Lds::V, valid - first, threadIdx.x);
        __syncthreads();
      }
    } else {
      __syncthreads();
    }
    next_num.there();
    num = next_num;
    RecordRows<NP> rec = next;
    now_v = next_v;
    if constexpr (MODE == KEEPING) {
      now_d[0] = next_d[0];
      now_d[1] = next_d[1];
    }
    if (MODE != KEEPING && c > chunk0) flush(c - 1);
    if (c + 1 < chunks) fetch(c + 1);
    if constexpr (MODE == KEEPING) {   // (behind the loads: the next barrier does not wait for these)
      if (c > chunk0) flush(c - 1);
      if (works) {
#pragma unroll
        for (int k = 0; k < KX; ++k) {
          auto put = [&](const auto& parts) {
#pragma unroll
            for (int t = 0; t < kStateParts<T>; ++t) p.states[state_at<DK>(bh, p.chunks, c, blocks, kStateParts<T>, t, col0 / 16) + k * 64 + lane] = parts.v[t];
          };
          if constexpr (sizeof(T) == 2) put(halves_of(s[2 * k], s[2 * k + 1]));
          else put(Parts<kStateParts<T>>::of(s[2 * k], s[2 * k + 1]));
        }
      }
    }
    if (works) {
      f32x4 x4[4] = {}, o4[4] = {};   // (of even and odd k)
      Parts<3> sp[KX];
#pragma unroll
      for (int k = 0; k < KX; k += 2) {
        Operand<T> rows_k[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) rows_k[j] = Operand<T>::template along<DK>(K, 16 * (j & 1) + m, k + j / 2, g);
        sp[k] = Parts<3>::of(s[2 * k], s[2 * k + 1]);
        sp[k + 1] = Parts<3>::of(s[2 * k + 2], s[2 * k + 3]);
        mma_turns<4, 2, PT, 3>([&](int j) -> const bf16x8 (&)[PT] { return rows_k[j].v; }, [&](int j) -> const bf16x8 (&)[3] { return sp[k + j / 2].v; }, x4);
      }
      f32x4 v[2], x[2];
      if constexpr (DIRECT_ROWS) {
        rec.template load<MODE == FORWARD>(reinterpret_cast<const bf16x8*>(buffer + Lds::SOLVE), reinterpret_cast<const bf16x8*>(buffer + Lds::PAIRS), lane);
        Operand<bf16>::across<64>(buffer + Lds::V, [&](uint32_t i) { return 16 * wave + i; }, m, g).widen(&v[0], &v[1]);
      }
      else now_v.widen(first, valid, takes, g, v);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[i] = num.gamma[i] * (x4[i] + x4[i + 2]);
        if constexpr (MODE == KEEPING) {
          float* const to = p.x + ((size_t)bh * p.chunks * kChunk + first + 16 * i + 4 * g) * (blocks * 32) + col;
#pragma unroll
          for (int e = 0; e < 4; ++e) to[e * blocks * 32] = x[i][e];
        }
      }
      f32x4 zs[2] = {v[0] - x[0], v[1] - x[1]}, u[2];
      const bool spoilt = MODE == FORWARD && !all_finite(zs);
      uint32_t from = kChunk;
      if (spoilt) from = clear_from_first(zs, g);
      const Parts<3> z = Parts<3>::of(zs[0], zs[1]);
      y[0] = y[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      mma_turns<2, 2, 3, 3>([&](int i) -> const bf16x8 (&)[3] { return rec.solve[i]; }, [&](int) -> const bf16x8 (&)[3] { return z.v; }, y);
      if constexpr (MODE != CARRYING)
#pragma unroll
      for (int k = 0; k < KX; k += 2) {
        Operand<T> rows_q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) rows_q[j] = Operand<T>::template along<DK>(Q, 16 * (j & 1) + m, k + j / 2, g);
        mma_turns<4, LESS, 3, PT>([&](int j) -> const bf16x8 (&)[3] { return sp[k + j / 2].v; }, [&](int j) -> const bf16x8 (&)[PT] { return rows_q[j].v; }, o4);
      }
      if (spoilt)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (16 * (i / 4) + 4 * g + i % 4 >= from) y[i / 4][i % 4] = __builtin_nanf("");
#pragma unroll
      for (int i = 0; i < 2; ++i) u[i] = num.beta[i] * y[i];
      const Parts<3> w = Parts<3>::of(num.left[0] * u[0], num.left[1] * u[1]);
      const bool spoils = MODE == FORWARD && !all_finite(u);
      if (spoils) from = clear_from_first(u, g);
      const Parts<NP> up = Parts<NP>::of(u[0], u[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) o[i] = p.scale * num.gamma_m[i] * (o4[i] + o4[i + 2]);
      if constexpr (MODE == FORWARD)
        mma_turns<2, LESS, NP, NP>([&](int) -> const bf16x8 (&)[NP] { return up.v; }, [&](int i) -> const bf16x8 (&)[NP] { return rec.pairs[i]; }, o);
      if (spoils)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          const uint32_t first = __shfl(from, 4 * g + e);   // of the column that the element is of
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (16 * i + m >= first) o[i][e] = __builtin_nanf("");
        }
      constexpr int TURN = PT == 1 ? TX : 4;
#pragma unroll
      for (int a0 = 0; a0 < TX; a0 += TURN) {
        Operand<T> cols_k[TURN];
        f32x4 part[TURN];
#pragma unroll
        for (int a = 0; a < TURN; ++a) {
          cols_k[a] = Operand<T>::template across<DK>(K, [&](uint32_t i) { return state_row(a0 + a, i); }, m, g);
          part[a] = num.keep(s[a0 + a]);
        }
        mma_turns<TURN, 2, PT, 3>([&](int a) -> const bf16x8 (&)[PT] { return cols_k[a].v; }, [&](int) -> const bf16x8 (&)[3] { return w.v; }, part);
#pragma unroll
        for (int a = 0; a < TURN; ++a) s[a0 + a] = part[a];
      }
      if constexpr (MODE == KEEPING) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const f32x4 d = four_of<T>(now_d[i], first + 16 * i + m < valid, col0 + 4 * g, dv);
          float dot = 0.0f;
#pragma unroll
          for (int e = 0; e < 4; ++e) dot = fmaf(d[e], o[i][e], dot);
          dot += __shfl_xor(dot, 16);
          o[i][0] = dot + __shfl_xor(dot, 32);
        }
      }
    }
  }
  if (chunk0 < chunks) flush(chunks - 1);
  if (MODE == FORWARD && works) {
    const uint32_t end = p.segment < (L - chunk0 * kChunk + kChunk - 1) / kChunk ? (chunk0 + p.segment) * kChunk : L;
    for (uint32_t t = chunks * kChunk + m; t < end; t += 16) store_four<T>(row_to<T>(p.out, b, t, h), p.out.wide, col0 + 4 * g, dv, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
  }
  float* to = seg + 1 == p.segments && p.to ? p.to + (int64_t)b * p.to_batch + (int64_t)h * p.to_head : nullptr;
  if (MODE == CARRYING) to = p.carried + ((size_t)bh * p.segments + seg) * p.each + (product ? dk * p.dv : 0);
  if (MODE == CARRYING && product && p.turned && on)
#pragma unroll
    for (int a = 0; a < TX; ++a) store_four<float>(to + dk * dk + col * dk, dk % 4 == 0, state_row(a, 4 * g), dk, s[a]);
  if (to && on)
#pragma unroll
    for (int a = 0; a < TX; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t row = state_row(a, 4 * g + r);
        if (row < dk) to[(size_t)row * dv + col] = s[a][r];
      }
}

// The states that segments start from, one behind the other: S <- P S + B, with what each segment carries; S takes the place of B.  BACK: of
// the gradients behind the segments, R <- P^T R + C.  A workgroup takes 64 columns, a wave 16 rows of them; the rows' parts meet in LDS, where
// they lie as operands, and the next segment's product is under way meanwhile.  Past segments without tokens a state goes as it is: of an
// identity's zeros, one that is not finite would spoil its column.  (A wave for 16 columns and all rows took 45 us for a
// segment: it takes all of P apart by itself.)
struct DeltaJoin {
  float* carried;            // [sequence, head][segment]: B or C, rows of dv
  const float* products;     // P (BACK: transposed), rows of dk
  const float* in;
  int64_t in_batch, in_head;
  size_t stride, product_stride;
  const int32_t* lengths;
  uint32_t L, H, dk, dv, slices, segments, segment;
};
template <int DK, bool BACK>
__global__ __launch_bounds__(4 * DK) void k_delta_join(DeltaJoin p) {
  constexpr int KX = DK / 32;
  __shared__ __attribute__((aligned(16))) bf16x8 lds[3][KX][4][64];
  const uint32_t slice = blockIdx.x % p.slices, bh = blockIdx.x / p.slices, h = bh % p.H, b = bh / p.H;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const uint32_t dk = p.dk, dv = p.dv, row = state_row(wave, 4 * g), of_m = state_row(wave, m);
  const uint32_t valid = __builtin_amdgcn_readfirstlane(valid_tokens(p.lengths, b, p.L)), chunks = (valid + kChunk - 1) / kChunk;
  uint32_t at[4][4];   // of the wave's elements
  bool on[4][4];
  f32x4 s[4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (uint32_t r = 0; r < 4; ++r) {
      const uint32_t col = 64 * slice + 16 * c + m;
      on[c][r] = col < dv && row + r < dk;
      at[c][r] = on[c][r] ? (row + r) * dv + col : 0;
      s[c][r] = p.in && on[c][r] ? p.in[(int64_t)b * p.in_batch + (int64_t)h * p.in_head + at[c][r]] : 0.0f;
    }
  f32x4 product[KX][2], add[4];
  const bool fast = dk % 4 == 0;   // (rows of whole vectors: what a segment carries starts with dk dv or more floats before them)
  auto load = [&](uint32_t i) {
    const uint32_t seg = BACK ? p.segments - 1 - i : i;
    const float* const from = p.carried + ((size_t)bh * p.segments + seg) * p.stride;
    const float* const P = p.products + ((size_t)bh * p.segments + seg) * p.product_stride;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) add[c][r] = from[at[c][r]];
    if (i + 1 == p.segments) return;   // (the last one's product leads nowhere)
    const float* const row_m = P + (of_m < dk ? of_m * dk : 0);
#pragma unroll
    for (int k = 0; k < KX; ++k)
#pragma unroll
      for (uint32_t e = 0; e < 8; e += 4) {
        const uint32_t place = 32 * k + 8 * g + e;
        if (fast) {
          product[k][e / 4] = *reinterpret_cast<const f32x4*>(row_m + (place < dk ? place : 0));
        } else {
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) product[k][e / 4][j] = row_m[place + j < dk ? place + j : 0];
        }
      }
  };
  load(0);
  for (uint32_t i = 0; i < p.segments; ++i) {
    const uint32_t seg = BACK ? p.segments - 1 - i : i;
    float* const to = p.carried + ((size_t)bh * p.segments + seg) * p.stride;
    f32x4 acc[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        acc[c][r] = on[c][r] ? add[c][r] : 0.0f;
        if (on[c][r]) to[at[c][r]] = s[c][r];
      }
    if (i + 1 == p.segments) break;
    if (seg * p.segment >= chunks) {
      load(i + 1);
      continue;
    }
    Parts<3> P[KX];
#pragma unroll
    for (int k = 0; k < KX; ++k) {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e)
        if (of_m >= dk || 32 * k + 8 * g + e >= dk) product[k][e / 4][e % 4] = 0.0f;
      P[k] = Parts<3>::of(product[k][0], product[k][1]);
    }
    load(i + 1);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const Parts<3> x = Parts<3>::of(s[c], s[c]);
#pragma unroll
      for (int t = 0; t < 3; ++t)
        reinterpret_cast<bf16x4*>(&lds[t][wave / 2][c][lane])[wave & 1] = __builtin_shufflevector(x.v[t], x.v[t], 0, 1, 2, 3);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < KX; ++k) {
      bf16x8 x[4][3];
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int t = 0; t < 3; ++t) x[c][t] = lds[t][k][c][lane];
      mma_turns<4, 2, 3, 3>([&](int) -> const bf16x8 (&)[3] { return P[k].v; }, [&](int c) -> const bf16x8 (&)[3] { return x[c]; }, acc);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) s[c] = acc[c];
    __syncthreads();
  }
}
