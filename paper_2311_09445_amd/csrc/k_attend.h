// One pass of linear attention over sequences (see seq_attention.hip for what the passes are), on the matrix cores.
// Part of seq_attention.hip (included inside namespace per); not a stand-alone header.
//
// A sequence is taken in chunks of 32 tokens.  With S the state before a chunk, f_i = c_out decay^(i+1-lag) and
// w_j = c_state decay^(n-1-j+lag) for the n tokens of the chunk,
//   out = diag(f) X S + (c_in X Y^T . decay^(i-j) for j <= i) Z,     S <- decay^n S + Y^T diag(w) Z.
// Everything is computed transposed (out^T = S^T X^T + ...), because then what one product leaves in registers is what the next
// one reads: the 16 x 16 result of a matrix instruction holds, in lane 16 g + m, column m and rows 4 g .. 4 g + 3, and its 32-deep
// operand column (or row) m and any eight places of the inner dimension, as long as both operands take the same ones.  Taking the
// places 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3, two results stacked are an operand: S^T, and the decayed products of pairs.
//
// A wave holds 16 NT columns of the state for all of dx in registers; the waves of a workgroup share the chunk's rows in LDS, and
// each works out the products of pairs for itself (3 tiles; sharing them would cost a barrier).

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kChunk = 32;

// Operand of 16 x 32 places: 8 of the inner dimension per lane.
template <typename T>
struct Operand;

template <>
struct Operand<bf16> {
  static constexpr uint32_t kWide = 8;                    // elements of 16 bytes
  static constexpr uint32_t kPadX = 8, kPadZ = 16;        // elements behind a row: rows read along their length, across it
  bf16x8 v;
  // Rows m of a tile, the inner dimension along them.
  __device__ __forceinline__ static Operand along(const bf16* row, uint32_t g) {
    const bf16x4 a = *reinterpret_cast<const bf16x4*>(row + 4 * g), b = *reinterpret_cast<const bf16x4*>(row + 16 + 4 * g);
    return {__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)};
  }
  // Columns m of a tile, the inner dimension across the rows (a transposing read: 16 lanes read 4 rows of 16 elements).
  __device__ __forceinline__ static Operand across(const bf16* tile, uint32_t stride, uint32_t m, uint32_t g) {
    typedef __attribute__((address_space(3))) s16x4 Lds;
    const bf16* at = tile + (4 * g + (m >> 2)) * stride + 4 * (m & 3);
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)at), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(at + 16 * stride));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const s16x8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return {__builtin_bit_cast(bf16x8, v)};
  }
  __device__ __forceinline__ static Operand of(f32x4 a, f32x4 b) {
    Operand o;
#pragma unroll
    for (int i = 0; i < 4; ++i) { o.v[i] = (bf16)a[i]; o.v[i + 4] = (bf16)b[i]; }
    return o;
  }
  __device__ __forceinline__ float at(int i) const { return (float)v[i]; }
  __device__ __forceinline__ static f32x4 mma(const Operand& a, const Operand& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
  }
};

template <>
struct Operand<float> {
  static constexpr uint32_t kWide = 4;
  static constexpr uint32_t kPadX = 4, kPadZ = 4;
  float v[8];
  __device__ __forceinline__ static Operand along(const float* row, uint32_t g) {
    return of(*reinterpret_cast<const f32x4*>(row + 4 * g), *reinterpret_cast<const f32x4*>(row + 16 + 4 * g));
  }
  __device__ __forceinline__ static Operand across(const float* tile, uint32_t stride, uint32_t m, uint32_t g) {
    Operand o;
    const float* at = tile + 4 * g * stride + m;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) { o.v[i] = at[i * stride]; o.v[i + 4] = at[(16 + i) * stride]; }
    return o;
  }
  __device__ __forceinline__ static Operand of(f32x4 a, f32x4 b) {
    Operand o;
#pragma unroll
    for (int i = 0; i < 4; ++i) { o.v[i] = a[i]; o.v[i + 4] = b[i]; }
    return o;
  }
  __device__ __forceinline__ float at(int i) const { return v[i]; }
  __device__ __forceinline__ static f32x4 mma(const Operand& a, const Operand& b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
  }
};

// What a wave's lane adds to the state: Z^T w in TERMS operands whose sum is the fp32 product to 8 TERMS bits.
template <typename T, int TERMS>
struct Scaled {
  Operand<T> part[TERMS];
  __device__ __forceinline__ Scaled(const Operand<T>& z, const f32x4& w0, const f32x4& w1) {
    f32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] = z.at(i) * w0[i]; b[i] = z.at(i + 4) * w1[i]; }
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
      part[t] = Operand<T>::of(a, b);
      if (t + 1 < TERMS)
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[i] -= part[t].at(i); b[i] -= part[t].at(i + 4); }
    }
  }
};

// decay^e for e >= 0 from its logarithm (which may be -infinity).
__device__ __forceinline__ float decay_power(float g, int e) { return e == 0 ? 1.0f : expf((float)e * g); }

// 32 rows of D elements on their way from memory to LDS, N pieces of 16 bytes in each thread's registers.
template <typename T, int D, int THREADS>
struct Piece {
  static constexpr uint32_t W = Operand<T>::kWide, PER_ROW = D / W, PIECES = kChunk * PER_ROW, N = (PIECES + THREADS - 1) / THREADS;
  typedef T Vec __attribute__((ext_vector_type(W)));
  Vec v[N];
  // Rows first .. first + n of a head's sequence of `valid` tokens (against time: counted from its end), columns col0 .. col0 + D.
  __device__ __forceinline__ void load(const SeqRows& r, const T* head, uint32_t first, uint32_t n, uint32_t valid, bool back, uint32_t col0, uint32_t width) {
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) {
      const uint32_t at = threadIdx.x + k * THREADS;
      const uint32_t row = at / PER_ROW, col = col0 + at % PER_ROW * W;
      v[k] = Vec(T(0.0f));
      if ((PIECES % THREADS == 0 || at < PIECES) && row < n && col < width) {
        const uint32_t i = first + row, t = back ? valid - 1 - i : i;
        const T* p = head + (int64_t)t * r.token + col;
        if (r.wide && col + W <= width) {
          v[k] = *reinterpret_cast<const Vec*>(p);
        } else {
#pragma unroll
          for (uint32_t e = 0; e < W; ++e)
            if (col + e < width) v[k][e] = p[e];
        }
      }
    }
  }
  __device__ __forceinline__ void store(T* lds, uint32_t stride) const {
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) {
      const uint32_t at = threadIdx.x + k * THREADS;
      if (PIECES % THREADS == 0 || at < PIECES) *reinterpret_cast<Vec*>(lds + at / PER_ROW * stride + at % PER_ROW * W) = v[k];
    }
  }
};

// Elements of one buffer of a chunk's rows.
template <typename T, int DX, int DZ, bool OUT>
constexpr uint32_t chunk_elements() {
  return kChunk * ((OUT ? 2 : 1) * (DX + Operand<T>::kPadX) + DZ + Operand<T>::kPadZ);
}

// OUT: the outputs are wanted too (else only the state that the piece of the sequence brings, from zeros).
template <typename T, int DX, int NT, int WAVES, int TERMS, bool OUT>
__global__ __launch_bounds__(64 * WAVES, 2) void k_attend(AttentionPasses all) {
  constexpr int THREADS = 64 * WAVES, DZ = 16 * NT * WAVES, TX = DX / 16, KX = DX / 32;
  constexpr uint32_t SX = DX + Operand<T>::kPadX, SZ = DZ + Operand<T>::kPadZ, BUFFER = chunk_elements<T, DX, DZ, OUT>();
  extern __shared__ __attribute__((aligned(16))) uint8_t lds_raw[];
  T* const lds = reinterpret_cast<T*>(lds_raw);
  // Workgroups go round the 8 dies by their number: the passes over the same rows sit on one die, one behind the other.
  const uint32_t which = blockIdx.x / 8 % all.count, item = blockIdx.x / (8 * all.count) * 8 + blockIdx.x % 8;
  if (item >= all.items) return;
  const AttentionPass& p = all.pass[which];
  const uint32_t slice = item % all.slices, seg = item / all.slices % all.segments, bh = item / all.slices / all.segments;
  const uint32_t h = bh % p.H, b = bh / p.H, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
  const uint32_t valid = valid_tokens(p.lengths, b, p.L), begin = seg * all.segment;
  const uint32_t end = valid < begin ? begin : valid - begin < all.segment ? valid : begin + all.segment;
  const uint32_t col0 = slice * DZ, col = col0 + wave * 16 * NT;   // first z column of the workgroup, of the wave
  const float decay = p.log_decay[h];
  const bool back = p.back != 0;
  const int lag = back ? 1 : 0;

  f32x4 S[TX][NT];
#pragma unroll
  for (int a = 0; a < TX; ++a)
#pragma unroll
    for (int c = 0; c < NT; ++c) S[a][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (OUT && p.in) {
    const float* in = p.in + (int64_t)b * p.in_batch + (int64_t)h * p.in_head + (int64_t)seg * p.in_segment;
#pragma unroll
    for (int a = 0; a < TX; ++a)
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t i = 16 * a + 4 * g + r, j = col + 16 * c + m;
          if (i < p.dx && j < p.dz) S[a][c][r] = in[i * p.in_x + j * p.in_z];
        }
  }

  const T* const xh = OUT ? row_of<T>(p.x, b, 0, h) : nullptr;
  const T* const yh = row_of<T>(p.y, b, 0, h);
  const T* const zh = row_of<T>(p.z, b, 0, h);
  Piece<T, DX, THREADS> px, py;
  Piece<T, DZ, THREADS> pz;
  auto fetch = [&](uint32_t first) {
    const uint32_t n = first < end ? (end - first < kChunk ? end - first : kChunk) : 0;
    if (OUT) px.load(p.x, xh, first, n, valid, back, 0, p.dx);
    py.load(p.y, yh, first, n, valid, back, 0, p.dx);
    pz.load(p.z, zh, first, n, valid, back, col0, p.dz);
  };

  // Powers of the decay: between the tokens of a pair (same tile; a tile apart), to the chunk's tokens, from them, over the chunk.
  f32x4 pair[2], into[2];
  float outof[2], keep = 0.0f;
  if (OUT) {
#pragma unroll
    for (int d = 0; d < 2; ++d) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = 16 * d + (int)m - (int)(4 * g) - r;
        pair[d][r] = e < 0 ? 0.0f : p.c_in * decay_power(decay, e);
      }
      outof[d] = p.c_out * decay_power(decay, 16 * d + (int)m + 1 - lag);
    }
  }
  auto weights = [&](int n) {
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = n - 1 - 16 * d - (int)(4 * g) - r;
        into[d][r] = e < 0 ? 0.0f : p.c_state * decay_power(decay, e + lag);
      }
    // S + (decay^n - 1) S: the power itself, rounded to 32 bits, would be off by the same 2^-25 in every chunk of a slow decay
    keep = expm1f((float)n * decay);
  };
  weights(kChunk);

  fetch(begin);
  for (uint32_t first = begin, turn = 0; first < end; first += kChunk, turn ^= 1) {
    T* const xs = lds + turn * BUFFER;
    T* const ys = OUT ? xs + kChunk * SX : xs;
    T* const zs = ys + kChunk * SX;
    if (OUT) px.store(xs, SX);
    py.store(ys, SX);
    pz.store(zs, SZ);
    __syncthreads();
    if (first + kChunk < end) fetch(first + kChunk);
    const uint32_t n = end - first < kChunk ? end - first : kChunk;
    if (n < kChunk) weights((int)n);

    Operand<T> z[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) z[c] = Operand<T>::across(zs + wave * 16 * NT + 16 * c, SZ, m, g);
    if (OUT) {
      f32x4 acc[NT][2], pt[3];
      const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < NT; ++c) acc[c][0] = acc[c][1] = zero;
      pt[0] = pt[1] = pt[2] = zero;
#pragma unroll
      for (int k = 0; k < KX; ++k) {
        const Operand<T> x0 = Operand<T>::along(xs + m * SX + 32 * k, g), x1 = Operand<T>::along(xs + (16 + m) * SX + 32 * k, g);
        const Operand<T> y0 = Operand<T>::along(ys + m * SX + 32 * k, g), y1 = Operand<T>::along(ys + (16 + m) * SX + 32 * k, g);
        pt[0] = Operand<T>::mma(y0, x0, pt[0]);
        pt[1] = Operand<T>::mma(y0, x1, pt[1]);
        pt[2] = Operand<T>::mma(y1, x1, pt[2]);
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          const Operand<T> s = Operand<T>::of(S[2 * k][c], S[2 * k + 1][c]);
          acc[c][0] = Operand<T>::mma(s, x0, acc[c][0]);
          acc[c][1] = Operand<T>::mma(s, x1, acc[c][1]);
        }
      }
      const Operand<T> p0 = Operand<T>::of(pt[0] * pair[0], zero), p1 = Operand<T>::of(pt[1] * pair[1], pt[2] * pair[0]);
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        acc[c][0] = Operand<T>::mma(z[c], p0, acc[c][0] * outof[0]);
        acc[c][1] = Operand<T>::mma(z[c], p1, acc[c][1] * outof[1]);
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const uint32_t row = 16 * d + m, j = col + 16 * c + 4 * g;
          if (row >= n || j >= p.dz) continue;
          const uint32_t i = first + row, t = back ? valid - 1 - i : i;
          if (p.out_f32) store4(row_to<float>(p.out, b, t, h) + j, acc[c][d], p.out.wide, p.dz - j);
          else store4(row_to<T>(p.out, b, t, h) + j, acc[c][d], p.out.wide, p.dz - j);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const Scaled<T, TERMS> zw(z[c], into[0], into[1]);
#pragma unroll
      for (int a = 0; a < TX; ++a) {
        const Operand<T> y = Operand<T>::across(ys + 16 * a, SX, m, g);
#pragma unroll
        for (int r = 0; r < 4; ++r) S[a][c][r] = fmaf(S[a][c][r], keep, S[a][c][r]);
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) S[a][c] = Operand<T>::mma(y, zw.part[t], S[a][c]);
      }
    }
  }

  float* const to = OUT ? p.to : p.part;
  if (to) {
    float* const S_out = OUT ? to + (int64_t)b * p.to_batch + (int64_t)h * p.to_head : to + ((size_t)bh * all.segments + seg) * p.dx * p.dz;
#pragma unroll
    for (int a = 0; a < TX; ++a)
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t i = 16 * a + 4 * g + r, j = col + 16 * c + m;
          if (i < p.dx && j < p.dz) S_out[i * p.dz + j] = S[a][c][r];
        }
  }
  if (!OUT || valid >= p.L) return;
  // tokens behind the valid ones: zeros
  const uint32_t width = p.dz - col0 < (uint32_t)DZ ? p.dz - col0 : DZ, from = begin > valid ? begin : valid;
  const uint32_t until = p.L - begin < all.segment ? p.L : begin + all.segment;
  for (uint32_t t = from + wave; t < until; t += WAVES)
    for (uint32_t j = lane; j < width; j += 64) {
      if (p.out_f32) row_to<float>(p.out, b, t, h)[col0 + j] = 0.0f;
      else row_to<T>(p.out, b, t, h)[col0 + j] = (T)0.0f;
    }
}

// The states that the segments of a sequence start from, from what each of them brings, in place; and the last state.
__global__ __launch_bounds__(256) void k_join(JoinPasses all) {
  const JoinPass& p = all.pass[blockIdx.y];
  const uint32_t per = p.dx * p.dz;
  const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (uint64_t)all.BH * per) return;
  const uint32_t bh = (uint32_t)(at / per), e = (uint32_t)(at % per), h = bh % all.H, b = bh / all.H;
  const uint32_t valid = valid_tokens(all.lengths, b, all.L);
  const float g = all.log_decay[h];
  float S = p.in ? p.in[(int64_t)b * p.in_batch + (int64_t)h * p.in_head + e] : 0.0f;
  float* part = p.part + (size_t)bh * all.segments * per + e;
  for (uint32_t s0 = 0; s0 < all.segments; s0 += 8) {
    float brought[8];
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) brought[k] = s0 + k < all.segments ? part[(size_t)(s0 + k) * per] : 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
      if (s0 + k >= all.segments) break;
      part[(size_t)(s0 + k) * per] = S;
      const uint32_t begin = (s0 + k) * all.segment;
      const uint32_t n = valid <= begin ? 0 : valid - begin < all.segment ? valid - begin : all.segment;
      if (n) S = fmaf(S, expm1f((float)n * g), S) + brought[k];
    }
  }
  if (p.to) p.to[(int64_t)b * p.to_batch + (int64_t)h * p.to_head + e] = S;
}
