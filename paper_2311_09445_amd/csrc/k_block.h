// Layer norm and dropout of rows.  Part of seq_block.hip (included inside namespace per).
//
// Rows are read in pieces of 16 bytes at any alignment; the last piece of a row whose width is no multiple of one ends with the row, and
// what it holds twice counts once.
//
// What bounds them: memory.  The norm of 32768 x 2048 in bfloat16 takes 52 us (5.2 TB/s; 44 where the last cache holds part of the rows from the call
// before; with weights element by element and a wave's row not ahead 78), dropout of as much with a residual 70 (5.7 TB/s).  The gradient of 8184 x 1537 takes 27: one round of workgroups, four rows to a wave
// (24, at 3.1 TB/s), and the sums' launch (a row to a workgroup of 256 lanes instead 35); of 32768 x 2048 88.

template <typename T>
struct Piece {
  static constexpr uint32_t W = 16 / sizeof(T);
  typedef T Vec __attribute__((ext_vector_type(W)));
  typedef Vec Loose __attribute__((aligned(sizeof(T))));   // (memory is read at any address that its elements may have)
};
__device__ __forceinline__ const char* block_row(const SeqRows& r, uint32_t row, uint32_t L, uint32_t H, uint32_t e) {
  const uint32_t h = row % H, tok = row / H;
  return static_cast<const char*>(r.d) + ((int64_t)(tok / L) * r.batch + (int64_t)(tok % L) * r.token + (int64_t)h * r.head) * (int64_t)e;
}
template <typename T>
__device__ __forceinline__ const T* row_at(const SeqRows& r, uint32_t row, const BlockArgs& a) {
  return reinterpret_cast<const T*>(block_row(r, row, a.L, a.H, sizeof(T)));
}

// A row held by LANES lanes, N pieces each; a piece's first column, and how many of its elements the piece before has as well.
template <typename T, int LANES, int N>
struct HeldRow {
  static constexpr uint32_t W = Piece<T>::W;
  static constexpr int ALL = N * W;
  uint32_t col[N], twice[N], whole;   // whole: the first pieces, which all lanes have
  bool on[N];
  __device__ __forceinline__ HeldRow(uint32_t lane, uint32_t dim) : whole(dim / (LANES * W)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t first = (lane + i * LANES) * W;
      on[i] = first < dim;
      col[i] = first + W <= dim ? first : dim - W;
      twice[i] = on[i] ? first - col[i] : W;
    }
  }
  __device__ __forceinline__ bool counts(int i, uint32_t e) const { return e >= twice[i]; }
  // (so that comparisons are made where they are used: held over a loop they would take two scalar registers for each element)
  __device__ __forceinline__ void again() {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(twice[i]));
  }
  // The sum of f(i) over the elements that count.
  template <typename F>
  __device__ __forceinline__ float sum(F f) const {
    float all = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if ((uint32_t)i < whole) {
#pragma unroll
        for (uint32_t e = 0; e < W; ++e) all += f(i * W + e);
      } else {
#pragma unroll
        for (uint32_t e = 0; e < W; ++e) all += counts(i, e) ? f(i * W + e) : 0.0f;
      }
    }
    return all;
  }
  typedef typename Piece<T>::Vec Raw[N];
  __device__ __forceinline__ void load(const T* row, Raw& v) const {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = *reinterpret_cast<const typename Piece<T>::Loose*>(row + (on[i] ? col[i] : 0));
  }
  __device__ __forceinline__ void widen(const Raw& v, float (&x)[ALL]) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (uint32_t e = 0; e < W; ++e) x[i * W + e] = as_float(v[i][e]);
  }
  __device__ __forceinline__ void load_plain(const float* row, float (&x)[ALL], float none) const {
    typedef Piece<float>::Loose Four;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (uint32_t e = 0; e < W; e += 4) {
        Piece<float>::Vec v = {none, none, none, none};
        if (row) v = *reinterpret_cast<const Four*>(row + (on[i] ? col[i] : 0) + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i * W + e + j] = v[j];
      }
  }
  __device__ __forceinline__ void store(T* row, const float (&x)[ALL]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (!on[i]) continue;
      typename Piece<T>::Vec v;
#pragma unroll
      for (uint32_t e = 0; e < W; ++e) v[e] = (T)x[i * W + e];
      *reinterpret_cast<typename Piece<T>::Loose*>(row + col[i]) = v;
    }
  }
};

// The sum over a wave, the same in every lane: four additions across 16 lanes, then the four of them in their order.
__device__ __forceinline__ float wave_sum(float x) {
  const int y = __builtin_bit_cast(int, sum16(x));
  auto lane = [&](int i) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(y, i)); };
  return (lane(0) + lane(16)) + (lane(32) + lane(48));
}
// Sums of a row's lanes, two at once: of 4 or 16 lanes, of a wave, or of the workgroup's four in their order.
template <int LANES>
__device__ __forceinline__ void row_sums(float* a, float* b, float (*lds)[2]) {
  if (LANES <= 16) {
    *a = LANES == 4 ? sum4(*a) : sum16(*a);
    *b = LANES == 4 ? sum4(*b) : sum16(*b);
    return;
  }
  *a = wave_sum(*a);
  *b = wave_sum(*b);
  if (LANES == 64) return;
  if ((threadIdx.x & 63) == 0) {
    lds[threadIdx.x >> 6][0] = *a;
    lds[threadIdx.x >> 6][1] = *b;
  }
  __syncthreads();
  *a = (lds[0][0] + lds[1][0]) + (lds[2][0] + lds[3][0]);
  *b = (lds[0][1] + lds[1][1]) + (lds[2][1] + lds[3][1]);
}

// Mean and reciprocal root of the variance of a row that is held: the variance from the differences, not from squares.
template <typename T, int LANES, int N>
__device__ __forceinline__ void standardise(const HeldRow<T, LANES, N>& at, float (&x)[N * Piece<T>::W], const BlockArgs& a, float* r, float (*lds)[4][2]) {
  float sum = at.sum([&](int i) { return x[i]; }), none = 0.0f;
  row_sums<LANES>(&sum, &none, lds[0]);
  const float mean = sum / (float)a.dim;
#pragma unroll
  for (int i = 0; i < at.ALL; ++i) x[i] -= mean;
  float square = at.sum([&](int i) { return x[i] * x[i]; });
  row_sums<LANES>(&square, &none, lds[1]);
  *r = 1.0f / sqrtf(square / (float)a.dim + a.eps);
}

// Which of a workgroup's rows a thread has part in.
template <int LANES>
__device__ __forceinline__ uint32_t row_of_block() {
  return LANES <= 16 ? threadIdx.x / LANES : LANES == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
}

// LANES 4, 16 or 64: 64, 16 or four rows to a workgroup.  Weights stay in registers from row to row.
template <typename T, int LANES, int N>
__global__ __launch_bounds__(256) void k_layer_norm(BlockArgs a) {
  constexpr int ALL = N * Piece<T>::W, ROWS = 256 / LANES;
  __shared__ float lds[2][4][2];
  const uint32_t lane = threadIdx.x % LANES;
  HeldRow<T, LANES, N> at(lane, a.dim);
  float w[ALL], b[ALL], x[ALL], r;
  typename HeldRow<T, LANES, N>::Raw next;
  const uint32_t rows = a.B * a.L * a.H, stride = gridDim.x * ROWS;   // (up to 2^31)
  uint32_t row = blockIdx.x * ROWS + row_of_block<LANES>();
  if (row < rows) at.load(row_at<T>(a.x, row, a), next);
  at.load_plain(a.weight, w, 1.0f);
  at.load_plain(a.bias, b, 0.0f);
  for (; row < rows; row += stride) {
    at.again();
    at.widen(next, x);
    if (row + stride < rows) at.load(row_at<T>(a.x, row + stride, a), next);
    standardise<T, LANES, N>(at, x, a, &r, lds);
#pragma unroll
    for (int i = 0; i < ALL; ++i) x[i] = fmaf(x[i] * r, w[i], b[i]);
    at.store(const_cast<T*>(row_at<T>(a.out, row, a)), x);
    if (LANES > 64) __syncthreads();
  }
}

// dx = r (h - mean h - xh mean(h xh)),  h = dout w,  xh = (x - mean) r;  the workgroup's sums of dout xh and of dout are left in `partial`.
template <typename T, int LANES, int N>
__global__ __launch_bounds__(256, 2) void k_layer_norm_back(BlockArgs a) {
  constexpr int W = Piece<T>::W, ALL = N * W, ROWS = 256 / LANES;
  __shared__ float lds[3][4][2];
  const uint32_t lane = threadIdx.x % LANES;
  HeldRow<T, LANES, N> at(lane, a.dim);
  float w[ALL], dw[ALL] = {}, db[ALL] = {}, x[ALL], d[ALL], r;
  typename HeldRow<T, LANES, N>::Raw next_x, next_d;
  const uint32_t rows = a.B * a.L * a.H, stride = gridDim.x * ROWS;   // (up to 2^31)
  uint32_t row = blockIdx.x * ROWS + row_of_block<LANES>();
  if (row < rows) {
    at.load(row_at<T>(a.x, row, a), next_x);
    at.load(row_at<T>(a.more, row, a), next_d);
  }
  at.load_plain(a.weight, w, 1.0f);
  for (; row < rows; row += stride) {
    at.again();
    at.widen(next_x, x);
    at.widen(next_d, d);
    if (row + stride < rows) {
      at.load(row_at<T>(a.x, row + stride, a), next_x);
      at.load(row_at<T>(a.more, row + stride, a), next_d);
    }
    standardise<T, LANES, N>(at, x, a, &r, lds);
#pragma unroll
    for (int i = 0; i < ALL; ++i) {
      x[i] *= r;
      dw[i] = fmaf(d[i], x[i], dw[i]);
      db[i] += d[i];
      d[i] *= w[i];
    }
    float sum = at.sum([&](int i) { return d[i]; }), along = at.sum([&](int i) { return d[i] * x[i]; });
    row_sums<LANES>(&sum, &along, lds[2]);
    sum /= (float)a.dim;
    along /= (float)a.dim;
#pragma unroll
    for (int i = 0; i < ALL; ++i) x[i] = r * (d[i] - sum - x[i] * along);
    at.store(const_cast<T*>(row_at<T>(a.out, row, a)), x);
    if (LANES > 64) __syncthreads();
  }
  // The waves' sums one after the other, lane by lane: element e of piece i of lane l at (i W + e) LANES + l, as k_norm_sums takes them.
  extern __shared__ float sums[];
  if (LANES < 64)
#pragma unroll
    for (int i = 0; i < ALL; ++i)
#pragma unroll
      for (int d = LANES; d < 64; d *= 2) {   // (the wave's rows)
        dw[i] += __shfl_xor(dw[i], d);
        db[i] += __shfl_xor(db[i], d);
      }
  constexpr int TURNS = LANES == 256 ? 1 : 4;
  const uint32_t wave = TURNS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int turn = 0; turn < TURNS; ++turn) {
    if (turn) __syncthreads();
    if (wave != (uint32_t)turn || (LANES < 64 && (threadIdx.x & 63) >= LANES)) continue;
    float* const to = (turn + 1 < TURNS ? sums : a.partial + (size_t)blockIdx.x * 2 * ALL * LANES) + lane;
#pragma unroll
    for (int i = 0; i < ALL; ++i) {
      to[i * LANES] = turn ? sums[i * LANES + lane] + dw[i] : dw[i];
      to[(ALL + i) * LANES] = turn ? sums[(ALL + i) * LANES + lane] + db[i] : db[i];
    }
  }
}

// Any width: a workgroup reads a row as often as it needs it, an element to a thread at a time; gradients add a row's part to the workgroup's own
// sums in memory.
template <typename T, bool BACK>
__global__ __launch_bounds__(256) void k_layer_norm_any(BlockArgs a) {
  __shared__ float lds[3][4][2];
  const uint32_t rows = a.B * a.L * a.H;
  float* const to = a.partial + (size_t)blockIdx.x * 2 * a.dim;
  if (BACK)
    for (uint32_t i = threadIdx.x; i < 2 * a.dim; i += 256) to[i] = 0.0f;
  __syncthreads();
  for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const T* x = row_at<T>(a.x, row, a);
    T* out = const_cast<T*>(row_at<T>(a.out, row, a));
    float sum = 0.0f, along = 0.0f;
    for (uint32_t i = threadIdx.x; i < a.dim; i += 256) sum += as_float(x[i]);
    row_sums<256>(&sum, &along, lds[0]);
    const float mean = sum / (float)a.dim;
    sum = along = 0.0f;
    for (uint32_t i = threadIdx.x; i < a.dim; i += 256) {
      const float y = as_float(x[i]) - mean;
      sum = fmaf(y, y, sum);
    }
    row_sums<256>(&sum, &along, lds[1]);
    const float r = 1.0f / sqrtf(sum / (float)a.dim + a.eps);
    if constexpr (BACK) {
      const T* d = row_at<T>(a.more, row, a);
      sum = along = 0.0f;
      for (uint32_t i = threadIdx.x; i < a.dim; i += 256) {
        const float y = (as_float(x[i]) - mean) * r, dy = as_float(d[i]), h = a.weight ? dy * a.weight[i] : dy;
        to[i] = fmaf(dy, y, to[i]);
        to[a.dim + i] += dy;
        sum += h;
        along = fmaf(h, y, along);
      }
      row_sums<256>(&sum, &along, lds[2]);
      sum /= (float)a.dim;
      along /= (float)a.dim;
      for (uint32_t i = threadIdx.x; i < a.dim; i += 256) {
        const float y = (as_float(x[i]) - mean) * r, dy = as_float(d[i]), h = a.weight ? dy * a.weight[i] : dy;
        out[i] = (T)(r * (h - sum - y * along));
      }
    } else {
      for (uint32_t i = threadIdx.x; i < a.dim; i += 256)
        out[i] = (T)fmaf((as_float(x[i]) - mean) * r, a.weight ? a.weight[i] : 1.0f, a.bias ? a.bias[i] : 0.0f);
    }
    __syncthreads();
  }
}

// The gradients of weight and bias from the sums that were left, in their order: 16 of them to a workgroup, 16 rows of sums at a time.  A row has
// `width` for the weight, then as many for the bias, by column (lanes 0) or by lane.
struct NormSums {
  const float* from;
  float *dweight, *dbias;
  uint32_t rows, dim, width, lanes, W;
};
__global__ __launch_bounds__(256) void k_norm_sums(NormSums p) {
  __shared__ float lds[16][17];
  const uint32_t c = threadIdx.x & 15, at = threadIdx.x >> 4, place = blockIdx.x * 16 + c, row = 2 * p.width;
  float sum = 0.0f;
  if (place < row) {
    const float* from = p.from + place;
    uint32_t i = at;
    for (; i + 7 * 16 < p.rows; i += 8 * 16) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = from[(size_t)(i + 16 * e) * row];
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += x[e];
    }
    for (; i < p.rows; i += 16) sum += from[(size_t)i * row];
  }
  lds[at][c] = sum;
  __syncthreads();
  if (at || place >= row) return;
  for (int i = 1; i < 16; ++i) sum += lds[i][c];
  uint32_t col = place % p.width;
  if (p.lanes) {
    const uint32_t k = col / p.lanes, first = (col % p.lanes + k / p.W * p.lanes) * p.W;
    col = (first + p.W <= p.dim ? first : p.dim - p.W) + k % p.W;
    if (first >= p.dim || col < first) return;
  }
  float* const to = place < p.width ? p.dweight : p.dbias;
  if (to) to[col] = sum;
}

// Philox4x32-10: four words of a counter and a key (Salmon et al., Parallel Random Numbers: As Easy as 1, 2, 3).
struct Words { uint32_t w[4]; };
__device__ __forceinline__ Words philox(uint64_t block, uint64_t offset, uint64_t seed) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Words{{c0, c1, c2, c3}};
}

// Eight elements to a thread: one block of random words.  PACKED: all tensors are packed, and end with a whole block but for the last thread's.
template <typename T, bool RESIDUAL, bool PACKED>
__global__ __launch_bounds__(256) void k_dropout(BlockArgs a, uint64_t n) {
  constexpr uint32_t W = Piece<T>::W;
  const uint64_t offset = a.offset + (a.d_offset ? (uint64_t)*a.d_offset : 0), blocks = (n + 7) / 8, stride = (uint64_t)gridDim.x * 256;
  const float factor = 65536.0f / (float)(65536u - a.border);
  for (uint64_t block = (uint64_t)blockIdx.x * 256 + threadIdx.x; block < blocks; block += stride) {
    const uint64_t first = block * 8;
    const uint32_t count = n - first < 8 ? (uint32_t)(n - first) : 8;
    auto kept_of = [&](const Words& r, uint32_t e) { return ((r.w[e / 2] >> (16 * (e & 1))) & 0xFFFFu) >= a.border; };
    if (PACKED && count == 8) {
      typename Piece<T>::Vec x[8 / W], y[8 / W];
#pragma unroll
      for (uint32_t i = 0; i < 8 / W; ++i) {
        x[i] = *reinterpret_cast<const typename Piece<T>::Loose*>(static_cast<const T*>(a.x.d) + first + i * W);
        if (RESIDUAL) y[i] = *reinterpret_cast<const typename Piece<T>::Loose*>(static_cast<const T*>(a.more.d) + first + i * W);
      }
      const Words r = philox(block, offset, a.seed);
#pragma unroll
      for (uint32_t i = 0; i < 8 / W; ++i) {
#pragma unroll
        for (uint32_t e = 0; e < W; ++e) {
          const float o = kept_of(r, i * W + e) ? as_float(x[i][e]) * factor : 0.0f;
          x[i][e] = (T)(RESIDUAL ? as_float(y[i][e]) + o : o);
        }
        *reinterpret_cast<typename Piece<T>::Loose*>(static_cast<T*>(a.out.d) + first + i * W) = x[i];
      }
      continue;
    }
    const Words r = philox(block, offset, a.seed);
    uint32_t row = (uint32_t)(first / a.dim);
    uint32_t col = (uint32_t)(first % a.dim);
    // (unrolled: words that are indexed by a number would lie in memory)
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
      if (e < count) {
        const float o = kept_of(r, e) ? as_float(row_at<T>(a.x, row, a)[col]) * factor : 0.0f;
        const_cast<T*>(row_at<T>(a.out, row, a))[col] = (T)(RESIDUAL ? as_float(row_at<T>(a.more, row, a)[col]) + o : o);
      }
      if (++col == a.dim) {
        col = 0;
        ++row;
      }
    }
  }
}
