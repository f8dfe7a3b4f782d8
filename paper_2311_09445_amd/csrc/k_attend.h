// One pass of linear attention over sequences (see seq_attention.hip for what the passes are), on the matrix cores.
// Part of seq_attention.hip (included inside namespace per); not a stand-alone header.
//
// A sequence is taken in chunks of 32 tokens.  With S the state before a chunk, f_i = c_out decay^(i+1-lag) and
// w_j = c_state decay^(n-1-j+lag) for the n tokens of the chunk,
//   out = diag(f) X S + (c_in X Y^T . decay^(i-j) for j <= i) Z,     S <- decay^n S + Y^T diag(w) Z.
// Everything is computed transposed (out^T = S^T X^T + ...), because then what one product leaves in registers is what the next
// one reads.  The 16 x 16 result of a matrix instruction holds, in lane 16 g + m, column m and rows 4 g .. 4 g + 3; a 32-deep operand
// holds column (or row) m and eight places of the inner dimension, whichever, if both operands take the same.  So two results
// stacked are an operand: S^T, and the decayed products of pairs.  Which row of the state is which place of dx is free too: row
// 4 g + r of tile 2 k + s is place 32 k + 8 g + 4 s + r, so that the operand it meets is eight elements in a row; the columns of a
// wave's two tiles are mixed likewise, so that a lane ends up with eight outputs in a row.
//
// A wave holds 16 NT columns of the state for all of dx in registers; the waves of a workgroup share the chunk's rows in LDS, and
// each works out the products of pairs for itself (3 tiles; sharing them would cost a barrier).  A gradient's workgroup may hold
// several heads that share a key and value, a team of waves each with rows of its own in LDS; what they bring to the shared output is
// added up in LDS, in the heads' order, behind one more barrier.
//
// Rows lie in LDS in pieces of 16 bytes, piece p of row r at place p ^ turn(r), so that reads along rows and across them meet the
// banks evenly without padding; memory can then be loaded straight into LDS, 64 pieces an instruction, several chunks ahead
// (DIRECT: bfloat16, rows made of pieces).  Rows in fp32, which are taken apart on the way, and rows of odd widths or alignments go
// through registers in pieces, two chunks ahead (PIECES); rows narrower than a piece or far apart one by one (ELEMENTS).

// What bounds it.  A workgroup by itself takes 0.8 us a chunk of 64 x 64 in bfloat16, 1.9 of 128 x 128: the chain from its barrier
// through LDS and two rounds of matrix instructions.  With the chip full it is memory: 768 workgroups of 64 x 64, three to a compute
// unit, take 2.8 us for a chunk each (4.5 TB/s), 2.7 without any of the products, 1.6 without the outputs; 65536 tokens of 16 heads of
// 128 x 128 take 255 us (4.2 TB/s; the least of 40 launches 231) behind 155 for their segments' states.

enum Way { ELEMENTS, PIECES, DIRECT };

// The column of the wave's that column m of tile c is.
template <int NT>
__device__ __forceinline__ uint32_t state_column(uint32_t c, uint32_t m) { return NT == 2 ? 8 * (m >> 2) + 4 * c + (m & 3) : 16 * c + m; }

// What a wave's lane adds to the state, Z^T w: in 32 bits, or in bfloat16 as operands whose sum holds 16 bits of it, 24 with the
// third.  (The state is fp32 whatever the rows are; where only rows in bfloat16 come of it, 16 bits lose nothing that shows.)
template <typename T>
struct Scaled;
template <>
struct Scaled<float> {
  Operand<float> part;
  __device__ __forceinline__ Scaled(const Operand<float>& z, const f32x4& w0, const f32x4& w1) {
    f32x4 a, b;
    z.widen(&a, &b);
    part = Operand<float>::of(a * w0, b * w1);
  }
  template <int TX>
  __device__ __forceinline__ void add(const Operand<float> (&y)[TX], f32x4 (&s)[TX], bool) const {
#pragma unroll
    for (int a = 0; a < TX; ++a) s[a] = Operand<float>::mma(y[a], part, s[a]);
  }
};
template <>
struct Scaled<bf16> {
  Operand<bf16> part[2];
  f32x4 rest0, rest1;
  __device__ __forceinline__ Scaled(const Operand<bf16>& z, const f32x4& w0, const f32x4& w1) {
    f32x4 u, v;
    z.widen(&rest0, &rest1);
    rest0 *= w0;
    rest1 *= w1;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      part[t] = Operand<bf16>::of(rest0, rest1);
      part[t].widen(&u, &v);
      rest0 -= u;
      rest1 -= v;
    }
  }
  template <int TX>
  __device__ __forceinline__ void add(const Operand<bf16> (&y)[TX], f32x4 (&s)[TX], bool exact) const {
    if (exact) {
      const Operand<bf16> third = Operand<bf16>::of(rest0, rest1);
#pragma unroll
      for (int a = 0; a < TX; ++a) s[a] = Operand<bf16>::mma(y[a], third, s[a]);
    }
#pragma unroll
    for (int a = 0; a < TX; ++a) s[a] = Operand<bf16>::mma(y[a], part[1], s[a]);
#pragma unroll
    for (int a = 0; a < TX; ++a) s[a] = Operand<bf16>::mma(y[a], part[0], s[a]);
  }
};

// The same straight into LDS, in bfloat16.  A wave's instruction fills 64 places one behind the other: 1 KiB of the chunk's tiles, which lie one
// behind the other too; the waves take these in turn.  Which piece belongs there is the lane's business: it asks for that one.
struct Fill {
  const uint8_t* base;   // (uniform) of the next chunk that is asked for
  int64_t step;          // (uniform) bytes to the one after it
  uint32_t offset;       // of the lane's piece within the chunk
  uint32_t row;          // of the chunk; kNoRow: a column behind the width
};
constexpr uint32_t kNoRow = 1u << 16;

template <typename T, int D>
__device__ __forceinline__ void fill_piece(Fill* d, const SeqRows& r, const T* head, uint32_t place, int64_t token, bool back, uint32_t col0, uint32_t width) {
  constexpr uint32_t PER_ROW = Tile<D>::PIECES, W = 8;
  const uint32_t row = place / PER_ROW, piece = place % PER_ROW ^ Tile<D>::turn(row);
  const int64_t bytes = r.token * (int64_t)sizeof(T);
  d->base = reinterpret_cast<const uint8_t*>(head + col0) + token * bytes;
  d->step = (back ? -(int64_t)kChunk : (int64_t)kChunk) * bytes;
  d->offset = (back ? kChunk - 1 - row : row) * (uint32_t)bytes + piece * 16;
  d->row = col0 + piece * W < width ? row : kNoRow;
}

// Bytes of a chunk's tiles, and how many chunks are held.  (The address that loads to LDS go to has 16 bits.)
template <typename T, int DX, int DZ, bool OUT>
constexpr uint32_t chunk_bytes() { return kChunk * ((OUT ? 2 : 1) * DX + DZ) * kParts<T> * sizeof(bf16); }
template <typename T, int DX, int DZ, bool OUT, Way WAY>
constexpr uint32_t ring() {
  if (WAY != DIRECT) return 2;
  const uint32_t n = 65536 / chunk_bytes<T, DX, DZ, OUT>();
  return n < 4 ? n : 4;
}

// A lane's outputs of one token, NT times four side by side, `left` elements before the end of the row.
template <typename O, int NT>
__device__ __forceinline__ void store_row(uint8_t* at, const f32x4 (&acc)[NT][2], int d, uint32_t left) {
  typedef O Vec __attribute__((ext_vector_type(4 * NT)));
  typedef Vec Loose __attribute__((aligned(sizeof(O))));
  O* const to = reinterpret_cast<O*>(at);
  if (left >= 4 * NT) {
    Vec o;
#pragma unroll
    for (int i = 0; i < 4 * NT; ++i) o[i] = (O)acc[i / 4][d][i % 4];
    *reinterpret_cast<Loose*>(to) = o;
    return;
  }
#pragma unroll
  for (uint32_t i = 0; i < 4 * NT; ++i)
    if (i < left) to[i] = (O)acc[i / 4][d][i % 4];
}
// The same where rows are whole pieces, as one instruction (two in fp32 and NT = 2): they are counted.  The compiler does not see
// that it is a store, so the wait states are here: behind it one, for its registers, which what follows may write; before it five, for
// its scalar registers, or 16 where its values come straight out of a matrix instruction (8 passes and 3).
template <bool STRAIGHT, typename V>
__device__ __forceinline__ void store_counted(uint8_t* base, uint32_t offset, const V& v) {
  if constexpr (STRAIGHT) asm volatile("s_nop 15\n\tglobal_store_dwordx4 %0, %1, %2\n\ts_nop 0" ::"v"(offset), "v"(v), "s"(base) : "memory");
  else if constexpr (sizeof(V) == 16) asm volatile("s_nop 4\n\tglobal_store_dwordx4 %0, %1, %2\n\ts_nop 0" ::"v"(offset), "v"(v), "s"(base) : "memory");
  else asm volatile("s_nop 4\n\tglobal_store_dwordx2 %0, %1, %2\n\ts_nop 0" ::"v"(offset), "v"(v), "s"(base) : "memory");
}
template <typename O, int NT>
__device__ __forceinline__ void store_row_counted(uint8_t* base, uint32_t offset, const f32x4 (&acc)[NT][2], int d) {
  if constexpr (sizeof(O) == 4) {
#pragma unroll
    for (int c = 0; c < NT; ++c) store_counted<true>(base, offset + 16 * c, acc[c][d]);
  } else {
    typedef O Vec __attribute__((ext_vector_type(4 * NT)));
    Vec o;
#pragma unroll
    for (int i = 0; i < 4 * NT; ++i) o[i] = (O)acc[i / 4][d][i % 4];
    store_counted<false>(base, offset, o);
  }
}

// Bytes of LDS: of a team's chunks, and of the outputs that teams add up.
template <typename T, int DX, int NT, int WAVES, bool OUT, Way WAY>
constexpr uint32_t team_bytes() { return ring<T, DX, 16 * NT * WAVES, OUT, WAY>() * chunk_bytes<T, DX, 16 * NT * WAVES, OUT>(); }
template <typename T, int DX, int NT, int WAVES, bool OUT, Way WAY, int TEAMS>
constexpr uint32_t lds_bytes() { return TEAMS * (team_bytes<T, DX, NT, WAVES, OUT, WAY>() + (TEAMS > 1 ? 2 * NT * WAVES * 1024 : 0)); }

// OUT: the outputs are wanted too (else only the state that the piece of the sequence brings, from zeros).
// TEAMS: heads of a workgroup, each a team of WAVES waves; a pass that is `summed` has one output for them.
template <typename T, int DX, int NT, int WAVES, bool OUT, Way WAY, int TEAMS>
__global__ __launch_bounds__(64 * WAVES * TEAMS, sizeof(T) == 4 && DX == 128 && OUT ? 1 : 2) void k_attend(AttentionPasses all) {
  constexpr int THREADS = 64 * WAVES, DZ = 16 * NT * WAVES, TX = DX / 16, KX = DX / 32;
  constexpr uint32_t BUFFER = chunk_bytes<T, DX, DZ, OUT>() / sizeof(bf16), RING = ring<T, DX, DZ, OUT, WAY>();
  extern __shared__ __attribute__((aligned(256))) uint8_t lds_raw[];
  const uint32_t team = TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.y) : 0;
  bf16* const lds = reinterpret_cast<bf16*>(lds_raw + team * team_bytes<T, DX, NT, WAVES, OUT, WAY>());
  f32x4* const sums = reinterpret_cast<f32x4*>(lds_raw + TEAMS * team_bytes<T, DX, NT, WAVES, OUT, WAY>());
  // Workgroups go round the 8 dies by their number: the passes over the same rows sit on one die.  (That spares little reading: those of
  // keys and values run against time, that of queries with it, and 2 x 16384 tokens of 16 heads of 128 x 128 miss L2 for 1.5 GB, where
  // nine readings and three writings by themselves are 1.6.)
  const uint32_t which = blockIdx.x / 8 % all.count, item = blockIdx.x / (8 * all.count) * 8 + blockIdx.x % 8;
  if (item >= all.items) return;
  const AttentionPass& p = all.pass[which];
  const uint32_t slice = item % all.slices, seg = item / all.slices % all.run, bh = item / all.slices / all.run * TEAMS + team;
  const uint32_t h = bh % p.H, b = bh / p.H, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (what the loop needs of the arguments is taken out of them here: behind its barriers they would be loaded again)
  const uint32_t L = p.L, dx = p.dx, dz = p.dz, segment = all.segment;
  const float decay = p.log_decay[h], c_state = p.c_state;
  const bool back = p.back != 0, out_f32 = p.out_f32 != 0;
  const bool last = OUT && p.to && seg + 1 == all.segments, exact = p.exact && (last || !OUT);   // (its state is an output)
  const bool summed = TEAMS > 1 && p.summed;
  const int lag = back ? 1 : 0;
  const uint32_t valid = valid_tokens(p.lengths, b, L), start = seg * segment;
  const uint32_t end = valid < start ? start : valid - start < segment ? valid : start + segment;
  const uint32_t col0 = slice * DZ, col = col0 + wave * 16 * NT;   // first z column of the workgroup, of the wave
  if (col0 >= dz) return;   // (a pass narrower than the launch's widest)

  f32x4 S[NT][TX];
#pragma unroll
  for (int a = 0; a < TX; ++a)
#pragma unroll
    for (int c = 0; c < NT; ++c) S[c][a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // A state out of memory (all asked for at once: places behind a width take the last one's, and are cleared when all are there).
  auto load = [&](const float* in, f32x4 (&to)[NT][TX]) __attribute__((always_inline)) {
    const uint32_t in_x = p.in_x, in_z = p.in_z;
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const uint32_t j = col + state_column<NT>(c, m), at = (j < dz ? j : dz - 1) * in_z;
#pragma unroll
      for (int a = 0; a < TX; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t i = state_row(a, 4 * g + r);
          to[c][a][r] = in[(i < dx ? i : dx - 1) * in_x + at];
        }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
      for (int a = 0; a < TX; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float s = to[c][a][r];
          asm("" : "+v"(s));   // (the load stays above: moved into the choice each would be waited for by itself)
          to[c][a][r] = state_row(a, 4 * g + r) < dx && col + state_column<NT>(c, m) < dz ? s : 0.0f;
        }
  };
  if (OUT && p.in) load(p.in + (int64_t)b * p.in_batch + (int64_t)h * p.in_head + (int64_t)seg * p.in_segment, S);

  const T* const xh = OUT ? row_of<T>(p.x, b, 0, h) : nullptr;
  const T* const yh = row_of<T>(p.y, b, 0, h);
  const T* const zh = row_of<T>(p.z, b, 0, h);
  const uint32_t out_size = out_f32 ? 4 : sizeof(T);
  const int64_t out_step = p.out.token * (int64_t)out_size;
  const bool out_near = WAY != ELEMENTS || p.out.near, out_wide = WAY == DIRECT || p.out.wide;
  uint8_t* const oh = OUT ? static_cast<uint8_t*>(p.out.d) + ((int64_t)b * p.out.batch + (int64_t)(h / p.out.share) * p.out.head) * out_size : nullptr;
  // Chunks on their way: staged in registers, or counted instructions that fill LDS.
  struct Rows {
    Staged<T, DX, WAY == DIRECT ? 1 << 20 : THREADS> x, y;
    Staged<T, DZ, WAY == DIRECT ? 1 << 20 : THREADS> z;
  } staged[2];
  constexpr uint32_t FILLS_X = OUT ? Tile<DX>::PIECES / 2 : 0, FILLS_Y = Tile<DX>::PIECES / 2, FILLS = FILLS_X + FILLS_Y + Tile<DZ>::PIECES / 2;
  constexpr uint32_t MINE = (FILLS + WAVES - 1) / WAVES;
  Fill fill[WAY == DIRECT ? MINE : 1];
  const bool whole = dx == DX && dz - col0 >= DZ;   // no piece lies behind a width
  const bool ends = dx % (16 / sizeof(T)) || dz % (16 / sizeof(T));
  const int64_t token0 = back ? (int64_t)valid - (int64_t)start - (int64_t)kChunk : (int64_t)start;   // lowest of the first chunk
  if (WAY == DIRECT) {
#pragma unroll
    for (uint32_t k = 0; k < MINE; ++k) {
      const uint32_t f = wave + WAVES * k;
      fill[k].row = kNoRow;
      if (f < FILLS_X) fill_piece<T, DX>(&fill[k], p.x, xh, f * 64 + lane, token0, back, 0, dx);
      else if (f < FILLS_X + FILLS_Y) fill_piece<T, DX>(&fill[k], p.y, yh, (f - FILLS_X) * 64 + lane, token0, back, 0, dx);
      else if (f < FILLS) fill_piece<T, DZ>(&fill[k], p.z, zh, (f - FILLS_X - FILLS_Y) * 64 + lane, token0, back, col0, dz);
    }
  }
  // Asks for the chunk from token `first` on (the chunks one after the other), to go to registers or to a place of the ring.
  auto fetch = [&](uint32_t first, uint32_t slot, Rows& to_rows) {
    const uint32_t n = first < end ? (end - first < kChunk ? end - first : kChunk) : 0;
    if (WAY == ELEMENTS) {
      if (OUT) to_rows.x.load(p.x, xh, first, n, valid, back, 0, dx);
      to_rows.y.load(p.y, yh, first, n, valid, back, 0, dx);
      to_rows.z.load(p.z, zh, first, n, valid, back, col0, dz);
      return;
    }
    if (WAY == PIECES) {
      if (OUT) to_rows.x.load_pieces(p.x, xh, first, end, valid, back, 0, dx);
      to_rows.y.load_pieces(p.y, yh, first, end, valid, back, 0, dx);
      to_rows.z.load_pieces(p.z, zh, first, end, valid, back, col0, dz);
      return;
    }
    const uint32_t to = slot * BUFFER * (uint32_t)sizeof(bf16) + wave * 1024;
    if (whole && n == kChunk) {
#pragma unroll
      for (uint32_t k = 0; k < MINE; ++k)
        if (FILLS % WAVES == 0 || wave + WAVES * k < FILLS) load_to_lds(to + WAVES * k * 1024, fill[k].base, fill[k].offset);
    } else {
#pragma unroll
      for (uint32_t k = 0; k < MINE; ++k) {
        if (FILLS % WAVES && wave + WAVES * k >= FILLS) continue;
        if (fill[k].row < n) load_to_lds(to + WAVES * k * 1024, fill[k].base, fill[k].offset);
        else *reinterpret_cast<f32x4*>(lds_raw + to + WAVES * k * 1024 + 16 * lane) = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
#pragma unroll
    for (uint32_t k = 0; k < MINE; ++k) fill[k].base += fill[k].step;
  };

  // Powers of the decay: lane e works out decay^e, the others ask it for what they need.  Between the tokens of a pair (same tile; a
  // tile apart), to the chunk's tokens, from them, over the chunk.
  const float power = lane == 0 ? 1.0f : expf((float)lane * decay);
  f32x4 pair[2], into[2];
  float outof[2];
  Keep keep{0.0f, false};
  if (OUT) {
#pragma unroll
    for (int d = 0; d < 2; ++d) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = 16 * d + (int)m - (int)(4 * g) - r;
        const float w = p.c_in * __shfl(power, e < 0 ? 0 : e);
        pair[d][r] = e < 0 ? 0.0f : w;
      }
      outof[d] = p.c_out * __shfl(power, 16 * d + (int)m + 1 - lag);
    }
  }
  auto weights = [&](int n) {
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = n - 1 - 16 * d - (int)(4 * g) - r;
        const float w = c_state * __shfl(power, e < 0 ? 0 : e + lag);
        into[d][r] = e < 0 ? 0.0f : w;
      }
    keep = keeps((float)n * decay);
    keep.half = __builtin_amdgcn_readfirstlane(keep.half);   // (the same in all lanes: a branch, not a choice for each element)
  };
  weights(kChunk);

  const bool stores = col < dz;           // the wave has outputs to store
  float worst = 0.0f;                     // not a number: one of the wave's outputs was none
  // One chunk: its rows into LDS, or in LDS, and those of a later one asked for; then its products.
  constexpr uint32_t AHEAD = WAY == DIRECT ? RING - 1 : WAY == PIECES ? 2 : 1;   // chunks asked for before the one at hand
  auto chunk = [&](uint32_t first, uint32_t slot, Rows& rows) __attribute__((always_inline)) {
    bf16* const xs = lds + slot * BUFFER;
    bf16* const ys = OUT ? xs + kParts<T> * Tile<DX>::SIZE : xs;
    bf16* const zs = ys + kParts<T> * Tile<DX>::SIZE;
    if (WAY == DIRECT) {
      // Behind the wave's parts of this chunk are those of the next RING - 2, at least FILLS / WAVES instructions each if they are
      // whole, and the outputs of the last RING - 1, two rows each.  That many may be left; towards the end none.
      constexpr int LOADS = (int)((RING - 2) * (FILLS / WAVES)), STORES = OUT ? 2 * (int)(RING - 1) : 0;
      if (end - first < (RING - 1) * kChunk) arrive<0>();
      else if (!OUT || !stores || first - start < (RING - 1) * kChunk) arrive<LOADS>();
      else if (NT == 2 && out_f32) arrive<LOADS + 2 * STORES>();
      else arrive<LOADS + STORES>();
      // (this barrier: all are through with the chunk before, whose place the next one takes)
      if (first + AHEAD * kChunk < end) fetch(first + AHEAD * kChunk, slot == 0 ? RING - 1 : slot - 1, rows);
    } else {
      if (WAY == PIECES && (!whole || end - first < kChunk)) {
        if (OUT) rows.x.clear(end - first, 0, dx);
        rows.y.clear(end - first, 0, dx);
        rows.z.clear(end - first, col0, dz);
      }
      if (OUT) rows.x.store(xs);
      rows.y.store(ys);
      rows.z.store(zs);
      if (WAY == PIECES && ends) {   // (behind the whole places, by the same lanes)
        if (OUT) rows.x.store_ends(xs, dx);
        rows.y.store_ends(ys, dx);
        rows.z.store_ends(zs, dz - col0);
      }
      __syncthreads();
      if (WAY == PIECES || first + AHEAD * kChunk < end) fetch(first + AHEAD * kChunk, 0, rows);
    }
    const uint32_t n = end - first < kChunk ? end - first : kChunk;
    if (n < kChunk) weights((int)n);

    Operand<T> z[NT], y[TX];
#pragma unroll
    for (int c = 0; c < NT; ++c) z[c] = Operand<T>::template across<DZ>(zs, [&](uint32_t i) { return wave * 16 * NT + state_column<NT>(c, i); }, m, g);
    f32x4 acc[NT][2];
    if (OUT) {
      f32x4 pt[3];
      const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < NT; ++c) acc[c][0] = acc[c][1] = zero;
      pt[0] = pt[1] = pt[2] = zero;
#pragma unroll
      for (int k = 0; k < KX; ++k) {
        const Operand<T> x0 = Operand<T>::template along<DX>(xs, m, k, g), x1 = Operand<T>::template along<DX>(xs, 16 + m, k, g);
        const Operand<T> y0 = Operand<T>::template along<DX>(ys, m, k, g), y1 = Operand<T>::template along<DX>(ys, 16 + m, k, g);
        pt[0] = Operand<T>::mma(y0, x0, pt[0]);
        pt[1] = Operand<T>::mma(y0, x1, pt[1]);
        pt[2] = Operand<T>::mma(y1, x1, pt[2]);
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          const Operand<T> s = Operand<T>::of(S[c][2 * k], S[c][2 * k + 1]);
          acc[c][0] = Operand<T>::mma(s, x0, acc[c][0]);
          acc[c][1] = Operand<T>::mma(s, x1, acc[c][1]);
        }
      }
      const Operand<T> p0 = Operand<T>::of(pt[0] * pair[0], zero), p1 = Operand<T>::of(pt[1] * pair[1], pt[2] * pair[0]);
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        acc[c][0] = Operand<T>::mma(z[c], p0, acc[c][0] * outof[0]);
        acc[c][1] = Operand<T>::mma(z[c], p1, acc[c][1] * outof[1]);
      }
    }
#pragma unroll
    for (int a = 0; a < TX; ++a) y[a] = Operand<T>::template across<DX>(ys, [&](uint32_t i) { return state_row(a, i); }, m, g);
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const Scaled<T> zw(z[c], into[0], into[1]);
      if (keep.half) {
#pragma unroll
        for (int a = 0; a < TX; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) S[c][a][r] = kept(S[c][a][r], Keep{keep.factor, true});
      } else {
#pragma unroll
        for (int a = 0; a < TX; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) S[c][a][r] = kept(S[c][a][r], Keep{keep.factor, false});
      }
      zw.add(y, S[c], exact);
    }
    if (!OUT) return;
    if (TEAMS > 1 && summed) {   // (the next chunk's barrier is between these reads and its sums)
      f32x4* const mine = sums + wave * 64 + lane;
      constexpr uint32_t TILE = WAVES * 64, TEAM = 2 * NT * TILE;
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int d = 0; d < 2; ++d) mine[team * TEAM + (2 * c + d) * TILE] = acc[c][d];
      __syncthreads();
      if (team >= 2) return;   // the first two teams add up and store a tile of tokens each
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          if (team != (uint32_t)d) continue;
          acc[c][d] = mine[(2 * c + d) * TILE];
#pragma unroll
          for (int other = 1; other < TEAMS; ++other) acc[c][d] += mine[other * TEAM + (2 * c + d) * TILE];
        }
    }
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) worst = __builtin_elementwise_maximum(worst, acc[c][d][r]);
    // out: four columns of a token in each tile of a lane, eight side by side in two
    const uint32_t j = col + (NT == 2 ? 8 : 4) * g;
    uint8_t* const base = oh + (back ? (int64_t)valid - (int64_t)first - (int64_t)kChunk : (int64_t)first) * out_step;
    if (WAY == DIRECT) {
      const uint32_t lower = (back ? kChunk - 1 - m : m) * (uint32_t)out_step + j * out_size;
      const uint32_t upper = lower + (back ? -16 : 16) * (uint32_t)out_step;
      if (out_f32) {
        if (m < n && j < dz) store_row_counted<float, NT>(base, lower, acc, 0);
        if (16 + m < n && j < dz) store_row_counted<float, NT>(base, upper, acc, 1);
      } else {
        if (m < n && j < dz) store_row_counted<T, NT>(base, lower, acc, 0);
        if (16 + m < n && j < dz) store_row_counted<T, NT>(base, upper, acc, 1);
      }
    } else if (out_near) {
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const uint32_t row = 16 * d + m;
        uint8_t* const at = base + ((back ? kChunk - 1 - row : row) * (uint32_t)out_step + j * out_size);
        if (row >= n || j >= dz || (summed && team != (uint32_t)d)) continue;
        if (out_f32) store_row<float, NT>(at, acc, d, dz - j);
        else store_row<T, NT>(at, acc, d, dz - j);
      }
    } else {
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const uint32_t row = 16 * d + m, i = first + row, t = back ? valid - 1 - i : i;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t e = col + state_column<NT>(c, 4 * g + r);
            if (row >= n || e >= dz || (summed && team != (uint32_t)d)) continue;
            if (out_f32) row_to<float>(p.out, b, t, h)[e] = acc[c][d][r];
            else row_to<T>(p.out, b, t, h)[e] = (T)acc[c][d][r];
          }
        }
    }
  };

  // The recurrence itself, token by token, over what the chunks have computed: for pieces of a sequence with values that are not
  // finite.  The product with Z takes each token of a chunk to all of them, with weight zero to those before it, and zero times such a
  // value is not zero.  That shows as outputs that are not numbers, which a chunk takes a maximum of (1 % of its time; looking at Z
  // before the product instead held up each chunk by up to 0.1 us).
  auto recur = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the stores that the compiler does not see)
#pragma unroll
    for (int a = 0; a < TX; ++a)
#pragma unroll
      for (int c = 0; c < NT; ++c) S[c][a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (p.in) load(p.in + (int64_t)b * p.in_batch + (int64_t)h * p.in_head + (int64_t)seg * p.in_segment, S);
    const Keep once = keeps(decay);
    float* const shared = reinterpret_cast<float*>(sums);
    for (uint32_t i = start; i < end; ++i) {
      const uint32_t t = back ? valid - 1 - i : i;
      const T *xr = xh + (int64_t)t * p.x.token, *yr = yh + (int64_t)t * p.y.token, *zr = zh + (int64_t)t * p.z.token;
      float zc[NT], sum[NT];
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        const uint32_t j = col + state_column<NT>(c, m);
        zc[c] = j < dz ? c_state * (float)zr[j] : 0.0f;
        sum[c] = 0.0f;
      }
#pragma unroll
      for (int a = 0; a < TX; ++a) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t row = state_row(a, 4 * g + r);
          if (row >= dx) continue;
          const float xv = (float)xr[row], yv = (float)yr[row];
#pragma unroll
          for (int c = 0; c < NT; ++c) {   // (against time what a token adds is decayed with the rest, behind its output)
            const float now = fmaf(yv, zc[c], back ? S[c][a][r] : kept(S[c][a][r], once));
            sum[c] = fmaf(xv, now, sum[c]);
            S[c][a][r] = back ? kept(now, once) : now;
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        sum[c] += __shfl_xor(sum[c], 16);
        sum[c] = p.c_out * (sum[c] + __shfl_xor(sum[c], 32));
      }
      const uint32_t place = wave * 16 * NT;
      if (TEAMS > 1 && summed) {
#pragma unroll
        for (int c = 0; c < NT; ++c)
          if (g == 0) shared[team * DZ + place + state_column<NT>(c, m)] = sum[c];
        __syncthreads();
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          sum[c] = shared[place + state_column<NT>(c, m)];
#pragma unroll
          for (int other = 1; other < TEAMS; ++other) sum[c] += shared[other * DZ + place + state_column<NT>(c, m)];
        }
        __syncthreads();
        if (team > 0) continue;
      }
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        const uint32_t j = col + state_column<NT>(c, m);
        if (g != 0 || j >= dz) continue;
        if (out_f32) row_to<float>(p.out, b, t, h)[j] = sum[c];
        else row_to<T>(p.out, b, t, h)[j] = (T)sum[c];
      }
    }
  };

  if (WAY == DIRECT) {
#pragma unroll
    for (uint32_t i = 0; i < AHEAD; ++i)
      if (start + i * kChunk < end) fetch(start + i * kChunk, i, staged[0]);
    for (uint32_t first = start, slot = 0; first < end; first += kChunk, slot = slot + 1 == RING ? 0 : slot + 1) chunk(first, slot, staged[0]);
  } else if (WAY == PIECES) {
    if (start < end) {
      fetch(start, 0, staged[0]);
      fetch(start + kChunk, 0, staged[1]);
    }
    for (uint32_t first = start; first < end; first += 2 * kChunk) {
      chunk(first, 0, staged[0]);
      if (first + kChunk < end) chunk(first + kChunk, 1, staged[1]);
    }
  } else {
    fetch(start, 0, staged[0]);
    for (uint32_t first = start, slot = 0; first < end; first += kChunk, slot ^= 1) chunk(first, slot, staged[0]);
  }

  if (OUT) {
    bool again = __any(worst != worst);
    if (TEAMS > 1 && summed) {   // (the teams' outputs are one: all or none)
      uint32_t* const seen = reinterpret_cast<uint32_t*>(sums);
      arrive<0>();
      if (lane == 0) seen[team * WAVES + wave] = again;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < TEAMS * WAVES; ++i) again = again || seen[i];
      again = __builtin_amdgcn_readfirstlane(again);
      __syncthreads();
    }
    if (__builtin_expect(again, 0)) recur();
  }
  if (last || !OUT) {
    float* const S_out = OUT ? p.to + (int64_t)b * p.to_batch + (int64_t)h * p.to_head : p.part + ((size_t)bh * all.segments + seg) * dx * dz;
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const uint32_t j = col + state_column<NT>(c, m);
      if (j >= dz) continue;
      float* const at = S_out + 8 * g * dz + j;
#pragma unroll
      for (int a = 0; a < TX; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (dx == DX || state_row(a, 4 * g + r) < dx) at[state_row(a, r) * dz] = S[c][a][r];
    }
  }
  if (!OUT || valid >= L || (summed && team > 0)) return;
  // tokens behind the valid ones: zeros
  const uint32_t width = dz - col0 < (uint32_t)DZ ? dz - col0 : DZ, from = start > valid ? start : valid;
  const uint32_t until = L - start < segment ? L : start + segment;
  const uint32_t piece = 16 / out_size, pieces = out_wide && width % piece == 0 ? width / piece : 0;
  if (pieces) {
    const uint32_t rows = THREADS / pieces, row = threadIdx.x / pieces;
    uint8_t* at = oh + (int64_t)(from + row) * out_step + (col0 * out_size + threadIdx.x % pieces * 16);
    if (row < rows)
      for (uint32_t t = from + row; t < until; t += rows, at += rows * out_step) *reinterpret_cast<f32x4*>(at) = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  } else {
    for (uint32_t t = from + wave; t < until; t += WAVES)
      for (uint32_t j = lane; j < width; j += 64) {
        if (out_f32) row_to<float>(p.out, b, t, h)[col0 + j] = 0.0f;
        else row_to<T>(p.out, b, t, h)[col0 + j] = (T)0.0f;
      }
  }
}

// The states that the segments of a sequence start from, from what each of those before brings, in place.
__global__ __launch_bounds__(256) void k_join(JoinPasses all) {
  const JoinPass& p = all.pass[blockIdx.y];
  const uint32_t per = p.dx * p.dz;
  const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (uint64_t)all.BH * per) return;
  const uint32_t bh = (uint32_t)(at / per), e = (uint32_t)(at % per), h = bh % all.H, b = bh / all.H;
  const uint32_t valid = valid_tokens(all.lengths, b, all.L), last = all.segments - 1;
  const float g = all.log_decay[h];
  float S = p.in ? p.in[(int64_t)b * p.in_batch + (int64_t)h * p.in_head + e] : 0.0f;
  float* part = p.part + (size_t)bh * all.segments * per + e;
  for (uint32_t s0 = 0; s0 < last; s0 += 8) {
    float brought[8];
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) brought[k] = s0 + k < last ? part[(size_t)(s0 + k) * per] : 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
      if (s0 + k >= last) break;
      part[(size_t)(s0 + k) * per] = S;
      const uint32_t begin = (s0 + k) * all.segment;
      const uint32_t n = valid <= begin ? 0 : valid - begin < all.segment ? valid - begin : all.segment;
      if (n) S = kept(S, keeps((float)n * g)) + brought[k];
    }
  }
  part[(size_t)last * per] = S;
}
