// What the kernels over chunks of a sequence share: rows as tiles in LDS, operands of the matrix instructions, what is left of a state.
#pragma once
#include "dev_seq.h"

namespace per {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kChunk = 32;

// Where row, piece of 32 rows of D elements of two bytes lies in LDS, in elements.
template <int D>
struct Tile {
  static constexpr uint32_t PIECES = D / 8, SIZE = kChunk * D;
  // What is read at once: 16 rows of one piece (along), for which the turns of 16 rows (those that share 256 bytes aside) differ; or
  // (across) rows 0 .. 7 of four pieces in a row.
  __device__ __forceinline__ static uint32_t turn(uint32_t row) {
    const uint32_t q = (row & 15) / (PIECES < 16 ? 16 / PIECES : 1);
    return PIECES >= 16 ? (q & 3) << 2 | q >> 2 : PIECES == 8 ? (q & 1) << 2 | q >> 1 : q;
  }
  __device__ __forceinline__ static uint32_t at(uint32_t row, uint32_t piece) { return row * D + (piece ^ turn(row)) * 8; }
};

// The place of the inner dimension that row m of tile a of a state is.
__device__ __forceinline__ uint32_t state_row(uint32_t a, uint32_t m) { return 32 * (a >> 1) + 8 * (m >> 2) + 4 * (a & 1) + (m & 3); }

// Operand of 16 x 32 places: 8 of the inner dimension per lane.  Where rows are bfloat16, what meets them (the state, the decayed
// products of pairs) is rounded to it once more as it becomes an operand.  In two parts each, outputs are off by 1.7e-3 as after one
// rounding, not 2.3e-3, but there are a third more matrix instructions and over half as many again of the others: 16 rows of 1024 tokens of 8
// heads of 128 x 128 45 -> 54 us and the gradient 89 -> 112, 2 x 16384 of 16 heads 395 -> 472, 32 x 512 of 64 x 64 21 -> 23.  Values in fp32 are taken apart into three in bfloat16, whose sum they
// are (8 bits each, cut off, not rounded: no part overflows), and products into six matrix instructions; the two products of 2^-24
// that are left out are of the size of fp32's own rounding.  (The matrix instructions of fp32 itself take 32 times as long as those of
// bfloat16, 5.3 times as long as six: a chunk of 64 x 64 took 3.1 us and takes 2.6, of 128 x 64 5.0 and 4.0.)  In LDS the parts are three tiles, one
// behind the other.
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Operand {
  static constexpr int PARTS = kParts<T>;
  bf16x8 v[PARTS];
  // A row of the tile, the inner dimension along it: 32 k + 8 g ..
  template <int D>
  __device__ __forceinline__ static Operand along(const bf16* tile, uint32_t row, uint32_t k, uint32_t g) {
    Operand o;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) o.v[i] = *reinterpret_cast<const bf16x8*>(tile + i * Tile<D>::SIZE + Tile<D>::at(row, 4 * k + g));
    return o;
  }
  // Columns column(0) .. column(15), of which four in a row are neighbours, the inner dimension across the 32 rows: a transposing
  // read, in which 16 lanes read 4 rows of 4 x 4 elements.
  template <int D, typename F>
  __device__ __forceinline__ static Operand across(const bf16* tile, F column, uint32_t m, uint32_t g) {
    typedef __attribute__((address_space(3))) s16x4 Lds;
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    Operand o;
    const uint32_t first = column(4 * (m & 3));
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
      const bf16* at = tile + i * Tile<D>::SIZE + Tile<D>::at(4 * g + (m >> 2), first >> 3) + (first & 4);
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)at), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(at + 16 * D));
      const s16x8 both = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
      o.v[i] = __builtin_bit_cast(bf16x8, both);
    }
    return o;
  }
  __device__ __forceinline__ static Operand of(f32x4 a, f32x4 b) {
    Operand o;
    if constexpr (PARTS == 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) { o.v[0][i] = (bf16)a[i]; o.v[0][i + 4] = (bf16)b[i]; }
    } else {
#pragma unroll
      for (int t = 0; t < PARTS; ++t) {
        u32x4 packed;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          packed[i] = upper_halves(a[2 * i], a[2 * i + 1]);
          packed[i + 2] = upper_halves(b[2 * i], b[2 * i + 1]);
        }
        if (t + 1 < PARTS)
#pragma unroll
          for (int i = 0; i < 4; ++i) { a[i] -= upper(a[i]); b[i] -= upper(b[i]); }
        o.v[t] = __builtin_bit_cast(bf16x8, packed);
      }
    }
    return o;
  }
  // A piece of 16 bytes, taken apart.
  typedef bf16 Piece __attribute__((ext_vector_type(16 / sizeof(T))));
  struct Pieces {
    Piece v[PARTS];
  };
  template <typename V>
  __device__ __forceinline__ static void cut(const V& piece, Pieces* p) {
    if constexpr (PARTS == 1) {
      p->v[0] = piece;
    } else {
      const Operand o = of(piece, piece);
#pragma unroll
      for (int t = 0; t < PARTS; ++t) p->v[t] = __builtin_shufflevector(o.v[t], o.v[t], 0, 1, 2, 3);
    }
  }
  __device__ __forceinline__ static float upper(float x) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xFFFF0000u); }
  __device__ __forceinline__ static uint32_t upper_halves(float x, float y) {   // packed
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, x), 0x07060302u);
  }
  // The values in fp32.
  __device__ __forceinline__ void widen(f32x4* a, f32x4* b) const {
    *a = *b = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int t = PARTS - 1; t >= 0; --t) {
      const u32x4 u = __builtin_bit_cast(u32x4, v[t]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float x[4] = {__builtin_bit_cast(float, u[i] << 16), __builtin_bit_cast(float, u[i] & 0xFFFF0000u),
                            __builtin_bit_cast(float, u[i + 2] << 16), __builtin_bit_cast(float, u[i + 2] & 0xFFFF0000u)};
        (*a)[2 * i] = t + 1 < PARTS ? (*a)[2 * i] + x[0] : x[0];
        (*a)[2 * i + 1] = t + 1 < PARTS ? (*a)[2 * i + 1] + x[1] : x[1];
        (*b)[2 * i] = t + 1 < PARTS ? (*b)[2 * i] + x[2] : x[2];
        (*b)[2 * i + 1] = t + 1 < PARTS ? (*b)[2 * i + 1] + x[3] : x[3];
      }
    }
  }
  __device__ __forceinline__ static f32x4 mma(const Operand& a, const Operand& b, f32x4 c) {
#pragma unroll
    for (int s = PARTS - 1; s >= 0; --s)   // parts s apart from the first of both, the smallest first
#pragma unroll
      for (int i = 0; i <= s; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[s - i], c, 0, 0, 0);
    return c;
  }
};

// 32 rows of D elements on their way from memory to LDS through the threads' registers.
template <typename T, int D, int THREADS>
struct Staged {
  static constexpr uint32_t W = 16 / sizeof(T), PER_ROW = D / W, ALL = kChunk * PER_ROW, N = (ALL + THREADS - 1) / THREADS;
  typedef T Vec __attribute__((ext_vector_type(W)));
  Vec v[N];
  // Rows first .. first + n of a head's sequence of `valid` tokens (against time: counted from its end), columns col0 .. col0 + D.
  __device__ __forceinline__ void load(const SeqRows& r, const T* head, uint32_t first, uint32_t n, uint32_t valid, bool back, uint32_t col0, uint32_t width) {
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) {
      const uint32_t at = threadIdx.x + k * THREADS;
      const uint32_t row = at / PER_ROW, col = col0 + at % PER_ROW * W;
      v[k] = Vec(T(0.0f));
      if ((ALL % THREADS == 0 || at < ALL) && row < n && col < width) {
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
  // The same in pieces, without a branch (a load in one is waited for at its end).  Rows behind the last, of which there is at least
  // one, take that one and are cleared on their way to LDS; pieces that reach behind the width end with it instead.
  __device__ __forceinline__ void load_pieces(const SeqRows& r, const T* head, uint32_t first, uint32_t end, uint32_t valid, bool back, uint32_t col0, uint32_t width) {
    typedef Vec Loose __attribute__((aligned(sizeof(T))));   // (memory is read at any address that its elements may have)
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) {
      const uint32_t at = threadIdx.x + k * THREADS;
      const uint32_t row = at / PER_ROW % kChunk, col = col0 + at % PER_ROW * W;
      const uint32_t i = first + row < end ? first + row : end - 1, t = back ? valid - 1 - i : i;
      v[k] = *reinterpret_cast<const Loose*>(head + (int64_t)t * r.token + (col + W <= width ? col : width - W));
    }
  }
  __device__ __forceinline__ void clear(uint32_t n, uint32_t col0, uint32_t width) {
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) {
      const uint32_t at = threadIdx.x + k * THREADS;
      const bool on = at / PER_ROW < n && col0 + at % PER_ROW * W < width;
#pragma unroll
      for (uint32_t e = 0; e < W; ++e) v[k][e] = on ? v[k][e] : T(0.0f);
    }
  }
  // A piece that ended with the width (columns width - W ..): its last `width % W` elements to the front of their place, zeros behind.
  __device__ __forceinline__ void store_ends(bf16* tile, uint32_t width) const {
    const uint32_t rest = width % W;
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) {
      const uint32_t at = threadIdx.x + k * THREADS;
      if (ALL % THREADS != 0 && at >= ALL) continue;
      const uint32_t row = at / PER_ROW, col = at % PER_ROW * W;
      if (col / W != width / W) continue;
      bf16* to = tile + Tile<D>::at(row, col / 8) + col % 8;
      typename Operand<T>::Pieces parts;
      Operand<T>::cut(v[k], &parts);
#pragma unroll
      for (int t = 0; t < kParts<T>; ++t) {
#pragma unroll
        for (uint32_t e = 0; e < W; ++e) to[t * Tile<D>::SIZE + e] = (bf16)0.0f;
#pragma unroll
        for (uint32_t e = 0; e < W; ++e)
          if (e + rest >= W) to[t * Tile<D>::SIZE + e + rest - W] = parts.v[t][e];
      }
    }
  }
  __device__ __forceinline__ void store(bf16* tile) const {
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) {
      const uint32_t at = threadIdx.x + k * THREADS;
      if (ALL % THREADS != 0 && at >= ALL) continue;
      const uint32_t row = at / PER_ROW, col = at % PER_ROW * W;
      bf16* to = tile + Tile<D>::at(row, col / 8) + col % 8;
      typename Operand<T>::Pieces parts;
      Operand<T>::cut(v[k], &parts);
#pragma unroll
      for (int t = 0; t < kParts<T>; ++t) *reinterpret_cast<decltype(&parts.v[t])>(to + t * Tile<D>::SIZE) = parts.v[t];
    }
  }
};

// 16 bytes of every active lane to LDS bytes `to` + 16 lane: in flight until the wait below.  (M0 is the compiler's own only for
// instructions that these kernels do not have.  The compiler does not see a memory instruction here, so the wait states between it
// and what may have set its scalar registers, five, are here.)
__device__ __forceinline__ void load_to_lds(uint32_t to, const uint8_t* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
// All but the wave's latest LEFT memory operations are done, its LDS operations too; then the workgroup's barrier.
template <int LEFT>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// What is left of a state over tokens whose decays' logarithms add up to x: S + (e^x - 1) S where more than half is (the power itself,
// rounded to 32 bits, would be off by the same 2^-25 in every chunk, or token, of a slow decay), e^x S where less is (the other form would be off
// by 2^-25 of what there was).
struct Keep { float factor; bool half; };
__device__ __forceinline__ Keep keeps(float x) { return x > -0.6931472f ? Keep{expm1f(x), true} : Keep{expf(x), false}; }
__device__ __forceinline__ float kept(float S, const Keep& k) { return k.half ? fmaf(S, k.factor, S) : S * k.factor; }

}  // namespace per
