// Values in fp32 taken apart into bfloat16, and products of what is taken apart.
#pragma once
#include "dev_tiles.h"

namespace per {

// N parts in bfloat16 whose sum holds 8 N + N - 1 bits of the values: each is what the ones before left, rounded.  (A value above the largest of
// bfloat16, 3.39e38, becomes infinite.)
template <int N>
struct Parts {
  bf16x8 v[N];
  __device__ __forceinline__ static Parts of(f32x4 a, f32x4 b) {
    typedef float Two __attribute__((ext_vector_type(2)));
    typedef bf16 Rounded __attribute__((ext_vector_type(2)));
    Two x[4] = {{a[0], a[1]}, {a[2], a[3]}, {b[0], b[1]}, {b[2], b[3]}};
    Parts o;
#pragma unroll
    for (int t = 0; t < N; ++t) {
      u32x4 packed;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        packed[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x[i], Rounded));
        if (t + 1 < N) {
          x[i][0] -= __builtin_bit_cast(float, packed[i] << 16);
          x[i][1] -= __builtin_bit_cast(float, packed[i] & 0xFFFF0000u);
        }
      }
      o.v[t] = __builtin_bit_cast(bf16x8, packed);
    }
    return o;
  }
};

// a b + c, of the products of parts those that are no smaller than 2^(-8 LEAST) of the first, the smallest first.
template <int LEAST = 2, int NA, int NB>
__device__ __forceinline__ f32x4 mma(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], f32x4 c) {
#pragma unroll
  for (int s = LEAST; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (s - i >= 0 && s - i < NB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[s - i], c, 0, 0, 0);
  return c;
}

// c[m] += a(m) b(m) for M products at once, in turn: an instruction that takes the result of the one before it waits for all of its passes.
template <int M, int LEAST, int NA, int NB, typename A, typename B>
__device__ __forceinline__ void mma_turns(A a, B b, f32x4 (&c)[M]) {
#pragma unroll
  for (int s = LEAST; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (s - i >= 0 && s - i < NB)
#pragma unroll
        for (int m = 0; m < M; ++m) c[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a(m)[i], b(m)[s - i], c[m], 0, 0, 0);
}

// LDS of a wave's own: written by some lanes, read by others behind this.
__device__ __forceinline__ void wave_sync() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// The sum over four lanes in a row; over the 16 lanes that share a lane's g.
#define PER_ADD_DPP(ctrl) x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, 0xF, 0xF, false))
__device__ __forceinline__ float sum4(float x) {
  PER_ADD_DPP(0xB1);    // lanes 1 apart
  PER_ADD_DPP(0x4E);    // 2 apart
  return x;
}
__device__ __forceinline__ float sum16(float x) {
  x = sum4(x);
  PER_ADD_DPP(0x141);   // 4: the half row turned around
  PER_ADD_DPP(0x140);   // 8: the row turned around
  return x;
}
#undef PER_ADD_DPP

// Sums over the 16 lanes that share a lane's g, of 16 values at once: value m in lane m.  Halves of the values and of the lanes meet.
__device__ __forceinline__ float sums16(float (&v)[16], uint32_t m) {
#define PER_MEET(n, ctrl, upper)                                                                                                    \
  _Pragma("unroll") for (int i = 0; i < n; ++i) {                                                                                   \
    const float keep = (upper) ? v[i + n] : v[i], give = (upper) ? v[i] : v[i + n];                                                 \
    v[i] = keep + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, give), ctrl, 0xF, 0xF, false));  \
  }
  PER_MEET(8, 0x140, m & 8)   // the row turned around
  PER_MEET(4, 0x141, m & 4)   // the half row
  PER_MEET(2, 0x4E, m & 2)
  PER_MEET(1, 0xB1, m & 1)
#undef PER_MEET
  return v[0];
}

}  // namespace per
