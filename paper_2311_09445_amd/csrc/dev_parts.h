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
    Parts o;
#pragma unroll
    for (int t = 0; t < N; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o.v[t][i] = (bf16)a[i];
        o.v[t][i + 4] = (bf16)b[i];
      }
      if (t + 1 < N)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i] -= (float)o.v[t][i];
          b[i] -= (float)o.v[t][i + 4];
        }
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

// LDS of a wave's own: written by some lanes, read by others behind this.
__device__ __forceinline__ void wave_sync() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// The sum over the 16 lanes that share a lane's g.
__device__ __forceinline__ float sum16(float x) {
#define PER_ADD_DPP(ctrl) x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, 0xF, 0xF, false))
  PER_ADD_DPP(0xB1);    // lanes 1 apart
  PER_ADD_DPP(0x4E);    // 2 apart
  PER_ADD_DPP(0x141);   // 4: the half row turned around
  PER_ADD_DPP(0x140);   // 8: the row turned around
#undef PER_ADD_DPP
  return x;
}

}  // namespace per
