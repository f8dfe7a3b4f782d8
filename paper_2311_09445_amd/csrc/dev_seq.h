// What the sequence operators' kernels share: element types, rows, turns.
#pragma once
#include "seq_geom.h"

namespace per {

typedef __bf16 bf16;

template <typename T>
__device__ __forceinline__ const T* row_of(const SeqRows& r, uint32_t b, uint32_t t, uint32_t h) {
  return static_cast<const T*>(r.d) + (int64_t)b * r.batch + (int64_t)t * r.token + (int64_t)(h / r.share) * r.head;
}
template <typename T>
__device__ __forceinline__ T* row_to(const SeqRows& r, uint32_t b, uint32_t t, uint32_t h) {
  return const_cast<T*>(row_of<T>(r, b, t, h));
}

template <typename T>
__device__ __forceinline__ float as_float(T x) { return (float)x; }

// Cosine and sine of position * freq.  The product is formed and taken to whole turns in 64 bits (in 32 bits the angle at
// position 2^20 is off by 0.06); what is left is below half a turn, exact to 2^-24 of one.
__device__ __forceinline__ void turn_of(int32_t position, float freq, float* c, float* s) {
  const double turns = (double)position * ((double)freq * 0.15915494309189533577);
  const float rest = (float)(2.0 * (turns - rint(turns)));
  sincospif(rest, s, c);
}

__device__ __forceinline__ uint32_t valid_tokens(const int32_t* lengths, uint32_t b, uint32_t L) {
  if (!lengths) return L;
  const int32_t n = lengths[b];
  return n < 0 ? 0u : (uint32_t)n < L ? (uint32_t)n : L;
}

}  // namespace per
