// Rotary positions, and norms of queries and keys for each head with the rotation in the same pass.
//
//   y = x r w,  r = 1 / sqrt(mean x^2 + eps);  pair (a, b) of y turned by theta = position * freq:
//   (m (a cos - b sin), m (a sin + b cos)); elements behind rot pass.
// The gradient turns dout back, then  h = dy w,  dx = r (h - x r mean(h x r)),  dw = sum dy x r.
#include "dev_seq.h"

namespace per {

namespace {

constexpr uint32_t kSums = 1024;   // most workgroups that leave sums for the weights' gradients

#include "k_rotate.h"

// Any width, alignment and layout: a wave per head, a lane holds elements lane, lane + 64, ... and the partner of each.
template <typename T, RotaryKind KIND>
__global__ __launch_bounds__(256) void k_rotate_any(RotaryArgs a) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = a.rot / 2;
  const uint32_t heads = a.side[0].heads + a.side[1].heads;
  const uint64_t items = (uint64_t)a.B * a.L * heads, stride = (uint64_t)gridDim.x * 4;
  float sums[2][4] = {};
  for (uint64_t it = (uint64_t)blockIdx.x * 4 + wave; it < items; it += stride) {
    uint32_t h = (uint32_t)(it % heads);
    const uint64_t tok = it / heads;
    const uint32_t b = (uint32_t)(tok / a.L), t = (uint32_t)(tok % a.L);
    const bool second = h >= a.side[0].heads;
    const RotarySide& sd = a.side[second];
    if (second) h -= a.side[0].heads;
    const T* x = row_of<T>(sd.x, b, t, h);
    const T* d = KIND == NORM_ROTATE_BACK ? row_of<T>(sd.dout, b, t, h) : nullptr;
    T* out = row_to<T>(sd.out, b, t, h);
    const int32_t pos = a.at ? a.at[(int64_t)b * a.at_batch + (int64_t)t * a.at_token] : (int32_t)t;
    float own[4], other[4], cs[4], sn[4], dy[4];
    float square = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t e = lane + 64 * i;
      own[i] = other[i] = dy[i] = 0.0f;
      cs[i] = 1.0f;
      sn[i] = 0.0f;
      if (e >= a.dim) continue;
      uint32_t partner = e, pair = 0;
      float sign = 0.0f;   // the turned element: own cos + sign partner sin
      if (e < a.rot) {
        if (a.layout == PER_SEQ_HALF) {
          partner = e < half ? e + half : e - half;
          pair = e < half ? e : e - half;
          sign = e < half ? -1.0f : 1.0f;
        } else {
          partner = e ^ 1u;
          pair = e >> 1;
          sign = (e & 1u) ? 1.0f : -1.0f;
        }
        turn_of(pos, a.freqs[pair], &cs[i], &sn[i]);
        cs[i] *= a.magnitude;
        sn[i] *= a.magnitude * sign * (KIND == NORM_ROTATE_BACK ? -1.0f : a.sign);
      }
      own[i] = as_float(x[e]);
      if (KIND == NORM_ROTATE_BACK) {
        dy[i] = as_float(d[e]);
        if (e < a.rot) dy[i] = dy[i] * cs[i] + as_float(d[partner]) * sn[i];
      } else {
        other[i] = as_float(x[partner]);
        if (KIND == NORM_ROTATE && sd.weight) other[i] *= sd.weight[partner];
      }
      square = fmaf(own[i], own[i], square);
    }
    float r = 1.0f;
    if (KIND != ROTATE) {
#pragma unroll
      for (int m = 32; m; m >>= 1) square += __shfl_xor(square, m);
      r = 1.0f / sqrtf(square / (float)a.dim + a.eps);
    }
    if (KIND == NORM_ROTATE_BACK) {
      float along = 0.0f;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t e = lane + 64 * i;
        own[i] *= r;
        sums[second][i] = fmaf(dy[i], own[i], sums[second][i]);
        if (e < a.dim && sd.weight) dy[i] *= sd.weight[e];
        along = fmaf(dy[i], own[i], along);
      }
#pragma unroll
      for (int m = 32; m; m >>= 1) along += __shfl_xor(along, m);
      along /= (float)a.dim;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t e = lane + 64 * i;
        if (e < a.dim) out[e] = (T)(r * (dy[i] - own[i] * along));
      }
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t e = lane + 64 * i;
        if (e >= a.dim) continue;
        if (KIND == NORM_ROTATE && sd.weight) own[i] *= sd.weight[e];
        if (e < a.rot) own[i] = own[i] * cs[i] + other[i] * sn[i];   // (those behind pass: zero times infinity would not be zero)
        out[e] = (T)(own[i] * r);
      }
    }
  }
  if (KIND != NORM_ROTATE_BACK) return;
  __shared__ float all[4][2][256];
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    all[wave][0][lane + 64 * i] = sums[0][i];
    all[wave][1][lane + 64 * i] = sums[1][i];
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < 2 * a.dim; i += 256) {
    const uint32_t s = i / a.dim, e = i % a.dim;
    a.partial[(size_t)blockIdx.x * 2 * a.dim + i] = (all[0][s][e] + all[1][s][e]) + (all[2][s][e] + all[3][s][e]);
  }
}

// The weights' gradients from the workgroups' sums, in their order: a workgroup takes 16 elements, 64 rows of sums at a time.
struct WeightSums {
  const float* from;
  uint32_t rows, stride;
  float* to;
};
struct WeightSumsOf {
  WeightSums side[2];
};
__global__ __launch_bounds__(1024) void k_weight_sums(WeightSumsOf both, uint32_t dim) {
  __shared__ float all[64][16];
  const WeightSums& w = both.side[blockIdx.y];
  const uint32_t e = threadIdx.x & 15, row = threadIdx.x >> 4, i = blockIdx.x * 16 + e;
  float sum = 0.0f;
  if (i < dim) {
    float s[kSums / 64];
#pragma unroll
    for (uint32_t k = 0; k < kSums / 64; ++k) s[k] = row + 64 * k < w.rows ? w.from[(size_t)(row + 64 * k) * w.stride + i] : 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < kSums / 64; ++k) sum += s[k];
  }
  all[row][e] = sum;
  __syncthreads();
  for (uint32_t m = 32; m; m >>= 1) {
    if (row < m) all[row][e] += all[row + m][e];
    __syncthreads();
  }
  if (row == 0 && i < dim && w.to) w.to[i] = all[0][e];
}

// Workgroups of a gradient: as the workspace is sized, before it is known which kernel takes it.
uint32_t sum_blocks(uint64_t tokens, uint32_t heads) {
  const uint64_t n = (tokens * heads + 3) / 4;
  return (uint32_t)(n < kSums ? (n > 2 ? n : 2) : kSums);
}

template <typename T, int W, RotaryKind KIND, bool INTERLEAVED>
hipError_t launch_units(const RotaryArgs& a, uint32_t blocks, hipStream_t s) {
  const uint32_t units = a.dim / (2 * W), most = a.tokens[0] > a.tokens[1] ? a.tokens[0] : a.tokens[1];
  const uint32_t lds = most * (a.rot / 2) * sizeof(float2);
  if (units <= 4) k_rotate_units<T, W, 4, KIND, INTERLEAVED><<<blocks, 256, lds, s>>>(a);
  else if (units <= 8) k_rotate_units<T, W, 8, KIND, INTERLEAVED><<<blocks, 256, lds, s>>>(a);
  else if (units <= 16) k_rotate_units<T, W, 16, KIND, INTERLEAVED><<<blocks, 256, lds, s>>>(a);
  else if (W <= 4 && units <= 32) k_rotate_units<T, W, W <= 4 ? 32 : 16, KIND, INTERLEAVED><<<blocks, 256, lds, s>>>(a);
  else k_rotate_units<T, W, W <= 2 ? 64 : 16, KIND, INTERLEAVED><<<blocks, 256, lds, s>>>(a);   // (dim is at most 256)
  return hipGetLastError();
}
template <typename T, int W>
hipError_t launch_units(RotaryKind kind, const RotaryArgs& a, uint32_t blocks, hipStream_t s) {
  const bool il = a.layout == PER_SEQ_INTERLEAVED;
  switch (kind) {
    case ROTATE: return il ? launch_units<T, W, ROTATE, true>(a, blocks, s) : launch_units<T, W, ROTATE, false>(a, blocks, s);
    case NORM_ROTATE: return il ? launch_units<T, W, NORM_ROTATE, true>(a, blocks, s) : launch_units<T, W, NORM_ROTATE, false>(a, blocks, s);
    default: return il ? launch_units<T, W, NORM_ROTATE_BACK, true>(a, blocks, s) : launch_units<T, W, NORM_ROTATE_BACK, false>(a, blocks, s);
  }
}

// Elements of the widest vectors (16 or 8 bytes) that all rows and the pairs' places allow; 0: none.
uint32_t vector_width(const RotaryArgs& a, RotaryKind kind, uint32_t element) {
  for (uint32_t w = 16 / element; w * element >= 8; w /= 2) {
    bool fits = a.dim % (2 * w) == 0 && a.rot % (2 * w) == 0;
    for (int i = 0; i < 2; ++i) {
      const RotarySide& sd = a.side[i];
      if (!sd.heads) continue;
      for (const SeqRows* r : {&sd.x, &sd.out, kind == NORM_ROTATE_BACK ? &sd.dout : &sd.x})
        fits = fits && reinterpret_cast<uintptr_t>(r->d) % (w * element) == 0 && r->batch % w == 0 && r->token % w == 0 && r->head % w == 0;
    }
    if (fits) return w;
  }
  return 0;
}

template <typename T>
hipError_t launch(RotaryKind kind, RotaryArgs a, float* dqw, float* dkw, hipStream_t s) {
  const uint32_t heads = a.side[0].heads + a.side[1].heads, most = sum_blocks((uint64_t)a.B * a.L, heads);
  const uint64_t tokens = (uint64_t)a.B * a.L;
  const uint32_t w = tokens && heads ? vector_width(a, kind, sizeof(T)) : 0;
  uint32_t blocks;
  hipError_t e;
  if (w) {
    // As many tokens to a workgroup as give its lanes eight units each (a gradient's sixteen), but fewer where that would leave the
    // chip without workgroups; their cosines take at most 32 KiB.
    const uint32_t units = a.dim / (2 * w), lanes = units <= 4 ? 4 : units <= 8 ? 8 : units <= 16 ? 16 : units <= 32 ? 32 : 64;
    const uint64_t fit = 4096 / (a.rot / 2 + 1);
    blocks = 0;
    for (int i = 0; i < 2; ++i) {
      const bool back = kind == NORM_ROTATE_BACK;
      const uint32_t of = back ? a.side[i].heads : heads;
      if (!of) continue;
      // (a gradient's workgroups are bounded by the room for their sums: shared out by heads, one at least)
      uint64_t room = back ? (uint64_t)most * of / heads : 1u << 20;
      if (back && i == 1 && room + a.blocks[0] > most) room = most - a.blocks[0];
      if (!room) room = 1;   // (there is one: `most` is two at least, and heads on the other side leave one)
      uint64_t n = (back ? 16 : 8) * 256 / lanes / of;
      const uint64_t share = back ? (tokens + room - 1) / room : tokens / 1024;
      if (n > share) n = share;
      if (n > fit) n = fit;
      a.tokens[i] = n ? (uint32_t)n : 1;
      a.tiles[i] = (uint32_t)((tokens + a.tokens[i] - 1) / a.tokens[i]);
      a.blocks[i] = a.tiles[i] < room ? a.tiles[i] : (uint32_t)room;
      blocks += a.blocks[i];
      if (!back) break;
    }
    e = w * sizeof(T) == 16 ? launch_units<T, 16 / sizeof(T)>(kind, a, blocks, s) : launch_units<T, 8 / sizeof(T)>(kind, a, blocks, s);
  } else {
    const uint64_t n = (tokens * heads + 3) / 4;
    blocks = kind == NORM_ROTATE_BACK ? most : (uint32_t)(n < 16384 ? n : 16384);
    if (kind == ROTATE) k_rotate_any<T, ROTATE><<<blocks, 256, 0, s>>>(a);
    else if (kind == NORM_ROTATE) k_rotate_any<T, NORM_ROTATE><<<blocks, 256, 0, s>>>(a);
    else k_rotate_any<T, NORM_ROTATE_BACK><<<blocks, 256, 0, s>>>(a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || kind != NORM_ROTATE_BACK || (!dqw && !dkw)) return e;
  WeightSumsOf sums{};
  for (int i = 0; i < 2; ++i)
    sums.side[i] = w ? WeightSums{a.partial + (i ? (size_t)a.blocks[0] * a.dim : 0), a.blocks[i], a.dim, i ? dkw : dqw}
                     : WeightSums{a.partial + i * a.dim, blocks, 2 * a.dim, i ? dkw : dqw};
  k_weight_sums<<<dim3((a.dim + 15) / 16, 2), 1024, 0, s>>>(sums, a.dim);
  return hipGetLastError();
}

}  // namespace

size_t rotary_work_bytes(uint64_t tokens, uint32_t heads, uint32_t dim) { return (size_t)sum_blocks(tokens, heads) * 2 * dim * sizeof(float); }

hipError_t launch_rotary(RotaryKind kind, uint32_t dtype, RotaryArgs a, float* dqw, float* dkw, hipStream_t s) {
  return dtype == PER_SEQ_BF16 ? launch<bf16>(kind, a, dqw, dkw, s) : launch<float>(kind, a, dqw, dkw, s);
}

}  // namespace per
