// Rotary positions, and norms of queries and keys for each head with the rotation in the same pass.
//
//   y = x r w,  r = 1 / sqrt(mean x^2 + eps);  pair (a, b) of y turned by theta = position * freq:
//   (m (a cos - b sin), m (a sin + b cos)); elements behind rot pass.
// The gradient turns dout back, then  h = dy w,  dx = r (h - x r mean(h x r)),  dw = sum dy x r.
#include "dev_seq.h"

namespace per {

namespace {

constexpr uint32_t kSums = 512;   // most workgroups that leave sums for the weights' gradients

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
        dy[i] = as_float(d[e]) * cs[i] + as_float(d[partner]) * sn[i];
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
        out[e] = (T)((own[i] * cs[i] + other[i] * sn[i]) * r);
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

// The weights' gradients from the workgroups' sums, in their order.
__global__ __launch_bounds__(256) void k_weight_sums(const float* partial, uint32_t blocks, uint32_t dim, float* dqw, float* dkw) {
  const uint32_t i = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;   // 32 lanes per element
  if (i >= 2 * dim) return;
  float sum = 0.0f;
  for (uint32_t b = lane; b < blocks; b += 32) sum += partial[(size_t)b * 2 * dim + i];
#pragma unroll
  for (int m = 16; m; m >>= 1) sum += __shfl_xor(sum, m);
  float* out = i < dim ? dqw : dkw;
  if (lane == 0 && out) out[i < dim ? i : i - dim] = sum;
}

uint32_t sum_blocks(uint64_t tokens, uint32_t heads) {
  const uint64_t n = (tokens * heads + 3) / 4;
  return (uint32_t)(n < kSums ? (n ? n : 1) : kSums);
}

template <typename T>
hipError_t launch(RotaryKind kind, const RotaryArgs& a, float* dqw, float* dkw, hipStream_t s) {
  const uint32_t heads = a.side[0].heads + a.side[1].heads;
  const uint64_t tokens = (uint64_t)a.B * a.L, waves = tokens * heads;
  if (kind == NORM_ROTATE_BACK) {
    const uint32_t blocks = sum_blocks(tokens, heads);
    k_rotate_any<T, NORM_ROTATE_BACK><<<blocks, 256, 0, s>>>(a);
    if (dqw || dkw) k_weight_sums<<<(2 * a.dim + 7) / 8, 256, 0, s>>>(a.partial, blocks, a.dim, dqw, dkw);
  } else {
    const uint64_t n = (waves + 3) / 4;
    const uint32_t blocks = (uint32_t)(n < 16384 ? n : 16384);
    if (kind == ROTATE) k_rotate_any<T, ROTATE><<<blocks, 256, 0, s>>>(a);
    else k_rotate_any<T, NORM_ROTATE><<<blocks, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

size_t rotary_work_bytes(uint64_t tokens, uint32_t heads, uint32_t dim) { return (size_t)sum_blocks(tokens, heads) * 2 * dim * sizeof(float); }

hipError_t launch_rotary(RotaryKind kind, uint32_t dtype, RotaryArgs a, float* dqw, float* dkw, hipStream_t s) {
  return dtype == PER_SEQ_BF16 ? launch<bf16>(kind, a, dqw, dkw, s) : launch<float>(kind, a, dqw, dkw, s);
}

}  // namespace per
