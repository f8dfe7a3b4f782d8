// Rotation and norm of heads whose rows can be moved in vectors.  Part of seq_rotate.hip (included inside namespace per).
//
// A head is taken in units of W pairs: two vectors of W elements, the partners of each other (half layout: W elements and those
// rot/2 further on; interleaved, and behind rot: 2 W elements in a row).  A lane takes one unit, the lanes of a head are LANES = the
// next power of two, and a workgroup takes the heads of `tokens` tokens, whose cosines and sines it works out once, in LDS.  The first
// vectors are asked for before the cosines are worked out.  A lane keeps two units in flight; one of a gradient, which reads twice as
// much for each and holds its sums besides: what counts there is waves (128 registers, four to a SIMD; with two units, and the sums of
// queries and keys in one workgroup, it took 187 and 37 us instead of 28.6 for 8184 tokens of 20 heads of 96).
// Memory bounds it: 32768 tokens of 40 heads of 128 in bfloat16 take 131 us (5.1 TB/s, a copy 5.2), rotation alone of 32 heads 107 (5.0).

template <typename T, int W>
struct Unit {
  typedef T Vec __attribute__((ext_vector_type(W)));
  // Partners a[i], b[i] from the two vectors and back.
  __device__ __forceinline__ static void split(const Vec& u, const Vec& v, bool interleaved, float* a, float* b) {
    float e[2 * W];
#pragma unroll
    for (int i = 0; i < W; ++i) { e[i] = as_float((T)u[i]); e[W + i] = as_float((T)v[i]); }
#pragma unroll
    for (int i = 0; i < W; ++i) { a[i] = interleaved ? e[2 * i] : e[i]; b[i] = interleaved ? e[2 * i + 1] : e[W + i]; }
  }
  __device__ __forceinline__ static void join(const float* a, const float* b, bool interleaved, Vec* u, Vec* v) {
    float e[2 * W];
#pragma unroll
    for (int i = 0; i < W; ++i) { e[interleaved ? 2 * i : i] = a[i]; e[interleaved ? 2 * i + 1 : W + i] = b[i]; }
#pragma unroll
    for (int i = 0; i < W; ++i) { (*u)[i] = (T)e[i]; (*v)[i] = (T)e[W + i]; }
  }
};

template <int LANES>
__device__ __forceinline__ float head_sum(float x) {
#pragma unroll
  for (int m = LANES / 2; m; m >>= 1) x += __shfl_xor(x, m);
  return x;
}

template <typename T, int W, int LANES, RotaryKind KIND, bool INTERLEAVED>
__global__ __launch_bounds__(256, KIND == NORM_ROTATE_BACK ? 4 : 2) void k_rotate_units(RotaryArgs a) {
  constexpr bool BACK = KIND == NORM_ROTATE_BACK, NORM = KIND != ROTATE;
  constexpr int GROUPS = 256 / LANES, kFlight = BACK ? 1 : 2;
  typedef typename Unit<T, W>::Vec Vec;
  extern __shared__ __attribute__((aligned(16))) float2 turns[];   // [tokens][rot/2]
  const uint32_t unit = threadIdx.x % LANES, group = threadIdx.x / LANES, half = a.rot / 2;
  const bool on = unit < a.dim / (2 * W), turned = on && unit < a.rot / (2 * W);
  uint32_t at_u = 2 * W * unit, at_v = at_u + W;      // where the unit's vectors are
  if (!INTERLEAVED && turned) { at_u = W * unit; at_v = half + W * unit; }
  const uint32_t total = a.B * a.L;
  const float per = 1.0f / (float)a.dim;
  // A gradient's workgroups are either's, queries' or keys'.
  const int from = BACK && blockIdx.x >= a.blocks[0] ? 1 : 0, until = BACK ? from + 1 : 2;
  const uint32_t block = from ? blockIdx.x - a.blocks[0] : blockIdx.x, blocks = BACK ? a.blocks[from] : gridDim.x;
  const uint32_t tokens = a.tokens[from], tiles = a.tiles[from];
  float sums[2 * W];
  if (BACK) {
#pragma unroll
    for (int i = 0; i < 2 * W; ++i) sums[i] = 0.0f;
  }
  for (uint32_t tile = block; tile < tiles; tile += blocks) {
    const uint32_t first = tile * tokens, n = total - first < tokens ? total - first : tokens;
    for (int side = from; side < until; ++side) {
      const RotarySide& sd = a.side[side];
      const uint32_t items = n * sd.heads;
      float wa[W], wb[W];
#pragma unroll
      for (int i = 0; i < W; ++i) wa[i] = wb[i] = 1.0f;
      if (NORM && sd.weight && on) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
          wa[i] = sd.weight[INTERLEAVED ? at_u + 2 * i : at_u + i];
          wb[i] = sd.weight[INTERLEAVED ? at_u + 2 * i + 1 : at_v + i];
        }
      }
      for (uint32_t it = group; it < items || (side == from && it == group); it += kFlight * GROUPS) {
        Vec u[kFlight], v[kFlight], du[kFlight], dv[kFlight];
        uint32_t token[kFlight];
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
          const uint32_t item = it + f * GROUPS;
          token[f] = item / (sd.heads ? sd.heads : 1);
          u[f] = v[f] = du[f] = dv[f] = Vec(T(0.0f));
          if (on && item < items) {
            const uint32_t tok = first + token[f], b = tok / a.L, t = tok % a.L, h = item % sd.heads;
            const T* x = row_of<T>(sd.x, b, t, h);
            u[f] = *reinterpret_cast<const Vec*>(x + at_u);
            v[f] = *reinterpret_cast<const Vec*>(x + at_v);
            if (BACK) {
              const T* d = row_of<T>(sd.dout, b, t, h);
              du[f] = *reinterpret_cast<const Vec*>(d + at_u);
              dv[f] = *reinterpret_cast<const Vec*>(d + at_v);
            }
          }
        }
        if (side == from && it == group) {   // (every wave comes here once per tile)
          if (tile != block) __syncthreads();   // (all are through with the tile before)
          for (uint32_t i = threadIdx.x; i < n * half; i += 256) {
            const uint32_t tok = first + i / half, b = tok / a.L, t = tok % a.L;
            const int32_t pos = a.at ? a.at[(int64_t)b * a.at_batch + (int64_t)t * a.at_token] : (int32_t)t;
            float c, s;
            turn_of(pos, a.freqs[i % half], &c, &s);
            turns[i] = float2{a.magnitude * c, a.magnitude * s * (BACK ? -1.0f : a.sign)};
          }
          __syncthreads();
        }
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
          const uint32_t item = it + f * GROUPS;
          if (item >= items) break;   // (the same for all lanes of a head)
          float xa[W], xb[W], ya[W], yb[W];
          Unit<T, W>::split(u[f], v[f], INTERLEAVED, xa, xb);
          float r = 1.0f;
          if (NORM) {
            float square = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) square = fmaf(xa[i], xa[i], fmaf(xb[i], xb[i], square));
            r = 1.0f / sqrtf(fmaf(head_sum<LANES>(square), per, a.eps));
          }
          const float2* cs = turns + token[f] * half + W * unit;
          if (BACK) {
            float da[W], db[W], along = 0.0f;
            Unit<T, W>::split(du[f], dv[f], INTERLEAVED, da, db);
#pragma unroll
            for (int i = 0; i < W; ++i) {
              float ga = da[i], gb = db[i];
              if (turned) {
                const float2 t = cs[i];
                ga = da[i] * t.x - db[i] * t.y;
                gb = da[i] * t.y + db[i] * t.x;
              }
              xa[i] *= r;
              xb[i] *= r;
              sums[i] = fmaf(ga, xa[i], sums[i]);
              sums[W + i] = fmaf(gb, xb[i], sums[W + i]);
              ya[i] = ga * wa[i];
              yb[i] = gb * wb[i];
              along = fmaf(ya[i], xa[i], fmaf(yb[i], xb[i], along));
            }
            along = head_sum<LANES>(along) * per;
#pragma unroll
            for (int i = 0; i < W; ++i) {
              ya[i] = r * fmaf(-xa[i], along, ya[i]);
              yb[i] = r * fmaf(-xb[i], along, yb[i]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
              if (NORM) {
                xa[i] *= r * wa[i];
                xb[i] *= r * wb[i];
              }
              ya[i] = xa[i];
              yb[i] = xb[i];
              if (turned) {
                const float2 t = cs[i];
                ya[i] = xa[i] * t.x - xb[i] * t.y;
                yb[i] = xa[i] * t.y + xb[i] * t.x;
              }
            }
          }
          if (on) {
            const uint32_t tok = first + token[f], b = tok / a.L, t = tok % a.L, h = item % sd.heads;
            T* out = row_to<T>(sd.out, b, t, h);
            Vec ou, ov;
            Unit<T, W>::join(ya, yb, INTERLEAVED, &ou, &ov);
            *reinterpret_cast<Vec*>(out + at_u) = ou;
            *reinterpret_cast<Vec*>(out + at_v) = ov;
          }
        }
      }
    }
  }
  if (!BACK) return;
  // sums of the workgroup: over the lanes of a wave that hold the same unit, then over the waves
  __shared__ float all[4][2 * W * LANES];
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 2 * W; ++i) {
    float s = sums[i];
#pragma unroll
    for (int m = LANES; m < 64; m <<= 1) s += __shfl_xor(s, m);
    if (lane < LANES) all[wave][lane * 2 * W + i] = s;
  }
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < a.dim; e += 256) {   // element e: of which unit, which place
    uint32_t un, place;
    if (INTERLEAVED) {
      un = e / (2 * W);
      place = (e & 1) * W + e % (2 * W) / 2;
    } else if (e < a.rot) {
      un = e % half / W;
      place = (e >= half ? W : 0) + e % half % W;
    } else {
      un = e / (2 * W);
      place = e % (2 * W);
    }
    const uint32_t at = un * 2 * W + place;
    a.partial[(size_t)blockIdx.x * a.dim + e] = (all[0][at] + all[1][at]) + (all[2][at] + all[3][at]);
  }
}
