// Rows of a residual block: layer norm with its gradient, and dropout.
#include "dev_parts.h"

namespace per {

namespace {

#include "k_block.h"

uint64_t count_of(const BlockArgs& a) { return (uint64_t)a.B * a.L * a.H; }

// Lanes and pieces of a row (pieces 0: any width).  A lane holds up to 32 elements.  Narrow rows take 4 or 16 lanes: of 64, a row of 16 would
// leave 62 idle (two million of them 904 us, of 16 lanes 202), and sums over many rows would be fewer and longer.
struct Shape { uint32_t lanes, pieces; };
Shape shape_of(uint32_t dtype, uint32_t dim) {
  const uint32_t W = dtype == PER_SEQ_BF16 ? 8 : 4, most = 32 / W;   // pieces of a lane
  if (dim < W || dim > 256 * most * W) return Shape{256, 0};
  const uint32_t lanes = dim <= 4 * 2 * W ? 4 : dim <= 16 * 2 * W ? 16 : dim <= 64 * most * W ? 64 : 256;
  uint32_t n = 1;
  while (lanes * n * W < dim) n *= 2;
  return Shape{lanes, n};
}
constexpr uint32_t kBlocks = 1024;     // workgroups of a norm: four to a compute unit
// Of a gradient: each leaves a row of sums, and two are on a compute unit at once.  Of 256, 512, 1024 workgroups, us: 8184 x 1537 33.5, 28.5, 35.6 (fp32 66, 54, 58);
// 32768 x 2048 105, 88, 91; 262144 x 128 67, 50, 46; 1100 x 5000 30, 29, 42; 64 x 256 alike.
constexpr uint32_t kBackBlocks = 512;

uint32_t sums_width(const Shape& s, uint32_t dtype, uint32_t dim) { return s.pieces ? s.lanes * s.pieces * (dtype == PER_SEQ_BF16 ? 8 : 4) : dim; }
uint32_t rows_each(const Shape& s) { return s.pieces ? 256 / s.lanes : 1; }
uint32_t back_blocks(const BlockArgs& a, uint32_t each) {
  const uint64_t need = (count_of(a) + each - 1) / each;
  return (uint32_t)(need < kBackBlocks ? need : kBackBlocks);
}

template <typename T, int LANES, int N>
hipError_t norm_as(const BlockArgs& a, bool back, hipStream_t s) {
  constexpr uint32_t each = 256 / LANES;
  if (back) {
    k_layer_norm_back<T, LANES, N><<<back_blocks(a, each), 256, LANES == 256 ? 0 : 2 * N * Piece<T>::W * LANES * sizeof(float), s>>>(a);
  } else {
    const uint64_t need = (count_of(a) + each - 1) / each;
    k_layer_norm<T, LANES, N><<<(uint32_t)(need < kBlocks ? need : kBlocks), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}
// FEWEST, MOST: the pieces that widths of these lanes come to (256 lanes are for rows that 64 do not hold).
template <typename T, int LANES, int FEWEST, int MOST>
hipError_t norm_pieces(const BlockArgs& a, uint32_t n, bool back, hipStream_t s) {
  if constexpr (FEWEST < MOST)
    if (n > (uint32_t)FEWEST) return norm_pieces<T, LANES, 2 * FEWEST, MOST>(a, n, back, s);
  return n == (uint32_t)FEWEST ? norm_as<T, LANES, FEWEST>(a, back, s) : hipErrorInvalidValue;
}
template <typename T>
hipError_t norm(uint32_t dtype, const BlockArgs& a, bool back, hipStream_t s) {
  const Shape shape = shape_of(dtype, a.dim);
  constexpr int MOST = 32 / Piece<T>::W;
  if (shape.lanes == 4) return norm_pieces<T, 4, 1, 2>(a, shape.pieces, back, s);
  if (shape.lanes == 16) return norm_pieces<T, 16, 1, 2>(a, shape.pieces, back, s);
  if (shape.lanes == 64) return norm_pieces<T, 64, 1, MOST>(a, shape.pieces, back, s);
  if (shape.pieces) return norm_pieces<T, 256, MOST / 2, MOST>(a, shape.pieces, back, s);
  if (back) {
    k_layer_norm_any<T, true><<<back_blocks(a, 1), 256, 0, s>>>(a);
  } else {
    const uint64_t need = count_of(a);
    k_layer_norm_any<T, false><<<(uint32_t)(need < kBlocks ? need : kBlocks), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

bool packed_rows(const SeqRows& r, const BlockArgs& a) {
  int64_t step = a.dim;
  if (a.H > 1 && r.head != step) return false;
  step *= a.H;
  if (a.L > 1 && r.token != step) return false;
  step *= a.L;
  return a.B == 1 || r.batch == step;
}
template <typename T, bool RESIDUAL>
hipError_t dropout(const BlockArgs& a, hipStream_t s) {
  const uint64_t n = count_of(a) * a.dim, need = ((n + 7) / 8 + 255) / 256;
  const uint32_t blocks = (uint32_t)(need < (1u << 20) ? need : 1u << 20);
  if (packed_rows(a.x, a) && packed_rows(a.out, a) && (!RESIDUAL || packed_rows(a.more, a))) k_dropout<T, RESIDUAL, true><<<blocks, 256, 0, s>>>(a, n);
  else k_dropout<T, RESIDUAL, false><<<blocks, 256, 0, s>>>(a, n);
  return hipGetLastError();
}

}  // namespace

size_t norm_work_bytes(uint32_t dtype, const BlockArgs& a) {
  const Shape shape = shape_of(dtype, a.dim);
  return (size_t)back_blocks(a, rows_each(shape)) * 2 * sums_width(shape, dtype, a.dim) * sizeof(float);
}

hipError_t launch_layer_norm(uint32_t dtype, const BlockArgs& a, hipStream_t s) {
  return dtype == PER_SEQ_BF16 ? norm<bf16>(dtype, a, false, s) : norm<float>(dtype, a, false, s);
}

hipError_t launch_layer_norm_backward(uint32_t dtype, const BlockArgs& a, hipStream_t s) {
  const Shape shape = shape_of(dtype, a.dim);
  NormSums p{a.partial, a.dweight, a.dbias, back_blocks(a, rows_each(shape)), a.dim, sums_width(shape, dtype, a.dim), shape.pieces ? shape.lanes : 0,
             dtype == PER_SEQ_BF16 ? 8u : 4u};
  if (count_of(a)) {
    const hipError_t e = dtype == PER_SEQ_BF16 ? norm<bf16>(dtype, a, true, s) : norm<float>(dtype, a, true, s);
    if (e != hipSuccess) return e;
  }
  if (!a.dweight && !a.dbias) return hipSuccess;
  k_norm_sums<<<(2 * p.width + 15) / 16, 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_dropout(uint32_t dtype, const BlockArgs& a, hipStream_t s) {
  if (dtype == PER_SEQ_BF16) return a.more.d ? dropout<bf16, true>(a, s) : dropout<bf16, false>(a, s);
  return a.more.d ? dropout<float, true>(a, s) : dropout<float, false>(a, s);
}

}  // namespace per
