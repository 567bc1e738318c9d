// Dropout and residual sum: out = res + m x, m the site's mask times its scale.
//
// Bounded by memory: 8 x 4096 x 2048 bf16 with a residual takes 68 us, 5.9 TB/s (a copy reaches 5.4).  The
// mask is made on the way: 16 bits an element, so a Philox block serves 8 columns, and the blocks of
// this size take 13 us of the vector units (with 32 bits an element it would be 25).
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

constexpr int kDropPieces = 4;   // pieces per thread, all loaded before the first is worked on

// A workgroup takes 256 * kDropPieces consecutive pieces of the rows laid end to end (per_row
// pieces each), a thread every 256th of them: one division finds its first row, steps of
// 256 pieces are (step_rows, step_pieces) with a carry.
template <class E, int M, class I, bool NT = false>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, int per_row, int step_rows, int step_pieces) {
  constexpr int EP = kPiece<E>;
  const int n = (int)a.n;
  const I q = (I)((int64_t)flat_block() * (256 * kDropPieces) + threadIdx.x);
  int64_t r = (int64_t)(q / (I)per_row);
  int c = (int)(q - (I)r * (I)per_row);
  uint4 x[kDropPieces], z[kDropPieces];
  int64_t row[kDropPieces];
  int col[kDropPieces];
#pragma unroll
  for (int k = 0; k < kDropPieces; ++k) {
    row[k] = r;
    col[k] = r < a.rows ? c * EP : -1;
    if (col[k] >= 0) {
      x[k] = load_row<E, M, NT>((const E*)a.x + r * a.ldx, col[k], n);
      if (a.res) z[k] = load_row<E, M, NT>((const E*)a.res + r * a.ldr, col[k], n);
    }
    r += step_rows;
    c += step_pieces;
    if (c >= per_row) {
      c -= per_row;
      ++r;
    }
  }
#pragma unroll
  for (int k = 0; k < kDropPieces; ++k) {
    if (col[k] < 0) continue;
    float v[EP], u[EP];
    unpack_row<E, M>(x[k], col[k], n, v);
    if (a.drop.on) drop_piece<E>(a.drop, (uint32_t)row[k], col[k], n, v);
    if (a.res) {
      unpack_row<E, M>(z[k], col[k], n, u);
#pragma unroll
      for (int j = 0; j < EP; ++j) v[j] += u[j];
    }
    store_row<E, M, NT>((E*)a.out + row[k] * a.ldo, col[k], n, v);
  }
}

template <class E>
static void launch_dropout_of(const DropoutArgs& a, hipStream_t st) {
  constexpr int EP = kPiece<E>;
  const int64_t per_row = ceil_div(a.n, EP), total = a.rows * per_row;
  const dim3 grid = flat_grid(ceil_div(total, 256 * kDropPieces));
  const int sr = (int)(256 / per_row), sp = (int)(256 % per_row);
  const bool small = total < ((int64_t)1 << 31);
  auto go = [&](auto kernel) { DPRC_LAUNCH(kernel, grid, dim3(256), 0, st, a, (int)per_row, sr, sp); };
  StreamRows stream(a.n * (int64_t)sizeof(E));
  stream.add(a.x, a.rows, a.ldx * sizeof(E));
  stream.add(a.res, a.rows, a.ldr * sizeof(E));
  stream.add(a.out, a.rows, a.ldo * sizeof(E));
  if (a.n < EP) go(dropout_kernel<E, kTiny, uint64_t>);
  else if (stream.yes()) go(dropout_kernel<E, kWhole, uint64_t, true>);
  else if (a.n % EP == 0 && small) go(dropout_kernel<E, kWhole, uint32_t>);
  else if (a.n % EP == 0) go(dropout_kernel<E, kWhole, uint64_t>);
  else if (small) go(dropout_kernel<E, kTail, uint32_t>);
  else go(dropout_kernel<E, kTail, uint64_t>);
}

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t st) {
  if (a.bf16) launch_dropout_of<uint16_t>(a, st);
  else launch_dropout_of<float>(a, st);
  return hipGetLastError();
}

}  // namespace dprc
