// Dropout, residual sum and norm of token rows (forward).
//
// Bounded by memory: a row is read once and held in registers from the sum through its mean,
// its variance about that mean and the output.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

constexpr int64_t kNormBlocks = 512;

// TPR threads hold a row of at most TPR * C columns, C each; a workgroup of max(256, TPR)
// threads works on 256 / TPR rows at a time and walks the rows with the grid, the next row's
// pieces loading while this one is reduced.  Weight and bias stay in registers for all rows.
template <class E, int M, int TPR, int C>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_kernel(NormArgs a) {
  constexpr int EP = kPiece<E>, V = C / EP, BLK = TPR > 256 ? TPR : 256, RPB = BLK / TPR;
  constexpr bool kHold = TPR < 1024;
  typedef RowSum<TPR, 1, BLK> Sum;
  __shared__ typename Sum::Buffer buf;
  int turn = 0;
  const int t = threadIdx.x % TPR, n = (int)a.n;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;

  uint4 x[V], z[V];
  auto load = [&](int64_t row) {
    row = std::min(row, a.rows - 1);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * EP;
      x[v] = load_row<E, M>((const E*)a.x + row * a.ldx, c, n);
      if (a.res) z[v] = load_row<E, M>((const E*)a.res + row * a.ldr, c, n);
    }
  };
  load(r);
  float w[C], b[C];
  auto load_wb = [&](int v) {
    const int c = (v * TPR + t) * EP;
    load_vec<EP>(a.w, a.wbf16, c, n, 1.f, w + v * EP);
    load_vec<EP>(a.b, a.wbf16, c, n, 0.f, b + v * EP);
  };
  if (kHold)
#pragma unroll
    for (int v = 0; v < V; ++v) load_wb(v);
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += step, r += step) {
    float s[C], u[EP], red[1] = {0.f}, mu = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * EP;
#pragma unroll
      for (int k = v * EP; k < v * EP + EP; ++k) s[k] = 0.f;
      if (c >= n) continue;
      unpack_row<E, M>(x[v], c, n, s + v * EP);
      if (a.drop.on) drop_piece<E>(a.drop, (uint32_t)r, c, s + v * EP);
      if (!a.res) continue;
      unpack_row<E, M>(z[v], c, n, u);
#pragma unroll
      for (int j = 0; j < EP; ++j) s[v * EP + j] += u[j];
    }
    load(r + step);
    if (!a.rms) {
#pragma unroll
      for (int k = 0; k < C; ++k) red[0] += s[k];
      Sum::run(red, buf, turn);
      mu = red[0] * a.inv_n;
      red[0] = 0.f;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * EP;
#pragma unroll
      for (int j = 0; j < EP; ++j) {
        const float d = (M == kWhole ? c : c + j) < n ? s[v * EP + j] - mu : 0.f;
        red[0] = fmaf(d, d, red[0]);
      }
    }
    Sum::run(red, buf, turn);
    const float rstd = 1.f / sqrtf(fmaf(red[0], a.inv_n, a.eps));
    if (r >= a.rows) continue;
    if (t == 0) {
      if (a.mean) a.mean[r] = mu;
      if (a.rstd) a.rstd[r] = rstd;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * EP;
      if (c >= n) continue;
      if (a.sum) store_row<E, M>((E*)a.sum + r * a.lds, c, n, s + v * EP);
      if (!kHold) load_wb(v);
#pragma unroll
      for (int j = 0; j < EP; ++j) u[j] = fmaf((s[v * EP + j] - mu) * rstd, w[v * EP + j], b[v * EP + j]);
      store_row<E, M>((E*)a.y + r * a.ldy, c, n, u);
    }
  }
}

// Rows longer than a workgroup's registers hold: three passes over the row (mean, variance,
// output), the sum made again in each.
template <class E, int M>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  constexpr int EP = kPiece<E>;
  typedef RowSum<1024, 1, 1024> Sum;
  __shared__ typename Sum::Buffer buf;
  int turn = 0;
  const int n = (int)a.n;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    auto piece = [&](int c, float* s) {
      float u[EP];
      unpack_row<E, M>(load_row<E, M>((const E*)a.x + r * a.ldx, c, n), c, n, s);
      if (a.drop.on) drop_piece<E>(a.drop, (uint32_t)r, c, s);
      if (a.res) {
        unpack_row<E, M>(load_row<E, M>((const E*)a.res + r * a.ldr, c, n), c, n, u);
#pragma unroll
        for (int j = 0; j < EP; ++j) s[j] += u[j];
      }
    };
    float s[EP], w[EP], b[EP], red[1] = {0.f}, mu = 0.f;
    if (!a.rms) {
      for (int c = threadIdx.x * EP; c < n; c += 1024 * EP) {
        piece(c, s);
#pragma unroll
        for (int j = 0; j < EP; ++j) red[0] += (M == kWhole || c + j < n) ? s[j] : 0.f;
      }
      Sum::run(red, buf, turn);
      mu = red[0] * a.inv_n;
      red[0] = 0.f;
    }
    for (int c = threadIdx.x * EP; c < n; c += 1024 * EP) {
      piece(c, s);
#pragma unroll
      for (int j = 0; j < EP; ++j) {
        const float d = (M == kWhole || c + j < n) ? s[j] - mu : 0.f;
        red[0] = fmaf(d, d, red[0]);
      }
    }
    Sum::run(red, buf, turn);
    const float rstd = 1.f / sqrtf(fmaf(red[0], a.inv_n, a.eps));
    for (int c = threadIdx.x * EP; c < n; c += 1024 * EP) {
      piece(c, s);
      if (a.sum) store_row<E, M>((E*)a.sum + r * a.lds, c, n, s);
      load_vec<EP>(a.w, a.wbf16, c, n, 1.f, w);
      load_vec<EP>(a.b, a.wbf16, c, n, 0.f, b);
#pragma unroll
      for (int j = 0; j < EP; ++j) s[j] = fmaf((s[j] - mu) * rstd, w[j], b[j]);
      store_row<E, M>((E*)a.y + r * a.ldy, c, n, s);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mu;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
}

// Threads per row: a power of two with 16 columns each (two bf16 or four fp32 pieces of every
// tensor in flight per thread), and two workgroups per CU.  32768 rows of 2048 bf16 with
// residual, dropout and statistics took 98 us so, 106 with four or eight per CU, 98 to 107
// with 32 columns per thread (196 registers) and, in the plain form, 92 against 49 with
// 8 columns (half as much in flight).
template <class E, int M>
static void launch_norm_of(const NormArgs& a, hipStream_t st) {
  auto go = [&](auto kernel, int block, int rows_per_block) {
    const int64_t blocks = std::min<int64_t>(ceil_div(a.rows, rows_per_block), kNormBlocks);
    DPRC_LAUNCH(kernel, dim3((unsigned)blocks), dim3(block), 0, st, a);
  };
  const int64_t n = a.n;
  if (n <= 64) return go(norm_kernel<E, M, 8, 8>, 256, 32);
  if constexpr (M != kTiny) {
    // At most one row per workgroup: a row's latency counts, 8 columns per thread (one row of 2048:
    // 2.9 us against 3.5, 512 rows: 4.1 against 4.5; from 1024 rows on it is slower).  Past
    // 4096 columns the two are alike.
    if (a.rows <= kNormBlocks && n > 512 && n <= 4096) {
      if (n <= 1024) return go(norm_kernel<E, M, 128, 8>, 256, 2);
      if (n <= 2048) return go(norm_kernel<E, M, 256, 8>, 256, 1);
      return go(norm_kernel<E, M, 512, 8>, 512, 1);
    }
    if (n <= 128) return go(norm_kernel<E, M, 8, 16>, 256, 32);
    if (n <= 256) return go(norm_kernel<E, M, 16, 16>, 256, 16);
    if (n <= 512) return go(norm_kernel<E, M, 32, 16>, 256, 8);
    if (n <= 1024) return go(norm_kernel<E, M, 64, 16>, 256, 4);
    if (n <= 2048) return go(norm_kernel<E, M, 128, 16>, 256, 2);
    if (n <= 4096) return go(norm_kernel<E, M, 256, 16>, 256, 1);
    if (n <= 8192) return go(norm_kernel<E, M, 512, 16>, 512, 1);
    if (n <= 16384) return go(norm_kernel<E, M, 1024, 16>, 1024, 1);
    go(norm_long_kernel<E, M>, 1024, 1);
  }
}

template <class E>
static void launch_norm_width(const NormArgs& a, hipStream_t st) {
  if (a.n < kPiece<E>) launch_norm_of<E, kTiny>(a, st);
  else if (a.n % kPiece<E> == 0) launch_norm_of<E, kWhole>(a, st);
  else launch_norm_of<E, kTail>(a, st);
}

hipError_t launch_norm(const NormArgs& a, hipStream_t st) {
  if (a.bf16) launch_norm_width<uint16_t>(a, st);
  else launch_norm_width<float>(a, st);
  return hipGetLastError();
}

}  // namespace dprc
