// Dropout, residual sum and norm of token rows, and the backward pass.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

template <class E>
__device__ __forceinline__ void sum_piece(const NormArgs& a, int64_t r, int64_t c, int m, float (&x)[8]) {
  load8((const E*)a.x + r * a.ldx + c, m, x);
  drop8(a.drop, (uint32_t)r, (uint32_t)(c >> 3), x);
  if (!a.res) return;
  float z[8];
  load8((const E*)a.res + r * a.ldr + c, m, z);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] += z[j];
}

// One workgroup per row, three passes over it: mean, variance, output.
template <class E>
__global__ __launch_bounds__(256) void norm_kernel(NormArgs a) {
  __shared__ float buf[4];
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    float x[8], mu = 0.f, t = 0.f;
    if (!a.rms) {
      for (int64_t c = 8 * threadIdx.x; c < a.n; c += 8 * 256) {
        sum_piece<E>(a, r, c, (int)std::min<int64_t>(8, a.n - c), x);
#pragma unroll
        for (int j = 0; j < 8; ++j) t += x[j];
      }
      mu = block_sum(t, buf) * a.inv_n;
      t = 0.f;
    }
    for (int64_t c = 8 * threadIdx.x; c < a.n; c += 8 * 256) {
      const int m = (int)std::min<int64_t>(8, a.n - c);
      sum_piece<E>(a, r, c, m, x);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < m) t = fmaf(x[j] - mu, x[j] - mu, t);
    }
    const float rstd = 1.f / sqrtf(fmaf(block_sum(t, buf), a.inv_n, a.eps));
    for (int64_t c = 8 * threadIdx.x; c < a.n; c += 8 * 256) {
      const int m = (int)std::min<int64_t>(8, a.n - c);
      sum_piece<E>(a, r, c, m, x);
      if (a.sum) store8((E*)a.sum + r * a.lds + c, m, x);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < m)
          x[j] = fmaf((x[j] - mu) * rstd, vec_entry(a.w, a.wbf16, c + j, 1.f), vec_entry(a.b, a.wbf16, c + j, 0.f));
      store8((E*)a.y + r * a.ldy + c, m, x);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mu;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
}

hipError_t launch_norm(const NormArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)std::min<int64_t>(a.rows, 65536));
  if (a.bf16) DPRC_LAUNCH((norm_kernel<uint16_t>), grid, dim3(256), 0, st, a);
  else DPRC_LAUNCH((norm_kernel<float>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

// ---- backward ---------------------------------------------------------------------------------

// xh and g = dy w of 8 columns of row r
template <class E>
__device__ __forceinline__ void back_piece(const NormBackArgs& a, int64_t r, int64_t c, int m, float mu, float rstd,
                                           float (&dy)[8], float (&xh)[8], float (&g)[8]) {
  load8((const E*)a.dy + r * a.lddy + c, m, dy);
  load8((const E*)a.s + r * a.lds + c, m, xh);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    xh[j] = j < m ? (xh[j] - mu) * rstd : 0.f;
    g[j] = j < m ? dy[j] * vec_entry(a.w, a.wbf16, c + j, 1.f) : 0.f;
  }
}

// dx and dh: one workgroup per row, two passes over it.
template <class E>
__global__ __launch_bounds__(256) void norm_back_rows_kernel(NormBackArgs a) {
  __shared__ float buf[4];
  const int64_t rows = a.B * a.T;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const float mu = a.rms ? 0.f : a.mean[r], rstd = a.rstd[r];
    float dy[8], xh[8], g[8], sg = 0.f, sgx = 0.f;
    for (int64_t c = 8 * threadIdx.x; c < a.n; c += 8 * 256) {
      back_piece<E>(a, r, c, (int)std::min<int64_t>(8, a.n - c), mu, rstd, dy, xh, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sg += g[j];
        sgx = fmaf(g[j], xh[j], sgx);
      }
    }
    sg = a.rms ? 0.f : block_sum(sg, buf) * a.inv_n;
    sgx = block_sum(sgx, buf) * a.inv_n;
    for (int64_t c = 8 * threadIdx.x; c < a.n; c += 8 * 256) {
      const int m = (int)std::min<int64_t>(8, a.n - c);
      back_piece<E>(a, r, c, m, mu, rstd, dy, xh, g);
      float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (a.ds) load8((const E*)a.ds + r * a.ldds + c, m, z);
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = fmaf(rstd, (g[j] - sg) - xh[j] * sgx, z[j]);
      if (a.dx) store8((E*)a.dx + r * a.lddx + c, m, z);
      drop8(a.drop, (uint32_t)r, (uint32_t)(c >> 3), z);
      if (a.dh) store8((E*)a.dh + r * a.lddh + c, m, z);
    }
  }
}

// dw and db: one thread per column and token split.
template <class E>
__global__ __launch_bounds__(256) void norm_back_cols_kernel(NormBackArgs a, int64_t col_blocks, int64_t blocks) {
  const int64_t blk = flat_block();
  if (blk >= blocks) return;
  const int64_t c = (blk % col_blocks) * 256 + threadIdx.x, is = blk / col_blocks;
  if (c >= a.n) return;
  const int64_t i = is / a.S, per = (a.T + a.S - 1) / a.S;
  const int64_t t0 = (is % a.S) * per, t1 = std::min<int64_t>(a.T, t0 + per);
  float dw = 0.f, db = 0.f;
  for (int64_t t = t0; t < t1; ++t) {
    const int64_t r = i * a.T + t;
    const float dy = to_f32(((const E*)a.dy)[r * a.lddy + c]);
    const float xh = (to_f32(((const E*)a.s)[r * a.lds + c]) - (a.rms ? 0.f : a.mean[r])) * a.rstd[r];
    dw = fmaf(dy, xh, dw);
    db += dy;
  }
  if (a.S > 1) {
    a.part[(is * 2 + 0) * a.n + c] = dw;
    a.part[(is * 2 + 1) * a.n + c] = db;
  } else {
    if (a.dw) a.dw[i * a.ldg + c] = dw;
    if (a.db) a.db[i * a.ldg + c] = db;
  }
}

int norm_back_splits(int64_t B, int64_t T, int64_t n) {
  const int64_t base = B * ceil_div(n, 256);
  return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(1024, base), T / 16));
}

hipError_t launch_norm_back(const NormBackArgs& a, hipStream_t st) {
  if (a.dw || a.db) {
    const int64_t cb = ceil_div(a.n, 256), blocks = a.B * a.S * cb;
    if (a.bf16) DPRC_LAUNCH((norm_back_cols_kernel<uint16_t>), flat_grid(blocks), dim3(256), 0, st, a, cb, blocks);
    else DPRC_LAUNCH((norm_back_cols_kernel<float>), flat_grid(blocks), dim3(256), 0, st, a, cb, blocks);
  }
  if (a.dx || a.dh) {
    const dim3 grid((unsigned)std::min<int64_t>(a.B * a.T, 65536));
    if (a.bf16) DPRC_LAUNCH((norm_back_rows_kernel<uint16_t>), grid, dim3(256), 0, st, a);
    else DPRC_LAUNCH((norm_back_rows_kernel<float>), grid, dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

// the token splits' partial sums of a sample, in their order
__global__ __launch_bounds__(256) void norm_back_sums_kernel(NormBackArgs a, int64_t col_blocks, int64_t blocks) {
  const int64_t blk = flat_block();
  if (blk >= blocks) return;
  const int64_t c = (blk % col_blocks) * 256 + threadIdx.x, i = blk / col_blocks;
  if (c >= a.n) return;
  float dw = 0.f, db = 0.f;
  for (int k = 0; k < a.S; ++k) {
    dw += a.part[((i * a.S + k) * 2 + 0) * a.n + c];
    db += a.part[((i * a.S + k) * 2 + 1) * a.n + c];
  }
  if (a.dw) a.dw[i * a.ldg + c] = dw;
  if (a.db) a.db[i * a.ldg + c] = db;
}

hipError_t launch_norm_back_sums(const NormBackArgs& a, hipStream_t st) {
  const int64_t cb = ceil_div(a.n, 256), blocks = a.B * cb;
  DPRC_LAUNCH(norm_back_sums_kernel, flat_grid(blocks), dim3(256), 0, st, a, cb, blocks);
  return hipGetLastError();
}

}  // namespace dprc
