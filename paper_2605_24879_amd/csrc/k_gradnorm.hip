// The joint norm of many tensors and their clipping: norm = sqrt(sum x^2), out = min(1, max_norm / norm) x.
//
// Bounded by memory (the tensors are read twice and written once), or by the launches for small models.
// Squares are taken and summed in fp64: a square of any fp32 value is exact there and can neither overflow nor
// vanish, and the conversions cost less than the loads.  The sums have a fixed order.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

// The chunk's tensor, and its rows and columns there.
struct GradChunk {
  int tensor;
  int64_t row, rows, col, cols;
};
__device__ __forceinline__ GradChunk grad_chunk(const GradArgs& a, int64_t c) {
  int i = 0;
  while (i + 1 < a.count && c >= a.t[i + 1].chunk0) ++i;
  const GradTensor& t = a.t[i];
  c -= t.chunk0;
  GradChunk k{i, 0, 1, 0, 0};
  if (t.cols >= kGradChunk) {
    const int64_t per = (t.cols + kGradChunk - 1) / kGradChunk;
    k.row = c / per;
    k.col = (c - k.row * per) * kGradChunk;
    k.cols = min(kGradChunk, t.cols - k.col);
  } else {
    const int64_t rows = kGradChunk / t.cols;
    k.row = c * rows;
    k.rows = min(rows, t.rows - k.row);
    k.cols = t.cols;
  }
  return k;
}

template <class E>
__device__ __forceinline__ double row_squares(const E* row, int64_t n, double t) {
  constexpr int EP = kPiece<E>;
  constexpr int U = 4;
  int64_t c = EP * threadIdx.x;
  for (; c + (U - 1) * EP * 256 + EP <= n; c += U * EP * 256) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_piece<E>(row + c + u * EP * 256);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[EP];
      unpack<E>(v[u], x);
#pragma unroll
      for (int j = 0; j < EP; ++j) t = fma((double)x[j], (double)x[j], t);
    }
  }
  for (; c < n; c += EP * 256) {
    if (c + EP <= n) {
      float x[EP];
      unpack<E>(load_piece<E>(row + c), x);
#pragma unroll
      for (int j = 0; j < EP; ++j) t = fma((double)x[j], (double)x[j], t);
    } else {
      for (int64_t j = c; j < n; ++j) {
        const double x = sizeof(E) == 2 ? (double)bf16_to_f32((uint32_t)row[j]) : (double)row[j];
        t = fma(x, x, t);
      }
    }
  }
  return t;
}

__device__ __forceinline__ double block_sum(double t) {
  __shared__ double buf[4];
  t = wave_sum(t);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = t;
  __syncthreads();
  t = buf[0] + buf[1] + buf[2] + buf[3];
  __syncthreads();
  return t;
}

__global__ __launch_bounds__(256) void grad_squares_kernel(GradArgs a) {
  double t = 0.0;
  for (int64_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const GradChunk k = grad_chunk(a, c);
    const GradTensor& g = a.t[k.tensor];
    for (int64_t r = k.row; r < k.row + k.rows; ++r) {
      if (g.bf16) t = row_squares<uint16_t>((const uint16_t*)g.x + r * g.ldx + k.col, k.cols, t);
      else t = row_squares<float>((const float*)g.x + r * g.ldx + k.col, k.cols, t);
    }
  }
  t = block_sum(t);
  if (threadIdx.x == 0) a.part[a.part0 + blockIdx.x] = t;
}

// The sum of all parts, the same in every workgroup.
__device__ __forceinline__ double grad_total(const GradArgs& a) {
  double t = 0.0;
  for (int k = threadIdx.x; k < a.parts; k += 256) t += a.part[k];
  return block_sum(t);
}

__global__ __launch_bounds__(256) void grad_norm_kernel(GradArgs a) {
  const double t = grad_total(a);
  if (threadIdx.x == 0) *a.norm = (float)sqrt(t);
}

// c x to out, the factor and the product in fp64 (a factor of fp32 could be subnormal where x is large).
// Nothing is read where c = 0 (a norm that is not finite), so that no NaN survives.
template <class E>
__device__ __forceinline__ void scale_row(const E* x, E* out, int64_t n, double c) {
  constexpr int EP = kPiece<E>;
  for (int64_t k = EP * threadIdx.x; k < n; k += EP * 256) {
    if (k + EP <= n) {
      float v[EP] = {};
      if (c != 0.0) unpack<E>(load_piece<E>(x + k), v);
#pragma unroll
      for (int j = 0; j < EP; ++j) v[j] = (float)((double)v[j] * c);
      store_piece<E>(out + k, pack<E>(v));
    } else {
      for (int64_t j = k; j < n; ++j) {
        if constexpr (sizeof(E) == 2)
          out[j] = c != 0.0 ? __builtin_bit_cast(uint16_t, (__bf16)(float)((double)bf16_to_f32(x[j]) * c)) : 0;
        else out[j] = c != 0.0 ? (float)((double)x[j] * c) : 0.f;
      }
    }
  }
}

__global__ __launch_bounds__(256) void grad_scale_kernel(GradArgs a) {
  const double norm = sqrt(grad_total(a));
  if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  const double c = !(norm <= 1.7976931348623157e308) ? 0.0 : norm <= a.max_norm ? 1.0 : a.max_norm / norm;
  for (int64_t q = blockIdx.x; q < a.chunks; q += gridDim.x) {
    const GradChunk k = grad_chunk(a, q);
    const GradTensor& g = a.t[k.tensor];
    if (c == 1.0 && g.out == g.x) continue;              // its values already
    for (int64_t r = k.row; r < k.row + k.rows; ++r) {
      if (g.bf16) scale_row<uint16_t>((const uint16_t*)g.x + r * g.ldx + k.col, (uint16_t*)g.out + r * g.ldo + k.col, k.cols, c);
      else scale_row<float>((const float*)g.x + r * g.ldx + k.col, (float*)g.out + r * g.ldo + k.col, k.cols, c);
    }
  }
}

hipError_t launch_grad_squares(const GradArgs& a, hipStream_t st) {
  DPRC_LAUNCH(grad_squares_kernel, dim3((unsigned)a.blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_grad_norm(const GradArgs& a, hipStream_t st) {
  DPRC_LAUNCH(grad_norm_kernel, dim3(1), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_grad_scale(const GradArgs& a, hipStream_t st) {
  DPRC_LAUNCH(grad_scale_kernel, dim3((unsigned)a.blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace dprc
