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
  if (t.cols >= a.chunk) {
    const int64_t per = (t.cols + a.chunk - 1) / a.chunk;
    k.row = c / per;
    k.col = (c - k.row * per) * a.chunk;
    k.cols = min(a.chunk, t.cols - k.col);
  } else {
    const int64_t rows = a.chunk / t.cols;
    k.row = c * rows;
    k.rows = min(rows, t.rows - k.row);
    k.cols = t.cols;
  }
  return k;
}

// Threads of a row of n columns: all of the workgroup, or a power of two of them with a piece each.
template <class E>
__device__ __forceinline__ int grad_tpr(int64_t n, int threads) {
  int tpr = 1;
  while (tpr < threads && tpr * kPiece<E> < n) tpr *= 2;
  return tpr;
}

__device__ __forceinline__ double get64(uint16_t x) { return (double)bf16_to_f32(x); }
__device__ __forceinline__ double get64(float x) { return (double)x; }

constexpr int kGradUnroll = 4;      // pieces loaded before the first is worked on

template <class E, bool NT>
__device__ __forceinline__ double row_squares(const E* row, int64_t n, int lane, int tpr, double t) {
  constexpr int EP = kPiece<E>, U = kGradUnroll;
  const int64_t step = (int64_t)EP * tpr;
  int64_t c = (int64_t)EP * lane;
  for (; c + (U - 1) * step + EP <= n; c += U * step) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_piece<E, NT>(row + c + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[EP];
      unpack<E>(v[u], x);
#pragma unroll
      for (int j = 0; j < EP; ++j) t = fma((double)x[j], (double)x[j], t);
    }
  }
  for (; c < n; c += step) {
    if (c + EP <= n) {
      float x[EP];
      unpack<E>(load_piece<E>(row + c), x);
#pragma unroll
      for (int j = 0; j < EP; ++j) t = fma((double)x[j], (double)x[j], t);
    } else {
      for (int64_t j = c; j < n; ++j) t = fma(get64(row[j]), get64(row[j]), t);
    }
  }
  return t;
}

template <class E, bool NT>
__device__ __forceinline__ double chunk_squares(const GradTensor& g, const GradChunk& k, int threads, double t) {
  const int tpr = grad_tpr<E>(k.cols, threads), lane = threadIdx.x & (tpr - 1);
  for (int64_t r = threadIdx.x / tpr; r < k.rows; r += threads / tpr)
    t = row_squares<E, NT>((const E*)g.x + (k.row + r) * g.ldx + k.col, k.cols, lane, tpr, t);
  return t;
}

template <int WAVES>
__device__ __forceinline__ double block_sum(double t) {
  __shared__ double buf[WAVES];
  t = wave_sum(t);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = t;
  __syncthreads();
  t = 0.0;
  for (int w = 0; w < WAVES; ++w) t += buf[w];
  __syncthreads();
  return t;
}

// Chunks before a.keep are read past the caches, which then hold the last ones when the scaling begins.  So for one launch
// (kGradTensors tensors).  Of several each keeps its own end, and they are scaled in the order of the squares: the later
// ones have pushed out what the first left.  113 fp32 tensors of 4.9 GB: 3063 us, norm alone 1143; 160 bf16 tensors of
// 512 MB: 578, norm alone 263 (launches of 256 workgroups one after the other).
__global__ __launch_bounds__(256) void grad_squares_kernel(GradArgs a) {
  double t = 0.0;
  for (int64_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const GradChunk k = grad_chunk(a, c);
    const GradTensor& g = a.t[k.tensor];
    if (c < a.keep) t = g.bf16 ? chunk_squares<uint16_t, true>(g, k, 256, t) : chunk_squares<float, true>(g, k, 256, t);
    else t = g.bf16 ? chunk_squares<uint16_t, false>(g, k, 256, t) : chunk_squares<float, false>(g, k, 256, t);
  }
  t = block_sum<4>(t);
  if (threadIdx.x == 0) a.part[a.part0 + blockIdx.x] = t;
}

// The sum of all parts, the same in every workgroup.
__device__ __forceinline__ double grad_total(const GradArgs& a) {
  double t = 0.0;
  for (int k = threadIdx.x; k < a.parts; k += 256) t += a.part[k];
  return block_sum<4>(t);
}

__global__ __launch_bounds__(256) void grad_norm_kernel(GradArgs a) {
  const double t = grad_total(a);
  if (threadIdx.x == 0) *a.norm = (float)sqrt(t);
}

// min(1, max_norm / norm), 0 for a norm that is not finite
__device__ __forceinline__ double grad_factor(const GradArgs& a, double norm) {
  return !(norm <= 1.7976931348623157e308) ? 0.0 : norm <= a.max_norm ? 1.0 : a.max_norm / norm;
}

// c x to out in fp32, or with WIDE in fp64: for a factor that fp32 holds in fewer bits, or not at all.
template <class E, bool NT, bool WIDE>
__device__ __forceinline__ void scale_row(const E* x, E* out, int64_t n, int lane, int tpr, double c) {
  constexpr int EP = kPiece<E>, U = kGradUnroll;
  const int64_t step = (int64_t)EP * tpr;
  const float cf = (float)c;
  auto times = [&](float v) __attribute__((always_inline)) { return WIDE ? (float)((double)v * c) : v * cf; };
  int64_t k = (int64_t)EP * lane;
  for (; k + (U - 1) * step + EP <= n; k += U * step) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_piece<E, NT>(x + k + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float y[EP];
      unpack<E>(v[u], y);
#pragma unroll
      for (int j = 0; j < EP; ++j) y[j] = times(y[j]);
      store_piece<E, NT>(out + k + u * step, pack<E>(y));
    }
  }
  for (; k < n; k += step) {
    if (k + EP <= n) {
      float y[EP];
      unpack<E>(load_piece<E>(x + k), y);
#pragma unroll
      for (int j = 0; j < EP; ++j) y[j] = times(y[j]);
      store_piece<E>(out + k, pack<E>(y));
    } else {
      for (int64_t j = k; j < n; ++j) {
        const float y = times((float)get64(x[j]));
        if constexpr (sizeof(E) == 2) out[j] = __builtin_bit_cast(uint16_t, (__bf16)y);
        else out[j] = y;
      }
    }
  }
}

// Zeros for c = 0 (a norm that is not finite): nothing is read, so that no NaN survives.
template <class E>
__device__ __forceinline__ void zero_row(E* out, int64_t n, int lane, int tpr) {
  constexpr int EP = kPiece<E>;
  for (int64_t k = (int64_t)EP * lane; k < n; k += (int64_t)EP * tpr) {
    if (k + EP <= n) store_piece<E>(out + k, uint4{0, 0, 0, 0});
    else
      for (int64_t j = k; j < n; ++j) out[j] = (E)0;
  }
}

template <class E, bool NT>
__device__ __forceinline__ void chunk_scale(const GradTensor& g, const GradChunk& k, int threads, double c) {
  if (c == 1.0 && g.out == g.x) return;                  // its values already
  const int tpr = grad_tpr<E>(k.cols, threads), lane = threadIdx.x & (tpr - 1);
  for (int64_t r = threadIdx.x / tpr; r < k.rows; r += threads / tpr) {
    const E* x = (const E*)g.x + (k.row + r) * g.ldx + k.col;
    E* out = (E*)g.out + (k.row + r) * g.ldo + k.col;
    if (c == 0.0) zero_row<E>(out, k.cols, lane, tpr);
    else if (c < 0x1p-100) scale_row<E, NT, true>(x, out, k.cols, lane, tpr, c);
    else scale_row<E, NT, false>(x, out, k.cols, lane, tpr, c);
  }
}

// From the launch's last chunk on: where it is the only launch, what the squares read last is still in the caches.
__global__ __launch_bounds__(256) void grad_scale_kernel(GradArgs a) {
  const double norm = sqrt(grad_total(a)), c = grad_factor(a, norm);
  if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  for (int64_t q = a.chunks - 1 - blockIdx.x; q >= 0; q -= gridDim.x) {
    const GradChunk k = grad_chunk(a, q);
    const GradTensor& g = a.t[k.tensor];
    if (a.keep > 0) {
      if (g.bf16) chunk_scale<uint16_t, true>(g, k, 256, c);
      else chunk_scale<float, true>(g, k, 256, c);
    } else {
      if (g.bf16) chunk_scale<uint16_t, false>(g, k, 256, c);
      else chunk_scale<float, false>(g, k, 256, c);
    }
  }
}

// Few elements in all: one workgroup does both.
__global__ __launch_bounds__(1024) void grad_small_kernel(GradArgs a) {
  double t = 0.0;
  for (int i = 0; i < a.count; ++i) {
    const GradTensor& g = a.t[i];
    const GradChunk k{i, 0, g.rows, 0, g.cols};
    t = g.bf16 ? chunk_squares<uint16_t, false>(g, k, 1024, t) : chunk_squares<float, false>(g, k, 1024, t);
  }
  const double norm = sqrt(block_sum<16>(t)), c = grad_factor(a, norm);
  if (a.norm && threadIdx.x == 0) *a.norm = (float)norm;
  for (int i = 0; i < a.count; ++i) {
    const GradTensor& g = a.t[i];
    const GradChunk k{i, 0, g.rows, 0, g.cols};
    if (g.bf16) chunk_scale<uint16_t, false>(g, k, 1024, c);
    else chunk_scale<float, false>(g, k, 1024, c);
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
hipError_t launch_grad_small(const GradArgs& a, hipStream_t st) {
  DPRC_LAUNCH(grad_small_kernel, dim3(1), dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace dprc
