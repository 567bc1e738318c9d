// Per-sample vector gradients G [B, n]: squared norms and clipped sums.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"

namespace dprc {

int vector_norm_splits(int64_t B, int64_t n) { return 1; }
int vector_sum_splits(int64_t B, int64_t n) { return 1; }

// one workgroup per sample
__global__ __launch_bounds__(256) void vector_norms_kernel(VectorArgs a) {
  __shared__ double buf[4];
  const int64_t i = flat_block();
  if (i >= a.B) return;
  double t = 0.0;
  for (int64_t c = threadIdx.x; c < a.n; c += 256) {
    const double v = a.G[i * a.ldg + c];
    t = fma(v, v, t);
  }
  t = wave_sum(t);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    const float v = (float)((buf[0] + buf[1]) + (buf[2] + buf[3]));
    a.out[i] = a.accumulate ? a.out[i] + v : v;
  }
}

hipError_t launch_vector_norms(const VectorArgs& a, hipStream_t st) {
  DPRC_LAUNCH(vector_norms_kernel, flat_grid(a.B), dim3(256), 0, st, a);
  return hipGetLastError();
}

// one thread per column
__global__ __launch_bounds__(256) void vector_sums_kernel(VectorArgs a) {
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < a.n; c += (int64_t)gridDim.x * 256) {
    float t = a.accumulate ? a.out[c] : 0.f;
    for (int64_t i = 0; i < a.B; ++i) {
      const float f = a.c[i];
      if (f != 0.f) t = fmaf(f, a.G[i * a.ldg + c], t);
    }
    a.out[c] = t;
  }
}

hipError_t launch_vector_sums(const VectorArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a.n, 256), 65536));
  DPRC_LAUNCH(vector_sums_kernel, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace dprc
