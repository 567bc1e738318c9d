// Dropout and residual sum: out = res + m x, m the site's mask times its scale.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

// One thread takes 8 columns of a row (one Philox block of mask bits) at a time.
template <class E>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, int64_t chunks) {
  const int64_t total = a.rows * chunks;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
    const int64_t r = q / chunks, c = 8 * (q - r * chunks);
    const int m = (int)std::min<int64_t>(8, a.n - c);
    float x[8], z[8];
    load8((const E*)a.x + r * a.ldx + c, m, x);
    drop8(a.drop, (uint32_t)r, (uint32_t)(c >> 3), x);
    if (a.res) {
      load8((const E*)a.res + r * a.ldr + c, m, z);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] += z[j];
    }
    store8((E*)a.out + r * a.ldo + c, m, x);
  }
}

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t st) {
  const int64_t chunks = ceil_div(a.n, 8);
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a.rows * chunks, 256), 65536));
  if (a.bf16) DPRC_LAUNCH((dropout_kernel<uint16_t>), grid, dim3(256), 0, st, a, chunks);
  else DPRC_LAUNCH((dropout_kernel<float>), grid, dim3(256), 0, st, a, chunks);
  return hipGetLastError();
}

}  // namespace dprc
