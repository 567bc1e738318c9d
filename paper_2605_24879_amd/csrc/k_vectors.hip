// Per-sample vector gradients G [B, n]: squared norms and clipped sums.  Bounded by memory, or by a
// launch's latency for the few vectors of a small batch.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

// Four columns from c (at any 4-byte address), or the row's last four where fewer are left: then the
// first `skip` of them belong to the thread before.
__device__ __forceinline__ void load4(const float* row, int64_t c, int64_t n, float (&x)[4]) {
  unpack<float>(load_piece(row + std::min(c, n - 4)), x);
}
__device__ __forceinline__ int skip4(int64_t c, int64_t n) { return (int)std::max<int64_t>(0, c + 4 - n); }

// ---- squared norms --------------------------------------------------------------------------------

constexpr int kNormUnroll = 8;

// A workgroup per sample and split, in fp64 (a sample's sum may mix large and small layers, and the
// conversions cost less than the loads).  TINY: fewer than four columns.
template <int BLK, bool TINY>
__global__ __launch_bounds__(BLK) void vector_norms_kernel(VectorArgs a, int64_t per, int64_t blocks) {
  __shared__ double buf[BLK / 64];
  const int64_t blk = flat_block();
  if (blk >= blocks) return;
  const int64_t i = blk / a.S, first = (blk - i * a.S) * per, last = std::min(a.n, first + per);
  const float* row = a.G + i * a.ldg;
  double t = 0.0;
  if (TINY) {
    if (threadIdx.x < a.n) t = (double)row[threadIdx.x] * row[threadIdx.x];
  } else {
    int64_t c = first + 4 * threadIdx.x;
    // whole rounds, all loads first
    for (; c + (kNormUnroll - 1) * 4 * BLK + 4 <= last; c += kNormUnroll * 4 * BLK) {
      float x[kNormUnroll][4];
#pragma unroll
      for (int u = 0; u < kNormUnroll; ++u) load4(row, c + u * 4 * BLK, a.n, x[u]);
#pragma unroll
      for (int u = 0; u < kNormUnroll; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) t = fma((double)x[u][j], (double)x[u][j], t);
    }
    float x[kNormUnroll][4];
#pragma unroll
    for (int u = 0; u < kNormUnroll; ++u) load4(row, c + u * 4 * BLK, a.n, x[u]);
#pragma unroll
    for (int u = 0; u < kNormUnroll; ++u) {
      const int64_t cu = c + u * 4 * BLK;
      if (cu >= last) continue;
      const int skip = skip4(cu, a.n);
#pragma unroll
      for (int j = 0; j < 4; ++j) t = j >= skip ? fma((double)x[u][j], (double)x[u][j], t) : t;
    }
  }
  t = wave_sum(t);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x > 0) return;
  t = 0.0;
  for (int k = 0; k < BLK / 64; ++k) t += buf[k];
  if (a.S > 1) static_cast<double*>(a.part)[blk] = t;
  else a.out[i] = a.accumulate ? a.out[i] + (float)t : (float)t;
}

// the sum of a sample's splits, in their order
__global__ __launch_bounds__(64) void vector_norm_splits_kernel(VectorArgs a) {
  const int64_t i = flat_block();
  if (i >= a.B) return;
  double t = 0.0;
  for (int k = threadIdx.x; k < a.S; k += 64) t += static_cast<const double*>(a.part)[i * a.S + k];
  t = wave_sum(t);
  if (threadIdx.x == 0) a.out[i] = a.accumulate ? a.out[i] + (float)t : (float)t;
}

// A sample's columns are split where one workgroup would take longer than a second launch: 8 x 300000
// went from 22.5 to 7.6 us with 16 splits, 16 x 135168 from 11.9 to 7.6 with 8; 8 x 67584 takes 5.7 us
// whole and 6.2 split, 256 x 135168 25.4 whole (5.4 TB/s).
int vector_norm_splits(int64_t B, int64_t n) {
  return n < 98304 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(128 / B, n >> 14));
}

hipError_t launch_vector_norms(const VectorArgs& a, hipStream_t st) {
  const int64_t per = round_up(ceil_div(a.n, (int64_t)a.S), 4), blocks = a.B * a.S;
  if (a.n < 4) DPRC_LAUNCH((vector_norms_kernel<64, true>), flat_grid(blocks), dim3(64), 0, st, a, per, blocks);
  else if (a.n <= 4096) DPRC_LAUNCH((vector_norms_kernel<256, false>), flat_grid(blocks), dim3(256), 0, st, a, per, blocks);
  else DPRC_LAUNCH((vector_norms_kernel<1024, false>), flat_grid(blocks), dim3(1024), 0, st, a, per, blocks);
  if (a.S > 1) DPRC_LAUNCH(vector_norm_splits_kernel, flat_grid(a.B), dim3(64), 0, st, a);
  return hipGetLastError();
}

// ---- clipped sums -----------------------------------------------------------------------------------

constexpr int kSumUnroll = 8;

// LANES threads of four columns each and 256 / LANES groups of samples a workgroup, whose sums
// meet in LDS; a.S > 1 splits the samples over workgroups too (partial sums [S][n]).  A
// dropped sample's values (c = 0) are read but never enter a sum.
template <int LANES, bool TINY>
__global__ __launch_bounds__(256) void vector_sums_kernel(VectorArgs a, int64_t per, int64_t col_blocks) {
  constexpr int G = 256 / LANES;
  __shared__ float sums[G][LANES][4];
  const int64_t blk = flat_block(), split = blk / col_blocks;
  if (split >= a.S) return;
  const int lane = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  const int64_t c = ((blk - split * col_blocks) * LANES + lane) * 4;
  const int64_t first = split * per, last = std::min(a.B, first + per);
  float t[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t i0 = first + grp; i0 < last; i0 += kSumUnroll * G) {
    float x[kSumUnroll][4], f[kSumUnroll];
#pragma unroll
    for (int u = 0; u < kSumUnroll; ++u) {
      const int64_t i = std::min(i0 + u * G, last - 1);
      f[u] = a.c[i];
      const float* row = a.G + i * a.ldg;
      if (TINY)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[u][j] = j < a.n ? row[j] : 0.f;
      else load4(row, c, a.n, x[u]);
    }
#pragma unroll
    for (int u = 0; u < kSumUnroll; ++u) {
      if (i0 + u * G >= last || f[u] == 0.f) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) t[j] = fmaf(f[u], x[u][j], t[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) sums[grp][lane][j] = t[j];
  __syncthreads();
  if (grp > 0 || c >= a.n) return;
  for (int g = 1; g < G; ++g)
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] += sums[g][lane][j];
  const int skip = TINY ? 0 : skip4(c, a.n);
  float* out = (a.S > 1 ? static_cast<float*>(a.part) + split * a.n : a.out) + (TINY ? 0 : std::min(c, a.n - 4));
  const bool add = a.S == 1 && a.accumulate;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j >= skip && (!TINY || j < a.n)) out[j] = add ? out[j] + t[j] : t[j];
}

__global__ __launch_bounds__(256) void vector_sum_splits_kernel(VectorArgs a) {
  const int64_t c = (int64_t)flat_block() * 256 + threadIdx.x;
  if (c >= a.n) return;
  float t = 0.f;
  for (int k = 0; k < a.S; ++k) t += static_cast<const float*>(a.part)[k * a.n + c];
  a.out[c] = a.accumulate ? a.out[c] + t : t;
}

// Long vectors fill the GPU with 256 columns a workgroup (256 x 135168: 28 us, 5.0 TB/s; 8 x 67584: 3.2 us
// against 3.6 with 64 columns); shorter ones take 64 columns and four times as many sample groups
// (256 x 256: 3.2 us against 6.9), and very many samples are split.
constexpr int64_t kLongVector = 16384;
int vector_sum_splits(int64_t B, int64_t n) {
  return n >= kLongVector ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(256 / ceil_div(n, 64), B >> 10));
}

hipError_t launch_vector_sums(const VectorArgs& a, hipStream_t st) {
  const int64_t per = ceil_div(a.B, (int64_t)a.S);
  if (a.n < 4) {
    DPRC_LAUNCH((vector_sums_kernel<16, true>), flat_grid(a.S), dim3(256), 0, st, a, per, (int64_t)1);
  } else if (a.n >= kLongVector) {
    const int64_t cb = ceil_div(a.n, 256);
    DPRC_LAUNCH((vector_sums_kernel<64, false>), flat_grid(cb * a.S), dim3(256), 0, st, a, per, cb);
  } else {
    const int64_t cb = ceil_div(a.n, 64);
    DPRC_LAUNCH((vector_sums_kernel<16, false>), flat_grid(cb * a.S), dim3(256), 0, st, a, per, cb);
  }
  if (a.S > 1) DPRC_LAUNCH(vector_sum_splits_kernel, flat_grid(ceil_div(a.n, 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace dprc
