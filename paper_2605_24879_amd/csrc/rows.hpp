// Token rows in 8-column pieces: loads, stores, dropout masks and sums over a workgroup.
#pragma once
#include "device.hpp"
#include "kernels.hpp"

namespace dprc {

__device__ __forceinline__ float to_f32(uint16_t h) { return bf16_to_f32(h); }
__device__ __forceinline__ float to_f32(float f) { return f; }
__device__ __forceinline__ void from_f32(float f, uint16_t& h) { h = (uint16_t)f32_to_bf16(f); }
__device__ __forceinline__ void from_f32(float f, float& h) { h = f; }

// the first m (at most 8) elements at p, zeros after them
template <class E>
__device__ __forceinline__ void load8(const E* p, int m, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = j < m ? to_f32(p[j]) : 0.f;
}

template <class E>
__device__ __forceinline__ void store8(E* p, int m, const float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < m) from_f32(x[j], p[j]);
}

// entry c of a weight or bias (fp32 or bf16), `none` without one
__device__ __forceinline__ float vec_entry(const void* v, int bf16, int64_t c, float none) {
  if (!v) return none;
  return bf16 ? bf16_to_f32(((const uint16_t*)v)[c]) : ((const float*)v)[c];
}

// x (columns 8 blk .. 8 blk + 7 of row r) through the site's dropout; a dropped element is 0
// whatever it was
__device__ __forceinline__ void drop8(const DropArgs& d, uint32_t r, uint32_t blk, float (&x)[8]) {
  if (!d.on) return;
  const u32x4 w = philox4x32_10(u32x4{blk, r, d.site, kStreamDropout}, d.key0, d.key1);
  const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t u = (j & 1) ? word[j >> 1] & 0xFFFF0000u : word[j >> 1] << 16;
    x[j] = u > d.lim ? x[j] * d.scale : 0.f;
  }
}

// sum over a workgroup of 256 threads, in every thread; `buf` is 4 floats of LDS
__device__ __forceinline__ float block_sum(float v, float* buf) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  return (buf[0] + buf[1]) + (buf[2] + buf[3]);
}

}  // namespace dprc
