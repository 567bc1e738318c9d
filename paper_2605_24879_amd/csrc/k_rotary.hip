// Rotary positions: features (a, b) of a head, the pair j < r of it, turned by the angle position * f_j:
//   a' = scale (a cos - b sin),  b' = scale (b cos + a sin)      (inverse: -sin),
// with a, b at features j and r + j (halves) or 2 j and 2 j + 1 (interleaved); features from 2 r on are copied.
// The inverse is the transpose, so it is the backward pass of the same call.
//
// Bounded by memory, or by a launch's latency for the few tokens of a serving step.  A workgroup takes whole
// tokens: their cosines and sines are made once for all heads of all tensors and kept in LDS.
// The angle is reduced to a fraction of a turn in 64 bits (in 32 a position of 10^6 would lose 0.06 of a
// radian); sine and cosine of the fraction are taken in 32.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

template <class E>
__device__ __forceinline__ void load8(const E* p, float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 8; k += kPiece<E>) unpack<E>(load_piece<E>(p + k), x + k);
}
template <class E>
__device__ __forceinline__ void store8(E* p, const float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 8; k += kPiece<E>) store_piece<E>(p + k, pack<E>(x + k));
}
__device__ __forceinline__ float get1(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float get1(const float* p) { return *p; }
__device__ __forceinline__ void put1(uint16_t* p, float x) {
  *p = __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ void put1(float* p, float x) { *p = x; }

__device__ __forceinline__ void turn(float2 cs, float& a, float& b) {
  const float c = a * cs.x - b * cs.y;
  b = b * cs.x + a * cs.y;
  a = c;
}

// Eight pairs from pair j on (or the r - j left), or eight features behind the pairs.
template <class X, class Y, bool INTERLEAVED>
__device__ __forceinline__ void rotary_unit(const X* x, Y* y, const float2* cs, int unit, int units, int r, int D) {
  if (unit >= units) {
    const int c = 2 * r + 8 * (unit - units);
    if (c + 8 <= D) {
      float v[8];
      load8<X>(x + c, v);
      store8<Y>(y + c, v);
    } else {
      for (int k = c; k < D; ++k) put1(y + k, get1(x + k));
    }
    return;
  }
  const int j = 8 * unit;
  if (j + 8 > r) {
    for (int k = j; k < r; ++k) {
      const int ia = INTERLEAVED ? 2 * k : k, ib = INTERLEAVED ? 2 * k + 1 : r + k;
      float a = get1(x + ia), b = get1(x + ib);
      turn(cs[k], a, b);
      put1(y + ia, a);
      put1(y + ib, b);
    }
    return;
  }
  float u[8], v[8];
  const int iu = INTERLEAVED ? 2 * j : j, iv = INTERLEAVED ? 2 * j + 8 : r + j;
  load8<X>(x + iu, u);
  load8<X>(x + iv, v);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if constexpr (INTERLEAVED) {
      if (k < 4) turn(cs[j + k], u[2 * k], u[2 * k + 1]);
      else turn(cs[j + k], v[2 * k - 8], v[2 * k - 7]);
    } else {
      turn(cs[j + k], u[k], v[k]);
    }
  }
  store8<Y>(y + iu, u);
  store8<Y>(y + iv, v);
}

template <class X, class Y, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  extern __shared__ __attribute__((aligned(16))) float2 cs[];
  const int64_t tokens = a.B * a.T, t0 = (int64_t)flat_block() * a.per_block;
  if (t0 >= tokens) return;
  const int n = (int)min((int64_t)a.per_block, tokens - t0), r = a.r;
  for (int s = threadIdx.x; s < n * r; s += 256) {
    const int k = s / r;
    const int64_t t = t0 + k;
    const double pos = (double)(a.pos ? a.pos[t] : a.start + t % a.T);
    double turns = pos * a.freqs[s - k * r] * 0.15915494309189533577;
    turns -= rint(turns);
    float sn, c;
    sincospif(2.f * (float)turns, &sn, &c);
    cs[s] = float2{a.scale * c, a.inverse ? -a.scale * sn : a.scale * sn};
  }
  __syncthreads();
  const int units = (r + 7) / 8, per_head = units + (a.D - 2 * r + 7) / 8, items = per_head * a.heads;
  for (int s = threadIdx.x; s < n * items; s += 256) {
    const int k = s / items, q = s - k * items;
    int head = q / per_head;
    const int unit = q - head * per_head;
    int i = 0;
    while (i + 1 < a.count && head >= a.x[i].H) head -= a.x[i++].H;
    const RotaryTensor& h = a.x[i];
    const int64_t b = (t0 + k) / a.T, t = t0 + k - b * a.T;
    rotary_unit<X, Y, INTERLEAVED>(static_cast<const X*>(h.x) + b * h.xb + t * h.xt + head * h.xh,
                                   static_cast<Y*>(h.y) + b * h.yb + t * h.yt + head * h.yh, cs + k * r, unit, units, r,
                                   a.D);
  }
}

hipError_t launch_rotary(RotaryArgs a, hipStream_t st) {
  const int64_t tokens = a.B * a.T, items = (int64_t)a.heads * ((a.r + 7) / 8 + (a.D - 2 * a.r + 7) / 8);
  int64_t per = std::max<int64_t>(1, 1280 / items);
  per = std::min<int64_t>({per, std::max<int64_t>(1, tokens / 512), 4096 / a.r});
  a.per_block = (int32_t)std::max<int64_t>(1, per);
  const dim3 grid = flat_grid(ceil_div(tokens, a.per_block));
  const size_t lds = sizeof(float2) * a.per_block * a.r;
  auto go = [&](auto kernel) { DPRC_LAUNCH(kernel, grid, dim3(256), lds, st, a); };
  auto types = [&](auto inter) {
    constexpr bool I = decltype(inter)::value;
    if (a.xbf16 && a.ybf16) go(rotary_kernel<uint16_t, uint16_t, I>);
    else if (a.xbf16) go(rotary_kernel<uint16_t, float, I>);
    else if (a.ybf16) go(rotary_kernel<float, uint16_t, I>);
    else go(rotary_kernel<float, float, I>);
  };
  if (a.interleaved) types(std::true_type{});
  else types(std::false_type{});
  return hipGetLastError();
}

}  // namespace dprc
