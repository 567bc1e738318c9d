// Rotary positions: features (a, b) of a head, the pair j < r of it, turned by the angle position * f_j:
//   a' = scale (a cos - b sin),  b' = scale (b cos + a sin)      (inverse: -sin),
// with a, b at features j and r + j (halves) or 2 j and 2 j + 1 (interleaved); features from 2 r on are copied.
// The inverse is the transpose, so it is the backward pass of the same call.
//
// Bounded by memory, or by a launch's latency for the few tokens of a serving step.  A workgroup takes whole
// tokens: their cosines and sines are made once for all heads of all tensors and kept in LDS.
// The angle is reduced to a fraction of a turn in 64 bits (in 32 a position of 10^6 would lose 0.06 of a
// radian), to an eighth of a turn beside whole quarters; sine and cosine of that are taken in 32.
// A thread takes eight pairs at a time, two 16-byte loads of bfloat16; the r mod 8 pairs left at the end of a head go as
// 4, 2 and 1 (one at a time: 138 us for 16 + 4 heads of 96 with r 13 and 2^15 tokens, results heads first, so 112;
// tokens first 88, with r 16 44).  32 + 8 heads of 64 bfloat16 features, 2^15 tokens: 72 us, 4.6 TB/s; with
// non-temporal loads and stores 77.  A step of 64 tokens: 3.8 us.  A workgroup reads x behind its angles' barrier, which
// adds their latencies: 12 us for 3063 tokens of 12 + 4 fp32 heads of 80, twice their bytes' time.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

// Eight features at any alignment of the element
template <class E>
__device__ __forceinline__ void load8(const E* p, float* x) {
#pragma unroll
  for (int k = 0; k < 8; k += kPiece<E>) unpack<E>(load_piece<E>(p + k), x + k);
}
template <class E>
__device__ __forceinline__ void store8(E* p, const float* x) {
#pragma unroll
  for (int k = 0; k < 8; k += kPiece<E>) store_piece<E>(p + k, pack<E>(x + k));
}

// The first n < 8 of them, as 4, 2 and 1; element i of what is loaded is in x[i] for the first four, then from x[4] on
// for the two and in x[6].
__device__ __forceinline__ void load_some(const uint16_t* p, int n, float* x) {
  if (n & 4) {
    const u32x2_any2 v = *reinterpret_cast<const u32x2_any2*>(p);
    x[0] = __uint_as_float(v[0] << 16); x[1] = __uint_as_float(v[0] & 0xFFFF0000u);
    x[2] = __uint_as_float(v[1] << 16); x[3] = __uint_as_float(v[1] & 0xFFFF0000u);
  }
  if (n & 2) {
    const uint32_t v = *reinterpret_cast<const u32_any2*>(p + (n & 4));
    x[4] = __uint_as_float(v << 16);
    x[5] = __uint_as_float(v & 0xFFFF0000u);
  }
  if (n & 1) x[6] = bf16_to_f32(p[n & 6]);
}
__device__ __forceinline__ void load_some(const float* p, int n, float* x) {
  if (n & 4) unpack<float>(load_piece<float>(p), x);
  if (n & 2) {
    x[4] = p[n & 4];
    x[5] = p[(n & 4) + 1];
  }
  if (n & 1) x[6] = p[n & 6];
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, bf16x2_t));
}
__device__ __forceinline__ void store_some(uint16_t* p, int n, const float* x) {
  if (n & 4) store_part(p, uint2{pack2(x[0], x[1]), pack2(x[2], x[3])});
  if (n & 2) store_part(p + (n & 4), pack2(x[4], x[5]));
  if (n & 1) p[n & 6] = (uint16_t)pack2(x[6], 0.f);
}
__device__ __forceinline__ void store_some(float* p, int n, const float* x) {
  if (n & 4) store_piece<float>(p, pack<float>(x));
  if (n & 2) {
    p[n & 4] = x[4];
    p[(n & 4) + 1] = x[5];
  }
  if (n & 1) p[n & 6] = x[6];
}
// where x[i] of these lies
__device__ __forceinline__ int some_at(int i, int n) { return i < 4 ? i : i < 6 ? (n & 4) + i - 4 : n & 6; }

__device__ __forceinline__ void turn(float2 cs, float& a, float& b) {
  const float c = a * cs.x - b * cs.y;
  b = b * cs.x + a * cs.y;
  a = c;
}

// Eight pairs from pair 8 * unit on (or the r - j left), or eight features behind the pairs.
template <class X, class Y, bool INTERLEAVED>
__device__ __forceinline__ void rotary_unit(const X* x, Y* y, const float2* cs, int unit, int units, int r, int D) {
  float u[8] = {}, v[8] = {};
  if (unit >= units) {
    const int c = 2 * r + 8 * (unit - units);
    if (c + 8 <= D) {
      load8<X>(x + c, v);
      store8<Y>(y + c, v);
    } else {
      load_some(x + c, D - c, v);
      store_some(y + c, D - c, v);
    }
    return;
  }
  const int j = 8 * unit, left = r - j;
  if (left >= 8) {
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
  } else if constexpr (INTERLEAVED) {                  // 4 pairs as 8 features, the others as 4 and 2
    const int rest = 2 * (left & 3), at = 2 * (r - (left & 3));
    if (left & 4) load8<X>(x + 2 * j, u);
    load_some(x + at, rest, v);
    if (left & 4) {
#pragma unroll
      for (int k = 0; k < 4; ++k) turn(cs[j + k], u[2 * k], u[2 * k + 1]);
      store8<Y>(y + 2 * j, u);
    }
    if (rest & 4) {
      turn(cs[at / 2], v[0], v[1]);
      turn(cs[at / 2 + 1], v[2], v[3]);
    }
    if (rest & 2) turn(cs[r - 1], v[4], v[5]);
    store_some(y + at, rest, v);
  } else {
    load_some(x + j, left, u);
    load_some(x + r + j, left, v);
#pragma unroll
    for (int k = 0; k < 7; ++k) turn(cs[min(j + some_at(k, left), r - 1)], u[k], v[k]);
    store_some(y + j, left, u);
    store_some(y + r + j, left, v);
  }
}

constexpr int kRotaryItems = 1280;   // units of a workgroup, where there are tokens for 512 such (2560: 5 to 15% slower; 640: within 4%)

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
    const double quarter = rint(4.0 * turns);            // an eighth of a turn at most is left to round to 32 bits
    float u, v;
    sincospif(2.f * (float)(turns - 0.25 * quarter), &u, &v);
    const int n = (int)quarter & 3;
    const float sn = n == 0 ? u : n == 1 ? v : n == 2 ? -u : -v, c = n == 0 ? v : n == 1 ? -u : n == 2 ? -v : u;
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
  int64_t per = std::max<int64_t>(1, kRotaryItems / items);
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
