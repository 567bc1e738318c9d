// Token rows in 16-byte pieces: loads, stores, dropout masks and sums over a row's threads.
//
// A piece is EP = 8 bf16 or 4 fp32 columns.  Rows may start at any alignment of their element
// (gfx950 takes 16-byte accesses at any address).
//
// Kernels that hold a whole row deal it to TPR threads: thread t has the pieces t, TPR + t, 2 TPR +
// t, ..., so a wave's loads are consecutive.  A piece that would reach past the row's end lies
// further left instead, on the row's last EP columns (piece_col), in part or wholly on columns of
// other threads.  There it holds what they hold and stores the same bits that they store; only
// sums over the row leave these columns out (owns).  So the loads and stores of a loop need no
// conditions.  (Every thread has its pieces of a row before any stores to it, also in place.)
// Rows of fewer than EP columns (kTiny) take element loads and stores, in instances of their own:
// beside the others these loads made every load of a loop wait for the one before.
//
// Kernels that come back to a row, or go through it piece by piece, keep to a piece's own columns:
//   kWhole  n is a multiple of EP;
//   kTail   the row's last piece is part of one: its thread loads the row's last EP elements,
//           shifts them down, and stores 8, 4 and 2 bytes;
//   kTiny   as above.
#pragma once
#include <type_traits>
#include "device.hpp"
#include "kernels.hpp"

namespace dprc {

// Threads of a row held whole: a power of two with 8 columns each (16 past 4096 columns).
inline int threads_per_row(int64_t n) {
  int tpr = 8;
  while (tpr < 512 && 8 * tpr < n) tpr *= 2;
  return tpr;
}

// Workgroups of a kernel that streams rows: one, two, three or four per CU, so that about 32 KB of loads are
// under way on each.  `ahead` bytes are those of a workgroup's rows in flight (the threads' columns within
// n only).  Fewer leave the memory waiting, more are slower again, as they reach over more
// pages at a time.  32768 x 2048 bf16 forwards with residual and dropout (16 KB a workgroup): 129, 97,
// 104, 106, 108 us with 1, 2, 3, 4, 8 per CU; without (8 KB): 92, 61, 51, 53, 56; backwards (24 KB): 135,
// 137, 144, 145, 139; 59 x 2402 x 130 fp32 backwards (25 KB): 82, 81, 82, 80; 8 x 4096 x 1111 bf16
// backwards (13 KB): 133, 97, 93, 96.
inline int64_t streaming_blocks(int64_t ahead) {
  const int64_t per_cu = (32768 + ahead / 2) / ahead;
  return 256 * (per_cu < 1 ? 1 : per_cu > 4 ? 4 : per_cu);
}

// Whether a call streams past the caches.  8 x 4096 x 2048 bf16: dropout (403 MB) 68 us with non-temporal
// accesses, 74 without; the fused norm (537 MB) 91 and 96, and a product with y that follows takes no
// longer.  4 x 4096 x 2048: the norm (268 MB) 45.5 and 44; 4 x 2048 x 2048 (134 MB): 26 and 23.6.
// Over 320 to 1000 MiB of both types, 512 to 16384 columns, times without against times with: dropout 7 to
// 11% longer; the norm with residual, dropout and sum 1% shorter to 9% longer; the norm alone 3% shorter
// (bf16 of 4096 columns, either type of 16384, from 540 MiB on) to 8% longer.
// Not for rows that share lines (97 fp32 columns backwards, 533 MB: 128 us and 109), and not for the backward
// pass, whose five streams took 133 to 157 us with them and 133 to 140 without, by where the tensors lay.
constexpr int64_t kStreamRowsBytes = (int64_t)300 << 20;
struct StreamRows {
  int64_t width, total = 0;      // bytes of a row's columns; of all tensors
  bool lines;
  explicit StreamRows(int64_t row_bytes) : width(row_bytes), lines(row_bytes % 128 == 0) {}
  void add(const void* p, int64_t rows, int64_t ld_bytes) {
    if (!p) return;
    total += rows * width;
    lines = lines && reinterpret_cast<uintptr_t>(p) % 128 == 0 && ld_bytes % 128 == 0;
  }
  bool yes() const { return lines && total >= kStreamRowsBytes; }
};

enum : int { kWide = 0, kTiny = 1, kWhole = 2, kTail = 3 };

template <class E>
constexpr int kPiece = 16 / (int)sizeof(E);

typedef uint32_t piece2_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t piece4_t __attribute__((ext_vector_type(4), aligned(4)));
template <class E>
using piece_t = std::conditional_t<sizeof(E) == 2, piece2_t, piece4_t>;
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// NT: non-temporal accesses, for calls whose tensors together are far larger than the 256 MB Infinity
// Cache and whose rows are whole 128-byte lines (StreamRows).
template <class E, bool NT = false>
__device__ __forceinline__ uint4 load_piece(const E* p) {
  const piece_t<E>* q = reinterpret_cast<const piece_t<E>*>(p);
  const piece_t<E> v = NT ? __builtin_nontemporal_load(q) : *q;
  return uint4{v[0], v[1], v[2], v[3]};
}

template <class E, bool NT = false>
__device__ __forceinline__ void store_piece(E* p, const uint4& v) {
  const piece_t<E> d = {v.x, v.y, v.z, v.w};
  piece_t<E>* q = reinterpret_cast<piece_t<E>*>(p);
  if (NT) __builtin_nontemporal_store(d, q);
  else *q = d;
}

// The piece of `row` at column c < n, for unpack_row at the same column.
template <class E, int M, bool NT = false>
__device__ __forceinline__ uint4 load_row(const E* row, int c, int n) {
  constexpr int EP = kPiece<E>;
  if constexpr (M != kTiny) return load_piece<E, NT>(row + min(c, n - EP));
  uint32_t h[EP];
#pragma unroll
  for (int j = 0; j < EP; ++j) {
    h[j] = 0;
    if (c + j < n) {
      if constexpr (sizeof(E) == 2) h[j] = row[c + j];
      else h[j] = __float_as_uint(row[c + j]);
    }
  }
  if constexpr (EP == 8) return uint4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
  else return uint4{h[0], h[1], h[2], h[3]};
}

template <class E>
__device__ __forceinline__ void unpack(const uint4& v, float* x) {
  if constexpr (sizeof(E) == 2) {
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(d[j] << 16);
      x[2 * j + 1] = __uint_as_float(d[j] & 0xFFFF0000u);
    }
  } else {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
}

// The columns c .. c + EP - 1 (c < n) of what load_row returned, zeros past the row's end.  (The
// shift is made here and not at the load, which would have to be waited for.)
template <class E, int M>
__device__ __forceinline__ void unpack_row(uint4 v, int c, int n, float* x) {
  constexpr int EP = kPiece<E>;
  if (M == kTail && c + EP > n) {
    const int over = EP - n % EP;                       // the same for every row: scalar branches
    if constexpr (EP == 8) {
      if (over & 4) v = uint4{v.z, v.w, 0u, 0u};
      if (over & 2) v = uint4{v.y, v.z, v.w, 0u};
      if (over & 1) v = shr_elems(v, 1);
    } else {
      if (over & 2) v = uint4{v.z, v.w, 0u, 0u};
      if (over & 1) v = uint4{v.y, v.z, v.w, 0u};
    }
  }
  unpack<E>(v, x);
}

// to E, nearest even
template <class E>
__device__ __forceinline__ uint4 pack(const float* x) {
  if constexpr (sizeof(E) == 2) {
    uint32_t d[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      d[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{x[2 * j], x[2 * j + 1]}, bf16x2_t));
    return uint4{d[0], d[1], d[2], d[3]};
  } else {
    return uint4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
}

// 8 or 4 bytes at any address that is aligned to an element
typedef uint32_t u32_any2 __attribute__((aligned(2)));
typedef uint32_t u32x2_any2 __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void store_part(void* p, uint32_t v) { *reinterpret_cast<u32_any2*>(p) = v; }
__device__ __forceinline__ void store_part(void* p, uint2 v) { *reinterpret_cast<u32x2_any2*>(p) = u32x2_any2{v.x, v.y}; }

// Piece at column c < n of an output row.
template <class E, int M, bool NT = false>
__device__ __forceinline__ void store_row(E* row, int c, int n, const float* x) {
  constexpr int EP = kPiece<E>;
  const uint4 v = pack<E>(x);
  if (M == kWhole || c + EP <= n) {
    store_piece<E, NT>(row + c, v);
    return;
  }
  // n - c < EP elements, as 8, 4 and 2 bytes
  const int m = n % EP;
  E* p = row + c;
  uint2 d{v.x, v.y};
  if (m * (int)sizeof(E) & 8) {
    store_part(p, d);
    d = uint2{v.z, v.w};
    p += 8 / sizeof(E);
  }
  if (m * (int)sizeof(E) & 4) {
    store_part(p, d.x);
    d.x = d.y;
    p += 4 / sizeof(E);
  }
  if constexpr (sizeof(E) == 2)
    if (m & 1) *p = (uint16_t)d.x;
}

// ---- pieces of rows held whole: kWide or kTiny ------------------------------------------------

// where the piece of column c lies, and whether its j-th column is its own
template <class E, int M>
__device__ __forceinline__ int piece_col(int c, int n) { return M == kTiny ? c : min(c, n - kPiece<E>); }
template <int M>
__device__ __forceinline__ bool owns(int c, int cc, int j, int n) { return M == kTiny ? c + j < n : cc + j >= c; }

// The piece of column c of the row `off` bytes after a base that the whole workgroup shares (the base
// stays in scalar registers, the offset in one vector register for a whole loop).
template <class E, int M, bool NT = false>
__device__ __forceinline__ uint4 load_at(const void* base, uint32_t off, int c, int n) {
  const char* p = static_cast<const char*>(base);
  if constexpr (M == kTiny) return load_row<E, kTiny>(reinterpret_cast<const E*>(p + off), c, n);
  else return load_piece<E, NT>(reinterpret_cast<const E*>(p + (off + (uint32_t)piece_col<E, M>(c, n) * (uint32_t)sizeof(E))));
}

template <class E, int M, bool NT = false>
__device__ __forceinline__ void store_at(void* base, uint32_t off, int c, int n, const float* x) {
  char* p = static_cast<char*>(base);
  if constexpr (M == kTiny) {
    if (c < n) store_row<E, kTiny>(reinterpret_cast<E*>(p + off), c, n, x);
  } else {
    store_piece<E, NT>(reinterpret_cast<E*>(p + (off + (uint32_t)piece_col<E, M>(c, n) * (uint32_t)sizeof(E))), pack<E>(x));
  }
}

// Entries c .. c + N - 1 of a weight or bias (fp32 or bf16), `none` without one and past its end.
template <int N>
__device__ __forceinline__ void load_vec(const void* v, int bf16, int c, int n, float none, float* x) {
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = none;
  if (!v || c >= n) return;
  if (bf16) {
    const uint16_t* p = (const uint16_t*)v + c;
    if (N == 8 && c + 8 <= n) {
      unpack<uint16_t>(load_piece(p), x);
      return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (c + j < n) x[j] = bf16_to_f32(p[j]);
  } else {
    const float* p = (const float*)v + c;
#pragma unroll
    for (int q = 0; q < N; q += 4) {
      if (c + q + 4 <= n) {
        unpack<float>(load_piece(p + q), x + q);
        continue;
      }
#pragma unroll
      for (int j = q; j < q + 4; ++j)
        if (c + j < n) x[j] = p[j];
    }
  }
}

// Philox4x32-10 with each round's two products taken whole (one v_mad_u64_u32 each, where high
// and low halves apart take two multiplies): 6.6e11 blocks/s against 5.2e11, in a loop of
// nothing else.
__device__ __forceinline__ u32x4 philox_mask(u32x4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    if (round) {
      k0 += 0x9E3779B9u;
      k1 += 0xBB67AE85u;
    }
    const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
    c = u32x4{(uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a};
  }
  return c;
}

// The mask words of the piece at column c of row r: 8 columns share a Philox block, two fp32 pieces half of
// it each.  A piece that was moved left (c no multiple of EP; all of a row's at the same place, n - EP)
// takes its words from two blocks.
template <class E>
__device__ __forceinline__ u32x4 drop_words(const DropArgs& d, uint32_t r, int c, int n) {
  constexpr int EP = kPiece<E>;
  u32x4 w = philox_mask(u32x4{(uint32_t)c >> 3, r, d.site, kStreamDropout}, d.key0, d.key1);
  if (c % EP == 0) {
    if (EP == 4 && (c & 4)) w = u32x4{w.z, w.w, 0u, 0u};
    return w;
  }
  u32x4 x = philox_mask(u32x4{((uint32_t)c >> 3) + 1u, r, d.site, kStreamDropout}, d.key0, d.key1);
  const int s = (n - EP) & 7;
  if (s & 4) w = u32x4{w.z, w.w, x.x, x.y}, x = u32x4{x.z, x.w, 0u, 0u};
  if (s & 2) w = u32x4{w.y, w.z, w.w, x.x}, x.x = x.y;
  if (s & 1) {
    auto join = [](uint32_t lo, uint32_t hi) { return lo >> 16 | hi << 16; };
    w = u32x4{join(w.x, w.y), join(w.y, w.z), join(w.z, w.w), join(w.w, x.x)};
  }
  return w;
}

// The piece through the site's dropout.  A dropped element is 0 whatever it was: it is replaced
// before the product with the scale.
template <class E>
__device__ __forceinline__ void drop_apply(const DropArgs& d, const u32x4& w, float* x) {
  const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < kPiece<E>; ++j)
    x[j] = (((j & 1) ? word[j >> 1] : word[j >> 1] << 16) > d.lim ? x[j] : 0.f) * d.scale;
}

template <class E>
__device__ __forceinline__ void drop_piece(const DropArgs& d, uint32_t r, int c, int n, float* x) {
  drop_apply<E>(d, drop_words<E>(d, r, c, n), x);
}

// ---- sums over groups of lanes ----------------------------------------------------------------
// Butterflies in vector registers: quad permutes for lanes 1 and 2 apart; the mirrors of 8 and of
// 16 lanes reach the other half of a group whose halves are uniform already; the lane swaps of
// gfx950 exchange rows of 16 and halves of 32.
template <int CTRL>
__device__ __forceinline__ float dpp_mov(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppMirror8 = 0x141, kDppMirror16 = 0x140, kDppRotate8 = 0x128;

// v of this lane plus v of the lane 16 (32) away
__device__ __forceinline__ float add_xor16(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ __forceinline__ float add_xor32(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// sum over aligned groups of L lanes (8, 16, 32 or 64), in every lane
template <int L>
__device__ __forceinline__ float lane_sum(float v) {
  v += dpp_mov<kDppXor1>(v);
  v += dpp_mov<kDppXor2>(v);
  v += dpp_mov<kDppMirror8>(v);
  if (L >= 16) v += dpp_mov<kDppMirror16>(v);
  if (L >= 32) v = add_xor16(v);
  if (L >= 64) v = add_xor32(v);
  return v;
}

// sum over the lanes of a wave that hold the same place in groups of L lanes, in every lane
template <int L>
__device__ __forceinline__ float group_sum(float v) {
  if (L <= 8) v += dpp_mov<kDppRotate8>(v);
  if (L <= 16) v = add_xor16(v);
  if (L <= 32) v = add_xor32(v);
  return v;
}

// Sums over a row's TPR threads, N values at once, in every thread.  Rows of several waves
// meet in LDS with one barrier a call: the calls of a kernel alternate between two buffers
// (`turn`), and a buffer is written again only after the barrier of the call between.
template <int TPR, int N, int BLK>
struct RowSum {
  static constexpr int kWaves = BLK / 64, kPer = TPR / 64;
  typedef float Buffer[2][N][TPR > 64 ? kWaves : 1];
  __device__ static __forceinline__ void run(float (&v)[N], Buffer& buf, int& turn) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lane_sum<(TPR < 64 ? TPR : 64)>(v[k]);
    if constexpr (TPR > 64) {
      const int wave = threadIdx.x >> 6, w0 = wave / kPer * kPer;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) buf[turn][k][wave] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < kPer; ++q) t += buf[turn][k][w0 + q];
        v[k] = t;
      }
      turn ^= 1;
    }
  }
};

}  // namespace dprc
