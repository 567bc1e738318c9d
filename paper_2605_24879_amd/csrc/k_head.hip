// Cross entropy of an output head S = h W^T over a vocabulary of V rows of W, without its logits.
//
//   forward:  l_tv = <h_t, W_v>;  lse_t = log sum_v exp l_tv;  loss_t = lse_t - l_t,y(t)
//   errors:   E_tv = g_t (exp(l_tv - lse_t) - [v = y(t)])      (0 where y(t) < 0)
//   backward: dh = E W  (and the weight's gradients h^T diag(c) E by the accumulation kernels)
//
// The logits exist only as matrix-core accumulators: the forward pass leaves each tile's running maximum
// and sum per token, the errors are formed from a tile made again and stored for a piece of the
// vocabulary at a time.  Bound by the matrix cores for more than a few hundred tokens, by reading W below.
//
// The tile of logits has the vocabulary as its rows and the tokens as its columns, so that an accumulator
// lane holds many logits of few tokens: the maximum and the sum over the vocabulary are sums over
// registers, with one exchange between the halves of the wave and one over the waves.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16_t;

constexpr float kLog2e = 1.44269504088896340736f;

// The tile of a workgroup: a contiguous share of the tiles for every XCD (workgroups are dealt to the 8 XCDs
// in turn), in groups of 4 row tiles walked column by column, so that 32 neighbours share 4 + 8 operand
// slabs in the XCD's L2.  (128000 x 8192 x 2048 in groups of 4, 8, 16, 32: 3225, 3258, 3288, 3810 us.)
__device__ __forceinline__ void tile_of(int64_t wg, int64_t tm_n, int64_t tn_n, int64_t& tm, int64_t& tn) {
  constexpr int GROUP = 4;
  const int64_t n = tm_n * tn_n, x = wg & 7;
  const int64_t lin = x * (n >> 3) + min(x, n & 7) + (wg >> 3);
  const int64_t group = lin / (GROUP * tn_n), r = lin - group * GROUP * tn_n, rows = min((int64_t)GROUP, tm_n - GROUP * group);
  tm = GROUP * group + r % rows;
  tn = r / rows;
}

// ---- products of tiles ----------------------------------------------------------------------------
// Accumulators as the 32 x 32 MFMAs hold them: WM x WN waves of XB x YB blocks; lane l of block (x, y) has
// rows 8 (q / 4) + 4 (l / 32) + q % 4, q < 16, of column l % 32.
//
// An operand is `rows` rows of `width` elements, ld apart.  KC: its rows are the tile's rows (columns), the
// contraction runs along them.  KR: the contraction runs over its rows, the tile's columns along them.

template <class E, int WM_, int WN_, int XB_, int YB_>
struct HeadTile {
  typedef E elem;
  static constexpr int WM = WM_, WN = WN_, XB = XB_, YB = YB_;
  static constexpr int MT = 32 * XB * WM, NT = 32 * YB * WN, threads = 64 * WM * WN;
};

constexpr int kHK = 64;               // contraction elements per bf16 slab

// The slabs in LDS, two of each operand.  KC: rows of 128 bytes, the eight 16-byte pieces of row r at piece ^
// (r & 7), so that a fragment read of 8 rows covers all banks.  KR: 64 rows of the tile's width, piece p of
// row r at p ^ swizzle_kr(r), so that the 4 (8) rows of a transposing read lie in different 32-byte (128-byte)
// parts of the banks.  Four arrays and not one: the compiler then knows that loads into one do not
// reach reads of another, and does not wait for them.
template <class TL, bool BKR>
struct HeadSlabs {
  static constexpr int A = TL::MT * kHK, B = TL::NT * kHK;
};
__device__ __forceinline__ int swizzle_kr(int r) { return ((r & 3) << 1) | (r & 8); }

// Eight elements at (row, col), zeros past the rows and the width, at any alignment.
__device__ __forceinline__ uint4 operand_piece(const HeadRows& X, int64_t row, int64_t col) {
  if (row >= X.rows || col >= X.width) return uint4{0, 0, 0, 0};
  const uint16_t* p = static_cast<const uint16_t*>(X.p);
  const int64_t at = row * X.ld + col, room = (X.rows - 1) * X.ld + X.width - 8;
  if (room < 0) return load8_elem(p + row * X.ld, col, X.width, true);
  const int64_t from = min(at, room);
  const u32x4_any v = *reinterpret_cast<const u32x4_any*>(p + from);
  return first_elems(shr_elems(uint4{v[0], v[1], v[2], v[3]}, (int)(at - from)), (int)min((int64_t)8, X.width - col));
}

// 64 lanes' 16-byte pieces at byte offsets `off` of the resource to 1024 bytes of LDS, in lane order; zeros
// where the offset is out of the resource's range.
typedef __attribute__((address_space(3))) void lds_void_t;
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, uint16_t* lds, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)lds, 16, (int)off, 0, 0, 0);
}

template <int V>
struct HInt {
  static constexpr int value = V;
};

// acc = sum over k in [k0, k1) of A[m0 + i][k] B[n0 + j][k] (BKR: B[k][n0 + j]), bf16 operands, k0 a multiple
// of kHK.  Slabs of kHK are double-buffered: while one is multiplied the next is loaded, straight into
// LDS where the operand's rows allow 16-byte pieces (VA, VB), else through registers.  A wave has the
// fragments of 16 contraction elements in registers ahead of their products, also across the slab's one
// barrier, and reads and products are issued in turn.  256 x 256 tiles of 128000 x 8192 x 2048: 1330
// TFLOP/s (the same loop as the compiler orders it 1146, all reads before all products 1270, four waves of
// 128 x 128 1217, tiles of 128 x 128 1093).
template <class TL, bool BKR, bool VA, bool VB>
__device__ __forceinline__ void head_product(const HeadRows& A, int64_t m0, const HeadRows& B, int64_t n0, int64_t k0,
                                             int64_t k1, f32x16_t (&acc)[TL::XB][TL::YB], uint16_t* la0, uint16_t* la1,
                                             uint16_t* lb0, uint16_t* lb1) {
  constexpr int XB = TL::XB, YB = TL::YB, TH = TL::threads;
  constexpr int PA = TL::MT * 8 / TH, PB = TL::NT * 8 / TH, BP = TL::NT / 8;     // pieces a thread; of a KR row
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int wave0 = 64 * (int)__builtin_amdgcn_readfirstlane(wv);
  const int wm = wv / TL::WN, wn = wv % TL::WN;
  auto kc_col = [](int s) { return 8 * ((s & 7) ^ ((s >> 3) & 7)); };
  auto kr_col = [](int s) { return 8 * ((s % BP) ^ (swizzle_kr(s / BP) & (BP - 1))); };
  // byte offsets of the thread's pieces in a slab
  uint32_t oa[PA], ob[PB];
#pragma unroll
  for (int r = 0; r < PA; ++r) {
    const int s = tid + TH * r;
    oa[r] = (uint32_t)(s >> 3) * (uint32_t)A.ld * 2u + 2u * kc_col(s);
  }
#pragma unroll
  for (int r = 0; r < PB; ++r) {
    const int s = tid + TH * r;
    if constexpr (BKR) ob[r] = n0 + kr_col(s) < B.width ? (uint32_t)(s / BP) * (uint32_t)B.ld * 2u + 2u * kr_col(s) : kOobOffset;
    else ob[r] = (uint32_t)(s >> 3) * (uint32_t)B.ld * 2u + 2u * kc_col(s);
  }
  // a resource over `tile` rows from row0 on, `skip` elements into them
  auto rsrc = [](const HeadRows& X, int64_t row0, int tile, int64_t skip) __attribute__((always_inline)) {
    const int64_t left = X.rows - row0;
    const uint32_t rows = (uint32_t)(left < 0 || skip >= X.width ? 0 : left < tile ? left : tile);
    return buffer_rsrc(static_cast<const uint16_t*>(X.p) + (rows ? row0 * X.ld + skip : 0),
                       rows ? rows * (uint32_t)X.ld * 2u - (uint32_t)skip * 2u : 0u);
  };
  uint4 ga[VA ? 1 : PA], gb[VB ? 1 : PB];
  auto gload = [&](int64_t k, auto u) __attribute__((always_inline)) {
    uint16_t* la = decltype(u)::value ? la1 : la0;
    uint16_t* lb = decltype(u)::value ? lb1 : lb0;
    const bool tail = k + kHK > A.width;               // columns past the rows' end
    if constexpr (VA) {
      const __amdgpu_buffer_rsrc_t ra = rsrc(A, m0, TL::MT, k);
      if (tail) {
#pragma unroll
        for (int r = 0; r < PA; ++r)
          load_to_lds(ra, la + 8 * (wave0 + TH * r), k + kc_col(tid + TH * r) < A.width ? oa[r] : kOobOffset);
      } else {
#pragma unroll
        for (int r = 0; r < PA; ++r) load_to_lds(ra, la + 8 * (wave0 + TH * r), oa[r]);
      }
    } else {
#pragma unroll
      for (int r = 0; r < PA; ++r) ga[r] = operand_piece(A, m0 + ((tid + TH * r) >> 3), k + kc_col(tid + TH * r));
    }
    if constexpr (VB && BKR) {
      const __amdgpu_buffer_rsrc_t rb = rsrc(B, k, kHK, n0);
#pragma unroll
      for (int r = 0; r < PB; ++r) load_to_lds(rb, lb + 8 * (wave0 + TH * r), ob[r]);
    } else if constexpr (VB) {
      const __amdgpu_buffer_rsrc_t rb = rsrc(B, n0, TL::NT, k);
      if (tail) {
#pragma unroll
        for (int r = 0; r < PB; ++r)
          load_to_lds(rb, lb + 8 * (wave0 + TH * r), k + kc_col(tid + TH * r) < B.width ? ob[r] : kOobOffset);
      } else {
#pragma unroll
        for (int r = 0; r < PB; ++r) load_to_lds(rb, lb + 8 * (wave0 + TH * r), ob[r]);
      }
    } else {
#pragma unroll
      for (int r = 0; r < PB; ++r) {
        const int s = tid + TH * r;
        gb[r] = BKR ? operand_piece(B, k + s / BP, n0 + kr_col(s)) : operand_piece(B, n0 + (s >> 3), k + kc_col(s));
      }
    }
  };
  // what went through registers to LDS, then every wave's slab is there and the other's reads are done
  auto arrive = [&](auto u) __attribute__((always_inline)) {
    uint16_t* la = decltype(u)::value ? la1 : la0;
    uint16_t* lb = decltype(u)::value ? lb1 : lb0;
    if constexpr (!VA) {
#pragma unroll
      for (int r = 0; r < PA; ++r) *reinterpret_cast<uint4*>(&la[8 * (tid + TH * r)]) = ga[r];
    }
    if constexpr (!VB) {
#pragma unroll
      for (int r = 0; r < PB; ++r) *reinterpret_cast<uint4*>(&lb[8 * (tid + TH * r)]) = gb[r];
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  };
#pragma unroll
  for (int x = 0; x < XB; ++x)
#pragma unroll
    for (int y = 0; y < YB; ++y)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[x][y][q] = 0.f;
  const int l32 = lane & 31, half = lane >> 5;
  const int g = lane >> 4, r4 = (lane & 15) >> 2, c4 = lane & 3;
  uint4 f0a[XB], f0b[YB], f1a[XB], f1b[YB];
  // the fragments of contraction elements 16 ks .. 16 ks + 15 of a slab
  auto frag = [&](uint4 (&av)[XB], uint4 (&bv)[YB], auto u, int ks) __attribute__((always_inline)) {
    const uint16_t* la = decltype(u)::value ? la1 : la0;
    const uint16_t* lb = decltype(u)::value ? lb1 : lb0;
#pragma unroll
    for (int y = 0; y < YB; ++y) {
      if constexpr (BKR) {
        // lane group g reads rows 8 (g / 2) + r4 (+ 4) of columns 16 (g % 2) + 4 c4 .. of the block
        const int row = 16 * ks + 8 * (g >> 1) + r4, col = 32 * (wn * YB + y) + 16 * (g & 1) + 4 * c4;
        const uint16_t* p = &lb[row * TL::NT + 8 * ((col >> 3) ^ (swizzle_kr(row) & (BP - 1))) + (col & 4)];
        bv[y] = make_u4(lds_read_tr16(p), lds_read_tr16(p + 4 * TL::NT));
      } else {
        const int row = 32 * (wn * YB + y) + l32;
        bv[y] = *reinterpret_cast<const uint4*>(&lb[row * kHK + 8 * ((2 * ks + half) ^ (row & 7))]);
      }
    }
#pragma unroll
    for (int x = 0; x < XB; ++x) {
      const int row = 32 * (wm * XB + x) + l32;
      av[x] = *reinterpret_cast<const uint4*>(&la[row * kHK + 8 * ((2 * ks + half) ^ (row & 7))]);
    }
  };
  auto phase = [&](uint4 (&na)[XB], uint4 (&nb)[YB], auto u, int ks, const uint4 (&av)[XB], const uint4 (&bv)[YB])
      __attribute__((always_inline)) {
    frag(na, nb, u, ks);
#pragma unroll
    for (int x = 0; x < XB; ++x)
#pragma unroll
      for (int y = 0; y < YB; ++y)
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, av[x]),
                                                            __builtin_bit_cast(bf16x8_t, bv[y]), acc[x][y], 0, 0, 0);
    constexpr int reads = XB + (BKR ? 2 : 1) * YB, products = XB * YB;
#pragma unroll
    for (int i = 0; i < reads; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);               // a read of LDS
      if (i < products) __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);   // a product
    }
    if constexpr (products > reads) __builtin_amdgcn_sched_group_barrier(0x8, products - reads, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  // the slab at k in buffers u, its first fragments in registers
  auto step = [&](int64_t k, auto u) __attribute__((always_inline)) {
    constexpr HInt<decltype(u)::value ^ 1> other{};
    gload(k + kHK < k1 ? k + kHK : (int64_t)1 << 40, other);           // past the end: nothing
    __builtin_amdgcn_sched_barrier(0);
    phase(f1a, f1b, u, 1, f0a, f0b);
    phase(f0a, f0b, u, 2, f1a, f1b);
    phase(f1a, f1b, u, 3, f0a, f0b);
    arrive(other);
    phase(f0a, f0b, other, 0, f1a, f1b);
  };
  gload(k0, HInt<0>{});
  arrive(HInt<0>{});
  frag(f0a, f0b, HInt<0>{}, 0);
  for (int64_t k = k0; k < k1; k += 2 * kHK) {       // (an odd number of slabs: the last one is zeros)
    step(k, HInt<0>{});
    step(k + kHK, HInt<1>{});
  }
  __syncthreads();                                     // all reads are done
}

// fp32 operands, on the fp32 matrix cores (products and sums in fp32): slabs of 16 in LDS as [k][row].
constexpr int kHKf = 16;

__device__ __forceinline__ float4 operand_piece_f32(const HeadRows& X, int64_t row, int64_t col) {
  float4 v{0.f, 0.f, 0.f, 0.f};
  if (row >= X.rows || col >= X.width) return v;
  const float* p = static_cast<const float*>(X.p) + row * X.ld + col;
  if (col + 4 <= X.width) {
    const uint4 d = load_piece<float>(p);
    return __builtin_bit_cast(float4, d);
  }
  v.x = p[0];
  if (col + 1 < X.width) v.y = p[1];
  if (col + 2 < X.width) v.z = p[2];
  return v;
}

template <class TL>
constexpr int head_lds_bytes_f32() {
  return 2 * 4 * kHKf * (TL::MT + 4 + TL::NT + 4);
}

template <class TL, bool BKR>
__device__ __forceinline__ void head_product_f32(const HeadRows& A, int64_t m0, const HeadRows& B, int64_t n0, int64_t k0,
                                                 int64_t k1, f32x16_t (&acc)[TL::XB][TL::YB], float* lds) {
  constexpr int XB = TL::XB, YB = TL::YB, LA = TL::MT + 4, LB = TL::NT + 4;
  constexpr int PA = TL::MT * kHKf / 4 / TL::threads, PB = TL::NT * kHKf / 4 / TL::threads;
  float* la[2] = {lds, lds + kHKf * LA};
  float* lb[2] = {lds + 2 * kHKf * LA, lds + 2 * kHKf * LA + kHKf * LB};
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int wm = wv / TL::WN, wn = wv % TL::WN, l32 = lane & 31, half = lane >> 5;
  float4 ga[PA], gb[PB];
  auto gload = [&](int64_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < PA; ++r) {
      const int s = tid + TL::threads * r;
      ga[r] = operand_piece_f32(A, m0 + (s >> 2), k + 4 * (s & 3));
    }
#pragma unroll
    for (int r = 0; r < PB; ++r) {
      const int s = tid + TL::threads * r;
      gb[r] = BKR ? operand_piece_f32(B, k + s / (TL::NT / 4), n0 + 4 * (s % (TL::NT / 4)))
                  : operand_piece_f32(B, n0 + (s >> 2), k + 4 * (s & 3));
    }
  };
  auto swrite = [&](int buf) __attribute__((always_inline)) {
    auto across = [&](float* l, int ld, int s, const float4& v) __attribute__((always_inline)) {
      float* o = l + 4 * (s & 3) * ld + (s >> 2);
      o[0] = v.x; o[ld] = v.y; o[2 * ld] = v.z; o[3 * ld] = v.w;
    };
#pragma unroll
    for (int r = 0; r < PA; ++r) across(la[buf], LA, tid + TL::threads * r, ga[r]);
#pragma unroll
    for (int r = 0; r < PB; ++r) {
      const int s = tid + TL::threads * r;
      if constexpr (BKR) *reinterpret_cast<float4*>(&lb[buf][s / (TL::NT / 4) * LB + 4 * (s % (TL::NT / 4))]) = gb[r];
      else across(lb[buf], LB, s, gb[r]);
    }
  };
#pragma unroll
  for (int x = 0; x < XB; ++x)
#pragma unroll
    for (int y = 0; y < YB; ++y)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[x][y][q] = 0.f;
  gload(k0);
  swrite(0);
  __syncthreads();
  int buf = 0;
  for (int64_t k = k0; k < k1; k += kHKf) {
    const bool more = k + kHKf < k1;
    if (more) gload(k + kHKf);
#pragma unroll
    for (int ks = 0; ks < kHKf / 2; ++ks) {
      float av[XB], bv[YB];
#pragma unroll
      for (int x = 0; x < XB; ++x) av[x] = la[buf][(2 * ks + half) * LA + 32 * (wm * XB + x) + l32];
#pragma unroll
      for (int y = 0; y < YB; ++y) bv[y] = lb[buf][(2 * ks + half) * LB + 32 * (wn * YB + y) + l32];
#pragma unroll
      for (int x = 0; x < XB; ++x)
#pragma unroll
        for (int y = 0; y < YB; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x2f32(av[x], bv[y], acc[x][y], 0, 0, 0);
    }
    if (more) swrite(buf ^ 1);
    __syncthreads();
    buf ^= 1;
  }
}

// ---- what becomes of a tile -----------------------------------------------------------------------

__device__ __forceinline__ int acc_row(int lane, int q) { return 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3); }

// (m, s): sum of exp(l) = s exp(m).  A maximum of -infinity (every logit is) counts as -1e38, so that no
// difference of infinities arises; a logit of +infinity or NaN makes s NaN.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  return float2{m, a.y * exp2f((a.x - m) * kLog2e) + b.y * exp2f((b.x - m) * kLog2e)};
}

// The tile's maximum and sum of every token: part[tile row][N].
template <class TL>
__device__ __forceinline__ void head_sums(const HeadArgs& a, int64_t tm, int64_t t0, f32x16_t (&acc)[TL::XB][TL::YB],
                                          float2* lds) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, wm = wv / TL::WN, wn = wv % TL::WN;
  const int64_t v0 = tm * TL::MT + 32 * TL::XB * wm;
  if (v0 + 32 * TL::XB > a.nv) {
#pragma unroll
    for (int x = 0; x < TL::XB; ++x)
#pragma unroll
      for (int q = 0; q < 16; ++q)
        if (v0 + 32 * x + acc_row(lane, q) >= a.nv) {
#pragma unroll
          for (int y = 0; y < TL::YB; ++y) acc[x][y][q] = -INFINITY;
        }
  }
#pragma unroll
  for (int y = 0; y < TL::YB; ++y) {
    float m = -1e38f;
#pragma unroll
    for (int x = 0; x < TL::XB; ++x)
#pragma unroll
      for (int q = 0; q < 16; ++q) m = fmaxf(m, acc[x][y][q]);
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float m2 = m * kLog2e;
    float s = 0.f;
#pragma unroll
    for (int x = 0; x < TL::XB; ++x)
#pragma unroll
      for (int q = 0; q < 16; ++q) s += __builtin_amdgcn_exp2f(fmaf(acc[x][y][q], kLog2e, -m2));
    s += __shfl_xor(s, 32, 64);
    if (lane < 32) lds[wm * TL::NT + 32 * (wn * TL::YB + y) + lane] = float2{m, s};
  }
  __syncthreads();
  for (int j = threadIdx.x; j < TL::NT; j += TL::threads) {
    float2 v = lds[j];
#pragma unroll
    for (int w = 1; w < TL::WM; ++w) v = join(v, lds[w * TL::NT + j]);
    if (t0 + j < a.N) a.part[tm * a.N + t0 + j] = v;
  }
}

// LDS for a tile of errors, token rows of MT: the 16-byte piece p of token t at p ^ (t & 31), so that the 32
// tokens of a block, one a lane, go to different banks.  Four arrays of 64 tokens, or one.
template <class TL>
struct HeadStage {
  typedef typename TL::elem E;
  static constexpr int EP = kPiece<E>, PPR = TL::MT / EP;
  static_assert(PPR == 32);
  E *p0, *p1, *p2, *p3;
  __device__ __forceinline__ E* piece(int token, int p) const {
    const int part = sizeof(E) == 2 ? token >> 6 : 0;
    E* base = part == 0 ? p0 : part == 1 ? p1 : part == 2 ? p2 : p3;
    return base + ((sizeof(E) == 2 ? token & 63 : token) * PPR + (p ^ (token & 31))) * EP;
  }
};

// The tile's errors, through LDS into token rows.
template <class TL>
__device__ __forceinline__ void head_errors(const HeadArgs& a, int64_t tm, int64_t t0, f32x16_t (&acc)[TL::XB][TL::YB],
                                            const HeadStage<TL>& stage) {
  typedef typename TL::elem E;
  constexpr int EP = kPiece<E>, PPR = TL::MT / EP;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, wm = wv / TL::WN, wn = wv % TL::WN;
  const int64_t vt = tm * TL::MT;                       // the tile's first column of this piece
  const int v0 = 32 * TL::XB * wm;                      // the wave's first in the tile
  const int end = (int)min((int64_t)TL::MT, a.nv - vt) - v0;       // its columns before the vocabulary's end
#pragma unroll
  for (int y = 0; y < TL::YB; ++y) {
    const int col = 32 * (wn * TL::YB + y) + (lane & 31);
    const int64_t t = t0 + col;
    const int64_t target = t < a.N ? a.target[t] : -1;
    const bool kept = target >= 0;
    const float lse = kept ? a.lse[t] : 0.f, g = kept ? a.g[t] : 0.f;
    const int64_t at64 = target - a.v0 - vt - v0;       // the target's place among the wave's columns
    const int at = kept && at64 >= 0 && at64 < 32 * TL::XB ? (int)at64 : -1;
    const float lse2 = lse * kLog2e;
    const bool rare = __any(at >= 0) || end < 32 * TL::XB;
#pragma unroll
    for (int x = 0; x < TL::XB; ++x)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        float e[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float l = acc[x][y][4 * q4 + q];
          if constexpr (sizeof(E) == 2) e[q] = g * __builtin_amdgcn_exp2f(fmaf(l, kLog2e, -lse2));
          else e[q] = g * expf(l - lse);
        }
        const int v = 32 * x + acc_row(lane, 4 * q4);
        if (rare) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (at == v + q) e[q] = g * expm1f(acc[x][y][4 * q4 + q] - lse);   // exp(x) - 1 without cancellation
            if (v + q >= end) e[q] = 0.f;
          }
        }
        E* o = stage.piece(col, (v0 + v) / EP) + (v & (EP - 1));
        if constexpr (sizeof(E) == 2) {
          const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{e[0], e[1]}, bf16x2_t));
          const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{e[2], e[3]}, bf16x2_t));
          *reinterpret_cast<uint2*>(o) = uint2{kept ? lo : 0u, kept ? hi : 0u};
        } else {
          *reinterpret_cast<float4*>(o) = kept ? float4{e[0], e[1], e[2], e[3]} : float4{0.f, 0.f, 0.f, 0.f};
        }
      }
  }
  __syncthreads();
  for (int s = threadIdx.x; s < TL::NT * PPR; s += TL::threads) {
    const int row = s / PPR, p = s % PPR;
    const int64_t t = t0 + row, v = vt + EP * p;
    if (t >= a.N || v >= a.width) continue;
    const E* from = stage.piece(row, p);
    E* to = static_cast<E*>(a.E) + t * a.lde + v;
    if (v + EP <= a.width) store_piece<E>(to, *reinterpret_cast<const uint4*>(from));
    else
      for (int j = 0; v + j < a.width; ++j) to[j] = from[j];
  }
}

// The tile written to, or added to, its place of a plane [N][d].
template <class TL>
__device__ __forceinline__ void head_store(const HeadBackArgs& a, float* plane, int64_t m0, int64_t n0,
                                           f32x16_t (&acc)[TL::XB][TL::YB]) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, wm = wv / TL::WN, wn = wv % TL::WN;
#pragma unroll
  for (int x = 0; x < TL::XB; ++x)
#pragma unroll
    for (int y = 0; y < TL::YB; ++y) {
      const int64_t col = n0 + 32 * (wn * TL::YB + y) + (lane & 31);
      if (col >= a.d) continue;
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int64_t row = m0 + 32 * (wm * TL::XB + x) + acc_row(lane, q);
        if (row >= a.N) continue;
        float* o = plane + row * a.d + col;
        *o = a.add ? *o + acc[x][y][q] : acc[x][y][q];
      }
    }
}

// ---- kernels --------------------------------------------------------------------------------------

// The logits' tiles.  bf16: rows of W in 16-byte pieces (VW) or at any alignment; h always in pieces.
template <class TL, bool ERRORS, bool VW>
__global__ __launch_bounds__(TL::threads) void head_logits_kernel(HeadArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t la0[HeadSlabs<TL, false>::A];
  __shared__ __attribute__((aligned(16))) uint16_t la1[HeadSlabs<TL, false>::A];
  __shared__ __attribute__((aligned(16))) uint16_t lb0[HeadSlabs<TL, false>::B];
  __shared__ __attribute__((aligned(16))) uint16_t lb1[HeadSlabs<TL, false>::B];
  static_assert(TL::NT == 64 || (TL::MT == 256 && TL::NT == 256));
  const int64_t tm_n = (a.nv + TL::MT - 1) / TL::MT, tn_n = (a.N + TL::NT - 1) / TL::NT;
  const int64_t wg = flat_block();
  if (wg >= tm_n * tn_n) return;
  int64_t tm, tn;
  tile_of(wg, tm_n, tn_n, tm, tn);
  f32x16_t acc[TL::XB][TL::YB];
  head_product<TL, false, VW, true>(a.W, tm * TL::MT, a.h, tn * TL::NT, 0, a.W.width, acc, la0, la1, lb0, lb1);
  if constexpr (ERRORS) head_errors<TL>(a, tm, tn * TL::NT, acc, HeadStage<TL>{la0, la1, lb0, lb1});
  else head_sums<TL>(a, tm, tn * TL::NT, acc, reinterpret_cast<float2*>(la0));
}

template <class TL, bool ERRORS>
__global__ __launch_bounds__(TL::threads) void head_logits_f32_kernel(HeadArgs a) {
  constexpr int MAIN = head_lds_bytes_f32<TL>(), TAIL = ERRORS ? 4 * TL::MT * TL::NT : 8 * TL::WM * TL::NT;
  __shared__ __attribute__((aligned(16))) char lds[MAIN > TAIL ? MAIN : TAIL];
  const int64_t tm_n = (a.nv + TL::MT - 1) / TL::MT, tn_n = (a.N + TL::NT - 1) / TL::NT;
  const int64_t wg = flat_block();
  if (wg >= tm_n * tn_n) return;
  int64_t tm, tn;
  tile_of(wg, tm_n, tn_n, tm, tn);
  f32x16_t acc[TL::XB][TL::YB];
  float* l = reinterpret_cast<float*>(lds);
  head_product_f32<TL, false>(a.W, tm * TL::MT, a.h, tn * TL::NT, 0, a.W.width, acc, l);
  if constexpr (ERRORS) head_errors<TL>(a, tm, tn * TL::NT, acc, HeadStage<TL>{l, l, l, l});
  else head_sums<TL>(a, tm, tn * TL::NT, acc, reinterpret_cast<float2*>(lds));
}

// dh's tiles: rows are tokens, columns features; blockIdx.z is the split of the piece's vocabulary.
template <class TL, bool VW>
__global__ __launch_bounds__(TL::threads) void head_back_kernel(HeadBackArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t la0[HeadSlabs<TL, true>::A];
  __shared__ __attribute__((aligned(16))) uint16_t la1[HeadSlabs<TL, true>::A];
  __shared__ __attribute__((aligned(16))) uint16_t lb0[HeadSlabs<TL, true>::B];
  __shared__ __attribute__((aligned(16))) uint16_t lb1[HeadSlabs<TL, true>::B];
  const int64_t tm_n = (a.N + TL::MT - 1) / TL::MT, tn_n = (a.d + TL::NT - 1) / TL::NT;
  const int64_t wg = flat_block();
  if (wg >= tm_n * tn_n) return;
  int64_t tm, tn;
  tile_of(wg, tm_n, tn_n, tm, tn);
  const int64_t k0 = blockIdx.z * a.per_split, k1 = min(a.E.width, k0 + a.per_split);
  f32x16_t acc[TL::XB][TL::YB];
  head_product<TL, true, true, VW>(a.E, tm * TL::MT, a.W, tn * TL::NT, k0, k1, acc, la0, la1, lb0, lb1);
  head_store<TL>(a, a.planes + blockIdx.z * a.N * a.d, tm * TL::MT, tn * TL::NT, acc);
}

template <class TL>
__global__ __launch_bounds__(TL::threads) void head_back_f32_kernel(HeadBackArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[head_lds_bytes_f32<TL>()];
  const int64_t tm_n = (a.N + TL::MT - 1) / TL::MT, tn_n = (a.d + TL::NT - 1) / TL::NT;
  const int64_t wg = flat_block();
  if (wg >= tm_n * tn_n) return;
  int64_t tm, tn;
  tile_of(wg, tm_n, tn_n, tm, tn);
  const int64_t k0 = blockIdx.z * a.per_split, k1 = min(a.E.width, k0 + a.per_split);
  f32x16_t acc[TL::XB][TL::YB];
  head_product_f32<TL, true>(a.E, tm * TL::MT, a.W, tn * TL::NT, k0, k1, acc, reinterpret_cast<float*>(lds));
  head_store<TL>(a, a.planes + blockIdx.z * a.N * a.d, tm * TL::MT, tn * TL::NT, acc);
}

// Joins the tiles' maxima and sums in a fixed order and takes the target's logit, summed in fp32.  16 tokens
// per workgroup: 64 groups of 16 lanes go through the tiles, then a wave per token multiplies h_t and
// W_y(t).  A target past the vocabulary makes both outputs NaN.
template <class E>
__global__ __launch_bounds__(1024) void head_join_kernel(HeadArgs a, int64_t tiles, float* loss, float* lse) {
  __shared__ float2 buf[64][16];
  __shared__ float out[16];
  const int64_t t0 = (int64_t)flat_block() * 16;
  if (t0 >= a.N) return;
  const int j = threadIdx.x & 15, grp = threadIdx.x >> 4, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  float2 v{-1e38f, 0.f};
  if (t0 + j < a.N)
    for (int64_t s = grp; s < tiles; s += 64) v = join(v, a.part[s * a.N + t0 + j]);
  buf[grp][j] = v;
  __syncthreads();
  if (threadIdx.x < 16) {
    for (int k = 1; k < 64; ++k) v = join(v, buf[k][j]);
    out[j] = v.x + logf(v.y);
  }
  __syncthreads();
  const int64_t t = t0 + wv;
  if (t >= a.N) return;
  const int64_t y = a.target[t];
  float dot = 0.f;
  if (y >= 0 && y < a.W.rows) {
    const E* h = static_cast<const E*>(a.h.p) + t * a.h.ld;
    const E* w = static_cast<const E*>(a.W.p) + y * a.W.ld;
    for (int64_t c = lane; c < a.W.width; c += 64) {
      if constexpr (sizeof(E) == 2) dot = fmaf(bf16_to_f32(h[c]), bf16_to_f32(w[c]), dot);
      else dot = fmaf(h[c], w[c], dot);
    }
  }
  dot = wave_sum(dot);
  if (lane > 0) return;
  const float z = y >= a.W.rows ? NAN : out[wv], l = z - dot;
  lse[t] = z;
  loss[t] = y < 0 ? 0.f : l < 0.f ? 0.f : l;           // a probability is at most 1
}

// h's rows laid out in 16-byte pieces, zeros behind the width, and with `target` in rows without a loss
// (whose values, NaN among them, have no part in any gradient).
template <class E>
__global__ __launch_bounds__(256) void head_rows_kernel(HeadRows X, const int64_t* target, E* out, int64_t ldo) {
  constexpr int EP = kPiece<E>;
  const int64_t ppr = ldo / EP, s = (int64_t)flat_block() * 256 + threadIdx.x;
  const int64_t row = s / ppr, c = EP * (s - row * ppr);
  if (row >= X.rows) return;
  const E* from = static_cast<const E*>(X.p) + row * X.ld;
  uint4 v{0, 0, 0, 0};
  if (!target || target[row] >= 0) {
    if (c + EP <= X.width) {
      v = load_piece<E>(from + c);
    } else {
      E x[EP];
#pragma unroll
      for (int j = 0; j < EP; ++j) x[j] = c + j < X.width ? from[c + j] : (E)0;
      v = *reinterpret_cast<const uint4*>(x);
    }
  }
  store_piece<E>(out + row * ldo + c, v);
}

// out = the sum of S planes [rows][cols], in their order, rounded once.
template <class E>
__global__ __launch_bounds__(256) void head_round_kernel(const float* planes, int S, int64_t rows, int64_t cols, E* out,
                                                         int64_t ldo) {
  const int64_t ppr = (cols + 3) / 4, s = (int64_t)flat_block() * 256 + threadIdx.x;
  const int64_t row = s / ppr, c = 4 * (s - row * ppr);
  if (row >= rows) return;
  const int m = (int)min((int64_t)4, cols - c);
  float x[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < S; ++k) {
    const float* p = planes + (k * rows + row) * cols + c;
    if (m == 4) {
      float u[4];
      unpack<float>(load_piece<float>(p), u);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] += u[j];
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (j < m) x[j] += p[j];
    }
  }
  E* o = out + row * ldo + c;
  if constexpr (sizeof(E) == 2) {
    const uint2 d{__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{x[0], x[1]}, bf16x2_t)),
                  __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{x[2], x[3]}, bf16x2_t))};
    if (m == 4) store_part(o, d);
    else {
      o[0] = (uint16_t)d.x;
      if (m > 1) o[1] = (uint16_t)(d.x >> 16);
      if (m > 2) o[2] = (uint16_t)d.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < m) o[j] = x[j];
  }
}

__global__ void head_one_kernel(float* one) { *one = 1.f; }

// ---- launches -------------------------------------------------------------------------------------

typedef HeadTile<uint16_t, 2, 4, 4, 2> TileWide;       // 256 x 256, eight waves of 128 x 64
typedef HeadTile<uint16_t, 8, 1, 1, 2> TileFew;        // 256 x 64, eight waves of 32 x 64: up to 64 tokens
typedef HeadTile<float, 2, 2, 2, 2> TileF32;           // 128 x 128, four waves of 64 x 64

int head_tile_rows(int bf16) { return bf16 ? TileWide::MT : TileF32::MT; }

template <class TL, bool ERRORS>
static void launch_logits(const HeadArgs& a, hipStream_t st) {
  const int64_t blocks = ceil_div(a.nv, TL::MT) * ceil_div(a.N, TL::NT);
  if (a.vec_w) DPRC_LAUNCH((head_logits_kernel<TL, ERRORS, true>), flat_grid(blocks), dim3(TL::threads), 0, st, a);
  else DPRC_LAUNCH((head_logits_kernel<TL, ERRORS, false>), flat_grid(blocks), dim3(TL::threads), 0, st, a);
}

template <bool ERRORS>
static hipError_t launch_head_logits(const HeadArgs& a, hipStream_t st) {
  if (!a.bf16) {
    const int64_t blocks = ceil_div(a.nv, TileF32::MT) * ceil_div(a.N, TileF32::NT);
    DPRC_LAUNCH((head_logits_f32_kernel<TileF32, ERRORS>), flat_grid(blocks), dim3(TileF32::threads), 0, st, a);
  } else if (a.N <= TileFew::NT) {
    launch_logits<TileFew, ERRORS>(a, st);
  } else {
    launch_logits<TileWide, ERRORS>(a, st);
  }
  return hipGetLastError();
}

hipError_t launch_head_sums(const HeadArgs& a, hipStream_t st) { return launch_head_logits<false>(a, st); }
hipError_t launch_head_errors(const HeadArgs& a, hipStream_t st) { return launch_head_logits<true>(a, st); }

hipError_t launch_head_join(const HeadArgs& a, float* loss, float* lse, hipStream_t st) {
  const int64_t tiles = ceil_div(a.nv, head_tile_rows(a.bf16)), blocks = ceil_div(a.N, 16);
  if (a.bf16) DPRC_LAUNCH(head_join_kernel<uint16_t>, flat_grid(blocks), dim3(1024), 0, st, a, tiles, loss, lse);
  else DPRC_LAUNCH(head_join_kernel<float>, flat_grid(blocks), dim3(1024), 0, st, a, tiles, loss, lse);
  return hipGetLastError();
}

HeadBackPlan head_back_plan(int64_t N, int64_t d, int64_t nv, int bf16, int32_t most) {
  const int64_t tile = bf16 ? 256 : 128, slab = bf16 ? kHK : kHKf;
  const int64_t tiles = ceil_div(N, tile) * ceil_div(d, tile), slabs = ceil_div(nv, slab);
  int64_t want = tiles >= 256 ? 1 : std::min<int64_t>(ceil_div(256, tiles), std::max<int64_t>(1, slabs / 16));
  if (most > 0) want = std::min<int64_t>(want, most);
  HeadBackPlan p;
  p.per_split = ceil_div(slabs, want) * slab;
  p.S = (int32_t)ceil_div(slabs * slab, p.per_split);
  return p;
}

hipError_t launch_head_back(const HeadBackArgs& a, hipStream_t st) {
  auto go = [&](auto kernel, int tile, int threads) {
    dim3 grid = flat_grid(ceil_div(a.N, tile) * ceil_div(a.d, tile));
    grid.z = (unsigned)a.S;
    DPRC_LAUNCH(kernel, grid, dim3(threads), 0, st, a);
  };
  if (!a.bf16) go(head_back_f32_kernel<TileF32>, TileF32::MT, TileF32::threads);
  else if (a.vec_w) go(head_back_kernel<TileWide, true>, TileWide::MT, TileWide::threads);
  else go(head_back_kernel<TileWide, false>, TileWide::MT, TileWide::threads);
  return hipGetLastError();
}

hipError_t launch_head_rows(const HeadRows& X, int bf16, const int64_t* target, void* out, int64_t ldo, hipStream_t st) {
  const int64_t blocks = ceil_div(X.rows * (ldo / (bf16 ? 8 : 4)), 256);
  if (bf16) DPRC_LAUNCH(head_rows_kernel<uint16_t>, flat_grid(blocks), dim3(256), 0, st, X, target, (uint16_t*)out, ldo);
  else DPRC_LAUNCH(head_rows_kernel<float>, flat_grid(blocks), dim3(256), 0, st, X, target, (float*)out, ldo);
  return hipGetLastError();
}

hipError_t launch_head_round(const float* planes, int S, int64_t rows, int64_t cols, int bf16, void* out, int64_t ldo,
                             hipStream_t st) {
  const int64_t blocks = ceil_div(rows * ceil_div(cols, 4), 256);
  if (bf16) DPRC_LAUNCH(head_round_kernel<uint16_t>, flat_grid(blocks), dim3(256), 0, st, planes, S, rows, cols, (uint16_t*)out, ldo);
  else DPRC_LAUNCH(head_round_kernel<float>, flat_grid(blocks), dim3(256), 0, st, planes, S, rows, cols, (float*)out, ldo);
  return hipGetLastError();
}

hipError_t launch_head_one(float* one, hipStream_t st) {
  DPRC_LAUNCH(head_one_kernel, dim3(1), dim3(1), 0, st, one);
  return hipGetLastError();
}

}  // namespace dprc
