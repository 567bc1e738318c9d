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
#include <type_traits>
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

// WK groups of waves take a part of every slab's contraction each.
template <class E, int WM_, int WN_, int XB_, int YB_, int RING = 2, int WK_ = 1>
struct HeadTile {
  typedef E elem;
  static constexpr int WM = WM_, WN = WN_, XB = XB_, YB = YB_, WK = WK_;
  static constexpr int ring = RING;                     // slabs in LDS
  static constexpr int MT = 32 * XB * WM, NT = 32 * YB * WN, threads = 64 * WM * WN * WK;
  static constexpr int EP = kPiece<E>;                  // elements of a 16-byte piece
  static constexpr int slab = 8 * EP;                   // contraction elements of a slab: 64 bf16, 32 fp32
};

// An operand is `rows` rows of `width` elements, ld apart.  KC: its rows are the tile's rows (columns), the
// contraction runs along them.  KR: the contraction runs over its rows, the tile's rows (columns) along them.
// A slab of it in LDS is 128 bytes for every row (column) of the tile; the banks are 256 bytes wide.  KC: rows of
// 128 bytes, piece p of row r at p ^ swizzle_kc(r), so that a fragment read of 16 rows covers all banks.  KR, bf16: rows
// of the tile's width, piece p of row r at p ^ swizzle_kr(r), so that the 64 bytes that half a wave reads of each of
// 4 rows do; fp32 fragments are read along the rows and need none.
__device__ __forceinline__ int swizzle_kc(int r) { return (r >> 1) & 7; }
template <class E>
__device__ __forceinline__ int swizzle_kr(int r, int pieces) {
  return sizeof(E) != 2 ? 0 : pieces == 8 ? (r & 2) << 1 : (r & 3) << 2;
}

// A piece at (row, col), zeros past the rows and the width, at any alignment of the element.
template <class E>
__device__ __forceinline__ uint4 operand_piece(const HeadRows& X, int64_t row, int64_t col) {
  if (row >= X.rows || col >= X.width) return uint4{0, 0, 0, 0};
  const E* p = static_cast<const E*>(X.p) + row * X.ld;
  if constexpr (sizeof(E) == 2) {
    const int64_t at = row * X.ld + col, room = (X.rows - 1) * X.ld + X.width - 8;
    if (room < 0) return load8_elem(p, col, X.width, true);
    const int64_t from = min(at, room);
    const u32x4_any v = *reinterpret_cast<const u32x4_any*>(static_cast<const E*>(X.p) + from);
    return first_elems(shr_elems(uint4{v[0], v[1], v[2], v[3]}, (int)(at - from)), (int)min((int64_t)8, X.width - col));
  } else {
    if (col + 4 <= X.width) return load_piece<E>(p + col);
    return uint4{__float_as_uint(p[col]), col + 1 < X.width ? __float_as_uint(p[col + 1]) : 0u,
                 col + 2 < X.width ? __float_as_uint(p[col + 2]) : 0u, 0u};
  }
}

// 64 lanes' 16-byte pieces at byte offsets `off` of the resource to 1024 bytes of LDS, in lane order; zeros
// where the offset is out of the resource's range.
typedef __attribute__((address_space(3))) void lds_void_t;
template <bool NT>
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, void* lds, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_t*)lds, 16, (int)off, 0, 0, NT ? kCachePolicyNT : 0);
}

// A workgroup's slabs, an array each: the compiler then knows that loads into one do not reach reads of another, and does
// not wait for them.
template <class TL>
struct HeadLds {
  typename TL::elem *a[TL::ring], *b[TL::ring];
};
template <class TL>
__device__ __forceinline__ HeadLds<TL> head_lds(typename TL::elem* a0, typename TL::elem* a1, typename TL::elem* a2,
                                                typename TL::elem* a3, typename TL::elem* b0, typename TL::elem* b1,
                                                typename TL::elem* b2, typename TL::elem* b3) {
  if constexpr (TL::ring == 2) return HeadLds<TL>{{a0, a1}, {b0, b1}};
  else if constexpr (TL::ring == 3) return HeadLds<TL>{{a0, a1, a2}, {b0, b1, b2}};
  else return HeadLds<TL>{{a0, a1, a2, a3}, {b0, b1, b2, b3}};
}

template <int V>
struct HInt {
  static constexpr int value = V;
};

// One operand's slabs of a tile of T rows (columns) from t0 on: loads, straight into LDS where its rows allow
// 16-byte pieces (VEC), else through registers.
// NT: past the caches.
template <class TL, int T, bool KR, bool VEC, bool NT = false>
struct HeadOperand {
  typedef typename TL::elem E;
  static constexpr int EP = TL::EP, P = T * 8 / TL::threads, RP = T / EP;    // pieces of a thread; of a KR row
  static constexpr bool direct = VEC;
  static_assert(T * 8 % TL::threads == 0);
  const HeadRows& X;
  int64_t t0;
  int wave0;                           // the wave's first thread
  uint32_t off[VEC ? P : 1];           // byte offsets of the thread's pieces in a slab
  uint4 reg[VEC ? 1 : P];

  static __device__ __forceinline__ int kc_col(int s) { return EP * ((s & 7) ^ swizzle_kc(s >> 3)); }
  static __device__ __forceinline__ int kr_col(int s) { return EP * ((s % RP) ^ swizzle_kr<E>(s / RP, RP)); }

  __device__ __forceinline__ HeadOperand(const HeadRows& X_, int64_t t) : X(X_), t0(t) {
    wave0 = 64 * (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if constexpr (VEC) {
#pragma unroll
      for (int r = 0; r < P; ++r) {
        const int s = threadIdx.x + TL::threads * r;
        const int row = KR ? s / RP : s >> 3, col = KR ? kr_col(s) : kc_col(s);
        off[r] = KR && t0 + col >= X.width ? kOobOffset : ((uint32_t)row * (uint32_t)X.ld + (uint32_t)col) * (uint32_t)sizeof(E);
      }
    }
  }
  // a resource over `n` rows from row0 on, `skip` elements into them
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(int64_t row0, int n, int64_t skip) const {
    const int64_t left = X.rows - row0;
    const uint32_t rows = (uint32_t)(left < 0 || skip >= X.width ? 0 : left < n ? left : n);
    return buffer_rsrc(static_cast<const E*>(X.p) + (rows ? row0 * X.ld + skip : 0),
                       rows ? (rows * (uint32_t)X.ld - (uint32_t)skip) * (uint32_t)sizeof(E) : 0u);
  }
  // the slab at k on its way to LDS
  __device__ __forceinline__ void load(int64_t k, E* lds) {
    if constexpr (VEC && KR) {
      const __amdgpu_buffer_rsrc_t r0 = rsrc(k, TL::slab, t0);
#pragma unroll
      for (int r = 0; r < P; ++r) load_to_lds<NT>(r0, lds + EP * (wave0 + TL::threads * r), off[r]);
    } else if constexpr (VEC) {
      const __amdgpu_buffer_rsrc_t r0 = rsrc(t0, T, k);
      if (TL::ring > 2 || k + TL::slab > X.width) {      // columns past the rows' end
#pragma unroll
        for (int r = 0; r < P; ++r)
          load_to_lds<NT>(r0, lds + EP * (wave0 + TL::threads * r),
                          k + kc_col(threadIdx.x + TL::threads * r) < X.width ? off[r] : kOobOffset);
      } else {
#pragma unroll
        for (int r = 0; r < P; ++r) load_to_lds<NT>(r0, lds + EP * (wave0 + TL::threads * r), off[r]);
      }
    } else {
#pragma unroll
      for (int r = 0; r < P; ++r) {
        const int s = threadIdx.x + TL::threads * r;
        reg[r] = KR ? operand_piece<E>(X, k + s / RP, t0 + kr_col(s)) : operand_piece<E>(X, t0 + (s >> 3), k + kc_col(s));
      }
    }
  }
  __device__ __forceinline__ void arrive(E* lds) const {
    if constexpr (!VEC) {
#pragma unroll
      for (int r = 0; r < P; ++r) *reinterpret_cast<uint4*>(lds + EP * (threadIdx.x + TL::threads * r)) = reg[r];
    }
  }
  // The fragment of the 32 rows (columns) from b on, for contraction elements 2 EP ks .. of the slab: the
  // lane's row b + l % 32, its EP elements from 2 EP ks + EP (l / 32) on.  (fp32: four MFMAs of K = 2 take the
  // elements i and EP + i of these.)
  static constexpr int reads = !KR ? 1 : sizeof(E) == 2 ? 2 : 4;
  static __device__ __forceinline__ uint4 frag(const E* lds, int b, int ks, int lane) {
    const int l32 = lane & 31, half = lane >> 5;
    if constexpr (!KR) {
      const int row = b + l32;
      return *reinterpret_cast<const uint4*>(&lds[row * TL::slab + EP * ((2 * ks + half) ^ swizzle_kc(row))]);
    } else if constexpr (sizeof(E) == 2) {
      // lane group g reads rows 8 (g / 2) + r4 (+ 4) of columns 16 (g % 2) + 4 c4 .. of the block
      const int g = lane >> 4, r4 = (lane & 15) >> 2, c4 = lane & 3;
      const int row = 16 * ks + 8 * (g >> 1) + r4, col = b + 16 * (g & 1) + 4 * c4;
      const E* p = &lds[row * T + EP * ((col >> 3) ^ swizzle_kr<E>(row, RP)) + (col & 4)];
      return make_u4(lds_read_tr16(p), lds_read_tr16(p + 4 * T));
    } else {
      const E* p = &lds[(8 * ks + 4 * half) * T + b + l32];
      return uint4{__float_as_uint(p[0]), __float_as_uint(p[T]), __float_as_uint(p[2 * T]), __float_as_uint(p[3 * T])};
    }
  }
};

// acc += the products of a wave's fragments
template <class E, int XB, int YB>
__device__ __forceinline__ void head_mfma(const uint4 (&av)[XB], const uint4 (&bv)[YB], f32x16_t (&acc)[XB][YB]) {
  if constexpr (sizeof(E) == 2) {
#pragma unroll
    for (int x = 0; x < XB; ++x)
#pragma unroll
      for (int y = 0; y < YB; ++y)
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, av[x]),
                                                            __builtin_bit_cast(bf16x8_t, bv[y]), acc[x][y], 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < XB; ++x)
#pragma unroll
        for (int y = 0; y < YB; ++y) {
          const float a = __uint_as_float(i == 0 ? av[x].x : i == 1 ? av[x].y : i == 2 ? av[x].z : av[x].w);
          const float b = __uint_as_float(i == 0 ? bv[y].x : i == 1 ? bv[y].y : i == 2 ? bv[y].z : bv[y].w);
          acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, acc[x][y], 0, 0, 0);
        }
  }
}

// acc = sum over k in [k0, k1) of A[i][k] B[j][k], i and j the tile's rows and columns; k0 a multiple of the
// slab.  fp32 products and sums (bf16 products are exact).  While a slab is multiplied the next TL::ring - 1 are on
// their way.  A wave has the next fragments in registers ahead of their products, also
// across the slab's one barrier, and reads and products are issued in turn.
// bf16, 256 x 256 tiles of 128000 x 8192 x 2048: 1330 TFLOP/s (the same loop as the compiler orders it 1146, all
// reads before all products 1270, four waves of 128 x 128 1217, tiles of 128 x 128 1093).
template <class TL, class OA, class OB>
__device__ __forceinline__ void head_product(OA A, OB B, int64_t k0, int64_t k1, f32x16_t (&acc)[TL::XB][TL::YB],
                                             const HeadLds<TL>& lds) {
  typedef typename TL::elem E;
  constexpr int XB = TL::XB, YB = TL::YB, RING = TL::ring;
  // loads that may still be under way when a slab is needed (all of them wait where a register is between)
  constexpr int later = OA::direct && OB::direct ? (RING - 2) * (OA::P + OB::P) : 0;
  static_assert(later < 64 && (RING == 2 || (OA::direct && OB::direct)));
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int wm = wv / TL::WN % TL::WM, wn = wv % TL::WN;
  auto gload = [&](int64_t k, auto u) __attribute__((always_inline)) {
    A.load(k < k1 ? k : (int64_t)1 << 40, lds.a[decltype(u)::value]);      // past the end: zeros
    B.load(k < k1 ? k : (int64_t)1 << 40, lds.b[decltype(u)::value]);
  };
  // what went through registers to LDS, then every wave's slab is there and the reads of the one before it are done
  auto arrive = [&](auto u) __attribute__((always_inline)) {
    A.arrive(lds.a[decltype(u)::value]);
    B.arrive(lds.b[decltype(u)::value]);
    if constexpr (later > 0) {                          // (with the fences all loads would be waited for)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(later) : "memory");
    } else {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
      __builtin_amdgcn_s_waitcnt(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    }
  };
#pragma unroll
  for (int x = 0; x < XB; ++x)
#pragma unroll
    for (int y = 0; y < YB; ++y)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[x][y][q] = 0.f;
  uint4 f0a[XB], f0b[YB], f1a[XB], f1b[YB];
  auto frag = [&](uint4 (&av)[XB], uint4 (&bv)[YB], auto u, int ks) __attribute__((always_inline)) {
    const E* la = lds.a[decltype(u)::value];
    const E* lb = lds.b[decltype(u)::value];
#pragma unroll
    for (int y = 0; y < YB; ++y) bv[y] = OB::frag(lb, 32 * (wn * YB + y), ks, lane);
#pragma unroll
    for (int x = 0; x < XB; ++x) av[x] = OA::frag(la, 32 * (wm * XB + x), ks, lane);
  };
  auto phase = [&](uint4 (&na)[XB], uint4 (&nb)[YB], auto u, int ks, const uint4 (&av)[XB], const uint4 (&bv)[YB])
      __attribute__((always_inline)) {
    frag(na, nb, u, ks);
    head_mfma<E, XB, YB>(av, bv, acc);
    constexpr int reads = XB * OA::reads + YB * OB::reads, products = XB * YB * (sizeof(E) == 2 ? 1 : 4);
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
    constexpr HInt<(decltype(u)::value + 1) % RING> next{};
    gload(k + (RING - 1) * TL::slab, HInt<(decltype(u)::value + RING - 1) % RING>{});
    __builtin_amdgcn_sched_barrier(0);
    phase(f1a, f1b, u, 1, f0a, f0b);
    phase(f0a, f0b, u, 2, f1a, f1b);
    phase(f1a, f1b, u, 3, f0a, f0b);
    arrive(next);
    phase(f0a, f0b, next, 0, f1a, f1b);
  };
  gload(k0, HInt<0>{});
  if constexpr (RING > 2) gload(k0 + TL::slab, HInt<1>{});
  if constexpr (RING > 3) gload(k0 + 2 * TL::slab, HInt<2>{});
  arrive(HInt<0>{});
  if constexpr (TL::WK > 1) {
    static_assert(TL::WK == 4 && TL::WM * TL::WN * XB * YB == 1 && TL::MT * TL::slab * sizeof(E) == 4096);
    auto quarter = [&](int64_t k, auto u) __attribute__((always_inline)) {
      gload(k + (RING - 1) * TL::slab, HInt<(decltype(u)::value + RING - 1) % RING>{});
      frag(f0a, f0b, u, wv);
      head_mfma<E, XB, YB>(f0a, f0b, acc);
      arrive(HInt<(decltype(u)::value + 1) % RING>{});
    };
    for (int64_t k = k0; k < k1; k += RING * TL::slab) {
      quarter(k, HInt<0>{});
      quarter(k + TL::slab, HInt<1>{});
      if constexpr (RING > 2) quarter(k + 2 * TL::slab, HInt<2>{});
      if constexpr (RING > 3) quarter(k + 3 * TL::slab, HInt<3>{});
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    // every wave has the sum of the four, in their order
    float* part[4] = {reinterpret_cast<float*>(lds.a[0]), reinterpret_cast<float*>(lds.a[1]),
                      reinterpret_cast<float*>(lds.b[0]), reinterpret_cast<float*>(lds.b[1])};
    float* own = wv == 0 ? part[0] : wv == 1 ? part[1] : wv == 2 ? part[2] : part[3];
#pragma unroll
    for (int q = 0; q < 16; ++q) own[64 * q + lane] = acc[0][0][q];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 16; ++q)
      acc[0][0][q] = part[0][64 * q + lane] + part[1][64 * q + lane] + part[2][64 * q + lane] + part[3][64 * q + lane];
    __syncthreads();
    return;
  }
  frag(f0a, f0b, HInt<0>{}, 0);
  for (int64_t k = k0; k < k1; k += RING * TL::slab) {  // (slabs past the end: zeros)
    step(k, HInt<0>{});
    step(k + TL::slab, HInt<1>{});
    if constexpr (RING > 2) step(k + 2 * TL::slab, HInt<2>{});
    if constexpr (RING > 3) step(k + 3 * TL::slab, HInt<3>{});
  }
  if constexpr (later > 0) __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();                                     // all loads have arrived, all reads are done
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
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, wm = wv / TL::WN % TL::WM, wn = wv % TL::WN;
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

// LDS for a tile, stored transposed: rows of MT elements for its columns, the 16-byte piece p of row t at
// p ^ (t & 31), so that the columns of a block, one a lane, go to different banks.  The four arrays of a
// product's slabs in turn, 128 bytes for every row of the tile each.
template <class TL>
struct HeadStage {
  typedef typename TL::elem E;
  static constexpr int EP = TL::EP, PPR = TL::MT / EP, TPA = 128 / (int)sizeof(E);   // pieces of a row; rows of an array
  static_assert(TL::NT <= 2 * TPA || TL::MT == TL::NT, "the arrays' sizes");
  E *p0, *p1, *p2, *p3;
  __device__ __forceinline__ E* piece(int t, int p) const {
    const int part = t / TPA;
    E* base = part == 0 ? p0 : part == 1 ? p1 : part == 2 ? p2 : p3;
    return base + ((t % TPA) * PPR + (p ^ (t & (PPR < 32 ? PPR - 1 : 31)))) * EP;
  }
};

// What the errors of a lane's tokens are formed with, one token in each of the wave's column blocks.  Loaded
// before the product, whose time hides the loads', and looked at after it.
template <class TL>
struct HeadTokens {
  int64_t target[TL::YB];
  float lse[TL::YB], g[TL::YB];
  __device__ __forceinline__ HeadTokens(const HeadArgs& a, int64_t t0) {
    const int wn = (threadIdx.x >> 6) % TL::WN;
#pragma unroll
    for (int y = 0; y < TL::YB; ++y) {                  // (past the last token: the last one's, not stored)
      const int64_t t = min(a.N - 1, t0 + 32 * (wn * TL::YB + y) + (threadIdx.x & 31));
      target[y] = a.target[t];
      lse[y] = a.lse[t];
      g[y] = a.g[t];
    }
  }
};

// The tile's errors, through LDS into token rows.
template <class TL>
__device__ __forceinline__ void head_errors(const HeadArgs& a, int64_t tm, int64_t t0, const HeadTokens<TL>& tok,
                                            f32x16_t (&acc)[TL::XB][TL::YB], const HeadStage<TL>& stage) {
  typedef typename TL::elem E;
  constexpr int EP = TL::EP, PPR = TL::MT / EP;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, wm = wv / TL::WN % TL::WM, wn = wv % TL::WN;
  const int64_t vt = tm * TL::MT;                       // the tile's first column of this piece
  const int v0 = 32 * TL::XB * wm;                      // the wave's first in the tile
  const int end = (int)min((int64_t)TL::MT, a.nv - vt); // the tile's columns before the vocabulary's end
#pragma unroll
  for (int y = 0; y < TL::YB; ++y) {
    const int col = 32 * (wn * TL::YB + y) + (lane & 31);
    const bool kept = tok.target[y] >= 0;
    const float g = tok.g[y], lse = tok.lse[y], lse2 = lse * kLog2e;
    // the target's or the vocabulary's end among the wave's rows: few waves
    const int64_t row = tok.target[y] - a.v0 - vt - v0;
    const int at = kept && row >= 0 && row < 32 * TL::XB ? (int)row : -1;
    const bool rare = __any(at >= 0) || end < v0 + 32 * TL::XB;
    float own = 0.f;                                    // the target's logit
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
        const int v = v0 + 32 * x + acc_row(lane, 4 * q4);
        if (rare) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            own = at == v - v0 + q ? acc[x][y][4 * q4 + q] : own;
            e[q] = v + q >= end ? 0.f : e[q];
          }
        }
        E* o = stage.piece(col, v / EP) + (v & (EP - 1));
        if constexpr (sizeof(E) == 2) {
          const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{e[0], e[1]}, bf16x2_t));
          const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{e[2], e[3]}, bf16x2_t));
          *reinterpret_cast<uint2*>(o) = uint2{kept ? lo : 0u, kept ? hi : 0u};
        } else {
          *reinterpret_cast<float4*>(o) = kept ? float4{e[0], e[1], e[2], e[3]} : float4{0.f, 0.f, 0.f, 0.f};
        }
      }
    if (at >= 0 && ((at >> 2) & 1) == (lane >> 5)) {     // exp(x) - 1 without cancellation
      const float e = g * expm1f(own - lse);
      E* o = stage.piece(col, (v0 + at) / EP) + (at & (EP - 1));
      if constexpr (sizeof(E) == 2) {
        *o = __builtin_bit_cast(uint16_t, (__bf16)e);
        if (a.lo && t0 + col < a.N) a.lo[t0 + col] = e - (float)(__bf16)e;
      } else {
        *o = e;
      }
    }
  }
  __syncthreads();
  // a thread stores one piece of every ROWS-th token, R of them read before the first is stored
  constexpr int ROWS = TL::threads / PPR, R = TL::NT / ROWS < 8 ? TL::NT / ROWS : 8;
  static_assert(TL::threads % PPR == 0 && TL::NT % (ROWS * R) == 0);
  const int p = threadIdx.x % PPR, row0 = threadIdx.x / PPR;
  const int64_t v = vt + EP * p, room = a.width - v;
  if (room <= 0) return;
  const int rows = (int)min((int64_t)TL::NT, a.N - t0);
  E* to = static_cast<E*>(a.E) + (t0 + row0) * a.lde + v;
  for (int row = row0; row < rows; row += ROWS * R) {
    uint4 w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = *reinterpret_cast<const uint4*>(stage.piece(row + ROWS * r, p));
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + ROWS * r < rows) {
        if (room >= EP) {
          if (a.stream) store_piece<E, true>(to, w[r]);
          else store_piece<E>(to, w[r]);
        } else {
          const E* from = stage.piece(row + ROWS * r, p);
          for (int j = 0; j < room; ++j) to[j] = from[j];
        }
      }
      to += ROWS * a.lde;
    }
  }
}

// ---- the target's entries to 16 bits ---------------------------------------------------------------
// E_t,y(t) = g_t (p - 1) is by far the largest entry of most rows, and tokens of one sample share g: its rounding
// to bf16 would be an error of up to 2^-8 of dh_t, and of a row of dW alike, in one direction for whole samples (an
// error of 0.0022 to 0.0028 of all of dh and dW where the results' own rounding is 0.0017).  What it loses, lo_t, joins
// the products as slabs of their own, formed in LDS:
//   dh:  64 tokens of the tile at a time, A their diagonal of lo_t, B the rows W_y(t);
//   dW:  up to 64 tokens whose target is among the tile's rows, in their order, A one lo_t in every row, B the
//        rows h_t.
template <class TL, bool AKR, bool VB>
__device__ __forceinline__ void head_targets(const HeadMulArgs& a, int split, int64_t m0, int64_t n0, int64_t k0, int64_t k1,
                                             f32x16_t (&acc)[TL::XB][TL::YB], uint16_t* la0, uint16_t* la1, uint16_t* lb0) {
  constexpr int TH = TL::threads, NW = TH / 64, PA = TL::MT * 8 / TH, PB = TL::NT * 8 / TH, RP = TL::NT / 8;
  typedef HeadOperand<TL, TL::MT, AKR, true> OA;
  typedef HeadOperand<TL, TL::NT, true, true> OB;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, wm = wv / TL::WN % TL::WM, wn = wv % TL::WN;
  // A's slab: the k-th entry, zero where there is none, at row `row` of the tile; B's: row(k) of the operand
  auto slab = [&](auto row_of, bool in, int row, float lo) __attribute__((always_inline)) {
    uint4 v[PB];
    bool there[PB];
#pragma unroll
    for (int r = 0; r < PB; ++r) {                      // all loads first: whole pieces (VB) need no condition
      const int s = tid + TH * r;
      const int64_t from = row_of(s / RP), col = n0 + OB::kr_col(s);
      there[r] = from >= 0 && col < a.B.width;
      if constexpr (VB) v[r] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.B.p) + (there[r] ? from * a.B.ld + col : 0));
      else v[r] = there[r] ? operand_piece<uint16_t>(a.B, from, col) : uint4{0, 0, 0, 0};
    }
#pragma unroll
    for (int r = 0; r < PA; ++r) *reinterpret_cast<uint4*>(&la0[8 * (tid + TH * r)]) = uint4{0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < PB; ++r) *reinterpret_cast<uint4*>(&lb0[8 * (tid + TH * r)]) = select4(there[r], v[r], uint4{0, 0, 0, 0});
    __syncthreads();
    if (in) {                                           // (at most the first 64 threads)
      const int at = AKR ? tid * TL::MT + 8 * ((row >> 3) ^ swizzle_kr<uint16_t>(tid, TL::MT / 8)) + (row & 7)
                         : row * TL::slab + 8 * ((tid >> 3) ^ swizzle_kc(row)) + (tid & 7);
      la0[at] = __builtin_bit_cast(uint16_t, (__bf16)lo);
    }
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      uint4 av[TL::XB], bv[TL::YB];
#pragma unroll
      for (int y = 0; y < TL::YB; ++y) bv[y] = OB::frag(lb0, 32 * (wn * TL::YB + y), ks, lane);
#pragma unroll
      for (int x = 0; x < TL::XB; ++x) av[x] = OA::frag(la0, 32 * (wm * TL::XB + x), ks, lane);
      head_mfma<uint16_t, TL::XB, TL::YB>(av, bv, acc);
    }
    __syncthreads();
  };
  if constexpr (!AKR) {
    auto place = [&](int64_t t) __attribute__((always_inline)) {   // the target's row of B, or -1
      const int64_t y = a.target[min(t, a.rows - 1)] - a.v0;
      return t < a.rows && y < a.B.rows ? y : (int64_t)-1;
    };
    for (int j = 64 * split; j < TL::MT && m0 + j < a.rows; j += 64 * a.S) {   // dealt to the splits
      const int64_t t = m0 + j + tid;
      const bool in = tid < 64 && place(t) >= 0;
      slab([&](int k) __attribute__((always_inline)) { return place(m0 + j + k); }, in, j + tid, in ? a.lo[t] : 0.f);
    }
  } else {
    constexpr int R = 4;                                // targets a thread looks at in a round
    int* list = reinterpret_cast<int*>(la1);            // tokens, and their rows of the tile
    uint8_t* rows = reinterpret_cast<uint8_t*>(list + R * TH + 64);
    int* counts = reinterpret_cast<int*>(rows + R * TH + 64);
    static_assert(5 * (R * TH + 64) + 4 * R * NW <= 128 * TL::MT && TL::MT <= 256);
    int n = 0;
    for (int64_t base = k0; base < k1; base += R * TH) {
      int64_t row[R];
      uint64_t mask[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t t = base + r * TH + tid;
        row[r] = t < k1 ? a.target[t] - a.v0 - m0 : -1;
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        mask[r] = __ballot(row[r] >= 0 && row[r] < TL::MT && m0 + row[r] < a.rows);
        if (lane == 0) counts[r * NW + wv] = __popcll(mask[r]);
      }
      __syncthreads();
      int before[R], total = n;
#pragma unroll
      for (int r = 0; r < R; ++r)
        for (int w = 0; w < NW; ++w) {
          if (w == wv) before[r] = total;
          total += counts[r * NW + w];
        }
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (mask[r] >> lane & 1) {
          const int at = before[r] + __popcll(mask[r] & (((uint64_t)1 << lane) - 1));
          list[at] = (int)(base + r * TH + tid);
          rows[at] = (uint8_t)row[r];
        }
      __syncthreads();
      n = total;
      if (n < 64 && base + R * TH < k1) continue;       // (the same for all threads)
      for (int g = 0; g < n; g += 64) {
        const bool in = tid < 64 && g + tid < n;
        const int own = in ? list[g + tid] : 0;
        slab([&](int k) __attribute__((always_inline)) { return g + k < n ? (int64_t)list[g + k] : (int64_t)-1; }, in,
             in ? rows[g + tid] : 0, in ? a.lo[own] : 0.f);
      }
      n = 0;
    }
  }
}

// The tile written to, or added to, its place of a plane [rows][cols], or rounded into the result's rows.
template <class TL>
__device__ __forceinline__ void head_store(const HeadMulArgs& a, int split, int64_t m0, int64_t n0,
                                           f32x16_t (&acc)[TL::XB][TL::YB]) {
  typedef typename TL::elem E;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, wm = wv / TL::WN % TL::WM, wn = wv % TL::WN;
  float* plane = a.planes + split * a.rows * a.cols;
#pragma unroll
  for (int x = 0; x < TL::XB; ++x)
#pragma unroll
    for (int y = 0; y < TL::YB; ++y) {
      const int64_t col = n0 + 32 * (wn * TL::YB + y) + (lane & 31);
      if (col >= a.cols) continue;
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int64_t row = m0 + 32 * (wm * TL::XB + x) + acc_row(lane, q);
        if (row >= a.rows) continue;
        const float v = acc[x][y][q];
        if (a.out) {
          E* o = static_cast<E*>(a.out) + row * a.ldo + col;
          if constexpr (sizeof(E) == 2) *o = __builtin_bit_cast(uint16_t, (__bf16)v);
          else *o = v;
        } else {
          float* o = plane + row * a.cols + col;
          *o = a.add ? *o + v : v;
        }
      }
    }
}

// ---- kernels --------------------------------------------------------------------------------------

// arrays for slabs of MT rows and NT columns, RING (2 to 4) of each
#define DPRC_HEAD_SLABS(E, MT, NT, SLAB, RING)                                        \
  __shared__ __attribute__((aligned(16))) E la0[MT * SLAB];                           \
  __shared__ __attribute__((aligned(16))) E la1[MT * SLAB];                           \
  __shared__ __attribute__((aligned(16))) E la2[RING > 2 ? MT * SLAB : 8];            \
  __shared__ __attribute__((aligned(16))) E la3[RING > 3 ? MT * SLAB : 8];            \
  __shared__ __attribute__((aligned(16))) E lb0[NT * SLAB];                           \
  __shared__ __attribute__((aligned(16))) E lb1[NT * SLAB];                           \
  __shared__ __attribute__((aligned(16))) E lb2[RING > 2 ? NT * SLAB : 8];            \
  __shared__ __attribute__((aligned(16))) E lb3[RING > 3 ? NT * SLAB : 8]
#define DPRC_HEAD_LDS(TL) head_lds<TL>(la0, la1, la2, la3, lb0, lb1, lb2, lb3)

// The logits' tiles.  Rows of W in 16-byte pieces (VW) or at any alignment; h always in pieces.
template <class TL, bool ERRORS, bool VW>
__global__ __launch_bounds__(TL::threads) void head_logits_kernel(HeadArgs a) {
  DPRC_HEAD_SLABS(typename TL::elem, TL::MT, TL::NT, TL::slab, TL::ring);
  const int64_t tm_n = (a.nv + TL::MT - 1) / TL::MT, tn_n = (a.N + TL::NT - 1) / TL::NT;
  const int64_t wg = flat_block();
  if (wg >= tm_n * tn_n) return;
  int64_t tm, tn;
  tile_of(wg, tm_n, tn_n, tm, tn);
  f32x16_t acc[TL::XB][TL::YB];
  constexpr bool STREAM = TL::NT < TL::MT;              // few tokens: every row of W is read once
  auto product = [&] {
    head_product<TL>(HeadOperand<TL, TL::MT, false, VW, STREAM>(a.W, tm * TL::MT),
                     HeadOperand<TL, TL::NT, false, true>(a.h, tn * TL::NT), 0, a.W.width, acc, DPRC_HEAD_LDS(TL));
  };
  if constexpr (ERRORS) {
    const HeadTokens<TL> tok(a, tn * TL::NT);
    product();
    head_errors<TL>(a, tm, tn * TL::NT, tok, acc, HeadStage<TL>{la0, la1, lb0, lb1});
  } else {
    product();
    head_sums<TL>(a, tm, tn * TL::NT, acc, reinterpret_cast<float2*>(la0));
  }
}

// A tile of A B, of one split of the contraction.  B's rows are the contraction's; so are A's with AKR.
template <class TL, bool AKR, bool VB>
__device__ __forceinline__ void head_mul(const HeadMulArgs& a, int64_t tm, int64_t tn, int split, const HeadLds<TL>& lds) {
  const int64_t k0 = split * a.per_split, k1 = min(a.K, k0 + a.per_split);
  f32x16_t acc[TL::XB][TL::YB];
  head_product<TL>(HeadOperand<TL, TL::MT, AKR, true>(a.A, tm * TL::MT),
                   HeadOperand<TL, TL::NT, true, VB>(a.B, tn * TL::NT), k0, k1, acc, lds);
  if constexpr (sizeof(typename TL::elem) == 2)
    head_targets<TL, AKR, VB>(a, split, tm * TL::MT, tn * TL::NT, k0, k1, acc, lds.a[0], lds.a[1], lds.b[0]);
  head_store<TL>(a, split, tm * TL::MT, tn * TL::NT, acc);
}

// blockIdx.z the split.
template <class TL, bool AKR, bool VB>
__global__ __launch_bounds__(TL::threads) void head_mul_kernel(HeadMulArgs a) {
  DPRC_HEAD_SLABS(typename TL::elem, TL::MT, TL::NT, TL::slab, TL::ring);
  const int64_t tm_n = (a.rows + TL::MT - 1) / TL::MT, tn_n = (a.cols + TL::NT - 1) / TL::NT;
  const int64_t wg = flat_block();
  if (wg >= tm_n * tn_n) return;
  int64_t tm, tn;
  tile_of(wg, tm_n, tn_n, tm, tn);
  head_mul<TL, AKR, VB>(a, tm, tn, blockIdx.z, DPRC_HEAD_LDS(TL));
}

// dh and dW in one launch, the tiles of every split of x, then those of y: neither's last round leaves CUs idle.  Gradients
// of N x d x V = 150 x 136 x 1009, 200 x 512 x 8000, 2000 x 512 x 8000 bf16 19, 33, 81 us, in two launches 25, 44, 107; fp32
// 24, 75, 412 and 30, 84, 425.
template <class TX, class TY, bool VB>
__global__ __launch_bounds__(TY::threads) void head_pair_kernel(HeadMulArgs x, HeadMulArgs y) {
  static_assert(TX::threads == TY::threads && TX::ring == TY::ring);
  typedef typename std::conditional<(TX::MT > TY::MT), TX, TY>::type TL;
  DPRC_HEAD_SLABS(typename TL::elem, TL::MT, TL::NT, TL::slab, TL::ring);
  auto tile = [&](auto t, const HeadMulArgs& a, int64_t wg, auto f) __attribute__((always_inline)) {
    typedef decltype(t) TL;
    const int64_t tm_n = (a.rows + TL::MT - 1) / TL::MT, tn_n = (a.cols + TL::NT - 1) / TL::NT, tiles = tm_n * tn_n;
    if (wg >= tiles * a.S) return wg - tiles * a.S;
    const int split = (int)(wg / tiles);
    int64_t tm, tn;
    tile_of(wg - split * tiles, tm_n, tn_n, tm, tn);
    f(tm, tn, split);
    return (int64_t)-1;
  };
  const int64_t wg = tile(TX{}, x, flat_block(), [&](int64_t tm, int64_t tn, int split) __attribute__((always_inline)) {
    head_mul<TX, false, VB>(x, tm, tn, split, DPRC_HEAD_LDS(TX)); });
  if (wg >= 0)
    tile(TY{}, y, wg, [&](int64_t tm, int64_t tn, int split) __attribute__((always_inline)) {
      head_mul<TY, true, true>(y, tm, tn, split, DPRC_HEAD_LDS(TY)); });
}

// Joins the tiles' maxima and sums in a fixed order and takes the target's logit, summed in fp32.  TPB tokens per
// workgroup: 64 / TPB groups of TPB lanes of every wave go through the tiles and are joined, then the waves; a
// wave per token multiplies h_t and W_y(t).  A target past the vocabulary makes both outputs NaN.
template <class E, int TPB>
__global__ __launch_bounds__(1024) void head_join_kernel(HeadArgs a, int64_t tiles, float* loss, float* lse) {
  __shared__ float2 buf[16][TPB];
  const int64_t t0 = (int64_t)flat_block() * TPB;
  if (t0 >= a.N) return;
  const int j = threadIdx.x % TPB, grp = threadIdx.x / TPB, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int64_t t = t0 + wv, y = wv < TPB && t < a.N ? a.target[t] : -1;
  float2 v{-1e38f, 0.f};
  if (t0 + j < a.N)
    for (int64_t s = grp; s < tiles; s += 1024 / TPB) v = join(v, a.part[s * a.N + t0 + j]);
#pragma unroll
  for (int off = TPB; off < 64; off *= 2) v = join(v, float2{__shfl_xor(v.x, off, 64), __shfl_xor(v.y, off, 64)});
  if (lane < TPB) buf[wv][lane] = v;
  __syncthreads();
  if (wv >= TPB || t >= a.N) return;
  v = buf[lane & 15][wv];
#pragma unroll
  for (int off = 1; off < 16; off *= 2) v = join(v, float2{__shfl_xor(v.x, off, 64), __shfl_xor(v.y, off, 64)});
  float dot = 0.f;
  if (y >= 0 && y < a.W.rows) {
    const HeadRows h{static_cast<const E*>(a.h.p) + t * a.h.ld, a.h.ld, 1, a.W.width};
    const HeadRows w{static_cast<const E*>(a.W.p) + y * a.W.ld, a.W.ld, 1, a.W.width};
    constexpr int EP = kPiece<E>;
    for (int64_t c = EP * lane; c < a.W.width; c += EP * 64) {
      float u[EP], v[EP];
      unpack<E>(operand_piece<E>(h, 0, c), u);
      unpack<E>(operand_piece<E>(w, 0, c), v);
#pragma unroll
      for (int j = 0; j < EP; ++j) dot = fmaf(u[j], v[j], dot);
    }
  }
  dot = wave_sum(dot);
  if (lane > 0) return;
  const float z = y >= a.W.rows ? NAN : v.x + logf(v.y), l = z - dot;
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

// ---- launches -------------------------------------------------------------------------------------

typedef HeadTile<uint16_t, 2, 4, 4, 2> TileWide;       // 256 x 256, eight waves of 128 x 64
typedef HeadTile<uint16_t, 2, 2, 2, 2> TileMid;        // 128 x 128, four waves of 64 x 64
typedef HeadTile<uint16_t, 2, 2, 1, 1> TileSmall;      // 64 x 64, four waves of 32 x 32
typedef HeadTile<uint16_t, 2, 2, 2, 2, 4> TileMidRing;
typedef HeadTile<uint16_t, 2, 2, 1, 1, 4> TileSmallRing;
typedef HeadTile<float, 2, 2, 2, 2> TileMidF32;
typedef HeadTile<float, 2, 2, 1, 1> TileSmallF32;
typedef HeadTile<float, 1, 1, 1, 1, 2, 4> TileLeastF32;  // 32 x 32, four waves of a quarter of the contraction
typedef HeadTile<float, 1, 1, 1, 1, 4, 4> TileLeastRingF32;
typedef HeadTile<uint16_t, 4, 1, 1, 2> TileFew;        // 128 x 64, four waves of 32 x 64
typedef HeadTile<uint16_t, 4, 1, 1, 2, 3> TileFewRing;
typedef HeadTile<float, 4, 1, 2, 1> TileFewF32;        // 256 x 32, four waves of 64 x 32

// Four slabs in LDS for bf16 tiles so few that they all run at once with them, and a contraction of 8 slabs or more: a slab
// is on its way while three are multiplied.  Loss of N x d x V = 100 x 2048 x 32000, 64 x 2048 x 8000 36, 25 us, with two
// 47, 32; dh of 500 x 1024 x 20000 with errors 98 and 104.  Shorter ones lose by it (dW of 8 tokens 33 and 31), fp32 products are
// as fast without.
static bool ring_tiles(int64_t m, int64_t n, int64_t K, int64_t S, int side, int bf16) {
  return bf16 && K >= 8 * TileMid::slab && ceil_div(m, side) * ceil_div(n, side) * S <= (side == 64 ? 512 : side == 128 ? 256 : 0);
}

// f(tile) with the ring's tile or the other.
template <class T, class R, class F>
static void ring_if(bool ring, T tile, R ringed, F&& f) {
  if (ring) f(ringed);
  else f(tile);
}

// The side of the tiles of an m x n result: the largest that leaves no CU without a tile, else small ones.
static int tile_side(int64_t m, int64_t n, int bf16) {
  if (bf16 && ceil_div(m, 256) * ceil_div(n, 256) >= 192) return 256;
  return ceil_div(m, 128) * ceil_div(n, 128) >= 192 ? 128 : 64;
}

// Rows of an m x n result that whole rounds of 256 x 256 tiles over the CUs take, or all of them where the last round is not
// nearly empty (they are then launches of their own, of smaller tiles).  3 rounds and 8, 40, 80, 104, 128 tiles, 2048 tokens,
// us with and without: d 2048, loss 189, 194, 200, 210, 211 and 206, 207, 209, 210, 211, errors and dW 452, 468, 491, 505, 510 and
// 491, 493, 502, 520, 502; d 1024, loss 192, 198, 206, 205, 210 and 200, 200, 202, 208, 208.
constexpr int64_t kHeadLastRound = 80;
static int64_t whole_rounds(int64_t m, int64_t n) {
  const int64_t tm = ceil_div(m, 256), tn = ceil_div(n, 256), last = ceil_div(tm * tn % 256, tn);   // rows of tiles
  return tm * tn < 256 || last * tn > kHeadLastRound || (tm - last) * tn < 192 ? m : std::min(m, 256 * (tm - last));
}

// Up to 64 tokens (32 in fp32) of a large vocabulary: tiles of all tokens and 128 (256) rows of W, which bounds the call and
// is read past the caches; bf16 with three slabs in LDS, two workgroups a CU.  64 tokens of 2048 and V 128256, 65536, 32000
// (32 tokens) bf16 96, 61, 37 us; two slabs 111, 67, 41, four (one workgroup a CU) 102, 66, 35; 256 rows and two slabs
// 102, 67, 53; d 512 and V 250000 53, with 256 rows 49.  Every wave reading rows of its own into registers: 3 times as slow.
static bool few_tokens(int64_t N, int64_t nv, int bf16) { return N <= (bf16 ? 64 : 32) && nv >= 64 * 256; }

// So few fp32 tiles of 64 x 64 that their contraction's length bounds them take 32 x 32, a quarter of it for each wave.  Loss of
// N x d x V = 16 x 4096 x 300, 64 x 2048 x 4096, 200 x 2048 x 2000 43, 30, 38 us, in tiles of 64 92, 54, 53; up to 256 of
// them 64 x 1024 x 12000 31 and 36, but 100 x 512 x 8000 24 and 22.
constexpr int64_t kHeadLeast = 128;

static int logits_side(int64_t N, int64_t nv, int bf16) {
  if (few_tokens(N, nv, bf16)) return 0;
  // one column of tiles: narrow ones, of which two share a CU
  const int side = tile_side(nv, N, bf16);
  if (!bf16 && side == 64 && ceil_div(nv, 64) * ceil_div(N, 64) <= kHeadLeast) return 32;
  return bf16 ? (N <= 128 ? std::min(side, 128) : side) : (N <= 64 ? 64 : side);
}

// Columns that whole rounds of large tiles over the CUs take; a last round of few tiles is a launch of its own, of smaller
// ones.
static int64_t logits_rounds(int64_t N, int64_t nv, int bf16) {
  return logits_side(N, nv, bf16) == 256 ? whole_rounds(nv, N) : nv;
}

static int64_t logits_tiles(int64_t N, int64_t nv, int bf16) {
  const int side = logits_side(N, nv, bf16);
  return ceil_div(nv, side > 0 ? side : bf16 ? TileFew::MT : TileFewF32::MT);
}

template <bool ERRORS>
static void launch_logits_part(const HeadArgs& a, hipStream_t st) {
  auto tiles = [&](auto tile) {
    typedef decltype(tile) TL;
    const dim3 grid = flat_grid(ceil_div(a.nv, TL::MT) * ceil_div(a.N, TL::NT));
    if (a.vec_w) DPRC_LAUNCH((head_logits_kernel<TL, ERRORS, true>), grid, dim3(TL::threads), 0, st, a);
    else if constexpr (TL::ring == 2) DPRC_LAUNCH((head_logits_kernel<TL, ERRORS, false>), grid, dim3(TL::threads), 0, st, a);
  };
  const int side = logits_side(a.N, a.nv, a.bf16);
  const bool ring = side > 0 && a.vec_w && ring_tiles(a.nv, a.N, a.W.width, 1, side, a.bf16);
  if (a.bf16) {
    if (side == 0) ring_if(a.vec_w, TileFew{}, TileFewRing{}, tiles);
    else if (side == 256) tiles(TileWide{});
    else if (side == 128) ring_if(ring, TileMid{}, TileMidRing{}, tiles);
    else ring_if(ring, TileSmall{}, TileSmallRing{}, tiles);
  } else {
    if (side == 0) tiles(TileFewF32{});
    else if (side == 128) tiles(TileMidF32{});
    else if (side == 64) tiles(TileSmallF32{});
    else ring_if(a.vec_w, TileLeastF32{}, TileLeastRingF32{}, tiles);
  }
}

template <bool ERRORS>
static hipError_t launch_head_logits(const HeadArgs& all, hipStream_t st) {
  const int64_t whole = logits_rounds(all.N, all.nv, all.bf16), e = all.bf16 ? 2 : 4;
  HeadArgs a = all;
  if (whole < all.nv) {
    a.nv = a.W.rows = a.width = whole;
    launch_logits_part<ERRORS>(a, st);
    a = all;
    a.nv = a.W.rows = all.nv - whole;
    a.v0 += whole;
    a.width -= whole;
    a.W.p = static_cast<const char*>(a.W.p) + whole * a.W.ld * e;
    if (ERRORS) a.E = static_cast<char*>(a.E) + whole * e;
    else a.part += logits_tiles(a.N, whole, a.bf16) * a.N;
  }
  launch_logits_part<ERRORS>(a, st);
  return hipGetLastError();
}

// tiles of the vocabulary that the sums leave
int64_t head_sum_tiles(int64_t N, int64_t nv, int bf16) {
  const int64_t whole = logits_rounds(N, nv, bf16);
  return logits_tiles(N, whole, bf16) + (whole < nv ? logits_tiles(N, nv - whole, bf16) : 0);
}

hipError_t launch_head_sums(const HeadArgs& a, hipStream_t st) { return launch_head_logits<false>(a, st); }
// E past the caches where it is larger than they are: 8192 x 65536 x 2048 1924 and 1898 us, 4096 x 50176 x 1024 504 and 472
// (without storing E at all 1780 and 418: every CU stores its tile at about the same time).
hipError_t launch_head_errors(HeadArgs a, hipStream_t st) {
  a.stream = a.N * a.width * (a.bf16 ? 2 : 4) > kStreamRowsBytes;
  return launch_head_logits<true>(a, st);
}

hipError_t launch_head_join(const HeadArgs& a, int64_t tiles, float* loss, float* lse, hipStream_t st) {
  auto go = [&](auto kernel, int tpb) { DPRC_LAUNCH(kernel, flat_grid(ceil_div(a.N, tpb)), dim3(1024), 0, st, a, tiles, loss, lse); };
  if (a.N <= 1024) {
    if (a.bf16) go(head_join_kernel<uint16_t, 4>, 4);
    else go(head_join_kernel<float, 4>, 4);
  } else {
    if (a.bf16) go(head_join_kernel<uint16_t, 16>, 16);
    else go(head_join_kernel<float, 16>, 16);
  }
  return hipGetLastError();
}

static HeadMulPlan split_plan(int64_t K, int64_t want, int side, int bf16) {
  const int64_t slab = bf16 ? TileWide::slab : TileMidF32::slab, slabs = ceil_div(K, slab);
  HeadMulPlan p;
  p.side = side;
  p.per_split = ceil_div(slabs, want) * slab;
  p.S = (int32_t)ceil_div(slabs * slab, p.per_split);
  return p;
}

// Long contractions are split among the largest tiles that then fill the CUs, short ones take smaller tiles.  dh of 500 and 4084
// tokens of 20000 x 1024 and 8000 x 256 bf16, with errors: 96 and 82 us, in tiles of 64 138 and 117.
HeadMulPlan head_mul_plan(int64_t rows, int64_t cols, int64_t K, int bf16) {
  const int64_t slabs = ceil_div(K, bf16 ? TileWide::slab : TileMidF32::slab);
  int side = tile_side(rows, cols, bf16);
  for (int large = bf16 ? 256 : 128; large > side; large /= 2)
    if (ceil_div(rows, large) * ceil_div(cols, large) * (slabs / 16) >= 192) side = large;
  const int64_t tiles = ceil_div(rows, side) * ceil_div(cols, side);
  const int64_t want = tiles >= 192 ? 1 : std::min<int64_t>(ceil_div(256, tiles), std::max<int64_t>(1, slabs / (side == 64 ? 4 : 16)));
  return split_plan(K, want, side, bf16);
}

// Rows that go with whole rounds of large tiles; the others are a product of their own with a plan of its own.
int64_t head_mul_rounds(int64_t rows, int64_t cols, int64_t K, int bf16) {
  const HeadMulPlan p = head_mul_plan(rows, cols, K, bf16);
  return bf16 && p.side == 256 && p.S == 1 ? whole_rounds(rows, cols) : rows;
}

HeadMulPlan head_mul_plan_like(const HeadMulPlan& p, int64_t K, int bf16) { return split_plan(K, p.S, p.side, bf16); }

template <bool AKR>
static void launch_mul(const HeadMulArgs& a, hipStream_t st) {
  auto go = [&](auto kernel, auto tile) {
    typedef decltype(tile) TL;
    dim3 grid = flat_grid(ceil_div(a.rows, TL::MT) * ceil_div(a.cols, TL::NT));
    grid.z = (unsigned)a.S;
    DPRC_LAUNCH(kernel, grid, dim3(TL::threads), 0, st, a);
  };
  auto rows = [&](auto tile) {
    typedef decltype(tile) TL;
    if constexpr (AKR) go(head_mul_kernel<TL, true, true>, tile);      // h's copy
    else if (a.vec_b) go(head_mul_kernel<TL, false, true>, tile);
    else if constexpr (TL::ring == 2) go(head_mul_kernel<TL, false, false>, tile);
  };
  const bool ring = a.vec_b && ring_tiles(a.rows, a.cols, a.per_split, a.S, a.side, a.bf16);
  if (a.bf16 && a.side == 256) rows(TileWide{});
  else if (a.bf16 && a.side == 128) ring_if(ring, TileMid{}, TileMidRing{}, rows);
  else if (a.bf16) ring_if(ring, TileSmall{}, TileSmallRing{}, rows);
  else if (a.side == 128) rows(TileMidF32{});
  else rows(TileSmallF32{});
}

hipError_t launch_head_mul(HeadMulArgs a, hipStream_t st) {
  if (a.akr) launch_mul<true>(a, st);
  else launch_mul<false>(a, st);
  return hipGetLastError();
}

bool head_mul_pairs(const HeadMulPlan& x, const HeadMulPlan& y) { return x.side <= 128 && y.side <= 128; }

hipError_t launch_head_pair(HeadMulArgs x, HeadMulArgs y, hipStream_t st) {
  auto go = [&](auto tx, auto ty) {
    typedef decltype(tx) TX;
    typedef decltype(ty) TY;
    const int64_t blocks = ceil_div(x.rows, TX::MT) * ceil_div(x.cols, TX::NT) * x.S + ceil_div(y.rows, TY::MT) * ceil_div(y.cols, TY::NT) * y.S;
    if (x.vec_b) DPRC_LAUNCH((head_pair_kernel<TX, TY, true>), flat_grid(blocks), dim3(TY::threads), 0, st, x, y);
    else if constexpr (TX::ring == 2) DPRC_LAUNCH((head_pair_kernel<TX, TY, false>), flat_grid(blocks), dim3(TY::threads), 0, st, x, y);
  };
  auto sides = [&](auto small, auto mid) {
    if (x.side == 128 && y.side == 128) go(mid, mid);
    else if (x.side == 128) go(mid, small);
    else if (y.side == 128) go(small, mid);
    else go(small, small);
  };
  const auto ring = [](const HeadMulArgs& a) { return a.side == 64 && a.vec_b && ring_tiles(a.rows, a.cols, a.per_split, a.S, 64, a.bf16); };
  if (ring(x) && ring(y)) go(TileSmallRing{}, TileSmallRing{});
  else if (x.bf16) sides(TileSmall{}, TileMid{});
  else sides(TileSmallF32{}, TileMidF32{});
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

}  // namespace dprc
