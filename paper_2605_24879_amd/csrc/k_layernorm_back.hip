// Backward pass of dropout, residual sum and norm, with the weight's and bias's gradient of every
// sample by itself.
//
// Bounded by memory: one pass over dy, s and ds writes dx and dh and sums dw and db on the way.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

// entries c .. c + N - 1 (N a multiple of 4) of a fp32 vector of n
template <int N>
__device__ __forceinline__ void store_vec(float* p, int c, int n, const float* x) {
#pragma unroll
  for (int q = 0; q < N; q += 4) {
    if (c + q + 4 <= n) {
      store_piece(p + c + q, pack<float>(x + q));
      continue;
    }
#pragma unroll
    for (int j = q; j < q + 4; ++j)
      if (c + j < n) p[c + j] = x[j];
  }
}

// TPR threads hold a row as in the forward pass, 256 / TPR row groups a workgroup.  A work item is
// a token split of a sample, whose rows its workgroup's groups take in turn, each thread summing
// dw and db of its own columns in registers; the groups' sums meet at the item's end, in lanes
// and in LDS.  With SOLO (samples shorter than a few rounds of the groups) an item is
// a sample for each group, and nothing is combined.
template <class E, int M, int TPR, int C, bool SOLO>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_back_kernel(NormBackArgs a, int64_t per, int64_t items) {
  constexpr int EP = kPiece<E>, V = C / EP, BLK = TPR > 256 ? TPR : 256, RPB = BLK / TPR;
  constexpr int G = SOLO ? 1 : (TPR < 64 ? BLK / 64 : RPB);      // sums to combine in LDS
  constexpr int kAhead = V <= 2 ? 2 : 1;                          // rows loading ahead
  typedef RowSum<TPR, 2, BLK> Sum;
  __shared__ typename Sum::Buffer buf;
  __shared__ float comb[G > 1 ? G - 1 : 1][2][G > 1 ? C : 1][G > 1 ? TPR : 1];
  int turn = 0;
  const int t = threadIdx.x % TPR, rg = threadIdx.x / TPR, n = (int)a.n;
  const bool grads = a.dw || a.db;

  float w[C];
#pragma unroll
  for (int v = 0; v < V; ++v) load_vec<EP>(a.w, a.wbf16, (v * TPR + t) * EP, n, 1.f, w + v * EP);

  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t i = SOLO ? it * RPB + rg : it / a.S;
    const int64_t first = SOLO ? 0 : (it - i * a.S) * per;
    const int64_t last = SOLO ? (i < a.B ? a.T : 0) : std::min<int64_t>(a.T, first + per);
    const int64_t trips = SOLO ? a.T : (last - first + RPB - 1) / RPB;
    int64_t tok = first + (SOLO ? 0 : rg);
    constexpr int kTokStep = SOLO ? 1 : RPB;

    struct Row {
      uint4 dy[V], s[V], ds[V];
      float mu, rstd;
    };
    auto load = [&](Row& x, int64_t token) {
      const int64_t r = std::min(i, a.B - 1) * a.T + std::min(token, a.T - 1);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + t) * EP;
        x.dy[v] = load_row<E, M>((const E*)a.dy + r * a.lddy, c, n);
        x.s[v] = load_row<E, M>((const E*)a.s + r * a.lds, c, n);
        if (a.ds) x.ds[v] = load_row<E, M>((const E*)a.ds + r * a.ldds, c, n);
      }
      if (!a.rms) x.mu = a.mean[r];
      x.rstd = a.rstd[r];
    };
    float dw[C], db[C];
#pragma unroll
    for (int k = 0; k < C; ++k) dw[k] = db[k] = 0.f;
    // one round: this row's sums, the loads of the row two rounds on, the mask, then the outputs
    auto round = [&](Row& x) {
      float g[C], xh[C], z[C], red[2] = {0.f, 0.f};
      const float rs = x.rstd, mu = a.rms ? 0.f : x.mu;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + t) * EP;
        if (tok >= last || c >= n) continue;
        unpack_row<E, M>(x.dy[v], c, n, g + v * EP);
        unpack_row<E, M>(x.s[v], c, n, xh + v * EP);
        if (a.ds) unpack_row<E, M>(x.ds[v], c, n, z + v * EP);
        else
#pragma unroll
          for (int k = v * EP; k < v * EP + EP; ++k) z[k] = 0.f;
#pragma unroll
        for (int k = v * EP; k < v * EP + EP; ++k) {
          xh[k] = (xh[k] - mu) * rs;
          db[k] += g[k];
          dw[k] = fmaf(g[k], xh[k], dw[k]);
          g[k] *= w[k];
          red[0] += g[k];
          red[1] = fmaf(g[k], xh[k], red[1]);
        }
      }
      load(x, tok + kAhead * kTokStep);
      const int64_t r = i * a.T + tok;
      u32x4 mask[V];
      const bool drop = a.dh && a.drop.on;
      if (drop)
#pragma unroll
        for (int v = 0; v < V; ++v) mask[v] = drop_words<E>(a.drop, (uint32_t)r, (v * TPR + t) * EP);
      Sum::run(red, buf, turn);
      const float mg = a.rms ? 0.f : red[0] * a.inv_n, mgx = red[1] * a.inv_n;
      if (tok < last)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int c = (v * TPR + t) * EP;
          if (c >= n) continue;
#pragma unroll
          for (int k = v * EP; k < v * EP + EP; ++k) z[k] = fmaf(rs, fmaf(-xh[k], mgx, g[k] - mg), z[k]);
          if (a.dx) store_row<E, M>((E*)a.dx + r * a.lddx, c, n, z + v * EP);
          if (!a.dh) continue;
          if (drop) drop_apply<E>(a.drop, mask[v], z + v * EP);
          store_row<E, M>((E*)a.dh + r * a.lddh, c, n, z + v * EP);
        }
      tok += kTokStep;
    };
    Row even, odd;
    load(even, tok);
    if constexpr (kAhead == 2) load(odd, tok + kTokStep);
    for (int64_t trip = 0; trip < trips; ++trip) {
      round(even);
      if constexpr (kAhead == 2)
        if (++trip < trips) round(odd);
    }
    if (!grads) continue;
    if (!SOLO) {
      if (TPR < 64)
#pragma unroll
        for (int k = 0; k < C; ++k) {
          dw[k] = group_sum<TPR>(dw[k]);
          db[k] = group_sum<TPR>(db[k]);
        }
      if constexpr (G > 1) {
        const int grp = TPR < 64 ? threadIdx.x >> 6 : rg;
        __syncthreads();                                  // the item before has read its sums
        if (grp > 0)
#pragma unroll
          for (int k = 0; k < C; ++k) {
            comb[grp - 1][0][k][t] = dw[k];
            comb[grp - 1][1][k][t] = db[k];
          }
        __syncthreads();
        if (grp == 0)
#pragma unroll
          for (int k = 0; k < C; ++k)
#pragma unroll
            for (int q = 0; q < G - 1; ++q) {
              dw[k] += comb[q][0][k][t];
              db[k] += comb[q][1][k][t];
            }
      }
    }
    if (SOLO ? i >= a.B : rg > 0) continue;
    float *pw = a.dw, *pb = a.db;
    if (!SOLO && a.S > 1) {
      pw = a.dw ? a.part + it * 2 * n : nullptr;
      pb = a.db ? a.part + it * 2 * n + n : nullptr;
    } else {
      if (pw) pw += i * a.ldg;
      if (pb) pb += i * a.ldg;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * EP;
      if (pw) store_vec<EP>(pw, c, n, dw + v * EP);
      if (pb) store_vec<EP>(pb, c, n, db + v * EP);
    }
  }
}

// ---- rows longer than a workgroup's registers hold -----------------------------------------------

// dx and dh: one workgroup per row, two passes over it.
template <class E, int M>
__global__ __launch_bounds__(1024) void norm_back_rows_kernel(NormBackArgs a) {
  constexpr int EP = kPiece<E>;
  typedef RowSum<1024, 2, 1024> Sum;
  __shared__ typename Sum::Buffer buf;
  int turn = 0;
  const int n = (int)a.n;
  const int64_t rows = a.B * a.T;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const float mu = a.rms ? 0.f : a.mean[r], rs = a.rstd[r];
    float g[EP], xh[EP], w[EP], z[EP], red[2] = {0.f, 0.f};
    auto piece = [&](int c) {
      unpack_row<E, M>(load_row<E, M>((const E*)a.dy + r * a.lddy, c, n), c, n, g);
      unpack_row<E, M>(load_row<E, M>((const E*)a.s + r * a.lds, c, n), c, n, xh);
      load_vec<EP>(a.w, a.wbf16, c, n, 1.f, w);
#pragma unroll
      for (int j = 0; j < EP; ++j) {
        xh[j] = (xh[j] - mu) * rs;
        g[j] *= w[j];
      }
    };
    for (int c = threadIdx.x * EP; c < n; c += 1024 * EP) {
      piece(c);
#pragma unroll
      for (int j = 0; j < EP; ++j) {
        red[0] += g[j];
        red[1] = fmaf(g[j], xh[j], red[1]);
      }
    }
    Sum::run(red, buf, turn);
    const float mg = a.rms ? 0.f : red[0] * a.inv_n, mgx = red[1] * a.inv_n;
    for (int c = threadIdx.x * EP; c < n; c += 1024 * EP) {
      piece(c);
#pragma unroll
      for (int j = 0; j < EP; ++j) z[j] = 0.f;
      if (a.ds) unpack_row<E, M>(load_row<E, M>((const E*)a.ds + r * a.ldds, c, n), c, n, z);
#pragma unroll
      for (int j = 0; j < EP; ++j) z[j] = fmaf(rs, fmaf(-xh[j], mgx, g[j] - mg), z[j]);
      if (a.dx) store_row<E, M>((E*)a.dx + r * a.lddx, c, n, z);
      if (!a.dh) continue;
      if (a.drop.on) drop_piece<E>(a.drop, (uint32_t)r, c, z);
      store_row<E, M>((E*)a.dh + r * a.lddh, c, n, z);
    }
  }
}

// dw and db: one thread per piece of columns and token split.
template <class E, int M>
__global__ __launch_bounds__(256) void norm_back_cols_kernel(NormBackArgs a, int64_t per, int64_t col_blocks,
                                                             int64_t blocks) {
  constexpr int EP = kPiece<E>;
  const int64_t blk = flat_block();
  if (blk >= blocks) return;
  const int n = (int)a.n;
  const int64_t it = blk / col_blocks, i = it / a.S;
  const int64_t c64 = ((blk - it * col_blocks) * 256 + threadIdx.x) * EP;
  if (c64 >= a.n) return;
  const int c = (int)c64;
  const int64_t first = (it - i * a.S) * per, last = std::min<int64_t>(a.T, first + per);
  float dw[EP], db[EP], g[EP], xh[EP];
#pragma unroll
  for (int j = 0; j < EP; ++j) dw[j] = db[j] = 0.f;
  for (int64_t tok = first; tok < last; ++tok) {
    const int64_t r = i * a.T + tok;
    const float mu = a.rms ? 0.f : a.mean[r], rs = a.rstd[r];
    unpack_row<E, M>(load_row<E, M>((const E*)a.dy + r * a.lddy, c, n), c, n, g);
    unpack_row<E, M>(load_row<E, M>((const E*)a.s + r * a.lds, c, n), c, n, xh);
#pragma unroll
    for (int j = 0; j < EP; ++j) {
      dw[j] = fmaf(g[j], (xh[j] - mu) * rs, dw[j]);
      db[j] += g[j];
    }
  }
  float* pw = a.S > 1 ? a.part + it * 2 * n : a.dw + i * a.ldg;
  float* pb = a.S > 1 ? a.part + it * 2 * n + n : a.db + i * a.ldg;
  if (a.dw) store_vec<EP>(pw, c, n, dw);
  if (a.db) store_vec<EP>(pb, c, n, db);
}

// ---- token splits -----------------------------------------------------------------------------

// Sums of a sample's token splits, 64 columns a workgroup: 16 groups of lanes take every 16th
// split, then each column's 16 sums are added in order.
__global__ __launch_bounds__(256) void norm_back_sums_kernel(NormBackArgs a, int64_t col_blocks, int64_t blocks) {
  __shared__ float sums[2][16][64];
  const int64_t blk = flat_block();
  if (blk >= blocks) return;
  const int64_t i = blk / col_blocks;
  const int n = (int)a.n, c0 = (int)(blk - i * col_blocks) * 64, q = (threadIdx.x & 15) * 4, grp = threadIdx.x >> 4;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (!(k ? a.db : a.dw)) continue;
    float t[4] = {0.f, 0.f, 0.f, 0.f}, u[4];
#pragma unroll 4
    for (int sp = grp; sp < a.S; sp += 16) {
      load_vec<4>(a.part + ((i * a.S + sp) * 2 + k) * n, 0, c0 + q, n, 0.f, u);
#pragma unroll
      for (int j = 0; j < 4; ++j) t[j] += u[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[k][grp][q + j] = t[j];
  }
  __syncthreads();
  const int k = threadIdx.x >> 6, c = c0 + (threadIdx.x & 63);
  float* out = k == 0 ? a.dw : a.db;
  if (k > 1 || !out || c >= n) return;
  float t = 0.f;
#pragma unroll
  for (int j = 0; j < 16; ++j) t += sums[k][j][threadIdx.x & 63];
  out[i * a.ldg + c] = t;
}

hipError_t launch_norm_back_sums(const NormBackArgs& a, hipStream_t st) {
  const int64_t cb = ceil_div(a.n, 64), blocks = a.B * cb;
  DPRC_LAUNCH(norm_back_sums_kernel, flat_grid(blocks), dim3(256), 0, st, a, cb, blocks);
  return hipGetLastError();
}

// ---- launch -------------------------------------------------------------------------------------

constexpr int64_t kNormBackLong = 8192;

// How a width is dealt out: TPR threads of C columns.  Small and few workgroups do best where every
// thread has two rows on their way (8 x 4096 x 2048 bf16 with ds, dropout and dh: 131 us with 256
// workgroups of <128, 16>, 140 with 512, 137 with 512 of <256, 8>, 187 with 256 of <256, 8> and one
// row ahead); up to 1024 columns <., 8> with 512 (n = 512: 37 us against 40 with 16 columns).
struct BackLayout {
  int tpr, cols;
};
static BackLayout back_layout(int64_t n, bool bf16) {
  if (n > 4096) return {512, 16};
  if (n > 2048) return {512, 8};
  if (n > 1024) return bf16 ? BackLayout{128, 16} : BackLayout{256, 8};
  int tpr = 8;
  while (8 * tpr < n) tpr *= 2;
  return {tpr, 8};
}
// rows that a workgroup works on at a time
static int64_t rows_at_once(int64_t n, bool bf16) {
  return n > kNormBackLong ? 1 : std::max(1, 256 / back_layout(n, bf16).tpr);
}

// Token splits of a sample: at least four rounds of rows each, and so many that the workgroups
// number 256, or 512 where that is better (bf16 rows of up to 1024 columns; fewer than 16 rounds a
// workgroup, where their latency is what counts: 16 x 333 x 1111 took 25 us with 448, 33 with 256).
int norm_back_splits(int64_t B, int64_t T, int64_t n, bool bf16) {
  const int64_t at_once = rows_at_once(n, bf16), rounds = ceil_div(T, at_once);
  const int64_t blocks = (bf16 && n <= 1024) || B * rounds < 16 * 256 ? 512 : 256;
  const int64_t S = std::max<int64_t>(1, std::min<int64_t>(ceil_div(blocks, B), rounds / 4));
  return (int)ceil_div(rounds, ceil_div(rounds, S));
}

template <class E, int M>
static void launch_norm_back_of(const NormBackArgs& a, hipStream_t st) {
  const int64_t n = a.n, at_once = rows_at_once(n, a.bf16);
  const int64_t per = ceil_div(ceil_div(a.T, at_once), (int64_t)a.S) * at_once;
  if (n > kNormBackLong) {
    if (a.dw || a.db) {
      const int64_t cb = ceil_div(n, 256 * kPiece<E>), blocks = a.B * a.S * cb;
      DPRC_LAUNCH((norm_back_cols_kernel<E, M>), flat_grid(blocks), dim3(256), 0, st, a, per, cb, blocks);
    }
    if (a.dx || a.dh) {
      const int64_t blocks = std::min<int64_t>(a.B * a.T, 512);
      DPRC_LAUNCH((norm_back_rows_kernel<E, M>), dim3((unsigned)blocks), dim3(1024), 0, st, a);
    }
    return;
  }
  // Many samples of fewer rows than a workgroup takes at a time: a sample for each row group.
  const bool solo = a.T < at_once && a.B > 512;
  const int64_t items = solo ? ceil_div(a.B, at_once) : a.B * a.S;
  const int64_t blocks = std::min<int64_t>(items, 1024);
  auto go = [&](auto kernel, int block) { DPRC_LAUNCH(kernel, dim3((unsigned)blocks), dim3(block), 0, st, a, per, items); };
  auto pick = [&](auto tpr, auto cols) {
    constexpr int TPR = decltype(tpr)::value, C = decltype(cols)::value;
    if constexpr (TPR < 256) {
      if (solo) return go(norm_back_kernel<E, M, TPR, C, true>, 256);
    }
    go(norm_back_kernel<E, M, TPR, C, false>, TPR > 256 ? TPR : 256);
  };
  using std::integral_constant;
  const integral_constant<int, 8> c8;
  const integral_constant<int, 16> c16;
  const BackLayout lay = back_layout(n, a.bf16);
  if (lay.tpr == 8) return pick(integral_constant<int, 8>(), c8);
  if constexpr (M != kTiny) {
    if (lay.tpr == 16) return pick(integral_constant<int, 16>(), c8);
    if (lay.tpr == 32) return pick(integral_constant<int, 32>(), c8);
    if (lay.tpr == 64) return pick(integral_constant<int, 64>(), c8);
    if (lay.tpr == 128 && lay.cols == 8) return pick(integral_constant<int, 128>(), c8);
    if constexpr (sizeof(E) == 2) {
      if (lay.tpr == 128) return pick(integral_constant<int, 128>(), c16);
    } else {
      if (lay.tpr == 256) return pick(integral_constant<int, 256>(), c8);
    }
    if (lay.cols == 8) return pick(integral_constant<int, 512>(), c8);
    pick(integral_constant<int, 512>(), c16);
  }
}

template <class E>
static void launch_norm_back_width(const NormBackArgs& a, hipStream_t st) {
  if (a.n < kPiece<E>) launch_norm_back_of<E, kTiny>(a, st);
  else if (a.n % kPiece<E> == 0) launch_norm_back_of<E, kWhole>(a, st);
  else launch_norm_back_of<E, kTail>(a, st);
}

hipError_t launch_norm_back(const NormBackArgs& a, hipStream_t st) {
  if (a.bf16) launch_norm_back_width<uint16_t>(a, st);
  else launch_norm_back_width<float>(a, st);
  return hipGetLastError();
}

}  // namespace dprc
