// Backward pass of dropout, residual sum and norm, with the weight's and bias's gradient of every
// sample by itself.
//
// With xh = (s - mu) rstd and g = dy w: dx = ds + rstd (g - mean(g) - xh mean(g xh)), dh = m dx, and for
// each sample dw = sum dy xh, db = sum dy.  Everything is fp32 but s itself, which the forward pass rounded
// to the tensors' type after its statistics were taken (s in fp32 would add as much traffic as dy
// and dx have in bf16): xh is off by that rounding times rstd.
//
// Bounded by memory: one pass over dy, s and ds writes dx and dh and sums dw and db on the way.  8 x 4096 x
// 2048 bf16 with everything takes 132 to 134 us, 5.1 TB/s, and 4 us to join the parts of dw and db; HBM
// carries 403 MB in and 273 MB out, no more than the tensors are.
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

// Which of ds and dh a call has: known at compile time, because the number of loads and stores of a
// round then is, and with it how many may still be under way when a row is waited for.  (Where a
// branch may skip a store, the compiler has to assume that it did, and waits for later loads.)
// kAny takes any set, dx = null too.
enum : int { kDs = 1, kDh = 2, kAny = 4 };

// TPR threads hold a row as in the forward pass, 256 / TPR row groups a workgroup; a round is a row for each
// of them.  The samples' rounds, laid end to end, are dealt out evenly (BackSplit), so a workgroup walks
// one sample's rounds or parts of several; each thread sums dw and db of its own columns in
// registers over a sample's rounds, the groups' sums meet in lanes and in LDS, and go to dw and db, or as a
// part of them to the workspace where other workgroups have the sample's other rounds.  With
// SOLO (samples shorter than a round) every group has samples of its own, and nothing is combined.
template <class E, int M, int TPR, int C, bool SOLO, int FL>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_back_kernel(NormBackArgs a) {
  constexpr int EP = kPiece<E>, V = C / EP, BLK = TPR > 256 ? TPR : 256, RPB = BLK / TPR;
  constexpr int G = SOLO ? 1 : (TPR < 64 ? BLK / 64 : RPB);      // sums to combine in LDS
  constexpr int kAhead = V <= 2 ? 2 : 1;                          // rows loading ahead
  // Rows of 1024 threads have 128 registers each, too few for dw and db, which lie in LDS (every thread its
  // own words), for the weights and for a row ahead (bf16 does without one too, in 91 to 122 registers).
  // 4096 x 16384 bf16 (dy, s, dx, dw, db) takes 104 to 109 us and 2048 x 16384 fp32 98 to 101, where two passes
  // over the rows took 168 and 167 (as many elements in rows of 9000: 137 and 100 against 182 and 164).
  // With more tensors, us (each once at 5.4 TB/s: 99, 99, 124):
  //            ds     dh     both
  //   bf16    130    133     157
  //   fp32    128    147     178     (28 registers spill with dh, 54 with both)
  constexpr bool kLean = TPR == 1024;
  typedef RowSum<TPR, 2, BLK> Sum;
  __shared__ typename Sum::Buffer buf;
  __shared__ float acc[2][kLean ? C : 1][kLean ? TPR : 1];
  __shared__ float comb[G > 1 ? G - 1 : 1][2][G > 1 ? C : 1][G > 1 ? TPR : 1];
  int turn = 0;
  const int t = threadIdx.x % TPR, rg = threadIdx.x / TPR, n = (int)a.n;
  const bool has_ds = FL & kAny ? a.ds != nullptr : (FL & kDs) != 0;
  const bool has_dh = FL & kAny ? a.dh != nullptr : (FL & kDh) != 0;
  const bool has_dx = FL & kAny ? a.dx != nullptr : true;
  const bool grads = a.dw || a.db;
  const float* mean = a.rms ? a.rstd : a.mean;                    // loaded either way
  // rows, and bytes, from the first row group's row to this one's
  const uint32_t apart = (uint32_t)(rg * (SOLO ? a.T : 1));
  const uint32_t gy = (uint32_t)(apart * a.lddy * sizeof(E)), gs = (uint32_t)(apart * a.lds * sizeof(E));
  const uint32_t gd = (uint32_t)(apart * a.ldds * sizeof(E));

  float w[C];
  auto load_w = [&](int v) { load_vec<EP>(a.w, a.wbf16, piece_col<E, M>((v * TPR + t) * EP, n), n, 1.f, w + v * EP); };
  if (!kLean)
#pragma unroll
    for (int v = 0; v < V; ++v) load_w(v);

  // this workgroup's samples (SOLO: every gridDim.x-th RPB of them) and rounds
  const BackSplit& sp = a.split;
  const int64_t q0 = SOLO ? 0 : sp.begin(blockIdx.x), q1 = SOLO ? 0 : sp.begin(blockIdx.x + 1);
  const int64_t i_first = SOLO ? (int64_t)blockIdx.x * RPB : q0 / sp.rounds, i_step = SOLO ? (int64_t)gridDim.x * RPB : 1;
  const int64_t i_end = SOLO ? a.B : (q1 + sp.rounds - 1) / sp.rounds;
  for (int64_t i0 = i_first; i0 < i_end; i0 += i_step) {
    const int64_t i = i0 + (SOLO ? rg : 0);
    // its tokens, kTokStep of them a round: the rounds in which every row group has a row, then the others
    constexpr int kTokStep = SOLO ? 1 : RPB;
    const int64_t first = SOLO ? 0 : std::max<int64_t>(q0 - i * sp.rounds, 0) * RPB;
    const int64_t last = SOLO ? a.T : std::min<int64_t>((q1 - i * sp.rounds) * RPB, a.T);
    const int64_t whole = kLean ? 0 : SOLO ? (i0 + RPB <= a.B ? a.T : 0) : (last - first) / RPB;
    const int64_t rest = SOLO ? a.T - whole : (last - first + RPB - 1) / RPB - whole;
    int64_t tok = first;

    struct Row {
      uint4 dy[V], s[V], ds[V];
      float mu, rstd;
    };
    auto load = [&](Row& x, int64_t token, bool live) {
      const int64_t r0 = i0 * a.T + token;
      const char* py = (const char*)a.dy + r0 * a.lddy * sizeof(E);
      const char* ps = (const char*)a.s + r0 * a.lds * sizeof(E);
      const char* pd = (const char*)a.ds + r0 * a.ldds * sizeof(E);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + t) * EP;
        x.dy[v] = load_at<E, M>(py, live ? gy : 0u, c, n);
        x.s[v] = load_at<E, M>(ps, live ? gs : 0u, c, n);
        if (has_ds) x.ds[v] = load_at<E, M>(pd, live ? gd : 0u, c, n);
      }
      x.mu = (mean + r0)[live ? apart : 0u];
      x.rstd = (a.rstd + r0)[live ? apart : 0u];
    };
    float dw[C], db[C];
#pragma unroll
    for (int k = 0; k < C; ++k) {
      dw[k] = db[k] = 0.f;
      if constexpr (kLean) acc[0][k][t] = acc[1][k][t] = 0.f;
    }
    // one round: this row's sums, the loads of the row kAhead rounds on (of `more` whole rounds), the
    // mask, then the outputs.  PART: only rows that are `live`.
    auto round = [&](Row& x, auto part, int64_t more, bool live) {
      constexpr bool PART = decltype(part)::value;
      float g[C], xh[C], z[C], red[2] = {0.f, 0.f};
      const float rs = x.rstd, mu = a.rms ? 0.f : x.mu;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + t) * EP, cc = piece_col<E, M>(c, n);
        if (kLean) load_w(v);
        unpack<E>(x.dy[v], g + v * EP);
        unpack<E>(x.s[v], xh + v * EP);
        if (has_ds) unpack<E>(x.ds[v], z + v * EP);
#pragma unroll
        for (int j = 0; j < EP; ++j) {
          const int k = v * EP + j;
          if (!has_ds) z[k] = 0.f;
          if (PART) g[k] = live ? g[k] : 0.f;
          xh[k] = (xh[k] - mu) * rs;
          if constexpr (kLean) {
            acc[0][k][t] = fmaf(g[k], xh[k], acc[0][k][t]);
            acc[1][k][t] += g[k];
          } else {
            db[k] += g[k];
            dw[k] = fmaf(g[k], PART && !live ? 0.f : xh[k], dw[k]);
          }
          g[k] *= w[k];
          const float own = owns<M>(c, cc, j, n) ? g[k] : 0.f;
          red[0] += own;
          red[1] = fmaf(own, owns<M>(c, cc, j, n) ? xh[k] : 0.f, red[1]);
        }
      }
      const int64_t r0 = i0 * a.T + tok;
      if (!PART) load(x, tok + std::min<int64_t>(kAhead, more - 1) * kTokStep, true);
      u32x4 mask[V];
      const bool drop = has_dh && a.drop.on;
      if (drop)
#pragma unroll
        for (int v = 0; v < V; ++v)
          mask[v] = drop_words<E>(a.drop, (uint32_t)r0 + apart, piece_col<E, M>((v * TPR + t) * EP, n), n);
      Sum::run(red, buf, turn);
      const float mg = a.rms ? 0.f : red[0] * a.inv_n, mgx = red[1] * a.inv_n;
      char* px = (char*)a.dx + r0 * a.lddx * sizeof(E);
      char* ph = (char*)a.dh + r0 * a.lddh * sizeof(E);
      if (!PART || live)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int c = (v * TPR + t) * EP;
#pragma unroll
          for (int k = v * EP; k < v * EP + EP; ++k) z[k] = fmaf(rs, fmaf(-xh[k], mgx, g[k] - mg), z[k]);
          if (has_dx) store_at<E, M>(px, (uint32_t)(apart * a.lddx * sizeof(E)), c, n, z + v * EP);
          if (!has_dh) continue;
          if (drop) drop_apply<E>(a.drop, mask[v], z + v * EP);
          store_at<E, M>(ph, (uint32_t)(apart * a.lddh * sizeof(E)), c, n, z + v * EP);
        }
      tok += kTokStep;
    };
    if (whole > 0) {
      Row ring[kAhead];
#pragma unroll
      for (int q = 0; q < kAhead; ++q) load(ring[q], first + std::min<int64_t>(q, whole - 1) * kTokStep, true);
      for (int64_t left = whole; left > 0; left -= kAhead)
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
          if (q < left) round(ring[q], std::false_type{}, left - q, true);
    }
    for (int64_t k = 0; k < rest; ++k) {
      const bool live = SOLO ? i < a.B : tok + rg < last;
      Row x;
      load(x, tok, live);
      round(x, std::true_type{}, 0, live);
    }
    if (!grads) continue;
    if constexpr (kLean)
#pragma unroll
      for (int k = 0; k < C; ++k) {
        dw[k] = acc[0][k][t];
        db[k] = acc[1][k][t];
      }
    if (!SOLO) {
      if (TPR < 64)
#pragma unroll
        for (int k = 0; k < C; ++k) {
          dw[k] = group_sum<TPR>(dw[k]);
          db[k] = group_sum<TPR>(db[k]);
        }
      if constexpr (G > 1) {
        const int grp = TPR < 64 ? threadIdx.x >> 6 : rg;
        __syncthreads();                                  // the sample before has read its sums
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
    float* pw = a.dw ? a.dw + i * a.ldg : nullptr;
    float* pb = a.db ? a.db + i * a.ldg : nullptr;
    if (!SOLO && (first > 0 || last < a.T)) {             // part of a sample: slot blockIdx.x + i is nobody else's
      float* part = a.part + (blockIdx.x + i) * 2 * n;
      pw = a.dw ? part : nullptr;
      pb = a.db ? part + n : nullptr;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * EP;
      if (c >= n) continue;
      if (pw) store_vec<EP>(pw, piece_col<E, M>(c, n), n, dw + v * EP);
      if (pb) store_vec<EP>(pb, piece_col<E, M>(c, n), n, db + v * EP);
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
      if (a.drop.on) drop_piece<E>(a.drop, (uint32_t)r, c, n, z);
      store_row<E, M>((E*)a.dh + r * a.lddh, c, n, z);
    }
  }
}

// dw and db: one thread per piece of columns and workgroup's share of the rounds (at_once rows each).
template <class E, int M>
__global__ __launch_bounds__(64) void norm_back_cols_kernel(NormBackArgs a, int at_once, int64_t col_blocks) {
  constexpr int EP = kPiece<E>, kRows = 4;
  const BackSplit& sp = a.split;
  const int64_t blk = flat_block() / col_blocks, c64 = ((flat_block() - blk * col_blocks) * 64 + threadIdx.x) * EP;
  if (blk >= sp.blocks || c64 >= a.n) return;
  const int c = (int)c64, n = (int)a.n;
  const int64_t q0 = sp.begin(blk), q1 = sp.begin(blk + 1);
  for (int64_t i = q0 / sp.rounds; i * sp.rounds < q1; ++i) {
    const int64_t first = std::max<int64_t>(q0 - i * sp.rounds, 0) * at_once;
    const int64_t last = std::min<int64_t>((q1 - i * sp.rounds) * at_once, a.T);
    float dw[EP], db[EP], g[EP], xh[EP];
#pragma unroll
    for (int j = 0; j < EP; ++j) dw[j] = db[j] = 0.f;
    for (int64_t t0 = first; t0 < last; t0 += kRows) {
      uint4 dy[kRows], s[kRows];
      float mu[kRows], rs[kRows];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int64_t r = i * a.T + std::min<int64_t>(t0 + k, last - 1);
        dy[k] = load_row<E, M>((const E*)a.dy + r * a.lddy, c, n);
        s[k] = load_row<E, M>((const E*)a.s + r * a.lds, c, n);
        mu[k] = a.rms ? 0.f : a.mean[r];
        rs[k] = a.rstd[r];
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        if (t0 + k >= last) continue;
        unpack_row<E, M>(dy[k], c, n, g);
        unpack_row<E, M>(s[k], c, n, xh);
#pragma unroll
        for (int j = 0; j < EP; ++j) {
          dw[j] = fmaf(g[j], (xh[j] - mu[k]) * rs[k], dw[j]);
          db[j] += g[j];
        }
      }
    }
    float* pw = a.dw ? a.dw + i * a.ldg : nullptr;
    float* pb = a.db ? a.db + i * a.ldg : nullptr;
    if (first > 0 || last < a.T) {
      float* part = a.part + (blk + i) * 2 * n;
      pw = a.dw ? part : nullptr;
      pb = a.db ? part + n : nullptr;
    }
    if (pw) store_vec<EP>(pw, c, n, dw);
    if (pb) store_vec<EP>(pb, c, n, db);
  }
}

// ---- sums of parts ----------------------------------------------------------------------------------

// dw and db of the samples whose rounds several workgroups had, 64 columns a workgroup: 16 groups of 16 lanes
// (four columns each) take every 16th part, all loads of four rounds first; then each column's
// 16 sums are added in order.
__global__ __launch_bounds__(256) void norm_back_sums_kernel(NormBackArgs a, int64_t col_blocks, int64_t blocks) {
  __shared__ float sums[2][16][64];
  const int64_t blk = flat_block();
  if (blk >= blocks) return;
  const int64_t i = blk / col_blocks, b0 = a.split.block_of(i * a.split.rounds);
  const int S = (int)(a.split.block_of((i + 1) * a.split.rounds - 1) - b0) + 1;
  if (S == 1) return;                                     // written whole
  const int n = (int)a.n, c0 = (int)(blk - i * col_blocks) * 64, q = (threadIdx.x & 15) * 4, grp = threadIdx.x >> 4;
  const int col = min(c0 + q, max(n - 4, 0)), skip = c0 + q - col;       // the last piece: `skip` columns to the left
  const float* part = a.part + (b0 + i) * 2 * n + col;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (!(k ? a.db : a.dw)) continue;
    float t[4] = {0.f, 0.f, 0.f, 0.f};
    if (n < 4) {
      for (int sp = grp; sp < S; sp += 16)
        for (int m = 0; m < n; ++m) t[m] += part[((int64_t)sp * 2 + k) * n + m];
    } else for (int sp = grp; sp < S; sp += 64) {
      float u[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) unpack<float>(load_piece(part + ((int64_t)min(sp + 16 * j, S - 1) * 2 + k) * n), u[j]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (sp + 16 * j < S)
#pragma unroll
          for (int m = 0; m < 4; ++m) t[m] += u[j][m];
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
      if (m >= skip) sums[k][grp][q + m - skip] = t[m];
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

// ---- launch -------------------------------------------------------------------------------------

// columns that a workgroup of 1024 threads holds; longer rows are read twice
constexpr int64_t kNormBackLong = 16384;

NormBackPlan norm_back_plan(int64_t B, int64_t T, int64_t n, int64_t elem_bytes, int tensors) {
  const bool wide = n > kNormBackLong;
  NormBackPlan p{};
  p.tpr = n > 8192 ? 1024 : threads_per_row(n);
  p.at_once = wide ? 1 : std::max(1, 256 / p.tpr);
  p.solo = T < p.at_once && B > 512;
  BackSplit& sp = p.split;
  sp.rounds = ceil_div(T, (int64_t)p.at_once);
  sp.total = B * sp.rounds;
  // Few rounds a sample, or many samples: none is cut.  (A cut costs a launch to join the parts, 3.5 us on
  // the GPU and as much on the host, as the four or five rounds that it saves: 4 x 12 x 2048 took 12.4 us
  // whole and 9.8 cut, 4 x 8 x 2048 9.2 and 9.8.  Of many samples whole ones gain where they come out even over
  // the workgroups, and lose where not, samples x 300 x 512 bf16: 1023 cut 207 us; whole 1024 194, 1025 233, 1280
  // 294, 1500 298, 2048 382, 2049 417.)
  sp.samples = sp.rounds <= 12 || B >= 1024 ? B : 0;
  if (p.solo) sp.blocks = std::min<int64_t>(ceil_div(B, (int64_t)p.at_once), 1024);
  else if (sp.samples) sp.blocks = std::min<int64_t>(B, 1024);
  // two rows of loads in flight, of more than 8192 columns one
  else sp.blocks = std::min<int64_t>(streaming_blocks((n > 8192 ? 1 : 2) * tensors * p.at_once * n * elem_bytes),
                                     std::max<int64_t>(B, sp.total / 4));
  p.parts = sp.samples ? 0 : sp.blocks + B;
  return p;
}

template <class E, int M>
static void launch_norm_back_long(const NormBackArgs& a, const NormBackPlan& p, hipStream_t st) {
  if (a.dw || a.db) {
    const int64_t cb = ceil_div(a.n, 64 * kPiece<E>);
    DPRC_LAUNCH((norm_back_cols_kernel<E, M>), flat_grid(a.split.blocks * cb), dim3(64), 0, st, a, p.at_once, cb);
  }
  if (a.dx || a.dh) {
    const int64_t blocks = std::min<int64_t>(a.B * a.T, 512);
    DPRC_LAUNCH((norm_back_rows_kernel<E, M>), dim3((unsigned)blocks), dim3(1024), 0, st, a);
  }
}

template <class E, int M>
static void launch_norm_back_of(const NormBackArgs& a, const NormBackPlan& p, hipStream_t st) {
  auto go = [&](auto kernel, int block) { DPRC_LAUNCH(kernel, dim3((unsigned)p.split.blocks), dim3(block), 0, st, a); };
  auto pick = [&](auto tpr, auto cols) {
    constexpr int TPR = decltype(tpr)::value, C = decltype(cols)::value, BLK = TPR > 256 ? TPR : 256;
    if constexpr (TPR < 256) {
      if (p.solo) return go(norm_back_kernel<E, M, TPR, C, true, kAny>, BLK);
    }
    if constexpr (M != kTiny) {
      if (a.dx && a.ds && a.dh) return go(norm_back_kernel<E, M, TPR, C, false, kDs | kDh>, BLK);
      if (a.dx && a.ds) return go(norm_back_kernel<E, M, TPR, C, false, kDs>, BLK);
      if (a.dx && a.dh) return go(norm_back_kernel<E, M, TPR, C, false, kDh>, BLK);
      if (a.dx) return go(norm_back_kernel<E, M, TPR, C, false, 0>, BLK);
    }
    go(norm_back_kernel<E, M, TPR, C, false, kAny>, BLK);
  };
  using std::integral_constant;
  const integral_constant<int, 8> c8;
  if (p.tpr == 8) return pick(integral_constant<int, 8>(), c8);
  if constexpr (M != kTiny) {
    if (p.tpr == 16) return pick(integral_constant<int, 16>(), c8);
    if (p.tpr == 32) return pick(integral_constant<int, 32>(), c8);
    if (p.tpr == 64) return pick(integral_constant<int, 64>(), c8);
    if (p.tpr == 128) return pick(integral_constant<int, 128>(), c8);
    if (p.tpr == 256) return pick(integral_constant<int, 256>(), c8);
    if (a.n <= 4096) return pick(integral_constant<int, 512>(), c8);
    if (p.tpr == 512) return pick(integral_constant<int, 512>(), integral_constant<int, 16>());
    pick(integral_constant<int, 1024>(), integral_constant<int, 16>());
  }
}

template <class E>
static void launch_norm_back_width(const NormBackArgs& a, const NormBackPlan& p, hipStream_t st) {
  constexpr int EP = kPiece<E>;
  // also rows so far apart that those of a workgroup's round leave 32-bit offsets go the long rows' way
  const int64_t apart = p.at_once * (p.solo ? a.T : 1) * (int64_t)sizeof(E);
  if (a.n > kNormBackLong || apart * std::max({a.lddy, a.lds, a.ldds, a.lddx, a.lddh}) >= ((int64_t)1 << 31)) {
    if (a.n < EP) launch_norm_back_long<E, kTiny>(a, p, st);
    else if (a.n % EP == 0) launch_norm_back_long<E, kWhole>(a, p, st);
    else launch_norm_back_long<E, kTail>(a, p, st);
  } else if (a.n < EP) {
    launch_norm_back_of<E, kTiny>(a, p, st);
  } else {
    launch_norm_back_of<E, kWide>(a, p, st);
  }
}

hipError_t launch_norm_back(const NormBackArgs& a, const NormBackPlan& p, hipStream_t st) {
  if (a.bf16) launch_norm_back_width<uint16_t>(a, p, st);
  else launch_norm_back_width<float>(a, p, st);
  if (p.parts > 0 && (a.dw || a.db)) {
    const int64_t cb = ceil_div(a.n, 64), blocks = a.B * cb;
    DPRC_LAUNCH(norm_back_sums_kernel, flat_grid(blocks), dim3(256), 0, st, a, cb, blocks);
  }
  return hipGetLastError();
}

}  // namespace dprc
