// Dropout, residual sum and norm of token rows (forward).
//
// Bounded by memory: a row is read once and held in registers from the sum through its mean, its
// variance about that mean (two sums one after the other: mean(s^2) - mu^2 would cancel) and the
// output.  Everything is fp32; y and s are rounded once, y from the unrounded s.  8 x 4096 x 2048 bf16
// with residual, dropout, statistics and bias takes 91 us, 5.9 TB/s (a copy reaches 5.4); one row of
// 2048 takes 2.7 us, a launch's latency.
#include <algorithm>
#include "device.hpp"
#include "kernels.hpp"
#include "rows.hpp"

namespace dprc {

// What a call has besides x and y: known at compile time, because the number of loads and stores of a
// row then is, and with it how many may still be under way when the next row is waited for.  kAny takes
// any set.
enum : int { kRes = 1, kSum = 2, kStats = 4, kAny = 8 };

// TPR threads hold a row of at most TPR * C columns, C each; a workgroup of max(256, TPR)
// threads works on 256 / TPR rows at a time and walks the rows with the grid, the next rows'
// pieces loading while this one is reduced.  Weight and bias stay in registers for all rows.
template <class E, int M, int TPR, int C, int FL, bool NT = false>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_kernel(NormArgs a) {
  constexpr int EP = kPiece<E>, V = C / EP, BLK = TPR > 256 ? TPR : 256, RPB = BLK / TPR;
  constexpr bool kHold = TPR < 1024;
  constexpr int kAhead = C == 8 ? 2 : 1;                          // rows loading ahead
  // fp32 rows of 1024 threads: 128 registers are too few for a row ahead (2048 x 16384 with residual and
  // sum 103 us without, 113 with it; bf16 4096 x 16384, which has them, 94 with it), and for the row itself:
  // without one ahead these instances still spill 10 to 30 registers, bf16 ones none
  constexpr bool kLean = TPR == 1024 && sizeof(E) == 4;
  typedef RowSum<TPR, 1, BLK> Sum;
  __shared__ typename Sum::Buffer buf;
  int turn = 0;
  const int t = threadIdx.x % TPR, rg = threadIdx.x / TPR, n = (int)a.n;
  const bool has_res = FL & kAny ? a.res != nullptr : (FL & kRes) != 0;
  const bool has_sum = FL & kAny ? a.sum != nullptr : (FL & kSum) != 0;
  const int64_t step = (int64_t)gridDim.x * RPB, r_first = (int64_t)blockIdx.x * RPB;
  // bytes from the first of the workgroup's rows to this thread's
  const uint32_t gx = (uint32_t)(rg * a.ldx * sizeof(E)), gr = (uint32_t)(rg * a.ldr * sizeof(E));
  const uint32_t gs = (uint32_t)(rg * a.lds * sizeof(E)), gy = (uint32_t)(rg * a.ldy * sizeof(E));

  struct Row {
    uint4 x[V], z[V];
  };
  auto load = [&](Row& q, int64_t r0, bool live) {
    const char* px = (const char*)a.x + r0 * a.ldx * sizeof(E);
    const char* pr = (const char*)a.res + r0 * a.ldr * sizeof(E);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (v * TPR + t) * EP;
      q.x[v] = load_at<E, M, NT>(px, live ? gx : 0u, c, n);
      if (has_res) q.z[v] = load_at<E, M, NT>(pr, live ? gr : 0u, c, n);
    }
  };
  float w[C], b[C];
  auto load_wb = [&](int v) {
    const int c = piece_col<E, M>((v * TPR + t) * EP, n);
    load_vec<EP>(a.w, a.wbf16, c, n, 1.f, w + v * EP);
    load_vec<EP>(a.b, a.wbf16, c, n, 0.f, b + v * EP);
  };
  int64_t r0 = r_first;
  // a round: the rows from r0 on, and the loads of those `ahead` rounds on.  PART: rows that are `live`.
  auto round = [&](Row& q, auto part, int64_t ahead, bool live) {
    constexpr bool PART = decltype(part)::value;
    float s[C], u[EP], red[1] = {0.f}, mu = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      unpack<E>(q.x[v], s + v * EP);
      if (a.drop.on)
        drop_piece<E>(a.drop, (uint32_t)r0 + (uint32_t)rg, piece_col<E, M>((v * TPR + t) * EP, n), n, s + v * EP);
      if (!has_res) continue;
      unpack<E>(q.z[v], u);
#pragma unroll
      for (int j = 0; j < EP; ++j) s[v * EP + j] += u[j];
    }
    if (!PART) load(q, r0 + ahead * step, true);
    if (!a.rms) {
#pragma unroll
      for (int k = 0; k < C; ++k) {
        const int c = (k / EP * TPR + t) * EP;
        red[0] += owns<M>(c, piece_col<E, M>(c, n), k % EP, n) ? s[k] : 0.f;
      }
      Sum::run(red, buf, turn);
      mu = red[0] * a.inv_n;
      red[0] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < C; ++k) {
      const int c = (k / EP * TPR + t) * EP;
      const float d = owns<M>(c, piece_col<E, M>(c, n), k % EP, n) ? s[k] - mu : 0.f;
      red[0] = fmaf(d, d, red[0]);
    }
    Sum::run(red, buf, turn);
    const float rstd = 1.f / sqrtf(fmaf(red[0], a.inv_n, a.eps));
    char* ps = (char*)a.sum + r0 * a.lds * sizeof(E);
    char* py = (char*)a.y + r0 * a.ldy * sizeof(E);
    if (!PART || live) {
      if (FL & kAny) {
        if (t == 0 && a.mean) a.mean[r0 + rg] = mu;
        if (t == 0 && a.rstd) a.rstd[r0 + rg] = rstd;
      } else if (FL & kStats) {                                   // by all of the row's threads
        (a.rms ? a.rstd : a.mean)[r0 + rg] = a.rms ? rstd : mu;
        a.rstd[r0 + rg] = rstd;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + t) * EP;
        if (has_sum) store_at<E, M, NT>(ps, gs, c, n, s + v * EP);
        if (!kHold) load_wb(v);
#pragma unroll
        for (int j = 0; j < EP; ++j) u[j] = fmaf((s[v * EP + j] - mu) * rstd, w[v * EP + j], b[v * EP + j]);
        store_at<E, M, NT>(py, gy, c, n, u);
      }
    }
    r0 += step;
  };
  // the rounds in which every row group has a row; then, for one workgroup, the last rows (or, without a
  // row ahead, all)
  const int64_t whole = kLean || a.rows - r_first < RPB ? 0 : (a.rows - r_first - RPB) / step + 1;
  Row ring[kAhead];
  if (whole > 0)
#pragma unroll
    for (int q = 0; q < kAhead; ++q) load(ring[q], r_first + std::min<int64_t>(q, whole - 1) * step, true);
  if (kHold)
#pragma unroll
    for (int v = 0; v < V; ++v) load_wb(v);
  for (int64_t left = whole; left > 0; left -= kAhead)
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
      if (q < left) round(ring[q], std::false_type{}, std::min<int64_t>(kAhead, left - q - 1), true);
  while ((RPB > 1 || kLean) && r0 < a.rows) {
    const bool live = r0 + rg < a.rows;
    load(ring[0], r0, live);
    round(ring[0], std::true_type{}, 0, live);
  }
}

// Rows longer than a workgroup's registers hold: three passes over the row (mean, variance,
// output), the sum made again in each.
template <class E, int M>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  constexpr int EP = kPiece<E>;
  typedef RowSum<1024, 1, 1024> Sum;
  __shared__ typename Sum::Buffer buf;
  int turn = 0;
  const int n = (int)a.n;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    auto piece = [&](int c, float* s) {
      float u[EP];
      unpack_row<E, M>(load_row<E, M>((const E*)a.x + r * a.ldx, c, n), c, n, s);
      if (a.drop.on) drop_piece<E>(a.drop, (uint32_t)r, c, n, s);
      if (a.res) {
        unpack_row<E, M>(load_row<E, M>((const E*)a.res + r * a.ldr, c, n), c, n, u);
#pragma unroll
        for (int j = 0; j < EP; ++j) s[j] += u[j];
      }
    };
    float s[EP], w[EP], b[EP], red[1] = {0.f}, mu = 0.f;
    if (!a.rms) {
      for (int c = threadIdx.x * EP; c < n; c += 1024 * EP) {
        piece(c, s);
#pragma unroll
        for (int j = 0; j < EP; ++j) red[0] += (M == kWhole || c + j < n) ? s[j] : 0.f;
      }
      Sum::run(red, buf, turn);
      mu = red[0] * a.inv_n;
      red[0] = 0.f;
    }
    for (int c = threadIdx.x * EP; c < n; c += 1024 * EP) {
      piece(c, s);
#pragma unroll
      for (int j = 0; j < EP; ++j) {
        const float d = (M == kWhole || c + j < n) ? s[j] - mu : 0.f;
        red[0] = fmaf(d, d, red[0]);
      }
    }
    Sum::run(red, buf, turn);
    const float rstd = 1.f / sqrtf(fmaf(red[0], a.inv_n, a.eps));
    for (int c = threadIdx.x * EP; c < n; c += 1024 * EP) {
      piece(c, s);
      if (a.sum) store_row<E, M>((E*)a.sum + r * a.lds, c, n, s);
      load_vec<EP>(a.w, a.wbf16, c, n, 1.f, w);
      load_vec<EP>(a.b, a.wbf16, c, n, 0.f, b);
#pragma unroll
      for (int j = 0; j < EP; ++j) s[j] = fmaf((s[j] - mu) * rstd, w[j], b[j]);
      store_row<E, M>((E*)a.y + r * a.ldy, c, n, s);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mu;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
}

constexpr int64_t kNormLong = 16384;

template <class E, int M>
static void launch_norm_of(const NormArgs& a, hipStream_t st) {
  const int64_t n = a.n;
  auto go = [&](auto tpr, auto cols) {
    constexpr int TPR = decltype(tpr)::value, C = decltype(cols)::value, BLK = TPR > 256 ? TPR : 256, RPB = BLK / TPR;
    const int64_t ahead = (C == 8 ? 2 : 1) * (a.res ? 2 : 1) * RPB * n * (int64_t)sizeof(E);
    const int64_t blocks = std::min<int64_t>(ceil_div(a.rows, RPB), streaming_blocks(ahead));
    auto launch = [&](auto kernel) { DPRC_LAUNCH(kernel, dim3((unsigned)blocks), dim3(BLK), 0, st, a); };
    const bool stats = a.rstd && (a.rms || a.mean), none = !a.rstd && !a.mean;
    if constexpr (M != kTiny && TPR >= 64) {                      // (narrower rows: not worth their instances)
      StreamRows stream(n * (int64_t)sizeof(E));
      stream.add(a.x, a.rows, a.ldx * sizeof(E));
      stream.add(a.res, a.rows, a.ldr * sizeof(E));
      stream.add(a.sum, a.rows, a.lds * sizeof(E));
      stream.add(a.y, a.rows, a.ldy * sizeof(E));
      if (stats && stream.yes()) {
        if (a.res && a.sum) return launch(norm_kernel<E, M, TPR, C, kRes | kSum | kStats, true>);
        if (!a.res && a.sum) return launch(norm_kernel<E, M, TPR, C, kSum | kStats, true>);
        if (!a.res && !a.sum) return launch(norm_kernel<E, M, TPR, C, kStats, true>);
      }
    }
    if constexpr (M != kTiny) {
      if (a.res && a.sum && stats) return launch(norm_kernel<E, M, TPR, C, kRes | kSum | kStats>);
      if (a.res && a.sum && none) return launch(norm_kernel<E, M, TPR, C, kRes | kSum>);
      if (!a.res && a.sum && stats) return launch(norm_kernel<E, M, TPR, C, kSum | kStats>);
      if (!a.res && !a.sum && stats) return launch(norm_kernel<E, M, TPR, C, kStats>);
      if (!a.res && !a.sum && none) return launch(norm_kernel<E, M, TPR, C, 0>);
    }
    launch(norm_kernel<E, M, TPR, C, kAny>);
  };
  using std::integral_constant;
  const integral_constant<int, 8> c8;
  const integral_constant<int, 16> c16;
  const int tpr = threads_per_row(n);
  if (tpr == 8) return go(integral_constant<int, 8>(), c8);
  if constexpr (M != kTiny) {
    if (tpr == 16) return go(integral_constant<int, 16>(), c8);
    if (tpr == 32) return go(integral_constant<int, 32>(), c8);
    if (tpr == 64) return go(integral_constant<int, 64>(), c8);
    if (tpr == 128) return go(integral_constant<int, 128>(), c8);
    if (tpr == 256) return go(integral_constant<int, 256>(), c8);
    if (n <= 4096) return go(integral_constant<int, 512>(), c8);
    if (n <= 8192) return go(integral_constant<int, 512>(), c16);
    go(integral_constant<int, 1024>(), c16);
  }
}

template <class E, int M>
static void launch_norm_long(const NormArgs& a, hipStream_t st) {
  const int64_t blocks = std::min<int64_t>(a.rows, 512);
  DPRC_LAUNCH((norm_long_kernel<E, M>), dim3((unsigned)blocks), dim3(1024), 0, st, a);
}

template <class E>
static void launch_norm_width(const NormArgs& a, hipStream_t st) {
  constexpr int EP = kPiece<E>;
  // also rows so far apart that the 32 of a workgroup leave 32-bit offsets go the long rows' way
  if (a.n > kNormLong || 32 * std::max({a.ldx, a.ldr, a.lds, a.ldy}) * (int64_t)sizeof(E) >= ((int64_t)1 << 31)) {
    if (a.n < EP) launch_norm_long<E, kTiny>(a, st);
    else if (a.n % EP == 0) launch_norm_long<E, kWhole>(a, st);
    else launch_norm_long<E, kTail>(a, st);
  } else if (a.n < EP) {
    launch_norm_of<E, kTiny>(a, st);
  } else {
    launch_norm_of<E, kWide>(a, st);
  }
}

hipError_t launch_norm(const NormArgs& a, hipStream_t st) {
  if (a.bf16) launch_norm_width<uint16_t>(a, st);
  else launch_norm_width<float>(a, st);
  return hipGetLastError();
}

}  // namespace dprc
