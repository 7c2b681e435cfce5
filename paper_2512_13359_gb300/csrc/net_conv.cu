// net_conv.cu -- short causal convolution along a trajectory (auvnet.h, net_causal_conv).
//
// y[t] = act(b + sum_{k < K} w[k] x[t - (K - 1) + k]), each channel with its own K weights.  Nothing is carried from step
// to step but the last K - 1 rows, so a sequence is cut into chunks of steps that know nothing of each other: a thread
// walks E adjacent channels of one env through one chunk with those rows in registers, and reads the K - 1 rows ahead of
// its chunk once more (backward: also those behind it, whose outputs the chunk's rows are part of).  128 steps of 4,096 envs x
// 256 channels of bf16, K = 4, silu: 115 us (4.8 TB/s) and 185 us (4.5 TB/s), of 81 and 122 that the bytes take.  What bounds
// them is not established: issue slots are half used and DRAM less than half busy, and what warps wait for most are their own
// products, but neither more warps nor more bytes on their way (below) made them faster.
#include <algorithm>

#include "net_common.cuh"

namespace auv {
namespace net {
namespace {

constexpr int kMaxTaps = 8;

struct Conv {
  int T, chunk, chunks;
  int64_t N, D;
  net_rows x, y, dy, dx;
  const float *w, *bias;
  const void* state;
  void* new_state;
  const void* dnew_state;
  void* dstate;
  const uint8_t *done, *done_prev;
  float* partial;               // backward: [blocks][K + 1][D]
};

template <typename T>
__device__ __forceinline__ const T* row_of(const net_rows& r, int64_t n, int64_t d) {
  return reinterpret_cast<const T*>(r.data) + n * r.inner + d;
}
// The flag of the end before step t.  Loaded long before it is asked for: nothing may wait for the load in between.
__device__ __forceinline__ uint8_t flag_at(const Conv& a, int t, int64_t n) {
  const uint8_t* p = t ? a.done : a.done_prev;
  return p ? p[(t ? (t - 1) * a.N : 0) + n] : (uint8_t)0;
}
__device__ __forceinline__ bool ended(const Conv& a, int t, int64_t n) { return flag_at(a, t, n) != 0; }

// E channels as pairs (of one channel: with a zero beside it).
template <typename T, int E>
__device__ __forceinline__ void to_pairs(const Raw<T, E>& w, F2 (&v)[(E + 1) / 2]) {
  float x[E];
  unpack<T, E>(w, x);
#pragma unroll
  for (int i = 0; i < (E + 1) / 2; ++i) v[i] = pair(x[2 * i], 2 * i + 1 < E ? x[(2 * i + 1) % E] : 0.0f);
}
template <typename T, int E>
__device__ __forceinline__ Raw<T, E> from_pairs(const F2 (&v)[(E + 1) / 2]) {
  float x[E + 1];
#pragma unroll
  for (int i = 0; i < (E + 1) / 2; ++i) split(v[i], x[2 * i], x[2 * i + 1]);
  float y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = x[e];
  return pack<T, E>(y);
}
__device__ __forceinline__ F2 zeros() { return pair(0.0f, 0.0f); }

// The last K - 1 rows of the sequence, zeros where an episode has ended since.  By the thread that read the old state,
// row i from row i + T or from x, first to last: new_state may be state.
template <typename T, int E, int K>
__device__ void store_window(const Conv& a, int64_t n, int64_t d) {
  if constexpr (K > 1) {
    uint32_t cut = 0;
    bool gone = false;
#pragma unroll
    for (int i = K - 2; i >= 0; --i) {
      const int next = a.T - K + 2 + i;              // the step after row i
      if (next >= 0 && next < a.T) gone = gone || ended(a, next, n);
      cut |= (uint32_t)gone << i;
    }
    const int64_t m = a.N * a.D, at = n * a.D + d;
    T* const out = reinterpret_cast<T*>(a.new_state) + at;
#pragma unroll 1
    for (int i = 0; i < K - 1; ++i) {
      const int s = a.T - K + 1 + i;
      Raw<T, E> w = {};
      if (!(cut >> i & 1u)) {
        if (s >= 0) w = *reinterpret_cast<const Raw<T, E>*>(row_of<T>(a.x, n, d) + s * a.x.outer);
        else if (a.state) w = *reinterpret_cast<const Raw<T, E>*>(reinterpret_cast<const T*>(a.state) + (i + a.T) * m + at);
      }
      *reinterpret_cast<Raw<T, E>*>(out + i * m) = w;
    }
  }
}

// The weights, w[j] of the row j steps back.
template <int E, int K>
__device__ __forceinline__ void load_taps(const Conv& a, int64_t d, F2 (&w)[K][(E + 1) / 2], F2 (&b)[(E + 1) / 2]) {
#pragma unroll
  for (int i = 0; i < (E + 1) / 2; ++i) {
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const float* const p = a.w + (K - 1 - j) * a.D + d + 2 * i;
      w[j][i] = pair(p[0], 2 * i + 1 < E ? p[1] : 0.0f);
    }
    b[i] = a.bias ? pair(a.bias[d + 2 * i], 2 * i + 1 < E ? a.bias[d + 2 * i + 1] : 0.0f) : zeros();
  }
}

// The K - 1 rows ahead of step t0, win[j - 1] the one j steps back, zeros where an episode has ended since.
template <typename T, int E, int K>
__device__ __forceinline__ void load_window(const Conv& a, int t0, int64_t n, int64_t d, F2 (&win)[K][(E + 1) / 2]) {
#pragma unroll
  for (int j = 1; j < K; ++j) {
    const int s = t0 - j;
    Raw<T, E> w = {};
    if (s >= 0) w = *reinterpret_cast<const Raw<T, E>*>(row_of<T>(a.x, n, d) + s * a.x.outer);
    else if (a.state)
      w = *reinterpret_cast<const Raw<T, E>*>(reinterpret_cast<const T*>(a.state) + (s + K - 1) * a.N * a.D + n * a.D + d);
    to_pairs<T, E>(w, win[j - 1]);
  }
  bool gone = false;                                 // ends between the rows (that before t0 is the walk's)
#pragma unroll
  for (int j = 2; j < K; ++j) {
    const int next = t0 - j + 1;
    if (next >= 0) gone = gone || ended(a, next, n);
    if (gone) {
#pragma unroll
      for (int i = 0; i < (E + 1) / 2; ++i) win[j - 1][i] = zeros();
    }
  }
}

constexpr int kForward = 128;

// A batch of steps' inputs is on its way while one is computed.  Eight channels a thread or four, four steps or eight, 12 warps
// an SM or 24: 114 to 119 us; chunks of 26 steps, with more rows read twice, 125.
template <typename T, int E, int K>
__global__ void __launch_bounds__(kForward, 4) k_conv(Conv a, bool act) {
  constexpr int P = (E + 1) / 2, kBatch = E == 8 ? 4 : 8;
  const int64_t m = blockIdx.x * (int64_t)kForward + threadIdx.x, per = a.D / E;
  if (m >= a.N * per) return;
  const int64_t n = m / per, d = (m - n * per) * E;
  const int t0 = blockIdx.y * a.chunk, t1 = min(a.T, t0 + a.chunk);
  using W = Raw<T, E>;
  F2 w[K][P], b[P], win[K][P];
  const T* x = row_of<T>(a.x, n, d) + t0 * a.x.outer;
  T* y = const_cast<T*>(row_of<T>(a.y, n, d)) + t0 * a.y.outer;
  const bool flagged = K > 1 && (a.done || a.done_prev);
  W next[kBatch];
  uint8_t next_flag[kBatch];
  const uint8_t* done = a.done + ((int64_t)t0 - 1) * a.N + n;       // of the end before a batch's first step; not read for step 0
  auto fetch = [&](int t) {
    if (t + kBatch <= t1) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) next[u] = *reinterpret_cast<const W*>(x + u * a.x.outer);
    } else {
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (t + u < t1) next[u] = *reinterpret_cast<const W*>(x + u * a.x.outer);
    }
    x += kBatch * a.x.outer;
    if (flagged) {
      if (t > 0 && t + kBatch <= t1 && a.done) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) next_flag[u] = done[u * a.N];
      } else {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) next_flag[u] = t + u < t1 ? flag_at(a, t + u, n) : (uint8_t)0;
      }
      done += kBatch * a.N;
    }
  };
#pragma unroll
  for (int u = 0; u < kBatch; ++u) next_flag[u] = 0;
  fetch(t0);
  load_taps<E, K>(a, d, w, b);
  load_window<T, E, K>(a, t0, n, d, win);
  if (blockIdx.y == 0 && a.new_state) store_window<T, E, K>(a, n, d);
#pragma unroll 1
  for (int t = t0; t < t1; t += kBatch) {
    W raw[kBatch];
    uint32_t ends = 0;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      raw[u] = next[u];
      ends |= (next_flag[u] ? 1u : 0u) << u;
    }
    fetch(t + kBatch);
    // PLAIN: a whole batch without an end: no questions
    auto walk = [&](auto plain) {
      constexpr bool kPlain = decltype(plain)::value;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (!kPlain && t + u >= t1) break;
        F2 r[P], p[P];
        to_pairs<T, E>(raw[u], r);
        if (!kPlain && (ends >> u & 1u)) {
#pragma unroll
          for (int j = 0; j < K; ++j)
#pragma unroll
            for (int i = 0; i < P; ++i) win[j][i] = zeros();
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
          p[i] = b[i];
#pragma unroll
          for (int j = K - 1; j > 0; --j) p[i] = fma2(w[j][i], win[j - 1][i], p[i]);
          p[i] = fma2(w[0][i], r[i], p[i]);
#pragma unroll
          for (int j = K - 1; j > 0; --j) win[j][i] = win[j - 1][i];
          win[0][i] = r[i];
          if (act) p[i] = p[i] * sigmoid2(p[i]);
        }
        *reinterpret_cast<W*>(y + u * a.y.outer) = from_pairs<T, E>(p);
      }
    };
    if (t + kBatch <= t1 && !ends) walk(std::true_type());
    else walk(std::false_type());
    y += kBatch * a.y.outer;
  }
}

// Backward.  With p the sums and dp = dy act'(p): dx[s] = sum_j w_j dp[s + j] over the steps s + j that see row s, so a row
// is done K - 1 steps after its own, or ahead of the step before which its episode ended.  The weights' gradients are
// summed in registers over all chunks of a thread, over the block's threads of the same channels, and over the blocks by
// k_conv_sums, each in a fixed order.  Inputs come by cp.async to slots of the thread's own, three batches of four steps
// ahead (six batches: 195 us for 185, eight leave half the warps: 347); a batch without an end, inside the chunk, is gone
// through without a question about its rows.
constexpr int kBackward = 128;
constexpr int kBack = 4, kRing = 4;                   // steps of a batch, batches in shared memory

template <typename T, int E, int K>
__global__ void __launch_bounds__(kBackward, K <= 4 ? 4 : 2) k_conv_back(Conv a, bool act, int side) {
  constexpr int P = (E + 1) / 2;
  using W = Raw<T, E>;
  constexpr bool kCopied = kAsync<T, E>;
  extern __shared__ uint4 smem[];
  __shared__ float part[kBackward][E];
  W* const ring = reinterpret_cast<W*>(smem) + threadIdx.x;       // slot (step, array) at (step % 16 * 2 + array) * kBackward
  const int lane = threadIdx.x % side, slot = threadIdx.x / side, slots = kBackward / side;
  const int64_t d = (blockIdx.x * (int64_t)side + lane) * E;
  const bool live = d < a.D;
  F2 w[K][P], b[P], dw[K][P], db[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    db[i] = zeros();
#pragma unroll
    for (int j = 0; j < K; ++j) dw[j][i] = zeros();
  }
  if (live) load_taps<E, K>(a, d, w, b);
  const int64_t m = a.N * a.D, items = live ? a.N * a.chunks : 0;
  const bool flagged = K > 1 && (a.done || a.done_prev);
  for (int64_t item = blockIdx.y * (int64_t)slots + slot; item < items; item += gridDim.y * (int64_t)slots) {
    const int64_t n = item % a.N;
    const int t0 = (int)(item / a.N) * a.chunk, t1 = min(a.T, t0 + a.chunk), last = min(a.T, t1 + K - 1);
    const T* const x = row_of<T>(a.x, n, d);
    const T* const dy = row_of<T>(a.dy, n, d);
    T* const dx = const_cast<T*>(row_of<T>(a.dx, n, d));
    const T* px = x + t0 * a.x.outer;
    const T* pdy = dy + t0 * a.dy.outer;
    auto copy = [&](int t) {
      if constexpr (kCopied) {
        W* const to = ring + (t - t0) % (kBack * kRing) * 2 * kBackward;
        if (t + kBack <= last) {
#pragma unroll
          for (int u = 0; u < kBack; ++u) {
            copy_async<sizeof(W)>(to + u * 2 * kBackward, px + u * a.x.outer);
            copy_async<sizeof(W)>(to + (u * 2 + 1) * kBackward, pdy + u * a.dy.outer);
          }
        } else {
#pragma unroll
          for (int u = 0; u < kBack; ++u)
            if (t + u < last) {
              copy_async<sizeof(W)>(to + u * 2 * kBackward, px + u * a.x.outer);
              copy_async<sizeof(W)>(to + (u * 2 + 1) * kBackward, pdy + u * a.dy.outer);
            }
        }
        px += kBack * a.x.outer, pdy += kBack * a.dy.outer;
        copy_commit();
      }
    };
    uint8_t next_flag[kBack];
    const uint8_t* done = a.done + ((int64_t)t0 - 1) * a.N + n;   // of the end before a batch's first step; not read for step 0
#pragma unroll
    for (int u = 0; u < kBack; ++u) next_flag[u] = 0;
    auto fetch_flags = [&](int t) {
      if (!flagged) return;
      if (t > 0 && t + kBack <= last && a.done) {
#pragma unroll
        for (int u = 0; u < kBack; ++u) next_flag[u] = done[u * a.N];
      } else {
#pragma unroll
        for (int u = 0; u < kBack; ++u) next_flag[u] = t + u < last ? flag_at(a, t + u, n) : (uint8_t)0;
      }
      done += kBack * a.N;
    };
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) copy(t0 + i * kBack);
    fetch_flags(t0);
    F2 win[K][P], acc[K][P];
    load_window<T, E, K>(a, t0, n, d, win);
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
      for (int i = 0; i < P; ++i) acc[j][i] = zeros();
    // rows that may still gain: of the sequence's own chunk, and ahead of the first step the state's
    int pending = t0 ? 0 : K - 1;
    auto put = [&](int s, F2 (&v)[P]) {
      if (s >= t0 && s < t1) *reinterpret_cast<W*>(dx + s * a.dx.outer) = from_pairs<T, E>(v);
      else if (s < 0 && t0 == 0 && a.dstate)
        *reinterpret_cast<W*>(reinterpret_cast<T*>(a.dstate) + (s + K - 1) * m + n * a.D + d) = from_pairs<T, E>(v);
    };
    auto step = [&](const W& rx, const W& rdy, bool counts) {
      F2 r[P], dp[P];
      to_pairs<T, E>(rx, r);
      to_pairs<T, E>(rdy, dp);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (act) {
          F2 p = b[i];
#pragma unroll
          for (int j = K - 1; j > 0; --j) p = fma2(w[j][i], win[j - 1][i], p);
          p = fma2(w[0][i], r[i], p);
          // s (1 + p (1 - s)): p - p s is off by 2^-24 p, of a slope near 1 where p is large
          const F2 s = sigmoid2(p), q = fma2(p * pair(-1.0f, -1.0f), s, p);
          dp[i] = dp[i] * fma2(s, q, s);
        }
        if (counts) {
          db[i] = db[i] + dp[i];
          dw[0][i] = fma2(dp[i], r[i], dw[0][i]);
#pragma unroll
          for (int j = 1; j < K; ++j) dw[j][i] = fma2(dp[i], win[j - 1][i], dw[j][i]);
        }
#pragma unroll
        for (int j = K - 1; j > 0; --j) {
          acc[j][i] = fma2(w[j][i], dp[i], acc[j - 1][i]);
          win[j][i] = win[j - 1][i];
        }
        acc[0][i] = w[0][i] * dp[i];
        win[0][i] = r[i];
      }
    };
    T* pdx = dx + (int64_t)(t0 - K + 1) * a.dx.outer;             // of the row that a step completes
#pragma unroll 1
    for (int tb = t0; tb < last; tb += kBack, pdx += kBack * a.dx.outer) {
      uint32_t flags = 0;
#pragma unroll
      for (int u = 0; u < kBack; ++u) flags |= (next_flag[u] ? 1u : 0u) << u;
      fetch_flags(tb + kBack);
      W* const from = ring + (tb - t0) % (kBack * kRing) * 2 * kBackward;
      W rx[kBack], rdy[kBack];
      if constexpr (kCopied) {
        copy_wait<kRing - 2>();
#pragma unroll
        for (int u = 0; u < kBack; ++u) rx[u] = from[u * 2 * kBackward], rdy[u] = from[(u * 2 + 1) * kBackward];
        copy(tb + (kRing - 1) * kBack);
      } else {
#pragma unroll
        for (int u = 0; u < kBack; ++u)
          if (tb + u < last) {
            rx[u] = *reinterpret_cast<const W*>(px);
            rdy[u] = *reinterpret_cast<const W*>(pdy);
            px += a.x.outer, pdy += a.dy.outer;
          }
      }
      if (!flags && pending == K - 1 && tb - (K - 1) >= t0 && tb + kBack <= t1) {
#pragma unroll
        for (int u = 0; u < kBack; ++u) {
          step(rx[u], rdy[u], true);
          *reinterpret_cast<W*>(pdx + u * a.dx.outer) = from_pairs<T, E>(acc[K - 1]);
        }
        continue;
      }
#pragma unroll
      for (int u = 0; u < kBack; ++u) {
        const int t = tb + u;
        if (t >= last) break;
        if (flags >> u & 1u) {
#pragma unroll
          for (int j = 1; j < K; ++j) {
            if (j <= pending) put(t - j, acc[j - 1]);
#pragma unroll
            for (int i = 0; i < P; ++i) win[j - 1][i] = zeros();
          }
          pending = 0;
        }
        step(rx[u], rdy[u], t < t1);
        if (pending == K - 1) put(t - (K - 1), acc[K - 1]);
        else ++pending;
      }
    }
    if constexpr (kCopied) copy_wait<0>();
    if (last == a.T) {                                // what is left passes into the state after the last step
#pragma unroll
      for (int j = 1; j < K; ++j) {
        if (j > pending) break;
        if (a.dnew_state) {
          F2 g[P];
          to_pairs<T, E>(*reinterpret_cast<const W*>(reinterpret_cast<const T*>(a.dnew_state) + (K - 1 - j) * m + n * a.D + d), g);
#pragma unroll
          for (int i = 0; i < P; ++i) acc[j - 1][i] = acc[j - 1][i] + g[i];
        }
        put(a.T - j, acc[j - 1]);
      }
    }
  }
  if (!a.partial) return;
  float* const out = a.partial + blockIdx.y * (K + 1) * a.D;
  for (int k = 0; k <= K; ++k) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      F2 q = db[i];
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (k == K - 1 - j) q = dw[j][i];
      float lo, hi;
      split(q, lo, hi);
      part[threadIdx.x][2 * i] = lo;
      if (2 * i + 1 < E) part[threadIdx.x][(2 * i + 1) % E] = hi;
    }
    __syncthreads();
    if (slot == 0 && live) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float v = 0.0f;
        for (int s = 0; s < slots; ++s) v += part[s * side + lane][e];
        out[k * a.D + d + e] = v;
      }
    }
    __syncthreads();
  }
}

// out[c] = sum over rows of partial[row][c], columns 0 .. split - 1 to one array and the rest to another.
constexpr int kSumCols = 8, kSumThreads = 512, kSumGroups = kSumThreads / kSumCols;
__global__ void __launch_bounds__(kSumThreads) k_conv_sums(const float* partial, int rows, int64_t cols, int64_t split, float* first,
                                                           float* second) {
  __shared__ float part[kSumThreads / 32][kSumCols];
  after_previous();
  const int lane = threadIdx.x % kSumCols, group = threadIdx.x / kSumCols;
  const int64_t c = blockIdx.x * (int64_t)kSumCols + lane;
  float v = 0.0f;
  if (c < cols) {
    const float* p = partial + group * cols + c;
#pragma unroll 4
    for (int r = group; r < rows; r += kSumGroups, p += kSumGroups * cols) v += *p;
  }
#pragma unroll
  for (int o = 16; o >= kSumCols; o /= 2) v += __shfl_down_sync(0xffffffffu, v, o);
  if (threadIdx.x % 32 < kSumCols) part[threadIdx.x / 32][lane] = v;
  __syncthreads();
  if (threadIdx.x >= kSumCols || c >= cols) return;
  v = 0.0f;
#pragma unroll
  for (int w = 0; w < kSumThreads / 32; ++w) v += part[w][lane];
  float* const to = c < split ? first : second;
  if (to) to[c < split ? c : c - split] = v;
}

// T = 0: the state passes as it is.
template <typename T>
__global__ void k_conv_none(int64_t m, const T* from, T* to) {
  const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
  if (i < m) {
    if (from) to[i] = from[i];
    else from_float(0.0f, to[i]);
  }
}
__global__ void k_conv_zero(int64_t m, float* to) {
  const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
  if (i < m) to[i] = 0.0f;
}

// Steps of a chunk: all of them where envs and channels make enough threads, else as few as fill the device, 16 at least.
int chunk_of(int64_t T, int64_t threads) {
  const int64_t want = (int64_t)sm_count() * 1024;
  int64_t chunks = std::max<int64_t>(1, std::min((want + threads - 1) / std::max<int64_t>(1, threads), T / 16));
  chunks = std::min<int64_t>(chunks, 65535);                   // a grid's second axis
  const int64_t chunk = (T + chunks - 1) / chunks;
  return (int)std::max<int64_t>(1, chunk);
}

struct BackPlan {
  int side, slots, chunk, chunks;
  int64_t tiles, blocks;        // of channels; along envs and chunks
};
BackPlan back_plan(int64_t T, int64_t N, int64_t D, int e) {
  BackPlan p;
  const int64_t per = (D + e - 1) / e;
  p.side = 1;
  while (p.side < per && p.side < kBackward) p.side *= 2;
  p.slots = kBackward / p.side;
  p.tiles = (per + p.side - 1) / p.side;
  p.chunk = chunk_of(T, N * per);
  p.chunks = (int)((T + p.chunk - 1) / p.chunk);
  const int64_t items = N * p.chunks, most = std::max<int64_t>(1, (int64_t)sm_count() * 4 / p.tiles);
  p.blocks = std::max<int64_t>(1, std::min((items + p.slots - 1) / p.slots, std::min<int64_t>(most, 65535)));
  return p;
}

// Channels of a thread, as many as every access can be aligned to: forward 16 bytes, with few taps and enough channels,
// else four, two or one.
int width_of(const net_conv* a, bool back) {
  const int z = type_size(a->dtype);
  const net_rows* rows[] = {&a->x, back ? &a->dy : &a->y, back ? &a->dx : &a->x};
  const void* flat[] = {a->state, back ? a->dnew_state : a->new_state, back ? a->dstate : nullptr};
  for (int e = !back && z == 2 && a->K <= 4 && a->N * a->D >= (int64_t)sm_count() * 8192 ? 8 : 4; e > 1; e /= 2) {
    bool fits = a->D % e == 0;
    for (const net_rows* r : rows) fits = fits && aligned(*r, a->T, a->N, z, e);
    for (const void* p : flat) fits = fits && reinterpret_cast<uintptr_t>(p) % ((size_t)z * e) == 0;
    if (fits) return e;
  }
  return 1;
}

template <typename T, int E, int K>
cudaError_t launch_taps(Conv& a, bool back, bool act, float* dw, float* dbias, cudaStream_t s) {
  if (!back) {
    const int64_t threads = a.N * (a.D / E);
    a.chunk = std::max(chunk_of(a.T, threads), K);
    a.chunks = (a.T + a.chunk - 1) / a.chunk;
    k_conv<T, E, K><<<dim3((unsigned)((threads + kForward - 1) / kForward), (unsigned)a.chunks), kForward, 0, s>>>(a, act);
    return cudaGetLastError();
  }
  if constexpr (E > 4) return cudaErrorInvalidValue;   // not asked for
  else {
  const BackPlan p = back_plan(a.T, a.N, a.D, E);
  a.chunk = p.chunk, a.chunks = p.chunks;
  if (!dw && !dbias) a.partial = nullptr;
  const auto kern = k_conv_back<T, E, K>;
  const int smem = kAsync<T, E> ? kBack * kRing * 2 * kBackward * (int)sizeof(T) * E : 0;
  cudaError_t e = smem > 40 * 1024 ? cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) : cudaSuccess;
  if (e != cudaSuccess) return e;
  kern<<<dim3((unsigned)p.tiles, (unsigned)p.blocks), kBackward, smem, s>>>(a, act, p.side);
  e = cudaGetLastError();
  if (e != cudaSuccess || !a.partial) return e;
  const int64_t cols = (K + 1) * a.D;
  return launch_after(k_conv_sums, dim3((unsigned)((cols + kSumCols - 1) / kSumCols)), kSumThreads, 0, s, a.partial, (int)p.blocks, cols,
                      K * a.D, dw,
                      dbias);
  }
}

template <typename T, int E>
cudaError_t launch_width(Conv& a, int K, bool back, bool act, float* dw, float* dbias, cudaStream_t s) {
  switch (K) {
    case 1: return launch_taps<T, E, 1>(a, back, act, dw, dbias, s);
    case 2: return launch_taps<T, E, 2>(a, back, act, dw, dbias, s);
    case 3: return launch_taps<T, E, 3>(a, back, act, dw, dbias, s);
    case 4: return launch_taps<T, E, 4>(a, back, act, dw, dbias, s);
  }
  if constexpr (E <= 4) {
    switch (K) {
      case 5: return launch_taps<T, E, 5>(a, back, act, dw, dbias, s);
      case 6: return launch_taps<T, E, 6>(a, back, act, dw, dbias, s);
      case 7: return launch_taps<T, E, 7>(a, back, act, dw, dbias, s);
      case 8: return launch_taps<T, E, 8>(a, back, act, dw, dbias, s);
    }
  }
  return cudaErrorInvalidValue;   // not asked for
}

template <typename T>
cudaError_t launch(Conv& a, const net_conv* p, bool back, cudaStream_t s) {
  const bool act = p->act == NET_ACT_SILU;
  if (a.T == 0 || a.N == 0) {
    const int64_t m = (p->K - 1) * a.N * a.D;
    const void* const from = back ? a.dnew_state : a.state;
    void* const to = back ? a.dstate : a.new_state;
    if (to && m)
      k_conv_none<T><<<(unsigned)((m + 255) / 256), 256, 0, s>>>(m, static_cast<const T*>(from), static_cast<T*>(to));
    if (back && p->dw) k_conv_zero<<<(unsigned)((p->K * a.D + 255) / 256), 256, 0, s>>>(p->K * a.D, p->dw);
    if (back && p->dbias) k_conv_zero<<<(unsigned)((a.D + 255) / 256), 256, 0, s>>>(a.D, p->dbias);
    return cudaGetLastError();
  }
  switch (width_of(p, back)) {
    case 8:
      if constexpr (sizeof(T) == 2) return launch_width<T, 8>(a, (int)p->K, back, act, p->dw, p->dbias, s);
    case 4: return launch_width<T, 4>(a, (int)p->K, back, act, p->dw, p->dbias, s);
    case 2: return launch_width<T, 2>(a, (int)p->K, back, act, p->dw, p->dbias, s);
    default: return launch_width<T, 1>(a, (int)p->K, back, act, p->dw, p->dbias, s);
  }
}

int check(const net_conv* p) {
  if (!p) return fail(AUV_ERR_INVALID, "argument block is NULL");
  if (p->struct_size != sizeof(net_conv))
    return fail(AUV_ERR_INVALID, "struct_size %u, expected %zu", p->struct_size, sizeof(net_conv));
  if (p->dtype > NET_FP16) return fail(AUV_ERR_INVALID, "dtype %u unknown", p->dtype);
  if (p->act != NET_ACT_NONE && p->act != NET_ACT_SILU) return fail(AUV_ERR_INVALID, "act %u is neither none nor silu", p->act);
  if (p->reserved) return fail(AUV_ERR_INVALID, "reserved is not 0");
  if (p->T < 0 || p->N < 0 || p->D < 0) return fail(AUV_ERR_INVALID, "negative size");
  if (p->K < 1) return fail(AUV_ERR_INVALID, "K < 1");
  if (p->K > kMaxTaps) return fail(AUV_ERR_UNSUPPORTED, "K past %d", kMaxTaps);
  const int64_t most = (int64_t)1 << 34;
  if (p->N > most || p->D > (1 << 24) || p->N * p->D > most || p->T > (1 << 30))
    return fail(AUV_ERR_UNSUPPORTED, "N * D past 2^34, D past 2^24 or T past 2^30");
  return AUV_OK;
}

int run(const net_conv* p, bool back, void* stream) {
  int rc = check(p);
  if (rc) return rc;
  if (p->D == 0 || (!back && p->N == 0)) return AUV_OK;
  const int z = type_size(p->dtype);
  struct { const net_rows* r; const char* name; bool out, used; } rows[] = {
      {&p->x, "x", false, true}, {&p->y, "y", true, !back}, {&p->dy, "dy", false, back}, {&p->dx, "dx", true, back}};
  if (p->T && p->N)
    for (const auto& q : rows)
      if (q.used && (rc = need_rows(*q.r, q.name, p->T, p->N, p->D, z, q.out))) return rc;
  if ((rc = need(p->w, "w", 4))) return rc;
  const bool states = p->K > 1 && p->N;
  struct { const void* p; const char* name; size_t align; bool used; } flat[] = {
      {p->bias, "bias", 4, true},      {p->state, "state", (size_t)z, states},
      {p->new_state, "new_state", (size_t)z, states && !back}, {p->dnew_state, "dnew_state", (size_t)z, states && back},
      {p->dstate, "dstate", (size_t)z, states && back},        {p->dw, "dw", 4, back},
      {p->dbias, "dbias", 4, back},    {p->done, "done", 1, true},
      {p->done_prev, "done_prev", 1, true}};
  for (const auto& q : flat)
    if (q.p && q.used && (rc = need(q.p, q.name, q.align))) return rc;
  const size_t bytes = net_causal_conv_workspace_bytes(p, back);
  if (bytes) {
    if (p->workspace_bytes < bytes) return fail(AUV_ERR_SIZE, "workspace of %zu bytes, %zu needed", p->workspace_bytes, bytes);
    if ((rc = need(p->workspace, "workspace", 16))) return rc;
  }
  Conv a = {(int)p->T, 0, 0, p->N, p->D, p->x, p->y, p->dy, p->dx, p->w, p->bias, p->state, p->new_state, p->dnew_state, p->dstate,
            p->done, p->done_prev, static_cast<float*>(p->workspace)};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p->dtype == NET_FP32   ? launch<float>(a, p, back, s)
                        : p->dtype == NET_BF16 ? launch<__nv_bfloat16>(a, p, back, s)
                                               : launch<__half>(a, p, back, s);
  return e == cudaSuccess ? AUV_OK : cuda_fail(e, back ? "net_causal_conv_backward" : "net_causal_conv");
}

}  // namespace
}  // namespace net
}  // namespace auv

extern "C" {

size_t net_causal_conv_workspace_bytes(const net_conv* a, int backward) {
  using namespace auv::net;
  if (!a || check(a) || !backward || !a->T || !a->N || !a->D || !(a->dw || a->dbias)) return 0;
  // whatever the alignment of arrays that are not there yet
  int64_t most = 0;
  for (int e = 1; e <= 4; e *= 2) most = std::max(most, back_plan(a->T, a->N, a->D, e).blocks);
  return sizeof(float) * (size_t)most * (size_t)((a->K + 1) * a->D);
}

int net_causal_conv(const net_conv* a, void* stream) { return auv::net::run(a, false, stream); }
int net_causal_conv_backward(const net_conv* a, void* stream) { return auv::net::run(a, true, stream); }

}  // extern "C"
