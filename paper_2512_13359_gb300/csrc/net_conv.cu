// net_conv.cu -- short causal convolution along a trajectory (auvnet.h, net_causal_conv).
//
// y[t] = act(b + sum_{k < K} w[k] x[t - (K - 1) + k]), each channel with its own K weights.  Nothing is carried from step
// to step but the last K - 1 rows, so a sequence is cut into chunks of steps that know nothing of each other: a thread
// walks E adjacent channels of one env through one chunk with those rows in registers, and reads the K - 1 rows ahead of
// its chunk once more (backward: also those behind it, whose outputs the chunk's rows are part of).
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
__device__ __forceinline__ bool ended(const Conv& a, int t, int64_t n) {
  const uint8_t* p = t ? a.done : a.done_prev;
  return p && p[(t ? (t - 1) * a.N : 0) + n];
}

// silu and its slope s (1 + u sigmoid(-u)).
__device__ __forceinline__ float silu(float u) {
  float s, o;
  gates(u, s, o);
  return u * s;
}
__device__ __forceinline__ float silu_slope(float u) {
  float s, o;
  gates(u, s, o);
  return s * fmaf(u, o, 1.0f);
}

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

template <int E, int K>
__device__ __forceinline__ void load_taps(const Conv& a, int64_t d, float (&w)[K][E], float (&b)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
#pragma unroll
    for (int j = 0; j < K; ++j) w[j][e] = a.w[(K - 1 - j) * a.D + d + e];    // of the row j steps back
    b[e] = a.bias ? a.bias[d + e] : 0.0f;
  }
}

// The K - 1 rows ahead of step t0, win[j - 1] the one j steps back, zeros where an episode has ended since.
template <typename T, int E, int K>
__device__ __forceinline__ void load_window(const Conv& a, int t0, int64_t n, int64_t d, float (&win)[K][E]) {
#pragma unroll
  for (int j = 1; j < K; ++j) {
    const int s = t0 - j;
#pragma unroll
    for (int e = 0; e < E; ++e) win[j - 1][e] = 0.0f;
    if (s >= 0) load<T, E>(row_of<T>(a.x, n, d) + s * a.x.outer, win[j - 1]);
    else if (a.state) load<T, E>(reinterpret_cast<const T*>(a.state) + (s + K - 1) * a.N * a.D + n * a.D + d, win[j - 1]);
  }
  bool gone = false;                                 // ends between the rows (that before t0 is the walk's)
#pragma unroll
  for (int j = 2; j < K; ++j) {
    const int next = t0 - j + 1;
    if (next >= 0) gone = gone || ended(a, next, n);
    if (gone) {
#pragma unroll
      for (int e = 0; e < E; ++e) win[j - 1][e] = 0.0f;
    }
  }
}

constexpr int kForward = 256;
constexpr int kBatch = 8;

template <typename T, int E, int K>
__global__ void __launch_bounds__(kForward) k_conv(Conv a, bool act) {
  const int64_t m = blockIdx.x * (int64_t)kForward + threadIdx.x, per = a.D / E;
  if (m >= a.N * per) return;
  const int64_t n = m / per, d = (m - n * per) * E;
  const int t0 = blockIdx.y * a.chunk, t1 = min(a.T, t0 + a.chunk);
  using W = Raw<T, E>;
  float w[K][E], b[E], win[K][E];
  const T* x = row_of<T>(a.x, n, d) + t0 * a.x.outer;
  T* y = const_cast<T*>(row_of<T>(a.y, n, d)) + t0 * a.y.outer;
  W next[kBatch];
  uint32_t flags = 0;
  auto fetch = [&](int t) {
    flags = 0;
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (t + u < t1) {
        next[u] = *reinterpret_cast<const W*>(x);
        x += a.x.outer;
        if (K > 1 && ended(a, t + u, n)) flags |= 1u << u;
      }
  };
  fetch(t0);
  load_taps<E, K>(a, d, w, b);
  load_window<T, E, K>(a, t0, n, d, win);
  if (blockIdx.y == 0 && a.new_state) store_window<T, E, K>(a, n, d);
  for (int t = t0; t < t1; t += kBatch) {
    W raw[kBatch];
    const uint32_t ends = flags;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) raw[u] = next[u];
    fetch(t + kBatch);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (t + u >= t1) break;
      float r[E], p[E];
      unpack<T, E>(raw[u], r);
      if (ends >> u & 1u) {
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
          for (int e = 0; e < E; ++e) win[j][e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        p[e] = b[e];
#pragma unroll
        for (int j = K - 1; j > 0; --j) p[e] = fmaf(w[j][e], win[j - 1][e], p[e]);
        p[e] = fmaf(w[0][e], r[e], p[e]);
#pragma unroll
        for (int j = K - 1; j > 0; --j) win[j][e] = win[j - 1][e];
        win[0][e] = r[e];
        if (act) p[e] = silu(p[e]);
      }
      store<T, E>(y, p);
      y += a.y.outer;
    }
  }
}

// Backward.  With p the sums and dp = dy act'(p): dx[s] = sum_j w_j dp[s + j] over the steps s + j that see row s, so a row
// is done K - 1 steps after its own, or ahead of the step before which its episode ended.  The weights' gradients are
// summed in registers over all chunks of a thread, over the block's threads of the same channels, and over the blocks by
// k_conv_sums, each in a fixed order.
constexpr int kBackward = 128;

template <typename T, int E, int K>
__global__ void __launch_bounds__(kBackward) k_conv_back(Conv a, bool act, int side) {
  __shared__ float part[kBackward][E];
  const int lane = threadIdx.x % side, slot = threadIdx.x / side, slots = kBackward / side;
  const int64_t d = (blockIdx.x * (int64_t)side + lane) * E;
  const bool live = d < a.D;
  using W = Raw<T, E>;
  float w[K][E], b[E], dw[K][E], db[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    db[e] = 0.0f;
#pragma unroll
    for (int j = 0; j < K; ++j) dw[j][e] = 0.0f;
  }
  if (live) load_taps<E, K>(a, d, w, b);
  const int64_t m = a.N * a.D, items = live ? a.N * a.chunks : 0;
  for (int64_t item = blockIdx.y * (int64_t)slots + slot; item < items; item += gridDim.y * (int64_t)slots) {
    const int64_t n = item % a.N;
    const int t0 = (int)(item / a.N) * a.chunk, t1 = min(a.T, t0 + a.chunk), last = min(a.T, t1 + K - 1);
    float win[K][E], acc[K][E];
    load_window<T, E, K>(a, t0, n, d, win);
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[j][e] = 0.0f;
    const T* const x = row_of<T>(a.x, n, d);
    const T* const dy = row_of<T>(a.dy, n, d);
    T* const dx = const_cast<T*>(row_of<T>(a.dx, n, d));
    // rows that may still gain: of the sequence's own chunk, and ahead of the first step the state's
    int pending = t0 ? 0 : K - 1;
    auto put = [&](int s, float (&v)[E]) {
      if (s >= t0 && s < t1) store<T, E>(dx + s * a.dx.outer, v);
      else if (s < 0 && t0 == 0 && a.dstate)
        store<T, E>(reinterpret_cast<T*>(a.dstate) + (s + K - 1) * m + n * a.D + d, v);
    };
    for (int tb = t0; tb < last; tb += kBatch) {
      W rx[kBatch], rdy[kBatch];
      uint32_t flags = 0;
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (tb + u < last) {
          rx[u] = *reinterpret_cast<const W*>(x + (tb + u) * a.x.outer);
          rdy[u] = *reinterpret_cast<const W*>(dy + (tb + u) * a.dy.outer);
          if (K > 1 && ended(a, tb + u, n)) flags |= 1u << u;
        }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int t = tb + u;
        if (t >= last) break;
        if (flags >> u & 1u) {
#pragma unroll
          for (int j = 1; j < K; ++j) {
            if (j <= pending) put(t - j, acc[j - 1]);
#pragma unroll
            for (int e = 0; e < E; ++e) win[j - 1][e] = 0.0f;
          }
          pending = 0;
        }
        float r[E], dp[E];
        unpack<T, E>(rx[u], r);
        unpack<T, E>(rdy[u], dp);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (act) {
            float p = b[e];
#pragma unroll
            for (int j = K - 1; j > 0; --j) p = fmaf(w[j][e], win[j - 1][e], p);
            dp[e] *= silu_slope(fmaf(w[0][e], r[e], p));
          }
          if (t < t1) {
            db[e] += dp[e];
            dw[0][e] = fmaf(dp[e], r[e], dw[0][e]);
#pragma unroll
            for (int j = 1; j < K; ++j) dw[j][e] = fmaf(dp[e], win[j - 1][e], dw[j][e]);
          }
#pragma unroll
          for (int j = K - 1; j > 0; --j) {
            acc[j][e] = fmaf(w[j][e], dp[e], acc[j - 1][e]);
            win[j][e] = win[j - 1][e];
          }
          acc[0][e] = w[0][e] * dp[e];
          win[0][e] = r[e];
        }
        if (pending == K - 1) put(t - (K - 1), acc[K - 1]);
        else ++pending;
      }
    }
    if (last == a.T) {                                // what is left passes into the state after the last step
#pragma unroll
      for (int j = 1; j < K; ++j) {
        if (j > pending) break;
        if (a.dnew_state) {
          float g[E];
          load<T, E>(reinterpret_cast<const T*>(a.dnew_state) + (K - 1 - j) * m + n * a.D + d, g);
#pragma unroll
          for (int e = 0; e < E; ++e) acc[j - 1][e] += g[e];
        }
        put(a.T - j, acc[j - 1]);
      }
    }
  }
  if (!a.partial) return;
  float* const out = a.partial + blockIdx.y * (K + 1) * a.D;
  for (int k = 0; k <= K; ++k) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float v = db[e];
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (k == K - 1 - j) v = dw[j][e];
      part[threadIdx.x][e] = v;
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
constexpr int kSumGroups = 32;
__global__ void __launch_bounds__(1024) k_conv_sums(const float* partial, int rows, int64_t cols, int64_t split, float* first,
                                                    float* second) {
  __shared__ float part[kSumGroups][33];
  after_previous();
  const int lane = threadIdx.x % 32, group = threadIdx.x / 32;
  const int64_t c = blockIdx.x * (int64_t)32 + lane;
  float v = 0.0f;
  if (c < cols)
    for (int r = group; r < rows; r += kSumGroups) v += partial[r * cols + c];
  part[group][lane] = v;
  __syncthreads();
  v = part[lane][group];
#pragma unroll
  for (int o = 16; o; o /= 2) v += __shfl_down_sync(0xffffffffu, v, o);
  const int64_t k = blockIdx.x * (int64_t)32 + group;
  if (lane == 0 && k < cols) {
    float* const to = k < split ? first : second;
    if (to) to[k < split ? k : k - split] = v;
  }
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
  const int64_t items = N * p.chunks, most = std::max<int64_t>(1, (int64_t)sm_count() * 8 / p.tiles);
  p.blocks = std::max<int64_t>(1, std::min((items + p.slots - 1) / p.slots, std::min<int64_t>(most, 65535)));
  return p;
}

// Channels of a thread: four where every access of four is aligned.
int width_of(const net_conv* a, bool back) {
  const int z = type_size(a->dtype);
  if (a->D % 4) return 1;
  const net_rows* rows[] = {&a->x, back ? &a->dy : &a->y, back ? &a->dx : &a->x};
  for (const net_rows* r : rows)
    if (!aligned(*r, a->T, a->N, z, 4)) return 1;
  const void* flat[] = {a->state, back ? a->dnew_state : a->new_state, back ? a->dstate : nullptr};
  for (const void* p : flat)
    if (reinterpret_cast<uintptr_t>(p) % ((size_t)z * 4)) return 1;
  return 4;
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
  const BackPlan p = back_plan(a.T, a.N, a.D, E);
  a.chunk = p.chunk, a.chunks = p.chunks;
  if (!dw && !dbias) a.partial = nullptr;
  k_conv_back<T, E, K><<<dim3((unsigned)p.tiles, (unsigned)p.blocks), kBackward, 0, s>>>(a, act, p.side);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !a.partial) return e;
  const int64_t cols = (K + 1) * a.D;
  return launch_after(k_conv_sums, dim3((unsigned)((cols + 31) / 32)), 1024, 0, s, a.partial, (int)p.blocks, cols, K * a.D, dw,
                      dbias);
}

template <typename T, int E>
cudaError_t launch_width(Conv& a, int K, bool back, bool act, float* dw, float* dbias, cudaStream_t s) {
  switch (K) {
    case 1: return launch_taps<T, E, 1>(a, back, act, dw, dbias, s);
    case 2: return launch_taps<T, E, 2>(a, back, act, dw, dbias, s);
    case 3: return launch_taps<T, E, 3>(a, back, act, dw, dbias, s);
    case 4: return launch_taps<T, E, 4>(a, back, act, dw, dbias, s);
    case 5: return launch_taps<T, E, 5>(a, back, act, dw, dbias, s);
    case 6: return launch_taps<T, E, 6>(a, back, act, dw, dbias, s);
    case 7: return launch_taps<T, E, 7>(a, back, act, dw, dbias, s);
    default: return launch_taps<T, E, 8>(a, back, act, dw, dbias, s);
  }
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
  if (width_of(p, back) == 4) return launch_width<T, 4>(a, (int)p->K, back, act, p->dw, p->dbias, s);
  return launch_width<T, 1>(a, (int)p->K, back, act, p->dw, p->dbias, s);
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
  const int64_t wide = back_plan(a->T, a->N, a->D, 4).blocks, narrow = back_plan(a->T, a->N, a->D, 1).blocks;
  return sizeof(float) * (size_t)std::max(wide, narrow) * (size_t)((a->K + 1) * a->D);
}

int net_causal_conv(const net_conv* a, void* stream) { return auv::net::run(a, false, stream); }
int net_causal_conv_backward(const net_conv* a, void* stream) { return auv::net::run(a, true, stream); }

}  // extern "C"
