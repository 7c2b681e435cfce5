// net_scan.cu -- gated linear recurrence along a trajectory (auvnet.h, net_gate_scan).
//
// h[t] = a c[t] + b v[t] with a = sigmoid(f[t]), b = 1 - a, c[t] = h[t - 1] or 0 where an episode ended: per channel a
// chain of affine maps.  The backward pass is the same chain from the last step to the first, in g[t], the gradient of
// c[t]: d[t] = dy[t] + g[t + 1], g[t] = a d[t] or 0.  Both move bytes and compute little (3 arrays of T N D forward, 6
// backward), so two kernels share the work by how much parallelism the channels give:
//
//  k_steps  one thread per E adjacent channels walks the steps.  Its inputs of the next 8 steps are on their way to
//           shared memory (cp.async to slots of its own: no barrier), so few threads keep HBM busy.  4,096 envs x 256
//           channels x 128 steps of bf16: forward 127 us (6.4 TB/s), backward 247 us (6.6 TB/s).
//  k_one    the same for a single step (65,536 envs x 256 channels of bf16: 34.4 us, 6.8 TB/s).
//  k_steps, k_join, k_steps: few channels, many steps: pieces of the sequence are folded to affine maps h -> A h + B,
//           the maps joined to the states before the pieces, and the pieces walked from those.
//  k_pieces few channels, fewer steps: both in one kernel, with the inputs read once (net_pieces.cu).
#include <algorithm>

#include "net_scan.cuh"

namespace auv {
namespace net {
namespace {

template <int E>
__device__ __forceinline__ void load_state(const float* p, float (&x)[E]) {
  if (p && E >= 4 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
#pragma unroll
    for (int e = 0; e + 3 < E; e += 4) {
      const float4 w = *reinterpret_cast<const float4*>(p + e);
      x[e] = w.x, x[e + 1] = w.y, x[e + 2] = w.z, x[e + 3] = w.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = p ? p[e] : 0.0f;
  }
}
template <int E>
__device__ __forceinline__ void store_state(float* p, const float (&x)[E]) {
  if (E >= 4 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
#pragma unroll
    for (int e = 0; e + 3 < E; e += 4) *reinterpret_cast<float4*>(p + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) p[e] = x[e];
  }
}

// One step of E channels: h (forward) or g (backward) is taken through it and its outputs are stored at y, or dv and
// df.  before: the state before step 0, asked for at that step alone (first).  ends: bit e for channel e.
template <typename T, int E, bool BACK>
__device__ __forceinline__ void step(const float (&ga)[E], const float (&gb)[E], const Raw<T, E>& rv, const Raw<T, E>& ry,
                                     const Raw<T, E>& rdy, bool first, const float* before, uint32_t ends, T* y, T* z,
                                     float (&h)[E]) {
  float v[E];
  unpack<T, E>(rv, v);
  if constexpr (!BACK) {
#pragma unroll
    for (int e = 0; e < E; ++e) h[e] = fmaf(ga[e], ends >> e & 1u ? 0.0f : h[e], gb[e] * v[e]);
    store<T, E>(y, h);
  } else {
    float c[E], dy[E], df[E], dv[E];
    if (!first) unpack<T, E>(ry, c);
    else load_state<E>(before, c);
    unpack<T, E>(rdy, dy);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool end = ends >> e & 1u;
      const float q = dy[e] + h[e];
      dv[e] = gb[e] * q;
      df[e] = ga[e] * dv[e] * ((end ? 0.0f : c[e]) - v[e]);
      h[e] = end ? 0.0f : ga[e] * q;
    }
    store<T, E>(y, dv);
    store<T, E>(z, df);
  }
}

// Whose flags a thread's channels follow: those of its first channel's env, and of the next env from some channel on
// (MIXED: arrays whose rows follow each other in memory are taken as one row, whose pieces may belong to two envs).
template <int E, bool MIXED>
struct Owner {
  int64_t env;
  uint32_t second;      // bits of the channels of the next env
  __device__ Owner(int64_t first, int64_t per) {
    env = first / per;
    const int split = (int)min((int64_t)E, (env + 1) * per - first);
    second = MIXED ? ((1u << E) - 1) & ~((1u << split) - 1) : 0u;
  }
  // The flags of step t as they are in memory, and from them bit e: channel e's episode ended before it.  Apart, since
  // the first is done long before the second: nothing may wait for the load in between.
  __device__ uint32_t load(const Scan& a, int t) const {
    const uint32_t one = end_flag(a, t, env);
    if constexpr (MIXED) return second ? one | end_flag(a, t, env + 1) << 8 : one;
    return one;
  }
  __device__ uint32_t ends(uint32_t flag) const {
    if constexpr (MIXED) return ((flag & 255u) ? ((1u << E) - 1) & ~second : 0u) | (flag >> 8 ? second : 0u);
    return flag ? (1u << E) - 1 : 0u;
  }
};

// T = 1, a rollout's step: nothing to walk, so few registers and many threads.
template <typename T, int E, bool BACK, bool MIXED>
__global__ void __launch_bounds__(256) k_one(Scan a, int64_t width) {
  const int64_t m = blockIdx.x * (int64_t)256 + threadIdx.x, per = a.D / E;
  if (m >= a.N * per) return;
  const int64_t n = m / per, d = (m - n * per) * E;
  using W = Raw<T, E>;
  auto get = [&](const net_rows& r) { return *reinterpret_cast<const W*>(base<T>(r, n, d)); };
  const W rf = get(a.f), rv = get(a.v), rdy = BACK ? get(a.dy) : rf;
  const float* const from = BACK ? a.dhT : a.h0;
  float h[E], f[E], ga[E], gb[E];
  load_state<E>(from ? from + m * E : nullptr, h);
  const Owner<E, MIXED> owner(m * E, width);
  const uint32_t ends = owner.ends(owner.load(a, 0));
  unpack<T, E>(rf, f);
#pragma unroll
  for (int e = 0; e < E; ++e) gates(f[e], ga[e], gb[e]);
  step<T, E, BACK>(ga, gb, rv, rv, rdy, true, a.h0 ? a.h0 + m * E : nullptr, ends,
                   const_cast<T*>(base<T>(BACK ? a.dv : a.y, n, d)), BACK ? const_cast<T*>(base<T>(a.df, n, d)) : nullptr,
                   h);
  float* const out = BACK ? a.dh0 : a.hT;
  if (out) store_state<E>(out + m * E, h);
}

constexpr int kStepThreads = 128;
// Steps on their way: of narrow pieces more, since few channels make few threads.
template <int E> constexpr int kAheadOf = E >= 4 ? 8 : 16;
// Steps whose gates are computed side by side before the chain runs through them: narrow pieces, of which few channels
// make few warps, wait for each other's latency otherwise.
template <int E> constexpr int kGroup = E == 4 ? 2 : 4;

// A sequence in pieces of `rows` steps: the maps of the pieces' channels, A [pieces][m] and B [pieces][m]; after k_join, B
// holds the states before the pieces.  A block takes adjacent pieces, `lanes` (a power of two) threads each.  One piece:
// rows = T, maps NULL.
struct Split {
  int rows, pieces, lanes;
  int64_t m;
  float* maps;
};

// SPLIT: in pieces, one a block (1) or several of few channels (2: their steps are then in no uniform registers, which
// takes 5 to 10 % longer where a piece fills the block).  FOLD: only their maps.
template <typename T, int E, bool BACK, bool MIXED, int SPLIT, bool FOLD>
__global__ void __launch_bounds__(kStepThreads) k_steps(Scan a, int64_t width, Split split) {
  using W = Raw<T, E>;
  using In = Inputs<T, BACK>;
  constexpr int K = In::kN, kAhead = kAsync<T, E> ? kAheadOf<E> : 8, kG = kAsync<T, E> ? kGroup<E> : kAhead;
  constexpr int kHeld = FOLD ? 2 : K;                          // arrays read: folding f, and v or dy
  constexpr int kX = FOLD && BACK ? 3 : 1;
  extern __shared__ uint4 smem[];
  W* const ring = reinterpret_cast<W*>(smem) + threadIdx.x;    // slot (u, i) at (u * kHeld + i) * kStepThreads
  const int lanes = SPLIT == 2 ? split.lanes : kStepThreads, lane = SPLIT == 2 ? threadIdx.x & (lanes - 1) : threadIdx.x;
  const int piece = SPLIT == 2 ? blockIdx.y * (kStepThreads / lanes) + threadIdx.x / lanes : SPLIT ? blockIdx.y : 0;
  const int64_t m = blockIdx.x * (int64_t)lanes + lane, per = a.D / E;
  if (m >= a.N * per || (SPLIT == 2 && piece >= split.pieces)) return;
  const int64_t n = m / per, d = (m - n * per) * E;
  In in(a, n, d);
  // steps before the piece, and its own
  const int skip = SPLIT ? piece * split.rows : 0, steps = SPLIT ? min(split.rows, a.T - skip) : a.T;
  if constexpr (SPLIT) {
#pragma unroll
    for (int i = 0; i < K; ++i) in.p[i] += skip * in.by[i];
  }
  static_assert(kAhead * E <= 32, "the flags of a round are one word");
  [[maybe_unused]] W reg[kAhead][kHeld];
  auto fetch = [&](int u, int s) {      // the piece's s-th step in the chain's order, one after the other
    if (s < steps) {
#pragma unroll
      for (int j = 0; j < kHeld; ++j) {
        const int i = j == 1 ? kX : j;
        if (i != 2 || skip + s < a.T - 1) {
          if constexpr (kAsync<T, E>) copy_async<sizeof(W)>(ring + (u * kHeld + j) * kStepThreads, in.p[i]);
          else reg[u][j] = *reinterpret_cast<const W*>(in.p[i]);
        }
        in.p[i] += in.by[i];
      }
    }
  };
  const bool flags = a.done || a.done_prev;
  const Owner<E, MIXED> owner(m * E, width);
  auto flag_of = [&](int s) { return flags && s < steps ? owner.load(a, BACK ? a.T - 1 - skip - s : skip + s) : 0u; };
  uint32_t flag[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    fetch(u, u);
    if (kAsync<T, E> && u % kG == kG - 1) copy_commit();
    flag[u] = flag_of(u);
  }
  float* const maps = SPLIT ? split.maps + piece * split.m + m * E : nullptr;
  const int64_t to_b = SPLIT ? split.pieces * split.m : 0;
  float h[E];
  [[maybe_unused]] Map q[E];
  if constexpr (FOLD) {
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = {1.0f, 0.0f};
  } else if constexpr (SPLIT) {
    after_previous();
    load_state<E>(maps + to_b, h);
  } else {
    load_state<E>(BACK ? (a.dhT ? a.dhT + m * E : nullptr) : (a.h0 ? a.h0 + m * E : nullptr), h);
  }
  const float* const h0 = a.h0 ? a.h0 + m * E : nullptr;
  const net_rows &ro = BACK ? a.dv : a.y, &rz = BACK ? a.df : a.y;
  T* y = const_cast<T*>(base<T>(ro, n, d)) + (BACK ? a.T - 1 - skip : skip) * ro.outer;
  T* z = BACK ? const_cast<T*>(base<T>(rz, n, d)) + (a.T - 1 - skip) * rz.outer : nullptr;
  const int64_t ys = BACK ? -ro.outer : ro.outer, zs = -rz.outer;
  for (int s0 = 0; s0 < steps; s0 += kAhead) {
    uint32_t ends = 0;
    if (flags) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) ends |= owner.ends(flag[u]) << (u * E);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) flag[u] = flag_of(s0 + kAhead + u);
    }
#pragma unroll
    for (int u0 = 0; u0 < kAhead; u0 += kG) {
      if (s0 + u0 >= steps) break;
      W w[kG][kHeld];
      if constexpr (kAsync<T, E>) copy_wait<kAhead / kG - 1>();
#pragma unroll
      for (int u = 0; u < kG; ++u)
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
          if constexpr (kAsync<T, E>) w[u][i] = ring[((u0 + u) * kHeld + i) * kStepThreads];
          else w[u][i] = reg[u][i];
        }
#pragma unroll
      for (int u = 0; u < kG; ++u) fetch(u0 + u, s0 + u0 + u + kAhead);
      if constexpr (kAsync<T, E>) copy_commit();
      float ga[kG][E], gb[kG][E];
#pragma unroll
      for (int u = 0; u < kG; ++u) {
        float f[E];
        unpack<T, E>(w[u][0], f);
#pragma unroll
        for (int e = 0; e < E; ++e) gates(f[e], ga[u][e], gb[u][e]);
      }
#pragma unroll
      for (int u = 0; u < kG; ++u) {
        const int s = s0 + u0 + u;
        const uint32_t end = ends >> ((u0 + u) * E);
        if (s < steps) {
          if constexpr (FOLD) {
            float x[E];
            unpack<T, E>(w[u][1], x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const bool cut = end >> e & 1u;
              if constexpr (BACK) q[e].B = cut ? 0.0f : ga[u][e] * (x[e] + q[e].B);
              else q[e].B = fmaf(ga[u][e], cut ? 0.0f : q[e].B, gb[u][e] * x[e]);
              q[e].A = cut ? -0.0f : q[e].A * ga[u][e];
            }
          } else {
            step<T, E, BACK>(ga[u], gb[u], w[u][1], w[u][BACK ? 2 : 0], w[u][BACK ? 3 : 0], skip + s == a.T - 1, h0, end, y,
                             z, h);
            y += ys;
            if constexpr (BACK) z += zs;
          }
        }
      }
    }
  }
  if constexpr (kAsync<T, E>) copy_wait<0>();
  if constexpr (FOLD) {
#pragma unroll
    for (int e = 0; e < E; ++e) h[e] = positive(q[e].A);
    store_state<E>(maps, h);
#pragma unroll
    for (int e = 0; e < E; ++e) h[e] = q[e].B;
    store_state<E>(maps + to_b, h);
  } else {
    float* const out = BACK ? a.dh0 : a.hT;
    if (out && skip + steps == a.T) store_state<E>(out + m * E, h);
  }
}

// The states before the pieces, in the place of B.  A block has 8 channels and all pieces: each of its 128 groups of 8
// lanes at most 16 adjacent pieces, whose maps it reads once (1,986 pieces of 250 channels: 16 us when it read them
// twice, 8 at a time).
constexpr int kJoinThreads = 1024, kJoinChannels = 8, kJoinGroups = kJoinThreads / kJoinChannels, kJoinHeld = 16;
constexpr int kMostPieces = kJoinGroups * kJoinHeld;
__global__ void __launch_bounds__(kJoinThreads) k_join(int pieces, int64_t m, float* maps, const float* from) {
  __shared__ Map warps[kJoinThreads / 32][kJoinChannels];
  after_previous();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, group = threadIdx.x / kJoinChannels;
  const int k = threadIdx.x % kJoinChannels;
  const int64_t c = blockIdx.x * (int64_t)kJoinChannels + k;
  const bool live = c < m;
  const int each = (pieces + kJoinGroups - 1) / kJoinGroups, p0 = min(pieces, group * each);
  const float* const A = maps + p0 * m + c;
  float* const B = maps + (pieces + (int64_t)p0) * m + c;
  const int n = live ? min(pieces, p0 + each) - p0 : 0;
  Map held[kJoinHeld];
#pragma unroll
  for (int i = 0; i < kJoinHeld; ++i) held[i] = i < n ? Map{A[i * m], B[i * m]} : Map{1.0f, 0.0f};
  Map q = {1.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kJoinHeld; ++i) q = then(q, held[i]);
#pragma unroll
  for (int o = kJoinChannels; o < 32; o *= 2) {
    const Map r = {__shfl_up_sync(0xffffffffu, q.A, o), __shfl_up_sync(0xffffffffu, q.B, o)};
    if (lane >= o) q = then(r, q);
  }
  if (lane >= 32 - kJoinChannels) warps[warp][k] = q;
  q = {__shfl_up_sync(0xffffffffu, q.A, kJoinChannels), __shfl_up_sync(0xffffffffu, q.B, kJoinChannels)};
  __syncthreads();
  float h = live && from ? from[c] : 0.0f;
  for (int w = 0; w < warp; ++w) h = apply(warps[w][k], h);
  if (lane >= kJoinChannels) h = apply(q, h);
#pragma unroll
  for (int i = 0; i < kJoinHeld; ++i) {
    if (i < n) B[i * m] = h;
    h = apply(held[i], h);
  }
}

// How the steps are gone through, by what each way costs (measured, in ns):
//  walked by a thread a channel or more: 100 a step forward, 190 backward, whatever the channels (up to HBM's pace);
//  in blocks, or clusters of them where channels are few (net_pieces.cu): 3,300 to 4,600 for every round of blocks, of
//    32 channels x 256 steps each (128 in fp32 and backward), that fit the SMs, two each (one backward in fp32; clusters
//    fill less of the device).  512 steps of bf16 forward, walked and so: 32,768 channels 49 and 34 us, 131,072 channels
//    87 and 121.  Rows that do not follow each other make a tile of their own however narrow they are: 512 steps of
//    4,096 envs x 8 channels as halves of one projection 51 and 103, 1,000 steps of 100 x 8 73 and 10;
//  in pieces whose maps are written, joined and walked from, where channels are few: 14,000, and their inputs twice, at
//    6 TB/s.  65,536 steps of 256 bf16 channels: 4,960 us walked, 74 in clusters, 49 so; 8,192 of 500: 18.6 in
//    clusters, 20 so; 8,192 of 64 envs x 1 fp32, halves of one projection: 532, 49 and 17.
enum class Way { kWalk, kBlocks, kPieces };
Way way_of(int T, int64_t m, const Tiles& t, int size, bool back) {
  if (T < 32) return Way::kWalk;
  const int64_t sms = sm_count(), tiles = t.wide;
  const bool clusters = tiles * 8 < sms, few = (m + 31) / 32 * 8 < sms, large = back && size == 4;
  const int64_t rows = back || size == 4 ? 128 : 256;
  const int64_t blocks = clusters ? std::min<int64_t>(128, t.narrow * 8) : large ? sms : 2 * sms;
  const double round = large ? (clusters ? 6600 : 3300) : back ? 3900 : size == 4 ? 3300 : 4600;
  const double walk = (double)T * (back ? 190 : 100);
  const double held = round * (double)((tiles * ((T + rows - 1) / rows) + blocks - 1) / blocks);
  const double pieces = 14000.0 + (double)T * (double)m * size * (back ? 8 : 5) / 6000.0;
  const bool split = few && pieces < held;
  if (walk <= (split ? pieces : held)) return Way::kWalk;
  return split ? Way::kPieces : Way::kBlocks;
}

// The pieces: for 1,024 threads an SM, of 32 steps at least.
Split split_of(int T, int64_t m, float* ws) {
  const int64_t threads = std::max<int64_t>(1, m / 4);
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>((int64_t)sm_count() * 1024 / threads, std::min(kMostPieces, T / 32)));
  const int rows = (int)((T + want - 1) / want);
  return {rows, (int)(((int64_t)T + rows - 1) / rows), kStepThreads, m, ws};
}

template <typename T, int E, bool BACK, bool MIXED, int SPLIT, bool FOLD>
cudaError_t launch_steps(const Scan& a, int64_t width, const Split& split, cudaStream_t s) {
  const int64_t blocks = (a.N * (a.D / E) + split.lanes - 1) / split.lanes;
  // slots: of a short sequence as many as it has steps, whole groups of them (a group is read whole)
  constexpr int kAhead = kAheadOf<E>, kG = kGroup<E>;
  const int ahead = split.rows < kAhead ? (split.rows + kG - 1) / kG * kG : kAhead;
  const int held = FOLD ? 2 : Inputs<T, BACK>::kN;
  const int smem = kAsync<T, E> ? ahead * held * kStepThreads * (int)sizeof(T) * E : 0;
  const auto kern = k_steps<T, E, BACK, MIXED, SPLIT, FOLD>;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
  }
  const int side = kStepThreads / split.lanes;   // pieces of a block
  const dim3 grid((unsigned)blocks, (unsigned)((split.pieces + side - 1) / side));
  if (SPLIT && !FOLD) return launch_after(kern, grid, kStepThreads, smem, s, a, width, split);
  kern<<<grid, kStepThreads, smem, s>>>(a, width, split);
  return cudaGetLastError();
}

template <typename T, int E, bool BACK, bool MIXED>
cudaError_t launch_walk(const Scan& a, int64_t width, const Split& split, cudaStream_t s) {
  if (a.T == 1) {
    k_one<T, E, BACK, MIXED><<<(unsigned)((a.N * (a.D / E) + 255) / 256), 256, 0, s>>>(a, width);
    return cudaGetLastError();
  }
  if constexpr (E <= 4) {
    if (!split.maps) return launch_steps<T, E, BACK, MIXED, 0, false>(a, width, split, s);
    Split p = split;
    const int64_t threads = a.N * (a.D / E);
    while (p.lanes > 8 && threads <= p.lanes / 2) p.lanes /= 2;
    const bool whole = p.lanes == kStepThreads;
    cudaError_t e = whole ? launch_steps<T, E, BACK, MIXED, 1, true>(a, width, p, s)
                          : launch_steps<T, E, BACK, MIXED, 2, true>(a, width, p, s);
    if (e != cudaSuccess) return e;
    e = launch_after(k_join, dim3((unsigned)((p.m + kJoinChannels - 1) / kJoinChannels)), kJoinThreads, 0, s, p.pieces, p.m,
                     p.maps, BACK ? a.dhT : a.h0);
    if (e != cudaSuccess) return e;
    return whole ? launch_steps<T, E, BACK, MIXED, 1, false>(a, width, p, s)
                 : launch_steps<T, E, BACK, MIXED, 2, false>(a, width, p, s);
  } else {
    return cudaErrorInvalidValue;   // not asked for
  }
}

template <typename T, bool BACK, bool MIXED>
cudaError_t launch_width(const Scan& a, int64_t width, int e, const Split& split, cudaStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (e == 8) return launch_walk<T, 8, BACK, MIXED>(a, width, split, s);
  if (e == 4) return launch_walk<T, 4, BACK, MIXED>(a, width, split, s);
  if (e == 2) return launch_walk<T, 2, BACK, MIXED>(a, width, split, s);
  return launch_walk<T, 1, BACK, false>(a, width, split, s);
}

// T = 0: the state passes as it is.
__global__ void k_none(int64_t m, const float* from, float* to) {
  const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
  if (i < m) to[i] = from ? from[i] : 0.0f;
}

template <typename T, bool BACK>
cudaError_t launch(const Scan& a, float* ws, cudaStream_t s) {
  const int64_t m = a.N * a.D, sms = sm_count();
  if (a.T == 0) {
    float* const to = BACK ? a.dh0 : a.hT;
    if (to) k_none<<<(unsigned)((m + 255) / 256), 256, 0, s>>>(m, BACK ? a.dhT : a.h0, to);
    return cudaGetLastError();
  }
  // Channels of a thread: for one step as many as 16 bytes hold; over many steps four, since half as many bytes a
  // thread make twice the threads (4,096 envs x 256 channels x 128 steps of bf16: 127 us, 137 with eight), and two
  // where four would leave fewer than 160 threads an SM (512 steps, 65,536 channels: 55 us, 75 with four; 131,072: 99
  // and 86).
  const net_rows* rows[] = {&a.f, &a.v, &a.y, &a.dy, &a.df, &a.dv};
  constexpr int kArrays = BACK ? 6 : 3;
  const Way way = way_of(a.T, m, tiles_of(a.N, a.D, rows, kArrays), sizeof(T), BACK);
  if (way == Way::kBlocks) return launch_pieces<T>(a, BACK, s);
  const Split split = way == Way::kPieces ? split_of(a.T, m, ws) : Split{a.T, 1, kStepThreads, m, nullptr};
  int most = 16 / (int)sizeof(T);
  if (a.T > 1) most = split.maps || m >= 4 * 160 * sms ? 4 : 2;
  auto fits = [&](int e, int64_t n) {
    for (int i = 0; i < kArrays; ++i)
      if (!aligned(*rows[i], a.T, n, sizeof(T), e)) return false;
    return true;
  };
  // Rows that follow each other in every array are one row.
  Scan flat = a;
  bool one_row = a.N > 1;
  for (int i = 0; i < kArrays; ++i) one_row = one_row && rows[i]->inner == a.D;
  flat.D = m, flat.N = 1;
  for (int e = most; e > 1; e /= 2) {
    if (a.D % e == 0 && fits(e, a.N)) return launch_width<T, BACK, false>(a, a.D, e, split, s);
    if (one_row && m % e == 0 && a.D >= e && fits(e, 1)) return launch_width<T, BACK, true>(flat, a.D, e, split, s);
  }
  return launch_width<T, BACK, false>(a, a.D, 1, split, s);
}

int check(const net_scan* p) {
  if (!p) return fail(AUV_ERR_INVALID, "argument block is NULL");
  if (p->struct_size != sizeof(net_scan))
    return fail(AUV_ERR_INVALID, "struct_size %u, expected %zu", p->struct_size, sizeof(net_scan));
  if (p->dtype > NET_FP16) return fail(AUV_ERR_INVALID, "dtype %u unknown", p->dtype);
  if (p->T < 0 || p->N < 0 || p->D < 0) return fail(AUV_ERR_INVALID, "negative size");
  const int64_t most = (int64_t)1 << 37;   // channels of a call: blocks stay below 2^31
  if (p->N > most || p->D > most || (p->N && p->D > most / p->N) || p->T > (1 << 30))
    return fail(AUV_ERR_UNSUPPORTED, "N * D past 2^37 or T past 2^30");
  return AUV_OK;
}

int run(const net_scan* p, bool back, void* stream) {
  int rc = check(p);
  if (rc) return rc;
  const int64_t M = p->N * p->D;
  if (M == 0) return AUV_OK;
  const int z = type_size(p->dtype);
  struct { const net_rows* r; const char* name; bool out, back; } rows[] = {
      {&p->f, "f", false, false}, {&p->v, "v", false, false}, {&p->y, "y", !back, false},
      {&p->dy, "dy", false, true}, {&p->df, "df", true, true}, {&p->dv, "dv", true, true}};
  if (p->T)
    for (const auto& q : rows)
      if ((back || !q.back) && (rc = need_rows(*q.r, q.name, p->T, p->N, p->D, z, q.out))) return rc;
  struct { const void* p; const char* name; size_t align; bool used; } flat[] = {
      {p->h0, "h0", 4, true}, {p->hT, "hT", 4, !back}, {p->dhT, "dhT", 4, back}, {p->dh0, "dh0", 4, back},
      {p->done, "done", 1, true}, {p->done_prev, "done_prev", 1, true}};
  for (const auto& q : flat)
    if (q.p && q.used && (rc = need(q.p, q.name, q.align))) return rc;
  const Scan a = {(int)p->T, p->N, p->D, p->f, p->v, p->y, p->dy, p->df, p->dv, p->h0, p->hT, p->dhT, p->dh0, p->done,
                  p->done_prev, p->N};
  const size_t bytes = net_gate_scan_workspace_bytes(p, back);
  if (bytes) {
    if (p->workspace_bytes < bytes) return fail(AUV_ERR_SIZE, "workspace of %zu bytes, %zu needed", p->workspace_bytes, bytes);
    if ((rc = need(p->workspace, "workspace", 16))) return rc;
  }
  float* const ws = static_cast<float*>(p->workspace);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (back)
    e = p->dtype == NET_FP32   ? launch<float, true>(a, ws, s)
        : p->dtype == NET_BF16 ? launch<__nv_bfloat16, true>(a, ws, s)
                               : launch<__half, true>(a, ws, s);
  else
    e = p->dtype == NET_FP32   ? launch<float, false>(a, ws, s)
        : p->dtype == NET_BF16 ? launch<__nv_bfloat16, false>(a, ws, s)
                               : launch<__half, false>(a, ws, s);
  return e == cudaSuccess ? AUV_OK : cuda_fail(e, back ? "net_gate_scan_backward" : "net_gate_scan");
}

}  // namespace
}  // namespace net
}  // namespace auv

extern "C" {

size_t net_gate_scan_workspace_bytes(const net_scan* a, int backward) {
  using namespace auv::net;
  if (!a || check(a) || !a->T || !a->N || !a->D) return 0;
  const int64_t m = a->N * a->D;
  const net_rows* const rows[] = {&a->f, &a->v, &a->y, &a->dy, &a->df, &a->dv};
  const int arrays = backward ? 6 : 3;
  auto split = [&](const Tiles& t) { return way_of((int)a->T, m, t, type_size(a->dtype), backward) == Way::kPieces; };
  bool there = true;
  for (int i = 0; i < arrays; ++i) there = there && rows[i]->data;
  if (!(there ? split(tiles_of(a->N, a->D, rows, arrays)) : split(tiles(a->N, a->D, true)) || split(tiles(a->N, a->D, false))))
    return 0;
  return sizeof(float) * 2 * (size_t)split_of((int)a->T, m, nullptr).pieces * (size_t)m;
}

int net_gate_scan(const net_scan* a, void* stream) { return auv::net::run(a, false, stream); }
int net_gate_scan_backward(const net_scan* a, void* stream) { return auv::net::run(a, true, stream); }

}  // extern "C"
