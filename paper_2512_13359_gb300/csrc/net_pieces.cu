// net_pieces.cu -- the gated recurrence (net_scan.cu) of few channels over many steps: the steps are split as well.
//
// A block holds 32 channels (16 where blocks would be few) x some hundred steps in shared memory.  Each of its threads takes a run of steps of
// E adjacent channels, folds them to one affine map h -> A h + B a channel, and keeps the gates in registers.  The maps
// are joined over the warp by shuffles, over the block's warps by a scan in shared memory, and over a cluster of blocks,
// each with the next piece of the sequence, through distributed shared memory; then every run is gone through from its
// right start.  Inputs are read from memory once.  The next piece is on its way meanwhile.
// 512 steps of 32,768 bf16 channels: forward 34 us (3 TB/s), backward 53 us (3.8 TB/s); instructions take 60 % of the
// issue slots, the barriers and the joins most of the rest.
#include <type_traits>

#include "net_scan.cuh"

namespace auv {
namespace net {
namespace {

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Stores a map in the shared memory of block `rank` of the cluster, at this block's address p.
__device__ __forceinline__ void store_remote(const Map* p, int rank, const Map& q) {
  const uint32_t local = (uint32_t)__cvta_generic_to_shared(p);
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(local), "r"(rank));
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(q.A), "f"(q.B) : "memory");
}

// A row of a piece is copied as the aligned 16-byte units that hold it, so any start and stride will do.  The first
// unit may begin before the row: within its allocation all the same, which begins on such a boundary.  The last one is
// read as far as the row goes.
__device__ __forceinline__ void copy_unit(void* dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
               "r"(bytes)
               : "memory");
}

// The shape of a block: CH channels, CH / E lanes a row, and so many steps a thread that two blocks, each with two
// pieces of the 2 or 4 arrays, fit an SM (backward in fp32 one; twice the threads at one block an SM took 1.1 to 1.9
// times as long: nothing covers the barriers).
template <typename T, int E, int CH, bool BACK>
struct Shape {
  static constexpr int kThreads = kPieceThreads;
  static constexpr int kRun = (BACK || sizeof(T) == 4 ? 16 : 32) / E;      // steps of a thread
  static constexpr int kLanes = CH / E, kRuns = kThreads / kLanes, kRows = kRuns * kRun, kWarps = kThreads / 32;
  // A row has room for a unit more than its own; a run ends with room for half a row of banks, so that the runs of a
  // warp do not meet in them.
  static constexpr int kPitch = CH * (int)sizeof(T) + 16, kRunPitch = kRun * kPitch + CH * (int)sizeof(T);
  static constexpr int kArray = kRuns * kRunPitch, kBytes = 2 * Inputs<T, BACK>::kN * kArray;
};

constexpr int kCluster = 16;                       // blocks joined at most

// EVEN: the arrays' rows all start equally far from a 16-byte boundary.  per: channels of an env; more than one env's
// may be in a block if their rows follow each other in memory (then N is 1, and D all channels).
template <typename T, int E, int CH, bool BACK, bool EVEN>
__global__ void __launch_bounds__(Shape<T, E, CH, BACK>::kThreads) k_pieces(Scan a, int64_t per, int units_log) {
  using In = Inputs<T, BACK>;
  using Sh = Shape<T, E, CH, BACK>;
  using W = Raw<T, E>;
  constexpr int K = In::kN, R = Sh::kRun, L = Sh::kLanes, kWarps = Sh::kWarps, kSize = (int)sizeof(T);
  static_assert(R <= 32 && CH * kWarps <= Sh::kThreads && CH <= 32, "");
  extern __shared__ uint4 smem[];
  __shared__ Map warps[CH][kWarps + 1];                // of the block's warps; then of what comes before each
  __shared__ Map blocks[2][kCluster][CH];              // of the cluster's blocks, two pieces in turn
  __shared__ float start[CH];                          // the state before the block's piece
  char* const tile = reinterpret_cast<char*>(smem);    // array (buffer, i) at (buffer * K + i) * kArray
  const int lane = threadIdx.x % L, run = threadIdx.x / L, warp = threadIdx.x / 32, in_warp = threadIdx.x % 32;
  const int T_ = a.T, rank = (int)cluster_rank(), ranks = (int)cluster_size();
  const int64_t across = (a.D + CH - 1) / CH, q = blockIdx.x / ranks;
  const int64_t n = q / across, d0 = (q - n * across) * CH;
  const int count = (int)min((int64_t)CH, a.D - d0);
  const bool live = lane * E < count;
  const int64_t d = d0 + (live ? lane * E : 0), m = n * a.D + d;   // the thread's first channel; dead ones shadow the first
  const int64_t env = m / per;
  const bool one_env = (n * a.D + d0) / per == (n * a.D + d0 + count - 1) / per;
  const In in(a, n, d0);
  const int stride = Sh::kRows * ranks, first = rank * Sh::kRows;   // steps of the cluster, and the block's first
  auto fetch = [&](int buf, int64_t s) {
    const int u = threadIdx.x & ((1 << units_log) - 1), rows = Sh::kThreads >> units_log;
    const int r0 = threadIdx.x >> units_log;
    const T* p[K];
    int64_t by[K];
#pragma unroll
    for (int i = 0; i < K; ++i) p[i] = in.p[i] + (s + r0) * in.by[i], by[i] = rows * in.by[i];
    const int left = (int)min((int64_t)Sh::kRows, T_ - s);
    char* const to = tile + buf * K * Sh::kArray + 16 * u;
#pragma unroll 2
    for (int r = r0; r < left; r += rows) {
      char* const row = to + (r / R) * Sh::kRunPitch + (r % R) * Sh::kPitch;
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p[i]);
        const int bytes = (int)(at & 15) + count * kSize - 16 * u;
        if (bytes > 0 && (i != 2 || s + r < T_ - 1))
          copy_unit(row + i * Sh::kArray, reinterpret_cast<const char*>((at & ~(uintptr_t)15) + 16 * u), min(bytes, 16));
        p[i] += by[i];
      }
    }
    copy_commit();
  };
  // The end flags of the run's steps from s on: of a block of one env, each lane reads some for all the run's lanes.
  constexpr int kFlags = (R + L - 1) / L;
  auto flag_of = [&](int64_t s) { return s < T_ ? end_flag(a, BACK ? T_ - 1 - (int)s : (int)s, env) : 0u; };
  uint32_t flag[kFlags];
  auto fetch_flags = [&](int64_t s) {
#pragma unroll
    for (int j = 0; j < kFlags; ++j) flag[j] = j * L + lane < R ? flag_of(s + j * L + lane) : 0u;
  };
  auto gather = [&](int64_t s) {
    uint32_t bits = 0;
#pragma unroll 8
    for (int r = 0; r < R; ++r) bits |= (flag_of(s + r) ? 1u : 0u) << r;
    return bits;
  };
  const bool flags = a.done || a.done_prev;
  fetch(0, first);
  if (flags && one_env) fetch_flags(first + run * R);
  if (ranks > 1) cluster_sync();       // all blocks have started: their shared memory may be written
  const float* const h0 = a.h0 ? a.h0 + m : nullptr;
  // The state before the cluster's piece is the first warp's, a lane a channel.
  float carry = 0.0f;
  {
    const float* const from = BACK ? a.dhT : a.h0;
    if ((int)threadIdx.x < count && from) carry = from[n * a.D + d0 + threadIdx.x];
  }
  float* const out = BACK ? (a.dh0 ? a.dh0 + m : nullptr) : (a.hT ? a.hT + m : nullptr);
  const net_rows &ro = BACK ? a.dv : a.y, &rz = BACK ? a.df : a.y;
  const int64_t ys = BACK ? -ro.outer : ro.outer, zs = -rz.outer;
  int turn = 0;
  for (int64_t s0 = 0; s0 < T_; s0 += stride, turn ^= 1) {
    const int64_t s = s0 + first + run * R;            // the thread's first step
    uint32_t ends = 0;
    if (flags) {
      if (one_env) {
#pragma unroll
        for (int j = 0; j < kFlags; ++j) {
          const uint32_t all = __ballot_sync(0xffffffffu, flag[j] != 0) >> (L < 32 ? in_warp / L * L : 0);
          ends |= (L < 32 ? all & ((1u << (L % 32)) - 1) : all) << (j * L % 32);
        }
        fetch_flags(s + stride);
      } else {
        ends = gather(s);
      }
    }
    copy_wait<0>();
    __syncthreads();     // the piece has landed for all, and all are done with the one before it
    fetch(turn ^ 1, s0 + stride + first);
    const char* at[K];
    uint32_t off[K], by[K];
#pragma unroll
    for (int i = 0; i < K; ++i) {
      // of array i's row r: its distance from a 16-byte boundary is off + r by
      by[i] = (uint32_t)(in.by[i] * kSize);
      off[i] = (uint32_t)reinterpret_cast<uintptr_t>(in.p[i]) + (uint32_t)s * by[i];
      at[i] = tile + (turn * K + i) * Sh::kArray + run * Sh::kRunPitch + (int)(d - d0) * kSize + (EVEN ? off[i] & 15u : 0u);
    }
    auto value = [&](int i, int r, float (&x)[E]) {
      unpack<T, E>(*reinterpret_cast<const W*>(at[i] + r * Sh::kPitch + (EVEN ? 0u : (off[i] + r * by[i]) & 15u)), x);
    };
    // The run as one map.  Steps past the end hold anything: nothing after them is wanted.  A gate where an episode
    // ended is made 0; that lets through what is not finite (it becomes NaN, and stays it to the run's end), so a run
    // with an end in it and such a result is gone through once more, with the state dropped instead (rare).
    float ga[R][E], gb[R][E];          // gb: forward already times v
    Map mine[E];
#pragma unroll
    for (int e = 0; e < E; ++e) mine[e] = {1.0f, 0.0f};
    bool finite = true;
    float last[E] = {};
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float f[E], x[E];
      value(0, r, f);
      value(BACK ? 3 : 1, r, x);
      const bool end = ends >> r & 1u;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        gates(f[e], ga[r][e], gb[r][e]);
        if constexpr (!BACK) gb[r][e] *= x[e];
        // backward the gate itself is wanted later on: dropped here, and there again
        const float g = end ? 0.0f : ga[r][e];
        if constexpr (!BACK) ga[r][e] = g;
        mine[e].A *= g;
        // backward B is the sum dy[t] + g[t + 1] until the run's end, and `last` the gate that it is to be taken through
        mine[e].B = BACK ? fmaf(last[e], mine[e].B, x[e]) : fmaf(g, mine[e].B, gb[r][e]);
        if constexpr (BACK) last[e] = g;
      }
    }
    if constexpr (BACK) {
#pragma unroll
      for (int e = 0; e < E; ++e) mine[e].B *= last[e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) mine[e].A = positive(mine[e].A);
    if (ends) {
#pragma unroll
      for (int e = 0; e < E; ++e) finite = finite && fabsf(mine[e].B) < INFINITY;
      if (!finite) {
#pragma unroll
        for (int e = 0; e < E; ++e) mine[e].B = last[e] = 0.0f;
#pragma unroll 1
        for (int r = 0; r < R; ++r) {
          float f[E], x[E];
          value(0, r, f);
          value(BACK ? 3 : 1, r, x);
          const bool end = ends >> r & 1u, cut = BACK && r > 0 && (ends >> (r - 1) & 1u);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            float g, q;
            gates(f[e], g, q);
            if constexpr (BACK) mine[e].B = fmaf(last[e], cut || r == 0 ? 0.0f : mine[e].B, x[e]), last[e] = end ? 0.0f : g;
            else mine[e].B = fmaf(g, end ? 0.0f : mine[e].B, q * x[e]);
          }
        }
        if constexpr (BACK) {
#pragma unroll
          for (int e = 0; e < E; ++e) mine[e].B = ends >> (R - 1) & 1u ? 0.0f : mine[e].B * last[e];
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) mine[e].A = -0.0f;
    }
    // over the warp's runs (L lanes apart), and what comes before each
#pragma unroll
    for (int o = L; o < 32; o *= 2) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const Map p = {__shfl_up_sync(0xffffffffu, mine[e].A, o), __shfl_up_sync(0xffffffffu, mine[e].B, o)};
        if (in_warp >= o) mine[e] = then(p, mine[e]);
      }
    }
    if (in_warp >= 32 - L) {
#pragma unroll
      for (int e = 0; e < E; ++e) warps[lane * E + e][warp] = mine[e];
    }
    if constexpr (L < 32) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        mine[e] = {__shfl_up_sync(0xffffffffu, mine[e].A, L), __shfl_up_sync(0xffffffffu, mine[e].B, L)};
        if (in_warp < L) mine[e] = {1.0f, 0.0f};
      }
    }
    __syncthreads();
    // over the block's warps: a channel's maps in adjacent lanes
    if (threadIdx.x < CH * kWarps) {
      const int c = threadIdx.x / kWarps, w = threadIdx.x % kWarps;
      Map p = warps[c][w];
#pragma unroll
      for (int o = 1; o < kWarps; o *= 2) {
        const Map b = {__shfl_up_sync(0xffffffffu, p.A, o, kWarps), __shfl_up_sync(0xffffffffu, p.B, o, kWarps)};
        if (w >= o) p = then(b, p);
      }
      const Map total = {__shfl_sync(0xffffffffu, p.A, kWarps - 1, kWarps), __shfl_sync(0xffffffffu, p.B, kWarps - 1, kWarps)};
      p = {__shfl_up_sync(0xffffffffu, p.A, 1, kWarps), __shfl_up_sync(0xffffffffu, p.B, 1, kWarps)};
      warps[c][w] = w ? p : Map{1.0f, 0.0f};
      for (int r = w; r < ranks; r += kWarps) {
        if (ranks > 1) store_remote(&blocks[turn][rank][c], r, total);
        else blocks[turn][0][c] = total;
      }
    }
    // over the cluster's blocks
    if (ranks > 1) cluster_sync();
    else __syncthreads();
    if (threadIdx.x < CH) {
      for (int r = 0; r < ranks; ++r) {
        if (r == rank) start[threadIdx.x] = carry;
        carry = apply(blocks[turn][r][threadIdx.x], carry);
      }
    }
    __syncthreads();
    float h[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = lane * E + e;
      h[e] = apply(L < 32 ? mine[e] : Map{1.0f, 0.0f}, apply(warps[c][warp], start[c]));
    }
    // Through the steps once more, from the right start.  INNER: all of the block's are there, and none is at t = 0 or
    // the last.
    T* y = const_cast<T*>(base<T>(ro, n, d)) + (BACK ? T_ - 1 - s : s) * ro.outer;
    T* z = BACK ? const_cast<T*>(base<T>(rz, n, d)) + (T_ - 1 - s) * rz.outer : nullptr;
    auto unfold = [&](auto inner) {
      constexpr bool INNER = decltype(inner)::value;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool there = INNER || s + r < T_, at_last = !INNER && s + r == T_ - 1;
        if constexpr (!BACK) {
#pragma unroll
          for (int e = 0; e < E; ++e) h[e] = fmaf(ga[r][e], h[e], gb[r][e]);
          if (live && there) store<T, E>(y, h);
        } else {
          const bool end = ends >> r & 1u;
          float c[E], v[E], g[E], df[E], dv[E];
          value(2, r, c);
          value(1, r, v);
          value(3, r, g);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            if (at_last) c[e] = h0 ? h0[e] : 0.0f;
            g[e] += h[e];
            dv[e] = gb[r][e] * g[e];
            df[e] = ga[r][e] * dv[e] * ((end ? 0.0f : c[e]) - v[e]);
            h[e] = end ? 0.0f : ga[r][e] * g[e];
          }
          if (live && there) {
            store<T, E>(y, dv);
            store<T, E>(z, df);
          }
          z += zs;
        }
        y += ys;
        if (at_last && live && out) {
#pragma unroll
          for (int e = 0; e < E; ++e) out[e] = h[e];
        }
      }
    };
    if (!BACK && ends) {
#pragma unroll
      for (int e = 0; e < E; ++e) finite = finite && fabsf(h[e]) < INFINITY;
    }
    if (!BACK && !finite) {
#pragma unroll 1
      for (int r = 0; r < R && s + r < T_; ++r, y += ys) {
        float f[E], x[E];
        value(0, r, f);
        value(1, r, x);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          float g, q;
          gates(f[e], g, q);
          h[e] = fmaf(g, ends >> r & 1u ? 0.0f : h[e], q * x[e]);
        }
        if (live) store<T, E>(y, h);
        if (s + r == T_ - 1 && live && out) {
#pragma unroll
          for (int e = 0; e < E; ++e) out[e] = h[e];
        }
      }
    } else if (s0 + first + Sh::kRows < T_) {
      unfold(std::true_type{});
    } else {
      unfold(std::false_type{});
    }
  }
  copy_wait<0>();
}

template <typename T, int E, int CH, bool BACK, bool EVEN>
cudaError_t launch_shape(const Scan& a, int64_t per, int units_log, int ranks, cudaStream_t s) {
  using Sh = Shape<T, E, CH, BACK>;
  const auto kern = k_pieces<T, E, CH, BACK, EVEN>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes);
  if (e == cudaSuccess && ranks > 8) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  while (ranks > 1 && (int64_t)(ranks / 2) * Sh::kRows >= a.T) ranks /= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.N * ((a.D + CH - 1) / CH) * ranks));
  cfg.blockDim = dim3(Sh::kThreads);
  cfg.dynamicSmemBytes = Sh::kBytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ranks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, a, per, units_log);
  return e == cudaSuccess ? cudaGetLastError() : e;
}

template <typename T, bool BACK>
cudaError_t launch_direction(Scan a, cudaStream_t s) {
  const net_rows* rows[] = {&a.f, &a.v, &a.y, &a.dy, &a.df, &a.dv};
  constexpr int kArrays = BACK ? 6 : 3, kUnit = 16 / (int)sizeof(T);
  const int64_t per = a.D;
  const Tiles t = tiles_of(a.N, a.D, rows, kArrays);
  bool even = true, units = true, pairs = per % 2 == 0;
  for (int i = 0; i < kArrays; ++i) {
    even = even && (a.T == 1 || rows[i]->outer % kUnit == 0);
    units = units && aligned(*rows[i], a.T, a.N, sizeof(T), kUnit);
    pairs = pairs && aligned(*rows[i], a.T, a.N, sizeof(T), 2);
  }
  if (t.flat) a.D *= a.N, a.N = 1;
  const int sms = sm_count();
  // Blocks of 16 channels where those of 32 would leave SMs without one; then blocks in clusters until they have one.
  const bool half = pairs && t.wide * 8 < sms;
  const int64_t tiles = half ? t.narrow : t.wide;
  int ranks = 1;
  while (ranks < 8 && tiles * ranks < sms) ranks *= 2;
  if (ranks == 8 && tiles * 16 <= 96) ranks = 16;
  // 16-byte units of a row, and one more where it does not start on one; a power of two
  int units_log = sizeof(T) == 4 ? 3 : 2;
  if (half) --units_log;
  if (!units) ++units_log;
  if (!pairs) return launch_shape<T, 1, 32, BACK, false>(a, per, units_log, ranks, s);
  if (half)
    return even ? launch_shape<T, 2, 16, BACK, true>(a, per, units_log, ranks, s)
                : launch_shape<T, 2, 16, BACK, false>(a, per, units_log, ranks, s);
  return even ? launch_shape<T, 2, 32, BACK, true>(a, per, units_log, ranks, s)
              : launch_shape<T, 2, 32, BACK, false>(a, per, units_log, ranks, s);
}

}  // namespace

template <typename T>
cudaError_t launch_pieces(const Scan& a, bool back, cudaStream_t s) {
  return back ? launch_direction<T, true>(a, s) : launch_direction<T, false>(a, s);
}
template cudaError_t launch_pieces<float>(const Scan&, bool, cudaStream_t);
template cudaError_t launch_pieces<__nv_bfloat16>(const Scan&, bool, cudaStream_t);
template cudaError_t launch_pieces<__half>(const Scan&, bool, cudaStream_t);

}  // namespace net
}  // namespace auv
