// net_norm.cu -- group norm with an activation, channels last (auvnet.h, net_group_norm).
//
// Two arrays of B S C forward, three backward, and a reduction over each group (S positions x C / G channels) before
// the elements can be finished: bytes again, if they are read once.
//
//  k_team, k_team_back      groups of a few thousand values: a team of lanes (of a warp, or a whole block) keeps a group
//                           in registers and goes from instance to instance.  A team's channels stay the same, so the
//                           backward pass sums dgamma and dbeta in registers and joins them once at its end.  65,536 x
//                           256 bf16, one group: forward 12.8 us (5.2 TB/s; half of it issuing instructions), backward
//                           28 us (3.6 TB/s; it waits for loads: 60 registers of weights and their sums leave two blocks
//                           an SM, 16 warps).
//  k_slab, k_slab_back      larger groups, as long as a cluster of blocks holds some adjacent ones of an instance in shared
//                           memory, each block some positions: statistics are joined through distributed shared memory.
//                           64 x 4,096 x 256 bf16, 32 groups: forward 60 us (4.5 TB/s), backward 136 us (3 TB/s): a block
//                           loads, joins and stores in turn, and three an SM cover that by half (issue slots 50 %).
//  k_part, k_stats, k_apply the rest: sums by chunk and channel, joined, and the elements read once more.  65,536 x 256
//  (.._back)                bf16 as one instance of 8 groups: forward 35 us, backward 63 us; as one group, whose chunks a
//                           single block joins, 108 and 100.
//
// Variances are those of deviations: in registers from the mean, else of up to 32 values from the first of them, joined
// by the distances of the means (Chan et al.).  All sums have a fixed order.
#include <algorithm>

#include "net_common.cuh"

namespace auv {
namespace net {
namespace {

struct Norm {
  int64_t B, S, C, G;
  net_rows x, y, dy, dx;
  const float *gamma, *beta;
  float *mean, *rstd, *dgamma, *dbeta;
  float eps;
  uint32_t act;
};

// Pairs of fp32 operations in one instruction, where there are pairs.
template <int E>
__device__ __forceinline__ void mul(float (&x)[E], const float (&y)[E]) {
  if constexpr (E == 1) {
    x[0] *= y[0];
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 r = __fmul2_rn(make_float2(x[e], x[e + 1]), make_float2(y[e], y[e + 1]));
      x[e] = r.x, x[e + 1] = r.y;
    }
  }
}
template <int E>
__device__ __forceinline__ void fma(const float (&x)[E], const float (&y)[E], const float (&z)[E], float (&o)[E]) {
  if constexpr (E == 1) {
    o[0] = fmaf(x[0], y[0], z[0]);
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 r = __ffma2_rn(make_float2(x[e], x[e + 1]), make_float2(y[e], y[e + 1]), make_float2(z[e], z[e + 1]));
      o[e] = r.x, o[e + 1] = r.y;
    }
  }
}
template <int E>
__device__ __forceinline__ void add(float (&x)[E], const float (&y)[E]) {
  if constexpr (E == 1) {
    x[0] += y[0];
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 r = __fadd2_rn(make_float2(x[e], x[e + 1]), make_float2(y[e], y[e + 1]));
      x[e] = r.x, x[e + 1] = r.y;
    }
  }
}
// The sum of x's values, halves together.
template <int E>
__device__ __forceinline__ float total(const float (&x)[E]) {
  if constexpr (E == 1) {
    return x[0];
  } else {
    float h[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) h[e] = x[e];
    float g[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) g[e] = x[E / 2 + e];
    add<E / 2>(h, g);
    return total<E / 2>(h);
  }
}
template <int E>
__device__ __forceinline__ void fill(float (&x)[E], float v) {
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = v;
}

// sigmoid(u) = 1 / (1 + 2^(-u log2 e)): three instructions a value, two of them the approximations'.  As with the gates,
// the rounded product makes it 2^-24 (|u| + 12) of itself off where it is small; where the exponential overflows it is 0.
template <int E>
__device__ __forceinline__ void sigmoid(const float (&u)[E], float (&s)[E]) {
  float one[E];
  fill<E>(one, 1.0f);
  fill<E>(s, -1.44269504088896341f);
  mul<E>(s, u);
#pragma unroll
  for (int e = 0; e < E; ++e) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(s[e]) : "f"(s[e]));
  add<E>(s, one);
#pragma unroll
  for (int e = 0; e < E; ++e) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s[e]) : "f"(s[e]));
}

// q = exp(-2 |u|) as 2^(-2 |u| log2 e), and r = 1 / (1 + q): tanh |u| = (1 - q) r.
__device__ __forceinline__ void tanh_parts(float u, float& q, float& r) {
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(q) : "f"(fabsf(u) * -2.88539008177792681f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + q));
}

// tanh.  Ahead of a 16-bit store by its parts, whose difference is off by some 3 units of 2^-24 whatever u: 13 of them
// relative to the result at |u| = 1/4, and below that Taylor's series to u^9 instead (what follows is 2^-26 of it there).
// 65,536 x 256 bf16: 19.3 us, 17.1 without the series (and 1 % off at 1e-6), 19.6 with tanhf; 64 x 4,096 x 256 in 32
// groups 73, 65 and 74.
template <typename T>
__device__ __forceinline__ float tanh_of(float u) {
  if constexpr (sizeof(T) == 4) {
    return tanhf(u);
  } else {
    float q, r;
    tanh_parts(u, q, r);
    const float w = u * u;
    float p = fmaf(62.0f / 2835.0f, w, -17.0f / 315.0f);
    p = fmaf(p, w, 2.0f / 15.0f);
    p = fmaf(p, w, -1.0f / 3.0f);
    return w < 0.0625f ? fmaf(u * w, p, u) : copysignf((1.0f - q) * r, u);
  }
}

// act(u); NaN passes relu.
template <typename T, int E>
__device__ __forceinline__ void activate(uint32_t act, float (&u)[E]) {
  if (act == NET_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < E; ++e) asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(u[e]) : "f"(u[e]));
  } else if (act == NET_ACT_SILU) {
    float s[E];
    sigmoid<E>(u, s);
    mul<E>(u, s);
  } else if (act == NET_ACT_TANH) {
#pragma unroll
    for (int e = 0; e < E; ++e) u[e] = tanh_of<T>(u[e]);
  }
}

// dz = dy act'(u) in place of dy; the slope of relu at 0 is 0.
template <typename T, int E>
__device__ __forceinline__ void slope(uint32_t act, const float (&u)[E], float (&dy)[E]) {
  if (act == NET_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < E; ++e) dy[e] = u[e] > 0.0f ? dy[e] : 0.0f;
  } else if (act == NET_ACT_SILU) {
    float s[E], v[E], one[E];
    sigmoid<E>(u, s);
    fill<E>(one, 1.0f);
    fill<E>(v, -1.0f);
    fma<E>(v, s, one, v);
    mul<E>(v, u);
    fma<E>(v, s, s, v);                // s (1 + u (1 - s))
    mul<E>(dy, v);
  } else if (act == NET_ACT_TANH) {
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float q, r;
      tanh_parts(u[e], q, r);
      v[e] = 4.0f * q * r * r;         // 1 - tanh^2, which as a difference has no digits left where tanh saturates
    }
    mul<E>(dy, v);
  }
}

template <typename T>
__device__ __forceinline__ T* at(const net_rows& r, int64_t i, int64_t j, int64_t k) {
  return reinterpret_cast<T*>(r.data) + i * r.outer + j * r.inner + k;
}

// E weights from channel c on (a multiple of E), or what stands for none.
template <int E>
__device__ __forceinline__ void load_weights(const float* w, int64_t c, float none, float (&x)[E]) {
  fill<E>(x, none);
  if (!w) return;
  if (E >= 4 && reinterpret_cast<uintptr_t>(w + c) % 16 == 0) {
#pragma unroll
    for (int e = 0; e + 3 < E; e += 4) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(w + c + e));
      x[e] = v.x, x[e + 1] = v.y, x[e + 2] = v.z, x[e + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = __ldg(w + c + e);
  }
}

// ------------------------------------------------------------------ clusters
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive(int ranks) {
  if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  cluster_wait();
}
// The value at this block's address p in the shared memory of block `rank`.
__device__ __forceinline__ float load_remote(const float* p, int rank) {
  uint32_t there;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(there) : "memory");
  return v;
}

// ------------------------------------------------------------------ teams
constexpr int kThreads = 256;
constexpr int kMostLanes = 512;      // of a team that is a block

// How teams cover a call: a group is `pieces` pieces of E channels, `wide` of them a position; a team has `lanes` lanes,
// a power of two: up to 32, or more, which are then a whole block.  A block has `groups` x `rows` teams, for that many
// adjacent groups of as many instances, and goes on by gridDim.x * rows instances.
struct Teams {
  int lanes, pieces, wide, groups, rows;
};

// How a team is made: LANES = 32 a whole warp, kAny some lanes of one, kBlock a block.
constexpr int kAny = 0, kBlock = -1;

// The sums over a team, in all its lanes.
template <int LANES, int N>
__device__ __forceinline__ void team_sum(float (&x)[N], int lanes) {
  if constexpr (LANES == kAny) {
    for (int o = lanes / 2; o; o /= 2) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], o);
    }
  } else {
#pragma unroll
    for (int o = 16; o; o /= 2) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], o);
    }
  }
  if constexpr (LANES == kBlock) {
    __shared__ float part[32][N];
    const int warps = blockDim.x / 32;
    __syncthreads();
    if (threadIdx.x % 32 == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) part[threadIdx.x / 32][i] = x[i];
    }
    __syncthreads();
    fill<N>(x, 0.0f);
    for (int w = 0; w < warps; ++w) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += part[w][i];
    }
  }
}

// 1 / sqrt(v): the approximation and a step of Newton's method; 0 for infinity, of which the step would make NaN.
__device__ __forceinline__ float inverse_root(float v) {
  const float r = rsqrtf(v);
  const float q = fmaf(-v * r, r, 1.0f);
  return v > 1e-30f && v < INFINITY ? fmaf(0.5f * r, q, r) : r;
}

// What a lane of a team works on.
template <int E, int SLOTS>
struct Lane {
  int lane, row;           // in the team; its instance among the block's
  int64_t g, c0;           // group, its first channel
  bool on;                 // whether the team has a group
  bool has[SLOTS];         // pieces that the lane has
  int s[SLOTS];            // their position
  int c[SLOTS];            // and first channel in the group
  __device__ Lane(const Norm& a, const Teams& t) {
    lane = threadIdx.x % t.lanes;
    const int team = threadIdx.x / t.lanes;
    row = team / t.groups;
    g = blockIdx.y * (int64_t)t.groups + team % t.groups;
    on = row < t.rows && g < a.G;
    c0 = on ? g * (a.C / a.G) : 0;
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      const int i = j * t.lanes + lane;
      has[j] = on && i < t.pieces;
      s[j] = has[j] ? i / t.wide : 0;
      c[j] = has[j] ? i - s[j] * t.wide : 0;
      c[j] *= E;
    }
  }
  // Where piece j of an array is, for instance 0.
  template <typename T>
  __device__ T* piece(const net_rows& r, int j) const {
    return at<T>(r, 0, s[j], c0 + c[j]);
  }
};

// What a lane reads of its next instances: N arrays' pieces of 16 bytes on their way to slots of its own in shared memory
// (65,536 x 256 bf16 forward: 12.8 us, 15.8 with registers), narrower ones in registers one instance ahead (65,536 x 250:
// 17.5 us, 21.1 with slots).
constexpr int kStages = 3;
template <typename T, int E, int SLOTS, int N>
struct Ahead {
  using W = Raw<T, E>;
  static constexpr bool kRing = sizeof(W) == 16;
  static constexpr int kDepth = kRing ? kStages : 1;
  const T* p[N][SLOTS];
  int64_t by[N];
  W* slots;              // (stage, i, j) at ((stage * N + i) * SLOTS + j) * blockDim.x
  W next[kRing ? 1 : N][kRing ? 1 : SLOTS];
  int stage;
  __device__ void begin(uint4* smem) { slots = reinterpret_cast<W*>(smem) + threadIdx.x, stage = 0; }
  static __host__ __device__ constexpr int bytes(int threads) {
    return kRing ? kStages * N * SLOTS * threads * (int)sizeof(W) : 0;
  }
  // The instance `kDepth` on from the one just taken (or the first few).
  __device__ void fetch(const bool (&has)[SLOTS], bool there, int to) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < SLOTS; ++j) {
        if (has[j] && there) {
          if constexpr (kRing) copy_async<sizeof(W)>(slots + ((to * N + i) * SLOTS + j) * blockDim.x, p[i][j]);
          else next[i][j] = *reinterpret_cast<const W*>(p[i][j]);
        }
        p[i][j] += by[i];
      }
    if constexpr (kRing) copy_commit();
  }
  __device__ void wait() {
    if constexpr (kRing) copy_wait<kStages - 1>();
  }
  __device__ void take(int i, int j, bool has, float (&x)[E]) {
    W w = {};
    if constexpr (kRing) {
      if (has) w = slots[((stage * N + i) * SLOTS + j) * blockDim.x];
    } else {
      if (has) w = next[i][j];
    }
    unpack<T, E>(w, x);
  }
  __device__ void step() { stage = stage + 1 == kDepth ? 0 : stage + 1; }
};

template <typename T, int E, int SLOTS, int LANES>
__global__ void __launch_bounds__(LANES == kBlock ? kMostLanes : kThreads) k_team(Norm a, Teams t) {
  const Lane<E, SLOTS> me(a, t);
  const float inv = 1.0f / (float)(a.S * (a.C / a.G));
  extern __shared__ uint4 smem[];
  float gamma[SLOTS][E], beta[SLOTS][E];
  Ahead<T, E, SLOTS, 1> in;
  T* py[SLOTS];
  const int first = blockIdx.x * t.rows + me.row, step = gridDim.x * t.rows, B = (int)a.B;
  const int64_t yy = step * a.y.outer;
  in.begin(smem);
  in.by[0] = step * a.x.outer;
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    in.p[0][j] = me.template piece<const T>(a.x, j) + first * a.x.outer;
    py[j] = me.template piece<T>(a.y, j) + first * a.y.outer;
  }
#pragma unroll
  for (int k = 0; k < in.kDepth; ++k) in.fetch(me.has, first + k * (int64_t)step < B, k);
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    load_weights<E>(me.has[j] ? a.gamma : nullptr, me.c0 + me.c[j], 1.0f, gamma[j]);
    load_weights<E>(me.has[j] ? a.beta : nullptr, me.c0 + me.c[j], 0.0f, beta[j]);
  }
  int64_t at_stats = first * a.G + me.g;
  const bool writes = me.on && me.lane == 0;
  // all lanes go round as often, for the shuffles
  int b = first;
  for (int left = (B - (int)blockIdx.x * t.rows + step - 1) / step; left > 0; --left, b += step) {
    float x[SLOTS][E];
    in.wait();
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) in.take(0, j, me.has[j], x[j]);    // 0 where the lane has none
    in.fetch(me.has, b + in.kDepth * (int64_t)step < B, in.stage);
    in.step();
    float part[E];
#pragma unroll
    for (int e = 0; e < E; ++e) part[e] = x[0][e];
#pragma unroll
    for (int j = 1; j < SLOTS; ++j) add<E>(part, x[j]);
    float sum[1] = {total<E>(part)};
    team_sum<LANES, 1>(sum, t.lanes);
    const float mean = sum[0] * inv;
    fill<E>(part, -mean);
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) add<E>(x[j], part);
    fill<E>(part, 0.0f);
#pragma unroll
    for (int j = 0; j < SLOTS; ++j)
      if (me.has[j]) fma<E>(x[j], x[j], part, part);
    sum[0] = total<E>(part);
    team_sum<LANES, 1>(sum, t.lanes);
    const float rstd = inverse_root(fmaf(sum[0], inv, a.eps));
    if (writes && b < B) {
      a.mean[at_stats] = mean;
      a.rstd[at_stats] = rstd;
    }
    at_stats += step * a.G;
    fill<E>(part, rstd);
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      mul<E>(x[j], part);
      fma<E>(gamma[j], x[j], beta[j], x[j]);
      activate<T, E>(a.act, x[j]);
      if (me.has[j] && b < B) store<T, E>(py[j], x[j]);
      py[j] += yy;
    }
  }
}

// weights: whether dbeta and dgamma are wanted.  Their sums by block go to partial [2][gridDim.x][C]; of few blocks, then
// a cluster (ranks of them), they are joined here.
template <typename T, int E, int SLOTS, int LANES>
__global__ void __launch_bounds__(LANES == kBlock ? kMostLanes : kThreads) k_team_back(Norm a, Teams t, bool weights, int ranks, float* partial) {
  extern __shared__ uint4 smem[];
  const Lane<E, SLOTS> me(a, t);
  const float inv = 1.0f / (float)(a.S * (a.C / a.G));
  float gamma[SLOTS][E], beta[SLOTS][E], db[SLOTS][E] = {}, dg[SLOTS][E] = {};
  Ahead<T, E, SLOTS, 2> in;
  T* pd[SLOTS];
  const int first = blockIdx.x * t.rows + me.row, step = gridDim.x * t.rows, B = (int)a.B;
  const int64_t dd = step * a.dx.outer;
  in.begin(smem);
  in.by[0] = step * a.x.outer, in.by[1] = step * a.dy.outer;
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    in.p[0][j] = me.template piece<const T>(a.x, j) + first * a.x.outer;
    in.p[1][j] = me.template piece<const T>(a.dy, j) + first * a.dy.outer;
    pd[j] = me.template piece<T>(a.dx, j) + first * a.dx.outer;
  }
#pragma unroll
  for (int k = 0; k < in.kDepth; ++k) in.fetch(me.has, first + k * (int64_t)step < B, k);
  int64_t at_stats = first * a.G + me.g;
  float nm = 0.0f, nr = 0.0f;
  auto fetch_stats = [&](int b) {
    if (me.on && b < B) nm = a.mean[at_stats], nr = a.rstd[at_stats];
    at_stats += step * a.G;
  };
  fetch_stats(first);
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    load_weights<E>(me.has[j] ? a.gamma : nullptr, me.c0 + me.c[j], 1.0f, gamma[j]);
    load_weights<E>(me.has[j] ? a.beta : nullptr, me.c0 + me.c[j], 0.0f, beta[j]);
  }
  int b = first;
  for (int left = (B - (int)blockIdx.x * t.rows + step - 1) / step; left > 0; --left, b += step) {
    float xh[SLOTS][E], dz[SLOTS][E], m[E], r[E];
    in.wait();
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      in.take(0, j, me.has[j], xh[j]);
      in.take(1, j, me.has[j], dz[j]);
    }
    in.fetch(me.has, b + in.kDepth * (int64_t)step < B, in.stage);
    in.step();
    fill<E>(m, -nm);
    fill<E>(r, nr);
    fetch_stats(b + step);
    float p0[E] = {}, p1[E] = {};
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      float u[E];
      add<E>(xh[j], m);
      mul<E>(xh[j], r);
      fma<E>(gamma[j], xh[j], beta[j], u);
      slope<T, E>(a.act, u, dz[j]);
      if (me.has[j] && b < B) {
        add<E>(db[j], dz[j]);
        fma<E>(dz[j], xh[j], dg[j], dg[j]);
        mul<E>(dz[j], gamma[j]);
        add<E>(p0, dz[j]);
        fma<E>(dz[j], xh[j], p1, p1);
      }
    }
    float w[2] = {total<E>(p0), total<E>(p1)};
    team_sum<LANES, 2>(w, t.lanes);
    // rstd (dz - avg(w) - xh avg(w xh))
    fill<E>(p0, -w[0] * inv);
    fill<E>(p1, -w[1] * inv);
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      add<E>(dz[j], p0);
      fma<E>(xh[j], p1, dz[j], dz[j]);
      mul<E>(dz[j], r);
      if (me.has[j] && b < B) store<T, E>(pd[j], dz[j]);
      pd[j] += dd;
    }
  }
  if (!weights) return;
  if constexpr (in.kRing) copy_wait<0>();
  __syncthreads();
  float* const sums = reinterpret_cast<float*>(smem);     // [2][teams of a block][lanes * SLOTS * E]
  // Each channel's sums: over the lanes that had it (a position each) and the block's instances.
  const int team = threadIdx.x / t.lanes, held = t.lanes * SLOTS * E, all = blockDim.x / t.lanes * held;
#pragma unroll
  for (int j = 0; j < SLOTS; ++j)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      sums[team * held + (j * t.lanes + me.lane) * E + e] = db[j][e];
      sums[all + team * held + (j * t.lanes + me.lane) * E + e] = dg[j][e];
    }
  __syncthreads();
  const int width = t.wide * E;
  for (int i = threadIdx.x; i < t.groups * width; i += blockDim.x) {
    const int64_t g = blockIdx.y * (int64_t)t.groups + i / width;
    if (g >= a.G) break;
    float b = 0.0f, w = 0.0f;
    for (int r = 0; r < t.rows; ++r)
      for (int k = i % width; k < t.pieces * E; k += width) {
        b += sums[(r * t.groups + i / width) * held + k];
        w += sums[all + (r * t.groups + i / width) * held + k];
      }
    const int64_t c = g * width + i % width;
    if (ranks) {                   // kept in the first row's place, which no other thread reads
      sums[i / width * held + i % width] = b;
      sums[all + i / width * held + i % width] = w;
    } else {
      partial[blockIdx.x * a.C + c] = b;
      partial[((int64_t)gridDim.x + blockIdx.x) * a.C + c] = w;
    }
  }
  if (!ranks) return;
  cluster_sync();
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < t.groups * width; i += blockDim.x) {
      const int64_t g = blockIdx.y * (int64_t)t.groups + i / width;
      if (g >= a.G) break;
      float b = 0.0f, w = 0.0f;
      for (int r = 0; r < ranks; ++r) {
        b += load_remote(sums + i / width * held + i % width, r);
        w += load_remote(sums + all + i / width * held + i % width, r);
      }
      const int64_t c = g * width + i % width;
      if (a.dbeta) a.dbeta[c] = b;
      if (a.dgamma) a.dgamma[c] = w;
    }
  }
  cluster_sync();                  // no block leaves before its sums are read
}

// dbeta and dgamma from [2][rows][C]: 32 columns of one a block, its warps over the rows.
constexpr int kJoinThreads = 1024;
__device__ __forceinline__ void join_weights(const Norm& a, const float* partial, int64_t rows, int64_t block, int which) {
  __shared__ float part[kJoinThreads / 32][32];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
  const int64_t c = block * 32 + lane;
  float s = 0.0f;
  if (c < a.C) {
    const float* p = partial + which * rows * a.C + c;
#pragma unroll 8
    for (int64_t r = warp; r < rows; r += warps) s += p[r * a.C];
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < a.C) {
    s = 0.0f;
    for (int w = 0; w < warps; ++w) s += part[w][lane];
    float* const out = which ? a.dgamma : a.dbeta;
    if (out) out[c] = s;
  }
}

__global__ void __launch_bounds__(kJoinThreads) k_weights(Norm a, const float* partial, int64_t rows) {
  after_previous();
  join_weights(a, partial, rows, blockIdx.x, blockIdx.y);
}

// ------------------------------------------------------------------ slabs
// A cluster holds S positions x `cols` pieces of E channels (whole groups of `wide` pieces, `groups` of them), each of
// its blocks `rows` positions; `side` rows of threads, a thread a piece of each `side`-th position.
struct Slab {
  int cols, wide, groups, side, rows, ranks, tiles;
};
constexpr int kSlabGroups = 8;             // of a slab at most
constexpr int kSlabRanks = 16;

// Stores v at this block's address p in the shared memory of every block of the cluster, all of which have started
// (cluster_arrive, a while ago), and waits for the others' stores.
__device__ __forceinline__ void exchange(float2* p, float2 v, bool mine, int ranks) {
  if (ranks > 1) cluster_wait();
  if (mine) {
    const uint32_t local = (uint32_t)__cvta_generic_to_shared(p);
    for (int r = 0; r < ranks; ++r) {
      uint32_t there;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(local), "r"(r));
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(v.x), "f"(v.y) : "memory");
    }
  }
  if (ranks > 1) cluster_sync();
  else __syncthreads();
}

template <typename T, int E>
struct SlabThread {
  int col, row, g, rank;       // piece, row of threads, group of the slab, block of the cluster
  int b, tile, c, s0, s1, n;   // instance, slab of it, first channel, the block's positions, the thread's pieces
  bool on;
  __device__ SlabThread(const Norm& a, const Slab& k) {
    rank = (int)cluster_rank();
    const unsigned q = blockIdx.x / (unsigned)k.ranks, i = q / (unsigned)k.tiles;
    b = (int)i;
    tile = (int)(q - i * k.tiles);
    row = threadIdx.x / (unsigned)k.cols;
    col = threadIdx.x - row * k.cols;
    g = col / (unsigned)k.wide;
    c = (tile * k.cols + col) * E;
    on = row < k.side && c < (int)a.C;
    s0 = (int)min(a.S, (int64_t)rank * k.rows);
    s1 = (int)min(a.S, (int64_t)s0 + k.rows);
    n = on && s0 + row < s1 ? (int)((unsigned)(s1 - s0 - row + k.side - 1) / (unsigned)k.side) : 0;
  }
  // Copies the thread's pieces of an array.
  __device__ void fetch(const net_rows& r, uint4* to, const Slab& k) const {
    const T* p = at<const T>(r, b, s0 + row, c);
    const int64_t by = k.side * r.inner;
    to += threadIdx.x;
#pragma unroll 4
    for (int i = 0; i < n; ++i, p += by, to += k.side * k.cols) copy_async<16>(to, p);
  }
};

// The sums of x over the threads of each group of the slab (in order), to group[g].
__device__ __forceinline__ void group_sums(float x, float* threads, float* group, const Slab& k) {
  threads[threadIdx.x] = x;
  __syncthreads();
  const int lane = threadIdx.x % 32, n = k.side * k.wide;
  for (int g = threadIdx.x / 32; g < k.groups; g += kThreads / 32) {
    float s = 0.0f;
    for (int i = lane; i < n; i += 32) s += threads[(unsigned)i / (unsigned)k.wide * k.cols + g * k.wide + (unsigned)i % (unsigned)k.wide];
#pragma unroll
    for (int o = 16; o; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) group[g] = s;
  }
  __syncthreads();
}

// A thread's values are summed once, as distances from its first piece; its mean and squared deviations from that mean
// are joined over the threads of a group, and over the cluster's blocks, by the distances of the means.
template <typename T, int E>
__global__ void __launch_bounds__(kThreads, 3) k_slab(Norm a, Slab k) {
  extern __shared__ uint4 data[];
  __shared__ float threads[2][kThreads], group[2][kSlabGroups];
  __shared__ float2 from[kSlabRanks][kSlabGroups], stats[kSlabGroups];   // mean, squared deviations; mean, rstd
  cluster_arrive(k.ranks);
  const SlabThread<T, E> me(a, k);
  me.fetch(a.x, data, k);
  copy_commit();
  float gamma[E], beta[E];
  load_weights<E>(me.on ? a.gamma : nullptr, me.c, 1.0f, gamma);
  load_weights<E>(me.on ? a.beta : nullptr, me.c, 0.0f, beta);
  copy_wait<0>();
  const uint4* const mine = data + threadIdx.x;
  const int n = me.n, by = k.side * k.cols, W = k.wide * E;
  float first[E] = {}, s1[E] = {}, s2[E] = {};
  if (n) {
    unpack<T, E>(mine[0], first);
#pragma unroll
    for (int e = 0; e < E; ++e) first[e] = -first[e];
  }
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    float x[E];
    unpack<T, E>(mine[i * by], x);
    add<E>(x, first);
    add<E>(s1, x);
    fma<E>(x, x, s2, s2);
  }
  const float inv = n ? 1.0f / (float)n : 0.0f;
  float mean = 0.0f, sq = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    s2[e] = fmaxf(fmaf(-s1[e] * inv, s1[e], s2[e]), 0.0f);
    s1[e] = fmaf(s1[e], inv, -first[e]);       // the channel's mean
    mean += s1[e];
    sq += s2[e];
  }
  mean *= 1.0f / E;
#pragma unroll
  for (int e = 0; e < E; ++e) sq = fmaf((s1[e] - mean) * (float)n, s1[e] - mean, sq);
  group_sums(mean * (float)(n * E), threads[0], group[0], k);
  const float here = (float)(me.s1 - me.s0) * (float)W;
  const float block = here > 0.0f ? group[0][me.g] / here : 0.0f;
  group_sums(fmaf((mean - block) * (float)(n * E), mean - block, sq), threads[1], group[1], k);
  const int mg = threadIdx.x;
  const bool joins = mg < k.groups;
  exchange(&from[me.rank][joins ? mg : 0],
           joins && here > 0.0f ? make_float2(group[0][mg] / here, group[1][mg]) : make_float2(0.0f, 0.0f), joins, k.ranks);
  if (joins) {
    const float all = 1.0f / ((float)a.S * (float)W), m0 = from[0][mg].x;
    auto size = [&](int r) { return (float)max((int64_t)0, min((int64_t)k.rows, a.S - (int64_t)r * k.rows)) * (float)W; };
    float m = 0.0f, v = 0.0f;
    for (int r = 0; r < k.ranks; ++r) m = fmaf(size(r), from[r][mg].x - m0, m);
    m = fmaf(m, all, m0);
    for (int r = 0; r < k.ranks; ++r) {
      const float d = from[r][mg].x - m, w = size(r);
      if (w > 0.0f) v += fmaf(w * d, d, from[r][mg].y);
    }
    const float rstd = inverse_root(fmaf(v, all, a.eps));
    stats[mg] = make_float2(m, rstd);
    const int64_t g = me.tile * (int64_t)k.groups + mg;
    if (me.rank == 0 && g < a.G) {
      a.mean[me.b * a.G + g] = m;
      a.rstd[me.b * a.G + g] = rstd;
    }
  }
  __syncthreads();
  if (!me.on) return;
  fill<E>(s1, -stats[me.g].x);
  fill<E>(s2, stats[me.g].y);
  mul<E>(gamma, s2);
  T* o = at<T>(a.y, me.b, me.s0 + me.row, me.c);
  const int64_t oy = k.side * a.y.inner;
#pragma unroll 4
  for (int i = 0; i < n; ++i, o += oy) {
    float x[E];
    unpack<T, E>(mine[i * by], x);
    add<E>(x, s1);
    fma<E>(gamma, x, beta, x);
    activate<T, E>(a.act, x);
    store<T, E>(o, x);
  }
}

// partial: [2][B * ranks][C], or NULL.
template <typename T, int E>
__global__ void __launch_bounds__(kThreads, 3) k_slab_back(Norm a, Slab k, float* partial) {
  extern __shared__ uint4 data[];
  __shared__ float sums[E][kThreads];
  __shared__ float2 from[kSlabRanks][kSlabGroups];
  __shared__ float own[2][kSlabGroups];
  cluster_arrive(k.ranks);
  const SlabThread<T, E> me(a, k);
  const int held = k.rows * k.cols;
  me.fetch(a.x, data, k);
  me.fetch(a.dy, data + held, k);
  float gamma[E], beta[E], shift[E], scale[E];
  load_weights<E>(me.on ? a.gamma : nullptr, me.c, 1.0f, gamma);
  load_weights<E>(me.on ? a.beta : nullptr, me.c, 0.0f, beta);
  const int W = k.wide * E;
  const int64_t stats = me.b * a.G + me.c / (unsigned)W;
  const float rstd = me.on ? a.rstd[stats] : 0.0f;
  fill<E>(shift, me.on ? -a.mean[stats] : 0.0f);
  fill<E>(scale, rstd);
  copy_commit();
  copy_wait<0>();
  const uint4 *const mx = data + threadIdx.x, *const my = mx + held;
  const int n = me.n, by = k.side * k.cols;
  float db[E] = {}, dg[E] = {};
  auto piece = [&](int i, float (&xh)[E], float (&dz)[E]) {
    float u[E];
    unpack<T, E>(mx[i * by], xh);
    unpack<T, E>(my[i * by], dz);
    add<E>(xh, shift);
    mul<E>(xh, scale);
    fma<E>(gamma, xh, beta, u);
    slope<T, E>(a.act, u, dz);
  };
#pragma unroll 2
  for (int i = 0; i < n; ++i) {
    float xh[E], dz[E];
    piece(i, xh, dz);
    add<E>(db, dz);
    fma<E>(dz, xh, dg, dg);
  }
  // Each channel's sums over the rows of threads, to the first row's places and out, and each group's, weighted: dbeta's,
  // then dgamma's (one array of sums leaves room for a third block an SM).
  const int64_t row = (int64_t)me.b * k.ranks + me.rank, rows = a.B * k.ranks;
  const int c0 = me.tile * k.cols * E, lane = threadIdx.x % 32;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
#pragma unroll
    for (int e = 0; e < E; ++e) sums[e][threadIdx.x] = which ? dg[e] : db[e];
    __syncthreads();
    for (int i = threadIdx.x; i < E * k.cols; i += kThreads) {
      const int e = (unsigned)i / (unsigned)k.cols, col = i - e * k.cols;
      float v = 0.0f;
      for (int r = 0; r < k.side; ++r) v += sums[e][r * k.cols + col];
      sums[e][col] = v;
      const int c = c0 + col * E + e;
      if (partial && c < a.C) partial[(which * rows + row) * a.C + c] = v;
    }
    __syncthreads();
    for (int g = threadIdx.x / 32; g < k.groups; g += kThreads / 32) {
      float v = 0.0f;
      for (int i = lane; i < W; i += 32) {
        const int col = g * k.wide + i / E, e = i % E, c = c0 + col * E + e;
        v = fmaf(c < a.C ? (a.gamma ? __ldg(a.gamma + c) : 1.0f) : 0.0f, sums[e][col], v);
      }
#pragma unroll
      for (int o = 16; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane == 0) own[which][g] = v;
    }
    __syncthreads();
  }
  const bool joins = (int)threadIdx.x < k.groups;
  const int mg = joins ? threadIdx.x : 0;
  exchange(&from[me.rank][mg], make_float2(own[0][mg], own[1][mg]), joins, k.ranks);
  if (!me.on) return;
  float2 w = make_float2(0.0f, 0.0f);
  for (int r = 0; r < k.ranks; ++r) w.x += from[r][me.g].x, w.y += from[r][me.g].y;
  const float all = 1.0f / (float)(a.S * W);
  float m1[E], m2[E];
  fill<E>(m1, -w.x * all);
  fill<E>(m2, -w.y * all);
  T* o = at<T>(a.dx, me.b, me.s0 + me.row, me.c);
  const int64_t oy = k.side * a.dx.inner;
#pragma unroll 2
  for (int i = 0; i < n; ++i, o += oy) {
    float xh[E], dz[E];
    piece(i, xh, dz);
    fma<E>(dz, gamma, m1, dz);
    fma<E>(xh, m2, dz, dz);
    mul<E>(dz, scale);
    store<T, E>(o, dz);
  }
}

// ------------------------------------------------------------------ chunks
// Larger groups: a block takes `rows` positions of `cols` pieces of E channels, kThreads / cols rows side by side.
struct Chunks {
  int cols;             // pieces of a block, up to 64
  int rows;             // positions of a block
  int64_t count;        // chunks of an instance
};

template <int E>
struct Place {
  int64_t b, chunk, c, s0, s1;
  int row, rows;        // the thread's first, and how many are side by side
  bool on;
  __device__ Place(const Norm& a, const Chunks& k) {
    b = blockIdx.x / k.count;
    chunk = blockIdx.x - b * k.count;
    row = threadIdx.x / k.cols;
    rows = kThreads / k.cols;
    c = (blockIdx.y * (int64_t)k.cols + threadIdx.x % k.cols) * E;
    on = c < a.C && row < rows;
    s0 = chunk * k.rows;
    s1 = min(a.S, s0 + k.rows);
  }
};

// Adds up the block's rows: x of the threads of a column, in the first row's.
template <int E>
__device__ __forceinline__ void join_rows(float (&x)[E], int cols) {
  __shared__ float part[E][kThreads];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e) part[e][threadIdx.x] = x[e];
  __syncthreads();
  if ((int)threadIdx.x < cols) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float s = 0.0f;
      for (int i = threadIdx.x; i < kThreads / cols * cols; i += cols) s += part[e][i];
      x[e] = s;
    }
  }
}

// Mean and sum of squared deviations of each chunk's channels: part[2][B * count][C].  A thread sums up to kRun of its
// rows at a time, as distances from the first of them, and joins those by the distances of their means; so are the
// threads joined.  n rows that are all far from the first, at distance k deviations, cancel n k^2 against the k^2 that it
// adds itself: with one first value for a chunk of 37,000 rows the variance was a tenth off.
constexpr int kRun = 32;
template <typename T, int E>
__global__ void __launch_bounds__(kThreads) k_part(Norm a, Chunks k, float* part) {
  __shared__ float means[E][kThreads], squares[E][kThreads];
  const Place<E> me(a, k);
  const int length = (int)(me.s1 - me.s0);
  float mean[E] = {}, m2[E] = {};
  if (me.on) {
    const T* p = at<T>(a.x, me.b, me.s0 + me.row, me.c);
    const int64_t by = me.rows * a.x.inner;
    int left = me.row < length ? (length - me.row + me.rows - 1) / me.rows : 0;
    float before = 0.0f;
    while (left > 0) {
      const int run = min(left, kRun);
      float first[E], s1[E] = {}, s2[E] = {};
      load<T, E>(p, first);
#pragma unroll 4
      for (int i = 0; i < run; ++i, p += by) {
        float x[E];
        load<T, E>(p, x);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float d = x[e] - first[e];
          s1[e] += d;
          s2[e] = fmaf(d, d, s2[e]);
        }
      }
      left -= run;
      const float inv = 1.0f / (float)run, share = (float)run / (before + (float)run);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float m = s1[e] * inv, d = first[e] + m - mean[e];
        m2[e] += fmaxf(fmaf(-m, s1[e], s2[e]), 0.0f) + d * (before * share) * d;
        mean[e] = fmaf(d, share, mean[e]);
      }
      before += (float)run;
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) means[e][threadIdx.x] = mean[e], squares[e][threadIdx.x] = m2[e];
  __syncthreads();
  const int each = length / me.rows, more = length % me.rows;        // rows of a thread: the first `more` one more
  const float inv = 1.0f / (float)length;
  for (int q = threadIdx.x; q < k.cols * E; q += kThreads) {
    const int e = q / k.cols, col = q - e * k.cols;
    const int64_t c = (blockIdx.y * (int64_t)k.cols + col) * E + e;
    if (c >= a.C) continue;
    const float m0 = means[e][col];
    float m = 0.0f, v = 0.0f;
    for (int i = 1; i < me.rows; ++i) m = fmaf((float)(each + (i < more)), means[e][i * k.cols + col] - m0, m);
    m = fmaf(m, inv, m0);
    for (int i = 0; i < me.rows; ++i) {
      const float w = (float)(each + (i < more)), d = means[e][i * k.cols + col] - m;
      if (w > 0.0f) v += fmaf(w * d, d, squares[e][i * k.cols + col]);
    }
    part[blockIdx.x * a.C + c] = m;
    part[((int64_t)gridDim.x + blockIdx.x) * a.C + c] = v;
  }
}

// Mean and rstd of a group, a block each, from its channels' chunks.
__global__ void __launch_bounds__(kJoinThreads) k_stats(Norm a, Chunks k, const float* part) {
  after_previous();
  const int64_t W = a.C / a.G, all = k.count * W;
  for (int64_t q = blockIdx.x; q < a.B * a.G; q += gridDim.x) {
    const int64_t b = q / a.G, c0 = q % a.G * W;
    const float* m = part + b * k.count * a.C + c0;
    const float* m2 = m + a.B * k.count * a.C;
    auto size = [&](int64_t chunk) { return (float)(min(a.S, (chunk + 1) * k.rows) - chunk * k.rows); };
    const float shift = m[0];
    float s[2] = {0.0f, 0.0f};
    for (int64_t i = threadIdx.x; i < all; i += blockDim.x) s[0] += size(i / W) * (m[i / W * a.C + i % W] - shift);
    team_sum<kBlock, 2>(s, 0);
    const float n = (float)a.S * (float)W, mean = shift + s[0] / n;
    s[0] = s[1] = 0.0f;
    for (int64_t i = threadIdx.x; i < all; i += blockDim.x) {
      const float d = m[i / W * a.C + i % W] - mean;
      s[0] += m2[i / W * a.C + i % W];
      s[1] = fmaf(size(i / W) * d, d, s[1]);
    }
    team_sum<kBlock, 2>(s, 0);
    if (threadIdx.x == 0) {
      a.mean[q] = mean;
      a.rstd[q] = 1.0f / sqrtf((s[0] + s[1]) / n + a.eps);
    }
  }
}

template <int E>
struct Weights {
  float gamma[E], beta[E], mean[E], rstd[E];
  __device__ Weights(const Norm& a, int64_t b, int64_t c) {
    load_weights<E>(a.gamma, c, 1.0f, gamma);
    load_weights<E>(a.beta, c, 0.0f, beta);
    const int64_t W = a.C / a.G;
    int64_t g = c / W, left = (g + 1) * W - c;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (left-- == 0) ++g, left = W - 1;
      mean[e] = a.mean[b * a.G + g];
      rstd[e] = a.rstd[b * a.G + g];
    }
  }
};

template <typename T, int E>
__global__ void __launch_bounds__(kThreads) k_apply(Norm a, Chunks k) {
  const Place<E> me(a, k);
  after_previous();
  if (!me.on) return;
  const Weights<E> w(a, me.b, me.c);
  const T* p = at<T>(a.x, me.b, me.s0 + me.row, me.c);
  T* o = at<T>(a.y, me.b, me.s0 + me.row, me.c);
  const int64_t by = me.rows * a.x.inner, oy = me.rows * a.y.inner;
#pragma unroll 4
  for (int64_t s = me.s0 + me.row; s < me.s1; s += me.rows, p += by, o += oy) {
    float x[E];
    load<T, E>(p, x);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = fmaf(w.gamma[e], (x[e] - w.mean[e]) * w.rstd[e], w.beta[e]);
    activate<T, E>(a.act, x);
    store<T, E>(o, x);
  }
}

// Sums of dz and dz xh of each chunk's channels: part[2][B * count][C].
template <typename T, int E>
__global__ void __launch_bounds__(kThreads) k_part_back(Norm a, Chunks k, float* part) {
  const Place<E> me(a, k);
  float db[E] = {}, dg[E] = {};
  if (me.on) {
    const Weights<E> w(a, me.b, me.c);
    const T* p = at<T>(a.x, me.b, me.s0 + me.row, me.c);
    const T* y = at<T>(a.dy, me.b, me.s0 + me.row, me.c);
    const int64_t by = me.rows * a.x.inner, yy = me.rows * a.dy.inner;
#pragma unroll 4
    for (int64_t s = me.s0 + me.row; s < me.s1; s += me.rows, p += by, y += yy) {
      float xh[E], dz[E], u[E];
      load<T, E>(p, xh);
      load<T, E>(y, dz);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        xh[e] = (xh[e] - w.mean[e]) * w.rstd[e];
        u[e] = fmaf(w.gamma[e], xh[e], w.beta[e]);
      }
      slope<T, E>(a.act, u, dz);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        db[e] += dz[e];
        dg[e] = fmaf(dz[e], xh[e], dg[e]);
      }
    }
  }
  join_rows<E>(db, k.cols);
  join_rows<E>(dg, k.cols);
  if (me.on && (int)threadIdx.x < k.cols) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      part[blockIdx.x * a.C + me.c + e] = db[e];
      part[((int64_t)gridDim.x + blockIdx.x) * a.C + me.c + e] = dg[e];
    }
  }
}

// avg(w) and avg(w xh) of a group, a block each: avg[2][B * G].  The blocks after those sum dbeta and dgamma.
__global__ void __launch_bounds__(kJoinThreads) k_stats_back(Norm a, Chunks k, const float* part, float* avg, int64_t groups) {
  after_previous();
  const int64_t rows = a.B * k.count;
  if (blockIdx.x >= groups) {
    join_weights(a, part, rows, (blockIdx.x - groups) / 2, (int)((blockIdx.x - groups) % 2));
    return;
  }
  const int64_t W = a.C / a.G, all = k.count * W;
  for (int64_t q = blockIdx.x; q < a.B * a.G; q += groups) {
    const int64_t b = q / a.G, c0 = q % a.G * W;
    const float* db = part + b * k.count * a.C + c0;
    const float* dg = db + rows * a.C;
    float s[2] = {0.0f, 0.0f};
    for (int64_t i = threadIdx.x; i < all; i += blockDim.x) {
      const float g = a.gamma ? a.gamma[c0 + i % W] : 1.0f;
      s[0] = fmaf(g, db[i / W * a.C + i % W], s[0]);
      s[1] = fmaf(g, dg[i / W * a.C + i % W], s[1]);
    }
    team_sum<kBlock, 2>(s, 0);
    if (threadIdx.x == 0) {
      const float inv = 1.0f / ((float)a.S * (float)W);
      avg[q] = s[0] * inv;
      avg[a.B * a.G + q] = s[1] * inv;
    }
  }
}

template <typename T, int E>
__global__ void __launch_bounds__(kThreads) k_apply_back(Norm a, Chunks k, const float* avg) {
  const Place<E> me(a, k);
  after_previous();
  if (!me.on) return;
  const Weights<E> w(a, me.b, me.c);
  float m1[E], m2[E];
  const int64_t W = a.C / a.G;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    m1[e] = avg[me.b * a.G + (me.c + e) / W];
    m2[e] = avg[(a.B + me.b) * a.G + (me.c + e) / W];
  }
  const T* p = at<T>(a.x, me.b, me.s0 + me.row, me.c);
  const T* y = at<T>(a.dy, me.b, me.s0 + me.row, me.c);
  T* o = at<T>(a.dx, me.b, me.s0 + me.row, me.c);
  const int64_t by = me.rows * a.x.inner, yy = me.rows * a.dy.inner, oy = me.rows * a.dx.inner;
#pragma unroll 4
  for (int64_t s = me.s0 + me.row; s < me.s1; s += me.rows, p += by, y += yy, o += oy) {
    float xh[E], dz[E], u[E];
    load<T, E>(p, xh);
    load<T, E>(y, dz);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      xh[e] = (xh[e] - w.mean[e]) * w.rstd[e];
      u[e] = fmaf(w.gamma[e], xh[e], w.beta[e]);
    }
    slope<T, E>(a.act, u, dz);
#pragma unroll
    for (int e = 0; e < E; ++e) dz[e] = w.rstd[e] * (w.gamma[e] * dz[e] - m1[e] - xh[e] * m2[e]);
    store<T, E>(o, dz);
  }
}

// No positions: the mean is 0, the variance too.
__global__ void k_empty(Norm a) {
  const int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x;
  if (i < a.B * a.G) {
    a.mean[i] = 0.0f;
    a.rstd[i] = 1.0f / sqrtf(a.eps);
  }
}

// ------------------------------------------------------------------ plans
struct Plan {
  bool team;
  int e, slots, threads;
  int join;             // blocks of a cluster that joins the weights' gradients, 0: none
  bool block;
  Teams t;
  dim3 grid;
  bool slab;
  Slab sl;
  int smem;
  Chunks k;
  int64_t stats;        // blocks that join groups
  size_t bytes;
};

int pow2_at_least(int64_t n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}

// By sizes, types, and the alignment of strides and data; pieces of up to `most_e` channels (the workspace's query asks
// for every alignment that arrays may come to have).
Plan make_plan(const net_norm* p, bool back, int most_e = 8) {
  Plan q = {};
  const int size = type_size(p->dtype), sms = sm_count();
  const int64_t W = p->C / p->G;
  const net_rows* rows[2][2] = {{&p->x, &p->y}, {&p->x, &p->dy}};
  auto fits = [&](int e) {
    bool ok = e <= most_e;
    for (const net_rows* r : rows[back])
      ok = ok && (p->B <= 1 || r->outer % e == 0) && (p->S <= 1 || r->inner % e == 0) &&
           reinterpret_cast<uintptr_t>(r->data) % ((size_t)size * e) == 0;
    if (back)
      ok = ok && (p->B <= 1 || p->dx.outer % e == 0) && (p->S <= 1 || p->dx.inner % e == 0) &&
           reinterpret_cast<uintptr_t>(p->dx.data) % ((size_t)size * e) == 0;
    return ok;
  };
  const int widest = 16 / size;
  // teams: pieces within a group
  q.e = widest;
  while (q.e > 1 && (W % q.e || !fits(q.e))) q.e = q.e > 2 ? 2 : 1;
  const int64_t pieces = W / q.e * (p->S < (1 << 20) ? p->S : 1 << 20);
  // Eight values a lane (four single ones): backward, six registers a value are weights, their sums and what comes next.
  const int most = std::min(4, 8 / q.e);
  q.team = pieces <= (int64_t)kMostLanes * most && p->G <= 65535;
  if (q.team) {
    q.block = pieces > 32 * most;
    int lanes = pow2_at_least((pieces + most - 1) / most);
    lanes = std::min(lanes, q.block ? kMostLanes : 32);
    q.slots = std::max(1, pow2_at_least((pieces + lanes - 1) / lanes));
    q.threads = q.block ? lanes : kThreads;
    const int teams = q.threads / lanes;
    const int groups = (int)std::min<int64_t>(p->G, teams), per = teams / groups;
    q.t = {lanes, (int)pieces, (int)(W / q.e), groups, per};
    const int64_t gy = (p->G + groups - 1) / groups, gx = (p->B + per - 1) / per;
    // as many blocks as the SMs hold at a time: each goes from instance to instance (a second round of blocks cost 8 us
    // of 29 backward at 65,536 x 256 bf16)
    const int resident = back ? 512 : q.e == 8 && !q.block ? 1280 : 1024;
    const int64_t want = std::max<int64_t>(1, (int64_t)sms * (resident / q.threads) / gy);
    q.grid = dim3((unsigned)std::min(gx, want), (unsigned)gy);
    // Few instances: a cluster of up to eight blocks joins dgamma and dbeta itself.  That saves a launch and the
    // workspace, 8 us of the host's 20 at 256 x 90, and costs some turns of the blocks.
    if (back && (p->dgamma || p->dbeta)) {
      if (gx <= 32) q.join = (int)std::min<int64_t>(gx, 8), q.grid.x = (unsigned)q.join;
      else q.bytes = sizeof(float) * 2 * q.grid.x * (size_t)p->C;
    }
    return q;
  }
  // slabs: whole groups side by side, in as few blocks as leave three an SM (72 KB each, backward 8 of them for sums;
  // then two, and clusters of 16).  128 bytes of a row at least where four blocks hold that (500 x 300 x 128 bf16: 22 us,
  // 28 with 64 bytes), else 64 (64 x 4,096 x 256: 60 us, 64 with 128 bytes).  Aligned pieces within a group alone.
  if (W % widest == 0 && fits(widest) && W / widest <= kThreads) {
    const int wide = (int)(W / widest), arrays = back ? 2 : 1;
    for (int least = kSlabGroups; least >= 4; least /= 2) {
      const int groups = (int)std::min<int64_t>(p->G, std::max(1, least / wide));
      const int cols = wide * groups, side = kThreads / cols;
      const int64_t row = (int64_t)cols * 16 * arrays;
      auto ranks_for = [&](int64_t bytes) {
        const int64_t rows = std::max<int64_t>(1, bytes / row);
        return (p->S + rows - 1) / rows;
      };
      int64_t ranks = ranks_for(back ? 64 * 1024 : 72 * 1024);
      if (least > 4 && ranks > 4) continue;
      if (ranks > 8) ranks = ranks_for(back ? 100 * 1024 : 108 * 1024);
      if (ranks > kSlabRanks) break;
      const int64_t tiles = (p->G + groups - 1) / groups;
      int r = pow2_at_least(ranks);
      // more blocks where there are few
      while (r < 8 && p->B * tiles * r < sms && p->S >= 2 * r * side) r *= 2;
      if (p->B * tiles * r > INT32_MAX) break;
      const int64_t rows = (p->S + r - 1) / r;
      q.slab = true;
      q.e = widest;
      q.sl = {cols, wide, groups, side, (int)rows, r, (int)tiles};
      q.grid = dim3((unsigned)(p->B * tiles * r));
      q.smem = (int)(rows * row);
      if (back && (p->dgamma || p->dbeta)) q.bytes = sizeof(float) * 2 * (size_t)(p->B * r) * p->C;
      return q;
    }
  }
  q.e = widest;
  while (q.e > 1 && (p->C % q.e || !fits(q.e))) q.e = q.e > 2 ? 2 : 1;
  const int64_t cols = (p->C + q.e - 1) / q.e;
  const int64_t across = (cols + 63) / 64;
  q.k.cols = (int)((cols + across - 1) / across);
  const int side = kThreads / q.k.cols;
  // four blocks an SM, but no more chunks of an instance than its statistics are soon joined from
  int64_t want = std::max<int64_t>(1, std::min<int64_t>(3 * sms, (int64_t)sms * 4 / std::max<int64_t>(1, across * p->B)));
  want = std::min(want, std::max<int64_t>(1, p->S / (side * 4)));
  int64_t per = (p->S + want - 1) / want;
  per = std::min<int64_t>(std::max<int64_t>(per, 1), 1 << 20);
  q.k.rows = (int)per;
  q.k.count = (p->S + per - 1) / per;
  q.grid = dim3((unsigned)(p->B * q.k.count), (unsigned)across);
  q.stats = std::min<int64_t>(p->B * p->G, 1 << 20);
  q.bytes = sizeof(float) * 2 * ((size_t)p->B * q.k.count * p->C + (back ? (size_t)p->B * p->G : 0));
  return q;
}

cudaError_t launch_weights(const Norm& a, const float* partial, int64_t rows, cudaStream_t s) {
  return launch_after(k_weights, dim3((unsigned)((a.C + 31) / 32), 2), kJoinThreads, 0, s, a, partial, rows);
}

template <typename... P, typename... A>
cudaError_t launch_cluster(void (*kern)(P...), dim3 grid, int threads, int smem, int ranks, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ranks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}

template <typename T, int E, int SLOTS, int LANES>
cudaError_t launch_team(const Norm& a, const Plan& q, bool back, float* ws, cudaStream_t s) {
  auto allow = [](const void* kern, int bytes) {
    return bytes <= 40 * 1024 ? cudaSuccess   // 48 KB with what a kernel declares itself
                              : cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  if (!back) {
    constexpr auto kern = k_team<T, E, SLOTS, LANES>;
    const int smem = Ahead<T, E, SLOTS, 1>::bytes(q.threads);
    const cudaError_t e = allow((const void*)kern, smem);
    if (e != cudaSuccess) return e;
    kern<<<q.grid, q.threads, smem, s>>>(a, q.t);
    return cudaGetLastError();
  }
  const bool weights = a.dgamma || a.dbeta;
  const int smem = std::max(weights ? 2 * q.threads * SLOTS * E * (int)sizeof(float) : 0,
                            Ahead<T, E, SLOTS, 2>::bytes(q.threads));
  const auto kern = k_team_back<T, E, SLOTS, LANES>;
  cudaError_t e = allow((const void*)kern, smem);
  if (e != cudaSuccess) return e;
  if (q.join) return launch_cluster(kern, q.grid, q.threads, smem, q.join, s, a, q.t, weights, q.join, ws);
  kern<<<q.grid, q.threads, smem, s>>>(a, q.t, weights, 0, ws);
  e = cudaGetLastError();
  return e == cudaSuccess && weights ? launch_weights(a, ws, q.grid.x, s) : e;
}

template <typename T, int E, int SLOTS>
cudaError_t launch_teams(const Norm& a, const Plan& q, bool back, float* ws, cudaStream_t s) {
  if (q.block) return launch_team<T, E, SLOTS, kBlock>(a, q, back, ws, s);
  if (q.t.lanes == 32) return launch_team<T, E, SLOTS, 32>(a, q, back, ws, s);
  return launch_team<T, E, SLOTS, kAny>(a, q, back, ws, s);
}

template <typename T, int E>
cudaError_t launch_teams(const Norm& a, const Plan& q, bool back, float* ws, cudaStream_t s) {
  if constexpr (E <= 2)
    if (q.slots == 4) return launch_teams<T, E, 4>(a, q, back, ws, s);
  if constexpr (E <= 4)
    if (q.slots == 2) return launch_teams<T, E, 2>(a, q, back, ws, s);
  return launch_teams<T, E, 1>(a, q, back, ws, s);
}

template <typename T>
cudaError_t launch_slab(const Norm& a, const Plan& q, bool back, float* ws, cudaStream_t s) {
  constexpr int E = 16 / sizeof(T);
  const bool weights = back && (a.dgamma || a.dbeta);
  const void* const kern = back ? (const void*)k_slab_back<T, E> : (const void*)k_slab<T, E>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, q.smem);
  if (e == cudaSuccess && q.sl.ranks > 8)
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  e = back ? launch_cluster(k_slab_back<T, E>, q.grid, kThreads, q.smem, q.sl.ranks, s, a, q.sl, weights ? ws : (float*)nullptr)
           : launch_cluster(k_slab<T, E>, q.grid, kThreads, q.smem, q.sl.ranks, s, a, q.sl);
  return e == cudaSuccess && weights ? launch_weights(a, ws, a.B * q.sl.ranks, s) : e;
}

template <typename T, int E>
cudaError_t launch_chunks(const Norm& a, const Plan& q, bool back, float* ws, cudaStream_t s) {
  cudaError_t e;
  // threads that join a group: by what there is of it
  const int join = q.k.count * (a.C / a.G) >= 1024 ? kJoinThreads : kThreads;
  if (!back) {
    k_part<T, E><<<q.grid, kThreads, 0, s>>>(a, q.k, ws);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    e = launch_after(k_stats, dim3((unsigned)q.stats), join, 0, s, a, q.k, (const float*)ws);
    return e != cudaSuccess ? e : launch_after(k_apply<T, E>, q.grid, kThreads, 0, s, a, q.k);
  }
  float* const avg = ws + 2 * a.B * q.k.count * a.C;
  const int64_t columns = a.dgamma || a.dbeta ? (a.C + 31) / 32 * 2 : 0;
  k_part_back<T, E><<<q.grid, kThreads, 0, s>>>(a, q.k, ws);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  e = launch_after(k_stats_back, dim3((unsigned)(q.stats + columns)), join, 0, s, a, q.k, (const float*)ws, avg, q.stats);
  return e != cudaSuccess ? e : launch_after(k_apply_back<T, E>, q.grid, kThreads, 0, s, a, q.k, (const float*)avg);
}

template <typename T>
cudaError_t launch(const Norm& a, const Plan& q, bool back, void* ws, cudaStream_t s) {
  constexpr int kWide = 16 / sizeof(T);
  float* const w = static_cast<float*>(ws);
  if (a.B == 0 || a.S == 0) {
    if (!back && a.B) k_empty<<<(unsigned)((a.B * a.G + kThreads - 1) / kThreads), kThreads, 0, s>>>(a);
    if (back && (a.dgamma || a.dbeta)) return launch_weights(a, nullptr, 0, s);
    return cudaGetLastError();
  }
  if (q.slab) return launch_slab<T>(a, q, back, w, s);
  if (!q.team) {
    if (q.e == kWide) return launch_chunks<T, kWide>(a, q, back, w, s);
    return q.e == 2 ? launch_chunks<T, 2>(a, q, back, w, s) : launch_chunks<T, 1>(a, q, back, w, s);
  }
  if (q.e == kWide) return launch_teams<T, kWide>(a, q, back, w, s);
  if (q.e == 2) return launch_teams<T, 2>(a, q, back, w, s);
  return launch_teams<T, 1>(a, q, back, w, s);
}

int check(const net_norm* p, bool back) {
  if (!p) return fail(AUV_ERR_INVALID, "argument block is NULL");
  if (p->struct_size != sizeof(net_norm))
    return fail(AUV_ERR_INVALID, "struct_size %u, expected %zu", p->struct_size, sizeof(net_norm));
  if (p->dtype > NET_FP16) return fail(AUV_ERR_INVALID, "dtype %u unknown", p->dtype);
  if (p->act > NET_ACT_TANH) return fail(AUV_ERR_INVALID, "act %u unknown", p->act);
  if (p->B < 0 || p->S < 0 || p->C < 0) return fail(AUV_ERR_INVALID, "negative size");
  if (p->G < 1 || p->C % p->G) return fail(AUV_ERR_INVALID, "G < 1, or C not a multiple of G");
  if (!back && !(p->eps >= 0.0f && p->eps < INFINITY)) return fail(AUV_ERR_INVALID, "eps negative or not finite");
  if (p->C > (1 << 20) || p->B > INT32_MAX / 2 || p->S > INT32_MAX || p->B * p->G > INT32_MAX)
    return fail(AUV_ERR_UNSUPPORTED, "C past 2^20, B past 2^30, or S or B * G past 2^31");
  return AUV_OK;
}

int run(const net_norm* p, bool back, void* stream) {
  int rc = check(p, back);
  if (rc) return rc;
  const int z = type_size(p->dtype);
  if (p->C == 0) return AUV_OK;
  if (p->B && p->S) {
    if ((rc = need_rows(p->x, "x", p->B, p->S, p->C, z, false))) return rc;
    if (!back && (rc = need_rows(p->y, "y", p->B, p->S, p->C, z, true))) return rc;
    if (back && ((rc = need_rows(p->dy, "dy", p->B, p->S, p->C, z, false)) ||
                 (rc = need_rows(p->dx, "dx", p->B, p->S, p->C, z, true))))
      return rc;
  }
  if (p->B && ((rc = need(p->mean, "mean", 4)) || (rc = need(p->rstd, "rstd", 4)))) return rc;
  if ((p->gamma && (rc = need(p->gamma, "gamma", 4))) || (p->beta && (rc = need(p->beta, "beta", 4)))) return rc;
  if (back && ((p->dgamma && (rc = need(p->dgamma, "dgamma", 4))) || (p->dbeta && (rc = need(p->dbeta, "dbeta", 4)))))
    return rc;
  const Plan q = make_plan(p, back);
  const size_t ws = p->B && p->S ? q.bytes : 0;
  if (ws) {
    if (p->workspace_bytes < ws)
      return fail(AUV_ERR_SIZE, "workspace of %zu bytes, %zu needed", p->workspace_bytes, ws);
    if ((rc = need(p->workspace, "workspace", 16))) return rc;
  }
  const Norm a = {p->B, p->S, p->C, p->G, p->x, p->y, p->dy, p->dx, p->gamma, p->beta, p->mean, p->rstd,
                  p->dgamma, p->dbeta, p->eps, p->act};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p->dtype == NET_FP32   ? launch<float>(a, q, back, p->workspace, s)
                        : p->dtype == NET_BF16 ? launch<__nv_bfloat16>(a, q, back, p->workspace, s)
                                               : launch<__half>(a, q, back, p->workspace, s);
  return e == cudaSuccess ? AUV_OK : cuda_fail(e, back ? "net_group_norm_backward" : "net_group_norm");
}

}  // namespace
}  // namespace net
}  // namespace auv

extern "C" {

size_t net_group_norm_workspace_bytes(const net_norm* a, int backward) {
  using namespace auv::net;
  if (!a || check(a, backward) || !a->B || !a->S || !a->C) return 0;
  if (a->x.data && (backward ? a->dy.data && a->dx.data : a->y.data != nullptr)) return make_plan(a, backward).bytes;
  net_norm any = *a;
  any.x = any.y = any.dy = any.dx = net_rows{};
  any.dgamma = any.dbeta = reinterpret_cast<float*>(16);      // wanted; not read here
  size_t most = 0;
  for (int e = 8; e; e /= 2) most = std::max(most, make_plan(&any, backward, e).bytes);
  return most;
}

int net_group_norm(const net_norm* a, void* stream) { return auv::net::run(a, false, stream); }
int net_group_norm_backward(const net_norm* a, void* stream) { return auv::net::run(a, true, stream); }

}  // extern "C"
