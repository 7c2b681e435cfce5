// net_select.cu -- selective state space scan along a trajectory (auvnet.h, net_select_scan): forward, entry points.
//
// Per channel and state a chain h = a c + u B with a = exp(e A), u = e x: S exponentials and 4 S products and sums a value
// of x, against 8 to 16 bytes of it, so with S = 16 the multi-function unit, the fp32 pipe and HBM are all near their
// limits.  k_select walks the steps with the states in registers (layout: net_select.cuh), B and C of four steps staged in
// shared memory by each warp for itself.  Sequences of few channels are cut into pieces: each is walked from 0 for its
// final state and the sum of its step sizes (the product of its decays is exp(A sum)), those are joined to the states
// before the pieces (k_select_join), and the pieces are walked from these.
//
// 128 steps of 4,096 envs x 256 channels x 16 states of bf16, states kept: 671 us (HBM alone 262, exponentials 230): 12 warps
// an SM, two channels a lane each, wait for their own instructions half of the time.  65,521 steps of 250 x 13 fp32: 162 us, of
// which 60 the fold, 85 the walk and the rest the join.
#include <algorithm>

#include "net_select.cuh"

namespace auv {
namespace net {
namespace {

constexpr int kWarps = 4;
constexpr int kBatch = 4;       // steps whose inputs are on their way while as many are computed

// FOLD: only the piece's final state from 0, and the sum of its step sizes (-1 where an episode ends in it: nothing
// passes through).
template <typename T, typename L, bool FOLD>
__global__ void __launch_bounds__(32 * kWarps, L::OWN > 1 ? 3 : L::SP == 8 ? 4 : 6) k_select(Select a) {
  constexpr int SP = L::SP, LS = L::LS, CC = L::CC, SW = L::SW, OWN = L::OWN, kSides = CC / OWN, R = L::R, RL = L::RL;
  using In = Staged<T, SW, kBatch, RL>;
  using W = Raw<T, OWN>;
  __shared__ __align__(16) float rows[kWarps][FOLD ? 1 : 2][R][kBatch * SW];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int64_t id = blockIdx.x * (int64_t)kWarps + warp;
  const int64_t envs_groups = (a.N * a.G + R - 1) / R;         // rows, or fours of them
  if (id >= envs_groups * a.tiles * a.pieces) return;
  const int tile = (int)(id % a.tiles), side = lane / RL, mine = lane % RL;
  id /= a.tiles;
  int g, piece;
  int64_t n;
  bool row_there = true;
  if constexpr (R == 1) {                                     // as below, but every lane's the same
    g = (int)(id % a.G);
    id /= a.G;
    n = id % a.N;
    piece = (int)(id / a.N);
  } else {
    const int64_t row = id % envs_groups * R + side;
    row_there = row < a.N * a.G;
    g = row_there ? (int)(row % a.G) : 0;
    n = row_there ? row / a.G : 0;
    piece = (int)(id / envs_groups);
  }
  float* const Bs = rows[warp][0][side];
  float* const Cs = rows[warp][FOLD ? 0 : 1][side];

  const int q = mine % LS, s0 = q * SP;
  const int first = tile * L::CW + mine / LS * CC;            // in the group
  const int own = first + q % kSides * OWN;
  const bool live = row_there && own < a.per, writes = live && q < kSides;   // OWN = 2: channels of a group are even in number
  const int64_t d = (int64_t)g * a.per + own;                 // own channels
  int64_t at[CC], at_weight[CC];
  bool there[CC];
#pragma unroll
  for (int c = 0; c < CC; ++c) {
    const int k = first + (q % kSides ^ c / OWN) * OWN + c % OWN;
    at_weight[c] = (int64_t)g * a.per + k;
    at[c] = n * a.D + at_weight[c];
    there[c] = row_there && k < a.per;
  }
  const int t0 = piece * a.piece, t1 = min(a.T, t0 + a.piece);
  const int64_t states = a.N * a.D * a.S;
  const bool gated = !FOLD && a.gate.data, flagged = a.done || a.done_prev;
  const T* px = row_at<T>(a.x, t0, n, d);
  const T* pdt = row_at<T>(a.dt, t0, n, d);
  const T* pgate = gated ? row_at<T>(a.gate, t0, n, d) : px;
  T* py = FOLD ? nullptr : const_cast<T*>(row_at<T>(a.y, t0, n, d));
  const int64_t in_row = (int64_t)g * a.S + mine % In::kSide;
  const T* pB = row_at<T>(a.B, t0 + mine / In::kSide, n, in_row);
  const T* pC = row_at<T>(a.C, t0 + mine / In::kSide, n, in_row);
  W rx[kBatch], rdt[kBatch], rgate[kBatch];
  In rB, rC;
  uint8_t rend = 0;
  const bool all_live = __all_sync(0xffffffffu, live);
  auto get = [](const T* p, int64_t at) { return *reinterpret_cast<const W*>(p + at); };
  auto fetch = [&](int t) {
    const int steps = t1 - t;
    if (steps <= 0) return;
    rend = flagged && mine < min(kBatch, steps) ? flag_at(a, t + mine, n) : (uint8_t)0;
    rB.load(pB, a.B.outer, steps, a.S, mine);
    if constexpr (!FOLD) rC.load(pC, a.C.outer, steps, a.S, mine);
    if (all_live && steps >= kBatch) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) rx[k] = get(px, k * a.x.outer), rdt[k] = get(pdt, k * a.dt.outer);
      if (gated) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) rgate[k] = get(pgate, k * a.gate.outer);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        rx[k] = rdt[k] = rgate[k] = W{};
        if (live && k < steps) {
          rx[k] = get(px, k * a.x.outer), rdt[k] = get(pdt, k * a.dt.outer);
          if (gated) rgate[k] = get(pgate, k * a.gate.outer);
        }
      }
    }
    px += kBatch * a.x.outer, pdt += kBatch * a.dt.outer, pB += kBatch * a.B.outer;
    if (gated) pgate += kBatch * a.gate.outer;
    if constexpr (!FOLD) pC += kBatch * a.C.outer;
  };
  fetch(t0);

  F2 h[CC][SP / 2], A2[CC][SP / 2];
  if constexpr (!FOLD) {
    if (a.pieces > 1) {
      after_previous();
      load_states<SP, CC>(a.maps + piece * states, at, there, s0, a.S, h);
    } else {
      load_states<SP, CC>(a.h0, at, there, s0, a.S, h);
    }
  } else {
#pragma unroll
    for (int c = 0; c < CC; ++c)
#pragma unroll
      for (int i = 0; i < SP / 2; ++i) h[c][i] = pair(0.0f, 0.0f);
  }
  load_states<SP, CC>(a.A, at_weight, there, s0, a.S, A2);
#pragma unroll
  for (int c = 0; c < CC; ++c)
#pragma unroll
    for (int i = 0; i < SP / 2; ++i) A2[c][i] = A2[c][i] * pair(kLog2e, kLog2e);
  float bias[OWN], skip[OWN], sum[OWN];
#pragma unroll
  for (int j = 0; j < OWN; ++j) {
    bias[j] = live && a.dt_bias ? a.dt_bias[d + j] : 0.0f;
    skip[j] = live && a.skip ? a.skip[d + j] : 0.0f;
    sum[j] = 0.0f;
  }
  bool cut = false;

#pragma unroll 1
  for (int ts = t0; ts < t1; ts += kBatch) {
    const int steps = t1 - ts;
    __syncwarp();                                             // the last batch's rows are read
    rB.put(Bs, mine);
    if constexpr (!FOLD) rC.put(Cs, mine);
    const uint32_t any_ends = flagged ? __ballot_sync(0xffffffffu, rend != 0) : 0u, ends = any_ends >> (side * RL % 32);
    float x[kBatch][OWN], e[kBatch][OWN], z[kBatch][OWN];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      unpack<T, OWN>(rx[k], x[k]);
      unpack<T, OWN>(rdt[k], e[k]);
#pragma unroll
      for (int j = 0; j < OWN; ++j) {
        e[k][j] = softplus(e[k][j] + bias[j]);
        z[k][j] = 1.0f;
      }
    }
    if (gated) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        unpack<T, OWN>(rgate[k], z[k]);
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
          float s, o;
          gates(z[k][j], s, o);
          z[k][j] *= s;
        }
      }
    }
    fetch(ts + kBatch);
    if constexpr (!FOLD)
      if (a.kept && ts % kKeep == 0) store_states<SP, CC>(a.kept + ts / kKeep * states, at, there, s0, a.S, h);
    __syncwarp();
    // PLAIN: four steps there are, and no end among them; straight through, which took 1.3 times as long with the questions
    auto walk = [&](auto plain) {
      constexpr bool kPlain = decltype(plain)::value;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (!kPlain && k >= steps) break;
        float es[CC], us[CC], u[OWN];
#pragma unroll
        for (int j = 0; j < OWN; ++j) u[j] = e[k][j] * x[k][j];
        to_lanes<CC, OWN>(e[k], es);
        to_lanes<CC, OWN>(u, us);
        F2 B[SP / 2], C[SP / 2];
        load_pairs<SP>(Bs + k * SW + s0, B);
        if constexpr (!FOLD) load_pairs<SP>(Cs + k * SW + s0, C);
        if (!kPlain && (ends >> k & 1u)) {
#pragma unroll
          for (int c = 0; c < CC; ++c)
#pragma unroll
            for (int i = 0; i < SP / 2; ++i) h[c][i] = pair(0.0f, 0.0f);
          cut = true;
        }
        float y[CC];
#pragma unroll
        for (int c = 0; c < CC; ++c) {
          const F2 e2 = pair(es[c], es[c]), u2 = pair(us[c], us[c]);
          F2 acc = pair(0.0f, 0.0f);
#pragma unroll
          for (int i = 0; i < SP / 2; ++i) {
            h[c][i] = fma2(decay_of(e2, A2[c][i]), h[c][i], u2 * B[i]);
            if constexpr (!FOLD) acc = i ? fma2(C[i], h[c][i], acc) : C[i] * h[c][i];
          }
          y[c] = total(acc);
        }
        if constexpr (FOLD) {
#pragma unroll
          for (int j = 0; j < OWN; ++j) sum[j] += e[k][j];
        } else {
          float p[OWN];
          over_states<LS, CC, OWN>(y, p);
#pragma unroll
          for (int j = 0; j < OWN; ++j) p[j] = fmaf(skip[j], x[k][j], p[j]) * z[k][j];
          if constexpr (OWN == 1) store_if(writes, py + k * a.y.outer, p[0]);
          else if (writes) store<T, OWN>(py + k * a.y.outer, p);
        }
      }
    };
    if (steps >= kBatch && !any_ends) walk(std::true_type());
    else walk(std::false_type());
    py += kBatch * a.y.outer;
  }
  if constexpr (FOLD) {
    store_states<SP, CC>(a.maps + piece * states, at, there, s0, a.S, h);
    if (writes) {
#pragma unroll
      for (int j = 0; j < OWN; ++j) a.sums[(int64_t)piece * a.N * a.D + n * a.D + d + j] = cut ? -1.0f : sum[j];
    }
  } else {
    if (a.hT && t1 == a.T) store_states<SP, CC>(a.hT, at, there, s0, a.S, h);
  }
}

// The states before the pieces (backward: their gradients behind the pieces), in the place of the pieces' own.  A block has
// some states and all pieces: each of its groups of threads folds adjacent pieces to one, those are joined over the block, and
// the groups go through their pieces once more from the state they begin with.  293 pieces of 4,000 states: 12 us in 64 groups,
// 40 by one thread a state, which is enough for a few pieces.
constexpr int kJoin = 512, kJoinGroups = 64, kJoinAhead = 4;
// A state behind a piece: that before it times the product of the piece's decays, 2^(A2 sum), and the piece's own.  The product
// may be out of fp32's range where the state behind it is not (2^140 of one of 2^-100): as 2^126, or 2^-126, and twice the root
// of the rest, so none of the factors is 0 or infinite, and a state of 0 stays 0 and an infinite one infinite, as step by step.
// 2^360 takes the smallest number past the largest, and 2^-360 the other way.  (Where the power is NaN, so is the piece's own.)
__device__ __forceinline__ float through_piece(float A2, float sum, float state, float own) {
  const float power = A2 * sum, most = fminf(fmaxf(power, -126.0f), 126.0f);
  const float root = ex2(fminf(fmaxf((power - most) * 0.5f, -117.0f), 117.0f));     // 1, mostly
  return fmaf(ex2(most), state * root * root, own);
}
__global__ void __launch_bounds__(kJoin) k_select_join(Select a, bool back, int groups) {
  __shared__ float sums[kJoin], owns[kJoin];
  after_previous();
  const int side = kJoin / groups;                              // states of the block
  const int k = threadIdx.x % side, group = threadIdx.x / side;
  const int64_t m = a.N * a.D * a.S, i = blockIdx.x * (int64_t)side + k;
  const bool live = i < m;
  const int64_t nd = live ? i / a.S : 0, all = a.N * a.D;
  const float A2 = live ? a.A[nd % a.D * a.S + i % a.S] * kLog2e : 0.0f;
  // pieces in the chain's order: backward the last one first
  const int each = (a.pieces + groups - 1) / groups, p0 = min(a.pieces, group * each);
  const int n = live ? min(a.pieces, p0 + each) - p0 : 0;
  const int64_t first = back ? a.pieces - 1 - p0 : p0, by = back ? -1 : 1;
  float total = 0.0f, state = 0.0f;
  auto through = [&](bool put) {
    for (int q = 0; q < n; q += kJoinAhead) {
      float sum[kJoinAhead], own[kJoinAhead];
#pragma unroll
      for (int u = 0; u < kJoinAhead; ++u)
        if (q + u < n) {
          sum[u] = a.sums[(first + (q + u) * by) * all + nd];
          own[u] = a.maps[(first + (q + u) * by) * m + i];
        }
#pragma unroll
      for (int u = 0; u < kJoinAhead; ++u)
        if (q + u < n) {
          if (put) a.maps[(first + (q + u) * by) * m + i] = state;
          else total = sum[u] < 0.0f || total < 0.0f ? -1.0f : total + sum[u];
          state = sum[u] < 0.0f ? own[u] : through_piece(A2, sum[u], state, own[u]);
        }
    }
  };
  if (groups > 1) through(false);
  sums[threadIdx.x] = total, owns[threadIdx.x] = state;
  __syncthreads();
  if (group == 0) {
    const float* const from = back ? a.dhT : a.h0;
    float h = live && from ? from[i] : 0.0f;
#pragma unroll 4
    for (int q = 0; q < groups; ++q) {
      const float sum = sums[q * side + k], own = owns[q * side + k];
      owns[q * side + k] = h;
      h = sum < 0.0f ? own : through_piece(A2, sum, h, own);
    }
  }
  __syncthreads();
  state = owns[threadIdx.x];
  through(true);
}

// One step, as in a rollout: the states are read, changed and written, so few registers and no staging; a warp takes its
// channels of one env after the other, A in registers (65,536 envs x 256 x 16 of bf16: 350 us, 6.5 TB/s).  wide: B's and C's
// values of a lane are aligned vectors, of a lane that has states (there); one past them (S = 24: the last of four) has zeros.
template <typename T, int SP>
__device__ __forceinline__ void load_row(const T* p, bool wide, bool there, int s0, int S, F2 (&v)[SP / 2]) {
  float x[SP];
  if (!there) {
#pragma unroll
    for (int i = 0; i < SP; ++i) x[i] = 0.0f;
  } else if (wide) {
    constexpr int E = SP * sizeof(T) > 16 ? 16 / sizeof(T) : SP;
#pragma unroll
    for (int i = 0; i < SP; i += E) {
      float y[E];
      load<T, E>(p + i, y);
#pragma unroll
      for (int e = 0; e < E; ++e) x[i + e] = y[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < SP; ++i) x[i] = s0 + i < S ? to_float(p[i]) : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < SP / 2; ++i) v[i] = pair(x[2 * i], x[2 * i + 1]);
}

// whole: every lane's channels and states are there, and whole sectors; then the next env's are on their way while one is
// computed.
constexpr int kOneWarps = 4;
template <int SP, int CC>
__device__ __forceinline__ void load_whole(const float* p, const int (&at)[CC], F2 (&h)[CC][SP / 2]) {
#pragma unroll
  for (int c = 0; c < CC; ++c) {
    if constexpr (SP == 8) {
      asm volatile("ld.global.v4.b64 {%0, %1, %2, %3}, [%4];"
                   : "=l"(h[c][0].v), "=l"(h[c][1].v), "=l"(h[c][2].v), "=l"(h[c][3].v)
                   : "l"(p + at[c])
                   : "memory");
    } else {
      const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(p + at[c]);
      h[c][0].v = w.x, h[c][1].v = w.y;
    }
  }
}
template <int SP, int CC>
__device__ __forceinline__ void store_whole(float* p, const int (&at)[CC], const F2 (&h)[CC][SP / 2]) {
#pragma unroll
  for (int c = 0; c < CC; ++c) {
    if constexpr (SP == 8)
      asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p + at[c]), "l"(h[c][0].v), "l"(h[c][1].v), "l"(h[c][2].v),
                   "l"(h[c][3].v)
                   : "memory");
    else
      *reinterpret_cast<ulonglong2*>(p + at[c]) = make_ulonglong2(h[c][0].v, h[c][1].v);
  }
}

template <typename T, typename L, bool WHOLE>
__global__ void __launch_bounds__(32 * kOneWarps, 4) k_select_one(Select a, bool wide) {
  constexpr int SP = L::SP, LS = L::LS, CC = L::CC, P = SP / 2;
  const int lane = threadIdx.x % 32;
  const int g = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles;
  const int64_t envs = gridDim.y * (int64_t)kOneWarps;                  // walked side by side
  int64_t n = blockIdx.y * (int64_t)kOneWarps + threadIdx.x / 32;
  if (n >= a.N) return;
  const int q = lane % LS, s0 = q * SP;
  const int first = tile * L::CW + lane / LS * CC, own = first + q % CC;
  const bool live = own < a.per, writes = live && q < CC;
  const int64_t d = (int64_t)g * a.per + own;
  int64_t at_weight[CC];
  int to[CC];                                                           // of an env's states
  bool there[CC];
#pragma unroll
  for (int c = 0; c < CC; ++c) {
    const int k = first + (q % CC ^ c);
    at_weight[c] = (int64_t)g * a.per + k;
    to[c] = (int)at_weight[c] * a.S + s0;
    there[c] = k < a.per;
  }
  F2 A2[CC][P];
  load_states<SP, CC>(a.A, at_weight, there, s0, a.S, A2);
  const float bias = live && a.dt_bias ? a.dt_bias[d] : 0.0f, skip = live && a.skip ? a.skip[d] : 0.0f;
#pragma unroll
  for (int c = 0; c < CC; ++c)
#pragma unroll
    for (int i = 0; i < P; ++i) A2[c][i] = A2[c][i] * pair(kLog2e, kLog2e);
  const int64_t in_row = (int64_t)g * a.S + s0, each = a.D * a.S;
  const bool gated = a.gate.data;
  T rx, rdt, rgate;
  uint8_t rend = 0;
  F2 next[CC][P], B[P], C[P];
  auto fetch = [&](int64_t n) {
    if constexpr (WHOLE) {
      if (a.h0) {
        load_whole<SP, CC>(a.h0 + n * each, to, next);
      } else {
#pragma unroll
        for (int c = 0; c < CC; ++c)
#pragma unroll
          for (int i = 0; i < P; ++i) next[c][i] = pair(0.0f, 0.0f);
      }
    } else {
      int64_t at[CC];
#pragma unroll
      for (int c = 0; c < CC; ++c) at[c] = n * a.D + at_weight[c];
      load_states<SP, CC>(a.h0, at, there, s0, a.S, next);
    }
    from_float(0.0f, rx);
    rdt = rgate = rx;
    if (WHOLE || live) {
      rx = *row_at<T>(a.x, 0, n, d);
      rdt = *row_at<T>(a.dt, 0, n, d);
      if (gated) rgate = *row_at<T>(a.gate, 0, n, d);
    }
    load_row<T, SP>(row_at<T>(a.B, 0, n, in_row), WHOLE || wide, WHOLE || s0 < a.S, s0, a.S, B);
    load_row<T, SP>(row_at<T>(a.C, 0, n, in_row), WHOLE || wide, WHOLE || s0 < a.S, s0, a.S, C);
    if (a.done_prev) rend = a.done_prev[n];
  };
  fetch(n);
  for (; n < a.N; n += envs) {
    F2 h[CC][P];
    int64_t at[CC];
#pragma unroll
    for (int c = 0; c < CC; ++c) {
      at[c] = n * a.D + at_weight[c];
#pragma unroll
      for (int i = 0; i < P; ++i) h[c][i] = next[c][i];
    }
    if (a.kept) store_states<SP, CC>(a.kept, at, there, s0, a.S, h);
    const float x = to_float(rx), e = WHOLE || live ? softplus(to_float(rdt) + bias) : 0.0f;
    float z = 1.0f;
    if (gated) {
      float s, o;
      z = to_float(rgate);
      gates(z, s, o);
      z *= s;
    }
    if (rend) {
#pragma unroll
      for (int c = 0; c < CC; ++c)
#pragma unroll
        for (int i = 0; i < P; ++i) h[c][i] = pair(0.0f, 0.0f);
    }
    F2 uB[P], oC[P];
#pragma unroll
    for (int i = 0; i < P; ++i) uB[i] = B[i], oC[i] = C[i];
    if (WHOLE && n + envs < a.N) fetch(n + envs);
    float es[CC], us[CC], y[CC];
    to_lanes<CC>(e, es);
    to_lanes<CC>(e * x, us);
#pragma unroll
    for (int c = 0; c < CC; ++c) {
      const F2 u2 = pair(us[c], us[c]);
      F2 acc;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        h[c][i] = fma2(decay_of(es[c], A2[c][i]), h[c][i], u2 * uB[i]);
        acc = i ? fma2(oC[i], h[c][i], acc) : oC[i] * h[c][i];
      }
      y[c] = total(acc);
    }
    if (a.hT) {
      if constexpr (WHOLE) store_whole<SP, CC>(a.hT + n * each, to, h);
      else store_states<SP, CC>(a.hT, at, there, s0, a.S, h);
    }
    store_if(writes, const_cast<T*>(row_at<T>(a.y, 0, n, d)), fmaf(skip, x, over_states<LS, CC>(y)) * z);
    if (!WHOLE && n + envs < a.N) fetch(n + envs);
  }
}

// T = 0: the states pass as they are.
__global__ void k_select_none(int64_t m, const float* from, float* to) {
  const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
  if (i < m) to[i] = from ? from[i] : 0.0f;
}

// No channels: sums over nothing.
template <typename T>
__global__ void k_select_no_channels(net_rows r, int64_t T_, int64_t N, int64_t k) {
  const int64_t step = gridDim.x * (int64_t)256;
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < T_ * N * k; i += step)
    from_float(0.0f, *const_cast<T*>(row_at<T>(r, i / (N * k), i / k % N, i % k)));
}

template <typename T, typename L, bool FOLD>
cudaError_t launch_walk(const Select& a, cudaStream_t s) {
  const int64_t warps = (a.N * a.G + L::R - 1) / L::R * a.tiles * a.pieces;
  const dim3 grid((unsigned)((warps + kWarps - 1) / kWarps));
  if (!FOLD && a.pieces > 1) return launch_after(k_select<T, L, FOLD>, grid, 32 * kWarps, 0, s, a);
  k_select<T, L, FOLD><<<grid, 32 * kWarps, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T, typename L>
cudaError_t launch_all(const Select& a, cudaStream_t s) {
  if (a.pieces > 1) {
    cudaError_t e = launch_walk<T, L, true>(a, s);
    if (e == cudaSuccess) e = launch_select_join(a, false, s);
    if (e != cudaSuccess) return e;
  }
  return launch_walk<T, L, false>(a, s);
}

template <typename T>
cudaError_t launch(const Select& a, cudaStream_t s) {
  if (a.rows > 1) return with_narrow_lanes(a.S, [&](auto l) { return launch_all<T, decltype(l)>(a, s); });
  if (a.wide) return with_wide_lanes(a.S, [&](auto l) { return launch_all<T, decltype(l)>(a, s); });
  return with_lanes(a.S, [&](auto l) {
    using L = decltype(l);
    if (a.T == 1) {
      const int z = sizeof(T);
      const int64_t side = (int64_t)a.G * a.tiles;
      const net_rows* rows[] = {&a.B, &a.C};
      bool wide = a.S % L::SP == 0;
      for (const net_rows* r : rows) wide = wide && aligned(*r, 1, a.N, z, std::min(L::SP, 16 / z));
      auto sectors = [&](const void* p) { return reinterpret_cast<uintptr_t>(p) % (4 * L::SP) == 0; };
      const bool whole = wide && a.S == L::SW && a.per % L::CW == 0 && sectors(a.h0) && sectors(a.hT);
      // as many warps as the SMs hold at a time walk the envs
      const int64_t few = (int64_t)sm_count() * 4, all = (a.N + kOneWarps - 1) / kOneWarps;
      const int64_t blocks = std::min<int64_t>(65535, std::max<int64_t>(1, std::min(all, (few + side - 1) / side)));
      const dim3 grid((unsigned)side, (unsigned)blocks);
      if (whole) k_select_one<T, L, true><<<grid, 32 * kOneWarps, 0, s>>>(a, true);
      else k_select_one<T, L, false><<<grid, 32 * kOneWarps, 0, s>>>(a, wide);
      return cudaGetLastError();
    }
    return launch_all<T, L>(a, s);
  });
}

int check(const net_select* p) {
  if (!p) return fail(AUV_ERR_INVALID, "argument block is NULL");
  if (p->struct_size != sizeof(net_select))
    return fail(AUV_ERR_INVALID, "struct_size %u, expected %zu", p->struct_size, sizeof(net_select));
  if (p->dtype > NET_FP16) return fail(AUV_ERR_INVALID, "dtype %u unknown", p->dtype);
  if (p->T < 0 || p->N < 0 || p->D < 0) return fail(AUV_ERR_INVALID, "negative size");
  if (p->S < 1 || p->G < 1) return fail(AUV_ERR_INVALID, "S or G < 1");
  if (p->D % p->G) return fail(AUV_ERR_INVALID, "D is no multiple of G");
  if (p->S > kMostStates) return fail(AUV_ERR_UNSUPPORTED, "S past %d", kMostStates);
  const int64_t most = (int64_t)1 << 32;
  if (p->N > most || p->D > (1 << 20) || p->G > (1 << 20) || p->N * std::max<int64_t>(p->D, p->G) > most || p->T > (1 << 30))
    return fail(AUV_ERR_UNSUPPORTED, "N * D or N * G past 2^32, D or G past 2^20, or T past 2^30");
  return AUV_OK;
}

Select of(const net_select* p, bool back, bool narrow = false) {
  Select a = {};
  a.T = (int)p->T, a.S = (int)p->S, a.G = (int)p->G, a.per = (int)(p->D / p->G), a.N = p->N, a.D = p->D;
  a.x = p->x, a.dt = p->dt, a.gate = p->gate, a.y = p->y, a.B = p->B, a.C = p->C, a.dy = p->dy, a.dx = p->dx;
  a.ddt = p->ddt, a.dgate = p->dgate, a.dB = p->dB, a.dC = p->dC;
  a.A = p->A, a.skip = p->skip, a.dt_bias = p->dt_bias, a.h0 = p->h0, a.hT = p->hT, a.kept = p->kept, a.dhT = p->dhT;
  a.dh0 = p->dh0, a.dA = p->dA, a.dskip = p->dskip, a.ddt_bias = p->ddt_bias, a.done = p->done, a.done_prev = p->done_prev;
  a.tiles = (a.per + lanes_channels(a.S) - 1) / lanes_channels(a.S);
  // pairs of channels a lane where every access of two is aligned and enough warps are left: pieces of a long sequence are
  // the shorter the more warps there are (65,521 steps of 250 channels x 13 fp32: 176 us in pairs, 161 not)
  const net_rows* rows[] = {&a.x, &a.dt, &a.gate, &a.y};
  const int z = type_size(p->dtype), tiles = (a.per + kWideChannels - 1) / kWideChannels;
  bool pairs = !back && !narrow && a.T > 1 && a.S <= kMostWide && a.per % 2 == 0;
  for (const net_rows* r : rows) pairs = pairs && aligned(*r, a.T, a.N, z, 2);
  a.wide = pairs && a.N * a.G * tiles >= (int64_t)sm_count() * 12;
  if (a.wide) a.tiles = tiles;
  // narrow groups: lanes that would be idle take other rows (1,374 steps of 1,137 envs x 2 groups of 8 channels x 16 fp32: 288 us,
  // 2,139 with a row a warp)
  a.rows = (back || a.T > 1) && a.per <= kNarrow && a.S <= kMostWide ? kSide4 : 1;
  if (a.rows > 1) a.wide = false, a.tiles = 1;
  select_pieces(a, back);
  return a;
}

// The workspace's parts, each on a 16-byte boundary, and its size.
size_t lay_out(Select& a, bool back, char* at) {
  size_t n = 0;
  auto part = [&](int64_t floats) {
    float* const p = reinterpret_cast<float*>(at + n);
    n += ((size_t)floats * 4 + 15) / 16 * 16;
    return floats ? p : nullptr;
  };
  const bool split = a.pieces > 1;
  a.sums = part(split ? a.pieces * a.N * a.D : 0);
  a.maps = part(split ? a.pieces * a.N * a.D * a.S : 0);
  if (back) {
    int64_t blocks;
    int rows;
    const int64_t slots = select_slots(a, &blocks, &rows);
    a.weights = part(slots * a.D * (a.S + 2));
    a.parts = part(blocks > 1 ? blocks * a.T * a.N * a.G * 2 * a.S : 0);
  }
  return n;
}

int run(const net_select* p, bool back, void* stream) {
  int rc = check(p);
  if (rc) return rc;
  const int z = type_size(p->dtype);
  const int64_t GS = p->G * p->S;
  if (p->D == 0) {
    const int64_t all = back ? p->T * p->N * GS : 0;
    const net_rows* const sums[] = {&p->dB, &p->dC};
    for (int i = 0; i < 2 && all; ++i) {
      if ((rc = need_rows(*sums[i], i ? "dC" : "dB", p->T, p->N, GS, z, true))) return rc;
      const unsigned blocks = (unsigned)std::min<int64_t>((all + 255) / 256, 65535);
      if (z == 4) k_select_no_channels<float><<<blocks, 256, 0, static_cast<cudaStream_t>(stream)>>>(*sums[i], p->T, p->N, GS);
      else k_select_no_channels<__half><<<blocks, 256, 0, static_cast<cudaStream_t>(stream)>>>(*sums[i], p->T, p->N, GS);
    }
    const cudaError_t e = all ? cudaGetLastError() : cudaSuccess;
    return e == cudaSuccess ? AUV_OK : cuda_fail(e, "net_select_scan_backward");
  }
  if (p->N == 0 && !back) return AUV_OK;
  const bool gate = p->gate.data != nullptr;
  struct { const net_rows* r; const char* name; bool out, used; int64_t k; } rows[] = {
      {&p->x, "x", false, true, p->D},        {&p->dt, "dt", false, true, p->D},   {&p->gate, "gate", false, gate, p->D},
      {&p->B, "B", false, true, GS},          {&p->C, "C", false, true, GS},       {&p->y, "y", true, !back, p->D},
      {&p->dy, "dy", false, back, p->D},      {&p->dx, "dx", true, back, p->D},    {&p->ddt, "ddt", true, back, p->D},
      {&p->dgate, "dgate", true, back && gate && p->dgate.data, p->D},
      {&p->dB, "dB", true, back, GS},         {&p->dC, "dC", true, back, GS}};
  if (p->T && p->N)
    for (const auto& q : rows)
      if (q.used && (rc = need_rows(*q.r, q.name, p->T, p->N, q.k, z, q.out))) return rc;
  if ((rc = need(p->A, "A", 4))) return rc;
  if (back && p->T && p->N && (rc = need(p->kept, "kept", 4))) return rc;
  struct { const void* p; const char* name; bool used; } flat[] = {
      {p->skip, "skip", true}, {p->dt_bias, "dt_bias", true}, {p->h0, "h0", !back}, {p->hT, "hT", !back}, {p->kept, "kept", !back},
      {p->dhT, "dhT", back}, {p->dh0, "dh0", back}, {p->dA, "dA", back}, {p->dskip, "dskip", back}, {p->ddt_bias, "ddt_bias", back}};
  for (const auto& q : flat)
    if (q.p && q.used && (rc = need(q.p, q.name, 4))) return rc;
  if (p->done && (rc = need(p->done, "done", 1))) return rc;
  if (p->done_prev && (rc = need(p->done_prev, "done_prev", 1))) return rc;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (p->T == 0 || p->N == 0) {
    const int64_t m = p->N * p->D * p->S;
    auto fill = [&](int64_t k, const float* from, float* to) {
      if (to && k) k_select_none<<<(unsigned)((k + 255) / 256), 256, 0, s>>>(k, from, to);
    };
    if (back) {
      fill(m, p->dhT, p->dh0);
      fill(p->D * p->S, nullptr, p->dA);
      fill(p->D, nullptr, p->dskip);
      fill(p->D, nullptr, p->ddt_bias);
    } else {
      fill(m, p->h0, p->hT);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? AUV_OK : cuda_fail(e, "net_select_scan");
  }
  Select a = of(p, back);
  const size_t bytes = lay_out(a, back, static_cast<char*>(p->workspace));
  if (bytes) {
    if (p->workspace_bytes < bytes) return fail(AUV_ERR_SIZE, "workspace of %zu bytes, %zu needed", p->workspace_bytes, bytes);
    if ((rc = need(p->workspace, "workspace", 16))) return rc;
  }
  cudaError_t e;
  if (back) {
    if (!gate) a.dgate.data = nullptr;
    e = p->dtype == NET_FP32   ? launch_select_back<float>(a, a.pieces > 1, s)
        : p->dtype == NET_BF16 ? launch_select_back<__nv_bfloat16>(a, a.pieces > 1, s)
                               : launch_select_back<__half>(a, a.pieces > 1, s);
  } else {
    e = p->dtype == NET_FP32 ? launch<float>(a, s) : p->dtype == NET_BF16 ? launch<__nv_bfloat16>(a, s) : launch<__half>(a, s);
  }
  return e == cudaSuccess ? AUV_OK : cuda_fail(e, back ? "net_select_scan_backward" : "net_select_scan");
}

}  // namespace

void select_pieces(Select& a, bool back) {
  const int64_t warps = (a.N * a.G + a.rows - 1) / a.rows * a.tiles, want = (int64_t)sm_count() * (!back ? 16 : a.S <= 8 ? 12 : 8);
  int64_t pieces = std::min(want / std::max<int64_t>(1, warps), (int64_t)a.T / 64);
  if (pieces < 2) pieces = 1;
  const int64_t piece = pieces == 1 ? a.T : ((a.T + pieces - 1) / pieces + kKeep - 1) / kKeep * kKeep;
  a.piece = (int)std::max<int64_t>(1, piece);
  a.pieces = a.T ? (a.T + a.piece - 1) / a.piece : 1;
}

cudaError_t launch_select_join(const Select& a, bool back, cudaStream_t s) {
  const int64_t m = a.N * a.D * a.S;
  int groups = 1;
  while (groups < kJoinGroups && a.pieces > 4 * groups) groups *= 2;
  const int side = kJoin / groups;
  return launch_after(k_select_join, dim3((unsigned)((m + side - 1) / side)), kJoin, 0, s, a, back, groups);
}

}  // namespace net
}  // namespace auv

extern "C" {

size_t net_select_scan_workspace_bytes(const net_select* p, int backward) {
  using namespace auv::net;
  if (!p || check(p) || !p->T || !p->N || !p->D) return 0;
  Select a = of(p, backward), b = of(p, backward, true);
  return std::max(lay_out(a, backward, nullptr), lay_out(b, backward, nullptr));
}

int net_select_scan(const net_select* a, void* stream) { return auv::net::run(a, false, stream); }
int net_select_scan_backward(const net_select* a, void* stream) { return auv::net::run(a, true, stream); }

}  // extern "C"
