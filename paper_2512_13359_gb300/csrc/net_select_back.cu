// net_select_back.cu -- gradients of the selective scan (auvnet.h, net_select_scan_backward).
//
// The chain of gradients runs from the last step to the first, and every step needs its states.  A segment of 16 steps
// starts again from its kept state: a first pass keeps the states before every 4th step (shared memory), then, last two
// steps first, a second pass holds a = exp(e A) and a c of two steps in registers and sums y and dC on its way, and the
// gradients run back through the two.  Per state and step some 16 fp32 operations and 2.25 exponentials.  Sums over a
// channel's states (y and the two that dx and ddt are made of) go over 1 to 16 lanes; dB and dC are sums over the channels
// of a group, over the lanes with one shuffle a value (each lane keeps half of its values at every level) and over the
// block's warps in shared memory at the end of a segment; groups wider than a block leave partial sums, which k_select_rows
// adds.  Weight gradients stay in registers over an env's piece.  Every sum has a fixed order.
//
// 128 steps of 4,096 envs x 256 channels x 16 states of bf16: 3.9 ms (the fp32 pipe alone 0.7): 255 registers a thread and 28 KB
// of shared memory a warp, either of them, leave 8 warps an SM, which wait for each other's latencies.  One channel a lane with 16 warps took 5.1 ms (every lane does a whole channel's
// and step's own work), four steps held instead of two 4.2 (spills).
#include <algorithm>

#include "net_select.cuh"

namespace auv {
namespace net {
namespace {

// Steps whose a and a c are held in registers (four: 176 registers of them, and spills), and from one kept start to the next.
constexpr int kHeld = 2, kSub = 4;

// Warps of a block: shared memory grows with the padded states.
constexpr int back_warps(int padded, int rows) {
  return rows > 1 ? 5 : padded <= 8 ? 4 : padded <= 16 ? 8 : padded <= 64 ? 4 : 2;
}
// Blocks of an SM: of up to 8 states a lane has one channel's, and three blocks of four warps fit (8,192 steps of 3 x 200
// channels x 8 fp16: 147 us, 200 with one block of eight).
constexpr int back_blocks(int padded, int rows) { return padded > 8 ? 1 : rows > 1 ? 2 : 3; }

// A warp's shared memory.  What multiplies pairs of states is there twice: copies in registers took a twelfth of all
// instructions.
template <typename L> struct Back {
  float B[L::R][kKeep][L::SW], C[L::R][kKeep][L::SW];
  static constexpr bool kTwice = L::CC == 2;    // one channel a lane: there is room for fewer, and copies are fewer too
  float4 eu[kKeep][32];                         // of the lane's own channel e, e, e x, e x; or e, x, p, dy silu'(gate)
  float2 pp[kTwice ? kKeep : 1][32], xq[kTwice ? kKeep : 1][32];   // p, p; x, dy silu'(gate)
  float slope[kKeep][32];                       // sigmoid(dt + dt_bias)
  float4 start[kKeep / kSub - 1][L::CC * L::SP / 4][32];   // the lane's states before steps 4, 8, 12
  float sums[L::R][kKeep][2][L::SW];            // dB and dC over a row's channels
};

// The order of a lane's pairs of states.  Sums over channels go over the lanes with the same q; at each level a lane keeps
// half of its values and gives half away.  Lanes that keep the upper half of the pairs have them first: what a lane keeps
// and gives then sits in the same registers everywhere, and nothing is selected.
template <typename L>
__device__ __forceinline__ int pair_order(int lane) {
  int order = 0;
  int bit = L::RL / 2;
#pragma unroll
  for (int n = L::SP / 4; n >= 1 && bit >= L::LS; n /= 2, bit /= 2) order |= lane & bit ? n : 0;
  return order;
}
__device__ __forceinline__ F2 other(F2 v, int bit) {
  float lo, hi;
  split(v, lo, hi);
  return pair(__shfl_xor_sync(0xffffffffu, lo, bit), __shfl_xor_sync(0xffffffffu, hi, bit));
}
// The sums of v over the warp's channels, to [SW] (to: the lane's states of it).
template <typename L>
__device__ __forceinline__ void put_sums(F2 (&v)[L::SP / 2], int lane, int order, float* to) {
  constexpr int P = L::SP / 2, LS = L::LS;
  int n = P, bit = L::RL / 2;
#pragma unroll
  for (int k = 0; k < 5; ++k)
    if (n > 1 && bit >= LS) {
      n /= 2;
#pragma unroll
      for (int i = 0; i < P / 2; ++i)
        if (i < n) v[i] = v[i] + other(v[i + n], bit);
      bit /= 2;
    }
  if (n > 1 || bit < LS) {                      // lanes ran out: pairs are left
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (i < n) {
        float2 w;
        split(v[i], w.x, w.y);
        *reinterpret_cast<float2*>(to + 2 * (i ^ order)) = w;
      }
    return;
  }
  float lo, hi;
  split(v[0], lo, hi);
  const bool up = lane & bit;
  float r = (up ? hi : lo) + __shfl_xor_sync(0xffffffffu, up ? lo : hi, bit);
  const int odd = up;
  int same = 0;
  bit /= 2;
#pragma unroll
  for (int k = 0; k < 5; ++k)
    if (bit >= LS) {
      r += __shfl_xor_sync(0xffffffffu, r, bit);
      same |= bit;
      bit /= 2;
    }
  if (!(lane & same)) to[2 * order + odd] = r;
}

// SP states of CC channels in the lane's order.
template <int SP, int CC>
__device__ __forceinline__ void load_ordered(const float* p, const int64_t (&at)[CC], const bool (&there)[CC], int s0, int order,
                                             int S, F2 (&h)[CC][SP / 2]) {
  const bool vec = S % 2 == 0 && reinterpret_cast<uintptr_t>(p) % 8 == 0;
#pragma unroll
  for (int c = 0; c < CC; ++c)
#pragma unroll
    for (int i = 0; i < SP / 2; ++i) {
      const int s = s0 + 2 * (i ^ order);
      const float* const q = p + at[c] * S + s;
      float2 w = make_float2(0.0f, 0.0f);
      if (p && there[c] && s < S) {
        if (vec) w = *reinterpret_cast<const float2*>(q);
        else w = make_float2(q[0], s + 1 < S ? q[1] : 0.0f);
      }
      h[c][i] = pair(w.x, w.y);
    }
}
template <int SP, int CC>
__device__ __forceinline__ void store_ordered(float* p, const int64_t (&at)[CC], const bool (&there)[CC], int s0, int order, int S,
                                              const F2 (&h)[CC][SP / 2]) {
  const bool vec = S % 2 == 0 && reinterpret_cast<uintptr_t>(p) % 8 == 0;
#pragma unroll
  for (int c = 0; c < CC; ++c)
#pragma unroll
    for (int i = 0; i < SP / 2; ++i) {
      const int s = s0 + 2 * (i ^ order);
      float* const q = p + at[c] * S + s;
      float2 w;
      split(h[c][i], w.x, w.y);
      if (there[c] && s < S) {
        if (vec) {
          *reinterpret_cast<float2*>(q) = w;
        } else {
          q[0] = w.x;
          if (s + 1 < S) q[1] = w.y;
        }
      }
    }
}
template <int P>
__device__ __forceinline__ void load_pairs(const float* row, int order, F2 (&v)[P]) {   // row: at the lane's states
#pragma unroll
  for (int i = 0; i < P; ++i) v[i].v = *reinterpret_cast<const uint64_t*>(row + 2 * (i ^ order));
}
template <int CC, int P>
__device__ __forceinline__ void clear(F2 (&h)[CC][P]) {
#pragma unroll
  for (int c = 0; c < CC; ++c)
#pragma unroll
    for (int i = 0; i < P; ++i) h[c][i] = pair(0.0f, 0.0f);
}
__device__ __forceinline__ void prefetch(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// rows: (env, group) pairs a block walks side by side, back_warps / rows warps each.
template <typename T, typename L>
__global__ void __launch_bounds__(32 * back_warps(L::SW, L::R), back_blocks(L::SW, L::R)) k_select_back(Select a, int rows) {
  constexpr bool kTwice = Back<L>::kTwice;
  constexpr int SP = L::SP, LS = L::LS, CC = L::CC, SW = L::SW, P = SP / 2, R = L::R, RL = L::RL;
  extern __shared__ __align__(16) uint8_t smem[];
  Back<L>* const all = reinterpret_cast<Back<L>*>(smem);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  Back<L>& m = all[warp];
  const int side = back_warps(SW, R) / rows;                    // warps of a row
  const int row = warp / side, sub = lane / RL, mine = lane % RL;
  const int blocks = (a.tiles + side - 1) / side;             // blocks along a group's channels
  const int g = blockIdx.x / blocks, block = blockIdx.x % blocks;
  const int tile = block * side + warp % side;

  const int q = mine % LS, s0 = q * SP, order = pair_order<L>(lane);
  const int first = tile * L::CW + mine / LS * CC, own = first + q % CC;
  const bool channel = own < a.per;
  const int64_t d = (int64_t)g * a.per + own;
  int64_t at_weight[CC];
  bool there[CC];
#pragma unroll
  for (int c = 0; c < CC; ++c) {
    const int k = first + (q % CC ^ c);
    at_weight[c] = (int64_t)g * a.per + k;
    there[c] = k < a.per;
  }
  if (a.pieces > 1) after_previous();
  F2 A2[CC][P], dA[CC][P];
  load_ordered<SP, CC>(a.A, at_weight, there, s0, order, a.S, A2);
#pragma unroll
  for (int c = 0; c < CC; ++c)
#pragma unroll
    for (int i = 0; i < P; ++i) A2[c][i] = A2[c][i] * pair(kLog2e, kLog2e);
  clear(dA);
  const float bias = channel && a.dt_bias ? a.dt_bias[d] : 0.0f, skip = channel && a.skip ? a.skip[d] : 0.0f;
  float dskip = 0.0f, dbias = 0.0f;
  const bool gated = a.gate.data, gate_out = a.dgate.data;
  const int64_t states = a.N * a.D * a.S, envs = (a.N + R - 1) / R, items = envs * a.pieces;
  float* const slot = a.weights + ((blockIdx.y * (int64_t)rows + row) * R + sub) * a.D * (a.S + 2);
  auto put_weights = [&] {
    store_ordered<SP, CC>(slot, at_weight, there, s0, order, a.S, dA);
    if (channel && q < CC) {
      slot[a.D * a.S + d] = dskip;
      slot[a.D * (a.S + 1) + d] = dbias;
    }
  };
  // every warp of a block makes the same number of rounds: the block's barriers are in them
  for (int64_t item0 = blockIdx.y * (int64_t)rows; item0 < items; item0 += gridDim.y * (int64_t)rows) {
    const bool real = item0 + row < items;
    const int64_t item = real ? item0 + row : 0;
    const int64_t env = item % envs * R + sub;
    const bool env_there = R == 1 || env < a.N;
    const int64_t n = env_there ? env : 0;
    const bool live = channel && env_there, writes = live && q < CC;
    const int piece = (int)(item / envs);
    const int t0 = piece * a.piece, t1 = real ? min(a.T, t0 + a.piece) : t0;
    const int segments = (min(a.T, a.piece) + kKeep - 1) / kKeep;       // of the longest piece
    int64_t at[CC];
    bool held[CC];                                        // the lane's channels of this env
#pragma unroll
    for (int c = 0; c < CC; ++c) {
      at[c] = n * a.D + at_weight[c];
      held[c] = there[c] && env_there;
    }
    F2 G[CC][P];
    load_ordered<SP, CC>(a.pieces > 1 ? a.maps + piece * states : a.dhT, at, held, s0, order, a.S, G);

    for (int seg = segments - 1; seg >= 0; --seg) {
      const int ts = t0 + seg * kKeep, steps = min(kKeep, t1 - ts);
      if (steps > 0) {
        const bool flagged = a.done || a.done_prev;
        const uint8_t rend = flagged && mine < steps ? flag_at(a, ts + mine, n) : (uint8_t)0;
        const uint8_t rend8 = R > 1 && flagged && mine + 8 < steps ? flag_at(a, ts + mine + 8, n) : (uint8_t)0;
        F2 h[CC][P];
        load_ordered<SP, CC>(a.kept + ts / kKeep * states, at, held, s0, order, a.S, h);
        stage<T, SW, RL>(a, a.B, ts, steps, n, g, mine, m.B[sub][0]);
        stage<T, SW, RL>(a, a.C, ts, steps, n, g, mine, m.C[sub][0]);
        const T* px = row_at<T>(a.x, ts, n, d);
        const T* pdt = row_at<T>(a.dt, ts, n, d);
        const T* pdy = row_at<T>(a.dy, ts, n, d);
        const T* pgate = gated ? row_at<T>(a.gate, ts, n, d) : px;
#pragma unroll 1
        for (int k0 = 0; k0 < steps; k0 += 8) {
          T rx[8], rdt[8], rgate[8], rdy[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            from_float(0.0f, rx[k]);
            rdt[k] = rgate[k] = rdy[k] = rx[k];
            if (live && k0 + k < steps) {
              rx[k] = *px;
              rdt[k] = *pdt;
              rdy[k] = *pdy;
              if (gated) rgate[k] = *pgate;
            }
            px += a.x.outer, pdt += a.dt.outer, pdy += a.dy.outer;
            if (gated) pgate += a.gate.outer;
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            float slope, p = to_float(rdy[k]), qy = 0.0f;
            const float e = softplus(to_float(rdt[k]) + bias, &slope);
            if (gated) {
              const float z = to_float(rgate[k]);
              float s, o;
              gates(z, s, o);
              qy = p * (s * fmaf(z, o, 1.0f));
              p *= z * s;
            }
            const float x = to_float(rx[k]), u = e * x;
            if constexpr (kTwice) {
              m.eu[k0 + k][lane] = live ? make_float4(e, e, u, u) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
              m.pp[k0 + k][lane] = make_float2(p, p);
              m.xq[k0 + k][lane] = make_float2(x, qy);
            } else {
              m.eu[k0 + k][lane] = make_float4(live ? e : 0.0f, x, p, qy);
            }
            m.slope[k0 + k][lane] = slope;
          }
        }
        if (ts > t0 && live) {                          // the next segment's rows, on their way to L2
          const int t = ts - kKeep + lane % kKeep;
          if (lane < kKeep) {
            prefetch(row_at<T>(a.x, t, n, d));
            prefetch(row_at<T>(a.dy, t, n, d));
          } else {
            prefetch(row_at<T>(a.dt, t, n, d));
            if (gated) prefetch(row_at<T>(a.gate, t, n, d));
          }
          prefetch(a.kept + (ts / kKeep - 1) * states + at[0] * a.S);
        }
        // ends of the lane's env, and of any of the warp's
        uint32_t ends = __ballot_sync(0xffffffffu, rend != 0), any_ends = ends;
        if constexpr (R > 1) {
          static_assert(RL == 8, "two flags a lane");
          const uint32_t upper = __ballot_sync(0xffffffffu, rend8 != 0);
          any_ends = (ends | ends >> 16) | (upper | upper >> 16) << 16;
          any_ends = ((any_ends | any_ends >> 8) & 255u) | ((any_ends >> 16 | any_ends >> 24) & 255u) << 8;
          ends = (ends >> (sub * RL) & 255u) | (upper >> (sub * RL) & 255u) << 8;
        }
        __syncwarp();
        // e, e x and p of step k, for both states of a pair
        auto inputs = [&](int k, F2 (&e)[CC], F2 (&u)[CC]) {
          if constexpr (kTwice) {
#pragma unroll
            for (int c = 0; c < CC; ++c) {
              const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(&m.eu[k][lane ^ c]);
              e[c].v = w.x, u[c].v = w.y;
            }
          } else {
            const float4 w = m.eu[k][lane];
            e[0] = pair(w.x, w.x);
            u[0] = pair(w.x * w.y, w.x * w.y);
          }
        };
        auto weights = [&](int k, F2 (&p)[CC]) {
          if constexpr (kTwice) {
#pragma unroll
            for (int c = 0; c < CC; ++c) p[c].v = *reinterpret_cast<const uint64_t*>(&m.pp[k][lane ^ c]);
          } else {
            p[0] = pair(m.eu[k][lane].z, m.eu[k][lane].z);
          }
        };
        const int subs = (steps + kSub - 1) / kSub;
        // COUNT steps forward: the states behind them.  plain: no end is among them (and, below, all of them are there).
        auto ahead = [&](auto plain, auto count, int first_step) {
          constexpr bool kPlain = decltype(plain)::value;
#pragma unroll
          for (int k = 0; k < decltype(count)::value; ++k) {
            const int i0 = first_step + k;
            F2 e[CC], u[CC], B[P];
            inputs(i0, e, u);
            load_pairs(m.B[sub][i0] + s0, order, B);
            if (!kPlain && (ends >> i0 & 1u)) clear(h);
#pragma unroll
            for (int c = 0; c < CC; ++c)
#pragma unroll
              for (int i = 0; i < P; ++i) h[c][i] = fma2(decay_of(e[c], A2[c][i]), h[c][i], u[c] * B[i]);
          }
        };
        T* pdx = const_cast<T*>(row_at<T>(a.dx, ts + subs * kSub, n, d));
        T* pddt = const_cast<T*>(row_at<T>(a.ddt, ts + subs * kSub, n, d));
        T* pdgate = gate_out ? const_cast<T*>(row_at<T>(a.dgate, ts + subs * kSub, n, d)) : pdx;
        // kHeld steps forward from the states h, and back.
        auto through = [&](auto plain, int first_step) {
          constexpr bool kPlain = decltype(plain)::value;
          F2 decay[kHeld][CC][P], passed[kHeld][CC][P];
          float y[kHeld];
#pragma unroll
          for (int k = 0; k < kHeld; ++k) {
            const int i0 = first_step + k;
            y[k] = 0.0f;
            if (kPlain || i0 < steps) {
              float yc[CC];
              F2 e[CC], u[CC], p[CC], B[P], C[P], sC[P];
              inputs(i0, e, u);
              weights(i0, p);
              load_pairs(m.B[sub][i0] + s0, order, B);
              load_pairs(m.C[sub][i0] + s0, order, C);
              if (!kPlain && (ends >> i0 & 1u)) clear(h);
#pragma unroll
              for (int c = 0; c < CC; ++c) {
                F2 acc;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                  decay[k][c][i] = decay_of(e[c], A2[c][i]);
                  passed[k][c][i] = decay[k][c][i] * h[c][i];
                  h[c][i] = fma2(u[c], B[i], passed[k][c][i]);
                  acc = i ? fma2(C[i], h[c][i], acc) : C[i] * h[c][i];
                  sC[i] = c ? fma2(p[c], h[c][i], sC[i]) : p[c] * h[c][i];
                }
                yc[c] = total(acc);
              }
              y[k] = over_states<LS, CC>(yc);
              put_sums<L>(sC, lane, order, &m.sums[sub][i0][1][s0]);
            }
          }
#pragma unroll
          for (int k = kHeld - 1; k >= 0; --k) {
            const int i0 = first_step + k;
            pdx -= a.dx.outer, pddt -= a.ddt.outer;
            if (gate_out) pdgate -= a.dgate.outer;
            if (kPlain || i0 < steps) {
              float by_B[CC], by_A[CC];
              F2 e[CC], u[CC], p[CC], B[P], C[P], sB[P];
              inputs(i0, e, u);
              weights(i0, p);
              load_pairs(m.B[sub][i0] + s0, order, B);
              load_pairs(m.C[sub][i0] + s0, order, C);
#pragma unroll
              for (int c = 0; c < CC; ++c) {
                F2 accB, accA;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                  const F2 f = fma2(p[c], C[i], G[c][i]), w = f * passed[k][c][i];
                  accB = i ? fma2(f, B[i], accB) : f * B[i];
                  accA = i ? fma2(w, A2[c][i], accA) : w * A2[c][i];
                  sB[i] = c ? fma2(u[c], f, sB[i]) : u[c] * f;
                  dA[c][i] = fma2(w, e[c], dA[c][i]);
                  G[c][i] = decay[k][c][i] * f;
                }
                by_B[c] = total(accB);
                by_A[c] = total(accA);
              }
              if (!kPlain && (ends >> i0 & 1u)) clear(G);
              const float sumB = over_states<LS, CC>(by_B), sumA = over_states<LS, CC>(by_A) * kLn2;
              put_sums<L>(sB, lane, order, &m.sums[sub][i0][0][s0]);
              float e1, p1, copy;
              split(e[0], e1, copy);
              split(p[0], p1, copy);
              float2 w;
              if constexpr (kTwice) w = m.xq[i0][lane];
              else w = make_float2(m.eu[i0][lane].y, m.eu[i0][lane].w);
              const float du = fmaf(w.x, sumB, sumA) * m.slope[i0][lane];
              store_if(writes, pdx, fmaf(e1, sumB, skip * p1));
              store_if(writes, pddt, du);
              if (gate_out) store_if(writes, pdgate, w.y * fmaf(skip, w.x, y[k]));
              dskip = fmaf(p1, w.x, dskip);
              dbias += du;
            }
          }
        };
        const auto plain = std::true_type();
        const auto any = std::false_type();
        const auto two = std::integral_constant<int, kHeld>();
        const auto four = std::integral_constant<int, kSub>();
#pragma unroll 1
        for (int block4 = 0; block4 + 1 < subs; ++block4) {        // the states before every 4th step but the first
          if (any_ends >> (block4 * kSub) & 15u) ahead(any, four, block4 * kSub);
          else ahead(plain, four, block4 * kSub);
#pragma unroll
          for (int c = 0; c < CC; ++c)
#pragma unroll
            for (int i = 0; i < P; i += 2) {
              float4 w;
              split(h[c][i], w.x, w.y);
              split(h[c][i + 1], w.z, w.w);
              m.start[block4][(c * SP + 2 * i) / 4][lane] = w;
            }
        }
#pragma unroll 1
        for (int half = subs * 2 - 1; half >= 0; --half) {
          const int block4 = half / 2, at0 = half * kHeld;
          if (block4) {
#pragma unroll
            for (int c = 0; c < CC; ++c)
#pragma unroll
              for (int i = 0; i < P; i += 2) {
                const float4 w = m.start[block4 - 1][(c * SP + 2 * i) / 4][lane];
                h[c][i] = pair(w.x, w.y);
                h[c][i + 1] = pair(w.z, w.w);
              }
          } else {
            load_ordered<SP, CC>(a.kept + ts / kKeep * states, at, held, s0, order, a.S, h);
          }
          if ((any_ends >> (block4 * kSub) & 15u) || at0 + kHeld > steps) {
            if (half & 1) ahead(any, two, at0 - kHeld);
            through(any, at0);
          } else {
            if (half & 1) ahead(plain, two, at0 - kHeld);
            through(plain, at0);
          }
        }
      }
      __syncthreads();
      // dB and dC of the segment over the row's warps, in their order
      if (R > 1 && steps > 0 && env_there) {
        for (int i = mine; i < steps * 2 * a.S; i += RL) {
          const int k = i / (2 * a.S), j = i % (2 * a.S), which = j >= a.S, s = which ? j - a.S : j;
          from_float(m.sums[sub][k][which][s], *const_cast<T*>(row_at<T>(which ? a.dC : a.dB, ts + k, n, (int64_t)g * a.S + s)));
        }
      } else if (R == 1 && steps > 0) {
        const int threads = 32 * side, me = threadIdx.x % threads;
        const Back<L>* const from = all + row * side;
        const int live_warps = min(side, a.tiles - block * side);
        for (int i = me; i < steps * 2 * a.S; i += threads) {
          const int k = i / (2 * a.S), j = i % (2 * a.S), which = j >= a.S, s = which ? j - a.S : j, t = ts + k;
          float v = 0.0f;
          for (int w = 0; w < live_warps; ++w) v += from[w].sums[0][k][which][s];
          if (blocks > 1) a.parts[((((int64_t)block * a.T + t) * a.N + n) * a.G + g) * 2 * a.S + j] = v;
          else from_float(v, *const_cast<T*>(row_at<T>(which ? a.dC : a.dB, t, n, (int64_t)g * a.S + s)));
        }
      }
      __syncthreads();
    }
    if (a.dh0 && piece == 0 && real) store_ordered<SP, CC>(a.dh0, at, held, s0, order, a.S, G);
    // weight gradients are summed over an item in registers, over a slot's items in memory: one chain through all of them
    // rounded away three times as much (4,096 x 128: 1.4e-6 of dA)
    if (real) {
      if (item0 != blockIdx.y * (int64_t)rows) {
        F2 before[CC][P];
        load_ordered<SP, CC>(slot, at_weight, there, s0, order, a.S, before);
#pragma unroll
        for (int c = 0; c < CC; ++c)
#pragma unroll
          for (int i = 0; i < P; ++i) dA[c][i] = dA[c][i] + before[c][i];
        if (channel && q < CC) {
          dskip += slot[a.D * a.S + d];
          dbias += slot[a.D * (a.S + 1) + d];
        }
      }
      put_weights();
      clear(dA);
      dskip = dbias = 0.0f;
    }
  }
  if (blockIdx.y * (int64_t)rows + row >= items) put_weights();         // a slot without an item
}

// The pieces' gradients from 0 behind them, and their sums of step sizes, as forward.
constexpr int kFoldWarps = 4, kFoldBatch = 4;
template <typename T, typename L>
__global__ void __launch_bounds__(32 * kFoldWarps) k_select_fold_back(Select a) {
  constexpr int SP = L::SP, LS = L::LS, CC = L::CC, SW = L::SW, R = L::R, RL = L::RL;
  using In = Staged<T, SW, kFoldBatch, RL>;
  __shared__ __align__(16) float rows[kFoldWarps][R][kFoldBatch * SW];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int64_t id = blockIdx.x * (int64_t)kFoldWarps + warp;
  const int64_t envs_groups = (a.N * a.G + R - 1) / R;         // rows, or fours of them
  if (id >= envs_groups * a.tiles * a.pieces) return;
  const int tile = (int)(id % a.tiles), sub = lane / RL, mine = lane % RL;
  id /= a.tiles;
  const int64_t row = id % envs_groups * R + sub;
  const bool row_there = R == 1 || row < a.N * a.G;
  const int g = row_there ? (int)(row % a.G) : 0;
  const int64_t n = row_there ? row / a.G : 0;
  const int piece = (int)(id / envs_groups);
  float* const Cs = rows[warp][sub];
  const int q = mine % LS, s0 = q * SP;
  const int first = tile * L::CW + mine / LS * CC, own = first + q % CC;
  const bool live = row_there && own < a.per;
  const int64_t d = (int64_t)g * a.per + own;
  int64_t at[CC], at_weight[CC];
  bool there[CC];
#pragma unroll
  for (int c = 0; c < CC; ++c) {
    const int k = first + (q % CC ^ c);
    at_weight[c] = (int64_t)g * a.per + k;
    at[c] = n * a.D + at_weight[c];
    there[c] = row_there && k < a.per;
  }
  const int t0 = piece * a.piece, t1 = min(a.T, t0 + a.piece);
  F2 G[CC][SP / 2], A2[CC][SP / 2];
  load_states<SP, CC>(a.A, at_weight, there, s0, a.S, A2);
#pragma unroll
  for (int c = 0; c < CC; ++c)
#pragma unroll
    for (int i = 0; i < SP / 2; ++i) {
      G[c][i] = pair(0.0f, 0.0f);
      A2[c][i] = A2[c][i] * pair(kLog2e, kLog2e);
    }
  const float bias = live && a.dt_bias ? a.dt_bias[d] : 0.0f;
  const bool gated = a.gate.data, flagged = a.done || a.done_prev;
  float sum = 0.0f;
  bool cut = false;
  // the last batch first, its inputs on their way while the one behind it is gone through
  const int last = t0 + (t1 - 1 - t0) / kFoldBatch * kFoldBatch;
  const T* pdt = row_at<T>(a.dt, last, n, d);
  const T* pdy = row_at<T>(a.dy, last, n, d);
  const T* pgate = gated ? row_at<T>(a.gate, last, n, d) : pdy;
  const T* pC = row_at<T>(a.C, last + mine / In::kSide, n, (int64_t)g * a.S + mine % In::kSide);
  T rdt[kFoldBatch], rgate[kFoldBatch], rdy[kFoldBatch];
  In rC;
  uint8_t rend = 0;
  auto fetch = [&](int t) {
    if (t < t0) return;
    const int steps = min(kFoldBatch, t1 - t);
    rend = flagged && mine < steps ? flag_at(a, t + mine, n) : (uint8_t)0;
    rC.load(pC, a.C.outer, steps, a.S, mine);
#pragma unroll
    for (int k = 0; k < kFoldBatch; ++k) {
      from_float(0.0f, rdt[k]);
      rgate[k] = rdy[k] = rdt[k];
      if (live && k < steps) {
        rdt[k] = pdt[k * a.dt.outer], rdy[k] = pdy[k * a.dy.outer];
        if (gated) rgate[k] = pgate[k * a.gate.outer];
      }
    }
    pdt -= kFoldBatch * a.dt.outer, pdy -= kFoldBatch * a.dy.outer, pC -= kFoldBatch * a.C.outer;
    if (gated) pgate -= kFoldBatch * a.gate.outer;
  };
  fetch(last);
#pragma unroll 1
  for (int ts = last; ts >= t0; ts -= kFoldBatch) {
    const int steps = t1 - ts;
    __syncwarp();                                             // the last batch's rows are read
    rC.put(Cs, mine);
    const uint32_t ends = flagged ? __ballot_sync(0xffffffffu, rend != 0) >> (sub * RL % 32) & 15u : 0u;
    float e[kFoldBatch], p[kFoldBatch];
#pragma unroll
    for (int k = 0; k < kFoldBatch; ++k) {
      e[k] = softplus(to_float(rdt[k]) + bias);
      p[k] = to_float(rdy[k]);
      if (gated) {
        const float z = to_float(rgate[k]);
        float s, o;
        gates(z, s, o);
        p[k] *= z * s;
      }
    }
    fetch(ts - kFoldBatch);
    __syncwarp();
    cut = cut || ends;
#pragma unroll
    for (int k = kFoldBatch - 1; k >= 0; --k) {
      if (k < steps) {
        float es[CC], ps[CC];
        to_lanes<CC>(e[k], es);
        to_lanes<CC>(p[k], ps);
        F2 C[SP / 2];
        load_pairs<SP>(Cs + k * SW + s0, C);
        sum += e[k];
#pragma unroll
        for (int c = 0; c < CC; ++c) {
          const F2 e2 = pair(es[c], es[c]), p2 = pair(ps[c], ps[c]);
#pragma unroll
          for (int i = 0; i < SP / 2; ++i) G[c][i] = decay_of(e2, A2[c][i]) * fma2(p2, C[i], G[c][i]);
        }
        if (ends >> k & 1u) clear(G);
      }
    }
  }
  store_states<SP, CC>(a.maps + piece * (a.N * a.D * a.S), at, there, s0, a.S, G);
  if (live && q < CC) a.sums[(int64_t)piece * a.N * a.D + n * a.D + d] = cut ? -1.0f : sum;
}

// dA, dskip and ddt_bias: the slots' sums added in order, 32 values a block.
constexpr int kGroups = 8;
__global__ void __launch_bounds__(32 * kGroups) k_select_weights(Select a, int64_t slots) {
  __shared__ float part[kGroups][32];
  after_previous();
  const int lane = threadIdx.x % 32, group = threadIdx.x / 32;
  const int64_t cols = a.D * (a.S + 2), c = blockIdx.x * (int64_t)32 + lane;
  float v = 0.0f;
  if (c < cols)
    for (int64_t r = group; r < slots; r += kGroups) v += a.weights[r * cols + c];
  part[group][lane] = v;
  __syncthreads();
  if (group || c >= cols) return;
  for (int k = 1; k < kGroups; ++k) v += part[k][lane];
  if (c < a.D * a.S) {
    if (a.dA) a.dA[c] = v;
  } else if (c < a.D * (a.S + 1)) {
    if (a.dskip) a.dskip[c - a.D * a.S] = v;
  } else if (a.ddt_bias) {
    a.ddt_bias[c - a.D * (a.S + 1)] = v;
  }
}

// dB and dC of groups of several blocks.
template <typename T>
__global__ void __launch_bounds__(256) k_select_rows(Select a, int64_t blocks) {
  after_previous();
  const int64_t each = (int64_t)a.T * a.N * a.G * 2 * a.S, step = gridDim.x * (int64_t)256;
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < each; i += step) {
    float v = 0.0f;
    for (int64_t b = 0; b < blocks; ++b) v += a.parts[b * each + i];
    const int64_t r = i / (2 * a.S);
    const int j = (int)(i % (2 * a.S)), g = (int)(r % a.G);
    const int64_t n = r / a.G % a.N, t = r / a.G / a.N;
    const bool which = j >= a.S;
    from_float(v, *const_cast<T*>(row_at<T>(which ? a.dC : a.dB, t, n, (int64_t)g * a.S + (which ? j - a.S : j))));
  }
}

}  // namespace

// How many partial sums of the weight gradients there are; *blocks: along a group's channels; *rows: of a block.
int64_t select_slots(const Select& a, int64_t* blocks, int* rows) {
  const int warps = back_warps(a.S, a.rows);
  int side = 1;
  while (a.rows == 1 && side < a.tiles && side < warps) side *= 2;
  *rows = warps / side;
  *blocks = (a.tiles + side - 1) / side;
  const int64_t items = ((a.N + a.rows - 1) / a.rows * a.pieces + *rows - 1) / *rows;
  const int64_t most = std::max<int64_t>(1, (int64_t)sm_count() * back_blocks(a.S, a.rows) / (*blocks * a.G));
  // as many rounds as the fullest slot makes, spread evenly
  const int64_t rounds = (items + most - 1) / most;
  return std::min<int64_t>((items + rounds - 1) / rounds, 65535) * *rows * a.rows;
}

template <typename T>
cudaError_t launch_select_back(const Select& a, bool split, cudaStream_t s) {
  int64_t blocks;
  int rows;
  const int64_t slots = select_slots(a, &blocks, &rows);
  auto all = [&](auto l) -> cudaError_t {
    using L = decltype(l);
    cudaError_t e;
    if (split) {
      const int64_t warps = (a.N * a.G + L::R - 1) / L::R * a.tiles * a.pieces;
      k_select_fold_back<T, L><<<(unsigned)((warps + kFoldWarps - 1) / kFoldWarps), 32 * kFoldWarps, 0, s>>>(a);
      if ((e = cudaGetLastError()) != cudaSuccess || (e = launch_select_join(a, true, s)) != cudaSuccess) return e;
    }
    const auto kern = k_select_back<T, L>;
    constexpr int kWarps = back_warps(L::SW, L::R);
    const int smem = (int)sizeof(Back<L>) * kWarps;
    static_assert((sizeof(Back<L>) * kWarps + 1024) * back_blocks(L::SW, L::R) <= 228 * 1024, "shared memory of an SM");
    if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return e;
    const dim3 grid((unsigned)(blocks * a.G), (unsigned)(slots / (rows * L::R)));
    if (split) return launch_after(kern, grid, 32 * kWarps, smem, s, a, rows);
    kern<<<grid, 32 * kWarps, smem, s>>>(a, rows);
    return cudaGetLastError();
  };
  cudaError_t e = a.rows > 1 ? with_narrow_lanes(a.S, all) : with_lanes(a.S, all);
  if (e != cudaSuccess) return e;
  if (a.dA || a.dskip || a.ddt_bias) {
    e = launch_after(k_select_weights, dim3((unsigned)((a.D * (a.S + 2) + 31) / 32)), 32 * kGroups, 0, s, a, slots);
    if (e != cudaSuccess) return e;
  }
  if (blocks > 1) {
    // not ahead of the kernel before last's end: an ordinary launch
    const int64_t each = (int64_t)a.T * a.N * a.G * 2 * a.S;
    k_select_rows<T><<<(unsigned)std::min<int64_t>((each + 255) / 256, (int64_t)sm_count() * 16), 256, 0, s>>>(a, blocks);
    e = cudaGetLastError();
  }
  return e;
}

template cudaError_t launch_select_back<float>(const Select&, bool, cudaStream_t);
template cudaError_t launch_select_back<__nv_bfloat16>(const Select&, bool, cudaStream_t);
template cudaError_t launch_select_back<__half>(const Select&, bool, cudaStream_t);

}  // namespace net
}  // namespace auv
