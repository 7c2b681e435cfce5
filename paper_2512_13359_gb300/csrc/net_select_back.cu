// net_select_back.cu -- gradients of the selective scan (auvnet.h, net_select_scan_backward).
//
// The chain of gradients runs from the last step to the first, and every step needs its states.  A segment of 16 steps
// starts again from its kept state: a first pass keeps the states before every 4th step (shared memory), then, last four
// steps first, a second pass holds a = exp(e A) and a c of four steps in registers and sums y and dC on its way, and the
// gradients run back through the four.  Per state and step some 13 fp32 operations and 1.75 exponentials.  Sums over a
// channel's states (y and the two that dx and ddt are made of) go over 1 to 16 lanes; dB and dC are sums over the channels
// of a group, over the lanes with one shuffle a value (each lane keeps half of its values at every level) and over the
// block's warps in shared memory at the end of a segment; groups wider than a block leave partial sums, which k_select_rows
// adds.  Weight gradients stay in registers over all envs and pieces of a warp.  Every sum has a fixed order.
#include <algorithm>

#include "net_select.cuh"

namespace auv {
namespace net {
namespace {

constexpr int kSub = 4;         // steps held in registers

// Warps of a block: shared memory grows with the padded states.
template <typename L> constexpr int kBackWarps = L::SW <= 32 ? 8 : L::SW <= 64 ? 4 : 2;

// A warp's shared memory.
template <typename L> struct Back {
  float B[kKeep][L::SW], C[kKeep][L::SW];
  float4 own[kKeep][32];                        // e, x, p, dy silu'(gate) of the lane's own channel
  float slope[kKeep][32];                       // sigmoid(dt + dt_bias)
  float4 start[kKeep / kSub][L::CC * L::SP / 4][32];   // the lane's states before steps 0, 4, 8, 12
  float sums[kKeep][2][L::SW];                  // dB and dC over the warp's channels
};

// Sums over the lanes with the same q of SP values: at each level a lane gives half of its values away.  Returns how many
// are left, the sums of values base, base + 1, ...; lanes whose bits in `same` are not 0 hold what another one holds too.
template <int SP, int LS>
__device__ __forceinline__ void over_channels(float (&v)[SP], int lane, int& base, int& same) {
  base = same = 0;
  int n = SP;
#pragma unroll
  for (int bit = 16; bit >= LS; bit /= 2) {
    if (n > 1) {
      n /= 2;
      const bool up = lane & bit;
#pragma unroll
      for (int i = 0; i < SP / 2; ++i)
        if (i < n) {
          const float give = up ? v[i] : v[i + n];
          v[i] = (up ? v[i + n] : v[i]) + __shfl_xor_sync(0xffffffffu, give, bit);
        }
      base += up ? n : 0;
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], bit);
      same |= bit;
    }
  }
}
template <int SP, int LS> constexpr int left_over() {
  int n = SP;
  for (int bit = 16; bit >= LS; bit /= 2) n = n > 1 ? n / 2 : 1;
  return n;
}
template <int SP, int LS>
__device__ __forceinline__ void put_sums(float (&v)[SP], int lane, float* to) {
  int base, same;
  over_channels<SP, LS>(v, lane, base, same);
  if (!(lane & same)) {
#pragma unroll
    for (int i = 0; i < left_over<SP, LS>(); ++i) to[base + i] = v[i];
  }
}

// rows: (env, group) pairs a block walks side by side, kBackWarps / rows warps each.
template <typename T, typename L>
__global__ void __launch_bounds__(32 * kBackWarps<L>, 1) k_select_back(Select a, int rows) {
  constexpr int SP = L::SP, LS = L::LS, CC = L::CC, SW = L::SW, kP = SP / 2;
  extern __shared__ __align__(16) uint8_t smem[];
  Back<L>* const all = reinterpret_cast<Back<L>*>(smem);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  Back<L>& m = all[warp];
  const int side = kBackWarps<L> / rows;                     // warps of a row
  const int row = warp / side;
  const int blocks = (a.tiles + side - 1) / side;             // blocks along a group's channels
  const int g = blockIdx.x / blocks, block = blockIdx.x % blocks;
  const int tile = block * side + warp % side;

  const int q = lane % LS, s0 = q * SP;
  const int first = tile * L::CW + lane / LS * CC, own = first + q % CC;
  const bool live = own < a.per, writes = live && q < CC;
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
  F2 A2[CC][kP], dA[CC][kP];
  load_states<SP, CC>(a.A, at_weight, there, s0, a.S, A2);
#pragma unroll
  for (int c = 0; c < CC; ++c)
#pragma unroll
    for (int i = 0; i < kP; ++i) {
      A2[c][i] = A2[c][i] * pair(kLog2e, kLog2e);
      dA[c][i] = pair(0.0f, 0.0f);
    }
  const float bias = live && a.dt_bias ? a.dt_bias[d] : 0.0f, skip = live && a.skip ? a.skip[d] : 0.0f;
  float dskip = 0.0f, dbias = 0.0f;
  const int64_t states = a.N * a.D * a.S, items = a.N * a.pieces;
  // every warp of a block makes the same number of rounds: the block's barriers are in them
  for (int64_t item0 = blockIdx.y * (int64_t)rows; item0 < items; item0 += gridDim.y * (int64_t)rows) {
    const int64_t item = min(item0 + row, items - 1);
    const bool real = item0 + row < items;
    const int64_t n = item % a.N;
    const int piece = (int)(item / a.N);
    const int t0 = piece * a.piece, t1 = min(a.T, t0 + a.piece);
    const int segments = (min(a.T, a.piece) + kKeep - 1) / kKeep;       // of the longest piece
    int64_t at[CC];
    bool put[CC];
#pragma unroll
    for (int c = 0; c < CC; ++c) {
      at[c] = n * a.D + at_weight[c];
      put[c] = there[c] && real;
    }
    F2 G[CC][kP];
    load_states<SP, CC>(a.pieces > 1 ? a.maps + piece * states : a.dhT, at, there, s0, a.S, G);

    for (int seg = segments - 1; seg >= 0; --seg) {
      const int ts = t0 + seg * kKeep, steps = min(kKeep, t1 - ts);
      if (steps > 0) {
        const uint32_t ends = ends_of(a, ts, n, lane);
        stage<T, SW>(a, a.B, ts, steps, n, g, lane, m.B[0]);
        stage<T, SW>(a, a.C, ts, steps, n, g, lane, m.C[0]);
        F2 h[CC][kP];
        load_states<SP, CC>(a.kept + ts / kKeep * states, at, there, s0, a.S, h);
#pragma unroll 1
        for (int k0 = 0; k0 < steps; k0 += 8) {
          T rx[8], rdt[8], rgate[8], rdy[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            from_float(0.0f, rx[k]);
            rdt[k] = rgate[k] = rdy[k] = rx[k];
            if (live && k0 + k < steps) {
              const int t = ts + k0 + k;
              rx[k] = *row_at<T>(a.x, t, n, d);
              rdt[k] = *row_at<T>(a.dt, t, n, d);
              rdy[k] = *row_at<T>(a.dy, t, n, d);
              if (a.gate.data) rgate[k] = *row_at<T>(a.gate, t, n, d);
            }
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            float slope, p = to_float(rdy[k]), qy = 0.0f;
            const float e = softplus(to_float(rdt[k]) + bias, &slope);
            if (a.gate.data) {
              const float z = to_float(rgate[k]);
              float s, o;
              gates(z, s, o);
              qy = p * (s * fmaf(z, o, 1.0f));
              p *= z * s;
            }
            m.own[k0 + k][lane] = make_float4(live ? e : 0.0f, to_float(rx[k]), p, qy);
            m.slope[k0 + k][lane] = slope;
          }
        }
        __syncwarp();
        auto channels = [&](int k, float (&e)[CC], float (&u)[CC], float (&p)[CC]) {
#pragma unroll
          for (int c = 0; c < CC; ++c) {
            const float4 w = m.own[k][lane ^ c];
            e[c] = w.x, u[c] = w.x * w.y, p[c] = w.z;
          }
        };
        const int subs = (steps + kSub - 1) / kSub;
#pragma unroll 1
        for (int sub = 0; sub < subs; ++sub) {            // the states before every 4th step
#pragma unroll
          for (int c = 0; c < CC; ++c)
#pragma unroll
            for (int i = 0; i < kP; i += 2) {
              float4 w;
              split(h[c][i], w.x, w.y);
              split(h[c][i + 1], w.z, w.w);
              m.start[sub][(c * SP + 2 * i) / 4][lane] = w;
            }
          if (sub + 1 < subs) {
#pragma unroll
            for (int k = 0; k < kSub; ++k) {
              const int i0 = sub * kSub + k;
              float e[CC], u[CC], p[CC];
              channels(i0, e, u, p);
              F2 B[kP];
              load_pairs<SP>(m.B[i0] + s0, B);
              const bool end = ends >> i0 & 1u;
#pragma unroll
              for (int c = 0; c < CC; ++c) {
                const F2 e2 = pair(e[c], e[c]), u2 = pair(u[c], u[c]);
#pragma unroll
                for (int i = 0; i < kP; ++i)
                  h[c][i] = fma2(ex2(e2 * A2[c][i]), end ? pair(0.0f, 0.0f) : h[c][i], u2 * B[i]);
              }
            }
          }
        }
#pragma unroll 1
        for (int sub = subs - 1; sub >= 0; --sub) {
          F2 decay[kSub][CC][kP], passed[kSub][CC][kP];
          float y[kSub];
#pragma unroll
          for (int c = 0; c < CC; ++c)
#pragma unroll
            for (int i = 0; i < kP; i += 2) {
              const float4 w = m.start[sub][(c * SP + 2 * i) / 4][lane];
              h[c][i] = pair(w.x, w.y);
              h[c][i + 1] = pair(w.z, w.w);
            }
#pragma unroll
          for (int k = 0; k < kSub; ++k) {
            const int i0 = sub * kSub + k;
            y[k] = 0.0f;
            if (i0 < steps) {
              float e[CC], u[CC], p[CC], yc[CC], dC[SP];
              channels(i0, e, u, p);
              F2 B[kP], C[kP], sC[kP];
              load_pairs<SP>(m.B[i0] + s0, B);
              load_pairs<SP>(m.C[i0] + s0, C);
              const bool end = ends >> i0 & 1u;
#pragma unroll
              for (int c = 0; c < CC; ++c) {
                const F2 e2 = pair(e[c], e[c]), u2 = pair(u[c], u[c]), p2 = pair(p[c], p[c]);
                F2 acc = pair(0.0f, 0.0f);
#pragma unroll
                for (int i = 0; i < kP; ++i) {
                  decay[k][c][i] = ex2(e2 * A2[c][i]);
                  passed[k][c][i] = end ? pair(0.0f, 0.0f) : decay[k][c][i] * h[c][i];
                  h[c][i] = fma2(u2, B[i], passed[k][c][i]);
                  acc = fma2(C[i], h[c][i], acc);
                  sC[i] = c ? fma2(p2, h[c][i], sC[i]) : p2 * h[c][i];
                }
                yc[c] = total(acc);
              }
              y[k] = over_states<LS, CC>(yc);
#pragma unroll
              for (int i = 0; i < kP; ++i) split(sC[i], dC[2 * i], dC[2 * i + 1]);
              put_sums<SP, LS>(dC, lane, &m.sums[i0][1][s0]);
            }
          }
#pragma unroll
          for (int k = kSub - 1; k >= 0; --k) {
            const int i0 = sub * kSub + k;
            if (i0 < steps) {
              float e[CC], u[CC], p[CC], by_B[CC], by_A[CC], dB[SP];
              channels(i0, e, u, p);
              F2 B[kP], C[kP], sB[kP];
              load_pairs<SP>(m.B[i0] + s0, B);
              load_pairs<SP>(m.C[i0] + s0, C);
              const bool end = ends >> i0 & 1u;
#pragma unroll
              for (int c = 0; c < CC; ++c) {
                const F2 e2 = pair(e[c], e[c]), u2 = pair(u[c], u[c]), p2 = pair(p[c], p[c]);
                F2 accB = pair(0.0f, 0.0f), accA = accB;
#pragma unroll
                for (int i = 0; i < kP; ++i) {
                  const F2 f = fma2(p2, C[i], G[c][i]), w = f * passed[k][c][i];
                  accB = fma2(f, B[i], accB);
                  accA = fma2(w, A2[c][i], accA);
                  sB[i] = c ? fma2(u2, f, sB[i]) : u2 * f;
                  dA[c][i] = fma2(w, real ? e2 : pair(0.0f, 0.0f), dA[c][i]);
                  G[c][i] = end ? pair(0.0f, 0.0f) : decay[k][c][i] * f;
                }
                by_B[c] = total(accB);
                by_A[c] = total(accA);
              }
              const float sumB = over_states<LS, CC>(by_B), sumA = over_states<LS, CC>(by_A) * kLn2;
#pragma unroll
              for (int i = 0; i < kP; ++i) split(sB[i], dB[2 * i], dB[2 * i + 1]);
              put_sums<SP, LS>(dB, lane, &m.sums[i0][0][s0]);
              const float4 w = m.own[i0][lane];
              const float du = fmaf(w.y, sumB, sumA) * m.slope[i0][lane];
              if (writes && real) {
                const int t = ts + i0;
                from_float(fmaf(w.x, sumB, skip * w.z), *const_cast<T*>(row_at<T>(a.dx, t, n, d)));
                from_float(du, *const_cast<T*>(row_at<T>(a.ddt, t, n, d)));
                if (a.dgate.data) from_float(w.w * fmaf(skip, w.y, y[k]), *const_cast<T*>(row_at<T>(a.dgate, t, n, d)));
                dskip = fmaf(w.z, w.y, dskip);
                dbias += du;
              }
            }
          }
        }
      }
      __syncthreads();
      // dB and dC of the segment over the row's warps, in their order
      if (steps > 0 && real) {
        const int threads = 32 * side, me = threadIdx.x % threads;
        const Back<L>* const from = all + row * side;
        const int live_warps = min(side, a.tiles - block * side);
        for (int i = me; i < steps * 2 * a.S; i += threads) {
          const int k = i / (2 * a.S), j = i % (2 * a.S), which = j >= a.S, s = which ? j - a.S : j, t = ts + k;
          float v = 0.0f;
          for (int w = 0; w < live_warps; ++w) v += from[w].sums[k][which][s];
          if (blocks > 1) a.parts[((((int64_t)block * a.T + t) * a.N + n) * a.G + g) * 2 * a.S + j] = v;
          else from_float(v, *const_cast<T*>(row_at<T>(which ? a.dC : a.dB, t, n, (int64_t)g * a.S + s)));
        }
      }
      __syncthreads();
    }
    if (a.dh0 && piece == 0) store_states<SP, CC>(a.dh0, at, put, s0, a.S, G);
  }
  if (a.weights) {
    float* const to = a.weights + (blockIdx.y * (int64_t)rows + row) * a.D * (a.S + 2);
    store_states<SP, CC>(to, at_weight, there, s0, a.S, dA);
    if (writes) {
      to[a.D * a.S + d] = dskip;
      to[a.D * (a.S + 1) + d] = dbias;
    }
  }
}

// The pieces' gradients from 0 behind them, and their sums of step sizes, as forward.
constexpr int kFoldWarps = 4;
template <typename T, typename L>
__global__ void __launch_bounds__(32 * kFoldWarps) k_select_fold_back(Select a) {
  constexpr int SP = L::SP, LS = L::LS, CC = L::CC, SW = L::SW;
  __shared__ __align__(16) float rows[kFoldWarps][kKeep * SW];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int64_t id = blockIdx.x * (int64_t)kFoldWarps + warp;
  if (id >= a.N * a.G * a.tiles * a.pieces) return;
  const int tile = (int)(id % a.tiles);
  id /= a.tiles;
  const int g = (int)(id % a.G);
  id /= a.G;
  const int64_t n = id % a.N;
  const int piece = (int)(id / a.N);
  float* const Cs = rows[warp];
  const int q = lane % LS, s0 = q * SP;
  const int first = tile * L::CW + lane / LS * CC, own = first + q % CC;
  const bool live = own < a.per;
  const int64_t d = (int64_t)g * a.per + own;
  int64_t at[CC], at_weight[CC];
  bool there[CC];
#pragma unroll
  for (int c = 0; c < CC; ++c) {
    const int k = first + (q % CC ^ c);
    at_weight[c] = (int64_t)g * a.per + k;
    at[c] = n * a.D + at_weight[c];
    there[c] = k < a.per;
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
  float sum = 0.0f;
  bool cut = false;
  for (int ts = t0 + (t1 - 1 - t0) / kKeep * kKeep; ts >= t0; ts -= kKeep) {
    const int steps = min(kKeep, t1 - ts);
    const uint32_t ends = ends_of(a, ts, n, lane);
    stage<T, SW>(a, a.C, ts, steps, n, g, lane, Cs);
    __syncwarp();
#pragma unroll 1
    for (int k0 = steps > 8 ? 8 : 0; k0 >= 0; k0 -= 8) {
      T rdt[8], rgate[8], rdy[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        from_float(0.0f, rdt[k]);
        rgate[k] = rdy[k] = rdt[k];
        if (live && k0 + k < steps) {
          const int t = ts + k0 + k;
          rdt[k] = *row_at<T>(a.dt, t, n, d);
          rdy[k] = *row_at<T>(a.dy, t, n, d);
          if (a.gate.data) rgate[k] = *row_at<T>(a.gate, t, n, d);
        }
      }
#pragma unroll
      for (int k = 7; k >= 0; --k) {
        if (k0 + k < steps) {
          float p = to_float(rdy[k]);
          const float e = live ? softplus(to_float(rdt[k]) + bias) : 0.0f;
          if (a.gate.data) {
            const float z = to_float(rgate[k]);
            float s, o;
            gates(z, s, o);
            p *= z * s;
          }
          float es[CC], ps[CC];
          to_lanes<CC>(e, es);
          to_lanes<CC>(p, ps);
          F2 C[SP / 2];
          load_pairs<SP>(Cs + (k0 + k) * SW + s0, C);
          const bool end = ends >> (k0 + k) & 1u;
          cut = cut || end;
          sum += e;
#pragma unroll
          for (int c = 0; c < CC; ++c) {
            const F2 e2 = pair(es[c], es[c]), p2 = pair(ps[c], ps[c]);
#pragma unroll
            for (int i = 0; i < SP / 2; ++i)
              G[c][i] = end ? pair(0.0f, 0.0f) : ex2(e2 * A2[c][i]) * fma2(p2, C[i], G[c][i]);
          }
        }
      }
    }
    __syncwarp();
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
  const int warps = a.S <= 32 ? 8 : a.S <= 64 ? 4 : 2;
  int side = 1;
  while (side < a.tiles && side < warps) side *= 2;
  *rows = warps / side;
  *blocks = (a.tiles + side - 1) / side;
  const int64_t items = (a.N * a.pieces + *rows - 1) / *rows;
  const int64_t most = std::max<int64_t>(1, (int64_t)sm_count() * (8 / warps) / (*blocks * a.G));
  // as many rounds as the fullest slot makes, spread evenly
  const int64_t rounds = (items + most - 1) / most;
  return std::min<int64_t>((items + rounds - 1) / rounds, 65535) * *rows;
}

template <typename T>
cudaError_t launch_select_back(const Select& a, bool split, cudaStream_t s) {
  int64_t blocks;
  int rows;
  const int64_t slots = select_slots(a, &blocks, &rows);
  cudaError_t e = with_lanes(a.S, [&](auto l) -> cudaError_t {
    using L = decltype(l);
    cudaError_t e;
    if (split) {
      const int64_t warps = a.N * a.G * a.tiles * a.pieces;
      k_select_fold_back<T, L><<<(unsigned)((warps + kFoldWarps - 1) / kFoldWarps), 32 * kFoldWarps, 0, s>>>(a);
      if ((e = cudaGetLastError()) != cudaSuccess || (e = launch_select_join(a, true, s)) != cudaSuccess) return e;
    }
    const auto kern = k_select_back<T, L>;
    const int smem = (int)sizeof(Back<L>) * kBackWarps<L>;
    static_assert(sizeof(Back<L>) * kBackWarps<L> <= 227 * 1024, "shared memory of a block");
    if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return e;
    const dim3 grid((unsigned)(blocks * a.G), (unsigned)(slots / rows));
    if (split) return launch_after(kern, grid, 32 * kBackWarps<L>, smem, s, a, rows);
    kern<<<grid, 32 * kBackWarps<L>, smem, s>>>(a, rows);
    return cudaGetLastError();
  });
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
