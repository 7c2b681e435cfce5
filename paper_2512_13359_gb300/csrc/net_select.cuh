// net_select.cuh -- what the kernels of the selective scan (net_select.cu, net_select_back.cu) share.
//
// Layout.  A warp has adjacent channels of one env n and group g, whose states all read the same B[t] and C[t].  LS lanes
// share CC channels: each of them holds SP of their S states (padded to LS * SP; what is padded has A = B = C = 0), of all
// CC channels, in pairs for the packed fp32 instructions.  Sums over states go over LS lanes, those over channels (dB, dC)
// over the others.  What is computed per channel and step, ahead of the states, is each lane's own for one channel.
#pragma once

#include "net_common.cuh"

namespace auv {
namespace net {

constexpr int kKeep = 16;       // steps from one kept state to the next
constexpr int kMostStates = 128;

struct Select {
  int T, S, G, per;             // per: channels of a group
  int piece, pieces;            // steps of a piece of the sequence, multiples of kKeep
  int tiles;                    // warps that a group's channels take
  bool wide;                    // forward: twice as many channels a lane
  int rows;                     // (env, group) pairs of a warp
  int64_t N, D;
  net_rows x, dt, gate, y, B, C, dy, dx, ddt, dgate, dB, dC;
  const float *A, *skip, *dt_bias, *h0;
  float *hT, *kept;
  const float* dhT;
  float *dh0, *dA, *dskip, *ddt_bias;
  const uint8_t *done, *done_prev;
  float *sums, *maps;           // pieces: [pieces][N][D] sums of step sizes, [pieces][N][D][S] states
  float *weights;               // backward: [slots][D][S + 2] sums of weight gradients
  float *parts;                 // backward, groups of several blocks: [blocks][T][N][G][2][S] sums of dB and dC
};

__device__ __forceinline__ float total(F2 a) {
  float lo, hi;
  split(a, lo, hi);
  return lo + hi;
}
__device__ __forceinline__ F2 ex2(F2 a) {
  float lo, hi;
  split(a, lo, hi);
  return pair(ex2(lo), ex2(hi));
}
constexpr float kLn2 = 0.693147180559945309f;
// exp(e A) of e and A log2 e.  The multi-function unit's 2^t is off by up to 2.4 of 2^-24 of it, and for t from -1 to -2^-8 by
// 0.3 to 0.45 towards 0 on average, which states add up over all steps that they remember.  kLift on the argument, in the
// product's own instruction, takes 0.26 of that off (where t is nearer to 0 it is 0.1 without and -0.16 with it), and 2^0 stays
// 1: states after 128 steps of 4,096 x 256 x 16 are 5.0e-7 off for 1.15e-6, with each exponential rounded to nearest 5.7e-7.
constexpr float kLift = 0x1.8p-26f;
__device__ __forceinline__ F2 decay_of(F2 e, F2 A2) { return ex2(fma2(e, A2, pair(kLift, kLift))); }
// The same, two instructions that hold the constant for one that needs it in registers: the single step has none to spare
// (65,536 envs x 256 x 16 of bf16: 350 us, 359 with a pair).
__device__ __forceinline__ F2 decay_of(float e, F2 A2) {
  float lo, hi;
  split(A2, lo, hi);
  return pair(ex2(fmaf(e, lo, kLift)), ex2(fmaf(e, hi, kLift)));
}

// softplus(v) = max(v, 0) + log(1 + q), q = exp(-|v|), and sigmoid(v) = 1 / (1 + q) or q / (1 + q).  log(1 + q) = 2 atanh(z)
// with z = q / (2 + q) <= 1/3: z times a polynomial in z^2 fitted on [0, 1/9] (Chebyshev, 8e-9 relative), so that a small
// step keeps its digits; off by a few units of 2^-24, and q by 2^-24 |v|.
__device__ __forceinline__ float softplus(float v, float* sigmoid = nullptr) {
  const float q = ex2(fabsf(v) * -kLog2e);
  const float z = __fdividef(q, 2.0f + q), w = z * z;
  float p = fmaf(w, 0.2815778f, 0.27965158f);
  p = fmaf(w, p, 0.40024596f);
  p = fmaf(w, p, 0.6666632f);
  p = fmaf(w, p, 2.0f);
  if (sigmoid) {
    const float r = __fdividef(1.0f, 1.0f + q);
    *sigmoid = v >= 0.0f ? r : q * r;
  }
  return fmaf(z, p, fmaxf(v, 0.0f));
}

// Sums over the lanes that share channels, of CC values a lane (its own OWN channels' first): those of its own.
template <int LS, int CC, int OWN>
__device__ __forceinline__ void over_states(const float (&v)[CC], float (&r)[OWN]) {
#pragma unroll
  for (int j = 0; j < OWN; ++j) {
    r[j] = v[j];
    if constexpr (CC > OWN) r[j] += __shfl_xor_sync(0xffffffffu, v[OWN + j], 1);
#pragma unroll
    for (int bit = CC / OWN; bit < LS; bit *= 2) r[j] += __shfl_xor_sync(0xffffffffu, r[j], bit);
  }
}
template <int LS, int CC>
__device__ __forceinline__ float over_states(const float (&v)[CC]) {
  float r[1];
  over_states<LS, CC, 1>(v, r);
  return r[0];
}

// Values of the lane's own channels to the lanes that share them: r[c] is that of the lane's c-th channel, its own first.
template <int CC, int OWN>
__device__ __forceinline__ void to_lanes(const float (&own)[OWN], float (&r)[CC]) {
#pragma unroll
  for (int j = 0; j < OWN; ++j) {
    r[j] = own[j];
    if constexpr (CC > OWN) r[OWN + j] = __shfl_xor_sync(0xffffffffu, own[j], 1);
  }
}
template <int CC>
__device__ __forceinline__ void to_lanes(float own, float (&r)[CC]) {
  const float v[1] = {own};
  to_lanes<CC, 1>(v, r);
}

template <typename T>
__device__ __forceinline__ const T* row_at(const net_rows& r, int64_t t, int64_t n, int64_t k) {
  return reinterpret_cast<const T*>(r.data) + t * r.outer + n * r.inner + k;
}
// The flag of the end before step t.
__device__ __forceinline__ uint8_t flag_at(const Select& a, int t, int64_t n) {
  const uint8_t* p = t ? a.done : a.done_prev;
  return p ? p[(t ? (t - 1) * a.N : 0) + n] : (uint8_t)0;
}
__device__ __forceinline__ bool ended(const Select& a, int t, int64_t n) { return flag_at(a, t, n) != 0; }
// Bit i: an episode ended before step t + i, of the 16 from t on.
__device__ __forceinline__ uint32_t ends_of(const Select& a, int t, int64_t n, int lane) {
  if (!a.done && !a.done_prev) return 0u;
  return __ballot_sync(0xffffffffu, lane < kKeep && t + lane < a.T && ended(a, t + lane, n));
}

// SP states of CC channels from s0 of an [.][S] array: pairs, zeros past S and for channels that are not there.  Whole
// sectors of 32 bytes a thread where S and the array allow them.
template <int SP>
__device__ __forceinline__ bool whole_sectors(const float* p, int S) {
  return S % SP == 0 && reinterpret_cast<uintptr_t>(p) % (4 * SP) == 0;
}
template <int SP, int CC>
__device__ __forceinline__ void load_states(const float* p, const int64_t (&at)[CC], const bool (&there)[CC], int s0, int S,
                                            F2 (&h)[CC][SP / 2]) {
  const bool vec = whole_sectors<SP>(p, S);
#pragma unroll
  for (int c = 0; c < CC; ++c) {
    const float* q = p + at[c] * S + s0;
#pragma unroll
    for (int i = 0; i < SP / 2; ++i) h[c][i] = pair(0.0f, 0.0f);
    if (!p || !there[c] || s0 >= S) continue;
    if (vec) {
      if constexpr (SP == 8) {
        asm volatile("ld.global.v4.b64 {%0, %1, %2, %3}, [%4];"
                     : "=l"(h[c][0].v), "=l"(h[c][1].v), "=l"(h[c][2].v), "=l"(h[c][3].v)
                     : "l"(q)
                     : "memory");
      } else {
        const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(q);
        h[c][0].v = w.x, h[c][1].v = w.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < SP / 2; ++i)
        h[c][i] = pair(s0 + 2 * i < S ? q[2 * i] : 0.0f, s0 + 2 * i + 1 < S ? q[2 * i + 1] : 0.0f);
    }
  }
}
template <int SP, int CC>
__device__ __forceinline__ void store_states(float* p, const int64_t (&at)[CC], const bool (&there)[CC], int s0, int S,
                                             const F2 (&h)[CC][SP / 2]) {
  const bool vec = whole_sectors<SP>(p, S);
#pragma unroll
  for (int c = 0; c < CC; ++c) {
    float* q = p + at[c] * S + s0;
    if (!there[c] || s0 >= S) continue;
    if (vec) {
      if constexpr (SP == 8) {
        asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(q), "l"(h[c][0].v), "l"(h[c][1].v), "l"(h[c][2].v),
                     "l"(h[c][3].v)
                     : "memory");
      } else {
        *reinterpret_cast<ulonglong2*>(q) = make_ulonglong2(h[c][0].v, h[c][1].v);
      }
    } else {
#pragma unroll
      for (int i = 0; i < SP / 2; ++i) {
        float lo, hi;
        split(h[c][i], lo, hi);
        if (s0 + 2 * i < S) q[2 * i] = lo;
        if (s0 + 2 * i + 1 < S) q[2 * i + 1] = hi;
      }
    }
  }
}

// The rows of B or C of up to 16 steps from t on, into [16][SW] fp32, zeros past S.
template <typename T, int SW, int RL>
__device__ __forceinline__ void stage(const Select& a, const net_rows& r, int t, int steps, int64_t n, int g, int lane, float* to) {
  constexpr int kSide = SW < RL ? SW : RL, kRows = RL / kSide;        // a lane's states stay, its rows are kRows apart
  const int s = lane % kSide, k = lane / kSide;
  const T* p = row_at<T>(r, t + k, n, (int64_t)g * a.S + s);
  const int64_t by = kRows * r.outer;
#pragma unroll
  for (int j = 0; j < kKeep / kRows; ++j) {
#pragma unroll
    for (int i = 0; i < SW / kSide; ++i)
      to[(k + j * kRows) * SW + s + i * kSide] = k + j * kRows < steps && s + i * kSide < a.S ? to_float(p[i * kSide]) : 0.0f;
    p += by;
  }
}

// The same for STEPS steps, in two parts: the loads, of a lane's values, and their way into shared memory.
// RL: lanes that a row's states are loaded by.
template <typename T, int SW, int STEPS, int RL = 32>
struct Staged {
  static constexpr int kSide = SW < RL ? SW : RL, kRows = RL / kSide;
  static constexpr int kDown = (STEPS + kRows - 1) / kRows, kAcross = SW / kSide;
  T v[kDown][kAcross];
  __device__ __forceinline__ void load(const T* p, int64_t by, int steps, int S, int lane) {   // p: the lane's first value
    const int s = lane % kSide, k = lane / kSide;
#pragma unroll
    for (int j = 0; j < kDown; ++j) {
#pragma unroll
      for (int i = 0; i < kAcross; ++i) {
        from_float(0.0f, v[j][i]);
        if (k + j * kRows < steps && s + i * kSide < S) v[j][i] = p[i * kSide];
      }
      p += kRows * by;
    }
  }
  __device__ __forceinline__ void put(float* to, int lane) const {
    const int s = lane % kSide, k = lane / kSide;
#pragma unroll
    for (int j = 0; j < kDown; ++j)
      if (STEPS % kRows == 0 || k + j * kRows < STEPS) {
#pragma unroll
        for (int i = 0; i < kAcross; ++i) to[(k + j * kRows) * SW + s + i * kSide] = to_float(v[j][i]);
      }
  }
};

// SP values of a staged row as pairs.
template <int SP>
__device__ __forceinline__ void load_pairs(const float* p, F2 (&v)[SP / 2]) {
#pragma unroll
  for (int i = 0; i < SP; i += 4) {
    const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(p + i);
    v[i / 2].v = w.x;
    v[i / 2 + 1].v = w.y;
  }
}

// How S states are laid over lanes.
// R: envs (with the same group, or groups) that a warp has side by side, of narrow groups, RL lanes each.
template <int SP_, int LS_, int CC_, int OWN_ = 1, int R_ = 1> struct Lanes {
  static constexpr int SP = SP_, LS = LS_, CC = CC_, OWN = OWN_;   // CC: OWN, or twice that
  static constexpr int R = R_, RL = 32 / R;
  static constexpr int SW = SP * LS;          // states, padded
  static constexpr int CW = RL / LS * CC;     // channels of a warp, or of a row of it
};
constexpr int kNarrow = 8, kSide4 = 4;         // groups of up to 8 channels, of up to 16 states: four rows a warp
template <typename F>
cudaError_t with_narrow_lanes(int S, F f) {
  if (S <= 4) return f(Lanes<4, 1, 1, 1, kSide4>());
  if (S <= 8) return f(Lanes<8, 1, 1, 1, kSide4>());
  return f(Lanes<8, 2, 2, 1, kSide4>());
}
template <typename F>
cudaError_t with_lanes(int S, F f) {
  if (S <= 4) return f(Lanes<4, 1, 1>());
  if (S <= 8) return f(Lanes<8, 1, 1>());
  if (S <= 16) return f(Lanes<8, 2, 2>());
  if (S <= 32) return f(Lanes<8, 4, 2>());
  if (S <= 64) return f(Lanes<8, 8, 2>());
  return f(Lanes<8, 16, 2>());
}
inline int lanes_channels(int S) { return S <= 16 ? 32 : S <= 32 ? 16 : S <= 64 ? 8 : 4; }
// Forward twice as many channels a lane: what a lane reads of B and C, and its addresses, serve twice the states (4,096 x 128
// x 256 x 16 bf16: 683 us, 822 with half as many).
template <typename F>
cudaError_t with_wide_lanes(int S, F f) {
  if (S <= 8) return f(Lanes<8, 1, 2, 2>());
  return f(Lanes<8, 2, 4, 2>());
}
constexpr int kMostWide = 16, kWideChannels = 64;   // states; channels of a warp

// The states before the pieces from the pieces' maps, in the maps' place (net_select.cu).
cudaError_t launch_select_join(const Select& a, bool back, cudaStream_t s);
template <typename T> cudaError_t launch_select_back(const Select& a, bool split, cudaStream_t s);
// Pieces and steps of a piece for warps that each walk T steps.
void select_pieces(Select& a, bool back);
int64_t select_slots(const Select& a, int64_t* blocks, int* rows);

}  // namespace net
}  // namespace auv
