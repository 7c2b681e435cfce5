// net_scan.cuh -- what the two kernels of the gated recurrence (net_scan.cu, net_pieces.cu) share.
#pragma once

#include "net_common.cuh"

namespace auv {
namespace net {

struct Scan {
  int T;
  int64_t N, D;
  net_rows f, v, y, dy, df, dv;
  const float* h0;
  float* hT;
  const float* dhT;
  float* dh0;
  const uint8_t *done, *done_prev;
  int64_t envs;          // of done: N, whatever of it has become channels
};

template <typename T>
__device__ __forceinline__ const T* base(const net_rows& r, int64_t n, int64_t d) {
  return reinterpret_cast<const T*>(r.data) + n * r.inner + d;
}

// The flag of step t of env n (0 where there are none).
__device__ __forceinline__ uint32_t end_flag(const Scan& a, int t, int64_t n) {
  const uint8_t* p = t ? a.done : a.done_prev;
  return p ? (uint32_t)__ldg(p + (t ? (t - 1) * a.envs : 0) + n) : 0u;
}

// The arrays of one step that a thread reads: f, v, and backward the state before the step and dy; from the chain's
// first step on (the last of the sequence backward).
template <typename T, bool BACK>
struct Inputs {
  static constexpr int kN = BACK ? 4 : 2;
  const T* p[kN];       // of the chain's first step (i = 2: the state before it)
  int64_t by[kN];       // from one step to the next
  __device__ Inputs(const Scan& a, int64_t n, int64_t d) {
    const net_rows* r[4] = {&a.f, &a.v, &a.y, &a.dy};
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      p[i] = base<T>(*r[i], n, d) + (BACK ? (a.T - 1 - (i == 2)) * r[i]->outer : 0);
      by[i] = BACK ? -r[i]->outer : r[i]->outer;
    }
  }
};

// An affine map h -> A h + B of one channel.  A piece with an episode end in it passes nothing on, whatever came
// before (NaN times 0 included): its A is -0, and the sign is asked for; gates are never negative.  A product of gates
// that would round to +0 is 2^-149 instead (`positive`), an error of the same size: what is infinite before a long piece
// is so after it, as it is when the steps are walked, and not the NaN of 0 times infinity.
struct Map {
  float A, B;
};
__device__ __forceinline__ bool cuts(float A) { return __float_as_uint(A) >> 31; }
__device__ __forceinline__ float positive(float A) { return __uint_as_float(max(__float_as_uint(A), 1u)); }
__device__ __forceinline__ Map then(const Map& p, const Map& q) {   // p, then q
  return cuts(q.A) ? q : Map{positive(p.A * q.A), fmaf(q.A, p.B, q.B)};
}
__device__ __forceinline__ float apply(const Map& q, float h) { return cuts(q.A) ? q.B : fmaf(q.A, h, q.B); }

// The tiles of 32 and of 16 channels that k_pieces makes of a step.  Rows that follow each other in every array are one
// row (flat); otherwise each env has tiles of its own, however few channels they hold.
struct Tiles {
  bool flat;
  int64_t wide, narrow;
};
inline Tiles tiles(int64_t N, int64_t D, bool flat) {
  if (flat) D *= N, N = 1;
  return {flat, N * ((D + 31) / 32), N * ((D + 15) / 16)};
}
inline Tiles tiles_of(int64_t N, int64_t D, const net_rows* const* rows, int arrays) {
  bool flat = true;
  for (int i = 0; i < arrays; ++i) flat = flat && (N == 1 || rows[i]->inner == D);
  return tiles(N, D, flat);
}

// Few channels, many steps (net_pieces.cu); back: the gradients.
constexpr int kPieceThreads = 256;
template <typename T> cudaError_t launch_pieces(const Scan& a, bool back, cudaStream_t s);

}  // namespace net
}  // namespace auv
