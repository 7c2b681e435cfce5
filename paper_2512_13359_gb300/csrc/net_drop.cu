// net_drop.cu -- dropout with a mask drawn from a counter where it is used (auvnet.h, net_dropout).
//
// Eight elements share a Philox4x32-10 block, 16 bits each.  It costs 40 instructions (two wide products and two
// three-way exclusive ors a round; the round keys come from the host), 5 an element, and what else an element takes
// some 7: at 16-bit types that is just under what HBM's pace leaves, so the generator runs while the loads are on their
// way, and where one mask serves all steps it is drawn once for several of them.
//
//  k_blocks  rows of whole blocks, aligned: a thread a block.  65,536 x 256 bf16: 11.8 us (5.7 TB/s), with a residual 15.3
//            (6.6 TB/s).
//  k_lanes   any other rows: a warp takes 32 blocks, its lanes adjacent pieces of E elements, as wide as the alignment
//            allows, 32 E apart from one turn to the next; keep bits come from their block's lane by a shuffle.
//            128 steps of 513 x 257 fp32 sharing a mask: 24.5 us (5.5 TB/s); bf16, each step its own: 34 us (2 TB/s).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "net_common.cuh"

namespace auv {
namespace net {
namespace {

struct Keys {
  uint32_t k[10][2];
};

struct Drop {
  int64_t T, N, D;
  net_rows x, r, y;
  int64_t steps;        // shared: steps of a thread
  bool drawn;           // whether there is a mask to draw (0 < p < 1)
  uint32_t limit;       // keep where 16 bits, as the upper half of a word, are not below it
  float scale;
  uint32_t d0, d1;
  Keys keys;
};

// The words of block q; zeros where none are drawn.
__device__ __forceinline__ uint4 words(const Drop& a, uint64_t q) {
  if (!a.drawn) return make_uint4(0u, 0u, 0u, 0u);
  uint32_t c0 = (uint32_t)q, c1 = (uint32_t)(q >> 32), c2 = a.d0, c3 = a.d1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ a.keys.k[r][0];
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ a.keys.k[r][1];
    c1 = (uint32_t)p1;
    c3 = (uint32_t)p0;
  }
  return make_uint4(c0, c1, c2, c3);
}
// Whether element i of the block is kept: the upper half of its word, or the lower half in the upper's place (what is
// below the upper half does not decide, the limit being 0 there).
__device__ __forceinline__ bool kept(const uint4& w, int i, uint32_t limit) {
  const uint32_t v = i < 4 ? (i < 2 ? w.x : w.y) : (i < 6 ? w.z : w.w);
  return (i & 1 ? v : v << 16) >= limit;
}
// All of a block's as bits.
__device__ __forceinline__ uint32_t keep_bits(const Drop& a, uint64_t q) {
  const uint4 w = words(a, q);
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) bits |= (kept(w, i, a.limit) ? 1u : 0u) << i;
  return bits;
}

template <typename T>
__device__ __forceinline__ T* data(const net_rows& r) { return reinterpret_cast<T*>(r.data); }

constexpr int kThreads = 256;

// Eight elements from x (+ r) to y.
template <typename T, bool RES>
struct Eight {
  uint4 x[sizeof(T) / 2], r[sizeof(T) / 2];
  __device__ void load(const T* px, const T* pr) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      x[i] = reinterpret_cast<const uint4*>(px)[i];
      if constexpr (RES) r[i] = reinterpret_cast<const uint4*>(pr)[i];
    }
  }
  __device__ void store(T* py, const uint4& drawn, uint32_t limit, float scale) const {
    constexpr int E = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      float v[E], w[E];
      unpack<T, E>(x[i], v);
      if constexpr (RES) unpack<T, E>(r[i], w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[e] = kept(drawn, i * E + e, limit) ? v[e] * scale : 0.0f;
        if constexpr (RES) v[e] += w[e];
      }
      reinterpret_cast<uint4*>(py)[i] = pack<T, E>(v);
    }
  }
};

// A block a thread; rows of `per` blocks.  SHARED: rows are the N of a step, and a thread takes several steps.
// Otherwise row t N + n, or one long row (FLAT), the last block of which may be of fewer elements.
template <typename T, bool RES, bool SHARED, bool FLAT>
__global__ void __launch_bounds__(kThreads) k_blocks(Drop a, int64_t total, int64_t per) {
  const int64_t q = blockIdx.x * (int64_t)kThreads + threadIdx.x;
  if (q >= total) return;
  const T *px = data<T>(a.x), *pr = data<T>(a.r);
  T* py = data<T>(a.y);
  if constexpr (SHARED) {
    const int64_t n = q / per, d = (q - n * per) * 8, t0 = blockIdx.y * a.steps, t1 = min(a.T, t0 + a.steps);
    px += n * a.x.inner + d + t0 * a.x.outer;
    py += n * a.y.inner + d + t0 * a.y.outer;
    if constexpr (RES) pr += n * a.r.inner + d + t0 * a.r.outer;
    constexpr int kAtOnce = 4;
    uint4 drawn;
    for (int64_t t = t0; t < t1; t += kAtOnce) {
      Eight<T, RES> v[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (t + u < t1) v[u].load(px + u * a.x.outer, RES ? pr + u * a.r.outer : nullptr);
      }
      if (t == t0) drawn = words(a, q);
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (t + u < t1) v[u].store(py + u * a.y.outer, drawn, a.limit, a.scale);
      }
      px += kAtOnce * a.x.outer;
      py += kAtOnce * a.y.outer;
      if constexpr (RES) pr += kAtOnce * a.r.outer;
    }
  } else {
    if constexpr (FLAT) {
      px += q * 8, py += q * 8, pr += q * 8;
      if (q * 8 + 8 > a.D) {
        const uint32_t bits = keep_bits(a, q);
        for (int i = 0; i < a.D - q * 8; ++i) {
          float v = bits >> i & 1u ? to_float(px[i]) * a.scale : 0.0f;
          if constexpr (RES) v += to_float(pr[i]);
          from_float(v, py[i]);
        }
        return;
      }
    } else {
      int64_t row, n, t;
      if (total <= 0xffffffff) {     // 32-bit divisions where they do
        row = (uint32_t)q / (uint32_t)per;
        t = (uint32_t)row / (uint32_t)a.N;
      } else {
        row = q / per;
        t = row / a.N;
      }
      n = row - t * a.N;
      const int64_t d = (q - row * per) * 8;
      px += t * a.x.outer + n * a.x.inner + d;
      py += t * a.y.outer + n * a.y.inner + d;
      if constexpr (RES) pr += t * a.r.outer + n * a.r.inner + d;
    }
    Eight<T, RES> v;
    v.load(px, pr);
    v.store(py, words(a, q), a.limit, a.scale);
  }
}

// 32 blocks a warp: elements e0 to e0 + 255 of the mask, of which those from `from` on, as many as a slab has, are its:
// the N rows of step t (their mask's elements begin at `from`), all T N rows (N is then their number, T = 1), or,
// SHARED, those of several steps alike.  I: what a slab's offsets fit.  A piece's place follows from that of the one
// 32 pieces before by additions.
template <typename T, int E, bool RES, bool SHARED, typename I>
__global__ void __launch_bounds__(kThreads) k_lanes(Drop a) {
  using W = Raw<T, E>;
  constexpr int kTurns = 8 / E;
  const int lane = threadIdx.x % 32;
  const int64_t slab = a.N * a.D;
  const int64_t warp = (blockIdx.x * (int64_t)kThreads + threadIdx.x) / 32;
  const I D = (I)a.D, rows = 32 * E / D, adv = 32 * E % D;
  const I sx = (I)a.x.inner, sy = (I)a.y.inner, sr = RES ? (I)a.r.inner : 0;
  const I byx = rows * sx + adv, byy = rows * sy + adv, byr = rows * sr + adv;   // 32 pieces on
  for (int64_t y = blockIdx.y; SHARED ? y == blockIdx.y : y < a.T; y += gridDim.y) {
    const int64_t from = SHARED ? 0 : y * slab, e0 = (from & ~(int64_t)7) + warp * 256;
    if (e0 >= from + slab) continue;
    const uint32_t bits = keep_bits(a, (uint64_t)(e0 >> 3) + lane);
    // the lane's first piece: its place among the slab's (the first few of a step's may be the step's before)
    const int64_t k = e0 + lane * E - from;
    const I first = (I)(k < 0 ? k + 8 * a.D : k);
    const I row = first / D, n = k < 0 ? row - 8 : row;
    I d = first - row * D;
    I atx[kTurns], aty[kTurns], atr[kTurns];
    atx[0] = n * sx + d, aty[0] = n * sy + d, atr[0] = RES ? n * sr + d : 0;
#pragma unroll
    for (int i = 1; i < kTurns; ++i) {
      d += adv;
      const bool wrap = d >= D;
      if (wrap) d -= D;
      atx[i] = atx[i - 1] + byx + (wrap ? sx - D : 0);
      aty[i] = aty[i - 1] + byy + (wrap ? sy - D : 0);
      atr[i] = RES ? atr[i - 1] + byr + (wrap ? sr - D : 0) : 0;
    }
    uint32_t mine[kTurns];
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
      mine[i] = __shfl_sync(0xffffffffu, bits, i * 4 * E + lane * E / 8) >> (lane * E % 8);
    const int64_t t0 = SHARED ? y * a.steps : y, t1 = SHARED ? min(a.T, t0 + a.steps) : y + 1;
    const T *px = data<T>(a.x) + t0 * a.x.outer, *pr = RES ? data<T>(a.r) + t0 * a.r.outer : nullptr;
    T* py = data<T>(a.y) + t0 * a.y.outer;
    auto pass = [&](auto whole) {
      auto there = [&](int i) { return decltype(whole)::value || (k + 32 * E * i >= 0 && k + 32 * E * i < slab); };
      for (int64_t t = t0; t < t1; ++t) {
        W x[kTurns];
        [[maybe_unused]] W r[kTurns];
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
          if (there(i)) {
            x[i] = *reinterpret_cast<const W*>(px + atx[i]);
            if constexpr (RES) r[i] = *reinterpret_cast<const W*>(pr + atr[i]);
          }
        }
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
          if (there(i)) {
            float v[E];
            [[maybe_unused]] float w[E];
            unpack<T, E>(x[i], v);
            if constexpr (RES) unpack<T, E>(r[i], w);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              v[e] = mine[i] >> e & 1u ? v[e] * a.scale : 0.0f;
              if constexpr (RES) v[e] += w[e];
            }
            *reinterpret_cast<W*>(py + aty[i]) = pack<T, E>(v);
          }
        }
        px += a.x.outer;
        py += a.y.outer;
        if constexpr (RES) pr += a.r.outer;
      }
    };
    if (e0 >= from && e0 + 256 <= from + slab) pass(std::true_type{});
    else pass(std::false_type{});
  }
}

template <typename T, int E, bool RES, bool SHARED>
cudaError_t launch_lanes(const Drop& a, dim3 grid, bool small, cudaStream_t s) {
  if (small) k_lanes<T, E, RES, SHARED, uint32_t><<<grid, kThreads, 0, s>>>(a);
  else k_lanes<T, E, RES, SHARED, int64_t><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T, bool RES>
cudaError_t launch(Drop a, bool shared, cudaStream_t s) {
  net_rows* const rows[3] = {&a.x, &a.y, &a.r};
  constexpr int kArrays = RES ? 3 : 2;
  // Rows that follow each other alike in every array are one axis (N), or one long row (D); a single step's or env's
  // axis is none.
  bool merge = !shared || a.T == 1, flat = true, vec = true;
  for (int i = 0; i < kArrays; ++i) {
    merge = merge && (a.T == 1 || a.N == 1 || rows[i]->outer == a.N * rows[i]->inner);
    flat = flat && (a.N == 1 || rows[i]->inner == a.D);
    vec = vec && aligned(*rows[i], a.T, a.N, sizeof(T), 16 / sizeof(T));
  }
  if (merge) {
    if (a.N == 1)
      for (int i = 0; i < kArrays; ++i) {
        flat = flat && (a.T == 1 || rows[i]->outer == a.D);
        rows[i]->inner = rows[i]->outer;
      }
    a.N *= a.T, a.T = 1;
    shared = false;
    if (flat) {
      a.D *= a.N, a.N = 1;
      vec = true;
      for (int i = 0; i < kArrays; ++i) vec = vec && aligned(*rows[i], 1, 1, sizeof(T), 16 / sizeof(T));
    }
  } else {
    flat = false;
  }
  const int64_t sms = sm_count();
  if (vec && (flat || a.D % 8 == 0)) {
    const int64_t per = (a.D + 7) / 8, total = per * a.N * (shared ? 1 : a.T);
    const unsigned blocks = (unsigned)((total + kThreads - 1) / kThreads);
    if (shared) {
      // as many steps a thread as leave every SM 2,048 threads
      const int64_t want = std::min<int64_t>(std::min<int64_t>(a.T, 65535), std::max<int64_t>(1, sms * 2048 / total));
      a.steps = (a.T + want - 1) / want;
      const dim3 grid(blocks, (unsigned)((a.T + a.steps - 1) / a.steps));
      k_blocks<T, RES, true, false><<<grid, kThreads, 0, s>>>(a, total, per);
    } else if (flat) {
      k_blocks<T, RES, false, true><<<blocks, kThreads, 0, s>>>(a, total, per);
    } else {
      k_blocks<T, RES, false, false><<<blocks, kThreads, 0, s>>>(a, total, per);
    }
    return cudaGetLastError();
  }
  const int64_t slab = a.N * a.D + (shared || a.T == 1 ? 0 : 7);
  const unsigned blocks = (unsigned)((slab + 8 * kThreads - 1) / (8 * kThreads));
  bool small = a.D <= INT32_MAX / 16 && a.N * a.D <= INT32_MAX / 2;
  for (int i = 0; i < kArrays; ++i) small = small && (a.N == 1 || rows[i]->inner <= (INT32_MAX - a.D) / a.N);
  int e = 4;
  for (int i = 0; i < kArrays; ++i)
    while (e > 1 && (a.D % e || !aligned(*rows[i], a.T, a.N, sizeof(T), e))) e /= 2;
  dim3 grid(blocks, (unsigned)std::min<int64_t>(a.T, 65535));
  if (shared) {
    const int64_t want = std::min<int64_t>(std::min<int64_t>(a.T, 65535), std::max<int64_t>(1, sms * 8 / blocks));
    a.steps = (a.T + want - 1) / want;
    grid.y = (unsigned)((a.T + a.steps - 1) / a.steps);
    if (e == 4) return launch_lanes<T, 4, RES, true>(a, grid, small, s);
    return e == 2 ? launch_lanes<T, 2, RES, true>(a, grid, small, s) : launch_lanes<T, 1, RES, true>(a, grid, small, s);
  }
  if (e == 4) return launch_lanes<T, 4, RES, false>(a, grid, small, s);
  return e == 2 ? launch_lanes<T, 2, RES, false>(a, grid, small, s) : launch_lanes<T, 1, RES, false>(a, grid, small, s);
}

template <typename T>
cudaError_t launch(const Drop& a, bool shared, cudaStream_t s) {
  return a.r.data ? launch<T, true>(a, shared, s) : launch<T, false>(a, shared, s);
}

int run(const net_drop* p, void* stream) {
  if (!p) return fail(AUV_ERR_INVALID, "argument block is NULL");
  if (p->struct_size != sizeof(net_drop))
    return fail(AUV_ERR_INVALID, "struct_size %u, expected %zu", p->struct_size, sizeof(net_drop));
  if (p->dtype > NET_FP16) return fail(AUV_ERR_INVALID, "dtype %u unknown", p->dtype);
  if (p->shared > 1 || p->reserved) return fail(AUV_ERR_INVALID, "shared not 0 or 1, or reserved not 0");
  if (p->T < 0 || p->N < 0 || p->D < 0) return fail(AUV_ERR_INVALID, "negative size");
  if (!(p->p >= 0.0 && p->p <= 1.0)) return fail(AUV_ERR_INVALID, "p outside [0, 1]");
  const int64_t most = (int64_t)1 << 40;
  if (p->T > most || p->N > most || p->D > most || (p->N && p->D > most / p->N) ||
      (p->T && p->N && p->D && p->N * p->D > most / p->T))
    return fail(AUV_ERR_UNSUPPORTED, "T * N * D past 2^40");
  if (!p->T || !p->N || !p->D) return AUV_OK;
  const int z = type_size(p->dtype);
  int rc;
  if ((rc = need_rows(p->x, "x", p->T, p->N, p->D, z, false)) ||
      (p->residual.data && (rc = need_rows(p->residual, "residual", p->T, p->N, p->D, z, false))) ||
      (rc = need_rows(p->y, "y", p->T, p->N, p->D, z, true)))
    return rc;
  const uint32_t thr = (uint32_t)std::floor(p->p * 65536.0 + 0.5);
  Drop a = {};
  a.T = p->T, a.N = p->N, a.D = p->D;
  a.x = p->x, a.r = p->residual, a.y = p->y;
  a.drawn = thr > 0 && thr < 65536;
  a.limit = thr < 65536 ? thr << 16 : 1u;               // of words that are not drawn, 0: all kept, or none
  a.scale = thr < 65536 ? (float)(65536.0 / (65536.0 - thr)) : 0.0f;
  a.d0 = (uint32_t)p->draw, a.d1 = (uint32_t)(p->draw >> 32);
  for (uint32_t r = 0; r < 10; ++r) {
    a.keys.k[r][0] = (uint32_t)p->seed + r * 0x9E3779B9u;
    a.keys.k[r][1] = (uint32_t)(p->seed >> 32) + r * 0xBB67AE85u;
  }
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p->dtype == NET_FP32   ? launch<float>(a, p->shared, s)
                        : p->dtype == NET_BF16 ? launch<__nv_bfloat16>(a, p->shared, s)
                                               : launch<__half>(a, p->shared, s);
  return e == cudaSuccess ? AUV_OK : cuda_fail(e, "net_dropout");
}

}  // namespace
}  // namespace net
}  // namespace auv

extern "C" int net_dropout(const net_drop* a, void* stream) { return auv::net::run(a, stream); }
