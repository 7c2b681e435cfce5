// net_ortho.cu -- orthogonalised updates by Newton-Schulz products (auvnet.h, net_orthogonalise).
//
// X <- a X + (b P + c P P) X with P = X X^T: per step the symmetric P, the symmetric Q = a I + b P + c P P, and Q X; of a
// matrix with more rows than columns P = X^T X and X Q, so that P is of the shorter side.  Nothing is transposed: an
// operand is read by rows or along its columns as the product wants it.
//
// fp32 values on tensor cores: v = hi + lo, two fp16 pieces of 11 bits each, and u v = hi hi + hi lo + lo hi, three MMAs
// into one fp32 accumulator; lo lo, 2^-22 of the product, is left out.  Scaled by powers of two the pieces' range holds
// every value to 2^-34 of the largest that can occur (the coefficients are checked for that).
//
// All products of a call are one cooperative launch, a block an SM, with barriers over all blocks between the products.
// Of a 128 x 128 or 128 x 256 tile a producer thread streams 128-byte-swizzled tiles of both pieces of both operands into a
// ring with TMA, one thread issues tcgen05.mma into tensor memory, and eight warps read the sums back, split them into
// pieces again and store them; of the symmetric products the tiles on and below the diagonal, stored on both sides of it.
//
// The tensor core cuts what it adds to an accumulator (each addition loses up to 2^-23 of it, always towards 0), which over
// K = 4096 came to 9e-5 of the result.  So a sum runs over 64 of K there, small products first, and those sums are added in
// registers, rounded to nearest, while the next 64 run into the other half of tensor memory (1e-6; 8 % of the time).
//
// 4,096 x 4,096 fp32, five steps: 3.0 to 3.1 ms on several boxes, 68 to 71 % of the measured bf16 rate in products (three for
// one, symmetric ones by half): large products are taken by pairs of blocks (below).  24 x 1,000 x 515 bf16: 780 to 790 us;
// 4 x 256 x 256 fp32: 162 us, latency of 15 products and barriers.
#include <cuda.h>

#include <algorithm>
#include <cmath>
#include <mutex>

#include "net_common.cuh"
#include "tc_ptx.cuh"

namespace auv {
namespace net {
namespace {

constexpr float kScaleX = 4096.0f, kScaleP = 512.0f, kScaleQ = 64.0f;     // of the stored pieces
constexpr int kBM = 128, kBK = 64;                                        // BK: 128 bytes of fp16
constexpr uint64_t kWaitLimitNs = 2000000000ull;

enum Kind { kP, kQ, kX, kLast };

// ---- sums of squares ----
// Of x, and of x times 2^100 and 2^-96: one of the three is in range wherever the largest |x| is, of up to 2^36 values.  2^-96:
// squares of the largest, 2^64, sum up to 2^100.  2^100: those of the smallest subnormal are 2^-98, and of sums below 1e-24
// (kLow) they come to less than 2^121.  What a sum from kLow on, or the scaled one of a sum from kHigh on, loses of squares
// below 2^-149 is 2^-34 of it at most.
constexpr float kUp = 0x1p100f, kDown = 0x1p-96f, kLow = 1e-24f, kHigh = 1e36f;
constexpr int kNormThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kNormThreads) k_squares(net_rows x, int64_t M, int64_t N, float* partial, int* error) {
  __shared__ float part[3][kNormThreads / 32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) error[0] = AUV_OK, error[1] = 0;     // and the barriers' count
  const T* const p = reinterpret_cast<const T*>(x.data) + blockIdx.y * x.outer;
  float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f;
  const int64_t all = M * N, step = gridDim.x * (int64_t)kNormThreads;
  int64_t i = blockIdx.x * (int64_t)kNormThreads + threadIdx.x;
  int64_t r = i / N, c = i - r * N;
  const int64_t dr = step / N, dc = step - dr * N;
  constexpr int kU = 4;
  while (i < all) {
    T v[kU];
    int n = 0;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      from_float(0.0f, v[u]);
      if (i < all) {
        v[u] = p[r * x.inner + c];
        ++n;
      }
      i += step, r += dr, c += dc;
      if (c >= N) c -= N, ++r;
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const float w = to_float(v[u]), up = w * kUp, down = w * kDown;
      s0 = fmaf(w, w, s0);
      s1 = fmaf(up, up, s1);
      s2 = fmaf(down, down, s2);
    }
  }
  float* const s[3] = {&s0, &s1, &s2};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
#pragma unroll
    for (int o = 16; o; o /= 2) *s[k] += __shfl_xor_sync(0xffffffffu, *s[k], o);
    if (threadIdx.x % 32 == 0) part[k][threadIdx.x / 32] = *s[k];
  }
  __syncthreads();
  if (threadIdx.x < 3) {
    float v = 0.0f;
    for (int w = 0; w < kNormThreads / 32; ++w) v += part[threadIdx.x][w];
    partial[(blockIdx.y * (int64_t)gridDim.x + blockIdx.x) * 3 + threadIdx.x] = v;
  }
}

// 1 / (|x| + eps) as two factors, from the blocks' sums (every thread of a block; fixed order).  Multiplied one after the other
// they keep x in range.  NaN where a value is not finite.
__device__ __forceinline__ float2 inverse_norm(const float* partial, int blocks, float eps) {
  __shared__ float part[3][kNormThreads / 32];
  float s[3] = {0.0f, 0.0f, 0.0f};
  for (int b = threadIdx.x; b < blocks; b += kNormThreads)
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k] += partial[b * 3 + k];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
#pragma unroll
    for (int o = 16; o; o /= 2) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
    if (threadIdx.x % 32 == 0) part[k][threadIdx.x / 32] = s[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    s[k] = 0.0f;
    for (int w = 0; w < kNormThreads / 32; ++w) s[k] += part[k][w];
  }
  if (s[0] >= kHigh) {                       // also infinite sums; NaN falls through
    if (isinf(s[2])) return make_float2(__uint_as_float(0x7fc00000u), 1.0f);
    return make_float2(1.0f / (sqrtf(s[2]) + eps * kDown), kDown);
  }
  if (s[0] < kLow && !isinf(eps * kUp)) return make_float2(kUp, 1.0f / (sqrtf(s[1]) + eps * kUp));     // else |x| is nothing to eps
  return make_float2(1.0f, 1.0f / (sqrtf(s[0]) + eps));
}

// x / (|x| + eps): as pieces, or as y.
template <typename T, bool PIECES>
__global__ void __launch_bounds__(kNormThreads) k_scaled(net_rows x, int64_t M, int64_t N, int64_t L, const float* partial,
                                                         int blocks, float eps, __half* out, int64_t ld, net_rows y) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  after_previous();
  const int64_t l = blockIdx.y;
  const float2 f = inverse_norm(partial + l * blocks * 3, blocks, eps);
  const T* const p = reinterpret_cast<const T*>(x.data) + l * x.outer;
  const int64_t all = M * N, step = gridDim.x * (int64_t)kNormThreads;
  int64_t i = blockIdx.x * (int64_t)kNormThreads + threadIdx.x;
  int64_t r = i / N, c = i - r * N;
  const int64_t dr = step / N, dc = step - dr * N;
  __half* const hi = out + l * M * ld;
  __half* const lo = hi + L * M * ld;
#pragma unroll 4
  for (; i < all; i += step) {
    float v = to_float(p[r * x.inner + c]) * f.x * f.y;
    if constexpr (PIECES) {
      v *= kScaleX;
      const __half h = __float2half_rn(v);
      hi[r * ld + c] = h;
      lo[r * ld + c] = __float2half_rn(v - __half2float(h));
    } else {
      from_float(v, reinterpret_cast<T*>(y.data)[l * y.outer + r * y.inner + c]);
    }
    r += dr, c += dc;
    if (c >= N) c -= N, ++r;
  }
}

// ---- products ----
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          tc::smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(tc::smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ uint64_t tile_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {   // 128-byte swizzle
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)((lbo >> 4) & 0x3FFFu) << 16 | (uint64_t)((sbo >> 4) & 0x3FFFu) << 32 |
         (uint64_t)1u << 46 | (uint64_t)2u << 61;
}
// fp16 operands, fp32 sums; bits 15, 16: A, B along M or N.
__host__ __device__ constexpr uint32_t idesc_f16(bool a_mn, bool b_mn, int M, int N) {
  return (1u << 4) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// A pair of blocks (a cluster of two) on one 256 x 256 tile: each loads its 128 rows of A and half of B's columns, and
// signals the first one's barrier.
__device__ __forceinline__ void tma_load_pair(void* dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          tc::smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t more) {
  if constexpr (PAIR)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
                 "l"(b), "r"(id), "r"(more)
                 : "memory");
  else
    tc::mma_ss(d, a, b, id, more);
}
// The barrier, of both blocks of a pair, when all products issued so far are done.
template <bool PAIR>
__device__ __forceinline__ void commit(uint64_t* bar) {
  if constexpr (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                     tc::smem_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
  else
    tc::mma_commit(bar);
}
template <bool PAIR>
__device__ __forceinline__ void alloc(uint32_t* dst, uint32_t cols) {
  if constexpr (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(dst)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    tc::tmem_alloc(dst, cols);
    tc::tmem_relinquish();
  }
}
template <bool PAIR>
__device__ __forceinline__ void dealloc(uint32_t at, uint32_t cols) {
  if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols) : "memory");
  else tc::tmem_dealloc(at, cols);
}
__device__ __forceinline__ void wait_landed(uint64_t* b, uint32_t phase) {
  const uint64_t t0 = tc::global_timer_ns();
  while (!tc::mbar_test(b, phase) && tc::global_timer_ns() - t0 < kWaitLimitNs) {
  }
}

// One of a step's products: result rows x cols, contraction K; which operands run along M or N.
struct Product {
  int kind, rows, cols, K, high, wide;   // high, wide: of a tile
  bool a_mn, b_mn;
};

struct Steps {
  CUtensorMap x_rows[2], x_cols[2], p, q;   // boxes of 128 rows; x_cols: of 64
  int L, M, N, s, steps, ldx, lds;          // s: the shorter side
  bool wide;                                // M <= N
  int tile[3];                              // columns of a tile of P, Q, X
  bool single;                              // a matrix is one tile of each
  float a, b, c;
  __half *x[2], *P, *Q;                     // pieces [2][L][rows][ld]
  net_rows y;
  int dtype;
  int* error;
  unsigned* arrived;                        // blocks at the barriers between products, and kGaveUp
  uint64_t limit;                           // of a wait, in ns
  int stuck;                                // self-test: the first block waits in vain behind this product
};

// Shared memory: a ring of two stages of 256-column tiles or of three of 128-column ones.
constexpr uint32_t kA = kBM * 128;           // one piece of A in a stage; of B: 128 bytes a column
constexpr uint32_t kRing = 196608, kTurn = 8 * 32 * 33 * 4;   // kTurn: a 32 x 32 block a storing warp
constexpr uint32_t kSmem = kRing + kTurn + 256 + 1024;
static_assert(kSmem <= 227 * 1024, "shared memory of a block");
__host__ __device__ constexpr int stages_of(int wide) { return wide > 128 ? 2 : 3; }
__host__ __device__ constexpr uint32_t stage_bytes(int wide) { return 2 * (kA + wide * 128); }
static_assert(stages_of(256) * stage_bytes(256) == kRing && stages_of(128) * stage_bytes(128) == kRing, "the ring");
struct Bars {
  uint64_t full[3], empty[3], sums[2], taken[2], drained;
  uint32_t tmem;
  int abort;
};
// Two warpgroups that store, and one with the producer and the issuer.  Registers: at launch 384 threads x 168 = 64,512;
// the storing warps, with up to 128 sums a thread, take 224, the others keep 56: 256 x 224 + 128 x 56 = 64,512.
constexpr int kStorers = 8, kProducer = 8, kIssuer = 9, kThreads = 384;
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 224;"); }
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 56;"); }

// A warp's 32 x 32 block of sums, a row a lane, is turned through shared memory so that four lanes have a row's 32 columns
// (64 bytes of a piece) and an access eight rows; a thread storing its own row took 2.1 us a 128 x 128 tile, and 4 to 5 us
// more where the block is also stored on the other side of the diagonal, a value at a time.

// Eight scaled values as pieces (a row's padding may be written).
__device__ __forceinline__ void store_pieces(__half* hi, int64_t to_lo, const float (&v)[8]) {
  uint32_t h[4], o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 w = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    const float2 f = __half22float2(w);
    const __half2 z = __floats2half2_rn(v[2 * i] - f.x, v[2 * i + 1] - f.y);
    h[i] = *reinterpret_cast<const uint32_t*>(&w);
    o[i] = *reinterpret_cast<const uint32_t*>(&z);
  }
  *reinterpret_cast<uint4*>(hi) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4*>(hi + to_lo) = make_uint4(o[0], o[1], o[2], o[3]);
}

// The block at (r0, c0) of a product that goes on as pieces, from turn[row * 33 + column]; with `mirror` its mirror image too.
template <int AHEAD>
__device__ __forceinline__ void store_block(const Steps& a, const Product& p, __half* out, int ld, int l, int r0, int c0, bool mirror,
                                            float* turn, int lane) {
  const int64_t to_lo = (int64_t)a.L * p.rows * ld, at = (int64_t)l * p.rows * ld;
  const int q = lane % 4 * 8;
  const float scale = p.kind == kP ? kScaleP / (kScaleX * kScaleX) : p.kind == kX ? 1.0f / kScaleQ : a.c * (kScaleQ / (kScaleP * kScaleP));
  const float fb = a.b * (kScaleQ / kScaleP);
  uint4 ph[AHEAD], po[AHEAD];                // P's values, on their way ahead of the stores
  auto fetch = [&](int i) {
    const int r = r0 + i * 8 + lane / 4;
    ph[i % AHEAD] = po[i % AHEAD] = make_uint4(0, 0, 0, 0);
    if (r < p.rows && c0 + q < p.cols) {
      const __half* const from = a.P + at + (int64_t)r * ld + c0 + q;
      ph[i % AHEAD] = *reinterpret_cast<const uint4*>(from);
      po[i % AHEAD] = *reinterpret_cast<const uint4*>(from + to_lo);
    }
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (p.kind == kQ && i % AHEAD == 0) {
#pragma unroll
      for (int k = i; k < i + AHEAD; ++k) fetch(k);
    }
    const int k = i * 8 + lane / 4, r = r0 + k, c = c0 + q;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = turn[k * 33 + q + e] * scale;
    if (p.kind == kQ) {
      float h[8], o[8];
      unpack<__half, 8>(ph[i % AHEAD], h);
      unpack<__half, 8>(po[i % AHEAD], o);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += fmaf(fb, h[e], fb * o[e]) + (c + e == r ? a.a * kScaleQ : 0.0f);
    }
    if (mirror) {
#pragma unroll
      for (int e = 0; e < 8; ++e) turn[k * 33 + q + e] = v[e];
    }
    if (r < p.rows && c < p.cols) store_pieces(out + at + (int64_t)r * ld + c, to_lo, v);
  }
  if (!mirror) return;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = i * 8 + lane / 4, r = c0 + k, c = r0 + q;
    if (r < p.rows && c < p.cols) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = turn[(q + e) * 33 + k];
      store_pieces(out + at + (int64_t)r * ld + c, to_lo, v);
    }
  }
}

// The block at (r0, c0) of the last product: y's rows start anywhere, the warp stores a row's values together.
template <typename T>
__device__ __forceinline__ void store_last(const Steps& a, int l, int r0, int c0, const float* turn, int lane) {
  if (c0 + lane >= a.N) return;
  T* p = reinterpret_cast<T*>(a.y.data) + l * a.y.outer + r0 * a.y.inner + c0 + lane;
#pragma unroll 8
  for (int i = 0; i < 32; ++i, p += a.y.inner)
    if (r0 + i < a.M) from_float(turn[i * 33 + lane] * (1.0f / (kScaleQ * kScaleX)), *p);
}

// Tiles of a product, of high x wide: number, and the t-th of a matrix.  Of symmetric results those that reach the diagonal
// or lie below it: row i of square tiles begins with number i (i + 1) / 2, of tiles twice as wide with about i^2 / 4.
__host__ __device__ inline int start_of(int i, int high, int wide) {
  return wide == high ? i * (i + 1) / 2 : (i / 2) * (i / 2 + 1) + (i & 1 ? i / 2 + 1 : 0);
}
__host__ __device__ inline int tiles_of(int kind, int rows, int cols, int high, int wide) {
  const int tm = (rows + high - 1) / high;
  return kind == kP || kind == kQ ? start_of(tm, high, wide) : tm * ((cols + wide - 1) / wide);
}
__device__ __forceinline__ void tile_at(const Product& p, int t, int& ti, int& tj) {
  if (p.kind != kP && p.kind != kQ) {
    // neighbours in groups of 8 tile rows: they read the same columns of B at about the same time
    const int tm = (p.rows + p.high - 1) / p.high, tn = (p.cols + p.wide - 1) / p.wide, group = t / (8 * tn), first = group * 8;
    const int most = min(8, tm - first), in = t - group * 8 * tn;
    ti = first + in % most, tj = in / most;
    return;
  }
  ti = (int)sqrtf((p.wide == p.high ? 2.0f : 4.0f) * t);
  while (start_of(ti, p.high, p.wide) > t) --ti;
  while (start_of(ti + 1, p.high, p.wide) <= t) ++ti;
  tj = t - start_of(ti, p.high, p.wide);
}

// Every block has arrived `round` times, and what they stored is seen, by TMA too.  Bounded.  A block that gave up, here or in
// the product before, says so ahead of its arrival, and the others give up with it: none goes on from a product that is not
// whole.  Returns whether to go on, the same to all threads.
constexpr unsigned kGaveUp = 1u << 31;
__device__ __forceinline__ bool all_blocks(const Steps& a, unsigned round, volatile int* abort) {
  asm volatile("fence.proxy.async.global;" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool in_vain = (int)round == a.stuck && blockIdx.x == 0;
    auto give_up = [&] {
      *abort = 1;
      asm volatile("red.relaxed.gpu.global.or.b32 [%0], %1;" ::"l"(a.arrived), "r"(kGaveUp) : "memory");
    };
    __threadfence();
    if (*abort) give_up();
    asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(a.arrived) : "memory");
    const uint64_t t0 = tc::global_timer_ns();
    for (unsigned it = 1; !*abort; ++it) {
      unsigned v;
      asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(a.arrived) : "memory");
      if (v & kGaveUp) *abort = 1;
      else if (v >= round * gridDim.x && !in_vain) break;
      else if ((it & 63u) == 0 && tc::global_timer_ns() - t0 > a.limit) give_up();
    }
  }
  const bool on = !__syncthreads_or(threadIdx.x == 0 && *abort);
  asm volatile("fence.proxy.async.global;" ::: "memory");
  return on;
}

// The same where every matrix is one tile of each product, always the same block's.
__device__ __forceinline__ bool this_block(volatile int* abort) {
  asm volatile("fence.proxy.async.global;" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) __threadfence();
  const bool on = !__syncthreads_or(threadIdx.x == 0 && *abort);
  asm volatile("fence.proxy.async.global;" ::: "memory");
  return on;
}

// After a wait that gave up: NaN in y where this block's tiles lie, whichever of them were stored.
template <typename T>
__device__ __forceinline__ void spoil(const Steps& a, int l, int m0, int n0, int wide) {
  T nan;
  from_float(__uint_as_float(0x7fc00000u), nan);
  T* const p = reinterpret_cast<T*>(a.y.data) + l * a.y.outer;
  for (int i = threadIdx.x; i < kBM * wide; i += kStorers * 32) {
    const int r = m0 + i / wide, c = n0 + i % wide;
    if (r < a.M && c < a.N) p[r * a.y.inner + c] = nan;
  }
}

// PAIR: blocks in clusters of two, each with 128 of a tile's 256 rows; the first one issues the products of both.
template <int BN, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) k_products(const __grid_constant__ Steps a) {
  constexpr int kCols = BN / 2;              // of a storing warp's row
  constexpr int kBlocks = PAIR ? 2 : 1, kHigh = kBlocks * kBM;
  const int rank = PAIR ? (int)tc::cluster_rank() : 0;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023u) & ~(uintptr_t)1023u);
  Bars* const bar = reinterpret_cast<Bars*>(smem + kRing + kTurn);
  volatile int* const abort = &bar->abort;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  if (tid == 0) {
    for (int s = 0; s < 3; ++s) {
      tc::mbar_init(&bar->full[s], 1);
      tc::mbar_init(&bar->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      tc::mbar_init(&bar->sums[b], 1);
      tc::mbar_init(&bar->taken[b], kStorers * kBlocks);
    }
    tc::mbar_init(&bar->drained, 1);
    bar->abort = 0;
    tc::mbar_fence_init();
  }
  if (warp == kProducer && lane < 6) {
    const CUtensorMap* const maps[6] = {&a.x_rows[0], &a.x_rows[1], &a.x_cols[0], &a.x_cols[1], &a.p, &a.q};
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(maps[lane])) : "memory");
  }
  if (warp == kIssuer) {
    alloc<PAIR>(&bar->tmem, 2 * BN);
  }
  tc::tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) tc::cluster_sync();    // the other block's barriers are there
  tc::tc_fence_after();
  const uint32_t tmem = bar->tmem;
  // The blocks' products and tiles, the same for every role: do(p, A, B, chunks, l, m0, n0, in).
  uint32_t chunk = 0;                        // of this block, over all tiles and products: each role counts its own
  uint32_t used = 0, parity = 0;             // bit s: stage s has been filled; an odd number of times
  auto all_tiles = [&](auto&& work) {
    for (int k = 0; k < a.steps * 3; ++k) {
      const int in = k / 3 & 1;                // which of the two X is read
      const bool last = k / 3 + 1 == a.steps;
      Product p;
      const CUtensorMap *A, *B;
      if (k % 3 == 0) {
        p = {kP, a.s, a.s, a.wide ? a.N : a.M, kHigh, a.tile[0], !a.wide, !a.wide};
        A = B = a.wide ? &a.x_rows[in] : &a.x_cols[in];
      } else if (k % 3 == 1) {
        p = {kQ, a.s, a.s, a.s, kHigh, a.tile[1], false, false};
        A = B = &a.p;
      } else {
        p = {last ? kLast : kX, a.M, a.N, a.s, kHigh, a.tile[2], false, a.wide};
        A = a.wide ? &a.q : &a.x_rows[in];
        B = a.wide ? &a.x_cols[in] : &a.q;
      }
      const int chunks = (p.K + kBK - 1) / kBK, each = tiles_of(p.kind, p.rows, p.cols, p.high, p.wide);
      int stage = 0;                           // the ring begins anew, with as many stages as these tiles leave
      const int64_t all = (int64_t)each * a.L;
      for (int64_t t = blockIdx.x / kBlocks; t < all; t += gridDim.x / kBlocks) {
        if (*abort) break;
        int ti, tj;
        const int l = (int)(t / each);
        tile_at(p, (int)(t % each), ti, tj);
        const int m0 = ti * kHigh + rank * kBM, n0 = tj * p.wide;
        work(p, A, B, chunks, l, m0, n0, in, stage);
      }
      if (k + 1 < a.steps * 3 && !(a.single ? this_block(abort) : all_blocks(a, (unsigned)k + 1, abort))) break;
    }
  };
  if (warp < kStorers) {
    more_registers();
    all_tiles([&](const Product& p, const CUtensorMap*, const CUtensorMap*, int chunks, int l, int m0, int n0, int in, int&) {
        float acc[kCols];
#pragma unroll
        for (int i = 0; i < kCols; ++i) acc[i] = 0.0f;
        bool ok = true;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16, half = warp / 4 * (p.wide / 2);
#pragma unroll 1
        for (int c = 0; c < chunks; ++c, ++chunk) {
          const uint32_t buf = chunk & 1u;
          ok = ok && tc::mbar_wait(&bar->sums[buf], chunk / 2 & 1u, abort, a.limit);
          if (!__all_sync(0xffffffffu, ok)) ok = false;
          tc::tc_fence_after();
          if (ok) {
#pragma unroll
            for (int j = 0; j < kCols; j += 64) {        // 64 columns on their way at a time
              if (j >= p.wide / 2) break;
              uint32_t r[32], q[32];
              tc::tmem_ld32(tmem + lanes + buf * BN + half + j, r);
              tc::tmem_ld32(tmem + lanes + buf * BN + half + j + 32, q);
              tc::tmem_ld_wait(r);
              tc::tmem_ld_wait(q);
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                acc[j + i] += __uint_as_float(r[i]);
                acc[j + 32 + i] += __uint_as_float(q[i]);
              }
            }
          }
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            // nothing but tensor memory has been read: no release at cluster scope, which waited 1 us for it to mean nothing
            if constexpr (PAIR)
              asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(tc::mapa(tc::smem_u32(&bar->taken[buf]), 0)) : "memory");
            else tc::mbar_arrive(&bar->taken[buf]);
          }
        }
        const int r0 = m0 + warp % 4 * 32;
        float* const turn = reinterpret_cast<float*>(smem + kRing) + warp * 32 * 33;
#pragma unroll
        for (int j = 0; j < kCols; j += 32) {
          if (j >= p.wide / 2) break;
          const int col = n0 + (int)half + j;
          float* const v = acc + j;
          if (!ok) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(0x7fc00000u);
          }
          if (r0 < p.rows && col < p.cols && (p.kind >= kX || col <= r0)) {
#pragma unroll
            for (int i = 0; i < 32; ++i) turn[lane * 33 + i] = v[i];
            __syncwarp();
            if (p.kind == kLast) {
              if (a.dtype == NET_FP32) store_last<float>(a, l, r0, col, turn, lane);
              else if (a.dtype == NET_BF16) store_last<__nv_bfloat16>(a, l, r0, col, turn, lane);
              else store_last<__half>(a, l, r0, col, turn, lane);
            } else {
              __half* const out = p.kind == kP ? a.P : p.kind == kQ ? a.Q : a.x[in ^ 1];
              const int ld = p.kind == kX ? a.ldx : a.lds;
              store_block<4>(a, p, out, ld, l, r0, col, p.kind != kX && col < r0, turn, lane);
            }
            __syncwarp();
          }
        }
    });
  } else {
    fewer_registers();
    if (warp == kProducer) {
      all_tiles([&](const Product& p, const CUtensorMap* A, const CUtensorMap* B, int chunks, int l, int m0, int n0, int, int& stage) {
        if (lane == 0)
          for (int c = 0; c < chunks; ++c) {
            const int s = stage;
            const int held = p.wide / kBlocks;        // columns of B in this block
            stage = s + 1 == stages_of(held) ? 0 : s + 1;
            if ((used >> s & 1u) && !tc::mbar_wait(&bar->empty[s], (parity >> s & 1u) ^ 1u, abort, a.limit)) break;
            used |= 1u << s, parity ^= 1u << s;
            if (rank == 0) tc::mbar_arrive_expect_tx(&bar->full[s], kBlocks * stage_bytes(held));
            uint8_t* to = smem + s * stage_bytes(held);
            auto load = [&](void* dst, const CUtensorMap* map, int x, int y, int z) {
              if constexpr (PAIR) tma_load_pair(dst, map, x, y, z, tc::mapa(tc::smem_u32(&bar->full[s]), 0));
              else tma_load_3d(dst, map, x, y, z, &bar->full[s]);
            };
            const int kk = c * kBK;
#pragma unroll
            for (int piece = 0; piece < 2; ++piece) {
              const int z = l + piece * a.L;
              if (p.a_mn) {
                load(to, A, m0, kk, z);
                load(to + 8192, A, m0 + 64, kk, z);
              } else {
                load(to, A, kk, m0, z);
              }
              to += kA;
            }
#pragma unroll
            for (int piece = 0; piece < 2; ++piece) {
              const int z = l + piece * a.L;
              if (p.b_mn) {
#pragma unroll
                for (int j = 0; j < BN; j += 64)
                  if (j < held) load(to + j * 128, B, n0 + rank * held + j, kk, z);
              } else {
#pragma unroll
                for (int j = 0; j < BN; j += 128)
                  if (j < held) load(to + j * 128, B, kk, n0 + rank * held + j, z);
              }
              to += held * 128;
            }
          }
        __syncwarp();
      });
    } else {
      all_tiles([&](const Product& p, const CUtensorMap*, const CUtensorMap*, int chunks, int, int, int, int, int& stage) {
        if (warp != kIssuer || rank) return;
        if (lane == 0) {
          const uint32_t id = idesc_f16(p.a_mn, p.b_mn, kHigh, p.wide);
          // 16 of K: 32 bytes along a row, or 16 rows of 128 bytes
          const uint32_t da = p.a_mn ? 2048 : 32, db = p.b_mn ? 2048 : 32, la = p.a_mn ? 8192 : 16, lb = p.b_mn ? 8192 : 16;
          for (int c = 0; c < chunks; ++c, ++chunk) {
            const int s = stage, held = p.wide / kBlocks;
            stage = s + 1 == stages_of(held) ? 0 : s + 1;
            const uint32_t buf = chunk & 1u, to = tmem + buf * BN;
            if (chunk >= 2 && !tc::mbar_wait(&bar->taken[buf], (chunk / 2 - 1) & 1u, abort, a.limit)) break;
            if (!tc::mbar_wait(&bar->full[s], parity >> s & 1u, abort, a.limit)) break;
            parity ^= 1u << s;
            tc::tc_fence_after();
            const uint32_t a0 = tc::smem_u32(smem + s * stage_bytes(held)), b0 = a0 + 2 * kA, next_b = held * 128;
            // the small products first: what the sum of the large ones is rounded by does not grow with them
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              const uint64_t ah = tile_desc(a0 + kk * da, la, 1024), al = tile_desc(a0 + kA + kk * da, la, 1024);
              const uint64_t bh = tile_desc(b0 + kk * db, lb, 1024), bl = tile_desc(b0 + next_b + kk * db, lb, 1024);
              mma<PAIR>(to, al, bh, id, kk > 0);
              mma<PAIR>(to, ah, bl, id, 1u);
            }
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma<PAIR>(to, tile_desc(a0 + kk * da, la, 1024), tile_desc(b0 + kk * db, lb, 1024), id, 1u);
            commit<PAIR>(&bar->empty[s]);
            commit<PAIR>(&bar->sums[buf]);
          }
        }
        __syncwarp();
      });
    }
  }
  // on the way out after a wait that gave up: nothing may land when the block has left
  if (warp == kIssuer && lane == 0) {
    if (rank == 0) commit<PAIR>(&bar->drained);
    wait_landed(&bar->drained, 0);
  }
  if (warp == kProducer && lane == 0 && *abort && rank == 0)     // those of both blocks signal here
    for (int s = 0; s < 3; ++s)
      if (used >> s & 1u) wait_landed(&bar->full[s], (parity >> s & 1u) ^ 1u);
  tc::tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) tc::cluster_sync();    // neither leaves while the other's memory is asked for
  if (tid == 0 && bar->abort) *a.error = AUV_ERR_TIMEOUT;
  if (warp < kStorers && bar->abort) {
    const Product p = {kLast, a.M, a.N, a.s, kHigh, a.tile[2], false, a.wide};
    const int each = tiles_of(kLast, a.M, a.N, kHigh, p.wide);
    for (int64_t t = blockIdx.x / kBlocks; t < (int64_t)each * a.L; t += gridDim.x / kBlocks) {
      int ti, tj;
      tile_at(p, (int)(t % each), ti, tj);
      const int l = (int)(t / each), m0 = ti * kHigh + rank * kBM, n0 = tj * p.wide;
      if (a.dtype == NET_FP32) spoil<float>(a, l, m0, n0, p.wide);
      else if (a.dtype == NET_BF16) spoil<__nv_bfloat16>(a, l, m0, n0, p.wide);
      else spoil<__half>(a, l, m0, n0, p.wide);
    }
  }
  if (warp == kIssuer) {
    tc::tc_fence_after();
    dealloc<PAIR>(tmem, 2 * BN);
  }
}

// ---------------------------------------------------------------- host side
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
  static EncodeFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeFn>(p);
    else
      cudaGetLastError();
  });
  return fn;
}

// Pieces [2 L][rows][ld], boxes of 64 columns x `box` rows.
bool make_map(CUtensorMap* map, const __half* at, int64_t cols, int64_t rows, int64_t ld, int64_t L, uint32_t box) {
  const EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)(2 * L)};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)(ld * rows) * 2};
  const cuuint32_t boxes[3] = {kBK, box, 1}, ones[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(at), dims, strides, boxes, ones,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Space {
  int64_t s, ldx, lds;          // shorter side; elements between rows of X, and of P and Q
  int blocks;                   // of a matrix's sum of squares
  size_t x[2], p, q, partial, bytes;
};
Space space(const net_ortho* a) {
  Space z;
  z.s = std::min(a->M, a->N);
  z.ldx = (a->N + 7) / 8 * 8, z.lds = (z.s + 7) / 8 * 8;
  const int64_t want = std::max<int64_t>(1, (int64_t)sm_count() * 4 / a->L);
  z.blocks = (int)std::max<int64_t>(1, std::min(want, a->M * a->N / (kNormThreads * 8)));
  size_t n = 256;               // the error word
  auto part = [&](size_t bytes) {
    const size_t at = n;
    n += (bytes + 255) / 256 * 256;
    return at;
  };
  z.partial = part((size_t)a->L * z.blocks * 3 * sizeof(float));
  const bool any = a->steps > 0;
  const size_t x = any ? (size_t)2 * a->L * a->M * z.ldx * 2 : 0, p = any ? (size_t)2 * a->L * z.s * z.lds * 2 : 0;
  z.x[0] = part(x), z.x[1] = part(a->steps > 1 ? x : 0), z.p = part(p), z.q = part(p);
  z.bytes = n;
  return z;
}

// The largest |a v + b v^3 + c v^5| of v in [0, top].
double highest(const float* k, double top) {
  auto at = [&](double v) { return std::fabs(v * (k[0] + v * v * (k[1] + v * v * k[2]))); };
  double most = at(top);
  const double A = 5.0 * k[2], B = 3.0 * k[1], C = k[0], disc = B * B - 4 * A * C;
  double w[2] = {A == 0.0 ? (B == 0.0 ? -1.0 : -C / B) : -1.0, -1.0};
  if (A != 0.0 && disc >= 0.0) w[0] = (-B + std::sqrt(disc)) / (2 * A), w[1] = (-B - std::sqrt(disc)) / (2 * A);
  for (double q : w)
    if (q > 0.0 && q < top * top) most = std::max(most, at(std::sqrt(q)));
  return most;
}

int check(const net_ortho* p) {
  if (!p) return fail(AUV_ERR_INVALID, "argument block is NULL");
  if (p->struct_size != sizeof(net_ortho))
    return fail(AUV_ERR_INVALID, "struct_size %u, expected %zu", p->struct_size, sizeof(net_ortho));
  if (p->dtype > NET_FP16) return fail(AUV_ERR_INVALID, "dtype %u unknown", p->dtype);
  if (p->reserved) return fail(AUV_ERR_INVALID, "reserved is not 0");
  if (p->steps > 64) return fail(AUV_ERR_INVALID, "more than 64 steps");
  if (!(p->eps >= 0.0f) || std::isinf(p->eps)) return fail(AUV_ERR_INVALID, "eps is no number from 0 on");
  for (float c : p->coef)
    if (!std::isfinite(c)) return fail(AUV_ERR_INVALID, "coef is not finite");
  if (p->L < 0 || p->M < 0 || p->N < 0) return fail(AUV_ERR_INVALID, "negative size");
  const int64_t most = 1 << 20, all = (int64_t)1 << 36;
  if (p->L > 65535 || p->M > most || p->N > most || std::min(p->M, p->N) > (1 << 15) || (p->L && p->M * p->N > all / p->L))
    return fail(AUV_ERR_UNSUPPORTED, "L past 65535, a side past 2^20, the shorter past 2^15, or L * M * N past 2^36");
  double top = 1.0;
  for (uint32_t k = 0; k < p->steps; ++k) {
    const double q = std::fabs(p->coef[0]) + std::fabs(p->coef[1]) * top * top + std::fabs(p->coef[2]) * top * top * top * top;
    top = highest(p->coef, top * 1.001);
    if (!(q <= 1000.0) || !(top <= 8.0))
      return fail(AUV_ERR_UNSUPPORTED, "coef takes singular values past 8, or its terms past 1000, in step %u", k);
  }
  return AUV_OK;
}

template <int BN, bool PAIR>
cudaError_t launch_products(const Steps& a, cudaStream_t s) {
  const auto kern = k_products<BN, PAIR>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != cudaSuccess) return e;
  // the blocks wait for each other: all of them, one an SM, or none; no more than the largest product has tiles
  const int blocks = PAIR ? 2 : 1, high = blocks * kBM;
  const int64_t tiles =
      (int64_t)std::max(tiles_of(kX, a.M, a.N, high, a.tile[2]), tiles_of(kP, a.s, a.s, high, std::min(a.tile[0], a.tile[1]))) * a.L;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(std::min<int64_t>(sm_count() / blocks, std::max<int64_t>(1, tiles)) * blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = blocks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = PAIR ? 2 : 1;
  if (PAIR) {                                // as many pairs as the device holds at a time: an SM may lie apart
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) cudaGetLastError();
    if (n < 1) return cudaErrorInvalidConfiguration;
    cfg.gridDim.x = std::min<unsigned>(cfg.gridDim.x, 2u * (unsigned)n);
  }
  return cudaLaunchKernelEx(&cfg, kern, a);
}

template <typename T>
cudaError_t launch(const net_ortho* a, const Space& z, int stuck, uint64_t limit, cudaStream_t s) {
  char* const ws = static_cast<char*>(a->workspace);
  float* const partial = reinterpret_cast<float*>(ws + z.partial);
  __half* const x[2] = {reinterpret_cast<__half*>(ws + z.x[0]), reinterpret_cast<__half*>(ws + z.x[1])};
  __half* const P = reinterpret_cast<__half*>(ws + z.p);
  __half* const Q = reinterpret_cast<__half*>(ws + z.q);
  const dim3 grid((unsigned)z.blocks, (unsigned)a->L);
  k_squares<T><<<grid, kNormThreads, 0, s>>>(a->x, a->M, a->N, partial, reinterpret_cast<int*>(ws));
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  if (a->steps == 0)
    return launch_after(k_scaled<T, false>, grid, kNormThreads, 0, s, a->x, a->M, a->N, a->L, partial, z.blocks, a->eps, nullptr,
                        (int64_t)0, a->y);
  e = launch_after(k_scaled<T, true>, grid, kNormThreads, 0, s, a->x, a->M, a->N, a->L, partial, z.blocks, a->eps, x[0], z.ldx, a->y);
  if (e != cudaSuccess) return e;
  Steps p = {};
  p.L = (int)a->L, p.M = (int)a->M, p.N = (int)a->N, p.s = (int)z.s, p.steps = (int)a->steps, p.ldx = (int)z.ldx, p.lds = (int)z.lds;
  p.wide = a->M <= a->N;
  p.a = a->coef[0], p.b = a->coef[1], p.c = a->coef[2];
  p.x[0] = x[0], p.x[1] = x[1], p.P = P, p.Q = Q;
  p.y = a->y, p.dtype = (int)a->dtype;
  p.error = reinterpret_cast<int*>(ws), p.arrived = reinterpret_cast<unsigned*>(ws) + 1;
  p.limit = limit, p.stuck = stuck;
  bool ok = make_map(&p.p, P, z.s, z.s, z.lds, a->L, kBM) && make_map(&p.q, Q, z.s, z.s, z.lds, a->L, kBM);
  for (int i = 0; i < 2 && ok; ++i) {
    const __half* const at = x[a->steps > 1 ? i : 0];
    ok = make_map(&p.x_rows[i], at, a->N, a->M, z.ldx, a->L, kBM) && make_map(&p.x_cols[i], at, a->N, a->M, z.ldx, a->L, kBK);
  }
  if (!ok) return cudaErrorInvalidValue;
  // Tiles: 128 x 256 read less of shared memory for a product than 128 x 128 (64 of K: 1.3 us of an SM, 0.7) and take longer to
  // store (4.5 us, 2.5), pairs of blocks on 256 x 256 read less still (1.0 us for both); the larger, the fewer and coarser are the
  // rounds over the SMs.  Of one form all three products of a step are, wide or narrow is each.
  const int kinds[3] = {kP, kQ, kX};
  double alone = 0.0, paired = 0.0;
  for (int k = 0; k < 3; ++k) {
    const int K = k == 0 ? std::max(p.M, p.N) : p.s, rows = k < 2 ? p.s : p.M, cols = k < 2 ? p.s : p.N;
    auto time = [&](int high, int wide, double chunk, double store) {
      const int64_t at_once = sm_count() / (high / kBM);
      const int64_t rounds = ((int64_t)tiles_of(kinds[k], rows, cols, high, wide) * p.L + at_once - 1) / at_once;
      return (double)rounds * ((K + kBK - 1) / kBK * chunk + store);
    };
    const double wide = time(kBM, 256, 1.3, 4.5), narrow = time(kBM, 128, 0.7, 2.5);
    p.tile[k] = wide < narrow ? 256 : 128;
    alone += std::min(wide, narrow);
    paired += time(2 * kBM, 256, 1.0, 4.5);
  }
  if (paired < alone) {
    p.tile[0] = p.tile[1] = p.tile[2] = 256;
    return launch_products<256, true>(p, s);
  }
  p.single = p.M <= 128 && p.N <= 128;
  if (p.single) p.tile[0] = p.tile[1] = p.tile[2] = 128;
  return p.tile[0] + p.tile[1] + p.tile[2] > 3 * 128 ? launch_products<256, false>(p, s) : launch_products<128, false>(p, s);
}

int run(const net_ortho* p, void* stream, int stuck = 0, uint64_t limit = kWaitLimitNs) {
  int rc = check(p);
  if (rc) return rc;
  if (!p->L || !p->M || !p->N) return AUV_OK;
  const int z = type_size(p->dtype);
  if ((rc = need_rows(p->x, "x", p->L, p->M, p->N, z, false)) || (rc = need_rows(p->y, "y", p->L, p->M, p->N, z, true))) return rc;
  const Space w = space(p);
  if (p->workspace_bytes < w.bytes) return fail(AUV_ERR_SIZE, "workspace of %zu bytes, %zu needed", p->workspace_bytes, w.bytes);
  if ((rc = need(p->workspace, "workspace", 256))) return rc;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p->dtype == NET_FP32   ? launch<float>(p, w, stuck, limit, s)
                        : p->dtype == NET_BF16 ? launch<__nv_bfloat16>(p, w, stuck, limit, s)
                                               : launch<__half>(p, w, stuck, limit, s);
  return e == cudaSuccess ? AUV_OK : cuda_fail(e, "net_orthogonalise");
}

}  // namespace
}  // namespace net
}  // namespace auv

extern "C" {

size_t net_orthogonalise_workspace_bytes(const net_ortho* a) {
  using namespace auv::net;
  return !a || check(a) || !a->L || !a->M || !a->N ? 0 : space(a).bytes;
}

int net_orthogonalise(const net_ortho* a, void* stream) { return auv::net::run(a, stream); }

int net_orthogonalise_selftest_timeout(const net_ortho* a, uint32_t product, uint32_t limit_us, void* stream) {
  using namespace auv::net;
  const int rc = check(a);
  if (rc) return rc;
  if (product < 1 || product >= a->steps * 3) return fail(AUV_ERR_INVALID, "product %u: not from 1 on and ahead of the last", product);
  if (limit_us < 1 || limit_us > 5000000) return fail(AUV_ERR_INVALID, "limit_us outside [1, 5e6]");
  return run(a, stream, (int)product, limit_us * 1000ull);
}

}  // extern "C"
