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
// One block computes a 128 x 128 or 128 x 256 tile: a producer thread streams 128-byte-swizzled tiles of both pieces of
// both operands into a ring with TMA, one thread issues tcgen05.mma into tensor memory, and eight warps read the sums back,
// split them into pieces again and store them; of the symmetric products the tiles on and below the diagonal, stored on
// both sides of it.  The products of a call follow each other by programmatic launches.
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

struct Product {
  int rows, cols, K, L;       // of the result; contraction; matrices
  int kind, tiles_n;
  float b, c, a;              // kQ
  __half* out;                // pieces [2][L][rows][ld]
  const __half* prev;         // kQ: P
  int ld;
  net_rows y;                 // kLast
  int dtype;
  int* error;
};

// ---- sums of squares ----
// Of x, and of x times 2^64 and 2^-64: one of the three is in range wherever the largest |x| is.
constexpr float kUp = 18446744073709551616.0f, kDown = 1.0f / 18446744073709551616.0f;
constexpr int kNormThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kNormThreads) k_squares(net_rows x, int64_t M, int64_t N, float* partial, int* error) {
  __shared__ float part[3][kNormThreads / 32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *error = AUV_OK;
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

// 1 / (|x| + eps) as two factors, from the blocks' sums (every thread of a block; fixed order).
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
  if (s[0] >= 1e30f) return make_float2(kDown, 1.0f / (sqrtf(s[2]) + eps * kDown));     // also infinite sums; NaN falls through
  if (s[0] < 1e-30f) return make_float2(kUp, 1.0f / (sqrtf(s[1]) + eps * kUp));
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
__device__ __forceinline__ void wait_landed(uint64_t* b, uint32_t phase) {
  const uint64_t t0 = tc::global_timer_ns();
  while (!tc::mbar_test(b, phase) && tc::global_timer_ns() - t0 < kWaitLimitNs) {
  }
}

template <int BN>
struct Tile {
  static constexpr int kStages = BN > 128 ? 2 : 3;
  static constexpr uint32_t kA = kBM * 128, kB = BN * 128;      // one piece of a stage
  static constexpr uint32_t kStage = 2 * (kA + kB);
  static constexpr uint32_t kSmem = kStages * kStage + 256 + 1024;
};
struct Bars {
  uint64_t full[3], empty[3], sums;
  uint32_t tmem;
  int abort;
};
constexpr int kEpilogue = 8, kProducer = 8, kIssuer = 9, kThreads = 320;

// 32 scaled values of row r from column c on, as pieces (whole 16-byte stores; a row's padding may be written).
__device__ __forceinline__ void store_pieces(const Product& p, int64_t l, int r, int c, const float (&v)[32], bool mirror) {
  const int64_t each = (int64_t)p.L * p.rows * p.ld;
  __half* const hi = p.out + (l * p.rows + r) * (int64_t)p.ld + c;
  uint32_t h[16], o[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const __half2 w = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    const float2 f = __half22float2(w);
    const __half2 z = __floats2half2_rn(v[2 * i] - f.x, v[2 * i + 1] - f.y);
    h[i] = *reinterpret_cast<const uint32_t*>(&w);
    o[i] = *reinterpret_cast<const uint32_t*>(&z);
  }
  if (r < p.rows) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + 8 * i < p.cols) {
        *reinterpret_cast<uint4*>(hi + 8 * i) = make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
        *reinterpret_cast<uint4*>(hi + each + 8 * i) = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
      }
    if (mirror) {                        // the lanes' rows are next to each other
      uint16_t* const to = reinterpret_cast<uint16_t*>(p.out) + (l * p.rows + c) * (int64_t)p.ld + r;
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (c + i < p.cols) {
          to[i * (int64_t)p.ld] = (uint16_t)(i & 1 ? h[i / 2] >> 16 : h[i / 2]);
          to[i * (int64_t)p.ld + each] = (uint16_t)(i & 1 ? o[i / 2] >> 16 : o[i / 2]);
        }
    }
  }
}

template <bool A_MN, bool B_MN, int BN>
__global__ void __launch_bounds__(kThreads, 1)
k_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, Product p) {
  using TL = Tile<BN>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023u) & ~(uintptr_t)1023u);
  Bars* const bar = reinterpret_cast<Bars*>(smem + TL::kStages * TL::kStage);
  volatile int* const abort = &bar->abort;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  int ti, tj;
  if (p.kind == kP || p.kind == kQ) {    // tiles on and below the diagonal
    const int t = blockIdx.x;
    ti = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while (ti * (ti + 1) / 2 > t) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
    tj = t - ti * (ti + 1) / 2;
  } else {
    ti = blockIdx.x / p.tiles_n, tj = blockIdx.x % p.tiles_n;
  }
  const int m0 = ti * kBM, n0 = tj * BN, l = blockIdx.y;
  const int chunks = (p.K + kBK - 1) / kBK;
  if (tid == 0) {
    for (int s = 0; s < TL::kStages; ++s) {
      tc::mbar_init(&bar->full[s], 1);
      tc::mbar_init(&bar->empty[s], 1);
    }
    tc::mbar_init(&bar->sums, 1);
    bar->abort = 0;
    tc::mbar_fence_init();
  }
  if (warp == kIssuer) {
    tc::tmem_alloc(&bar->tmem, BN);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  after_previous();
  const uint32_t tmem = bar->tmem;

  if (warp == kProducer) {
    if (lane == 0) {
      int c = 0;
      for (; c < chunks; ++c) {
        const int s = c % TL::kStages;
        if (c >= TL::kStages && !tc::mbar_wait(&bar->empty[s], (uint32_t)(c / TL::kStages - 1) & 1u, abort, kWaitLimitNs)) break;
        tc::mbar_arrive_expect_tx(&bar->full[s], TL::kStage);
        uint8_t* to = smem + s * TL::kStage;
        const int k = c * kBK;
#pragma unroll
        for (int piece = 0; piece < 2; ++piece) {
          const int z = l + piece * p.L;
          if (A_MN) {
            tma_load_3d(to, &map_a, m0, k, z, &bar->full[s]);
            tma_load_3d(to + 8192, &map_a, m0 + 64, k, z, &bar->full[s]);
          } else {
            tma_load_3d(to, &map_a, k, m0, z, &bar->full[s]);
          }
          to += TL::kA;
        }
#pragma unroll
        for (int piece = 0; piece < 2; ++piece) {
          const int z = l + piece * p.L;
#pragma unroll
          for (int j = 0; j < BN; j += B_MN ? 64 : 128) {
            if (B_MN) tma_load_3d(to + j * 128, &map_b, n0 + j, k, z, &bar->full[s]);
            else tma_load_3d(to + j * 128, &map_b, k, n0 + j, z, &bar->full[s]);
          }
          to += TL::kB;
        }
      }
      if (*abort)                        // the copies still in flight
        for (int s = 0; s < TL::kStages; ++s) {
          const int fills = c / TL::kStages + (s < c % TL::kStages ? 1 : 0);
          if (fills > 0) wait_landed(&bar->full[s], (uint32_t)(fills - 1) & 1u);
        }
    }
    __syncwarp();
  } else if (warp == kIssuer) {
    if (lane == 0) {
      constexpr uint32_t kId = idesc_f16(A_MN, B_MN, kBM, BN);
      for (int c = 0; c < chunks; ++c) {
        const int s = c % TL::kStages;
        if (!tc::mbar_wait(&bar->full[s], (uint32_t)(c / TL::kStages) & 1u, abort, kWaitLimitNs)) break;
        tc::tc_fence_after();
        const uint32_t a0 = tc::smem_u32(smem + s * TL::kStage), b0 = a0 + 2 * TL::kA;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          // 16 of K: 32 bytes along a row, or 16 rows of 128 bytes
          const uint32_t da = A_MN ? kk * 2048 : kk * 32, db = B_MN ? kk * 2048 : kk * 32;
          const uint32_t la = A_MN ? 8192 : 16, lb = B_MN ? 8192 : 16;
          const uint64_t ah = tile_desc(a0 + da, la, 1024), al = tile_desc(a0 + TL::kA + da, la, 1024);
          const uint64_t bh = tile_desc(b0 + db, lb, 1024), bl = tile_desc(b0 + TL::kB + db, lb, 1024);
          tc::mma_ss(tmem, al, bh, kId, c > 0 || kk > 0);
          tc::mma_ss(tmem, ah, bl, kId, 1u);
          tc::mma_ss(tmem, ah, bh, kId, 1u);
        }
        tc::mma_commit(&bar->empty[s]);
      }
      tc::mma_commit(&bar->sums);
      wait_landed(&bar->sums, 0);        // tensor memory is freed below
    }
    __syncwarp();
  } else {
    const bool ok = tc::mbar_wait(&bar->sums, 0, abort, kWaitLimitNs);
    tc::tc_fence_after();
    const int row = m0 + warp % 4 * 32 + lane;
    const uint32_t from = tmem + ((uint32_t)(warp % 4 * 32) << 16);
    float* const turn = reinterpret_cast<float*>(smem) + warp * 32 * 33;   // the ring is done with
#pragma unroll 1
    for (int j = warp / 4 * 32; j < BN; j += 64) {
      const int col = n0 + j;
      if (col >= p.cols) break;
      uint32_t acc[32];
      tc::tmem_ld32(from + j, acc);
      tc::tmem_ld_wait(acc);
      float v[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = ok ? __uint_as_float(acc[i]) : __uint_as_float(0x7fc00000u);
      if (p.kind == kP) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= kScaleP / (kScaleX * kScaleX);
        store_pieces(p, l, row, col, v, ti != tj);
      } else if (p.kind == kQ) {
        const float fc = p.c * (kScaleQ / (kScaleP * kScaleP)), fb = p.b * (kScaleQ / kScaleP);
        const int64_t each = (int64_t)p.L * p.rows * p.ld;
        const __half* const prev = p.prev + ((int64_t)l * p.rows + row) * p.ld + col;
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          uint4 h = make_uint4(0, 0, 0, 0), o = h;
          if (row < p.rows && col + i < p.cols) {
            h = *reinterpret_cast<const uint4*>(prev + i);
            o = *reinterpret_cast<const uint4*>(prev + each + i);
          }
          float hf[8], of[8];
          unpack<__half, 8>(h, hf);
          unpack<__half, 8>(o, of);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            v[i + e] = fmaf(fc, v[i + e], fmaf(fb, hf[e], fb * of[e])) + (col + i + e == row ? p.a * kScaleQ : 0.0f);
        }
        store_pieces(p, l, row, col, v, ti != tj);
      } else if (p.kind == kX) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= 1.0f / kScaleQ;
        store_pieces(p, l, row, col, v, false);
      } else {                           // y's rows start anywhere: turned, the warp stores a row's values together
#pragma unroll
        for (int i = 0; i < 32; ++i) turn[lane * 33 + i] = v[i] * (1.0f / (kScaleQ * kScaleX));
        __syncwarp();
        const int r0 = m0 + warp % 4 * 32;
        if (col + lane < p.cols)
          for (int i = 0; i < 32 && r0 + i < p.rows; ++i) {
            const float w = turn[i * 33 + lane];
            const int64_t at = l * p.y.outer + (r0 + i) * p.y.inner + col + lane;
            if (p.dtype == NET_FP32) reinterpret_cast<float*>(p.y.data)[at] = w;
            else if (p.dtype == NET_BF16) from_float(w, reinterpret_cast<__nv_bfloat16*>(p.y.data)[at]);
            else from_float(w, reinterpret_cast<__half*>(p.y.data)[at]);
          }
        __syncwarp();
      }
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (tid == 0 && bar->abort) *p.error = AUV_ERR_TIMEOUT;
  if (warp == kIssuer) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, BN);
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

template <bool A_MN, bool B_MN, int BN>
cudaError_t launch_product(const CUtensorMap& A, const CUtensorMap& B, Product& p, cudaStream_t s) {
  const auto kern = k_product<A_MN, B_MN, BN>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Tile<BN>::kSmem);
  if (e != cudaSuccess) return e;
  const int64_t tm = (p.rows + kBM - 1) / kBM;
  p.tiles_n = (p.cols + BN - 1) / BN;
  const int64_t tiles = p.kind == kP || p.kind == kQ ? tm * (tm + 1) / 2 : tm * p.tiles_n;
  return launch_after(kern, dim3((unsigned)tiles, (unsigned)p.L), kThreads, Tile<BN>::kSmem, s, A, B, p);
}

template <typename T>
cudaError_t launch(const net_ortho* a, const Space& z, cudaStream_t s) {
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
  const bool wide = a->M <= a->N;
  CUtensorMap rows[2], cols[2], pm, qm;            // of x, read by rows and along columns
  bool ok = make_map(&pm, P, z.s, z.s, z.lds, a->L, kBM) && make_map(&qm, Q, z.s, z.s, z.lds, a->L, kBM);
  for (int i = 0; i < 2 && ok; ++i) {
    const __half* const at = x[a->steps > 1 ? i : 0];
    ok = make_map(&rows[i], at, a->N, a->M, z.ldx, a->L, kBM) && make_map(&cols[i], at, a->N, a->M, z.ldx, a->L, kBK);
  }
  if (!ok) return cudaErrorInvalidValue;
  Product p = {};
  p.L = (int)a->L;
  p.a = a->coef[0], p.b = a->coef[1], p.c = a->coef[2];
  p.error = reinterpret_cast<int*>(ws);
  p.y = a->y, p.dtype = (int)a->dtype;
  for (uint32_t k = 0; k < a->steps; ++k) {
    const int i = k & 1;
    p.kind = kP, p.rows = p.cols = (int)z.s, p.K = (int)std::max(a->M, a->N), p.out = P, p.ld = (int)z.lds;
    e = wide ? launch_product<false, false, 128>(rows[i], rows[i], p, s) : launch_product<true, true, 128>(cols[i], cols[i], p, s);
    if (e != cudaSuccess) return e;
    p.kind = kQ, p.K = (int)z.s, p.out = Q, p.prev = P;
    if ((e = launch_product<false, false, 128>(pm, pm, p, s)) != cudaSuccess) return e;
    p.kind = k + 1 == a->steps ? kLast : kX, p.rows = (int)a->M, p.cols = (int)a->N, p.out = x[i ^ 1], p.ld = (int)z.ldx;
    // wide tiles where they still fill the device
    const bool large = ((a->M + 127) / 128) * ((a->N + 255) / 256) * a->L >= sm_count();
    if (wide) e = large ? launch_product<false, true, 256>(qm, cols[i], p, s) : launch_product<false, true, 128>(qm, cols[i], p, s);
    else e = large ? launch_product<false, false, 256>(rows[i], qm, p, s) : launch_product<false, false, 128>(rows[i], qm, p, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

int run(const net_ortho* p, void* stream) {
  int rc = check(p);
  if (rc) return rc;
  if (!p->L || !p->M || !p->N) return AUV_OK;
  const int z = type_size(p->dtype);
  if ((rc = need_rows(p->x, "x", p->L, p->M, p->N, z, false)) || (rc = need_rows(p->y, "y", p->L, p->M, p->N, z, true))) return rc;
  const Space w = space(p);
  if (p->workspace_bytes < w.bytes) return fail(AUV_ERR_SIZE, "workspace of %zu bytes, %zu needed", p->workspace_bytes, w.bytes);
  if ((rc = need(p->workspace, "workspace", 256))) return rc;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p->dtype == NET_FP32   ? launch<float>(p, w, s)
                        : p->dtype == NET_BF16 ? launch<__nv_bfloat16>(p, w, s)
                                               : launch<__half>(p, w, s);
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

}  // extern "C"
