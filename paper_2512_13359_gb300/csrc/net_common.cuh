// net_common.cuh -- what the network operators (net_scan.cu, net_norm.cu, net_drop.cu) share: moves of a thread's
// channels between memory and fp32 registers, the gate function, and the checks of an argument block.
#pragma once

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <type_traits>

#include "auvenv.h"
#include "auvnet.h"

namespace auv {
namespace net {

// A thread's piece of a row in memory: E channels of type T in one access.
template <int BYTES> struct Word;
template <> struct Word<2> { using type = uint16_t; };
template <> struct Word<4> { using type = uint32_t; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<16> { using type = uint4; };

template <typename T, int E> using Raw = typename Word<(int)sizeof(T) * E>::type;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_float(float x, float& r) { r = x; }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16& r) { r = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_float(float x, __half& r) { r = __float2half_rn(x); }

// Pairs of 16-bit values by words: a shift and a mask, or one conversion, for two.
template <typename T>
__device__ __forceinline__ void unpack_pair(uint32_t w, float& lo, float& hi) {
  if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
  } else {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    lo = f.x, hi = f.y;
  }
}
template <typename T>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}

template <typename T, int E>
__device__ __forceinline__ void unpack(const Raw<T, E>& w, float (&x)[E]) {
  union { Raw<T, E> w; T t[E]; uint32_t u[(sizeof(T) * E + 3) / 4]; } v;
  v.w = w;
  if constexpr (sizeof(T) == 4 || E == 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = to_float(v.t[e]);
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 2) unpack_pair<T>(v.u[e / 2], x[e], x[e + 1]);
  }
}

template <typename T, int E>
__device__ __forceinline__ Raw<T, E> pack(const float (&x)[E]) {
  union U { Raw<T, E> w; T t[E]; uint32_t u[(sizeof(T) * E + 3) / 4]; __device__ U() {} } v;
  if constexpr (sizeof(T) == 4 || E == 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) from_float(x[e], v.t[e]);
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 2) v.u[e / 2] = pack_pair<T>(x[e], x[e + 1]);
  }
  return v.w;
}

template <typename T, int E>
__device__ __forceinline__ void load(const T* p, float (&x)[E]) {
  unpack<T, E>(*reinterpret_cast<const Raw<T, E>*>(p), x);
}

template <typename T, int E>
__device__ __forceinline__ void store(T* p, const float (&x)[E]) {
  *reinterpret_cast<Raw<T, E>*>(p) = pack<T, E>(x);
}

// sigmoid(x) and sigmoid(-x) from q = exp(-|x|), taken as 2^(-|x| log2 e): 1 / (1 + q) and q / (1 + q), neither of them
// 1 - the other, which has no digits left where the gate is nearly shut.  The product with log2 e is rounded, so q, and
// with it the smaller gate, is off by up to 2^-24 (|x| + 12) of itself; below 2^-126 it is 0.  The larger is right to a
// few units of 2^-24.  Eight instructions.
__device__ __forceinline__ void gates(float x, float& a, float& b) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(x) * -1.44269504088896341f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  const float q = e * r;
  a = x >= 0.0f ? r : q;
  b = x >= 0.0f ? q : r;
}

template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(d), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Two-byte pieces (odd widths or strides of 16-bit types) have no asynchronous copy.
template <typename T, int E> constexpr bool kAsync = sizeof(T) * E >= 4;

// Kernels of one call follow each other closely: the next one's blocks are set up while the last of the one before run,
// and wait here for its stores.
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... A>
cudaError_t launch_after(void (*kern)(P...), dim3 grid, int threads, int smem, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}

// ---------------------------------------------------------------- host side
int fail(int code, const char* fmt, ...);
int cuda_fail(cudaError_t e, const char* what);
// Device memory of the current device, aligned to `align`.
int need(const void* p, const char* name, size_t align);
// The same for rows (ni x nj rows of nk elements of `size` bytes): strides not
// negative; of an output, no two rows on the same memory.
int need_rows(const net_rows& r, const char* name, int64_t ni, int64_t nj, int64_t nk, int size, bool output);
int sm_count();

// Whether every access of E channels of r is aligned.
inline bool aligned(const net_rows& r, int64_t ni, int64_t nj, int size, int e) {
  return reinterpret_cast<uintptr_t>(r.data) % ((size_t)size * e) == 0 && (ni <= 1 || r.outer % e == 0) &&
         (nj <= 1 || r.inner % e == 0);
}

inline int type_size(uint32_t dtype) { return dtype == NET_FP32 ? 4 : 2; }

}  // namespace net
}  // namespace auv
