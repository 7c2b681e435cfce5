// net_drop.cu -- dropout with a mask drawn from a counter where it is used (auvnet.h, net_dropout).
#include <cmath>

#include "auv_device.cuh"
#include "net_common.cuh"

namespace auv {
namespace net {
namespace {

struct Drop {
  int64_t T, N, D;
  net_rows x, r, y;
  bool shared;
  uint32_t thr;
  float scale;
  uint32_t k0, k1, d0, d1;
};

template <typename T>
__device__ __forceinline__ T* at(const net_rows& r, int64_t t, int64_t n, int64_t d) {
  return reinterpret_cast<T*>(r.data) + t * r.outer + n * r.inner + d;
}

// One element a thread.
template <typename T>
__global__ void k_drop(Drop a) {
  const int64_t total = a.T * a.N * a.D;
  for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t d = i % a.D, row = i / a.D, n = row % a.N, t = row / a.N;
    const uint64_t e = a.shared ? n * a.D + d : i;
    const uint64_t q = e >> 3;
    const uint4 w = philox10((uint32_t)q, (uint32_t)(q >> 32), a.d0, a.d1, a.k0, a.k1);
    const int k = (int)(e & 7);
    const uint32_t word = k < 4 ? (k < 2 ? w.x : w.y) : (k < 6 ? w.z : w.w);
    const uint32_t u = k & 1 ? word >> 16 : word & 0xffffu;
    float o = u < a.thr ? 0.0f : to_float(*at<T>(a.x, t, n, d)) * a.scale;
    if (a.r.data) o += to_float(*at<T>(a.r, t, n, d));
    from_float(o, *at<T>(a.y, t, n, d));
  }
}

template <typename T>
cudaError_t launch(const Drop& a, cudaStream_t s) {
  const int64_t blocks = (a.T * a.N * a.D + 255) / 256;
  k_drop<T><<<(unsigned)(blocks < (1 << 30) ? blocks : (1 << 30)), 256, 0, s>>>(a);
  return cudaGetLastError();
}

int run(const net_drop* p, void* stream) {
  if (!p) return fail(AUV_ERR_INVALID, "argument block is NULL");
  if (p->struct_size != sizeof(net_drop))
    return fail(AUV_ERR_INVALID, "struct_size %u, expected %zu", p->struct_size, sizeof(net_drop));
  if (p->dtype > NET_FP16) return fail(AUV_ERR_INVALID, "dtype %u unknown", p->dtype);
  if (p->shared > 1 || p->reserved) return fail(AUV_ERR_INVALID, "shared not 0 or 1, or reserved not 0");
  if (p->T < 0 || p->N < 0 || p->D < 0) return fail(AUV_ERR_INVALID, "negative size");
  if (!(p->p >= 0.0 && p->p <= 1.0)) return fail(AUV_ERR_INVALID, "p outside [0, 1]");
  const int64_t most = (int64_t)1 << 50;
  if (p->T > most || p->N > most || p->D > most || (p->N && p->D > most / p->N) ||
      (p->T && p->N && p->D && p->N * p->D > most / p->T))
    return fail(AUV_ERR_UNSUPPORTED, "T * N * D past 2^50");
  if (!p->T || !p->N || !p->D) return AUV_OK;
  const int z = type_size(p->dtype);
  int rc;
  if ((rc = need_rows(p->x, "x", p->T, p->N, p->D, z, false)) ||
      (p->residual.data && (rc = need_rows(p->residual, "residual", p->T, p->N, p->D, z, false))) ||
      (rc = need_rows(p->y, "y", p->T, p->N, p->D, z, true)))
    return rc;
  const uint32_t thr = (uint32_t)std::floor(p->p * 65536.0 + 0.5);
  const float scale = thr < 65536 ? (float)(65536.0 / (65536.0 - thr)) : 0.0f;
  const Drop a = {p->T, p->N, p->D, p->x, p->residual, p->y, p->shared != 0, thr, scale,
                  (uint32_t)p->seed, (uint32_t)(p->seed >> 32), (uint32_t)p->draw, (uint32_t)(p->draw >> 32)};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p->dtype == NET_FP32   ? launch<float>(a, s)
                        : p->dtype == NET_BF16 ? launch<__nv_bfloat16>(a, s)
                                               : launch<__half>(a, s);
  return e == cudaSuccess ? AUV_OK : cuda_fail(e, "net_dropout");
}

}  // namespace
}  // namespace net
}  // namespace auv

extern "C" int net_dropout(const net_drop* a, void* stream) { return auv::net::run(a, stream); }
