// net_norm.cu -- group norm with an activation, channels last (auvnet.h, net_group_norm).
#include "net_common.cuh"

namespace auv {
namespace net {
namespace {

struct Norm {
  int64_t B, S, C, G;
  net_rows x, y, dy, dx;
  const float *gamma, *beta;
  float *mean, *rstd, *dgamma, *dbeta;
  float eps;
  uint32_t act;
};

// act(u) and act'(u); the slope of relu at 0 is 0.
__device__ __forceinline__ float act_value(uint32_t act, float u) {
  if (act == NET_ACT_RELU) return u > 0.0f || u != u ? u : 0.0f;
  if (act == NET_ACT_SILU) {
    float s, r;
    gates(u, s, r);
    return u * s;
  }
  return act == NET_ACT_TANH ? tanhf(u) : u;
}

__device__ __forceinline__ float act_slope(uint32_t act, float u) {
  if (act == NET_ACT_RELU) return u > 0.0f ? 1.0f : 0.0f;
  if (act == NET_ACT_SILU) {
    float s, r;
    gates(u, s, r);
    return s * fmaf(u, r, 1.0f);
  }
  if (act == NET_ACT_TANH) {
    const float t = tanhf(u);
    return fmaf(-t, t, 1.0f);
  }
  return 1.0f;
}

template <typename T>
__device__ __forceinline__ T* at(const net_rows& r, int64_t i, int64_t j, int64_t k) {
  return reinterpret_cast<T*>(r.data) + i * r.outer + j * r.inner + k;
}

constexpr int kThreads = 128;

__device__ float block_sum(float x) {
  __shared__ float part[kThreads / 32];
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = x;
  __syncthreads();
  float s = 0.0f;
  for (int w = 0; w < kThreads / 32; ++w) s += part[w];
  return s;
}

template <typename T>
__device__ __forceinline__ float value(const net_rows& r, int64_t i, int64_t j, int64_t k) {
  return to_float(*at<T>(r, i, j, k));
}

// One group of one instance a block.
template <typename T>
__global__ void k_norm(Norm a) {
  const int64_t W = a.C / a.G, n = a.S * W;
  for (int64_t q = blockIdx.x; q < a.B * a.G; q += gridDim.x) {
    const int64_t b = q / a.G, c0 = q % a.G * W;
    float s = 0.0f;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) s += value<T>(a.x, b, i / W, c0 + i % W);
    const float mean = block_sum(s) / (float)max(n, (int64_t)1);
    s = 0.0f;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) {
      const float d = value<T>(a.x, b, i / W, c0 + i % W) - mean;
      s = fmaf(d, d, s);
    }
    const float rstd = 1.0f / sqrtf(block_sum(s) / (float)max(n, (int64_t)1) + a.eps);
    for (int64_t i = threadIdx.x; i < n; i += kThreads) {
      const int64_t j = i / W, c = c0 + i % W;
      const float xh = (value<T>(a.x, b, j, c) - mean) * rstd;
      from_float(act_value(a.act, fmaf(a.gamma ? a.gamma[c] : 1.0f, xh, a.beta ? a.beta[c] : 0.0f)),
                 *at<T>(a.y, b, j, c));
    }
    if (threadIdx.x == 0) {
      a.mean[q] = mean;
      a.rstd[q] = rstd;
    }
  }
}

template <typename T>
__device__ __forceinline__ void slope_at(const Norm& a, int64_t b, int64_t j, int64_t c, float mean, float rstd,
                                         float& dz, float& xh) {
  xh = (value<T>(a.x, b, j, c) - mean) * rstd;
  dz = value<T>(a.dy, b, j, c) *
       act_slope(a.act, fmaf(a.gamma ? a.gamma[c] : 1.0f, xh, a.beta ? a.beta[c] : 0.0f));
}

template <typename T>
__global__ void k_norm_dx(Norm a) {
  const int64_t W = a.C / a.G, n = a.S * W;
  for (int64_t q = blockIdx.x; q < a.B * a.G; q += gridDim.x) {
    const int64_t b = q / a.G, c0 = q % a.G * W;
    const float mean = a.mean[q], rstd = a.rstd[q];
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) {
      const int64_t c = c0 + i % W;
      float dz, xh;
      slope_at<T>(a, b, i / W, c, mean, rstd, dz, xh);
      const float w = (a.gamma ? a.gamma[c] : 1.0f) * dz;
      s1 += w;
      s2 = fmaf(w, xh, s2);
    }
    s1 = block_sum(s1) / (float)n;
    s2 = block_sum(s2) / (float)n;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) {
      const int64_t j = i / W, c = c0 + i % W;
      float dz, xh;
      slope_at<T>(a, b, j, c, mean, rstd, dz, xh);
      from_float(rstd * ((a.gamma ? a.gamma[c] : 1.0f) * dz - s1 - xh * s2), *at<T>(a.dx, b, j, c));
    }
  }
}

// One channel a block.
template <typename T>
__global__ void k_norm_dparam(Norm a) {
  const int64_t c = blockIdx.x, g = c / (a.C / a.G), n = a.B * a.S;
  float s1 = 0.0f, s2 = 0.0f;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) {
    const int64_t b = i / a.S;
    float dz, xh;
    slope_at<T>(a, b, i % a.S, c, a.mean[b * a.G + g], a.rstd[b * a.G + g], dz, xh);
    s1 += dz;
    s2 = fmaf(dz, xh, s2);
  }
  s1 = block_sum(s1);
  s2 = block_sum(s2);
  if (threadIdx.x == 0) {
    if (a.dbeta) a.dbeta[c] = s1;
    if (a.dgamma) a.dgamma[c] = s2;
  }
}

template <typename T>
cudaError_t launch(const Norm& a, bool back, cudaStream_t s) {
  const int64_t q = a.B * a.G;
  const unsigned blocks = (unsigned)(q < (1 << 30) ? q : (1 << 30));
  if (!back) {
    if (q) k_norm<T><<<blocks, kThreads, 0, s>>>(a);
  } else {
    if (q && a.S) k_norm_dx<T><<<blocks, kThreads, 0, s>>>(a);
    if (a.dgamma || a.dbeta) k_norm_dparam<T><<<(unsigned)a.C, kThreads, 0, s>>>(a);
  }
  return cudaGetLastError();
}

int check(const net_norm* p, bool back) {
  if (!p) return fail(AUV_ERR_INVALID, "argument block is NULL");
  if (p->struct_size != sizeof(net_norm))
    return fail(AUV_ERR_INVALID, "struct_size %u, expected %zu", p->struct_size, sizeof(net_norm));
  if (p->dtype > NET_FP16) return fail(AUV_ERR_INVALID, "dtype %u unknown", p->dtype);
  if (p->act > NET_ACT_TANH) return fail(AUV_ERR_INVALID, "act %u unknown", p->act);
  if (p->B < 0 || p->S < 0 || p->C < 0) return fail(AUV_ERR_INVALID, "negative size");
  if (p->G < 1 || p->C % p->G) return fail(AUV_ERR_INVALID, "G < 1, or C not a multiple of G");
  if (!back && !(p->eps >= 0.0f && p->eps < INFINITY)) return fail(AUV_ERR_INVALID, "eps negative or not finite");
  const int64_t most = (int64_t)1 << 50;
  if (p->C > (1 << 24) || p->G > (1 << 24) || p->B > most || p->S > most || (p->B && p->S > most / p->B))
    return fail(AUV_ERR_UNSUPPORTED, "C or G past 2^24, or B * S past 2^50");
  return AUV_OK;
}

int run(const net_norm* p, bool back, void* stream) {
  int rc = check(p, back);
  if (rc) return rc;
  const int z = type_size(p->dtype);
  if (p->C == 0) return AUV_OK;
  if (p->B && p->S) {
    if ((rc = need_rows(p->x, "x", p->B, p->S, p->C, z, false))) return rc;
    if (!back && (rc = need_rows(p->y, "y", p->B, p->S, p->C, z, true))) return rc;
    if (back && ((rc = need_rows(p->dy, "dy", p->B, p->S, p->C, z, false)) ||
                 (rc = need_rows(p->dx, "dx", p->B, p->S, p->C, z, true))))
      return rc;
  }
  if (p->B && ((rc = need(p->mean, "mean", 4)) || (rc = need(p->rstd, "rstd", 4)))) return rc;
  if ((p->gamma && (rc = need(p->gamma, "gamma", 4))) || (p->beta && (rc = need(p->beta, "beta", 4)))) return rc;
  if (back && ((p->dgamma && (rc = need(p->dgamma, "dgamma", 4))) || (p->dbeta && (rc = need(p->dbeta, "dbeta", 4)))))
    return rc;
  const size_t ws = net_group_norm_workspace_bytes(p, back);
  if (ws) {
    if (p->workspace_bytes < ws)
      return fail(AUV_ERR_SIZE, "workspace of %zu bytes, %zu needed", p->workspace_bytes, ws);
    if ((rc = need(p->workspace, "workspace", 16))) return rc;
  }
  const Norm a = {p->B, p->S, p->C, p->G, p->x, p->y, p->dy, p->dx, p->gamma, p->beta, p->mean, p->rstd,
                  p->dgamma, p->dbeta, p->eps, p->act};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p->dtype == NET_FP32   ? launch<float>(a, back, s)
                        : p->dtype == NET_BF16 ? launch<__nv_bfloat16>(a, back, s)
                                               : launch<__half>(a, back, s);
  return e == cudaSuccess ? AUV_OK : cuda_fail(e, back ? "net_group_norm_backward" : "net_group_norm");
}

}  // namespace
}  // namespace net
}  // namespace auv

extern "C" {

size_t net_group_norm_workspace_bytes(const net_norm* a, int backward) {
  (void)a;
  (void)backward;
  return 0;
}

int net_group_norm(const net_norm* a, void* stream) { return auv::net::run(a, false, stream); }
int net_group_norm_backward(const net_norm* a, void* stream) { return auv::net::run(a, true, stream); }

}  // extern "C"
