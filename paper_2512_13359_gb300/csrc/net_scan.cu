// net_scan.cu -- gated linear recurrence along a trajectory (auvnet.h, net_gate_scan): h[t] = a c[t] + (1 - a) v[t],
// a = sigmoid(f[t]), c[t] = h[t - 1] or 0 where an episode ended.
#include "net_common.cuh"

namespace auv {
namespace net {
namespace {

struct Scan {
  int64_t T, N, D;
  net_rows f, v, y, dy, df, dv;
  const float* h0;
  float* hT;
  const float* dhT;
  float* dh0;
  const uint8_t *done, *done_prev;
};

__device__ __forceinline__ bool ended(const Scan& a, int64_t t, int64_t n) {
  const uint8_t* p = t ? (a.done ? a.done + (t - 1) * a.N + n : nullptr) : (a.done_prev ? a.done_prev + n : nullptr);
  return p && *p;
}

template <typename T>
__device__ __forceinline__ T* at(const net_rows& r, int64_t t, int64_t n, int64_t d) {
  return reinterpret_cast<T*>(r.data) + t * r.outer + n * r.inner + d;
}

// One channel of one env a thread, step after step.
template <typename T>
__global__ void k_scan(Scan a) {
  const int64_t m = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  if (m >= a.N * a.D) return;
  const int64_t n = m / a.D, d = m % a.D;
  float h = a.h0 ? a.h0[m] : 0.0f;
  for (int64_t t = 0; t < a.T; ++t) {
    float f[1], v[1], ga, gb;
    load<T, 1>(at<T>(a.f, t, n, d), f);
    load<T, 1>(at<T>(a.v, t, n, d), v);
    gates(f[0], ga, gb);
    if (ended(a, t, n)) h = 0.0f;
    h = fmaf(ga, h, gb * v[0]);
    const float o[1] = {h};
    store<T, 1>(at<T>(a.y, t, n, d), o);
  }
  if (a.hT) a.hT[m] = h;
}

template <typename T>
__global__ void k_scan_back(Scan a) {
  const int64_t m = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
  if (m >= a.N * a.D) return;
  const int64_t n = m / a.D, d = m % a.D;
  float g = a.dhT ? a.dhT[m] : 0.0f;
  for (int64_t t = a.T - 1; t >= 0; --t) {
    float f[1], v[1], dy[1], c[1], ga, gb;
    load<T, 1>(at<T>(a.f, t, n, d), f);
    load<T, 1>(at<T>(a.v, t, n, d), v);
    load<T, 1>(at<T>(a.dy, t, n, d), dy);
    if (t) load<T, 1>(at<T>(a.y, t - 1, n, d), c);
    else c[0] = a.h0 ? a.h0[m] : 0.0f;
    gates(f[0], ga, gb);
    const bool e = ended(a, t, n);
    if (e) c[0] = 0.0f;
    const float q = dy[0] + g;
    const float dv[1] = {gb * q}, df[1] = {ga * gb * (c[0] - v[0]) * q};
    store<T, 1>(at<T>(a.dv, t, n, d), dv);
    store<T, 1>(at<T>(a.df, t, n, d), df);
    g = e ? 0.0f : ga * q;
  }
  if (a.dh0) a.dh0[m] = g;
}

template <typename T>
cudaError_t launch(const Scan& a, bool back, cudaStream_t s) {
  const int64_t blocks = (a.N * a.D + 127) / 128;
  if (back) k_scan_back<T><<<(unsigned)blocks, 128, 0, s>>>(a);
  else k_scan<T><<<(unsigned)blocks, 128, 0, s>>>(a);
  return cudaGetLastError();
}

int run(const net_scan* p, bool back, void* stream) {
  if (!p) return fail(AUV_ERR_INVALID, "argument block is NULL");
  if (p->struct_size != sizeof(net_scan))
    return fail(AUV_ERR_INVALID, "struct_size %u, expected %zu", p->struct_size, sizeof(net_scan));
  if (p->dtype > NET_FP16) return fail(AUV_ERR_INVALID, "dtype %u unknown", p->dtype);
  if (p->T < 0 || p->N < 0 || p->D < 0) return fail(AUV_ERR_INVALID, "negative size");
  const int64_t most = (int64_t)1 << 37;   // channels of a call: blocks stay below 2^31
  if (p->N > most || p->D > most || (p->N && p->D > most / p->N) || p->T > ((int64_t)1 << 50))
    return fail(AUV_ERR_UNSUPPORTED, "N * D past 2^37 or T past 2^50");
  const int64_t M = p->N * p->D;
  if (M == 0) return AUV_OK;
  const int z = type_size(p->dtype);
  int rc;
  struct { const net_rows* r; const char* name; bool out, back; } rows[] = {
      {&p->f, "f", false, false}, {&p->v, "v", false, false}, {&p->y, "y", !back, false},
      {&p->dy, "dy", false, true}, {&p->df, "df", true, true}, {&p->dv, "dv", true, true}};
  if (p->T)
    for (const auto& q : rows)
      if ((back || !q.back) && (rc = need_rows(*q.r, q.name, p->T, p->N, p->D, z, q.out))) return rc;
  struct { const void* p; const char* name; size_t align; bool used; } flat[] = {
      {p->h0, "h0", 4, true}, {p->hT, "hT", 4, !back}, {p->dhT, "dhT", 4, back}, {p->dh0, "dh0", 4, back},
      {p->done, "done", 1, true}, {p->done_prev, "done_prev", 1, true}};
  for (const auto& q : flat)
    if (q.p && q.used && (rc = need(q.p, q.name, q.align))) return rc;
  const Scan a = {p->T, p->N, p->D, p->f, p->v, p->y, p->dy, p->df, p->dv, p->h0, p->hT, p->dhT, p->dh0, p->done,
                  p->done_prev};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = p->dtype == NET_FP32   ? launch<float>(a, back, s)
                        : p->dtype == NET_BF16 ? launch<__nv_bfloat16>(a, back, s)
                                               : launch<__half>(a, back, s);
  return e == cudaSuccess ? AUV_OK : cuda_fail(e, back ? "net_gate_scan_backward" : "net_gate_scan");
}

}  // namespace
}  // namespace net
}  // namespace auv

extern "C" {

int net_gate_scan(const net_scan* a, void* stream) { return auv::net::run(a, false, stream); }
int net_gate_scan_backward(const net_scan* a, void* stream) { return auv::net::run(a, true, stream); }

}  // extern "C"
