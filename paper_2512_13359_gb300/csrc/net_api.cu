// net_api.cu -- the network operators' error text and argument checks.
#include <atomic>
#include <cstdarg>

#include "net_common.cuh"

namespace auv {
namespace net {

namespace {
thread_local char g_err[256] = "";
}

int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return code;
}

int cuda_fail(cudaError_t e, const char* what) { return fail(AUV_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e)); }

int need(const void* p, const char* name, size_t align) {
  if (!p) return fail(AUV_ERR_INVALID, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % align) return fail(AUV_ERR_SIZE, "%s not %zu-byte aligned", name, align);
  cudaPointerAttributes a;
  if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
    cudaGetLastError();
    return fail(AUV_ERR_SIZE, "%s is not device memory", name);
  }
  if (a.type == cudaMemoryTypeManaged) return AUV_OK;
  if (a.type != cudaMemoryTypeDevice) return fail(AUV_ERR_SIZE, "%s is not device memory", name);
  int cur = -1;
  const cudaError_t e = cudaGetDevice(&cur);
  if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
  if (a.device != cur)
    return fail(AUV_ERR_INVALID, "%s lives on device %d but device %d is current", name, a.device, cur);
  return AUV_OK;
}

int need_rows(const net_rows& r, const char* name, int64_t ni, int64_t nj, int64_t nk, int size, bool output) {
  const int rc = need(r.data, name, size);
  if (rc) return rc;
  const int64_t most = INT64_MAX / 16;
  if (r.outer < 0 || r.inner < 0) return fail(AUV_ERR_INVALID, "%s: negative stride", name);
  if ((ni > 1 && r.outer > most / ni) || (nj > 1 && r.inner > most / nj))
    return fail(AUV_ERR_INVALID, "%s: strides past 2^59 elements", name);
  if (output) {
    const int64_t o = ni > 1 ? r.outer : INT64_MAX, i = nj > 1 ? r.inner : INT64_MAX;
    const bool by_outer = nj <= 1 ? o >= nk : i >= nk && (ni <= 1 || o >= (nj - 1) * i + nk);
    const bool by_inner = ni <= 1 ? i >= nk : o >= nk && (nj <= 1 || i >= (ni - 1) * o + nk);
    if (!by_outer && !by_inner) return fail(AUV_ERR_SIZE, "%s: rows of an output overlap", name);
  }
  return AUV_OK;
}

int sm_count() {
  static std::atomic<int> known[64];
  int dev = 0, n = 152;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64) return n;
  const int k = known[dev].load(std::memory_order_relaxed);
  if (k) return k;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return 152;
  }
  known[dev].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace net
}  // namespace auv

extern "C" const char* net_last_error(void) { return auv::net::g_err; }
