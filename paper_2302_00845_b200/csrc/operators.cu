// State shared by the training operators: per-device lookups and the status word their kernels raise.
#include <atomic>

#include "operators.cuh"
#include "ptx.cuh"

namespace {
__device__ int g_ops_status;
constexpr int kMaxDevices = 64;
CdgOpsDevice g_ops[kMaxDevices];
std::atomic<int> g_ready[kMaxDevices];
std::atomic<long long> g_wait_limit{kCdgWaitCycles};
}  // namespace

int cdg_ops_device(const CdgOpsDevice **out) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return CDGRAB_ERR_DEVICE; }
  if (dev < 0 || dev >= kMaxDevices) return CDGRAB_ERR_DEVICE;
  if (!g_ready[dev].load(std::memory_order_acquire)) {
    int major = 0, sms = 0;
    void *p = nullptr;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess || major != 10 ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaGetSymbolAddress(&p, g_ops_status) != cudaSuccess) {
      cudaGetLastError();
      return CDGRAB_ERR_DEVICE;
    }
    // two threads that arrive together write the same values
    g_ops[dev].index = dev;
    g_ops[dev].sms = sms;
    g_ops[dev].status = static_cast<int *>(p);
    g_ready[dev].store(1, std::memory_order_release);
  }
  *out = &g_ops[dev];
  return CDGRAB_OK;
}

long long cdg_ops_wait_limit() { return g_wait_limit.load(std::memory_order_relaxed); }

extern "C" int cdgrab_operators_wait_limit(long long cycles) {
  if (cycles < 0 || cycles > (1ll << 40)) return CDGRAB_ERR_INVALID;
  g_wait_limit.store(cycles > 0 ? cycles : kCdgWaitCycles, std::memory_order_relaxed);
  return CDGRAB_OK;
}

extern "C" int cdgrab_operators_status(void) {
  const CdgOpsDevice *d = nullptr;
  const int rc = cdg_ops_device(&d);
  if (rc != CDGRAB_OK) return rc;
  if (cudaDeviceSynchronize() != cudaSuccess) { cudaGetLastError(); return CDGRAB_ERR_CUDA; }
  int st = 0;
  if (cudaMemcpy(&st, d->status, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess) { cudaGetLastError(); return CDGRAB_ERR_CUDA; }
  if (st != 0 && cudaMemset(d->status, 0, sizeof(int)) != cudaSuccess) { cudaGetLastError(); return CDGRAB_ERR_CUDA; }
  return st & CDG_ST_TIMEOUT ? CDGRAB_ERR_TIMEOUT : CDGRAB_OK;
}
