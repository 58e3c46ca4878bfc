// State shared by the training operators: per-device lookups and the status word their kernels raise.
#include <atomic>
#include <climits>
#include <cstring>

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
  // one report a call: what else the word holds stays for the next (written before this returns: a later launch may report on a stream
  // that does not wait for the copy)
  const int said = st & CDG_ST_TIMEOUT ? CDG_ST_TIMEOUT : st, rest = st & ~said;
  if (st != 0 && (cudaMemcpy(d->status, &rest, sizeof(int), cudaMemcpyHostToDevice) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess)) {
    cudaGetLastError();
    return CDGRAB_ERR_CUDA;
  }
  return said & CDG_ST_TIMEOUT ? CDGRAB_ERR_TIMEOUT : said & CDG_ST_INDEX ? CDGRAB_ERR_INVALID : CDGRAB_OK;
}

namespace {
// the fields of a record, eight bytes each, in turn
struct Record {
  const unsigned char *p;
  bool ok = true;            // every number fitted its parameter
  template <typename T> T take() { T v; memcpy(&v, p, sizeof(T)); p += sizeof(T); return v; }
  long long wide() { return take<long long>(); }
  int narrow() {
    const long long v = wide();
    ok = ok && v >= INT_MIN && v <= INT_MAX;
    return (int)v;
  }
  unsigned word() {
    const long long v = wide();
    ok = ok && v >= 0 && v <= (long long)UINT_MAX;
    return (unsigned)v;
  }
  void *pointer() { return reinterpret_cast<void *>(wide()); }
};
}  // namespace

extern "C" int cdgrab_call(int call, const void *record) {
  if (!record) return CDGRAB_ERR_INVALID;
  Record r = {static_cast<const unsigned char *>(record)};
  // (fields are taken one statement after another: the order of a call's arguments is not given)
  switch (call) {
    case CDGRAB_CALL_EMBEDDING_FORWARD: {
      const long long groups = r.wide(), length = r.wide();
      const int cols = r.narrow(), vocab = r.narrow(), bits = r.narrow();
      const void *tokens = r.pointer();
      const long long token_stride = r.wide(), padding = r.wide();
      const double scale = r.take<double>();
      const int dtype = r.narrow();
      const void *table = r.pointer();
      const long long table_stride = r.wide();
      const int out_dtype = r.narrow();
      void *y = r.pointer();
      const long long y_stride = r.wide();
      void *stream = r.pointer();
      return !r.ok ? CDGRAB_ERR_INVALID
                   : cdgrab_embedding_forward(groups, length, cols, vocab, bits, tokens, token_stride, padding, (float)scale, dtype, table,
                                              table_stride, out_dtype, y, y_stride, stream);
    }
    case CDGRAB_CALL_EMBEDDING_BACKWARD: {
      const int m = r.narrow();
      const long long groups = r.wide(), length = r.wide();
      const int cols = r.narrow(), vocab = r.narrow(), bits = r.narrow();
      const void *tokens = r.pointer();
      const long long token_stride = r.wide(), padding = r.wide();
      const double scale = r.take<double>();
      const int dtype = r.narrow();
      const void *dy = r.pointer();
      const long long dy_stride = r.wide();
      const int grad_dtype = r.narrow();
      void *dtable = r.pointer();
      const long long worker_stride = r.wide(), row_stride = r.wide();
      const int accumulate = r.narrow();
      void *workspace = r.pointer();
      const long long bytes = r.wide();
      void *stream = r.pointer();
      return !r.ok ? CDGRAB_ERR_INVALID
                   : cdgrab_embedding_backward(m, groups, length, cols, vocab, bits, tokens, token_stride, padding, (float)scale, dtype, dy,
                                               dy_stride, grad_dtype, dtable, worker_stride, row_stride, accumulate, workspace, bytes, stream);
    }
    case CDGRAB_CALL_DROPOUT_FORWARD:
    case CDGRAB_CALL_DROPOUT_BACKWARD: {
      const long long rows = r.wide(), cols = r.wide();
      const int dtype = r.narrow();
      const void *x = r.pointer();
      const long long xs = r.wide();
      const int out_dtype = r.narrow();
      const bool forward = call == CDGRAB_CALL_DROPOUT_FORWARD;
      const void *res = forward ? r.pointer() : nullptr;
      const long long rs = forward ? r.wide() : 0;
      void *y = r.pointer();
      const long long ys = r.wide();
      const double p = r.take<double>();
      const unsigned long long seed = r.take<unsigned long long>();
      const unsigned which = r.word(), step = r.word();
      const long long *step_dev = static_cast<const long long *>(r.pointer());
      void *stream = r.pointer();
      return !r.ok ? CDGRAB_ERR_INVALID
             : forward ? cdgrab_dropout_forward(rows, cols, dtype, x, xs, out_dtype, res, rs, y, ys, p, seed, which, step, step_dev, stream)
                       : cdgrab_dropout_backward(rows, cols, dtype, x, xs, out_dtype, y, ys, p, seed, which, step, step_dev, stream);
    }
    case CDGRAB_CALL_ROTARY_FORWARD: {
      const cdgrab_rotary_shape shape = r.take<cdgrab_rotary_shape>();
      const void *q = r.pointer(), *k = r.pointer();
      const float *qw = static_cast<const float *>(r.pointer()), *kw = static_cast<const float *>(r.pointer());
      const void *pos = r.pointer();
      const int bits = r.narrow();
      const long long pos_stride = r.wide();
      const int32_t *lens = static_cast<const int32_t *>(r.pointer());
      void *qo = r.pointer(), *ko = r.pointer(), *stream = r.pointer();
      return !r.ok ? CDGRAB_ERR_INVALID : cdgrab_rotary_forward(&shape, q, k, qw, kw, pos, bits, pos_stride, lens, qo, ko, stream);
    }
    case CDGRAB_CALL_ROTARY_BACKWARD: {
      const cdgrab_rotary_shape shape = r.take<cdgrab_rotary_shape>();
      const int m = r.narrow();
      const void *dq = r.pointer(), *dk = r.pointer(), *q = r.pointer(), *k = r.pointer();
      const float *qw = static_cast<const float *>(r.pointer()), *kw = static_cast<const float *>(r.pointer());
      const void *pos = r.pointer();
      const int bits = r.narrow();
      const long long pos_stride = r.wide();
      const int32_t *lens = static_cast<const int32_t *>(r.pointer());
      void *qo = r.pointer(), *ko = r.pointer();
      const int grad_dtype = r.narrow();
      void *dqw = r.pointer(), *dkw = r.pointer();
      const long long worker_stride = r.wide();
      void *workspace = r.pointer();
      const long long bytes = r.wide();
      void *stream = r.pointer();
      return !r.ok ? CDGRAB_ERR_INVALID
                   : cdgrab_rotary_backward(&shape, m, dq, dk, q, k, qw, kw, pos, bits, pos_stride, lens, qo, ko, grad_dtype, dqw, dkw,
                                            worker_stride, workspace, bytes, stream);
    }
    default: return CDGRAB_ERR_INVALID;
  }
}
