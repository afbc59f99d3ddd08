// Host helpers of the training operators.
#include "train_ops.cuh"

namespace ps {
namespace train {
namespace {
constexpr int kMaxDevices = 64;
std::atomic<int> g_sms[kMaxDevices];
}  // namespace

int device_sms() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
    (void)cudaGetLastError();
    return 148;
  }
  int n = g_sms[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
      (void)cudaGetLastError();
      return 148;
    }
    g_sms[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

cudaError_t allow_smem(const void* kern, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < kMaxDevices ? 1ull << dev : 0;
  if (bit && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

ps_status check_workspace(const Err& err, const char* who, const void* ws, size_t have, size_t need) {
  char text[160];
  if (!ws || !aligned(ws, kAlign)) {
    std::snprintf(text, sizeof(text), "%s: the workspace must be 256-byte aligned device memory", who);
    return err(PS_ERR_INVALID_ARG, text);
  }
  if (have < need) {
    std::snprintf(text, sizeof(text), "%s: workspace of %zu bytes, %zu are needed", who, have, need);
    return err(PS_ERR_CAPACITY, text);
  }
  return PS_OK;
}

}  // namespace train
}  // namespace ps

using namespace ps::train;

extern "C" ps_status ps_train_poll(void* stream) {
  cudaStream_t st = (cudaStream_t)stream;
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  const cudaError_t asked = cudaStreamIsCapturing(st, &capture);
  if (asked != cudaSuccess || capture != cudaStreamCaptureStatusNone) {
    (void)cudaGetLastError();
    return PS_ERR_INVALID_ARG;
  }
  int words[2] = {0, 0};
  cudaError_t e = attn_take_status(&words[0], st);
  if (e == cudaSuccess) e = loss_take_status(&words[1], st);
  const cudaError_t done = cudaStreamSynchronize(st);   // (whatever failed: the words must not be written once they are gone)
  if (e != cudaSuccess || done != cudaSuccess) {
    (void)cudaGetLastError();
    return PS_ERR_CUDA;
  }
  return (words[0] | words[1]) & ps::kStatTimeout ? PS_ERR_TIMEOUT : PS_OK;
}

extern "C" ps_status ps_debug_train_wait_expires(int loss, long long limit_cycles, int* status, void* stream) {
  if (limit_cycles < 0 || limit_cycles > 4000000000LL) return PS_ERR_INVALID_ARG;
  const cudaError_t e = loss ? loss_wait_expires(limit_cycles, status, (cudaStream_t)stream)
                             : attn_wait_expires(limit_cycles, status, (cudaStream_t)stream);
  if (e == cudaSuccess) return PS_OK;
  (void)cudaGetLastError();
  return PS_ERR_CUDA;
}
