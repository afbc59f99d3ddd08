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
