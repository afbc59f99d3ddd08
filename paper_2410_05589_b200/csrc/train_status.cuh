// The device's word for waits that ran out in calls of the training operators without a status word of their own: one per
// source file that includes this, in the library's own memory, so that neither a call nor a captured graph has to keep it.
#pragma once
#include "train_ops.cuh"
#include "umma_gemm.cuh"

namespace ps {
namespace train {
namespace {

__device__ int g_status;

__device__ __forceinline__ void report_timeout(int* status) { atomicOr(status ? status : &g_status, kStatTimeout); }

// Reads and clears the word of the current device on the stream; *word is there once the stream has been waited for.
cudaError_t take_word(int* word, cudaStream_t st) {
  void* p = nullptr;
  cudaError_t e = cudaGetSymbolAddress(&p, g_status);
  if (e == cudaSuccess) e = cudaMemcpyAsync(word, p, sizeof(int), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaMemsetAsync(p, 0, sizeof(int), st);
  return e;
}

// A bounded wait on a barrier that nothing completes, reported as the operators' kernels do.
__global__ void k_wait_expires(long long limit, int* status) {
  __shared__ uint64_t bar;
  __shared__ int abort_flag;
  if (threadIdx.x == 0) {
    umma::mbar_init(&bar, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (!umma::mbar_wait(&bar, 0, &abort_flag, limit)) report_timeout(status);
  }
}
cudaError_t wait_expires(long long limit, int* status, cudaStream_t st) {
  k_wait_expires<<<1, 32, 0, st>>>(limit, status);
  return cudaGetLastError();
}

}  // namespace
}  // namespace train
}  // namespace ps
