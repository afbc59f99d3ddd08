// What the training operators (group_attn*.cu, lm_loss*.cu, embed_rows.cu) share on the host: they have no context, so
// errors go to the caller's buffer and answers of a device are asked once per device.
#pragma once
#include <cstdio>

#include "ps_internal.cuh"

namespace ps {
namespace train {

// Where a call reports: the caller's text buffer.
struct Err {
  char* text;
  size_t cap;
  ps_status operator()(ps_status s, const char* what) const {
    if (text && cap) std::snprintf(text, cap, "%s", what);
    return s;
  }
  ps_status cuda(cudaError_t e, const char* what) const {
    if (e == cudaSuccess) return PS_OK;
    (void)cudaGetLastError();
    if (text && cap) std::snprintf(text, cap, "%s: %s", what, cudaGetErrorString(e));
    return PS_ERR_CUDA;
  }
};

constexpr size_t kAlign = 256;
inline size_t up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }
inline bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// Multiprocessors of the current device (148 where none can be asked: sizes are worked out without a device too).
int device_sms();
// Lets `kern` have `bytes` of dynamic shared memory on the current device; `done`: one word per kernel, a bit per device.
cudaError_t allow_smem(const void* kern, int bytes, std::atomic<uint64_t>& done);

// Slices of a workspace, one behind the other (behind kAlign bytes, so that none is empty: 0 bytes mean sizes that are refused).
struct Carve {
  char* base;
  size_t at = kAlign;
  explicit Carve(void* ws) : base((char*)ws) {}
  template <class T>
  T* take(size_t n) {
    T* p = base ? reinterpret_cast<T*>(base + at) : nullptr;
    at += up(n * sizeof(T));
    return p;
  }
};
// What a wait that ran out leaves in the words of calls without one of their own (train_status.cuh), and one that does.
cudaError_t attn_take_status(int* word, cudaStream_t st);
cudaError_t loss_take_status(int* word, cudaStream_t st);
cudaError_t attn_wait_expires(long long limit, int* status, cudaStream_t st);
cudaError_t loss_wait_expires(long long limit, int* status, cudaStream_t st);
ps_status check_workspace(const Err& err, const char* who, const void* ws, size_t have, size_t need);

}  // namespace train
}  // namespace ps
