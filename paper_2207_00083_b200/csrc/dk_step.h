// Shared by the operators around the masked products (dk_norm.cu, dk_xent.cu, dk_ortho.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "dk_internal.h"

namespace dk {

// Plans that size a workspace without a context assume at most this many SMs.
constexpr int kMaxSms = 160;

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Words with which the last CTA of several finds that it is the last; zero at the start of every kernel that uses them
// and left at zero by it.
inline unsigned int* step_counters(const dk_ctx* ctx) { return ctx->d_step; }

// Makes the context's device current for the length of a call.
struct OnDevice {
  int prev, dev;
  bool ok;
  explicit OnDevice(int d) : prev(-1), dev(d), ok(false) {
    if (cudaGetDevice(&prev) != cudaSuccess) return;
    ok = prev == d || cudaSetDevice(d) == cudaSuccess;
  }
  ~OnDevice() {
    if (ok && prev != dev) cudaSetDevice(prev);
  }
};

// The most dynamic shared memory that any call gives a kernel, told to the runtime once per kernel and device and never
// lowered after: another thread's context may be about to launch the same kernel with more than this call needs.
// (One SmemLimit, static, per kernel; a CTA of `threads` that re-partitions its registers needs `pool` of them.)
struct SmemLimit {
  std::atomic<bool> done[64];
};
template <typename K>
dk_status allow_smem(SmemLimit& limit, int device, K kern, int bytes, int threads = 0, int pool = 0) {
  if (device < 0 || device >= 64) return DK_ERR_UNSUPPORTED;
  if (limit.done[device].load(std::memory_order_acquire)) return DK_OK;
  if (pool > 0) {
    cudaFuncAttributes fa;
    if (cudaFuncGetAttributes(&fa, kern) != cudaSuccess) return DK_ERR_CUDA;
    if (fa.numRegs * threads < pool) return DK_ERR_UNSUPPORTED;
  }
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return DK_ERR_CUDA;
  limit.done[device].store(true, std::memory_order_release);
  return DK_OK;
}

// Programmatic dependent launch: the next kernel of the stream may be set up while this one runs (its own call of this
// function then waits for this one's end and its writes).  At the start of kernels that follow one another closely.
__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void chained_launch() {
  allow_next();
  wait_for_previous();
}
template <typename... K, typename... A>
cudaError_t launch_chained(void (*kern)(K...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

}  // namespace dk
