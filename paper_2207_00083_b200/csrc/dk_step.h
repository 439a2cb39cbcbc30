// Shared by the operators around the masked products (dk_norm.cu, dk_xent.cu, dk_ortho.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "dk_internal.h"

namespace dk {

// Plans that size a workspace without a context assume at most this many SMs.
constexpr int kMaxSms = 160;

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

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

}  // namespace dk
