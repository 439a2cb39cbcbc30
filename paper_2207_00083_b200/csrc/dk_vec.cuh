// Vectors of consecutive fp32 or bf16 elements, and moments of values: shared by the normalisations.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include <type_traits>

#include "dk.h"

namespace dk {

// VEC consecutive elements: as stored (Raw, one access of at most 16 bytes) and as fp32
template <int DT, int VEC>
struct Vec {
  static constexpr int BYTES = VEC * (DT == DK_F32 ? 4 : 2);
  using Raw = typename std::conditional<
      BYTES == 16, uint4,
      typename std::conditional<BYTES == 8, uint2,
                                typename std::conditional<BYTES == 4, uint32_t, uint16_t>::type>::type>::type;
  static __device__ __forceinline__ Raw get(const void* base, long long e) {
    return *reinterpret_cast<const Raw*>(static_cast<const char*>(base) + e * (BYTES / VEC));
  }
  static __device__ __forceinline__ void put(void* base, long long e, const Raw r) {
    *reinterpret_cast<Raw*>(static_cast<char*>(base) + e * (BYTES / VEC)) = r;
  }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[VEC]) {
    if constexpr (DT == DK_F32) {
      const float* f = reinterpret_cast<const float*>(&r);
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = f[i];
    } else if constexpr (VEC == 1) {
      v[0] = __uint_as_float((uint32_t)r << 16);
    } else {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  static __device__ __forceinline__ Raw pack(const float (&v)[VEC]) {
    Raw r;
    if constexpr (DT == DK_F32) {
      float* f = reinterpret_cast<float*>(&r);
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] = v[i];
    } else if constexpr (VEC == 1) {
      const __nv_bfloat16 t = __float2bfloat16_rn(v[0]);
      r = *reinterpret_cast<const uint16_t*>(&t);
    } else {
      uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&t);
      }
    }
    return r;
  }
  static __device__ __forceinline__ void load(const void* base, long long e, float (&v)[VEC]) {
    unpack(get(base, e), v);
  }
  static __device__ __forceinline__ void store(void* base, long long e, const float (&v)[VEC]) { put(base, e, pack(v)); }
};

// The low words of eight, shifted down by `off` bytes, 0 to 14 (even; fp32: a multiple of four): a vector that starts `off`
// bytes behind an aligned one.
template <int DT>
__device__ __forceinline__ uint4 shifted(const uint4& x, const uint4& y, int off) {
  uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  if (off & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (off & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  if (DT == DK_BF16 && (off & 2)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// (count, mean, sum of squared deviations) of the union of two sets
struct Moments {
  float n, mean, m2;
};
__device__ __forceinline__ Moments join(const Moments a, const Moments b) {
  const float n = a.n + b.n;
  if (b.n == 0.f) return a;
  if (a.n == 0.f) return b;
  const float d = b.mean - a.mean, f = __fdividef(b.n, n);
  return {n, fmaf(d, f, a.mean), a.m2 + b.m2 + d * d * a.n * f};
}
__device__ __forceinline__ Moments warp_join(Moments m) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Moments t;
    t.n = __shfl_xor_sync(0xffffffffu, m.n, o);
    t.mean = __shfl_xor_sync(0xffffffffu, m.mean, o);
    t.m2 = __shfl_xor_sync(0xffffffffu, m.m2, o);
    // (both lanes of a pair join in the same order)
    m = (threadIdx.x & o) ? join(t, m) : join(m, t);
  }
  return m;
}

// Two fp32 values in a 64-bit register pair: one instruction does both (rounded each as by itself).
struct F2 {
  unsigned long long v;
};
__device__ __forceinline__ F2 f2(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ F2 f2(float both) { return f2(both, both); }
__device__ __forceinline__ float2 split(F2 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
  return r;
}
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ float sum(F2 a) {
  const float2 t = split(a);
  return t.x + t.y;
}

}  // namespace dk
