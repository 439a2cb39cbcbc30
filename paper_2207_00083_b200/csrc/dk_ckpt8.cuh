// The 8-bit form in which a checkpoint holds a tensor of rows x d values: whole numbers q of 8 bits under a power of two
// for each 32 consecutive values of a row,
//   value = q*2^(b - 127),  |q| <= 127,
// the rows of q padded with zeros to whole blocks, then the bytes b.  The power of two is the least under which no value
// of the block rounds beyond 127, so a value is off by at most half a step, at most 1/127 of the block's largest magnitude (but
// of blocks below 63.75*2^-126, whose step is the least there is, 2^-126).
// Powers of two, not max/127: x/2^k and q*2^k are exact, so what a value becomes
// does not depend on how the division is done, and q*2^k is a bf16 number, which the tensor cores take without another
// rounding.  The largest b is 248: the few values from 127.5*2^121 on, which would round to 2^128, become 127*2^121, off by up to
// a whole step (a mask of the type's largest magnitude among them).  b = 255: the block held an infinity or a NaN, and all its values are NaN.
#pragma once

#include <stdint.h>

#include "dk_vec.cuh"

namespace dk {
namespace ckpt8 {

constexpr int kBlock = 32;

__host__ __device__ inline int padded(int d) { return (d + kBlock - 1) / kBlock * kBlock; }
__host__ __device__ inline long long code_bytes(long long rows, int d) { return rows * padded(d); }
__host__ __device__ inline long long total_bytes(long long rows, int d) {
  return rows * padded(d) + rows * (padded(d) / kBlock);
}

// A block's byte from the bits of its largest magnitude, and what brings its values to steps.  Adding 2^16 carries into the
// exponent exactly where the largest value would round to 128 steps of 2^-6 of its binade, that is from 127.5/64 on.
constexpr uint32_t kLargest = 248u;
struct Scale {
  uint32_t byte;
  float steps;           // values times this are steps
  bool rare;             // values beyond the range, infinities or NaN
};
__device__ __forceinline__ Scale scale_of(uint32_t most) {
  Scale s;
  const int t = min(max((int)((most + 0x10000u) >> 23), 7), 254);
  s.byte = (uint32_t)(t - 6);
  s.steps = __uint_as_float((uint32_t)(260 - t) << 23);
  s.rare = most >= 0x7f7f0000u;
  if (most >= 0x7f800000u) s.byte = 255u;
  return s;
}
// (of byte 255: infinity, which times the code 0 is NaN)
__device__ __forceinline__ float step_of(uint32_t b) { return __uint_as_float(b << 23); }

// Four codes.  1.5*2^23 + v has the nearest whole number to v (halves to even) in its low bits, two's complement.
__device__ __forceinline__ uint32_t pack4(float x, float y, float z, float w, float f) {
  const float2 m = split(fma(f2(x, y), f2(f), f2(12582912.f))), n = split(fma(f2(z, w), f2(f), f2(12582912.f)));
  return __byte_perm(__byte_perm(__float_as_uint(m.x), __float_as_uint(m.y), 0x0040),
                     __byte_perm(__float_as_uint(n.x), __float_as_uint(n.y), 0x0040), 0x5410);
}
// VEC codes at `to` (aligned to VEC bytes)
template <int VEC>
__device__ __forceinline__ void put_codes(uint8_t* to, const float (&x)[VEC], const Scale& s) {
  constexpr int W = VEC == 8 ? 2 : 1;
  uint32_t w[W];
  if (!s.rare) {
#pragma unroll
    for (int i = 0; i < W; ++i)
      w[i] = pack4(x[4 * i], VEC > 1 ? x[(4 * i + 1) % VEC] : 0.f, VEC > 2 ? x[(4 * i + 2) % VEC] : 0.f,
                   VEC > 2 ? x[(4 * i + 3) % VEC] : 0.f, s.steps);
  } else {
    // largest magnitudes become 127 of the largest steps; a block with an infinity or a NaN holds zeros
    const float most = 127.f * step_of(kLargest);
    float v[4 * W];
#pragma unroll
    for (int i = 0; i < 4 * W; ++i) v[i] = i < VEC ? fminf(fmaxf(x[i % VEC], -most), most) : 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i)
      w[i] = s.byte == 255u ? 0u : pack4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], s.steps);
  }
  if constexpr (VEC == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
  else if constexpr (VEC == 4) *reinterpret_cast<uint32_t*>(to) = w[0];
  else if constexpr (VEC == 2) *reinterpret_cast<uint16_t*>(to) = (uint16_t)w[0];
  else *to = (uint8_t)w[0];
}

// VEC codes and the byte of their block, as loaded
template <int VEC>
struct Raw {
  uint32_t w[VEC == 8 ? 2 : 1];
  uint32_t b;
};
template <int VEC>
__device__ __forceinline__ Raw<VEC> get_codes(const uint8_t* codes) {
  Raw<VEC> r;
  if constexpr (VEC == 8) {
    const uint2 u = *reinterpret_cast<const uint2*>(codes);
    r.w[0] = u.x; r.w[1] = u.y;
  } else if constexpr (VEC == 4) {
    r.w[0] = *reinterpret_cast<const uint32_t*>(codes);
  } else if constexpr (VEC == 2) {
    r.w[0] = *reinterpret_cast<const uint16_t*>(codes);
  } else {
    r.w[0] = *codes;
  }
  return r;
}
template <int VEC>
__device__ __forceinline__ Raw<VEC> get(const uint8_t* codes, const uint8_t* exps) {
  Raw<VEC> r = get_codes<VEC>(codes);
  r.b = *exps;
  return r;
}
// (a code with its sign bit turned over, put into the low bits of 2^23, is 2^23 + 128 + q)
constexpr float kBias = 8388736.f;
template <int VEC>
__device__ __forceinline__ float biased(const Raw<VEC>& r, int i) {
  return __uint_as_float(__byte_perm(r.w[i / 4] ^ 0x80808080u, 0x4b000000u, 0x7540u | (uint32_t)(i & 3)));
}
template <int VEC>
__device__ __forceinline__ void unpack(const Raw<VEC>& r, float (&v)[VEC]) {
  const float s = step_of(r.b);
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = (biased<VEC>(r, i) - kBias) * s;
}

// largest of three magnitudes; a NaN is passed on
__device__ __forceinline__ float abs_max(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// the largest magnitude (as bits) over the lanes of a block: 32/VEC neighbours, `lanes` of the warp taking part
template <int VEC>
__device__ __forceinline__ uint32_t block_most(const float (&v)[VEC], unsigned lanes = 0xffffffffu) {
  float f = abs_max(v[0], v[VEC > 1 ? 1 : 0], v[VEC > 2 ? 2 : 0]);
#pragma unroll
  for (int i = 3; i < VEC; i += 2) f = abs_max(f, v[i], v[i + 1 < VEC ? i + 1 : i]);
  uint32_t m = __float_as_uint(f);
  if constexpr (VEC == 1) {
    return __reduce_max_sync(lanes, m);
  } else {
#pragma unroll
    for (int o = kBlock / VEC / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(lanes, m, o));
    return m;
  }
}

}  // namespace ckpt8
}  // namespace dk
