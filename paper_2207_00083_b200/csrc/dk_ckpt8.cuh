// The 8-bit form in which a checkpoint holds a tensor of rows x d values: whole numbers q of 8 bits under a power of two
// for each 32 consecutive values of a row,
//   value = q*2^(b - 127),  |q| <= 127,
// the rows of q padded with zeros to whole blocks, then the bytes b.  The power of two is the least under which no value
// of the block rounds beyond 127, so a value is off by at most half a step, at
// most 1/127 of the block's largest magnitude.  Powers of two, not max/127: x/2^k and q*2^k are exact, so what a value becomes
// does not depend on how the division is done, and q*2^k is a bf16 number, which the tensor cores take without another
// rounding.  The largest b is 248: the few values beyond 127.5*2^121, which would round to 2^128, become 127*2^121 (a mask
// of the type's largest magnitude among them).  b = 255: the block held an infinity or a NaN, and all its values are NaN.
#pragma once

#include <stdint.h>

namespace dk {
namespace ckpt8 {

constexpr int kBlock = 32;

__host__ __device__ inline int padded(int d) { return (d + kBlock - 1) / kBlock * kBlock; }
__host__ __device__ inline long long code_bytes(long long rows, int d) { return rows * padded(d); }
__host__ __device__ inline long long total_bytes(long long rows, int d) {
  return rows * padded(d) + rows * (padded(d) / kBlock);
}

// the byte of a block from the bits of its largest magnitude.  Adding 2^16 carries into the exponent exactly where the
// largest value would round to 128 steps of 2^-6 of its binade, that is from 127.5/64 on.
constexpr uint32_t kLargest = 248u;
__device__ __forceinline__ uint32_t exponent_byte(uint32_t most) {
  return most >= 0x7f800000u ? 255u : (uint32_t)min(max(1, (int)((most + 0x10000u) >> 23) - 6), (int)kLargest);
}
__device__ __forceinline__ float to_steps(uint32_t b) { return __uint_as_float(b == 255u ? 0u : (254u - b) << 23); }
// (of byte 255: infinity, which times the code 0 is NaN)
__device__ __forceinline__ float step_of(uint32_t b) { return __uint_as_float(b << 23); }

// Four codes.  1.5*2^23 + v has the nearest whole number to v (halves to even) in its low bits, two's complement.
__device__ __forceinline__ uint32_t pack4(float x, float y, float z, float w, float f) {
  constexpr float kMagic = 12582912.f;
  const uint32_t a = __float_as_uint(fmaf(x, f, kMagic)), b = __float_as_uint(fmaf(y, f, kMagic));
  const uint32_t c = __float_as_uint(fmaf(z, f, kMagic)), d = __float_as_uint(fmaf(w, f, kMagic));
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// VEC codes at `to` (aligned to VEC bytes)
template <int VEC>
__device__ __forceinline__ void put_codes(uint8_t* to, const float (&x)[VEC], uint32_t b) {
  const float f = to_steps(b);
  float v[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = x[i];
  if (b == kLargest) {
    const float most = 127.f * step_of(kLargest);
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = fminf(fmaxf(v[i], -most), most);
  }
  const uint32_t live = b == 255u ? 0u : 0xffffffffu;
  if constexpr (VEC == 8) {
    *reinterpret_cast<uint2*>(to) =
        make_uint2(pack4(v[0], v[1], v[2], v[3], f) & live, pack4(v[4], v[5], v[6], v[7], f) & live);
  } else if constexpr (VEC == 4) {
    *reinterpret_cast<uint32_t*>(to) = pack4(v[0], v[1], v[2], v[3], f) & live;
  } else if constexpr (VEC == 2) {
    *reinterpret_cast<uint16_t*>(to) = (uint16_t)(pack4(v[0], v[1], 0.f, 0.f, f) & live);
  } else {
    *to = (uint8_t)(pack4(v[0], 0.f, 0.f, 0.f, f) & live);
  }
}

// VEC codes and the byte of their block, as loaded
template <int VEC>
struct Raw {
  uint32_t w[VEC == 8 ? 2 : 1];
  uint32_t b;
};
template <int VEC>
__device__ __forceinline__ Raw<VEC> get(const uint8_t* codes, const uint8_t* exps) {
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

// the largest magnitude (as bits) over the lanes of a block: 32/VEC neighbours
template <int VEC>
__device__ __forceinline__ uint32_t block_most(const float (&v)[VEC]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < VEC; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  if constexpr (VEC == 1) return __reduce_max_sync(0xffffffffu, m);
#pragma unroll
  for (int o = kBlock / VEC / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}

}  // namespace ckpt8
}  // namespace dk
