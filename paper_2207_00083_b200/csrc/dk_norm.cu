// Group normalisation with an activation, channels-last, forward and backward.
//
//   z = (x - mean)*rstd*gamma + beta,  y = act(z),  statistics per sample and group of channels
//   d = dy*act'(z),  dgamma = sum d*xhat,  dbeta = sum d
//   dx = rstd*(q - mean(q) - xhat*mean(q*xhat)),  q = d*gamma
//
// A sample's pixels are cut into slabs.  The first kernel of either direction
// reads a slab once and leaves its sums, the second joins the slabs of a sample
// in a fixed order, the third reads the tensors again and writes the result.
// Every thread keeps one vector of consecutive channels of one group at a time.
//
// Variance.  The sums of a thread are taken about its own first value, so that
// cancellation is bounded by its number of values (at most kMaxPix pixels) and
// not by how far the mean lies from zero; the (count, mean, sum of squared
// deviations) of threads and slabs are then joined pairwise,
//   M2 = M2a + M2b + (mean_b - mean_a)^2 * na*nb/(na + nb).
#include <cuda_bf16.h>

#include "dk_internal.h"
#include "dk_step.h"

namespace dk {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPix = 64;        // pixels a thread adds up about one pivot
constexpr int kMaxC = 16384;

template <int DT, int VEC>
struct Vec {
  static __device__ __forceinline__ void load(const void* base, long long e, float (&v)[VEC]) {
    if constexpr (DT == DK_F32) {
      const float* p = static_cast<const float*>(base) + e;
      if constexpr (VEC == 4) {
        const float4 t = *reinterpret_cast<const float4*>(p);
        v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
      } else if constexpr (VEC == 2) {
        const float2 t = *reinterpret_cast<const float2*>(p);
        v[0] = t.x; v[1] = t.y;
      } else {
        v[0] = *p;
      }
    } else {
      const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(base) + e;
      if constexpr (VEC == 1) {
        v[0] = __bfloat162float(*p);
      } else {
        uint32_t w[VEC / 2];
        if constexpr (VEC == 8) {
          const uint4 t = *reinterpret_cast<const uint4*>(p);
          w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w;
        } else if constexpr (VEC == 4) {
          const uint2 t = *reinterpret_cast<const uint2*>(p);
          w[0] = t.x; w[1] = t.y;
        } else {
          w[0] = *reinterpret_cast<const uint32_t*>(p);
        }
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
          v[2 * i] = __uint_as_float(w[i] << 16);
          v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
      }
    }
  }
  static __device__ __forceinline__ void store(void* base, long long e, const float (&v)[VEC]) {
    if constexpr (DT == DK_F32) {
      float* p = static_cast<float*>(base) + e;
      if constexpr (VEC == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
      else if constexpr (VEC == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
      else *p = v[0];
    } else {
      __nv_bfloat16* p = static_cast<__nv_bfloat16*>(base) + e;
      if constexpr (VEC == 1) {
        *p = __float2bfloat16_rn(v[0]);
      } else {
        uint32_t w[VEC / 2];
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
          const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
        if constexpr (VEC == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (VEC == 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
      }
    }
  }
};

// z*sigmoid(z): exp(-z) overflows to infinity for very negative z, the quotient is then -0
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == DK_ACT_NONE) return z;
  if (act == DK_ACT_RELU) return z < 0.f ? 0.f : z;        // (a NaN stays a NaN)
  return z / (1.f + __expf(-z));
}
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == DK_ACT_NONE) return 1.f;
  if (act == DK_ACT_RELU) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
  const float e = __expf(-fabsf(z)), r = 1.f / (1.f + e);
  const float s = z >= 0.f ? r : e * r;                    // sigmoid(z), no overflow on either side
  return s * (1.f + z * (1.f - s));
}

// (count, mean, sum of squared deviations) of the union of two sets
struct Moments {
  float n, mean, m2;
};
__device__ __forceinline__ Moments join(const Moments a, const Moments b) {
  const float n = a.n + b.n;
  if (b.n == 0.f) return a;
  if (a.n == 0.f) return b;
  const float d = b.mean - a.mean, f = b.n / n;
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

struct NormParams {
  const void* x;
  const void* dy;
  void* out;
  const float* gamma;
  const float* beta;
  float* stats;           // [n][groups][2]
  float* part;            // forward: [n][slabs][groups][3]; backward: [n][slabs][c][2]
  float* gsum;            // backward: [n][groups][2] means of q and q*xhat
  float* csum;            // backward: [n][c][2]
  float* dgamma;
  float* dbeta;
  long long n;
  int pix, c, groups, cg, slabs, slab_pix, act;
  int TX, TY;             // threads along the channel vectors, and along the pixels
  float eps;
};

template <int DT, int VEC>
__global__ void __launch_bounds__(kThreads) norm_stats_kernel(const NormParams p) {
  extern __shared__ float sm[];
  const int cv = p.c / VEC;
  const int tx = threadIdx.x % p.TX, ty = threadIdx.x / p.TX;
  const long long s = blockIdx.x / p.slabs;
  const int slab = blockIdx.x % p.slabs;
  const int p0 = slab * p.slab_pix, p1 = min(p.pix, p0 + p.slab_pix);
  const long long base = (s * p.pix) * (long long)p.c;
  if (ty < p.TY) {
    for (int v = tx; v < cv; v += p.TX) {
      Moments tot{0.f, 0.f, 0.f};
      for (int b = p0 + ty; b < p1; b += p.TY * kMaxPix) {
        float pivot = 0.f, s1 = 0.f, s2 = 0.f;
        int cnt = 0;
        for (int i = b; i < p1 && cnt < kMaxPix; i += p.TY, ++cnt) {
          float a[VEC];
          Vec<DT, VEC>::load(p.x, base + (long long)i * p.c + v * VEC, a);
          if (cnt == 0) pivot = a[0];
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float d = a[k] - pivot;
            s1 += d;
            s2 = fmaf(d, d, s2);
          }
        }
        const float n = (float)(cnt * VEC), m = s1 / n;
        tot = join(tot, Moments{n, pivot + m, fmaxf(0.f, fmaf(-s1, m, s2))});
        if (!(s2 - s2 == 0.f)) tot.m2 = s2;        // (a NaN or an infinity is passed on, not clamped away)
      }
      float* e = sm + 3 * ((size_t)ty * cv + v);
      e[0] = tot.n; e[1] = tot.mean; e[2] = tot.m2;
    }
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int vg = p.cg / VEC, items = vg * p.TY;
  for (int g = warp; g < p.groups; g += kThreads / 32) {
    Moments m{0.f, 0.f, 0.f};
    for (int i = lane; i < items; i += 32) {
      const float* e = sm + 3 * ((size_t)(i / vg) * cv + g * vg + i % vg);
      m = join(m, Moments{e[0], e[1], e[2]});
    }
    m = warp_join(m);
    if (lane == 0) {
      float* o = p.part + 3 * ((s * p.slabs + slab) * p.groups + g);
      o[0] = m.n; o[1] = m.mean; o[2] = m.m2;
    }
  }
}

// one warp per sample and group: joins the slabs
__global__ void __launch_bounds__(kThreads) norm_join_kernel(const NormParams p) {
  const long long i = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (i >= p.n * p.groups) return;
  const long long s = i / p.groups;
  const int g = (int)(i % p.groups);
  Moments m{0.f, 0.f, 0.f};
  for (int b = lane; b < p.slabs; b += 32) {
    const float* e = p.part + 3 * ((s * p.slabs + b) * p.groups + g);
    m = join(m, Moments{e[0], e[1], e[2]});
  }
  m = warp_join(m);
  if (lane == 0) {
    p.stats[2 * i] = m.mean;
    p.stats[2 * i + 1] = 1.f / sqrtf(m.m2 / m.n + p.eps);
  }
}

template <int DT, int VEC>
__global__ void __launch_bounds__(kThreads) norm_apply_kernel(const NormParams p) {
  const int cv = p.c / VEC;
  const int tx = threadIdx.x % p.TX, ty = threadIdx.x / p.TX;
  if (ty >= p.TY) return;
  const long long s = blockIdx.x / p.slabs;
  const int slab = blockIdx.x % p.slabs;
  const int p0 = slab * p.slab_pix, p1 = min(p.pix, p0 + p.slab_pix);
  const long long base = (s * p.pix) * (long long)p.c;
  for (int v = tx; v < cv; v += p.TX) {
    const int g = v * VEC / p.cg;
    const float mean = p.stats[2 * (s * p.groups + g)], rstd = p.stats[2 * (s * p.groups + g) + 1];
    float ga[VEC], be[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) { ga[k] = p.gamma[v * VEC + k] * rstd; be[k] = p.beta[v * VEC + k]; }
    for (int i = p0 + ty; i < p1; i += p.TY) {
      float a[VEC];
      const long long e = base + (long long)i * p.c + v * VEC;
      Vec<DT, VEC>::load(p.x, e, a);
#pragma unroll
      for (int k = 0; k < VEC; ++k) a[k] = act_value(fmaf(a[k] - mean, ga[k], be[k]), p.act);
      Vec<DT, VEC>::store(p.out, e, a);
    }
  }
}

// sums of d and d*xhat over a slab, per channel
template <int DT, int VEC>
__global__ void __launch_bounds__(kThreads) norm_bwd_sums_kernel(const NormParams p) {
  extern __shared__ float sm[];
  const int cv = p.c / VEC;
  const int tx = threadIdx.x % p.TX, ty = threadIdx.x / p.TX;
  const long long s = blockIdx.x / p.slabs;
  const int slab = blockIdx.x % p.slabs;
  const int p0 = slab * p.slab_pix, p1 = min(p.pix, p0 + p.slab_pix);
  const long long base = (s * p.pix) * (long long)p.c;
  if (ty < p.TY) {
    for (int v = tx; v < cv; v += p.TX) {
      const int g = v * VEC / p.cg;
      const float mean = p.stats[2 * (s * p.groups + g)], rstd = p.stats[2 * (s * p.groups + g) + 1];
      float ga[VEC], be[VEC], s0[VEC], s1[VEC];
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        ga[k] = p.gamma[v * VEC + k]; be[k] = p.beta[v * VEC + k];
        s0[k] = 0.f; s1[k] = 0.f;
      }
      for (int i = p0 + ty; i < p1; i += p.TY) {
        float a[VEC], dy[VEC];
        const long long e = base + (long long)i * p.c + v * VEC;
        Vec<DT, VEC>::load(p.x, e, a);
        Vec<DT, VEC>::load(p.dy, e, dy);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float xh = (a[k] - mean) * rstd;
          const float d = dy[k] * act_slope(fmaf(xh, ga[k], be[k]), p.act);
          s0[k] += d;
          s1[k] = fmaf(d, xh, s1[k]);
        }
      }
      float* e = sm + 2 * ((size_t)ty * p.c + v * VEC);
#pragma unroll
      for (int k = 0; k < VEC; ++k) { e[2 * k] = s0[k]; e[2 * k + 1] = s1[k]; }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * p.c; i += kThreads) {
    float t = 0.f;
    for (int y = 0; y < p.TY; ++y) t += sm[(size_t)2 * y * p.c + i];
    p.part[(s * p.slabs + slab) * 2 * p.c + i] = t;
  }
}

// one block per sample: joins the slabs per channel, then the channels per group
__global__ void __launch_bounds__(kThreads) norm_bwd_join_kernel(const NormParams p) {
  extern __shared__ float sm[];      // [c][2]
  const long long s = blockIdx.x;
  for (int i = threadIdx.x; i < 2 * p.c; i += kThreads) {
    float t = 0.f;
    for (int b = 0; b < p.slabs; ++b) t += p.part[(s * p.slabs + b) * 2 * p.c + i];
    sm[i] = t;
    p.csum[s * 2 * p.c + i] = t;
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float inv = 1.f / ((float)p.pix * (float)p.cg);
  for (int g = warp; g < p.groups; g += kThreads / 32) {
    float a = 0.f, b = 0.f;
    for (int i = lane; i < p.cg; i += 32) {
      const int ch = g * p.cg + i;
      a = fmaf(p.gamma[ch], sm[2 * ch], a);
      b = fmaf(p.gamma[ch], sm[2 * ch + 1], b);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, o);
      b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if (lane == 0) {
      p.gsum[2 * (s * p.groups + g)] = a * inv;
      p.gsum[2 * (s * p.groups + g) + 1] = b * inv;
    }
  }
}

// dgamma and dbeta: sums over the samples, one warp per channel
__global__ void __launch_bounds__(kThreads) norm_param_kernel(const NormParams p) {
  const int ch = (blockIdx.x * kThreads + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  if (ch >= p.c) return;
  float a = 0.f, b = 0.f;
  for (long long s = lane; s < p.n; s += 32) {
    a += p.csum[(s * p.c + ch) * 2];
    b += p.csum[(s * p.c + ch) * 2 + 1];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b += __shfl_xor_sync(0xffffffffu, b, o);
  }
  if (lane == 0) { p.dbeta[ch] = a; p.dgamma[ch] = b; }
}

template <int DT, int VEC>
__global__ void __launch_bounds__(kThreads) norm_bwd_apply_kernel(const NormParams p) {
  const int cv = p.c / VEC;
  const int tx = threadIdx.x % p.TX, ty = threadIdx.x / p.TX;
  if (ty >= p.TY) return;
  const long long s = blockIdx.x / p.slabs;
  const int slab = blockIdx.x % p.slabs;
  const int p0 = slab * p.slab_pix, p1 = min(p.pix, p0 + p.slab_pix);
  const long long base = (s * p.pix) * (long long)p.c;
  for (int v = tx; v < cv; v += p.TX) {
    const int g = v * VEC / p.cg;
    const long long sg = 2 * (s * p.groups + g);
    const float mean = p.stats[sg], rstd = p.stats[sg + 1], m0 = p.gsum[sg], m1 = p.gsum[sg + 1];
    float ga[VEC], be[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) { ga[k] = p.gamma[v * VEC + k]; be[k] = p.beta[v * VEC + k]; }
    for (int i = p0 + ty; i < p1; i += p.TY) {
      float a[VEC], dy[VEC];
      const long long e = base + (long long)i * p.c + v * VEC;
      Vec<DT, VEC>::load(p.x, e, a);
      Vec<DT, VEC>::load(p.dy, e, dy);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float xh = (a[k] - mean) * rstd;
        const float d = dy[k] * act_slope(fmaf(xh, ga[k], be[k]), p.act);
        a[k] = rstd * (fmaf(d, ga[k], -m0) - xh * m1);
      }
      Vec<DT, VEC>::store(p.out, e, a);
    }
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct NormPlan {
  int vec, TX, TY, slabs, slab_pix;
  size_t part, gsum, csum, total;      // workspace offsets in bytes
};

dk_status check_norm(const dk_norm* q) {
  if (!q) return DK_ERR_INVALID_ARG;
  if (q->act < DK_ACT_NONE || q->act > DK_ACT_SILU) return DK_ERR_INVALID_ARG;
  if (q->dtype != DK_F32 && q->dtype != DK_BF16) return DK_ERR_INVALID_ARG;
  if (!(q->eps >= 0.f)) return DK_ERR_INVALID_ARG;
  if (q->n < 0 || q->h < 1 || q->w < 1 || q->c < 1 || q->groups < 1) return DK_ERR_SHAPE;
  if (q->c > kMaxC || q->c % q->groups) return DK_ERR_SHAPE;
  const long long pix = (long long)q->h * q->w;
  if (pix >= (1LL << 31) || (double)q->n * (double)pix * q->c >= 1e15) return DK_ERR_SHAPE;
  return DK_OK;
}

NormPlan plan_norm(const dk_norm& q, int sms) {
  NormPlan p;
  const int cg = q.c / q.groups;
  p.vec = q.dtype == DK_F32 ? 4 : 8;
  while (cg % p.vec) p.vec /= 2;
  const int cv = q.c / p.vec;
  p.TX = cv < kThreads ? cv : kThreads;
  p.TY = kThreads / p.TX;
  const int pix = q.h * q.w;
  // slabs: at least four blocks per SM where the tensor has that much, each thread at least four pixels
  long long want = q.n > 0 ? (4LL * sms + q.n - 1) / q.n : 1;
  long long most = ((long long)pix + 4 * p.TY - 1) / (4 * p.TY);
  const long long least = ((long long)pix + 16LL * p.TY - 1) / (16LL * p.TY);   // 16 pixels a thread are enough
  if (want < least) want = least;
  if (want > most) want = most;
  if (want < 1) want = 1;
  p.slab_pix = (int)((pix + want - 1) / want);
  p.slabs = (pix + p.slab_pix - 1) / p.slab_pix;
  const size_t fwd = (size_t)q.n * p.slabs * q.groups * 3, bwd = (size_t)q.n * p.slabs * q.c * 2;
  size_t off = 0;
  p.part = off; off += ((fwd > bwd ? fwd : bwd) * sizeof(float) + 255) / 256 * 256;
  p.gsum = off; off += ((size_t)q.n * q.groups * 2 * sizeof(float) + 255) / 256 * 256;
  p.csum = off; off += ((size_t)q.n * q.c * 2 * sizeof(float) + 255) / 256 * 256;
  p.total = off;
  return p;
}

template <typename F>
dk_status with_smem(F kern, size_t bytes) {
  if (bytes > 48 * 1024 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) !=
                               cudaSuccess)
    return DK_ERR_CUDA;
  return DK_OK;
}

template <int DT, int VEC>
dk_status run_fwd(const NormParams& p, cudaStream_t st) {
  const size_t smem = (size_t)3 * p.TY * (p.c / VEC) * sizeof(float);
  if (with_smem(norm_stats_kernel<DT, VEC>, smem) != DK_OK) return DK_ERR_CUDA;
  const unsigned grid = (unsigned)(p.n * p.slabs);
  norm_stats_kernel<DT, VEC><<<grid, kThreads, smem, st>>>(p);
  norm_join_kernel<<<(unsigned)((p.n * p.groups * 32 + kThreads - 1) / kThreads), kThreads, 0, st>>>(p);
  norm_apply_kernel<DT, VEC><<<grid, kThreads, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? DK_OK : DK_ERR_CUDA;
}

template <int DT, int VEC>
dk_status run_bwd(const NormParams& p, cudaStream_t st) {
  const size_t smem = (size_t)2 * p.TY * p.c * sizeof(float), smem_j = (size_t)2 * p.c * sizeof(float);
  if (with_smem(norm_bwd_sums_kernel<DT, VEC>, smem) != DK_OK) return DK_ERR_CUDA;
  if (with_smem(norm_bwd_join_kernel, smem_j) != DK_OK) return DK_ERR_CUDA;
  const unsigned grid = (unsigned)(p.n * p.slabs);
  norm_bwd_sums_kernel<DT, VEC><<<grid, kThreads, smem, st>>>(p);
  norm_bwd_join_kernel<<<(unsigned)p.n, kThreads, smem_j, st>>>(p);
  norm_param_kernel<<<(unsigned)((p.c * 32 + kThreads - 1) / kThreads), kThreads, 0, st>>>(p);
  norm_bwd_apply_kernel<DT, VEC><<<grid, kThreads, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? DK_OK : DK_ERR_CUDA;
}

template <bool FWD>
dk_status dispatch(const NormParams& p, int dtype, int vec, cudaStream_t st) {
#define DK_NORM_CASE(DT, V) \
  if (dtype == DT && vec == V) return FWD ? run_fwd<DT, V>(p, st) : run_bwd<DT, V>(p, st)
  DK_NORM_CASE(DK_F32, 4);
  DK_NORM_CASE(DK_F32, 2);
  DK_NORM_CASE(DK_F32, 1);
  DK_NORM_CASE(DK_BF16, 8);
  DK_NORM_CASE(DK_BF16, 4);
  DK_NORM_CASE(DK_BF16, 2);
  DK_NORM_CASE(DK_BF16, 1);
#undef DK_NORM_CASE
  return DK_ERR_UNSUPPORTED;
}

dk_status begin(dk_ctx* ctx, const dk_norm* q, NormPlan* pl, NormParams* p) {
  *pl = plan_norm(*q, ctx->sm_count);
  if (!ctx->ws || ctx->ws_bytes < pl->total) return DK_ERR_WORKSPACE;
  if (q->n * pl->slabs >= (1LL << 31) || q->n * q->groups >= (1LL << 31) / 32) return DK_ERR_SHAPE;
  char* ws = static_cast<char*>(ctx->ws);
  p->part = reinterpret_cast<float*>(ws + pl->part);
  p->gsum = reinterpret_cast<float*>(ws + pl->gsum);
  p->csum = reinterpret_cast<float*>(ws + pl->csum);
  p->n = q->n;
  p->pix = q->h * q->w; p->c = q->c; p->groups = q->groups; p->cg = q->c / q->groups;
  p->slabs = pl->slabs; p->slab_pix = pl->slab_pix; p->act = q->act;
  p->TX = pl->TX; p->TY = pl->TY; p->eps = q->eps;
  return DK_OK;
}

}  // namespace
}  // namespace dk

using namespace dk;

extern "C" {

dk_status dk_norm_workspace_bytes(const dk_norm* q, size_t* bytes) {
  if (!bytes) return DK_ERR_INVALID_ARG;
  dk_status s = check_norm(q);
  if (s != DK_OK) return s;
  *bytes = plan_norm(*q, kMaxSms).total;
  return DK_OK;
}

dk_status dk_group_norm_fwd(dk_ctx* ctx, const dk_norm* q, const void* x, const float* gamma, const float* beta,
                            void* y, float* stats, void* stream) {
  dk_status s = check_norm(q);
  if (s != DK_OK) return s;
  if (!ctx) return DK_ERR_INVALID_ARG;
  if (q->n == 0) return DK_OK;              // (tensors without elements may be NULL)
  if (!x || !gamma || !beta || !y || !stats) return DK_ERR_INVALID_ARG;
  if (!aligned_to(x, 16) || !aligned_to(y, 16) || !aligned_to(gamma, 16) || !aligned_to(beta, 16) ||
      !aligned_to(stats, 16))
    return DK_ERR_INVALID_ARG;
  NormPlan pl;
  NormParams p = {};
  s = begin(ctx, q, &pl, &p);
  if (s != DK_OK) return s;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  p.x = x; p.out = y; p.gamma = gamma; p.beta = beta; p.stats = stats;
  ProfScope ps(ctx, DK_KERNEL_OTHER, 3, st);
  return dispatch<true>(p, q->dtype, pl.vec, st);
}

dk_status dk_group_norm_bwd(dk_ctx* ctx, const dk_norm* q, const void* dy, const void* x, const float* gamma,
                            const float* beta, const float* stats, void* dx, float* dgamma, float* dbeta,
                            void* stream) {
  dk_status s = check_norm(q);
  if (s != DK_OK) return s;
  if (!ctx || !dgamma || !dbeta) return DK_ERR_INVALID_ARG;
  if (q->n > 0 && (!dy || !x || !gamma || !beta || !stats || !dx)) return DK_ERR_INVALID_ARG;
  if (!aligned_to(dy, 16) || !aligned_to(x, 16) || !aligned_to(gamma, 16) || !aligned_to(beta, 16) ||
      !aligned_to(stats, 16) || !aligned_to(dx, 16) || !aligned_to(dgamma, 16) || !aligned_to(dbeta, 16))
    return DK_ERR_INVALID_ARG;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (q->n == 0) {
    DK_CUDA_CHECK(cudaMemsetAsync(dgamma, 0, (size_t)q->c * sizeof(float), st));
    DK_CUDA_CHECK(cudaMemsetAsync(dbeta, 0, (size_t)q->c * sizeof(float), st));
    return DK_OK;
  }
  NormPlan pl;
  NormParams p = {};
  s = begin(ctx, q, &pl, &p);
  if (s != DK_OK) return s;
  p.x = x; p.dy = dy; p.out = dx; p.gamma = gamma; p.beta = beta; p.stats = const_cast<float*>(stats);
  p.dgamma = dgamma; p.dbeta = dbeta;
  ProfScope ps(ctx, DK_KERNEL_OTHER, 4, st);
  return dispatch<false>(p, q->dtype, pl.vec, st);
}

}  // extern "C"
