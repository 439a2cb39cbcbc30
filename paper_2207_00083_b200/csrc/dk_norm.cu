// Group normalisation with an activation, channels-last, forward and backward.
//
//   z = (x - mean)*rstd*gamma + beta,  y = act(z),  statistics per sample and group of channels
//   d = dy*act'(z),  dgamma = sum d*xhat,  dbeta = sum d
//   dx = rstd*(q - mean(q) - xhat*mean(q*xhat)),  q = d*gamma
//
// Either direction needs sums over a sample before it can write its first value.
//   norm_sample_kernel: small items (a sample's pixels in a block of channels), one CTA each; the second reading
//     comes from L1 or L2.
//   norm_sums_kernel + norm_apply_kernel: larger samples in slabs, one CTA each.  The CTA that is the last of its
//     sample to leave its sums joins them (in the slabs' order, whichever CTA that is).
// HBM-bound; what it takes to get there is enough loads in flight: eight 16-byte loads per thread, up to 64 warps per
// SM, CTAs that live long enough (192 KiB slabs) for their start and their closing reduction not to count.  Measured on
// 64x224x224x64 bf16 (411 MB; a copy takes 137 us, a read 57): sums 76 us, values 137 us.  Reading once instead, with
// the slabs kept in shared memory or L2 until co-resident CTAs have exchanged their sums, was built four ways and took
// 375 to 614 us: the exchange leaves too few warps for every dependent step.  Chunks of samples that fit in L2, two
// launches each, took 290 to 670 us: each launch costs some 15 us of ramp and tail.
//
// Variance.  A thread's sums are taken about the first value of each batch of eight vectors, so cancellation is
// bounded by the few dozen values that share a pivot and not by how far the mean lies from zero; the (count, mean,
// sum of squared deviations) of batches, threads and slabs are then joined pairwise,
//   M2 = M2a + M2b + (mean_b - mean_a)^2 * na*nb/(na + nb).
#include "dk_ckpt8.cuh"
#include "dk_internal.h"
#include "dk_step.h"
#include "dk_vec.cuh"

namespace dk {
namespace {

constexpr int kThreads = 256;      // slab kernels
constexpr int kLoads = 8;          // vectors of one tensor a thread has in flight
constexpr int kMaxC = 16384;
// Pixels of an image: a loop's index passes the last pixel by less than a step, at most kLoads * 512 threads' pixels, and
// stays below 2^31.  (Unsigned indices would do without the limit and cost the backward sums 1 to 2 %.)
constexpr long long kMaxPix = (1LL << 31) - 4096;

// z*sigmoid(z) = z/(1 + exp(-z)): exp overflows to infinity for very negative z, the quotient is then -0
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == DK_ACT_NONE) return z;
  if (act == DK_ACT_RELU) return z < 0.f ? 0.f : z;        // (a NaN stays a NaN)
  return __fdividef(z, 1.f + __expf(-z));
}
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == DK_ACT_NONE) return 1.f;
  if (act == DK_ACT_RELU) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
  const float e = __expf(-fabsf(z)), r = __fdividef(1.f, 1.f + e);
  const float s = z >= 0.f ? r : e * r;                    // sigmoid(z), no overflow on either side
  return s * (1.f + z * (1.f - s));
}

struct NormParams {
  const void* x;          // (null where x comes from a checkpoint)
  const uint8_t* codes;   // the checkpoint: rows of dp codes, and the exponents of their blocks
  const uint8_t* exps;
  const void* dy;
  void* out;
  const float* gamma;
  const float* beta;
  float* stats;           // [n][groups][2]
  float* part;            // forward: [n][slabs][groups][3]; backward: [n][slabs][c][2]
  float* gsum;            // backward: [n][groups][2] means of q and q*xhat
  float* csum;            // backward: [rows][c][2], a row per sample (slab kernels) or per CTA of a channel block
  float* dgamma;
  float* dbeta;
  unsigned int* count;    // [n] slabs of a sample that have left their sums; zero between calls
  long long n;
  long long rows;         // of csum
  int pix, c, groups, cg, slabs, slab_pix, act;
  uint8_t* keep_codes;    // forward: the checkpoint that is written
  uint8_t* keep_exps;
  int dp;                 // codes of a checkpoint's row
  int TX, TY;             // threads along the channel vectors, and along the pixels
  int param_blocks;       // of norm_apply_kernel
  int cb;                 // channels of an item of norm_sample_kernel
  float eps;
};

// The vectors of x at one place of each pixel of a sample, as given (K8 = false) or from a checkpoint.
template <int DT, int VEC, bool K8>
struct XVectors;
template <int DT, int VEC>
struct XVectors<DT, VEC, false> {
  using Raw = typename Vec<DT, VEC>::Raw;
  const void* x;
  long long base;
  int c;
  __device__ __forceinline__ XVectors(const NormParams& p, long long, int, long long at) : x(p.x), base(at), c(p.c) {}
  __device__ __forceinline__ Raw get(int i) const { return Vec<DT, VEC>::get(x, base + (long long)i * c); }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[VEC]) { Vec<DT, VEC>::unpack(r, v); }
};
template <int DT, int VEC>
struct XVectors<DT, VEC, true> {
  using Raw = ckpt8::Raw<VEC>;
  const uint8_t* codes;
  const uint8_t* exps;
  int dp;
  __device__ __forceinline__ XVectors(const NormParams& p, long long s, int ch, long long)
      : codes(p.codes + s * p.pix * (long long)p.dp + ch),
        exps(p.exps + s * p.pix * (long long)(p.dp / ckpt8::kBlock) + ch / ckpt8::kBlock), dp(p.dp) {}
  __device__ __forceinline__ Raw get(int i) const {
    return ckpt8::get<VEC>(codes + (long long)i * dp, exps + (long long)i * (dp / ckpt8::kBlock));
  }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[VEC]) { ckpt8::unpack<VEC>(r, v); }
};

// where a vector of a sample's first pixel is kept
__device__ __forceinline__ uint8_t* kept_codes(const NormParams& p, long long s, int ch) {
  return p.keep_codes + s * p.pix * (long long)p.dp + ch;
}
__device__ __forceinline__ uint8_t* kept_exps(const NormParams& p, long long s, int ch) {
  return p.keep_exps + s * p.pix * (long long)(p.dp / ckpt8::kBlock) + ch / ckpt8::kBlock;
}

// Sums of the pixels [b, e) (every TY-th from ty on) of the channel vector at `base`: forward, about a pivot per batch.
template <int DT, int VEC>
__device__ __forceinline__ Moments sum_moments(const void* x, long long base, int b, int e, int c, int TY) {
  Moments tot{0.f, 0.f, 0.f};
  for (int i0 = b; i0 < e; i0 += kLoads * TY) {
    typename Vec<DT, VEC>::Raw raw[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      if (i0 + u * TY < e) raw[u] = Vec<DT, VEC>::get(x, base + (long long)(i0 + u * TY) * c);
    float pivot = 0.f, s1 = 0.f, s2 = 0.f;
    int cnt = 0;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      if (i0 + u * TY < e) {
        cnt += VEC;
        float a[VEC];
        Vec<DT, VEC>::unpack(raw[u], a);
        if (u == 0) pivot = a[0];
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float d = a[k] - pivot;
          s1 += d;
          s2 = fmaf(d, d, s2);
        }
      }
    }
    const float n = (float)cnt, m = __fdividef(s1, n);
    tot = join(tot, Moments{n, pivot + m, fmaxf(0.f, fmaf(-s1, m, s2))});
    if (!(s2 - s2 == 0.f)) tot.m2 = s2;      // (a NaN or an infinity is passed on, not clamped away)
  }
  return tot;
}

// The same for the backward pass: sums of d and d*xhat per channel of the vector.  z is formed by the very expression of
// write_values, so that at ReLU's kink the sums, dx and the forward call's y agree on which elements are active.
template <int DT, int VEC, int ACT, bool K8>
__device__ __forceinline__ void sum_gradients(const XVectors<DT, VEC, K8>& x, const void* dy, long long base, int b, int e, int c, int TY,
                                              const float (&mean)[VEC], const float (&rstd)[VEC],
                                              const float (&ga)[VEC], const float (&be)[VEC], float (&sb)[VEC],
                                              float (&sg)[VEC]) {
  constexpr int L = kLoads / 2;
  float f[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) f[k] = ga[k] * rstd[k];
  for (int i0 = b; i0 < e; i0 += L * TY) {
    typename XVectors<DT, VEC, K8>::Raw rx[L];
    typename Vec<DT, VEC>::Raw rd[L];
#pragma unroll
    for (int u = 0; u < L; ++u)
      if (i0 + u * TY < e) {
        rx[u] = x.get(i0 + u * TY);
        rd[u] = Vec<DT, VEC>::get(dy, base + (long long)(i0 + u * TY) * c);
      }
#pragma unroll
    for (int u = 0; u < L; ++u)
      if (i0 + u * TY < e) {
        float a[VEC], d[VEC];
        x.unpack(rx[u], a);
        Vec<DT, VEC>::unpack(rd[u], d);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float dev = a[k] - mean[k];
          const float t = d[k] * act_slope(fmaf(dev, f[k], be[k]), ACT);
          sb[k] += t;
          sg[k] = fmaf(t, dev * rstd[k], sg[k]);
        }
      }
  }
}

// The values of those pixels: y, or dx given the means m0 of q and m1 of q*xhat.  KEEP: and the checkpoint of x, whose blocks
// of 32 channels lie in neighbouring lanes of the same pixel (codes, exps: of this vector in the sample's first pixel).
template <int DT, int VEC, int ACT, bool FWD, bool K8, bool KEEP>
__device__ __forceinline__ void write_values(const XVectors<DT, VEC, K8>& x, const void* dy, void* out, long long base, int b, int e,
                                             int c, int TY, const float (&mean)[VEC], const float (&rstd)[VEC],
                                             const float (&m0)[VEC], const float (&m1)[VEC], const float (&ga)[VEC],
                                             const float (&be)[VEC], uint8_t* codes, uint8_t* exps, int dp) {
  constexpr int L = FWD || VEC < 8 ? 4 : 2;
  // z = (x - mean)*f + beta;  dx = rstd*((d*gamma - m0) - (x - mean)*c1)
  float f[VEC], c1[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) { f[k] = ga[k] * rstd[k]; c1[k] = rstd[k] * m1[k]; }
  for (int i0 = b; i0 < e; i0 += L * TY) {
    typename XVectors<DT, VEC, K8>::Raw rx[L];
    typename Vec<DT, VEC>::Raw rd[FWD ? 1 : L];
#pragma unroll
    for (int u = 0; u < L; ++u)
      if (i0 + u * TY < e) {
        rx[u] = x.get(i0 + u * TY);
        if constexpr (!FWD) rd[u] = Vec<DT, VEC>::get(dy, base + (long long)(i0 + u * TY) * c);
      }
#pragma unroll
    for (int u = 0; u < L; ++u)
      if (i0 + u * TY < e) {
        float a[VEC];
        x.unpack(rx[u], a);
        if constexpr (KEEP) {
          constexpr unsigned LANES = 32 / VEC == 32 ? 0xffffffffu : (1u << (32 / VEC)) - 1u;
          const int lane = threadIdx.x & 31;
          const ckpt8::Scale s = ckpt8::scale_of(ckpt8::block_most<VEC>(a, LANES << (lane & ~(32 / VEC - 1) & 31)));
          ckpt8::put_codes<VEC>(codes + (long long)(i0 + u * TY) * dp, a, s);
          if ((lane & (32 / VEC - 1)) == 0) exps[(long long)(i0 + u * TY) * (dp / ckpt8::kBlock)] = (uint8_t)s.byte;
        }
        if constexpr (FWD) {
#pragma unroll
          for (int k = 0; k < VEC; ++k) a[k] = act_value(fmaf(a[k] - mean[k], f[k], be[k]), ACT);
        } else {
          float d[VEC];
          Vec<DT, VEC>::unpack(rd[u], d);
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float t = a[k] - mean[k];
            const float q = d[k] * act_slope(fmaf(t, f[k], be[k]), ACT) * ga[k];
            a[k] = rstd[k] * ((q - m0[k]) - t * c1[k]);
          }
        }
        Vec<DT, VEC>::store(out, base + (long long)(i0 + u * TY) * c, a);
      }
  }
}

// Called by the whole CTA after its sums are in global memory: true in the CTA that is the sample's last (which leaves
// the counter at zero for the next call).
__device__ __forceinline__ bool last_to_arrive(const NormParams& p, long long s) {
  __shared__ unsigned int last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.count + s, 1u) + 1u == (unsigned int)p.slabs;
  __syncthreads();
  if (last) {
    __threadfence();
    if (threadIdx.x == 0) p.count[s] = 0u;
  }
  return last != 0u;
}

// Sums over the slabs b = r, r + R, ... of NC columns (every kThreads-th from i on) of [slabs][C2], in the slabs' order; U
// slabs' loads are in flight (one CTA reads them all, so it waits for L2 rather than for its bandwidth).
template <int U, int NC>
__device__ __forceinline__ void join_slabs(const float* part, int slabs, int C2, int r, int R, int i, float* to) {
  float t[NC];
#pragma unroll
  for (int k = 0; k < NC; ++k) t[k] = 0.f;
  for (int b = r; b < slabs; b += U * R) {
    float v[U][NC];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < NC; ++k)
        if (b + u * R < slabs && i + k * kThreads < C2) v[u][k] = __ldcg(part + (long long)(b + u * R) * C2 + i + k * kThreads);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < NC; ++k)
        if (b + u * R < slabs && i + k * kThreads < C2) t[k] += v[u][k];
  }
#pragma unroll
  for (int k = 0; k < NC; ++k)
    if (i + k * kThreads < C2) to[i + k * kThreads] = t[k];
}

// Sums of one slab.  Dynamic shared memory: forward [TY][c/VEC][3], backward [TY][c][2] floats.
template <int DT, int VEC, int ACT, bool FWD, bool K8>
__global__ void __launch_bounds__(kThreads) norm_sums_kernel(const NormParams p) {
  extern __shared__ float sm[];
  chained_launch();
  const int cv = p.c / VEC;
  const int tx = threadIdx.x % p.TX, ty = threadIdx.x / p.TX;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long s = blockIdx.x / p.slabs;
  const int slab = blockIdx.x % p.slabs;
  const int p0 = slab * p.slab_pix, p1 = (int)min((unsigned)p.pix, (unsigned)p0 + p.slab_pix);
  const long long base = s * p.pix * (long long)p.c;
  if (ty < p.TY) {
    for (int v = tx; v < cv; v += p.TX) {
      if constexpr (FWD) {
        const Moments m = sum_moments<DT, VEC>(p.x, base + v * VEC, p0 + ty, p1, p.c, p.TY);
        float* e = sm + 3 * ((size_t)ty * cv + v);
        e[0] = m.n; e[1] = m.mean; e[2] = m.m2;
      } else {
        float mean[VEC], rstd[VEC], ga[VEC], be[VEC], sb[VEC], sg[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float2 st = __ldg(reinterpret_cast<const float2*>(p.stats) + s * p.groups + (v * VEC + k) / p.cg);
          mean[k] = st.x; rstd[k] = st.y;
          ga[k] = __ldg(p.gamma + v * VEC + k); be[k] = __ldg(p.beta + v * VEC + k);
          sb[k] = sg[k] = 0.f;
        }
        sum_gradients<DT, VEC, ACT, K8>(XVectors<DT, VEC, K8>(p, s, v * VEC, base + v * VEC), p.dy, base + v * VEC, p0 + ty, p1, p.c, p.TY, mean, rstd, ga, be, sb, sg);
        float* e = sm + 2 * ((size_t)ty * p.c + v * VEC);
#pragma unroll
        for (int k = 0; k < VEC; ++k) { e[2 * k] = sb[k]; e[2 * k + 1] = sg[k]; }
      }
    }
  }
  __syncthreads();
  if constexpr (FWD) {
    const int vg = p.cg / VEC;
    for (int g = warp; g < p.groups; g += kThreads / 32) {
      Moments m{0.f, 0.f, 0.f};
      for (int i = lane; i < vg * p.TY; i += 32) {
        const float* e = sm + 3 * ((size_t)(i / vg) * cv + g * vg + i % vg);
        m = join(m, Moments{e[0], e[1], e[2]});
      }
      m = warp_join(m);
      if (lane == 0) {
        float* o = p.part + 3 * ((s * p.slabs + slab) * p.groups + g);
        __stcg(o, m.n); __stcg(o + 1, m.mean); __stcg(o + 2, m.m2);
      }
    }
    if (!last_to_arrive(p, s)) return;
    for (int g = warp; g < p.groups; g += kThreads / 32) {
      Moments m{0.f, 0.f, 0.f};
      for (int b = lane; b < p.slabs; b += 32) {
        const float* e = p.part + 3 * ((s * p.slabs + b) * p.groups + g);
        m = join(m, Moments{__ldcg(e), __ldcg(e + 1), __ldcg(e + 2)});
      }
      m = warp_join(m);
      if (lane == 0)
        reinterpret_cast<float2*>(p.stats)[s * p.groups + g] = make_float2(m.mean, 1.f / sqrtf(m.m2 / m.n + p.eps));
    }
  } else {
    for (int i = threadIdx.x; i < 2 * p.c; i += kThreads) {
      float t = 0.f;
      for (int y = 0; y < p.TY; ++y) t += sm[(size_t)2 * y * p.c + i];
      __stcg(p.part + (s * p.slabs + slab) * 2 * p.c + i, t);
    }
    if (!last_to_arrive(p, s)) return;
    // the sample's sums per channel: the slabs are dealt to R rows of threads, whose sums are joined in order
    const int C2 = 2 * p.c, R = C2 < kThreads ? kThreads / C2 : 1;
    const float* part = p.part + s * p.slabs * C2;
    if (C2 < kThreads) {
      const int r = (int)threadIdx.x / C2;
      if (r < R) join_slabs<8, 1>(part, p.slabs, C2, r, R, (int)threadIdx.x % C2, sm + r * C2);
    } else {
      for (int i0 = 0; i0 < C2; i0 += 2 * kThreads) join_slabs<8, 2>(part, p.slabs, C2, 0, 1, i0 + (int)threadIdx.x, sm);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < C2; i += kThreads) {
      float t = sm[i];
      for (int r = 1; r < R; ++r) t += sm[r * C2 + i];
      sm[i] = t;
      p.csum[s * C2 + i] = t;
    }
    __syncthreads();
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
      if (lane == 0) reinterpret_cast<float2*>(p.gsum)[s * p.groups + g] = make_float2(a * inv, b * inv);
    }
  }
}

// dgamma and dbeta of 16 channels: sums over the rows of csum, 16 threads each take every 16th row
__device__ __forceinline__ void param_sums(const NormParams& p, int block) {
  __shared__ float2 sm[16][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
  const int ch = block * 16 + x;
  float2 t = make_float2(0.f, 0.f);
  if (ch < p.c) {
#pragma unroll 8
    for (long long r = y; r < p.rows; r += 16) {
      const float2 v = __ldg(reinterpret_cast<const float2*>(p.csum) + r * p.c + ch);
      t.x += v.x; t.y += v.y;
    }
  }
  sm[y][x] = t;
  __syncthreads();
  if (y == 0 && ch < p.c) {
    for (int i = 1; i < 16; ++i) { t.x += sm[i][x].x; t.y += sm[i][x].y; }
    p.dbeta[ch] = t.x;
    p.dgamma[ch] = t.y;
  }
}
__global__ void __launch_bounds__(256) norm_param_kernel(const NormParams p) {
  chained_launch();
  param_sums(p, blockIdx.x);
}

// The values.  A vector may hold channels of several groups.  Backward: the first p.param_blocks CTAs form the
// parameters' gradients instead.
template <int DT, int VEC, int ACT, bool FWD, bool K8, bool KEEP>
__global__ void __launch_bounds__(kThreads) norm_apply_kernel(const NormParams p) {
  chained_launch();
  if constexpr (!FWD) {
    if ((int)blockIdx.x < p.param_blocks) {
      param_sums(p, blockIdx.x);
      return;
    }
  }
  const int cv = p.c / VEC;
  const int tx = threadIdx.x % p.TX, ty = threadIdx.x / p.TX;
  if (ty >= p.TY) return;
  // the slabs read last by the sums are taken first: they are the likeliest to be in L2 still
  const unsigned int block = gridDim.x - 1 - blockIdx.x;
  const long long s = block / p.slabs;
  const int slab = block % p.slabs;
  const int p0 = slab * p.slab_pix, p1 = (int)min((unsigned)p.pix, (unsigned)p0 + p.slab_pix);
  const long long base = s * p.pix * (long long)p.c;
  for (int v = tx; v < cv; v += p.TX) {
    float mean[VEC], rstd[VEC], m0[VEC], m1[VEC], ga[VEC], be[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const long long sg = s * p.groups + (v * VEC + k) / p.cg;
      const float2 st = __ldg(reinterpret_cast<const float2*>(p.stats) + sg);
      const float2 ms = FWD ? make_float2(0.f, 0.f) : __ldg(reinterpret_cast<const float2*>(p.gsum) + sg);
      mean[k] = st.x; rstd[k] = st.y; m0[k] = ms.x; m1[k] = ms.y;
      ga[k] = __ldg(p.gamma + v * VEC + k); be[k] = __ldg(p.beta + v * VEC + k);
    }
    write_values<DT, VEC, ACT, FWD, K8, KEEP>(XVectors<DT, VEC, K8>(p, s, v * VEC, base + v * VEC), p.dy, p.out, base + v * VEC, p0 + ty, p1, p.c,
                                              p.TY, mean, rstd, m0, m1, ga, be, kept_codes(p, s, v * VEC),
                                              kept_exps(p, s, v * VEC), p.dp);
  }
}

// Items that one CTA does by itself: all pixels of a sample in a block of p.cb channels (whole groups).  The grid is a
// multiple of the number of blocks, so a CTA keeps its channels.  Dynamic shared memory: [TY][cb/VEC][3] or, backward,
// [TY][cb][2], then [groups of a block][2].
constexpr int kSampleThreads = 512;
template <int DT, int VEC, int ACT, bool FWD, bool K8, bool KEEP>
__global__ void __launch_bounds__(kSampleThreads, 2) norm_sample_kernel(const NormParams p) {
  extern __shared__ float sm[];
  constexpr int NS = FWD ? 3 : 2;
  float* const st = sm + (FWD ? 3 * p.TY * p.TX : 2 * p.TY * p.cb);
  const int tx = threadIdx.x % p.TX, ty = threadIdx.x / p.TX;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const bool active = ty < p.TY;
  const int nblk = p.c / p.cb, blk = blockIdx.x % nblk, gpb = p.cb / p.cg, g0 = blk * gpb;
  const int ch0 = blk * p.cb + tx * VEC;                     // this thread's first channel
  const int g = active ? tx * VEC / p.cg : 0, vg = p.cg / VEC;      // its group within the block
  const float inv = 1.f / ((float)p.pix * (float)p.cg);
  float ga[VEC], be[VEC], cb[VEC], cg[VEC];      // cb, cg: this thread's part of dbeta and dgamma
#pragma unroll
  for (int k = 0; k < VEC; ++k) {
    ga[k] = active ? __ldg(p.gamma + ch0 + k) : 0.f;
    be[k] = active ? __ldg(p.beta + ch0 + k) : 0.f;
    cb[k] = cg[k] = 0.f;
  }
  for (long long s = blockIdx.x / nblk; s < p.n; s += gridDim.x / nblk) {
    const long long base = s * p.pix * (long long)p.c + ch0;
    float2 given = make_float2(0.f, 0.f);
    if (active) {
      float* e = sm + NS * (ty * p.TX + tx);
      if constexpr (FWD) {
        const Moments m = sum_moments<DT, VEC>(p.x, base, ty, p.pix, p.c, p.TY);
        e[0] = m.n; e[1] = m.mean; e[2] = m.m2;
      } else {
        given = __ldg(reinterpret_cast<const float2*>(p.stats) + s * p.groups + g0 + g);
        float sb[VEC], sg[VEC], a = 0.f, b = 0.f;
#pragma unroll
        for (int k = 0; k < VEC; ++k) sb[k] = sg[k] = 0.f;
        float mean[VEC], rstd[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) { mean[k] = given.x; rstd[k] = given.y; }
        sum_gradients<DT, VEC, ACT, K8>(XVectors<DT, VEC, K8>(p, s, ch0, base), p.dy, base, ty, p.pix, p.c, p.TY, mean, rstd, ga, be, sb, sg);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          cb[k] += sb[k]; cg[k] += sg[k];
          a = fmaf(ga[k], sb[k], a);
          b = fmaf(ga[k], sg[k], b);
        }
        e[0] = a; e[1] = b;
      }
    }
    __syncthreads();
    for (int gi = warp; gi < gpb; gi += warps) {
      Moments m{0.f, 0.f, 0.f};
      for (int i = lane; i < vg * p.TY; i += 32) {
        const float* e = sm + NS * ((i / vg) * p.TX + gi * vg + i % vg);
        if constexpr (FWD) m = join(m, Moments{e[0], e[1], e[2]});
        else { m.n += e[0]; m.mean += e[1]; }
      }
      if constexpr (FWD) {
        m = warp_join(m);
      } else {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          m.n += __shfl_xor_sync(0xffffffffu, m.n, o);
          m.mean += __shfl_xor_sync(0xffffffffu, m.mean, o);
        }
      }
      if (lane == 0) {
        const float2 r = FWD ? make_float2(m.mean, 1.f / sqrtf(m.m2 / m.n + p.eps)) : make_float2(m.n * inv, m.mean * inv);
        st[2 * gi] = r.x; st[2 * gi + 1] = r.y;
        if (FWD) reinterpret_cast<float2*>(p.stats)[s * p.groups + g0 + gi] = r;
      }
    }
    __syncthreads();
    if (active) {
      const float t0 = st[2 * g], t1 = st[2 * g + 1];
      float mean[VEC], rstd[VEC], m0[VEC], m1[VEC];
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        mean[k] = FWD ? t0 : given.x; rstd[k] = FWD ? t1 : given.y;
        m0[k] = t0; m1[k] = t1;
      }
      write_values<DT, VEC, ACT, FWD, K8, KEEP>(XVectors<DT, VEC, K8>(p, s, ch0, base), p.dy, p.out, base, ty, p.pix, p.c, p.TY, mean,
                                                rstd, m0, m1, ga, be, kept_codes(p, s, ch0), kept_exps(p, s, ch0), p.dp);
    }
    // (the next sample's sums go to `sm`, which was read before the second barrier; `st` is written after another one)
  }
  if constexpr (!FWD) {
    __syncthreads();
    if (active) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        sm[2 * (ty * p.cb + tx * VEC + k)] = cb[k];
        sm[2 * (ty * p.cb + tx * VEC + k) + 1] = cg[k];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.cb; i += blockDim.x) {
      float t = 0.f;
      for (int y = 0; y < p.TY; ++y) t += sm[2 * y * p.cb + i];
      p.csum[((size_t)(blockIdx.x / nblk) * p.c + blk * p.cb) * 2 + i] = t;
    }
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
constexpr long long kItemBytes = 128 * 1024;       // of x (and dy) in an item of norm_sample_kernel
constexpr long long kSampleTotal = 32LL << 20;     // of x (and dy) in the call
constexpr long long kSlabBytes = 192 * 1024;       // of x

struct NormPlan {
  int vec, wide;                       // channels of a vector within one group, and whatever the group
  int TX[2], TY[2];                    // of the slab kernels with either vector
  bool sample[2];                      // forward, backward: by norm_sample_kernel
  int cb, sTX, sTY, threads;           // of norm_sample_kernel
  int slabs, slab_pix;
  size_t part, gsum, csum, count, total;      // workspace offsets in bytes
};

dk_status check_norm(const dk_norm* q) {
  if (!q) return DK_ERR_INVALID_ARG;
  if (q->act < DK_ACT_NONE || q->act > DK_ACT_SILU) return DK_ERR_INVALID_ARG;
  if (q->dtype != DK_F32 && q->dtype != DK_BF16) return DK_ERR_INVALID_ARG;
  if (!(q->eps >= 0.f)) return DK_ERR_INVALID_ARG;
  if (q->n < 0 || q->h < 1 || q->w < 1 || q->c < 1 || q->groups < 1) return DK_ERR_SHAPE;
  if (q->c > kMaxC || q->c % q->groups) return DK_ERR_SHAPE;
  const long long pix = (long long)q->h * q->w;
  if (pix > kMaxPix || (double)q->n * (double)pix * q->c >= 1e15) return DK_ERR_SHAPE;
  return DK_OK;
}

constexpr int kSampleGrid = kMaxSms * 16;            // most CTAs of the sample kernel

NormPlan plan_norm(const dk_norm& q) {
  NormPlan p;
  const int es = q.dtype == DK_F32 ? 4 : 2;
  const int cg = q.c / q.groups;
  p.vec = 16 / es;
  while (cg % p.vec) p.vec /= 2;
  p.wide = 16 / es;
  while (q.c % p.wide) p.wide /= 2;
  const int pix = q.h * q.w;
  const long long bytes = (long long)q.c * pix * es;
  for (int w = 0; w < 2; ++w) {
    const int n = q.c / (w ? p.wide : p.vec);
    p.TX[w] = n < kThreads ? n : kThreads;
    p.TY[w] = kThreads / p.TX[w];
  }
  // Channel blocks of norm_sample_kernel: as few as give two items per SM, each with 128 bytes of a pixel (a line).
  int nblk = 1;
  for (int d = 1; d <= q.groups; ++d) {
    if (q.groups % d) continue;
    const int c = q.c / d;
    if (d > 1 && c * es < 128) break;
    nblk = d;
    if (q.n * d >= 2 * 148 && c / p.vec <= kSampleThreads) break;
  }
  p.cb = q.c / nblk;
  p.sTX = p.cb / p.vec;
  // threads: up to 512, four vectors each where the item has that many
  const long long vecs = (long long)p.sTX * pix;
  long long threads = (vecs + 3) / 4;
  if (threads > kSampleThreads) threads = kSampleThreads;
  if (threads < p.sTX) threads = p.sTX;
  p.sTY = (int)(threads / p.sTX);
  if (p.sTY < 1) p.sTY = 1;
  p.threads = (p.sTX * p.sTY + 31) / 32 * 32;
  // Taken for small items: one launch instead of two and no joining of slabs.  With more than kSampleTotal to move, two
  // launches whose CTAs stream longer are faster unless the items are tiny (3200x22x23x64 bf16: 160 against 110 us;
  // 128x14x14x256 fp32, 25 MB: 20 against 41; 8192 samples of 4 KiB: 59 against 102).
  for (int bwd = 0; bwd < 2; ++bwd) {
    const long long item = (long long)p.cb * pix * es * (1 + bwd), total = bytes * q.n * (1 + bwd);
    p.sample[bwd] = p.sTX <= kSampleThreads && item <= kItemBytes && (total <= kSampleTotal || item <= 16 * 1024);
  }
  // Slabs of the others: about kSlabBytes, and as many as make whole waves of four CTAs per SM (27x37x53x60 bf16
  // backward: 783 CTAs, 1.3 waves, 20.5 us; 567 CTAs, one wave, 18.4 us); but each thread four pixels.
  constexpr long long kWave = 4 * 148;
  long long waves = (long long)((double)q.n * (double)bytes / kSlabBytes / kWave + 0.5);
  if (waves < 1) waves = 1;
  long long want = q.n > 0 ? waves * kWave / q.n : 1;
  const long long most = ((long long)pix + 4 * p.TY[1] - 1) / (4 * p.TY[1]);
  if (want > most) want = most;
  if (want < 1) want = 1;
  p.slab_pix = (int)((pix + want - 1) / want);
  p.slabs = (int)(((long long)pix + p.slab_pix - 1) / p.slab_pix);
  size_t part = 0, rows_c = kSampleGrid;
  if (!p.sample[0]) part = (size_t)q.n * p.slabs * q.groups * 3;
  if (!p.sample[1]) {
    const size_t b = (size_t)q.n * p.slabs * q.c * 2;
    if (b > part) part = b;
    rows_c = (size_t)q.n;
  } else if ((size_t)q.n < rows_c) {
    rows_c = (size_t)q.n;
  }
  size_t off = 0;
  p.part = off; off += (part * sizeof(float) + 255) / 256 * 256;
  p.gsum = off; off += ((size_t)q.n * q.groups * 2 * sizeof(float) + 255) / 256 * 256;
  p.csum = off; off += (rows_c * q.c * 2 * sizeof(float) + 255) / 256 * 256;
  p.count = off; off += q.n > kStepCounters ? ((size_t)q.n * sizeof(unsigned int) + 255) / 256 * 256 : 0;
  p.total = off;
  return p;
}

// most dynamic shared memory of any call: the forward sums of kMaxC channels that share no vector
constexpr int kMaxSmem = 3 * kMaxC * (int)sizeof(float);

// whole samples: one launch, and one for the parameters' gradients
template <int DT, int VEC, int ACT, bool FWD, bool K8, bool KEEP>
dk_status run_sample(NormParams p, const NormPlan& pl, int device, int sms, cudaStream_t st) {
  auto kern = norm_sample_kernel<DT, VEC, ACT, FWD, K8, KEEP>;
  p.TX = pl.sTX; p.TY = pl.sTY; p.cb = pl.cb;
  const int nblk = p.c / p.cb;
  const size_t smem =
      ((FWD ? (size_t)3 * p.TY * p.TX : (size_t)2 * p.TY * p.cb) + 2 * (size_t)(p.cb / p.cg)) * sizeof(float);
  static SmemLimit limit;
  if (smem > 40 * 1024) {
    const dk_status r = allow_smem(limit, device, kern, kMaxSmem);
    if (r != DK_OK) return r;
  }
  long long per = (long long)(sms < kMaxSms ? sms : kMaxSms) * (2048 / pl.threads > 16 ? 16 : 2048 / pl.threads) / nblk;
  if (per < 1) per = 1;
  if (per > p.n) per = p.n;
  p.rows = per;
  kern<<<(unsigned)(per * nblk), pl.threads, smem, st>>>(p);
  if (cudaGetLastError() != cudaSuccess) return DK_ERR_CUDA;
  if (!FWD) DK_CUDA_CHECK(launch_chained(norm_param_kernel, dim3((unsigned)((p.c + 15) / 16)), 256, 0, st, p));
  return DK_OK;
}

// slabs: sums (forward with vectors within a group, backward per channel), then values
template <int DT, int VEC, int ACT, bool FWD, bool K8>
dk_status run_sums(NormParams p, const NormPlan& pl, int device, cudaStream_t st) {
  auto kern = norm_sums_kernel<DT, VEC, ACT, FWD, K8>;
  p.TX = pl.TX[FWD ? 0 : 1]; p.TY = pl.TY[FWD ? 0 : 1];
  size_t smem = FWD ? (size_t)3 * p.TY * (p.c / VEC) : (size_t)2 * p.TY * p.c;
  if (!FWD && smem < (size_t)2 * kThreads) smem = 2 * kThreads;
  smem *= sizeof(float);
  static SmemLimit limit;
  if (smem > 40 * 1024) {
    const dk_status r = allow_smem(limit, device, kern, kMaxSmem);
    if (r != DK_OK) return r;
  }
  return launch_chained(kern, dim3((unsigned)(p.n * p.slabs)), kThreads, smem, st, p) == cudaSuccess ? DK_OK
                                                                                                     : DK_ERR_CUDA;
}
template <int DT, int VEC, int ACT, bool FWD, bool K8, bool KEEP>
dk_status run_apply(NormParams p, const NormPlan& pl, cudaStream_t st) {
  p.TX = pl.TX[1]; p.TY = pl.TY[1];
  p.rows = p.n;
  p.param_blocks = FWD ? 0 : (p.c + 15) / 16;
  return launch_chained(norm_apply_kernel<DT, VEC, ACT, FWD, K8, KEEP>, dim3((unsigned)(p.n * p.slabs + p.param_blocks)), kThreads, 0,
                        st, p) == cudaSuccess
             ? DK_OK
             : DK_ERR_CUDA;
}

#define DK_NORM_ACTS(DT, V, CALL)                                       \
  do {                                                                  \
    if (p.act == DK_ACT_NONE) return CALL(DT, V, DK_ACT_NONE);          \
    if (p.act == DK_ACT_RELU) return CALL(DT, V, DK_ACT_RELU);          \
    return CALL(DT, V, DK_ACT_SILU);                                    \
  } while (0)
#define DK_NORM_TYPES(VECTOR, CALL)                                     \
  do {                                                                  \
    if (dtype == DK_F32) {                                              \
      if ((VECTOR) == 4) DK_NORM_ACTS(DK_F32, 4, CALL);                 \
      if ((VECTOR) == 2) DK_NORM_ACTS(DK_F32, 2, CALL);                 \
      DK_NORM_ACTS(DK_F32, 1, CALL);                                    \
    }                                                                   \
    if ((VECTOR) == 8) DK_NORM_ACTS(DK_BF16, 8, CALL);                  \
    if ((VECTOR) == 4) DK_NORM_ACTS(DK_BF16, 4, CALL);                  \
    if ((VECTOR) == 2) DK_NORM_ACTS(DK_BF16, 2, CALL);                  \
    DK_NORM_ACTS(DK_BF16, 1, CALL);                                     \
  } while (0)

template <bool FWD, bool K8, bool KEEP>
dk_status dispatch_sample(const NormParams& p, const NormPlan& pl, int dtype, int device, int sms, cudaStream_t st) {
#define DK_NORM_CALL(DT, V, ACT) run_sample<DT, V, ACT, FWD, K8, KEEP>(p, pl, device, sms, st)
  DK_NORM_TYPES(pl.vec, DK_NORM_CALL);
#undef DK_NORM_CALL
}
template <bool FWD, bool K8>
dk_status dispatch_sums(const NormParams& p, const NormPlan& pl, int dtype, int device, cudaStream_t st) {
#define DK_NORM_CALL(DT, V, ACT) run_sums<DT, V, FWD ? DK_ACT_NONE : ACT, FWD, K8>(p, pl, device, st)
  DK_NORM_TYPES(FWD ? pl.vec : pl.wide, DK_NORM_CALL);
#undef DK_NORM_CALL
}
template <bool FWD, bool K8, bool KEEP>
dk_status dispatch_apply(const NormParams& p, const NormPlan& pl, int dtype, cudaStream_t st) {
#define DK_NORM_CALL(DT, V, ACT) run_apply<DT, V, ACT, FWD, K8, KEEP>(p, pl, st)
  DK_NORM_TYPES(pl.wide, DK_NORM_CALL);
#undef DK_NORM_CALL
}

template <bool FWD, bool K8, bool KEEP>
dk_status dispatch(const NormParams& p, const NormPlan& pl, int dtype, int device, int sms, cudaStream_t st) {
  if (pl.sample[FWD ? 0 : 1]) return dispatch_sample<FWD, K8, KEEP>(p, pl, dtype, device, sms, st);
  if (p.n > kStepCounters) DK_CUDA_CHECK(cudaMemsetAsync(p.count, 0, (size_t)p.n * sizeof(unsigned int), st));
  const dk_status s = dispatch_sums<FWD, K8>(p, pl, dtype, device, st);
  return s == DK_OK ? dispatch_apply<FWD, K8, KEEP>(p, pl, dtype, st) : s;
}

dk_status begin(dk_ctx* ctx, const dk_norm* q, NormPlan* pl, NormParams* p) {
  *pl = plan_norm(*q);
  if (!ctx->ws || ctx->ws_bytes < pl->total) return DK_ERR_WORKSPACE;
  if (q->n * pl->slabs >= (1LL << 31)) return DK_ERR_SHAPE;
  char* ws = static_cast<char*>(ctx->ws);
  p->part = reinterpret_cast<float*>(ws + pl->part);
  p->gsum = reinterpret_cast<float*>(ws + pl->gsum);
  p->csum = reinterpret_cast<float*>(ws + pl->csum);
  p->count = q->n > kStepCounters ? reinterpret_cast<unsigned int*>(ws + pl->count) : step_counters(ctx);
  p->n = q->n;
  p->pix = q->h * q->w; p->c = q->c; p->groups = q->groups; p->cg = q->c / q->groups;
  p->slabs = pl->slabs; p->slab_pix = pl->slab_pix; p->act = q->act;
  p->eps = q->eps;
  return DK_OK;
}

// kernels of a call, for the launch counters
int launches(const NormPlan& pl, bool fwd) { return pl.sample[fwd ? 0 : 1] && fwd ? 1 : 2; }

// kept: a checkpoint of x is written too
dk_status norm_forward(dk_ctx* ctx, const dk_norm* q, const void* x, const float* gamma, const float* beta, void* y,
                       float* stats, void* ckpt, bool kept, void* stream) {
  dk_status s = check_norm(q);
  if (s != DK_OK) return s;
  if (!ctx) return DK_ERR_INVALID_ARG;
  if (q->n == 0) return DK_OK;              // (tensors without elements may be NULL)
  if (!x || !gamma || !beta || !y || !stats || (kept && !ckpt)) return DK_ERR_INVALID_ARG;
  if (!aligned_to(x, 16) || !aligned_to(y, 16) || !aligned_to(gamma, 16) || !aligned_to(beta, 16) ||
      !aligned_to(stats, 16) || !aligned_to(ckpt, 16))
    return DK_ERR_INVALID_ARG;
  NormPlan pl;
  NormParams p = {};
  s = begin(ctx, q, &pl, &p);
  if (s != DK_OK) return s;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  p.x = x; p.out = y; p.gamma = gamma; p.beta = beta; p.stats = stats;
  // A checkpoint is written with the values where its blocks of 32 channels lie in one warp: whole blocks in a pixel and, for
  // items of blocks of channels, in an item.  Else by a launch of its own, first: y may be x.  (64x56x56x64 fp32, both
  // directions: 99 us with two launches, 92 with one; 27x37x53x60 takes two.)
  const bool with = kept && q->c % ckpt8::kBlock == 0 && (!pl.sample[0] || pl.cb % ckpt8::kBlock == 0);
  ProfScope ps(ctx, DK_KERNEL_OTHER, launches(pl, true) + (kept && !with ? 1 : 0), st);
  if (with) {
    p.keep_codes = static_cast<uint8_t*>(ckpt);
    p.keep_exps = p.keep_codes + ckpt8::code_bytes(q->n * p.pix, q->c);
    p.dp = q->c;
    return dispatch<true, false, true>(p, pl, q->dtype, ctx->device, ctx->sm_count, st);
  }
  if (kept) {
    const dk_ckpt8 k{q->n * p.pix, q->c, q->dtype};
    s = launch_ckpt8(k, true, x, nullptr, ckpt, ctx->sm_count, st);
    if (s != DK_OK) return s;
  }
  return dispatch<true, false, false>(p, pl, q->dtype, ctx->device, ctx->sm_count, st);
}

// K8: x is a checkpoint
template <bool K8>
dk_status norm_backward(dk_ctx* ctx, const dk_norm* q, const void* dy, const void* x, const float* gamma,
                        const float* beta, const float* stats, void* dx, float* dgamma, float* dbeta, void* stream) {
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
  if (K8) {
    p.dp = ckpt8::padded(q->c);
    p.codes = static_cast<const uint8_t*>(x);
    p.exps = p.codes + ckpt8::code_bytes(q->n * p.pix, q->c);
  } else {
    p.x = x;
  }
  p.dy = dy; p.out = dx; p.gamma = gamma; p.beta = beta; p.stats = const_cast<float*>(stats);
  p.dgamma = dgamma; p.dbeta = dbeta;
  ProfScope ps(ctx, DK_KERNEL_OTHER, launches(pl, false), st);
  return dispatch<false, K8, false>(p, pl, q->dtype, ctx->device, ctx->sm_count, st);
}

}  // namespace
}  // namespace dk

using namespace dk;

extern "C" {

dk_status dk_norm_workspace_bytes(const dk_norm* q, size_t* bytes) {
  if (!bytes) return DK_ERR_INVALID_ARG;
  dk_status s = check_norm(q);
  if (s != DK_OK) return s;
  *bytes = plan_norm(*q).total;
  return DK_OK;
}

dk_status dk_group_norm_fwd(dk_ctx* ctx, const dk_norm* q, const void* x, const float* gamma, const float* beta,
                            void* y, float* stats, void* stream) {
  return norm_forward(ctx, q, x, gamma, beta, y, stats, nullptr, false, stream);
}

dk_status dk_group_norm_fwd_ckpt8(dk_ctx* ctx, const dk_norm* q, const void* x, const float* gamma, const float* beta,
                                  void* y, float* stats, void* ckpt, void* stream) {
  return norm_forward(ctx, q, x, gamma, beta, y, stats, ckpt, true, stream);
}

dk_status dk_group_norm_bwd(dk_ctx* ctx, const dk_norm* q, const void* dy, const void* x, const float* gamma,
                            const float* beta, const float* stats, void* dx, float* dgamma, float* dbeta,
                            void* stream) {
  return norm_backward<false>(ctx, q, dy, x, gamma, beta, stats, dx, dgamma, dbeta, stream);
}

dk_status dk_group_norm_bwd_ckpt8(dk_ctx* ctx, const dk_norm* q, const void* dy, const void* ckpt, const float* gamma,
                                  const float* beta, const float* stats, void* dx, float* dgamma, float* dbeta,
                                  void* stream) {
  return norm_backward<true>(ctx, q, dy, ckpt, gamma, beta, stats, dx, dgamma, dbeta, stream);
}

}  // extern "C"
