// The orthogonalised update: Newton-Schulz products on the tensor cores.
//
//   X = x/(|x|_F + eps);   per step  A = X X^T,  B = a I + b A + c A A,  X = B X;   out = keep*out + scale*X
// (from the right, A = X^T X and X = X B, when the matrix is tall: A always has the shorter side.)
//
// fp32 accuracy throughout: X, A and B are kept as two fp16 terms under fixed powers of two (|X|_F <= 1 to begin with
// and the polynomial keeps every singular value below sqrt(2), so the ranges are known), three products per step, fp32
// sums.  16 bits alone would not do: the polynomial multiplies small singular values by a at every step (485 times
// over five), and the rounding of the large ones with them.  A and A A are symmetric, so only the tiles on and below
// the diagonal are formed.
#include <math.h>

#include <type_traits>

#include "dk_gemm16.cuh"

namespace dk {
namespace {

using g16::Operand;
using g16::Params;

constexpr int BN = 256;
constexpr int kSumBlocks = 1184;                 // partial sums of squares per matrix
// powers of two of the stored terms: |X| < 8, |A| < 8, |B| < 32
constexpr float kX = 8192.f, kA = 8192.f, kB = 2048.f;

template <int DT>
__device__ __forceinline__ float load1(const void* p, size_t i) {
  if constexpr (DT == DK_F32) return __ldg(static_cast<const float*>(p) + i);
  else return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

// sums of squares in fp64: neither tiny nor huge gradients leave its range
template <int DT>
__global__ void __launch_bounds__(256) ortho_sumsq_kernel(const void* x, long long per, double* part) {
  chained_launch();
  __shared__ double s[8];
  constexpr int V = DT == DK_F32 ? 4 : 8;              // elements of 16 bytes
  constexpr int U = 4;                                 // loads in flight
  const size_t base = (size_t)blockIdx.y * per;
  // (every matrix but the first may start off a 16-byte boundary)
  const long long head = (long long)((V - base % V) % V) < per ? (long long)((V - base % V) % V) : per;
  const long long vecs = (per - head) / V;
  const uint4* xv = reinterpret_cast<const uint4*>(static_cast<const char*>(x) + (base + head) * (16 / V));
  double t = 0.0;
  auto add = [&](double v) { t = fma(v, v, t); };
  const long long step = (long long)gridDim.x * 256;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < vecs; i += U * step) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = i + u * step < vecs ? __ldg(xv + i + u * step) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (DT == DK_F32) {
          add((double)__uint_as_float(w[k]));
        } else {
          add((double)__uint_as_float(w[k] << 16));
          add((double)__uint_as_float(w[k] & 0xffff0000u));
        }
      }
    }
  }
  if (blockIdx.x == 0) {
    if ((long long)threadIdx.x < head) add((double)load1<DT>(x, base + threadIdx.x));
    const long long rest = head + vecs * V + threadIdx.x;
    if (rest < per && (long long)threadIdx.x < V) add((double)load1<DT>(x, base + rest));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 8; ++i) t += s[i];
    part[blockIdx.y * gridDim.x + blockIdx.x] = t;
  }
}

// What brings x to |X|_F = 1 and to X's power of two: x*f.x*f.y, where f.x is a power of two.  One fp32 factor would be
// infinite for norms (and eps) below 2^-115, and the zeros of x then NaN, and subnormal above 2^139.  (In 64 bits the
// kernel of the smallest matrices takes 1 us longer.)
__device__ __forceinline__ float2 norm_factor(double sum_of_squares, double eps) {
  const double f = (double)kX / (sqrt(sum_of_squares) + eps);
  const float p = f > 0x1p64 ? 0x1p64f : f < 0x1p-64 ? 0x1p-64f : 1.f;
  return make_float2(p, (float)(f / (double)p));
}

// X as two fp16 terms, rows padded to `pitch` with zeros
template <int DT>
__global__ void __launch_bounds__(256)
ortho_load_kernel(const void* x, const double* part, int nparts, double eps, long long m, int n, int pitch, __half* hi,
                  __half* lo) {
  chained_launch();
  __shared__ float2 f;
  if (threadIdx.x < 32) {
    double t = 0.0;
    for (int i = threadIdx.x; i < nparts; i += 32) t += part[blockIdx.y * nparts + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (threadIdx.x == 0) f = norm_factor(t, eps);
  }
  __syncthreads();
  const float2 fac = f;
  const int n8 = pitch / 8;
  const size_t src = (size_t)blockIdx.y * m * n, dst = (size_t)blockIdx.y * m * pitch;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < m * n8; i += (long long)gridDim.x * 256) {
    const long long r = i / n8;
    const int c = (int)(i - r * n8) * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < n ? load1<DT>(x, src + (size_t)r * n + c + j) * fac.x * fac.y : 0.f;
    g16::store_planes<8>(hi + dst + r * pitch + c, lo + dst + r * pitch + c, v, 8);
  }
}

// Joins the slices of a symmetric product (its tiles on and below the diagonal) in order and writes both halves as two
// fp16 terms: poly = 0: A = sum * f;  1: B = (a I + b A + c*sum*f) * kB with A from its own terms.
struct SymArgs {
  const float* part;
  int ks, nbatch, s, pitch_part, pitch;
  float f;
  int poly;
  float a, b, c;
  const __half* a_hi;
  const __half* a_lo;
  __half* hi;
  __half* lo;
};
__global__ void __launch_bounds__(256) ortho_sym_kernel(const SymArgs q) {
  chained_launch();
  __shared__ float tile[32][33];
  const int bi = blockIdx.y, bj = blockIdx.x, batch = blockIdx.z;
  if (bj > bi) return;
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const size_t plane = (size_t)batch * q.s * q.pitch;
  const size_t slice = (size_t)q.nbatch * q.s * q.pitch_part;
  for (int r = ty; r < 32; r += 8) {
    const int i = bi * 32 + r, j = bj * 32 + tx;
    float v = 0.f;
    if (i < q.s && j < q.s) {
      const size_t at = ((size_t)batch * q.s + i) * q.pitch_part + j;
      v = q.part[at];
      for (int k = 1; k < q.ks; ++k) v += q.part[at + k * slice];
      v *= q.f;
      if (q.poly) {
        const size_t e = plane + (size_t)i * q.pitch + j;
        const float av = (__half2float(q.a_hi[e]) + __half2float(q.a_lo[e])) * (1.f / kA);
        v = fmaf(q.c, v, q.b * av);
        if (i == j) v += q.a;
        v *= kB;
      }
    }
    tile[r][tx] = v;
  }
  __syncthreads();
  for (int r = ty; r < 32; r += 8) {
    // below (or on) the diagonal as formed, above it mirrored
    int i = bi * 32 + r, j = bj * 32 + tx;
    float v = (bi == bj && tx > r) ? tile[tx][r] : tile[r][tx];
    if (i < q.s && j < q.pitch) {
      const __half h = __float2half_rn(v);
      q.hi[plane + (size_t)i * q.pitch + j] = h;
      q.lo[plane + (size_t)i * q.pitch + j] = __float2half_rn(v - __half2float(h));
    }
    if (bi != bj) {
      i = bj * 32 + r; j = bi * 32 + tx;
      v = tile[tx][r];
      if (i < q.s && j < q.pitch) {
        const __half h = __float2half_rn(v);
        q.hi[plane + (size_t)i * q.pitch + j] = h;
        q.lo[plane + (size_t)i * q.pitch + j] = __float2half_rn(v - __half2float(h));
      }
    }
  }
}

// The same from a product that is finished where it is formed (tiles of the small kernel): this thread's NH columns of
// its row, on or below the diagonal, and their mirror images.
struct EpiSym {
  static constexpr bool kAhead = true;
  SymArgs q;
  // A at this thread's columns (both terms of each in a word), from the mirrored positions: neighbours across the lanes
  template <int NH>
  __device__ __forceinline__ void fetch(int batch, int row, int col0, uint32_t (&a)[NH]) const {
    const size_t mirror = (size_t)batch * q.s * q.pitch + (size_t)col0 * q.pitch + row;
    const uint16_t* hi = reinterpret_cast<const uint16_t*>(q.a_hi) + mirror;
    const uint16_t* lo = reinterpret_cast<const uint16_t*>(q.a_lo) + mirror;
    const int last = q.poly ? min(NH - 1, (row < q.s ? row : -1) - col0) : -1;
#pragma unroll
    for (int j = 0; j < NH; ++j) {
      a[j] = 0u;
      if (j <= last) a[j] = (uint32_t)hi[(size_t)j * q.pitch] | (uint32_t)lo[(size_t)j * q.pitch] << 16;
    }
  }
  template <int NH>
  __device__ __forceinline__ void operator()(const Params&, float (&acc)[NH], int batch, int row, int col0, char* sm,
                                             const uint32_t (&a)[NH]) const {
    const int lane = threadIdx.x & 31, row0 = row - lane;
    if (row0 >= q.s || col0 >= q.s || col0 > row0 + 31) return;      // (nothing there on or below the diagonal)
    const size_t plane = (size_t)batch * q.s * q.pitch;
#pragma unroll
    for (int j = 0; j < NH; ++j) {
      float v = acc[j] * q.f;
      if (q.poly) {
        const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&a[j]));
        v = fmaf(q.c, v, q.b * ((t.x + t.y) * (1.f / kA)));
        if (col0 + j == row) v += q.a;
        v *= kB;
      }
      acc[j] = v;
    }
    const size_t to = plane + (size_t)row0 * q.pitch + col0;
    constexpr int W = NH < 32 ? NH : 32;
#pragma unroll
    for (int c0 = 0; c0 < NH; c0 += W) {
      uint32_t h[W / 2], l[W / 2];
      g16::to_terms<W>(acc, c0, h, l);
      // elements on and below the diagonal only: what lies above it is the mirror image of others
      auto put = [&](__half* dst, int r, int c, const uint4& u) {
        const int count = min(row0 + r, q.s - 1) - (col0 + c0 + c) + 1;
        if (row0 + r < q.s && count > 0) g16::put_piece16(dst + to + (size_t)r * q.pitch + c0 + c, u, count);
      };
      g16::warp_block_16<W>(h, sm, [&](int r, int c, const uint4& u) { put(q.hi, r, c, u); });
      g16::warp_block_16<W>(l, sm, [&](int r, int c, const uint4& u) { put(q.lo, r, c, u); });
      // the mirror image: both terms of an element in a word, [column][row], and eight rows of a column to a store
      uint32_t* words = reinterpret_cast<uint32_t*>(sm);
      __syncwarp();
#pragma unroll
      for (int j = 0; j < W; ++j)
        words[j * 32 + lane] = j & 1 ? __byte_perm(h[j / 2], l[j / 2], 0x7632) : __byte_perm(h[j / 2], l[j / 2], 0x5410);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < W / 8; ++i) {
        const int c = i * 8 + lane / 4, r = (lane % 4) * 8, col = col0 + c0 + c;
        const uint4 u = *reinterpret_cast<const uint4*>(words + c * 32 + r), v = *reinterpret_cast<const uint4*>(words + c * 32 + r + 4);
        const uint4 hi = make_uint4(__byte_perm(u.x, u.y, 0x5410), __byte_perm(u.z, u.w, 0x5410),
                                    __byte_perm(v.x, v.y, 0x5410), __byte_perm(v.z, v.w, 0x5410));
        const uint4 lo = make_uint4(__byte_perm(u.x, u.y, 0x7632), __byte_perm(u.z, u.w, 0x7632),
                                    __byte_perm(v.x, v.y, 0x7632), __byte_perm(v.z, v.w, 0x7632));
        const int first = row0 + r;
        if (col >= q.s || first >= q.s) continue;
        const size_t at = plane + (size_t)col * q.pitch + first;
        if (col < first) {                 // strictly below the diagonal (the pitch has room for whole pieces)
          *reinterpret_cast<uint4*>(q.hi + at) = hi;
          *reinterpret_cast<uint4*>(q.lo + at) = lo;
        } else {
          const uint32_t hw[4] = {hi.x, hi.y, hi.z, hi.w}, lw[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (first + k < q.s && first + k > col) {
              reinterpret_cast<uint16_t*>(q.hi)[at + k] = (uint16_t)(k & 1 ? hw[k / 2] >> 16 : hw[k / 2] & 0xffffu);
              reinterpret_cast<uint16_t*>(q.lo)[at + k] = (uint16_t)(k & 1 ? lw[k / 2] >> 16 : lw[k / 2] & 0xffffu);
            }
          }
        }
      }
    }
  }
};

// the result of a step: the next X as two terms (hi given), or the update itself
struct XArgs {
  __half* hi;
  __half* lo;
  long long pitch;             // of the terms
  void* out;
  int n, dtype;                // (dtype: ortho_x_kernel's)
  float f;                     // undoes the operands' powers of two (and brings X to its own)
  float scale, keep;
};
constexpr int kTerms = 2;            // OUT: DK_F32, DK_BF16 or this
template <int OUT>
struct EpiX {
  static constexpr bool kAhead = false;
  XArgs a;
  template <int NH>
  __device__ __forceinline__ void operator()(const Params& p, float (&acc)[NH], int batch, int, int row, int col0,
                                             char* sm) const {
    const int row0 = row - (int)(threadIdx.x & 31);
    if (row0 >= p.M || col0 >= p.N) return;
    const size_t first = (size_t)batch * p.M + row0;
    const int rows = p.M - row0, cols = p.N - col0;
    const float f = OUT == kTerms ? a.f : a.f * a.scale;
#pragma unroll
    for (int j = 0; j < NH; ++j) acc[j] *= f;
    const size_t to = first * (OUT == kTerms ? a.pitch : (long long)a.n) + col0;
    if constexpr (OUT == kTerms) {
      g16::store_terms<NH>(acc, sm, a.hi + to, a.lo + to, a.pitch, rows, cols);
    } else if constexpr (OUT == DK_F32) {
      float* out = static_cast<float*>(a.out) + to;
      g16::warp_rows_f32<NH>(acc, sm, [&](int r, int c, float4 u) {
        if (r >= rows || c >= cols) return;
        float* o = out + (size_t)r * a.n + c;
        if (a.keep != 0.f) {
          u.x = fmaf(a.keep, o[0], u.x);
          if (c + 1 < cols) u.y = fmaf(a.keep, o[1], u.y);
          if (c + 2 < cols) u.z = fmaf(a.keep, o[2], u.z);
          if (c + 3 < cols) u.w = fmaf(a.keep, o[3], u.w);
        }
        g16::put_piece32(o, u, cols - c);
      });
    } else {
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + to;
      if (a.keep != 0.f) {
#pragma unroll
        for (int j = 0; j < NH; ++j)
          if (row < p.M && j < cols) acc[j] = fmaf(a.keep, __bfloat162float(out[(size_t)(row - row0) * a.n + j]), acc[j]);
      }
      g16::warp_rows_bf16<NH>(acc, sm, [&](int r, int c, const uint4& u) {
        if (r < rows && c < cols) g16::put_piece16(out + (size_t)r * a.n + c, u, cols - c);
      });
    }
  }
};

// the same from slices of the contraction (part given), or from X's own terms (no step at all)
__global__ void __launch_bounds__(256)
ortho_x_kernel(const XArgs a, const float* part, int ks, int pitch_part, const __half* x_hi, const __half* x_lo,
               long long rows, int pitch_x) {
  chained_launch();
  const int n8 = (a.n + 7) / 8;
  const size_t slice = (size_t)rows * pitch_part;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows * n8; i += (long long)gridDim.x * 256) {
    const long long r = i / n8;
    const int c = (int)(i - r * n8) * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = 0.f;
      if (c + j < a.n) {
        if (part != nullptr) {
          const size_t at = (size_t)r * pitch_part + c + j;
          v[j] = part[at];
          for (int k = 1; k < ks; ++k) v[j] += part[at + k * slice];
        } else {
          const size_t at = (size_t)r * pitch_x + c + j;
          v[j] = __half2float(x_hi[at]) + __half2float(x_lo[at]);
        }
        v[j] *= a.f;
      }
    }
    if (a.hi != nullptr) {
      g16::store_planes<8>(a.hi + r * a.pitch + c, a.lo + r * a.pitch + c, v, 8);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (c + j >= a.n) break;
        const size_t e = (size_t)r * a.n + c + j;
        if (a.dtype == DK_F32) {
          float* o = static_cast<float*>(a.out) + e;
          *o = a.keep != 0.f ? fmaf(a.keep, *o, a.scale * v[j]) : a.scale * v[j];
        } else {
          __nv_bfloat16* o = static_cast<__nv_bfloat16*>(a.out) + e;
          *o = __float2bfloat16_rn(a.keep != 0.f ? fmaf(a.keep, __bfloat162float(*o), a.scale * v[j]) : a.scale * v[j]);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Short sides of at most 128: the whole call in one kernel.  What bounds such matrices is not the products but 15
// launches of them, one after the other.  Here a gang of co-resident CTAs holds the matrix, each `C` columns (of the
// wide orientation) as two fp16 terms in shared memory for all steps.  Per step a CTA forms its columns' share of A on
// the tensor core and leaves it in global memory; the gang meets; every CTA adds the shares up (gangs of more than
// kDirect first add up a slice each and meet again), forms B = a I + b A + c A A by itself, and multiplies its own
// columns.  One block layout serves all three products: [128 rows][64 columns], 128-byte rows swizzled, is the K-major
// operand of X X^T and the MN-major operand of B X.
// ---------------------------------------------------------------------------
constexpr int kResThreads = 256;
constexpr int kMaxColumns = 256;        // of a CTA
constexpr int kDirect = 28 * 1024;      // elements of A times CTAs of the gang

constexpr int kBlock = 128 * 128;            // bytes of one [128][64] fp16 block
// What the tensor pipe loses per 16 contraction elements, one instruction (see kLossSquares).  What it gives back is an
// average; in A A, which the polynomial's first steps amplify most, what is left is halved by three accumulators
// (against plain fp32, 64x576: 1.5 times its error with one, 0.9 with three; 128x1152: 1.2 and 0.75; 2 us of 120).
// (A A's own constant is the best of 0, 0.3, .. 1.7 over short sides of 16 to 128.)
constexpr float kResLossSquares = 1.1f / 16777216.f, kResLossAA = 1.5f / 16777216.f, kResLossMixed = 0.3f / 16777216.f;

struct ResArgs {
  const void* x;
  void* out;
  double* sums;            // [batch][gang]
  float* part;             // [2][batch][gang][128 columns][128 rows], see `mine`
  float* asum;             // [batch][128][128]
  unsigned int* count;     // [batch], zero at the start and at the end
  int m, n, s, L, tall, steps, C, gang;
  float a, b, c, scale, keep;
  double eps;
  unsigned int spin_cap;
  int withhold;            // test hook: the first CTA waits at its n-th meeting without arriving (-1 = off)
  int* status;
};

__device__ __forceinline__ uint64_t desc_mn_blocks(uint32_t smem_addr) {      // as g16::desc_mn, blocks of 128 rows
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr >> 4) & 0x3FFF);
  d |= (uint64_t)(kBlock >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
// byte of (row, column) in consecutive [128][64] blocks
__device__ __forceinline__ uint32_t block_at(int row, int col) {
  return (uint32_t)((col >> 6) * kBlock + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4) + (col & 7) * 2);
}
// eight consecutive columns (col a multiple of 8) as two terms
__device__ __forceinline__ void put8(unsigned char* hi, unsigned char* lo, int row, int col, const float* v) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const __half2 t = __floats2half2_rn(v[2 * q], v[2 * q + 1]);
    h[q] = *reinterpret_cast<const uint32_t*>(&t);
    l[q] = g16::pack_f16(v[2 * q] - __low2float(t), v[2 * q + 1] - __high2float(t));
  }
  const uint32_t at = block_at(row, col);
  *reinterpret_cast<uint4*>(hi + at) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4*>(lo + at) = make_uint4(l[0], l[1], l[2], l[3]);
}

template <int DT>
__global__ void __launch_bounds__(kResThreads, 1) ortho_resident_kernel(const ResArgs q) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bar;
  __shared__ uint32_t tmem_slot;
  __shared__ int failed;
  __shared__ double dsum[kResThreads / 32];
  unsigned char* const base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                               ~static_cast<uintptr_t>(1023));
  const int nblk = q.C / 64;
  unsigned char* const xh = base;
  unsigned char* const xl = xh + nblk * kBlock;
  unsigned char* const ah = xl + nblk * kBlock;
  unsigned char* const al = ah + 2 * kBlock;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane;
  const int mat = blockIdx.x / q.gang, g = blockIdx.x % q.gang;
  const int c0 = g * q.C, cols = min(q.C, q.L - c0);
  const size_t mbase = (size_t)mat * q.m * q.n;

  chained_launch();
  if (threadIdx.x == 0) {
    tc::mbar_init(&bar, 1);
    failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&tmem_slot)),
                 "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = tmem_slot, lanes = (uint32_t)(quad * 32) << 16;

  unsigned int epoch = 0;
  const unsigned int silent = blockIdx.x == 0 ? (unsigned int)(q.withhold + 1) : 0u;      // 0: at no meeting
  uint32_t phase = 0;
  // the gang's CTAs meet; what they wrote to global memory before is visible after
  auto meet = [&]() -> bool {
    ++epoch;
    __syncthreads();
    if (threadIdx.x == 0) {
      __threadfence();
      atomicAdd(q.count + mat, epoch == silent ? 0u : 1u);
      const unsigned int target = epoch * (unsigned int)q.gang;
      bool ok = false;
      for (unsigned int i = 0; i < q.spin_cap; ++i) {
        unsigned int v;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(q.count + mat) : "memory");
        if (v >= target) { ok = true; break; }
      }
      if (!ok) failed = 1;
    }
    __syncthreads();
    return failed == 0;
  };
  // all products issued so far are complete
  auto products_done = [&]() -> bool {
    bool ok = tc::mbar_wait(&bar, phase, &failed, q.spin_cap);
    phase ^= 1u;
    tc::tc_fence_after();
    return !__syncthreads_or(!ok);
  };
  auto operands_ready = [&]() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
  };

  // ---- the columns, brought to |X|_F = 1 ----
  // Lines of the stored matrix: rows of the wide orientation, or columns where it is tall; a warp takes four lines at a
  // time, a lane every 32nd element of 128.
  const int lines = q.tall ? cols : q.s, length = q.tall ? q.s : cols;
  const size_t line0 = mbase + (q.tall ? (size_t)c0 * q.n : (size_t)c0);
  auto fetch = [&](int l0, int e0, float (&v)[16]) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int l = l0 + 8 * u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int e = e0 + 32 * j;
        v[4 * u + j] = l < lines && e < length ? load1<DT>(q.x, line0 + (size_t)l * q.n + e) : 0.f;
      }
    }
  };
  {
    double t[4] = {0.0, 0.0, 0.0, 0.0};
    for (int e0 = lane; e0 < length; e0 += 128)
      for (int l0 = warp; l0 < lines; l0 += 32) {
        float v[16];
        fetch(l0, e0, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) t[i & 3] = fma((double)v[i], (double)v[i], t[i & 3]);
      }
    double sum = (t[0] + t[1]) + (t[2] + t[3]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) dsum[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int i = 1; i < kResThreads / 32; ++i) sum += dsum[i];
      __stcg(q.sums + (size_t)mat * q.gang + g, sum);
    }
    // meanwhile: rows and columns that do not exist are zero
    for (int i = threadIdx.x; i < 2 * nblk * kBlock / 16; i += kResThreads)
      reinterpret_cast<uint4*>(xh)[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  bool alive = meet();
  if (alive) {
    double t = 0.0;
    for (int i = lane; i < q.gang; i += 32) t += __ldcg(q.sums + (size_t)mat * q.gang + i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    const float2 f = norm_factor(t, q.eps);
    for (int e0 = lane; e0 < length; e0 += 128)
      for (int l0 = warp; l0 < lines; l0 += 32) {
        float v[16];
        fetch(l0, e0, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int l = l0 + 8 * (i >> 2), e = e0 + 32 * (i & 3);
          if (l < lines && e < length) {
            const uint32_t at = q.tall ? block_at(e, l) : block_at(l, e);
            const float w = v[i] * f.x * f.y;
            const __half h = __float2half_rn(w);
            *reinterpret_cast<__half*>(xh + at) = h;
            *reinterpret_cast<__half*>(xl + at) = __float2half_rn(w - __half2float(h));
          }
        }
      }
  }

  constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(128 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);      // fp16, 128 x 128
  const uint32_t idesc_x = (1u << 4) | (1u << 16) | ((uint32_t)(q.C >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
  const uint32_t uxh = tc::smem_u32(xh), uxl = tc::smem_u32(xl), uah = tc::smem_u32(ah), ual = tc::smem_u32(al);
  // Shares of A: two sets, used by even and odd steps.  A gang that adds all shares up directly meets once a step, so a
  // CTA may store its share of step k + 1 while a slower one still reads those of step k; it stores the share of step
  // k + 2 only after the meeting of step k + 1, where every CTA arrives with its reading of step k behind it.
  const size_t set = (size_t)gridDim.x * 128 * 128, mine = ((size_t)mat * q.gang + g) * 128 * 128;
  // instructions (of 16) that cover the columns and the shorter side: zeros beyond them are not multiplied
  const int kcols = (cols + 15) / 16, ks = (q.s + 15) / 16;
  // 32 columns of this thread's row: the products with a low term (from column 0 of tensor memory), and those of high
  // terms, `k` instructions in accumulators of `per` from column `first`, with what the instructions lose given back
  auto sum_of = [&](uint32_t col, uint32_t first, int k, int per, float loss, float* to) {
    g16::ld32(tmem + lanes + col, to);
    for (int k0 = 0; k0 < k; k0 += per, first += 128u) {
      float t[32];
      g16::ld32(tmem + lanes + first + col, t);
      tc::tc_wait_ld();
      const float f = (float)min(per, k - k0) * loss;
#pragma unroll
      for (int j = 0; j < 32; ++j) to[j] += fmaf(t[j], f, t[j]);
    }
  };
  for (int step = 0; alive && step < q.steps; ++step) {
    // ---- this CTA's share of A ----
    operands_ready();
    if (threadIdx.x == 0) {
      for (int k = 0; k < kcols; ++k) {
        const uint64_t h = tc::make_desc<128>(uxh + (k >> 2) * kBlock) + 2 * (k & 3);
        const uint64_t l = tc::make_desc<128>(uxl + (k >> 2) * kBlock) + 2 * (k & 3);
        g16::mma_f16(tmem + 128u, h, h, idesc, k ? 1u : 0u);
        g16::mma_f16(tmem, h, l, idesc, k ? 1u : 0u);
        g16::mma_f16(tmem, l, h, idesc, 1u);
      }
      tc::tc_commit(&bar);
    }
    if (!products_done()) { alive = false; break; }
    float A[64];
#pragma unroll
    for (int c = 0; c < 64; c += 32) sum_of((uint32_t)(half * 64 + c), 128u, kcols, kcols, kResLossSquares, A + c);
    if (q.gang > 1) {
      float* const part = q.part + (step & 1) * set;
      if (row < q.s) {
#pragma unroll
        for (int j = 0; j < 64; ++j)
          if (half * 64 + j < q.s) __stcg(part + mine + (half * 64 + j) * 128 + row, A[j]);
      }
      if (!meet()) { alive = false; break; }
      // The shares are added up in order, every thread taking elements (column i / s, row i % s) of its own, and pass to
      // the threads that need them through the room of A's terms.
      const float* shares = part + (size_t)mat * q.gang * 128 * 128;
      float* const sums = reinterpret_cast<float*>(ah);          // [column][row]
      const int all = q.s * q.s;
      int parts = q.gang;
      // elements [lo, hi): U per thread and D shares at a time, all loads in flight
      auto add_some = [&](auto U_, auto D_, int lo, int hi, float* to, bool global) {
        constexpr int U = decltype(U_)::value, D = decltype(D_)::value;
        for (int i0 = lo + (int)threadIdx.x; i0 < hi; i0 += U * kResThreads) {
          float t[U];
          int at[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int i = min(i0 + u * kResThreads, hi - 1);      // (the last element again rather than a branch)
            at[u] = i / q.s * 128 + i % q.s;
            t[u] = 0.f;
          }
          for (int k = 0; k < parts; k += D) {
            float v[D][U];
#pragma unroll
            for (int d = 0; d < D; ++d)
#pragma unroll
              for (int u = 0; u < U; ++u) v[d][u] = __ldcg(shares + (size_t)min(k + d, parts - 1) * 128 * 128 + at[u]);
#pragma unroll
            for (int d = 0; d < D; ++d)
#pragma unroll
              for (int u = 0; u < U; ++u) t[u] += k + d < parts ? v[d][u] : 0.f;
          }
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (global) __stcg(to + at[u], t[u]);
            else to[at[u]] = t[u];
          }
        }
      };
      auto add_up = [&](int lo, int hi, float* to, bool global) {
        using std::integral_constant;
        if (parts == 1) add_some(integral_constant<int, 32>(), integral_constant<int, 1>(), lo, hi, to, global);
        else if (hi - lo > 2 * kResThreads) add_some(integral_constant<int, 8>(), integral_constant<int, 4>(), lo, hi, to, global);
        else add_some(integral_constant<int, 2>(), integral_constant<int, 16>(), lo, hi, to, global);
      };
      if (all * q.gang > kDirect) {
        float* sum = q.asum + (size_t)mat * 128 * 128;
        const int per = (all + q.gang - 1) / q.gang;
        add_up(min(all, g * per), min(all, (g + 1) * per), sum, true);
        if (!meet()) { alive = false; break; }
        shares = sum;
        parts = 1;
      }
      add_up(0, all, sums, false);
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 64; ++j) A[j] = row < q.s && half * 64 + j < q.s ? sums[(half * 64 + j) * 128 + row] : 0.f;
      __syncthreads();
    }
    // ---- A's terms, A A (in up to three accumulators), B's terms in their place ----
#pragma unroll
    for (int j = 0; j < 64; j += 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) A[j + k] *= kA / (kX * kX);
      put8(ah, al, row, half * 64 + j, A + j);
    }
    const int per = (ks + 2) / 3;
    operands_ready();
    if (threadIdx.x == 0) {
      for (int k = 0; k < ks; ++k) {
        const uint64_t h = tc::make_desc<128>(uah + (k >> 2) * kBlock) + 2 * (k & 3);
        const uint64_t l = tc::make_desc<128>(ual + (k >> 2) * kBlock) + 2 * (k & 3);
        g16::mma_f16(tmem + 128u * (uint32_t)(1 + k / per), h, h, idesc, k % per ? 1u : 0u);
        g16::mma_f16(tmem, h, l, idesc, k ? 1u : 0u);
        g16::mma_f16(tmem, l, h, idesc, 1u);
      }
      tc::tc_commit(&bar);
    }
    if (!products_done()) { alive = false; break; }
#pragma unroll
    for (int c = 0; c < 64; c += 32) {
      float t[32];
      sum_of((uint32_t)(half * 64 + c), 128u, ks, per, kResLossAA, t);
#pragma unroll
      for (int j = 0; j < 32; j += 8) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          v[k] = fmaf(q.c, t[j + k] * (1.f / (kA * kA)), q.b * (A[c + j + k] * (1.f / kA)));
          if (half * 64 + c + j + k == row) v[k] += q.a;
          v[k] *= kB;
        }
        put8(ah, al, row, half * 64 + c + j, v);
      }
    }
    // ---- this CTA's columns of B X ----
    operands_ready();
    if (threadIdx.x == 0) {
      const uint64_t xhd = desc_mn_blocks(uxh), xld = desc_mn_blocks(uxl);
      for (int k = 0; k < ks; ++k) {         // 16 rows of X each
        const uint64_t bh = tc::make_desc<128>(uah + (k >> 2) * kBlock) + 2 * (k & 3);
        const uint64_t bl = tc::make_desc<128>(ual + (k >> 2) * kBlock) + 2 * (k & 3);
        g16::mma_f16(tmem + 256u, bh, xhd + 128 * k, idesc_x, k ? 1u : 0u);
        g16::mma_f16(tmem, bh, xld + 128 * k, idesc_x, k ? 1u : 0u);
        g16::mma_f16(tmem, bl, xhd + 128 * k, idesc_x, 1u);
      }
      tc::tc_commit(&bar);
    }
    if (!products_done()) { alive = false; break; }
    const bool last = step + 1 == q.steps;
    for (int c = half * (q.C / 2); c < (half + 1) * (q.C / 2); c += 32) {
      float t[32];
      sum_of((uint32_t)c, 256u, ks, ks, kResLossMixed, t);
      if (!last) {
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
#pragma unroll
          for (int k = 0; k < 8; ++k) t[j + k] *= 1.f / kB;
          put8(xh, xl, row, c + j, t + j);
        }
      } else if (row < q.s) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          if (c + j < cols) {
            const size_t e = q.tall ? mbase + (size_t)(c0 + c + j) * q.n + row : mbase + (size_t)row * q.n + c0 + c + j;
            const float v = t[j] * (1.f / (kB * kX)) * q.scale;
            if constexpr (DT == DK_F32) {
              float* o = static_cast<float*>(q.out) + e;
              *o = q.keep != 0.f ? fmaf(q.keep, *o, v) : v;
            } else {
              __nv_bfloat16* o = static_cast<__nv_bfloat16*>(q.out) + e;
              *o = __float2bfloat16_rn(q.keep != 0.f ? fmaf(q.keep, __bfloat162float(*o), v) : v);
            }
          }
        }
      }
    }
  }

  // ---- teardown: the last CTA of the gang leaves the counter at zero ----
  tc::tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) {
    if (failed) atomicExch(q.status, (int)DK_ERR_TIMEOUT);
    else if (atomicAdd(q.count + mat, 1u) + 1u == (epoch + 1u) * (unsigned int)q.gang) q.count[mat] = 0u;
  }
  if (failed) {      // (products may be in flight still: time for them to end)
    for (int i = 0; i < 64; ++i) __nanosleep(16384);
    __syncthreads();
  }
  if (warp == 0) {
    tc::tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
size_t up(size_t v) { return (v + 1023) / 1024 * 1024; }

struct Plan {
  bool tall;
  int s, np, sp;               // shorter side; pitches of X and of the square matrices
  size_t off_sum, off_x[2], off_a, off_b, off_part, off_asum, total;
  size_t x_plane, s_plane;     // elements of one term of all matrices
};

Plan plan_ortho(const dk_ortho& q) {
  Plan p;
  p.tall = q.m > q.n;
  p.s = p.tall ? q.n : q.m;
  p.np = (q.n + 7) / 8 * 8;
  p.sp = (p.s + 7) / 8 * 8;
  p.x_plane = (size_t)q.batch * q.m * p.np;
  p.s_plane = (size_t)q.batch * p.s * p.sp;
  size_t off = 0;
  p.off_sum = off; off += up((size_t)q.batch * kSumBlocks * sizeof(double));
  for (int i = 0; i < 2; ++i) { p.off_x[i] = off; off += up(p.x_plane * 4); }
  p.off_a = off; off += up(p.s_plane * 4);
  p.off_b = off; off += up(p.s_plane * 4);
  // Slices of a product: every (tile, slice) has a pair of its own, but a slice of a symmetric product takes the room of
  // the whole square, up to twice its tiles.  A symmetric product always goes through them.  (The resident kernel's two
  // sets of shares, 64 KiB for each of at most kMaxSms CTAs, take half of this room.)
  size_t part = (size_t)2 * (kMaxSms / 2) * g16::TILE_M * BN * sizeof(float);
  static_assert(2 * 128 * 128 * kMaxSms <= 2 * (kMaxSms / 2) * g16::TILE_M * BN, "room for two sets of shares");
  const size_t square = (size_t)q.batch * p.s * p.sp * sizeof(float);
  if (square > part) part = square;
  p.off_part = off; off += up(part);
  p.off_asum = off; off += p.s <= 128 ? up((size_t)(q.batch < kMaxSms ? q.batch : kMaxSms) * 128 * 128 * sizeof(float)) : 0;
  p.total = off;
  return p;
}

// Columns per CTA of the resident kernel (0: it does not take the call): 128, whose share of A is one accumulator's
// sum, or more where that leaves more CTAs than SMs.
int resident_columns(const dk_ortho& q, const Plan& pl, int sms) {
  if (pl.s > 128 || q.steps < 1) return 0;
  const int L = pl.tall ? q.m : q.n;
  if (sms > kMaxSms) sms = kMaxSms;
  for (int C = L <= 64 ? 64 : 128; C <= kMaxColumns; C += 64)
    if ((long long)q.batch * ((L + C - 1) / C) <= sms) return C;
  return 0;
}

dk_status check_ortho(const dk_ortho* q) {
  if (!q) return DK_ERR_INVALID_ARG;
  if (q->dtype != DK_F32 && q->dtype != DK_BF16) return DK_ERR_INVALID_ARG;
  if (q->batch < 1 || q->m < 1 || q->n < 1 || q->m > 65536 || q->n > 65536 || q->batch > 4096) return DK_ERR_SHAPE;
  if (q->steps < 0 || q->steps > 32) return DK_ERR_SHAPE;
  if ((double)q->batch * q->m * q->n > 4e10) return DK_ERR_SHAPE;
  if (!(q->eps >= 0.f) || !(fabsf(q->a) + 2.f * fabsf(q->b) + 4.f * fabsf(q->c) <= 31.f)) return DK_ERR_INVALID_ARG;
  return DK_OK;
}

// What the tensor pipe loses per stage when it adds, in 2^-24 of the sum (the large tiles add all three products into one
// accumulator, the small ones the low terms' apart): measured on sums of squares 6.6 and 4.4, of products of random sign
// 3.6 and 1.2, within 0.7 of that for chunks of 1 to 8 stages and contractions of 64 to 4096.  X X^T and A A have their
// weight on the diagonal, a sum of squares.
constexpr float kUlp = 1.f / 16777216.f;
constexpr float kLossSquares[2] = {6.6f * kUlp, 4.4f * kUlp}, kLossMixed[2] = {3.6f * kUlp, 1.2f * kUlp};

// Stages added up in tensor memory: as even as at most four allow.  What is lost in A A counts most (the polynomial's
// first steps amplify it, the more the smaller the matrices are): up to a short side of 512 each stage is promoted
// (against plain fp32, at 4 stages and at 1: 256x2304 2.2 times its error and 0.8, 320x10000 2.7 and 1.2, 512x4608
// 1.05 and 0.8, for 1-5 % of the call; 1001x1961 0.8 and 0.5, 4096x25088 0.7 and 0.35 for 4 % and 10 % are not taken).
int chunk_of(const g16::Tiling& t, int most) {
  const int chunks = (t.kb_per_split + most - 1) / most;
  return (t.kb_per_split + chunks - 1) / chunks;
}

Params gemm_params(const g16::Tiling& t, const dk_ortho& q, long long M, long long N, bool sym, int most = 4) {
  Params p = {};
  p.MT = t.MT; p.NT = t.NT; p.nbatch = q.batch; p.sym = sym ? 1 : 0; p.tiles = t.tiles;
  p.KB = t.KB; p.ksplit = t.ksplit; p.kb_per_split = t.kb_per_split;
  p.M = (int)M; p.N = (int)N;
  p.bf16 = 0;
  p.chunk = chunk_of(t, most);
  p.comp = sym ? kLossSquares[0] : kLossMixed[0];
  p.comp_small = sym ? kLossSquares[1] : kLossMixed[1];
  return p;
}

unsigned grid_of(long long items, int sms) {
  long long b = (items + 255) / 256;
  if (b > (long long)sms * 8) b = (long long)sms * 8;
  return b < 1 ? 1u : (unsigned)b;
}

dk_status orthogonalize(dk_ctx* ctx, const dk_ortho& q, const Plan& pl, const void* x, float scale, float keep,
                        void* out, cudaStream_t st) {
  char* ws = static_cast<char*>(ctx->ws);
  const int sms = ctx->sm_count;
  double* sums = reinterpret_cast<double*>(ws + pl.off_sum);
  float* part = reinterpret_cast<float*>(ws + pl.off_part);
  __half* xs[2] = {reinterpret_cast<__half*>(ws + pl.off_x[0]), reinterpret_cast<__half*>(ws + pl.off_x[1])};
  __half* am = reinterpret_cast<__half*>(ws + pl.off_a);
  __half* bm = reinterpret_cast<__half*>(ws + pl.off_b);
  const long long per = (long long)q.m * q.n;

  if (const int C = resident_columns(q, pl, sms)) {
    ResArgs r = {};
    r.x = x; r.out = out; r.sums = sums; r.part = part;
    r.asum = reinterpret_cast<float*>(ws + pl.off_asum);
    r.count = step_counters(ctx);
    r.m = q.m; r.n = q.n; r.s = pl.s; r.L = pl.tall ? q.m : q.n; r.tall = pl.tall; r.steps = q.steps; r.C = C;
    r.gang = (r.L + C - 1) / C;
    r.a = q.a; r.b = q.b; r.c = q.c; r.scale = scale; r.keep = keep; r.eps = (double)q.eps;
    r.spin_cap = (unsigned)ctx->opt.v[DK_OPT_SPIN_LIMIT];
    r.withhold = ctx->opt.v[DK_OPT_TEST_WITHHOLD];
    ctx->opt.v[DK_OPT_TEST_WITHHOLD] = -1;
    r.status = device_status_word(ctx);
    auto kern = q.dtype == DK_F32 ? ortho_resident_kernel<DK_F32> : ortho_resident_kernel<DK_BF16>;
    const int smem = (2 * (C / 64) + 4) * kBlock + 1024, most = (2 * (kMaxColumns / 64) + 4) * kBlock + 1024;
    if (most > tc_smem_optin(ctx)) return DK_ERR_UNSUPPORTED;
    static SmemLimit limit[2];
    const dk_status s = allow_smem(limit[q.dtype == DK_F32 ? 0 : 1], ctx->device, kern, most);
    if (s != DK_OK) return s;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(q.batch * r.gang));
    cfg.blockDim = dim3(kResThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
    cfg.attrs = at;
    cfg.numAttrs = r.gang > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, r) == cudaSuccess ? DK_OK : DK_ERR_CUDA;
  }

  int nb = (int)((per + 8191) / 8192);
  if (nb > kSumBlocks) nb = kSumBlocks;
  const dim3 gs((unsigned)nb, (unsigned)q.batch);
  const dim3 gl(grid_of((long long)q.m * pl.np / 8, sms), (unsigned)q.batch);
  if (q.dtype == DK_F32) {
    DK_CUDA_CHECK(launch_chained(ortho_sumsq_kernel<DK_F32>, gs, 256, 0, st,
                                 x, per, sums));
    DK_CUDA_CHECK(launch_chained(ortho_load_kernel<DK_F32>, gl, 256, 0, st,
                                 x, sums, nb, (double)q.eps, q.m, q.n, pl.np, xs[0], xs[0] + pl.x_plane));
  } else {
    DK_CUDA_CHECK(launch_chained(ortho_sumsq_kernel<DK_BF16>, gs, 256, 0, st,
                                 x, per, sums));
    DK_CUDA_CHECK(launch_chained(ortho_load_kernel<DK_BF16>, gl, 256, 0, st,
                                 x, sums, nb, (double)q.eps, q.m, q.n, pl.np, xs[0], xs[0] + pl.x_plane));
  }

  XArgs fin = {};
  fin.out = out; fin.n = q.n; fin.dtype = q.dtype; fin.scale = scale; fin.keep = keep;
  const long long rows = (long long)q.batch * q.m;
  if (q.steps == 0) {
    fin.f = 1.f / kX;
    DK_CUDA_CHECK(launch_chained(ortho_x_kernel, dim3(grid_of(rows * ((q.n + 7) / 8), sms)), 256, 0, st,
                                 fin, nullptr, 0, 0, xs[0], xs[0] + pl.x_plane, rows, pl.np));
    return cudaGetLastError() == cudaSuccess ? DK_OK : DK_ERR_CUDA;
  }

  const g16::Tiling tg = g16::plan(pl.s, pl.s, pl.tall ? q.m : q.n, q.batch, true, sms, 3);
  const g16::Tiling tp = g16::plan(pl.s, pl.s, pl.s, q.batch, true, sms, 3);
  const g16::Tiling tx = g16::plan(q.m, q.n, pl.s, q.batch, false, sms, 3, true);
  const int pitch_s = (pl.s + 3) / 4 * 4, pitch_x = (q.n + 3) / 4 * 4;
  const unsigned nt = (unsigned)((pl.sp + 31) / 32);
  SymArgs sa = {};
  sa.part = part; sa.nbatch = q.batch; sa.s = pl.s; sa.pitch_part = pitch_s; sa.pitch = pl.sp;
  sa.a = q.a; sa.b = q.b; sa.c = q.c;
  sa.a_hi = am; sa.a_lo = am + pl.s_plane;
  const Operand A{am, am + pl.s_plane, pl.s, pl.s, pl.sp, (long long)pl.s * pl.sp};
  const Operand B{bm, bm + pl.s_plane, pl.s, pl.s, pl.sp, (long long)pl.s * pl.sp};

  for (int k = 0; k < q.steps; ++k) {
    __half* cur = xs[k & 1];
    __half* nxt = xs[(k + 1) & 1];
    const Operand X{cur, cur + pl.x_plane, q.m, q.n, pl.np, (long long)q.m * pl.np};
    // A
    const g16::EpiPartial ep{part, pitch_s};
    Params p = gemm_params(tg, q, pl.s, pl.s, true);
    dk_status s;
    sa.ks = tg.ksplit; sa.f = kA / (kX * kX); sa.poly = 0; sa.hi = am; sa.lo = am + pl.s_plane;
    if (tg.cs) {
      s = pl.tall ? g16::product<3, true, true>(ctx, tg, X, X, p, EpiSym{sa}, st)
                  : g16::product<3, false, false>(ctx, tg, X, X, p, EpiSym{sa}, st);
      if (s != DK_OK) return s;
    } else {
      s = pl.tall ? g16::launch<3, true, true, BN>(ctx, X, X, p, ep, st)
                  : g16::launch<3, false, false, BN>(ctx, X, X, p, ep, st);
      if (s != DK_OK) return s;
      count_launches(ctx, DK_KERNEL_OTHER, 1);
      DK_CUDA_CHECK(launch_chained(ortho_sym_kernel, dim3(nt, nt, (unsigned)q.batch), 256, 0, st, sa));
    }
    // B
    p = gemm_params(tp, q, pl.s, pl.s, true, pl.s <= 512 ? 1 : 4);
    sa.ks = tp.ksplit; sa.f = 1.f / (kA * kA); sa.poly = 1; sa.hi = bm; sa.lo = bm + pl.s_plane;
    if (tp.cs) {
      s = g16::product<3, false, false>(ctx, tp, A, A, p, EpiSym{sa}, st);
      if (s != DK_OK) return s;
    } else {
      s = g16::launch<3, false, false, BN>(ctx, A, A, p, ep, st);
      if (s != DK_OK) return s;
      count_launches(ctx, DK_KERNEL_OTHER, 1);
      DK_CUDA_CHECK(launch_chained(ortho_sym_kernel, dim3(nt, nt, (unsigned)q.batch), 256, 0, st, sa));
    }
    // X
    XArgs xa = fin;
    if (k + 1 < q.steps) {
      xa.hi = nxt; xa.lo = nxt + pl.x_plane; xa.pitch = pl.np;
      xa.f = 1.f / kB;
    } else {
      xa.f = 1.f / (kB * kX);
    }
    p = gemm_params(tx, q, q.m, q.n, false);
    if (!tx.cs && tx.ksplit > 1) {
      const g16::EpiPartial ex{part, pitch_x};
      s = pl.tall ? g16::launch<3, false, false, BN>(ctx, X, B, p, ex, st)
                  : g16::launch<3, false, true, BN>(ctx, B, X, p, ex, st);
      if (s != DK_OK) return s;
      count_launches(ctx, DK_KERNEL_OTHER, 1);
      DK_CUDA_CHECK(launch_chained(ortho_x_kernel, dim3(grid_of(rows * ((q.n + 7) / 8), sms)), 256, 0, st,
                                 xa, part, tx.ksplit, pitch_x, nullptr, nullptr, rows, 0));
    } else {
      auto x_product = [&](auto epi) {
        return pl.tall ? g16::product<3, false, false, true>(ctx, tx, X, B, p, epi, st)
                       : g16::product<3, false, true, true>(ctx, tx, B, X, p, epi, st);
      };
      s = k + 1 < q.steps ? x_product(EpiX<kTerms>{xa})
          : q.dtype == DK_F32 ? x_product(EpiX<DK_F32>{xa}) : x_product(EpiX<DK_BF16>{xa});
      if (s != DK_OK) return s;
    }
  }
  return cudaGetLastError() == cudaSuccess ? DK_OK : DK_ERR_CUDA;
}

}  // namespace
}  // namespace dk

using namespace dk;

extern "C" {

dk_status dk_ortho_workspace_bytes(const dk_ortho* q, size_t* bytes) {
  if (!bytes) return DK_ERR_INVALID_ARG;
  dk_status s = check_ortho(q);
  if (s != DK_OK) return s;
  *bytes = plan_ortho(*q).total;
  return DK_OK;
}

dk_status dk_orthogonalize(dk_ctx* ctx, const dk_ortho* q, const void* x, float scale, float keep, void* out,
                           void* stream) {
  if (!ctx || !x || !out || x == out) return DK_ERR_INVALID_ARG;
  if (!aligned_to(x, 16) || !aligned_to(out, 16)) return DK_ERR_INVALID_ARG;
  dk_status s = check_ortho(q);
  if (s != DK_OK) return s;
  const Plan pl = plan_ortho(*q);
  if (!ctx->ws || ctx->ws_bytes < pl.total) return DK_ERR_WORKSPACE;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // (kernels that join slices are counted where they are launched)
  ProfScope ps(ctx, DK_KERNEL_OTHER, resident_columns(*q, pl, ctx->sm_count) ? 1 : q->steps ? 2 + 3 * q->steps : 3, st);
  return orthogonalize(ctx, *q, pl, x, scale, keep, out, st);
}

}  // extern "C"
