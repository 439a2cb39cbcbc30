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

#include "dk_gemm16.cuh"

namespace dk {
namespace {

using g16::Operand;
using g16::Params;

constexpr int BN = 256;
constexpr int kSumBlocks = 256;                 // partial sums of squares per matrix
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
  const size_t base = (size_t)blockIdx.y * per;
  double t = 0.0;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < per; i += (long long)gridDim.x * 256) {
    const double v = (double)load1<DT>(x, base + i);
    t = fma(v, v, t);
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

// X as two fp16 terms, rows padded to `pitch` with zeros
template <int DT>
__global__ void __launch_bounds__(256)
ortho_load_kernel(const void* x, const double* part, int nparts, double eps, long long m, int n, int pitch, __half* hi,
                  __half* lo) {
  chained_launch();
  __shared__ float f;
  if (threadIdx.x < 32) {
    double t = 0.0;
    for (int i = threadIdx.x; i < nparts; i += 32) t += part[blockIdx.y * nparts + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (threadIdx.x == 0) f = (float)((double)kX / (sqrt(t) + eps));
  }
  __syncthreads();
  const float fac = f;
  const int n8 = pitch / 8;
  const size_t src = (size_t)blockIdx.y * m * n, dst = (size_t)blockIdx.y * m * pitch;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < m * n8; i += (long long)gridDim.x * 256) {
    const long long r = i / n8;
    const int c = (int)(i - r * n8) * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < n ? load1<DT>(x, src + (size_t)r * n + c + j) * fac : 0.f;
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

// the result of a step: the next X as two terms (hi given), or the update itself
struct XArgs {
  __half* hi;
  __half* lo;
  long long pitch;             // of the terms
  void* out;
  int n, dtype;
  float f;                     // undoes the operands' powers of two (and brings X to its own)
  float scale, keep;
  int vec;
};
struct EpiX {
  XArgs a;
  template <int NH>
  __device__ __forceinline__ void operator()(const Params& p, float (&acc)[NH], int batch, int, int row,
                                             int col0) const {
    if (row >= p.M || col0 >= p.N) return;
    const int count = min(NH, p.N - col0);
    if (a.hi != nullptr) {
      const size_t e = ((size_t)batch * p.M + row) * a.pitch + col0;
#pragma unroll
      for (int j = 0; j < NH; ++j) acc[j] *= a.f;
      g16::store_planes<NH>(a.hi + e, a.lo + e, acc, count);
      return;
    }
    const size_t e = ((size_t)batch * p.M + row) * a.n + col0;
    const float s = a.f * a.scale;
    if (a.dtype == DK_F32) {
      float* o = static_cast<float*>(a.out) + e;
#pragma unroll
      for (int j = 0; j < NH; ++j) {
        acc[j] *= s;
        if (a.keep != 0.f && j < count) acc[j] = fmaf(a.keep, o[j], acc[j]);
      }
      g16::store_f32<NH>(o, acc, count, a.vec != 0);
    } else {
      __nv_bfloat16* o = static_cast<__nv_bfloat16*>(a.out) + e;
#pragma unroll
      for (int j = 0; j < NH; ++j) {
        acc[j] *= s;
        if (a.keep != 0.f && j < count) acc[j] = fmaf(a.keep, __bfloat162float(o[j]), acc[j]);
      }
      g16::store_bf16<NH>(o, acc, count, a.vec != 0);
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
// host side
// ---------------------------------------------------------------------------
size_t up(size_t v) { return (v + 1023) / 1024 * 1024; }

struct Plan {
  bool tall;
  int s, np, sp;               // shorter side; pitches of X and of the square matrices
  size_t off_sum, off_x[2], off_a, off_b, off_part, total;
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
  // the whole square, up to twice its tiles.  A symmetric product always goes through them.
  size_t part = (size_t)2 * (kMaxSms / 2) * g16::TILE_M * BN * sizeof(float);
  const size_t square = (size_t)q.batch * p.s * p.sp * sizeof(float);
  if (square > part) part = square;
  p.off_part = off; off += up(part);
  p.total = off;
  return p;
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

Params gemm_params(const g16::Tiling& t, const dk_ortho& q, long long M, long long N, bool sym) {
  Params p = {};
  p.MT = t.MT; p.NT = t.NT; p.nbatch = q.batch; p.sym = sym ? 1 : 0; p.tiles = t.tiles;
  p.KB = t.KB; p.ksplit = t.ksplit; p.kb_per_split = t.kb_per_split;
  p.M = (int)M; p.N = (int)N;
  p.bf16 = 0;
  p.chunk = 2;
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
  const int sms = ctx->sm_count, pairs = sms / 2;
  double* sums = reinterpret_cast<double*>(ws + pl.off_sum);
  float* part = reinterpret_cast<float*>(ws + pl.off_part);
  __half* xs[2] = {reinterpret_cast<__half*>(ws + pl.off_x[0]), reinterpret_cast<__half*>(ws + pl.off_x[1])};
  __half* am = reinterpret_cast<__half*>(ws + pl.off_a);
  __half* bm = reinterpret_cast<__half*>(ws + pl.off_b);
  const long long per = (long long)q.m * q.n;

  int nb = (int)((per + 2047) / 2048);
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

  const size_t es = q.dtype == DK_F32 ? 4 : 2;
  XArgs fin = {};
  fin.out = out; fin.n = q.n; fin.dtype = q.dtype; fin.scale = scale; fin.keep = keep;
  fin.vec = (size_t)q.n * es % 16 == 0;
  const long long rows = (long long)q.batch * q.m;
  if (q.steps == 0) {
    fin.f = 1.f / kX;
    DK_CUDA_CHECK(launch_chained(ortho_x_kernel, dim3(grid_of(rows * ((q.n + 7) / 8), sms)), 256, 0, st,
                                 fin, nullptr, 0, 0, xs[0], xs[0] + pl.x_plane, rows, pl.np));
    return cudaGetLastError() == cudaSuccess ? DK_OK : DK_ERR_CUDA;
  }

  const g16::Tiling tg = g16::plan(pl.s, pl.s, pl.tall ? q.m : q.n, BN, q.batch, true, pairs, 4);
  const g16::Tiling tp = g16::plan(pl.s, pl.s, pl.s, BN, q.batch, true, pairs, 4);
  const g16::Tiling tx = g16::plan(q.m, q.n, pl.s, BN, q.batch, false, pairs, 4);
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
    Params p = gemm_params(tg, q, pl.s, pl.s, true);
    const g16::EpiPartial ep{part, pitch_s};
    dk_status s = pl.tall ? g16::launch<3, true, true, BN>(ctx, X, X, p, ep, st)
                          : g16::launch<3, false, false, BN>(ctx, X, X, p, ep, st);
    if (s != DK_OK) return s;
    sa.ks = tg.ksplit; sa.f = kA / (kX * kX); sa.poly = 0; sa.hi = am; sa.lo = am + pl.s_plane;
    DK_CUDA_CHECK(launch_chained(ortho_sym_kernel, dim3(nt, nt, (unsigned)q.batch), 256, 0, st,
                                 sa));
    // B
    p = gemm_params(tp, q, pl.s, pl.s, true);
    s = g16::launch<3, false, false, BN>(ctx, A, A, p, ep, st);
    if (s != DK_OK) return s;
    sa.ks = tp.ksplit; sa.f = 1.f / (kA * kA); sa.poly = 1; sa.hi = bm; sa.lo = bm + pl.s_plane;
    DK_CUDA_CHECK(launch_chained(ortho_sym_kernel, dim3(nt, nt, (unsigned)q.batch), 256, 0, st,
                                 sa));
    // X
    XArgs xa = fin;
    if (k + 1 < q.steps) {
      xa.hi = nxt; xa.lo = nxt + pl.x_plane; xa.pitch = pl.np;
      xa.f = 1.f / kB;
    } else {
      xa.f = 1.f / (kB * kX);
    }
    p = gemm_params(tx, q, q.m, q.n, false);
    if (tx.ksplit > 1) {
      const g16::EpiPartial ex{part, pitch_x};
      s = pl.tall ? g16::launch<3, false, false, BN>(ctx, X, B, p, ex, st)
                  : g16::launch<3, false, true, BN>(ctx, B, X, p, ex, st);
      if (s != DK_OK) return s;
      DK_CUDA_CHECK(launch_chained(ortho_x_kernel, dim3(grid_of(rows * ((q.n + 7) / 8), sms)), 256, 0, st,
                                 xa, part, tx.ksplit, pitch_x, nullptr, nullptr, rows, 0));
    } else {
      s = pl.tall ? g16::launch<3, false, false, BN>(ctx, X, B, p, EpiX{xa}, st)
                  : g16::launch<3, false, true, BN>(ctx, B, X, p, EpiX{xa}, st);
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
  ProfScope ps(ctx, DK_KERNEL_OTHER, 2 + 5 * q->steps, st);
  return orthogonalize(ctx, *q, pl, x, scale, keep, out, st);
}

}  // extern "C"
