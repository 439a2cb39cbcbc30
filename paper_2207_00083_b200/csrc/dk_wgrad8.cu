// Weight gradient of a linear layer from the 8-bit checkpoint of its input: dW = keep*dW + scale*dy^T.x, db likewise.
//
// The product contracts over rows, across which the checkpoint's powers of two change; so a block's power cannot leave the
// sum, and the tensor cores' 8-bit formats (whose scales run along the contraction) do not apply.  But q*2^k is a bf16
// number as it stands.  bf16: dy and x enter unrounded, one product.  fp32: dy as two fp16 terms under a power of two of
// each output (its column of dy, its row of dW), x as one fp16 plane under a power of two of the whole checkpoint (q*2^k
// is an fp16 number for 33 powers of two, subnormals included), two products.
//   wgrad8_columns_kernel: sums (db) and largest magnitudes of dy's columns; bf16: the operand from the checkpoint; fp32: its
//     largest exponent
//   wgrad8_prep_kernel: fp32: the operands
//   the product (dk_gemm16.cuh), both operands read across their rows in place
// Large products are bound by the tensor cores (16384 rows, 4096 x 4096 bf16: 431 us, 1.28 PFLOP/s, and 453
// with db, for which dy is read once more), products of few rows by the writing of dW (256 rows, 25088 x 4096 fp32: 125 us for 411 MB, floor 64), small ones
// by the chain of launches (64 rows, 512 x 1000 fp32: 13 us).
#include <math.h>

#include "dk_ckpt8.cuh"
#include "dk_gemm16.cuh"
#include "dk_vec.cuh"

namespace dk {
namespace {

using g16::magnitude;
using g16::Operand;
using g16::Params;
using g16::pow2;
using g16::scale_exp;

constexpr int kThreads = 256;
constexpr int kMaxParts = 148;           // parts of the rows in which columns are summed, but of
constexpr long long kPartRows = 1 << 15; // rows at most each
constexpr int kMaxBlocks = 148;          // of wgrad8_columns_kernel that look at the exponents

struct Wg8 {
  const void* dy;
  const uint8_t* codes;
  const uint8_t* exps;
  void* x16;                 // [rows][dp]
  void* hi;                  // [rows][op] (dy's terms, or a copy with whole pitch)
  void* lo;
  float* sums;               // [parts][op]
  unsigned int* most;        // [parts][op]
  unsigned int* most_all;
  unsigned int* block_exp;   // [blocks]: largest exponent; block_exp[kMaxBlocks]: of all
  float* db;
  long long rows;
  unsigned int* count;       // [strips], zero between launches
  int d, dp, out, op, strips, parts, blocks, copy_dy, with_sums;
  float scale, keep;
};

// the checkpoint's power of two: its largest step becomes 2^8, so the largest value is below 2^15
__device__ __forceinline__ int x_exp(unsigned int largest) {
  const int s = 8 - ((int)largest - 127);
  return largest == 0u ? 0 : min(s, 126);
}

// The checkpoint's values as operands, eight a thread.
template <int DT>
__device__ __forceinline__ void expand(const Wg8& a, int s, long long i0, long long step) {
  constexpr int U = 4;
  const long long units = a.rows * (a.dp / 8);
  for (long long i = i0; i < units; i += U * step) {
    ckpt8::Raw<8> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * step < units) r[u] = ckpt8::get<8>(a.codes + (i + u * step) * 8, a.exps + (i + u * step) / 4);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u * step >= units) continue;
      float v[8];
      uint32_t w[4];
      if constexpr (DT == DK_F32) {
        if (r[u].b != 255u) r[u].b = (uint32_t)min(max((int)r[u].b + s, 0), 254);
        ckpt8::unpack<8>(r[u], v);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = g16::pack_f16(v[2 * k], v[2 * k + 1]);
      } else {
        ckpt8::unpack<8>(r[u], v);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = __byte_perm(__float_as_uint(v[2 * k]), __float_as_uint(v[2 * k + 1]), 0x7632);
      }
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.x16) + (i + u * step) * 8) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// Columns of dy: their sums and (fp32) largest magnitudes, over parts of the rows; a CTA has a strip of 32 vectors of 16
// bytes.  bf16: rows of no whole vectors are copied to a pitch of such; and the
// CTAs behind those of dy expand the checkpoint, so nothing else comes before the product.  fp32: they look for the
// checkpoint's largest exponent.  The last CTA of a strip to be done joins its parts.  (bf16: three CTAs an SM, for the sake of
// what expands the checkpoint: 1000 rows, 8192 by 1024 without db 29 us, with two 30.)
template <int DT, int VEC>
__global__ void __launch_bounds__(kThreads, DT == DK_BF16 ? 3 : 2) wgrad8_columns_kernel(const Wg8 a) {
  chained_launch();
  constexpr int FULL = DT == DK_F32 ? 4 : 8, NV = FULL / VEC, U = NV >= 4 ? 4 : 8 / NV;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, columns = a.with_sums ? a.strips * a.parts : 0;
  if ((int)blockIdx.x >= columns) {
    const long long i0 = (long long)(blockIdx.x - columns) * kThreads + threadIdx.x, step = (long long)(gridDim.x - columns) * kThreads;
    if constexpr (DT == DK_BF16) {
      expand<DT>(a, 0, i0, step);
    } else {
      // (four bytes at a time; those of the end, and 255, by themselves)
      const long long n = a.rows * (a.dp / ckpt8::kBlock);
      unsigned int e = 0;
      for (long long i = i0; i < n / 4; i += step) {
        const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(a.exps) + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const unsigned int b = w >> 8 * k & 255u;
          e = max(e, b == 255u ? 0u : b);
        }
      }
      for (long long i = n / 4 * 4 + i0; i < n; i += step) e = max(e, a.exps[i] == 255u ? 0u : (unsigned)a.exps[i]);
      e = __reduce_max_sync(0xffffffffu, e);
      __shared__ unsigned int se[8];
      if (lane == 0) se[warp] = e;
      __syncthreads();
      if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < 8; ++w) e = max(e, se[w]);
        a.block_exp[blockIdx.x - columns] = e;
      }
    }
    return;
  }
  const int strip = blockIdx.x % a.strips, part = blockIdx.x / a.strips, c0 = strip * 32 * FULL + lane * VEC;
  const long long per = (a.rows + a.parts - 1) / a.parts;
  const long long r0 = part * per, r1 = min(a.rows, r0 + per);
  // A thread's sums: of kFold rows at a time, then, in shared memory, of those.  (A wide dy has few parts, one from 37889 bf16
  // or 18945 fp32 outputs on: all of a thread's rows one after the other would lose what is small beside the sum so far.)
  constexpr int kFold = 64;
  __shared__ float ss[8][32 * FULL + 1];
  __shared__ unsigned int sm[DT == DK_F32 ? 8 : 1][32 * FULL + 1];
  float* const mine = ss[warp] + lane * VEC;
  float s[NV][VEC];
  unsigned int m[NV][VEC];
  int ahead = 0;                     // rows in s
  bool folded = false;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < VEC; ++k) { s[j][k] = 0.f; m[j][k] = 0u; }
  for (long long r = r0 + warp; r < r1; r += 8 * U) {
    if ((ahead += U) > kFold) {
      ahead = U;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          mine[j * 32 * VEC + k] = folded ? mine[j * 32 * VEC + k] + s[j][k] : s[j][k];
          s[j][k] = 0.f;
        }
      folded = true;
    }
    typename Vec<DT, VEC>::Raw raw[U][NV];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (r + 8 * u < r1 && c0 + j * 32 * VEC < a.out) raw[u][j] = Vec<DT, VEC>::get(a.dy, (r + 8 * u) * a.out + c0 + j * 32 * VEC);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = c0 + j * 32 * VEC;
        if (r + 8 * u >= r1 || c >= a.op) continue;
        if (c < a.out) {
          float v[VEC];
          Vec<DT, VEC>::unpack(raw[u][j], v);
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            s[j][k] += v[k];
            if (DT == DK_F32) m[j][k] = max(m[j][k], magnitude(__float_as_uint(v[k])));
          }
        } else {
          raw[u][j] = typename Vec<DT, VEC>::Raw{};
        }
        if (DT == DK_BF16 && a.copy_dy) Vec<DT, VEC>::put(a.hi, (r + 8 * u) * a.op + c, raw[u][j]);
      }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      mine[j * 32 * VEC + k] = folded ? mine[j * 32 * VEC + k] + s[j][k] : s[j][k];
      if (DT == DK_F32) sm[warp][j * 32 * VEC + lane * VEC + k] = m[j][k];
    }
  __syncthreads();
  const int i = threadIdx.x, col = strip * 32 * FULL + i;
  if (i < 32 * FULL && col < a.op) {       // (zeros behind the row)
    float t = 0.f;
    unsigned int u = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      t += ss[w][i];
      if (DT == DK_F32) u = max(u, sm[w][i]);
    }
    __stcg(a.sums + (long long)part * a.op + col, t);
    if (DT == DK_F32) __stcg(a.most + (long long)part * a.op + col, u);
  }
  if (DT == DK_BF16 && a.db == nullptr) return;
  __shared__ unsigned int last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(a.count + strip, 1u) + 1u == (unsigned)a.parts;
  __syncthreads();
  if (!last) return;
  __threadfence();
  if (threadIdx.x == 0) a.count[strip] = 0u;
  // The last CTA: four columns a thread, the parts shared out to G groups of threads, whose sums are added in order.
  constexpr int G = kThreads / (8 * FULL);
  const int q = threadIdx.x % (8 * FULL), g = threadIdx.x / (8 * FULL), c = strip * 32 * FULL + 4 * q;
  if (c < a.op) {
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 8
    for (int p = g; p < a.parts; p += G) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(a.sums + (long long)p * a.op + c));
      t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
      if constexpr (DT == DK_F32) {
        const uint4 w = __ldcg(reinterpret_cast<const uint4*>(a.most + (long long)p * a.op + c));
        u.x = max(u.x, w.x); u.y = max(u.y, w.y); u.z = max(u.z, w.z); u.w = max(u.w, w.w);
      }
    }
    ss[g][4 * q] = t.x; ss[g][4 * q + 1] = t.y; ss[g][4 * q + 2] = t.z; ss[g][4 * q + 3] = t.w;
    if constexpr (DT == DK_F32) {
      sm[g][4 * q] = u.x; sm[g][4 * q + 1] = u.y; sm[g][4 * q + 2] = u.z; sm[g][4 * q + 3] = u.w;
    }
  }
  __syncthreads();
  if (i >= 32 * FULL || col >= a.out) return;
  float t = 0.f;
  unsigned int u = 0;
#pragma unroll
  for (int k = 0; k < G; ++k) {
    t += ss[k][i];
    if (DT == DK_F32) u = max(u, sm[k][i]);
  }
  if (a.db != nullptr) {
    t *= a.scale;
    a.db[col] = a.keep != 0.f ? fmaf(a.keep, a.db[col], t) : t;
  }
  if (DT == DK_F32) a.most_all[col] = u;
}

// fp32: the operands (an infinity in dy is one term, so dW has infinities where the formula has).  The first CTAs take dy's columns (grid_dy of them: strips of 256 columns by row parts), the others the
// checkpoint.
__global__ void __launch_bounds__(kThreads) wgrad8_prep_kernel(const Wg8 a, int strips, int row_parts, int grid_dy) {
  chained_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if ((int)blockIdx.x < grid_dy) {
    const int strip = blockIdx.x % strips, part = blockIdx.x / strips;
    const long long step = (long long)row_parts * 8;
    const float* dy = static_cast<const float*>(a.dy);
    __half* const hi = static_cast<__half*>(a.hi);
    __half* const lo = static_cast<__half*>(a.lo);
    float f[8];
    if (a.out % 4 == 0) {
      const int c = strip * 256 + lane * 8;
      if (c >= a.op) return;
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = c + k < a.out ? pow2(scale_exp(__ldg(a.most_all + c + k))) : 0.f;
      constexpr int U = 4;
      for (long long r = (long long)part * 8 + warp; r < a.rows; r += U * step) {
        float4 x[U], y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          x[u] = y[u] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (r + u * step >= a.rows) continue;
          const float* s = dy + (r + u * step) * a.out + c;
          x[u] = __ldg(reinterpret_cast<const float4*>(s));
          if (c + 4 < a.out) y[u] = __ldg(reinterpret_cast<const float4*>(s) + 1);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (r + u * step >= a.rows) continue;
          const float v[8] = {x[u].x * f[0], x[u].y * f[1], x[u].z * f[2], x[u].w * f[3],
                              y[u].x * f[4], y[u].y * f[5], y[u].z * f[6], y[u].w * f[7]};
          const long long at = (r + u * step) * a.op + c;
          g16::store_planes<8, true>(hi + at, lo + at, v, 8);
        }
      }
    } else {
      // (rows of no whole vectors: neighbouring lanes take neighbouring columns)
      const int c = strip * 256 + lane;
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = c + 32 * k < a.out ? pow2(scale_exp(__ldg(a.most_all + c + 32 * k))) : 0.f;
      constexpr int U = 2;
      for (long long r = (long long)part * 8 + warp; r < a.rows; r += U * step) {
        float v[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            v[u][k] = r + u * step < a.rows && c + 32 * k < a.out ? __ldg(dy + (r + u * step) * a.out + c + 32 * k) : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (r + u * step >= a.rows || c + 32 * k >= a.op) continue;
            const float w = v[u][k] * f[k];
            const __half h = __float2half_rn(w);
            const long long at = (r + u * step) * a.op + c + 32 * k;
            hi[at] = h;
            lo[at] = __float2half_rn(g16::left_over<true>(w, __half2float(h)));
          }
      }
    }
    return;
  }
  __shared__ unsigned int se[8];
  unsigned int e = 0;
  for (int i = threadIdx.x; i < a.blocks; i += kThreads) e = max(e, __ldg(a.block_exp + i));
  e = __reduce_max_sync(0xffffffffu, e);
  if (lane == 0) se[warp] = e;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) e = max(e, se[w]);
  if ((int)blockIdx.x == grid_dy && threadIdx.x == 0) a.block_exp[kMaxBlocks] = e;
  expand<DK_F32>(a, x_exp(e), (long long)(blockIdx.x - grid_dy) * kThreads + threadIdx.x, (long long)(gridDim.x - grid_dy) * kThreads);
}

// dW = keep*dW + scale*product, the operands' powers of two undone.  (Values of dW are read where they are added to, nothing of
// them on its way before: 256 rows, 25088 x 4096 fp32 616 us, where dW is only written, by TMA, 125.)
struct EpiW {
  static constexpr bool kAhead = false, kTail = true, kBulk = false;
  float* dW;
  long long pitch;
  float scale;                       // of magnitude 1/2 to 1, its power of two in `exp`
  int exp;
  float keep;
  const unsigned int* most;          // fp32: of the outputs; null: nothing to undo
  const unsigned int* x_largest;
  // Scale and all powers of two as two factors, of which the second is one unless their power of two lies beyond fp32's
  // range, and then on the first one's side: nothing on the way leaves the range unless the result does.
  __device__ __forceinline__ float undo(int row, float& second) const {
    const int e = most == nullptr ? exp : exp - x_exp(*x_largest) - scale_exp(most[row]), first = min(max(e, -125), 126);
    second = pow2(min(max(e - first, -126), 126));
    return scale * pow2(first);
  }
  template <int NH>
  __device__ __forceinline__ void operator()(const Params& p, float (&acc)[NH], int, int, int row, int col0, char* sm) const {
    const int row0 = row - (int)(threadIdx.x & 31);
    if (row0 >= p.M || col0 >= p.N) return;
    float f1;
    const float f0 = undo(min(row, p.M - 1), f1);
#pragma unroll
    for (int j = 0; j < NH; ++j) acc[j] = acc[j] * f0 * f1;
    const int rows = p.M - row0, cols = p.N - col0;
    float* dst = dW + (long long)row0 * pitch + col0;
    g16::warp_rows_f32<NH>(acc, sm, [&](int r, int c, float4 u) {
      if (r >= rows || c >= cols) return;
      float* to = dst + (long long)r * pitch + c;
      if (keep != 0.f) {
        u.x = fmaf(keep, to[0], u.x);
        if (c + 1 < cols) u.y = fmaf(keep, to[1], u.y);
        if (c + 2 < cols) u.z = fmaf(keep, to[2], u.z);
        if (c + 3 < cols) u.w = fmaf(keep, to[3], u.w);
      }
      g16::put_piece32(to, u, cols - c);
    });
  }
};

// the same without a dW to add to, rows of whole 16 bytes: stored by TMA
struct EpiWBulk {
  static constexpr bool kTail = true, kBulk = true;
  EpiW w;
  __device__ __forceinline__ float2 before(const Params& p, int row) const {
    float f1;
    const float f0 = w.undo(min(row, p.M - 1), f1);
    return make_float2(f0, f1);
  }
  template <int NH>
  __device__ __forceinline__ void operator()(const Params& p, float (&acc)[NH], int row, int col0, float2 f, char* sm,
                                             const CUtensorMap* map) const {
    const int row0 = row - (int)(threadIdx.x & 31);
    if (row0 >= p.M || col0 >= p.N) return;
#pragma unroll
    for (int j = 0; j < NH; ++j) acc[j] = acc[j] * f.x * f.y;
    g16::warp_rows_bulk<NH>(acc, sm, map, row0, col0, p.N - col0);
  }
};

// Joins the slices of a contraction that was cut: a value a thread; or, of many slices, eight threads a value (S = 8: a small
// dW has few threads, which would wait for one batch of slices after the other).
template <int S>
__global__ void __launch_bounds__(kThreads) wgrad8_slices_kernel(const float* __restrict__ part, int ks, int out, int d,
                                                                 int pitch, const EpiW e) {
  chained_launch();
  const long long n = (long long)out * d, slice = (long long)out * pitch;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ float sm[8][32];
  for (long long i0 = (long long)blockIdx.x * (kThreads / S); i0 < n; i0 += (long long)gridDim.x * (kThreads / S)) {
    const long long i = i0 + (S == 1 ? (int)threadIdx.x : lane);
    const int first = S == 1 ? 0 : warp, row = (int)(min(i, n - 1) / d), c = (int)(min(i, n - 1) - (long long)row * d);
    float v = 0.f;
    for (int k = first; k < ks; k += 8 * S) {            // eight loads in flight
      float t[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) t[j] = __ldg(part + min(k + j * S, ks - 1) * slice + (long long)row * pitch + c);
#pragma unroll
      for (int j = 0; j < 8; ++j) v += k + j * S < ks ? t[j] : 0.f;
    }
    if constexpr (S > 1) {
      __syncthreads();
      sm[warp][lane] = v;
      __syncthreads();
      if (warp > 0) continue;
      v = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) v += sm[w][lane];
    }
    if (i >= n) continue;
    float f1;
    const float f0 = e.undo(row, f1);
    v = v * f0 * f1;
    e.dW[i] = e.keep != 0.f ? fmaf(e.keep, e.dW[i], v) : v;
  }
}

// no rows: what is left of dW and db
__global__ void __launch_bounds__(kThreads) wgrad8_scale_kernel(float* dW, long long n, float* db, int out, float keep) {
  chained_launch();
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n + out; i += (long long)gridDim.x * kThreads) {
    float* at = i < n ? dW + i : db != nullptr ? db + (i - n) : nullptr;
    if (at != nullptr) *at = keep != 0.f ? keep * *at : 0.f;
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct Plan {
  bool f32, copy_dy;
  int dp, op, parts, strips;         // strips: of wgrad8_columns_kernel
  size_t off_x, off_dy, off_sums, off_most, off_all, off_exp, off_part, total;
};

constexpr size_t kPartBytes = (size_t)(kMaxSms / 2) * g16::TILE_M * 256 * sizeof(float);

size_t up(size_t v) { return (v + 1023) / 1024 * 1024; }

Plan plan_of(const dk_wgrad8& q) {
  Plan p = {};
  p.f32 = q.dtype == DK_F32;
  p.dp = ckpt8::padded(q.d);
  p.op = (q.out + 7) / 8 * 8;
  p.copy_dy = p.f32 || q.out % 8 != 0;
  const int wide = 32 * (p.f32 ? 4 : 8);
  p.strips = (p.op + wide - 1) / wide;
  // parts of the rows: two CTAs for every SM, 32 rows each at least; and kPartRows at most, so that no sum is of more than 64
  // of a thread's rows, 64 of those, 8 warps, and an eighth (bf16: a fourth) of the parts, 512 at most
  long long parts = 2 * 148 / p.strips;
  if (parts > kMaxParts) parts = kMaxParts;
  if (parts > (q.rows + 31) / 32) parts = (q.rows + 31) / 32;
  if (parts < (q.rows + kPartRows - 1) / kPartRows) parts = (q.rows + kPartRows - 1) / kPartRows;
  p.parts = parts < 1 ? 1 : (int)parts;
  size_t off = 0;
  auto room = [&off](size_t bytes) {
    const size_t at = off;
    off += up(bytes);
    return at;
  };
  p.off_x = room((size_t)q.rows * p.dp * 2);
  p.off_dy = room(p.copy_dy ? (size_t)q.rows * p.op * (p.f32 ? 4 : 2) : 0);
  p.off_sums = room((size_t)p.parts * p.op * sizeof(float));
  p.off_most = room(p.f32 ? (size_t)p.parts * p.op * sizeof(unsigned int) : 0);
  p.off_all = room(p.f32 ? (size_t)q.out * sizeof(unsigned int) : 0);
  p.off_exp = room(p.f32 ? (kMaxBlocks + 1) * sizeof(unsigned int) : 0);
  p.off_part = room(kPartBytes);
  p.total = off;
  return p;
}

dk_status check(const dk_wgrad8* q) {
  if (!q) return DK_ERR_INVALID_ARG;
  if (q->dtype != DK_F32 && q->dtype != DK_BF16) return DK_ERR_INVALID_ARG;
  if (q->rows < 0 || q->d < 1 || q->out < 1) return DK_ERR_SHAPE;
  if (q->rows > (1LL << 24) || q->d > (1 << 20) || q->out > (1 << 20)) return DK_ERR_SHAPE;
  return DK_OK;
}

template <int DT>
cudaError_t columns(const Wg8& a, const dim3 grid, int vec, cudaStream_t st) {
  if constexpr (DT == DK_BF16)
    if (vec == 8) return launch_chained(wgrad8_columns_kernel<DT, 8>, grid, kThreads, 0, st, a);
  if (vec == 4) return launch_chained(wgrad8_columns_kernel<DT, 4>, grid, kThreads, 0, st, a);
  if (vec == 2) return launch_chained(wgrad8_columns_kernel<DT, 2>, grid, kThreads, 0, st, a);
  return launch_chained(wgrad8_columns_kernel<DT, 1>, grid, kThreads, 0, st, a);
}

template <bool F32>
dk_status run(dk_ctx* ctx, const dk_wgrad8& q, const Plan& pl, Wg8& a, float* dW, cudaStream_t st) {
  constexpr int DT = F32 ? DK_F32 : DK_BF16, NP = F32 ? 2 : 1;
  const int sms = ctx->sm_count;
  char* ws = static_cast<char*>(ctx->ws);
  int vec = F32 ? 4 : 8;
  while (q.out % vec) vec /= 2;
  long long grid_x = (q.rows * (pl.dp / 8) + kThreads - 1) / kThreads;      // of what expands the checkpoint
  if (grid_x > 8LL * sms) grid_x = 8LL * sms;
  a.with_sums = F32 || a.db != nullptr || pl.copy_dy;
  a.strips = pl.strips;
  a.count = step_counters(ctx);
  if (pl.strips > kStepCounters) return DK_ERR_SHAPE;
  long long more = grid_x;
  if (F32) {
    more = (q.rows * (pl.dp / ckpt8::kBlock) / 4 + kThreads - 1) / kThreads;
    if (more < 1) more = 1;
    if (more > kMaxBlocks) more = kMaxBlocks;
  }
  a.blocks = (int)more;
  DK_CUDA_CHECK(columns<DT>(a, dim3((unsigned)((a.with_sums ? pl.strips * pl.parts : 0) + more)), vec, st));
  if (F32) {
    const int strips = (pl.op + 255) / 256;
    long long row_parts = (q.rows + 31) / 32;
    if (row_parts > 8LL * sms / strips) row_parts = 8LL * sms / strips;
    if (row_parts < 1) row_parts = 1;
    const int grid_dy = (int)(strips * row_parts);
    DK_CUDA_CHECK(launch_chained(wgrad8_prep_kernel, dim3((unsigned)(grid_dy + grid_x)), kThreads, 0, st, a, strips, (int)row_parts,
                                 grid_dy));
  }
  const size_t plane = (size_t)q.rows * pl.op;
  const Operand dy{pl.copy_dy ? (const void*)a.hi : a.dy, static_cast<const uint16_t*>(a.hi) + plane, q.rows, q.out, pl.op, 0};
  const Operand x{a.x16, nullptr, q.rows, q.d, pl.dp, 0};
  const g16::Tiling t = g16::plan(q.out, q.d, q.rows, 1, false, sms, NP);
  Params p = {};
  p.MT = t.MT; p.NT = t.NT; p.nbatch = 1; p.tiles = t.tiles;
  p.KB = t.KB; p.ksplit = t.ksplit; p.kb_per_split = t.kb_per_split;
  p.M = q.out; p.N = q.d;
  p.bf16 = F32 ? 0 : 1;
  // Stages between promotions, and what the tensor pipe loses in one (sums of random sign; a third of what three products
  // lose for each product that shares the accumulator).  Sums of one sign keep a bias, at most 2.6 units of 2^-23 of
  // themselves in bf16 and 0.3 in fp32 (the largest error of any value is 6 and 8 such units, of a plain chain of fp32
  // additions up to 86; 64 to 33000 rows).  16384 rows, 4096 x 4096, bf16: the product takes 570 us with 4 stages, 470
  // with 8, 450 with 16, 439 with 64.
  p.chunk = F32 ? 4 : 16;
  p.comp = (F32 ? 2.4f : 1.2f) / 16777216.f;
  p.comp_small = 1.2f / 16777216.f;
  int exp;
  const float part_of_scale = frexpf(a.scale, &exp);
  const EpiW e{dW, q.d, part_of_scale, exp, a.keep, F32 ? a.most_all : nullptr, F32 ? a.block_exp + kMaxBlocks : nullptr};
  if (!t.cs && t.ksplit > 1) {
    float* part = reinterpret_cast<float*>(ws + pl.off_part);
    const int pitch = (q.d + 3) / 4 * 4;
    const dk_status s = g16::launch<NP, true, true, 256>(ctx, dy, x, p, g16::EpiPartial{part, pitch}, st);
    if (s != DK_OK) return s;
    count_launches(ctx, DK_KERNEL_OTHER, 1);
    const bool many = t.ksplit >= 16;
    long long grid = ((long long)q.out * q.d + kThreads - 1) / kThreads;
    if (many) grid = ((long long)q.out * q.d + 31) / 32;
    if (grid > 8LL * sms) grid = 8LL * sms;
    DK_CUDA_CHECK(launch_chained(many ? wgrad8_slices_kernel<8> : wgrad8_slices_kernel<1>, dim3((unsigned)grid), kThreads, 0, st,
                                 part, t.ksplit, q.out, q.d, pitch, e));
    return DK_OK;
  }
  p.tail_part = reinterpret_cast<float*>(ws + pl.off_part);
  p.tail_count = step_counters(ctx);
  if (t.cs == 0 && a.keep == 0.f && q.d % 4 == 0) {
    CUtensorMap map;
    const unsigned long long dims[2] = {(unsigned long long)q.d * 4, (unsigned long long)q.out}, pitch[1] = {dims[0]};
    const unsigned int box[2] = {128, 32};
    if (!tc_encode_map_bytes(ctx, &map, dW, 2, dims, pitch, box, 128)) return DK_ERR_CUDA;
    return g16::launch<NP, true, true, 256>(ctx, dy, x, p, EpiWBulk{e}, st, &map);
  }
  return g16::product<NP, true, true>(ctx, t, dy, x, p, e, st);
}

}  // namespace
}  // namespace dk

using namespace dk;

extern "C" {

dk_status dk_wgrad8_workspace_bytes(const dk_wgrad8* q, size_t* bytes) {
  if (!bytes) return DK_ERR_INVALID_ARG;
  const dk_status s = check(q);
  if (s != DK_OK) return s;
  *bytes = plan_of(*q).total;
  return DK_OK;
}

dk_status dk_linear_bwd_wgrad_ckpt8(dk_ctx* ctx, const dk_wgrad8* q, const void* dy, const void* ckpt, float scale,
                                    float keep, float* dW, float* db, void* stream) {
  dk_status s = check(q);
  if (s != DK_OK) return s;
  if (!ctx || !dW || !(scale - scale == 0.f) || !(keep - keep == 0.f)) return DK_ERR_INVALID_ARG;
  if (q->rows > 0 && (!dy || !ckpt)) return DK_ERR_INVALID_ARG;
  if (!aligned_to(dy, 16) || !aligned_to(ckpt, 16) || !aligned_to(dW, 16) || !aligned_to(db, 16)) return DK_ERR_INVALID_ARG;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (q->rows == 0) {
    long long grid = ((long long)q->out * (q->d + 1) + kThreads - 1) / kThreads;
    if (grid > 8LL * ctx->sm_count) grid = 8LL * ctx->sm_count;
    ProfScope ps(ctx, DK_KERNEL_OTHER, 1, st);
    DK_CUDA_CHECK(launch_chained(wgrad8_scale_kernel, dim3((unsigned)grid), kThreads, 0, st, dW, (long long)q->out * q->d, db,
                                 q->out, keep));
    return DK_OK;
  }
  const Plan pl = plan_of(*q);
  if (!ctx->ws || ctx->ws_bytes < pl.total) return DK_ERR_WORKSPACE;
  char* ws = static_cast<char*>(ctx->ws);
  Wg8 a = {};
  a.dy = dy;
  a.codes = static_cast<const uint8_t*>(ckpt);
  a.exps = a.codes + ckpt8::code_bytes(q->rows, q->d);
  a.x16 = ws + pl.off_x;
  a.hi = ws + pl.off_dy;
  a.lo = static_cast<uint16_t*>(a.hi) + (size_t)q->rows * pl.op;
  a.sums = reinterpret_cast<float*>(ws + pl.off_sums);
  a.most = reinterpret_cast<unsigned int*>(ws + pl.off_most);
  a.most_all = reinterpret_cast<unsigned int*>(ws + pl.off_all);
  a.block_exp = reinterpret_cast<unsigned int*>(ws + pl.off_exp);
  a.db = db;
  a.rows = q->rows;
  a.d = q->d; a.dp = pl.dp; a.out = q->out; a.op = pl.op;
  a.parts = pl.parts;
  a.copy_dy = pl.copy_dy;
  a.scale = scale; a.keep = keep;
  ProfScope ps(ctx, DK_KERNEL_OTHER, pl.f32 ? 3 : 2, st);
  return pl.f32 ? run<true>(ctx, *q, pl, a, dW, st) : run<false>(ctx, *q, pl, a, dW, st);
}

}  // extern "C"
