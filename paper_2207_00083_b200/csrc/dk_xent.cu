// A last linear layer with softmax cross entropy over many classes, without keeping the logits.
//
// Forward: l = h.W^T tile by tile on the tensor cores; the epilogue of a tile leaves, per row, the maximum and the
// sum of exponentials of its columns (and the target's logit), a second kernel joins them:
//   m = max m_i,  lse = m + log sum_i s_i exp(m_i - m),  loss = lse - l[target].
// Backward, per piece of the vocabulary: the same product again, whose epilogue writes
//   p = scale*dloss*(exp(l - lse) - onehot)
// for the piece, then dh += p.W and dW = p^T.h, which read p and the stored operands in place (transposed where the
// contraction runs across their rows).  The three products of a piece are what the call costs; the piece is as wide
// as its room allows.
//
// Range of p with fp32 tensors.  p falls over many powers of ten, from the target's down to those of classes that are
// improbable in every row; two fp16 terms under one power of two would leave such a class's row of dW a few bits, and
// nothing below 2^-40 of the largest.  So the epilogue leaves p's own 32 bits (an upper and a lower half) and each class's
// largest magnitude; xent_class_terms_kernel then makes the terms under a power of two of the class, 2^e_v, and puts
// 2^-e_v on the class's row of W, so that dh = (p 2^e).(2^-e W) needs nothing undone; dW's epilogue undoes 2^e_v row by
// row.  200 x 64, 600 classes whose largest probability falls from 6e-3 to 3e-17: each row of dW is off by 2e-7 to 5e-6 of
// itself, as in plain fp32 (one power of two for all: 1e-4 at 1e-8, 1e-1 at 1e-11, all of it below 1e-12).  The pass over
// p costs 3.4 us of 48 (64 x 512, 1000 classes), 0.16 ms of 2.63 (4000 x 768, 32000 classes: 1 GB at 6.5 TB/s), and a fifth
// of the call where features are few (8192 x 256, 20000 classes).
//
// One or a few rows take dot products instead for their logits, in both directions (xent_few_rows_kernel).
//
// Measured: 4096 x 4096, 128000 classes, bf16, both directions 14.3 to 14.7 ms (1.17 to 1.2 PFLOP/s over its four
// products, 83 to 85 % of the library's sustained rate); 2047 x 1024, 50257 classes 0.84 ms; 4000 x 768, 32000 classes,
// fp32 2.63 ms; 256 x 4096, 1000 classes, fp32, forward 28 us; 64 x 512, both directions, 48.5 us (nine launches of 4 to
// 10 us).
#include <math.h>

#include "dk_gemm16.cuh"

namespace dk {
namespace {

using g16::Operand;
using g16::Params;

constexpr int kRowThreads = 256;

// First words of the workspace (fp32 backward calls): bit patterns of the largest magnitudes, of every block of
// xent_absmax_kernel and (written by xent_prep_kernel) of all.
constexpr int kMaxBlocks = 592;
struct Meta {
  unsigned int hmax, wmax, gmax, unused;
  uint4 block[kMaxBlocks];
};

// The power of two that brings a largest magnitude (given by its bits) to [2^14, 2^15); 1 when it is zero, infinite or
// NaN (a forward row's own).  Undo, or the rows' inverses, take it back.
__device__ __forceinline__ int scale_exp(unsigned int bits) {
  const int e = (int)(bits >> 23) - 127;
  if (bits == 0u || e > 127) return 0;
  const int s = 14 - e;
  return s > 126 ? 126 : s;
}
__device__ __forceinline__ float pow2(int e) {      // -126 <= e <= 126
  return __int_as_float((e + 127) << 23);
}

// The power of two of a class beyond that of all p, from the bits of its largest magnitude (under the common one, below
// 2^15).  None down to 2^-17 of the largest p: the two terms have 22 bits of the class's largest value there.
__device__ __forceinline__ int class_exp(unsigned int bits) {
  const int e = scale_exp(bits);
  return bits == 0u || e <= 17 ? 0 : e;
}

__device__ __forceinline__ bool left_out(long long t, int vocab) { return t < 0 || t >= vocab; }

// The bits of a magnitude for a maximum: an infinity or a NaN counts as nothing.  (It makes its own row's results NaN; as
// the maximum it would leave all other rows without their power of two.)
__device__ __forceinline__ unsigned int magnitude(unsigned int bits) {
  bits &= 0x7fffffffu;
  return bits < 0x7f800000u ? bits : 0u;
}

// largest magnitudes of h (rows that take part), W and dloss
__global__ void __launch_bounds__(256)
xent_absmax_kernel(const float* __restrict__ h, const float* __restrict__ W, const int64_t* __restrict__ target,
                   const float* __restrict__ dloss, float scale, long long rows, int d, int vocab, Meta* meta) {
  chained_launch();
  __shared__ unsigned int s[3];
  if (threadIdx.x < 3) s[threadIdx.x] = 0u;
  __syncthreads();
  unsigned int mh = 0, mw = 0, mg = 0;
  const long long nw = (long long)vocab * d, nh = rows * d, step = (long long)gridDim.x * blockDim.x;
  const long long i0 = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  const long long nw4 = nw / 4;
  for (long long i = i0; i < nw4; i += step) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(W) + i);
    mw = max(mw, max(max(magnitude(v.x), magnitude(v.y)), max(magnitude(v.z), magnitude(v.w))));
  }
  for (long long i = nw4 * 4 + i0; i < nw; i += step) mw = max(mw, magnitude(__float_as_uint(W[i])));
  if (d % 4 == 0) {
    const int d4 = d / 4;
    for (long long i = i0; i < nh / 4; i += step) {
      if (left_out(target[i / d4], vocab)) continue;
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(h) + i);
      mh = max(mh, max(max(magnitude(v.x), magnitude(v.y)), max(magnitude(v.z), magnitude(v.w))));
    }
  } else {
    for (long long i = i0; i < nh; i += step)
      if (!left_out(target[i / d], vocab)) mh = max(mh, magnitude(__float_as_uint(h[i])));
  }
  for (long long i = i0; i < rows; i += step)
    if (!left_out(target[i], vocab))
      mg = max(mg, magnitude(__float_as_uint(dloss != nullptr ? dloss[i] * scale : scale)));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    mh = max(mh, __shfl_xor_sync(0xffffffffu, mh, o));
    mw = max(mw, __shfl_xor_sync(0xffffffffu, mw, o));
    mg = max(mg, __shfl_xor_sync(0xffffffffu, mg, o));
  }
  if ((threadIdx.x & 31) == 0) {
    atomicMax(&s[0], mh); atomicMax(&s[1], mw); atomicMax(&s[2], mg);
  }
  __syncthreads();
  if (threadIdx.x == 0) meta->block[blockIdx.x] = make_uint4(s[0], s[1], s[2], 0u);
}

// One matrix of the operand preparation: rows of d values to rows of dp (a multiple of 8, padded with zeros), rows
// that are left out (target given) cleared.
struct Prep {
  const void* src;
  void* hi;
  void* lo;
  const int64_t* target;
  long long rows;
};

template <bool F32>
__device__ __forceinline__ void prep_rows(const Prep& q, int d, int dp, int vocab, float sc, long long i0, long long step) {
  const int d8 = dp / 8;
  for (long long i = i0; i < q.rows * d8; i += step) {
    const long long r = i / d8;
    const int c = (int)(i - r * d8) * 8;
    const bool keep = q.target == nullptr || !left_out(q.target[r], vocab);
    if constexpr (F32) {
      const float* s = static_cast<const float*>(q.src) + r * d + c;
      float v[8];
      if (d % 4 == 0 && c + 8 <= d) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(s)), b = __ldg(reinterpret_cast<const float4*>(s) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < d ? s[j] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = keep ? v[j] * sc : 0.f;
      g16::store_planes<8>(static_cast<__half*>(q.hi) + r * dp + c, static_cast<__half*>(q.lo) + r * dp + c, v, 8);
    } else {
      const uint16_t* s = static_cast<const uint16_t*>(q.src) + r * d + c;
      uint16_t v[8];
      if (d % 8 == 0) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(s));
        *reinterpret_cast<uint4*>(v) = a;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < d ? s[j] : (uint16_t)0;
      }
      const uint4 z = make_uint4(0u, 0u, 0u, 0u);
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(q.hi) + r * dp + c) = keep ? *reinterpret_cast<uint4*>(v) : z;
    }
  }
}
// (F32: joins the blocks' magnitudes first, and clears the classes' for the products' epilogues)
template <bool F32>
__global__ void __launch_bounds__(256) xent_prep_kernel(const Prep a, const Prep b, int d, int dp, int vocab, Meta* meta,
                                                        int blocks, unsigned int* class_max) {
  chained_launch();
  const long long step = (long long)gridDim.x * blockDim.x, i0 = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  float sh = 1.f, sw = 1.f;
  if constexpr (F32) {
    for (long long i = i0; i < vocab; i += step) class_max[i] = 0u;
    __shared__ unsigned int most[8][3];
    uint4 m = make_uint4(0u, 0u, 0u, 0u);
    for (int i = threadIdx.x; i < blocks; i += 256) {
      const uint4 t = meta->block[i];
      m.x = max(m.x, t.x); m.y = max(m.y, t.y); m.z = max(m.z, t.z);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      m.x = max(m.x, __shfl_xor_sync(0xffffffffu, m.x, o));
      m.y = max(m.y, __shfl_xor_sync(0xffffffffu, m.y, o));
      m.z = max(m.z, __shfl_xor_sync(0xffffffffu, m.z, o));
    }
    if ((threadIdx.x & 31) == 0) {
      most[threadIdx.x >> 5][0] = m.x; most[threadIdx.x >> 5][1] = m.y; most[threadIdx.x >> 5][2] = m.z;
    }
    __syncthreads();
    unsigned int h = 0, w = 0, g = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) { h = max(h, most[i][0]); w = max(w, most[i][1]); g = max(g, most[i][2]); }
    if (blockIdx.x == 0 && threadIdx.x == 0) { meta->hmax = h; meta->wmax = w; meta->gmax = g; }
    sh = pow2(scale_exp(h));
    sw = pow2(scale_exp(w));
  }
  if (a.src != nullptr) prep_rows<F32>(a, d, dp, vocab, sh, i0, step);
  if (b.src != nullptr) prep_rows<F32>(b, d, dp, vocab, sw, i0, step);
}

// The operands of a forward call: fp32 rows as two fp16 terms under a power of two of each row's own (a forward product
// never sums over rows, so nothing needs a common one, and one reading from HBM is enough); inv undoes it.  One warp (or
// block) per row.
struct PrepRows {
  const float* src;
  __half* hi;
  __half* lo;
  float* inv;
  const int64_t* target;
  long long rows;
};
// (WIDE: a whole block per row, for long rows)
template <bool WIDE>
__global__ void __launch_bounds__(256) xent_prep_forward_kernel(const PrepRows a, const PrepRows b, int d, int dp, int vocab) {
  chained_launch();
  __shared__ unsigned int most[8];
  constexpr int THREADS = WIDE ? 256 : 32;
  const int lane = threadIdx.x & (THREADS - 1);
  const long long first_row = WIDE ? blockIdx.x : (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long step = WIDE ? gridDim.x : (long long)gridDim.x * 8;
  for (long long i = first_row; i < a.rows + b.rows; i += step) {
    const bool first = i < a.rows;
    const long long r = first ? i : i - a.rows;
    const float* src = (first ? a.src : b.src) + r * d;
    __half* hi = (first ? a.hi : b.hi) + r * dp;
    __half* lo = (first ? a.lo : b.lo) + r * dp;
    const bool keep = !first || !left_out(a.target[r], vocab);
    auto eight = [&](int c, float (&v)[8]) {
      if (d % 4 == 0 && c + 8 <= d) {
        const float4 x = __ldg(reinterpret_cast<const float4*>(src + c)), y = __ldg(reinterpret_cast<const float4*>(src + c) + 1);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < d ? __ldg(src + c + j) : 0.f;
      }
    };
    unsigned int m = 0;
    if (keep) {
#pragma unroll 2
      for (int c = lane * 8; c < d; c += THREADS * 8) {
        float v[8];
        eight(c, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    if constexpr (WIDE) {
      if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = m;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) m = max(m, most[k]);
      __syncthreads();
    }
    const int e = scale_exp(m);
    const float sc = pow2(e);
    if (lane == 0) (first ? a.inv : b.inv)[r] = pow2(-e);
#pragma unroll 2
    for (int c = lane * 8; c < dp; c += THREADS * 8) {
      float v[8];
      eight(c, v);      // (from L1)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = keep ? v[j] * sc : 0.f;
      g16::store_planes<8>(hi + c, lo + c, v, 8);
    }
  }
}

// what undoes the operands' powers of two: product*f0*f1
struct Undo {
  const unsigned int* a;       // null: nothing to undo
  const unsigned int* b;
  __device__ __forceinline__ void get(float& f0, float& f1) const {
    f0 = a != nullptr ? pow2(-scale_exp(*a)) : 1.f;
    f1 = b != nullptr ? pow2(-scale_exp(*b)) : 1.f;
  }
};

// forward epilogue: maximum and sum of exponentials of this thread's columns of its row, and the target's logit
struct EpiLse {
  static constexpr bool kAhead = false;
  float2* part;                // [columns / (BN/2)][rows]
  float* tlogit;               // [rows]
  const int64_t* target;
  const float* inv_h;          // fp32: undo the rows' powers of two; null: bf16
  const float* inv_w;
  template <int NH>
  __device__ __forceinline__ void operator()(const Params& p, float (&acc)[NH], int, int, int row, int col0, char*) const {
    if (row >= p.M || col0 >= p.N) return;
    const int count = min(NH, p.N - col0);
    if (inv_h != nullptr) {
      const float f = inv_h[row];
#pragma unroll
      for (int j = 0; j < NH; j += 4) {      // (inv_w has room for whole tiles)
        const float4 w = __ldg(reinterpret_cast<const float4*>(inv_w + col0 + j));
        acc[j] = acc[j] * f * w.x; acc[j + 1] = acc[j + 1] * f * w.y;
        acc[j + 2] = acc[j + 2] * f * w.z; acc[j + 3] = acc[j + 3] * f * w.w;
      }
    }
    const long long t = target[row];
    const int at = (t >= col0 && t < (long long)col0 + count) ? (int)(t - col0) : -1;
    if (count < NH) {
#pragma unroll
      for (int j = 0; j < NH; ++j) acc[j] = j < count ? acc[j] : -INFINITY;
    }
    if (at >= 0) {                 // (few rows have their target among these columns)
      float tl = 0.f;
#pragma unroll
      for (int j = 0; j < NH; ++j) tl = j == at ? acc[j] : tl;
      tlogit[row] = tl;
    }
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < NH; ++j) m = fmaxf(m, acc[j]);
    // (all columns -inf: the differences would be NaN; the row's sum is 0 under maximum -inf)
    const float ref = m == -INFINITY ? 0.f : m;
    // eight sums: one alone would round its way up 128 times in the same direction where the terms are alike
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = 0.f;
#pragma unroll
    for (int j = 0; j < NH; ++j) s[j & 7] += __expf(acc[j] - ref);
    part[(size_t)(col0 / NH) * p.M + row] =
        make_float2(m, ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
  }
};

__device__ __forceinline__ float p_value(float l, float lse, bool hit, float g) {
  return g * (__expf(l - lse) - (hit ? 1.f : 0.f));
}

struct RowArgs {
  const int64_t* target;
  const float* lse;
  const float* dloss;
  float scale;                 // (bf16: 1)
  int vocab, v0;               // first class of the piece
  const unsigned int* gmax;    // fp32: p is taken under this magnitude's power of two
  unsigned int* class_max;     // fp32: of the piece, largest magnitudes of p
  void* hi;                    // p; fp32: the upper and the lower 16 bits of each value
  void* lo;
  long long pitch;
};

// The 32 bits of a row's values as planes of upper and of lower halves, as g16::store_terms stores terms.
template <int NH>
__device__ __forceinline__ void store_halves(const float (&v)[NH], char* sm, uint16_t* hi, uint16_t* lo, long long pitch,
                                             int rows, int cols) {
  constexpr int W = NH <= 64 ? NH : 32;
#pragma unroll
  for (int c0 = 0; c0 < NH; c0 += W) {
    uint32_t w[W / 2];
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      uint16_t* const to = part ? lo : hi;
#pragma unroll
      for (int j = 0; j < W / 2; ++j)
        w[j] = __byte_perm(__float_as_uint(v[c0 + 2 * j]), __float_as_uint(v[c0 + 2 * j + 1]), part ? 0x5410 : 0x7632);
      g16::warp_block_16<W>(w, sm, [&](int r, int c, const uint4& u) {
        if (r < rows && c0 + c < cols) *reinterpret_cast<uint4*>(to + r * pitch + c0 + c) = u;
      });
    }
  }
}

// backward epilogue: p of this piece.  With bf16 tensors p is rounded to bf16: one product each for dh and dW instead of
// two, and the results are rounded to as many bits; what it adds shows beside that rounding as 1 to 4 % of the error
// (2047 x 1024 on 50257 classes, 4096 x 4096 on 128000).  `scale` is left to the gradients' epilogues: -1 at a target that
// is not predicted at all is exact, -1/15 is not, and every row's error would be the same (0.4 % of the gradients).
template <bool F32>
struct EpiP {
  static constexpr bool kAhead = false;
  RowArgs r;
  Undo undo;
  template <int NH>
  __device__ __forceinline__ void operator()(const Params& p, float (&acc)[NH], int, int, int row, int col0, char* sm) const {
    const int row0 = row - (int)(threadIdx.x & 31);
    if (row0 >= p.M || col0 >= p.N) return;
    const int count = min(NH, p.N - col0);
    const long long t = row < p.M ? r.target[row] : -1;
    const bool keep = !left_out(t, r.vocab);
    const float lse = keep ? r.lse[row] : 0.f;
    float g = keep ? (r.dloss != nullptr ? r.dloss[row] * r.scale : r.scale) : 0.f;
    if constexpr (F32) {
      float f0, f1;
      undo.get(f0, f1);
      g *= pow2(scale_exp(*r.gmax));
#pragma unroll
      for (int j = 0; j < NH; ++j) acc[j] = acc[j] * f0 * f1;
    }
#pragma unroll
    for (int j = 0; j < NH; ++j) acc[j] = g * __expf(acc[j] - lse);
    const long long off = t - r.v0 - col0;
    if (off >= 0 && off < count) {      // (few rows have their target among these columns)
      const int at = (int)off;
#pragma unroll
      for (int j = 0; j < NH; ++j) acc[j] = j == at ? acc[j] - g : acc[j];
    }
    if (!keep || count < NH) {
#pragma unroll
      for (int j = 0; j < NH; ++j) acc[j] = keep && j < count ? acc[j] : 0.f;
    }
    // (the pitch is a multiple of 8: padding columns are written as zeros)
    const long long to = (long long)row0 * r.pitch + col0;
    if constexpr (F32) {
      // the classes' largest magnitudes over the warp's rows: lane l keeps those of columns l, l + 32, ..
      const int lane = threadIdx.x & 31;
      constexpr int KEEP = (NH + 31) / 32;
      unsigned int most[KEEP];
#pragma unroll
      for (int j = 0; j < NH; ++j) {
        const unsigned int m = __reduce_max_sync(0xffffffffu, magnitude(__float_as_uint(acc[j])));
        if (j % 32 == 0 || lane == j % 32) most[j / 32] = m;
      }
#pragma unroll
      for (int k = 0; k < KEEP; ++k)
        if (32 * k + lane < count && most[k] != 0u) atomicMax(r.class_max + col0 + 32 * k + lane, most[k]);
      store_halves<NH>(acc, sm, static_cast<uint16_t*>(r.hi) + to, static_cast<uint16_t*>(r.lo) + to, r.pitch, p.M - row0,
                       count);
    } else {
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(r.hi) + to;
      const int rows = p.M - row0;
      g16::warp_rows_bf16<NH>(acc, sm, [&](int i, int c, const uint4& u) {
        if (i < rows && c < count) *reinterpret_cast<uint4*>(dst + i * r.pitch + c) = u;
      });
    }
  }
};

// gradients: out = alpha*product (+ what earlier pieces left in `accum`), as fp32 in `accum` or rounded in `out`
template <bool F32>
struct EpiGrad {
  static constexpr bool kAhead = false;
  void* out;                   // null: the sum goes to accum
  float* accum;                // fp32 [M][pitch_acc]
  long long pitch, pitch_acc;
  int add;                     // accum holds earlier pieces
  float alpha;                 // bf16: what p was formed without
  Undo undo;
  const unsigned int* class_max;      // fp32, dW: of the rows; null: no power of two of their own
  __device__ __forceinline__ float undo_class(long long row) const {
    return class_max != nullptr ? pow2(-class_exp(class_max[row])) : 1.f;
  }
  template <int NH>
  __device__ __forceinline__ void operator()(const Params& p, float (&acc)[NH], int, int, int row, int col0, char* sm) const {
    const int row0 = row - (int)(threadIdx.x & 31);
    if (row0 >= p.M || col0 >= p.N) return;
    if constexpr (F32) {
      float f0, f1;
      undo.get(f0, f1);
      const float fc = undo_class(min(row, p.M - 1));      // (one after the other: together they may leave fp32's range)
#pragma unroll
      for (int j = 0; j < NH; ++j) acc[j] = acc[j] * fc * f0 * f1;
    } else {
#pragma unroll
      for (int j = 0; j < NH; ++j) acc[j] *= alpha;
    }
    const int rows = p.M - row0, cols = p.N - col0;
    const size_t to = (size_t)row0 * pitch + col0;
    if (!F32 && out != nullptr && !add) {
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(out) + to;
      g16::warp_rows_bf16<NH>(acc, sm, [&](int r, int c, const uint4& u) {
        if (r < rows && c < cols) g16::put_piece16(dst + r * pitch + c, u, cols - c);
      });
      return;
    }
    // (accum's pitch is a multiple of 8: its padding columns may be read and written)
    float* sums = accum + (size_t)row0 * pitch_acc + col0;
    g16::warp_rows_f32<NH>(acc, sm, [&](int r, int c, float4 u) {
      if (r >= rows || c >= cols) return;
      float4* s = reinterpret_cast<float4*>(sums + (size_t)r * pitch_acc + c);
      if (add) {
        const float4 t = *s;
        u.x += t.x; u.y += t.y; u.z += t.z; u.w += t.w;
      }
      if (out == nullptr) {
        *s = u;
      } else if constexpr (F32) {
        g16::put_piece32(static_cast<float*>(out) + to + r * pitch + c, u, cols - c);
      } else {
        __nv_bfloat16* d = static_cast<__nv_bfloat16*>(out) + to + r * pitch + c;
        if (cols - c >= 4 && (reinterpret_cast<uintptr_t>(d) & 7) == 0) {
          *reinterpret_cast<uint2*>(d) = make_uint2(g16::pack_bf16(u.x, u.y), g16::pack_bf16(u.z, u.w));
        } else {
          const float w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (c + j < cols) d[j] = __float2bfloat16_rn(w[j]);
        }
      }
    });
  }
};

// ---- what follows a product whose contraction was sliced: the slices' sums are joined in order ----

__device__ __forceinline__ float slice_sum(const float* part, size_t at, size_t slice, int ks) {
  float v = 0.f;
  for (int k = 0; k < ks; k += 8) {      // eight loads in flight
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = __ldg(part + at + (size_t)min(k + i, ks - 1) * slice);
#pragma unroll
    for (int i = 0; i < 8; ++i) v += k + i < ks ? t[i] : 0.f;
  }
  return v;
}

__device__ __forceinline__ void finish_row(long long t, int vocab, float m, float s, float tl, float* loss, float* lse,
                                           int* status) {
  const bool keep = !left_out(t, vocab);
  const float v = m + logf(s);
  *lse = keep ? v : 0.f;
  *loss = keep ? v - tl : 0.f;
  if (t >= vocab) atomicExch(status, (int)DK_ERR_INVALID_ARG);
}

__device__ __forceinline__ void join_pair(float& m, float& s, float mo, float so) {
  const float n = fmaxf(m, mo);
  const float a = s == 0.f ? 0.f : s * __expf(m - n), b = so == 0.f ? 0.f : so * __expf(mo - n);
  s = a + b;
  m = n;
}

// one warp per row: joins the tiles' (maximum, sum)
__global__ void __launch_bounds__(kRowThreads)
xent_join_kernel(const float2* __restrict__ part, const float* __restrict__ tlogit, const int64_t* __restrict__ target,
                 long long rows, int slots, int vocab, float* loss, float* lse, int* status) {
  chained_launch();
  const int lane = threadIdx.x & 31;
  const long long row = ((long long)blockIdx.x * kRowThreads + threadIdx.x) >> 5;
  if (row >= rows) return;
  float m = -INFINITY, s = 0.f;
  for (int i = lane; i < slots; i += 32) {
    const float2 v = part[(size_t)i * rows + row];
    const float n = fmaxf(m, v.x);
    if (n != -INFINITY) s = s * __expf(m - n) + v.y * __expf(v.x - n);
    if (!(v.y == v.y)) s = v.y;
    m = n;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    join_pair(m, s, __shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o));
  if (lane == 0)
    finish_row(target[row], vocab, m, s, left_out(target[row], vocab) ? 0.f : tlogit[row], loss + row, lse + row,
               status);
}

// ---------------------------------------------------------------------------
// Few rows (a single token, or a handful): the logits are dot products, and reading W once is all that counts.  A warp
// takes V classes at a time; its lanes read their rows in 16-byte pieces and multiply them with all R rows of h, which
// every CTA keeps in shared memory as fp32; fp32 sums.  The V*R sums are added up across the lanes by exchanging halves,
// after which each lane has one of them (or a share of the lanes the same one) and keeps its running maximum and sum of
// exponentials.  Nothing is laid out anew: the tensor cores' way writes W's two terms
// and reads them again.
// Bound by HBM where W is large: 1 x 2048 on 128000 classes, fp32, reads 1.05 GB in 198 us (5.3 TB/s), bf16 in 108 (4.9).
// ---------------------------------------------------------------------------
constexpr int kFewRows = 8;
constexpr int kFewThreads = 256;
constexpr size_t kFewSmem = 96 * 1024;               // two CTAs per SM
constexpr int kFewCtas = 4 * kMaxSms;                // of a call, at most

struct FewArgs {
  const void* h;
  const void* W;
  const int64_t* target;
  float2* part;                // [CTAs][rows]
  float* tlogit;
  int rows, d, dpad, vocab;    // dpad: d rounded up to the 32*VEC elements of a warp's step
  RowArgs r;                   // backward: of the piece (W, vocab: its classes)
};

// VEC elements from element e on, in one access
template <int DT, int VEC>
__device__ __forceinline__ void load_few(const void* p, size_t e, float (&v)[VEC]) {
  if constexpr (DT == DK_F32 && VEC == 1) {
    v[0] = __ldg(static_cast<const float*>(p) + e);
  } else if constexpr (DT == DK_F32) {
    const float4 u = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(p) + e));
    v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
  } else if constexpr (VEC == 1) {
    v[0] = __bfloat162float(static_cast<const __nv_bfloat16*>(p)[e]);
  } else {
    uint32_t u[VEC / 2];
    const __nv_bfloat16* b = static_cast<const __nv_bfloat16*>(p) + e;
    if constexpr (VEC == 8) {
      const uint4 w = __ldg(reinterpret_cast<const uint4*>(b));
      u[0] = w.x; u[1] = w.y; u[2] = w.z; u[3] = w.w;
    } else {
      u[0] = __ldg(reinterpret_cast<const uint32_t*>(b));
    }
#pragma unroll
    for (int j = 0; j < VEC / 2; ++j) {
      v[2 * j] = __uint_as_float(u[j] << 16);
      v[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
    }
  }
}

// P: the backward call's p instead, from logits of the very same bits.  (A logit formed in another way differs from the
// one in lse by some 2^-22 of its terms, which is all that p has at the target where the model is sure: 4 x 256, 1000
// classes, dh off by 7e-5 of itself at p = 0.986 and by 2.8 times itself at 1 - 2e-6; now 1e-5 and 0.2, which is lse's
// rounding.)
template <int DT, int VEC, int R, int V, bool P>
__global__ void __launch_bounds__(kFewThreads) xent_few_rows_kernel(const FewArgs q) {
  chained_launch();
  extern __shared__ float hs[];                      // [R][dpad]
  __shared__ float2 joined[kFewThreads / 32][R];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int Q = VEC >= 4 ? 4 : VEC;              // elements of one access to shared memory
  constexpr int STEP = 32 * VEC;
  // Within a step of shared memory the lanes' first Q elements come first (then their next ones), so that a warp's
  // accesses are whole.  (What the rows above q.rows and the padding hold is never used.)
  const unsigned per = (unsigned)(q.d / VEC), all = per * (unsigned)q.rows;
  for (unsigned i0 = threadIdx.x; i0 < all; i0 += 4 * kFewThreads) {
    float v[4][VEC];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * kFewThreads < all) load_few<DT, VEC>(q.h, (size_t)(i0 + u * kFewThreads) * VEC, v[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const unsigned i = i0 + u * kFewThreads;
      if (i < all) {
        const unsigned r = i / per, c = i - r * per;           // vector c of the row: lane c % 32 of step c / 32
        float* to = hs + (size_t)r * q.dpad + c / 32 * STEP + c % 32 * Q;
#pragma unroll
        for (int j = 0; j < VEC; ++j) to[j / Q * 32 * Q + j % Q] = v[u][j];
      }
    }
  }
  __syncthreads();

  constexpr int kAtOnce = 4 / V;                     // steps whose loads are in flight together
  constexpr int N = V * R;                           // sums per step of a warp, a power of two
  constexpr int SHIFT = N == 1 ? 5 : N == 4 ? 3 : N == 8 ? 2 : N == 16 ? 1 : 0;
  static_assert(N << SHIFT == 32, "sums of a warp");
  const int mine = lane >> SHIFT, myv = mine / R, myr = mine % R;
  const long long t = myr < q.rows ? q.target[myr] : -1;
  float m = -INFINITY, s = 0.f;
  const bool keep = P && !left_out(t, q.r.vocab), writes = myr < q.rows && (lane & ((1 << SHIFT) - 1)) == 0;
  const float lse = keep ? q.r.lse[myr] : 0.f;
  float g = keep ? (q.r.dloss != nullptr ? q.r.dloss[myr] * q.r.scale : q.r.scale) : 0.f;
  if constexpr (P && DT == DK_F32) g *= pow2(scale_exp(*q.r.gmax));
  for (int v0 = (blockIdx.x * (kFewThreads / 32) + warp) * V; v0 < q.vocab; v0 += gridDim.x * (kFewThreads / 32) * V) {
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = 0.f;
    size_t row[V];
#pragma unroll
    for (int v = 0; v < V; ++v) row[v] = (size_t)min(v0 + v, q.vocab - 1) * q.d;      // (the last class again, not used)
#pragma unroll kAtOnce
    for (int k = lane * VEC; k < q.d; k += STEP) {
      float w[V][VEC];
#pragma unroll
      for (int v = 0; v < V; ++v) load_few<DT, VEC>(q.W, row[v] + k, w[v]);
      const float* at = hs + (k - lane * VEC) + lane * Q;
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int part = 0; part < VEC / Q; ++part) {
          const float* from = at + r * q.dpad + part * 32 * Q;
          float g[Q];
          if constexpr (Q == 4) {
            const float4 u = *reinterpret_cast<const float4*>(from);
            g[0] = u.x; g[1] = u.y; g[2] = u.z; g[3] = u.w;
          } else if constexpr (Q == 2) {
            const float2 u = *reinterpret_cast<const float2*>(from);
            g[0] = u.x; g[1] = u.y;
          } else {
            g[0] = *from;
          }
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < Q; ++j) x[v * R + r] = fmaf(w[v][part * Q + j], g[j], x[v * R + r]);
        }
      }
    }
    // sum i ends up in the lanes whose upper bits are i
#pragma unroll
    for (int o = 16, n = N / 2; o > 0; o >>= 1, n >>= 1) {
      if (n > 0) {
        const bool upper = lane & o;
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
          if (i < n) {
            const float keep = upper ? x[i + n] : x[i], give = upper ? x[i] : x[i + n];
            x[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
          }
      } else {
        x[0] += __shfl_xor_sync(0xffffffffu, x[0], o);
      }
    }
    const float l = x[0];
    if constexpr (P) {
      const int v = v0 + myv;
      if (v < q.vocab && writes) {
        const float p = keep ? p_value(l, lse, t - q.r.v0 == v, g) : 0.f;
        const size_t to = (size_t)myr * q.r.pitch + v;
        if constexpr (DT == DK_F32) {
          const unsigned int bits = __float_as_uint(p), most = magnitude(bits);
          static_cast<uint16_t*>(q.r.hi)[to] = (uint16_t)(bits >> 16);
          static_cast<uint16_t*>(q.r.lo)[to] = (uint16_t)(bits & 0xffffu);
          if (most > __ldcg(q.r.class_max + v)) atomicMax(q.r.class_max + v, most);
        } else {
          static_cast<__nv_bfloat16*>(q.r.hi)[to] = __float2bfloat16_rn(p);
        }
      }
    } else if (v0 + myv < q.vocab) {
      if (v0 + myv == t) q.tlogit[myr] = l;
      const float n = fmaxf(m, l);
      if (n != -INFINITY) s = s * __expf(m - n) + __expf(l - n);
      if (!(l == l)) s = l;
      m = n;
    }
  }
  if constexpr (!P) {
    // the V lanes of a row, then the warps, in order
#pragma unroll
    for (int o = R << SHIFT; o < 32; o <<= 1)
      join_pair(m, s, __shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o));
    if (myv == 0 && (lane & ((1 << SHIFT) - 1)) == 0) joined[warp][myr] = make_float2(m, s);
    __syncthreads();
    if ((int)threadIdx.x < q.rows) {
      float2 a = joined[0][threadIdx.x];
#pragma unroll
      for (int i = 1; i < kFewThreads / 32; ++i) join_pair(a.x, a.y, joined[i][threadIdx.x].x, joined[i][threadIdx.x].y);
      q.part[(size_t)blockIdx.x * q.rows + threadIdx.x] = a;
    }
  }
}

// one block per row of sliced logits
__global__ void __launch_bounds__(kRowThreads)
xent_slices_lse_kernel(const float* __restrict__ part, int ks, long long rows, int vocab, int pitch,
                       const int64_t* __restrict__ target, const float* __restrict__ inv_h,
                       const float* __restrict__ inv_w, float* loss, float* lse, int* status) {
  chained_launch();
  __shared__ float sm[kRowThreads / 32], ss[kRowThreads / 32], st;
  const long long row = blockIdx.x;
  const float f0 = inv_h != nullptr ? inv_h[row] : 1.f;
  const size_t slice = (size_t)rows * pitch;
  const long long t = target[row];
  float m = -INFINITY, s = 0.f;
  if (threadIdx.x == 0) st = 0.f;
  __syncthreads();
  for (int v = threadIdx.x; v < vocab; v += kRowThreads) {
    const float l = slice_sum(part, (size_t)row * pitch + v, slice, ks) * f0 * (inv_w != nullptr ? inv_w[v] : 1.f);
    if (v == t) st = l;
    const float n = fmaxf(m, l);
    if (n != -INFINITY) s = s * __expf(m - n) + __expf(l - n);
    if (!(l == l)) s = l;
    m = n;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float mo = __shfl_xor_sync(0xffffffffu, m, o), so = __shfl_xor_sync(0xffffffffu, s, o);
    const float n = fmaxf(m, mo);
    const float a = s == 0.f ? 0.f : s * __expf(m - n), b = so == 0.f ? 0.f : so * __expf(mo - n);
    s = a + b;
    m = n;
  }
  if ((threadIdx.x & 31) == 0) { sm[threadIdx.x >> 5] = m; ss[threadIdx.x >> 5] = s; }
  __syncthreads();
  if (threadIdx.x == 0) {
    float M = sm[0];
    for (int i = 1; i < kRowThreads / 32; ++i) M = fmaxf(M, sm[i]);
    float S = 0.f;
    for (int i = 0; i < kRowThreads / 32; ++i) S += ss[i] == 0.f ? 0.f : ss[i] * __expf(sm[i] - M);
    finish_row(t, vocab, M, S, st, loss + row, lse + row, status);
  }
}

// eight values' upper and lower halves
__device__ __forceinline__ void put_halves(const uint32_t (&w)[8], uint16_t* hi, uint16_t* lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    h[j] = __byte_perm(w[2 * j], w[2 * j + 1], 0x7632);
    l[j] = __byte_perm(w[2 * j], w[2 * j + 1], 0x5410);
  }
  *reinterpret_cast<uint4*>(hi) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4*>(lo) = make_uint4(l[0], l[1], l[2], l[3]);
}

template <bool F32>
__global__ void __launch_bounds__(256)
xent_slices_p_kernel(const float* __restrict__ part, int ks, long long rows, int n, int pitch, const RowArgs r,
                     const Undo undo) {
  chained_launch();
  float f0, f1;
  undo.get(f0, f1);
  const size_t slice = (size_t)rows * pitch;
  const int n8 = (int)(r.pitch / 8);
  const float gs = F32 ? pow2(scale_exp(*r.gmax)) : 1.f;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < rows * n8;
       i += (long long)gridDim.x * blockDim.x) {
    const long long row = i / n8;
    const int c = (int)(i - row * n8) * 8;
    const long long t = r.target[row];
    const bool keep = !left_out(t, r.vocab);
    const float lse = keep ? r.lse[row] : 0.f;
    const float g = keep ? (r.dloss != nullptr ? r.dloss[row] * r.scale : r.scale) * gs : 0.f;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      v[j] = keep && c + j < n
                 ? p_value(slice_sum(part, (size_t)row * pitch + c + j, slice, ks) * f0 * f1, lse, t - r.v0 == c + j, g)
                 : 0.f;
    if constexpr (F32) {
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = __float_as_uint(v[j]);
        const unsigned int m = magnitude(w[j]);
        if (c + j < n && m > __ldcg(r.class_max + c + j)) atomicMax(r.class_max + c + j, m);
      }
      put_halves(w, static_cast<uint16_t*>(r.hi) + row * r.pitch + c, static_cast<uint16_t*>(r.lo) + row * r.pitch + c);
    } else {
      *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(r.hi) + row * r.pitch + c) =
          make_uint4(g16::pack_bf16(v[0], v[1]), g16::pack_bf16(v[2], v[3]), g16::pack_bf16(v[4], v[5]),
                     g16::pack_bf16(v[6], v[7]));
    }
  }
}

// Between the product that forms p and those that read it (fp32): p's halves become, in place, two fp16 terms under the
// class's power of two; the rows of W of classes that have one of their own are laid out anew with its inverse.
struct ClassArgs {
  void* hi;
  void* lo;
  long long rows, pitch;       // of p; the pitch a multiple of 8
  const unsigned int* class_max;
  int n, d, dp;                // classes of the piece, features
  const float* W;              // the piece's rows, as given and as terms
  __half* w_hi;
  __half* w_lo;
  const unsigned int* wmax;
};
// A warp has 256 classes (512 bytes of either plane) and every eighth of the block's rows.  The classes written last, which
// are the likeliest to be in L2, come first.
constexpr int kTermRows = 4;             // of a warp, in flight together
__global__ void __launch_bounds__(256) xent_class_terms_kernel(const ClassArgs q) {
  chained_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = (int)(gridDim.y - 1 - blockIdx.y) * 256 + lane * 8;
  const long long per = (q.rows + gridDim.x - 1) / gridDim.x, end = min(q.rows, (blockIdx.x + 1) * per);
  if (c < q.pitch) {
    // (what lies behind the last class is zero in p)
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = c + j < q.n ? pow2(class_exp(__ldg(q.class_max + c + j))) : 0.f;
    for (long long r = blockIdx.x * per + warp; r < end; r += 8 * kTermRows) {
      uint4 a[kTermRows], b[kTermRows];
#pragma unroll
      for (int u = 0; u < kTermRows; ++u)
        if (r + 8 * u < end) {
          a[u] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(q.hi) + (r + 8 * u) * q.pitch + c);
          b[u] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(q.lo) + (r + 8 * u) * q.pitch + c);
        }
#pragma unroll
      for (int u = 0; u < kTermRows; ++u)
        if (r + 8 * u < end) {
          const uint32_t aw[4] = {a[u].x, a[u].y, a[u].z, a[u].w}, bw[4] = {b[u].x, b[u].y, b[u].z, b[u].w};
          float v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j)
            v[j] = __uint_as_float(__byte_perm(bw[j / 2], aw[j / 2], j & 1 ? 0x7632 : 0x5410)) * f[j];
          g16::store_planes<8>(static_cast<__half*>(q.hi) + (r + 8 * u) * q.pitch + c,
                               static_cast<__half*>(q.lo) + (r + 8 * u) * q.pitch + c, v, 8);
        }
    }
  }
  // a warp looks at the classes of its lanes, and lays out those that need it together
  const long long warps = (long long)gridDim.x * gridDim.y * 8;
  const long long first = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 8 + warp;
  for (long long r0 = first; r0 < q.n; r0 += 32 * warps) {
    const long long mine = r0 + lane * warps;
    const int e_mine = mine < q.n ? class_exp(__ldg(q.class_max + mine)) : 0;
    for (unsigned left = __ballot_sync(0xffffffffu, e_mine != 0); left != 0u; left &= left - 1u) {
      const int l = __ffs(left) - 1;
      const long long r = r0 + l * warps;
      const float f = pow2(-__shfl_sync(0xffffffffu, e_mine, l)), sw = pow2(scale_exp(*q.wmax));
      const float* src = q.W + r * q.d;
      for (int c8 = lane * 8; c8 < q.dp; c8 += 256) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c8 + j < q.d ? __ldg(src + c8 + j) * sw * f : 0.f;
        g16::store_planes<8>(q.w_hi + r * q.dp + c8, q.w_lo + r * q.dp + c8, v, 8);
      }
    }
  }
}

template <bool F32>
__global__ void __launch_bounds__(256)
xent_slices_grad_kernel(const float* __restrict__ part, int ks, long long rows, int n, int pitch,
                        const EpiGrad<F32> e) {
  chained_launch();
  float f0, f1;
  e.undo.get(f0, f1);
  const size_t slice = (size_t)rows * pitch;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < rows * n;
       i += (long long)gridDim.x * blockDim.x) {
    const long long row = i / n;
    const int c = (int)(i - row * n);
    float v = slice_sum(part, (size_t)row * pitch + c, slice, ks);
    v = F32 ? v * e.undo_class(row) * f0 * f1 : v * e.alpha;
    float* a = e.accum + row * e.pitch_acc + c;
    if (e.add) v += *a;
    if (e.out == nullptr) *a = v;
    else if constexpr (F32) static_cast<float*>(e.out)[row * e.pitch + c] = v;
    else static_cast<__nv_bfloat16*>(e.out)[row * e.pitch + c] = __float2bfloat16_rn(v);
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
constexpr int BN = 256;
// Room for p of one piece (both terms).  Wider pieces mean fewer readings and writings of dh's sums and fewer launches:
// 4096x4096x128000 bf16 15.2 ms with 128 MiB, 14.8 with 256, 14.7 with 512; 4000x768x32000 fp32 2.82, 2.63, 2.58 ms.
constexpr long long kPieceBytes = 256LL << 20;

size_t up(size_t v) { return (v + 1023) / 1024 * 1024; }

struct Plan {
  bool f32, copy_w, copy_h;    // fwd: operands are laid out anew (fp32 terms, or rows that do not start on 16 bytes)
  int dp, vp, pieces;
  size_t off_h, off_w, off_p, off_acc, off_part, off_slots, off_tl, off_inv, off_class, total;
};

// slices of a product: every (tile, slice) has at most one pair's tile of fp32 sums
constexpr size_t kPartBytes = (size_t)(kMaxSms / 2) * g16::TILE_M * BN * sizeof(float);

// Both sides of the rule, in us (rows x d, classes; here | tensor cores): fp32 1 x 4096, 1000 19.5 | 29.7; 3 x 1538, 6216
// 34 | 55; 8 x 1024, 50257 69 | 200; 1 x 2048, 128000 198 | 752; but 1 x 12288, 64 36 | 26: a warp walks its row alone.  h takes
// its room of shared memory in 1, 4 or 8 rows: 2 to 4 rows stop at 6144 features, 5 to 8 at 3072.
// bf16, where the tensor cores read W as it is: 1 x 2048, 128000 108 | 146, but 4 rows 144 | 124.  A lone class has
// probability one exactly: both directions have to see the same logit, so it takes the backward call's way.
bool takes_few_rows(const dk_xent& q) {
  if (q.vocab < 2 || q.d > 8192) return false;
  if (q.dtype == DK_BF16) return q.rows == 1;
  const size_t r = q.rows == 1 ? 1 : q.rows <= 4 ? 4 : kFewRows;
  return q.rows <= kFewRows && r * (((size_t)q.d + 127) / 128 * 128) * sizeof(float) <= kFewSmem;
}

// `forward`: the room of dk_linear_xent_fwd alone, whose plan it is (a row against 128000 classes of 2048 features, fp32:
// 6 KiB; both directions 1.07 GB)
Plan plan_xent(const dk_xent& q, bool forward) {
  Plan p;
  p.f32 = q.dtype == DK_F32;
  p.dp = (q.d + 7) / 8 * 8;
  const bool few = forward && takes_few_rows(q);
  p.copy_w = !few && (p.f32 || q.d % 8 != 0);
  p.copy_h = p.copy_w;
  const size_t es = p.f32 ? 4 : 2;             // bytes of one operand element, both terms
  const long long T = q.rows > 0 ? q.rows : 1;
  long long vp = kPieceBytes / (T * (long long)es) / BN * BN;
  if (vp < 2 * BN) vp = 2 * BN;
  if (vp >= q.vocab) vp = q.vocab;
  p.pieces = (int)((q.vocab + vp - 1) / vp);
  if (p.pieces > 1) {                           // even pieces
    vp = (q.vocab + p.pieces - 1) / p.pieces;
    vp = (vp + BN - 1) / BN * BN;
    p.pieces = (int)((q.vocab + vp - 1) / vp);
  }
  p.vp = (int)((vp + 7) / 8 * 8);
  size_t off = 0;
  auto room = [&off](bool needed, size_t bytes) {
    const size_t at = off;
    off += needed ? up(bytes) : 0;
    return at;
  };
  room(!forward, sizeof(Meta));
  p.off_h = room(!forward || p.copy_h, (size_t)T * p.dp * es);
  p.off_w = room(p.copy_w, (size_t)q.vocab * p.dp * es);
  p.off_p = room(!forward, (size_t)T * p.vp * es);
  p.off_acc = room(!forward && p.pieces > 1, (size_t)T * p.dp * 4);
  p.off_part = room(!few, kPartBytes);
  // (maximum, sum) per row and the columns one thread finishes: BN/2 in the large tiles; in the small ones, of which
  // there are at most kSmallCtas CTAs with SMALL rows each, two to a CTA; per row and CTA of the dot products
  size_t slots = ((size_t)q.vocab + BN / 2 - 1) / (BN / 2) * T;
  if (slots < (size_t)g16::kSmallCtas * 2 * g16::SMALL) slots = (size_t)g16::kSmallCtas * 2 * g16::SMALL;
  if (few) slots = (size_t)kFewCtas * T;
  p.off_slots = room(forward, slots * sizeof(float2));
  p.off_tl = room(forward, (size_t)T * sizeof(float));
  // (inverse powers of two of the rows; those of W in whole tiles)
  p.off_inv = room(forward && !few && p.f32, ((size_t)T + 4 + (size_t)q.vocab + 256) * sizeof(float));
  p.off_class = room(!forward && p.f32, ((size_t)q.vocab + 8) * sizeof(unsigned int));
  p.total = off;
  return p;
}

size_t workspace_of(const dk_xent& q, bool forward) {
  const size_t f = plan_xent(q, true).total, b = plan_xent(q, false).total;
  return forward || f > b ? f : b;
}

dk_status check_xent(const dk_xent* q) {
  if (!q) return DK_ERR_INVALID_ARG;
  if (q->dtype != DK_F32 && q->dtype != DK_BF16) return DK_ERR_INVALID_ARG;
  if (q->rows < 0 || q->d < 1 || q->vocab < 1) return DK_ERR_SHAPE;
  if (q->rows > (1LL << 24) || q->d > (1 << 20) || q->vocab > (1 << 24)) return DK_ERR_SHAPE;
  return DK_OK;
}

Params gemm_params(const g16::Tiling& t, long long M, long long N, bool f32) {
  Params p = {};
  p.MT = t.MT; p.NT = t.NT; p.nbatch = 1; p.sym = 0; p.tiles = t.tiles;
  p.KB = t.KB; p.ksplit = t.ksplit; p.kb_per_split = t.kb_per_split;
  p.M = (int)M; p.N = (int)N;
  p.bf16 = f32 ? 0 : 1;
  p.chunk = f32 ? 2 : 16;
  // what the tensor pipe loses per stage in sums of random sign (large tiles, small tiles; measured, see g16::Params)
  p.comp = f32 ? 3.6f / 16777216.f : 0.f;
  p.comp_small = f32 ? 1.2f / 16777216.f : 0.f;
  return p;
}

unsigned grid_of(long long items, int sms) {
  long long b = (items + 255) / 256;
  if (b > (long long)sms * 8) b = (long long)sms * 8;
  return b < 1 ? 1u : (unsigned)b;
}

struct Call {
  dk_ctx* ctx;
  const dk_xent* q;
  Plan pl;
  char* ws;
  cudaStream_t st;
  Operand h, w;
  Undo undo_hw;
  const float *inv_h, *inv_w;
  Meta* meta() const { return reinterpret_cast<Meta*>(ws); }
  unsigned int* class_max() const { return reinterpret_cast<unsigned int*>(ws + pl.off_class); }
  float* part() const { return reinterpret_cast<float*>(ws + pl.off_part); }
};

// Lays out what the products read.  Backward: h always, rows that are left out cleared, so that what they hold meets no
// product (bf16: a copy), and fp32 operands under one power of two each.
template <bool F32>
dk_status prepare(Call& c, const void* h, const void* W, const int64_t* target, const float* dloss, float scale,
                  bool backward) {
  const dk_xent& q = *c.q;
  const Plan& pl = c.pl;
  const bool copy_h = pl.copy_h || backward;
  __half* hh = reinterpret_cast<__half*>(c.ws + pl.off_h);
  __half* wh = reinterpret_cast<__half*>(c.ws + pl.off_w);
  const long long nh = q.rows * pl.dp, nw = (long long)q.vocab * pl.dp;
  const int sms = c.ctx->sm_count;
  c.undo_hw = Undo{nullptr, nullptr};
  c.inv_h = c.inv_w = nullptr;
  if (F32 && !backward) {
    float* inv_h = reinterpret_cast<float*>(c.ws + pl.off_inv);
    float* inv_w = inv_h + (q.rows + 3) / 4 * 4;
    const PrepRows a{static_cast<const float*>(h), hh, hh + nh, inv_h, target, q.rows};
    const PrepRows b{static_cast<const float*>(W), wh, wh + nw, inv_w, nullptr, q.vocab};
    // (a block per row keeps one reading of 2048 elements or more in flight: 256 + 1000 rows of 4096 in 14 us by warps)
    const bool wide = q.d >= 1024;
    DK_CUDA_CHECK(launch_chained(wide ? xent_prep_forward_kernel<true> : xent_prep_forward_kernel<false>,
                                 dim3(grid_of((q.rows + q.vocab) * (wide ? 256 : 32), sms)), 256, 0, c.st, a, b, q.d, pl.dp,
                                 q.vocab));
    c.inv_h = inv_h;
    c.inv_w = inv_w;
  } else if (copy_h || pl.copy_w) {
    Prep a = {}, b = {};
    if (copy_h) a = Prep{h, hh, hh + nh, target, q.rows};
    if (pl.copy_w) b = Prep{W, wh, wh + nw, nullptr, q.vocab};
    Meta* meta = c.meta();
    unsigned blocks = grid_of((nw + nh) / 4, sms);
    if (blocks > kMaxBlocks) blocks = kMaxBlocks;
    if (F32) {
      DK_CUDA_CHECK(launch_chained(xent_absmax_kernel, dim3(blocks), 256, 0, c.st, static_cast<const float*>(h),
                                   static_cast<const float*>(W), target, dloss, scale, q.rows, q.d, q.vocab, meta));
      c.undo_hw = Undo{&meta->hmax, &meta->wmax};
    }
    DK_CUDA_CHECK(launch_chained(xent_prep_kernel<F32>,
                                 dim3(grid_of(((copy_h ? nh : 0) + (pl.copy_w ? nw : 0)) / 8, sms)), 256, 0, c.st, a, b, q.d,
                                 pl.dp, q.vocab, meta, (int)blocks, c.class_max()));
  }
  c.h = Operand{copy_h ? (const void*)hh : h, hh + nh, q.rows, q.d, pl.dp, 0};
  c.w = Operand{pl.copy_w ? (const void*)wh : W, wh + nw, q.vocab, q.d, pl.dp, 0};
  return DK_OK;
}

template <int DT, int VEC, int R, int V, bool P>
dk_status few_rows(dk_ctx* ctx, FewArgs a, float* loss, float* lse, cudaStream_t st) {
  a.dpad = (a.d + 32 * VEC - 1) / (32 * VEC) * (32 * VEC);
  const size_t smem = (size_t)R * a.dpad * sizeof(float);
  auto kern = xent_few_rows_kernel<DT, VEC, R, V, P>;
  static SmemLimit limit;
  const dk_status r = allow_smem(limit, ctx->device, kern, (int)kFewSmem);
  if (r != DK_OK) return r;
  long long per_sm = (long long)(200 * 1024 / (smem + 2048));
  if (per_sm > 4) per_sm = 4;
  const int classes = kFewThreads / 32 * V;
  long long grid = ((long long)a.vocab + classes - 1) / classes;
  if (grid > per_sm * ctx->sm_count) grid = per_sm * ctx->sm_count;
  if (grid > kFewCtas) grid = kFewCtas;
  DK_CUDA_CHECK(launch_chained(kern, dim3((unsigned)grid), kFewThreads, smem, st, a));
  if (!P)
    DK_CUDA_CHECK(launch_chained(xent_join_kernel, dim3((unsigned)((a.rows * 32 + kRowThreads - 1) / kRowThreads)),
                                 kRowThreads, 0, st, a.part, a.tlogit, a.target, (long long)a.rows, (int)grid, a.vocab, loss,
                                 lse, device_status_word(ctx)));
  return cudaGetLastError() == cudaSuccess ? DK_OK : DK_ERR_CUDA;
}

template <int DT, int VEC, int R, bool P>
dk_status few_rows(dk_ctx* ctx, const FewArgs& a, float* loss, float* lse, cudaStream_t st) {
  // four classes at a time where each warp still has some; one where there would be idle SMs
  const bool four = (long long)a.vocab >= 4LL * 4 * (kFewThreads / 32) * ctx->sm_count;
  return four ? few_rows<DT, VEC, R, 4, P>(ctx, a, loss, lse, st) : few_rows<DT, VEC, R, 1, P>(ctx, a, loss, lse, st);
}

// (what either direction takes follows from the call's sizes alone, so that both form a row's logits alike)
template <int DT, int VEC, bool P>
dk_status few_rows(dk_ctx* ctx, const FewArgs& a, float* loss, float* lse, cudaStream_t st) {
  if (a.rows == 1) return few_rows<DT, VEC, 1, P>(ctx, a, loss, lse, st);
  if constexpr (DT == DK_F32) {
    if (a.rows <= 4) return few_rows<DT, VEC, 4, P>(ctx, a, loss, lse, st);
    return few_rows<DT, VEC, 8, P>(ctx, a, loss, lse, st);
  }
  return DK_ERR_UNSUPPORTED;
}

template <bool P>
dk_status few_rows(dk_ctx* ctx, bool f32, const FewArgs& a, float* loss, float* lse, cudaStream_t st) {
  if (f32)
    return a.d % 4 == 0 ? few_rows<DK_F32, 4, P>(ctx, a, loss, lse, st) : few_rows<DK_F32, 1, P>(ctx, a, loss, lse, st);
  return a.d % 8 == 0   ? few_rows<DK_BF16, 8, P>(ctx, a, loss, lse, st)
         : a.d % 2 == 0 ? few_rows<DK_BF16, 2, P>(ctx, a, loss, lse, st)
                        : few_rows<DK_BF16, 1, P>(ctx, a, loss, lse, st);
}

template <bool F32>
dk_status forward(Call& c, const int64_t* target, float* loss, float* lse) {
  constexpr int NP = F32 ? 3 : 1;
  const dk_xent& q = *c.q;
  const Plan& pl = c.pl;
  const g16::Tiling t = g16::plan(q.rows, q.vocab, q.d, 1, false, c.ctx->sm_count, NP);
  Params p = gemm_params(t, q.rows, q.vocab, F32);
  int* status = device_status_word(c.ctx);
  dk_status s;
  if (!t.cs && t.ksplit > 1) {
    const int pitch = (q.vocab + 3) / 4 * 4;
    s = g16::launch<NP, false, false, BN>(c.ctx, c.h, c.w, p, g16::EpiPartial{c.part(), pitch}, c.st);
    if (s != DK_OK) return s;
    DK_CUDA_CHECK(launch_chained(xent_slices_lse_kernel, dim3((unsigned)q.rows), kRowThreads, 0, c.st,
                                 c.part(), t.ksplit, q.rows, q.vocab, pitch, target, c.inv_h, c.inv_w, loss, lse, status));
  } else {
    float2* slots = reinterpret_cast<float2*>(c.ws + pl.off_slots);
    float* tl = reinterpret_cast<float*>(c.ws + pl.off_tl);
    s = g16::product<NP, false, false>(c.ctx, t, c.h, c.w, p, EpiLse{slots, tl, target, c.inv_h, c.inv_w}, c.st);
    if (s != DK_OK) return s;
    const int cols = t.cs ? g16::SMALL / 2 / t.cs : BN / 2;      // columns a thread of the product finishes
    const int nslots = (q.vocab + cols - 1) / cols;
    DK_CUDA_CHECK(launch_chained(xent_join_kernel, dim3((unsigned)((q.rows * 32 + kRowThreads - 1) / kRowThreads)), kRowThreads, 0, c.st,
                                 slots, tl, target, q.rows, nslots, q.vocab, loss, lse, status));
  }
  return cudaGetLastError() == cudaSuccess ? DK_OK : DK_ERR_CUDA;
}

template <bool F32>
dk_status backward(Call& c, const void* h, const void* W, const int64_t* target, const float* lse, const float* dloss, float scale,
                   void* dh, void* dW) {
  constexpr int NP = F32 ? 3 : 1;
  const dk_xent& q = *c.q;
  const Plan& pl = c.pl;
  const long long T = q.rows;
  const int sms = c.ctx->sm_count;
  const size_t es = F32 ? 4 : 2;
  __half* ph = reinterpret_cast<__half*>(c.ws + pl.off_p);
  float* accum = reinterpret_cast<float*>(c.ws + pl.off_acc);
  const Undo undo_pw{F32 ? &c.meta()->gmax : nullptr, F32 ? &c.meta()->wmax : nullptr};
  const Undo undo_ph{F32 ? &c.meta()->gmax : nullptr, F32 ? &c.meta()->hmax : nullptr};
  for (int i = 0; i < pl.pieces; ++i) {
    const int v0 = i * pl.vp, nv = q.vocab - v0 < pl.vp ? q.vocab - v0 : pl.vp;
    const long long pitch_p = (nv + 7) / 8 * 8;
    __half* pl_lo = ph + T * pitch_p;
    Operand w = c.w;
    w.hi = static_cast<const __half*>(c.w.hi) + (size_t)v0 * pl.dp;
    w.lo = static_cast<const __half*>(c.w.lo) + (size_t)v0 * pl.dp;
    w.rows = nv;
    const Operand pop{ph, pl_lo, T, nv, pitch_p, 0};
    const RowArgs r{target, lse, dloss, F32 ? scale : 1.f, q.vocab, v0, &c.meta()->gmax, c.class_max() + v0, ph, pl_lo, pitch_p};

    // p of the piece
    g16::Tiling t = g16::plan(T, nv, q.d, 1, false, sms, NP);
    Params p = gemm_params(t, T, nv, F32);
    dk_status s;
    if (takes_few_rows(q)) {
      const FewArgs a = {h, static_cast<const char*>(W) + (size_t)v0 * q.d * es, target, nullptr, nullptr, (int)T, q.d, 0, nv, r};
      s = few_rows<true>(c.ctx, F32, a, nullptr, nullptr, c.st);
      if (s != DK_OK) return s;
    } else if (!t.cs && t.ksplit > 1) {
      const int pitch = (nv + 3) / 4 * 4;
      s = g16::launch<NP, false, false, BN>(c.ctx, c.h, w, p, g16::EpiPartial{c.part(), pitch}, c.st);
      if (s != DK_OK) return s;
      count_launches(c.ctx, DK_KERNEL_OTHER, 1);
      DK_CUDA_CHECK(launch_chained(xent_slices_p_kernel<F32>, dim3(grid_of(T * pitch_p / 8, c.ctx->sm_count)), 256, 0, c.st,
                                 c.part(), t.ksplit, T, nv, pitch, r, c.undo_hw));
    } else {
      s = g16::product<NP, false, false>(c.ctx, t, c.h, w, p, EpiP<F32>{r, c.undo_hw}, c.st);
      if (s != DK_OK) return s;
    }

    if constexpr (F32) {
      const ClassArgs a{ph, pl_lo, T, pitch_p, r.class_max, nv, q.d, pl.dp, static_cast<const float*>(W) + (size_t)v0 * q.d,
                        static_cast<__half*>(const_cast<void*>(w.hi)), static_cast<__half*>(const_cast<void*>(w.lo)),
                        &c.meta()->wmax};
      const unsigned strips = (unsigned)((pitch_p + 255) / 256);
      // parts of the rows: 32 rows each, or as many parts as give every class a warp that lays its row of W out
      long long parts = (T + 31) / 32 > 32 ? (T + 31) / 32 : 32;
      if (parts > 8LL * sms / strips) parts = 8LL * sms / strips;
      if (parts < 1) parts = 1;
      DK_CUDA_CHECK(launch_chained(xent_class_terms_kernel, dim3((unsigned)parts, strips), 256, 0, c.st, a));
    }

    // dh += p.W
    const bool last = i + 1 == pl.pieces;
    EpiGrad<F32> e{last ? dh : nullptr, accum, q.d, pl.dp, i > 0, scale, undo_pw, nullptr};
    t = g16::plan(T, q.d, nv, 1, false, sms, NP);
    p = gemm_params(t, T, q.d, F32);
    if (!t.cs && t.ksplit > 1) {
      const int pitch = (q.d + 3) / 4 * 4;
      s = g16::launch<NP, false, true, BN>(c.ctx, pop, w, p, g16::EpiPartial{c.part(), pitch}, c.st);
      if (s != DK_OK) return s;
      count_launches(c.ctx, DK_KERNEL_OTHER, 1);
      DK_CUDA_CHECK(launch_chained(xent_slices_grad_kernel<F32>, dim3(grid_of(T * q.d, c.ctx->sm_count)), 256, 0, c.st,
                                 c.part(), t.ksplit, T, q.d, pitch, e));
    } else {
      s = g16::product<NP, false, true>(c.ctx, t, pop, w, p, e, c.st);
      if (s != DK_OK) return s;
    }

    // dW of the piece = p^T.h
    e = EpiGrad<F32>{static_cast<char*>(dW) + (size_t)v0 * q.d * es, nullptr, q.d, 0, 0, scale, undo_ph, F32 ? r.class_max : nullptr};
    t = g16::plan(nv, q.d, T, 1, false, sms, NP);
    p = gemm_params(t, nv, q.d, F32);
    if (!t.cs && t.ksplit > 1) {
      const int pitch = (q.d + 3) / 4 * 4;
      s = g16::launch<NP, true, true, BN>(c.ctx, pop, c.h, p, g16::EpiPartial{c.part(), pitch}, c.st);
      if (s != DK_OK) return s;
      count_launches(c.ctx, DK_KERNEL_OTHER, 1);
      DK_CUDA_CHECK(launch_chained(xent_slices_grad_kernel<F32>, dim3(grid_of((long long)nv * q.d, c.ctx->sm_count)), 256, 0, c.st,
                                 c.part(), t.ksplit, nv, q.d, pitch, e));
    } else {
      s = g16::product<NP, true, true>(c.ctx, t, pop, c.h, p, e, c.st);
      if (s != DK_OK) return s;
    }
    if (cudaGetLastError() != cudaSuccess) return DK_ERR_CUDA;
  }
  return DK_OK;
}

dk_status begin(dk_ctx* ctx, const dk_xent* q, bool forward, void* stream, Call* c) {
  c->ctx = ctx;
  c->q = q;
  c->pl = plan_xent(*q, forward);
  c->ws = static_cast<char*>(ctx->ws);
  c->st = static_cast<cudaStream_t>(stream);
  return ctx->ws && ctx->ws_bytes >= c->pl.total ? DK_OK : DK_ERR_WORKSPACE;
}

}  // namespace
}  // namespace dk

using namespace dk;

extern "C" {

dk_status dk_xent_workspace_bytes(const dk_xent* q, size_t* bytes) {
  if (!bytes) return DK_ERR_INVALID_ARG;
  dk_status s = check_xent(q);
  if (s != DK_OK) return s;
  *bytes = workspace_of(*q, false);
  return DK_OK;
}

dk_status dk_xent_fwd_workspace_bytes(const dk_xent* q, size_t* bytes) {
  if (!bytes) return DK_ERR_INVALID_ARG;
  dk_status s = check_xent(q);
  if (s != DK_OK) return s;
  *bytes = workspace_of(*q, true);
  return DK_OK;
}

dk_status dk_linear_xent_fwd(dk_ctx* ctx, const dk_xent* q, const void* h, const void* W, const int64_t* target,
                             float* loss, float* lse, void* stream) {
  dk_status s = check_xent(q);
  if (s != DK_OK) return s;
  if (!ctx) return DK_ERR_INVALID_ARG;
  if (q->rows == 0) return DK_OK;           // (tensors without elements may be NULL)
  if (!h || !W || !target || !loss || !lse) return DK_ERR_INVALID_ARG;
  if (!aligned_to(h, 16) || !aligned_to(W, 16) || !aligned_to(target, 16) || !aligned_to(loss, 16) ||
      !aligned_to(lse, 16))
    return DK_ERR_INVALID_ARG;
  Call c;
  s = begin(ctx, q, true, stream, &c);
  if (s != DK_OK) return s;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  const bool few = takes_few_rows(*q);
  ProfScope ps(ctx, DK_KERNEL_OTHER, 2 + (!few && c.pl.copy_w ? 1 : 0), c.st);
  if (few) {
    const FewArgs a = {h, W, target, reinterpret_cast<float2*>(c.ws + c.pl.off_slots),
                       reinterpret_cast<float*>(c.ws + c.pl.off_tl), (int)q->rows, q->d, 0, q->vocab, {}};
    return few_rows<false>(ctx, c.pl.f32, a, loss, lse, c.st);
  }
  if (c.pl.f32) {
    s = prepare<true>(c, h, W, target, nullptr, 1.f, false);
    return s == DK_OK ? forward<true>(c, target, loss, lse) : s;
  }
  s = prepare<false>(c, h, W, target, nullptr, 1.f, false);
  return s == DK_OK ? forward<false>(c, target, loss, lse) : s;
}

dk_status dk_linear_xent_bwd(dk_ctx* ctx, const dk_xent* q, const void* h, const void* W, const int64_t* target,
                             const float* lse, const float* dloss, float scale, void* dh, void* dW, void* stream) {
  dk_status s = check_xent(q);
  if (s != DK_OK) return s;
  if (!ctx || !dW) return DK_ERR_INVALID_ARG;
  if (q->rows > 0 && (!h || !W || !target || !lse || !dh)) return DK_ERR_INVALID_ARG;
  if (!aligned_to(h, 16) || !aligned_to(W, 16) || !aligned_to(target, 16) || !aligned_to(lse, 16) ||
      !aligned_to(dloss, 16) || !aligned_to(dh, 16) || !aligned_to(dW, 16))
    return DK_ERR_INVALID_ARG;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  if (q->rows == 0) {
    DK_CUDA_CHECK(cudaMemsetAsync(dW, 0, (size_t)q->vocab * q->d * (q->dtype == DK_F32 ? 4 : 2),
                                  static_cast<cudaStream_t>(stream)));
    return DK_OK;
  }
  Call c;
  s = begin(ctx, q, false, stream, &c);
  if (s != DK_OK) return s;
  // (slices of a product that are joined by a kernel of their own are counted where that is launched)
  ProfScope ps(ctx, DK_KERNEL_OTHER, c.pl.f32 ? 2 + 4 * c.pl.pieces : 1 + 3 * c.pl.pieces, c.st);
  if (c.pl.f32) {
    s = prepare<true>(c, h, W, target, dloss, scale, true);
    return s == DK_OK ? backward<true>(c, h, W, target, lse, dloss, scale, dh, dW) : s;
  }
  s = prepare<false>(c, h, W, target, dloss, scale, true);
  return s == DK_OK ? backward<false>(c, h, W, target, lse, dloss, scale, dh, dW) : s;
}

}  // extern "C"
