// Activation checkpoints in 8 bits: a tensor to its 8-bit form (dk_ckpt8.cuh) and back.
//
// Bound by HBM.  A thread takes one vector of 16 bytes of the tensor (4 fp32 or 8 bf16 values) at a time, of which U are in
// flight; the 8 or 4 neighbouring lanes of a block of 32 values exchange their largest magnitude.  Rows whose length is no
// multiple of the vector start anywhere, and are read by single elements (as two aligned vectors, shifted: 40000 x 1693 bf16
// 64 us, by elements 59; 28286 x 1693 fp32 66 and 45).  bf16 rows are written in aligned vectors, their codes being shifted
// instead (40000 x 1693: 55 us, by elements 189), fp32 rows by elements (28286 x 1693: 57 us, in vectors 51; but 3000000 x
// 33, where every eighth vector has a row's end in it: 130 and 239).  64*224*224 x 64 bf16, stored and brought back: 184 us for 1.25 GB, 6.8
// TB/s, what a copy does; 196 x 512 fp32: 8.6 us for the two launches.
#include "dk_ckpt8.cuh"
#include "dk_internal.h"
#include "dk_step.h"
#include "dk_vec.cuh"

namespace dk {
namespace {

constexpr int kThreads = 256;

struct Args {
  const void* x;             // store: the tensor; load: unused
  void* y;                   // load: the tensor
  uint8_t* codes;
  uint8_t* exps;
  long long units;           // vectors of all padded rows; load, SHIFTED: of the tensor
  long long elements;
  unsigned long long recip;  // 2^64/per rounded up: i/per is its high product with i (exact for i*per < 2^64)
  int d, per;                // per: vectors of a padded row
  int dp;
};

// How rows lie: whole vectors and whole blocks (one flat array), whole vectors, or neither.  SHIFTED: neither, and bf16 to be
// written.
enum { FLAT = 0, WHOLE = 1, RAGGED = 2, SHIFTED = 3 };

// vector i of the padded rows, as stored (zero behind the row)
template <int DT, int VEC, int WAY>
__device__ __forceinline__ typename Vec<DT, VEC>::Raw load_unit(const Args& a, long long i) {
  using V = Vec<DT, VEC>;
  if constexpr (WAY == FLAT) return V::get(a.x, i * VEC);
  const long long row = __umul64hi((unsigned long long)i, a.recip);
  const int c = (int)(i - row * a.per) * VEC;
  if constexpr (WAY == WHOLE) {
    if (c < a.d) return V::get(a.x, row * a.d + c);
    return typename V::Raw{};
  } else {
    float v[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      float t[1] = {0.f};
      if (c + k < a.d) Vec<DT, 1>::load(a.x, row * a.d + c + k, t);
      v[k] = t[0];
    }
    return V::pack(v);
  }
}

template <int DT, int WAY, int U>
__global__ void __launch_bounds__(kThreads) ckpt8_store_kernel(const Args a) {
  constexpr int VEC = DT == DK_F32 ? 4 : 8;
  chained_launch();
  const long long i0 = (long long)blockIdx.x * (kThreads * U) + threadIdx.x;
  typename Vec<DT, VEC>::Raw raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    raw[u] = {};
    if (i0 + u * kThreads < a.units) raw[u] = load_unit<DT, VEC, WAY>(a, i0 + u * kThreads);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long i = i0 + u * kThreads;
    float v[VEC];
    Vec<DT, VEC>::unpack(raw[u], v);
    const ckpt8::Scale s = ckpt8::scale_of(ckpt8::block_most<VEC>(v));
    if (i < a.units) {
      ckpt8::put_codes<VEC>(a.codes + i * VEC, v, s);
      if ((threadIdx.x & (ckpt8::kBlock / VEC - 1)) == 0) a.exps[i * VEC / ckpt8::kBlock] = (uint8_t)s.byte;
    }
  }
}

template <int DT, int WAY, int U>
__global__ void __launch_bounds__(kThreads) ckpt8_load_kernel(const Args a) {
  constexpr int VEC = DT == DK_F32 ? 4 : 8;
  chained_launch();
  const long long i0 = (long long)blockIdx.x * (kThreads * U) + threadIdx.x;
  if constexpr (WAY != SHIFTED) {
    ckpt8::Raw<VEC> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * kThreads;
      if (i < a.units) r[u] = ckpt8::get<VEC>(a.codes + i * VEC, a.exps + i * VEC / ckpt8::kBlock);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * kThreads;
      if (i >= a.units) continue;
      float v[VEC];
      ckpt8::unpack<VEC>(r[u], v);
      if constexpr (WAY == FLAT) {
        Vec<DT, VEC>::store(a.y, i * VEC, v);
        continue;
      }
      const long long row = __umul64hi((unsigned long long)i, a.recip);
      const int c = (int)(i - row * a.per) * VEC;
      if constexpr (WAY == WHOLE) {
        if (c < a.d) Vec<DT, VEC>::store(a.y, row * a.d + c, v);
      } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k)
          if (c + k < a.d) {
            const float t[1] = {v[k]};
            Vec<DT, 1>::store(a.y, row * a.d + c + k, t);
          }
      }
    }
  } else {
    // A vector of the tensor: codes from c on, of one row; at a row's end and the tensor's, by single elements.
    constexpr int W = VEC / 4 + 1;
    uint32_t w[U][W], b0[U], b1[U];
    long long row[U];
    int c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * kThreads;
      row[u] = a.d == 1 ? i * VEC : __umul64hi((unsigned long long)i * VEC, a.recip);
      c[u] = (int)(i * VEC - row[u] * a.d);
      if (i >= a.units || c[u] + VEC > a.d) continue;
      const uint32_t* from = reinterpret_cast<const uint32_t*>(a.codes + row[u] * a.dp + (c[u] & ~3));
      const uint8_t* exps = a.exps + row[u] * (a.dp / ckpt8::kBlock);
#pragma unroll
      for (int k = 0; k < W; ++k) w[u][k] = k < W - 1 || (c[u] & 3) ? __ldg(from + k) : 0u;
      b0[u] = __ldg(exps + c[u] / ckpt8::kBlock);
      b1[u] = __ldg(exps + (c[u] + VEC - 1) / ckpt8::kBlock);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * kThreads;
      if (i >= a.units) continue;
      float v[VEC];
      if (c[u] + VEC <= a.d) {
        ckpt8::Raw<VEC> r;
#pragma unroll
        for (int k = 0; k < W - 1; ++k) r.w[k] = __funnelshift_r(w[u][k], w[u][k + 1], 8 * (c[u] & 3));
        const int left = ckpt8::kBlock - c[u] % ckpt8::kBlock;      // values of the first block
#pragma unroll
        for (int k = 0; k < VEC; ++k)
          v[k] = (ckpt8::biased<VEC>(r, k) - ckpt8::kBias) * ckpt8::step_of(k < left ? b0[u] : b1[u]);
        Vec<DT, VEC>::store(a.y, i * VEC, v);
      } else {
        long long at = row[u];
        for (int k = 0, col = c[u]; k < VEC && i * VEC + k < a.elements; ++k, ++col) {
          if (col == a.d) { ++at; col = 0; }
          float t[1];
          ckpt8::unpack<1>(ckpt8::get<1>(a.codes + at * a.dp + col, a.exps + at * (a.dp / ckpt8::kBlock) + col / ckpt8::kBlock), t);
          Vec<DT, 1>::store(a.y, i * VEC + k, t);
        }
      }
    }
  }
}

dk_status check(const dk_ckpt8* q) {
  if (!q) return DK_ERR_INVALID_ARG;
  if (q->dtype != DK_F32 && q->dtype != DK_BF16) return DK_ERR_INVALID_ARG;
  if (q->rows < 0 || q->d < 1) return DK_ERR_SHAPE;
  if (q->d > (1 << 20) || (double)q->rows * ckpt8::padded(q->d) > 1e12) return DK_ERR_SHAPE;
  return DK_OK;
}

template <int DT, int WAY>
cudaError_t launch_one(const Args& a, bool store, bool many, cudaStream_t st) {
  constexpr int LOAD = DT == DK_BF16 && WAY == RAGGED ? SHIFTED : WAY;
  const int u = many ? 4 : 1;
  const dim3 grid((unsigned)((a.units + kThreads * u - 1) / (kThreads * u)));
  auto kern = store ? (many ? ckpt8_store_kernel<DT, WAY, 4> : ckpt8_store_kernel<DT, WAY, 1>)
                    : (many ? ckpt8_load_kernel<DT, LOAD, 4> : ckpt8_load_kernel<DT, LOAD, 1>);
  return launch_chained(kern, grid, kThreads, 0, st, a);
}
template <int DT>
cudaError_t launch_way(const Args& a, bool store, bool many, cudaStream_t st) {
  if (a.d == a.dp) return launch_one<DT, FLAT>(a, store, many, st);
  if (a.d % (DT == DK_F32 ? 4 : 8) == 0) return launch_one<DT, WHOLE>(a, store, many, st);
  return launch_one<DT, RAGGED>(a, store, many, st);
}

}  // namespace

// x -> checkpoint (store) or checkpoint -> y, in one launch
dk_status launch_ckpt8(const dk_ckpt8& q, bool store, const void* x, void* y, void* ckpt, int sms, cudaStream_t st) {
  const int vec = q.dtype == DK_F32 ? 4 : 8;
  Args a = {};
  a.x = x; a.y = y;
  a.codes = static_cast<uint8_t*>(ckpt);
  a.exps = a.codes + ckpt8::code_bytes(q.rows, q.d);
  a.d = q.d;
  a.dp = ckpt8::padded(q.d);
  a.per = a.dp / vec;
  a.units = q.rows * a.per;
  a.elements = q.rows * q.d;
  int by = a.per;
  if (!store && q.dtype == DK_BF16 && q.d % vec != 0) {           // (SHIFTED)
    a.units = (a.elements + vec - 1) / vec;
    by = q.d;
  }
  a.recip = ~0ull / (unsigned)by + 1;          // (0 for 1)
  // four vectors a thread where that leaves every SM its threads, one for the sake of latency otherwise
  const bool many = a.units >= 4LL * 2048 * sms;
  const cudaError_t e = q.dtype == DK_F32 ? launch_way<DK_F32>(a, store, many, st) : launch_way<DK_BF16>(a, store, many, st);
  return e == cudaSuccess ? DK_OK : DK_ERR_CUDA;
}

}  // namespace dk

using namespace dk;

extern "C" {

dk_status dk_ckpt8_bytes(const dk_ckpt8* q, size_t* bytes) {
  if (!bytes) return DK_ERR_INVALID_ARG;
  const dk_status s = check(q);
  if (s != DK_OK) return s;
  *bytes = (size_t)ckpt8::total_bytes(q->rows, q->d);
  return DK_OK;
}

static dk_status run_ckpt8(dk_ctx* ctx, const dk_ckpt8* q, bool store, const void* x, void* y, void* ckpt, void* stream) {
  const dk_status s = check(q);
  if (s != DK_OK) return s;
  if (!ctx) return DK_ERR_INVALID_ARG;
  if (q->rows == 0) return DK_OK;              // (tensors without elements may be NULL)
  const void* t = store ? x : y;
  if (!t || !ckpt || !aligned_to(t, 16) || !aligned_to(ckpt, 16)) return DK_ERR_INVALID_ARG;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope ps(ctx, DK_KERNEL_OTHER, 1, st);
  return launch_ckpt8(*q, store, x, y, ckpt, ctx->sm_count, st);
}

dk_status dk_ckpt8_store(dk_ctx* ctx, const dk_ckpt8* q, const void* x, void* ckpt, void* stream) {
  return run_ckpt8(ctx, q, true, x, nullptr, ckpt, stream);
}

dk_status dk_ckpt8_load(dk_ctx* ctx, const dk_ckpt8* q, const void* ckpt, void* x, void* stream) {
  return run_ckpt8(ctx, q, false, nullptr, x, const_cast<void*>(ckpt), stream);
}

}  // extern "C"
