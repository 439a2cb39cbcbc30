// Activation checkpoints in 8 bits: a tensor to its 8-bit form (dk_ckpt8.cuh) and back.
//
// Bound by HBM.  A thread takes one vector of 16 bytes of the tensor (4 fp32 or 8 bf16 values) at a time, of which U are in
// flight; the 8 or 4 neighbouring lanes of a block of 32 values exchange their largest magnitude.  Rows whose length is no
// multiple of the vector are read by single elements.
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
  long long units;           // vectors of all padded rows
  unsigned long long recip;  // 2^64/per rounded up: i/per is its high product with i (exact for i < 2^50)
  int d, per;                // per: vectors of a padded row
  int dp;
};

template <int DT, int VEC, bool WHOLE>
__device__ __forceinline__ void load_unit(const void* x, long long row, int c, int d, float (&v)[VEC]) {
  if constexpr (WHOLE) {
    if (c < d) {
      Vec<DT, VEC>::load(x, row * d + c, v);
      return;
    }
  }
#pragma unroll
  for (int k = 0; k < VEC; ++k) {
    v[k] = 0.f;
    if (!WHOLE && c + k < d) {
      float t[1];
      Vec<DT, 1>::load(x, row * d + c + k, t);
      v[k] = t[0];
    }
  }
}

template <int DT, bool WHOLE, int U>
__global__ void __launch_bounds__(kThreads) ckpt8_store_kernel(const Args a) {
  constexpr int VEC = DT == DK_F32 ? 4 : 8;
  chained_launch();
  const long long i0 = (long long)blockIdx.x * (kThreads * U) + threadIdx.x;
  float v[U][VEC];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long i = i0 + u * kThreads;
    const long long row = __umul64hi((unsigned long long)i, a.recip);
    if (i < a.units) {
      load_unit<DT, VEC, WHOLE>(a.x, row, (int)(i - row * a.per) * VEC, a.d, v[u]);
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[u][k] = 0.f;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long i = i0 + u * kThreads;
    const ckpt8::Scale s = ckpt8::scale_of(ckpt8::block_most<VEC>(v[u]));
    if (i < a.units) {
      ckpt8::put_codes<VEC>(a.codes + i * VEC, v[u], s);
      if ((threadIdx.x & (ckpt8::kBlock / VEC - 1)) == 0) a.exps[i * VEC / ckpt8::kBlock] = (uint8_t)s.byte;
    }
  }
}

template <int DT, bool WHOLE, int U>
__global__ void __launch_bounds__(kThreads) ckpt8_load_kernel(const Args a) {
  constexpr int VEC = DT == DK_F32 ? 4 : 8;
  chained_launch();
  const long long i0 = (long long)blockIdx.x * (kThreads * U) + threadIdx.x;
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
    const long long row = __umul64hi((unsigned long long)i, a.recip);
    const int c = (int)(i - row * a.per) * VEC;
    float v[VEC];
    ckpt8::unpack<VEC>(r[u], v);
    if constexpr (WHOLE) {
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
}

dk_status check(const dk_ckpt8* q) {
  if (!q) return DK_ERR_INVALID_ARG;
  if (q->dtype != DK_F32 && q->dtype != DK_BF16) return DK_ERR_INVALID_ARG;
  if (q->rows < 0 || q->d < 1) return DK_ERR_SHAPE;
  if (q->d > (1 << 20) || (double)q->rows * ckpt8::padded(q->d) > 1e12) return DK_ERR_SHAPE;
  return DK_OK;
}

template <int DT, bool WHOLE, int U>
cudaError_t launch_one(const Args& a, bool store, cudaStream_t st) {
  const dim3 grid((unsigned)((a.units + kThreads * U - 1) / (kThreads * U)));
  return launch_chained(store ? ckpt8_store_kernel<DT, WHOLE, U> : ckpt8_load_kernel<DT, WHOLE, U>, grid, kThreads, 0, st, a);
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
  a.recip = ~0ull / (unsigned)a.per + 1;
  const bool whole = q.d % vec == 0;
  // four vectors a thread where that leaves every SM its threads, one for the sake of latency otherwise
  const bool many = a.units >= 4LL * 2048 * sms;
  cudaError_t e;
#define DK_CKPT8(DT)                                                                                              \
  e = whole ? (many ? launch_one<DT, true, 4>(a, store, st) : launch_one<DT, true, 1>(a, store, st))              \
            : (many ? launch_one<DT, false, 4>(a, store, st) : launch_one<DT, false, 1>(a, store, st))
  if (q.dtype == DK_F32) DK_CKPT8(DK_F32);
  else DK_CKPT8(DK_BF16);
#undef DK_CKPT8
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
