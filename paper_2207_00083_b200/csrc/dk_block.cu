// The norms before and after a residual block, fused with its gate and residual scale, forward and backward.
//
//   u^ = (u - mean_u)*rstd_u,  h' = keep*h + scale*gate*post*u^,  h^ = (h' - mean_h)*rstd_h,  n = h^*pre + shift
//   q = dn*pre,  D = dh' + rstd_h*(q - mean(q) - h^*mean(q*h^)),  dh = keep*D
//   s = scale*gate*post*D,  du = rstd_u*(s - mean(s) - u^*mean(s*u^))
//   E = scale*D*u^:  dgate = sum E*post over the gate's rows,  dpost = sum E*gate,  dpre = sum dn*h^,  dshift = sum dn
// (root mean square: the means that are subtracted are zero, and rstd = 1/sqrt(mean(x^2) + eps)).
//
// A row is a team's: 4 to 32 lanes, or a CTA; a thread has sixteen of its values in registers, so a row is read once.  A team
// takes consecutive rows; backward it keeps the sums over rows of its columns in registers, and the rows of one gate are
// never split unevenly, so a gate's sums are either one team's, written at once, or of a fixed number of teams, joined in
// order by block_sums_kernel.  Rows above 8192 values have kernels of their own.
#include "dk_ckpt8.cuh"
#include "dk_internal.h"
#include "dk_step.h"
#include "dk_vec.cuh"

namespace dk {
namespace {

constexpr int kMaxD = 16384;
constexpr int kHeld = 8192;            // longest rows that are held in registers
// Values of a thread, and threads of a CTA at most (they share out the registers).
template <int DT>
constexpr int kValues = DT == DK_F32 ? 8 : 16;
template <int DT>
constexpr int kFwdThreads = DT == DK_F32 ? 768 : 512;
template <int DT>
constexpr int kBwdThreads = DT == DK_F32 ? 576 : 512;
constexpr int kMostSmem = 227 * 1024 - 2048;
constexpr int kSmallTeams = 256;       // threads of a CTA whose teams are lanes of a warp

struct BlockArgs {
  const void* h;
  const void* u;
  const uint8_t *ch, *eh, *cu, *eu;      // h and u as checkpoints: codes and exponents (backward: read, forward: written)
  uint8_t *kh, *keh, *ku, *keu;
  const float *gate, *post, *pre, *shift;
  void *h_out, *n;
  float4* stats;
  const void *dh_out, *dn;
  void *dh, *du;
  float* dgate;
  float* part;             // [3][CTAs][d]: dpre, dshift, dpost
  float* part_e;           // [teams or CTAs][d]
  long long rows, per;     // per: rows of a gate
  long long chunk;         // rows of a team
  int split;               // teams that share a gate's rows (0: a team has whole gates)
  int join_e;              // E is joined over a CTA's teams
  int d, dp, tl, teams;    // tl: threads of a team; teams: of a CTA
  int stages, team_smem;   // rows of a team's ring, bytes of its shared memory
  int shifted;             // dshift is asked for
  int layer;
  float eps, keep, scale, inv_d;
};

// sums over a team; `sm` [2][32][N], in turns, so that one barrier per sum is enough
template <int N>
__device__ __forceinline__ void team_sum(float (&v)[N], int tl, float* sm, int& turn) {
  for (int o = min(tl, 32) >> 1; o > 0; o >>= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  }
  if (tl > 32) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float* b = sm + turn * 32 * N;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) b[warp * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane < (tl >> 5) ? b[lane * N + i] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
    turn ^= 1;
  }
}

template <int VEC>
__device__ __forceinline__ void load_param(const float* p, int c, float (&v)[VEC]) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int k = 0; k < VEC; k += 4) {
      const float4 t = __ldg(reinterpret_cast<const float4*>(p + c + k));
      v[k] = t.x; v[k + 1] = t.y; v[k + 2] = t.z; v[k + 3] = t.w;
    }
  } else if constexpr (VEC == 2) {
    const float2 t = __ldg(reinterpret_cast<const float2*>(p + c));
    v[0] = t.x; v[1] = t.y;
  } else {
    v[0] = __ldg(p + c);
  }
}
template <int VEC>
__device__ __forceinline__ void load_gate(const float* p, int c, float (&v)[VEC]) {
  if (p != nullptr) {
    load_param<VEC>(p, c, v);
  } else {
#pragma unroll
    for (int k = 0; k < VEC; ++k) v[k] = 1.f;
  }
}

// mean and 1/sqrt(variance + eps) of a row from its values v[NV][VEC], of which live(j) say which vectors exist
template <int NV, int VEC>
__device__ __forceinline__ float2 row_moments(const float (&v)[NV][VEC], const bool (&live)[NV], const BlockArgs& a,
                                              float* sm, int& turn) {
  float mean = 0.f;
  if (a.layer) {
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (live[j]) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) s[0] += v[j][k];
      }
    team_sum<1>(s, a.tl, sm, turn);
    mean = s[0] * a.inv_d;
  }
  float s[1] = {0.f};
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (live[j]) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float t = v[j][k] - mean;
        s[0] = fmaf(t, t, s[0]);
      }
    }
  team_sum<1>(s, a.tl, sm, turn);
  return make_float2(mean, 1.f / sqrtf(fmaf(s[0], a.inv_d, a.eps)));
}

template <int VEC>
__device__ __forceinline__ void keep_vector(uint8_t* codes, uint8_t* exps, const float (&v)[VEC], long long row, int c,
                                            const BlockArgs& a, bool valid) {
  const uint32_t b = ckpt8::exponent_byte(ckpt8::block_most<VEC>(v));
  if (valid && c < a.dp) {
    ckpt8::put_codes<VEC>(codes + row * a.dp + c, v, b);
    if (c % ckpt8::kBlock == 0) exps[row * (a.dp / ckpt8::kBlock) + c / ckpt8::kBlock] = (uint8_t)b;
  }
}

// Wide rows, a CTA each: sixteen values of a thread.
template <int DT, int VEC, int NV>
__global__ void __launch_bounds__(1024) block_fwd_wide_kernel(const BlockArgs a) {
  chained_launch();
  __shared__ float sm[2 * 32];
  int turn = 0;
  const int lane = threadIdx.x;
  const long long row = blockIdx.x;
  constexpr bool valid = true;
  float h[NV][VEC], u[NV][VEC];
  bool live[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * a.tl + lane) * VEC;
    live[j] = c < a.d;
#pragma unroll
    for (int k = 0; k < VEC; ++k) h[j][k] = u[j][k] = 0.f;
    if (live[j]) {
      Vec<DT, VEC>::load(a.h, row * a.d + c, h[j]);
      if (a.u != nullptr) Vec<DT, VEC>::load(a.u, row * a.d + c, u[j]);
    }
  }
  if (a.kh != nullptr) {
#pragma unroll
    for (int j = 0; j < NV; ++j) keep_vector<VEC>(a.kh, a.keh, h[j], row, (j * a.tl + lane) * VEC, a, valid);
  }
  float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
  if (a.u != nullptr) {
    if (a.ku != nullptr) {
#pragma unroll
      for (int j = 0; j < NV; ++j) keep_vector<VEC>(a.ku, a.keu, u[j], row, (j * a.tl + lane) * VEC, a, valid);
    }
    const float2 m = row_moments<NV, VEC>(u, live, a, sm, turn);
    st.x = m.x; st.y = m.y;
    const float* gate = a.gate != nullptr ? a.gate + row / a.per * a.d : nullptr;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (live[j]) {
        const int c = (j * a.tl + lane) * VEC;
        float post[VEC], g[VEC];
        load_param<VEC>(a.post, c, post);
        load_gate<VEC>(gate, c, g);
#pragma unroll
        for (int k = 0; k < VEC; ++k)
          h[j][k] = fmaf(a.keep, h[j][k], a.scale * (g[k] * ((u[j][k] - m.x) * m.y * post[k])));
        Vec<DT, VEC>::store(a.h_out, row * a.d + c, h[j]);
      }
  }
  if (a.n != nullptr) {
    const float2 m = row_moments<NV, VEC>(h, live, a, sm, turn);
    st.z = m.x; st.w = m.y;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (live[j]) {
        const int c = (j * a.tl + lane) * VEC;
        float pre[VEC];
        load_param<VEC>(a.pre, c, pre);
#pragma unroll
        for (int k = 0; k < VEC; ++k) h[j][k] = (h[j][k] - m.x) * m.y * pre[k];
        if (a.shift != nullptr) {
          float b[VEC];
          load_param<VEC>(a.shift, c, b);
#pragma unroll
          for (int k = 0; k < VEC; ++k) h[j][k] += b[k];
        }
        Vec<DT, VEC>::store(a.n, row * a.d + c, h[j]);
      }
  }
  if (a.stats != nullptr && lane == 0) a.stats[row] = st;
}

// One vector of h or u of the backward pass.
template <int DT, int VEC, bool KEPT>
__device__ __forceinline__ void load_kept(const void* x, const uint8_t* codes, const uint8_t* exps, long long row, int c,
                                          const BlockArgs& a, float (&v)[VEC]) {
  if constexpr (KEPT) {
    ckpt8::unpack<VEC>(ckpt8::get<VEC>(codes + row * a.dp + c, exps + row * (a.dp / ckpt8::kBlock) + c / ckpt8::kBlock), v);
  } else {
    Vec<DT, VEC>::load(x, row * a.d + c, v);
  }
}

// What the phases of the backward pass need of a vector: u^, h^, q = dn*pre, dn and the gradient dh'
template <int VEC>
struct Cell {
  float uh[VEC], hh[VEC], dn[VEC], dho[VEC];
};
template <int DT, int VEC, bool KEPT>
__device__ __forceinline__ void load_cell(Cell<VEC>& e, const BlockArgs& a, long long row, int c, const float* gate,
                                          const float4& st) {
  load_kept<DT, VEC, KEPT>(a.h, a.ch, a.eh, row, c, a, e.hh);
  if (a.dn != nullptr) Vec<DT, VEC>::load(a.dn, row * a.d + c, e.dn);
  if (a.dh_out != nullptr) Vec<DT, VEC>::load(a.dh_out, row * a.d + c, e.dho);
  if (a.post != nullptr) {
    load_kept<DT, VEC, KEPT>(a.u, a.cu, a.eu, row, c, a, e.uh);
    float post[VEC], g[VEC];
    load_param<VEC>(a.post, c, post);
    load_gate<VEC>(gate, c, g);
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      e.uh[k] = (e.uh[k] - st.x) * st.y;
      e.hh[k] = fmaf(a.keep, e.hh[k], a.scale * (g[k] * (e.uh[k] * post[k])));
    }
  }
#pragma unroll
  for (int k = 0; k < VEC; ++k) e.hh[k] = (e.hh[k] - st.z) * st.w;
}

// Wide rows, a CTA each: read again in each phase, sums over rows in shared memory ([3][d]: E, dpre, dshift).
template <int DT, int VEC, int NV, bool KEPT>
__global__ void __launch_bounds__(1024) block_bwd_wide_kernel(const BlockArgs a) {
  extern __shared__ float dyn[];
  __shared__ float sm[2 * 32 * 2];
  chained_launch();
  int turn = 0;
  const int lane = threadIdx.x;
  const long long team = blockIdx.x;
  long long r0, r1;
  if (a.split) {
    const long long seg = team / a.split;
    r0 = seg * a.per + team % a.split * a.chunk;
    r1 = min(min(r0 + a.chunk, (seg + 1) * a.per), a.rows);
  } else {
    r0 = team * a.chunk;
    r1 = min(r0 + a.chunk, a.rows);
  }
  float* const my_post = a.part + (2LL * gridDim.x + blockIdx.x) * a.d;      // this CTA's sums of dpost
  for (int j = 0; j < NV; ++j) {
    const int c = (j * a.tl + lane) * VEC;
    if (c < a.d) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        dyn[c + k] = dyn[a.d + c + k] = dyn[2 * a.d + c + k] = 0.f;
        if (a.post != nullptr) my_post[c + k] = 0.f;
      }
    }
  }
  // D of a vector whose cell and dn*pre are given
  auto gradient = [&](const Cell<VEC>& e, const float (&q)[VEC], const float4& st, float m0, float m1, float (&D)[VEC]) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      D[k] = a.dh_out != nullptr ? e.dho[k] : 0.f;
      if (a.dn != nullptr) D[k] = fmaf(st.w, q[k] - m0 - e.hh[k] * m1, D[k]);
    }
  };
  auto scaled = [&](const Cell<VEC>& e, int c, float (&q)[VEC]) {
    if (a.dn == nullptr) return;
    float pre[VEC];
    load_param<VEC>(a.pre, c, pre);
#pragma unroll
    for (int k = 0; k < VEC; ++k) q[k] = e.dn[k] * pre[k];
  };
  auto factors = [&](const float* gate, int c, float (&f)[VEC]) {
    float g[VEC];
    load_param<VEC>(a.post, c, f);
    load_gate<VEC>(gate, c, g);
#pragma unroll
    for (int k = 0; k < VEC; ++k) f[k] *= a.scale * g[k];
  };
  for (long long row = r0; row < r1; ++row) {
    const long long seg = row / a.per;
    const float* gate = a.gate != nullptr ? a.gate + seg * a.d : nullptr;
    const float4 st = __ldg(a.stats + row);
    Cell<VEC> e;
    float q[VEC], f[VEC], D[VEC], v[VEC];
    float m[2] = {0.f, 0.f};
    if (a.dn != nullptr) {
      for (int j = 0; j < NV; ++j) {
        const int c = (j * a.tl + lane) * VEC;
        if (c >= a.d) continue;
        load_cell<DT, VEC, KEPT>(e, a, row, c, gate, st);
        scaled(e, c, q);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          dyn[a.d + c + k] = fmaf(e.dn[k], e.hh[k], dyn[a.d + c + k]);
          dyn[2 * a.d + c + k] += e.dn[k];
          m[0] += q[k];
          m[1] = fmaf(q[k], e.hh[k], m[1]);
        }
      }
      team_sum<2>(m, a.tl, sm, turn);
    }
    const float m0 = a.layer ? m[0] * a.inv_d : 0.f, m1 = m[1] * a.inv_d;
    float t[2] = {0.f, 0.f};
    for (int j = 0; j < NV; ++j) {
      const int c = (j * a.tl + lane) * VEC;
      if (c >= a.d) continue;
      load_cell<DT, VEC, KEPT>(e, a, row, c, gate, st);
      scaled(e, c, q);
      gradient(e, q, st, m0, m1, D);
      if (a.post == nullptr) {
        Vec<DT, VEC>::store(a.dh, row * a.d + c, D);
        continue;
      }
      factors(gate, c, f);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        dyn[c + k] = fmaf(a.scale * D[k], e.uh[k], dyn[c + k]);
        const float s = D[k] * f[k];
        t[0] += s;
        t[1] = fmaf(s, e.uh[k], t[1]);
      }
    }
    if (a.post == nullptr) continue;
    team_sum<2>(t, a.tl, sm, turn);
    const float t0 = a.layer ? t[0] * a.inv_d : 0.f, t1 = t[1] * a.inv_d;
    const bool last = row + 1 == r1 || (row + 1) / a.per != seg;      // of a gate's rows
    for (int j = 0; j < NV; ++j) {
      const int c = (j * a.tl + lane) * VEC;
      if (c >= a.d) continue;
      load_cell<DT, VEC, KEPT>(e, a, row, c, gate, st);
      scaled(e, c, q);
      gradient(e, q, st, m0, m1, D);
      factors(gate, c, f);
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[k] = a.keep * D[k];
      Vec<DT, VEC>::store(a.dh, row * a.d + c, v);          // (dh may be dh_out: only here)
#pragma unroll
      for (int k = 0; k < VEC; ++k) v[k] = st.y * (D[k] * f[k] - t0 - e.uh[k] * t1);
      Vec<DT, VEC>::store(a.du, row * a.d + c, v);
      if (last) {
        float post[VEC], g[VEC];
        load_param<VEC>(a.post, c, post);
        load_gate<VEC>(gate, c, g);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float s = dyn[c + k];
          my_post[c + k] = fmaf(g[k], s, my_post[c + k]);
          if (a.gate != nullptr && a.split == 0) a.dgate[seg * a.d + c + k] = s * post[k];
          if (a.split == 0) dyn[c + k] = 0.f;
        }
      }
    }
  }
  // what the CTA has summed up over its rows
  const long long slab = (long long)gridDim.x * a.d;
  for (int j = 0; j < NV; ++j) {
    const int c = (j * a.tl + lane) * VEC;
    if (c >= a.d) continue;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const long long at = (long long)blockIdx.x * a.d + c + k;
      if (a.dn != nullptr) {
        a.part[at] = dyn[a.d + c + k];
        a.part[slab + at] = dyn[2 * a.d + c + k];
      }
      if (a.gate != nullptr && a.split != 0) a.part_e[at] = dyn[c + k];
    }
  }
}

// ---------------------------------------------------------------------------
// The same with rows on their way into shared memory while others are worked on: a team has a ring of kStages rows of each
// tensor, filled by asynchronous copies two rows ahead.  Rows of whole 16-byte vectors: a thread copies the vectors that it
// reads itself.  Others: copied in 16-byte pieces from the boundary before them on (the last piece no further than the
// tensor's end), and read by single values, so that every length streams alike.  The copies of the next row are waited for
// before a barrier of this row's sums, which hands them to the whole team; the copies issued at a row's start go where the
// row before lay, whose last reading is before that row's last barrier.
//
// What bounds it besides HBM is instructions: bf16 rows from checkpoints leave some 55 per value at the rate of HBM.  So a
// thread has sixteen values, over which a row's sums, its copies and its scalars are shared out (eight: 86 and 91 per
// value forward and backward, 261 and 272 us for 16384 x 4096; 512 threads a row), and works on pairs, two to an
// instruction.
// ---------------------------------------------------------------------------
constexpr int kMostWarps = 24;               // of a team

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// a row of a tensor of `rows` rows of `bytes` bytes, 16-byte aligned, by a whole team
__device__ __forceinline__ void copy_row(uint32_t dst, const void* base, long long row, int bytes, long long rows, int lane,
                                         int tl) {
  const long long at = row * bytes, from = at & ~15LL;
  const int n = ((int)(at & 15) + bytes + 15) >> 4;
  const char* src = static_cast<const char*>(base) + from;
  for (int i = lane; i < n; i += tl) {
    const long long left = rows * bytes - from - i * 16LL;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + i * 16), "l"(src + i * 16),
                 "r"(left >= 16 ? 16 : (int)left)
                 : "memory");
  }
}
__host__ __device__ inline int row_room(int bytes) { return (bytes + 15 + 15) / 16 * 16; }

// A team and a thread's place in it.  Its values: VEC at a time, 2 * P/VEC vectors tl*VEC apart; as pairs in that order.
struct Team {
  int lane, tl, warps;         // warps: of a team that is the CTA, else 0
  float* sm;                   // [2][2*kMostWarps], zero behind the team's warps
  int turn;
};
__device__ __forceinline__ void team_sync(const Team& t) {
  if (t.warps) __syncthreads(); else __syncwarp();
}
__device__ __forceinline__ float team_sum1(float x, Team& t) {
  if (t.tl < 32) {
    for (int o = t.tl >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (t.warps == 0) return x;
  float* s = t.sm + t.turn * 2 * kMostWarps;
  t.turn ^= 1;
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
  __syncthreads();
  F2 y = f2(0.f);
#pragma unroll
  for (int w = 0; w < kMostWarps; w += 4)
    if (w < t.warps) {
      const float4 v = *reinterpret_cast<const float4*>(s + w);
      y = y + (f2(v.x, v.y) + f2(v.z, v.w));
    }
  return sum(y);
}
__device__ __forceinline__ void team_sum2(float& a, float& b, Team& t) {
  if (t.tl < 32) {
    for (int o = t.tl >> 1; o > 0; o >>= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, o);
      b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    return;
  }
  const int lane = threadIdx.x & 31;
  const bool upper = lane & 16;      // the lower half of the warp goes on with a, the upper with b
  float x = (upper ? b : a) + __shfl_xor_sync(0xffffffffu, upper ? a : b, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (t.warps == 0) {
    const float y = __shfl_xor_sync(0xffffffffu, x, 16);
    a = upper ? y : x;
    b = upper ? x : y;
    return;
  }
  float* s = t.sm + t.turn * 2 * kMostWarps;
  t.turn ^= 1;
  if ((lane & 15) == 0) s[(threadIdx.x >> 5) * 2 + (lane >> 4)] = x;
  __syncthreads();
  F2 y = f2(0.f);
#pragma unroll
  for (int w = 0; w < kMostWarps; w += 2)
    if (w < t.warps) {
      const float4 v = *reinterpret_cast<const float4*>(s + 2 * w);
      y = y + (f2(v.x, v.y) + f2(v.z, v.w));
    }
  const float2 r = split(y);
  a = r.x;
  b = r.y;
}

template <int VEC>
__device__ __forceinline__ int column(int e, const Team& t) { return ((e / VEC) * t.tl + t.lane) * VEC + e % VEC; }

template <int DT, int VEC, int P>
__device__ __forceinline__ void take(const char* row, const Team& t, int d, F2 (&v)[P]) {
  float x[2 * P];
#pragma unroll
  for (int e = 0; e < 2 * P; e += VEC) {
    const int c = column<VEC>(e, t);
    float y[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) y[k] = 0.f;
    if (c < d) Vec<DT, VEC>::load(row, c, y);
#pragma unroll
    for (int k = 0; k < VEC; ++k) x[e + k] = y[k];
  }
#pragma unroll
  for (int i = 0; i < P; ++i) v[i] = f2(x[2 * i], x[2 * i + 1]);
}
// A row of a checkpoint: the codes as numbers (WHOLE: and each vector's step, else each value's).
template <int VEC, int P>
__device__ __forceinline__ void take_codes(const char* codes, const char* exps, const Team& t, int dp, F2 (&v)[P]) {
#pragma unroll
  for (int e = 0; e < 2 * P; e += (VEC > 1 ? VEC : 2)) {
    if constexpr (VEC > 1) {
      const int c = column<VEC>(e, t);
      ckpt8::Raw<VEC> r = {};
      if (c < dp)
        r = ckpt8::get<VEC>(reinterpret_cast<const uint8_t*>(codes) + c, reinterpret_cast<const uint8_t*>(exps) + c / ckpt8::kBlock);
      const F2 step = f2(ckpt8::step_of(r.b));
#pragma unroll
      for (int k = 0; k < VEC; k += 2)
        v[(e + k) / 2] = (f2(ckpt8::biased<VEC>(r, k), ckpt8::biased<VEC>(r, k + 1)) + f2(-ckpt8::kBias)) * step;
    } else {
      float x[2], s[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c = column<1>(e + k, t);
        ckpt8::Raw<1> r = {};
        if (c < dp)
          r = ckpt8::get<1>(reinterpret_cast<const uint8_t*>(codes) + c, reinterpret_cast<const uint8_t*>(exps) + c / ckpt8::kBlock);
        x[k] = ckpt8::biased<1>(r, 0);
        s[k] = ckpt8::step_of(r.b);
      }
      v[e / 2] = (f2(x[0], x[1]) + f2(-ckpt8::kBias)) * f2(s[0], s[1]);
    }
  }
}
template <int DT, int VEC, int P>
__device__ __forceinline__ void give(void* base, long long row, const Team& t, int d, const F2 (&v)[P]) {
  char* const to = static_cast<char*>(base) + row * d * (DT == DK_F32 ? 4 : 2);
#pragma unroll
  for (int e = 0; e < 2 * P; e += VEC) {
    const int c = column<VEC>(e, t);
    if (c >= d) continue;
    float y[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const float2 p = split(v[(e + k) / 2]);
      y[k] = (e + k) & 1 ? p.y : p.x;
    }
    Vec<DT, VEC>::store(to, c, y);
  }
}
// a parameter's values of this thread (0 behind the row; null: `otherwise`)
template <int VEC, int P>
__device__ __forceinline__ void take_param(const float* p, const Team& t, int d, float otherwise, F2 (&v)[P]) {
  float x[2 * P];
#pragma unroll
  for (int e = 0; e < 2 * P; e += VEC) {
    const int c = column<VEC>(e, t);
    float y[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) y[k] = c < d ? otherwise : 0.f;
    if (c < d && p != nullptr) load_param<VEC>(p, c, y);
#pragma unroll
    for (int k = 0; k < VEC; ++k) x[e + k] = y[k];
  }
#pragma unroll
  for (int i = 0; i < P; ++i) v[i] = f2(x[2 * i], x[2 * i + 1]);
}
// a thread's values to fp32 `to`, which only it reads again or which is a part of the sums over rows
template <int VEC, int P>
__device__ __forceinline__ void give_sums(float* to, const Team& t, int d, const F2 (&v)[P]) {
#pragma unroll
  for (int e = 0; e < 2 * P; e += VEC) {
    const int c = column<VEC>(e, t);
    if (c >= d) continue;
    if constexpr (VEC == 1) {
      const float2 y = split(v[e / 2]);
      to[c] = e & 1 ? y.y : y.x;
    } else if constexpr (VEC == 2) {
      *reinterpret_cast<float2*>(to + c) = split(v[e / 2]);
    } else {
#pragma unroll
      for (int k = 0; k < VEC; k += 4) {
        const float2 x = split(v[(e + k) / 2]), y = split(v[(e + k) / 2 + 1]);
        *reinterpret_cast<float4*>(to + c + k) = make_float4(x.x, x.y, y.x, y.y);
      }
    }
  }
}
// (from shared memory: what give_sums has put there)
template <int VEC, int P>
__device__ __forceinline__ void take_own(const float* p, const Team& t, int d, F2 (&v)[P]) {
#pragma unroll
  for (int e = 0; e < 2 * P; e += (VEC > 1 ? VEC : 2)) {
    const int c = column<VEC>(e, t);
    if constexpr (VEC == 2) {
      float2 x = make_float2(0.f, 0.f);
      if (c < d) x = *reinterpret_cast<const float2*>(p + c);
      v[e / 2] = f2(x.x, x.y);
    } else if constexpr (VEC > 2) {
#pragma unroll
      for (int k = 0; k < VEC; k += 4) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < d) x = *reinterpret_cast<const float4*>(p + c + k);
        v[(e + k) / 2] = f2(x.x, x.y);
        v[(e + k) / 2 + 1] = f2(x.z, x.w);
      }
    } else {
      const int c1 = column<1>(e + 1, t);
      v[e / 2] = f2(c < d ? p[c] : 0.f, c1 < d ? p[c1] : 0.f);
    }
  }
}
// gate*post*scale
template <int VEC, int P>
__device__ __forceinline__ void take_factors(const BlockArgs& a, long long seg, const Team& t, F2 (&gps)[P]) {
  F2 g[P];
  take_param<VEC>(a.gate != nullptr ? a.gate + seg * a.d : nullptr, t, a.d, 1.f, g);
  take_param<VEC>(a.post, t, a.d, 0.f, gps);
#pragma unroll
  for (int i = 0; i < P; ++i) gps[i] = gps[i] * g[i] * f2(a.scale);
}
// the next gate's row on its way into L2
__device__ __forceinline__ void fetch_gate(const BlockArgs& a, long long seg, const Team& t) {
  for (int c = t.lane * 32; c < a.d; c += t.tl * 32)
    asm volatile("prefetch.global.L2 [%0];" ::"l"(a.gate + seg * a.d + c));
}

// 1/sqrt(x): the instruction's 22 bits and one step of Newton's method
__device__ __forceinline__ float inverse_root(float x) {
  const float r = rsqrtf(x);
  return x > 1e-36f && x < 1e36f ? fmaf(r * 0.5f, fmaf(-x * r, r, 1.f), r) : 1.f / sqrtf(x);
}
// (x - mean) in place of x, and 1/sqrt(variance + eps)
template <int VEC, int P>
__device__ __forceinline__ float2 normalise(F2 (&v)[P], const BlockArgs& a, bool ragged, Team& t) {
  float mean = 0.f;
  if (a.layer) {
    F2 s = v[0];
#pragma unroll
    for (int i = 1; i < P; ++i) s = s + v[i];
    mean = team_sum1(sum(s), t) * a.inv_d;
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = v[i] + f2(-mean);
    if (ragged) {                  // (deviations of values that do not exist count as zero)
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float2 x = split(v[i]);
        v[i] = f2(column<VEC>(2 * i, t) < a.d ? x.x : 0.f, column<VEC>(2 * i + 1, t) < a.d ? x.y : 0.f);
      }
    }
  }
  F2 s = v[0] * v[0];
#pragma unroll
  for (int i = 1; i < P; ++i) s = fma(v[i], v[i], s);
  const float m2 = team_sum1(sum(s), t);
  return make_float2(mean, inverse_root(fmaf(m2, a.inv_d, a.eps)));
}

// Codes and exponents of a row.
template <int VEC, int P>
__device__ __forceinline__ void keep_row(uint8_t* codes, uint8_t* exps, long long row, const BlockArgs& a, bool valid,
                                         const Team& t, const F2 (&v)[P]) {
  uint8_t* const to = codes + row * a.dp;
  uint8_t* const to_e = exps + row * (a.dp / ckpt8::kBlock);
#pragma unroll
  for (int e = 0; e < 2 * P; e += VEC) {
    if (e > 0 && (e / VEC) * t.tl * VEC >= a.dp) continue;      // (nothing of the row there, whatever the lane)
    float x[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const float2 p = split(v[(e + k) / 2]);
      x[k] = (e + k) & 1 ? p.y : p.x;
    }
    const uint32_t b = ckpt8::exponent_byte(ckpt8::block_most<VEC>(x));
    const int c = column<VEC>(e, t);
    if (valid && c < a.dp) {
      ckpt8::put_codes<VEC>(to + c, x, b);
      if (c % ckpt8::kBlock == 0) to_e[c / ckpt8::kBlock] = (uint8_t)b;
    }
  }
}

// A tensor's row into a stage: WHOLE, by the threads that read it; else by the team.
template <int VEC, int BYTES, int N>
__device__ __forceinline__ void copy_own(uint32_t dst, const void* base, long long row, int n, const Team& t) {
  // N values of a thread, VEC of BYTES bytes together, n in the row
  const char* src = static_cast<const char*>(base) + row * n * (BYTES / VEC);
#pragma unroll
  for (int e = 0; e < N; e += VEC) {
    const int c = column<VEC>(e, t);
    if (c < n) copy_async<BYTES>(dst + c * (BYTES / VEC), src + c * (BYTES / VEC));
  }
}
template <int DT, int VEC>
__device__ __forceinline__ void copy_tensor(uint32_t dst, const void* base, long long row, const BlockArgs& a, const Team& t) {
  constexpr int ES = DT == DK_F32 ? 4 : 2;
  if constexpr (VEC * ES == 16) copy_own<VEC, 16, kValues<DT>>(dst, base, row, a.d, t);
  else copy_row(dst, base, row, a.d * ES, a.rows, t.lane, t.tl);
}
template <int DT, int VEC>
__device__ __forceinline__ void copy_codes(uint32_t dst, const uint8_t* base, long long row, const BlockArgs& a, const Team& t) {
  if constexpr (VEC >= 4) copy_own<VEC, VEC, kValues<DT>>(dst, base, row, a.dp, t);
  else copy_row(dst, base, row, a.dp, a.rows, t.lane, t.tl);
}

__device__ __forceinline__ Team make_team(const BlockArgs& a, float* sm) {
  Team t;
  t.lane = threadIdx.x % a.tl; t.tl = a.tl;
  t.warps = a.tl > 32 ? a.tl >> 5 : 0;
  t.sm = sm;
  t.turn = 0;
  for (int i = threadIdx.x; i < 4 * kMostWarps; i += blockDim.x) sm[i] = 0.f;
  return t;
}

template <int DT, int VEC>
__global__ void __launch_bounds__(kFwdThreads<DT>) block_fwd_rows_kernel(const BlockArgs a) {
  constexpr int kStages = 3;
  extern __shared__ __align__(16) char ring[];
  __shared__ __align__(16) float sm[4 * kMostWarps];
  constexpr int ES = DT == DK_F32 ? 4 : 2, kPairs = kValues<DT> / 2;
  Team t = make_team(a, sm);
  const int team_in = threadIdx.x / a.tl;
  const long long r0 = ((long long)blockIdx.x * a.teams + team_in) * a.chunk, r1 = min(a.rows, r0 + a.chunk);
  const int bytes = a.d * ES, room = row_room(bytes), stage = 2 * room;
  char* const mine = ring + (size_t)team_in * a.team_smem;
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  const bool branch = a.u != nullptr;
  chained_launch();
  auto issue = [&](long long row, int slot) {
    if (row < r1) {
      copy_tensor<DT, VEC>(mine_at + slot * stage, a.h, row, a, t);
      if (branch) copy_tensor<DT, VEC>(mine_at + slot * stage + room, a.u, row, a, t);
    }
    copies_done();
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) issue(r0 + s, s);
  F2 gps[kPairs], pre[kPairs];
  long long seg = branch && r0 < r1 ? r0 / a.per : 0, seg_end = (seg + 1) * a.per;
  if (branch) take_factors<VEC>(a, seg, t, gps);
  take_param<VEC>(a.pre, t, a.d, 0.f, pre);
  const bool ragged = column<VEC>(2 * kPairs - 1, t) >= a.d;
  wait_copies<kStages - 2>();
  team_sync(t);
  int slot = 0;
  for (long long row = r0; row < r0 + a.chunk; ++row) {
    const bool valid = row < r1;
    if (a.tl >= 32 && !valid) break;                 // (a team of whole warps has no other team's lanes in them)
    const char* at = mine + slot * stage;
    const int off = VEC * ES == 16 ? 0 : (int)((row * bytes) & 15), d = valid ? a.d : 0;
    issue(row + kStages - 1, slot == 0 ? kStages - 1 : slot - 1);
    F2 h[kPairs];
    take<DT, VEC>(at + off, t, d, h);
    if (a.kh != nullptr) keep_row<VEC>(a.kh, a.keh, row, a, valid, t, h);
    float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.n == nullptr) wait_copies<kStages - 2>();
    if (branch) {
      F2 u[kPairs];
      take<DT, VEC>(at + room + off, t, d, u);
      if (a.ku != nullptr) keep_row<VEC>(a.ku, a.keu, row, a, valid, t, u);
      if (valid && row == seg_end) {
        seg_end += a.per;
        take_factors<VEC>(a, ++seg, t, gps);
      }
      if (row + 1 == seg_end && row + 1 < r1) fetch_gate(a, seg + 1, t);
      const float2 m = normalise<VEC>(u, a, ragged, t);
      st.x = m.x; st.y = m.y;
#pragma unroll
      for (int k = 0; k < kPairs; ++k) h[k] = fma(f2(a.keep), h[k], gps[k] * (u[k] * f2(m.y)));
      if (valid) give<DT, VEC>(a.h_out, row, t, a.d, h);
    }
    if (a.n != nullptr) {
      wait_copies<kStages - 2>();
      const float2 m = normalise<VEC>(h, a, ragged, t);
      st.z = m.x; st.w = m.y;
#pragma unroll
      for (int k = 0; k < kPairs; ++k) h[k] = h[k] * f2(m.y) * pre[k];
      if (a.shift != nullptr) {
        F2 shift[kPairs];
        take_param<VEC>(a.shift, t, a.d, 0.f, shift);
#pragma unroll
        for (int k = 0; k < kPairs; ++k) h[k] = h[k] + shift[k];
      }
      if (valid) give<DT, VEC>(a.n, row, t, a.d, h);
    }
    if (a.stats != nullptr && t.lane == 0 && valid) a.stats[row] = st;
    if (t.warps == 0) __syncwarp();
    slot = slot + 1 == kStages ? 0 : slot + 1;
  }
  wait_copies<0>();
}

// Beside the ring a team has [d] fp32 of gate*post*scale, where the teams have several gates (split = 0) of dpost, and of
// dshift where that is asked for.
template <int DT, int VEC, bool KEPT>
__global__ void __launch_bounds__(kBwdThreads<DT>) block_bwd_rows_kernel(const BlockArgs a) {
  extern __shared__ __align__(16) char ring[];
  __shared__ __align__(16) float sm[4 * kMostWarps];
  constexpr int ES = DT == DK_F32 ? 4 : 2, kPairs = kValues<DT> / 2;
  Team t = make_team(a, sm);
  const int team_in = threadIdx.x / a.tl;
  const long long team = (long long)blockIdx.x * a.teams + team_in;
  const int bytes = a.d * ES, eb = a.dp / ckpt8::kBlock;
  const int room = row_room(bytes), room_k = row_room(KEPT ? a.dp : bytes), room_e = KEPT ? row_room(eb) : 0;
  // a stage: dh', dn, h, u and the exponents of both
  const int at_h = 2 * room, at_u = at_h + room_k, at_eh = at_u + room_k, at_eu = at_eh + room_e, stage = at_eu + room_e;
  const int own = row_room(a.d * 4), stages = a.stages;
  char* const mine = ring + (size_t)team_in * a.team_smem;
  float* const factors = reinterpret_cast<float*>(mine + stages * stage);
  float* const posts = factors + own / 4;
  float* const shifts = a.split == 0 ? posts + own / 4 : posts;
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  const bool branch = a.post != nullptr, norm = a.dn != nullptr;
  long long r0, r1, seg;
  if (a.split) {
    seg = team / a.split;
    r0 = seg * a.per + team % a.split * a.chunk;
    r1 = min(min(r0 + a.chunk, (seg + 1) * a.per), a.rows);
  } else {
    r0 = team * a.chunk;
    r1 = min(r0 + a.chunk, a.rows);
    seg = r0 / a.per;
  }
  if (r0 >= r1) seg = 0;
  long long seg_end = (seg + 1) * a.per;
  chained_launch();
  auto issue = [&](long long row, int slot) {
    if (row < r1) {
      const uint32_t to = mine_at + slot * stage;
      if (a.dh_out != nullptr) copy_tensor<DT, VEC>(to, a.dh_out, row, a, t);
      if (norm) copy_tensor<DT, VEC>(to + room, a.dn, row, a, t);
      if constexpr (KEPT) {
        copy_codes<DT, VEC>(to + at_h, a.ch, row, a, t);
        copy_row(to + at_eh, a.eh, row, eb, a.rows, t.lane, t.tl);
        if (branch) {
          copy_codes<DT, VEC>(to + at_u, a.cu, row, a, t);
          copy_row(to + at_eu, a.eu, row, eb, a.rows, t.lane, t.tl);
        }
      } else {
        copy_tensor<DT, VEC>(to + at_h, a.h, row, a, t);
        if (branch) copy_tensor<DT, VEC>(to + at_u, a.u, row, a, t);
      }
    }
    copies_done();
  };
  for (int s = 0; s < stages - 1; ++s) issue(r0 + s, s);
  const F2 zero = f2(0.f);
  F2 E[kPairs], spre[kPairs];
#pragma unroll
  for (int k = 0; k < kPairs; ++k) E[k] = spre[k] = zero;
  if (branch) {
    F2 gps[kPairs];
    take_factors<VEC>(a, seg, t, gps);
    give_sums<VEC>(factors, t, a.d, gps);
    if (a.split == 0) give_sums<VEC>(posts, t, a.d, E);
  }
  if (a.shifted) give_sums<VEC>(shifts, t, a.d, E);
  float4 next = r0 < r1 ? __ldg(a.stats + r0) : make_float4(0.f, 0.f, 0.f, 0.f);
  if (stages == 3) wait_copies<1>(); else wait_copies<0>();
  team_sync(t);
  int slot = 0;
  for (long long row = r0; row < r0 + a.chunk; ++row) {
    const bool valid = row < r1;
    if (a.tl >= 32 && !valid) break;
    const char* at = mine + slot * stage;
    const int off = VEC * ES == 16 ? 0 : (int)((row * bytes) & 15), off_e = (int)((row * eb) & 15);
    const int d = valid ? a.d : 0, dp = valid ? a.dp : 0;
    issue(row + stages - 1, slot == 0 ? stages - 1 : slot - 1);
    const float4 st = next;
    if (row + 1 < r1) next = __ldg(a.stats + row + 1);
    if (branch && valid) {
      if (row == seg_end) {
        F2 gps[kPairs];
        seg_end += a.per;
        take_factors<VEC>(a, ++seg, t, gps);
        give_sums<VEC>(factors, t, a.d, gps);
      }
      if (row + 1 == seg_end && row + 1 < r1) fetch_gate(a, seg + 1, t);
    }
    // u^ and h^; sums of q = dn*pre and q*h^
    F2 uh[kPairs], hh[kPairs];
    if constexpr (KEPT) take_codes<VEC>(at + at_h, at + at_eh + off_e, t, dp, hh);
    else take<DT, VEC>(at + at_h + off, t, d, hh);
    if (branch) {
      if constexpr (KEPT) take_codes<VEC>(at + at_u, at + at_eu + off_e, t, dp, uh);
      else take<DT, VEC>(at + at_u + off, t, d, uh);
      F2 gps[kPairs];
      take_own<VEC>(factors, t, a.d, gps);
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        uh[k] = (uh[k] + f2(-st.x)) * f2(st.y);
        hh[k] = fma(f2(a.keep), hh[k], gps[k] * uh[k]);
      }
    }
    float m0 = 0.f, m1 = 0.f;
    if (norm) {
      F2 dn[kPairs], pre[kPairs], s0 = zero, s1 = zero;
      take<DT, VEC>(at + room + off, t, d, dn);
      take_param<VEC>(a.pre, t, a.d, 0.f, pre);
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        hh[k] = (hh[k] + f2(-st.z)) * f2(st.w);
        spre[k] = fma(dn[k], hh[k], spre[k]);
        const F2 q = dn[k] * pre[k];
        s0 = s0 + q;
        s1 = fma(q, hh[k], s1);
      }
      m0 = sum(s0);
      m1 = sum(s1);
      if (a.shifted) {
        take_own<VEC>(shifts, t, a.d, pre);
#pragma unroll
        for (int k = 0; k < kPairs; ++k) pre[k] = pre[k] + dn[k];
        give_sums<VEC>(shifts, t, a.d, pre);
      }
    }
    team_sum2(m0, m1, t);
    m0 = a.layer ? m0 * a.inv_d : 0.f;
    m1 *= a.inv_d;
    // D in h^'s place
    if (norm) {
      F2 dn[kPairs], pre[kPairs];      // (again, from shared memory and L1: held, they would cost the registers of a row)
      take<DT, VEC>(at + room + off, t, d, dn);
      take_param<VEC>(a.pre, t, a.d, 0.f, pre);
#pragma unroll
      for (int k = 0; k < kPairs; ++k) hh[k] = f2(st.w) * fma(hh[k], f2(-m1), fma(dn[k], pre[k], f2(-m0)));
    } else {
#pragma unroll
      for (int k = 0; k < kPairs; ++k) hh[k] = zero;
    }
    if (a.dh_out != nullptr) {
      F2 dh[kPairs];
      take<DT, VEC>(at + off, t, d, dh);
#pragma unroll
      for (int k = 0; k < kPairs; ++k) hh[k] = hh[k] + dh[k];
    }
    float t0 = 0.f, t1 = 0.f;
    if (branch) {
      F2 v[kPairs], s0 = zero, s1 = zero;
#pragma unroll
      for (int k = 0; k < kPairs; ++k) v[k] = f2(a.keep) * hh[k];
      if (valid) give<DT, VEC>(a.dh, row, t, a.d, v);
      take_own<VEC>(factors, t, a.d, v);
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        E[k] = fma(hh[k], uh[k], E[k]);
        hh[k] = hh[k] * v[k];
        s0 = s0 + hh[k];
        s1 = fma(hh[k], uh[k], s1);
      }
      t0 = sum(s0);
      t1 = sum(s1);
    } else if (valid) {
      give<DT, VEC>(a.dh, row, t, a.d, hh);
    }
    if (stages == 3) wait_copies<1>(); else wait_copies<0>();
    team_sum2(t0, t1, t);
    if (branch) {
      t0 = a.layer ? t0 * a.inv_d : 0.f;
      t1 *= a.inv_d;
#pragma unroll
      for (int k = 0; k < kPairs; ++k) hh[k] = f2(st.y) * fma(uh[k], f2(-t1), hh[k] + f2(-t0));
      if (valid) {
        give<DT, VEC>(a.du, row, t, a.d, hh);
        if (a.split == 0 && (row + 1 == r1 || row + 1 == seg_end)) {      // the end of a gate's rows
          F2 g[kPairs], v[kPairs];
          take_param<VEC>(a.gate + seg * a.d, t, a.d, 1.f, g);
          take_own<VEC>(posts, t, a.d, v);
#pragma unroll
          for (int k = 0; k < kPairs; ++k) {
            E[k] = E[k] * f2(a.scale);
            v[k] = fma(g[k], E[k], v[k]);
          }
          give_sums<VEC>(posts, t, a.d, v);
          take_param<VEC>(a.post, t, a.d, 0.f, g);
#pragma unroll
          for (int k = 0; k < kPairs; ++k) {
            g[k] = g[k] * E[k];
            E[k] = zero;
          }
          give_sums<VEC>(a.dgate + seg * a.d, t, a.d, g);
        }
      }
    }
    if (t.warps == 0) __syncwarp();
    slot = slot + 1 == stages ? 0 : slot + 1;
  }
  wait_copies<0>();

  // what the team has summed up over its rows
  F2 v[kPairs];
  if (branch && a.split != 0) {
#pragma unroll
    for (int k = 0; k < kPairs; ++k) E[k] = E[k] * f2(a.scale);
    if (a.gate != nullptr && !a.join_e) give_sums<VEC>(a.part_e + team * a.d, t, a.d, E);
  }
  const long long slab = (long long)gridDim.x * a.d;
  float* const joined = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int which = 3; which >= 0; --which) {                 // E, dpost, dshift, dpre
    if (which == 0 ? !norm : which == 1 ? !a.shifted : !branch) continue;
    if (which == 3 && !a.join_e) continue;
    float* to = (which == 3 ? a.part_e : a.part + which * slab) + (long long)blockIdx.x * a.d;
    if (which == 2) {
      if (a.split == 0) {
        take_own<VEC>(posts, t, a.d, v);
      } else {
        take_param<VEC>(a.gate != nullptr ? a.gate + seg * a.d : nullptr, t, a.d, 1.f, v);
#pragma unroll
        for (int k = 0; k < kPairs; ++k) v[k] = v[k] * E[k];
      }
    }
    if (which == 1) take_own<VEC>(shifts, t, a.d, v);
    const F2(&of)[kPairs] = which == 0 ? spre : which == 3 ? E : v;
    if (a.teams > 1) {
      // (at the start of each team's ring, which has room for a row of fp32; what is its own lies behind the ring)
      __syncthreads();
      give_sums<VEC>(joined + team_in * (a.team_smem / 4), t, a.d, of);
      __syncthreads();
      for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
        float s = 0.f;
        for (int i = 0; i < a.teams; ++i) s += joined[i * (a.team_smem / 4) + c];
        to[c] = s;
      }
    } else {
      give_sums<VEC>(to, t, a.d, of);
    }
  }
}

// Joins the parts in order: 32 columns of one output per CTA, 16 rows of threads.
struct SumArgs {
  const float* part;
  const float* part_e;
  const float* post;
  float *dpre, *dshift, *dpost, *dgate;
  long long ctas, gates;
  int d, split;            // parts of a gate
};
__global__ void __launch_bounds__(512) block_sums_kernel(const SumArgs a) {
  chained_launch();
  __shared__ float sm[16][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + x;
  const long long what = blockIdx.y;
  const bool of_gate = what >= 3;
  float* out = what == 0 ? a.dpre : what == 1 ? a.dshift : what == 2 ? a.dpost : a.dgate + (what - 3) * a.d;
  const float* from = of_gate ? a.part_e + (what - 3) * a.split * a.d : a.part + what * a.ctas * a.d;
  const long long n = of_gate ? a.split : a.ctas;
  if (what < 3 && out == nullptr) return;
  float s = 0.f;
  if (c < a.d) {
#pragma unroll 8
    for (long long i = y; i < n; i += 16) s += __ldg(from + i * a.d + c);
  }
  sm[y][x] = s;
  __syncthreads();
  if (y == 0 && c < a.d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += sm[i][x];
    out[c] = of_gate ? s * a.post[c] : s;
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct BlockPlan {
  bool wide, whole;              // rows above the limit; rows of whole vectors
  int tl, teams, stages;
  int smem;                      // of a team, or of the wide backward kernel's sums
  long long chunk, nteams, ctas;
  // backward
  long long gates;
  int split, join_e;
  size_t part_e, total;
};

dk_status check_block(const dk_block* q) {
  if (!q) return DK_ERR_INVALID_ARG;
  if (q->kind != DK_BLOCK_RMS && q->kind != DK_BLOCK_LAYER) return DK_ERR_INVALID_ARG;
  if (q->dtype != DK_F32 && q->dtype != DK_BF16) return DK_ERR_INVALID_ARG;
  if (!(q->eps >= 0.f) || !(q->keep - q->keep == 0.f) || !(q->scale - q->scale == 0.f)) return DK_ERR_INVALID_ARG;
  if (q->rows < 0 || q->d < 1 || q->d > kMaxD || q->rows_per_gate < 1) return DK_ERR_SHAPE;
  if ((double)q->rows * q->d > 1e12 || q->rows > (1LL << 31) - 1) return DK_ERR_SHAPE;
  return DK_OK;
}

// What a call asks for beside its sizes: rows_per_gate counts, h and u come from checkpoints, dshift.
struct Asked {
  bool gated, held, shifted;
};
BlockPlan plan_block(const dk_block& q, bool backward, const Asked& asked) {
  BlockPlan p = {};
  const bool f32 = q.dtype == DK_F32;
  const int es = f32 ? 4 : 2, vec = 16 / es, dp = ckpt8::padded(q.d);
  const int values = f32 ? kValues<DK_F32> : kValues<DK_BF16>;
  const int most = backward ? (f32 ? kBwdThreads<DK_F32> : kBwdThreads<DK_BF16>) : f32 ? kFwdThreads<DK_F32> : kFwdThreads<DK_BF16>;
  const long long per = asked.gated && q.rows_per_gate < q.rows ? q.rows_per_gate : q.rows;
  p.gates = per > 0 ? (q.rows + per - 1) / per : 0;
  p.whole = q.d % vec == 0;
  int threads = (dp + values - 1) / values;
  if (threads <= 32) {
    // (a block of 32 values lies in one vector of neighbouring lanes)
    p.tl = ckpt8::kBlock / (p.whole ? vec : !f32 && q.d % 2 == 0 ? 2 : 1);
    while (p.tl < threads) p.tl *= 2;
    p.teams = kSmallTeams / p.tl;
  } else {
    p.tl = (threads + 31) / 32 * 32;
    p.teams = 1;
  }
  // A team's ring of three rows, or of two where that lets an SM hold more teams.
  const int row = row_room(q.d * es), room = 220 * 1024;
  long long ctas = 0;
  for (int stages = 3; stages >= 2; --stages) {
    int smem = stages * 2 * row;
    if (backward)
      smem = stages * (2 * row + 2 * (asked.held ? row_room(dp) + row_room(dp / ckpt8::kBlock) : row)) +
             (1 + (p.gates > 1) + asked.shifted) * row_room(q.d * 4);
    int teams = p.teams;
    while (teams > 1 && teams * smem > room / 2) teams /= 2;
    long long c = most / (p.tl * teams);
    if (c > room / ((long long)smem * teams + 1024)) c = room / ((long long)smem * teams + 1024);
    if (smem * teams > kMostSmem || c < 1) c = smem * teams <= kMostSmem ? 1 : 0;
    if (c * teams > ctas * (ctas ? p.teams : 1)) {
      ctas = c;
      p.smem = smem;
      p.stages = stages;
      if (teams < p.teams) p.teams = teams;
    }
    if (!backward) break;
  }
  p.wide = q.d > kHeld || p.tl > most || ctas == 0;
  if (p.wide) {
    p.tl = ((dp + 15) / 16 + 31) / 32 * 32;
    p.teams = 1;
    p.smem = backward ? 3 * q.d * (int)sizeof(float) : 0;
    ctas = 1;
  }
  // Rows of a team: as many as give every SM the CTAs that its registers and shared memory hold.
  const long long want = 148 * ctas * p.teams;
  long long chunk = (q.rows + want - 1) / want;
  if (chunk < 1) chunk = 1;
  if (!backward) {
    p.chunk = p.wide ? 1 : chunk;
    p.nteams = (q.rows + p.chunk - 1) / p.chunk;
    p.ctas = (p.nteams + p.teams - 1) / p.teams;
    return p;
  }
  if (per <= chunk && p.gates > 1) {
    p.split = 0;
    p.chunk = (chunk + per - 1) / per * per;
    p.nteams = (q.rows + p.chunk - 1) / p.chunk;
  } else {
    // (no more teams than are resident together: 152 instead of 144 CTAs of 148 take twice the time)
    long long k = p.gates > 0 ? want / p.gates : 1;
    if (k < 1) k = 1;
    if (k > per) k = per > 0 ? per : 1;
    p.chunk = (per + k - 1) / k;
    p.split = p.chunk > 0 ? (int)((per + p.chunk - 1) / p.chunk) : 1;
    p.nteams = p.gates * p.split;
  }
  p.ctas = (p.nteams + p.teams - 1) / p.teams;
  p.join_e = p.gates <= 1;
  if (p.join_e) p.split = (int)p.ctas;       // (of one gate: what is joined is a part per CTA)
  const size_t part = (size_t)3 * p.ctas * q.d * sizeof(float);
  p.part_e = (part + 255) / 256 * 256;
  const size_t e = p.split ? (size_t)(p.join_e ? p.ctas : p.ctas * p.teams) * q.d * sizeof(float) : 0;
  p.total = p.part_e + (e + 255) / 256 * 256;
  return p;
}

template <int DT, int VEC>
dk_status launch_fwd(const BlockArgs& a, const BlockPlan& p, int device, cudaStream_t st) {
  const dim3 grid((unsigned)p.ctas);
  const int threads = p.tl * p.teams;
  if (p.wide)
    return launch_chained(block_fwd_wide_kernel<DT, VEC, 16 / VEC>, grid, threads, 0, st, a) == cudaSuccess ? DK_OK : DK_ERR_CUDA;
  auto kern = block_fwd_rows_kernel<DT, VEC>;
  static SmemLimit limit;
  const dk_status s = allow_smem(limit, device, kern, kMostSmem);
  if (s != DK_OK) return s;
  return launch_chained(kern, grid, threads, (size_t)p.smem * p.teams, st, a) == cudaSuccess ? DK_OK : DK_ERR_CUDA;
}

template <int DT, int VEC, bool KEPT>
dk_status launch_bwd(const BlockArgs& a, const BlockPlan& p, int device, cudaStream_t st) {
  const dim3 grid((unsigned)p.ctas);
  const int threads = p.tl * p.teams;
  auto run = [&](auto kern, SmemLimit& limit) {
    const dk_status s = allow_smem(limit, device, kern, kMostSmem);
    if (s != DK_OK) return s;
    return launch_chained(kern, grid, threads, (size_t)p.smem * p.teams, st, a) == cudaSuccess ? DK_OK : DK_ERR_CUDA;
  };
  static SmemLimit limits[2];
  return p.wide ? run(block_bwd_wide_kernel<DT, VEC, 16 / VEC, KEPT>, limits[0]) : run(block_bwd_rows_kernel<DT, VEC, KEPT>, limits[1]);
}
template <int DT, int VEC>
dk_status launch_bwd(const BlockArgs& a, const BlockPlan& p, bool kept, int device, cudaStream_t st) {
  return kept ? launch_bwd<DT, VEC, true>(a, p, device, st) : launch_bwd<DT, VEC, false>(a, p, device, st);
}

dk_status backward(dk_ctx* ctx, const dk_block* q, bool kept, const void* dh_out, const void* dn, const void* h,
                   const void* u, const float* gate, const float* post, const float* pre, const float* stats, void* dh,
                   void* du, float* dgate, float* dpost, float* dpre, float* dshift, void* stream) {
  dk_status s = check_block(q);
  if (s != DK_OK) return s;
  // a branch: u, post, their gradients and, with a gate, its gradient; a norm after the sum: dn, pre, dpre
  const bool rows = q->rows > 0;
  if (!ctx || (post == nullptr) != (dpost == nullptr) || (gate == nullptr) != (dgate == nullptr) || (gate && !post))
    return DK_ERR_INVALID_ARG;
  if ((pre == nullptr) != (dpre == nullptr) || (dshift && !pre) || (!post && !pre)) return DK_ERR_INVALID_ARG;
  if (rows && ((u == nullptr) != (post == nullptr) || (du == nullptr) != (post == nullptr))) return DK_ERR_INVALID_ARG;
  if (rows && ((dn == nullptr) != (pre == nullptr) || (!dn && !dh_out) || !h || !stats || !dh)) return DK_ERR_INVALID_ARG;
  const void* all[] = {dh_out, dn, h, u, gate, post, pre, stats, dh, du, dgate, dpost, dpre, dshift};
  for (const void* t : all)
    if (!aligned_to(t, 16)) return DK_ERR_INVALID_ARG;
  if (rows && (dh == h || dh == dn || dh == u || (du && (du == dh || du == h || du == u || du == dn || du == dh_out))))
    return DK_ERR_INVALID_ARG;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!rows) {
    for (float* t : {dpost, dpre, dshift})
      if (t) DK_CUDA_CHECK(cudaMemsetAsync(t, 0, (size_t)q->d * sizeof(float), st));
    return DK_OK;
  }
  const BlockPlan p = plan_block(*q, true, Asked{gate != nullptr, kept, dshift != nullptr});
  if (!ctx->ws || ctx->ws_bytes < p.total) return DK_ERR_WORKSPACE;
  if (p.ctas >= (1LL << 31)) return DK_ERR_SHAPE;
  BlockArgs a = {};
  a.h = h; a.u = u;
  if (kept) {
    a.ch = static_cast<const uint8_t*>(h);
    a.eh = a.ch + ckpt8::code_bytes(q->rows, q->d);
    a.cu = static_cast<const uint8_t*>(u);
    if (u) a.eu = a.cu + ckpt8::code_bytes(q->rows, q->d);
  }
  a.gate = gate; a.post = post; a.pre = pre;
  a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
  a.dh_out = dh_out; a.dn = dn; a.dh = dh; a.du = du; a.dgate = dgate;
  a.part = static_cast<float*>(ctx->ws);
  a.part_e = reinterpret_cast<float*>(static_cast<char*>(ctx->ws) + p.part_e);
  a.rows = q->rows;
  a.per = gate != nullptr && q->rows_per_gate < q->rows ? q->rows_per_gate : q->rows;
  a.chunk = p.chunk;
  // (with one gate p.split counts the CTAs' parts; its teams' rows are consecutive either way)
  a.split = p.split ? (int)((a.per + p.chunk - 1) / p.chunk) : 0;
  a.join_e = p.join_e && gate != nullptr;
  a.shifted = dshift != nullptr;
  a.d = q->d; a.dp = ckpt8::padded(q->d); a.tl = p.tl; a.teams = p.teams; a.stages = p.stages; a.team_smem = p.smem;
  a.layer = q->kind == DK_BLOCK_LAYER;
  a.eps = q->eps; a.keep = q->keep; a.scale = q->scale; a.inv_d = 1.f / (float)q->d;
  ProfScope ps(ctx, DK_KERNEL_OTHER, 2, st);
  if (q->dtype == DK_F32)
    s = p.whole ? launch_bwd<DK_F32, 4>(a, p, kept, ctx->device, st) : launch_bwd<DK_F32, 1>(a, p, kept, ctx->device, st);
  else
    s = p.whole           ? launch_bwd<DK_BF16, 8>(a, p, kept, ctx->device, st)
        : q->d % 2 == 0 ? launch_bwd<DK_BF16, 2>(a, p, kept, ctx->device, st)
                        : launch_bwd<DK_BF16, 1>(a, p, kept, ctx->device, st);
  if (s != DK_OK) return s;
  const bool gates = gate != nullptr && p.split != 0;
  const SumArgs v{a.part, a.part_e, post, dpre, dshift, dpost, dgate, p.ctas, p.gates, q->d, p.split};
  const dim3 grid((unsigned)((q->d + 31) / 32), (unsigned)(3 + (gates ? p.gates : 0)));
  DK_CUDA_CHECK(launch_chained(block_sums_kernel, grid, 512, 0, st, v));
  return DK_OK;
}

}  // namespace
}  // namespace dk

using namespace dk;

extern "C" {

dk_status dk_block_workspace_bytes(const dk_block* q, size_t* bytes) {
  if (!bytes) return DK_ERR_INVALID_ARG;
  const dk_status s = check_block(q);
  if (s != DK_OK) return s;
  *bytes = 0;
  if (q->rows > 0)
    for (int way = 0; way < 8; ++way) {
      const size_t n = plan_block(*q, true, Asked{(way & 1) != 0, (way & 2) != 0, (way & 4) != 0}).total;
      if (n > *bytes) *bytes = n;
    }
  return DK_OK;
}

dk_status dk_block_norm_fwd(dk_ctx* ctx, const dk_block* q, const void* h, const void* u, const float* gate,
                            const float* post, const float* pre, const float* shift, void* h_out, void* n, float* stats,
                            void* ckpt_h, void* ckpt_u, void* stream) {
  const dk_status s = check_block(q);
  if (s != DK_OK) return s;
  if (!ctx) return DK_ERR_INVALID_ARG;
  if (q->rows == 0) return DK_OK;              // (tensors without elements may be NULL)
  // a branch: u, post and h_out; a norm after the sum: pre and n
  if (!h || (u == nullptr) != (post == nullptr) || (u == nullptr) != (h_out == nullptr)) return DK_ERR_INVALID_ARG;
  if ((gate && !u) || (ckpt_u && !u) || (n == nullptr) != (pre == nullptr) || (shift && !pre) || (!u && !n))
    return DK_ERR_INVALID_ARG;
  const void* all[] = {h, u, gate, post, pre, shift, h_out, n, stats, ckpt_h, ckpt_u};
  for (const void* t : all)
    if (!aligned_to(t, 16)) return DK_ERR_INVALID_ARG;
  if ((n && (n == h || n == u || n == h_out)) || (h_out && h_out == u) || (ckpt_h && ckpt_h == ckpt_u))
    return DK_ERR_INVALID_ARG;
  const BlockPlan p = plan_block(*q, false, Asked{});
  if (p.ctas >= (1LL << 31)) return DK_ERR_SHAPE;
  BlockArgs a = {};
  a.h = h; a.u = u; a.gate = gate; a.post = post; a.pre = pre; a.shift = shift;
  a.h_out = h_out; a.n = n; a.stats = reinterpret_cast<float4*>(stats);
  const long long codes = ckpt8::code_bytes(q->rows, q->d);
  a.kh = static_cast<uint8_t*>(ckpt_h);
  a.ku = static_cast<uint8_t*>(ckpt_u);
  if (a.kh) a.keh = a.kh + codes;
  if (a.ku) a.keu = a.ku + codes;
  a.rows = q->rows;
  a.per = gate != nullptr && q->rows_per_gate < q->rows ? q->rows_per_gate : q->rows;
  a.chunk = p.chunk;
  a.d = q->d; a.dp = ckpt8::padded(q->d); a.tl = p.tl; a.teams = p.teams; a.stages = p.stages; a.team_smem = p.smem;
  a.layer = q->kind == DK_BLOCK_LAYER;
  a.eps = q->eps; a.keep = q->keep; a.scale = q->scale; a.inv_d = 1.f / (float)q->d;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope ps(ctx, DK_KERNEL_OTHER, 1, st);
  if (q->dtype == DK_F32)
    return p.whole ? launch_fwd<DK_F32, 4>(a, p, ctx->device, st) : launch_fwd<DK_F32, 1>(a, p, ctx->device, st);
  return p.whole           ? launch_fwd<DK_BF16, 8>(a, p, ctx->device, st)
         : q->d % 2 == 0 ? launch_fwd<DK_BF16, 2>(a, p, ctx->device, st)
                         : launch_fwd<DK_BF16, 1>(a, p, ctx->device, st);
}

dk_status dk_block_norm_bwd(dk_ctx* ctx, const dk_block* q, const void* dh_out, const void* dn, const void* h, const void* u,
                            const float* gate, const float* post, const float* pre, const float* stats, void* dh, void* du,
                            float* dgate, float* dpost, float* dpre, float* dshift, void* stream) {
  return backward(ctx, q, false, dh_out, dn, h, u, gate, post, pre, stats, dh, du, dgate, dpost, dpre, dshift, stream);
}

dk_status dk_block_norm_bwd_ckpt8(dk_ctx* ctx, const dk_block* q, const void* dh_out, const void* dn, const void* ckpt_h,
                                  const void* ckpt_u, const float* gate, const float* post, const float* pre,
                                  const float* stats, void* dh, void* du, float* dgate, float* dpost, float* dpre,
                                  float* dshift, void* stream) {
  return backward(ctx, q, true, dh_out, dn, ckpt_h, ckpt_u, gate, post, pre, stats, dh, du, dgate, dpost, dpre, dshift,
                  stream);
}

}  // extern "C"
