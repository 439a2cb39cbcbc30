// The norms before and after a residual block, fused with its gate and residual scale, forward and backward.
//
//   u^ = (u - mean_u)*rstd_u,  h' = keep*h + scale*gate*post*u^,  h^ = (h' - mean_h)*rstd_h,  n = h^*pre + shift
//   q = dn*pre,  D = dh' + rstd_h*(q - mean(q) - h^*mean(q*h^)),  dh = keep*D
//   s = scale*gate*post*D,  du = rstd_u*(s - mean(s) - u^*mean(s*u^))
//   E = scale*D*u^:  dgate = sum E*post over the gate's rows,  dpost = sum E*gate,  dpre = sum dn*h^,  dshift = sum dn
// (root mean square: the means that are subtracted are zero, and rstd = 1/sqrt(mean(x^2) + eps)).
//
// A row is a team's: 4 to 32 lanes, or a CTA; a thread has sixteen (fp32: eight) of its values in registers, so a row is read
// once.  A team takes consecutive rows; backward it keeps the sums over rows of its columns in registers, and the rows of one
// gate are never split unevenly, so a gate's sums are either one team's, written at once, or of a fixed number of teams,
// joined in order by block_sums_kernel.  Rows that a CTA's registers or shared memory do not hold have kernels of their own, which read a
// row three times backward: from 8193 bf16 and 6145 fp32 values forward, from 4609 fp32 backward, and bf16 backward from 8193, or
// where several gates a team, shift's gradient and rows of no whole vectors ask for more shared memory, from 6377 on at the
// earliest.
#include "dk_ckpt8.cuh"
#include "dk_internal.h"
#include "dk_step.h"
#include "dk_vec.cuh"

namespace dk {
namespace {

constexpr int kMaxD = 16384;
constexpr int kHeld = 8192;            // longest rows that are held in registers (bf16; fp32: 8 values a thread)
// Values of a thread, and threads of a CTA at most (they share out the registers).
template <int DT>
constexpr int kValues = DT == DK_BF16 ? 16 : 8;
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
  int rows, per, chunk;    // per: rows of a gate; chunk: of a team
  int split;               // teams that share a gate's rows (0: a team has whole gates)
  int join_e;              // E is joined over a CTA's teams
  int d, dp, tl, teams;    // tl: threads of a team; teams: of a CTA
  int stages, team_smem;   // rows of a team's ring, bytes of its shared memory
  unsigned spin_cap;       // polls of a wait
  int withhold;            // test hook: the first team arms its n-th row but copies nothing from there on (-1 = off)
  int* status;
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
  const ckpt8::Scale s = ckpt8::scale_of(ckpt8::block_most<VEC>(v));
  if (valid && c < a.dp) {
    ckpt8::put_codes<VEC>(codes + row * a.dp + c, v, s);
    if (c % ckpt8::kBlock == 0) exps[row * (a.dp / ckpt8::kBlock) + c / ckpt8::kBlock] = (uint8_t)s.byte;
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

// rstd as what brings deviations to normalised values.  mean*rstd beyond fp32's range is the mark of a row of one value (where
// values differ it is below 2^24*sqrt(d)), whose normalised values are zero.  They are made so, because the kernels with values
// in registers have zeros where a row has none, and (0 - mean)*rstd there is to be a number.
__device__ __forceinline__ float normaliser(float mean, float rstd) {
  const float inf = __int_as_float(0x7f800000);
  return fabsf(mean * rstd) == inf && rstd < inf ? 0.f : rstd;
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
    const float ru = normaliser(st.x, st.y);
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      e.uh[k] = (e.uh[k] - st.x) * ru;
      e.hh[k] = fmaf(a.keep, e.hh[k], a.scale * (g[k] * (e.uh[k] * post[k])));
    }
  }
  const float rh = normaliser(st.z, st.w);
#pragma unroll
  for (int k = 0; k < VEC; ++k) e.hh[k] = (e.hh[k] - st.z) * rh;
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
    r1 = min(min(r0 + a.chunk, (seg + 1) * a.per), (long long)a.rows);
  } else {
    r0 = team * a.chunk;
    r1 = min(r0 + a.chunk, (long long)a.rows);
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
// The same with rows on their way into shared memory while others are worked on: a team has a ring of two or three rows of
// each tensor, filled by asynchronous copies.  A team of whole warps has one lane issue bulk copies of whole rows, from the
// 16-byte boundary before a row to the one behind it (no further than the tensor's end: the last row's odd bytes are copied
// by hand), so every length streams alike and the other threads spend nothing on it; they wait on the stage's barrier.
// Teams of fewer lanes copy with cp.async, the vectors that they read themselves or 16-byte pieces.  The copies issued at a
// row's start go where the row before lay, whose last reading is before that row's last barrier.
//
// What bounds it besides HBM is instructions: bf16 rows from checkpoints leave some 55 per value at the rate of HBM and four a
// cycle; there are 37 forward and 54 backward, of which 15 warps an SM issue 2.0 and 2.3 a cycle (16384 x 4096: 134 and 181
// us).  So a thread has sixteen values, over which a row's sums, its copies and its scalars are shared out (eight: 86 and 91 per
// value forward and backward, 261 and 272 us for 16384 x 4096; 512 threads a row), and works on pairs, two to an
// instruction.
// ---------------------------------------------------------------------------
constexpr int kMostWarps = 24;               // of a team
constexpr int kMostStages = 3, kBulkTeams = kSmallTeams / 32, kMostSources = 6;

// What a stage is made of: tensors (rows of `bytes` bytes) and where their rows go.  In shared memory: a lane each.
struct Source {
  const void* base;
  int bytes, at;
};
struct Sources {
  Source of[kMostSources];
  int n;
  __device__ __forceinline__ void add(const void* base, int bytes, int at) {
    if (base != nullptr) of[n++] = Source{base, bytes, at};
  }
};

__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

__host__ __device__ inline int row_room(int bytes) { return (bytes + 15) / 16 * 16; }
// A row of a tensor in a stage; RAGGED: its vectors are read as two of a row that starts anywhere, and rows on their way out
// have 16 bytes before them.
__host__ __device__ inline int stage_room(int bytes, bool ragged) { return row_room(bytes) + (ragged ? 48 : 0); }

// 1/sqrt(x): the instruction's 22 bits and one step of Newton's method
__device__ __forceinline__ float inverse_root(float x) {
  const float r = rsqrtf(x);
  return x > 1e-36f && x < 1e36f ? fmaf(r * 0.5f, fmaf(-x * r, r, 1.f), r) : 1.f / sqrtf(x);
}

// A team and a thread's place in it.  Its N values: NV vectors of VEC, tl*VEC apart; as P pairs in that order.
// How rows lie.  FULL: rows of multiples of 32*N values; every thread of every team has all of its values, and teams are
// whole warps.  WHOLE: rows of whole 16-byte vectors.  Others start anywhere (`off` bytes behind a 16-byte boundary, the same
// for the whole row).  RAGGED, bf16: a vector is read as two of the stage's and shifted, and written to shared memory first,
// from where the team stores the row in whole aligned vectors (and its two ends by single values).  PAIRS and SINGLES, fp32:
// two values to an access where rows have an even number, else one.  Both sides: 16384 x 1001 bf16 takes 66 us forward and
// 115 backward as RAGGED, 130 and 143 as SINGLES; 4095 x 2050 fp32 62 and 82, but 47 and 60 as PAIRS (a shift serves four
// values there, not eight).
enum { FULL = 0, WHOLE = 1, RAGGED = 2, PAIRS = 3, SINGLES = 4 };
template <int DT, int WAY>
struct Team {
  static constexpr int ES = DT == DK_F32 ? 4 : 2, VEC = WAY == PAIRS ? 2 : WAY == SINGLES ? 1 : 16 / ES;
  static constexpr int N = kValues<DT>, NV = N / VEC, P = N / 2;
  static constexpr bool NARROW = WAY >= PAIRS;
  using Pairs = F2[P];
  int lane, tl, warps;         // warps: of a team that is the CTA, else 0
  int c0, cs;                  // first column, and from one vector to the next
  int d;
  bool lives[NV];              // vectors of which a value exists
  bool ragged;                 // not all of them
  float* sm;                   // [2][2*kMostWarps], zero behind the team's warps
  int turn;
  // bulk copies (whole warps)
  bool bulk;
  uint64_t* full;              // barriers of the ring's stages
  volatile int* abort_flag;

  __device__ __forceinline__ Team(const BlockArgs& a, float* shared, uint64_t* bars, volatile int* flag, int sources) {
    lane = threadIdx.x % a.tl; tl = a.tl;
    warps = a.tl > 32 ? a.tl >> 5 : 0;
    c0 = lane * VEC; cs = tl * VEC; d = a.d;
#pragma unroll
    for (int j = 0; j < NV; ++j) lives[j] = column(j) < a.d;
    ragged = WAY == RAGGED ? column(NV - 1) + VEC > a.d : !live(NV - 1);
    sm = shared;
    turn = 0;
    for (int i = threadIdx.x; i < 4 * kMostWarps; i += blockDim.x) sm[i] = 0.f;
    bulk = WAY == FULL || tl >= 32;
    full = bars + (bulk ? threadIdx.x / tl * kMostStages : 0);
    abort_flag = flag;
    if (threadIdx.x == 0) *flag = 0;
    if (bulk && lane == 0) {
      for (int i = 0; i < kMostStages; ++i)
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_at(full + i)), "r"(sources) : "memory");
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
  }
  // Waits for a stage's copies.  A wait that runs out raises the CTA's flag, after which none waits; what is then computed is
  // not the result, and the status says so.
  __device__ __forceinline__ void wait_row(int slot, uint32_t phase, const BlockArgs& a) const {
    if (!bulk) return;
    const uint32_t bar = shared_at(full + slot);
    for (unsigned i = 0; i < a.spin_cap; ++i) {
      uint32_t ok;
      asm volatile(
          "{\n\t.reg .pred p;\n\t"
          "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(ok)
          : "r"(bar), "r"(phase)
          : "memory");
      if (ok || *abort_flag) return;
    }
    *abort_flag = 1;
  }
  // One lane: its tensor's row into a stage at `to`.
  __device__ __forceinline__ void bulk_row(uint32_t to, const Source& src, int row, int rows, int slot) const {
    const long long at = (long long)row * src.bytes, from = at & ~15LL, left = (long long)rows * src.bytes - from;
    const int end = (int)(at & 15) + src.bytes, size = (int)min((long long)(end + 15 & ~15), left & ~15LL);
    const uint32_t dst = to + src.at, bar = shared_at(full + slot);
    const char* p = static_cast<const char*>(src.base) + from;
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(size) : "memory");
    if (size > 0)
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(p),
                   "r"(size), "r"(bar)
                   : "memory");
    for (int i = size; i < end; ++i)      // (handed to the team by a barrier before the row is read)
      asm volatile("st.shared.u8 [%0], %1;" ::"r"(dst + i), "r"((uint32_t) * reinterpret_cast<const uint8_t*>(p + i)) : "memory");
  }
  // The team's first lanes, one for each tensor.
  __device__ __forceinline__ void issue_bulk(uint32_t to, const Sources& from, int row, int r0, int r1, int slot,
                                             const BlockArgs& a) const {
    if (lane < from.n && row < r1 && issues(row - r0, slot, a)) bulk_row(to, from.of[lane], row, a.rows, slot);
  }
  // Whether a team's i-th row is copied: not once a wait has run out; nor, under the test hook, from the n-th on, which is
  // armed for bytes that nothing brings.
  __device__ __forceinline__ bool issues(int i, int slot, const BlockArgs& a) const {
    if (*abort_flag) return false;
    if (a.withhold < 0 || blockIdx.x > 0 || i < a.withhold) return true;
    if (i == a.withhold)
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], 16;" ::"r"(shared_at(full + slot)) : "memory");
    return false;
  }
  // at the kernel's end: after a wait that ran out, time for copies in flight to land
  __device__ __forceinline__ void leave(const BlockArgs& a) const {
    if (!bulk || !*abort_flag) return;
    if (lane == 0 && a.status != nullptr) atomicExch(a.status, (int)DK_ERR_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(16384);
  }
  __device__ __forceinline__ int column(int j) const { return c0 + j * cs; }
  __device__ __forceinline__ bool live(int j) const { return WAY == FULL || lives[j]; }
  __device__ __forceinline__ bool live(int j, int k) const { return WAY == RAGGED ? column(j) + k < d : live(j); }
  __device__ __forceinline__ void sync() const {
    if (warps) __syncthreads(); else __syncwarp();
  }
  // (behind a sum, which is a barrier only for teams of several warps)
  __device__ __forceinline__ void after_sum() const {
    if (!warps) __syncwarp();
  }

  __device__ __forceinline__ float sum1(float x) {
    if (WAY != FULL && tl < 32) {
      for (int o = tl >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      return x;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (warps == 0) return x;
    float* s = sm + turn * 2 * kMostWarps;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    F2 y = f2(0.f);
    for (int w = 0; w < warps; w += 8) {
      const float4 u = *reinterpret_cast<const float4*>(s + w), v = *reinterpret_cast<const float4*>(s + w + 4);
      y = y + ((f2(u.x, u.y) + f2(u.z, u.w)) + (f2(v.x, v.y) + f2(v.z, v.w)));
    }
    return sum(y);
  }
  __device__ __forceinline__ void sum2(float& a, float& b) {
    if (WAY != FULL && tl < 32) {
      for (int o = tl >> 1; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
      }
      return;
    }
    const int l = threadIdx.x & 31;
    const bool upper = l & 16;      // the lower half of the warp goes on with a, the upper with b
    float x = (upper ? b : a) + __shfl_xor_sync(0xffffffffu, upper ? a : b, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (warps == 0) {
      const float y = __shfl_xor_sync(0xffffffffu, x, 16);
      a = upper ? y : x;
      b = upper ? x : y;
      return;
    }
    float* s = sm + turn * 2 * kMostWarps;
    turn ^= 1;
    if ((l & 15) == 0) s[(threadIdx.x >> 5) * 2 + (l >> 4)] = x;
    __syncthreads();
    F2 y = f2(0.f);
    for (int w = 0; w < warps; w += 4) {
      const float4 u = *reinterpret_cast<const float4*>(s + 2 * w), v = *reinterpret_cast<const float4*>(s + 2 * w + 4);
      y = y + ((f2(u.x, u.y) + f2(u.z, u.w)) + (f2(v.x, v.y) + f2(v.z, v.w)));
    }
    const float2 r = split(y);
    a = r.x;
    b = r.y;
  }

  // values of a row in a stage, `off` bytes behind `row` (zero where there are none)
  __device__ __forceinline__ void take(const char* row, int off, bool valid, Pairs& v) const {
    float x[N];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      typename Vec<DT, VEC>::Raw r = {};
      if ((WAY == FULL || valid) && live(j)) {
        if constexpr (WAY == RAGGED) {
          const uint4* at = reinterpret_cast<const uint4*>(row + column(j) * ES);
          r = shifted<DT>(at[0], at[1], off);
        } else {
          r = Vec<DT, VEC>::get(row + off, column(j));
        }
      }
      float y[VEC];
      Vec<DT, VEC>::unpack(r, y);
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[j * VEC + k] = y[k];
    }
    if (WAY == RAGGED && ragged) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = live(i / VEC, i % VEC) ? x[i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = f2(x[2 * i], x[2 * i + 1]);
  }
  // A result's row: RAGGED, to `out` first, from where the team stores it (`flush`, behind a barrier); else at once.
  __device__ __forceinline__ void give(void* base, int row, const Pairs& v, char* out) const {
    char* const to = WAY == RAGGED ? out : static_cast<char*>(base) + (long long)row * (d * ES);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float y[VEC];
      vector(v, j, y);
      if (live(j)) Vec<DT, VEC>::store(to, column(j), y);
    }
  }
  // (`out` has 16 bytes of room before the row)
  __device__ __forceinline__ void flush(void* base, int row, const char* out) const {
    if constexpr (WAY == RAGGED) {
      const long long at = (long long)row * (d * ES);
      const int off = (int)(at & 15), bytes = d * ES, n = (off + bytes + 15) >> 4;
      char* const to = static_cast<char*>(base) + (at - off);
      for (int q = lane; q < n; q += tl) {
        const uint4* from = reinterpret_cast<const uint4*>(out) + q;
        const uint4 w = off == 0 ? from[0] : shifted<DT>(from[-1], from[0], 16 - off);
        const int lo = q == 0 ? off : 0, hi = min(16, off + bytes - q * 16);
        if (lo == 0 && hi == 16) {
          *reinterpret_cast<uint4*>(to + q * 16) = w;
        } else {
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int i = 0; i < 16 / ES; ++i) {
            if (i * ES < lo || i * ES >= hi) continue;
            if constexpr (DT == DK_F32) *reinterpret_cast<uint32_t*>(to + q * 16 + i * 4) = u[i];
            else *reinterpret_cast<uint16_t*>(to + q * 16 + i * 2) = (uint16_t)(i & 1 ? u[i / 2] >> 16 : u[i / 2]);
          }
        }
      }
    }
  }
  static __device__ __forceinline__ void vector(const Pairs& v, int j, float (&y)[VEC]) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const float2 p = split(v[(j * VEC + k) / 2]);
      y[k] = (j * VEC + k) & 1 ? p.y : p.x;
    }
  }
  // fp32 of this thread's columns (0 behind the row): a parameter's, or what give_f32 has put there
  __device__ __forceinline__ void take_f32(const float* p, Pairs& v) const { load_f32<WAY == RAGGED>(p, v); }
  __device__ __forceinline__ void give_f32(float* p, const Pairs& v) const { store_f32<WAY == RAGGED>(p, v); }
  // the same in the team's own shared memory, whole vectors
  __device__ __forceinline__ void take_own(const float* p, Pairs& v) const { load_f32<false>(p, v); }
  __device__ __forceinline__ void give_own(float* p, const Pairs& v) const { store_f32<false>(p, v); }
  template <bool SINGLE>
  __device__ __forceinline__ void load_f32(const float* p, Pairs& v) const {
    float x[N];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const float* const at = p + column(j);
      float y[VEC];
#pragma unroll
      for (int k = 0; k < VEC; ++k) y[k] = 0.f;
      if constexpr (SINGLE || VEC == 1) {
#pragma unroll
        for (int k = 0; k < VEC; ++k)
          if (live(j, k)) y[k] = at[k];
      } else if constexpr (VEC == 2) {
        float2 f = make_float2(0.f, 0.f);
        if (live(j)) f = *reinterpret_cast<const float2*>(at);
        y[0] = f.x; y[1] = f.y;
      } else {
#pragma unroll
        for (int k = 0; k < VEC; k += 4) {
          float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
          if (live(j)) f = *reinterpret_cast<const float4*>(at + k);
          y[k] = f.x; y[k + 1] = f.y; y[k + 2] = f.z; y[k + 3] = f.w;
        }
      }
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[j * VEC + k] = y[k];
    }
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = f2(x[2 * i], x[2 * i + 1]);
  }
  template <bool SINGLE>
  __device__ __forceinline__ void store_f32(float* p, const Pairs& v) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float y[VEC];
      vector(v, j, y);
      float* const at = p + column(j);
      if constexpr (SINGLE || VEC == 1) {
#pragma unroll
        for (int k = 0; k < VEC; ++k)
          if (live(j, k)) at[k] = y[k];
      } else if constexpr (VEC == 2) {
        if (live(j)) *reinterpret_cast<float2*>(at) = make_float2(y[0], y[1]);
      } else {
#pragma unroll
        for (int k = 0; k < VEC; k += 4)
          if (live(j)) *reinterpret_cast<float4*>(at + k) = make_float4(y[k], y[k + 1], y[k + 2], y[k + 3]);
      }
    }
  }
  // gate*post*scale of a gate's rows
  __device__ __forceinline__ void take_factors(const BlockArgs& a, int seg, Pairs& f) const {
    take_f32(a.post, f);
#pragma unroll
    for (int i = 0; i < P; ++i) f[i] = f[i] * f2(a.scale);
    if (a.gate != nullptr) {
      Pairs g;
      take_f32(a.gate + (long long)seg * a.d, g);
#pragma unroll
      for (int i = 0; i < P; ++i) f[i] = f[i] * g[i];
    }
  }
  // the next gate's row on its way into L2
  __device__ __forceinline__ void fetch_gate(const BlockArgs& a, int seg) const {
    for (int c = lane * 32; c < a.d; c += tl * 32)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(a.gate + (long long)seg * a.d + c));
  }

  // Teams of less than a warp: a row of a tensor into a stage by the threads that read it; or in 16-byte pieces, none of which
  // reaches beyond the tensor.
  __device__ __forceinline__ void copy_pieces(uint32_t dst, const void* base, int row, int bytes, int rows) const {
    const long long at = (long long)row * bytes, from = at & ~15LL;
    const int n = ((int)(at & 15) + bytes + 15) >> 4, left = (int)min((long long)rows * bytes - from, (long long)n * 16);
    const char* src = static_cast<const char*>(base) + from;
    for (int i = lane; i < n; i += tl)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + i * 16), "l"(src + i * 16),
                   "r"(min(16, left - i * 16))
                   : "memory");
  }
  __device__ __forceinline__ void copy_tensor(uint32_t dst, const void* base, int row, const BlockArgs& a) const {
    if constexpr (WAY >= RAGGED) {
      copy_pieces(dst, base, row, d * ES, a.rows);
    } else {
      const char* src = static_cast<const char*>(base) + (long long)row * (d * ES);
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (live(j)) copy_async<16>(dst + column(j) * ES, src + column(j) * ES);
    }
  }
  __device__ __forceinline__ void copy_codes(uint32_t dst, const uint8_t* base, int row, const BlockArgs& a) const {
    if constexpr (NARROW) {
      copy_pieces(dst, base, row, a.dp, a.rows);
    } else {
      const uint8_t* src = base + (long long)row * a.dp;
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (live(j)) copy_async<VEC>(dst + column(j), src + column(j));
    }
  }
  // A row of a checkpoint: codes from the stage; the exponents of a thread's vectors fetched a row ahead, NARROW from the stage.
  struct Bytes {
    uint32_t b[NARROW ? 1 : NV];
  };
  __device__ __forceinline__ void fetch_bytes(const uint8_t* exps, int row, const BlockArgs& a, Bytes& b) const {
    if constexpr (!NARROW) {
      const uint8_t* e = exps + (long long)row * (a.dp / ckpt8::kBlock);
#pragma unroll
      for (int j = 0; j < NV; ++j) b.b[j] = live(j) ? __ldg(e + column(j) / ckpt8::kBlock) : 0u;
    }
  }
  __device__ __forceinline__ void take_codes(const char* codes, const char* exps, const Bytes& b, bool valid, Pairs& v) const {
    float x[N], s[N];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      ckpt8::Raw<VEC> r = {};
      if ((WAY == FULL || valid) && live(j)) {
        r = ckpt8::get_codes<VEC>(reinterpret_cast<const uint8_t*>(codes) + column(j));
        r.b = NARROW ? reinterpret_cast<const uint8_t*>(exps)[column(j) / ckpt8::kBlock] : b.b[NARROW ? 0 : j];
      }
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        x[j * VEC + k] = ckpt8::biased<VEC>(r, k);
        s[j * VEC + k] = ckpt8::step_of(r.b);
      }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = (f2(x[2 * i], x[2 * i + 1]) + f2(-ckpt8::kBias)) * f2(s[2 * i], s[2 * i + 1]);
  }
  // codes and exponents of a row
  __device__ __forceinline__ void keep_row(uint8_t* codes, uint8_t* exps, int row, const BlockArgs& a, bool valid,
                                           const Pairs& v) const {
    uint8_t* const to = codes + (long long)row * a.dp;
    uint8_t* const to_e = exps + (long long)row * (a.dp / ckpt8::kBlock);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (WAY != FULL && j > 0 && j * cs >= a.dp) continue;             // (nothing of the row there, whatever the lane)
      float x[VEC];
      vector(v, j, x);
      const ckpt8::Scale s = ckpt8::scale_of(ckpt8::block_most<VEC>(x));
      const int c = column(j);
      if (WAY == FULL || (valid && c < a.dp)) {
        ckpt8::put_codes<VEC>(to + c, x, s);
        if (c % ckpt8::kBlock == 0) to_e[c / ckpt8::kBlock] = (uint8_t)s.byte;
      }
    }
  }
  // (x - mean) in place of x, and 1/sqrt(variance + eps)
  __device__ __forceinline__ float2 normalise(Pairs& v, const BlockArgs& a) {
    float mean = 0.f;
    if (a.layer) {
      F2 s = v[0];
#pragma unroll
      for (int i = 1; i < P; ++i) s = s + v[i];
      mean = sum1(sum(s)) * a.inv_d;
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = v[i] + f2(-mean);
      if (ragged) {                  // (deviations of values that do not exist count as zero)
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const float2 x = split(v[i]);
          v[i] = f2(live(2 * i / VEC, 2 * i % VEC) ? x.x : 0.f, live((2 * i + 1) / VEC, (2 * i + 1) % VEC) ? x.y : 0.f);
        }
      }
    }
    F2 s = v[0] * v[0];
#pragma unroll
    for (int i = 1; i < P; ++i) s = fma(v[i], v[i], s);
    const float m2 = sum1(sum(s));
    return make_float2(mean, inverse_root(fmaf(m2, a.inv_d, a.eps)));
  }
};

template <int DT, int WAY>
__global__ void __launch_bounds__(kFwdThreads<DT>) block_fwd_rows_kernel(const BlockArgs a) {
  constexpr int kStages = kMostStages;
  using T = Team<DT, WAY>;
  constexpr int P = T::P;
  extern __shared__ __align__(16) char ring[];
  __shared__ __align__(16) float sm[4 * kMostWarps];
  __shared__ __align__(8) uint64_t bars[kMostStages * kBulkTeams];
  __shared__ int flag;
  __shared__ Sources sources;
  const bool branch = a.u != nullptr;
  T t(a, sm, bars, &flag, branch ? 2 : 1);
  const int team_in = threadIdx.x / a.tl;
  const int r0 = (int)min((long long)a.rows, ((long long)blockIdx.x * a.teams + team_in) * a.chunk), r1 = r0 + min(a.rows - r0, a.chunk);
  const int bytes = a.d * T::ES, room = stage_room(bytes, WAY >= RAGGED), stage = 2 * room;
  char* const mine = ring + (size_t)team_in * a.team_smem;
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  // (behind the ring, RAGGED: rows on their way out, and shift)
  char* const out = mine + kStages * stage + 16;
  float* const shifts = reinterpret_cast<float*>(mine + kStages * stage + (WAY == RAGGED ? 2 * room : 0));
  if (threadIdx.x == 0) {
    sources.n = 0;
    sources.add(a.h, bytes, 0);
    sources.add(a.u, bytes, room);
  }
  __syncthreads();
  chained_launch();
  auto issue = [&](int row, int slot) {
    if (t.bulk) {
      t.issue_bulk(mine_at + slot * stage, sources, row, r0, r1, slot, a);
      return;
    }
    if (row < r1) {
      t.copy_tensor(mine_at + slot * stage, a.h, row, a);
      if (branch) t.copy_tensor(mine_at + slot * stage + room, a.u, row, a);
    }
    copies_done();
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) issue(r0 + s, s);
  F2 gps[P], pre[P];
  int seg = branch && r0 < r1 ? r0 / a.per : 0;
  long long seg_end = (long long)(seg + 1) * a.per;
  if (branch) t.take_factors(a, seg, gps);
  if (a.n != nullptr) t.take_f32(a.pre, pre);
  if (a.shift != nullptr) {
    F2 v[P];
    t.take_f32(a.shift, v);
    t.give_own(shifts, v);
  }
  if (!t.bulk) wait_copies<kStages - 2>();
  t.sync();
  int slot = 0, before = -1;      // RAGGED: the row whose n is still on its way out
  uint32_t phase = 0;
  for (int i = 0; i < a.chunk; ++i) {
    const int row = r0 + i;
    const bool valid = WAY == FULL || row < r1;
    if ((WAY == FULL || a.tl >= 32) && row >= r1) break;                 // (a team of whole warps has no other team's lanes in them)
    const char* at = mine + slot * stage;
    const int off = WAY >= RAGGED ? (int)(((long long)row * bytes) & 15) : 0;
    issue(row + kStages - 1, slot == 0 ? kStages - 1 : slot - 1);
    t.wait_row(slot, phase, a);
    F2 h[P];
    t.take(at, off, valid, h);
    if (a.kh != nullptr) t.keep_row(a.kh, a.keh, row, a, valid, h);
    float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!t.bulk && a.n == nullptr) wait_copies<kStages - 2>();
    if (branch) {
      F2 u[P];
      t.take(at + room, off, valid, u);
      if (a.ku != nullptr) t.keep_row(a.ku, a.keu, row, a, valid, u);
      if (valid && row == seg_end) {
        seg_end += a.per;
        t.take_factors(a, ++seg, gps);
      }
      if (row + 1 == seg_end && row + 1 < r1) t.fetch_gate(a, seg + 1);
      const float2 m = t.normalise(u, a);
      if (WAY == RAGGED) {
        t.after_sum();
        if (before >= 0) t.flush(a.n, before, out + room);
      }
      st.x = m.x; st.y = m.y;
#pragma unroll
      for (int k = 0; k < P; ++k) h[k] = fma(f2(a.keep), h[k], gps[k] * (u[k] * f2(m.y)));
      if (valid) t.give(a.h_out, row, h, out);
    }
    if (a.n != nullptr) {
      if (!t.bulk) wait_copies<kStages - 2>();
      const float2 m = t.normalise(h, a);
      if (WAY == RAGGED) {
        t.after_sum();
        if (branch && valid) t.flush(a.h_out, row, out);
      }
      st.z = m.x; st.w = m.y;
#pragma unroll
      for (int k = 0; k < P; ++k) h[k] = h[k] * f2(m.y) * pre[k];
      if (a.shift != nullptr) {
        F2 shift[P];
        t.take_own(shifts, shift);
#pragma unroll
        for (int k = 0; k < P; ++k) h[k] = h[k] + shift[k];
      }
      if (valid) t.give(a.n, row, h, out + room);
    }
    if (WAY == RAGGED) {
      // (n waits for the next row's first sum; with one norm alone there is no sum between its rows' ways out)
      before = a.n != nullptr && valid ? row : -1;
      if (a.n == nullptr || !branch) {
        t.sync();
        if (valid) t.flush(a.n != nullptr ? a.n : a.h_out, row, a.n != nullptr ? out + room : out);
        before = -1;
        t.sync();
      }
    }
    if (a.stats != nullptr && t.lane == 0 && valid) a.stats[row] = st;
    if (t.warps == 0) __syncwarp();
    if (++slot == kStages) { slot = 0; phase ^= 1u; }
  }
  wait_copies<0>();
  if (WAY == RAGGED) {
    t.sync();
    if (before >= 0) t.flush(a.n, before, out + room);
  }
  t.leave(a);
}

// Beside the ring a team has [d] fp32 of gate*post*scale, of pre (from L1, which the copies pass through, each reading of it
// stood in the row's way: 243 us for 16384 x 4096 bf16 against 182), where the teams have several gates (split = 0) of dpost, and of dshift where
// that is asked for.
template <int DT, int WAY, bool KEPT>
__global__ void __launch_bounds__(kBwdThreads<DT>) block_bwd_rows_kernel(const BlockArgs a) {
  using T = Team<DT, WAY>;
  constexpr int P = T::P;
  extern __shared__ __align__(16) char ring[];
  __shared__ __align__(16) float sm[4 * kMostWarps];
  __shared__ __align__(8) uint64_t bars[kMostStages * kBulkTeams];
  __shared__ int flag;
  __shared__ Sources sources;
  const bool branch = a.post != nullptr, norm = a.dn != nullptr;
  T t(a, sm, bars, &flag, (a.dh_out != nullptr) + norm + (KEPT && T::NARROW ? 2 : 1) * (1 + branch));
  const int team_in = threadIdx.x / a.tl;
  const long long team = (long long)blockIdx.x * a.teams + team_in;
  const int bytes = a.d * T::ES, eb = a.dp / ckpt8::kBlock;
  const int room = stage_room(bytes, WAY >= RAGGED), room_k = KEPT ? row_room(a.dp) : room;
  const int room_e = KEPT && T::NARROW ? stage_room(eb, true) : 0;
  // a stage: dh', dn, h, u and, NARROW, the exponents of both
  const int at_h = 2 * room, at_u = at_h + room_k, at_eh = at_u + room_k, at_eu = at_eh + room_e, stage = at_eu + room_e;
  const int own = row_room(a.dp * 4), stages = a.stages;
  char* const mine = ring + (size_t)team_in * a.team_smem;
  char* const out = mine + stages * stage + 16;      // (RAGGED: rows on their way out)
  float* const factors = reinterpret_cast<float*>(mine + stages * stage + (WAY == RAGGED ? 2 * room : 0));
  float* const pres = factors + own / 4;
  float* const posts = pres + own / 4;
  float* const shifts = a.split == 0 ? posts + own / 4 : posts;
  const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
  if (threadIdx.x == 0) {
    sources.n = 0;
    sources.add(a.dh_out, bytes, 0);
    sources.add(a.dn, bytes, room);
    sources.add(KEPT ? (const void*)a.ch : a.h, KEPT ? a.dp : bytes, at_h);
    sources.add(KEPT ? (const void*)a.cu : a.u, KEPT ? a.dp : bytes, at_u);
    if (KEPT && T::NARROW) {
      sources.add(a.eh, eb, at_eh);
      sources.add(branch ? a.eu : nullptr, eb, at_eu);
    }
  }
  __syncthreads();
  int r0, r1, seg;
  {
    long long f, e;
    if (a.split) {
      seg = (int)(team / a.split);
      f = (long long)seg * a.per + (long long)(team - (long long)seg * a.split) * a.chunk;
      e = min(min(f + a.chunk, (long long)(seg + 1) * a.per), (long long)a.rows);
    } else {
      f = team * a.chunk;
      e = min(f + a.chunk, (long long)a.rows);
      seg = (int)(f / a.per);
    }
    if (f >= e) { f = e = 0; seg = 0; }        // (a CTA's last teams may have nothing)
    r0 = (int)f; r1 = (int)e;
  }
  long long seg_end = (long long)(seg + 1) * a.per;
  chained_launch();
  auto issue = [&](int row, int slot) {
    const uint32_t to = mine_at + slot * stage;
    if (t.bulk) {
      t.issue_bulk(to, sources, row, r0, r1, slot, a);
      return;
    }
    if (row < r1) {
      if (a.dh_out != nullptr) t.copy_tensor(to, a.dh_out, row, a);
      if (norm) t.copy_tensor(to + room, a.dn, row, a);
      if constexpr (KEPT) {
        t.copy_codes(to + at_h, a.ch, row, a);
        if (T::NARROW) t.copy_pieces(to + at_eh, a.eh, row, eb, a.rows);
        if (branch) {
          t.copy_codes(to + at_u, a.cu, row, a);
          if (T::NARROW) t.copy_pieces(to + at_eu, a.eu, row, eb, a.rows);
        }
      } else {
        t.copy_tensor(to + at_h, a.h, row, a);
        if (branch) t.copy_tensor(to + at_u, a.u, row, a);
      }
    }
    copies_done();
  };
  for (int s = 0; s < stages - 1; ++s) issue(r0 + s, s);
  const F2 zero = f2(0.f);
  F2 E[P], spre[P];
#pragma unroll
  for (int k = 0; k < P; ++k) E[k] = spre[k] = zero;
  if (branch) {
    F2 f[P];
    t.take_factors(a, seg, f);
    t.give_own(factors, f);
    if (a.split == 0) t.give_own(posts, E);
  }
  if (a.shifted) t.give_own(shifts, E);
  if (norm) {
    F2 f[P];
    t.take_f32(a.pre, f);
    t.give_own(pres, f);
  }
  float4 next = make_float4(0.f, 0.f, 0.f, 0.f);
  typename T::Bytes bytes_h = {}, bytes_u = {};
  auto fetch = [&](int row) {
    if (row >= r1) {
      next = make_float4(0.f, 0.f, 0.f, 0.f);      // (of a row that a team does not have)
      return;
    }
    next = __ldg(a.stats + row);
    if constexpr (KEPT) {
      t.fetch_bytes(a.eh, row, a, bytes_h);
      if (branch) t.fetch_bytes(a.eu, row, a, bytes_u);
    }
  };
  fetch(r0);
  if (!t.bulk) {
    if (stages == 3) wait_copies<1>(); else wait_copies<0>();
  }
  t.sync();
  int slot = 0;
  uint32_t phase = 0;
  for (int i = 0; i < a.chunk; ++i) {
    const int row = r0 + i;
    const bool valid = WAY == FULL || row < r1;
    if ((WAY == FULL || a.tl >= 32) && row >= r1) break;
    const char* at = mine + slot * stage;
    const int off = WAY >= RAGGED ? (int)(((long long)row * bytes) & 15) : 0;
    const int off_e = T::NARROW ? (int)(((long long)row * eb) & 15) : 0;
    issue(row + stages - 1, slot == 0 ? stages - 1 : slot - 1);
    t.wait_row(slot, phase, a);
    const float4 st = next;
    if (branch && valid) {
      if (row == seg_end) {
        F2 f[P];
        seg_end += a.per;
        t.take_factors(a, ++seg, f);
        t.give_own(factors, f);
      }
      if (row + 1 == seg_end && row + 1 < r1) t.fetch_gate(a, seg + 1);
    }
    // u^ and h^; sums of q = dn*pre and q*h^
    F2 uh[P], hh[P];
    if constexpr (KEPT) t.take_codes(at + at_h, at + at_eh + off_e, bytes_h, valid, hh);
    else t.take(at + at_h, off, valid, hh);
    if (branch) {
      if constexpr (KEPT) t.take_codes(at + at_u, at + at_eu + off_e, bytes_u, valid, uh);
      else t.take(at + at_u, off, valid, uh);
      F2 f[P];
      t.take_own(factors, f);
      const float ru = normaliser(st.x, st.y);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        uh[k] = (uh[k] + f2(-st.x)) * f2(ru);
        hh[k] = fma(f2(a.keep), hh[k], f[k] * uh[k]);
      }
    }
    fetch(row + 1);
    float m0 = 0.f, m1 = 0.f;
    if (norm) {
      F2 dn[P], pre[P], s0 = zero, s1 = zero;
      t.take(at + room, off, valid, dn);
      t.take_own(pres, pre);
      const float rh = normaliser(st.z, st.w);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        hh[k] = (hh[k] + f2(-st.z)) * f2(rh);
        spre[k] = fma(dn[k], hh[k], spre[k]);
        const F2 q = dn[k] * pre[k];
        s0 = s0 + q;
        s1 = fma(q, hh[k], s1);
      }
      m0 = sum(s0);
      m1 = sum(s1);
      if (a.shifted) {
        t.take_own(shifts, pre);
#pragma unroll
        for (int k = 0; k < P; ++k) pre[k] = pre[k] + dn[k];
        t.give_own(shifts, pre);
      }
    }
    t.sum2(m0, m1);
    m0 = a.layer ? m0 * a.inv_d : 0.f;
    m1 *= a.inv_d;
    // D in h^'s place
    if (norm) {
      F2 dn[P], pre[P];      // (again, from shared memory: held, they would cost the registers of a row)
      t.take(at + room, off, valid, dn);
      t.take_own(pres, pre);
#pragma unroll
      for (int k = 0; k < P; ++k) hh[k] = f2(st.w) * fma(hh[k], f2(-m1), fma(dn[k], pre[k], f2(-m0)));
    } else {
#pragma unroll
      for (int k = 0; k < P; ++k) hh[k] = zero;
    }
    if (a.dh_out != nullptr) {
      F2 dh[P];
      t.take(at, off, valid, dh);
#pragma unroll
      for (int k = 0; k < P; ++k) hh[k] = hh[k] + dh[k];
    }
    float t0 = 0.f, t1 = 0.f;
    if (branch) {
      F2 v[P], s0 = zero, s1 = zero;
#pragma unroll
      for (int k = 0; k < P; ++k) v[k] = f2(a.keep) * hh[k];
      if (valid) t.give(a.dh, row, v, out);
      t.take_own(factors, v);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        E[k] = fma(hh[k], uh[k], E[k]);
        hh[k] = hh[k] * v[k];
        s0 = s0 + hh[k];
        s1 = fma(hh[k], uh[k], s1);
      }
      t0 = sum(s0);
      t1 = sum(s1);
    } else if (valid) {
      t.give(a.dh, row, hh, out);
    }
    if (!t.bulk) {
      if (stages == 3) wait_copies<1>(); else wait_copies<0>();
    }
    if (WAY == RAGGED) {
      t.sync();
      if (valid) t.flush(a.dh, row, out);
    }
    t.sum2(t0, t1);
    if (branch) {
      t0 = a.layer ? t0 * a.inv_d : 0.f;
      t1 *= a.inv_d;
#pragma unroll
      for (int k = 0; k < P; ++k) hh[k] = f2(st.y) * fma(uh[k], f2(-t1), hh[k] + f2(-t0));
      if (valid) {
        t.give(a.du, row, hh, out + room);
        if (a.split == 0 && (row + 1 == r1 || row + 1 == seg_end)) {      // the end of a gate's rows
          F2 g[P], v[P];
          t.take_f32(a.gate + (long long)seg * a.d, g);
          t.take_own(posts, v);
#pragma unroll
          for (int k = 0; k < P; ++k) {
            E[k] = E[k] * f2(a.scale);
            v[k] = fma(g[k], E[k], v[k]);
          }
          t.give_own(posts, v);
          t.take_f32(a.post, g);
#pragma unroll
          for (int k = 0; k < P; ++k) {
            g[k] = g[k] * E[k];
            E[k] = zero;
          }
          t.give_f32(a.dgate + (long long)seg * a.d, g);
        }
      }
    }
    // (at once: held back until the next row's sum, as the forward pass does with n, the way out costs registers: 148 us for
    // 16384 x 1001 against 114)
    if (WAY == RAGGED && branch) {
      t.sync();
      if (valid) t.flush(a.du, row, out + room);
    }
    if (t.warps == 0) __syncwarp();
    if (++slot == stages) { slot = 0; phase ^= 1u; }
  }
  wait_copies<0>();
  t.leave(a);

  // what the team has summed up over its rows
  F2 v[P];
  if (branch && a.split != 0) {
#pragma unroll
    for (int k = 0; k < P; ++k) E[k] = E[k] * f2(a.scale);
    if (a.gate != nullptr && !a.join_e) t.give_f32(a.part_e + team * a.d, E);
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
        t.take_own(posts, v);
      } else if (a.gate == nullptr) {
#pragma unroll
        for (int k = 0; k < P; ++k) v[k] = E[k];
      } else {
        t.take_f32(a.gate + (long long)seg * a.d, v);
#pragma unroll
        for (int k = 0; k < P; ++k) v[k] = v[k] * E[k];
      }
    }
    if (which == 1) t.take_own(shifts, v);
    const F2(&of)[P] = which == 0 ? spre : which == 3 ? E : v;
    if (a.teams > 1) {
      // (at the start of each team's ring, which has room for a row of fp32; what is its own lies behind the ring)
      __syncthreads();
      t.give_own(joined + team_in * (a.team_smem / 4), of);
      __syncthreads();
      for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
        float s = 0.f;
        for (int k = 0; k < a.teams; ++k) s += joined[k * (a.team_smem / 4) + c];
        to[c] = s;
      }
    } else {
      t.give_f32(to, of);
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
  bool wide, whole, full;        // rows above the limit; rows of whole vectors; and of whole warps
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
  if ((double)q->rows * q->d > 1e12 || q->rows > (1LL << 30)) return DK_ERR_SHAPE;
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
  const int most = backward ? (f32 ? kBwdThreads<DK_F32> : kBwdThreads<DK_BF16>) : f32 ? kFwdThreads<DK_F32> : kFwdThreads<DK_BF16>;
  const long long per = asked.gated && q.rows_per_gate < q.rows ? q.rows_per_gate : q.rows;
  p.gates = per > 0 ? (q.rows + per - 1) / per : 0;
  p.whole = q.d % vec == 0;
  const int values = f32 ? kValues<DK_F32> : kValues<DK_BF16>;
  p.full = q.d % (32 * values) == 0;
  const int threads = (dp + values - 1) / values;
  if (threads <= 32) {
    // (a block of 32 values lies in one vector of neighbouring lanes)
    p.tl = ckpt8::kBlock / (p.whole || !f32 ? vec : q.d % 2 == 0 ? 2 : 1);
    while (p.tl < threads) p.tl *= 2;
    p.teams = kSmallTeams / p.tl;
  } else {
    p.tl = (threads + 31) / 32 * 32;
    p.teams = 1;
  }
  // A team's ring of three rows, or of two where that lets an SM hold more teams; and as many rows to a team as give every SM
  // the CTAs that its registers and shared memory hold.  (Backward, teams with several gates each need room for dpost.)
  const int row = stage_room(q.d * es, !p.whole), f32s = row_room(dp * 4), out = p.whole || f32 ? 0 : 2 * row, room = 220 * 1024;
  const int exps = f32 && !p.whole ? stage_room(dp / ckpt8::kBlock, true) : 0;
  const int teams_most = p.teams;
  long long ctas = 0, want = 0, chunk = 0;
  for (int posts = 0; posts < 2; ++posts) {
    ctas = 0;
    for (int stages = 3; stages >= 2; --stages) {
      int smem = stages * 2 * row + out + f32s;
      if (backward) smem = stages * (2 * row + 2 * (asked.held ? row_room(dp) + exps : row)) + out + (2 + posts + asked.shifted) * f32s;
      int teams = teams_most;
      while (teams > 1 && teams * smem > room / 2) teams /= 2;
      long long c = most / (p.tl * teams);
      if (c > room / ((long long)smem * teams + 1024)) c = room / ((long long)smem * teams + 1024);
      if (c < 1) c = (long long)smem * teams <= kMostSmem ? 1 : 0;
      if (c * teams > ctas * p.teams || (ctas == 0 && c > 0)) {
        ctas = c;
        p.smem = smem;
        p.stages = stages;
        p.teams = teams;
      }
      if (!backward) break;
    }
    want = 148 * ctas * p.teams;
    chunk = want > 0 ? (q.rows + want - 1) / want : 1;
    if (!backward || p.gates <= 1 || per > chunk) break;
  }
  p.wide = q.d > kHeld || p.tl > most || ctas == 0;
  if (p.wide) {
    p.tl = ((dp + 15) / 16 + 31) / 32 * 32;
    p.teams = 1;
    p.smem = backward ? 3 * q.d * (int)sizeof(float) : 0;
    ctas = 1;
  }
  if (p.wide) {
    want = 148;
    chunk = (q.rows + want - 1) / want;
  }
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

template <typename K>
dk_status launch_rows(K kern, SmemLimit& limit, const BlockArgs& a, const BlockPlan& p, int smem, int device, cudaStream_t st) {
  const dk_status s = allow_smem(limit, device, kern, kMostSmem);
  if (s != DK_OK) return s;
  return launch_chained(kern, dim3((unsigned)p.ctas), p.tl * p.teams, (size_t)smem, st, a) == cudaSuccess ? DK_OK : DK_ERR_CUDA;
}
// (rows above the limit: vectors as wide as all rows' alignment allows)
template <int DT, int VEC>
dk_status launch_fwd_wide(const BlockArgs& a, const BlockPlan& p, int device, cudaStream_t st) {
  static SmemLimit limit;
  return launch_rows(block_fwd_wide_kernel<DT, VEC, 16 / VEC>, limit, a, p, 0, device, st);
}
template <int DT, int VEC>
dk_status launch_bwd_wide(const BlockArgs& a, const BlockPlan& p, bool kept, int device, cudaStream_t st) {
  static SmemLimit limits[2];
  return kept ? launch_rows(block_bwd_wide_kernel<DT, VEC, 16 / VEC, true>, limits[0], a, p, p.smem, device, st)
              : launch_rows(block_bwd_wide_kernel<DT, VEC, 16 / VEC, false>, limits[1], a, p, p.smem, device, st);
}
template <int DT, int WAY>
dk_status launch_fwd_rows(const BlockArgs& a, const BlockPlan& p, int device, cudaStream_t st) {
  static SmemLimit limit;
  return launch_rows(block_fwd_rows_kernel<DT, WAY>, limit, a, p, p.smem * p.teams, device, st);
}
template <int DT, int WAY>
dk_status launch_bwd_rows(const BlockArgs& a, const BlockPlan& p, bool kept, int device, cudaStream_t st) {
  static SmemLimit limits[2];
  const int smem = p.smem * p.teams;
  return kept ? launch_rows(block_bwd_rows_kernel<DT, WAY, true>, limits[0], a, p, smem, device, st)
              : launch_rows(block_bwd_rows_kernel<DT, WAY, false>, limits[1], a, p, smem, device, st);
}
template <int DT>
dk_status launch_fwd(const BlockArgs& a, const BlockPlan& p, int device, cudaStream_t st) {
  if (p.wide) {
    if constexpr (DT == DK_BF16)
      if (p.whole) return launch_fwd_wide<DT, 8>(a, p, device, st);
    if constexpr (DT == DK_F32)
      if (p.whole) return launch_fwd_wide<DT, 4>(a, p, device, st);
    return a.d % 2 == 0 ? launch_fwd_wide<DT, 2>(a, p, device, st) : launch_fwd_wide<DT, 1>(a, p, device, st);
  }
  if (p.full) return launch_fwd_rows<DT, FULL>(a, p, device, st);
  if (p.whole) return launch_fwd_rows<DT, WHOLE>(a, p, device, st);
  if constexpr (DT == DK_BF16) return launch_fwd_rows<DT, RAGGED>(a, p, device, st);
  else return a.d % 2 == 0 ? launch_fwd_rows<DT, PAIRS>(a, p, device, st) : launch_fwd_rows<DT, SINGLES>(a, p, device, st);
}
template <int DT>
dk_status launch_bwd(const BlockArgs& a, const BlockPlan& p, bool kept, int device, cudaStream_t st) {
  if (p.wide) {
    if constexpr (DT == DK_BF16)
      if (p.whole) return launch_bwd_wide<DT, 8>(a, p, kept, device, st);
    if constexpr (DT == DK_F32)
      if (p.whole) return launch_bwd_wide<DT, 4>(a, p, kept, device, st);
    return a.d % 2 == 0 ? launch_bwd_wide<DT, 2>(a, p, kept, device, st) : launch_bwd_wide<DT, 1>(a, p, kept, device, st);
  }
  if (p.full) return launch_bwd_rows<DT, FULL>(a, p, kept, device, st);
  if (p.whole) return launch_bwd_rows<DT, WHOLE>(a, p, kept, device, st);
  if constexpr (DT == DK_BF16) return launch_bwd_rows<DT, RAGGED>(a, p, kept, device, st);
  else return a.d % 2 == 0 ? launch_bwd_rows<DT, PAIRS>(a, p, kept, device, st) : launch_bwd_rows<DT, SINGLES>(a, p, kept, device, st);
}

// how long the kernels of bulk copies wait
void take_waits(dk_ctx* ctx, const BlockPlan& p, BlockArgs& a) {
  a.spin_cap = (unsigned)ctx->opt.v[DK_OPT_SPIN_LIMIT];
  a.status = device_status_word(ctx);
  a.withhold = -1;
  if (!p.wide && p.tl >= 32) {
    a.withhold = ctx->opt.v[DK_OPT_TEST_WITHHOLD];
    ctx->opt.v[DK_OPT_TEST_WITHHOLD] = -1;
  }
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
  a.rows = (int)q->rows;
  a.per = (int)(gate != nullptr && q->rows_per_gate < q->rows ? q->rows_per_gate : q->rows);
  a.chunk = (int)p.chunk;
  // (with one gate p.split counts the CTAs' parts; its teams' rows are consecutive either way)
  a.split = p.split ? (int)((a.per + p.chunk - 1) / p.chunk) : 0;
  a.join_e = p.join_e && gate != nullptr;
  a.shifted = dshift != nullptr;
  take_waits(ctx, p, a);
  a.d = q->d; a.dp = ckpt8::padded(q->d); a.tl = p.tl; a.teams = p.teams; a.stages = p.stages; a.team_smem = p.smem;
  a.layer = q->kind == DK_BLOCK_LAYER;
  a.eps = q->eps; a.keep = q->keep; a.scale = q->scale; a.inv_d = 1.f / (float)q->d;
  ProfScope ps(ctx, DK_KERNEL_OTHER, 2, st);
  s = q->dtype == DK_F32 ? launch_bwd<DK_F32>(a, p, kept, ctx->device, st) : launch_bwd<DK_BF16>(a, p, kept, ctx->device, st);
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
  a.rows = (int)q->rows;
  a.per = (int)(gate != nullptr && q->rows_per_gate < q->rows ? q->rows_per_gate : q->rows);
  a.chunk = (int)p.chunk;
  a.d = q->d; a.dp = ckpt8::padded(q->d); a.tl = p.tl; a.teams = p.teams; a.stages = p.stages; a.team_smem = p.smem;
  a.layer = q->kind == DK_BLOCK_LAYER;
  a.eps = q->eps; a.keep = q->keep; a.scale = q->scale; a.inv_d = 1.f / (float)q->d;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  take_waits(ctx, p, a);
  ProfScope ps(ctx, DK_KERNEL_OTHER, 1, st);
  return q->dtype == DK_F32 ? launch_fwd<DK_F32>(a, p, ctx->device, st) : launch_fwd<DK_BF16>(a, p, ctx->device, st);
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
