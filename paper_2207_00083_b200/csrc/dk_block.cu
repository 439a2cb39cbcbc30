// The norms before and after a residual block, fused with its gate and residual scale, forward and backward.
//
//   u^ = (u - mean_u)*rstd_u,  h' = keep*h + scale*gate*post*u^,  h^ = (h' - mean_h)*rstd_h,  n = h^*pre + shift
//   q = dn*pre,  D = dh' + rstd_h*(q - mean(q) - h^*mean(q*h^)),  dh = keep*D
//   s = scale*gate*post*D,  du = rstd_u*(s - mean(s) - u^*mean(s*u^))
//   E = scale*D*u^:  dgate = sum E*post over the gate's rows,  dpost = sum E*gate,  dpre = sum dn*h^,  dshift = sum dn
// (root mean square: the means that are subtracted are zero, and rstd = 1/sqrt(mean(x^2) + eps)).
//
// A row is a team's: 4 to 32 lanes, or a CTA; a thread has eight of its values (sixteen forward, above 8192) in registers,
// so a row is read once.  Deviations are summed about the mean of the values in registers.  Backward, a team takes
// consecutive rows and keeps the sums over rows of its columns in registers; the rows of one gate are never split
// unevenly, so a gate's sums are either one team's, written at once, or of a fixed number of teams, joined in order by
// block_sums_kernel.  Rows above 4096 values are read again in each phase of the backward pass (from L2) and their sums
// over rows kept in shared memory.
#include "dk_ckpt8.cuh"
#include "dk_internal.h"
#include "dk_step.h"
#include "dk_vec.cuh"

namespace dk {
namespace {

constexpr int kMaxD = 16384;
constexpr int kHeld = 4096;            // values of a row that the backward pass holds in registers
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

template <int DT, int VEC, int NV>
__global__ void __launch_bounds__(1024) block_fwd_kernel(const BlockArgs a) {
  chained_launch();
  __shared__ float sm[2 * 32];
  int turn = 0;
  const int lane = threadIdx.x % a.tl;
  const long long row = (long long)blockIdx.x * a.teams + threadIdx.x / a.tl;
  const bool valid = row < a.rows;
  float h[NV][VEC], u[NV][VEC];
  bool live[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * a.tl + lane) * VEC;
    live[j] = valid && c < a.d;
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
    const float* gate = a.gate != nullptr && valid ? a.gate + row / a.per * a.d : nullptr;
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
  if (a.stats != nullptr && lane == 0 && valid) a.stats[row] = st;
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
                                          const float4& st, bool again) {
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

// BIG: rows that are read again in each phase, sums over rows in shared memory ([3][d]: E, dpre, dshift).
template <int DT, int VEC, int NV, bool KEPT, bool BIG>
__global__ void __launch_bounds__(BIG ? 1024 : 512) block_bwd_kernel(const BlockArgs a) {
  extern __shared__ float dyn[];         // BIG: sums; else [teams][d], where a CTA's teams join theirs
  __shared__ float sm[2 * 32 * 2];
  chained_launch();
  int turn = 0;
  const int lane = threadIdx.x % a.tl, team_in = threadIdx.x / a.tl;
  const long long team = (long long)blockIdx.x * a.teams + team_in;
  long long r0, r1;
  if (a.split) {
    const long long seg = team / a.split;
    r0 = seg * a.per + team % a.split * a.chunk;
    r1 = min(min(r0 + a.chunk, (seg + 1) * a.per), a.rows);
  } else {
    r0 = team * a.chunk;
    r1 = min(r0 + a.chunk, a.rows);
  }
  constexpr int NA = BIG ? 1 : NV;
  float E[NA][VEC], spre[NA][VEC], sshift[NA][VEC], spost[NA][VEC];
#pragma unroll
  for (int j = 0; j < NA; ++j)
#pragma unroll
    for (int k = 0; k < VEC; ++k) E[j][k] = spre[j][k] = sshift[j][k] = spost[j][k] = 0.f;
  float* const big_post = a.part + (2LL * gridDim.x + blockIdx.x) * a.d;      // (BIG: this CTA's sums of dpost)
  if constexpr (BIG) {
    for (int j = 0; j < NV; ++j) {
      const int c = (j * a.tl + lane) * VEC;
      if (c < a.d) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          dyn[c + k] = dyn[a.d + c + k] = dyn[2 * a.d + c + k] = 0.f;
          if (a.post != nullptr) big_post[c + k] = 0.f;
        }
      }
    }
  }

  for (long long i = 0; i < a.chunk; ++i) {
    const long long row = r0 + i;
    const bool valid = row < r1;
    if (a.tl >= 32 && !valid) break;                 // (a team of whole warps has no other team's lanes in them)
    const long long seg = valid ? row / a.per : 0;
    const float* gate = a.gate != nullptr ? a.gate + seg * a.d : nullptr;
    const float4 st = valid ? __ldg(a.stats + row) : make_float4(0.f, 0.f, 0.f, 0.f);
    Cell<VEC> cell[NA];
    float m[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * a.tl + lane) * VEC;
      if (!(valid && c < a.d)) continue;
      Cell<VEC>& e = cell[BIG ? 0 : j];
      load_cell<DT, VEC, KEPT>(e, a, row, c, gate, st, false);
      if (a.dn != nullptr) {
        float pre[VEC];
        load_param<VEC>(a.pre, c, pre);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          if constexpr (BIG) {
            dyn[a.d + c + k] = fmaf(e.dn[k], e.hh[k], dyn[a.d + c + k]);
            dyn[2 * a.d + c + k] += e.dn[k];
          } else {
            spre[j][k] = fmaf(e.dn[k], e.hh[k], spre[j][k]);
            sshift[j][k] += e.dn[k];
          }
          const float q = e.dn[k] * pre[k];
          m[0] += q;
          m[1] = fmaf(q, e.hh[k], m[1]);
          e.dn[k] = q;
        }
      }
    }
    if (a.dn != nullptr) team_sum<2>(m, a.tl, sm, turn);
    const float m0 = a.layer ? m[0] * a.inv_d : 0.f, m1 = m[1] * a.inv_d;
    float t[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * a.tl + lane) * VEC;
      if (!(valid && c < a.d)) continue;
      Cell<VEC>& e = cell[BIG ? 0 : j];
      if constexpr (BIG) {
        load_cell<DT, VEC, KEPT>(e, a, row, c, gate, st, true);
        if (a.dn != nullptr) {
          float pre[VEC];
          load_param<VEC>(a.pre, c, pre);
#pragma unroll
          for (int k = 0; k < VEC; ++k) e.dn[k] *= pre[k];
        }
      }
      float D[VEC], v[VEC];
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        D[k] = a.dh_out != nullptr ? e.dho[k] : 0.f;
        if (a.dn != nullptr) D[k] = fmaf(st.w, e.dn[k] - m0 - e.hh[k] * m1, D[k]);
        v[k] = a.post != nullptr ? a.keep * D[k] : D[k];
      }
      // (dh may be dh_out: nothing reads this vector of it again, but BIG's last phase)
      if (!BIG || a.post == nullptr) Vec<DT, VEC>::store(a.dh, row * a.d + c, v);
      if (a.post != nullptr) {
        float post[VEC], g[VEC];
        load_param<VEC>(a.post, c, post);
        load_gate<VEC>(gate, c, g);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float sd = a.scale * D[k];
          if constexpr (BIG) dyn[c + k] = fmaf(sd, e.uh[k], dyn[c + k]);
          else E[j][k] = fmaf(sd, e.uh[k], E[j][k]);
          const float s = sd * g[k] * post[k];
          t[0] += s;
          t[1] = fmaf(s, e.uh[k], t[1]);
          e.dn[k] = s;
        }
      }
    }
    if (a.post != nullptr) {
      team_sum<2>(t, a.tl, sm, turn);
      const float t0 = a.layer ? t[0] * a.inv_d : 0.f, t1 = t[1] * a.inv_d;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * a.tl + lane) * VEC;
        if (!(valid && c < a.d)) continue;
        Cell<VEC>& e = cell[BIG ? 0 : j];
        if constexpr (BIG) {
          load_cell<DT, VEC, KEPT>(e, a, row, c, gate, st, true);
          float post[VEC], g[VEC], pre[VEC], v[VEC];
          load_param<VEC>(a.post, c, post);
          load_gate<VEC>(gate, c, g);
          if (a.dn != nullptr) load_param<VEC>(a.pre, c, pre);
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            float D = a.dh_out != nullptr ? e.dho[k] : 0.f;
            if (a.dn != nullptr) D = fmaf(st.w, e.dn[k] * pre[k] - m0 - e.hh[k] * m1, D);
            v[k] = a.keep * D;
            e.dn[k] = a.scale * D * g[k] * post[k];
          }
          Vec<DT, VEC>::store(a.dh, row * a.d + c, v);
        }
        float v[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = st.y * (e.dn[k] - t0 - e.uh[k] * t1);
        Vec<DT, VEC>::store(a.du, row * a.d + c, v);
      }
      // the end of a gate's rows
      if (valid && (row + 1 == r1 || (row + 1) / a.per != seg)) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int c = (j * a.tl + lane) * VEC;
          if (c >= a.d) continue;
          float post[VEC], g[VEC];
          load_param<VEC>(a.post, c, post);
          load_gate<VEC>(gate, c, g);
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            float& s = BIG ? dyn[c + k] : E[BIG ? 0 : j][k];
            if constexpr (BIG) big_post[c + k] = fmaf(g[k], s, big_post[c + k]);
            else spost[j][k] = fmaf(g[k], s, spost[j][k]);
            if (a.gate != nullptr && a.split == 0) a.dgate[seg * a.d + c + k] = s * post[k];
            if (a.split == 0) s = 0.f;
          }
        }
      }
    }
  }

  // what the team has summed up over its rows
  if (a.post != nullptr && a.gate != nullptr && a.split != 0 && !a.join_e) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * a.tl + lane) * VEC;
      if (c >= a.d) continue;
#pragma unroll
      for (int k = 0; k < VEC; ++k) a.part_e[team * a.d + c + k] = BIG ? dyn[c + k] : E[BIG ? 0 : j][k];
    }
  }
  const long long slab = (long long)gridDim.x * a.d;
#pragma unroll
  for (int which = 0; which < 4; ++which) {            // dpre, dshift, dpost, E
    if (which < 2 && a.dn == nullptr) continue;
    if (which >= 2 && a.post == nullptr) continue;
    if (which == 3 && !a.join_e) continue;
    float* to = (which == 3 ? a.part_e : a.part + which * slab) + (long long)blockIdx.x * a.d;
    if constexpr (BIG) {
      if (which == 2) continue;                        // (there already)
      const float* from = dyn + (which == 3 ? 0 : which + 1) * a.d;
      for (int j = 0; j < NV; ++j) {
        const int c = (j * a.tl + lane) * VEC;
        if (c < a.d) {
#pragma unroll
          for (int k = 0; k < VEC; ++k) to[c + k] = from[c + k];
        }
      }
    } else {
      float* mine = a.teams > 1 ? dyn + team_in * a.d : to;
      if (a.teams > 1) __syncthreads();
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * a.tl + lane) * VEC;
        if (c < a.d) {
#pragma unroll
          for (int k = 0; k < VEC; ++k)
            mine[c + k] = which == 0 ? spre[j][k] : which == 1 ? sshift[j][k] : which == 2 ? spost[j][k] : E[j][k];
        }
      }
      if (a.teams > 1) {
        __syncthreads();
        for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
          float s = 0.f;
          for (int i = 0; i < a.teams; ++i) s += dyn[i * a.d + c];
          to[c] = s;
        }
      }
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
  int vec, per_thread;           // values of a vector, and of a thread
  int tl, teams;
  bool big;
  // backward
  long long chunk, nteams, ctas, gates;
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

// `gated`: rows_per_gate counts
BlockPlan plan_block(const dk_block& q, bool backward, bool gated) {
  BlockPlan p = {};
  const int full = q.dtype == DK_F32 ? 4 : 8;
  p.vec = full;
  while (q.d % p.vec) p.vec /= 2;
  const int dp = ckpt8::padded(q.d);
  p.big = backward && q.d > kHeld;
  p.per_thread = q.d > (backward ? kHeld : 8192) ? 16 : 8;
  const int threads = (dp + p.per_thread - 1) / p.per_thread;
  if (threads <= 32) {
    p.tl = ckpt8::kBlock / p.vec;            // (a block of 32 values lies in one vector of neighbouring lanes)
    while (p.tl < threads) p.tl *= 2;
    p.teams = kSmallTeams / p.tl;
  } else {
    p.tl = (threads + 31) / 32 * 32;
    p.teams = 1;
  }
  if (!backward) return p;
  // Rows of a team: as many as give every SM its threads.
  const long long per = gated && q.rows_per_gate < q.rows ? q.rows_per_gate : q.rows;
  long long resident = p.teams > 1 ? 3 * p.teams : 768 / p.tl;
  if (resident < 1) resident = 1;
  const long long want = 148 * resident;
  long long chunk = (q.rows + want - 1) / want;
  if (chunk < 1) chunk = 1;
  p.gates = per > 0 ? (q.rows + per - 1) / per : 0;
  if (per <= chunk && p.gates > 1) {
    p.split = 0;
    p.chunk = (chunk + per - 1) / per * per;
    p.nteams = (q.rows + p.chunk - 1) / p.chunk;
  } else {
    const long long k = per > 0 ? (per + chunk - 1) / chunk : 1;
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
cudaError_t launch_fwd(const BlockArgs& a, const BlockPlan& p, cudaStream_t st) {
  const dim3 grid((unsigned)((a.rows + p.teams - 1) / p.teams));
  const int threads = p.tl * p.teams;
  return p.per_thread == 8 ? launch_chained(block_fwd_kernel<DT, VEC, 8 / VEC>, grid, threads, 0, st, a)
                           : launch_chained(block_fwd_kernel<DT, VEC, 16 / VEC>, grid, threads, 0, st, a);
}

template <int DT, int VEC, bool KEPT>
dk_status launch_bwd(const BlockArgs& a, const BlockPlan& p, int device, cudaStream_t st) {
  const dim3 grid((unsigned)p.ctas);
  const int threads = p.tl * p.teams;
  cudaError_t e;
  if (p.big) {
    auto kern = block_bwd_kernel<DT, VEC, 16 / VEC, KEPT, true>;
    static SmemLimit limit;
    const dk_status s = allow_smem(limit, device, kern, 3 * kMaxD * (int)sizeof(float));
    if (s != DK_OK) return s;
    e = launch_chained(kern, grid, threads, (size_t)3 * a.d * sizeof(float), st, a);
  } else {
    const size_t smem = p.teams > 1 ? (size_t)p.teams * a.d * sizeof(float) : 0;
    e = launch_chained(block_bwd_kernel<DT, VEC, 8 / VEC, KEPT, false>, grid, threads, smem, st, a);
  }
  return e == cudaSuccess ? DK_OK : DK_ERR_CUDA;
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
  const BlockPlan p = plan_block(*q, true, gate != nullptr);
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
  a.d = q->d; a.dp = ckpt8::padded(q->d); a.tl = p.tl; a.teams = p.teams;
  a.layer = q->kind == DK_BLOCK_LAYER;
  a.eps = q->eps; a.keep = q->keep; a.scale = q->scale; a.inv_d = 1.f / (float)q->d;
  ProfScope ps(ctx, DK_KERNEL_OTHER, 2, st);
#define DK_BLOCK_BWD(DT, V)                                                             \
  s = kept ? launch_bwd<DT, V, true>(a, p, ctx->device, st) : launch_bwd<DT, V, false>(a, p, ctx->device, st)
  if (q->dtype == DK_F32) {
    if (p.vec == 4) DK_BLOCK_BWD(DK_F32, 4);
    else if (p.vec == 2) DK_BLOCK_BWD(DK_F32, 2);
    else DK_BLOCK_BWD(DK_F32, 1);
  } else {
    if (p.vec == 8) DK_BLOCK_BWD(DK_BF16, 8);
    else if (p.vec == 4) DK_BLOCK_BWD(DK_BF16, 4);
    else if (p.vec == 2) DK_BLOCK_BWD(DK_BF16, 2);
    else DK_BLOCK_BWD(DK_BF16, 1);
  }
#undef DK_BLOCK_BWD
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
    for (bool gated : {false, true}) {
      const size_t n = plan_block(*q, true, gated).total;
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
  const BlockPlan p = plan_block(*q, false, false);
  BlockArgs a = {};
  a.h = h; a.u = u; a.gate = gate; a.post = post; a.pre = pre; a.shift = shift;
  a.h_out = h_out; a.n = n; a.stats = reinterpret_cast<float4*>(stats);
  const long long codes = ckpt8::code_bytes(q->rows, q->d);
  a.kh = static_cast<uint8_t*>(ckpt_h);
  a.ku = static_cast<uint8_t*>(ckpt_u);
  if (a.kh) a.keh = a.kh + codes;
  if (a.ku) a.keu = a.ku + codes;
  a.rows = q->rows;
  a.per = q->rows_per_gate;
  a.d = q->d; a.dp = ckpt8::padded(q->d); a.tl = p.tl; a.teams = p.teams;
  a.layer = q->kind == DK_BLOCK_LAYER;
  a.eps = q->eps; a.keep = q->keep; a.scale = q->scale; a.inv_d = 1.f / (float)q->d;
  OnDevice dev(ctx->device);
  if (!dev.ok) return DK_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ProfScope ps(ctx, DK_KERNEL_OTHER, 1, st);
  cudaError_t e;
  if (q->dtype == DK_F32)
    e = p.vec == 4 ? launch_fwd<DK_F32, 4>(a, p, st) : p.vec == 2 ? launch_fwd<DK_F32, 2>(a, p, st) : launch_fwd<DK_F32, 1>(a, p, st);
  else
    e = p.vec == 8   ? launch_fwd<DK_BF16, 8>(a, p, st)
        : p.vec == 4 ? launch_fwd<DK_BF16, 4>(a, p, st)
        : p.vec == 2 ? launch_fwd<DK_BF16, 2>(a, p, st)
                     : launch_fwd<DK_BF16, 1>(a, p, st);
  return e == cudaSuccess ? DK_OK : DK_ERR_CUDA;
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
