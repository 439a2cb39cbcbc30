// Matrix products C = A.B^T of 16-bit operands on CTA pairs (tcgen05 kind::f16, cta_group::2), for the operators
// around the masked products: bf16 operands as they are, or fp32 operands as two fp16 terms each,
//   v*2^s = hi + lo + e,  hi = fp16(v*2^s),  lo = fp16(v*2^s - hi),  |e| <= 2^-22 |v*2^s| (absolute 2^-25 below),
// of which hi.hi + hi.lo + lo.hi are kept (lo.lo is 2^-22 of the product), or hi.B + lo.B where B needs
// no second term.  fp16 terms run at the full 16-bit rate of the tensor cores, twice that of TF32, at the same 22
// significant bits; what they lack is range, which the common power of two 2^s supplies.
//
// A pair computes a 256 x BN tile: each CTA stages its own 128 rows of A and its half of the BN rows of B, 64
// contraction elements (128 bytes) per stage.  An operand is K-major (rows contiguous along the contraction) or
// MN-major (contiguous along M or N: a stored matrix used transposed needs no transposed copy).  Roles, barriers and
// bounded waits are those of the masked products' pair kernel (dk_tc_pair.cuh).
//
// The tensor pipe truncates when it adds, a loss of about half a unit of the accumulator per addition whatever is added.
// So the accumulator in tensor memory takes `chunk` stages at a time and the epilogue warps add the chunks up in fp32
// registers, rounding to nearest.  What is lost within a chunk is a bias, the same relative amount again and again where
// the terms have one sign (the squares on the diagonal of X X^T), and `comp`, per stage, gives it back on average.  Two
// accumulators of BN columns let the epilogue of one tile run beside the products of the next.  (The small tiles have
// columns to spare: there the products with a low term have an accumulator of their own, 2^-11 times as large, whose
// losses do not count.)
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "dk_step.h"
#include "dk_tc_pair.cuh"

namespace dk {
namespace g16 {

using tc::smem_u32;

constexpr int BK = 64;                       // contraction elements per stage: one 128-byte swizzle span
constexpr int ROWS = 128;                    // rows of A per CTA = TMEM lanes
constexpr int TILE_M = 256;
constexpr int kEpi = 8;                      // epilogue warps per CTA
constexpr int kThreadsG = 32 * (4 + kEpi);

struct Params {
  int MT, NT, nbatch;          // tiles along M (256 rows), along N (BN rows), matrices
  int sym;                     // 1: C is symmetric, only tiles with mt >= nt (needs BN = 256)
  int tiles;                   // tiles of one matrix
  int group;                   // tiles along M that are walked before the next tile along N
  int KB, ksplit, kb_per_split;
  int chunk;                   // stages added up in tensor memory before promotion
  float comp, comp_small;      // relative loss of a stage's additions that promotion makes good (large, small tiles)
  int nitems;                  // nbatch * tiles * ksplit
  int nstages;
  unsigned spin_cap;
  int withhold;                // test hook: the producer arms its n-th stage but issues no copy (-1 = off)
  int bf16;                    // operand type: 1 bf16, 0 fp16
  int M, N;
  int* status;
  // The last wave (epilogues with kTail; one matrix, ksplit = 1): tiles from tail_from on are cut into tail_slices slices
  // of tail_kb stages, whose sums the last of a tile's slices to be done joins.
  int tail_from, tail_slices, tail_kb;
  float* tail_part;            // [slice of a tile][16 warps][32 lanes][128]
  unsigned int* tail_count;    // [tile][16], zero between launches
};

// What an epilogue asks of the pair kernel: kTail (see above), kBulk (it stores by TMA, through the map that B's second plane
// would have had; its stores are waited for at the end).
template <class E, class = void>
struct Asks {
  static constexpr bool tail = false, bulk = false;
};
template <class E>
struct Asks<E, std::void_t<decltype(E::kTail)>> {
  static constexpr bool tail = E::kTail, bulk = E::kBulk;
};

// shared memory of an epilogue warp
template <class E>
constexpr int kRowsMem = Asks<E>::bulk ? 8192 : 4096;

// a stored matrix: `rows` rows of `cols` contiguous elements, `pitch` elements apart (a multiple of 8), one or two
// planes
struct Operand {
  const void* hi;
  const void* lo;
  long long rows, cols, pitch, batch_stride;     // in elements
};

template <bool TAIL = false>
__device__ __forceinline__ void item_tile(const Params& p, int w, int& batch, int& ks, int& mt, int& nt) {
  int t;
  if (TAIL && w >= p.tail_from) {
    ks = (w - p.tail_from) % p.tail_slices;
    t = p.tail_from + (w - p.tail_from) / p.tail_slices;
  } else {
    ks = w % p.ksplit;
    t = w / p.ksplit;
  }
  batch = t / p.tiles;
  t -= batch * p.tiles;
  if (p.sym) {
    mt = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (mt * (mt + 1) / 2 > t) --mt;
    while ((mt + 1) * (mt + 2) / 2 <= t) ++mt;
    nt = t - mt * (mt + 1) / 2;
  } else {
    const int per = p.group * p.NT, gi = t / per, m0 = gi * p.group;
    const int gm = min(p.group, p.MT - m0);
    t -= gi * per;
    nt = t / gm;
    mt = m0 + t - nt * gm;
  }
}

// the stages of an item, and which slice of its contraction it is
template <bool TAIL>
__device__ __forceinline__ int item_stages(const Params& p, int w, int& kb_lo, int& kb_hi) {
  const bool tail = TAIL && w >= p.tail_from;
  const int ks = tail ? (w - p.tail_from) % p.tail_slices : w % p.ksplit, per = tail ? p.tail_kb : p.kb_per_split;
  kb_lo = ks * per;
  kb_hi = min(p.KB, kb_lo + per);
  return ks;
}

// A slice of the last wave: leaves the warp's sums, and, where it is the last of its tile's slices, joins them in the slices'
// order.  True: `acc` is the whole sum.  (Done warp by warp: no barrier between the warps of a tile is needed.)
template <int NH>
__device__ __forceinline__ bool join_tail(const Params& p, int w, uint32_t rank, int epi_warp, float (&acc)[NH]) {
  const int lane = threadIdx.x & 31, item = w - p.tail_from, ks = item % p.tail_slices, tile = item / p.tail_slices;
  const int mine = (int)rank * kEpi + epi_warp;
  auto at = [&](int slice) {      // [4 columns][lane]
    return reinterpret_cast<float4*>(p.tail_part) + (((size_t)tile * p.tail_slices + slice) * (2 * kEpi) + mine) * (32 * NH / 4) + lane;
  };
#pragma unroll
  for (int j = 0; j < NH; j += 4) __stcg(at(ks) + j / 4 * 32, make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]));
  __threadfence();
  __syncwarp();
  unsigned int done = 0;
  if (lane == 0) done = atomicAdd(p.tail_count + tile * 2 * kEpi + mine, 1u) + 1u;
  done = __shfl_sync(0xffffffffu, done, 0);
  if (done != (unsigned)p.tail_slices) return false;
  __threadfence();
  if (lane == 0) p.tail_count[tile * 2 * kEpi + mine] = 0u;
#pragma unroll
  for (int j = 0; j < NH; ++j) acc[j] = 0.f;
  for (int s = 0; s < p.tail_slices; ++s) {
#pragma unroll
    for (int j = 0; j < NH; j += 4) {
      const float4 v = __ldcg(at(s) + j / 4 * 32);
      acc[j] += v.x; acc[j + 1] += v.y; acc[j + 2] += v.z; acc[j + 3] += v.w;
    }
  }
  return true;
}

__device__ __forceinline__ void mma_f16_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void ld32(uint32_t taddr, float* v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

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

// The bits of a magnitude for a maximum: an infinity or a NaN counts as nothing.  (It makes its own row's results NaN; as
// the maximum it would leave all other rows without their power of two.)
__device__ __forceinline__ unsigned int magnitude(unsigned int bits) {
  bits &= 0x7fffffffu;
  return bits < 0x7f800000u ? bits : 0u;
}

// Descriptor of an MN-major tile: [64 contraction rows][64 elements] boxes of 8 KiB, 8-row groups 1 KiB apart, the
// next 64 elements of M or N in the next box.
__device__ __forceinline__ uint64_t desc_mn(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr >> 4) & 0x3FFF);
  d |= (uint64_t)(8192 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// `rows` rows (of M or N) from r0 on, contraction elements from k0 on, of one plane
template <bool MN, int NROWS>
__device__ __forceinline__ void load_tile(unsigned char* dst, const CUtensorMap* map, uint32_t bar, int r0, int k0,
                                          int batch) {
  if constexpr (MN) {
#pragma unroll
    for (int i = 0; i < NROWS / 64; ++i)
      tc::tma_pair_load_3d(dst + i * 8192, map, bar, (r0 + 64 * i) * 2, k0, batch);
  } else {
    tc::tma_pair_load_3d(dst, map, bar, k0 * 2, r0, batch);
  }
}

// planes of A and of B: 1 and 1 (one product), 2 and 1 (two), 2 and 2 (three)
template <int NPROD>
constexpr int kPlanesA = NPROD == 1 ? 1 : 2;
template <int NPROD>
constexpr int kPlanesB = NPROD == 3 ? 2 : 1;

template <int NPROD, int BN>
__host__ __device__ constexpr int stage_bytes() { return (kPlanesA<NPROD> * ROWS + kPlanesB<NPROD> * BN / 2) * 128; }

// Epi: __device__ void operator()(const Params&, float (&acc)[BN/2], int batch, int ks, int row, int col0, char* sm) is
// called by every epilogue thread with its row of C and its BN/2 columns from col0 on (row and columns may lie outside
// C), by whole warps of 32 consecutive rows; sm: 4 KiB of the warp's own (see warp_pieces).
template <int NPROD, bool AMN, bool BMN, int BN, class Epi>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreadsG, 1)
gemm16_kernel(const __grid_constant__ CUtensorMap map_a_hi, const __grid_constant__ CUtensorMap map_a_lo,
              const __grid_constant__ CUtensorMap map_b_hi, const __grid_constant__ CUtensorMap map_b_lo, const Params p,
              const Epi epi) {
  constexpr bool TAIL = Asks<Epi>::tail;
  constexpr int A_BYTES = ROWS * 128, B_BYTES = BN / 2 * 128;
  constexpr int PL = kPlanesA<NPROD>;
  constexpr int STAGE = stage_bytes<NPROD, BN>();
  constexpr int NH = BN / 2;
  static_assert(BN == 256 || BN == 128, "tile width");
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                         ~static_cast<uintptr_t>(1023));
  char* rows_mem = reinterpret_cast<char*>(smem + (size_t)p.nstages * STAGE);
  unsigned char* ctrl = reinterpret_cast<unsigned char*>(rows_mem + kEpi * kRowsMem<Epi>);
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(ctrl);      // used in the leader only
  uint64_t* empty_bar = full_bar + tc::kMaxStages;
  uint64_t* tfull_bar = empty_bar + tc::kMaxStages;
  uint64_t* tempty_bar = tfull_bar + 2;                        // used in the leader only
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tempty_bar + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;

  // what follows up to wait_for_previous touches nothing that an earlier kernel writes
  allow_next();
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.nstages; ++s) { tc::mbar_init(full_bar + s, 1); tc::mbar_init(empty_bar + s, 1); }
    for (int b = 0; b < 2; ++b) { tc::mbar_init(tfull_bar + b, 1); tc::mbar_init(tempty_bar + b, 2 * kEpi); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::cluster_sync_all();
  tc::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  wait_for_previous();

  static_assert(40 * 128 + 232 * 256 <= 168 * kThreadsG, "setmaxnreg budget exceeds the CTA's register pool");
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;" ::: "memory");
    if (warp == 0) {
      // ---------------- TMA producer (both CTAs) ----------------
      if (lane == 0) {
        int stage = 0, issued = 0;
        uint32_t phase = 0;
        bool alive = true;
        for (int w = pair; alive && w < p.nitems; w += npairs) {
          int batch, ks, mt, nt, kb_lo, kb_hi;
          item_tile<TAIL>(p, w, batch, ks, mt, nt);
          item_stages<TAIL>(p, w, kb_lo, kb_hi);
          const int m0 = mt * TILE_M + (int)rank * ROWS, n0 = nt * BN + (int)rank * (BN / 2);
          for (int kb = kb_lo; kb < kb_hi; ++kb) {
            if (!tc::mbar_wait(empty_bar + stage, phase ^ 1u, abort_flag, p.spin_cap)) { alive = false; break; }
            if (rank == 0) tc::mbar_expect_tx(full_bar + stage, (uint32_t)(2 * STAGE));
            if (issued++ == p.withhold) { alive = false; break; }
            unsigned char* st = smem + (size_t)stage * STAGE;
            const uint32_t bar = tc::mapa_shared(smem_u32(full_bar + stage), 0u);
            load_tile<AMN, ROWS>(st, &map_a_hi, bar, m0, kb * BK, batch);
            load_tile<BMN, BN / 2>(st + PL * A_BYTES, &map_b_hi, bar, n0, kb * BK, batch);
            if constexpr (NPROD >= 2) load_tile<AMN, ROWS>(st + A_BYTES, &map_a_lo, bar, m0, kb * BK, batch);
            if constexpr (NPROD == 3)
              load_tile<BMN, BN / 2>(st + PL * A_BYTES + B_BYTES, &map_b_lo, bar, n0, kb * BK, batch);
            if (++stage == p.nstages) { stage = 0; phase ^= 1u; }
          }
        }
      }
    } else if (warp == 1 && rank == 0) {
      // ---------------- MMA issuer (leader only) ----------------
      if (lane == 0) {
        const uint32_t idesc = (1u << 4) | ((uint32_t)p.bf16 << 7) | ((uint32_t)p.bf16 << 10) |
                               ((AMN ? 1u : 0u) << 15) | ((BMN ? 1u : 0u) << 16) | ((uint32_t)(BN >> 3) << 17) |
                               ((uint32_t)(TILE_M >> 4) << 24);
        // 16 contraction elements: 32 bytes along a K-major row, 16 rows of an MN-major box; in 16-byte units
        constexpr uint64_t STEP_A = AMN ? 128 : 2, STEP_B = BMN ? 128 : 2;
        int stage = 0;
        uint32_t phase = 0, acc_it = 0;
        bool alive = true;
        for (int w = pair; alive && w < p.nitems; w += npairs) {
          int kb_lo, kb_hi;
          item_stages<TAIL>(p, w, kb_lo, kb_hi);
          for (int kb = kb_lo; alive && kb < kb_hi; kb += p.chunk, ++acc_it) {
            const uint32_t buf = acc_it & 1u, aphase = (acc_it >> 1) & 1u;
            if (!tc::mbar_wait(tempty_bar + buf, aphase ^ 1u, abort_flag, p.spin_cap)) { alive = false; break; }
            tc::tc_fence_after();
            const uint32_t d_tmem = tmem_base + buf * 256u;
            const int kb_end = min(kb_hi, kb + p.chunk);
            for (int k = kb; k < kb_end; ++k) {
              if (!tc::mbar_wait(full_bar + stage, phase, abort_flag, p.spin_cap)) { alive = false; break; }
              tc::tc_fence_after();
              const uint32_t st = smem_u32(smem + (size_t)stage * STAGE);
              const uint64_t a_hi = AMN ? desc_mn(st) : tc::make_desc<128>(st);
              const uint64_t b_hi = BMN ? desc_mn(st + PL * A_BYTES) : tc::make_desc<128>(st + PL * A_BYTES);
              const bool first = k == kb;
#pragma unroll
              for (int kk = 0; kk < BK / 16; ++kk) {
                mma_f16_pair(d_tmem, a_hi + kk * STEP_A, b_hi + kk * STEP_B, idesc, (first && kk == 0) ? 0u : 1u);
                constexpr uint64_t LO_A = A_BYTES / 16, LO_B = B_BYTES / 16;
                if constexpr (NPROD == 3)
                  mma_f16_pair(d_tmem, a_hi + kk * STEP_A, b_hi + LO_B + kk * STEP_B, idesc, 1u);
                if constexpr (NPROD >= 2)
                  mma_f16_pair(d_tmem, a_hi + LO_A + kk * STEP_A, b_hi + kk * STEP_B, idesc, 1u);
              }
              tc::tc_pair_commit(empty_bar + stage);
              if (++stage == p.nstages) { stage = 0; phase ^= 1u; }
            }
            if (alive) tc::tc_pair_commit(tfull_bar + buf);
          }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;" ::: "memory");
    // ---------------- epilogue: warps 4..11 of both CTAs ----------------
    const int quad = warp & 3, half = (warp - 4) >> 2;
    uint32_t acc_it = 0;
    bool alive = true;
    float acc[NH];
    for (int w = pair; alive && w < p.nitems; w += npairs) {
      int batch, ks, mt, nt, kb_lo, kb_hi;
      item_tile<TAIL>(p, w, batch, ks, mt, nt);
      item_stages<TAIL>(p, w, kb_lo, kb_hi);
      [[maybe_unused]] float2 ahead;      // (what `before` reads is on its way while the products run)
      if constexpr (Asks<Epi>::bulk) ahead = epi.before(p, mt * TILE_M + (int)rank * ROWS + quad * 32 + lane);
      for (int kb = kb_lo; kb < kb_hi; kb += p.chunk, ++acc_it) {
        const uint32_t buf = acc_it & 1u, aphase = (acc_it >> 1) & 1u;
        if (!tc::mbar_wait(tfull_bar + buf, aphase, abort_flag, p.spin_cap)) { alive = false; break; }
        tc::tc_fence_after();
        const uint32_t t = tmem_base + buf * 256u + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * NH);
        const float comp = p.comp * (float)min(p.chunk, kb_hi - kb);
        if (kb == kb_lo) {
#pragma unroll
          for (int c = 0; c < NH; c += 32) ld32(t + (uint32_t)c, acc + c);
          tc::tc_wait_ld();
          if (comp != 0.f) {
#pragma unroll
            for (int j = 0; j < NH; ++j) acc[j] = fmaf(acc[j], comp, acc[j]);
          }
        } else {
#pragma unroll
          for (int c = 0; c < NH; c += 32) {
            float tmp[32];
            ld32(t + (uint32_t)c, tmp);
            tc::tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[c + j] += fmaf(tmp[j], comp, tmp[j]);
          }
        }
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_cluster(tc::mapa_shared(smem_u32(tempty_bar + buf), 0u));
      }
      if (!alive) break;
      if constexpr (TAIL) {
        if (w >= p.tail_from && !join_tail<NH>(p, w, rank, warp - 4, acc)) continue;
      }
      if constexpr (Asks<Epi>::bulk)
        epi(p, acc, mt * TILE_M + (int)rank * ROWS + quad * 32 + lane, nt * BN + half * NH, ahead,
            rows_mem + (warp - 4) * kRowsMem<Epi>, &map_b_lo);
      else
        epi(p, acc, batch, ks, mt * TILE_M + (int)rank * ROWS + quad * 32 + lane, nt * BN + half * NH,
            rows_mem + (warp - 4) * 4096);
    }
    if constexpr (Asks<Epi>::bulk) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }

  // ---------------- teardown ----------------
  tc::tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (threadIdx.x == 0 && p.status != nullptr) atomicExch(p.status, (int)DK_ERR_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(16384);
    __syncthreads();
  }
  tc::cluster_sync_all();
  if (warp == 1) {
    tc::tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// ---------------------------------------------------------------------------
// Few tiles: 128 x 128 tiles of single CTAs, one tile per cluster of CS CTAs that share its contraction.  Each CTA
// sums its slice, leaves the sums in shared memory, and takes CS-th of the tile's columns, whose slices it adds up over
// distributed shared memory in the slices' order.  Nothing goes through global memory and no second kernel joins it.
// ---------------------------------------------------------------------------
constexpr int SMALL = 128;

__device__ __forceinline__ void mma_f16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr)
               : "memory");
  return v;
}
template <bool MN, int NROWS>
__device__ __forceinline__ void load_tile_cta(unsigned char* dst, const CUtensorMap* map, uint64_t* bar, int r0, int k0,
                                              int batch) {
  if constexpr (MN) {
#pragma unroll
    for (int i = 0; i < NROWS / 64; ++i) tc::tma_load_3d(dst + i * 8192, map, bar, (r0 + 64 * i) * 2, k0, batch);
  } else {
    tc::tma_load_3d(dst, map, bar, k0 * 2, r0, batch);
  }
}

template <int NPROD, bool AMN, bool BMN, int CS, class Epi>
__global__ void __launch_bounds__(kThreadsG, 1)
gemm16_small_kernel(const __grid_constant__ CUtensorMap map_a_hi, const __grid_constant__ CUtensorMap map_a_lo,
                    const __grid_constant__ CUtensorMap map_b_hi, const __grid_constant__ CUtensorMap map_b_lo,
                    const Params p, const Epi epi) {
  constexpr int OP = SMALL * 128;                  // bytes of one operand plane in a stage
  constexpr int PL = kPlanesA<NPROD>;
  constexpr int STAGE = (PL + kPlanesB<NPROD>) * OP;
  // Columns of tensor memory between the two accumulators.  With two or three products each is followed by the low terms'
  // own; with three so that hi.hi and hi.lo are one instruction over both planes of B (they lie one after the other) and
  // A's rows are read from shared memory once for both (update of 3 x 512x4608 294 -> 288 us, of 1961x1001 273 -> 268).
  constexpr uint32_t ACC = NPROD >= 2 ? 256u : 128u;
  constexpr int NC = SMALL / 2;                    // columns a thread holds (8 epilogue warps: 4 x 32 rows, 2 halves)
  constexpr int NH = NC / CS;                      // columns it finishes
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                         ~static_cast<uintptr_t>(1023));
  unsigned char* ctrl = smem + (size_t)p.nstages * STAGE;
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(ctrl);
  uint64_t* empty_bar = full_bar + tc::kMaxStages;
  uint64_t* tfull_bar = empty_bar + tc::kMaxStages;
  uint64_t* tempty_bar = tfull_bar + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tempty_bar + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % CS;
  int batch, ks, mt, nt;
  item_tile(p, blockIdx.x / CS, batch, ks, mt, nt);
  const int kb_lo = min(p.KB, rank * p.kb_per_split), kb_hi = min(p.KB, kb_lo + p.kb_per_split);

  allow_next();
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.nstages; ++s) { tc::mbar_init(full_bar + s, 1); tc::mbar_init(empty_bar + s, 1); }
    for (int b = 0; b < 2; ++b) { tc::mbar_init(tfull_bar + b, 1); tc::mbar_init(tempty_bar + b, kEpi); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  wait_for_previous();

  const int quad = warp & 3, half = (warp - 4) >> 2;
  const int row = quad * 32 + lane;
  float acc[NC];
  uint32_t ahead[Epi::kAhead ? NH : 1];            // what the epilogue reads, fetched while the products run
  if (warp == 0) {
    if (lane == 0) {
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      const int m0 = mt * SMALL, n0 = nt * SMALL;
      for (int kb = kb_lo; kb < kb_hi; ++kb) {
        if (!tc::mbar_wait(empty_bar + stage, phase ^ 1u, abort_flag, p.spin_cap)) break;
        tc::mbar_expect_tx(full_bar + stage, (uint32_t)STAGE);
        if (issued++ == p.withhold) break;
        unsigned char* st = smem + (size_t)stage * STAGE;
        load_tile_cta<AMN, SMALL>(st, &map_a_hi, full_bar + stage, m0, kb * BK, batch);
        load_tile_cta<BMN, SMALL>(st + PL * OP, &map_b_hi, full_bar + stage, n0, kb * BK, batch);
        if constexpr (NPROD >= 2) load_tile_cta<AMN, SMALL>(st + OP, &map_a_lo, full_bar + stage, m0, kb * BK, batch);
        if constexpr (NPROD == 3)
          load_tile_cta<BMN, SMALL>(st + PL * OP + OP, &map_b_lo, full_bar + stage, n0, kb * BK, batch);
        if (++stage == p.nstages) { stage = 0; phase ^= 1u; }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | ((uint32_t)p.bf16 << 7) | ((uint32_t)p.bf16 << 10) | ((AMN ? 1u : 0u) << 15) |
                             ((BMN ? 1u : 0u) << 16) | ((uint32_t)(SMALL >> 3) << 17) | ((uint32_t)(SMALL >> 4) << 24);
      const uint32_t idesc_both = idesc + ((uint32_t)(SMALL >> 3) << 17);
      constexpr uint64_t STEP_A = AMN ? 128 : 2, STEP_B = BMN ? 128 : 2, LO = OP / 16;
      int stage = 0;
      uint32_t phase = 0, acc_it = 0;
      bool alive = true;
      for (int kb = kb_lo; alive && kb < kb_hi; kb += p.chunk, ++acc_it) {
        const uint32_t buf = acc_it & 1u, aphase = (acc_it >> 1) & 1u;
        if (!tc::mbar_wait(tempty_bar + buf, aphase ^ 1u, abort_flag, p.spin_cap)) break;
        tc::tc_fence_after();
        const uint32_t d_tmem = tmem_base + buf * ACC;
        const int kb_end = min(kb_hi, kb + p.chunk);
        for (int k = kb; k < kb_end; ++k) {
          if (!tc::mbar_wait(full_bar + stage, phase, abort_flag, p.spin_cap)) { alive = false; break; }
          tc::tc_fence_after();
          const uint32_t st = smem_u32(smem + (size_t)stage * STAGE);
          const uint64_t a_hi = AMN ? desc_mn(st) : tc::make_desc<128>(st);
          const uint64_t b_hi = BMN ? desc_mn(st + PL * OP) : tc::make_desc<128>(st + PL * OP);
#pragma unroll
          for (int kk = 0; kk < BK / 16; ++kk) {
            const bool first = k == kb && kk == 0;
            if constexpr (NPROD == 1) {
              mma_f16(d_tmem, a_hi + kk * STEP_A, b_hi + kk * STEP_B, idesc, first ? 0u : 1u);
            } else if constexpr (NPROD == 2) {
              mma_f16(d_tmem, a_hi + kk * STEP_A, b_hi + kk * STEP_B, idesc, first ? 0u : 1u);
              mma_f16(d_tmem + 128u, a_hi + LO + kk * STEP_A, b_hi + kk * STEP_B, idesc, first && acc_it < 2 ? 0u : 1u);
            } else {
              if (first && acc_it >= 2) {      // a new sum of high terms, the low terms' goes on
                mma_f16(d_tmem, a_hi + kk * STEP_A, b_hi + kk * STEP_B, idesc, 0u);
                mma_f16(d_tmem + 128u, a_hi + kk * STEP_A, b_hi + LO + kk * STEP_B, idesc, 1u);
              } else {
                mma_f16(d_tmem, a_hi + kk * STEP_A, b_hi + kk * STEP_B, idesc_both, first ? 0u : 1u);
              }
              mma_f16(d_tmem + 128u, a_hi + LO + kk * STEP_A, b_hi + kk * STEP_B, idesc, 1u);
            }
          }
          tc::tc_commit(empty_bar + stage);
          if (++stage == p.nstages) { stage = 0; phase ^= 1u; }
        }
        if (alive) tc::tc_commit(tfull_bar + buf);
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    if constexpr (Epi::kAhead) epi.fetch(batch, mt * SMALL + row, nt * SMALL + rank * (SMALL / CS) + half * NH, ahead);
    uint32_t acc_it = 0;
#pragma unroll
    for (int j = 0; j < NC; ++j) acc[j] = 0.f;
    for (int kb = kb_lo; kb < kb_hi; kb += p.chunk, ++acc_it) {
      const uint32_t buf = acc_it & 1u, aphase = (acc_it >> 1) & 1u;
      if (!tc::mbar_wait(tfull_bar + buf, aphase, abort_flag, p.spin_cap)) break;
      tc::tc_fence_after();
      const uint32_t t = tmem_base + buf * ACC + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * NC);
      const float comp = p.comp_small * (float)min(p.chunk, kb_hi - kb);
#pragma unroll
      for (int c = 0; c < NC; c += 32) {
        float tmp[32];
        ld32(t + (uint32_t)c, tmp);
        tc::tc_wait_ld();
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[c + j] += fmaf(tmp[j], comp, tmp[j]);
      }
      if (NPROD >= 2 && kb + p.chunk >= kb_hi) {           // (nothing overwrites them: this was the last chunk)
        for (uint32_t b = 0; b <= min(acc_it, 1u); ++b) {
#pragma unroll
          for (int c = 0; c < NC; c += 32) {
            float tmp[32];
            ld32(tmem_base + b * ACC + 128u + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * NC + c), tmp);
            tc::tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[c + j] += tmp[j];
          }
        }
      }
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tempty_bar + buf);
    }
    if constexpr (CS > 1) {
      // [column / 4][row][column % 4]: every product of this CTA is done, its stages are free
      float4* red = reinterpret_cast<float4*>(smem);
#pragma unroll
      for (int j = 0; j < NC; j += 4)
        red[(half * NC + j) / 4 * SMALL + row] = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
    }
  }
  const bool failed = __syncthreads_or(*abort_flag != 0);
  if constexpr (CS > 1) tc::cluster_sync_all();
  if (warp >= 4 && !failed) {
    const int c0 = rank * (SMALL / CS) + half * NH;        // first of the columns this thread finishes
    float fin[NH];
    if constexpr (CS > 1) {
#pragma unroll
      for (int j = 0; j < NH; ++j) fin[j] = 0.f;
      const uint32_t mine = smem_u32(smem) + (uint32_t)((c0 / 4 * SMALL + row) * 16);
      float4 t[CS][NH / 4];
#pragma unroll
      for (int r = 0; r < CS; ++r) {
        const uint32_t from = tc::mapa_shared(mine, (uint32_t)r);
#pragma unroll
        for (int j = 0; j < NH / 4; ++j) t[r][j] = ld_cluster4(from + (uint32_t)(j * SMALL * 16));
      }
#pragma unroll
      for (int r = 0; r < CS; ++r) {
#pragma unroll
        for (int j = 0; j < NH / 4; ++j) {
          fin[4 * j] += t[r][j].x; fin[4 * j + 1] += t[r][j].y; fin[4 * j + 2] += t[r][j].z; fin[4 * j + 3] += t[r][j].w;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NH; ++j) fin[j] = acc[j];
    }
    // (the stages behind the cluster's sums are free)
    char* sm = reinterpret_cast<char*>(smem + SMALL * SMALL * 4) + (warp - 4) * 4096;
    if constexpr (Epi::kAhead) epi(p, fin, batch, mt * SMALL + row, nt * SMALL + c0, sm, ahead);
    else epi(p, fin, batch, 0, mt * SMALL + row, nt * SMALL + c0, sm);
  }
  // ---------------- teardown ----------------
  tc::tc_fence_before();
  __syncthreads();
  if (failed) {
    if (threadIdx.x == 0 && p.status != nullptr) atomicExch(p.status, (int)DK_ERR_TIMEOUT);
    for (int i = 0; i < 64; ++i) __nanosleep(16384);
    __syncthreads();
  }
  if constexpr (CS > 1) tc::cluster_sync_all();      // no CTA leaves while its sums are being read
  if (warp == 1) {
    tc::tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// ---------------------------------------------------------------------------
// epilogues shared by the operators
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 t = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}
// what the first of two terms leaves of a value; INF: nothing of an infinity, whose products then have the first term's
template <bool INF>
__device__ __forceinline__ float left_over(float v, float first) {
  return INF && fabsf(first) == __int_as_float(0x7f800000) ? 0.f : v - first;
}
// two fp16 terms of v[j]
template <int NV, bool INF = false>
__device__ __forceinline__ void store_planes(__half* hi, __half* lo, const float (&v)[NV], int count) {
  // (pitches are multiples of 8 and padding columns may be written: they are zero, as the operands' are)
#pragma unroll
  for (int j = 0; j < NV; j += 8) {
    if (j < count) {
      uint32_t h[4], l[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float a = v[j + 2 * q], b = v[j + 2 * q + 1];
        const __half2 t = __floats2half2_rn(a, b);
        h[q] = *reinterpret_cast<const uint32_t*>(&t);
        l[q] = pack_f16(left_over<INF>(a, __low2float(t)), left_over<INF>(b, __high2float(t)));
      }
      *reinterpret_cast<uint4*>(hi + j) = make_uint4(h[0], h[1], h[2], h[3]);
      *reinterpret_cast<uint4*>(lo + j) = make_uint4(l[0], l[1], l[2], l[3]);
    }
  }
}

// A thread holds columns of its row, the 32 lanes 32 rows.  Stored like that, every store instruction touches 32 lines
// and the tile's epilogue takes 14000 cycles, longer than the products of a short contraction (256 x 256 x 512: 12600).
// So a warp turns 16-byte pieces over in shared memory (their places exchanged within a row against bank conflicts): P
// pieces of its row go in from every thread, and f(r, q, piece) gets piece q of row r, P neighbouring lanes a row.
// P * 512 bytes of `sm`.
template <int P, class F>
__device__ __forceinline__ void warp_pieces(const uint4 (&v)[P], char* sm, F f) {
  static_assert(P == 1 || P == 2 || P == 4 || P == 8, "pieces of a row");
  const int lane = threadIdx.x & 31;
  auto place = [](int r, int q) { return (r * P + (q ^ ((r * P >> 3) & (P - 1)))) * 16; };
  __syncwarp();
#pragma unroll
  for (int q = 0; q < P; ++q) *reinterpret_cast<uint4*>(sm + place(lane, q)) = v[q];
  __syncwarp();
  uint4 t[P];
#pragma unroll
  for (int i = 0; i < P; ++i) t[i] = *reinterpret_cast<const uint4*>(sm + place(i * (32 / P) + lane / P, lane % P));
#pragma unroll
  for (int i = 0; i < P; ++i) f(i * (32 / P) + lane / P, lane % P, t[i]);
}
// fp32 values of a row, W at a time: f(r, c, value of columns c .. c+3)
template <int NH, class F>
__device__ __forceinline__ void warp_rows_f32(const float (&v)[NH], char* sm, F f) {
  constexpr int W = NH < 32 ? NH : 32;
#pragma unroll
  for (int c = 0; c < NH; c += W) {
    uint4 t[W / 4];
#pragma unroll
    for (int q = 0; q < W / 4; ++q)
      t[q] = make_uint4(__float_as_uint(v[c + 4 * q]), __float_as_uint(v[c + 4 * q + 1]), __float_as_uint(v[c + 4 * q + 2]),
                        __float_as_uint(v[c + 4 * q + 3]));
    warp_pieces<W / 4>(t, sm, [&](int r, int q, const uint4& u) {
      f(r, c + 4 * q, make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)));
    });
  }
}
// 16-bit values of a block of W <= 64 columns, two to a word: f(r, c, columns c .. c+7 of the block)
template <int W, class F>
__device__ __forceinline__ void warp_block_16(const uint32_t (&v)[W / 2], char* sm, F f) {
  uint4 t[W / 8];
#pragma unroll
  for (int q = 0; q < W / 8; ++q) t[q] = make_uint4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
  warp_pieces<W / 8>(t, sm, [&](int r, int q, const uint4& u) { f(r, 8 * q, u); });
}
// bf16 of a row's values: f(r, c, columns c .. c+7)
template <int NH, class F>
__device__ __forceinline__ void warp_rows_bf16(const float (&v)[NH], char* sm, F f) {
  constexpr int W = NH < 64 ? NH : 64;
#pragma unroll
  for (int c = 0; c < NH; c += W) {
    uint32_t w[W / 2];
#pragma unroll
    for (int j = 0; j < W / 2; ++j) w[j] = pack_bf16(v[c + 2 * j], v[c + 2 * j + 1]);
    warp_block_16<W>(w, sm, [&](int r, int k, const uint4& u) { f(r, c + k, u); });
  }
}
// two fp16 terms of W of a thread's values from v[c] on
template <int W, int NH>
__device__ __forceinline__ void to_terms(const float (&v)[NH], int c, uint32_t (&hi)[W / 2], uint32_t (&lo)[W / 2]) {
#pragma unroll
  for (int j = 0; j < W / 2; ++j) {
    const float a = v[c + 2 * j], b = v[c + 2 * j + 1];
    const __half2 t = __floats2half2_rn(a, b);
    hi[j] = *reinterpret_cast<const uint32_t*>(&t);
    lo[j] = pack_f16(a - __low2float(t), b - __high2float(t));
  }
}
// a piece of eight 16-bit (four 32-bit) elements of which `count` exist
__device__ __forceinline__ void put_piece16(void* dst, const uint4& u, int count) {
  if (count >= 8 && (reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
    *static_cast<uint4*>(dst) = u;
  } else {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint16_t* d = static_cast<uint16_t*>(dst);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < count) d[j] = (uint16_t)(j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu);
  }
}
__device__ __forceinline__ void put_piece32(float* dst, const float4& u, int count) {
  if (count >= 4 && (reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
    *reinterpret_cast<float4*>(dst) = u;
  } else {
    const float w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < count) dst[j] = w[j];
  }
}
// rows of two fp16 terms to planes whose pitch is a multiple of 8 (padding columns may be written); rows, cols: how many
// of the warp's 32 rows and of the columns exist
template <int NH>
__device__ __forceinline__ void store_terms(const float (&v)[NH], char* sm, __half* hi, __half* lo, long long pitch, int rows,
                                            int cols) {
  constexpr int W = NH <= 64 ? NH : 32;            // (of 128: 32 at a time spill 52 bytes a thread, 64 at a time 640)
#pragma unroll
  for (int c0 = 0; c0 < NH; c0 += W) {
    uint32_t h[W / 2], l[W / 2];
    to_terms<W>(v, c0, h, l);
    warp_block_16<W>(h, sm, [&](int r, int c, const uint4& u) {
      if (r < rows && c0 + c < cols) *reinterpret_cast<uint4*>(hi + r * pitch + c0 + c) = u;
    });
    warp_block_16<W>(l, sm, [&](int r, int c, const uint4& u) {
      if (r < rows && c0 + c < cols) *reinterpret_cast<uint4*>(lo + r * pitch + c0 + c) = u;
    });
  }
}

// fp32 rows of a warp stored by TMA: 32 columns at a time through the two halves of the warp's 8 KiB of shared memory
// (128-byte rows, their 16-byte pieces exchanged as the 128-byte swizzle has them, so the writes meet no bank twice).  The
// map clips what lies outside the matrix.  A tile of 256 x 256 takes half the instructions of warp_rows_f32 (256 rows, 25088
// x 4096 fp32: 1568 tiles of four stages, the product takes 172 us with warp_rows_f32, 121 with one half, 110 with two).
// A piece goes to the half that the piece before did not, whose store is the only one that may still read: but a tile may have
// had one piece or three (1 to 32 or 65 to 96 columns left of 128) and ended where this one begins, so a tile's first piece
// waits for all of them.  (They had the time that the tile's sums took: no slower.  Counting a warp's pieces over its tiles
// instead costs registers: that product's call 128 us against 126, of bf16 118 against 114.)
template <int NH>
__device__ __forceinline__ void warp_rows_bulk(const float (&v)[NH], char* sm, const CUtensorMap* map, int row0, int col0, int cols) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int c = 0; c < NH; c += 32) {
    if (c >= cols) break;
    char* const to = sm + (c / 32 & 1) * 4096;
    if (lane == 0) {
      if (c == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      else asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
    }
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q)
      *reinterpret_cast<float4*>(to + lane * 128 + ((q ^ (lane & 7)) << 4)) =
          make_float4(v[c + 4 * q], v[c + 4 * q + 1], v[c + 4 * q + 2], v[c + 4 * q + 3]);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"((col0 + c) * 4),
                   "r"(row0), "r"(smem_u32(to))
                   : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
}

// fp32 partial sums of a contraction slice: part[ks][batch][M][pitch]
struct EpiPartial {
  static constexpr bool kAhead = false;
  float* part;
  int pitch;             // multiple of 4
  template <int NH>
  __device__ __forceinline__ void operator()(const Params& p, float (&acc)[NH], int batch, int ks, int row, int col0,
                                             char* sm) const {
    const int row0 = row - (int)(threadIdx.x & 31);
    if (row0 >= p.M || col0 >= p.N) return;
    float* dst = part + ((size_t)(ks * p.nbatch + batch) * p.M + row0) * pitch + col0;
    const int rows = p.M - row0, cols = p.N - col0;
    warp_rows_f32<NH>(acc, sm, [&](int r, int c, const float4& u) {
      if (r < rows && c < cols) *reinterpret_cast<float4*>(dst + (size_t)r * pitch + c) = u;
    });
  }
};

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// How a product is computed: `cs` = 0: 256 x 256 tiles of CTA pairs, `ksplit` slices of the contraction with partial
// sums in global memory; cs > 0: 128 x 128 tiles, clusters of cs CTAs sharing the contraction.
constexpr int kSmallCtas = 8 * kMaxSms;      // most CTAs of a product in small tiles
struct Tiling {
  int cs;
  int narrow;                  // cs = 0: tiles of 256 x 128
  int MT, NT, tiles, KB, ksplit, kb_per_split;
};

// Cost in cycles of either way, from what was measured: a stage (64 contraction elements) of the pair's tile takes 512
// cycles per product, of the small tile 256, but what binds the small tile is shared memory, where its operands arrive
// and every product reads them again (taken as 16 KiB per operand plane at 50 bytes per cycle, 1311 cycles for three
// products; with A's rows read once for both planes of B the slope over the contraction is 1430 to 1520 cycles where 128 to
// 144 CTAs are at work, 64 KiB each through L2); some 9000 cycles go
// to a launch's start, fill and epilogue, 6000 more to joining a cluster's slices, 24000 to the partial sums' way through
// global memory and a second kernel.  Clusters of four and eight do not tile the GPCs: 33 and 15 of them are resident at
// once on 148 SMs.  `narrow`: the caller has a kernel of three products for pair tiles of 256 x 128 too (the update's X:
// 3 x 512x4608, 216 tiles instead of 108 on 74 pairs, 300 us -> 293 for the whole update; 4 x 130x5000 251 -> 236).
inline Tiling plan(long long M, long long N, long long K, int nbatch, bool sym, int sms, int nprod,
                   bool narrow = false) {
  Tiling best = {};
  double least = 0;
  const int KB = (int)((K + BK - 1) / BK);
  for (int cs = 0; cs <= 8; cs = cs ? 2 * cs : 1) {
    const int tm = cs ? SMALL : TILE_M;
    Tiling t = {};
    t.cs = cs;
    const long long MT = (M + tm - 1) / tm, NT = (N + tm - 1) / tm;
    const long long tiles = sym ? MT * (MT + 1) / 2 : MT * NT;
    if (tiles * nbatch >= (1LL << 26)) { if (cs) continue; }
    t.MT = (int)MT; t.NT = (int)NT; t.tiles = (int)tiles;
    t.KB = KB;
    double cost;
    if (cs == 0) {
      const int pairs = sms / 2;
      int want = (int)(pairs / (tiles * nbatch));
      if (want < 1) want = 1;
      int per = (KB + want - 1) / want;
      if (per < 4) per = 4;
      if (per > KB) per = KB;
      t.kb_per_split = per;
      t.ksplit = (KB + per - 1) / per;
      const double waves = (double)((tiles * nbatch * t.ksplit + pairs - 1) / pairs);
      cost = waves * per * 512.0 * nprod + 9000.0 + (t.ksplit > 1 ? 24000.0 : 0.0);
    } else {
      if (cs > 1 && KB < 2 * cs) continue;             // at least two stages each
      const long long ctas = tiles * nbatch * cs;
      if (ctas > kSmallCtas) continue;
      const long long resident = cs <= 2 ? sms / cs : cs == 4 ? sms * 33 / 148 : sms * 15 / 148;
      const double waves = (double)((tiles * nbatch + resident - 1) / resident);
      t.kb_per_split = (KB + cs - 1) / cs;
      t.ksplit = 1;
      const double stage = (nprod + 1) * 16384.0 / 50.0;
      cost = waves * (t.kb_per_split * (stage > 256.0 * nprod ? stage : 256.0 * nprod) + 9000.0 + (cs > 1 ? 6000.0 : 0.0));
    }
    if (cs == 0 || cost < least) { least = cost; best = t; }
  }
  // Pair tiles of 256 x 128 instead of 256 x 256: a stage of three products takes 1150 cycles (operands through shared
  // memory) against 1600, but they fill whole waves better, and their epilogue is half as long (3000 cycles against
  // 6000, which a short contraction does not hide).
  if (narrow && !best.cs && best.ksplit == 1) {
    const int pairs = sms / 2;
    Tiling t = best;
    t.narrow = 1;
    t.NT = (int)((N + 127) / 128);
    auto cost = [&](const Tiling& v, double stage, double epilogue) {
      const double waves = (double)(((long long)v.MT * v.NT * nbatch + pairs - 1) / pairs);
      return waves * (KB * stage > epilogue ? KB * stage : epilogue) + epilogue;
    };
    if ((long long)t.MT * t.NT * nbatch < (1LL << 26) && cost(t, 1150.0, 3000.0) < cost(best, 1600.0, 6000.0)) {
      t.tiles = t.MT * t.NT;
      best = t;
    }
  }
  return best;
}

inline bool make_map(const dk_ctx* ctx, CUtensorMap* m, const void* base, const Operand& o, int nbatch, bool mn,
                     int box_rows) {
  const unsigned long long dims[3] = {(unsigned long long)o.cols * 2, (unsigned long long)o.rows,
                                      (unsigned long long)nbatch};
  const unsigned long long str[2] = {(unsigned long long)o.pitch * 2,
                                     (unsigned long long)(nbatch > 1 ? o.batch_stride : o.pitch * o.rows) * 2};
  const unsigned int box[3] = {128, mn ? (unsigned)BK : (unsigned)box_rows, 1};
  return tc_encode_map_bytes(ctx, m, base, 3, dims, str, box, 128);
}

template <int NPROD, bool AMN, bool BMN, int CS, class Epi>
dk_status launch_small(dk_ctx* ctx, const Operand& A, const Operand& B, Params p, const Epi& epi, cudaStream_t st) {
  static SmemLimit limit;
  CUtensorMap ma, mal, mb, mbl;
  if (!make_map(ctx, &ma, A.hi, A, p.nbatch, AMN, SMALL) || !make_map(ctx, &mb, B.hi, B, p.nbatch, BMN, SMALL))
    return DK_ERR_CUDA;
  mal = ma; mbl = mb;
  if ((NPROD >= 2 && !make_map(ctx, &mal, A.lo, A, p.nbatch, AMN, SMALL)) ||
      (NPROD == 3 && !make_map(ctx, &mbl, B.lo, B, p.nbatch, BMN, SMALL)))
    return DK_ERR_CUDA;
  constexpr int STAGE = (kPlanesA<NPROD> + kPlanesB<NPROD>) * SMALL * 128;
  constexpr int CTRL = (2 * tc::kMaxStages + 4) * 8 + 16;
  p.nstages = NPROD == 3 ? 3 : NPROD == 2 ? 4 : 6;
  const int smem = p.nstages * STAGE + CTRL + 1024;
  if (smem > tc_smem_optin(ctx)) return DK_ERR_UNSUPPORTED;
  auto kern = gemm16_small_kernel<NPROD, AMN, BMN, CS, Epi>;
  const dk_status r = allow_smem(limit, ctx->device, kern, smem);
  if (r != DK_OK) return r;
  p.ksplit = 1;
  p.nitems = p.nbatch * p.tiles;
  p.group = p.MT < 16 ? p.MT : 16;
  p.spin_cap = (unsigned)ctx->opt.v[DK_OPT_SPIN_LIMIT];
  p.withhold = ctx->opt.v[DK_OPT_TEST_WITHHOLD];
  ctx->opt.v[DK_OPT_TEST_WITHHOLD] = -1;
  p.status = device_status_word(ctx);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.nitems * CS));
  cfg.blockDim = dim3(kThreadsG);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = CS;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = CS > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, ma, mal, mb, mbl, p, epi) == cudaSuccess ? DK_OK : DK_ERR_CUDA;
}

// p: MT, NT, nbatch, sym, tiles, KB, ksplit, kb_per_split, M, N, chunk are set by the caller
template <int NPROD, bool AMN, bool BMN, int BN, class Epi>
dk_status launch(dk_ctx* ctx, const Operand& A, const Operand& B, Params p, const Epi& epi, cudaStream_t st,
                 const CUtensorMap* out = nullptr) {
  static_assert(!Asks<Epi>::bulk || NPROD < 3, "the second plane of B has the map");
  static SmemLimit limit;
  CUtensorMap ma, mal, mb, mbl;
  if (!make_map(ctx, &ma, A.hi, A, p.nbatch, AMN, ROWS) || !make_map(ctx, &mb, B.hi, B, p.nbatch, BMN, BN / 2))
    return DK_ERR_CUDA;
  mal = ma; mbl = mb;
  if (Asks<Epi>::bulk) {
    if (out == nullptr) return DK_ERR_INVALID_ARG;
    mbl = *out;
  }
  if ((NPROD >= 2 && !make_map(ctx, &mal, A.lo, A, p.nbatch, AMN, ROWS)) ||
      (NPROD == 3 && !make_map(ctx, &mbl, B.lo, B, p.nbatch, BMN, BN / 2)))
    return DK_ERR_CUDA;
  constexpr int STAGE = stage_bytes<NPROD, BN>();
  constexpr int CTRL = (2 * tc::kMaxStages + 4) * 8 + 16;
  constexpr int ROWS_MEM = kEpi * kRowsMem<Epi>;
  p.nstages = (227 * 1024 - 1024 - CTRL - ROWS_MEM) / STAGE;
  if (p.nstages > tc::kMaxStages) p.nstages = tc::kMaxStages;
  const int smem = p.nstages * STAGE + ROWS_MEM + CTRL + 1024;
  if (smem > tc_smem_optin(ctx)) return DK_ERR_UNSUPPORTED;
  auto kern = gemm16_kernel<NPROD, AMN, BMN, BN, Epi>;
  // (the setmaxnreg split draws on threads * registers at launch; a smaller pool would wait forever)
  const dk_status r = allow_smem(limit, ctx->device, kern, smem, kThreadsG, 40 * 128 + 232 * 256);
  if (r != DK_OK) return r;
  p.nitems = p.nbatch * p.tiles * p.ksplit;
  p.group = p.MT < 16 ? p.MT : 16;
  p.spin_cap = (unsigned)ctx->opt.v[DK_OPT_SPIN_LIMIT];
  p.withhold = ctx->opt.v[DK_OPT_TEST_WITHHOLD];
  ctx->opt.v[DK_OPT_TEST_WITHHOLD] = -1;
  p.status = device_status_word(ctx);
  int pairs = ctx->sm_count / 2;
  if constexpr (Asks<Epi>::tail) {
    // What the last wave leaves idle, against what joining a tile's slices takes (some 12000 cycles: 128 KiB a CTA written
    // and read again through L2).  16384 rows, 4096 x 4096: 256 tiles on 74 pairs, 3.46 waves.
    p.tail_from = p.tiles;
    p.tail_slices = 1;
    const int rest = p.tiles % pairs;
    int slices = rest > 0 ? pairs / rest : 1;
    const int kb = (p.KB + slices - 1) / slices;
    slices = (p.KB + kb - 1) / kb;
    if (slices > 1 && (p.KB - kb) * 512 * NPROD > 12000 && rest * 2 * kEpi <= kStepCounters && p.tail_part != nullptr) {
      p.tail_from = p.tiles - rest;
      p.tail_slices = slices;
      p.tail_kb = kb;
      p.nitems = p.tail_from + rest * slices;
    }
  }
  if (pairs > p.nitems) pairs = p.nitems;
  return launch_chained(kern, dim3(2 * (unsigned)pairs), kThreadsG, (size_t)smem, st, ma, mal, mb, mbl, p, epi) == cudaSuccess
             ? DK_OK
             : DK_ERR_CUDA;
}

// The product by the way `t` says; `epi` finishes its elements (t.cs > 0, or t.ksplit == 1 and an epilogue that has
// nothing to fetch ahead).
template <int NPROD, bool AMN, bool BMN, bool NARROW = false, class Epi>
dk_status product(dk_ctx* ctx, const Tiling& t, const Operand& A, const Operand& B, const Params& p, const Epi& epi,
                  cudaStream_t st) {
  if constexpr (NARROW) {
    if (t.narrow) return launch<NPROD, AMN, BMN, 128, Epi>(ctx, A, B, p, epi, st);
  }
  if constexpr (!Epi::kAhead) {
    if (t.cs == 0) return launch<NPROD, AMN, BMN, 256, Epi>(ctx, A, B, p, epi, st);
  }
  switch (t.cs) {
    case 1: return launch_small<NPROD, AMN, BMN, 1, Epi>(ctx, A, B, p, epi, st);
    case 2: return launch_small<NPROD, AMN, BMN, 2, Epi>(ctx, A, B, p, epi, st);
    case 4: return launch_small<NPROD, AMN, BMN, 4, Epi>(ctx, A, B, p, epi, st);
    case 8: return launch_small<NPROD, AMN, BMN, 8, Epi>(ctx, A, B, p, epi, st);
  }
  return DK_ERR_UNSUPPORTED;
}

}  // namespace g16
}  // namespace dk
