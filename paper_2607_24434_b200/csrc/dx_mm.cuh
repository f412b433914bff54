// The matrix products of the batch operators: one persistent kernel skeleton on the 5th-generation tensor cores.
//
//   D[lane m, column n] = sum_k A[m, k] B[n, k]     bf16 operands, fp32 accumulators in tensor memory
//
// A tile is 128 lanes per CTA and up to 256 columns.  CG = 1: a CTA by itself.  CG = 2: a pair of CTAs on two SMs whose
// tensor cores work as one on 256 lanes; each CTA fetches its own 128 rows of A and HALF of the columns' rows of B, so
// a stage of the contraction costs 32 KB of L2 reads per SM instead of 48 KB for the same products per SM.
//
// The contraction goes in blocks of 64 elements through a ring of shared-memory stages that tensor-map copies (TMA) fill:
// rows of 128 bytes in the 128-byte swizzle that tcgen05.mma reads.  Either operand may be "K-major" (its rows lie along
// the contraction) or "MN-major" (its rows lie across it: a box holds 64 contraction rows of 64 lanes or columns), so
// that transposed weights and products over the rows themselves need no transposed copy.  Rows may be gathered by index
// (tile::gather4, four rows of 128 bytes per copy); an index outside the matrix reads zeros.
//
// Warps: 0-3 take finished tiles out of tensor memory (lanes 32 w .. 32 w + 31), 4 issues the copies, 5 owns the tensor
// memory and issues the products (one lane; in a pair only the first CTA's).  Two accumulators take turns, so a tile
// is stored while the next one is multiplied.  Every wait is bounded; one that runs out raises the CTA's abort flag,
// after which nothing more is copied or multiplied, copies and products in flight are waited for (bounded), tensor
// memory is freed and DX_DEV_WAIT_EXPIRED stands in the status word.
#pragma once

#include <cuda.h>

#include "dx_internal.cuh"
#include "dx_stream.cuh"

namespace {

constexpr int kMmThreads = 192;
constexpr int kMmK = 64;                    // contraction elements of a stage: 128 bytes of a row
constexpr int kMmA = 128 * kMmK * 2;        // bytes of a CTA's 128 rows of A in a stage
constexpr int kMmMaxStages = 8;

// ---- PTX ---------------------------------------------------------------------------------------------------------
// In a pair, every copy reports to the FIRST CTA's barrier: its address is the local one with the CTA bit cleared.
constexpr uint32_t kFirstCta = 0xFEFFFFFFu;

template <int CG>
__device__ __forceinline__ void tma2(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar & kFirstCta) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tma3(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar & kFirstCta) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tma5(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int u, int v, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(u), "r"(v), "r"(bar & kFirstCta) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(u), "r"(v), "r"(bar) : "memory");
}
// four rows of the matrix, 128 bytes of each (the map's box is one row high)
template <int CG>
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap* map, int x, int r0, int r1, int r2, int r3,
                                            uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar & kFirstCta) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Shared-memory matrix descriptors, 128-byte swizzle (bits 61..63 = 2), descriptor version 1 (bit 46).
// K-major: groups of eight rows are 1024 bytes apart (sbo); a step of 16 contraction elements is 32 bytes further.
// MN-major: boxes of 64 lanes (columns) x 64 contraction rows of 128 bytes; eight contraction rows are 1024 bytes apart
// (sbo), the next 64 lanes 8192 (lbo); a step of 16 contraction rows is 2048 bytes further.
__device__ __forceinline__ uint64_t mm_desc(uint32_t addr, bool mn_major) {
  const uint32_t lo = ((addr & 0x3FFFFu) >> 4) | ((mn_major ? 8192u >> 4 : 1u) << 16);
  const uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);
  return (uint64_t)hi << 32 | lo;
}
// fp32 accumulators, bf16 operands, the operands' majors, columns / 8, lanes / 16
__host__ __device__ constexpr uint32_t mm_idesc(bool a_mn, bool b_mn, int lanes, int columns) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(columns >> 3) << 17) | ((uint32_t)(lanes >> 4) << 24);
}
template <int CG>
__device__ __forceinline__ void mm_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CG == 2)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives at the barrier (in a pair: at both CTAs' barriers of this offset) once all products issued so far are done
template <int CG>
__device__ __forceinline__ void mm_commit(uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void mm_tmem_alloc(uint32_t where, uint32_t columns) {
  if constexpr (CG == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::);
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
}
template <int CG>
__device__ __forceinline__ void mm_tmem_free(uint32_t base, uint32_t columns) {
  if constexpr (CG == 2)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
  else
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}
__device__ __forceinline__ void mm_ld32(uint32_t taddr, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// arrive at the first CTA's barrier of this offset
__device__ __forceinline__ void arrive_at_first(uint32_t bar) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, 0;\n\t"
               "mbarrier.arrive.release.cluster.shared::cluster.b64 _, [a];\n\t}" ::"r"(bar) : "memory");
}
// Wait of the warps that store finished tiles: lane 0 polls with pauses, so that their scheduler partitions stay free for
// the copying and the multiplying warp.
__device__ __forceinline__ bool mm_store_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t limit, int lane) {
  int ok = 1;
  if (lane == 0) {
    ok = 0;
    for (uint32_t it = 0; it < limit; ++it) {
      if (mbar_try_wait(bar, parity)) { ok = 1; break; }
      if ((it & 15u) == 15u && *abort_flag) break;
      __nanosleep(32);
    }
    if (!ok) *abort_flag = 1;
  }
  return __shfl_sync(0xffffffffu, ok, 0) != 0;
}

// ---- parameters ----------------------------------------------------------------------------------------------------
struct MmMaps {
  CUtensorMap a, b;       // boxes of rows
  CUtensorMap ag, bg;     // the same matrices for gathered rows
};
struct MmParams {
  int n_groups, n_rows;          // groups; rows of the sorted order (offsets lie in 0 .. n_rows)
  int lanes, columns, kdim;      // extents of D's lanes and columns and of the contraction, where they are not rows
  int a_rows, b_rows;            // rows of the matrices that are gathered from (an index outside reads zeros)
  const int32_t* offsets;        // [n_groups + 1]
  const int32_t* a_index;        // sorted row -> index / a_div = row of A's matrix (null: the row itself)
  const int32_t* b_index;
  int a_div, b_div;
  // output: element (row of column n, lane m) at out + row * ld + m
  void* out;
  int64_t ld;
  int64_t group_stride;          // elements between the groups' outputs (products over rows)
  const int32_t* scatter;        // sorted row -> row of out (null: itself)
  int out_rows;
  const float* addend;           // fp32, added to the products, laid out like out
  // SwiGLU
  void* save;                    // [n_rows, 2 I] gate and up products
  int64_t ld_save;
  const void* gate_up;
  int64_t ld_gate_up;
  const float* pair_w;           // weight of pair q
  int n_pairs;
  void* act_w;
  int64_t ld_act;
  float* partial;                // [warps of lanes][n_rows] shares of the pair weights' gradients
  // loss
  const int32_t* n_live;         // rows that count
  const int32_t* targets;        // [..] by original row
  const float* row_weight;
  float2* part;                  // [column tiles][pitch] (maximum, sum) of a tile
  int part_pitch;
  float* target_logit;           // [n_live]
  const float* lse;              // [n_live]
  const float* row_loss;         // [n_live]
  int column0;                   // first column's word
  int32_t* dev_status;
  uint32_t wait_limit;
};

// Which operand comes from where
enum MmForm {
  kRows,      // lanes: rows of W_e (K-major); columns: sorted rows (K-major, gathered or not)
  kRowsT,     // lanes: columns of W_e (MN-major); columns: sorted rows
  kSwiglu,    // as kRows, the lanes eight gate rows and eight up rows in turns
  kOuter,     // lanes, columns: columns of two matrices of rows (both MN-major); the contraction goes over a group's rows
  kHead       // lanes: live rows (gathered, K-major); columns: rows of W
};
__host__ __device__ constexpr bool mm_a_mn(int form) { return form == kRowsT || form == kOuter; }
__host__ __device__ constexpr bool mm_b_mn(int form) { return form == kOuter; }

struct MmShared {
  unsigned long long full[kMmMaxStages];
  unsigned long long empty[kMmMaxStages];
  unsigned long long acc_full[2], acc_empty[2], drained;
  uint32_t tmem_base;
  int abort_flag;
  int tiles;                     // of the launch
  int off[DX_MAX_E + 1];         // first row of a group, and behind it its end where the next begins elsewhere
  int cnt[DX_MAX_E];
  int before[DX_MAX_E + 1];      // row tiles in front of a group
};

struct MmTile {
  int e;          // group
  int m0;         // first lane's index (of the tile, not of the CTA)
  int n0;         // first column's index; for rows as columns: the sorted row
  int ncols;      // columns that exist
  int row0, rows; // (contraction over rows) the group's rows
  int kblocks;
};

template <int FORM, int CG, int BN>
struct MmSchedule {
  const MmParams& p;
  const MmShared* s;
  int m_tiles, n_tiles, e;
  __device__ MmSchedule(const MmParams& p_, const MmShared* s_) : p(p_), s(s_), e(0) {
    const int lanes = FORM == kHead ? s->cnt[0] : p.lanes;
    m_tiles = (lanes + 128 * CG - 1) / (128 * CG);
    n_tiles = (p.columns + BN - 1) / BN;
  }
  // (tiles are asked for in ascending order)
  __device__ __forceinline__ MmTile get(int t) {
    MmTile r;
    if constexpr (FORM == kOuter) {
      const int per = m_tiles * n_tiles;
      r.e = t / per;
      const int rest = t - r.e * per;
      const int nt = rest / m_tiles;
      r.m0 = (rest - nt * m_tiles) * 128 * CG;
      r.n0 = nt * BN;
      r.ncols = min(BN, p.columns - r.n0);
      r.row0 = s->off[r.e];
      r.rows = s->cnt[r.e];
      r.kblocks = (r.rows + kMmK - 1) / kMmK;
    } else if constexpr (FORM == kHead) {
      const int nt = t / m_tiles;
      r.e = 0;
      r.m0 = (t - nt * m_tiles) * 128 * CG;
      r.n0 = nt * BN;
      r.ncols = min(BN, p.columns - r.n0);
      r.row0 = 0;
      r.rows = s->cnt[0];
      r.kblocks = (p.kdim + kMmK - 1) / kMmK;
    } else {
      const int nt = t / m_tiles;
      while (e + 1 < p.n_groups && s->before[e + 1] <= nt) ++e;
      r.e = e;
      r.m0 = (t - nt * m_tiles) * 128 * CG;
      // a group's rows are split evenly over its tiles
      const int cnt = s->cnt[e], k = s->before[e + 1] - s->before[e], j = nt - s->before[e];
      const int each = (cnt + k - 1) / k, width = (each + 16 * CG - 1) / (16 * CG) * (16 * CG);
      r.n0 = s->off[e] + j * width;
      r.ncols = min(width, cnt - j * width);
      r.row0 = r.n0;
      r.rows = r.ncols;
      r.kblocks = (p.kdim + kMmK - 1) / kMmK;
    }
    return r;
  }
};
// columns of the products of a tile
template <int CG>
__device__ __forceinline__ int mm_width(int ncols) { return (ncols + 16 * CG - 1) / (16 * CG) * (16 * CG); }

// row of the matrix that sorted row r takes (-1, which reads zeros, where the index points outside)
__device__ __forceinline__ int mm_source(const int32_t* index, int div, int r, int n_rows, int32_t* dev_status) {
  if (!index) return r;
  const int q = __ldg(index + r);
  const int row = q < 0 ? -1 : div == 1 ? q : q / div;
  if (row >= 0 && row < n_rows) return row;
  atomicExch(dev_status, (int32_t)DX_DEV_BAD_ROW);
  return -1;
}

template <int FORM, int CG, int BN, int STAGES, class Epilogue>
__global__ void __launch_bounds__(kMmThreads, 1)
dx_mm_kernel(const __grid_constant__ MmMaps maps, const __grid_constant__ MmParams p) {
  constexpr int kHalf = BN / CG;                       // columns whose rows a CTA fetches
  constexpr int kB = (kHalf < 32 ? 32 : kHalf) * kMmK * 2;
  constexpr int kStage = kMmA + kB;
  constexpr bool A_MN = mm_a_mn(FORM), B_MN = mm_b_mn(FORM);
  constexpr uint32_t kAccCols = BN < 32 ? 32 : BN, kTmemCols = 2 * kAccCols;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  MmShared* s = reinterpret_cast<MmShared*>(ring + (size_t)STAGES * kStage);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cta_rank() : 0u;
  const int unit = blockIdx.x / CG, n_units = gridDim.x / CG;
  volatile int* abort_flag = &s->abort_flag;

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(smem_u32(&s->full[i]), 1);
      mbar_init(smem_u32(&s->empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&s->acc_full[i]), 1);
      mbar_init(smem_u32(&s->acc_empty[i]), 4 * CG);
    }
    mbar_init(smem_u32(&s->drained), 1);
    s->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (FORM != kHead) tma_prefetch_map(&maps.a);
    tma_prefetch_map(FORM != kHead && FORM != kOuter && p.b_index ? &maps.bg : &maps.b);
    if (FORM == kHead || FORM == kOuter) tma_prefetch_map(&maps.ag);
  }
  if (warp == 5) mm_tmem_alloc<CG>(smem_u32(&s->tmem_base), kTmemCols);
  dx_pdl_wait();
  // the groups: rows outside [0, n_rows) and ends in front of their beginnings are cut off and reported
  if (warp == 0) {
    int run = 0;
    for (int e0 = 0; e0 < p.n_groups; e0 += 32) {
      const int e = e0 + lane;
      int lo = 0, hi = 0;
      if (e < p.n_groups) {
        if (FORM == kHead) {
          hi = __ldg(p.n_live);
        } else {
          lo = __ldg(p.offsets + e);
          hi = __ldg(p.offsets + e + 1);
        }
        const int a = min(max(lo, 0), p.n_rows), b = min(max(hi, a), p.n_rows);
        if (a != lo || b != hi) atomicExch(p.dev_status, (int32_t)DX_DEV_BAD_OFFSETS);
        lo = a;
        hi = b;
        s->off[e] = lo;
        s->cnt[e] = hi - lo;
      }
      int tiles = (hi - lo + BN - 1) / BN, sum = tiles;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += o;
      }
      if (e < p.n_groups) s->before[e] = run + sum - tiles;
      run += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) s->before[p.n_groups] = run;
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2) pair_sync();     // (the other CTA's barriers exist)
  tc_fence_after();
  const uint32_t tmem = s->tmem_base;
  MmSchedule<FORM, CG, BN> schedule(p, s);
  const int total = FORM == kOuter ? p.n_groups * schedule.m_tiles * schedule.n_tiles
                    : FORM == kHead ? schedule.m_tiles * schedule.n_tiles
                                    : s->before[p.n_groups] * schedule.m_tiles;

  if (warp == 4) {
    // ------------------------------------------------------------------------------------------------------ copies
    uint32_t slot = 0, phase = 0, issued = 0;
    bool alive = true;
    for (int t = unit; t < total && alive; t += n_units) {
      const MmTile tile = schedule.get(t);
      if (tile.kblocks == 0) continue;
      const int width = mm_width<CG>(tile.ncols), half = width / CG;
      const int m0 = tile.m0 + (int)rank * 128;
      constexpr int kIdx = (FORM == kHead ? 1 : (kHalf + 127) / 128);
      int rows_at[kIdx][4];
      uint32_t bytes;
      bool gathered = false;
      if constexpr (FORM == kHead) {
        bytes = kMmA + kB;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = m0 + 4 * lane + i;
          rows_at[0][i] = r < tile.rows ? mm_source(p.a_index, 1, r, p.a_rows, p.dev_status) : -1;
        }
      } else if constexpr (FORM == kOuter) {
        bytes = kMmA + (uint32_t)((half + 63) / 64) * 8192u;
      } else {
        gathered = p.b_index != nullptr;
        if (gathered) {
          bytes = kMmA + (uint32_t)((half + 3) / 4) * 512u;
#pragma unroll
          for (int j = 0; j < kIdx; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int c = (int)rank * half + 128 * j + 4 * lane + i;
              rows_at[j][i] = c < tile.ncols ? mm_source(p.b_index, p.b_div, tile.n0 + c, p.b_rows, p.dev_status) : -1;
            }
        } else {
          bytes = kMmA + (uint32_t)((half + 31) / 32) * 4096u;
        }
      }
      // (products over rows: lane l looks up rows 4 (l % 16) .. + 3 of a block, one block ahead of the copies)
      int ra[4] = {-1, -1, -1, -1}, rb[4] = {-1, -1, -1, -1};
      auto look_up = [&](int k0) {
        const bool tail = tile.rows - k0 < kMmK;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int q = k0 + 4 * (lane & 15) + i;
          if (p.a_index || tail)
            ra[i] = q < tile.rows ? mm_source(p.a_index, p.a_div, tile.row0 + q, p.a_rows, p.dev_status) : -1;
          if (p.b_index || tail)
            rb[i] = q < tile.rows ? mm_source(p.b_index, p.b_div, tile.row0 + q, p.b_rows, p.dev_status) : -1;
        }
      };
      if constexpr (FORM == kOuter) look_up(0);
      for (int kb = 0; kb < tile.kblocks; ++kb) {
        int ok = 1;
        if (lane == 0) {
          ok = mbar_wait(smem_u32(&s->empty[slot]), phase ^ 1u, abort_flag, p.wait_limit) ? 1 : 0;
          if (ok && rank == 0) mbar_arrive_expect_tx(smem_u32(&s->full[slot]), bytes * CG);
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) { alive = false; break; }
        const uint32_t bar = smem_u32(&s->full[slot]);
        const uint32_t da = smem_u32(ring + (size_t)slot * kStage), db = da + kMmA;
        const int k0 = kb * kMmK;
        if constexpr (FORM == kOuter) {
          // A block of 64 rows of the group; the last one takes its rows one by one, so that the rows behind the
          // group's last come as zeros (in both operands: nothing of another group's, not even a NaN, gets in).
          const bool tail = tile.rows - k0 < kMmK;
          const int x = m0, y = tile.n0 + (int)rank * half, nb = (half + 63) / 64;
          if (!p.a_index && !tail) {
            if (lane < 2) tma2<CG>(da + lane * 8192u, &maps.a, x + 64 * lane, tile.row0 + k0, bar);
          } else {
            const int g = lane & 15, j = lane >> 4;
            tma_gather4<CG>(da + j * 8192u + g * 512u, &maps.ag, x + 64 * j, ra[0], ra[1], ra[2], ra[3], bar);
          }
          if (!p.b_index && !tail) {
            if (lane < nb) tma2<CG>(db + lane * 8192u, &maps.b, y + 64 * lane, tile.row0 + k0, bar);
          } else {
            const int g = lane & 15;
            for (int j = lane >> 4; j < nb; j += 2)
              tma_gather4<CG>(db + j * 8192u + g * 512u, &maps.bg, y + 64 * j, rb[0], rb[1], rb[2], rb[3], bar);
          }
          if (kb + 1 < tile.kblocks) look_up(k0 + kMmK);
        } else {
          if constexpr (FORM == kHead) {
            tma_gather4<CG>(da + lane * 512u, &maps.ag, k0, rows_at[0][0], rows_at[0][1], rows_at[0][2], rows_at[0][3], bar);
            if (lane < kHalf / 128)
              tma2<CG>(db + lane * 16384u, &maps.b, k0, p.column0 + tile.n0 + (int)rank * half + 128 * lane, bar);
          } else {
            if constexpr (FORM == kRows) {
              if (lane == 0) tma3<CG>(da, &maps.a, k0, m0, tile.e, bar);
            } else if constexpr (FORM == kSwiglu) {
              if (lane == 0) tma5<CG>(da, &maps.a, k0, 0, 0, m0 / 16, tile.e, bar);
            } else {
              if (lane < 2) tma3<CG>(da + lane * 8192u, &maps.a, m0 + 64 * lane, k0, tile.e, bar);
            }
            if (gathered) {
#pragma unroll
              for (int j = 0; j < kIdx; ++j)
                if (128 * j + 4 * lane < half)
                  tma_gather4<CG>(db + j * 16384u + lane * 512u, &maps.bg, k0, rows_at[j][0], rows_at[j][1], rows_at[j][2],
                                  rows_at[j][3], bar);
            } else if (32 * lane < half) {
              tma2<CG>(db + lane * 4096u, &maps.b, k0, tile.n0 + (int)rank * half + 32 * lane, bar);
            }
          }
        }
        __syncwarp();
        ++issued;
        if (++slot == STAGES) { slot = 0; phase ^= 1u; }
      }
    }
    if (rank == 0 && lane == 0 && *abort_flag) {
      // something gave up: no copy may still be landing when the shared memory is released
      const uint32_t back = issued < STAGES ? issued : STAGES;
      for (uint32_t k = 1; k <= back; ++k) {
        const uint32_t j = issued - k;
        for (uint32_t spin = 0; spin < DX_WAIT_LIMIT_DEFAULT; ++spin)
          if (mbar_try_wait(smem_u32(&s->full[j % STAGES]), (j / STAGES) & 1u)) break;
      }
    }
  } else if (warp == 5) {
    // ---------------------------------------------------------------------------------------------------- products
    if (rank == 0 && lane == 0) {
      uint32_t slot = 0, phase = 0;
      int turn = 0;
      bool alive = true;
      for (int t = unit; t < total && alive; t += n_units) {
        const MmTile tile = schedule.get(t);
        if (tile.kblocks == 0) continue;
        const uint32_t idesc = mm_idesc(A_MN, B_MN, 128 * CG, mm_width<CG>(tile.ncols));
        const int buf = turn & 1;
        if (!mbar_wait(smem_u32(&s->acc_empty[buf]), (uint32_t)((turn >> 1) & 1) ^ 1u, abort_flag, p.wait_limit)) break;
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)buf * kAccCols;
        for (int kb = 0; kb < tile.kblocks; ++kb) {
          if (!mbar_wait(smem_u32(&s->full[slot]), phase, abort_flag, p.wait_limit)) { alive = false; break; }
          tc_fence_after();
          const uint32_t at = smem_u32(ring + (size_t)slot * kStage);
          const uint64_t a = mm_desc(at, A_MN), b = mm_desc(at + kMmA, B_MN);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            mm_mma<CG>(d, a + (uint64_t)(i * (A_MN ? 128 : 2)), b + (uint64_t)(i * (B_MN ? 128 : 2)), idesc,
                       (kb | i) != 0 ? 1u : 0u);
          mm_commit<CG>(smem_u32(&s->empty[slot]));
          if (++slot == STAGES) { slot = 0; phase ^= 1u; }
        }
        if (!alive) break;
        mm_commit<CG>(smem_u32(&s->acc_full[buf]));
        ++turn;
      }
      if (*abort_flag) {
        mm_commit<CG>(smem_u32(&s->drained));
        for (uint32_t spin = 0; spin < DX_WAIT_LIMIT_DEFAULT; ++spin)
          if (mbar_try_wait(smem_u32(&s->drained), 0)) break;
      }
    }
  } else {
    // ---------------------------------------------------------------------------------------------- finished tiles
    Epilogue epi(p, lane);
    int turn = 0;
    for (int t = unit; t < total; t += n_units) {
      const MmTile tile = schedule.get(t);
      const int lane0 = tile.m0 + (int)rank * 128 + 32 * warp;      // index of the warp's first lane
      epi.begin(tile, lane0, (int)rank * 4 + warp);
      if (tile.kblocks == 0) {                                       // (an empty group's product over its rows)
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = 0.0f;
        for (int c = 0; c < tile.ncols; c += 32) epi.chunk(tile, lane0, c, v);
        continue;
      }
      const int buf = turn & 1;
      if (!mm_store_wait(smem_u32(&s->acc_full[buf]), (uint32_t)(turn >> 1) & 1u, abort_flag, p.wait_limit, lane)) break;
      tc_fence_after();
      const uint32_t base = tmem + ((uint32_t)(32 * warp) << 16) + (uint32_t)buf * kAccCols;
      for (int c = 0; c < tile.ncols; c += 32) {
        float v[32];
        mm_ld32(base + (uint32_t)c, v);
        if (c + 32 >= tile.ncols) {     // the accumulator may be written again
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if constexpr (CG == 2) arrive_at_first(smem_u32(&s->acc_empty[buf]));
            else mbar_arrive(smem_u32(&s->acc_empty[buf]));
          }
        }
        epi.chunk(tile, lane0, c, v);
      }
      epi.end(tile, lane0, t);
      ++turn;
    }
  }
  __syncwarp();
  tc_fence_before();
  if constexpr (CG == 2) pair_sync();
  else __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.dev_status, (int32_t)DX_DEV_WAIT_EXPIRED);
  if (warp == 5) mm_tmem_free<CG>(tmem, kTmemCols);
}

template <int CG, int BN, int STAGES>
constexpr size_t mm_smem() {
  constexpr int half = BN / CG < 32 ? 32 : BN / CG;
  return 1024 + (size_t)STAGES * (kMmA + half * kMmK * 2) + sizeof(MmShared);
}

// ---- host ----------------------------------------------------------------------------------------------------------
template <int FORM, int CG, int BN, int STAGES, class Epilogue>
cudaError_t mm_launch(dx_ctx* ctx, const MmMaps& maps, const MmParams& p, long long max_tiles, cudaStream_t st) {
  auto kernel = dx_mm_kernel<FORM, CG, BN, STAGES, Epilogue>;
  constexpr size_t smem = mm_smem<CG, BN, STAGES>();
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  long long units = ctx->sm_count / CG;
  if (max_tiles < units) units = max_tiles;
  if (units < 1) units = 1;
  return dx_launch_pdl(false, kernel, dim3((unsigned)(units * CG)), dim3(kMmThreads), smem, st, CG, maps, p);
}

}  // namespace

// Tensor map of a bf16 matrix (or stack of them) with rows of `box[0]` = 64 elements in the 128-byte swizzle; dims / strides
// in elements, strides[i] of dimension i + 1.  Returns false where the driver refuses it.
bool dx_tensor_map(CUtensorMap* out, const void* base, int rank, const uint64_t* dims, const uint64_t* strides,
                   const uint32_t* box);
// ... of [rows][cols], boxes of 64 columns by box_rows rows (1: for gathered rows)
bool dx_matrix_map(CUtensorMap* out, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows);
