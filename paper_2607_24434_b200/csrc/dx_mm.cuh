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
// that transposed weights and products over the rows themselves need no transposed copy.  Rows gathered by index come in
// 16-byte pieces (cp.async) from four to six warps of their own, which write the same swizzle; an index outside the matrix reads
// zeros.  (Tensor-map copies of four gathered rows took 85 to 120 clocks each, whoever issued them: 2.8 to 3.8 ms where rows
// in place take 1.0 ms, 98304 rows x 2048 x 2816.)
//
// Warps: 0-7 take finished tiles out of tensor memory (lanes 32 (w % 4) .. + 31, every other chunk of columns), 8 asks for A and
// 10 for B (one of them where only one operand comes by tensor map), 9 owns the tensor memory and issues the products (in a pair
// only the first CTA's), those from 12 on gather.  Two accumulators take turns, so a tile is stored while the next one is
// multiplied; of a contraction longer than a section (below) one takes the sections and the other holds their sum.
//
// Every wait is bounded; one that runs out raises the CTA's abort flag, after which nothing more is copied or multiplied.  When
// all warps of the CTA have come to their ends, copies and products in flight are waited for (bounded; a warp that issued its
// last ones may have been done long before another one gave up), tensor memory is freed and DX_DEV_WAIT_EXPIRED stands in the
// status word.
#pragma once

#include <cuda.h>

#include "dx_internal.cuh"
#include "dx_stream.cuh"

namespace {

constexpr int kMmStoring = 8;               // storing warps: two for each quarter of the tile's lanes, which share its columns
enum { kWarpA = 8, kWarpMma = 9, kWarpB = 10, kWarpGather = 12 };
__host__ __device__ constexpr int mm_threads(int gathering) { return gathering ? 32 * (kWarpGather + gathering) : 352; }
constexpr int kMmK = 64;                    // contraction elements of a stage: 128 bytes of a row
constexpr int kMmA = 128 * kMmK * 2;        // bytes of a CTA's 128 rows of A in a stage
constexpr int kMmMaxStages = 8;
constexpr uint32_t kDrainPolls = 1u << 16;  // of a barrier that may never complete, after something gave up
constexpr int kDealt = 4;                   // (a panel's)
// rows per group up to which tiles have 64 columns, and, products with transposed matrices, 64 and 128
constexpr int kFewestRows = 8, kFewRows = 32, kSomeRows = 96;
constexpr int kPanel = 256;                 // columns of a panel: a tile's, so that a tile's rows lie close together
// The tensor cores' additions to an accumulator truncate, so what is lost grows with their number: of one group's fp32 weight
// gradient 7e-7 of its rms after 768 rows, 4e-6 after 4096, 1e-4 after 98304, 1.2e-3 after 2^20 (operands of one sign: 5e-7,
// 7e-6, 6e-4, 7e-3).  So a long contraction goes in sections, each from zero, which the storing warps add up in fp32, rounded to
// nearest: 4e-6 (7e-6) from 4096 rows on.  Blocks of kMmK of a section: 4096 terms where the result leaves in fp32; where it is
// rounded to bf16, 32768, which lose a tenth of that rounding's half step.  A section's end costs the tensor core the time of the
// addition, some 1700 clocks beside the 33000 that 64 blocks of a pair take: fp32 gradient of 2816 x 2048 over 98304 rows in one
// group 1025 -> 1070 us, in eight 805 -> 808; products of 4096 x 4096 x 16384 396 -> 419 us.
constexpr int kSectionFp32 = 64, kSectionBf16 = 512;

// ---- PTX ---------------------------------------------------------------------------------------------------------
// In a pair, every copy reports to the FIRST CTA's barrier: its address is the local one with the CTA bit cleared.
constexpr uint32_t kFirstCta = 0xFEFFFFFFu;

template <int CG>
__device__ __forceinline__ void tma2(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar & kFirstCta) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tma3(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar & kFirstCta) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tma5(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int u, int v, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(u), "r"(v), "r"(bar & kFirstCta) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(u), "r"(v), "r"(bar) : "memory");
}
// 16 bytes, or (bytes = 0) zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// boxes of shared memory to a matrix (what lies outside it is left out), by one lane; the copies of a group are waited for
// together
__device__ __forceinline__ void tma_store2(const CUtensorMap* map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y),
               "r"(src) : "memory");
}
__device__ __forceinline__ void tma_store3(const CUtensorMap* map, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y),
               "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// ... have read their shared memory
__device__ __forceinline__ void tma_store_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
// ... are done
__device__ __forceinline__ void tma_store_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Shared-memory matrix descriptors, 128-byte swizzle (bits 61..63 = 2), descriptor version 1 (bit 46).
// K-major: groups of eight rows are 1024 bytes apart (sbo); a step of 16 contraction elements is 32 bytes further.
// MN-major: boxes of 64 lanes (columns) x 64 contraction rows of 128 bytes; eight contraction rows are 1024 bytes apart
// (sbo), the next 64 lanes 8192 (lbo); a step of 16 contraction rows is 2048 bytes further.
// (As two words: only the low one changes from product to product.)
__device__ __forceinline__ uint32_t mm_desc_lo(uint32_t addr, bool mn_major) {
  return ((addr & 0x3FFFFu) >> 4) | ((mn_major ? 8192u >> 4 : 1u) << 16);
}
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
// fp32 accumulators, bf16 operands, the operands' majors, columns / 8, lanes / 16
__host__ __device__ constexpr uint32_t mm_idesc(bool a_mn, bool b_mn, int lanes, int columns) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(columns >> 3) << 17) | ((uint32_t)(lanes >> 4) << 24);
}
template <int CG>
__device__ __forceinline__ void mm_mma(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CG == 2)
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHi) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHi) : "memory");
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
// 32 lanes x 16 columns, a lane per thread
__device__ __forceinline__ void mm_ld16(uint32_t taddr, float (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
        "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void mm_st16(uint32_t taddr, const float (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"f"(r[0]),
      "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "f"(r[8]), "f"(r[9]), "f"(r[10]), "f"(r[11]),
      "f"(r[12]), "f"(r[13]), "f"(r[14]), "f"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void mm_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
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
// 32 lanes x 32 (16) columns in the fragments of an 8 x 8 matrix load: thread t holds, for the 16 lanes from 16 h and the
// eight columns from 8 n, v[h][4 n + {0, 1}] = lane t / 4, columns 2 (t % 4) + {0, 1} and v[h][4 n + {2, 3}] = lane 8 + t / 4.
template <int COLS>
struct Fragments {
  float v[2][COLS / 2];
};
// (asked for here; the values are there after mm_ld_wait, which therefore names them)
__device__ __forceinline__ void mm_ld_frag(uint32_t taddr, Fragments<32>& x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float(&r)[16] = x.v[h];
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
          "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
        : "r"(taddr + (uint32_t)h * (16u << 16)));
  }
}
__device__ __forceinline__ void mm_ld_frag(uint32_t taddr, Fragments<16>& x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float(&r)[8] = x.v[h];
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
                 : "r"(taddr + (uint32_t)h * (16u << 16)));
  }
}
template <int N>
__device__ __forceinline__ void mm_ld_wait(float (&a)[N], float (&b)[N]) {
  if constexpr (N == 16)
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(a[0]), "+f"(a[1]), "+f"(a[2]), "+f"(a[3]), "+f"(a[4]), "+f"(a[5]), "+f"(a[6]), "+f"(a[7]), "+f"(a[8]),
                   "+f"(a[9]), "+f"(a[10]), "+f"(a[11]), "+f"(a[12]), "+f"(a[13]), "+f"(a[14]), "+f"(a[15]), "+f"(b[0]),
                   "+f"(b[1]), "+f"(b[2]), "+f"(b[3]), "+f"(b[4]), "+f"(b[5]), "+f"(b[6]), "+f"(b[7]), "+f"(b[8]), "+f"(b[9]),
                   "+f"(b[10]), "+f"(b[11]), "+f"(b[12]), "+f"(b[13])
                 :
                 : "memory");
  else
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(a[0]), "+f"(a[1]), "+f"(a[2]), "+f"(a[3]), "+f"(a[4]), "+f"(a[5]), "+f"(a[6]), "+f"(a[7]), "+f"(b[0]),
                   "+f"(b[1]), "+f"(b[2]), "+f"(b[3]), "+f"(b[4]), "+f"(b[5]), "+f"(b[6]), "+f"(b[7])
                 :
                 : "memory");
  // (an asm statement takes thirty operands: the last two of 32 follow the others through one more)
  if constexpr (N == 16) asm volatile("" : "+f"(b[14]), "+f"(b[15]), "+f"(a[0]) : : "memory");
}
__device__ __forceinline__ void mm_ld_wait(float (&a)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(a[0]), "+f"(a[1]), "+f"(a[2]), "+f"(a[3]), "+f"(a[4]), "+f"(a[5]), "+f"(a[6]), "+f"(a[7]), "+f"(a[8]),
                 "+f"(a[9]), "+f"(a[10]), "+f"(a[11]), "+f"(a[12]), "+f"(a[13]), "+f"(a[14]), "+f"(a[15])
               :
               : "memory");
}
// four 8 x 8 matrices of 16-bit elements, transposed: lanes 8 j .. 8 j + 7 name the rows of matrix j
__device__ __forceinline__ void stmatrix_t(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d)
               : "memory");
}
__device__ __forceinline__ void ldmatrix_t(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts16(uint32_t at, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void sts4(uint32_t at, float v) {
  asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.4426950408889634f;
// 1 / (1 + exp(-x)): good to a few 2^-22 of itself (the argument's rounding adds 2^-24 |x|), 0 below -87
__device__ __forceinline__ float sigmoid(float x) { return rcp(1.0f + ex2(-kLog2e * x)); }
// two fp32 operations in one instruction
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float x, float y) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void f2_get(F2 a, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(a)); }
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint32_t bf16_pair(F2 a) {
  float x, y;
  f2_get(a, x, y);
  const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&b);
}
__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {   // rounded to nearest even
  const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&b);
}
__device__ __forceinline__ float2 bf16_unpair(uint32_t u) {
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// One lane of a warp that goes through a loop together: what it computes stays in uniform registers, where copies and products
// take their operands from.  (With one lane in a branch of its own, every operand is moved there again for every instruction:
// 100 to 150 clocks for a copy, 400 for the four products of a stage.)
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a wait for what both CTAs of a pair have written
__device__ __forceinline__ bool pair_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t limit) {
  for (uint32_t it = 0; it <= limit; ++it) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
    if ((it & 63u) == 63u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
// Arrive at the first CTA's barrier of this offset.  What is handed on lies in this CTA's shared or tensor memory and is read
// by its own SM's tensor core, so the default release at CTA scope orders it; a release at cluster scope costs a memory barrier
// of its own for every stage (stages then took 2600 clocks instead of 700).
__device__ __forceinline__ void arrive_at_first(uint32_t bar) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, 0;\n\t"
               "mbarrier.arrive.shared::cluster.b64 _, [a];\n\t}" ::"r"(bar) : "memory");
}
// A whole warp's wait: all lanes go on or none (those behind a lane that gave up would wait for it at their next exchange).
template <bool PAIR = false>
__device__ __forceinline__ bool mm_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t limit) {
  const bool mine = PAIR ? pair_wait(bar, parity, abort_flag, limit) : mbar_wait(bar, parity, abort_flag, limit);
  return __all_sync(0xffffffffu, mine) != 0;
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
  CUtensorMap b_few;      // of fewer rows
  CUtensorMap out[3];     // outputs that go out in boxes
  CUtensorMap in;         // (SwiGLU gradient) gate and up
};
// Division of 0 <= q < 2^31 by a constant d of the launch: q factor >> shift with shift = 31 + ceil(log2 d) and
// factor = ceil(2^shift / d) < 2^32 (exact: factor d - 2^shift < d <= 2^(shift - 31), so the error stays below 1 / d).
// d = 1: factor 0.
struct MmDiv {
  uint32_t factor, shift;
};
inline MmDiv mm_div(int d) {
  if (d <= 1) return {0u, 0u};
  uint32_t s = 0;
  while ((1u << s) < (uint32_t)d) ++s;
  return {(uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d), 31 + s};
}
struct MmParams {
  int n_groups, n_rows;          // groups; rows of the sorted order (offsets lie in 0 .. n_rows)
  int lanes, columns, kdim;      // extents of D's lanes and columns and of the contraction, where they are not rows
  const void *a_src, *b_src;     // matrices that rows are gathered from (bf16), their rows and pitches; an index outside
  int a_rows, b_rows;            // reads zeros
  int64_t a_ld, b_ld;
  const int32_t* offsets;        // [n_groups + 1]
  const int32_t* a_index;        // sorted row -> index / a_div = row of A's matrix (null: the row itself)
  const int32_t* b_index;        // ... / b_div = row of B's (null: the row itself; rows as columns: row / b_div)
  MmDiv a_div, b_div;
  // output: element (row of column n, lane m) at out + row * ld + m
  void* out;
  int64_t ld;
  const int32_t* scatter;        // sorted row -> row of out (null: itself)
  int out_rows;
  const float* addend;           // fp32, added to the products, laid out like out
  // SwiGLU
  void* save;                    // [n_rows, 2 I] gate and up products
  int64_t ld_save;
  const float* pair_w;           // weight of pair q
  int n_pairs;
  void* act_w;
  int64_t ld_act;
  float* partial;                // [warps of lanes][n_rows] shares of the pair weights' gradients
  // Groups of *n_live rows each, group_rows apart, instead of offsets, that share out one product's contraction: kDealt blocks of
  // kMmK rows of the one matrix in turns, from its end (which was read last) to its beginning.  The rows' elements stand in
  // panels of kPanel columns, one below the other, group_rows rows each.
  const int32_t* n_live;         // (loss) rows that count
  int group_rows;
  int shared_out;                // blocks of kMmK rows of the matrix (0: a matrix per group)
  int b_panel;                   // (products over rows) rows of a panel of B (0: no panels)
  // loss
  float* logits;                 // [n_live][ld_logits], kept where that is little
  int64_t ld_logits;
  int panel;                     // rows of a panel of dz
  const int32_t* live;           // the rows that count
  const int32_t* targets;        // [..] by original row
  const float* row_weight;
  float2* part;                  // (maximum, sum) of halves of column tiles
  int64_t part_half, part_row;   // from one half, one row to the next
  float* target_logit;           // [n_live]
  const float* lse;              // [n_live]
  const float* row_loss;         // [n_live]
  int column0;                   // first column's word
  int tile_width;                // columns of a tile (0: BN)
  uint32_t a_box;                // rows of a copy of A
  int section;                   // blocks of the contraction that one accumulator takes
  int32_t* dev_status;
  uint32_t wait_limit;
};

// Which operand comes from where
enum MmForm {
  kRows,      // lanes: rows of W_e (K-major); columns: sorted rows (K-major, gathered or not)
  kRowsT,     // lanes: columns of W_e (MN-major); columns: sorted rows
  kSwiglu,    // as kRows, the lanes eight gate rows and eight up rows in turns
  kOuter,     // lanes, columns: columns of two matrices of rows (both MN-major); the contraction goes over a group's rows
  kHead       // lanes: rows (K-major); columns: rows of W
};
__host__ __device__ constexpr bool mm_a_mn(int form) { return form == kRowsT || form == kOuter; }
__host__ __device__ constexpr bool mm_b_mn(int form) { return form == kOuter; }
// both operands (may) come by tensor map: a warp for each
__host__ __device__ constexpr bool mm_two_copiers(int form, bool gather) { return form == kOuter || !gather; }

struct __align__(16) MmShared {
  unsigned long long full[kMmMaxStages];
  unsigned long long empty[kMmMaxStages];
  unsigned long long acc_full[2], acc_empty[2], drained;
  unsigned long long fetched[kMmStoring][2];   // what a storing warp reads beside the accumulators
  uint32_t tmem_base;
  int abort_flag;
  int off[DX_MAX_E], cnt[DX_MAX_E];      // a group's first row, its rows
  int before[DX_MAX_E + 1];      // row tiles in front of a group
};

struct MmTile {
  int e;          // group
  int m0;         // first lane's index (of the tile, not of the CTA)
  int n0;         // first column's index; for rows as columns: the sorted row
  int ncols;      // columns that exist
  int row0, rows; // (contraction over rows) the group's rows; (kHead) number of the column tile, rows that count
  int kblocks;
  __device__ __forceinline__ MmTile uniform_copy() const {
    return {uniform(e), uniform(m0), uniform(n0), uniform(ncols), uniform(row0), uniform(rows), uniform(kblocks)};
  }
};

template <int FORM, int CG, int BN>
struct MmSchedule {
  const MmParams& p;
  const MmShared* s;
  int m_tiles, n_tiles, width, e;
  __device__ MmSchedule(const MmParams& p_, const MmShared* s_) : p(p_), s(s_), e(0) {
    const int lanes = FORM == kHead ? s->cnt[0] : p.lanes;
    m_tiles = (lanes + 128 * CG - 1) / (128 * CG);
    width = FORM == kHead && p.tile_width ? p.tile_width : BN;
    n_tiles = (p.columns + width - 1) / width;
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
      r.n0 = nt * width;
      r.ncols = min(width, p.columns - r.n0);
      r.row0 = nt;
      r.rows = s->cnt[0];
      r.kblocks = (p.kdim + kMmK - 1) / kMmK;
    } else {
      const int nt = t / m_tiles;
      int last = p.n_groups - 1;                      // (the last group that begins at or before tile nt)
      while (e < last) {
        const int mid = (e + last + 1) >> 1;
        if (s->before[mid] <= nt) e = mid;
        else last = mid - 1;
      }
      r.e = e;
      r.m0 = (t - nt * m_tiles) * 128 * CG;
      // a group's rows are split evenly over its tiles
      const int cnt = s->cnt[e], k = s->before[e + 1] - s->before[e], j = nt - s->before[e];
      const int each = (cnt + k - 1) / k, width = (each + 16 * CG - 1) / (16 * CG) * (16 * CG);
      r.n0 = s->off[e] + j * width;
      r.ncols = min(width, cnt - j * width);
      r.row0 = r.n0;
      r.rows = r.ncols;
      if (p.shared_out) {
        const int turn = kDealt * p.n_groups, turns = p.shared_out / turn;
        r.kblocks = turns * kDealt + min(max(p.shared_out - turns * turn - kDealt * e, 0), kDealt);
      } else {
        r.kblocks = (p.kdim + kMmK - 1) / kMmK;
      }
    }
    return r;
  }
};
// barriers of a storing warp's own fetches, and what bounds its waits
struct MmFetch {
  uint32_t bar;
  volatile int* abort_flag;
  uint32_t limit;
};
// columns of the products of a tile
template <int CG>
__device__ __forceinline__ int mm_width(int ncols) { return (ncols + 16 * CG - 1) / (16 * CG) * (16 * CG); }

// Row of the matrix that an index (a pair, say) stands for; -1, which reads zeros, where it points outside.  Kept apart from the
// load of the index: several loads are to be in flight before the first is looked at.
__device__ __forceinline__ int mm_row(int q, MmDiv div, int n_rows, int32_t* dev_status) {
  const int row = q < 0 ? -1 : div.factor == 0u ? q : (int)((uint64_t)(uint32_t)q * div.factor >> div.shift);
  if (row >= 0 && row < n_rows) return row;
  atomicExch(dev_status, (int32_t)DX_DEV_BAD_ROW);
  return -1;
}

// LONG: some tile's contraction may go in sections
template <int FORM, bool GATHER, int CG, int BN, int STAGES, class Epilogue, bool LONG>
__global__ void __launch_bounds__(mm_threads(GATHER ? Epilogue::kGathering : 0), 1)
dx_mm_kernel(const __grid_constant__ MmMaps maps, const __grid_constant__ MmParams p) {
  constexpr int kHalf = BN / CG;                       // columns whose rows a CTA fetches
  constexpr int kB = (kHalf < 32 ? 32 : kHalf) * kMmK * 2;
  constexpr int kStage = kMmA + kB;
  constexpr bool A_MN = mm_a_mn(FORM), B_MN = mm_b_mn(FORM), kTwo = mm_two_copiers(FORM, GATHER);
  constexpr uint32_t kAccCols = BN < 32 ? 32 : BN, kTmemCols = 2 * kAccCols;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char* staging = ring + (size_t)STAGES * kStage;
  MmShared* s = reinterpret_cast<MmShared*>(staging + kMmStoring * Epilogue::kStaging);
  static_assert(Epilogue::kStaging % 512 == 0);

  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cta_rank() : 0u;
  const int unit = blockIdx.x / CG, n_units = gridDim.x / CG;
  volatile int* abort_flag = &s->abort_flag;

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(smem_u32(&s->full[i]), (kTwo ? 2 : 1) + (GATHER ? CG : 0));
      mbar_init(smem_u32(&s->empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&s->acc_full[i]), 1);
      mbar_init(smem_u32(&s->acc_empty[i]), kMmStoring * CG);
    }
    mbar_init(smem_u32(&s->drained), 1);
    for (int i = 0; i < 2 * kMmStoring; ++i) mbar_init(smem_u32(&s->fetched[i >> 1][i & 1]), 1);
    s->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_map(&maps.a);
    if (!GATHER || FORM == kOuter) tma_prefetch_map(&maps.b);
  }
  if (warp == kWarpMma) mm_tmem_alloc<CG>(smem_u32(&s->tmem_base), kTmemCols);
  dx_pdl_wait();
  dx_pdl_trigger();      // (what follows may take its place on the SMs as they become free; it waits for this grid to end)
  // the groups: rows outside [0, n_rows) and ends in front of their beginnings are cut off and reported
  if (warp == 0) {
    int run = 0;
    for (int e0 = 0; e0 < p.n_groups; e0 += 32) {
      const int e = e0 + lane;
      int lo = 0, hi = 0;
      if (e < p.n_groups) {
        if (FORM == kHead) {
          hi = __ldg(p.n_live);
        } else if (p.n_live) {
          lo = e * p.group_rows;
          hi = lo + __ldg(p.n_live);
        } else {
          lo = __ldg(p.offsets + e);
          hi = __ldg(p.offsets + e + 1);
        }
        const int a = min(max(lo, 0), p.n_rows), b = min(max(hi, a), p.n_rows);
        if (a != lo || b != hi) atomicExch(p.dev_status, (int32_t)DX_DEV_BAD_OFFSETS);
        lo = a;
        hi = b;
        if (DX_BOUNDS(e < DX_MAX_E, p.dev_status)) {
          s->off[e] = lo;
          s->cnt[e] = hi - lo;
        }
      }
      int tiles = (hi - lo + BN - 1) / BN, sum = tiles;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += o;
      }
      if (e < p.n_groups && DX_BOUNDS(e < DX_MAX_E, p.dev_status)) s->before[e] = run + sum - tiles;
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
  uint32_t issued = 0;      // (copying warps) stages asked for

  if (warp == kWarpA || (kTwo && warp == kWarpB)) {
    // ------------------------------------------------------------------------------------------------------ copies
    // (the one of them where only one operand comes by tensor map)
    const bool for_a = warp == kWarpA, for_b = warp == kWarpB;
    uint32_t slot = 0, phase = 0;
    bool alive = true;
    auto shared_row = [&](int e, int kb) {
      return (p.shared_out - 1 - (kb / kDealt * p.n_groups + e) * kDealt - kb % kDealt) * kMmK;
    };
    for (int t = unit; t < total && alive; t += n_units) {
      const MmTile tile = schedule.get(t).uniform_copy();
      const int half = mm_width<CG>(tile.ncols) / CG, m0 = tile.m0 + (int)rank * 128;
      const int n0 = tile.n0 + (int)rank * half;
      // rows as columns: copies of 128 rows, or of 32 where those would bring twice what is needed
      const bool big = FORM == kHead || (kHalf >= 128 && half > 64);
      const int nb = FORM == kOuter ? (half + 63) / 64
                     : FORM == kHead ? kHalf / 128 : big ? (half + 127) / 128 : (half + 31) / 32;
      const uint32_t box = FORM == kOuter ? 8192u : big ? 16384u : 4096u;   // bytes of a copy of B
      for (int kb = 0; kb < tile.kblocks; ++kb) {
        const int k0 = kb * kMmK;
        // Products over rows: a group's last block, where it is not full, is gathered with zeros behind the last row (in
        // both operands: nothing of another group's rows, not even a NaN, gets in).
        const bool tail = FORM == kOuter && tile.rows - k0 < kMmK;
        const bool here = FORM != kOuter || (!tail && !(for_a ? p.a_index : p.b_index));
        if (!mm_wait(smem_u32(&s->empty[slot]), phase ^ 1u, abort_flag, p.wait_limit)) { alive = false; break; }
        const uint32_t bar = smem_u32(&s->full[slot]);
        const uint32_t da = smem_u32(ring + (size_t)slot * kStage), db = da + kMmA;
        if (elect_one()) {
          const uint32_t bytes = for_a ? (FORM == kHead ? p.a_box * 128u : (uint32_t)kMmA) : nb * box;
          if (rank == 0) mbar_arrive_expect_tx(bar, here ? bytes * CG : 0u);
          if (here && for_a) {
            if constexpr (FORM == kRows) {
              tma3<CG>(da, &maps.a, k0, m0, tile.e, bar);
            } else if constexpr (FORM == kSwiglu) {
              tma5<CG>(da, &maps.a, k0, 0, 0, m0 / 16, tile.e, bar);
            } else if constexpr (FORM == kRowsT) {
              const int y = p.shared_out ? shared_row(tile.e, kb) : k0, z = p.shared_out ? 0 : tile.e;
              tma3<CG>(da, &maps.a, m0, y, z, bar);
              tma3<CG>(da + 8192u, &maps.a, m0 + 64, y, z, bar);
            } else if constexpr (FORM == kOuter) {
              tma2<CG>(da, &maps.a, m0, tile.row0 + k0, bar);
              tma2<CG>(da + 8192u, &maps.a, m0 + 64, tile.row0 + k0, bar);
            } else {
              tma2<CG>(da, &maps.a, k0, m0, bar);
            }
          }
          if (here && for_b) {
            if constexpr (FORM == kOuter) {
              const int x = p.b_panel ? n0 % kPanel : n0, y = p.b_panel ? n0 / kPanel * p.b_panel : 0;
              for (int j = 0; j < nb; ++j) tma2<CG>(db + j * 8192u, &maps.b, x + 64 * j, y + tile.row0 + k0, bar);
            } else if constexpr (FORM == kHead) {
#pragma unroll
              for (int j = 0; j < kHalf / 128; ++j) tma2<CG>(db + j * 16384u, &maps.b, k0, p.column0 + n0 + 128 * j, bar);
            } else {
              int x = k0, y = n0;
              if (FORM == kRowsT && p.shared_out) {
                const int at = shared_row(tile.e, kb);
                x = at % kPanel;
                y += (at / kPanel - tile.e) * p.group_rows;
              }
              if (big) {
                for (int j = 0; j < nb; ++j) tma2<CG>(db + j * 16384u, &maps.b, x, y + 128 * j, bar);
              } else {
                for (int j = 0; j < nb; ++j) tma2<CG>(db + j * 4096u, &maps.b_few, x, y + 32 * j, bar);
              }
            }
          }
        }
        __syncwarp();
        ++issued;
        if (++slot == STAGES) { slot = 0; phase ^= 1u; }
      }
    }
  } else if (GATHER && warp >= kWarpGather) {
    // ----------------------------------------------------------------------------------------------- gathered rows
    // Each of the four or six warps does every fourth or sixth stage by itself: its fixed costs (waiting for the slot, for the
    // pieces to land, making them visible to the tensor core) are spread over the time of as many stages.  A stage takes a warp
    // some 2800 clocks, most of them to issue the copies, and its products 512: with four warps they wait for it.  Eight lanes
    // bring 128 bytes of a row, the warp four rows at a time: row 4 i + lane / 8; lane l looks up rows l, l + 32, ...
    // (A warp asks for a slot when it has filled the one kGathering stages in front.  That one's own slot was empty then, so no
    // slot is more than one turn behind what is asked of it: its barrier's phase tells turns apart.)
    constexpr uint32_t kGathering = Epilogue::kGathering;
    static_assert(kGathering <= STAGES);
    const int g = warp - kWarpGather, sub = lane >> 3, piece = lane & 7;
    // where row 4 i + sub's piece goes: rows of one i parity share their place in the swizzle
    const uint32_t place[2] = {(uint32_t)(sub * 128 + ((piece ^ sub) << 4)), (uint32_t)(sub * 128 + ((piece ^ (4 + sub)) << 4))};
    // (what a copy of no bytes names as its source)
    const unsigned char* zeros = reinterpret_cast<const unsigned char*>(p.b_src);
    uint32_t base = 0;              // stages in front of the tile
    bool alive = true;
    for (int t = unit; t < total && alive; t += n_units) {
      const MmTile tile = schedule.get(t).uniform_copy();
      const int half = mm_width<CG>(tile.ncols) / CG, m0 = tile.m0 + (int)rank * 128;
      const int n0 = tile.n0 + (int)rank * half;
      constexpr int kRegs = FORM == kOuter ? 2 : (kHalf + 31) / 32;
      const int here = min(half, tile.ncols - (int)rank * half);      // rows as columns
      // what this lane has looked up: a row's place in its matrix, in pieces of 16 bytes, and which lanes' rows exist
      uint32_t at_a[2], at_b[kRegs], ok_a[2], ok_b[kRegs];
      auto resolve = [&](int q, bool in, bool indexed, MmDiv div, int n_rows, int64_t ld, uint32_t& at, uint32_t& ok) {
        int row = !in ? -1 : indexed ? mm_row(q, div, n_rows, p.dev_status) : q;
        if (in && !indexed && !DX_BOUNDS(q >= 0 && q < n_rows, p.dev_status)) row = -1;
        at = (uint32_t)max(row, 0) * (uint32_t)(ld >> 3);
        ok = __ballot_sync(0xffffffffu, row >= 0);
      };
      // eight copies of four rows each: first where they come from, then the copies (one after the other they would wait for
      // their own address every time)
      auto copy_rows = [&](uint32_t dst, const unsigned char* from, uint32_t at, uint32_t ok, bool in, uint32_t offset) {
        uint32_t src[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) src[i] = __shfl_sync(0xffffffffu, at, 4 * i + sub);
        if (ok == 0xffffffffu && in) {
#pragma unroll
          for (int i = 0; i < 8; ++i) copy16(dst + place[i & 1] + i * 512u, from + (uint64_t)src[i] * 16u + offset, 16u);
        } else {
          const uint32_t mine = in ? ok >> sub : 0u;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            copy16(dst + place[i & 1] + i * 512u, (mine >> (4 * i)) & 1u ? from + (uint64_t)src[i] * 16u + offset : zeros,
                   ((mine >> (4 * i)) & 1u) * 16u);
        }
      };
      if constexpr (FORM != kOuter) {
        int q[kRegs];
#pragma unroll
        for (int j = 0; j < kRegs; ++j)
          q[j] = 32 * j + lane >= here || !DX_BOUNDS(n0 >= 0 && n0 + 32 * j + lane < p.n_rows, p.dev_status) ? 0
                 : p.b_index ? __ldg(p.b_index + n0 + 32 * j + lane) : n0 + 32 * j + lane;
#pragma unroll
        for (int j = 0; j < kRegs; ++j)
          resolve(q[j], 32 * j + lane < here, true, p.b_div, p.b_rows, p.b_ld, at_b[j], ok_b[j]);
      }
      // (products over rows: the rows of the warp's next stage are looked up a turn ahead)
      int next_a[2], next_b[2];
      auto ask = [&](int k0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = k0 + 32 * j + lane;
          const bool in = r < tile.rows && DX_BOUNDS(tile.row0 >= 0 && tile.row0 + r < p.n_rows, p.dev_status);
          next_a[j] = in && p.a_index ? __ldg(p.a_index + tile.row0 + r) : 0;
          next_b[j] = in && p.b_index ? __ldg(p.b_index + tile.row0 + r) : 0;
        }
      };
      const int first = (int)((uint32_t)g + kGathering - base % kGathering) % (int)kGathering;
      if constexpr (FORM == kOuter) ask(first * kMmK);
      for (int kb = first; kb < tile.kblocks; kb += (int)kGathering) {
        const int k0 = kb * kMmK;
        const uint32_t n = base + (uint32_t)kb, slot = n % STAGES, phase = (n / STAGES) & 1u;
        const bool tail = FORM == kOuter && tile.rows - k0 < kMmK;
        const bool do_a = FORM == kOuter && (p.a_index || tail), do_b = FORM == kOuter && (p.b_index || tail);
        if constexpr (FORM == kOuter) {
          if (do_a || do_b) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int r = k0 + 32 * j + lane;
              const bool in = r < tile.rows;
              resolve(p.a_index ? next_a[j] : tile.row0 + r, in, p.a_index != nullptr, p.a_div, p.a_rows, p.a_ld, at_a[j],
                      ok_a[j]);
              resolve(p.b_index ? next_b[j] : tile.row0 + r, in, p.b_index != nullptr, p.b_div, p.b_rows, p.b_ld, at_b[j],
                      ok_b[j]);
            }
            ask(k0 + (int)kGathering * kMmK);
          }
        }
        if (!mm_wait(smem_u32(&s->empty[slot]), phase ^ 1u, abort_flag, p.wait_limit)) { alive = false; break; }
        const uint32_t da = smem_u32(ring + (size_t)slot * kStage), db = da + kMmA;
        if constexpr (FORM == kOuter) {
          // columns x0 + 64 b + 8 piece of a matrix: inside it, or zeros
          if (do_a) {
            const unsigned char* from = reinterpret_cast<const unsigned char*>(p.a_src) + 2 * (int64_t)(m0 + 8 * piece);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              copy_rows(da + j * 4096u, from, at_a[j], ok_a[j],
                        m0 + 8 * piece < p.lanes, 0);
              copy_rows(da + 8192u + j * 4096u, from, at_a[j], ok_a[j],
                        m0 + 64 + 8 * piece < p.lanes, 128);
            }
          }
          if (do_b) {
            const int64_t x = p.b_panel ? (int64_t)(n0 / kPanel) * p.b_panel * kPanel + n0 % kPanel : n0;
            const unsigned char* from = reinterpret_cast<const unsigned char*>(p.b_src) + 2 * (x + 8 * piece);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
              for (int b = 0; b < kHalf / 64; ++b)
                if (64 * b < half)
                  copy_rows(db + b * 8192u + j * 4096u, from, at_b[j], ok_b[j], n0 + 64 * b + 8 * piece < p.columns, 128 * b);
            }
          }
        } else {
          // (rows that do not exist come as zeros; they only ever meet lanes or columns that do not exist either)
          const bool in = k0 + 8 * piece < p.kdim;
          const unsigned char* from = zeros + 2 * (int64_t)(k0 + 8 * piece);
#pragma unroll
          for (int j = 0; j < kRegs; ++j)
            if (32 * j < here) copy_rows(db + j * 4096u, from, at_b[j], ok_b[j], in, 0);
        }
        asm volatile("cp.async.wait_all;\n\tfence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          if constexpr (CG == 2) arrive_at_first(smem_u32(&s->full[slot]));
          else mbar_arrive(smem_u32(&s->full[slot]));
        }
      }
      base += (uint32_t)tile.kblocks;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == kWarpMma) {
    // ---------------------------------------------------------------------------------------------------- products
    if (rank == 0) {
      uint32_t slot = 0, phase = 0;
      int turn = 0;
      uint32_t parity = 0, held = 0;      // (LONG) bit b: of accumulator b's next turn; the accumulator whose turn it is
      bool alive = true;
      const uint32_t ring_a = mm_desc_lo(smem_u32(ring), A_MN), ring_b = mm_desc_lo(smem_u32(ring) + kMmA, B_MN);
      for (int t = unit; t < total && alive; t += n_units) {
        const MmTile tile = schedule.get(t).uniform_copy();
        if (tile.kblocks == 0) continue;
        const uint32_t idesc = mm_idesc(A_MN, B_MN, 128 * CG, mm_width<CG>(tile.ncols));
        const uint32_t buf = LONG ? held : (uint32_t)turn & 1u;
        // (a long contraction's sections take turns on one accumulator; the other one holds their sum)
        auto empty = [&] {
          const uint32_t odd = LONG ? (parity >> buf) & 1u : (uint32_t)(turn >> 1) & 1u;
          if (!mm_wait(smem_u32(&s->acc_empty[buf]), odd ^ 1u, abort_flag, p.wait_limit)) return false;
          tc_fence_after();
          if (LONG) parity ^= 1u << buf;
          return true;
        };
        int begin = 0, end = LONG ? min(p.section, tile.kblocks) : tile.kblocks;
        if (!empty()) break;
        const uint32_t d = tmem + buf * kAccCols;
        for (int kb = 0; kb < tile.kblocks; ++kb) {
          if (LONG && kb == end) {
            if (!empty()) { alive = false; break; }
            begin = end;
            end = min(end + p.section, tile.kblocks);
          }
          if (!mm_wait<CG == 2>(smem_u32(&s->full[slot]), phase, abort_flag, p.wait_limit)) { alive = false; break; }
          // (no tcgen05 fence: the stage was written in, or made visible to, the tensor core's proxy; a fence drains the pipe)
          const uint32_t a = ring_a + slot * (uint32_t)(kStage >> 4), b = ring_b + slot * (uint32_t)(kStage >> 4);
          if (elect_one()) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              mm_mma<CG>(d, a + (uint32_t)(i * (A_MN ? 128 : 2)), b + (uint32_t)(i * (B_MN ? 128 : 2)), idesc,
                         (kb != begin) | (i != 0) ? 1u : 0u);
            mm_commit<CG>(smem_u32(&s->empty[slot]));
            if (kb + 1 == end) mm_commit<CG>(smem_u32(&s->acc_full[buf]));
          }
          __syncwarp();
          if (++slot == STAGES) { slot = 0; phase ^= 1u; }
        }
        if (!alive) break;
        ++turn;
        if constexpr (LONG) {
          // (the accumulator that holds a sum is handed back like one that held products)
          if (tile.kblocks > p.section) parity ^= 2u >> buf;
          else held ^= 1u;
        }
      }
    }
  } else if (warp < kMmStoring) {
    // ---------------------------------------------------------------------------------------------- finished tiles
    constexpr int kCols = Epilogue::kCols;      // columns of a chunk
    const int quarter = warp & 3, share = warp >> 2;
    Epilogue epi(p, maps, lane, share, smem_u32(staging) + (uint32_t)warp * Epilogue::kStaging,
                 MmFetch{smem_u32(&s->fetched[warp][0]), abort_flag, p.wait_limit});
    int turn = 0;
    uint32_t parity = 0, held = 0;              // (LONG) as the products'
    MmTile next = {};
    if (unit < total) next = schedule.get(unit);
    for (int t = unit; t < total; t += n_units) {
      const MmTile tile = next;
      const bool more = t + n_units < total;
      if (more) next = schedule.get(t + n_units);
      const int lane0 = tile.m0 + (int)rank * 128 + 32 * quarter;   // index of the warp's first lane
      // (what everything the epilogues store is placed by)
      if (!DX_BOUNDS(tile.e >= 0 && tile.e < p.n_groups && tile.m0 >= 0 && tile.n0 >= 0 && tile.ncols > 0 && tile.ncols <= BN &&
                         tile.n0 + tile.ncols <= (FORM == kOuter || FORM == kHead ? p.columns : p.n_rows) &&
                         tile.row0 >= 0 && tile.rows >= 0 && (FORM != kOuter || tile.row0 + tile.rows <= p.n_rows),
                     p.dev_status))
        break;
      epi.begin(tile, lane0, kCols * share, next, more);
      typename Epilogue::Values v;
      if (tile.kblocks == 0) {                                       // (an empty group's product over its rows)
        epi.zero(v);
        for (int c = kCols * share; c < tile.ncols && lane0 < p.lanes; c += 2 * kCols) epi.chunk(tile, lane0, c, v, [] {});
        continue;
      }
      const int lanes = FORM == kHead ? tile.rows : p.lanes;
      const int end = lane0 >= lanes ? 0 : (tile.ncols + Epilogue::kRound - 1) / Epilogue::kRound * Epilogue::kRound;
      const uint32_t quarters = tmem + ((uint32_t)(32 * quarter) << 16);
      const uint32_t buf = LONG ? held : (uint32_t)turn & 1u;
      uint32_t from = buf;                     // the accumulator that the tile is taken from
      auto taken = [&]() {                     // it may be written again
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (CG == 2) arrive_at_first(smem_u32(&s->acc_empty[from]));
          else mbar_arrive(smem_u32(&s->acc_empty[from]));
        }
      };
      auto full = [&] {
        const uint32_t odd = LONG ? (parity >> buf) & 1u : (uint32_t)(turn >> 1) & 1u;
        if (!mm_store_wait(smem_u32(&s->acc_full[buf]), odd, abort_flag, p.wait_limit, lane)) return false;
        tc_fence_after();
        if (LONG) parity ^= 1u << buf;
        return true;
      };
      if (!full()) break;
      bool alive = true;
      for (int kb = 0; LONG && tile.kblocks > p.section; kb += p.section) {
        // A section of a long contraction: this warp's part of it is added to its part of the other accumulator.  That one is
        // free of products: its last ones were taken out, by this warp too, before this tile, and it is handed back after it.
        const uint32_t part = quarters + buf * kAccCols, sum = quarters + (buf ^ 1u) * kAccCols;
#pragma unroll 1
        for (int c0 = kCols * share; c0 < end; c0 += 2 * kCols) {
#pragma unroll 1
          for (int i = 0; i < kCols; i += 16) {
            float x[16], y[16];
            mm_ld16(part + (uint32_t)(c0 + i), x);
            if (kb > 0) {
              mm_ld16(sum + (uint32_t)(c0 + i), y);
              mm_ld_wait(x, y);
#pragma unroll
              for (int j = 0; j < 16; ++j) x[j] += y[j];
              mm_st16(sum + (uint32_t)(c0 + i), x);
            } else {
              mm_ld_wait(x);
              mm_st16(sum + (uint32_t)(c0 + i), x);
            }
          }
        }
        mm_st_wait();
        taken();
        if (kb + p.section >= tile.kblocks) {
          from = buf ^ 1u;
          break;
        }
        if (!full()) { alive = false; break; }
      }
      if (!alive) break;
      const uint32_t base = quarters + from * kAccCols;
      int c = kCols * share;
      if (c >= end) {
        taken();
      } else if constexpr (Epilogue::kBefore) {
        // a chunk is on its way out of tensor memory while the one in front of it is stored
        typename Epilogue::Values coming;
        epi.load(base + (uint32_t)c, coming);
        for (; c < end; c += 2 * kCols) {
          epi.arrived(coming);
          v = coming;
          if (c + 2 * kCols < end) epi.load(base + (uint32_t)(c + 2 * kCols), coming);
          else taken();
          epi.chunk(tile, lane0, c, v, [] {});
        }
      } else {
        for (; c < end; c += 2 * kCols) {
          epi.load(base + (uint32_t)c, v);
          epi.chunk(tile, lane0, c, v, [&] { if (c + 2 * kCols >= end) taken(); });
        }
      }
      epi.end(tile);
      ++turn;
      if (LONG && from == buf) held ^= 1u;
    }
    epi.finish();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();          // (nobody of this CTA issues anything more, or gives up)
  if (*abort_flag) {
    // Neither a copy nor a product may be on its way when the shared memory, the tensor memory and in a pair the first CTA's
    // barriers are released.  (The other CTA of a pair waits at pair_sync.  If only that one gave up, all products of this one
    // are done: each of its tiles was stored.)
    if (warp == kWarpMma && rank == 0) {
      if (elect_one()) mm_commit<CG>(smem_u32(&s->drained));      // (by the lane that issued the products)
      __syncwarp();
      for (uint32_t spin = 0; spin < DX_WAIT_LIMIT_DEFAULT; ++spin)
        if (mbar_try_wait(smem_u32(&s->drained), 0)) break;
    } else if (warp == kWarpA || (kTwo && warp == kWarpB)) {
      // Stages that both operands were asked for complete on their barriers; for one that only one operand was asked for, or a
      // box of a storing warp, there is nothing to wait on, so the rest is time, a thousand times what a copy takes.
      if (rank == 0 && warp == kWarpA) {
        const uint32_t back = issued < STAGES ? issued : STAGES;
        for (uint32_t k = 1; k <= back; ++k) {
          const uint32_t j = issued - k;
          for (uint32_t spin = 0; spin < kDrainPolls; ++spin)
            if (mbar_try_wait(smem_u32(&s->full[j % STAGES]), (j / STAGES) & 1u)) break;
        }
      }
      for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    __syncwarp();
  }
  if constexpr (CG == 2) pair_sync();
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(p.dev_status, (int32_t)DX_DEV_WAIT_EXPIRED);
  if (warp == kWarpMma) mm_tmem_free<CG>(tmem, kTmemCols);
}

template <int CG, int BN, int STAGES, class Epilogue>
constexpr size_t mm_smem() {
  constexpr int half = BN / CG < 32 ? 32 : BN / CG;
  return 1024 + (size_t)STAGES * (kMmA + half * kMmK * 2) + (sizeof(MmShared) + 127) / 128 * 128 +
         kMmStoring * Epilogue::kStaging;
}

// ---- host ----------------------------------------------------------------------------------------------------------
template <int FORM, bool GATHER, int CG, int BN, int STAGES, class Epilogue, bool LONG>
cudaError_t mm_launch(dx_ctx* ctx, const MmMaps& maps, const MmParams& p, long long max_tiles, cudaStream_t st) {
  auto kernel = dx_mm_kernel<FORM, GATHER, CG, BN, STAGES, Epilogue, LONG>;
  constexpr size_t smem = mm_smem<CG, BN, STAGES, Epilogue>();
  static_assert(smem <= 227 * 1024);
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  long long units = ctx->sm_count / CG;
  if (max_tiles < units) units = max_tiles;
  if (units < 1) units = 1;
  return dx_launch_pdl((ctx->pdl_mask & DX_PDL_EXPERTS) != 0, kernel, dim3((unsigned)(units * CG)),
                       dim3(mm_threads(GATHER ? Epilogue::kGathering : 0)), smem, st, CG, maps, p);
}
// A kernel of its own for long contractions: in one for both, the code for their sections cost SwiGLU of 98304 gathered rows 5 %
// (867 -> 916 us: registers) and weight gradients of five rows per group as much (47.2 -> 49.5 us).
template <int FORM, bool GATHER, int CG, int BN, int STAGES, class Epilogue>
cudaError_t mm_launch(dx_ctx* ctx, const MmMaps& maps, const MmParams& p, long long max_tiles, cudaStream_t st) {
  const int most = ((FORM == kOuter ? p.n_rows : p.kdim) - 1) / kMmK + 1;      // blocks of a tile's contraction
  return most > p.section ? mm_launch<FORM, GATHER, CG, BN, STAGES, Epilogue, true>(ctx, maps, p, max_tiles, st)
                          : mm_launch<FORM, GATHER, CG, BN, STAGES, Epilogue, false>(ctx, maps, p, max_tiles, st);
}

}  // namespace

// Tensor map of a bf16 matrix (or stack of them) with rows of `box[0]` = 64 elements in the 128-byte swizzle; dims / strides
// in elements, strides[i] of dimension i + 1.  Returns false where the driver refuses it.
bool dx_tensor_map(CUtensorMap* out, const void* base, int rank, const uint64_t* dims, const uint64_t* strides,
                   const uint32_t* box);
// Tensor map for boxes of box[0] x box[1] elements of fp32 or bf16 in the swizzle of box[0]'s bytes (32, 64 or 128).
bool dx_box_map(CUtensorMap* out, const void* base, bool fp32, int rank, const uint64_t* dims, const uint64_t* strides,
                const uint32_t* box);
// ... of [rows][cols], boxes of 64 columns by box_rows rows
bool dx_matrix_map(CUtensorMap* out, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows);
