// Cross entropy of hidden rows against a vocabulary (spec_head_loss): with z = W h, per row
//     loss = log sum_v exp(z_v) - z_target,      dz = weight * (softmax(z) - 1_target),      dh = W^T dz,     dW = dz^T h
// with dz in pieces of the vocabulary, and the logits kept only where that is worth their bytes.
//
//   1. the rows that count (a target, a weight other than 0) are listed in order and copied next to each other: the others cost
//      nothing below, whatever they hold
//   2. products of the listed rows with the whole vocabulary; of every tile a row keeps (maximum, sum of exponentials) and,
//      where the tile holds it, the target's logit
//   3. the tiles' pairs are joined: loss, log of the sum
//   4. (gradients) for each piece of the vocabulary dz, from kept logits or from the products once more, then dh += dz W and
//      dW = dz^T h as products of the kernel of the grouped experts with one group
// dz is rounded to bf16 once: it is the tensor cores' operand, and carried in two parts (a bf16 value and what it leaves) both
// gradients' products would double, 2.2 of the 3.6 ms of 4096 rows.  The rounding is what dh and dW are off by beside their own:
// 1.9e-3 to 2.6e-3 of their rms against 64 bits where the output's rounding alone is 1.7e-3.
// A second pass over the products costs 2 N V H operations beside the 6 N V H of loss and gradients; what it saves is N V logits
// in fp32 (they cannot be kept in bf16: a logit of 20 would be off by 0.06, its probability by 6 %), which cross to memory and
// back at some 5.5 TB/s.  So long hidden rows keep them where there is room (4096 rows, 102400 words, H = 2048: all gradients
// 4.11 ms, recomputed 4.73; 32768 words: H = 2048 1.30 ms, recomputed 1.47, H = 1024 0.87, recomputed 0.81; 256 rows, 102400
// words, H = 4096: 0.64, recomputed 0.81).  For few rows -- a verified block -- the logits are little and the head's bytes are
// the time: there they are always kept, and the vocabulary is dealt out to blocks whose shares of dh different SMs sum, in fp32,
// added up in order afterwards (dh alone has no more tiles than H / 128: 16 of 148 SMs at H = 2048).
//
// 16 rows x 102400 words x 2048: 147 to 159 us with dh, of which the head's two ways from memory are 130; the loss alone 76 (65).
// 4096 rows (a quarter of them padding) with both gradients 3.60 to 3.80 ms, the three products 2.8 at the rate that the power
// cap allows; 4096 rows, loss alone 1.10 ms.
#include "dx_mm.cuh"

namespace {

// ---- 1: which rows count -------------------------------------------------------------------------------------------
// One CTA, a thread for every 1/1024 of the rows: counted, summed over the CTA, listed.  live[i]: the i-th row that counts; rows
// that do not have loss 0 (a target outside the vocabulary, and a weight other than 0: NaN).
constexpr int kListed = 256;      // rows up to which every row's CTA counts those in front of it
__device__ __forceinline__ bool row_counts(const int32_t* targets, const float* row_weight, int r, int V, bool& bad) {
  const int t = __ldg(targets + r);
  const float w = row_weight ? __ldg(row_weight + r) : 1.0f;
  bad = (t < -1 || t >= V) && w != 0.0f;      // (what a row of weight 0 has for a target does not matter)
  return t >= 0 && t < V && w != 0.0f;
}
__global__ void __launch_bounds__(1024) dx_head_rows_kernel(const int32_t* targets, const float* row_weight, int N, int V,
                                                            int32_t* live, int32_t* n_live, float* loss,
                                                            int32_t* dev_status) {
  __shared__ int sums[32];
  dx_pdl_wait();
  dx_pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int each = (N + 1023) / 1024, lo = min(N, (int)threadIdx.x * each), hi = min(N, lo + each);
  int count = 0;
#pragma unroll 4
  for (int r = lo; r < hi; ++r) {
    bool bad;
    const bool in = row_counts(targets, row_weight, r, V, bad);
    if (bad) atomicExch(dev_status, (int32_t)DX_DEV_BAD_TOKEN);
    if (!in && loss) loss[r] = bad ? __int_as_float(0x7fffffff) : 0.0f;
    count += in ? 1 : 0;
  }
  int sum = count;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += o;
  }
  if (lane == 31) sums[warp] = sum;
  __syncthreads();
  int at = sum - count, all = 0;
#pragma unroll
  for (int w = 0; w < 32; ++w) {
    at += w < warp ? sums[w] : 0;
    all += sums[w];
  }
#pragma unroll 4
  for (int r = lo; r < hi; ++r) {
    bool bad;
    if (row_counts(targets, row_weight, r, V, bad) && DX_BOUNDS(at < N, dev_status)) live[at++] = r;
  }
  if (threadIdx.x == 0) {
    n_live[0] = 0;        // (offsets of the one group that the products of the gradients see)
    n_live[1] = all;
  }
}
// Few rows (a thread for each): a CTA per row counts those in front of its own and does both.  One launch instead of two and
// no list to wait for.
__global__ void __launch_bounds__(kListed) dx_head_few_kernel(const int32_t* targets, const float* row_weight, int N, int V,
                                                              const __nv_bfloat16* h, int64_t ldh, int H, int32_t* live,
                                                              int32_t* n_live, float* loss, __nv_bfloat16* out,
                                                              int32_t* dev_status) {
  dx_pdl_wait();
  dx_pdl_trigger();
  const int mine = blockIdx.x, r = threadIdx.x;
  bool bad = false, own_bad;
  const bool in_front = r < mine && row_counts(targets, row_weight, r, V, bad);
  const int at = __syncthreads_count(in_front);
  const bool in = row_counts(targets, row_weight, mine, V, own_bad);
  if (r == 0) {
    if (own_bad) atomicExch(dev_status, (int32_t)DX_DEV_BAD_TOKEN);
    if (!in && loss) loss[mine] = own_bad ? __int_as_float(0x7fffffff) : 0.0f;
    if (in && DX_BOUNDS(at < N, dev_status)) live[at] = mine;
    if (mine == N - 1) {
      n_live[0] = 0;
      n_live[1] = at + (in ? 1 : 0);
    }
  }
  if (!in || !DX_BOUNDS(at < N, dev_status)) return;
  for (int i = r * 8; i < H; i += kListed * 8)
    *reinterpret_cast<uint4*>(out + (int64_t)at * H + i) = __ldg(reinterpret_cast<const uint4*>(h + mine * ldh + i));
}
// the listed rows next to each other: four rows per CTA
__global__ void __launch_bounds__(256) dx_head_pack_kernel(const __nv_bfloat16* h, int64_t ldh, int H, const int32_t* live,
                                                           const int32_t* n_live, int N, __nv_bfloat16* out,
                                                           int32_t* dev_status) {
  dx_pdl_wait();
  dx_pdl_trigger();
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= __ldg(n_live) || !DX_BOUNDS(row < N && live[row] >= 0 && live[row] < N, dev_status)) return;
  const __nv_bfloat16* from = h + (int64_t)__ldg(live + row) * ldh;
  for (int i = (threadIdx.x & 63) * 8; i < H; i += 512)
    *reinterpret_cast<uint4*>(out + (int64_t)row * H + i) = __ldg(reinterpret_cast<const uint4*>(from + i));
}

// 32 bytes of a row per store: a thread has a row of its own, and less than a sector would be written twice
__device__ __forceinline__ void store_sector(void* at, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void store32(float* at, const float (&v)[32], int n) {   // (n: whole sectors of them)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (8 * i >= n) break;
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[8 * i + j]);
    store_sector(at + 8 * i, w);
  }
}
__device__ __forceinline__ void store32(__nv_bfloat16* at, const float (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = bf16_pair(v[16 * i + 2 * j], v[16 * i + 2 * j + 1]);
    store_sector(at + 16 * i, w);
  }
}

// ---- 2: (maximum, sum) of a half of a tile's columns (every other 32), a row per thread ----------------------------------
template <bool KEEP>
struct RowSums {
  const MmParams& p;
  const int lane, share;
  int row, target;
  float top, sum;
  static constexpr bool kBefore = false;
  static constexpr int kStaging = 0, kCols = 32, kRound = 1, kGathering = 0;
  struct Values {
    float v[32];
  };
  __device__ RowSums(const MmParams& p_, const MmMaps&, int lane_, int share_, uint32_t, MmFetch)
      : p(p_), lane(lane_), share(share_) {}
  __device__ __forceinline__ void finish() {}
  __device__ __forceinline__ void load(uint32_t taddr, Values& x) { mm_ld32(taddr, x.v); }
  __device__ __forceinline__ void zero(Values&) {}
  __device__ __forceinline__ void begin(const MmTile& t, int lane0, int, const MmTile&, bool) {
    row = lane0 + lane < t.rows ? lane0 + lane : -1;
    if (!DX_BOUNDS(row < p.n_rows, p.dev_status)) row = -1;
    target = row >= 0 ? __ldg(p.targets + __ldg(p.live + row)) - t.n0 : -1;   // (its place among the tile's columns)
    top = -INFINITY;
    sum = 0.0f;
  }
  template <class Taken>
  __device__ __forceinline__ void chunk(const MmTile& t, int, int c0, Values& x, Taken taken) {
    taken();
    float(&v)[32] = x.v;
    const int left = t.ncols - c0;
    if (KEEP && row >= 0 && DX_BOUNDS(t.n0 + c0 + (left < 32 ? (left + 7) / 8 * 8 : 32) <= p.ld_logits, p.dev_status))
      store32(p.logits + (int64_t)row * p.ld_logits + t.n0 + c0, v, left);
    if (left < 32) {
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (c >= left) v[c] = -INFINITY;
    }
    const int at = target - c0;
    if (__any_sync(0xffffffffu, at >= 0 && at < 32)) {
      float z = 0.0f;
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (c == at) z = v[c];
      if (at >= 0 && at < min(32, left)) p.target_logit[row] = z;
    }
    float m = v[0];
#pragma unroll
    for (int c = 1; c < 32; ++c) m = fmaxf(m, v[c]);
    m = fmaxf(m, top);
    const float from = m == -INFINITY ? 0.0f : m;      // (all -inf so far: exp(-inf - 0) = 0)
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < 32; ++c) s[c & 3] += ex2((v[c] - from) * kLog2e);
    sum = sum * ex2((top - from) * kLog2e) + ((s[0] + s[1]) + (s[2] + s[3]));
    top = m;
  }
  __device__ __forceinline__ void end(const MmTile& t) {
    if (row >= 0) p.part[(t.row0 * 2 + share) * p.part_half + row * p.part_row] = make_float2(top, sum);
  }
};

// ---- 3: joined over the tiles ----------------------------------------------------------------------------------------
// 32 rows per CTA, a lane each; 32 warps take the tiles in turns.  The loss is (maximum - target's logit) + log of the sum
// relative to the maximum, so that a confident row's loss is not a difference of two large numbers.  With gradients also the
// zeros of the rows that do not count.
__global__ void __launch_bounds__(1024) dx_head_join_kernel(const float2* part, int part_pitch, int tiles, const int32_t* live,
                                                           const int32_t* n_live_at, const float* target_logit, float* loss,
                                                           float* lse, float* row_loss, const int32_t* targets,
                                                           const float* row_weight, int N, int V, int H,
                                                           __nv_bfloat16* dh, int64_t ld_dh, int32_t* dev_status) {
  __shared__ float tops[32][32];
  __shared__ double sums[32][32];
  dx_pdl_wait();
  dx_pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x * 32 + lane;
  const int n_live = __ldg(n_live_at);
  float top = -INFINITY;
  double sum = 0.0;        // (hundreds of tiles: their additions would be the largest error of the loss)
  if (row < n_live) {
    for (int i = warp; i < tiles; i += 256) {     // (eight of them under way at a time)
      float2 q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        q[j] = i + 32 * j < tiles ? __ldg(part + (int64_t)(i + 32 * j) * part_pitch + row) : make_float2(-INFINITY, 0.0f);
      float m = top;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, q[j].x);
      const float from = m == -INFINITY ? 0.0f : m;
      sum *= ex2((top - from) * kLog2e);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += q[j].y * ex2((q[j].x - from) * kLog2e);
      top = m;
    }
  }
  tops[warp][lane] = top;
  sums[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && row < n_live && DX_BOUNDS(row < N && live[row] >= 0 && live[row] < N, dev_status)) {
    float m = tops[0][lane];
#pragma unroll
    for (int w = 1; w < 32; ++w) m = fmaxf(m, tops[w][lane]);
    const float from = m == -INFINITY ? 0.0f : m;
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < 32; ++w) s += sums[w][lane] * ex2((tops[w][lane] - from) * kLog2e);
    const double log_sum = log(s);
    const float l = (float)(((double)m - (double)target_logit[row]) + log_sum);
    if (loss) loss[live[row]] = l;
    lse[row] = (float)((double)m + log_sum);
    row_loss[row] = l;
  }
  if (!dh) return;
  for (int r = blockIdx.x * 32 + warp; r < min(N, blockIdx.x * 32 + 32); r += 32) {
    const int t = __ldg(targets + r);
    if (t >= 0 && t < V && (!row_weight || __ldg(row_weight + r) != 0.0f)) continue;
    for (int i = lane; i < H / 8; i += 32) *reinterpret_cast<uint4*>(dh + r * ld_dh + 8 * i) = make_uint4(0u, 0u, 0u, 0u);
  }
}

// ---- 4: dz of a tile ---------------------------------------------------------------------------------------------------
// p - 1 at the target is -(1 - exp(-loss)): where the row is confident that is not the difference of two rounded numbers.
struct StoreDz {
  const MmParams& p;
  const int lane, share;
  int row, target;
  float lse, weight, at_target;
  static constexpr bool kBefore = false;
  static constexpr int kStaging = 0, kCols = 32, kGathering = 0;
  static constexpr int kRound = 64;      // (the products of the gradients read whole blocks of 64)
  struct Values {
    float v[32];
  };
  __device__ StoreDz(const MmParams& p_, const MmMaps&, int lane_, int share_, uint32_t, MmFetch)
      : p(p_), lane(lane_), share(share_) {}
  __device__ __forceinline__ void finish() {}
  __device__ __forceinline__ void load(uint32_t taddr, Values& x) { mm_ld32(taddr, x.v); }
  __device__ __forceinline__ void zero(Values&) {}
  __device__ __forceinline__ void begin(const MmTile& t, int lane0, int, const MmTile&, bool) {
    row = lane0 + lane < t.rows ? lane0 + lane : -1;
    if (!DX_BOUNDS(row < p.n_rows, p.dev_status)) row = -1;
    target = -1;
    lse = weight = at_target = 0.0f;
    if (row >= 0) {
      const int r = __ldg(p.live + row);
      target = __ldg(p.targets + r) - p.column0 - t.n0;
      weight = p.row_weight ? __ldg(p.row_weight + r) : 1.0f;
      lse = __ldg(p.lse + row);
      at_target = weight * expm1f(-__ldg(p.row_loss + row));
    }
  }
  __device__ __forceinline__ void end(const MmTile&) {}
  template <class Taken>
  __device__ __forceinline__ void chunk(const MmTile& t, int, int c0, Values& x, Taken taken) {
    taken();
    float(&v)[32] = x.v;
#pragma unroll
    for (int c = 0; c < 32; ++c) v[c] = weight * ex2((v[c] - lse) * kLog2e);
    const int at = target - c0;
    if (__any_sync(0xffffffffu, at >= 0 && at < 32)) {
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (c == at) v[c] = at_target;
    }
    if (t.ncols - c0 < 32) {
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (c >= t.ncols - c0) v[c] = 0.0f;
    }
    if (row < 0 || !DX_BOUNDS(row < p.panel && t.n0 % kPanel == 0 && c0 + 32 <= kPanel, p.dev_status)) return;
    store32(reinterpret_cast<__nv_bfloat16*>(p.out) + ((int64_t)(t.n0 / kPanel) * p.panel + row) * kPanel + c0, v);
  }
};

// ... from logits that were kept, eight words of a row (lse, row_loss of that row; target: its place among the eight)
__device__ __forceinline__ uint4 dz_of(const float* logits, float weight, float lse, float row_loss, int target, int left) {
  float z[8];
  asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(z[0]), "=f"(z[1]), "=f"(z[2]), "=f"(z[3]), "=f"(z[4]), "=f"(z[5]), "=f"(z[6]), "=f"(z[7]) : "l"(logits));
  const float at_target = target >= 0 && target < 8 ? weight * expm1f(-row_loss) : 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    z[i] = weight * ex2((z[i] - lse) * kLog2e);
    if (i == target) z[i] = at_target;
    if (i >= left) z[i] = 0.0f;
  }
  return make_uint4(bf16_pair(z[0], z[1]), bf16_pair(z[2], z[3]), bf16_pair(z[4], z[5]), bf16_pair(z[6], z[7]));
}
// words v0 .. v0 + len of all rows (blockIdx.x): dz of a piece
__global__ void __launch_bounds__(256) dx_head_dz_kernel(const float* logits, int64_t ld_logits, int v0, int len,
                                                         const int32_t* live, const int32_t* n_live,
                                                         const int32_t* targets, const float* row_weight,
                                                         const float* lse, const float* row_loss, __nv_bfloat16* dz, int panel,
                                                         int32_t* dev_status) {
  dx_pdl_wait();
  dx_pdl_trigger();
  const int row = blockIdx.x, v = (blockIdx.y * 256 + threadIdx.x) * 8;
  if (row >= __ldg(n_live) || v >= (len + 63) / 64 * 64 ||
      !DX_BOUNDS(row < panel && live[row] >= 0 && live[row] < panel && v0 + v + 8 <= ld_logits, dev_status))
    return;
  const int r = __ldg(live + row);
  *reinterpret_cast<uint4*>(dz + ((int64_t)(v / kPanel) * panel + row) * kPanel + v % kPanel) =
      dz_of(logits + row * ld_logits + v0 + v, row_weight ? __ldg(row_weight + r) : 1.0f, __ldg(lse + row), __ldg(row_loss + row),
            __ldg(targets + r) - v0 - v, len - v);
}
// Little work (N V): a CTA joins the tiles of one row (blockIdx.y) ...
// ... and, where the logits were kept, goes on to eight elements of dz per thread; all CTAs of a row join it in the same order (a
// kernel for that, between this one and the products, took 8 us where this takes 2).
__global__ void __launch_bounds__(256) dx_head_row_kernel(const float* logits, int64_t ld_logits, int V, const int32_t* live,
                                                         const int32_t* n_live, const int32_t* targets,
                                                         const float* row_weight, const float2* part, int halves,
                                                         const float* target_logit, float* loss, float* lses, float* row_losses,
                                                         __nv_bfloat16* dz, int panel, int H, __nv_bfloat16* dh, int64_t ld_dh,
                                                         int32_t* dev_status) {
  __shared__ float tops[8], row_loss_at, lse_at;
  __shared__ double sums[8];
  dx_pdl_wait();
  dx_pdl_trigger();
  const int row = blockIdx.y, v0 = (blockIdx.x * 256 + threadIdx.x) * 8, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x == 0 && dh) {          // (of the rows as they were given)
    bool bad;
    if (!row_counts(targets, row_weight, row, V, bad))
      for (int i = threadIdx.x; i < H / 8; i += 256)
        *reinterpret_cast<uint4*>(dh + row * ld_dh + 8 * i) = make_uint4(0u, 0u, 0u, 0u);
  }
  if (row >= __ldg(n_live) || !DX_BOUNDS(row < panel && live[row] >= 0 && live[row] < panel, dev_status)) return;
  const int r = __ldg(live + row), target = __ldg(targets + r) - v0;
  const float weight = row_weight ? __ldg(row_weight + r) : 1.0f, z_target = __ldg(target_logit + row);
  const bool here = logits && v0 < (V + 63) / 64 * 64;
  part += (int64_t)row * halves;
  float top = -INFINITY;
  double sum = 0.0;
  for (int i = threadIdx.x; i < halves; i += 1024) {
    float2 q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = i + 256 * j < halves ? __ldg(part + i + 256 * j) : make_float2(-INFINITY, 0.0f);
    const float m = fmaxf(top, fmaxf(fmaxf(q[0].x, q[1].x), fmaxf(q[2].x, q[3].x))), from = m == -INFINITY ? 0.0f : m;
    sum *= ex2((top - from) * kLog2e);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += q[j].y * ex2((q[j].x - from) * kLog2e);
    top = m;
  }
  float m = top;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  if (lane == 0) tops[warp] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) m = fmaxf(m, tops[w]);
  const float from = m == -INFINITY ? 0.0f : m;
  sum *= ex2((top - from) * kLog2e);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) sums[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < 8; ++w) sum += sums[w];
    const double log_sum = log(sum);
    if (lane == 0) {
      row_loss_at = (float)(((double)m - (double)z_target) + log_sum);
      lse_at = (float)((double)m + log_sum);
      if (blockIdx.x == 0) {
        if (loss) loss[r] = row_loss_at;
        lses[row] = lse_at;
        row_losses[row] = row_loss_at;
      }
    }
  }
  __syncthreads();
  if (!here || !DX_BOUNDS(v0 + 8 <= ld_logits, dev_status)) return;
  *reinterpret_cast<uint4*>(dz + ((int64_t)(v0 / kPanel) * panel + row) * kPanel + v0 % kPanel) =
      dz_of(logits + row * ld_logits + v0, weight, lse_at, row_loss_at, target, V - v0);
}

// dh of the rows that count: the blocks' shares in order, rounded once
__global__ void __launch_bounds__(128) dx_head_sum_kernel(const float* share, int blocks, int rows, int H, const int32_t* live,
                                                          const int32_t* n_live, __nv_bfloat16* dh, int64_t ld_dh,
                                                          int32_t* dev_status) {
  dx_pdl_wait();
  dx_pdl_trigger();
  const int row = blockIdx.y, i = (blockIdx.x * 128 + threadIdx.x) * 4;
  if (row >= __ldg(n_live) || i >= H || !DX_BOUNDS(row < rows && live[row] >= 0 && live[row] < rows, dev_status)) return;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int b = 0; b < blocks; ++b) {
    const float4 q = __ldcs(reinterpret_cast<const float4*>(share + ((int64_t)b * rows + row) * H + i));
    s = make_float4(s.x + q.x, s.y + q.y, s.z + q.z, s.w + q.w);
  }
  *reinterpret_cast<uint2*>(dh + (int64_t)__ldg(live + row) * ld_dh + i) = make_uint2(bf16_pair(s.x, s.y), bf16_pair(s.z, s.w));
}

// ---- workspace -----------------------------------------------------------------------------------------------------
constexpr size_t kPieceBest = size_t(256) << 20;   // bytes of dz of a piece with which more would gain nothing
// Logits are kept where there are few (half of L2), and, up to 2 GB, where hidden rows are so long that a logit's second product
// takes longer than its way to memory and back (measured above: the two meet a little above H = 1024).
constexpr size_t kKeepFew = size_t(64) << 20, kKeepMost = size_t(2) << 30;
constexpr int kKeepFrom = 1280;

constexpr int kByRow = 1 << 21;      // words up to which every CTA of a row joins its tiles (V^2 / 2^18 pairs are read)
constexpr int kFewest = 32768;       // rows up to which a CTA per row (and block) will do

struct HeadPlan {
  bool by_row;               // a CTA or more for each row joins its tiles
  bool keep;                 // logits are kept
  int tiles;                 // of the first pass, along the vocabulary
  int piece;                 // words of a piece (a multiple of 256)
  int blocks;                // shares of dh that are summed apart
  size_t live, n_live, rows, part, target_logit, lse, row_loss, dh_acc, logits, share, dz, bytes;
  int pitch;                 // rows of a half tile's sums (where they are joined by themselves)
  int width;                 // words of a tile of the first pass
  int64_t ld_logits;
};
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// `space`: bytes there are (0: as many as are of use)
HeadPlan head_plan(int sm_count, int N, int V, int H, bool grad, size_t space) {
  HeadPlan s = {};
  if (sm_count < 2) sm_count = 2;
  const int64_t words = ((int64_t)V + 255) / 256 * 256;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += up256(bytes);
    return here;
  };
  s.pitch = (N + 31) / 32 * 32;
  s.n_live = take(8);
  s.live = take((size_t)N * 4);
  s.target_logit = take((size_t)N * 4);
  s.lse = take((size_t)N * 4);
  s.row_loss = take((size_t)N * 4);
  s.rows = take((size_t)N * H * 2);
  // Few rows: the width with which the tiles fill the GPU best (the last round is rarely full: 400 tiles of 256 words are 2.7
  // rounds of 148 SMs, 427 of 240 are 2.9).  More rows: narrower tiles would fetch the rows more often than they save.
  s.width = 256;
  if (N <= 128) {
    int64_t best = 0;
    for (int w = 256; w >= 128; w -= 16) {
      const int64_t cost = ((V + w - 1) / w + sm_count - 1) / sm_count * w;
      if (best == 0 || cost < best) {
        best = cost;
        s.width = w;
      }
    }
  }
  s.tiles = (V + s.width - 1) / s.width;
  s.part = take((size_t)s.tiles * 2 * s.pitch * sizeof(float2));
  s.by_row = (size_t)N * words * 4 <= kKeepFew && words <= kByRow && N <= kFewest;
  s.blocks = 1;
  s.piece = (int)words;
  s.bytes = at;
  if (!grad) return s;
  const size_t fixed = at, column = (size_t)N * 2;
  // words of a piece: all of them, or as many as the space allows, in pieces of equal length
  int64_t piece = (int64_t)(kPieceBest / column / 256 * 256);
  if (piece < 256 || space == 1) piece = 256;
  const size_t kept = (size_t)N * words * 4;
  const bool worth = s.by_row || (H >= kKeepFrom && kept <= kKeepMost);
  for (int level = space == 1 ? 2 : worth ? 0 : 1;; ++level) {
    // (0: the logits are kept; 1: they are not; 2: nor shares of dh, and as many words as are left room for)
    const bool lean = level == 2;
    at = fixed;
    s.keep = level == 0;
    if (lean) {
      const size_t rest = up256((size_t)N * H * 4);
      piece = space > fixed + rest ? (int64_t)((space - fixed - rest) / column / 256 * 256) : 256;
      if (piece < 256) piece = 256;
    }
    if (piece > words) piece = words;
    const int64_t pieces = (words + piece - 1) / piece;
    piece = (words / 256 + pieces - 1) / pieces * 256;
    s.blocks = 1;
    if (!lean && N <= kFewest) {
      // dh has few tiles where there are few rows, and rarely a multiple of what runs at a time: a piece's words are dealt out
      // to as many blocks as fill the GPU best, their shares of dh summed apart.  Rates in words and bytes per microsecond: a
      // pair of CTAs multiplies 256 x 256 x 64 in a third of a microsecond; few rows wait for the head's bytes instead.
      const bool few = N <= kSomeRows;          // (one tile of them)
      const int64_t tiles = few ? (H + 127) / 128 : ((H + 255) / 256) * (int64_t)((N + 255) / 256);
      const int64_t units = few ? sm_count : sm_count / 2;
      const double wave = few ? (double)piece * 256.0 * units / 6e6 : (double)piece / 64.0 * 0.33;
      double least = 0.0;
      for (int n = 1; n <= 32 && n <= piece / 256; ++n) {
        const double cost = (double)pieces * (double)((n * tiles + units - 1) / units) * wave / n +
                            (n > 1 ? n * (double)N * H * 8.0 / 6e6 + 4.0 : 0.0);
        if (n == 1 || cost < least) {
          least = cost;
          s.blocks = n;
        }
      }
    }
    s.piece = (int)piece;
    s.ld_logits = words;
    if (s.keep) s.logits = take(kept);
    if (s.blocks > 1) s.share = take((size_t)s.blocks * N * H * 4);
    else if (pieces > 1 || lean) s.dh_acc = take((size_t)N * H * 4);
    s.dz = take(column * piece);
    s.bytes = at;
    if (lean || space == 0 || space >= s.bytes) return s;
  }
}

template <class Epilogue>
cudaError_t launch_head(dx_ctx* ctx, const MmMaps& m, const MmParams& p, cudaStream_t st) {
  // up to 128 rows: a pair of CTAs would multiply 128 rows of nothing
  const bool few = p.n_rows <= 128;
  const long long lanes = few ? 128 : 256;
  const int width = p.tile_width ? p.tile_width : 256;
  const long long tiles = ((p.n_rows + lanes - 1) / lanes) * ((p.columns + width - 1) / width);
  return few ? mm_launch<kHead, false, 1, 256, 4, Epilogue>(ctx, m, p, tiles, st)
             : mm_launch<kHead, false, 2, 256, 6, Epilogue>(ctx, m, p, tiles, st);
}

}  // namespace

void dx_head_loss_workspace(int sm_count, int N, int V, int H, int grad, size_t* least, size_t* best) {
  *best = head_plan(sm_count, N, V, H, grad != 0, 0).bytes;
  *least = head_plan(sm_count, N, V, H, grad != 0, 1).bytes;
  if (*best < *least) *best = *least;
}

cudaError_t dx_launch_head_loss(dx_ctx* ctx, const DxHeadLoss& a, cudaStream_t st, int* n_launches) {
  const bool grad = a.dh != nullptr || a.dW != nullptr;
  const HeadPlan s = head_plan(ctx->sm_count, a.N, a.V, a.H, grad, a.workspace_bytes);
  unsigned char* ws = reinterpret_cast<unsigned char*>(a.workspace);
  int32_t* live = reinterpret_cast<int32_t*>(ws + s.live);
  int32_t* n_live = reinterpret_cast<int32_t*>(ws + s.n_live);
  float2* part = reinterpret_cast<float2*>(ws + s.part);
  float* target_logit = reinterpret_cast<float*>(ws + s.target_logit);
  float* lse = reinterpret_cast<float*>(ws + s.lse);
  float* row_loss = reinterpret_cast<float*>(ws + s.row_loss);
  float* dh_acc = reinterpret_cast<float*>(ws + s.dh_acc);
  float* logits = reinterpret_cast<float*>(ws + s.logits);
  float* share = reinterpret_cast<float*>(ws + s.share);
  __nv_bfloat16* dz = reinterpret_cast<__nv_bfloat16*>(ws + s.dz);
  __nv_bfloat16* dh = reinterpret_cast<__nv_bfloat16*>(a.dh);
  __nv_bfloat16* rows = reinterpret_cast<__nv_bfloat16*>(ws + s.rows);
  int n = 0;
  cudaError_t e = cudaSuccess;
  auto launched = [&](cudaError_t err) {
    e = err;
    if (e == cudaSuccess) ++n;
    *n_launches = n;
    return e == cudaSuccess;
  };

  MmMaps m = {};
  // (few rows: copies of no more rows than that; what else the lanes' place in a stage holds meets no row that counts)
  const int box = a.N <= 32 ? 32 : 128;
  if (!dx_matrix_map(&m.a, rows, a.N, a.H, a.H, box) || !dx_matrix_map(&m.b, a.W, a.V, a.H, a.ldw, 128))
    return cudaErrorInvalidValue;
  MmParams p = {};
  p.n_groups = 1;
  p.n_rows = a.N;
  p.n_live = n_live + 1;
  p.columns = a.V;
  p.kdim = a.H;
  p.live = live;
  p.a_box = (uint32_t)box;
  p.targets = a.targets;
  p.row_weight = a.row_weight;
  p.part = part;
  p.part_half = s.by_row ? 1 : s.pitch;
  p.part_row = s.by_row ? 2 * s.tiles : 1;
  p.target_logit = target_logit;
  p.lse = lse;
  p.row_loss = row_loss;
  p.logits = logits;
  p.ld_logits = s.ld_logits;
  p.dev_status = ctx->dev_status;
  p.wait_limit = ctx->wait_limit;
  p.section = kSectionFp32;

  const bool pdl = (ctx->pdl_mask & DX_PDL_EXPERTS) != 0;
  if (a.N <= kListed) {
    if (!launched(dx_launch_pdl(pdl, dx_head_few_kernel, dim3(a.N), dim3(kListed), 0, st, 1, a.targets, a.row_weight, a.N, a.V,
                                reinterpret_cast<const __nv_bfloat16*>(a.h), a.ldh, a.H, live, n_live, a.loss, rows,
                                ctx->dev_status))) return e;
  } else {
    if (!launched(dx_launch_pdl(pdl, dx_head_rows_kernel, dim3(1), dim3(1024), 0, st, 1, a.targets, a.row_weight, a.N, a.V, live,
                                n_live, a.loss, ctx->dev_status))) return e;
    if (!launched(dx_launch_pdl(pdl, dx_head_pack_kernel, dim3((a.N + 3) / 4), dim3(256), 0, st, 1,
                                reinterpret_cast<const __nv_bfloat16*>(a.h), a.ldh, a.H, live, n_live + 1, a.N, rows,
                                ctx->dev_status))) return e;
  }
  p.tile_width = s.width;
  if (!launched(s.keep ? launch_head<RowSums<true>>(ctx, m, p, st) : launch_head<RowSums<false>>(ctx, m, p, st))) return e;
  p.tile_width = 0;
  if (s.by_row) {
    // (logits that are kept become dz in the same launch)
    if (!launched(dx_launch_pdl(pdl, dx_head_row_kernel, dim3(s.keep ? (a.V + 2047) / 2048 : 1, a.N), dim3(256), 0, st, 1,
                                s.keep ? logits : nullptr, s.ld_logits, a.V, live, n_live + 1, a.targets, a.row_weight, part,
                                2 * s.tiles, target_logit, a.loss, lse, row_loss, dz, a.N, a.H, dh, a.ld_dh,
                                ctx->dev_status))) return e;
  } else if (!launched(dx_launch_pdl(pdl, dx_head_join_kernel, dim3((a.N + 31) / 32), dim3(1024), 0, st, 1, part, s.pitch,
                              2 * s.tiles, live, n_live + 1, target_logit, a.loss, lse, row_loss, a.targets, a.row_weight,
                              a.N, a.V, a.H, dh, a.ld_dh, ctx->dev_status))) return e;
  if (!grad) return e;

  for (int64_t v0 = 0; v0 < a.V; v0 += s.piece) {
    const int len = (int)(a.V - v0 < s.piece ? a.V - v0 : s.piece);
    const bool first = v0 == 0, last = v0 + len == a.V;
    if (s.keep && !s.by_row) {
      if (!launched(dx_launch_pdl(pdl, dx_head_dz_kernel, dim3(a.N, (len + 2047) / 2048), dim3(256), 0, st, 1, logits,
                                  s.ld_logits, (int)v0, len, live, n_live + 1, a.targets, a.row_weight, lse, row_loss, dz, a.N,
                                  ctx->dev_status))) return e;
    } else if (!s.keep) {
      MmParams q = p;
      q.columns = len;
      q.column0 = (int)v0;
      q.out = dz;
      q.panel = a.N;
      if (!launched(launch_head<StoreDz>(ctx, m, q, st))) return e;
    }
    if (a.dh) {
      DxGroupedMm g = {};
      g.x = dz;
      g.x_rows = a.N;
      g.ldx = kPanel;
      g.w = reinterpret_cast<const unsigned char*>(a.W) + v0 * a.ldw * 2;
      g.n_groups = s.blocks;
      g.n = len;
      g.k = a.H;
      g.transposed = 1;
      g.ldw = a.ldw;
      g.w_stride = (int64_t)len * a.ldw;
      g.n_rows = s.blocks * a.N;
      g.gather_div = 1;
      g.w_rows = len;
      g.group_rows = a.N;
      g.n_live = n_live + 1;
      if (s.blocks > 1) {
        g.y = share;
        g.y_fp32 = 1;
        g.y_rows = g.n_rows;
        g.ldy = a.H;
        g.addend = first ? nullptr : share;
      } else {
        g.scatter = live;
        g.y = last ? a.dh : (void*)dh_acc;
        g.y_fp32 = last ? 0 : 1;
        g.y_rows = a.N;
        g.ldy = last ? a.ld_dh : a.H;
        g.addend = first ? nullptr : dh_acc;
      }
      if (!launched(dx_launch_grouped_mm(ctx, g, st))) return e;
      if (s.blocks > 1 && last) {
        if (!launched(dx_launch_pdl(pdl, dx_head_sum_kernel, dim3((a.H + 511) / 512, a.N), dim3(128), 0, st, 1, share,
                                    s.blocks, a.N, a.H, live, n_live + 1, dh, a.ld_dh, ctx->dev_status))) return e;
      }
    }
    if (a.dW) {
      DxGroupedDw g = {};
      g.dy = dz;
      g.dy_rows = a.N;
      g.ld_dy = kPanel;
      g.dy_panels = 1;
      g.x = rows;
      g.x_rows = a.N;
      g.ldx = a.H;
      g.n_groups = 1;
      g.n = len;
      g.k = a.H;
      g.offsets = n_live;
      g.n_rows = a.N;
      g.dy_div = g.x_div = 1;
      g.dw = reinterpret_cast<unsigned char*>(a.dW) + v0 * a.ld_dW * 2;
      g.ld_dw = a.ld_dW;
      g.dw_stride = (int64_t)len * a.ld_dW;
      if (!launched(dx_launch_grouped_dw(ctx, g, st))) return e;
    }
  }
  return e;
}
