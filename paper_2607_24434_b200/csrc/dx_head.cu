// Cross entropy of hidden rows against a vocabulary (spec_head_loss): with z = W h, per row
//     loss = log sum_v exp(z_v) - z_target,      dz = weight * (softmax(z) - 1_target),      dh = W^T dz,     dW = dz^T h
// in pieces of the vocabulary; logits exist as tiles in tensor memory only.
//
//   1. the rows that count (a target, a weight other than 0) are listed in order: the others cost nothing below
//   2. products of the listed rows with the whole vocabulary; of every tile a row keeps (maximum, sum of exponentials) and,
//      where the tile holds it, the target's logit
//   3. the tiles' pairs are joined: loss, log of the sum
//   4. (gradients) for each piece of the vocabulary the products once more, now straight to dz (rounded to bf16 once), then
//      dh += dz W and dW = dz^T h as products of the kernel of the grouped experts with one group
// The second pass over the products costs 2 N V H operations beside the 6 N V H of loss and gradients; what it saves is
// N V logits in fp32 (they cannot be kept in bf16: a logit of 20 would be off by 0.06, its probability by 6 %).
#include "dx_mm.cuh"

namespace {

// ---- 1: which rows count -------------------------------------------------------------------------------------------
// One CTA; every turn takes 1024 rows.  live[i]: the i-th row that counts; rows that do not have loss 0 (a target outside the
// vocabulary: NaN).
__global__ void __launch_bounds__(1024) dx_head_rows_kernel(const int32_t* targets, const float* row_weight, int N, int V,
                                                            int32_t* live, int32_t* n_live, float* loss,
                                                            int32_t* dev_status) {
  __shared__ int sums[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int base = 0;
  for (int r0 = 0; r0 < N; r0 += 1024) {
    const int r = r0 + threadIdx.x;
    bool in = false;
    if (r < N) {
      const int t = __ldg(targets + r);
      const bool bad = t < -1 || t >= V;
      in = t >= 0 && !bad && (!row_weight || __ldg(row_weight + r) != 0.0f);
      if (bad) atomicExch(dev_status, (int32_t)DX_DEV_BAD_TOKEN);
      if (!in && loss) loss[r] = bad ? __int_as_float(0x7fffffff) : 0.0f;
    }
    const unsigned int m = __ballot_sync(0xffffffffu, in);
    if (lane == 0) sums[warp] = __popc(m);
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 32; ++w) {
      before += w < warp ? sums[w] : 0;
      all += sums[w];
    }
    if (in) live[base + before + __popc(m & ((1u << lane) - 1u))] = r;
    base += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    n_live[0] = 0;        // (offsets of the one group that the products of the gradients see)
    n_live[1] = base;
  }
}

// ---- 2: (maximum, sum) of a half of a tile's columns (every other 32), a row per thread ---------------------------------------------------------
struct RowSums {
  const MmParams& p;
  const int lane, share;
  int row, target;
  float top, sum;
  static constexpr int kStaging = 0, kCols = 32;
  struct Values {
    float v[32];
  };
  __device__ RowSums(const MmParams& p_, int lane_, int share_, uint32_t) : p(p_), lane(lane_), share(share_) {}
  __device__ __forceinline__ void load(uint32_t taddr, Values& x) { mm_ld32(taddr, x.v); }
  __device__ __forceinline__ void zero(Values&) {}
  __device__ __forceinline__ void begin(const MmTile& t, int lane0, int) {
    row = lane0 + lane < t.rows ? lane0 + lane : -1;
    target = row >= 0 ? __ldg(p.targets + __ldg(p.a_index + row)) - t.n0 : -1;   // (its place among the tile's columns)
    top = -INFINITY;
    sum = 0.0f;
  }
  __device__ __forceinline__ void chunk(const MmTile& t, int, int c0, Values& x) {
    float(&v)[32] = x.v;
    const int left = t.ncols - c0;
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
    if (row >= 0) p.part[(int64_t)((t.n0 >> 8) * 2 + share) * p.part_pitch + row] = make_float2(top, sum);
  }
};

// ---- 3: joined over the tiles ----------------------------------------------------------------------------------------
// 32 rows per CTA, a lane each; eight warps take the tiles in turns.  The loss is (maximum - target's logit) + log of the sum
// relative to the maximum, so that a confident row's loss is not a difference of two large numbers.  With gradients also the
// zeros of the rows that do not count.
__global__ void __launch_bounds__(256) dx_head_join_kernel(const float2* part, int part_pitch, int tiles, const int32_t* live,
                                                           const int32_t* n_live_at, const float* target_logit, float* loss,
                                                           float* lse, float* row_loss, const int32_t* targets,
                                                           const float* row_weight, int N, int V, int H,
                                                           __nv_bfloat16* dh, int64_t ld_dh) {
  __shared__ float tops[8][32], sums[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x * 32 + lane;
  const int n_live = __ldg(n_live_at);
  float top = -INFINITY, sum = 0.0f;
  if (row < n_live) {
    for (int i = warp; i < tiles; i += 8) {
      const float2 q = part[(int64_t)i * part_pitch + row];
      const float m = fmaxf(top, q.x), from = m == -INFINITY ? 0.0f : m;
      sum = sum * ex2((top - from) * kLog2e) + q.y * ex2((q.x - from) * kLog2e);
      top = m;
    }
  }
  tops[warp][lane] = top;
  sums[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && row < n_live) {
    float m = tops[0][lane];
#pragma unroll
    for (int w = 1; w < 8; ++w) m = fmaxf(m, tops[w][lane]);
    const float from = m == -INFINITY ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += sums[w][lane] * ex2((tops[w][lane] - from) * kLog2e);
    const double log_sum = log((double)s);
    const float l = (float)(((double)m - (double)target_logit[row]) + log_sum);
    if (loss) loss[live[row]] = l;
    lse[row] = (float)((double)m + log_sum);
    row_loss[row] = l;
  }
  if (!dh) return;
  for (int r = blockIdx.x * 32 + warp; r < min(N, blockIdx.x * 32 + 32); r += 8) {
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
  static constexpr int kStaging = 0, kCols = 32;
  struct Values {
    float v[32];
  };
  __device__ StoreDz(const MmParams& p_, int lane_, int share_, uint32_t) : p(p_), lane(lane_), share(share_) {}
  __device__ __forceinline__ void load(uint32_t taddr, Values& x) { mm_ld32(taddr, x.v); }
  __device__ __forceinline__ void zero(Values&) {}
  __device__ __forceinline__ void begin(const MmTile& t, int lane0, int) {
    row = lane0 + lane < t.rows ? lane0 + lane : -1;
    target = -1;
    lse = weight = at_target = 0.0f;
    if (row >= 0) {
      const int r = __ldg(p.a_index + row);
      target = __ldg(p.targets + r) - p.column0 - t.n0;
      weight = p.row_weight ? __ldg(p.row_weight + r) : 1.0f;
      lse = __ldg(p.lse + row);
      at_target = weight * expm1f(-__ldg(p.row_loss + row));
    }
  }
  __device__ __forceinline__ void end(const MmTile&) {}
  __device__ __forceinline__ void chunk(const MmTile& t, int, int c0, Values& x) {
    float(&v)[32] = x.v;
#pragma unroll
    for (int c = 0; c < 32; ++c) v[c] = weight * ex2((v[c] - lse) * kLog2e);
    const int at = target - c0;
    if (__any_sync(0xffffffffu, at >= 0 && at < 32)) {
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (c == at) v[c] = at_target;
    }
    if (row < 0) return;
    uint32_t w[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      w[c] = bf16_pair(v[2 * c], v[2 * c + 1]);
    }
    // (columns behind the piece's last are not read: the matrices of the gradients end there)
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out) + (int64_t)row * p.ld + t.n0 + c0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(out + 16 * i), "r"(w[8 * i]), "r"(w[8 * i + 1]),
                   "r"(w[8 * i + 2]), "r"(w[8 * i + 3]), "r"(w[8 * i + 4]), "r"(w[8 * i + 5]), "r"(w[8 * i + 6]),
                   "r"(w[8 * i + 7]) : "memory");
  }
};

// ---- workspace -----------------------------------------------------------------------------------------------------
constexpr size_t kPieceBest = size_t(256) << 20;   // bytes of dz of a piece with which more would gain nothing

struct HeadSpace {
  size_t live, n_live, part, target_logit, lse, row_loss, dh_acc, dz, fixed;
  int pitch;
};
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

HeadSpace head_space(int N, int V, int H, bool grad) {
  HeadSpace s;
  s.pitch = (N + 31) / 32 * 32;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += up256(bytes);
    return here;
  };
  s.n_live = take(8);
  s.live = take((size_t)N * 4);
  s.target_logit = take((size_t)N * 4);
  s.lse = take((size_t)N * 4);
  s.row_loss = take((size_t)N * 4);
  s.part = take((size_t)((V + 255) / 256) * 2 * s.pitch * sizeof(float2));
  s.dh_acc = take(grad ? (size_t)N * H * 4 : 0);
  s.dz = at;
  s.fixed = at;
  return s;
}

template <class Epilogue>
cudaError_t launch_head(dx_ctx* ctx, const MmMaps& m, const MmParams& p, cudaStream_t st) {
  // up to 128 rows: a pair of CTAs would multiply 128 rows of nothing
  const bool few = p.n_rows <= 128;
  const long long lanes = few ? 128 : 256;
  const long long tiles = ((p.n_rows + lanes - 1) / lanes) * ((p.columns + 255) / 256);
  return few ? mm_launch<kHead, true, 1, 256, 4, Epilogue>(ctx, m, p, tiles, st)
             : mm_launch<kHead, true, 2, 256, 6, Epilogue>(ctx, m, p, tiles, st);
}

}  // namespace

void dx_head_loss_workspace(int N, int V, int H, int grad, size_t* least, size_t* best) {
  const HeadSpace s = head_space(N, V, H, grad != 0);
  const size_t column = (size_t)N * 2, all = ((size_t)V + 255) / 256 * 256;
  *least = s.fixed + (grad ? column * 256 : 0);
  size_t want = kPieceBest / column / 256 * 256;
  if (want < 256) want = 256;
  if (want > all) want = all;
  *best = s.fixed + (grad ? column * want : 0);
}

cudaError_t dx_launch_head_loss(dx_ctx* ctx, const DxHeadLoss& a, cudaStream_t st, int* n_launches) {
  const bool grad = a.dh != nullptr || a.dW != nullptr;
  const HeadSpace s = head_space(a.N, a.V, a.H, grad);
  unsigned char* ws = reinterpret_cast<unsigned char*>(a.workspace);
  int32_t* live = reinterpret_cast<int32_t*>(ws + s.live);
  int32_t* n_live = reinterpret_cast<int32_t*>(ws + s.n_live);
  float2* part = reinterpret_cast<float2*>(ws + s.part);
  float* target_logit = reinterpret_cast<float*>(ws + s.target_logit);
  float* lse = reinterpret_cast<float*>(ws + s.lse);
  float* row_loss = reinterpret_cast<float*>(ws + s.row_loss);
  float* dh_acc = reinterpret_cast<float*>(ws + s.dh_acc);
  const int tiles = (a.V + 255) / 256;
  int n = 0;

  MmMaps m = {};
  if (!dx_matrix_map(&m.b, a.W, a.V, a.H, a.ldw, 128)) return cudaErrorInvalidValue;
  MmParams p = {};
  p.n_groups = 1;
  p.n_rows = a.N;
  p.n_live = n_live + 1;
  p.columns = a.V;
  p.kdim = a.H;
  p.a_src = a.h;
  p.a_ld = a.ldh;
  p.a_rows = a.N;
  p.a_index = live;
  p.targets = a.targets;
  p.row_weight = a.row_weight;
  p.part = part;
  p.part_pitch = s.pitch;
  p.target_logit = target_logit;
  p.lse = lse;
  p.row_loss = row_loss;
  p.dev_status = ctx->dev_status;
  p.wait_limit = ctx->wait_limit;

  dx_head_rows_kernel<<<1, 1024, 0, st>>>(a.targets, a.row_weight, a.N, a.V, live, n_live, a.loss, ctx->dev_status);
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) { ++n; e = launch_head<RowSums>(ctx, m, p, st); }
  if (e == cudaSuccess) {
    ++n;
    dx_head_join_kernel<<<(a.N + 31) / 32, 256, 0, st>>>(part, s.pitch, 2 * tiles, live, n_live + 1, target_logit, a.loss, lse,
                                                         row_loss, a.targets, a.row_weight, a.N, a.V, a.H,
                                                         reinterpret_cast<__nv_bfloat16*>(a.dh), a.ld_dh);
    e = cudaGetLastError();
    if (e == cudaSuccess) ++n;
  }
  if (grad && e == cudaSuccess) {
    void* dz = ws + s.dz;
    const size_t column = (size_t)a.N * 2;
    long long piece = (long long)((a.workspace_bytes - s.fixed) / column / 256 * 256);
    if (piece > (long long)tiles * 256) piece = (long long)tiles * 256;
    // (pieces of equal length)
    const int pieces = (int)((tiles * 256LL + piece - 1) / piece);
    piece = ((tiles + pieces - 1) / pieces) * 256LL;
    for (int64_t v0 = 0; v0 < a.V && e == cudaSuccess; v0 += piece) {
      const int len = (int)(a.V - v0 < piece ? a.V - v0 : piece);
      const bool first = v0 == 0, last = v0 + len == a.V;
      MmParams q = p;
      q.columns = len;
      q.column0 = (int)v0;
      q.out = dz;
      q.ld = piece;
      e = launch_head<StoreDz>(ctx, m, q, st);
      if (e != cudaSuccess) break;
      ++n;
      const unsigned char* W = reinterpret_cast<const unsigned char*>(a.W) + v0 * a.ldw * 2;
      if (a.dh) {
        DxGroupedMm g = {};
        g.x = dz;
        g.x_rows = a.N;
        g.ldx = piece;
        g.w = W;
        g.n_groups = 1;
        g.n = len;
        g.k = a.H;
        g.transposed = 1;
        g.ldw = a.ldw;
        g.w_stride = (int64_t)len * a.ldw;
        g.offsets = n_live;
        g.n_rows = a.N;
        g.gather_div = 1;
        g.scatter = live;
        g.y = last ? a.dh : (void*)dh_acc;
        g.y_fp32 = last ? 0 : 1;
        g.y_rows = a.N;
        g.ldy = last ? a.ld_dh : a.H;
        g.addend = first ? nullptr : dh_acc;
        e = dx_launch_grouped_mm(ctx, g, st);
        if (e != cudaSuccess) break;
        ++n;
      }
      if (a.dW) {
        DxGroupedDw g = {};
        g.dy = dz;
        g.dy_rows = a.N;
        g.ld_dy = piece;
        g.x = a.h;
        g.x_rows = a.N;
        g.ldx = a.ldh;
        g.n_groups = 1;
        g.n = len;
        g.k = a.H;
        g.offsets = n_live;
        g.n_rows = a.N;
        g.gather_x = live;
        g.dy_div = g.x_div = 1;
        g.dw = reinterpret_cast<unsigned char*>(a.dW) + v0 * a.ld_dW * 2;
        g.ld_dw = a.ld_dW;
        g.dw_stride = (int64_t)len * a.ld_dW;
        e = dx_launch_grouped_dw(ctx, g, st);
        if (e == cudaSuccess) ++n;
      }
    }
  }
  *n_launches = n;
  return e;
}
