// The experts of Eq. 4 for whole batches of tokens: products of rows, sorted by expert, with their experts' matrices
// (moe_grouped_mm), SwiGLU on top of them (moe_grouped_swiglu), the gradients of both (moe_grouped_swiglu_backward,
// moe_grouped_mm_dw).  One persistent tcgen05 kernel (dx_mm.cuh) with different operands and different ways out.
//
// In all of them the LANES of a tile are the contiguous dimension of the output and its COLUMNS the output's rows: weights
// are the fixed 128 lanes of a CTA, and the ragged number of an expert's rows is the width of the products, which
// tcgen05.mma takes in steps of 16 -- a group of 5 rows costs 16 columns, not 128.
#include "dx_mm.cuh"

namespace {

// The two lanes 2 i, 2 i + 1 hold two neighbouring elements of columns c and c + 1; after the exchange the even lane has
// both elements of column c and the odd lane both of column c + 1.
__device__ __forceinline__ void pair_up(float v0, float v1, int odd, float& x, float& y) {
  const float got = __shfl_xor_sync(0xffffffffu, odd ? v0 : v1, 1);
  x = odd ? got : v0;
  y = odd ? v1 : got;
}
__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {   // rounded to nearest even
  const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&b);
}
__device__ __forceinline__ float2 bf16_unpair(uint32_t u) {
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ void put2(float* at, float x, float y) { *reinterpret_cast<float2*>(at) = make_float2(x, y); }
__device__ __forceinline__ void put2(__nv_bfloat16* at, float x, float y) {
  *reinterpret_cast<uint32_t*>(at) = bf16_pair(x, y);
}
// sorted row of a chunk's column `c0 + lane` (-1: none)
__device__ __forceinline__ int sorted_row(const MmTile& t, int c0, int lane) {
  return c0 + lane < t.ncols ? t.n0 + c0 + lane : -1;
}
__device__ __forceinline__ int scattered(const MmParams& p, int row) {
  if (row < 0 || !p.scatter) return row;
  const int to = __ldg(p.scatter + row);
  if (to >= 0 && to < p.out_rows) return to;
  atomicExch(p.dev_status, (int32_t)DX_DEV_BAD_ROW);
  return -1;
}

// out[row of the column][lane] = D (+ addend), rounded once
template <class T, bool ADD>
struct StoreRows {
  const MmParams& p;
  const int lane, odd;
  __device__ StoreRows(const MmParams& p_, int lane_) : p(p_), lane(lane_), odd(lane_ & 1) {}
  __device__ void begin(const MmTile&, int, int) {}
  __device__ void end(const MmTile&, int, int) {}
  __device__ __forceinline__ void chunk(const MmTile& t, int lane0, int c0, const float (&v)[32]) {
    const int mine = scattered(p, sorted_row(t, c0, lane));
    const int m = (lane0 + lane) & ~1;
    const bool in = m < p.lanes;
    T* out = reinterpret_cast<T*>(p.out) + m;
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      float x, y;
      pair_up(v[c], v[c + 1], odd, x, y);
      const int row = __shfl_sync(0xffffffffu, mine, c + odd);
      if (row >= 0 && in) {
        if constexpr (ADD) {
          const float2 a = *reinterpret_cast<const float2*>(p.addend + (int64_t)row * p.lanes + m);
          x += a.x;
          y += a.y;
        }
        put2(out + (int64_t)row * p.ld, x, y);
      }
    }
  }
};

// out of group e: [columns][lanes], element (n, m) = D
template <class T>
struct StoreOuter {
  const MmParams& p;
  const int lane, odd;
  __device__ StoreOuter(const MmParams& p_, int lane_) : p(p_), lane(lane_), odd(lane_ & 1) {}
  __device__ void begin(const MmTile&, int, int) {}
  __device__ void end(const MmTile&, int, int) {}
  __device__ __forceinline__ void chunk(const MmTile& t, int lane0, int c0, const float (&v)[32]) {
    const int m = (lane0 + lane) & ~1;
    const bool in = m < p.lanes;
    T* out = reinterpret_cast<T*>(p.out) + (int64_t)t.e * p.group_stride + (int64_t)(t.n0 + c0 + odd) * p.ld + m;
    const int left = t.ncols - c0 - odd;
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      float x, y;
      pair_up(v[c], v[c + 1], odd, x, y);
      if (c < left && in) put2(out + (int64_t)c * p.ld, x, y);
    }
  }
};

// act = silu(gate) * up from the fp32 products; SAVE: the products themselves, rounded once, for the backward pass.
// Lane r of 16: r < 8 gate row 8 b + r, else up row 8 b + r - 8 (b = block of eight).
template <bool SAVE>
struct StoreSwiglu {
  const MmParams& p;
  const int lane, odd;
  __device__ StoreSwiglu(const MmParams& p_, int lane_) : p(p_), lane(lane_), odd(lane_ & 1) {}
  __device__ void begin(const MmTile&, int, int) {}
  __device__ void end(const MmTile&, int, int) {}
  __device__ __forceinline__ void chunk(const MmTile& t, int lane0, int c0, const float (&v)[32]) {
    const int n_inter = p.lanes >> 1;
    const int up = (lane >> 3) & 1;
    const int i = ((lane0 + lane) >> 4) * 8 + (lane & 7);
    const bool in = i < n_inter;
    const int at = i & ~1;
    if constexpr (SAVE) {
      __nv_bfloat16* save = reinterpret_cast<__nv_bfloat16*>(p.save) + (int64_t)(t.n0 + c0 + odd) * p.ld_save +
                            (up ? n_inter : 0) + at;
      const int left = t.ncols - c0 - odd;
#pragma unroll
      for (int c = 0; c < 32; c += 2) {
        float x, y;
        pair_up(v[c], v[c + 1], odd, x, y);
        if (c < left && in) put2(save + (int64_t)c * p.ld_save, x, y);
      }
    }
    // the gate lane takes the even columns of a pair, the up lane the odd ones
    float a[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float got = __shfl_xor_sync(0xffffffffu, up ? v[2 * j] : v[2 * j + 1], 8);
      const float g = up ? got : v[2 * j], u = up ? v[2 * j + 1] : got;
      a[j] = fast_silu(g) * u;
    }
    __nv_bfloat16* act = reinterpret_cast<__nv_bfloat16*>(p.out) + (int64_t)(t.n0 + c0 + 2 * odd + up) * p.ld + at;
    const int left = t.ncols - c0 - 2 * odd - up;
#pragma unroll
    for (int j = 0; j < 16; j += 2) {      // columns 2 j + up and 2 j + 2 + up
      float x, y;
      pair_up(a[j], a[j + 1], odd, x, y);
      if (2 * j < left && in) put2(act + (int64_t)(2 * j) * p.ld, x, y);
    }
  }
};

// D = W_down^T dy = the gradient of an unweighted act.  With q the row's pair, w its weight, s = sigmoid(gate):
//   d gate = w D up s (1 + gate (1 - s)),  d up = w D gate s,  act_w = w gate s up,  share of d w = sum over lanes of D gate s up.
// A pair of weight 0 contributes nothing, whatever its rows hold.
struct StoreSwigluGrad {
  const MmParams& p;
  const int lane, odd;
  int part;
  __device__ StoreSwigluGrad(const MmParams& p_, int lane_) : p(p_), lane(lane_), odd(lane_ & 1), part(0) {}
  __device__ void begin(const MmTile& t, int lane0, int) { part = lane0 >> 5; }
  __device__ void end(const MmTile&, int, int) {}
  __device__ __forceinline__ void chunk(const MmTile& t, int lane0, int c0, const float (&v)[32]) {
    const int n_inter = p.lanes;
    const int m = (lane0 + lane) & ~1;
    const bool in = m < n_inter;
    const int mine = sorted_row(t, c0, lane);
    float weight = 0.0f;
    if (mine >= 0) {
      const int q = p.b_index ? __ldg(p.b_index + mine) : mine;
      if (q >= 0 && q < p.n_pairs) weight = p.pair_w ? __ldg(p.pair_w + q) : 1.0f;
      else atomicExch(p.dev_status, (int32_t)DX_DEV_BAD_ROW);
    }
    const int row0 = t.n0 + c0 + odd, left = t.ncols - c0 - odd;
    const __nv_bfloat16* gu = reinterpret_cast<const __nv_bfloat16*>(p.gate_up) + (int64_t)row0 * p.ld_gate_up + m;
    uint32_t gate[16], up[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const bool there = 2 * j < left && in;
      gate[j] = there ? __ldg(reinterpret_cast<const uint32_t*>(gu + (int64_t)(2 * j) * p.ld_gate_up)) : 0u;
      up[j] = there ? __ldg(reinterpret_cast<const uint32_t*>(gu + (int64_t)(2 * j) * p.ld_gate_up + n_inter)) : 0u;
    }
    __nv_bfloat16* dgu = reinterpret_cast<__nv_bfloat16*>(p.out) + (int64_t)row0 * p.ld + m;
    __nv_bfloat16* actw = reinterpret_cast<__nv_bfloat16*>(p.act_w) + (int64_t)row0 * p.ld_act + m;
    float dw[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      float a[2];
      pair_up(v[2 * j], v[2 * j + 1], odd, a[0], a[1]);
      const float w = __shfl_sync(0xffffffffu, weight, 2 * j + odd);
      const float2 g2 = bf16_unpair(gate[j]), u2 = bf16_unpair(up[j]);
      const float g[2] = {g2.x, g2.y}, u[2] = {u2.x, u2.y};
      float dg[2], du[2], aw[2];
      dw[j] = 0.0f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float e = __expf(-fabsf(g[i])), r = __fdividef(1.0f, 1.0f + e);      // sigmoid of either sign
        const float sg = g[i] >= 0.0f ? r : e * r, not_sg = g[i] >= 0.0f ? e * r : r;
        const float gs = g[i] * sg, act = gs * u[i], d = w * a[i];
        dg[i] = d * u[i] * fmaf(gs, not_sg, sg);
        du[i] = d * gs;
        aw[i] = w * act;
        dw[j] = fmaf(a[i], act, dw[j]);
        if (w == 0.0f) dg[i] = du[i] = aw[i] = 0.0f;
      }
      const bool there = 2 * j < left && in;
      if (!there || w == 0.0f) dw[j] = 0.0f;
      if (there) {
        put2(dgu + (int64_t)(2 * j) * p.ld, dg[0], dg[1]);
        put2(dgu + (int64_t)(2 * j) * p.ld + n_inter, du[0], du[1]);
        put2(actw + (int64_t)(2 * j) * p.ld_act, aw[0], aw[1]);
      }
    }
    // sixteen lanes of one parity hold shares of the same sixteen columns: folded so that lane l ends with column l
#pragma unroll
    for (int h = 8; h >= 1; h >>= 1) {
      const bool high = (lane & (2 * h)) != 0;
#pragma unroll
      for (int j = 0; j < h; ++j) {
        const float got = __shfl_xor_sync(0xffffffffu, high ? dw[j] : dw[j + h], 2 * h);
        dw[j] = (high ? dw[j + h] : dw[j]) + got;
      }
    }
    if (p.partial && mine >= 0) p.partial[(int64_t)part * p.n_rows + mine] = dw[0];
  }
};

// d pair_w[q] = sum of the shares, in order
__global__ void __launch_bounds__(256) dx_pair_weight_grad_kernel(const float* partial, int parts, int n_rows,
                                                                  const int32_t* offsets, int n_groups,
                                                                  const int32_t* index, int n_pairs, float* d_pair_w) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  const int lo = max(0, __ldg(offsets)), hi = min(n_rows, __ldg(offsets + n_groups));
  if (r < lo || r >= hi) return;
  const int q = index ? __ldg(index + r) : r;
  if (q < 0 || q >= n_pairs) return;
  float sum = 0.0f;
#pragma unroll 8
  for (int i = 0; i < parts; ++i) sum += __ldg(partial + (int64_t)i * n_rows + r);
  d_pair_w[q] = sum;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return fn;
}

}  // namespace

bool dx_tensor_map(CUtensorMap* out, const void* base, int rank, const uint64_t* dims, const uint64_t* strides,
                   const uint32_t* box) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  cuuint64_t d[5], s[4];
  cuuint32_t b[5], one[5] = {1, 1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) {
    d[i] = dims[i];
    b[i] = box[i];
    if (i + 1 < rank) s[i] = strides[i] * 2;
  }
  return encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), d, s, b, one,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool dx_matrix_map(CUtensorMap* out, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows}, strides[1] = {(uint64_t)ld};
  const uint32_t box[2] = {64, (uint32_t)box_rows};
  return dx_tensor_map(out, base, 2, dims, strides, box);
}

namespace {

// Few rows per group: the weights' bytes are the time, so tiles are small (128 lanes: twice as many CTAs have one, and eight
// stages of 24 KB keep 128 KB of weights in flight per SM).  Otherwise pairs of CTAs with 256 lanes x 256 columns.
bool few_rows(const dx_ctx* ctx, int64_t rows, int groups) { return rows <= 32 * (int64_t)groups; }

template <int FORM, class Epilogue>
cudaError_t launch_rows(dx_ctx* ctx, const MmMaps& maps, const MmParams& p, cudaStream_t st) {
  const bool few = few_rows(ctx, p.n_rows, p.n_groups);
  const long long lanes = few ? 128 : 256, bn = few ? 64 : 256;
  // (every group may end in a tile that is not full)
  const long long most = ((p.lanes + lanes - 1) / lanes) *
                         ((p.n_rows + bn - 1) / bn + (p.n_groups < p.n_rows ? p.n_groups : p.n_rows));
  return few ? mm_launch<FORM, 1, 64, 8, Epilogue>(ctx, maps, p, most, st)
             : mm_launch<FORM, 2, 256, 6, Epilogue>(ctx, maps, p, most, st);
}

// tensor maps of the rows (columns of D) and of the weights, [groups][n][k] or [groups][2][inter][k]
bool rows_map(MmMaps* m, const void* x, int64_t x_rows, int cols, int64_t ldx, bool gathered) {
  return gathered ? dx_matrix_map(&m->bg, x, x_rows, cols, ldx, 1) : dx_matrix_map(&m->b, x, x_rows, cols, ldx, 32);
}

MmParams base_params(const dx_ctx* ctx, const int32_t* offsets, int groups, int rows) {
  MmParams p = {};
  p.offsets = offsets;
  p.n_groups = groups;
  p.n_rows = rows;
  p.a_div = p.b_div = 1;
  p.dev_status = ctx->dev_status;
  p.wait_limit = ctx->wait_limit;
  return p;
}

}  // namespace

cudaError_t dx_launch_grouped_mm(dx_ctx* ctx, const DxGroupedMm& a, cudaStream_t st) {
  MmMaps m = {};
  MmParams p = base_params(ctx, a.offsets, a.n_groups, a.n_rows);
  const int n_in = a.transposed ? a.n : a.k, n_out = a.transposed ? a.k : a.n;
  p.lanes = n_out;
  p.kdim = n_in;
  p.b_rows = a.x_rows;
  p.b_index = a.gather;
  p.b_div = a.gather_div;
  p.out = a.y;
  p.ld = a.ldy;
  p.scatter = a.scatter;
  p.out_rows = a.y_rows;
  p.addend = a.addend;
  const uint64_t dims[3] = {(uint64_t)a.k, (uint64_t)a.n, (uint64_t)a.n_groups};
  const uint64_t strides[2] = {(uint64_t)a.ldw, (uint64_t)a.w_stride};
  const uint32_t box[3] = {64, a.transposed ? 64u : 128u, 1};
  if (!dx_tensor_map(&m.a, a.w, 3, dims, strides, box) || !rows_map(&m, a.x, a.x_rows, n_in, a.ldx, a.gather != nullptr))
    return cudaErrorInvalidValue;
  if (a.transposed) {
    if (a.addend)
      return a.y_fp32 ? launch_rows<kRowsT, StoreRows<float, true>>(ctx, m, p, st)
                      : launch_rows<kRowsT, StoreRows<__nv_bfloat16, true>>(ctx, m, p, st);
    return a.y_fp32 ? launch_rows<kRowsT, StoreRows<float, false>>(ctx, m, p, st)
                    : launch_rows<kRowsT, StoreRows<__nv_bfloat16, false>>(ctx, m, p, st);
  }
  return a.y_fp32 ? launch_rows<kRows, StoreRows<float, false>>(ctx, m, p, st)
                  : launch_rows<kRows, StoreRows<__nv_bfloat16, false>>(ctx, m, p, st);
}

cudaError_t dx_launch_grouped_swiglu(dx_ctx* ctx, const DxGroupedMm& a, void* gate_up, int64_t ld_gate_up, cudaStream_t st) {
  MmMaps m = {};
  MmParams p = base_params(ctx, a.offsets, a.n_groups, a.n_rows);
  const int n_inter = a.n / 2;
  p.lanes = a.n;
  p.kdim = a.k;
  p.b_rows = a.x_rows;
  p.b_index = a.gather;
  p.b_div = a.gather_div;
  p.out = a.y;
  p.ld = a.ldy;
  p.save = gate_up;
  p.ld_save = ld_gate_up;
  // a tile's lanes: eight gate rows, the same eight up rows, the next eight ...
  const uint64_t dims[5] = {(uint64_t)a.k, 8, 2, (uint64_t)(n_inter / 8), (uint64_t)a.n_groups};
  const uint64_t strides[4] = {(uint64_t)a.ldw, (uint64_t)(n_inter * a.ldw), (uint64_t)(8 * a.ldw), (uint64_t)a.w_stride};
  const uint32_t box[5] = {64, 8, 2, 8, 1};
  if (!dx_tensor_map(&m.a, a.w, 5, dims, strides, box) || !rows_map(&m, a.x, a.x_rows, a.k, a.ldx, a.gather != nullptr))
    return cudaErrorInvalidValue;
  return gate_up ? launch_rows<kSwiglu, StoreSwiglu<true>>(ctx, m, p, st)
                 : launch_rows<kSwiglu, StoreSwiglu<false>>(ctx, m, p, st);
}

int dx_swiglu_grad_parts(int n_inter) { return (n_inter + 255) / 256 * 8; }

cudaError_t dx_launch_grouped_swiglu_grad(dx_ctx* ctx, const DxGroupedMm& a, const void* gate_up, int64_t ld_gate_up,
                                          const float* pair_w, int n_pairs, void* act_w, int64_t ld_act, float* partial,
                                          float* d_pair_w, cudaStream_t st, int* n_launches) {
  MmMaps m = {};
  MmParams p = base_params(ctx, a.offsets, a.n_groups, a.n_rows);
  p.lanes = a.k;
  p.kdim = a.n;
  p.b_rows = a.x_rows;
  p.b_index = a.gather;
  p.b_div = a.gather_div;
  p.out = a.y;
  p.ld = a.ldy;
  p.gate_up = gate_up;
  p.ld_gate_up = ld_gate_up;
  p.pair_w = pair_w;
  p.n_pairs = n_pairs;
  p.act_w = act_w;
  p.ld_act = ld_act;
  p.partial = d_pair_w ? partial : nullptr;
  const uint64_t dims[3] = {(uint64_t)a.k, (uint64_t)a.n, (uint64_t)a.n_groups};
  const uint64_t strides[2] = {(uint64_t)a.ldw, (uint64_t)a.w_stride};
  const uint32_t box[3] = {64, 64, 1};
  if (!dx_tensor_map(&m.a, a.w, 3, dims, strides, box) || !rows_map(&m, a.x, a.x_rows, a.n, a.ldx, a.gather != nullptr))
    return cudaErrorInvalidValue;
  cudaError_t e = launch_rows<kRowsT, StoreSwigluGrad>(ctx, m, p, st);
  *n_launches = 1;
  if (e != cudaSuccess || !d_pair_w) return e;
  // (lanes of a tile behind the last are no shares: only warps with lanes that exist wrote theirs)
  const int parts = (a.k + 31) / 32;
  dx_pair_weight_grad_kernel<<<(a.n_rows + 255) / 256, 256, 0, st>>>(partial, parts, a.n_rows, a.offsets, a.n_groups, a.gather,
                                                                     n_pairs, d_pair_w);
  *n_launches = 2;
  return cudaGetLastError();
}

cudaError_t dx_launch_grouped_dw(dx_ctx* ctx, const DxGroupedDw& a, cudaStream_t st) {
  MmMaps m = {};
  MmParams p = base_params(ctx, a.offsets, a.n_groups, a.n_rows);
  p.lanes = a.k;
  p.columns = a.n;
  p.a_rows = a.x_rows;
  p.b_rows = a.dy_rows;
  p.a_index = a.gather_x;
  p.a_div = a.x_div;
  p.b_index = a.gather_dy;
  p.b_div = a.dy_div;
  p.out = a.dw;
  p.ld = a.ld_dw;
  p.group_stride = a.dw_stride;
  if (!dx_matrix_map(&m.a, a.x, a.x_rows, a.k, a.ldx, 64) || !dx_matrix_map(&m.ag, a.x, a.x_rows, a.k, a.ldx, 1) ||
      !dx_matrix_map(&m.b, a.dy, a.dy_rows, a.n, a.ld_dy, 64) || !dx_matrix_map(&m.bg, a.dy, a.dy_rows, a.n, a.ld_dy, 1))
    return cudaErrorInvalidValue;
  const long long tiles = (long long)a.n_groups * ((a.k + 255) / 256) * ((a.n + 255) / 256);
  return a.dw_fp32 ? mm_launch<kOuter, 2, 256, 6, StoreOuter<float>>(ctx, m, p, tiles, st)
                   : mm_launch<kOuter, 2, 256, 6, StoreOuter<__nv_bfloat16>>(ctx, m, p, tiles, st);
}
