// The weighted sum of a token's experts and its gradient (moe_combine_tokens, moe_combine_tokens_backward):
//     y[t] = sum_j w[t, j] z[t k + j];      dz[t k + j] = w[t, j] dy[t],   dw[t, j] = <z[t k + j], dy[t]>
// Rows of k neighbours in fp32 or bf16, sums in fp32 in the order of j, rounded once.  Bound by the rows' bytes: every element is
// touched once, in 16-byte vectors, the k rows of a token by the same threads with all loads in flight.  16384 tokens x 6 x 2048
// bf16: 73 to 75 us, 97 to 100 % of the copy rate.  The gradient of 4999 x 4 x 1000 fp32, of which nearly half is written: 36.5
// to 37.2 us, 76 % (with the loads of each row behind its own weight's test, 41.8).
#include <type_traits>

#include "dx_internal.cuh"

namespace {

// 16 bytes of a row: four fp32 or eight bf16 elements
template <class T>
struct Piece {
  static constexpr int kN = 16 / (int)sizeof(T);
  uint4 raw;
  __device__ __forceinline__ void load(const T* p) { raw = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(float (&v)[kN]) const {
    const uint32_t u[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        v[i] = __uint_as_float(u[i]);
      } else {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      }
    }
  }
};
__device__ __forceinline__ uint32_t pair(float x, float y) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&b);
}
template <int N>
__device__ __forceinline__ void put(float* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}
template <int N>
__device__ __forceinline__ void put(__nv_bfloat16* p, const float (&v)[N]) {
  if constexpr (N == 8)
    *reinterpret_cast<uint4*>(p) = make_uint4(pair(v[0], v[1]), pair(v[2], v[3]), pair(v[4], v[5]), pair(v[6], v[7]));
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(pair(v[0], v[1]), pair(v[2], v[3]));
}
__device__ __forceinline__ float weight_of(const float* w, int64_t q) { return w ? __ldg(w + q) : 1.0f; }

// blockDim.x threads go along a row, blockDim.y tokens are done at a time
template <class Tz, class Ty, int K>
__global__ void __launch_bounds__(256) dx_combine_kernel(const Tz* z, int64_t ldz, const float* w, int n_tokens, int pieces,
                                                         Ty* y, int64_t ldy) {
  constexpr int kN = Piece<Tz>::kN;
  dx_pdl_wait();
  dx_pdl_trigger();
  const int t = blockIdx.x * blockDim.y + threadIdx.y;
  if (t >= n_tokens) return;
  float weight[K];
#pragma unroll
  for (int j = 0; j < K; ++j) weight[j] = weight_of(w, (int64_t)t * K + j);
  const Tz* row = z + (int64_t)t * K * ldz;
  for (int i = threadIdx.x; i < pieces; i += blockDim.x) {
    Piece<Tz> x[K];
#pragma unroll
    for (int j = 0; j < K; ++j)
      if (weight[j] != 0.0f) x[j].load(row + j * ldz + kN * i);     // (a weight of 0: the row is not looked at)
    float s[kN] = {};
#pragma unroll
    for (int j = 0; j < K; ++j)
      if (weight[j] != 0.0f) {
        float v[kN];
        x[j].get(v);
#pragma unroll
        for (int q = 0; q < kN; ++q) s[q] = fmaf(weight[j], v[q], s[q]);
      }
    put(y + (int64_t)t * ldy + kN * i, s);
  }
}

// WARPS warps per token: one where there are tokens enough to fill the GPU
template <class T, int K, int WARPS>
__global__ void __launch_bounds__(256) dx_combine_grad_kernel(const T* dy, int64_t ld_dy, const T* z, int64_t ldz,
                                                              const float* w, int n_tokens, int pieces, T* dz, int64_t ld_dz,
                                                              float* dw) {
  constexpr int kN = Piece<T>::kN;
  __shared__ float share[8][K];
  dx_pdl_wait();
  dx_pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x * (8 / WARPS) + warp / WARPS, part = warp % WARPS;
  float sum[K] = {};
  if (t < n_tokens) {
    float weight[K];
#pragma unroll
    for (int j = 0; j < K; ++j) weight[j] = weight_of(w, (int64_t)t * K + j);
    for (int i = part * 32 + lane; i < pieces; i += 32 * WARPS) {
      Piece<T> d, x[K];
      d.load(dy + (int64_t)t * ld_dy + kN * i);
      if (dw) {
#pragma unroll
        for (int j = 0; j < K; ++j) x[j].load(z + ((int64_t)t * K + j) * ldz + kN * i);
      }
      float g[kN];
      d.get(g);
#pragma unroll
      for (int j = 0; j < K; ++j) {
        if (dw) {
          float v[kN];
          x[j].get(v);
#pragma unroll
          for (int q = 0; q < kN; ++q) sum[j] = fmaf(v[q], g[q], sum[j]);
        }
        if (dz) {
          float o[kN];
#pragma unroll
          for (int q = 0; q < kN; ++q) o[q] = weight[j] != 0.0f ? weight[j] * g[q] : 0.0f;
          put(dz + ((int64_t)t * K + j) * ld_dz + kN * i, o);
        }
      }
    }
  }
  if (!dw) return;
#pragma unroll
  for (int j = 0; j < K; ++j) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
    if (lane == 0) share[warp][j] = sum[j];
  }
  if constexpr (WARPS > 1) __syncthreads();
  else __syncwarp();
  if (part == 0 && lane < K && t < n_tokens) {
    float s = share[warp][lane];
    for (int i = 1; i < WARPS; ++i) s += share[warp + i][lane];
    const int64_t q = (int64_t)t * K + lane;
    dw[q] = isfinite(s) || weight_of(w, q) != 0.0f ? s : 0.0f;      // (a row that was taken out may hold anything)
  }
}

template <class Tz, class Ty, int K>
cudaError_t combine(bool pdl, const void* z, int64_t ldz, const float* w, int n, int H, void* y, int64_t ldy, cudaStream_t st) {
  const int pieces = H / Piece<Tz>::kN;
  int along = 8;
  while (along < pieces && along < 256) along *= 2;
  const dim3 block(along, 256 / along);
  return dx_launch_pdl(pdl, dx_combine_kernel<Tz, Ty, K>, dim3((n + block.y - 1) / block.y), block, 0, st, 1,
                       reinterpret_cast<const Tz*>(z), ldz, w, n, pieces, reinterpret_cast<Ty*>(y), ldy);
}
template <class T, int K>
cudaError_t combine_grad(bool pdl, const void* dy, const void* z, int64_t ld_dy, int64_t ldz, const float* w, int n, int H,
                         void* dz, int64_t ld_dz, float* dw, cudaStream_t st) {
  const int pieces = H / Piece<T>::kN;
  const T *d = reinterpret_cast<const T*>(dy), *x = reinterpret_cast<const T*>(z);
  T* o = reinterpret_cast<T*>(dz);
  if (n < 2048 && pieces > 32)
    return dx_launch_pdl(pdl, dx_combine_grad_kernel<T, K, 8>, dim3(n), dim3(256), 0, st, 1, d, ld_dy, x, ldz, w, n, pieces, o,
                         ld_dz, dw);
  return dx_launch_pdl(pdl, dx_combine_grad_kernel<T, K, 1>, dim3((n + 7) / 8), dim3(256), 0, st, 1, d, ld_dy, x, ldz, w, n,
                       pieces, o, ld_dz, dw);
}
// f(the number of rows of a token as a constant)
template <class F>
cudaError_t with_k(int k, F f) {
  switch (k) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 3: return f(std::integral_constant<int, 3>());
    case 4: return f(std::integral_constant<int, 4>());
    case 5: return f(std::integral_constant<int, 5>());
    case 6: return f(std::integral_constant<int, 6>());
    case 7: return f(std::integral_constant<int, 7>());
    default: return f(std::integral_constant<int, 8>());
  }
}
static_assert(DX_MAX_TOPK == 8);

}  // namespace

cudaError_t dx_launch_combine(dx_ctx* ctx, const void* z, int fp32, int64_t ldz, const float* w, int n_tokens, int k, int H,
                              void* y, int y_fp32, int64_t ldy, cudaStream_t st) {
  const bool pdl = (ctx->pdl_mask & DX_PDL_EXPERTS) != 0;
  return with_k(k, [&](auto K) {
    if (fp32)
      return y_fp32 ? combine<float, float, K.value>(pdl, z, ldz, w, n_tokens, H, y, ldy, st)
                    : combine<float, __nv_bfloat16, K.value>(pdl, z, ldz, w, n_tokens, H, y, ldy, st);
    return y_fp32 ? combine<__nv_bfloat16, float, K.value>(pdl, z, ldz, w, n_tokens, H, y, ldy, st)
                  : combine<__nv_bfloat16, __nv_bfloat16, K.value>(pdl, z, ldz, w, n_tokens, H, y, ldy, st);
  });
}

cudaError_t dx_launch_combine_grad(dx_ctx* ctx, const void* dy, const void* z, int fp32, int64_t ld_dy, int64_t ldz,
                                   const float* w, int n_tokens, int k, int H, void* dz, int64_t ld_dz, float* dw,
                                   cudaStream_t st) {
  const bool pdl = (ctx->pdl_mask & DX_PDL_EXPERTS) != 0;
  return with_k(k, [&](auto K) {
    return fp32 ? combine_grad<float, K.value>(pdl, dy, z, ld_dy, ldz, w, n_tokens, H, dz, ld_dz, dw, st)
                : combine_grad<__nv_bfloat16, K.value>(pdl, dy, z, ld_dy, ldz, w, n_tokens, H, dz, ld_dz, dw, st);
  });
}
