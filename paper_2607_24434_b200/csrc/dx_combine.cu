// The weighted sum of a token's experts and its gradient (moe_combine_tokens, moe_combine_tokens_backward):
//     y[t] = sum_j w[t, j] z[t k + j];      dz[t k + j] = w[t, j] dy[t],   dw[t, j] = <z[t k + j], dy[t]>
// Rows of k neighbours in fp32 or bf16, sums in fp32 in the order of j, rounded once.  Bound by the rows' bytes: every
// element is touched once, in 16-byte vectors, the k rows of a token by the same threads with all loads in flight.
#include "dx_internal.cuh"

namespace {

struct Vec8 {
  float v[8];
};
__device__ __forceinline__ Vec8 load8(const float* p) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ Vec8 load8(const __nv_bfloat16* p) {
  const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p));
  const uint32_t u[4] = {a.x, a.y, a.z, a.w};
  Vec8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.v[2 * i] = __uint_as_float(u[i] << 16);
    r.v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
  return r;
}
__device__ __forceinline__ void store8(float* p, const Vec8& x) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x.v[0], x.v[1], x.v[2], x.v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x.v[4], x.v[5], x.v[6], x.v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const Vec8& x) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x.v[2 * i], x.v[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}

// blockDim.x threads go along a row, blockDim.y tokens are done at a time
template <class Tz, class Ty>
__global__ void __launch_bounds__(256) dx_combine_kernel(const Tz* z, int64_t ldz, const float* w, int n_tokens, int k, int vecs,
                                                         Ty* y, int64_t ldy) {
  const int t = blockIdx.x * blockDim.y + threadIdx.y;
  if (t >= n_tokens) return;
  float weight[DX_MAX_TOPK];
#pragma unroll
  for (int j = 0; j < DX_MAX_TOPK; ++j) weight[j] = j >= k ? 0.0f : w ? __ldg(w + (int64_t)t * k + j) : 1.0f;
  const Tz* row = z + (int64_t)t * k * ldz;
  for (int i = threadIdx.x; i < vecs; i += blockDim.x) {
    Vec8 x[DX_MAX_TOPK];
#pragma unroll
    for (int j = 0; j < DX_MAX_TOPK; ++j)
      if (weight[j] != 0.0f) x[j] = load8(row + j * ldz + 8 * i);     // (a weight of 0: the row is not looked at)
    Vec8 s = {};
#pragma unroll
    for (int j = 0; j < DX_MAX_TOPK; ++j)
      if (weight[j] != 0.0f)
#pragma unroll
        for (int q = 0; q < 8; ++q) s.v[q] = fmaf(weight[j], x[j].v[q], s.v[q]);
    store8(y + (int64_t)t * ldy + 8 * i, s);
  }
}

// A warp per token; WARPS of them share one token where there are few.
template <class T, int WARPS>
__global__ void __launch_bounds__(256) dx_combine_grad_kernel(const T* dy, int64_t ld_dy, const T* z, int64_t ldz,
                                                              const float* w, int n_tokens, int k, int vecs, T* dz,
                                                              int64_t ld_dz, float* dw) {
  __shared__ float share[8][DX_MAX_TOPK];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x * (8 / WARPS) + warp / WARPS, part = warp % WARPS;
  float sum[DX_MAX_TOPK] = {};
  if (t < n_tokens) {
    float weight[DX_MAX_TOPK];
#pragma unroll
    for (int j = 0; j < DX_MAX_TOPK; ++j) weight[j] = j >= k ? 0.0f : w ? __ldg(w + (int64_t)t * k + j) : 1.0f;
    for (int i = part * 32 + lane; i < vecs; i += 32 * WARPS) {
      const Vec8 d = load8(dy + (int64_t)t * ld_dy + 8 * i);
#pragma unroll
      for (int j = 0; j < DX_MAX_TOPK; ++j) {
        if (j >= k) break;
        const int64_t r = (int64_t)t * k + j;
        Vec8 out = {};
        if (weight[j] != 0.0f) {
          if (dw) {
            const Vec8 x = load8(z + r * ldz + 8 * i);
#pragma unroll
            for (int q = 0; q < 8; ++q) sum[j] = fmaf(x.v[q], d.v[q], sum[j]);
          }
#pragma unroll
          for (int q = 0; q < 8; ++q) out.v[q] = weight[j] * d.v[q];
        }
        if (dz) store8(dz + r * ld_dz + 8 * i, out);
      }
    }
  }
  if (!dw) return;
#pragma unroll
  for (int j = 0; j < DX_MAX_TOPK; ++j) {
    if (j >= k) break;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
    if (lane == 0) share[warp][j] = sum[j];
  }
  if constexpr (WARPS > 1) __syncthreads();
  else __syncwarp();
  if (part == 0 && lane < k && t < n_tokens) {
    float s = share[warp][lane];
    for (int i = 1; i < WARPS; ++i) s += share[warp + i][lane];
    dw[(int64_t)t * k + lane] = s;
  }
}

template <class Tz, class Ty>
cudaError_t combine(const void* z, int64_t ldz, const float* w, int n, int k, int H, void* y, int64_t ldy, cudaStream_t st) {
  const int vecs = H / 8;
  int along = 8;
  while (along < vecs && along < 256) along *= 2;
  const dim3 block(along, 256 / along);
  dx_combine_kernel<Tz, Ty><<<(n + block.y - 1) / block.y, block, 0, st>>>(
      reinterpret_cast<const Tz*>(z), ldz, w, n, k, vecs, reinterpret_cast<Ty*>(y), ldy);
  return cudaGetLastError();
}

template <class T>
cudaError_t combine_grad(const void* dy, const void* z, int64_t ld_dy, int64_t ldz, const float* w, int n, int k, int H,
                         void* dz, int64_t ld_dz, float* dw, cudaStream_t st) {
  const int vecs = H / 8;
  const T *d = reinterpret_cast<const T*>(dy), *x = reinterpret_cast<const T*>(z);
  T* o = reinterpret_cast<T*>(dz);
  if (n < 2048 && vecs > 32)
    dx_combine_grad_kernel<T, 8><<<n, 256, 0, st>>>(d, ld_dy, x, ldz, w, n, k, vecs, o, ld_dz, dw);
  else
    dx_combine_grad_kernel<T, 1><<<(n + 7) / 8, 256, 0, st>>>(d, ld_dy, x, ldz, w, n, k, vecs, o, ld_dz, dw);
  return cudaGetLastError();
}

}  // namespace

cudaError_t dx_launch_combine(const void* z, int fp32, int64_t ldz, const float* w, int n_tokens, int k, int H, void* y,
                              int y_fp32, int64_t ldy, cudaStream_t st) {
  if (fp32)
    return y_fp32 ? combine<float, float>(z, ldz, w, n_tokens, k, H, y, ldy, st)
                  : combine<float, __nv_bfloat16>(z, ldz, w, n_tokens, k, H, y, ldy, st);
  return y_fp32 ? combine<__nv_bfloat16, float>(z, ldz, w, n_tokens, k, H, y, ldy, st)
                : combine<__nv_bfloat16, __nv_bfloat16>(z, ldz, w, n_tokens, k, H, y, ldy, st);
}

cudaError_t dx_launch_combine_grad(const void* dy, const void* z, int fp32, int64_t ld_dy, int64_t ldz, const float* w,
                                   int n_tokens, int k, int H, void* dz, int64_t ld_dz, float* dw, cudaStream_t st) {
  return fp32 ? combine_grad<float>(dy, z, ld_dy, ldz, w, n_tokens, k, H, dz, ld_dz, dw, st)
              : combine_grad<__nv_bfloat16>(dy, z, ld_dy, ldz, w, n_tokens, k, H, dz, ld_dz, dw, st);
}
