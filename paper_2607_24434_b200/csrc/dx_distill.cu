// Distillation from a teacher's top log probabilities (Eq. 8 with the teacher cut to a short list), per row t:
//   q = softmax(z / T);  p_j = e^{l_j} over the listed words, renormalised to sum 1 or -- with the tail bucket -- as they
//   are, the rest r = 1 - sum p in one bucket that is compared with R = sum of q over the unlisted words:
//     L = sum_j p_j (log p_j - log q_j)  [ + r (log r - log R) ]
//     dL/dz_v = ( beta q_v - p_v ) / T  for listed v,   ( beta - r / R ) q_v / T  otherwise,  beta = sum p + r
// One launch reads each logit once and writes each gradient once: a cluster of CTAs holds the row in shared memory
// between the statistics and the gradient.
//
// The unlisted words are summed apart from the listed ones (whose places in shared memory are set to -inf before the
// sweep), relative to their own maximum: R never comes out of a difference of nearly equal sums, and neither R nor the
// factor r / R can under- or overflow however far the listed words stand above the rest.  Per-row scalars (teacher
// mass, loss) are 64-bit: the loss is a small difference of logarithms.
#include "dx_rows.cuh"

namespace {

constexpr int kListLanes = DX_MAX_TEACHER / 32;   // list entries per lane of the warp that handles the list

struct DistillParams {
  const void* logits;
  int N, V, k, tail;
  long long ld, ld_d;
  const int32_t* ids;
  const float* lp;
  float c, T;                 // log2(e) / T, T
  const float* weight;
  float* loss;
  void* dlogits;
  int32_t* dev_status;
};

struct MaxSum {
  float m, s;
};
__device__ __forceinline__ MaxSum join(MaxSum x, MaxSum y, float c) {
  const float m = fmaxf(x.m, y.m);
  return MaxSum{m, x.s * row_ex2((x.m - m) * c) + y.s * row_ex2((y.m - m) * c)};
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ void copy16(uint4* dst_smem, const uint4* src) {
  const uint32_t d = static_cast<uint32_t>(__cvta_generic_to_shared(dst_smem));
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
}

template <typename T, bool kGrad>
__global__ void __launch_bounds__(kRowThreads, 4) dx_distill_kernel(DistillParams p, int C) {
  using V16 = RowVec<T>;
  extern __shared__ uint4 s_row[];                 // this CTA's vectors of the row
  __shared__ MaxSum s_warp[kRowWarps];
  __shared__ MaxSum s_cta;
  __shared__ float s_coef, s_ref;
  __shared__ unsigned int s_edge;                  // head (bits 0..7) and tail (8..15) elements that are listed
  __shared__ int s_used;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = C > 1 ? (int)cluster_rank() : 0;
  const int t = blockIdx.x / C;
  const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
  T* out = kGrad ? reinterpret_cast<T*>(p.dlogits) + (size_t)t * (size_t)p.ld_d : nullptr;
  const RowSplit sp = row_split(row, p.V, rank, C);
  const int n_vec = sp.v_hi - sp.v_lo;
  const bool has_head = rank == 0 && tid < sp.head, has_tail = rank == C - 1 && tid < sp.tail;
  const int tail0 = p.V - sp.tail;
  // gradient vectors can be stored as such where the output row is aligned like the input row
  const bool same_align = kGrad && ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row)) & 15u) == 0;
  const float c = p.c;
  const float w = p.weight ? p.weight[t] : 1.f;

  // ---- the teacher's list (first warp): ids in range, an id counts once
  int id[kListLanes];
  bool live = false;
  if (warp == 0) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kListLanes; ++i) {
      const int j = lane + 32 * i;
      id[i] = j < p.k ? p.ids[(size_t)t * p.k + j] : -1;
      bad |= id[i] < -1 || id[i] >= p.V;
      if (id[i] < 0 || id[i] >= p.V) id[i] = -1;
      live |= id[i] >= 0;
    }
    if (bad && rank == 0) *p.dev_status = DX_DEV_BAD_TOKEN;
    live = __any_sync(0xffffffffu, live);
    if (lane == 0) {
      s_used = live;
      s_edge = 0;
    }
  }
  __syncthreads();
  if (w == 0.f || !s_used) {   // (the same for every CTA of the row) nothing to learn: the logits are not looked at
    if (rank == 0 && tid == 0 && p.loss) p.loss[t] = 0.f;
    if (kGrad) {
      if (has_head) out[tid] = V16::round(0.f);
      if (has_tail) out[tail0 + tid] = V16::round(0.f);
      for (int i = tid; i < n_vec; i += kRowThreads) {
        const int e = sp.head + (sp.v_lo + i) * V16::kN;
        if (same_align) {
          *reinterpret_cast<uint4*>(out + e) = make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
          for (int q = 0; q < V16::kN; ++q) out[e + q] = V16::round(0.f);
        }
      }
    }
    return;
  }
  // ---- the row on its way into shared memory
  const uint4* src = reinterpret_cast<const uint4*>(row + sp.head) + sp.v_lo;
  for (int i = tid; i < n_vec; i += kRowThreads) copy16(s_row + i, src + i);
  asm volatile("cp.async.commit_group;" ::: "memory");
  float edge_head = has_head ? V16::load(row + tid) : -INFINITY;
  float edge_tail = has_tail ? V16::load(row + tail0 + tid) : -INFINITY;

  // ---- list statistics relative to the largest listed logit, while the row arrives
  float z[kListLanes];
  double pj[kListLanes];
  float z_ref = 0.f, sum_e = 0.f;
  double mass = 0.0, p_log_p = 0.0, p_u = 0.0;
  if (warp == 0) {
#pragma unroll
    for (int i = 0; i < kListLanes; ++i) {
      z[i] = -INFINITY;
      pj[i] = 0.0;
      if (32 * i < p.k) {
        unsigned int same = __match_any_sync(0xffffffffu, id[i]);
        if (__ffs(same) - 1 != lane) id[i] = -1;   // an earlier lane has it
#pragma unroll
        for (int h = 0; h < i; ++h) {
          for (int o = 0; o < 32; ++o) {
            const int other = __shfl_sync(0xffffffffu, id[h], o);
            if (other == id[i]) id[i] = -1;
          }
        }
      }
      if (id[i] >= 0) {
        z[i] = V16::load(row + id[i]);
        pj[i] = exp((double)p.lp[(size_t)t * p.k + lane + 32 * i]);
      }
    }
    z_ref = z[0];
#pragma unroll
    for (int i = 1; i < kListLanes; ++i) z_ref = fmaxf(z_ref, z[i]);
    z_ref = fmaxf(warp_max(z_ref), -FLT_MAX);
#pragma unroll
    for (int i = 0; i < kListLanes; ++i) mass += pj[i];
    mass = warp_sum(mass);
    const double norm = p.tail || !(mass > 0.0) ? 1.0 : 1.0 / mass;
    double se = 0.0;
#pragma unroll
    for (int i = 0; i < kListLanes; ++i) {
      pj[i] *= norm;
      if (id[i] >= 0) {
        const double u = ((double)z[i] - (double)z_ref) / (double)p.T;
        se += (double)expf((float)u);
        if (pj[i] > 0.0) {
          p_log_p += pj[i] * log(pj[i]);
          p_u += pj[i] * u;
        } else {
          p_log_p += pj[i];   // (0, or the NaN of a NaN entry)
        }
      }
    }
    p_log_p = warp_sum(p_log_p);
    p_u = warp_sum(p_u);
    sum_e = (float)warp_sum(se);
    mass *= norm;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  // ---- listed places are taken out of the row
  if (warp == 0) {
#pragma unroll
    for (int i = 0; i < kListLanes; ++i) {
      if (id[i] < 0) continue;
      if (id[i] < sp.head) {
        atomicOr(&s_edge, 1u << id[i]);
      } else if (id[i] >= tail0) {
        atomicOr(&s_edge, 256u << (id[i] - tail0));
      } else {
        const int e = id[i] - sp.head - sp.v_lo * V16::kN;
        if (e >= 0 && e < n_vec * V16::kN) reinterpret_cast<T*>(s_row)[e] = V16::round(-INFINITY);
      }
    }
  }
  __syncthreads();
  const bool head_listed = has_head && (s_edge >> tid & 1u), tail_listed = has_tail && (s_edge >> (8 + tid) & 1u);
  if (head_listed) edge_head = -INFINITY;
  if (tail_listed) edge_tail = -INFINITY;
  // ---- maximum and sum of exponentials of the unlisted words
  MaxSum st{-FLT_MAX, 0.f};
  if (has_head || has_tail) {
    st.m = fmaxf(st.m, fmaxf(edge_head, edge_tail));
    if (has_head) st.s += row_ex2((edge_head - st.m) * c);
    if (has_tail) st.s += row_ex2((edge_tail - st.m) * c);
  }
  const unsigned long long c2 = f2_pack(c, c);
  constexpr int kUnroll = 4;
  for (int i = tid; i < n_vec; i += kUnroll * kRowThreads) {
    uint4 v[kUnroll];
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      v[u] = i + u * kRowThreads < n_vec
                 ? s_row[i + u * kRowThreads]
                 : make_uint4(V16::kNegInfWord, V16::kNegInfWord, V16::kNegInfWord, V16::kNegInfWord);
      top = fmaxf(top, V16::largest(v[u]));
    }
    if (top > st.m) {
      st.s *= row_ex2((st.m - top) * c);
      st.m = top;
    }
    const unsigned long long nm2 = f2_pack(-st.m, -st.m);
    unsigned long long s2 = f2_pack(st.s, 0.f);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
      for (int q = 0; q < V16::kN / 2; ++q) {
        float x0, x1;
        f2_unpack(f2_mul(f2_add(V16::pair(v[u], q), nm2), c2), x0, x1);
        s2 = f2_add(s2, f2_pack(row_ex2(x0), row_ex2(x1)));
      }
    }
    float s0, s1;
    f2_unpack(s2, s0, s1);
    st.s = s0 + s1;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    st = join(st, MaxSum{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o)}, c);
  if (lane == 0) s_warp[warp] = st;
  __syncthreads();
  if (C > 1) {
    if (tid == 0) {
      MaxSum x = s_warp[0];
      for (int r = 1; r < kRowWarps; ++r) x = join(x, s_warp[r], c);
      s_cta = x;
    }
    __syncthreads();
    cluster_arrive();
    cluster_wait();
  }
  // ---- the row's scalars (first warp of every CTA, the same arithmetic in the same order)
  float coef_listed = 0.f;    // beta q_j = coef_listed * e^{(z_j - z_ref) / T}
  if (warp == 0) {
    MaxSum x{-FLT_MAX, 0.f};
    if (C > 1) {
      if (lane < C) {
        const uint32_t a = cluster_addr(&s_cta, lane);
        x = MaxSum{cluster_load_f32(a), cluster_load_f32(a + 4)};
      }
    } else if (lane < kRowWarps) {
      x = s_warp[lane];
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
      x = join(x, MaxSum{__shfl_xor_sync(0xffffffffu, x.m, o), __shfl_xor_sync(0xffffffffu, x.s, o)}, c);
    x.m = __shfl_sync(0xffffffffu, x.m, 0);
    x.s = __shfl_sync(0xffffffffu, x.s, 0);
    const double T64 = (double)p.T;
    const float M = fmaxf(x.m, z_ref);
    const double du_rest = ((double)x.m - (double)M) / T64, du_list = ((double)z_ref - (double)M) / T64;
    const float w_rest = x.s > 0.f ? expf((float)du_rest) : x.s, w_list = expf((float)du_list);
    const double S = (double)w_rest * (double)x.s + (double)w_list * (double)sum_e;
    const double log_S = log(S);
    // - sum_j p_j log q_j = -( sum p_j (z_j - z_ref) / T + P (z_ref - M) / T - P log S )
    double loss = p_log_p - (p_u + mass * (du_list - log_S));
    double beta = mass, coef = 0.0;
    double rest = 0.0;
    if (p.tail) {
      rest = 1.0 - mass;
      if (rest < 0.0) rest = 0.0;
      beta = mass + rest;
      if (rest > 0.0) loss += rest * (log(rest) - (du_rest + log((double)x.s) - log_S));
    }
    if (x.s != 0.f) coef = beta * (double)w_rest / S - rest / (double)x.s;
    const bool none = S == 0.0;      // nothing but -inf in the row
    if (none) {
      coef = 0.0;
      loss = beta > 0.0 ? INFINITY : 0.0;
    }
    coef_listed = none ? 0.f : (float)(beta * (double)w_list / S);
    if (lane == 0) {
      s_coef = (float)(coef * (double)w / T64);
      s_ref = x.m;
      if (rank == 0 && p.loss) p.loss[t] = (float)loss;
    }
#pragma unroll
    for (int i = 0; i < kListLanes; ++i)
      if (none) pj[i] = 0.0;
  }
  __syncwarp();
  if (C > 1) cluster_arrive();   // this CTA is done with the others' shared memory (waited for before it ends)
  if (kGrad) {
    __syncthreads();
    const float coef = s_coef, ref = s_ref;
    if (has_head && !head_listed) out[tid] = V16::round(coef * row_ex2((edge_head - ref) * c));
    if (has_tail && !tail_listed) out[tail0 + tid] = V16::round(coef * row_ex2((edge_tail - ref) * c));
    const unsigned long long nm2 = f2_pack(-ref, -ref), k2 = f2_pack(coef, coef);
    T* out_vec = out + sp.head + (long long)sp.v_lo * V16::kN;
#pragma unroll 2
    for (int i = tid; i < n_vec; i += kRowThreads) {
      const uint4 v = s_row[i];
      float g[V16::kN];
#pragma unroll
      for (int q = 0; q < V16::kN / 2; ++q) {
        float x0, x1;
        f2_unpack(f2_mul(f2_add(V16::pair(v, q), nm2), c2), x0, x1);
        f2_unpack(f2_mul(f2_pack(row_ex2(x0), row_ex2(x1)), k2), g[2 * q], g[2 * q + 1]);
      }
      if (same_align) {
        *reinterpret_cast<uint4*>(out_vec + (long long)i * V16::kN) = V16::pack(g);
      } else {
#pragma unroll
        for (int q = 0; q < V16::kN; ++q) out_vec[(long long)i * V16::kN + q] = V16::round(g[q]);
      }
    }
    __syncthreads();
    // listed words: over the zeros the sweep has left in their places
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < kListLanes; ++i) {
        if (id[i] < 0) continue;
        const int e = id[i] - sp.head - sp.v_lo * V16::kN;
        const bool mine = id[i] < sp.head ? rank == 0 : id[i] >= tail0 ? rank == C - 1 : e >= 0 && e < n_vec * V16::kN;
        if (mine) {
          const double u = ((double)z[i] - (double)z_ref) / (double)p.T;
          const double d = (double)coef_listed * (double)expf((float)u) - pj[i];
          out[id[i]] = V16::round((float)(d * (double)w / (double)p.T));
        }
      }
    }
  }
  __syncwarp();
  if (C > 1) cluster_wait();
}

template <typename T, bool kGrad>
cudaError_t launch(dx_ctx* ctx, const DistillParams& p, cudaStream_t st) {
  // CTAs per row: few enough bytes per CTA that four fit an SM (one loads while another computes or stores), and as
  // many as fill the GPU when there are few rows
  const long long bytes = (long long)p.V * (long long)sizeof(T);
  const int slots = 4 * ctx->sm_count;
  int C = 1;
  while (C < DX_ROW_CLUSTER_MAX &&
         (bytes > (long long)C * DX_ROW_SLICE_BYTES ||
          ((long long)p.N * C * 2 <= slots && (long long)C * 2 * kRowThreads * 16 <= bytes)))
    C *= 2;
  const long long n_vec = bytes / 16 + 1;
  const size_t smem = (size_t)((n_vec + C - 1) / C + 1) * 16;
  return dx_launch_pdl(false, dx_distill_kernel<T, kGrad>, dim3((unsigned)p.N * C), dim3(kRowThreads), smem, st, C, p, C);
}

template <typename K>
cudaError_t prepare(K kernel, int smem) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  return e;
}

}  // namespace

// (2 KB of the opt-in limit stay for the kernel's static variables)
size_t dx_distill_max_row_bytes(const dx_ctx* ctx) {
  return (size_t)(ctx->smem_optin - 2048 - 64) * DX_ROW_CLUSTER_MAX;
}

cudaError_t dx_distill_prepare(const dx_ctx* ctx) {
  const int smem = ctx->smem_optin - 2048;
  cudaError_t e = prepare(dx_distill_kernel<float, true>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<float, false>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<__nv_bfloat16, true>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<__nv_bfloat16, false>, smem);
  return e;
}

cudaError_t dx_launch_distill(dx_ctx* ctx, const void* logits, int dtype, int N, int V, long long ld,
                              const int32_t* teacher_ids, const float* teacher_logprobs, int k, int tail,
                              float temperature, const float* row_weight, float* loss, void* dlogits, long long ld_d,
                              cudaStream_t st) {
  DistillParams p{logits, N, V, k, tail, ld, ld_d, teacher_ids, teacher_logprobs,
                  (float)(1.4426950408889634 / (double)temperature), temperature, row_weight, loss, dlogits,
                  ctx->dev_status};
  if (dtype == DX_DTYPE_FP32) return dlogits ? launch<float, true>(ctx, p, st) : launch<float, false>(ctx, p, st);
  return dlogits ? launch<__nv_bfloat16, true>(ctx, p, st) : launch<__nv_bfloat16, false>(ctx, p, st);
}
