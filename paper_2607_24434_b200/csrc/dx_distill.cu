// Distillation from a teacher's top log probabilities (Eq. 8 with the teacher cut to a short list), per row t:
//   q = softmax(z / T);  p_j = e^{l_j} over the listed words, renormalised to sum 1 or -- with the tail bucket -- as they
//   are, the rest r = 1 - sum p in one bucket that is compared with R = sum of q over the unlisted words:
//     L = sum_j p_j (log p_j - log q_j)  [ + r (log r - log R) ]
//     dL/dz_v = ( beta q_v - p_v ) / T  for listed v,   ( beta - r / R ) q_v / T  otherwise,  beta = sum p + r
// One launch reads each logit once and writes each gradient once: a cluster of CTAs holds the row in shared memory
// between the statistics and the gradient.
//
// The unlisted words are summed apart from the listed ones, relative to their own maximum: R never comes out of a
// difference of nearly equal sums, and neither R nor the factor r / R can under- or overflow however far the listed
// words stand above the rest.  The sweep leaves vectors that hold a listed word out (a bit per vector says so); a thread
// per list entry adds what else is in them afterwards.  Per-row scalars (teacher mass, loss) are 64-bit: the loss is a
// small difference of logarithms.
#include "dx_rows.cuh"

namespace {

constexpr int kUnroll = 4;
constexpr int kStaticBytes = 1024;                // at least the kernel's static shared memory
constexpr int kListWarps = DX_MAX_TEACHER / 32;   // thread j < k has list entry j

struct DistillParams {
  const void* logits;
  int N, V, k, tail;
  long long ld, ld_d;
  const int32_t* ids;
  const float* lp;
  float c, c_lo, T;           // log2(e) / T in two parts, T
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

// What the list entries of one warp contribute, relative to the warp's largest listed logit (unnormalised p).
struct ListPart {
  double mass, p_log_p, p_u, sum_e;
  float z_ref;
  int pad;
};

template <typename T, bool kGrad>
__global__ void __launch_bounds__(kRowThreads, 4) dx_distill_kernel(DistillParams p, int C) {
  using V16 = RowVec<T>;
  extern __shared__ uint4 s_dyn[];                 // bit u of byte [chunk][thread]: vector u of that chunk holds a listed
  unsigned int* s_mark = reinterpret_cast<unsigned int*>(s_dyn);   // word; behind it (kGrad) the CTA's vectors of the row
  __shared__ MaxSum s_warp[kRowWarps];
  __shared__ MaxSum s_cta;
  __shared__ ListPart s_list[kListWarps];
  __shared__ int s_ids[DX_MAX_TEACHER];
  __shared__ float s_coef, s_ref, s_max;
  __shared__ double s_norm, s_beta;
  __shared__ unsigned int s_edge;                  // head (bits 0..7) and tail (8..15) elements that are listed
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = C > 1 ? (int)cluster_rank() : 0;
  const int t = blockIdx.x / C;
  const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
  T* out = kGrad ? reinterpret_cast<T*>(p.dlogits) + (size_t)t * (size_t)p.ld_d : nullptr;
  const RowSplit sp = row_split(row, p.V, rank, C);
  const int n_vec = sp.v_hi - sp.v_lo;
  const int chunks = (n_vec + kUnroll * kRowThreads - 1) / (kUnroll * kRowThreads);
  uint4* s_row = s_dyn + chunks * (kRowThreads / 16);
  const bool has_head = rank == 0 && tid < sp.head, has_tail = rank == C - 1 && tid < sp.tail;
  const int tail0 = p.V - sp.tail;
  // gradient vectors can be stored as such where the output row is aligned like the input row
  const bool same_align = kGrad && ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row)) & 15u) == 0;
  const float c = p.c;
  const float w = p.weight ? p.weight[t] : 1.f;

  // ---- the teacher's list
  int id = -1;
  if (tid < p.k) {
    id = p.ids[(size_t)t * p.k + tid];
    if (id < -1 || id >= p.V) {
      if (rank == 0) *p.dev_status = DX_DEV_BAD_TOKEN;
      id = -1;
    }
  }
  for (int i = tid; i < chunks * (kRowThreads / 4); i += kRowThreads) s_mark[i] = 0;
  if (tid < DX_MAX_TEACHER) s_ids[tid] = id;
  if (tid == 0) s_edge = 0;
  const int live = __syncthreads_or(id >= 0);
  if (w == 0.f || !live) {   // (the same for every CTA of the row) nothing to learn: the logits are not looked at
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
  // marks; `vec` is the slice's vector an entry lies in (-1: not this CTA's, or a head / tail element)
  int vec = -1;
  bool mine = false;
  if (id >= 0) {
    if (id < sp.head) {
      mine = rank == 0;
      atomicOr(&s_edge, 1u << id);
    } else if (id >= tail0) {
      mine = rank == C - 1;
      atomicOr(&s_edge, 256u << (id - tail0));
    } else {
      const int v = (id - sp.head) / V16::kN - sp.v_lo;
      mine = v >= 0 && v < n_vec;
      if (mine) vec = v;
    }
  }
  const int m_byte = vec / (kUnroll * kRowThreads) * kRowThreads + vec % kRowThreads;     // (of entries with vec >= 0)
  const unsigned int m_bit = 1u << ((m_byte & 3) * 8 + vec / kRowThreads % kUnroll);
  if (vec >= 0) atomicOr(&s_mark[m_byte >> 2], m_bit);
  // an id counts once, with its first entry
  if (warp * 32 < p.k) {
    const unsigned int same = __match_any_sync(0xffffffffu, id);
    if (__ffs(same) - 1 != lane) id = -1;
    for (int j = 0; j < warp * 32; ++j)
      if (s_ids[j] == id) id = -1;
  }
  if (id < 0) {
    mine = false;
    vec = -1;
  }
  float z = -INFINITY;
  double pj = 0.0;
  if (id >= 0 && (mine || rank == 0)) {
    z = V16::load(row + id);
    pj = exp((double)p.lp[(size_t)t * p.k + tid]);
  }
  if (rank == 0 && warp * 32 < p.k) {
    const float z_ref = fmaxf(warp_max(z), -FLT_MAX);
    const double u = ((double)z - (double)z_ref) / (double)p.T;
    const double se = warp_sum(id >= 0 ? (double)expf((float)u) : 0.0);
    const double mass = warp_sum(pj);
    const bool has = pj > 0.0;                        // (a NaN entry makes the mass NaN, and with it the loss)
    const double plp = warp_sum(has ? pj * log(pj) : 0.0), pu = warp_sum(has ? pj * u : 0.0);
    if (lane == 0) s_list[warp] = ListPart{mass, plp, pu, se, z_ref, 0};
  }
  __syncthreads();
  const unsigned int edge = s_edge;
  const bool head_listed = has_head && (edge >> tid & 1u), tail_listed = has_tail && (edge >> (8 + tid) & 1u);
  // ---- maximum and sum of exponentials of the unlisted words
  MaxSum st{-FLT_MAX, 0.f};
  const unsigned long long c2 = f2_pack(c, c), cl2 = f2_pack(p.c_lo, p.c_lo);
  const float edge_head = has_head ? V16::load(row + tid) : -INFINITY;
  const float edge_tail = has_tail ? V16::load(row + tail0 + tid) : -INFINITY;
  auto single = [&](float x) {
    if (x > st.m) {
      st.s *= row_ex2((st.m - x) * c);
      st.m = x;
    }
    st.s += row_ex2((x - st.m) * c);
  };
  if (has_head && !head_listed) single(edge_head);
  if (has_tail && !tail_listed) single(edge_tail);
  unsigned long long s2 = f2_pack(st.s, 0.f);
  auto add = [&](const uint4* v, int n_v, unsigned int skip) {
    float top;
    if (skip == 0) {
      top = V16::largest(v, n_v);
    } else {
      top = -INFINITY;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (u < n_v && !(skip >> u & 1u)) top = fmaxf(top, V16::largest(v[u]));
    }
    if (top > st.m) {
      float s0, s1;
      f2_unpack(s2, s0, s1);
      s2 = f2_pack((s0 + s1) * row_ex2((st.m - top) * c), 0.f);
      st.m = top;
    }
    const unsigned long long nm2 = f2_pack(-st.m, -st.m);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (u < n_v && !(skip >> u & 1u)) {
#pragma unroll
        for (int q = 0; q < V16::kN / 2; ++q) {
          // (the factor in two parts: rounded to one, it would shift the exponents of all words the same way)
          const unsigned long long d2 = f2_add(V16::pair(v[u], q), nm2);
          float x0, x1;
          f2_unpack(f2_fma(d2, cl2, f2_mul(d2, c2)), x0, x1);
          s2 = f2_add(s2, f2_pack(row_ex2(x0), row_ex2(x1)));
        }
      }
    }
  };
  for (int ch = 0, i = tid; ch < chunks; ++ch, i += kUnroll * kRowThreads) {
    const unsigned int skip = reinterpret_cast<const unsigned char*>(s_mark)[ch * kRowThreads + tid];
    uint4 v[kUnroll];
    if (i + (kUnroll - 1) * kRowThreads < n_vec) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) v[u] = row_vec_stream(row, sp, sp.v_lo + i + u * kRowThreads);
      if (kGrad) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) s_row[i + u * kRowThreads] = v[u];
      }
      add(v, kUnroll, skip);
    } else {
#pragma unroll
      for (int u = 0; u < kUnroll - 1; ++u)
        if (i + u * kRowThreads < n_vec) v[u] = row_vec_stream(row, sp, sp.v_lo + i + u * kRowThreads);
#pragma unroll
      for (int u = 0; u < kUnroll - 1; ++u) {
        if (i + u * kRowThreads < n_vec) {
          if (kGrad) s_row[i + u * kRowThreads] = v[u];
          if (!(skip >> u & 1u)) add(v + u, 1, 0);
        }
      }
    }
  }
  {
    float s0, s1;
    f2_unpack(s2, s0, s1);
    st.s = s0 + s1;
  }
  __syncthreads();
  // ---- the vectors left out: the first entry that lies in one takes it
  if (vec >= 0 && (atomicAnd(&s_mark[m_byte >> 2], ~m_bit) & m_bit)) {
    const uint4 v = row_vec_stream(row, sp, sp.v_lo + vec);
    const int e0 = sp.head + (sp.v_lo + vec) * V16::kN;
    unsigned int listed = 0;
    for (int j = 0; j < p.k; ++j) {
      const int e = s_ids[j] - e0;
      if (e >= 0 && e < V16::kN) listed |= 1u << e;
    }
#pragma unroll
    for (int q = 0; q < V16::kN / 2; ++q) {
      float x0, x1;
      f2_unpack(V16::pair(v, q), x0, x1);
      if (!(listed >> (2 * q) & 1u)) single(x0);
      if (!(listed >> (2 * q + 1) & 1u)) single(x1);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    st = join(st, MaxSum{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o)}, c);
  if (lane == 0) s_warp[warp] = st;
  __syncthreads();
  if (C > 1) {
    if (warp == 0) {
      MaxSum x = lane < kRowWarps ? s_warp[lane] : MaxSum{-FLT_MAX, 0.f};
#pragma unroll
      for (int o = kRowWarps / 2; o > 0; o >>= 1)
        x = join(x, MaxSum{__shfl_xor_sync(0xffffffffu, x.m, o), __shfl_xor_sync(0xffffffffu, x.s, o)}, c);
      if (lane == 0) s_cta = x;
      __syncwarp();
    }
    cluster_arrive();
    cluster_wait();
  }
  // ---- the row's scalars (first warp of every CTA, the same arithmetic in the same order)
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
    // the list's parts (the first CTA has them)
    double mass = 0.0, p_log_p = 0.0, p_u = 0.0, sum_e = 0.0;
    float z_ref = -FLT_MAX;
    if (lane < kListWarps && lane * 32 < p.k) {
      if (C > 1) {
        const uint32_t a = cluster_addr(&s_list[lane], 0);
        mass = cluster_load_f64(a);
        p_log_p = cluster_load_f64(a + 8);
        p_u = cluster_load_f64(a + 16);
        sum_e = cluster_load_f64(a + 24);
        z_ref = cluster_load_f32(a + 32);
      } else {
        const ListPart l = s_list[lane];
        mass = l.mass; p_log_p = l.p_log_p; p_u = l.p_u; sum_e = l.sum_e; z_ref = l.z_ref;
      }
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
      x = join(x, MaxSum{__shfl_xor_sync(0xffffffffu, x.m, o), __shfl_xor_sync(0xffffffffu, x.s, o)}, c);
    x.m = __shfl_sync(0xffffffffu, x.m, 0);
    x.s = __shfl_sync(0xffffffffu, x.s, 0);
    const double T64 = (double)p.T;
    const float M = fmaxf(x.m, warp_max(z_ref));
    // list sums relative to M
    const double du = ((double)z_ref - (double)M) / T64;
    sum_e = sum_e > 0.0 || sum_e != sum_e ? sum_e * exp(du) : 0.0;
    p_u += mass > 0.0 ? mass * du : 0.0;
#pragma unroll
    for (int o = kListWarps / 2; o > 0; o >>= 1) {
      mass += __shfl_xor_sync(0xffffffffu, mass, o);
      p_log_p += __shfl_xor_sync(0xffffffffu, p_log_p, o);
      p_u += __shfl_xor_sync(0xffffffffu, p_u, o);
      sum_e += __shfl_xor_sync(0xffffffffu, sum_e, o);
    }
    if (lane == 0) {
      double norm = 1.0;
      if (!p.tail && mass != 1.0 && mass != 0.0) {    // p' = norm p:  sum p' log p' = norm (sum p log p + mass log norm)
        norm = 1.0 / mass;
        p_log_p = norm * (p_log_p - mass * log(mass));
        p_u *= norm;
        mass = mass == mass ? 1.0 : mass;
      }
      const double du_rest = ((double)x.m - (double)M) / T64;
      const double w_rest = x.s > 0.f ? exp(du_rest) : (double)x.s;
      const double S = w_rest * (double)x.s + sum_e;
      const double log_S = log(S);
      double loss = p_log_p - (p_u - mass * log_S);
      double rest = 0.0, coef = 0.0;
      if (p.tail) {
        rest = 1.0 - mass;
        if (rest < 0.0) rest = 0.0;
        if (rest > 0.0) loss += rest * (log(rest) - (du_rest + log((double)x.s) - log_S));
      }
      const double beta = mass + rest;
      if (x.s != 0.f) coef = beta * w_rest / S - rest / (double)x.s;
      double listed = beta / S;
      if (S == 0.0) {                                 // nothing but -inf in the row
        listed = coef = norm = 0.0;
        loss = beta > 0.0 ? INFINITY : 0.0;
      }
      s_coef = (float)(coef * (double)w / T64);
      s_ref = x.m;
      s_max = M;
      s_norm = norm;
      s_beta = listed;
      if (rank == 0 && p.loss) p.loss[t] = (float)loss;
    }
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
    // listed words: over what the sweep has left in their places
    if (mine) {
      const double u = ((double)z - (double)s_max) / (double)p.T;
      const double d = (z == -INFINITY ? 0.0 : s_beta * exp(u)) - pj * s_norm;
      out[id] = V16::round((float)(d * (double)w / (double)p.T));
    }
  }
  __syncwarp();
  if (C > 1) cluster_wait();
}

template <typename T, bool kGrad>
cudaError_t launch(dx_ctx* ctx, const DistillParams& p, cudaStream_t st) {
  // CTAs per row: few enough bytes per CTA that four fit an SM (one loads while another computes or stores), and as many
  // as fill the GPU when there are few rows.  (Without the gradient nothing has to fit; the same split gives the same
  // loss, bit for bit.)
  const long long bytes = (long long)p.V * (long long)sizeof(T);
  const int slots = 4 * ctx->sm_count;
  int C = 1;
  while (C < DX_ROW_CLUSTER_MAX &&
         (bytes > (long long)C * DX_ROW_SLICE_BYTES ||
          ((long long)p.N * C * 2 <= slots && (long long)C * 2 * kRowThreads * 16 <= bytes)))
    C *= 2;
  const long long slice = (bytes / 16 + C - 1) / C;      // vectors of a CTA, at most
  const long long chunks = (slice + kUnroll * kRowThreads - 1) / (kUnroll * kRowThreads);
  const size_t smem = (size_t)(chunks * kRowThreads + (kGrad ? slice * 16 : 0));
  return dx_launch_pdl(false, dx_distill_kernel<T, kGrad>, dim3((unsigned)p.N * C), dim3(kRowThreads), smem, st, C, p, C);
}

template <typename K>
cudaError_t prepare(K kernel, int smem) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  return e;
}

}  // namespace

// (of the opt-in limit 1 KB stays for the kernel's static variables, 4 KB for the marks: a byte per 64 of the row)
size_t dx_distill_max_row_bytes(const dx_ctx* ctx) {
  return (size_t)(ctx->smem_optin - kStaticBytes - 4096) * DX_ROW_CLUSTER_MAX;
}

cudaError_t dx_distill_prepare(const dx_ctx* ctx) {
  const int smem = ctx->smem_optin - kStaticBytes;
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
  const double c = 1.4426950408889634 / (double)temperature;
  DistillParams p{logits, N, V, k, tail, ld, ld_d, teacher_ids, teacher_logprobs,
                  (float)c, (float)(c - (double)(float)c), temperature, row_weight, loss, dlogits, ctx->dev_status};
  if (dtype == DX_DTYPE_FP32) return dlogits ? launch<float, true>(ctx, p, st) : launch<float, false>(ctx, p, st);
  return dlogits ? launch<__nv_bfloat16, true>(ctx, p, st) : launch<__nv_bfloat16, false>(ctx, p, st);
}
