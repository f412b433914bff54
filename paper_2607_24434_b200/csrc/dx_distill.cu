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
// words stand above the rest.  A bit per vector tells the sweep which vectors hold listed words; a small hash table says
// which of their elements, and those count as -inf.  A ninth warp does the arithmetic on the list while the other eight
// stream the row.  The warps' sums go straight into the shared memory of all CTAs of the row, so that one cluster
// barrier is all that stands between the sweep and the gradient.  Per-row scalars of the loss are 64-bit (it is a small
// difference of logarithms) and are not waited for by the gradient.
#include "dx_rows.cuh"

namespace {

constexpr int kUnroll = 2;
constexpr float kSlack = 8.f;                     // powers of two by which an element may exceed its sum's reference
constexpr int kStaticBytes = 5632;                // at least the kernel's static shared memory
constexpr int kLists = DX_MAX_TEACHER / 32;       // list entries per lane of the list's warp
constexpr int kHash = 2 * DX_MAX_TEACHER;
constexpr int kThreads = kRowThreads + 32;        // eight warps that stream, one that handles the list
constexpr int kWarps = kThreads / 32;

struct DistillParams {
  const void* logits;
  int N, V, k, tail;
  long long ld, ld_d;
  const int32_t* ids;
  const float* lp;
  float c, c_lo;              // log2(e) / T in two parts
  double inv_T;
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
// What the gradient needs to know of the list: the largest listed logit, sum_j e^{(z_j - z_ref) / T}, the teacher's mass
// with and of the tail bucket, and what its p_j are multiplied with.
struct ListSums {
  float z_ref, sum_e, beta, rest, norm;
};

__device__ __forceinline__ void copy16(uint4* dst_smem, const uint4* src) {
  const uint32_t d = static_cast<uint32_t>(__cvta_generic_to_shared(dst_smem));
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
}
// vector `v` with the elements in `drop` at -inf
template <typename T>
__device__ __forceinline__ void mask_vector(uint4& v, unsigned int drop) {
  uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (sizeof(T) == 4) {
      if (drop >> q & 1u) x[q] = 0xff800000u;
    } else {
      if (drop >> (2 * q) & 1u) x[q] = (x[q] & 0xffff0000u) | 0xff80u;
      if (drop >> (2 * q + 1) & 1u) x[q] = (x[q] & 0xffffu) | 0xff800000u;
    }
  }
  v = make_uint4(x[0], x[1], x[2], x[3]);
}

// (maximum, sum) of a warp's lanes; every lane gets them
__device__ __forceinline__ MaxSum warp_join(MaxSum x, float c) {
  const float m = warp_max(x.m);
  float s = x.s * row_ex2((x.m - m) * c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return MaxSum{m, s};
}

template <typename T, bool kGrad>
__global__ void __launch_bounds__(kThreads, 4) dx_distill_kernel(DistillParams p, int C) {
  using V16 = RowVec<T>;
  extern __shared__ uint4 s_row[];                 // (kGrad) the CTA's vectors of the row
  // bit q of a thread's pair of words: its q-th vector holds a listed word
  __shared__ __align__(16) unsigned int s_mark[2 * kRowThreads];
  __shared__ __align__(16) int s_key[kHash];                       // vectors that hold listed words (-1: free) ...
  __shared__ __align__(16) unsigned int s_drop[kHash];             // ... and which of their elements those are
  __shared__ MaxSum s_all[DX_ROW_CLUSTER_MAX * kWarps];   // sums of all warps of all CTAs of the row
  __shared__ ListSums s_list;
  __shared__ unsigned int s_edge;                  // head (bits 0..7) and tail (8..15) elements that are listed
  __shared__ int s_live;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool list_warp = warp == kRowWarps;
  const int rank = C > 1 ? (int)cluster_rank() : 0;
  const int t = blockIdx.x / C;
  const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
  T* out = kGrad ? reinterpret_cast<T*>(p.dlogits) + (size_t)t * (size_t)p.ld_d : nullptr;
  const RowSplit sp = row_split(row, p.V, rank, C);
  const int n_vec = sp.v_hi - sp.v_lo;
  const int tail0 = p.V - sp.tail;
  // gradient vectors can be stored as such where the output row is aligned like the input row
  const bool same_align = kGrad && ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row)) & 15u) == 0;
  const float c = p.c;
  if (C > 1) cluster_arrive();

  // ---- the row on its way into shared memory, in two parts that can be waited for one by one (every thread copies
  // what it reads itself); the list warp marks the listed words meanwhile
  const int deep = (n_vec + kRowThreads - 1) / kRowThreads;        // vectors of a thread, at most
  const int part = ((deep + 1) / 2 + kUnroll - 1) / kUnroll * kUnroll;
  int id[kLists];                                  // list warp: entry lane + 32 i
  float w;
  if (list_warp) {
#pragma unroll
    for (int i = 0; i < kLists; ++i) id[i] = lane + 32 * i < p.k ? p.ids[(size_t)t * p.k + lane + 32 * i] : -1;
    w = p.weight ? p.weight[t] : 1.f;
#pragma unroll
    for (int i = 0; i < 2 * kRowThreads / 128; ++i) reinterpret_cast<uint4*>(s_mark)[lane + 32 * i] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < kHash / 128; ++i) {
      reinterpret_cast<int4*>(s_key)[lane + 32 * i] = make_int4(-1, -1, -1, -1);
      reinterpret_cast<uint4*>(s_drop)[lane + 32 * i] = make_uint4(0, 0, 0, 0);
    }
    if (lane == 0) s_edge = 0;
    __syncwarp();
    bool live = false, bad = false;
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
      if (32 * i >= p.k) continue;
      bad |= id[i] < -1 || id[i] >= p.V;
      if (id[i] < 0 || id[i] >= p.V) id[i] = -1;
      live |= id[i] >= 0;
      // an id counts once, with its first entry: the first of equal lanes, and not if an earlier 32 have left its bit
      const unsigned int same = __match_any_sync(0xffffffffu, id[i]);
      if (__ffs(same) - 1 != lane) id[i] = -1;
      if (id[i] >= 0) {
        unsigned int bit, old;
        if (id[i] < sp.head) {
          bit = 1u << id[i];
          old = atomicOr(&s_edge, bit);
        } else if (id[i] >= tail0) {
          bit = 256u << (id[i] - tail0);
          old = atomicOr(&s_edge, bit);
        } else {
          const int x = (id[i] - sp.head) / V16::kN;
          int h = x & (kHash - 1);
          for (int tries = 0; tries < kHash; ++tries) {   // (at most kHash / 2 keys: a free or equal one is found)
            const int key = atomicCAS(&s_key[h], -1, x);
            if (key == -1 || key == x) break;
            h = (h + 1) & (kHash - 1);
          }
          bit = 1u << ((id[i] - sp.head) % V16::kN);
          old = atomicOr(&s_drop[h], bit);
          const int mine = x - sp.v_lo;
          if (mine >= 0 && mine < n_vec) {
            const int q = mine / kRowThreads;
            atomicOr(&s_mark[2 * (mine % kRowThreads) + (q >> 5)], 1u << (q & 31));
          }
        }
        if (old & bit) id[i] = -1;
      }
      __syncwarp();
    }
    if (bad && rank == 0) *p.dev_status = DX_DEV_BAD_TOKEN;
    live = __any_sync(0xffffffffu, live);
    if (lane == 0) s_live = live;
  } else {
    if (kGrad) {
      const uint4* src = reinterpret_cast<const uint4*>(row + sp.head) + sp.v_lo;
#pragma unroll 4
      for (int q = 0; q < deep; ++q) {
        if (q == part) asm volatile("cp.async.commit_group;" ::: "memory");
        if (tid + q * kRowThreads < n_vec) copy16(s_row + tid + q * kRowThreads, src + tid + q * kRowThreads);
      }
      if (part >= deep) asm volatile("cp.async.commit_group;" ::: "memory");
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    w = p.weight ? p.weight[t] : 1.f;
  }
  __syncthreads();
  if (w == 0.f || !s_live) {   // (the same for every CTA of the row) nothing to learn: the logits do not matter
    if (rank == 0 && tid == 0 && p.loss) p.loss[t] = 0.f;
    if (kGrad) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncthreads();         // (in place: nobody overwrites what is still being copied)
      if (rank == 0 && tid < sp.head) out[tid] = V16::round(0.f);
      if (rank == C - 1 && tid < sp.tail) out[tail0 + tid] = V16::round(0.f);
      for (int i = tid; i < n_vec; i += kThreads) {
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
  const unsigned int edge = s_edge;
  const bool head_in = !list_warp && rank == 0 && tid < sp.head && !(edge >> tid & 1u);      // this thread's unlisted
  const bool tail_in = !list_warp && rank == C - 1 && tid < sp.tail && !(edge >> (8 + tid) & 1u);   // edge elements
  float edge_head = -INFINITY, edge_tail = -INFINITY;
  MaxSum st{-FLT_MAX, 0.f};
  const unsigned long long c2 = f2_pack(c, c);
  float pj[kLists], e[kLists];                     // list warp: p_j, e^{(z_j - z_ref) / T}
  double mass = 0.0, p_log_p = 0.0, p_u = 0.0;     // ... and, in the first CTA, sums over the list
  if (!list_warp) {
    // ---- maximum and sum of exponentials of the unlisted words
    const unsigned long long cl2 = f2_pack(p.c_lo, p.c_lo);
    const uint2 marks = *reinterpret_cast<const uint2*>(s_mark + 2 * tid);
    const uint4 none4 = make_uint4(V16::kNegInfWord, V16::kNegInfWord, V16::kNegInfWord, V16::kNegInfWord);
    unsigned long long s2 = f2_pack(0.f, 0.f);
    // All warps start from the largest unlisted element of their first chunk as the reference of the exponents; a thread
    // takes another only when it meets an element more than 2^kSlack times as likely.
#pragma unroll 1
    for (int q = 0, arrived = 0; q < deep; q += kUnroll) {
      if (kGrad && q >= arrived) {
        if (arrived == 0) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        arrived = arrived == 0 ? part : deep;
      }
      uint4 v[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = tid + (q + u) * kRowThreads;
        v[u] = none4;                                // (adds nothing)
        if (i < n_vec) v[u] = kGrad ? s_row[i] : row_vec_stream(row, sp, sp.v_lo + i);
      }
      const unsigned int marked = (q < 32 ? marks.x >> q : marks.y >> (q - 32)) & ((1u << kUnroll) - 1u);
      if (marked) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          if (marked >> u & 1u) {
            const int vec = sp.v_lo + tid + (q + u) * kRowThreads;
            int h = vec & (kHash - 1);
            for (int tries = 0; tries < kHash && s_key[h] != vec; ++tries) h = (h + 1) & (kHash - 1);
            mask_vector<T>(v[u], s_drop[h]);
          }
        }
      }
      const float top = V16::largest(v, kUnroll);
      if (q == 0) {
        st.m = fmaxf(warp_max(top), -FLT_MAX);
      } else if ((top - st.m) * c > kSlack) {
        float s0, s1;
        f2_unpack(s2, s0, s1);
        s2 = f2_pack((s0 + s1) * row_ex2((st.m - top) * c), 0.f);
        st.m = top;
      }
      const unsigned long long nm2 = f2_pack(-st.m, -st.m);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
        for (int h = 0; h < V16::kN / 2; ++h) {
          // (the factor in two parts: rounded to one, it would shift the exponents of all words the same way)
          const unsigned long long d2 = f2_add(V16::pair(v[u], h), nm2);
          float x0, x1;
          f2_unpack(f2_fma(d2, cl2, f2_mul(d2, c2)), x0, x1);
          s2 = f2_add(s2, f2_pack(row_ex2(x0), row_ex2(x1)));
        }
      }
    }
    float s0, s1;
    f2_unpack(s2, s0, s1);
    st.s = s0 + s1;
    if (head_in || tail_in) {
      edge_head = head_in ? V16::load(row + tid) : -INFINITY;
      edge_tail = tail_in ? V16::load(row + tail0 + tid) : -INFINITY;
      const float top = fmaxf(edge_head, edge_tail);
      if (top > st.m) {
        st.s *= row_ex2((st.m - top) * c);
        st.m = top;
      }
      if (head_in) st.s += row_ex2((edge_head - st.m) * c);
      if (tail_in) st.s += row_ex2((edge_tail - st.m) * c);
    }
    st = warp_join(st, c);
  } else {
    // ---- the list (log p_j is what the caller has given)
    float z[kLists], lp[kLists], top = -FLT_MAX;
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
      z[i] = id[i] >= 0 ? V16::load(row + id[i]) : -INFINITY;
      lp[i] = id[i] >= 0 ? p.lp[(size_t)t * p.k + lane + 32 * i] : -INFINITY;
      top = fmaxf(top, z[i]);
    }
    ListSums l{warp_max(top), 0.f, 0.f, 0.f, 1.f};
    double se = 0.0;
#pragma unroll
    for (int i = 0; i < kLists; ++i) {
      e[i] = pj[i] = 0.f;
      if (32 * i >= p.k) continue;
      const double u = ((double)z[i] - (double)l.z_ref) * p.inv_T;
      e[i] = id[i] >= 0 ? expf((float)u) : 0.f;
      const double pd = exp((double)lp[i]);          // (a NaN entry makes the mass NaN, and with it the loss)
      pj[i] = (float)pd;
      se += (double)e[i];
      mass += pd;
      if (pd > 0.0) {
        p_log_p += pd * (double)lp[i];
        p_u += pd * u;
      }
    }
    se = warp_sum(se);
    mass = warp_sum(mass);
    p_log_p = warp_sum(p_log_p);
    p_u = warp_sum(p_u);
    if (!p.tail && mass != 0.0) {                    // p' = p / mass:  sum p' log p' = (sum p log p) / mass - log mass
      const double norm = 1.0 / mass;
      l.norm = (float)norm;
      p_log_p = p_log_p * norm - log(mass);
      p_u *= norm;
      mass = mass == mass ? 1.0 : mass;
    }
    const double rest = p.tail && mass < 1.0 ? 1.0 - mass : 0.0;
    l.sum_e = (float)se;
    l.beta = (float)(mass + rest);
    l.rest = (float)rest;
    if (lane == 0) s_list = l;
  }
  // ---- sums of the warp, to all CTAs of the row (the list warp has none)
  if (C > 1) {
    __syncwarp();
    cluster_wait();                                  // (all CTAs of the row have started)
    if (!list_warp && lane < C) {
      const uint32_t a = cluster_addr(&s_all[rank * kRowWarps + warp], lane);
      cluster_store_f32(a, st.m);
      cluster_store_f32(a + 4, st.s);
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
  } else {
    if (!list_warp && lane == 0) s_all[warp] = st;
    __syncthreads();
  }
  // ---- the row's scalars (every warp, the same arithmetic in the same order)
  MaxSum x{-FLT_MAX, 0.f};
  for (int i = lane; i < C * kRowWarps; i += 32) x = join(x, s_all[i], c);
  x = warp_join(x, c);
  const ListSums l = s_list;
  const float M = fmaxf(x.m, l.z_ref);
  // (fp32: the gradient's factors; a sum that is NaN stays NaN)
  const float w_rest = x.s > 0.f ? row_ex2((x.m - M) * c) : x.s;
  const float w_list = row_ex2((l.z_ref - M) * c);
  const float S = w_rest * x.s + w_list * l.sum_e;
  const float scale = w * (float)p.inv_T;
  if (kGrad && !list_warp) {
    float coef = 0.f;
    if (x.s != 0.f && S != 0.f) coef = (l.beta * w_rest / S - l.rest / x.s) * scale;
    if (head_in) out[tid] = V16::round(coef * row_ex2((edge_head - x.m) * c));
    if (tail_in) out[tail0 + tid] = V16::round(coef * row_ex2((edge_tail - x.m) * c));
    const unsigned long long nm2 = f2_pack(-x.m, -x.m), k2 = f2_pack(coef, coef);
    T* out_vec = out + sp.head + (long long)sp.v_lo * V16::kN;
    auto gradient = [&](const uint4& y, float (&g)[V16::kN]) {
#pragma unroll
      for (int q = 0; q < V16::kN / 2; ++q) {
        float x0, x1;
        f2_unpack(f2_mul(f2_add(V16::pair(y, q), nm2), c2), x0, x1);
        f2_unpack(f2_mul(f2_pack(row_ex2(x0), row_ex2(x1)), k2), g[2 * q], g[2 * q + 1]);
      }
    };
    if (same_align) {
#pragma unroll 2
      for (int i = tid; i < n_vec; i += kRowThreads) {
        float g[V16::kN];
        gradient(s_row[i], g);
        *reinterpret_cast<uint4*>(out_vec + (long long)i * V16::kN) = V16::pack(g);
      }
    } else {
#pragma unroll 1
      for (int i = tid; i < n_vec; i += kRowThreads) {
        float g[V16::kN];
        gradient(s_row[i], g);
#pragma unroll
        for (int q = 0; q < V16::kN; ++q) out_vec[(long long)i * V16::kN + q] = V16::round(g[q]);
      }
    }
  }
  if (list_warp && rank == 0 && p.loss) {
    const double du_rest = ((double)x.m - (double)M) * p.inv_T, du_list = ((double)l.z_ref - (double)M) * p.inv_T;
    const double S64 = (x.s > 0.f ? exp(du_rest) : 1.0) * (double)x.s + exp(du_list) * (double)l.sum_e;
    const double log_S = log(S64);
    const double rest = p.tail && mass < 1.0 ? 1.0 - mass : 0.0;
    // - sum_j p_j log q_j = -( sum p_j (z_j - z_ref) / T + P (z_ref - M) / T - P log S )
    double loss = p_log_p - (p_u + (mass != 0.0 ? mass * (du_list - log_S) : 0.0));
    if (rest > 0.0) loss += rest * (log(rest) - (du_rest + log((double)x.s) - log_S));
    if (S64 == 0.0) loss = mass + rest > 0.0 ? INFINITY : 0.0;   // nothing but -inf in the row
    if (lane == 0) p.loss[t] = (float)loss;
  }
  if (kGrad) {
    if (list_warp) {                                 // gradients of this CTA's listed words
      const float f = S == 0.f ? 0.f : l.beta * w_list / S;
#pragma unroll
      for (int i = 0; i < kLists; ++i) {
        e[i] = S == 0.f ? 0.f : (f * e[i] - pj[i] * l.norm) * scale;
        const int v_at = (id[i] - sp.head) / V16::kN - sp.v_lo;
        if (id[i] < sp.head ? rank != 0 : id[i] >= tail0 ? rank != C - 1 : v_at < 0 || v_at >= n_vec) id[i] = -1;
      }
    }
    __syncthreads();
    // ... over what the sweep has left in their places
    if (list_warp) {
#pragma unroll
      for (int i = 0; i < kLists; ++i)
        if (id[i] >= 0) out[id[i]] = V16::round(e[i]);
    }
  }
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
  const size_t smem = kGrad ? (size_t)slice * 16 : 0;
  return dx_launch_pdl(false, dx_distill_kernel<T, kGrad>, dim3((unsigned)p.N * C), dim3(kThreads), smem, st, C, p, C);
}

template <typename K>
cudaError_t prepare(K kernel, int smem) {
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  return e;
}

}  // namespace

size_t dx_distill_max_row_bytes(const dx_ctx* ctx) {
  return (size_t)(ctx->smem_optin - kStaticBytes - 16) * DX_ROW_CLUSTER_MAX;
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
                  (float)c, (float)(c - (double)(float)c), 1.0 / (double)temperature, row_weight, loss, dlogits, ctx->dev_status};
  if (dtype == DX_DTYPE_FP32) return dlogits ? launch<float, true>(ctx, p, st) : launch<float, false>(ctx, p, st);
  return dlogits ? launch<__nv_bfloat16, true>(ctx, p, st) : launch<__nv_bfloat16, false>(ctx, p, st);
}
