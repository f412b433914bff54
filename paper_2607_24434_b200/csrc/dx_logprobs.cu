// Log probabilities of given tokens, entropy and the most likely alternatives of rows of logits:
//   u_v = (z_v - max z) / T,  S = sum_v e^{u_v},  log p_v = u_v - log S,  H = log S - (sum_v u_v e^{u_v}) / S.
// (Both terms of H are non-negative, nothing cancels.)  The n alternatives are the largest z, ties to the lower id.
//
// One pass: every logit is read from HBM once.  Threads carry (running maximum, S, sum u e^u); a chunk of four
// 16-byte vectors shares one rescaling.  Alternatives ride along as each thread's largest logit and the vector it
// sits in.  Of those, one warp picks a threshold that at least n and at most kFlagCap threads reach; only elements of
// these threads can be among the n largest, so they alone are read again (from L2) against the threshold, and the few
// elements that pass are ranked by counting.  A row of few-row calls is split over a cluster of up to 16 CTAs, whose
// statistics and candidate lists the first CTA joins through distributed shared memory: no workspace, no atomics
// on device memory, one launch, the same result on every run.
#include "dx_rows.cuh"

namespace {

constexpr int kUnroll = 4;
constexpr int kFlagCap = 64;      // threads whose elements are looked at again
constexpr int kCandCap = 1024;    // elements that may pass the threshold before the slow path takes over

struct LogprobParams {
  const void* logits;
  int N, V, n_top;
  long long ld;
  const int32_t* tokens;
  float c, T;                     // log2(e) / T, T
  float* logprob;
  float* entropy;
  int32_t* top_ids;
  float* top_logprobs;
  int32_t* dev_status;
};

// (value, index) as one integer, larger = earlier: higher value, then lower index.  Zero means "no element".
// -0 counts as +0; a NaN comes after -inf.
__device__ __forceinline__ unsigned long long top_key(float v, int idx) {
  const unsigned int hi = v == v ? dx_orderable(v + 0.f) : 0x007ffffeu;
  return ((unsigned long long)hi << 32) | (unsigned long long)(~(unsigned int)idx);
}
__device__ __forceinline__ float key_value(unsigned long long key) {
  const unsigned int u = (unsigned int)(key >> 32);
  if (u == 0x007ffffeu) return __uint_as_float(0x7fc00000u);
  return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u);
}

struct Stats {
  float m, s, a;   // maximum, sum of e^u, sum of (z - m) e^u
};
// brings the sums to another reference maximum m >= st.m (NaN sums stay NaN).  Where the factor vanishes so does the
// old sum: the distance may then be as large as that of a mask of the type's lowest value, and is not multiplied out.
__device__ __forceinline__ void rebase(Stats& st, float m, float c) {
  const float d = st.m - m, f = row_ex2(d * c);
  st.a = f > 0.f ? fmaf(d, st.s, st.a) * f : 0.f;
  st.s *= f;
  st.m = m;
}
__device__ __forceinline__ Stats join(Stats x, Stats y, float c) {
  const float m = fmaxf(x.m, y.m);
  rebase(x, m, c);
  rebase(y, m, c);
  return Stats{m, x.s + y.s, x.a + y.a};
}

template <typename T>
__device__ __forceinline__ float element(const T* row, long long i) { return RowVec<T>::load(row + i); }

template <typename T>
__device__ __forceinline__ uint4 row_vec(const T* row, const RowSplit& sp, int v) {
  return __ldg(reinterpret_cast<const uint4*>(row + sp.head) + v);
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads, 4) dx_logprobs_kernel(LogprobParams p, int C) {
  using V16 = RowVec<T>;
  __shared__ Stats s_warp[kRowWarps];
  __shared__ Stats s_cta;
  __shared__ unsigned long long s_keys[kRowThreads];
  __shared__ unsigned long long s_cand[kCandCap];
  __shared__ unsigned long long s_top[DX_MAX_TOP];
  __shared__ unsigned long long s_tau;
  __shared__ int s_flag[kFlagCap];
  __shared__ int s_nflag, s_ncand;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = C > 1 ? (int)cluster_rank() : 0;
  const int t = blockIdx.x / C;
  const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
  const RowSplit sp = row_split(row, p.V, rank, C);
  const float c = p.c;

  // ---- the pass over the row
  Stats st{-FLT_MAX, 0.f, 0.f};
  float best = -INFINITY;
  int pos = -1;                   // of `best`: vector >= 0, or -2 - element for a head / tail element
  // the head and the tail element of this thread, if any; a thread meets its elements in the order of their ids, so that
  // the first of several equal maxima is the one it keeps
  const int extra = rank == 0 && tid < sp.head ? tid : -1;
  const int extra2 = rank == C - 1 && tid < sp.tail ? p.V - sp.tail + tid : -1;
  auto single = [&](int i) {
    if (i < 0) return;
    const float z = element(row, i);
    if (z > best || (pos == -1 && z >= best)) { best = z; pos = -2 - i; }
    if (z > st.m) rebase(st, z, c);
    const float u = max_nan(z - st.m, -FLT_MAX), x = row_ex2(u * c);
    st.s += x;
    st.a = fmaf(u, x, st.a);
  };
  single(extra);
  unsigned long long s2 = f2_pack(st.s, 0.f), a2 = f2_pack(st.a, 0.f);
  const unsigned long long c2 = f2_pack(c, c);
  auto chunk = [&](const uint4* v, int n, int first) {
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (u < n) {
        const float vm = V16::largest(v[u]);
        if (vm > best || (pos == -1 && vm >= best)) { best = vm; pos = first + u * kRowThreads; }
        top = fmaxf(top, vm);
      }
    }
    if (top > st.m) {
      float s0, s1, a0, a1;
      f2_unpack(s2, s0, s1);
      f2_unpack(a2, a0, a1);
      st.s = s0 + s1;
      st.a = a0 + a1;
      rebase(st, top, c);
      s2 = f2_pack(st.s, 0.f);
      a2 = f2_pack(st.a, 0.f);
    }
    const unsigned long long nm2 = f2_pack(-st.m, -st.m);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (u < n) {
#pragma unroll
        for (int q = 0; q < V16::kN / 2; ++q) {
          float d0, d1, x0, x1;
          f2_unpack(f2_add(V16::pair(v[u], q), nm2), d0, d1);
          // (a masked logit of -inf: the difference stays finite so that its product with e^u = 0 is 0)
          const unsigned long long d2 = f2_pack(max_nan(d0, -FLT_MAX), max_nan(d1, -FLT_MAX));
          f2_unpack(f2_mul(d2, c2), x0, x1);
          const unsigned long long e2 = f2_pack(row_ex2(x0), row_ex2(x1));
          s2 = f2_add(s2, e2);
          a2 = f2_fma(d2, e2, a2);
        }
      }
    }
  };
  int i = sp.v_lo + tid;
  uint4 v[kUnroll];
  for (; i + (kUnroll - 1) * kRowThreads < sp.v_hi; i += kUnroll * kRowThreads) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) v[u] = row_vec(row, sp, i + u * kRowThreads);
    chunk(v, kUnroll, i);
  }
  int left = 0;
#pragma unroll
  for (int u = 0; u < kUnroll - 1; ++u) {
    const bool in = i + u * kRowThreads < sp.v_hi;
    v[u] = in ? row_vec(row, sp, i + u * kRowThreads) : make_uint4(0, 0, 0, 0);
    left += in ? 1 : 0;
  }
#pragma unroll
  for (int u = 0; u < kUnroll - 1; ++u)
    if (u < left) chunk(v + u, 1, i + u * kRowThreads);
  {
    float s0, s1, a0, a1;
    f2_unpack(s2, s0, s1);
    f2_unpack(a2, a0, a1);
    st.s = s0 + s1;
    st.a = a0 + a1;
  }
  single(extra2);
  // ---- statistics of the CTA
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Stats y;
    y.m = __shfl_xor_sync(0xffffffffu, st.m, o);
    y.s = __shfl_xor_sync(0xffffffffu, st.s, o);
    y.a = __shfl_xor_sync(0xffffffffu, st.a, o);
    st = join(st, y, c);
  }
  if (lane == 0) s_warp[warp] = st;
  // ---- the CTA's n largest elements
  const int n = p.n_top;
  if (n > 0) {
    unsigned long long key = 0;
    if (pos >= 0) {
      const uint4 w = row_vec(row, sp, pos);
      float x[V16::kN];
#pragma unroll
      for (int q = 0; q < V16::kN / 2; ++q) f2_unpack(V16::pair(w, q), x[2 * q], x[2 * q + 1]);
      int j = 0;
#pragma unroll
      for (int q = V16::kN - 1; q >= 0; --q) j = x[q] == best ? q : j;
      key = top_key(best, sp.head + pos * V16::kN + j);
    } else if (pos <= -2) {
      key = top_key(best, -2 - pos);
    } else {   // nothing but NaN, or no element at all
      const int first = extra >= 0 ? extra : (sp.v_lo + tid < sp.v_hi ? sp.head + (sp.v_lo + tid) * V16::kN : extra2);
      if (first >= 0) key = top_key(__uint_as_float(0x7fc00000u), first);
    }
    s_keys[tid] = key;
    if (tid < n) s_top[tid] = 0;
    if (tid == 0) s_nflag = s_ncand = 0;
    __syncthreads();
    if (warp == 0) {
      unsigned long long k[kRowThreads / 32];
      unsigned int any = 0u, all = ~0u;
      int have = 0;
#pragma unroll
      for (int q = 0; q < kRowThreads / 32; ++q) {
        k[q] = s_keys[lane + 32 * q];
        have += k[q] != 0;
        any |= (unsigned int)(k[q] >> 32);
        all &= (unsigned int)(k[q] >> 32);
      }
      have = __reduce_add_sync(0xffffffffu, have);
      unsigned long long tau = 1;
      if (have > kFlagCap) {
        // the bits all high words agree on, then bit by bit the largest threshold that n keys reach, until few enough do
        any = __reduce_or_sync(0xffffffffu, any);
        all = __reduce_and_sync(0xffffffffu, all);
        const int same = __clz(any ^ all);
        unsigned int hi = same ? any & ~(same >= 32 ? 0u : 0xffffffffu >> same) : 0u;
        int count = kRowThreads;
        for (int b = 31 - same; b >= 0 && count > kFlagCap; --b) {
          const unsigned int cand = hi | (1u << b);
          int r = 0;
#pragma unroll
          for (int q = 0; q < kRowThreads / 32; ++q) r += (unsigned int)(k[q] >> 32) >= cand;
          r = __reduce_add_sync(0xffffffffu, r);
          if (r >= n) { hi = cand; count = r; }
        }
        tau = (unsigned long long)hi << 32;
        for (int b = 31; b >= 0 && count > kFlagCap; --b) {   // many equal maxima: the order of their indices
          const unsigned long long cand = tau | (1ull << b);
          int r = 0;
#pragma unroll
          for (int q = 0; q < kRowThreads / 32; ++q) r += k[q] >= cand;
          r = __reduce_add_sync(0xffffffffu, r);
          if (r >= n) { tau = cand; count = r; }
        }
        if (tau == 0) tau = 1;
      }
      if (lane == 0) s_tau = tau;
    }
    __syncthreads();
    const unsigned long long tau = s_tau;
    if (key >= tau) {
      const int q = atomicAdd(&s_nflag, 1);
      if (q < kFlagCap) s_flag[q] = tid;
    }
    __syncthreads();
    auto offer = [&](float z, int idx) {
      const unsigned long long k = top_key(z, idx);
      if (k >= tau) {
        const int q = atomicAdd(&s_ncand, 1);
        if (q < kCandCap) s_cand[q] = k;
      }
    };
    const int nflag = s_nflag;
    for (int f = warp; f < min(nflag, kFlagCap); f += kRowWarps) {
      const int who = s_flag[f];
      for (int w = sp.v_lo + who + lane * kRowThreads; w < sp.v_hi; w += 32 * kRowThreads) {
        const uint4 x = row_vec(row, sp, w);
#pragma unroll
        for (int q = 0; q < V16::kN / 2; ++q) {
          float x0, x1;
          f2_unpack(V16::pair(x, q), x0, x1);
          offer(x0, sp.head + w * V16::kN + 2 * q);
          offer(x1, sp.head + w * V16::kN + 2 * q + 1);
        }
      }
      if (lane == 0 && rank == 0 && who < sp.head) offer(element(row, who), who);
      if (lane == 0 && rank == C - 1 && who < sp.tail)
        offer(element(row, p.V - sp.tail + who), p.V - sp.tail + who);
    }
    __syncthreads();
    const int ncand = s_ncand;
    if (ncand <= kCandCap && nflag <= kFlagCap) {
      for (int x = tid; x < ncand; x += kRowThreads) {
        const unsigned long long k = s_cand[x];
        int r = 0;
        for (int y = 0; y < ncand; ++y) r += s_cand[y] > k;
        if (r < n) s_top[r] = k;
      }
    } else {
      // a few threads hold nearly all of the row's largest elements: find them one after the other
      unsigned long long last = ~0ull;
      for (int r = 0; r < n; ++r) {
        unsigned long long k = 0;
        auto look = [&](float z, int idx) {
          const unsigned long long o = top_key(z, idx);
          if (o < last && o > k) k = o;
        };
        for (int w = sp.v_lo + tid; w < sp.v_hi; w += kRowThreads) {
          const uint4 x = row_vec(row, sp, w);
#pragma unroll
          for (int q = 0; q < V16::kN / 2; ++q) {
            float x0, x1;
            f2_unpack(V16::pair(x, q), x0, x1);
            look(x0, sp.head + w * V16::kN + 2 * q);
            look(x1, sp.head + w * V16::kN + 2 * q + 1);
          }
        }
        if (extra >= 0) look(element(row, extra), extra);
        if (extra2 >= 0) look(element(row, extra2), extra2);
        s_keys[tid] = k;
        __syncthreads();
        for (int o = kRowThreads / 2; o > 0; o >>= 1) {
          if (tid < o && s_keys[tid + o] > s_keys[tid]) s_keys[tid] = s_keys[tid + o];
          __syncthreads();
        }
        last = s_keys[0];
        if (tid == 0) s_top[r] = last;
        __syncthreads();
        if (last == 0) break;
      }
    }
  }
  __syncthreads();
  if (tid == 0) {
    Stats x = s_warp[0];
    for (int w = 1; w < kRowWarps; ++w) x = join(x, s_warp[w], c);
    s_cta = x;
  }
  // ---- the first CTA of the row joins and writes
  if (C > 1) {
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    if (rank == 0) {
      if (tid == 0) {
        Stats x = s_cta;
        for (int r = 1; r < C; ++r) {
          const uint32_t a = cluster_addr(&s_cta, r);
          x = join(x, Stats{cluster_load_f32(a), cluster_load_f32(a + 4), cluster_load_f32(a + 8)}, c);
        }
        s_warp[0] = x;   // (s_cta stays what the other CTAs might still be told it is)
      }
      for (int q = tid; q < C * n; q += kRowThreads)
        s_cand[q] = cluster_load_u64(cluster_addr(&s_top[q % n], q / n));
      __syncthreads();
      for (int q = tid; q < C * n; q += kRowThreads) {
        const unsigned long long k = s_cand[q];
        int r = 0;
        for (int y = 0; y < C * n; ++y) r += s_cand[y] > k;
        if (k != 0 && r < n) s_keys[r] = k;
      }
    }
    cluster_arrive();   // (this CTA has read all it wants of the others)
    cluster_wait();
    if (rank != 0) return;
  }
  __syncthreads();
  const Stats x = C > 1 ? s_warp[0] : s_cta;
  const unsigned long long* top = C > 1 ? s_keys : s_top;
  // a row of nothing but -inf has no distribution: probabilities 0, entropy 0
  const bool none = x.s == 0.f;
  const float log_s = logf(x.s);
  if (tid == 0) {
    if (p.logprob) {
      const int tok = p.tokens[t];
      float lp = 0.f;
      if (tok >= 0 && tok < p.V) {
        lp = none ? -INFINITY : (element(row, tok) - x.m) / p.T - log_s;
      } else if (tok != -1) {
        lp = __uint_as_float(0x7fc00000u);
        *p.dev_status = DX_DEV_BAD_TOKEN;
      }
      p.logprob[t] = lp;
    }
    if (p.entropy) p.entropy[t] = none ? 0.f : log_s - x.a / x.s / p.T;
  }
  if (tid < n) {
    const unsigned long long k = top[tid];
    p.top_ids[(size_t)t * n + tid] = (int32_t)(~(unsigned int)k);
    p.top_logprobs[(size_t)t * n + tid] = none ? -INFINITY : (key_value(k) - x.m) / p.T - log_s;
  }
}

template <typename T>
cudaError_t launch(dx_ctx* ctx, const LogprobParams& p, cudaStream_t st) {
  // As many CTAs per row as fill the GPU (four per SM), while each still has a vector for every thread.
  const int slots = 4 * ctx->sm_count;
  int C = 1;
  while (C < DX_ROW_CLUSTER_MAX && (long long)p.N * C * 2 <= slots &&
         (long long)C * 2 * kRowThreads * RowVec<T>::kN <= p.V)
    C *= 2;
  return dx_launch_pdl(false, dx_logprobs_kernel<T>, dim3((unsigned)p.N * C), dim3(kRowThreads), 0, st, C, p, C);
}

}  // namespace

cudaError_t dx_logprobs_prepare() {
  cudaError_t e = cudaFuncSetAttribute(dx_logprobs_kernel<float>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(dx_logprobs_kernel<__nv_bfloat16>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  return e;
}

cudaError_t dx_launch_logprobs(dx_ctx* ctx, const void* logits, int dtype, int N, int V, long long ld,
                               const int32_t* tokens, float temperature, int n_top, float* logprob, float* entropy,
                               int32_t* top_ids, float* top_logprobs, cudaStream_t st) {
  LogprobParams p{logits, N, V, n_top, ld, tokens, (float)(1.4426950408889634 / (double)temperature), temperature,
                  logprob, entropy, top_ids, top_logprobs, ctx->dev_status};
  return dtype == DX_DTYPE_FP32 ? launch<float>(ctx, p, st) : launch<__nv_bfloat16>(ctx, p, st);
}
