// Log probabilities of given tokens, entropy and the most likely alternatives of rows of logits:
//   u_v = (z_v - m) / T,  S = sum_v e^{u_v},  log p_v = u_v - log S,  H = log S - (sum_v u_v e^{u_v}) / S.
// The reference m is one of the row's logits, the largest or one at least 2^-8 (kSlack) times as likely: where it is not
// the largest, log S and log p_v + log S reach up to log 2^8 = 5.5 and cancel, so H and log p_v are good to a few steps of
// 5.5 in 32 bits (2e-6) besides the error of the sums; log p_v <= 0 and H >= 0 hold all the same, the reference's own mass
// being at least 2^-8 of the largest's.  The n alternatives are the largest z, ties to the lower id.
//
// One pass: every logit is read from HBM once.  Threads carry (a reference near the maximum, S, sum u e^u)
// relative to it, three 16-byte vectors at a time.  Alternatives ride along as each thread's largest logit, one per segment of its
// share of the row.  From the threads' maxima one warp picks a threshold that at least n and at most n + kFlagSlack
// threads reach; only the runs (thread, segment) that reach it can hold one of the n largest, so they alone -- one or
// two percent of the row -- are read again, and the few elements that pass are ranked by counting.  Where more threads
// share the threshold (a row of equal or masked words), what exceeds it is taken the same way and the equal elements in
// the order of their ids.  A row of few-row calls is split over a cluster of up to 16 CTAs, whose statistics and lists
// the first CTA joins through distributed shared memory: no workspace, no atomics on device memory, one launch, the
// same result on every run.
//
// What bounds it: without alternatives HBM and the exponentials (2048 x 102400 bf16: 75 us, 87 % of the measured copy
// bandwidth); with 20 alternatives 93 us, 70 % (86 us in a loop over one batch, part of which is still in L2; so are the
// other figures of variants here): the second look and its barriers stop a CTA's loads for a quarter of its row, and the
// other three CTAs of the SM do not cover all of it (a ninth warp that did the selection alone: 106 us).
// Few rows are a chain of latencies: 1 x 102400 9 us, 16 x 163840 fp32 12 us.
#include "dx_rows.cuh"

namespace {

constexpr int kUnroll = 3;        // vectors at a time, as many on their way (2: 101 us, 4: 96 us, 3: 87 us for the batch above)
constexpr float kSlack = 8.f;      // powers of two by which an element may exceed the reference of its thread's sums
constexpr int kSegments = 8;      // parts of a thread's share of the row that have a maximum of their own
constexpr int kFlagSlack = 12;    // the threshold may be reached by n + this many threads
constexpr int kRunCap = (DX_MAX_TOP + kFlagSlack) * kSegments;   // (thread, segment) runs looked at again
constexpr int kCandCap = 768;     // elements that may pass the threshold before the slow path takes over

struct LogprobParams {
  const void* logits;
  int N, V, n_top;
  long long ld;
  const int32_t* tokens;
  float c, T, dc;                 // log2(e) / T rounded, T, what the rounding has left out (times ln 2)
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
  float m, s, a;   // reference, sum of e^{(z - m) / T}, sum of (z - m) e^{(z - m) / T}
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

// the sums of a warp's lanes, relative to their largest reference; every lane gets them
__device__ __forceinline__ Stats warp_join(Stats x, float c) {
  rebase(x, warp_max(x.m), c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
    x.a += __shfl_xor_sync(0xffffffffu, x.a, o);
  }
  return x;
}

template <typename T>
__device__ __forceinline__ float element(const T* row, long long i) { return RowVec<T>::load(row + i); }

template <typename T>
__device__ __forceinline__ uint4 row_vec(const T* row, const RowSplit& sp, int v) {
  return __ldg(reinterpret_cast<const uint4*>(row + sp.head) + v);
}
// Which elements can be among the n largest: those of the runs listed (thread, segment), and the head / tail elements.
template <typename T>
struct Picker {
  const T* row;
  RowSplit sp;
  int V, rank, C, n, seg_vecs;          // vectors of one thread in one segment
  unsigned long long* cand;             // [kCandCap + DX_MAX_TOP]
  int* n_cand;
  int32_t* dev_status;

  // (`least`: the smallest value wanted; a NaN is taken where -inf is)
  __device__ __forceinline__ void offer(float z, int idx, float least) const {
    if (!(z < least) && (z == z || least == -INFINITY)) {
      const int q = atomicAdd(n_cand, 1);
      if (q < kCandCap) cand[q] = top_key(z, idx);
    }
  }
  // every element of the listed runs that is not below `least`
  __device__ __forceinline__ void rescan(const int* runs, int n_runs, float least) const {
    using V16 = RowVec<T>;
    const float inv = 1.f / (float)seg_vecs;
    const int items = n_runs * seg_vecs;
#pragma unroll 1
    for (int x = threadIdx.x; x < items; x += 2 * kRowThreads) {
      int v[2];
      uint4 w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int y = x + h * kRowThreads;
        int r = (int)(((float)y + 0.5f) * inv);           // y / seg_vecs, one off at most where y passes 24 bits
        r += (y >= (r + 1) * seg_vecs) - (y < r * seg_vecs);
        const int run = y < items && DX_BOUNDS(r >= 0 && r < n_runs, dev_status) ? runs[r] : 0;
        v[h] = sp.v_lo + run % kRowThreads + (run / kRowThreads * seg_vecs + y - r * seg_vecs) * kRowThreads;
        if (y >= items || v[h] >= sp.v_hi) v[h] = -1;
        if (v[h] >= 0) w[h] = row_vec(row, sp, v[h]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (v[h] < 0 || (V16::largest(w[h]) < least)) continue;
#pragma unroll
        for (int q = 0; q < V16::kN / 2; ++q) {
          float x0, x1;
          f2_unpack(V16::pair(w[h], q), x0, x1);
          offer(x0, sp.head + v[h] * V16::kN + 2 * q, least);
          offer(x1, sp.head + v[h] * V16::kN + 2 * q + 1, least);
        }
      }
    }
    if (rank == 0 && threadIdx.x < sp.head) offer(element(row, threadIdx.x), threadIdx.x, least);
    if (rank == C - 1 && threadIdx.x < sp.tail)
      offer(element(row, V - sp.tail + threadIdx.x), V - sp.tail + threadIdx.x, least);
  }
  // the first n elements, in the order of their ids, whose key has the high word `hi`; returns how many there are
  // (at most n), their keys in out[0 .. )
  __device__ __forceinline__ int first_equal(unsigned int hi, unsigned long long* out, int* s_scan) const {
    using V16 = RowVec<T>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int found = 0;
    const int tiles = (sp.v_hi - sp.v_lo + kRowThreads - 1) / kRowThreads;
    for (int tile = -1; tile <= tiles && found < n; ++tile) {
      unsigned int mask = 0;
      int first = 0;
      if (tile == -1) {
        first = threadIdx.x;
        if (rank == 0 && threadIdx.x < sp.head) mask = (unsigned int)(top_key(element(row, first), 0) >> 32) == hi;
      } else if (tile == tiles) {
        first = V - sp.tail + threadIdx.x;
        if (rank == C - 1 && threadIdx.x < sp.tail)
          mask = (unsigned int)(top_key(element(row, first), 0) >> 32) == hi;
      } else {
        const int v = sp.v_lo + tile * kRowThreads + threadIdx.x;
        first = sp.head + v * V16::kN;
        if (v < sp.v_hi) {
          const uint4 w = row_vec(row, sp, v);
#pragma unroll
          for (int q = 0; q < V16::kN / 2; ++q) {
            float x0, x1;
            f2_unpack(V16::pair(w, q), x0, x1);
            mask |= (unsigned int)((unsigned int)(top_key(x0, 0) >> 32) == hi) << (2 * q);
            mask |= (unsigned int)((unsigned int)(top_key(x1, 0) >> 32) == hi) << (2 * q + 1);
          }
        }
      }
      int at = __popc(mask);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, at, o);
        if (lane >= o) at += y;
      }
      if (lane == 31) s_scan[warp] = at;
      __syncthreads();
      int total = 0;
      at += found - __popc(mask);
      for (int w = 0; w < kRowWarps; ++w) {
        at += w < warp ? s_scan[w] : 0;
        total += s_scan[w];
      }
      for (; mask && at < n; mask &= mask - 1, ++at)
        if (DX_BOUNDS(at >= 0 && out + at < cand + kCandCap + DX_MAX_TOP, dev_status))
          out[at] = ((unsigned long long)hi << 32) | (unsigned long long)(~(unsigned int)(first + __ffs(mask) - 1));
      found += total;
      __syncthreads();
    }
    return min(found, n);
  }
};

template <typename T>
__global__ void __launch_bounds__(kRowThreads, 4) dx_logprobs_kernel(LogprobParams p, int C) {
  using V16 = RowVec<T>;
  __shared__ Stats s_warp[kRowWarps];
  __shared__ Stats s_cta;
  __shared__ float s_seg[kSegments][kRowThreads];          // largest element of each thread in each segment
  __shared__ unsigned long long s_cand[kCandCap + DX_MAX_TOP];
  __shared__ unsigned long long s_top[DX_MAX_TOP], s_out[DX_MAX_TOP];
  __shared__ unsigned long long s_in[DX_ROW_CLUSTER_MAX * DX_MAX_TOP], s_floor;   // (first CTA) the lists of all CTAs
  __shared__ Stats s_stats[DX_ROW_CLUSTER_MAX];
  __shared__ unsigned int s_keys[kRowThreads];
  __shared__ unsigned int s_tau;
  __shared__ int s_runs[kRunCap];
  __shared__ int s_scan[kRowWarps];
  __shared__ int s_nrun, s_ncand, s_ties;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = C > 1 ? (int)cluster_rank() : 0;
  const int t = blockIdx.x / C;
  const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
  const RowSplit sp = row_split(row, p.V, rank, C);
  const float c = p.c;
  const int n = p.n_top;

  if (C > 1) cluster_arrive();
  // ---- the pass over the row
  Stats st{-FLT_MAX, 0.f, 0.f};
  float best = -INFINITY;
  // All warps start from the largest element of their first chunk as the reference of the exponents; a thread takes
  // another only when it meets an element more than 2^kSlack times as likely (the sums stay far from fp32's limits, and
  // what they lose is a few bits of the entropy's last place).
  unsigned long long s2 = 0ull, a2 = 0ull;
  const unsigned long long c2 = f2_pack(c, c);
  auto take = [&]() {
    float s0, s1, a0, a1;
    f2_unpack(s2, s0, s1);
    f2_unpack(a2, a0, a1);
    st.s = s0 + s1;
    st.a = a0 + a1;
  };
  const int n_vec = sp.v_hi - sp.v_lo;
  const int chunks = (n_vec + kUnroll * kRowThreads - 1) / (kUnroll * kRowThreads);
  const int seg_chunks = max(1, (chunks + kSegments - 1) / kSegments);
  const uint4 none4 = make_uint4(V16::kNegInfWord, V16::kNegInfWord, V16::kNegInfWord, V16::kNegInfWord);
  float seg = -INFINITY;
  int g = 0, in_seg = 0;
  const uint4* src = reinterpret_cast<const uint4*>(row + sp.head) + sp.v_lo + tid;
  auto fetch = [&](uint4 (&x)[kUnroll], int ch) {
    if ((ch + 1) * (kUnroll * kRowThreads) <= n_vec) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) x[u] = load_stream(src + u * kRowThreads);
    } else {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        x[u] = none4;                                      // (adds nothing to any sum)
        if ((ch * kUnroll + u) * kRowThreads + tid < n_vec) x[u] = load_stream(src + u * kRowThreads);
      }
    }
    src += kUnroll * kRowThreads;
  };
  uint4 ahead[kUnroll];
  fetch(ahead, 0);
#pragma unroll 1
  for (int ch = 0; ch < chunks; ++ch) {
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) v[u] = ahead[u];
    if (ch + 1 < chunks) fetch(ahead, ch + 1);
    const float top = V16::largest(v, kUnroll);
    if (ch == 0) {
      st.m = fmaxf(warp_max(top), -FLT_MAX);
    } else if ((top - st.m) * c > kSlack) {
      take();
      rebase(st, top, c);
      s2 = f2_pack(st.s, 0.f);
      a2 = f2_pack(st.a, 0.f);
    }
    const unsigned long long nm2 = f2_pack(-st.m, -st.m);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
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
    seg = fmaxf(seg, top);
    if (++in_seg == seg_chunks) {
      if (DX_BOUNDS(g < kSegments, p.dev_status)) s_seg[g++][tid] = seg;
      best = fmaxf(best, seg);
      seg = -INFINITY;
      in_seg = 0;
    }
  }
  if (in_seg > 0 && DX_BOUNDS(g < kSegments, p.dev_status)) {
    s_seg[g][tid] = seg;
    best = fmaxf(best, seg);
  }
  take();
  // the head and the tail element of this thread, if any
  const int extra = rank == 0 && tid < sp.head ? tid : -1;
  const int extra2 = rank == C - 1 && tid < sp.tail ? p.V - sp.tail + tid : -1;
#pragma unroll 1
  for (int e = 0; e < 2; ++e) {
    const int i = e ? extra2 : extra;
    if (i < 0) continue;
    const float z = element(row, i);
    best = fmaxf(best, z);
    if (z > st.m) rebase(st, z, c);
    const float u = max_nan(z - st.m, -FLT_MAX), x = row_ex2(u * c);
    st.s += x;
    st.a = fmaf(u, x, st.a);
  }
  // ---- statistics of the CTA
  st = warp_join(st, c);
  if (lane == 0) s_warp[warp] = st;
  // ---- the CTA's n largest elements
  if (n > 0) {
    // (best is -inf for a thread that met nothing but -inf and NaN; zero: no element at all)
    const bool any = extra >= 0 || extra2 >= 0 || sp.v_lo + tid < sp.v_hi;
    const unsigned int mine = any ? dx_orderable(best + 0.f) : 0u;
    s_keys[tid] = mine;
    if (tid < n) s_top[tid] = 0;
    if (tid == 0) s_nrun = s_ncand = 0;
    __syncthreads();
    if (warp == 0) {
      unsigned int k[kRowThreads / 32];
      unsigned int some = 0u, all = ~0u;
      int have = 0;
#pragma unroll
      for (int q = 0; q < kRowThreads / 32; ++q) {
        k[q] = s_keys[lane + 32 * q];
        have += k[q] != 0;
        some |= k[q];
        all &= k[q];
      }
      have = __reduce_add_sync(0xffffffffu, have);
      unsigned int tau = 1;
      int count = have;
      const int enough = n + kFlagSlack;
      if (have > enough) {
        // the bits all keys agree on, then bit by bit the largest threshold that n keys reach, until few enough do
        some = __reduce_or_sync(0xffffffffu, some);
        all = __reduce_and_sync(0xffffffffu, all);
        const int same = __clz(some ^ all);
        const int first = (31 - same) | 1;                 // (-1: all keys are equal)
        tau = first < 0 ? some : some & ~((2u << first) - 1u);
        // (two bits at a time: the three counts of one step share a reduction)
        for (int b = first; b > 0 && count > enough; b -= 2) {
          const unsigned int step = 1u << (b - 1);
          unsigned int r = 0;
#pragma unroll
          for (int q = 0; q < kRowThreads / 32; ++q)
            r += (k[q] >= tau + step) + (k[q] >= tau + 2 * step) * 1024u + (k[q] >= tau + 3 * step) * (1024u * 1024u);
          r = __reduce_add_sync(0xffffffffu, r);
#pragma unroll
          for (int h = 2; h >= 0; --h) {
            const int reached = (int)(r >> (10 * h) & 1023u);
            if (reached >= n) {
              tau += (unsigned int)(h + 1) * step;
              count = reached;
              break;
            }
          }
        }
        if (tau == 0) tau = 1;
      }
      if (lane == 0) {
        s_tau = tau;
        s_ties = count > enough;      // tau is then a value that many threads share, and fewer than n exceed
      }
    }
    __syncthreads();
    const unsigned int tau = s_tau;
    const bool ties = s_ties != 0;
    Picker<T> pick{row, sp, p.V, rank, C, n, seg_chunks * kUnroll, s_cand, &s_ncand, p.dev_status};
    // (a threshold that everything reaches takes NaN in as well)
    const unsigned int low = ties ? tau + 1u : tau <= 0x007fffffu ? 1u : tau;
    if (ties ? mine > tau : mine >= tau) {
      const int segs = min(kSegments, (chunks + seg_chunks - 1) / seg_chunks);
      for (int g = 0; g < segs; ++g) {
        if (low == 1u || dx_orderable(s_seg[g][tid] + 0.f) >= low) {
          const int q = atomicAdd(&s_nrun, 1);
          if (q < kRunCap) s_runs[q] = g * kRowThreads + tid;
        }
      }
    }
    __syncthreads();
    pick.rescan(s_runs, min(s_nrun, kRunCap), low <= 0x007fffffu ? -INFINITY : key_value((unsigned long long)low << 32));
    __syncthreads();
    int ncand = s_ncand;
    if (ties && ncand <= kCandCap) {
      ncand += pick.first_equal(tau, s_cand + ncand, s_scan);
      // (fewer than n numbers in all: NaN follow)
      if (tau == 0x007fffffu && ncand < n) ncand += pick.first_equal(0x007ffffeu, s_cand + ncand, s_scan);
    }
    if (ncand <= kCandCap + DX_MAX_TOP && s_ncand <= kCandCap && s_nrun <= kRunCap) {
      __syncthreads();
      for (int x = tid; x < ncand; x += kRowThreads) {
        const unsigned long long k = s_cand[x];
        int r = 0;
        for (int y = 0; y < ncand; ++y) r += s_cand[y] > k;
        if (r < n) s_top[r] = k;
      }
    } else {
      // a few threads hold more large elements than the list takes: find the n largest one after the other
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
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const unsigned long long y = __shfl_xor_sync(0xffffffffu, k, o);
          k = y > k ? y : k;
        }
        __syncthreads();
        if (lane == 0) s_cand[warp] = k;
        __syncthreads();
        last = s_cand[0];
        for (int w = 1; w < kRowWarps; ++w) last = s_cand[w] > last ? s_cand[w] : last;
        if (tid == 0) s_top[r] = last;
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
  // ---- the first CTA of the row joins and writes: the others put their sums and lists into its shared memory
  Stats x{0.f, 0.f, 0.f};
  if (C > 1) {
    __syncthreads();
    cluster_wait();                                        // (all CTAs of the row have started)
    if (tid < n) cluster_store_u64(cluster_addr(&s_in[rank * n + tid], 0), s_top[tid]);
    if (tid == 0) {
      const uint32_t a = cluster_addr(&s_stats[rank], 0);
      cluster_store_f32(a, s_cta.m);
      cluster_store_f32(a + 4, s_cta.s);
      cluster_store_f32(a + 8, s_cta.a);
      s_ncand = 0;
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
    if (warp == 0) {
      x = lane < C ? s_stats[lane] : Stats{-FLT_MAX, 0.f, 0.f};
      // What at least n elements reach: the n-th of any one CTA, and the least of their m-th if m per CTA make n.
      const int m = (n + C - 1) / C;
      unsigned long long floor = 0, least = ~0ull;
      if (n > 0 && lane < C) {
        floor = s_in[lane * n + n - 1];
        least = s_in[lane * n + m - 1];
      }
      x = warp_join(x, c);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) {
        const unsigned long long f = __shfl_xor_sync(0xffffffffu, floor, o), l = __shfl_xor_sync(0xffffffffu, least, o);
        floor = f > floor ? f : floor;
        least = l < least ? l : least;
      }
      if (lane == 0) {
        s_warp[0] = x;
        s_floor = least > floor ? least : floor;
      }
    }
    __syncthreads();
    const unsigned long long floor = s_floor;
    for (int q = tid; q < C * n; q += kRowThreads) {
      const unsigned long long k = s_in[q];
      if (k != 0 && k >= floor) {
        const int at = atomicAdd(&s_ncand, 1);
        if (DX_BOUNDS(at < kCandCap + DX_MAX_TOP, p.dev_status)) s_cand[at] = k;
      }
    }
    __syncthreads();
    const int ncand = s_ncand;
    for (int q = tid; q < ncand; q += kRowThreads) {
      const unsigned long long k = s_cand[q];
      int r = 0;
      for (int y = 0; y < ncand; ++y) r += s_cand[y] > k;
      if (r < n) s_out[r] = k;
    }
  }
  __syncthreads();
  x = C > 1 ? s_warp[0] : s_cta;
  const unsigned long long* top = C > 1 ? s_out : s_top;
  // a row of nothing but -inf has no distribution: probabilities 0, entropy 0
  const bool none = x.s == 0.f;
  // (c is log2(e) / T rounded to fp32: what the rounding takes from every exponent, to first order)
  const float log_s = logf(fmaf(p.dc, x.a, x.s));
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
    (void)DX_BOUNDS(~(unsigned int)k < (unsigned int)p.V, p.dev_status);
    p.top_ids[(size_t)t * n + tid] = (int32_t)(~(unsigned int)k);
    p.top_logprobs[(size_t)t * n + tid] = none ? -INFINITY : (key_value(k) - x.m) / p.T - log_s;
  }
}

template <typename T>
cudaError_t launch(dx_ctx* ctx, const LogprobParams& p, cudaStream_t st) {
  // As many CTAs per row as fill the GPU (four per SM), while each still has a vector for every thread (a row of 102400 bf16
  // alone: 9.1 us, with one CTA 11.7; sixteen of 163840 fp32: 11.6 and 19.7 us).
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
  const double c = 1.4426950408889634 / (double)temperature;
  LogprobParams p{logits, N, V, n_top, ld, tokens, (float)c, temperature,
                  (float)((c - (double)(float)c) * 0.6931471805599453), logprob, entropy, top_ids, top_logprobs,
                  ctx->dev_status};
  return dtype == DX_DTYPE_FP32 ? launch<float>(ctx, p, st) : launch<__nv_bfloat16>(ctx, p, st);
}
