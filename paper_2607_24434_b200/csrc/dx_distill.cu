// Distillation from a teacher's top log probabilities (Eq. 8 with the teacher cut to a short list), per row t:
//   q = softmax(z / T);  p_j = e^{l_j} over the listed words, renormalised to sum 1 or -- with the tail bucket -- as they
//   are, the rest r = 1 - sum p in one bucket that is compared with R = sum of q over the unlisted words:
//     L = sum_j p_j (log p_j - log q_j)  [ + r (log r - log R) ]
//     dL/dz_v = ( beta q_v - p_v ) / T  for listed v,   ( beta - r / R ) q_v / T  otherwise,  beta = sum p + r
// One launch reads each logit once and writes each gradient once: a cluster of CTAs holds the row in shared memory
// between the statistics and the gradient, and each vector's place takes the next row's vector as soon as it has been
// read for the last time.
//
// The unlisted words are summed apart from the listed ones, relative to a reference of their own: R never comes out of a
// difference of nearly equal sums, and neither R nor the factor r / R can under- or overflow however far the listed words
// stand above the rest.  A bit per vector says which vectors hold listed words, a small hash table which of their
// elements; those become -inf in shared memory in front of the sweep.  A ninth warp does the arithmetic on the list while
// the other eight go over the row: in 64 bits for the loss, the listed words' gradient and, with a tail bucket, the
// unlisted words' factor (all are small differences), in 32 bits and first of all for what the eight wait for otherwise.
// It also says a row ahead whether there is anything to learn from the next row: rows without weight or list are not
// fetched.  The warps' sums go straight into the shared memory of all CTAs of the row, so that one cluster barrier is all
// that stands between the sweep and the gradient; without a gradient nobody waits at all, and a row's sums are collected
// while the next row is summed.
//
// What bounds it: HBM for fp32 (1024 x 163840 with gradient 254 us, 82 % of the measured copy bandwidth, with a tail
// bucket 259; loss alone 119 us, 88 %); for bf16 there are twice as many exponentials per byte and the two that a logit
// needs with a gradient keep their pipe busy for 55 % of the time (2048 x 102400, list of 64: 164 us, 79 %, with a tail
// bucket 166).  The loss alone needs one exponential per logit, but goes through shared memory, marks and barriers like
// the gradient: 96 us, 68 %, where the log probabilities of the same rows, which stay in registers, take 75.  Short rows
// pay the fixed part of a row per warp -- about half as many instructions as a sweep of 25 vectors -- more often: 8192 x
// 32000 bf16 217 us, 75 %, loss alone 111.
#include <cmath>

#include "dx_rows.cuh"

namespace {

constexpr int kUnroll = 4;
constexpr float kSlack = 8.f;                     // powers of two by which an element may exceed its sum's reference
constexpr int kStaticBytes = 5120;                // at least the kernel's static shared memory
constexpr int kHash = 2 * DX_MAX_TEACHER;
constexpr int kThreads = kRowThreads + 32;        // eight warps that stream, one that handles the list

struct DistillParams {
  const void* logits;
  int N, V, k, tail;
  int half, late;             // 16-bit words of marks per thread; the vector of a thread that begins its second half
  long long ld, ld_d;
  const int32_t* ids;
  const float* lp;
  float c, c_lo;              // log2(e) / T in two parts
  double inv_T, c64;          // c64: log2(e) / T
  float inv_Tf;
  const float* weight;
  float* loss;
  void* dlogits;
  int32_t* dev_status;
};
// vectors of a row that each of its C CTAs has room for
template <typename T>
__host__ __device__ __forceinline__ long long slice_vectors(int V, int C) {
  return ((long long)V * (long long)sizeof(T) / 16 + C - 1) / C;
}

// log2(e) / T in two parts, the first rounded down: rounded to one, it would shift the exponents of all words the same way,
// and a gradient that is a small difference of q and p would show it.
struct Factor {
  float hi, lo;
};
__device__ __forceinline__ float scaled_ex2(float d, Factor f) { return row_ex2(fmaf(d, f.lo, d * f.hi)); }

struct MaxSum {
  float m, s;
};
__device__ __forceinline__ MaxSum join(MaxSum x, MaxSum y, Factor c) {
  const float m = fmaxf(x.m, y.m);
  return MaxSum{m, x.s * scaled_ex2(x.m - m, c) + y.s * scaled_ex2(y.m - m, c)};
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// What the gradient needs to know of the list: the largest listed logit, sum_j e^{(z_j - z_ref) / T}, the teacher's mass.
struct ListSums {
  float z_ref, sum_e, mass;
};
// What the loss of a row is made of.  64-bit logarithms are long chains: kRing rows are finished at a time, a lane each.
constexpr int kRing = 16;
struct LossTerms {
  double mass, p_log_p, p_u, sum_e;
  float z_ref, rest_m, rest_s;
  int t;
};

__device__ __forceinline__ void copy16(uint32_t dst_smem, const uint4* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst_smem), "l"(src) : "memory");
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
__device__ __forceinline__ MaxSum warp_join(MaxSum x, Factor c) {
  const float m = warp_max(x.m);
  float s = x.s * scaled_ex2(x.m - m, c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return MaxSum{m, s};
}

// Barrier of all nine warps (the two roles meet it at different places of the program).
__device__ __forceinline__ void cta_barrier() { asm volatile("bar.sync 0, %0;" ::"n"(kThreads) : "memory"); }

// The sums of a row, from all warps of its CTAs and from the list.
struct RowSums {
  MaxSum rest;                // unlisted words
  ListSums l;
  float M;                    // the larger of the two references
  float w_rest, w_list, S;    // factors that bring the two sums to M; the whole sum relative to it
};
__device__ __forceinline__ RowSums row_sums(const MaxSum* all, const ListSums& l, int n, Factor c) {
  RowSums r;
  const int lane = threadIdx.x & 31;
  MaxSum x = lane < n ? all[lane] : MaxSum{-FLT_MAX, 0.f};
  for (int i = lane + 32; i < n; i += 32) x = join(x, all[i], c);
  r.rest = warp_join(x, c);
  r.l = l;
  r.M = fmaxf(r.rest.m, l.z_ref);
  // (fp32: the gradient's factors; a sum that is NaN stays NaN)
  r.w_rest = r.rest.s > 0.f ? scaled_ex2(r.rest.m - r.M, c) : r.rest.s;
  r.w_list = scaled_ex2(l.z_ref - r.M, c);
  r.S = r.w_rest * r.rest.s + r.w_list * l.sum_e;
  return r;
}

// 2^((m - ref) c) to 2^-32, for exponents from -1000 to 500 (less counts as none, more as 500): Taylor's polynomial of
// e^t on |t| <= ln 2 / 2.  c32: c in 32 bits, for the comparisons with the limits.
__device__ __forceinline__ double ex2_64(float m, float ref, double c, float c32) {
  const float about = (m - ref) * c32;
  const double y = ((double)m - (double)ref) * c;
  const double big = y + 6755399441055744.0;            // 1.5 * 2^52: the nearest integer is in the low word
  const double t = (y - (big - 6755399441055744.0)) * 0.6931471805599453, t2 = t * t, t4 = t2 * t2;
  const double lo = fma(t2, fma(t, 1.0 / 6.0, 0.5), 1.0 + t);
  const double hi = fma(t2, fma(t, 1.0 / 5040.0, 1.0 / 720.0), fma(t, 1.0 / 120.0, 1.0 / 24.0));
  const double x = fma(t4, fma(t4, 1.0 / 40320.0, hi), lo);
  const int up = __double2hiint(x) + (__double2loint(big) << 20);
  return about < -1000.f ? 0.0 : about > 500.f ? 3.273390607896142e150 : __hiloint2double(up, __double2loint(x));
}
// A row's sums in 64 bits: R over the unlisted words, relative to e^{ref / T}; w: what brings the listed words' sum to
// that reference.  (Where the list stands more than 2^500 above the rest, or 2^1000 below, the smaller of the two counts
// for nothing.)
struct Row64 {
  float ref;
  double R, w;
};
__device__ __forceinline__ Row64 row_sums64(const MaxSum* all, float z_ref, int n, double c, float c32) {
  Row64 r{-FLT_MAX, 0.0, 0.0};
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int i = lane; i < n; i += 32) r.ref = fmaxf(r.ref, all[i].m);
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r.ref) : "f"(r.ref));   // (a third of the time of five shuffles)
#pragma unroll 1
  for (int i = lane; i <= n; i += 32) {                 // (place n: the list)
    const double x = ex2_64(i < n ? all[i].m : z_ref, r.ref, c, c32);
    if (i < n) r.R += (double)all[i].s * x;
    else r.w = x;
  }
  r.R = warp_sum(r.R);
  r.w = __shfl_sync(0xffffffffu, r.w, n & 31);
  return r;
}
// beta / S - rest / R of a row with a tail bucket, relative to the same reference.  The two quotients cancel where the
// student's tail is close to the teacher's; with S = R + P, P the listed words' sum, and beta = mass + rest they are one
// fraction whose numerator is a difference in 64 bits.  What is left is the error of R's own exponentials, 1e-8 to 2e-8
// (rms) of rest / R for a student within 1e-4 of its teacher at 2000 to 163840 words; as two quotients in 32 bits it was
// 1.7e-7 to 3e-7.  The 64-bit chain costs 0.2 us a row (2048 x 102400 bf16: 164 -> 166 us).
__device__ __forceinline__ float tail_factor(const Row64& r, double mass, double sum_e) {
  const double rest = mass < 1.0 ? 1.0 - mass : 0.0, P = r.w * sum_e, S = r.R + P;
  const double scale = __hiloint2double(0x7fe00000 - (__double2hiint(S) & 0x7ff00000), 0);   // brings S to [1, 2)
  return __fdividef(__fdividef((float)((r.R * mass - rest * P) * scale), (float)(S * scale)), (float)r.R);
}

// kLists: list entries per lane of the list's warp, at least k / 32: two up to 64 words, four up to 128 (four for all: 170 us
// instead of 164.6 for the batch above, 62 instead of 46 us for 4096 x 1001; lists of 128 words 184 us)
template <typename T, bool kGrad, int kLists>
__global__ void __launch_bounds__(kThreads, kGrad ? 2 : 3) dx_distill_kernel(DistillParams p, int C, int buffers) {
  using V16 = RowVec<T>;
  // [buffers][kRowThreads][half] 16-bit words -- bit q of a thread's words: its q-th vector holds a listed word -- and
  // behind them the CTA's vectors of the row
  // (on a 128-byte border: 16 bytes beside a 32-byte one cost a tenth of the time)
  extern __shared__ __align__(128) uint4 s_dyn[];
  __shared__ __align__(16) unsigned int s_hash[2][kHash];   // vector + 1 << 8 | its listed elements; 0: free
  __shared__ MaxSum s_all[2][DX_ROW_CLUSTER_MAX * kRowWarps];   // sums of all warps of all CTAs of the row
  __shared__ ListSums s_list[2];
  __shared__ double s_list64[2][2];                // (tail bucket) the teacher's mass on the list, the student's sum in 64 bits
  __shared__ unsigned int s_edge[2];               // head (bits 0..7) and tail (8..15) elements that are listed
  __shared__ float2 s_weight[2];                   // x = 0: nothing to learn from the row; y = 0: from the row behind
  __shared__ LossTerms s_ring[kRing];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = C > 1 ? (int)cluster_rank() : 0;
  const int n_rows = gridDim.x / C;                // rows in flight: row t is followed by row t + n_rows
  const Factor c{p.c, p.c_lo};
  const int half = p.half;
  unsigned int* s_mark = reinterpret_cast<unsigned int*>(s_dyn);
  if (C > 1) cluster_arrive();

  // Both roles walk the same rows and meet at the same barriers: one of the CTA in front of a row (its marks are there,
  // the previous row's gradient has been stored), one of all CTAs of the row between the sums and the gradient.  The
  // sums are kept in two sets, taken in turn by the rows that have any: a CTA that is one row ahead cannot overwrite
  // what another still reads, and it cannot be two rows ahead of that barrier.
  if (warp == kRowWarps) {
    // ==== the list warp
    int id[kLists];                                // entry lane + 32 i (-1: unused, out of range, listed before)
    int raw[kLists];                               // ... of the row behind, as given
    float w = 0.f, weight = 0.f;                   // weight of the row behind; of the row that is marked
    // The list's part in a row: logits and log p_j, on their way while the row in front is worked on; then per entry
    // e^{(z_j - z_ref) / T} -- later the word's gradient, stored when the next row begins -- and p_j, the sums for the
    // gradient, and the sums for the loss (log p_j is what the caller has given).
    float z[kLists], lp[kLists], g[kLists];
    double e[kLists], pj[kLists], norm = 1.0;      // (64 bits: where q is close to p, their difference shows every rounding)
    int at[kLists];
    T* last_out = nullptr;
    ListSums l{};
    double mass = 0.0, p_log_p = 0.0, p_u = 0.0, sum_e = 0.0;
    auto load_ids = [&](int t) {
      if (t >= p.N) return;
#pragma unroll
      for (int i = 0; i < kLists; ++i) raw[i] = lane + 32 * i < p.k ? p.ids[(size_t)t * p.k + lane + 32 * i] : -1;
      w = p.weight ? p.weight[t] : 1.f;
    };
    // The ids of row t are at hand, those of the row behind it are asked for: early in the row in front of t, so that they
    // are there when that row ends (asked for among the marks they kept everyone waiting, 2 % of a loss alone).
    auto take_ids = [&](int t) {
#pragma unroll
      for (int i = 0; i < kLists; ++i) id[i] = raw[i];
      weight = w;
      load_ids(t + n_rows);
    };
    // whether there is something to learn from the row behind, for those who fetch it
    auto announce = [&](int t, int b) {
      if (t >= p.N) return;
      bool any = false;
#pragma unroll
      for (int i = 0; i < kLists; ++i) any |= raw[i] >= 0 && raw[i] < p.V;
      any = __any_sync(0xffffffffu, any);
      if (lane == 0) s_weight[b].y = any && w != 0.f ? 1.f : 0.f;
    };
    auto mark = [&](int t, int b) {                // ids -> marks, hash table and state of buffer b
      if (t >= p.N) return;
      const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
#pragma unroll
      for (int i = 0; i < kLists; ++i) {
        const bool in = id[i] >= 0 && id[i] < p.V;
        z[i] = in ? V16::load(row + id[i]) : -INFINITY;
        lp[i] = in ? p.lp[(size_t)t * p.k + lane + 32 * i] : -INFINITY;
      }
      const RowSplit sp = row_split(row, p.V, rank, C);
      const int n_vec = sp.v_hi - sp.v_lo, tail0 = p.V - sp.tail;
      unsigned int* marks = s_mark + b * half * (kRowThreads / 2);
      for (int i = lane; i < half * (kRowThreads / 8); i += 32)
        reinterpret_cast<uint4*>(marks)[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < kHash / 128; ++i) reinterpret_cast<uint4*>(s_hash[b])[lane + 32 * i] = make_uint4(0, 0, 0, 0);
      if (lane == 0) s_edge[b] = 0;
      __syncwarp();
      bool live = false, bad = false;
#pragma unroll
      for (int i = 0; i < kLists; ++i) {
        if (32 * i >= p.k) continue;
        int x = id[i];
        bad |= x < -1 || x >= p.V;
        if (x < 0 || x >= p.V) x = -1;
        live |= x >= 0;
        // an id counts once, with its first entry: the first of equal lanes, and not if an earlier 32 have left its bit
        const unsigned int same = __match_any_sync(0xffffffffu, x);
        if (__ffs(same) - 1 != lane) x = -1;
        if (x >= 0) {
          unsigned int bit, old;
          if (x < sp.head) {
            bit = 1u << x;
            old = atomicOr(&s_edge[b], bit);
          } else if (x >= tail0) {
            bit = 256u << (x - tail0);
            old = atomicOr(&s_edge[b], bit);
          } else {
            const int vec = (x - sp.head) / V16::kN;
            const unsigned int key = (unsigned int)(vec + 1) << 8;
            bit = 1u << ((x - sp.head) % V16::kN);
            old = 0;
            int h = vec & (kHash - 1);
            for (int tries = 0; tries < kHash; ++tries) {   // (at most kHash / 2 vectors: a free or equal one is found)
              const unsigned int found = atomicCAS(&s_hash[b][h], 0u, key | bit);
              if (found == 0u) break;
              if ((found & 0xffffff00u) == key) {
                old = atomicOr(&s_hash[b][h], bit);
                break;
              }
              h = (h + 1) & (kHash - 1);
            }
            const int mine = vec - sp.v_lo;
            if (mine >= 0 && mine < n_vec) {
              const int q = mine / kRowThreads, at = (mine % kRowThreads) * half + (q >> 4);
              if (DX_BOUNDS(q < 16 * half, p.dev_status)) atomicOr(&marks[at >> 1], 1u << ((at & 1) * 16 + (q & 15)));
            }
          }
          if (old & bit) x = -1;
        }
        id[i] = x;
        __syncwarp();
      }
      if (bad && rank == 0) *p.dev_status = DX_DEV_BAD_TOKEN;
      live = __any_sync(0xffffffffu, live);
      if (lane == 0) s_weight[b].x = live ? weight : 0.f;
    };
    // the teacher's part in the row whose ids and log p_j are at hand: p_j, their mass, sum p log p, renormalisation
    auto teacher = [&](const int (&ids)[kLists]) {
      mass = p_log_p = 0.0;
      // (a renormalised list is taken relative to its largest entry: only differences count, and no exponential of it
      // over- or underflows)
      float top = 0.f;
      if (!p.tail) {
        top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kLists; ++i)
          if (ids[i] >= 0) top = fmaxf(top, lp[i]);
        top = warp_max(top);
        if (top == -INFINITY) top = 0.f;
      }
#pragma unroll
      for (int i = 0; i < kLists; ++i) {
        pj[i] = 0.0;
        if (32 * i >= p.k) continue;
        const double x = (double)lp[i] - (double)top;
        const double pd = ids[i] >= 0 ? exp(x) : 0.0;   // (a NaN makes the mass NaN, and with it the loss)
        pj[i] = pd;
        mass += pd;
        if (pd > 0.0) p_log_p += pd * x;
      }
      mass = warp_sum(mass);
      p_log_p = warp_sum(p_log_p);
      norm = 1.0;
      if (!p.tail && mass != 0.0) {                // p' = p / mass:  sum p' log p' = (sum p log p) / mass - log mass
        norm = 1.0 / mass;
        p_log_p = p_log_p * norm - log(mass);
        mass = mass == mass ? 1.0 : mass;
      }
    };
    // the student's part in 64 bits, for the loss, the listed words' gradient and, with a tail bucket, the unlisted
    // words' factor
    auto student = [&]() {
      p_u = sum_e = 0.0;
#pragma unroll
      for (int i = 0; i < kLists; ++i) {
        e[i] = 0.0;
        if (32 * i >= p.k) continue;
        const double u = ((double)z[i] - (double)l.z_ref) * p.inv_T;
        e[i] = at[i] >= 0 ? exp(u) : 0.0;
        sum_e += e[i];
        if (pj[i] > 0.0) p_u += pj[i] * u;
      }
      sum_e = warp_sum(sum_e);
    };
    // the largest listed logit
    auto list_top = [&]() {
      float top = -FLT_MAX;
#pragma unroll
      for (int i = 0; i < kLists; ++i) {
        at[i] = id[i];
        if (at[i] < 0) z[i] = -INFINITY;           // (unused, or listed before)
        top = fmaxf(top, z[i]);
      }
      l.z_ref = warp_max(top);
    };
    // what the sweep's warps wait for: 32 bits are enough where the gradient's factor is one quotient, and are there sooner
    auto publish = [&](int slot) {
      if (!p.tail) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kLists; ++i)
          if (32 * i < p.k && at[i] >= 0) s += expf((float)(((double)z[i] - (double)l.z_ref) * p.inv_T));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        l.sum_e = s;
      } else {
        l.sum_e = (float)sum_e;
        if (lane == 0) {
          s_list64[slot][0] = mass;
          s_list64[slot][1] = sum_e;
        }
      }
      l.mass = (float)mass;
      if (lane == 0) s_list[slot] = l;
      __syncwarp();
    };
    auto store_listed = [&]() {                    // over what the sweep has left in their places
      if constexpr (kGrad) {
        if (!last_out) return;
#pragma unroll
        for (int i = 0; i < kLists; ++i)
          if (at[i] >= 0 && DX_BOUNDS(at[i] < p.V, p.dev_status)) last_out[at[i]] = V16::round(g[i]);
        last_out = nullptr;
      }
    };
    int in_ring = 0;
    auto finish = [&]() {                          // the losses of the rows in the ring
      if (lane >= in_ring) return;
      const LossTerms x = s_ring[lane];
      if (!DX_BOUNDS(x.t >= 0 && x.t < p.N, p.dev_status)) return;
      const float M = fmaxf(x.rest_m, x.z_ref);
      const double rest = p.tail && x.mass < 1.0 ? 1.0 - x.mass : 0.0;
      const double du_rest = ((double)x.rest_m - (double)M) * p.inv_T;
      const double du_list = ((double)x.z_ref - (double)M) * p.inv_T;
      const double S = (x.rest_s > 0.f ? exp(du_rest) : 1.0) * (double)x.rest_s + exp(du_list) * x.sum_e;
      const double log_S = log(S);
      // - sum_j p_j log q_j = -( sum p_j (z_j - z_ref) / T + P (z_ref - M) / T - P log S )
      double loss = x.p_log_p - (x.p_u + (x.mass != 0.0 ? x.mass * (du_list - log_S) : 0.0));
      if (rest > 0.0) loss += rest * (log(rest) - (du_rest + log((double)x.rest_s) - log_S));
      if (S == 0.0) loss = x.mass + rest > 0.0 ? INFINITY : 0.0;   // nothing but -inf in the row
      p.loss[x.t] = (float)loss;
    };
    auto keep = [&](const RowSums& r, int t) {     // a row's terms into the ring
      if (lane == 0) s_ring[in_ring] = LossTerms{mass, p_log_p, p_u, sum_e, l.z_ref, r.rest.m, r.rest.s, t};
      __syncwarp();
      if (++in_ring == kRing) {
        finish();
        __syncwarp();
        in_ring = 0;
      }
    };
    int t = blockIdx.x / C, turn = 0;
    int pending = -1;                              // (loss alone) the row whose sums are still to be collected
    auto collect = [&]() {
      if (pending < 0) return;
      if (C > 1) cluster_wait();
      if (rank == 0) keep(row_sums(s_all[turn ^ 1], l, C * kRowWarps, c), pending);
      pending = -1;
    };
    load_ids(t);
    take_ids(t);
    mark(t, 0);
    if (C > 1) cluster_wait();                     // (all CTAs of the row have started)
#pragma unroll 1
    for (int it = 0; t < p.N; ++it, t += n_rows) {
      announce(t + n_rows, it & (buffers - 1));
      cta_barrier();
      if (!kGrad) collect();
      if (kGrad && it == 0) teacher(id);           // (of later rows it is ready by now)
      store_listed();
      const float scale = s_weight[it & (buffers - 1)].x * p.inv_Tf;
      if (s_weight[it & (buffers - 1)].x == 0.f) {   // nothing to learn from this row
        if (rank == 0 && lane == 0 && p.loss) p.loss[t] = 0.f;
        take_ids(t + n_rows);
        mark(t + n_rows, (it + 1) & (buffers - 1));
        if (kGrad) teacher(id);
        continue;
      }
      const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
      list_top();
      take_ids(t + n_rows);
      const bool wide = kGrad && p.tail != 0;
      if (kGrad && !wide) publish(turn);
      if (C > 1 && !wide) cluster_arrive();
      if (!kGrad) teacher(at);
      student();
      if (wide) {
        publish(turn);
        if (C > 1) cluster_arrive();
      }
      p_u = warp_sum(p_u) * norm;                  // (no one waits for this sum)
      mark(t + n_rows, (it + 1) & (buffers - 1));
      __syncwarp();
      if (!kGrad) {
        pending = t;
        turn ^= 1;
        continue;
      }
      if (C > 1) cluster_wait();
      else cta_barrier();
      const RowSums r = row_sums(s_all[turn], l, C * kRowWarps, c);
      turn ^= 1;
      if (kGrad) {
        const double w_list = ex2_64(l.z_ref, r.rest.m, p.c64, c.hi), S = (double)r.rest.s + w_list * sum_e;
        const double f = S == 0.0 ? 0.0 : (p.tail && mass < 1.0 ? 1.0 : mass) * w_list / S;
        last_out = reinterpret_cast<T*>(p.dlogits) + (size_t)t * (size_t)p.ld_d;
        const RowSplit sp = row_split(row, p.V, rank, C);
#pragma unroll
        for (int i = 0; i < kLists; ++i) {
          g[i] = S == 0.0 ? 0.f : (float)(f * e[i] - pj[i] * norm) * scale;
          const int v = (at[i] - sp.head) / V16::kN;
          if (at[i] < sp.head ? rank != 0 : at[i] >= p.V - sp.tail ? rank != C - 1 : v < sp.v_lo || v >= sp.v_hi) at[i] = -1;
        }
      }
      if (rank == 0 && p.loss) keep(r, t);
      teacher(id);
    }
    if (kGrad) {
      finish();
      __syncwarp();
      cta_barrier();
      store_listed();
    } else {
      cta_barrier();
      collect();
      finish();
    }
    return;
  }

  // ==== the eight warps that go over the row
  // this thread's vectors of the row: every 4096 bytes from here
  const uint32_t s_mine =
      static_cast<uint32_t>(__cvta_generic_to_shared(s_dyn + buffers * half * (kRowThreads / 8) + tid));
  const unsigned long long c2 = f2_pack(c.hi, c.hi), cl2 = f2_pack(p.c_lo, p.c_lo);
  const uint4 none4 = make_uint4(V16::kNegInfWord, V16::kNegInfWord, V16::kNegInfWord, V16::kNegInfWord);
  int t = blockIdx.x / C, turn = 0;
  bool pending = false;                            // (loss alone) arrived at the cluster's barrier, not waited
  const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
  RowSplit sp = row_split(row, p.V, rank, C);
  // Every thread copies the vectors tid, tid + 256, ... that it reads itself, in two groups: those in front of `late` can
  // be waited for alone.
  const int late = p.late;
  {
    const uint4* src = reinterpret_cast<const uint4*>(row + sp.head) + sp.v_lo;
    const int n_vec = sp.v_hi - sp.v_lo, deep = (n_vec + kRowThreads - 1) / kRowThreads;
#pragma unroll 2
    for (int q = 0; q < deep; ++q) {
      if (q == late) asm volatile("cp.async.commit_group;" ::: "memory");
      const int i = tid + q * kRowThreads;
      if (i < n_vec && DX_BOUNDS(i < slice_vectors<T>(p.V, C), p.dev_status)) copy16(s_mine + q * kRowThreads * 16, src + i);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  if (C > 1) cluster_wait();                       // (all CTAs of the row have started)
#pragma unroll 1
  for (int it = 0; t < p.N; ++it) {
    const int b = it & (buffers - 1);
    T* out = kGrad ? reinterpret_cast<T*>(p.dlogits) + (size_t)t * (size_t)p.ld_d : nullptr;
    const int n_vec = sp.v_hi - sp.v_lo, deep = (n_vec + kRowThreads - 1) / kRowThreads;
    const int tail0 = p.V - sp.tail;
    const bool has_head = rank == 0 && tid < sp.head, has_tail = rank == C - 1 && tid < sp.tail;
    // gradient vectors can be stored as such where the output row is aligned like the input row
    const bool same_align = kGrad && ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row)) & 15u) == 0;
    T* out_vec = out + sp.head + (long long)sp.v_lo * V16::kN;
    // the next row: its vectors take the places of this one's as soon as those have been read for the last time
    const T* next = row + (size_t)n_rows * (size_t)p.ld;
    t += n_rows;
    const RowSplit np = t < p.N ? row_split(next, p.V, rank, C) : sp;
    const uint4* fetch = reinterpret_cast<const uint4*>(next + np.head) + np.v_lo + tid;
    cta_barrier();
    const float2 wn = s_weight[b];                 // (a row there is nothing to learn from stays where it is)
    const bool more = t < p.N && wn.y != 0.f && DX_BOUNDS(np.v_hi - np.v_lo <= slice_vectors<T>(p.V, C), p.dev_status);
    const int next_vecs = more ? np.v_hi - np.v_lo : 0, next_deep = (next_vecs + kRowThreads - 1) / kRowThreads;
    const int plain = min(n_vec, next_vecs ? next_vecs : n_vec);
    const float w = wn.x;
    float coef = 0.f, ref = 0.f;                   // gradient of an unlisted word: coef * e^{(z - ref) / T}
    float edge_head = -INFINITY, edge_tail = -INFINITY;
    bool head_in = has_head, tail_in = has_tail;   // this thread's edge elements that are not listed
    if (w != 0.f) {                                // (the same for every CTA of the row)
      const unsigned int edge = s_edge[b];
      head_in = has_head && !(edge >> tid & 1u);
      tail_in = has_tail && !(edge >> (8 + tid) & 1u);
      // ---- sum of exponentials of the unlisted words
      MaxSum st{-FLT_MAX, 0.f};
      const unsigned short* marks = reinterpret_cast<const unsigned short*>(s_mark) + (b * kRowThreads + tid) * half;
      unsigned long long s2 = f2_pack(0.f, 0.f);
      // The listed words are left out of the sums: their elements of this thread's vectors q0 .. q1 - 1 become -inf where
      // they lie (a warp has a handful per row; the sweep knows nothing of them).
      auto leave_out = [&](int q0, int q1) {
#pragma unroll 1
        for (int w16 = q0 >> 4; w16 << 4 < q1; ++w16) {
          unsigned int marked = marks[w16];
          if (w16 << 4 < q0) marked &= ~0u << (q0 & 15);
          if (q1 - (w16 << 4) < 16) marked &= (1u << (q1 - (w16 << 4))) - 1u;
#pragma unroll 1
          for (; marked; marked &= marked - 1) {
            const int q = (w16 << 4) + __ffs(marked) - 1, vec = sp.v_lo + tid + q * kRowThreads;
            int h = vec & (kHash - 1);
            for (int tries = 0; tries < kHash && s_hash[b][h] >> 8 != (unsigned int)vec + 1u; ++tries)
              h = (h + 1) & (kHash - 1);
            if (!DX_BOUNDS(tid + q * kRowThreads < n_vec && s_hash[b][h] >> 8 == (unsigned int)vec + 1u, p.dev_status))
              continue;
            uint4 v = load_shared(s_mine + q * kRowThreads * 16);
            mask_vector<T>(v, s_hash[b][h]);
            store_shared(s_mine + q * kRowThreads * 16, v);
          }
        }
        __syncwarp();
      };
      // All warps start from the largest unlisted element of their first vectors as the reference of the exponents; a
      // thread takes another only when it meets an element more than 2^kSlack times as likely.
      auto add = [&](uint4 (&v)[kUnroll], int q, int n_v) {
        const float top = n_v == 1 ? V16::largest(v[0]) : V16::largest(v, kUnroll);
        if (q == 0) {
          st.m = fmaxf(warp_max(top), -FLT_MAX);
        } else if ((top - st.m) * c.hi > kSlack) {
          float s0, s1;
          f2_unpack(s2, s0, s1);
          s2 = f2_pack((s0 + s1) * scaled_ex2(st.m - top, c), 0.f);
          st.m = top;
        }
        const unsigned long long nm2 = f2_pack(-st.m, -st.m);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          if (u >= n_v) continue;
#pragma unroll
          for (int h = 0; h < V16::kN / 2; ++h) {
            const unsigned long long d2 = f2_add(V16::pair(v[u], h), nm2);
            float x0, x1;
            f2_unpack(f2_fma(d2, cl2, f2_mul(d2, c2)), x0, x1);
            s2 = f2_add(s2, f2_pack(row_ex2(x0), row_ex2(x1)));
          }
        }
      };
      uint32_t held = s_mine;
      int q = 0;
      auto second_half = [&]() {                     // the vectors from `late` on are there; the next row's first half is asked for
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (!kGrad) asm volatile("cp.async.commit_group;" ::: "memory");
        leave_out(late, deep);
      };
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      leave_out(0, late);
#pragma unroll 1
      for (; (q + kUnroll) * kRowThreads <= (kGrad ? n_vec : plain); q += kUnroll) {
        if (q == late) second_half();
        uint4 v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) v[u] = load_shared(held + u * kRowThreads * 16);
        add(v, q, kUnroll);
        if (!kGrad && next_vecs) {
#pragma unroll
          for (int u = 0; u < kUnroll; ++u) copy16(held + u * kRowThreads * 16, fetch + u * kRowThreads);
        }
        held += kUnroll * kRowThreads * 16;
        if (!kGrad) fetch += kUnroll * kRowThreads;
      }
#pragma unroll 1
      for (; q < (kGrad ? deep : max(deep, next_deep)); q += kUnroll) {   // what is left: less than kUnroll vectors per
        if (q == late) second_half();                                     // thread, and one more for some
        uint4 v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int i = tid + (q + u) * kRowThreads;
          v[u] = none4;                                          // (adds nothing)
          if (i < n_vec) v[u] = load_shared(held + u * kRowThreads * 16);
        }
        // (a single vector: the warps that have no second one)
        if ((q + 1) * kRowThreads + (tid & ~31) < n_vec) add(v, q, kUnroll);
        else add(v, q, 1);
        if (!kGrad) {
#pragma unroll
          for (int u = 0; u < kUnroll; ++u)
            if (tid + (q + u) * kRowThreads < next_vecs) copy16(held + u * kRowThreads * 16, fetch + u * kRowThreads);
          fetch += kUnroll * kRowThreads;
        }
        held += kUnroll * kRowThreads * 16;
      }
      if (!kGrad) asm volatile("cp.async.commit_group;" ::: "memory");
      float s0, s1;
      f2_unpack(s2, s0, s1);
      st.s = s0 + s1;
      if (head_in || tail_in) {
        edge_head = head_in ? V16::load(row + tid) : -INFINITY;
        edge_tail = tail_in ? V16::load(row + tail0 + tid) : -INFINITY;
        const float top = fmaxf(edge_head, edge_tail);
        if (top > st.m) {
          st.s *= scaled_ex2(st.m - top, c);
          st.m = top;
        }
        if (head_in) st.s += scaled_ex2(edge_head - st.m, c);
        if (tail_in) st.s += scaled_ex2(edge_tail - st.m, c);
      }
      __syncwarp();
      st = warp_join(st, c);
      if (!kGrad) {
        // The loss alone is the first CTA's business: its list warp collects the sums while these warps are a row ahead
        // (at the latest when the second row behind has its own to give).
        if (C > 1) {
          if (pending) cluster_wait();
          if (lane == 0) {
            const uint32_t a = cluster_addr(&s_all[turn][rank * kRowWarps + warp], 0);
            cluster_store_f32(a, st.m);
            cluster_store_f32(a + 4, st.s);
          }
          __syncwarp();
          cluster_arrive();
          pending = true;
        } else if (lane == 0) {
          s_all[turn][warp] = st;                  // (read behind the barrier in front of the next row)
        }
      } else if (C > 1) {                          // to all CTAs of the row
        if (lane < C) {
          const uint32_t a = cluster_addr(&s_all[turn][rank * kRowWarps + warp], lane);
          cluster_store_f32(a, st.m);
          cluster_store_f32(a + 4, st.s);
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
      } else {
        if (lane == 0) s_all[turn][warp] = st;
        cta_barrier();
      }
      if (kGrad) {
        const int n = C * kRowWarps;
        if (p.tail) {
          const Row64 r = row_sums64(s_all[turn], s_list[turn].z_ref, n, p.c64, c.hi);
          ref = r.ref;
          if (r.R != 0.0) coef = tail_factor(r, s_list64[turn][0], s_list64[turn][1]) * (w * p.inv_Tf);
        } else {
          const RowSums r = row_sums(s_all[turn], s_list[turn], n, c);
          ref = r.rest.m;
          if (r.rest.s != 0.f && r.S != 0.f) coef = __fdividef(r.l.mass * r.w_rest, r.S) * (w * p.inv_Tf);
        }
      }
      turn ^= 1;
    } else {
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (!kGrad) {
        for (int q = 0; q < next_deep; ++q) {
          if (q == late) asm volatile("cp.async.commit_group;" ::: "memory");
          if (tid + q * kRowThreads < next_vecs) copy16(s_mine + q * kRowThreads * 16, fetch + q * kRowThreads);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
    }
    // ---- the gradient (zeros where there is nothing to learn)
    if (kGrad) {
      if (head_in) out[tid] = V16::round(w == 0.f ? 0.f : coef * scaled_ex2(edge_head - ref, c));
      if (tail_in) out[tail0 + tid] = V16::round(w == 0.f ? 0.f : coef * scaled_ex2(edge_tail - ref, c));
      const unsigned long long nm2 = f2_pack(-ref, -ref), k2 = f2_pack(coef, coef);
      auto gradient = [&](const uint4& v) {
        float g[V16::kN];
#pragma unroll
        for (int h = 0; h < V16::kN / 2; ++h) {
          float x0, x1;
          const unsigned long long d2 = f2_add(V16::pair(v, h), nm2);
          f2_unpack(f2_fma(d2, cl2, f2_mul(d2, c2)), x0, x1);
          f2_unpack(f2_mul(f2_pack(row_ex2(x0), row_ex2(x1)), k2), g[2 * h], g[2 * h + 1]);
        }
        return V16::pack(g);
      };
      uint4* store = reinterpret_cast<uint4*>(out_vec) + tid;
      uint32_t held = s_mine;
      const int whole = same_align && w != 0.f ? plain : 0;
      int q = 0;
#pragma unroll 1
      for (; (q + kUnroll) * kRowThreads <= whole; q += kUnroll) {
        if (q == late) asm volatile("cp.async.commit_group;" ::: "memory");
        uint4 v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) v[u] = load_shared(held + u * kRowThreads * 16);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) store[u * kRowThreads] = gradient(v[u]);
        if (next_vecs) {
#pragma unroll
          for (int u = 0; u < kUnroll; ++u) copy16(held + u * kRowThreads * 16, fetch + u * kRowThreads);
        }
        held += kUnroll * kRowThreads * 16;
        fetch += kUnroll * kRowThreads;
        store += kUnroll * kRowThreads;
      }
      // the rest, rows of another alignment than the logits', rows there is nothing to learn from (rows of the same
      // length differ by one vector at most, where their alignment differs)
#pragma unroll 1
      for (; q < max(deep, next_deep); ++q, held += kRowThreads * 16, fetch += kRowThreads, store += kRowThreads) {
        if (q == late) asm volatile("cp.async.commit_group;" ::: "memory");
        const int i = tid + q * kRowThreads;
        if (i < n_vec) {
          const uint4 v = w == 0.f ? make_uint4(0, 0, 0, 0) : gradient(load_shared(held));   // (whatever the logits hold)
          if (same_align) {
            *store = v;
          } else {
            T* at = out_vec + (long long)i * V16::kN;
#pragma unroll
            for (int h = 0; h < V16::kN; ++h) at[h] = V16::element(v, h);
          }
        }
        if (i < next_vecs) copy16(held, fetch);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    row = next;
    sp = np;
  }
  cta_barrier();
  if (!kGrad && C > 1 && pending) cluster_wait();
}

// clusters of C CTAs that run on the GPU at a time (asked once per context and size)
template <typename T, bool kGrad, int kLists>
cudaError_t max_clusters(dx_ctx* ctx, int C, size_t smem, int* out) {
  DxClusterCount& known = ctx->distill_clusters[(sizeof(T) == 4 ? 4 : 0) + (kGrad ? 2 : 0) + (kLists == 4 ? 1 : 0)];
  if (known.cluster != C || known.smem != smem) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(C * ctx->sm_count);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    cudaError_t e = cudaOccupancyMaxActiveClusters(&n, dx_distill_kernel<T, kGrad, kLists>, &cfg);
    if (e != cudaSuccess) return e;
    known = DxClusterCount{C, smem, n};
  }
  *out = known.count;
  return cudaSuccess;
}

template <typename T, bool kGrad, int kLists>
cudaError_t launch(dx_ctx* ctx, const DistillParams& p, cudaStream_t st) {
  // CTAs per row: few enough bytes per CTA that two fit an SM (one works while the other waits for its row; four with half
  // the slice took 182 us where two took 172), and as many as fill the GPU when there are few rows (8 x 102400 bf16: 8.0 us,
  // without that 9.9).  (The same with and without the gradient: so is the loss, bit for bit.)
  const long long bytes = (long long)p.V * (long long)sizeof(T);
  const int slots = 2 * ctx->sm_count;
  int C = 1;
  while (C < DX_ROW_CLUSTER_MAX &&
         (bytes > (long long)C * DX_ROW_SLICE_BYTES ||
          ((long long)p.N * C * 2 <= slots && (long long)C * 2 * kRowThreads * 16 <= bytes)))
    C *= 2;
  const long long slice = slice_vectors<T>(p.V, C);
  DistillParams q = p;
  q.half = (int)((slice + kRowThreads * 16 - 1) / (kRowThreads * 16));
  if (q.half < 1) q.half = 1;
  q.late = (int)(slice / kRowThreads & ~(2 * kUnroll - 1)) / 2;
  const size_t held = (size_t)slice * 16;
  // As many clusters as run at a time, each going from row to row with the next row's logits and marks on their way;
  // rows so long that only one set of marks fits get a cluster each.
  const int buffers = held + 2 * 512 * (size_t)q.half + kStaticBytes <= (size_t)ctx->smem_optin ? 2 : 1;
  const size_t smem = held + buffers * 512 * (size_t)q.half;
  int rows = p.N;
  if (buffers == 2) {
    int active = 0;
    cudaError_t e = max_clusters<T, kGrad, kLists>(ctx, C, smem, &active);
    if (e != cudaSuccess) return e;
    if (active < 1) return cudaErrorInvalidConfiguration;
    if (rows > active) rows = active;
  }
  return dx_launch_pdl(false, dx_distill_kernel<T, kGrad, kLists>, dim3((unsigned)rows * C), dim3(kThreads), smem, st, C, q, C,
                       buffers);
}

template <typename T, bool kGrad>
cudaError_t launch_lists(dx_ctx* ctx, const DistillParams& p, cudaStream_t st) {
  return p.k <= 64 ? launch<T, kGrad, 2>(ctx, p, st) : launch<T, kGrad, 4>(ctx, p, st);
}

template <typename K>
cudaError_t prepare(K kernel, int smem) {
  // (what the row's slices are sized by must hold for the kernel as it was compiled)
  cudaFuncAttributes a;
  cudaError_t e = cudaFuncGetAttributes(&a, kernel);
  if (e == cudaSuccess && a.sharedSizeBytes > (size_t)kStaticBytes) e = cudaErrorInvalidConfiguration;
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  return e;
}

}  // namespace

size_t dx_distill_max_row_bytes(const dx_ctx* ctx) {
  return (size_t)(ctx->smem_optin - kStaticBytes - 2048 - 16) * DX_ROW_CLUSTER_MAX;
}

cudaError_t dx_distill_prepare(const dx_ctx* ctx) {
  const int smem = ctx->smem_optin - kStaticBytes;
  cudaError_t e = prepare(dx_distill_kernel<float, true, 2>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<float, true, 4>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<float, false, 2>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<float, false, 4>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<__nv_bfloat16, true, 2>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<__nv_bfloat16, true, 4>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<__nv_bfloat16, false, 2>, smem);
  if (e == cudaSuccess) e = prepare(dx_distill_kernel<__nv_bfloat16, false, 4>, smem);
  return e;
}

cudaError_t dx_launch_distill(dx_ctx* ctx, const void* logits, int dtype, int N, int V, long long ld,
                              const int32_t* teacher_ids, const float* teacher_logprobs, int k, int tail,
                              float temperature, const float* row_weight, float* loss, void* dlogits, long long ld_d,
                              cudaStream_t st) {
  // the first part rounded down, the second positive: a masked logit (-inf) stays -inf times either
  const double c = 1.4426950408889634 / (double)temperature;
  float c_hi = (float)c;
  if ((double)c_hi >= c) c_hi = nextafterf(c_hi, 0.f);
  DistillParams p{logits, N, V, k, tail, 0, 0, ld, ld_d, teacher_ids, teacher_logprobs,
                  c_hi, (float)(c - (double)c_hi), 1.0 / (double)temperature, c, (float)(1.0 / (double)temperature), row_weight, loss, dlogits, ctx->dev_status};
  if (dtype == DX_DTYPE_FP32) return dlogits ? launch_lists<float, true>(ctx, p, st) : launch_lists<float, false>(ctx, p, st);
  return dlogits ? launch_lists<__nv_bfloat16, true>(ctx, p, st) : launch_lists<__nv_bfloat16, false>(ctx, p, st);
}
