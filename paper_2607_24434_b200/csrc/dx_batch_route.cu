// Routing of whole batches: scores, selection with a balance bias and expert groups, gate weights, and the permutation
// of the token-expert pairs by expert; and the gradient of the gate weights with respect to the router logits.
//
//   score   r_e = softmax(z)_e or sigmoid(z_e);   selection value  v_e = r_e + b_e   (z_e itself where there is no bias: the
//   scores are monotone in the logits, and logits can be compared without any rounding)
//   groups  of E / G consecutive experts are ranked by their largest value, or by the sum of their two largest; the best
//   `keep` of them stay;  the k largest values among the experts left are selected, ties to the lower id
//   gate    w_j = scale * r_j  or  scale * r_j / sum_i r_i
//
// The selection is that of 64-bit arithmetic (without a bias: of the logits, exactly).  It is made on unique 32-bit keys
// first: a lane holds eight consecutive experts, whose keys are 24 bits of the value and the reversed expert id -- with a
// bias the value's place between the smallest and the largest that a score plus a bias can have, without one the leading
// bits of the logit (all of a bf16 logit).  A sorting network and k + 1 rounds of a maximum over the token's lanes put them
// in order.  Where two neighbours of the result are closer than keys and arithmetic can tell apart (one token in a thousand
// with a bias and 64 experts), the picks are put in order by their 64-bit values, and where that cannot settle it the whole
// warp makes the token's selection again in 64 bits.  Groups whose scores are as close get theirs from the two or three
// experts concerned.  Biases whose common part is more than about nine times their spread and the scores' leave the keys
// nothing of the scores: every token is then selected in 64 bits (biases of 0.05 randn + 10: 40 us instead of 13.4 at 16384 x
// 64, 157 instead of 39 at 32768 x 256 in groups).
//
// Two launches for a large batch: selection with one histogram of experts per CTA, then the permutation, clusters of
// CTAs adding up the histograms in front of them (a stable counting sort without atomics on device memory; the order
// does not depend on timing).  A small batch is one CTA and one launch.
//
// What bounds it: at 64 experts latencies -- one pass per warp, two launches (16384 fp32 tokens, top-6 with a bias: 13.2 us,
// 7.0 of them the selection); at 256 experts instruction issue (32768 bf16 tokens, top-8 with a bias: 33 us, 39 us with
// groups, 10.7 of them the permutation).  The rare paths are kept short and the parameters in constant memory: cold code
// and a copy of the parameters per thread had made the first two 17 and 53 us.
#include "dx_internal.cuh"

namespace {

constexpr int kThreadsLog = 9;
constexpr int kThreads = 1 << kThreadsLog;
constexpr int kWarps = kThreads / 32;
constexpr int kEpl = 8;           // experts per lane
// How far the difference of two 32-bit selection values may be off, relative to 1 + the largest bias: exponential and
// reciprocal of a score are good to 2^-22 and 2^-23, a softmax's sum adds as much again, the exponent's rounding and the
// addition of the bias half a step each; less than 8e-7 per value.
constexpr float kScoreError = 2e-6f;

struct BatchRouteParams {
  const void* logits;
  int N, E, k;
  long long ld;
  const float* bias;
  int score_fn, norm, groups, keep, group_score;
  float scale;
  int vec;                        // rows can be read in 16-byte vectors
  int per_cta;                    // tokens per CTA
  int32_t* topk_ids;
  float* topk_w;
  int32_t* offsets;
  int32_t* perm;
  int32_t* counts;                // [CTAs][E] context scratch
  int32_t* dev_status;
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }

// Eight consecutive logits of a row; places past the last expert are -inf.
__device__ __forceinline__ void load8(const float* row, int e0, int E, bool vec, float (&z)[kEpl]) {
  if (vec && e0 + kEpl <= E) {
    const float4 a = *reinterpret_cast<const float4*>(row + e0), b = *reinterpret_cast<const float4*>(row + e0 + 4);
    z[0] = a.x; z[1] = a.y; z[2] = a.z; z[3] = a.w; z[4] = b.x; z[5] = b.y; z[6] = b.z; z[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < kEpl; ++i) z[i] = e0 + i < E ? row[e0 + i] : -INFINITY;
  }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* row, int e0, int E, bool vec, float (&z)[kEpl]) {
  if (vec && e0 + kEpl <= E) {
    const uint4 a = *reinterpret_cast<const uint4*>(row + e0);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      z[2 * i] = __uint_as_float(w[i] << 16);
      z[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEpl; ++i) z[i] = e0 + i < E ? to_f(row[e0 + i]) : -INFINITY;
  }
}
__device__ __forceinline__ void store8(float* row, int e0, int E, bool vec, const float (&z)[kEpl]) {
  if (vec && e0 + kEpl <= E) {
    *reinterpret_cast<float4*>(row + e0) = make_float4(z[0], z[1], z[2], z[3]);
    *reinterpret_cast<float4*>(row + e0 + 4) = make_float4(z[4], z[5], z[6], z[7]);
  } else {
#pragma unroll
    for (int i = 0; i < kEpl; ++i)
      if (e0 + i < E) row[e0 + i] = z[i];
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* row, int e0, int E, bool vec, const float (&z)[kEpl]) {
  if (vec && e0 + kEpl <= E) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(z[2 * i + 1]), "f"(z[2 * i]));
    *reinterpret_cast<uint4*>(row + e0) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < kEpl; ++i)
      if (e0 + i < E) row[e0 + i] = __float2bfloat16_rn(z[i]);
  }
}
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// reductions over the G lanes that share a token
template <int G>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int G>
__device__ __forceinline__ unsigned int lanes_umax(unsigned int v) {
  if constexpr (G == 32) {
    return __reduce_max_sync(0xffffffffu, v);
  } else {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  }
}

__device__ __forceinline__ float min_nan(float a, float b) {   // a NaN on either side stays
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float sigmoid_f(float z) { return 1.f / (1.f + expf(-z)); }

// Larger double -> larger integer; -inf (masked experts) -> 1 or more, 0 is left for what is excluded.
__device__ __forceinline__ unsigned long long orderable64(double v) {
  const unsigned long long u = (unsigned long long)__double_as_longlong(v + 0.0);
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

// Puts a token right that 32 bits cannot settle, by a whole warp: lane j < k returns the j-th id.  Lane j <= k has the
// token's j-th pick, `behind` is the key after those, s_row holds E doubles of the warp.
//   The true selection is among the first k + 1 picks unless the key behind them is as close to the border as well; then
// their exact values put them in order: the logits, or the sigmoid in 64 bits and the bias.  Otherwise (`whole`, or a
// softmax's scores, which need the whole row) the selection is made again from the logits in 64 bits.
//   Loops stay rolled and exponentials are calls: few tokens come here, each of them brings this code in from L2 once
// per SM, and the kernel ends with the last one (16384 x 64 fp32, selection alone: 9.8 us unrolled).
__device__ __noinline__ double exact_exp(double x) { return exp(x); }
__device__ __noinline__ double exact_sigmoid(double x) { return 1.0 / (1.0 + exact_exp(-x)); }
template <typename T>
__device__ __noinline__ int settle(const BatchRouteParams& p, const T* row, double* s_row, unsigned int pick,
                                   unsigned int behind, bool whole, unsigned int near) {
  const int lane = threadIdx.x & 31;
  const bool softmax = p.score_fn == DX_SCORE_SOFTMAX;
  const unsigned int border = __shfl_sync(0xffffffffu, pick, p.k - 1);
  whole = whole || (p.bias && softmax) || (behind != 0 && (border >> 8) - (behind >> 8) <= near);
  if (!whole) {
    const int id = pick != 0 ? 255 - (int)(pick & 255u) : DX_MAX_E;
    const float x = pick != 0 ? to_f(row[id]) : -INFINITY;
    double v = (double)x;
    if (p.bias && x > -INFINITY) v = exact_sigmoid(v) + (double)p.bias[id];
    if (!(x > -INFINITY) || !(v == v)) v = -INFINITY;   // (nothing that is not a number is compared)
    int rank = 0;
#pragma unroll 1
    for (int j = 0; j <= p.k; ++j) {
      const double o = __shfl_sync(0xffffffffu, v, j);
      const int oe = __shfl_sync(0xffffffffu, id, j);
      rank += o > v || (o == v && oe < id);
    }
    int* order = reinterpret_cast<int*>(s_row);
    __syncwarp();
    if (pick != 0 && DX_BOUNDS(rank <= p.k, p.dev_status)) order[rank] = id;
    __syncwarp();
    const int mine = order[lane];
    __syncwarp();
    return mine;
  }
  const bool scores = p.bias != nullptr || (p.groups > 1 && p.group_score != DX_GROUP_MAX);
  double m = -INFINITY, s = 0.0;
  if (scores && softmax) {
#pragma unroll 1
    for (int e = lane; e < p.E; e += 32) m = fmax(m, (double)to_f(row[e]));
    for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (m == -INFINITY) m = 0.0;
#pragma unroll 1
    for (int e = lane; e < p.E; e += 32) s += exact_exp((double)to_f(row[e]) - m);
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
  __syncwarp();
#pragma unroll 1
  for (int e = lane; e < p.E; e += 32) {
    const float z = to_f(row[e]);
    double v = (double)z;
    if (scores) v = softmax ? exact_exp(v - m) / s : exact_sigmoid(v);
    if (p.bias) v += (double)p.bias[e];
    if (!(z > -INFINITY) || !(v == v)) v = -INFINITY;
    s_row[e] = v;
  }
  __syncwarp();
  unsigned int kept = 0xffffffffu;
  const int per = p.E / p.groups;
  if (p.groups > 1) {
    double a = -INFINITY, b = -INFINITY;
    if (lane < p.groups) {
      int at = lane % per;                           // (start apart: the lanes read different banks)
#pragma unroll 1
      for (int i = 0; i < per; ++i) {
        const double x = s_row[lane * per + at];
        if (x > a) { b = a; a = x; }
        else if (x > b) b = x;
        at = at + 1 == per ? 0 : at + 1;
      }
      if (p.group_score != DX_GROUP_MAX && b > -INFINITY) a += b;
    }
    int r = 0;
#pragma unroll 1
    for (int g = 0; g < p.groups; ++g) {
      const double o = __shfl_sync(0xffffffffu, a, g);
      r += o > a || (o == a && g < lane);
    }
    kept = __ballot_sync(0xffffffffu, lane < p.groups && r < p.keep);
  }
  // keys: without a bias the experts themselves are compared by their logits
  unsigned long long key[kEpl];
#pragma unroll
  for (int i = 0; i < kEpl; ++i) {
    const int e = lane + 32 * i;
    key[i] = 0ull;
    if (e < p.E && (p.groups == 1 || (kept >> (e / per) & 1u))) {
      const double v = s_row[e];
      key[i] = orderable64(p.bias || v == -INFINITY ? v : (double)to_f(row[e]));
    }
  }
  int mine = 0, head_e = 0;
#pragma unroll 1
  for (int j = 0; j < p.k; ++j) {
    // the lane's first (its lowest expert among equals), then the warp's: high word, low word, expert
    unsigned long long head = 0;
#pragma unroll
    for (int i = 0; i < kEpl; ++i) {
      if (key[i] > head) {
        head = key[i];
        head_e = lane + 32 * i;
      }
    }
    const unsigned int hi = __reduce_max_sync(0xffffffffu, (unsigned int)(head >> 32));
    const unsigned int lo = __reduce_max_sync(0xffffffffu, (unsigned int)(head >> 32) == hi ? (unsigned int)head : 0u);
    const unsigned long long best = (unsigned long long)hi << 32 | lo;
    const int e = (int)__reduce_min_sync(0xffffffffu, head == best ? (unsigned int)head_e : 0xffffu);
    if (lane == j) mine = e;
#pragma unroll
    for (int i = 0; i < kEpl; ++i)
      if (lane + 32 * i == e) key[i] = 0;
  }
  __syncwarp();
  return mine;
}

// Ranks of the groups of a warp's tokens (G lanes each, 1 << gl_log lanes per group) where 32-bit scores leave the border
// open; the scores are sigmoids.  `open`: the lane's group is close to the border; `cand`: those of the lane's experts e0
// + i that can be among the two largest of such a group (two or three, mostly).  Their exact values give the group's
// score in 64 bits; the others keep theirs, which are on their side of the border whatever their last bits.
template <typename T>
__device__ __noinline__ int settle_groups(const BatchRouteParams& p, const T* row, const float* bias, int e0, bool open,
                                          unsigned int cand, float gs, int gl_log, int G) {
  const int lane = threadIdx.x & 31, grp = (lane & (G - 1)) >> gl_log, base = lane & ~(G - 1);
  double a = -INFINITY, b = -INFINITY;
#pragma unroll 1
  while (__any_sync(0xffffffffu, cand != 0)) {
    const int e = e0 + __ffs(cand) - 1;
    const bool in = cand && DX_BOUNDS(e < p.E, p.dev_status);
    const double v = in ? exact_sigmoid((double)to_f(row[e])) + (double)bias[e] : -INFINITY;
    __syncwarp();
    cand &= cand - 1;
    if (v > a) { b = a; a = v; }
    else if (v > b) b = v;
  }
#pragma unroll 1
  for (int o = 1; o < 1 << gl_log; o <<= 1) {
    const double oa = __shfl_xor_sync(0xffffffffu, a, o), ob = __shfl_xor_sync(0xffffffffu, b, o);
    b = fmax(fmax(b, ob), fmin(a, oa));
    a = fmax(a, oa);
  }
  const double g = !open ? (double)gs : p.group_score == DX_GROUP_MAX || b == -INFINITY ? a : a + b;
  int r = 0;
#pragma unroll 1
  for (int i = 0; i < p.groups; ++i) {
    const double o = __shfl_sync(0xffffffffu, g, base + (i << gl_log));
    r += o > g || (o == g && i < grp);
  }
  return r;
}

// Where the pairs of a CTA's tokens go: s_base[e] = first place of expert e's.  The pairs are taken kTile at a time, a
// contiguous stretch of 32 * kDeep per warp, so that equal experts keep the order of their pairs.
constexpr int kDeep = 2;
constexpr int kTile = kWarps * 32 * kDeep;
struct Pairs {
  int id[kDeep];
  unsigned int same[kDeep];   // the warp's lanes with the same expert
};
__device__ __forceinline__ void load_pairs(const int32_t* ids, long long p0, int at, int n, Pairs& q) {
  const int first = at + (threadIdx.x >> 5) * 32 * kDeep + (threadIdx.x & 31);
#pragma unroll
  for (int d = 0; d < kDeep; ++d) q.id[d] = first + 32 * d < n ? ids[p0 + first + 32 * d] : -1;
}
// pairs of each expert per warp
__device__ __forceinline__ void count_pairs(Pairs& q, int E, int (*s_hist)[DX_MAX_E], int32_t* dev_status) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int e = lane; e < E; e += 32) s_hist[warp][e] = 0;
  __syncwarp();
#pragma unroll
  for (int d = 0; d < kDeep; ++d) {
    if (!DX_BOUNDS(q.id[d] < E, dev_status)) q.id[d] = -1;
    q.same[d] = __match_any_sync(0xffffffffu, q.id[d]);
    if (q.id[d] >= 0 && __ffs(q.same[d]) - 1 == lane) s_hist[warp][q.id[d]] += __popc(q.same[d]);
    __syncwarp();
  }
}
// ... turned into the pairs of the warps in front; s_total[e] += those of all warps
__device__ __forceinline__ void front_of_warps(int E, int (*s_hist)[DX_MAX_E], int* s_total) {
  for (int e = threadIdx.x; e < E; e += kThreads) {
    int c[kWarps], x = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) c[w] = s_hist[w][e];
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      s_hist[w][e] = x;
      x += c[w];
    }
    s_total[e] = x;
  }
}
// (a place past the permutation can only come of counts that another call has overwritten -- the context's scratch shared by
// streams that are not ordered: it is not written)
__device__ __forceinline__ void scatter_pairs(const Pairs& q, long long first_pair, const int* s_base,
                                              int (*s_hist)[DX_MAX_E], const BatchRouteParams& p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long first = first_pair + warp * 32 * kDeep + lane;
#pragma unroll
  for (int d = 0; d < kDeep; ++d) {
    const int x = q.id[d] >= 0 ? s_hist[warp][q.id[d]] : 0;
    __syncwarp();
    if (q.id[d] >= 0) {
      const int at = s_base[q.id[d]] + x + __popc(q.same[d] & ((1u << lane) - 1u));
      if ((unsigned int)at < (unsigned int)(p.N * p.k)) p.perm[at] = (int32_t)(first + 32 * d);
      else (void)DX_BOUNDS(false, p.dev_status);
      if (__ffs(q.same[d]) - 1 == lane) s_hist[warp][q.id[d]] = x + __popc(q.same[d]);
    }
    __syncwarp();
  }
}
// the tiles from the first on (whose counts are in place, s_total and s_base filled)
__device__ __forceinline__ void place_pairs(const BatchRouteParams& p, long long p0, int n, int (*s_hist)[DX_MAX_E],
                                            int* s_base, int* s_total, Pairs& q) {
  const int E = p.E;
#pragma unroll 1
  for (int at = 0; at < n; at += kTile) {
    if (at > 0) {
      load_pairs(p.topk_ids, p0, at, n, q);
      __syncthreads();                               // (the tile in front has been placed)
      for (int e = threadIdx.x; e < E; e += kThreads) s_base[e] += s_total[e];
      count_pairs(q, E, s_hist, p.dev_status);
      __syncthreads();
      front_of_warps(E, s_hist, s_total);
      __syncthreads();
    }
    scatter_pairs(q, p0 + at, s_base, s_hist, p);
  }
}

// exclusive prefix over E <= kThreads counts; thread e passes count e and gets the sum of the counts in front of it
__device__ __forceinline__ int prefix_counts(int c, int* s_scan) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = c;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_scan[warp] = x;
  __syncthreads();
  int before_warp = 0;
  for (int w = 0; w < warp; ++w) before_warp += s_scan[w];
  return before_warp + x - c;
}

// Score as the keys see it: ex2 and rcp of the hardware, good to 2^-22 and 1 step; |z| adds |z| 2^-24 to the exponent,
// and |z| sigmoid'(z) stays below 0.23.
__device__ __forceinline__ float sigmoid_fast(float z) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}
__device__ __forceinline__ float exp_fast(float x) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * 1.4426950408889634f));
  return e;
}

// G lanes per token.  What the selection goes by: the logits, or scores (a bias, or groups ranked by a sum).
enum { kByLogits, kBySigmoid, kBySoftmax };
template <typename T, int G, int kBy>
__global__ void __launch_bounds__(kThreads, 2) dx_batch_route_kernel(const __grid_constant__ BatchRouteParams p) {
  constexpr int kTok = 32 / G;                       // tokens a warp works on side by side
  constexpr int kPicks = G == 4 ? 3 : G == 8 ? 2 : 1;   // picks (of k + 1) per lane
  constexpr int kGateLanes = G < DX_MAX_TOPK ? G : DX_MAX_TOPK;   // the lanes that have the selected experts
  constexpr bool kScores = kBy != kByLogits;
  constexpr unsigned int kMask = G == 32 ? 0xffffffffu : (1u << (G % 32)) - 1u;
  __shared__ int s_count[DX_MAX_E];
  __shared__ __align__(16) float s_bias[DX_MAX_E];
  __shared__ unsigned char s_gid[DX_MAX_E];
  __shared__ int s_base[DX_MAX_E];
  __shared__ int s_scan[kWarps];
  __shared__ __align__(16) union {
    double exact[kWarps][DX_MAX_E];                  // 64-bit scores of the token a warp selects again, or its values
    int hist[kWarps][DX_MAX_E];
  } s_mem;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % G, tok = lane / G;
  const int E = p.E, k = p.k, e0 = sub * kEpl;
  const int per = E / p.groups;
  // a group is a whole number of lanes, a power of two of them: its score comes out of a few exchanges
  const int gl = per / kEpl;
  const bool lane_groups = p.groups > 1 && per % kEpl == 0 && (gl & (gl - 1)) == 0;
  const int gl_log = lane_groups ? __ffs(gl) - 1 : 0;
  const bool biased = kScores && p.bias != nullptr;
  const bool softmax = kScores ? kBy == kBySoftmax : p.score_fn == DX_SCORE_SOFTMAX;
  dx_pdl_trigger();            // (the permutation waits for this kernel's end before it reads anything)
  for (int e = threadIdx.x; e < DX_MAX_E; e += kThreads) {
    s_count[e] = 0;
    const float b = biased && e < E ? p.bias[e] : 0.f;
    s_bias[e] = b == b ? b : -INFINITY;              // (a NaN would be in no place of any order)
    s_gid[e] = (unsigned char)(min(e, E - 1) / per);
  }
  __syncthreads();
  // keys of biased values: their place in [least bias, 1 + greatest bias]
  float key_mul = 0.f, key_add = 0.f, bias_abs = 0.f;
  bool key_ok = true;
  unsigned int near = 0;                             // keys of that many quanta or fewer apart are not told apart
  if (biased) {
    float lo = INFINITY, hi = -INFINITY;
    for (int e = lane; e < E; e += 32) {
      if (s_bias[e] > -INFINITY) lo = fminf(lo, s_bias[e]);   // (experts at -inf get the key of the masked ones)
      hi = fmaxf(hi, s_bias[e]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    bias_abs = fmaxf(fabsf(lo), fabsf(hi));
    // value -> 2^23 + quanta: the low 24 bits of the float are the quanta, bit 23 being zero (at least 8, masked experts have 1: key_add's
    // share is rounded, by less than 4 up to the bound that follows)
    key_mul = 8388000.f / (1.f + hi - lo);
    const float shift = 8.f - lo * key_mul;
    key_add = 8388608.f + shift;
    key_ok = fabsf(shift) < 6e7f && key_mul > 0.f;   // (infinite or far-off biases: every token is selected in 64 bits)
    near = 4u + (unsigned int)fminf(kScoreError * (1.f + bias_abs) * key_mul, 8e6f);
  }
  const float4* bias8 = reinterpret_cast<const float4*>(s_bias + min(e0, DX_MAX_E - kEpl));

  const long long t_lo = (long long)blockIdx.x * p.per_cta;
  const long long t_hi = min((long long)p.N, t_lo + p.per_cta);
#pragma unroll 1
  for (long long t0 = t_lo + warp * kTok; t0 < t_hi; t0 += kWarps * kTok) {
    const bool active = t0 + tok < t_hi;
    const long long t = active ? t0 + tok : t_hi - 1;   // (lanes without a token repeat the last one and write nothing)
    const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
    float z[kEpl];                                   // logits, then values; -inf: masked (a NaN is)
    load8(row, e0, E, p.vec != 0, z);
    float m = -INFINITY, inv = 0.f;
    bool odd = false;                                // a sum that is not a number: no score says anything
    if (softmax && (kScores || !p.norm)) {
      float s = 0.f, bad = 0.f;
#pragma unroll
      for (int i = 0; i < kEpl; ++i) {
        m = fmaxf(m, z[i]);
        bad += z[i] != z[i] ? 1.f : 0.f;
      }
      m = lanes_max<G>(m);
#pragma unroll
      for (int i = 0; i < kEpl; ++i) s += z[i] > -INFINITY ? exp_fast(z[i] - m) : 0.f;
      s = lanes_sum<G>(s + (bad > 0.f ? __uint_as_float(0x7fc00000u) : 0.f));
      odd = s != s;
      inv = s;
    }
    bool doubt = biased && !key_ok;
    unsigned int kept = 0xffffffffu;
    if (kScores) {
      const float rcp = softmax ? 1.f / inv : 0.f;
      const float4 b0 = bias8[0], b1 = bias8[1];
      const float b[kEpl] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
      float least = z[0];
#pragma unroll
      for (int i = 1; i < kEpl; ++i) least = min_nan(least, z[i]);
      unsigned int masked = 0;                       // (masked experts are rare: a warp that has none skips them)
      if (__any_sync(0xffffffffu, !(least > -INFINITY) || odd)) {
#pragma unroll
        for (int i = 0; i < kEpl; ++i) masked |= (unsigned int)(!(z[i] > -INFINITY) || odd) << i;
      }
#pragma unroll
      for (int i = 0; i < kEpl; ++i)
        z[i] = (softmax ? exp_fast(z[i] - m) * rcp : sigmoid_fast(z[i])) + b[i];
      if (__any_sync(0xffffffffu, masked != 0)) {
#pragma unroll
        for (int i = 0; i < kEpl; ++i) z[i] = masked >> i & 1u ? -INFINITY : z[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kEpl; ++i) z[i] = fmaxf(z[i], -INFINITY);
    }
    // ---- groups
    if (p.groups > 1) {
      float g1 = -INFINITY, g2 = -INFINITY;          // two largest values of the group
      if (lane_groups) {
#pragma unroll
        for (int i = 0; i < kEpl; ++i) {
          g2 = fmaxf(g2, fminf(g1, z[i]));
          g1 = fmaxf(g1, z[i]);
        }
        for (int o = 1; o < gl; o <<= 1) {
          const float o1 = __shfl_xor_sync(0xffffffffu, g1, o), o2 = __shfl_xor_sync(0xffffffffu, g2, o);
          g2 = fmaxf(fmaxf(g2, o2), fminf(g1, o1));
          g1 = fmaxf(g1, o1);
        }
      } else {
        float* stage = reinterpret_cast<float*>(s_mem.exact[warp]) + tok * G * kEpl;
#pragma unroll
        for (int i = 0; i < kEpl; ++i) stage[e0 + i] = z[i];
        __syncwarp();
        if (sub < p.groups) {
          int at = sub % per;                        // (start apart: the lanes read different banks)
          for (int i = 0; i < per; ++i) {
            const float x = stage[sub * per + at];
            g2 = fmaxf(g2, fminf(g1, x));
            g1 = fmaxf(g1, x);
            at = at + 1 == per ? 0 : at + 1;
          }
        }
        __syncwarp();
      }
      const float gs = p.group_score == DX_GROUP_MAX || g2 == -INFINITY ? g1 : g1 + g2;
      // A group's rank is the number of groups in front of it, counted by its lanes side by side (lane g has group g
      // where a group is not a number of lanes); scores that the arithmetic cannot tell apart at the border raise the doubt.
      const int grp = sub >> gl_log;
      int r = 0;
      for (int i0 = 0; i0 < p.groups; i0 += 1 << gl_log) {
        const int i = i0 + (sub & ((1 << gl_log) - 1));
        const float o = __shfl_sync(0xffffffffu, gs, tok * G + (min(i, p.groups - 1) << gl_log));
        r += i < p.groups && (o > gs || (o == gs && i < grp));
      }
      for (int o = 1; o < 1 << gl_log; o <<= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
      if (grp >= p.groups) r = DX_MAX_GROUPS;
      const unsigned int last = __ballot_sync(0xffffffffu, r == p.keep - 1) >> (tok * G) & kMask;
      const unsigned int next = __ballot_sync(0xffffffffu, r == p.keep) >> (tok * G) & kMask;   // (keep < groups)
      const float g_in = __shfl_sync(0xffffffffu, gs, tok * G + __ffs(last) - 1);
      const float g_out = __shfl_sync(0xffffffffu, gs, tok * G + __ffs(next) - 1);
      // (logits are compared as they are; infinite on both sides: not close)
      if (kScores) {
        const float err = kScoreError * (1.f + bias_abs);
        const bool open = fabsf(g_in - g_out) <= 2.f * err;
        if (kBy == kBySigmoid && lane_groups) {
          if (__any_sync(0xffffffffu, open)) {
            const bool mine = open && grp < p.groups && (fabsf(gs - g_in) <= 2.f * err || fabsf(gs - g_out) <= 2.f * err);
            const float from = (p.group_score == DX_GROUP_MAX ? g1 : g2) - err;
            unsigned int cand = 0;
#pragma unroll
            for (int i = 0; i < kEpl; ++i) cand |= (unsigned int)(mine && z[i] >= from && z[i] > -INFINITY) << i;
            r = settle_groups(p, row, s_bias, e0, mine, cand, gs, gl_log, G);
            if (grp >= p.groups) r = DX_MAX_GROUPS;
          }
        } else {
          doubt |= open;
        }
      }
      kept = __ballot_sync(0xffffffffu, r < p.keep) >> (tok * G) & kMask;   // by lane
    }
    if (kScores && !biased) {                        // (the scores were for the groups; experts go by their logits)
      load8(row, e0, E, p.vec != 0, z);
#pragma unroll
      for (int i = 0; i < kEpl; ++i) z[i] = fmaxf(z[i], -INFINITY);
    }
    // ---- unique keys; 0: excluded or no expert
    unsigned int key[kEpl];
#pragma unroll
    for (int i = 0; i < kEpl; ++i) {
      const unsigned int id = (unsigned int)(255 - e0 - i);
      if (biased) {   // (not a number, or below: masked)
        key[i] = __byte_perm(__float_as_uint(fmaxf(fmaf(z[i], key_mul, key_add), 8388609.f)), id, 0x2104);
      } else {
        key[i] = __byte_perm(dx_orderable(z[i] + 0.f), id, 0x3214);
      }
    }
    // (where the lane's experts stay or go together, it is enough that the lane has no first key)
    const bool on = e0 < E && (p.groups == 1 || !lane_groups || (kept >> sub & 1u));
    if (!lane_groups && (p.groups > 1 || (E & (kEpl - 1)) != 0)) {
#pragma unroll
      for (int i = 0; i < kEpl; ++i) {
        const bool in = e0 + i < E && (kept >> s_gid[min(e0 + i, DX_MAX_E - 1)] & 1u);
        key[i] = in ? key[i] : 0u;
      }
    }
    // ---- the lane's keys in descending order (19 exchanges: the network of Bose and Nelson, 1962)
#define DX_EXCHANGE(a, c) { const unsigned int hi_ = max(key[a], key[c]), lo_ = min(key[a], key[c]); key[a] = hi_; key[c] = lo_; }
    DX_EXCHANGE(0, 1) DX_EXCHANGE(2, 3) DX_EXCHANGE(4, 5) DX_EXCHANGE(6, 7)
    DX_EXCHANGE(0, 2) DX_EXCHANGE(1, 3) DX_EXCHANGE(4, 6) DX_EXCHANGE(5, 7)
    DX_EXCHANGE(1, 2) DX_EXCHANGE(5, 6) DX_EXCHANGE(0, 4) DX_EXCHANGE(3, 7)
    DX_EXCHANGE(1, 5) DX_EXCHANGE(2, 6)
    DX_EXCHANGE(1, 4) DX_EXCHANGE(3, 6)
    DX_EXCHANGE(2, 4) DX_EXCHANGE(3, 5)
    DX_EXCHANGE(3, 4)
#undef DX_EXCHANGE
    // ---- k + 1 rounds: lane j of the token's lanes keeps pick j (j + G, j + 2 G); a lane's next key comes out of shared
    // memory when its first has been taken
    unsigned int pick[kPicks] = {};
    unsigned int* list = reinterpret_cast<unsigned int*>(s_mem.exact[warp]) + lane;
    __syncwarp();
#pragma unroll
    for (int i = 1; i < kEpl; ++i) list[i * 32] = key[i];
    list[kEpl * 32] = 0u;
    unsigned int head = on ? key[0] : 0u;
    list += 32;
#pragma unroll 1
    for (int j = 0, at = sub; j <= k; ++j, --at) {
      const unsigned int top = lanes_umax<G>(head);
#pragma unroll
      for (int h = 0; h < kPicks; ++h)
        if (at == -h * G) pick[h] = top;             // (j == h * G + sub)
      if (head == top && top != 0u) {
        head = *list;
        list += 32;
      }
    }
    __syncwarp();
    // ---- the picks' logits, and neighbours that 32 bits cannot tell apart
    int id[kPicks];
    float x[kPicks];
    unsigned int below[kPicks];
    bool close = false;
#pragma unroll
    for (int h = 0; h < kPicks; ++h) {
      id[h] = 255 - (int)(pick[h] & 255u);
      const bool in = h * G + sub <= k && pick[h] != 0 && DX_BOUNDS(id[h] >= 0 && id[h] < E, p.dev_status);
      x[h] = in ? to_f(row[id[h]]) : -INFINITY;
      below[h] = __shfl_sync(0xffffffffu, pick[h], tok * G + (sub + 1) % G);
      if (h + 1 < kPicks) {                          // (the last lane's neighbour is the first lane's next pick)
        const unsigned int w = __shfl_sync(0xffffffffu, pick[h + 1 < kPicks ? h + 1 : h], tok * G);
        if (sub == G - 1) below[h] = w;
      }
      // (the keys of bf16 logits hold all of them)
      if (kScores || sizeof(T) == 4)
        close |= h * G + sub < k && below[h] != 0 && (pick[h] >> 8) - (below[h] >> 8) <= near;
    }
    if (__any_sync(0xffffffffu, close)) {
      close = false;
#pragma unroll
      for (int h = 0; h < kPicks; ++h) {
        const int j = h * G + sub;                   // neighbours j and j + 1 (j + 1 == k: the first that is left out)
        if (j < k && below[h] != 0 && x[h] > -INFINITY && (pick[h] >> 8) - (below[h] >> 8) <= near) {
          const int eb = 255 - (int)(below[h] & 255u);
          const float xb = to_f(row[eb]);
          // equal logits under equal biases are a true tie, in the right order already -- but at the border only if
          // equal keys are equal logits
          bool tie = x[h] == xb || !(xb > -INFINITY);
          if (biased && xb > -INFINITY) tie = tie && s_bias[id[h]] == s_bias[eb];
          if (j + 1 == k && xb > -INFINITY) tie = tie && !biased && sizeof(T) == 2;
          close |= !tie;
        }
      }
    }
    const bool unsure = (__ballot_sync(0xffffffffu, close) >> (tok * G) & kMask) != 0;
    const unsigned int open = __ballot_sync(0xffffffffu, doubt || unsure);
    if (open != 0) {
      const unsigned int behind = lanes_umax<G>(head);
#pragma unroll 1
      for (int q = 0; q < kTok; ++q) {
        if (!(open >> (q * G) & 1u)) continue;       // (the same for the whole warp)
        const long long tq = min(t0 + q, t_hi - 1);
        unsigned int mine = 0;                       // pick j of the token in lane j
#pragma unroll
        for (int h = 0; h < kPicks; ++h) {
          const unsigned int y = __shfl_sync(0xffffffffu, pick[h], q * G + sub);
          if (tok == h) mine = y;
        }
        const int got = settle(p, reinterpret_cast<const T*>(p.logits) + (size_t)tq * (size_t)p.ld, s_mem.exact[warp], mine,
                               __shfl_sync(0xffffffffu, behind, q * G), __shfl_sync(0xffffffffu, (int)doubt, q * G) != 0, near);
#pragma unroll
        for (int h = 0; h < kPicks; ++h) {
          const int y = __shfl_sync(0xffffffffu, got, (sub + h * G) % 32);
          if (tok == q && h * G + sub < k && DX_BOUNDS(y >= 0 && y < E, p.dev_status)) {
            id[h] = y;
            x[h] = to_f(row[y]);
          }
        }
      }
    }
    // ---- gate weights of the selected experts
    constexpr int kH = G < DX_MAX_TOPK ? 2 : 1;      // pairs per lane
    float w[kH], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int h = 0; h < kH; ++h) {
      if (h * G + sub >= k) x[h] = -INFINITY;
      top = fmaxf(top, x[h]);
    }
    if (p.norm) top = lanes_max<kGateLanes>(top);
#pragma unroll
    for (int h = 0; h < kH; ++h) {
      // Renormalised gates are ratios: softmax needs no more of the row than e^{x - top}, and sigmoid(x) is e^x to 32
      // bits where it is small enough to underflow.
      const bool ratio = p.norm && (softmax || top < -64.f);
      const float ref = softmax || ratio ? (p.norm ? top : m) : 0.f;
      const float e = expf(softmax || ratio ? x[h] - ref : -x[h]);
      w[h] = x[h] == -INFINITY ? 0.f : softmax || ratio ? e : __fdividef(1.f, 1.f + e);
      sum += w[h];
    }
    float f = p.scale;
    if (p.norm) {
      sum = lanes_sum<kGateLanes>(sum);
      f = sum > 0.f || sum != sum ? p.scale / sum : 0.f;
    } else if (softmax) {
      // (the keys' fast sum is not good enough for the gates)
      float z8[kEpl], s = 0.f;
      load8(row, e0, E, p.vec != 0, z8);
#pragma unroll
      for (int i = 0; i < kEpl; ++i) s += z8[i] == -INFINITY ? 0.f : expf(z8[i] - m);
      s = lanes_sum<G>(s);
      f = s > 0.f || s != s ? p.scale / s : 0.f;
    }
#pragma unroll
    for (int h = 0; h < kH; ++h) {
      const int j = h * G + sub;
      if (active && j < k && DX_BOUNDS(id[h] >= 0 && id[h] < E, p.dev_status)) {
        p.topk_ids[t * k + j] = id[h];
        p.topk_w[t * k + j] = w[h] * f;
        atomicAdd(&s_count[id[h]], 1);
      }
    }
  }
  if (!p.perm) return;
  __syncthreads();
  if (gridDim.x > 1) {
    for (int e = threadIdx.x; e < E; e += kThreads) p.counts[(size_t)blockIdx.x * E + e] = s_count[e];
    return;
  }
  // one CTA: the whole permutation here
  const int c = threadIdx.x < E ? s_count[threadIdx.x] : 0;
  const int at = prefix_counts(c, s_scan);
  if (threadIdx.x < E) {
    s_base[threadIdx.x] = at;
    p.offsets[threadIdx.x] = at;
  }
  if (threadIdx.x == 0) p.offsets[E] = p.N * k;
  __syncthreads();
  Pairs q;
  load_pairs(p.topk_ids, 0, 0, p.N * k, q);
  count_pairs(q, E, s_mem.hist, p.dev_status);
  __syncthreads();
  front_of_warps(E, s_mem.hist, s_count);
  __syncthreads();
  place_pairs(p, 0, p.N * k, s_mem.hist, s_base, s_count, q);
}

// Clusters of kPermCluster CTAs share the sums over the histograms: CTA r of a cluster adds up every kPermCluster-th part
// of them, once over all CTAs (the experts' totals) and once over those in front of the cluster; its threads take the
// experts several times over.  What needs the CTA's own pairs alone is done while the sums are on their way.
constexpr int kPermCluster = 8;
__global__ void __launch_bounds__(kThreads) dx_batch_permute_kernel(BatchRouteParams p, int n_ctas, int e_log) {
  __shared__ int s_hist[kWarps][DX_MAX_E];
  __shared__ int s_base[DX_MAX_E], s_total[DX_MAX_E];
  __shared__ int s_scan[kWarps];
  __shared__ int2 s_part[DX_MAX_E];
  const int E = p.E, e = threadIdx.x & ((1 << e_log) - 1), seg = threadIdx.x >> e_log, segs_log = kThreadsLog - e_log;
  const int rank = blockIdx.x % kPermCluster, first = blockIdx.x - rank;   // (clusters are runs of the grid)
  const long long t_lo = (long long)blockIdx.x * p.per_cta;
  const long long t_hi = min((long long)p.N, t_lo + p.per_cta);
  const int n = t_lo < t_hi ? (int)(t_hi - t_lo) * p.k : 0;
  if (threadIdx.x < DX_MAX_E) s_part[threadIdx.x] = make_int2(0, 0);
  __syncthreads();
  dx_pdl_wait();               // (launched while the selection drains)
  Pairs q;
  load_pairs(p.topk_ids, t_lo * p.k, 0, n, q);
  const int32_t* col = p.counts + e;
  int front = 0, total = 0, near = 0;
  if (e < E) {
    const int all_lo = n_ctas * rank / kPermCluster;
    const int all_hi = n_ctas * (rank + 1) / kPermCluster;
    const int lo = all_lo + ((all_hi - all_lo) * seg >> segs_log), hi = all_lo + ((all_hi - all_lo) * (seg + 1) >> segs_log);
    // (short code: every instruction of this kernel comes out of L2 once, and that is a good part of its time)
    const int32_t* at = col + (size_t)lo * E;
#pragma unroll 8
    for (int b = lo; b < hi; ++b, at += E) {
      const int c = *at;
      total += c;
      front += b < first ? c : 0;
    }
    // (the CTAs of the cluster in front of this one; up to two experts per warp lane: four loads side by side)
    at = col + (size_t)(first + seg) * E;
#pragma unroll
    for (int i = 0; i < 4; ++i, at += (size_t)E << segs_log)
      if (first + seg + (i << segs_log) < min((int)blockIdx.x, n_ctas)) near += *at;
  }
  count_pairs(q, E, s_hist, p.dev_status);
  if (e < E) {
    atomicAdd(&s_part[e].x, total);
    atomicAdd(&s_part[e].y, front);
  }
  __syncthreads();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  if (threadIdx.x < DX_MAX_E) s_base[threadIdx.x] = 0;
  front_of_warps(E, s_hist, s_total);
  __syncthreads();
  if (e < E && near != 0) atomicAdd(&s_base[e], near);
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  total = front = 0;
  if (threadIdx.x < E) {
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(&s_part[threadIdx.x]));
#pragma unroll
    for (int r = 0; r < kPermCluster; ++r) {
      uint32_t a;
      int x, y;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(mine), "r"(r));
      asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "r"(a) : "memory");
      total += x;
      front += y;
    }
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  const int at = prefix_counts(total, s_scan);       // (a barrier of the CTA among it: s_base is complete)
  if (threadIdx.x < E) {
    s_base[threadIdx.x] += at + front;
    if (blockIdx.x == 0) p.offsets[threadIdx.x] = at;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[E] = p.N * p.k;
  __syncthreads();
  place_pairs(p, t_lo * p.k, n, s_hist, s_base, s_total, q);
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- backward ---------------------------------------------------------------------------------------------------------
// With S = sum_i r_i over the selected and g the gradient of the gates,
//   dL/dr_j = scale * g_j   or   scale * (g_j - sum_i g_i r_i / S) / S,
// sigmoid: dz_e = dL/dr_e r_e (1 - r_e);  softmax: dz_e = r_e (dL/dr_e - sum_j dL/dr_j r_j), dL/dr zero for experts that
// were not selected.  For renormalised gates that last sum is zero, so only softmax gates that are not renormalised
// have a gradient outside the selection, and only they need the whole row of logits.
constexpr int kGradThreads = 256;   // (512: 17.7 us instead of 14.5, cold)
constexpr int kGradWarps = kGradThreads / 32;

struct RouteGradParams {
  const void* logits;
  int N, E, k;
  long long ld;
  const int32_t* ids;
  const float* dw;
  int score_fn, norm;
  float scale;
  int vec_in, vec_out;
  void* dlogits;
  long long ld_d;
  int32_t* dev_status;
};

// A pair of a token: lane j of the token's lanes holds pair j (id -1: none).
struct Pair {
  int id;
  float g, x;                 // gradient of the gate, logit
};
template <typename T>
__device__ __forceinline__ Pair load_pair(const RouteGradParams& p, long long t, const T* row, int j) {
  Pair q{-1, 0.f, -INFINITY};
  if (j < p.k) {
    q.id = p.ids[t * p.k + j];
    q.g = p.dw[t * p.k + j] * p.scale;
    if (q.id < 0 || q.id >= p.E) {
      *p.dev_status = DX_DEV_BAD_EXPERT_ID;
      q.id = -1;
      q.g = 0.f;
    } else {
      q.x = to_f(row[q.id]);
    }
  }
  return q;
}
// an expert listed twice gets the sum of its pairs' gradients (`tok`: the token's place in the warp)
template <int G>
__device__ __forceinline__ float sum_duplicates(int id, float g, int tok, int k) {
  const unsigned int same = __match_any_sync(0xffffffffu, id < 0 ? -1 - (int)(threadIdx.x & 31) : tok << 16 | id);
  float both = g;
  if (__any_sync(0xffffffffu, __popc(same) > 1)) {
    both = 0.f;
    for (int j = 0; j < k; ++j) {
      const int src = tok * G + j;
      const float og = __shfl_sync(0xffffffffu, g, src);
      if (same >> src & 1u) both += og;
    }
  }
  return both;
}

// Gradients that are zero outside the selection: a warp takes four tokens, eight lanes for the pairs of each, writes
// the zeros of their rows with all lanes and then the selected experts' places.  Bound by HBM: 65536 x 256 bf16 14.5 us
// with cold inputs, 76 % of the measured copy bandwidth (as one dense pass over rows of both: 25.6 us).
template <typename T>
__global__ void __launch_bounds__(kGradThreads) dx_route_grad_sparse_kernel(RouteGradParams p) {
  constexpr int G = DX_MAX_TOPK, kTok = 32 / G, kN = 16 / sizeof(T);
  const int lane = threadIdx.x & 31, sub = lane % G, tok = lane / G;
  const int E = p.E;
  const bool softmax = p.score_fn == DX_SCORE_SOFTMAX;
  const long long warps = (long long)gridDim.x * kGradWarps;
#pragma unroll 1
  for (long long t0 = ((long long)blockIdx.x * kGradWarps + (threadIdx.x >> 5)) * kTok; t0 < p.N; t0 += warps * kTok) {
    const bool active = t0 + tok < p.N;
    const long long t = active ? t0 + tok : p.N - 1;
    const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
    T* out0 = reinterpret_cast<T*>(p.dlogits) + (size_t)t0 * (size_t)p.ld_d;
    const int rows = (int)min((long long)kTok, p.N - t0);
    // the pairs' loads are on their way while the zeros are written
    const Pair q = load_pair(p, t, row, sub);
    for (int r = 0; r < rows; ++r) {
      T* out = out0 + (size_t)r * (size_t)p.ld_d;
      if (p.vec_out) {
        for (int e = lane * kN; e + kN <= E; e += 32 * kN) *reinterpret_cast<uint4*>(out + e) = make_uint4(0, 0, 0, 0);
        if (lane < E % kN) store1(out + E - E % kN + lane, 0.f);
      } else {
        for (int e = lane; e < E; e += 32) store1(out + e, 0.f);
      }
    }
    const float top = lanes_max<G>(q.x);
    // renormalised gates: a common factor of the scores cancels (e^{x - top} for softmax; sigmoid(x) is e^x where it is
    // small)
    const bool ratio = softmax || (p.norm && top < -64.f);
    const float e = expf(ratio ? q.x - top : -q.x);
    const float r = q.x == -INFINITY ? 0.f : ratio ? e : 1.f / (1.f + e);
    const float slope = softmax ? 1.f : sigmoid_f(-q.x);             // 1 - sigmoid
    float g = q.g;
    if (p.norm) {
      const float S = lanes_sum<G>(r);
      const float mean = lanes_sum<G>(g * (r / S));    // (shares first: an only expert's is 1 and its gradient zero)
      g = S == 0.f || q.id < 0 ? 0.f : (g - mean) / S;
    }
    const float both = sum_duplicates<G>(q.id, g, tok, p.k);
    __syncwarp();                                      // the zeros are written before the selected experts' places are
    if (active && q.id >= 0)
      store1(reinterpret_cast<T*>(p.dlogits) + (size_t)t * (size_t)p.ld_d + q.id, both * r * slope);
    __syncwarp();
  }
}

// Softmax gates that are not renormalised: every expert's logit has a gradient.  G lanes per token, at least eight.
template <typename T, int G>
__global__ void __launch_bounds__(kGradThreads) dx_route_grad_dense_kernel(RouteGradParams p) {
  constexpr int kTok = 32 / G;
  const int lane = threadIdx.x & 31, sub = lane % G, tok = lane / G;
  const int E = p.E, e0 = sub * kEpl;
  const long long warps = (long long)gridDim.x * kGradWarps;
#pragma unroll 1
  for (long long t0 = ((long long)blockIdx.x * kGradWarps + (threadIdx.x >> 5)) * kTok; t0 < p.N; t0 += warps * kTok) {
    const bool active = t0 + tok < p.N;
    const long long t = active ? t0 + tok : p.N - 1;
    const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
    T* out = reinterpret_cast<T*>(p.dlogits) + (size_t)t * (size_t)p.ld_d;
    float d[kEpl];
    load8(row, e0, E, p.vec_in != 0, d);
    const Pair q = load_pair(p, t, row, sub);
    float m = d[0], s = 0.f;
#pragma unroll
    for (int i = 1; i < kEpl; ++i) m = fmaxf(m, d[i]);
    m = lanes_max<G>(m);
#pragma unroll
    for (int i = 0; i < kEpl; ++i) {
      d[i] = d[i] == -INFINITY ? 0.f : expf(d[i] - m);
      s += d[i];
    }
    s = lanes_sum<G>(s);
    const float inv = s == 0.f ? 0.f : 1.f / s;
    const float r = q.x == -INFINITY ? 0.f : expf(q.x - m) * inv;
    const float dot = lanes_sum<G>(q.g * r);
#pragma unroll
    for (int i = 0; i < kEpl; ++i) d[i] *= -inv * dot;
    const float both = sum_duplicates<G>(q.id, q.g, tok, p.k);
    if (active) store8(out, e0, E, p.vec_out != 0, d);
    __syncwarp();                                      // the row is written before the selected experts' places are
    if (active && q.id >= 0) store1(out + q.id, r * (both - dot));
    __syncwarp();
  }
}

template <typename T, int kBy>
cudaError_t launch_route(int grid, const BatchRouteParams& p, cudaStream_t st) {
  if (p.E <= 4 * kEpl && p.groups <= 4) dx_batch_route_kernel<T, 4, kBy><<<grid, kThreads, 0, st>>>(p);
  else if (p.E <= 8 * kEpl && p.groups <= 8) dx_batch_route_kernel<T, 8, kBy><<<grid, kThreads, 0, st>>>(p);
  else if (p.E <= 16 * kEpl && p.groups <= 16) dx_batch_route_kernel<T, 16, kBy><<<grid, kThreads, 0, st>>>(p);
  else dx_batch_route_kernel<T, 32, kBy><<<grid, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}
template <typename T>
cudaError_t launch_route(int grid, const BatchRouteParams& p, cudaStream_t st) {
  // (the logits stand for the scores wherever only their order counts)
  const bool scores = p.bias != nullptr || (p.groups > 1 && p.group_score != DX_GROUP_MAX);
  if (!scores) return launch_route<T, kByLogits>(grid, p, st);
  return p.score_fn == DX_SCORE_SOFTMAX ? launch_route<T, kBySoftmax>(grid, p, st) : launch_route<T, kBySigmoid>(grid, p, st);
}
template <typename T>
cudaError_t launch_grad(int grid, const RouteGradParams& p, cudaStream_t st) {
  if (p.score_fn != DX_SCORE_SOFTMAX || p.norm) dx_route_grad_sparse_kernel<T><<<grid, kGradThreads, 0, st>>>(p);
  else if (p.E <= 8 * kEpl) dx_route_grad_dense_kernel<T, 8><<<grid, kGradThreads, 0, st>>>(p);
  else if (p.E <= 16 * kEpl) dx_route_grad_dense_kernel<T, 16><<<grid, kGradThreads, 0, st>>>(p);
  else dx_route_grad_dense_kernel<T, 32><<<grid, kGradThreads, 0, st>>>(p);
  return cudaGetLastError();
}
bool rows_aligned(const void* base, long long ld, int elem) {
  return reinterpret_cast<uintptr_t>(base) % 16 == 0 && ld * elem % 16 == 0;
}

}  // namespace

cudaError_t dx_launch_batch_route(dx_ctx* ctx, const dx_route_desc& d, const void* logits, int dtype, int N,
                                  long long ld, const float* bias, int32_t* topk_ids, float* topk_w, int32_t* offsets,
                                  int32_t* perm, cudaStream_t st, int* n_launches) {
  const int elem = dtype == DX_DTYPE_FP32 ? 4 : 2;
  BatchRouteParams p{};
  p.logits = logits;
  p.N = N; p.E = d.n_experts; p.k = d.top_k; p.ld = ld; p.bias = bias;
  p.score_fn = d.score_fn; p.norm = d.norm_topk; p.groups = d.n_groups; p.keep = d.topk_groups;
  if (p.keep == p.groups) p.groups = p.keep = 1;      // every group stays
  p.group_score = d.group_score;
  p.scale = d.routed_scale;
  p.vec = rows_aligned(logits, ld, elem) ? 1 : 0;
  p.topk_ids = topk_ids; p.topk_w = topk_w; p.offsets = offsets; p.perm = perm;
  p.counts = ctx->route_counts;
  p.dev_status = ctx->dev_status;
  // One CTA up to two turns of its warps (128 tokens of 64 experts: 8.1 us against 7.1 us for two launches, the second of
  // which costs the host 3 us; four turns: 10.9 against 7.1 us), else at most two per SM, each with whole turns.
  const int lanes = p.E <= 4 * kEpl && p.groups <= 4 ? 4 : p.E <= 8 * kEpl && p.groups <= 8 ? 8
                    : p.E <= 16 * kEpl && p.groups <= 16 ? 16 : 32;
  const int turn = kWarps * (32 / lanes);
  const int max_ctas = DX_ROUTE_CTAS_PER_SM * ctx->sm_count;
  p.per_cta = N <= 2 * turn ? N : (int)((((long long)N + max_ctas - 1) / max_ctas + turn - 1) / turn * turn);
  const int grid = (int)(((long long)N + p.per_cta - 1) / p.per_cta);
  cudaError_t e = dtype == DX_DTYPE_FP32 ? launch_route<float>(grid, p, st) : launch_route<__nv_bfloat16>(grid, p, st);
  *n_launches = 1;
  if (e == cudaSuccess && perm && grid > 1) {
    const unsigned int padded = (unsigned)((grid + kPermCluster - 1) / kPermCluster * kPermCluster);
    e = dx_launch_pdl((ctx->pdl_mask & DX_PDL_ROUTE) != 0, dx_batch_permute_kernel, dim3(padded), dim3(kThreads), 0, st, kPermCluster, p, grid,
                      p.E <= 32 ? 5 : p.E <= 64 ? 6 : p.E <= 128 ? 7 : 8);
    *n_launches = 2;
  }
  return e;
}

cudaError_t dx_launch_route_grad(dx_ctx* ctx, const dx_route_desc& d, const void* logits, int dtype, int N,
                                 long long ld, const int32_t* topk_ids, const float* d_topk_w, void* d_logits,
                                 long long ld_d, cudaStream_t st) {
  const int elem = dtype == DX_DTYPE_FP32 ? 4 : 2;
  RouteGradParams p{logits, N, d.n_experts, d.top_k, ld, topk_ids, d_topk_w, d.score_fn, d.norm_topk, d.routed_scale,
                    rows_aligned(logits, ld, elem) ? 1 : 0, rows_aligned(d_logits, ld_d, elem) ? 1 : 0, d_logits, ld_d,
                    ctx->dev_status};
  // four tokens per warp and turn, fewer where every expert's logit has a gradient and E takes more lanes
  const bool dense = d.score_fn == DX_SCORE_SOFTMAX && !d.norm_topk;
  const int turn = kGradWarps * (!dense || d.n_experts <= 8 * kEpl ? 4 : d.n_experts <= 16 * kEpl ? 2 : 1);
  long long grid = ((long long)N + turn - 1) / turn;
  const long long most = 8ll * ctx->sm_count;
  if (grid > most) grid = most;
  return dtype == DX_DTYPE_FP32 ? launch_grad<float>((int)grid, p, st) : launch_grad<__nv_bfloat16>((int)grid, p, st);
}
