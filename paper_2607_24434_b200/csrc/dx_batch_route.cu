// Routing of whole batches: scores, selection with a balance bias and expert groups, gate weights, and the permutation
// of the token-expert pairs by expert; and the gradient of the gate weights with respect to the router logits.
//
//   score   r_e = softmax(z)_e or sigmoid(z_e);   selection value  v_e = r_e + b_e   (z_e itself where there is no bias: the
//   scores are monotone in the logits, and logits can be compared without any rounding)
//   groups  of E / G consecutive experts are ranked by their largest value, or by the sum of their two largest; the best
//   `keep` of them stay;  the k largest values among the experts left are selected, ties to the lower id
//   gate    w_j = scale * r_j  or  scale * r_j / sum_i r_i
//
// The selection is that of exact arithmetic.  It is made in 32 bits first: a lane holds eight consecutive experts, their
// values become unique integer keys (24 bits of the value's place in the token's range, then the reversed expert id),
// which a sorting network and k + 1 rounds of a maximum over the token's lanes put in order.  Where two neighbours of
// the result are closer than the arithmetic can tell apart (about one token in a thousand), the whole warp makes that
// token's selection again with 64-bit scores.
//
// Two launches for a large batch: selection with one histogram of experts per CTA, then the permutation, every CTA
// adding up the histograms in front of it (a stable counting sort without atomics on device memory; the order does not
// depend on timing).  A small batch is one CTA and one launch.
#include "dx_internal.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kEpl = 8;           // experts per lane
// How far the difference of two 32-bit selection values may be off, relative to the largest score + bias: expf is good
// to 2 steps of 2^-23, the row's sum and the difference in its exponent add as much again, the quotient and the
// addition of the bias half a step each; less than 8e-7 per value.
constexpr float kScoreError = 2e-6f;
constexpr float kKeyRange = 256.f;   // values this far below the token's largest share one key

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
__device__ __forceinline__ float lanes_min(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v = fminf(v, __shfl_xor_sync(0xffffffffu, v, o));
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
  if (G == 32) return __reduce_max_sync(0xffffffffu, v);
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

__device__ __forceinline__ bool finite_f(float x) { return fabsf(x) <= 3.402823466e38f; }
__device__ __forceinline__ float sigmoid_f(float z) { return 1.f / (1.f + expf(-z)); }

// (value, expert) in the order of selection: larger value first, then the lower expert; masked experts (value -inf)
// behind all others, excluded ones (expert -1) never
struct Pick {
  double v;
  int e;
};
__device__ __forceinline__ bool before(const Pick& a, const Pick& b) {
  if (a.e < 0 || b.e < 0) return b.e < 0 && a.e >= 0;
  return a.v > b.v || (a.v == b.v && a.e < b.e);
}

// The selection of one token in 64 bits by a whole warp (lane j < k + 1 ... receives the j-th id in `mine`).
// s_row: E doubles of the warp.
template <typename T>
__device__ __noinline__ int select_exact(const BatchRouteParams& p, const T* row, double* s_row) {
  const int lane = threadIdx.x & 31;
  double m = -INFINITY, s = 0.0;
  const bool scores = p.bias != nullptr || (p.groups > 1 && p.group_score != DX_GROUP_MAX);
  if (p.score_fn == DX_SCORE_SOFTMAX && scores) {
    for (int e = lane; e < p.E; e += 32) m = fmax(m, (double)to_f(row[e]));
    for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (m > -INFINITY)
      for (int e = lane; e < p.E; e += 32) s += exp((double)to_f(row[e]) - m);
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
  auto score = [&](int e) {   // -inf marks a masked expert
    const double z = (double)to_f(row[e]);
    if (!(z > -INFINITY)) return (double)-INFINITY;
    double r = z;
    if (scores) r = p.score_fn == DX_SCORE_SOFTMAX ? exp(z - m) / s : 1.0 / (1.0 + exp(-z));
    if (p.bias) r += (double)p.bias[e];
    return r == r ? r : (double)-INFINITY;
  };
  for (int e = lane; e < p.E; e += 32) s_row[e] = score(e);
  __syncwarp();
  unsigned int kept = 0xffffffffu;
  const int per = p.E / p.groups;
  if (p.groups > 1) {
    double a = -INFINITY, b = -INFINITY;
    if (lane < p.groups) {
      for (int i = 0; i < per; ++i) {
        const double v = s_row[lane * per + i];
        if (v > a) { b = a; a = v; }
        else if (v > b) b = v;
      }
      if (p.group_score != DX_GROUP_MAX && b > -INFINITY) a += b;
    }
    int r = 0;
    for (int g = 0; g < p.groups; ++g) {
      const double o = __shfl_sync(0xffffffffu, a, g);
      r += o > a || (o == a && g < lane);
    }
    kept = __ballot_sync(0xffffffffu, lane < p.groups && r < p.keep);
  }
  // without a bias the experts themselves are compared by their logits
  Pick last{INFINITY, -1};
  bool first = true;
  int mine = -1;
  for (int j = 0; j < p.k; ++j) {
    Pick best{0.0, -1};
    for (int e = lane; e < p.E; e += 32) {
      if (p.groups > 1 && !(kept >> (e / per) & 1u)) continue;
      double v = s_row[e];
      if (scores && !p.bias && v > -INFINITY) v = (double)to_f(row[e]);
      const Pick c{v, e};
      if ((first || before(last, c)) && before(c, best)) best = c;
    }
    for (int o = 16; o > 0; o >>= 1) {
      const Pick c{__shfl_xor_sync(0xffffffffu, best.v, o), __shfl_xor_sync(0xffffffffu, best.e, o)};
      if (before(c, best)) best = c;
    }
    last = best;
    first = false;
    if (lane == j) mine = best.e;
  }
  __syncwarp();
  return mine;
}

// Where the pairs of this CTA go: base[e] = first place of expert e's pairs of this CTA.  The pairs of the CTA's tokens
// are taken in runs of 32, a contiguous stretch of them per warp, so that equal experts keep the order of their pairs.
__device__ __forceinline__ void place_pairs(const int32_t* ids, long long p0, int n, int E, int (*s_hist)[DX_MAX_E],
                                            const int* s_base, int32_t* perm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int run = (n + kWarps * 32 - 1) / (kWarps * 32) * 32;
  const int lo = min(n, warp * run), hi = min(n, lo + run);
  for (int e = lane; e < E; e += 32) s_hist[warp][e] = 0;
  __syncwarp();
  for (int i = lo; i < hi; i += 32) {
    const int id = i + lane < hi ? ids[p0 + i + lane] : -1;
    const unsigned int same = __match_any_sync(0xffffffffu, id);
    if (id >= 0 && __ffs(same) - 1 == lane) s_hist[warp][id] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kThreads) {
    int at = s_base[e];
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const int c = s_hist[w][e];
      s_hist[w][e] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int i = lo; i < hi; i += 32) {
    const int id = i + lane < hi ? ids[p0 + i + lane] : -1;
    const unsigned int same = __match_any_sync(0xffffffffu, id);
    const int at = id >= 0 ? s_hist[warp][id] : 0;
    __syncwarp();
    if (id >= 0) {
      perm[at + __popc(same & ((1u << lane) - 1u))] = (int32_t)(p0 + i + lane);
      if (__ffs(same) - 1 == lane) s_hist[warp][id] = at + __popc(same);
    }
    __syncwarp();
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

template <typename T, int G>
__global__ void __launch_bounds__(kThreads) dx_batch_route_kernel(BatchRouteParams p) {
  constexpr int kTok = 32 / G;                       // tokens a warp works on side by side
  __shared__ int s_count[DX_MAX_E];
  __shared__ int s_hist[kWarps][DX_MAX_E];
  __shared__ int s_base[DX_MAX_E];
  __shared__ int s_scan[kWarps];
  __shared__ double s_exact[kWarps][DX_MAX_E];
  float* s_vals = reinterpret_cast<float*>(s_exact[threadIdx.x >> 5]);   // (the general group path stages values here)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % G, tok = lane / G;
  const int E = p.E, k = p.k, e0 = sub * kEpl;
  const int per = E / p.groups;
  // a group is a whole number of lanes, a power of two of them: its score comes out of a few exchanges
  const int gl = per / kEpl;
  const bool lane_groups = p.groups > 1 && per % kEpl == 0 && (gl & (gl - 1)) == 0;
  for (int e = threadIdx.x; e < E; e += kThreads) s_count[e] = 0;
  __syncthreads();

  float b[kEpl];
  float bmax = 0.f;
#pragma unroll
  for (int i = 0; i < kEpl; ++i) {
    b[i] = p.bias && e0 + i < E ? p.bias[e0 + i] : 0.f;
    bmax = fmaxf(bmax, fabsf(b[i]));
  }
  bmax = lanes_max<G>(bmax);
  int gid[kEpl];                                     // groups of this lane's experts (general path)
#pragma unroll
  for (int i = 0; i < kEpl; ++i) gid[i] = p.groups > 1 ? min(e0 + i, E - 1) / per : 0;

  const long long t_lo = (long long)blockIdx.x * p.per_cta;
  const long long t_hi = min((long long)p.N, t_lo + p.per_cta);
  for (long long t0 = t_lo + warp * kTok; t0 < t_hi; t0 += kWarps * kTok) {
    const bool active = t0 + tok < t_hi;
    const long long t = active ? t0 + tok : t_hi - 1;   // (lanes without a token repeat the last one and write nothing)
    const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
    float z[kEpl], v[kEpl];
    load8(row, e0, E, p.vec != 0, z);
    // ---- scores and selection values; masked experts have value -inf
    float m = -INFINITY, ssum = 0.f, rmax = 1.f;
    if (p.score_fn == DX_SCORE_SOFTMAX) {
#pragma unroll
      for (int i = 0; i < kEpl; ++i) m = fmaxf(m, z[i]);
      m = lanes_max<G>(m);
#pragma unroll
      for (int i = 0; i < kEpl; ++i) ssum += z[i] == -INFINITY ? 0.f : expf(z[i] - m);
      ssum = lanes_sum<G>(ssum);
    }
    const bool scores = p.bias != nullptr || (p.groups > 1 && p.group_score != DX_GROUP_MAX);
    float rs[kEpl];
#pragma unroll
    for (int i = 0; i < kEpl; ++i) {
      const bool masked = !(z[i] > -INFINITY);
      float r = z[i];
      if (scores) r = p.score_fn == DX_SCORE_SOFTMAX ? expf(z[i] - m) / ssum : sigmoid_f(z[i]);
      rs[i] = masked ? -INFINITY : r + b[i];
      v[i] = masked ? -INFINITY : p.bias ? rs[i] : z[i];
    }
    if (p.score_fn == DX_SCORE_SOFTMAX) rmax = 1.f / ssum;
    bool doubt = false;
    // ---- groups
    unsigned int kept = 0xffffffffu;
    if (p.groups > 1) {
      float g1 = -INFINITY, g2 = -INFINITY;            // two largest values of the group
      if (lane_groups) {
#pragma unroll
        for (int i = 0; i < kEpl; ++i) {
          g2 = fmaxf(g2, fminf(g1, rs[i]));
          g1 = fmaxf(g1, rs[i]);
        }
        for (int o = 1; o < gl; o <<= 1) {
          const float o1 = __shfl_xor_sync(0xffffffffu, g1, o), o2 = __shfl_xor_sync(0xffffffffu, g2, o);
          g2 = fmaxf(fmaxf(g2, o2), fminf(g1, o1));
          g1 = fmaxf(g1, o1);
        }
        // lane g of the token's lanes takes group g
        g1 = __shfl_sync(0xffffffffu, g1, tok * G + min(sub, p.groups - 1) * gl);
        g2 = __shfl_sync(0xffffffffu, g2, tok * G + min(sub, p.groups - 1) * gl);
      } else {
        float* stage = s_vals + tok * G * kEpl;
#pragma unroll
        for (int i = 0; i < kEpl; ++i) stage[e0 + i] = rs[i];
        __syncwarp();
        if (sub < p.groups) {
          int at = sub % per;                          // (start apart: the lanes read different banks)
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
      // rank of this lane's group; neighbours at the border too close to tell apart raise the doubt
      const float eps = scores ? 2.f * kScoreError * (rmax + bmax) : 0.f;
      int r = 0;
      bool close = false;
      for (int g = 0; g < p.groups; ++g) {
        const float o = __shfl_sync(0xffffffffu, gs, tok * G + g);
        r += o > gs || (o == gs && g < sub);
        close |= g != sub && fabsf(o - gs) <= eps && finite_f(o) && finite_f(gs);
      }
      const bool in = sub < p.groups;
      const unsigned int mask = (G == 32 ? 0xffffffffu : ((1u << G) - 1u)) << (tok * G);
      kept = (__ballot_sync(0xffffffffu, in && r < p.keep) & mask) >> (tok * G);
      const bool border = in && close && scores && p.keep < p.groups && (r == p.keep - 1 || r == p.keep);
      doubt = (__ballot_sync(0xffffffffu, border) & mask) != 0;
    }
    // ---- unique keys: 24 bits of the value within the token's range, then the reversed id
    float lo = INFINITY, hi = -INFINITY;
    const int e_id = e0;
#pragma unroll
    for (int i = 0; i < kEpl; ++i) {
      if (finite_f(v[i])) {
        lo = fminf(lo, v[i]);
        hi = fmaxf(hi, v[i]);
      }
    }
    hi = lanes_max<G>(hi);
    lo = fmaxf(lanes_min<G>(lo), hi - kKeyRange);
    const float span = hi - lo;
    const float quanta = span > 0.f ? 16777000.f / span : 0.f;
    doubt |= hi > lo && !finite_f(quanta);             // (a range too narrow for the factor: the keys say nothing)
    unsigned int key[kEpl];
#pragma unroll
    for (int i = 0; i < kEpl; ++i) {
      const int e = e_id + i;
      unsigned int q = 1;                              // masked
      if (v[i] > -INFINITY) q = v[i] == INFINITY ? 0xffffffu : 2u + (unsigned int)fminf(fmaxf((v[i] - lo) * quanta, 0.f), 16777000.f);
      if (p.groups > 1) {
        const int g = lane_groups ? sub / gl : gid[i];
        if (!(kept >> g & 1u)) q = 0;
      }
      key[i] = e < E ? (q << 8 | (unsigned int)(255 - e)) : 0u;
      if (q == 0) key[i] = 0;                          // excluded: never selected
    }
    // ---- the lane's keys in descending order (19 exchanges)
#define DX_EXCHANGE(a, c) { const unsigned int hi_ = max(key[a], key[c]), lo_ = min(key[a], key[c]); key[a] = hi_; key[c] = lo_; }
    DX_EXCHANGE(0, 1) DX_EXCHANGE(2, 3) DX_EXCHANGE(4, 5) DX_EXCHANGE(6, 7)
    DX_EXCHANGE(0, 2) DX_EXCHANGE(1, 3) DX_EXCHANGE(4, 6) DX_EXCHANGE(5, 7)
    DX_EXCHANGE(1, 2) DX_EXCHANGE(5, 6) DX_EXCHANGE(0, 4) DX_EXCHANGE(3, 7)
    DX_EXCHANGE(1, 5) DX_EXCHANGE(2, 6)
    DX_EXCHANGE(1, 4) DX_EXCHANGE(3, 6)
    DX_EXCHANGE(2, 4) DX_EXCHANGE(3, 5)
    DX_EXCHANGE(3, 4)
#undef DX_EXCHANGE
    // ---- k + 1 rounds: lane j of the token's lanes gets the j-th key (a token of four lanes keeps two apiece)
    unsigned int mine = 0, mine2 = 0, mine3 = 0;
    for (int j = 0; j <= k; ++j) {
      const unsigned int top = lanes_umax<G>(key[0]);
      const bool won = key[0] == top && top != 0;
#pragma unroll
      for (int i = 0; i < kEpl - 1; ++i) key[i] = won ? key[i + 1] : key[i];
      key[kEpl - 1] = won ? 0 : key[kEpl - 1];
      if (j % G == sub) {
        if (j < G) mine = top;
        else if (j < 2 * G) mine2 = top;
        else mine3 = top;
      }
    }
    // ---- neighbours too close for 32 bits (equal logits and biases are a true tie, in the right order already)
    const float slack = p.bias ? kScoreError * (rmax + bmax) * quanta : 0.f;
    const unsigned int near = 4u + (unsigned int)fminf(slack, 1.6e7f);
#pragma unroll
    for (int h = 0; h < (G == 4 ? 3 : G == 8 ? 2 : 1); ++h) {
      const unsigned int a = h == 0 ? mine : h == 1 ? mine2 : mine3;
      const unsigned int up = __shfl_sync(0xffffffffu, h == 0 ? mine : h == 1 ? mine2 : mine3, tok * G + (sub + 1) % G);
      const unsigned int wrap = __shfl_sync(0xffffffffu, h == 0 ? mine2 : h == 1 ? mine3 : 0u, tok * G);
      const unsigned int c = sub == G - 1 ? wrap : up;
      const int j = h * G + sub;                       // neighbours j and j + 1
      bool close = j < k && a != 0 && c != 0 && (a >> 8) >= 2u && (c >> 8) >= 2u && (a >> 8) - (c >> 8) <= near;
      if (close && j + 1 < k) {
        const int ea = 255 - (int)(a & 255u), ec = 255 - (int)(c & 255u);
        const float za = to_f(row[ea]), zc = to_f(row[ec]);
        if (za == zc && (!p.bias || p.bias[ea] == p.bias[ec])) close = false;
      }
      const unsigned int mask = (G == 32 ? 0xffffffffu : ((1u << G) - 1u)) << (tok * G);
      doubt |= (__ballot_sync(0xffffffffu, close) & mask) != 0;
    }
    int id0 = 255 - (int)(mine & 255u), id1 = 255 - (int)(mine2 & 255u);
    unsigned int redo = __ballot_sync(0xffffffffu, doubt);
    for (int q = 0; q < kTok; ++q) {
      if (!(redo >> (q * G) & 1u)) continue;           // (the same for the whole warp)
      const long long tq = min(t0 + q, t_hi - 1);
      const T* rq = reinterpret_cast<const T*>(p.logits) + (size_t)tq * (size_t)p.ld;
      const int got = select_exact(p, rq, s_exact[warp]);
      const int x0 = __shfl_sync(0xffffffffu, got, sub), x1 = __shfl_sync(0xffffffffu, got, (sub + G) % 32);
      if (tok == q) {
        id0 = x0;
        id1 = x1;
      }
    }
    // ---- gate weights of the selected experts
    const bool on0 = sub < k, on1 = G < DX_MAX_TOPK && sub + G < k;
    const float x0 = on0 ? to_f(row[id0]) : -INFINITY, x1 = on1 ? to_f(row[id1]) : -INFINITY;
    auto gate = [&](float x, float top) {   // e^{x - top}: renormalised softmax gates need nothing else of the row
      return x == -INFINITY ? 0.f : expf(x - top);
    };
    float w0, w1, sum = 1.f;
    if (p.norm) {
      const float top = lanes_max<G>(fmaxf(x0, x1));
      if (p.score_fn == DX_SCORE_SOFTMAX) {
        w0 = gate(x0, top);
        w1 = gate(x1, top);
      } else {
        // (sigmoid(x) is e^x to 32 bits where it is this small: the ratio survives the underflow)
        w0 = top < -64.f ? gate(x0, top) : x0 == -INFINITY ? 0.f : sigmoid_f(x0);
        w1 = top < -64.f ? gate(x1, top) : x1 == -INFINITY ? 0.f : sigmoid_f(x1);
      }
      sum = lanes_sum<G>(w0 + w1);
    } else if (p.score_fn == DX_SCORE_SOFTMAX) {
      w0 = gate(x0, m) / ssum;
      w1 = gate(x1, m) / ssum;
      if (m == -INFINITY) w0 = w1 = 0.f;
    } else {
      w0 = x0 == -INFINITY ? 0.f : sigmoid_f(x0);
      w1 = x1 == -INFINITY ? 0.f : sigmoid_f(x1);
    }
    const float f = sum > 0.f || sum != sum ? p.scale / sum : 0.f;
    if (active) {
      if (on0) {
        p.topk_ids[t * k + sub] = id0;
        p.topk_w[t * k + sub] = w0 * f;
        atomicAdd(&s_count[id0], 1);
      }
      if (on1) {
        p.topk_ids[t * k + sub + G] = id1;
        p.topk_w[t * k + sub + G] = w1 * f;
        atomicAdd(&s_count[id1], 1);
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
  place_pairs(p.topk_ids, 0, p.N * k, E, s_hist, s_base, p.perm);
}

// Clusters of kPermCluster CTAs share the sums over the histograms: CTA r of a cluster adds up every kPermCluster-th part
// of them, once over all CTAs (the experts' totals) and once over those in front of the cluster.
constexpr int kPermCluster = 8;
__global__ void __launch_bounds__(kThreads) dx_batch_permute_kernel(BatchRouteParams p, int n_ctas) {
  __shared__ int s_hist[kWarps][DX_MAX_E];
  __shared__ int s_base[DX_MAX_E];
  __shared__ int s_scan[kWarps];
  __shared__ int2 s_part[DX_MAX_E];
  const int E = p.E, e = threadIdx.x;
  const int rank = blockIdx.x % kPermCluster, first = blockIdx.x - rank;   // (clusters are runs of the grid)
  const int32_t* col = p.counts + e;
  int front = 0, total = 0;
  if (e < E) {
    const int lo = (int)((long long)n_ctas * rank / kPermCluster), hi = (int)((long long)n_ctas * (rank + 1) / kPermCluster);
#pragma unroll 8
    for (int b = lo; b < hi; ++b) {
      const int c = col[(size_t)b * E];
      total += c;
      front += b < first ? c : 0;
    }
    s_part[e] = make_int2(total, front);
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (e < E) {
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(&s_part[e]));
    total = front = 0;
#pragma unroll
    for (int r = 0; r < kPermCluster; ++r) {
      uint32_t a;
      int x, y;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(mine), "r"(r));
      asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "r"(a) : "memory");
      total += x;
      front += y;
    }
    for (int b = first; b < min((int)blockIdx.x, n_ctas); ++b) front += col[(size_t)b * E];
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  const int at = prefix_counts(total, s_scan);
  if (e < E) {
    s_base[e] = at + front;
    if (blockIdx.x == 0) p.offsets[e] = at;
  }
  if (blockIdx.x == 0 && e == 0) p.offsets[E] = p.N * p.k;
  __syncthreads();
  const long long t_lo = (long long)blockIdx.x * p.per_cta;
  const long long t_hi = min((long long)p.N, t_lo + p.per_cta);
  if (t_lo < t_hi) place_pairs(p.topk_ids, t_lo * p.k, (int)(t_hi - t_lo) * p.k, E, s_hist, s_base, p.perm);
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- backward ---------------------------------------------------------------------------------------------------------
// With S = sum_i r_i over the selected and g the gradient of the gates,
//   dL/dr_j = scale * g_j   or   scale * (g_j - sum_i g_i r_i / S) / S,
// sigmoid: dz_e = dL/dr_e r_e (1 - r_e);  softmax: dz_e = r_e (dL/dr_e - sum_j dL/dr_j r_j), dL/dr zero for experts that
// were not selected.  For renormalised gates that last sum is zero, so only softmax gates that are not renormalised
// have a gradient outside the selection, and only they need the whole row of logits.
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

template <typename T, int G>
__global__ void __launch_bounds__(kThreads) dx_route_grad_kernel(RouteGradParams p) {
  constexpr int kTok = 32 / G;
  const int lane = threadIdx.x & 31, sub = lane % G, tok = lane / G;
  const int E = p.E, k = p.k, e0 = sub * kEpl;
  const long long warps = (long long)gridDim.x * kWarps;
  for (long long t0 = ((long long)blockIdx.x * kWarps + (threadIdx.x >> 5)) * kTok; t0 < p.N; t0 += warps * kTok) {
    const bool active = t0 + tok < p.N;
    const long long t = active ? t0 + tok : p.N - 1;
    const T* row = reinterpret_cast<const T*>(p.logits) + (size_t)t * (size_t)p.ld;
    T* out = reinterpret_cast<T*>(p.dlogits) + (size_t)t * (size_t)p.ld_d;
    // the pairs of the token: lane j of its lanes takes pair j (a token of four lanes two apiece)
    int id[2];
    float g[2], x[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int j = sub + h * G;
      const bool on = j < k && (h == 0 || G < DX_MAX_TOPK);
      id[h] = on ? p.ids[t * k + j] : -1;
      g[h] = on ? p.dw[t * k + j] * p.scale : 0.f;
      if (on && (id[h] < 0 || id[h] >= E)) {
        *p.dev_status = DX_DEV_BAD_EXPERT_ID;
        id[h] = -1;
        g[h] = 0.f;
      }
      x[h] = id[h] >= 0 ? to_f(row[id[h]]) : -INFINITY;
    }
    const bool dense = p.score_fn == DX_SCORE_SOFTMAX && !p.norm;
    float d[kEpl];
    float r[2], slope[2] = {1.f, 1.f};                 // scores of the pairs; sigmoid: 1 - r
    float dot = 0.f;
    if (dense) {
      float m = -INFINITY, s = 0.f;
      load8(row, e0, E, p.vec_in != 0, d);
#pragma unroll
      for (int i = 0; i < kEpl; ++i) m = fmaxf(m, d[i]);
      m = lanes_max<G>(m);
#pragma unroll
      for (int i = 0; i < kEpl; ++i) {
        d[i] = d[i] == -INFINITY ? 0.f : expf(d[i] - m);
        s += d[i];
      }
      s = lanes_sum<G>(s);
      const float inv = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
      for (int h = 0; h < 2; ++h) r[h] = x[h] == -INFINITY ? 0.f : expf(x[h] - m) * inv;
      dot = lanes_sum<G>(g[0] * r[0] + g[1] * r[1]);
#pragma unroll
      for (int i = 0; i < kEpl; ++i) d[i] *= -inv * dot;
    } else {
      const float top = lanes_max<G>(fmaxf(x[0], x[1]));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // renormalised gates: a common factor of the scores cancels (e^{x - top} for softmax; sigmoid(x) is e^x where
        // it is small)
        const bool ratio = p.score_fn == DX_SCORE_SOFTMAX || (p.norm && top < -64.f);
        r[h] = x[h] == -INFINITY ? 0.f : ratio ? expf(x[h] - top) : sigmoid_f(x[h]);
        if (p.score_fn != DX_SCORE_SOFTMAX) slope[h] = sigmoid_f(-x[h]);
      }
      if (p.norm) {
        const float S = lanes_sum<G>(r[0] + r[1]);
        const float mean = lanes_sum<G>(g[0] * r[0] + g[1] * r[1]) / S;
#pragma unroll
        for (int h = 0; h < 2; ++h) g[h] = S == 0.f || id[h] < 0 ? 0.f : (g[h] - mean) / S;
      }
#pragma unroll
      for (int i = 0; i < kEpl; ++i) d[i] = 0.f;
    }
    // an expert listed twice gets the sum of its pairs' gradients
    float both[2] = {0.f, 0.f};
    for (int j = 0; j < k; ++j) {
      const int src = tok * G + j % G;
      const int oi = __shfl_sync(0xffffffffu, j < G ? id[0] : id[1], src);
      const float og = __shfl_sync(0xffffffffu, j < G ? g[0] : g[1], src);
#pragma unroll
      for (int h = 0; h < 2; ++h) both[h] += oi == id[h] ? og : 0.f;
    }
    if (active) store8(out, e0, E, p.vec_out != 0, d);
    __syncwarp();                                      // the row is written before the selected experts' places are
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (active && id[h] >= 0)
        store1(out + id[h], r[h] * (both[h] - dot) * slope[h]);
  }
}

template <typename T>
cudaError_t launch_route(int grid, const BatchRouteParams& p, cudaStream_t st) {
  if (p.E <= 4 * kEpl && p.groups <= 4) dx_batch_route_kernel<T, 4><<<grid, kThreads, 0, st>>>(p);
  else if (p.E <= 8 * kEpl && p.groups <= 8) dx_batch_route_kernel<T, 8><<<grid, kThreads, 0, st>>>(p);
  else if (p.E <= 16 * kEpl && p.groups <= 16) dx_batch_route_kernel<T, 16><<<grid, kThreads, 0, st>>>(p);
  else dx_batch_route_kernel<T, 32><<<grid, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}
template <typename T>
cudaError_t launch_grad(int grid, const RouteGradParams& p, cudaStream_t st) {
  if (p.E <= 4 * kEpl) dx_route_grad_kernel<T, 4><<<grid, kThreads, 0, st>>>(p);
  else if (p.E <= 8 * kEpl) dx_route_grad_kernel<T, 8><<<grid, kThreads, 0, st>>>(p);
  else if (p.E <= 16 * kEpl) dx_route_grad_kernel<T, 16><<<grid, kThreads, 0, st>>>(p);
  else dx_route_grad_kernel<T, 32><<<grid, kThreads, 0, st>>>(p);
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
  // one CTA up to 64 tokens (a second launch would cost more than the work), else at most two per SM
  const int max_ctas = 2 * ctx->sm_count;
  int grid = N <= 64 ? 1 : (N + 31) / 32;
  if (grid > max_ctas) grid = max_ctas;
  p.per_cta = (N + grid - 1) / grid;
  grid = (N + p.per_cta - 1) / p.per_cta;
  cudaError_t e = dtype == DX_DTYPE_FP32 ? launch_route<float>(grid, p, st) : launch_route<__nv_bfloat16>(grid, p, st);
  *n_launches = 1;
  if (e == cudaSuccess && perm && grid > 1) {
    const unsigned int padded = (unsigned)((grid + kPermCluster - 1) / kPermCluster * kPermCluster);
    e = dx_launch_pdl(false, dx_batch_permute_kernel, dim3(padded), dim3(kThreads), 0, st, kPermCluster, p, grid);
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
  long long grid = ((long long)N + 31) / 32;
  const long long most = 8ll * ctx->sm_count;
  if (grid > most) grid = most;
  return dtype == DX_DTYPE_FP32 ? launch_grad<float>((int)grid, p, st) : launch_grad<__nv_bfloat16>((int)grid, p, st);
}
