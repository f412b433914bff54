// Device helpers of the kernels that go over rows of logits: 16-byte vectors of fp32 / bf16 values, the running
// (maximum, sum of exponentials) of a softmax, and the exchange between the CTAs of a cluster that share a row.
#pragma once

#include <cuda_bf16.h>
#include <float.h>
#include <stdint.h>

#include "dx_internal.cuh"

namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;

__device__ __forceinline__ float row_ex2(float x) {   // 2^x, results below 2^-126 become zero
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN on either side stays
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// Two fp32 values in one 64-bit register: Blackwell adds, multiplies and multiply-adds both in one instruction.
__device__ __forceinline__ unsigned long long f2_pack(float lo, float hi) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void f2_unpack(unsigned long long v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ unsigned long long f2_add(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long f2_mul(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long f2_fma(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// A 16-byte vector of row elements: kN of them, pair i of them as two fp32 values, their largest (NaN ignored unless
// all are NaN).
template <typename T>
struct RowVec;
template <>
struct RowVec<float> {
  static constexpr int kN = 4;
  static constexpr uint32_t kNegInfWord = 0xff800000u;
  static __device__ __forceinline__ unsigned long long pair(const uint4& v, int i) {
    return i == 0 ? f2_pack(__uint_as_float(v.x), __uint_as_float(v.y))
                  : f2_pack(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  static __device__ __forceinline__ float largest(const uint4& v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ float largest(const uint4* v, int n) {   // (n is known after inlining)
    float m = largest(v[0]);
#pragma unroll
    for (int u = 1; u < 4; ++u)
      if (u < n) m = fmaxf(m, largest(v[u]));
    return m;
  }
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ float round(float x) { return x; }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float element(const uint4& v, int i) {
    return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
  }
};
template <>
struct RowVec<__nv_bfloat16> {
  static constexpr int kN = 8;
  static constexpr uint32_t kNegInfWord = 0xff80ff80u;
  static __device__ __forceinline__ uint32_t word(const uint4& v, int i) {
    return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
  }
  static __device__ __forceinline__ unsigned long long pair(const uint4& v, int i) {
    const uint32_t w = word(v, i);
    return f2_pack(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ uint32_t largest2(const uint4& v) { return max2(max2(v.x, v.y), max2(v.z, v.w)); }
  static __device__ __forceinline__ float larger_half(uint32_t m) {
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
  static __device__ __forceinline__ float largest(const uint4& v) { return larger_half(largest2(v)); }
  static __device__ __forceinline__ float largest(const uint4* v, int n) {   // (n is known after inlining)
    uint32_t m = largest2(v[0]);
#pragma unroll
    for (int u = 1; u < 4; ++u)
      if (u < n) m = max2(m, largest2(v[u]));
    return larger_half(m);
  }
  static __device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ __nv_bfloat16 round(float x) { return __float2bfloat16_rn(x); }
  static __device__ __forceinline__ __nv_bfloat16 element(const uint4& v, int i) {
    return __ushort_as_bfloat16((unsigned short)(word(v, i >> 1) >> (16 * (i & 1))));
  }
  // one rounding of at most half a bf16 step, 2^-8 relative
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint4 r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.x) : "f"(f[1]), "f"(f[0]));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.y) : "f"(f[3]), "f"(f[2]));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.z) : "f"(f[5]), "f"(f[4]));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.w) : "f"(f[7]), "f"(f[6]));
    return r;
  }
};

// A row of V elements starting at any multiple of its element size: `head` elements in front of the first 16-byte
// boundary, `nvec` aligned vectors, `tail` elements behind them.  The CTAs of a cluster take consecutive runs of the
// vectors; the first one also takes the head, the last one the tail (one element per thread).
struct RowSplit {
  int head, tail;
  int nvec, v_lo, v_hi;
};
template <typename T>
__device__ __forceinline__ RowSplit row_split(const T* row, int V, int rank, int n_ranks) {
  RowSplit s;
  const int mis = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
  s.head = mis ? min(V, RowVec<T>::kN - mis) : 0;
  s.nvec = (V - s.head) / RowVec<T>::kN;
  s.tail = V - s.head - s.nvec * RowVec<T>::kN;
  const int shift = __ffs(n_ranks) - 1;   // (a power of two)
  s.v_lo = (int)(((long long)s.nvec * rank) >> shift);
  s.v_hi = (int)(((long long)s.nvec * (rank + 1)) >> shift);
  return s;
}

// (each logit is read once; L1 is left to what is read again)
__device__ __forceinline__ uint4 load_stream(const uint4* p) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p)
               : "memory");
  return r;
}
__device__ __forceinline__ uint4 load_shared(uint32_t addr) {
  uint4 r;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr) : "memory");
  return r;
}

__device__ __forceinline__ void store_shared(uint32_t addr, const uint4& v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// ---- clusters ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// address of this CTA's shared-memory word `p` in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank) {
  uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(p)), r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_store_f32(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ void cluster_store_u64(uint32_t addr, unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}

}  // namespace
