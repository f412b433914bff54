// The experts of Eq. 4 for whole batches of tokens: products of rows, sorted by expert, with their experts' matrices
// (moe_grouped_mm), SwiGLU on top of them (moe_grouped_swiglu), the gradients of both (moe_grouped_swiglu_backward,
// moe_grouped_mm_dw).  One persistent tcgen05 kernel (dx_mm.cuh) with different operands and different ways out.
//
// In all of them the LANES of a tile are the contiguous dimension of the output and its COLUMNS the output's rows: weights
// are the fixed 128 lanes of a CTA, and the ragged number of an expert's rows is the width of the products, which
// tcgen05.mma takes in steps of 16 -- a group of 5 rows costs 16 columns, not 128.
//
// Bounds and measurements, 64 experts of which a token takes six, H = 2048, I = 1408, calls one after the other.  One token:
// the weights' bytes (34.6 MB, 5.4 us at the copy rate) fetched by 96 CTAs of 148 SMs behind a chain of launch, offsets and
// first stage: 12.2 us; SwiGLU (69 MB, 132 CTAs) 16.5.  700 tokens, SwiGLU gradient: 370 MB of weights, 98 us with the gates'
// sums.  16384 tokens: the products (669 us at the burst rate, 813 at the sustained one) under the power cap, W^T x 940 to 1015
// us, SwiGLU that keeps its products 993 to 1060.  Weight gradients of many rows: 1.5 GB of fp32 results, gathered rows and
// operands through the SMs' path to L2, which is 74 % busy, the tensor pipe 45 % (8192 tokens 619 to 676 us, 335 by the
// products alone); of few rows the results (64 rows per group 4.9 TB/s in fp32, 4.7 in bf16).
#include <limits.h>

#include "dx_mm.cuh"

namespace {

// ---- out of tensor memory ------------------------------------------------------------------------------------------
// A warp turns 32 lanes x 32 (16) columns around in shared memory: fragments as the tensor memory gives them (mm_ld_frag),
// rounded and stored as transposed 8 x 8 matrices -- a column's lanes next to each other -- in the swizzle of a tensor map, which
// takes them from there (what the map cannot cut off -- the rows behind a group's last, rows scattered by index -- goes out in
// 16-byte pieces).  Some 40 instructions for 1024 elements; exchanged by shuffles they took over 200, and the storing warps, not
// the products, were what a tile waited for.

// bf16: 64 bytes per column, pieces of 16 bytes in an order that keeps the eight columns of a matrix in different banks
__device__ __forceinline__ uint32_t piece64(int column, int piece) {
  return (uint32_t)(column * 64 + ((piece ^ ((column >> 1) & 3)) << 4));
}
// four pieces of lanes, packed pairs of columns: matrix j = piece j, eight columns from 8 n
__device__ __forceinline__ void stage64(uint32_t at, int lane, int n, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  stmatrix_t(at + piece64(8 * n + (lane & 7), lane >> 3), a, b, c, d);
}
template <int COLS>
__device__ __forceinline__ void stage_bf16(uint32_t at, int lane, const Fragments<COLS>& x) {
#pragma unroll
  for (int n = 0; n < COLS / 8; ++n)
    stage64(at, lane, n, bf16_pair(x.v[0][4 * n], x.v[0][4 * n + 1]), bf16_pair(x.v[0][4 * n + 2], x.v[0][4 * n + 3]),
            bf16_pair(x.v[1][4 * n], x.v[1][4 * n + 1]), bf16_pair(x.v[1][4 * n + 2], x.v[1][4 * n + 3]));
}
// fp32: 128 bytes per column, pieces of 16 bytes in an order that keeps eight columns in different banks
__device__ __forceinline__ uint32_t piece128(int column, int piece) {
  return (uint32_t)(column * 128 + ((piece ^ (column & 7)) << 4));
}
template <int COLS>
__device__ __forceinline__ void stage_fp32(uint32_t at, int lane, const Fragments<COLS>& x) {
#pragma unroll
  for (int odd = 0; odd < 2; ++odd) {
    // column 8 n + r, lanes 16 h + 8 q + lane / 4: piece 4 h + 2 q + lane / 16, of which only the last part differs by lane
    const int r = 2 * (lane & 3) + odd;
    const uint32_t mine = at + piece128(r, lane >> 4) + ((lane >> 2) & 3) * 4;
#pragma unroll
    for (int n = 0; n < COLS / 8; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 2; ++q)
          sts4((mine ^ (uint32_t)((4 * h + 2 * q) << 4)) + (uint32_t)(n * 1024), x.v[h][4 * n + 2 * q + odd]);
  }
}

// sorted row of a chunk's column `c0 + lane` (-1: none)
__device__ __forceinline__ int sorted_row(const MmTile& t, int c0, int lane) {
  return c0 + lane < t.ncols ? t.n0 + c0 + lane : -1;
}
template <int COLS>
struct FragmentEpilogue {
  // Warps that gather: as many as the ring has stages, six, where 96 registers do (20 warps; of 98304 gathered rows SwiGLU that
  // keeps its products 922 us with four of them, 897 with six; of 49152 the weight gradient in fp32 591 and 567, in bf16 477 and
  // 454, W x 451 and 435: in turns, in bursts of 80 ms), four where 128 are needed.
  static constexpr int kCols = COLS, kRound = 1, kGathering = 4;
  static constexpr bool kBefore = true;
  using Values = Fragments<COLS>;
  const MmParams& p;
  const MmMaps& maps;
  const int lane;
  const uint32_t at;       // the warp's staging
  __device__ FragmentEpilogue(const MmParams& p_, const MmMaps& maps_, int lane_, int, uint32_t at_, MmFetch)
      : p(p_), maps(maps_), lane(lane_), at(at_) {}
  // the boxes that the staging went out in have been read
  __device__ __forceinline__ void writable() {
    if (lane == 0) tma_store_read();
    __syncwarp();
  }
  // the staging is what the tensor map's copies are to see
  __device__ __forceinline__ void written() {
    proxy_fence();
    __syncwarp();
  }
  __device__ __forceinline__ void finish() {
    if (lane == 0) tma_store_done();
  }
  __device__ __forceinline__ void load(uint32_t taddr, Values& x) { mm_ld_frag(taddr, x); }
  __device__ __forceinline__ void arrived(Values& x) { mm_ld_wait(x.v[0], x.v[1]); }
  __device__ __forceinline__ void zero(Values& x) {
#pragma unroll
    for (int i = 0; i < COLS / 2; ++i) x.v[0][i] = x.v[1][i] = 0.0f;
  }
  __device__ __forceinline__ void begin(const MmTile&, int, int, const MmTile&, bool) {}
  __device__ __forceinline__ void end(const MmTile&) {}
};

// Staged columns (bf16) to rows `mine` (of lane = column) of a matrix; m: first of the warp's 32 elements in a row.
// (First all reads, then all writes: a read and the write of what it brought would each wait for the one in front.)
template <int COLS>
__device__ __forceinline__ void flush_bf16(const MmParams& p, int lane, uint32_t at, int mine, int m, __nv_bfloat16* out,
                                           int64_t ld) {
  const int piece = lane & 3, x = m + 8 * piece;
  uint4 u[COLS / 8];
  int row[COLS / 8];
#pragma unroll
  for (int i = 0; i < COLS / 8; ++i) u[i] = lds16(at + piece64(8 * i + (lane >> 2), piece));
#pragma unroll
  for (int i = 0; i < COLS / 8; ++i) row[i] = __shfl_sync(0xffffffffu, mine, 8 * i + (lane >> 2));
#pragma unroll
  for (int i = 0; i < COLS / 8; ++i)
    if (row[i] >= 0 && x < p.lanes) *reinterpret_cast<uint4*>(out + (int64_t)row[i] * ld + x) = u[i];
}
// fp32 columns (plus what is to be added) in pieces
template <class T, bool ADD, int COLS>
__device__ __forceinline__ void flush_fp32(const MmParams& p, int lane, uint32_t at, int mine, int m, T* out, int64_t ld) {
  if constexpr (sizeof(T) == 4) {
    const int x = m + 4 * (lane & 7);
    uint4 u[COLS / 4];
    float4 a[COLS / 4];
    int row[COLS / 4];
#pragma unroll
    for (int i = 0; i < COLS / 4; ++i) row[i] = __shfl_sync(0xffffffffu, mine, 4 * i + (lane >> 3));
#pragma unroll
    for (int i = 0; i < COLS / 4; ++i) {
      a[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (ADD && row[i] >= 0 && x < p.lanes) a[i] = *reinterpret_cast<const float4*>(p.addend + (int64_t)row[i] * p.lanes + x);
    }
#pragma unroll
    for (int i = 0; i < COLS / 4; ++i) u[i] = lds16(at + piece128(4 * i + (lane >> 3), lane & 7));
#pragma unroll
    for (int i = 0; i < COLS / 4; ++i)
      if (row[i] >= 0 && x < p.lanes)
        *reinterpret_cast<float4*>(out + (int64_t)row[i] * ld + x) =
            make_float4(__uint_as_float(u[i].x) + a[i].x, __uint_as_float(u[i].y) + a[i].y, __uint_as_float(u[i].z) + a[i].z,
                        __uint_as_float(u[i].w) + a[i].w);
  } else {      // (summed in fp32, then rounded)
    const int x = m + 8 * (lane & 3);
#pragma unroll
    for (int i = 0; i < COLS / 8; ++i) {
      const int column = 8 * i + (lane >> 2), row = __shfl_sync(0xffffffffu, mine, column);
      const uint4 u = lds16(at + piece128(column, 2 * (lane & 3))), w = lds16(at + piece128(column, 2 * (lane & 3) + 1));
      if (row >= 0 && x < p.lanes) {
        const float4* a = reinterpret_cast<const float4*>(p.addend + (int64_t)row * p.lanes + x);
        const float4 a0 = a[0], a1 = a[1];
        *reinterpret_cast<uint4*>(out + (int64_t)row * ld + x) =
            make_uint4(bf16_pair(__uint_as_float(u.x) + a0.x, __uint_as_float(u.y) + a0.y),
                       bf16_pair(__uint_as_float(u.z) + a0.z, __uint_as_float(u.w) + a0.w),
                       bf16_pair(__uint_as_float(w.x) + a1.x, __uint_as_float(w.y) + a1.y),
                       bf16_pair(__uint_as_float(w.z) + a1.z, __uint_as_float(w.w) + a1.w));
      }
    }
  }
}
template <class T, bool ADD>
constexpr int store_cols() { return sizeof(T) == 2 && !ADD ? 32 : 16; }
constexpr int kStoreStaging = 2048;      // 32 columns of 64 bytes, 16 of 128

// out[row of the column][lane] = D (+ addend), rounded once.  Whole chunks whose rows follow one another go out as a box.
template <class T, bool ADD>
struct StoreRows : FragmentEpilogue<store_cols<T, ADD>()> {
  using Base = FragmentEpilogue<store_cols<T, ADD>()>;
  static constexpr int kStaging = kStoreStaging, kGathering = 6;
  using Base::Base;
  int next;      // where column `lane` of the next chunk goes (looked up a chunk ahead)
  __device__ __forceinline__ void look_up(const MmTile& t, int c0) {
    const int row = this->lane < Base::kCols ? sorted_row(t, c0, this->lane) : -1;
    const bool look = row >= 0 && this->p.scatter && DX_BOUNDS(row < this->p.n_rows, this->p.dev_status);
    next = look ? __ldg(this->p.scatter + row) : row;
  }
  __device__ __forceinline__ void begin(const MmTile& t, int, int c0, const MmTile&, bool) { look_up(t, c0); }
  template <class Taken>
  __device__ __forceinline__ void chunk(const MmTile& t, int lane0, int c0, const typename Base::Values& x, Taken) {
    const MmParams& p = this->p;
    int mine = next;
    if (p.scatter && this->lane < Base::kCols && sorted_row(t, c0, this->lane) >= 0 && (mine < 0 || mine >= p.out_rows)) {
      atomicExch(p.dev_status, (int32_t)DX_DEV_BAD_ROW);
      mine = -1;
    }
    if (!DX_BOUNDS(mine < this->p.out_rows, p.dev_status)) mine = -1;
    look_up(t, c0 + 2 * Base::kCols);
    this->writable();
    if constexpr (sizeof(T) == 2 && !ADD) stage_bf16(this->at, this->lane, x);
    else stage_fp32(this->at, this->lane, x);
    if (!ADD && !p.scatter && c0 + Base::kCols <= t.ncols) {
      this->written();
      if (this->lane == 0) {
        tma_store2(&this->maps.out[0], lane0, t.n0 + c0, this->at);
        tma_store_commit();
      }
    } else {
      __syncwarp();
      if constexpr (sizeof(T) == 2 && !ADD)
        flush_bf16<Base::kCols>(p, this->lane, this->at, mine, lane0, reinterpret_cast<T*>(p.out), p.ld);
      else
        flush_fp32<T, ADD, Base::kCols>(p, this->lane, this->at, mine, lane0, reinterpret_cast<T*>(p.out), p.ld);
      __syncwarp();
    }
  }
};

// out of group e: [columns][lanes], element (n, m) = D.  Every chunk is a box: the matrix ends where its columns do.
template <class T, int GATHERING>
struct StoreOuter : FragmentEpilogue<store_cols<T, false>()> {
  using Base = FragmentEpilogue<store_cols<T, false>()>;
  static constexpr int kStaging = kStoreStaging, kGathering = GATHERING;
  using Base::Base;
  template <class Taken>
  __device__ __forceinline__ void chunk(const MmTile& t, int lane0, int c0, const typename Base::Values& x, Taken) {
    this->writable();
    if constexpr (sizeof(T) == 2) stage_bf16(this->at, this->lane, x);
    else stage_fp32(this->at, this->lane, x);
    this->written();
    if (this->lane == 0) {
      tma_store3(&this->maps.out[0], lane0, t.n0 + c0, t.e, this->at);
      tma_store_commit();
    }
  }
};

// act = silu(gate) * up from the fp32 products; SAVE: the products themselves, rounded once, for the backward pass.
// Of 16 lanes the first eight are gate rows, the others the same eight up rows: a thread holds both of an element.
// 16 elements of a row per warp: 32 bytes per column, the halves in turns so that eight columns meet different banks.
template <bool SAVE>
struct StoreSwiglu : FragmentEpilogue<32> {
  static constexpr int kArea = 32 * 32, kStaging = (SAVE ? 3 : 1) * kArea, kGathering = 6;
  using FragmentEpilogue<32>::FragmentEpilogue;
  static __device__ __forceinline__ uint32_t half32(int column, int h) {
    return (uint32_t)(column * 32 + ((h ^ ((column >> 2) & 1)) << 4));
  }
  // matrices: (eight elements h, eight columns n)
  __device__ __forceinline__ void stage(uint32_t to, const uint32_t (&a)[2][4]) {
#pragma unroll
    for (int n = 0; n < 4; n += 2)
      stmatrix_t(to + half32(8 * (n + (lane >> 4)) + (lane & 7), (lane >> 3) & 1), a[0][n], a[1][n], a[0][n + 1], a[1][n + 1]);
  }
  __device__ __forceinline__ void pieces(uint32_t from, const MmTile& t, int c0, int i, __nv_bfloat16* out, int64_t ld) {
    out += (int64_t)(t.n0 + c0 + (lane >> 1)) * ld + i;
    uint4 u[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) u[k] = lds16(from + half32(16 * k + (lane >> 1), lane & 1));
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (16 * k + (lane >> 1) < t.ncols - c0 && i < (p.lanes >> 1) &&
          DX_BOUNDS(t.n0 + c0 + 16 * k + (lane >> 1) < p.n_rows, p.dev_status))
        *reinterpret_cast<uint4*>(out + (int64_t)(16 * k) * ld) = u[k];
  }
  template <class Taken>
  __device__ __forceinline__ void chunk(const MmTile& t, int lane0, int c0, const Values& x, Taken) {
    const float(&v)[2][16] = x.v;
    const int n_inter = p.lanes >> 1, i0 = lane0 >> 1;      // the warp's 16 elements
    uint32_t a[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < 4; ++n)
        a[h][n] = bf16_pair(v[h][4 * n] * sigmoid(v[h][4 * n]) * v[h][4 * n + 2],
                            v[h][4 * n + 1] * sigmoid(v[h][4 * n + 1]) * v[h][4 * n + 3]);
    writable();
    stage(at, a);
    if constexpr (SAVE) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int n = 0; n < 4; ++n) a[h][n] = bf16_pair(v[h][4 * n + 2 * g], v[h][4 * n + 2 * g + 1]);
        stage(at + (1 + g) * kArea, a);
      }
    }
    if (c0 + 32 <= t.ncols) {
      written();
      if (lane == 0) {
        tma_store2(&maps.out[0], i0, t.n0 + c0, at);
        if constexpr (SAVE) {
          tma_store2(&maps.out[1], i0, t.n0 + c0, at + kArea);
          tma_store2(&maps.out[2], i0, t.n0 + c0, at + 2 * kArea);
        }
        tma_store_commit();
      }
    } else {
      __syncwarp();
      const int i = i0 + 8 * (lane & 1);
      pieces(at, t, c0, i, reinterpret_cast<__nv_bfloat16*>(p.out), p.ld);
      if constexpr (SAVE) {
        __nv_bfloat16* save = reinterpret_cast<__nv_bfloat16*>(p.save);
        pieces(at + kArea, t, c0, i, save, p.ld_save);
        pieces(at + 2 * kArea, t, c0, i, save + n_inter, p.ld_save);
      }
      __syncwarp();
    }
  }
};

// D = W_down^T dy = the gradient of an unweighted act.  With q the row's pair, w its weight, s = sigmoid(gate):
//   d gate = w D up s (1 + gate (1 - s)),  d up = w D gate s,  act_w = w gate s up,
//   share of d w = sum over lanes of D gate s up.
// The rows of a pair of weight 0 get zeros, whatever they hold.  gate and up come as boxes, a chunk ahead; their place in the
// staging takes the gradients, which go out as boxes.  (In pieces through registers, every element crossed the load/store path
// six times: 458 us, 49152 rows x 2048 x 1408, where boxes took 423 in the same run; 396 to 421 now.)  Nothing is at its limit
// there -- an instruction in 38 % of the cycles, tensor pipe 47 %, DRAM 50 %, path to L2 40 %: what bounds it is the chain of
// each chunk -- its products' way out of tensor memory, exponential and reciprocal, stores, fence, box -- with two storing
// warps per scheduler and no registers to have two chunks under way.
struct StoreSwigluGrad : FragmentEpilogue<16> {
  static constexpr bool kBefore = false;      // (no registers for two chunks: this one is waited for where it is needed)
  // of a column 64 bytes of gate, then 64 of up; behind the sixteen columns act_w; two chunks; the weights of 128 columns
  static constexpr int kArea = 16 * 64, kBuffer = 3 * kArea, kStaging = 2 * kBuffer + 512;
  static __device__ __forceinline__ uint32_t piece2(int column, int up, int piece) {
    return (uint32_t)(column * 128 + up * 64 + ((piece ^ (column & 3)) << 4));
  }
  const int share;
  const MmFetch own;
  uint32_t turn = 0;         // chunks so far
  bool asked = false;        // the next chunk's gate and up are on their way
  bool gone = false;         // a chunk's did not come in time: nothing more is asked for
  MmTile next;
  bool more = false, first = true;
  int q[4];
  float w4[4];
  __device__ StoreSwigluGrad(const MmParams& p_, const MmMaps& maps_, int lane_, int share_, uint32_t at_, MmFetch own_)
      : FragmentEpilogue<16>(p_, maps_, lane_, share_, at_, own_), share(share_), own(own_) {}
  // gate and up of chunk number `n`, which is (tile, c0); its buffer has been read
  __device__ __forceinline__ void fetch(uint32_t n, const MmTile& t, int lane0, int c0) {
    if (lane == 0) {
      const uint32_t bar = own.bar + (n & 1u) * 8u, to = at + (n & 1u) * kBuffer;
      mbar_arrive_expect_tx(bar, 2 * kArea);
      tma3<1>(to, &maps.in, lane0, 0, t.n0 + c0, bar);
    }
  }
  // whether any chunk of a tile is the warp's
  __device__ __forceinline__ bool chunks(const MmTile& t, int lane0, int c0) const { return lane0 < p.lanes && c0 < t.ncols; }
  // The weights of the warp's share of a tile's columns, all at once.  An index and the weight behind it are two trips to L2:
  // they are asked for while the tile in front is still being stored.
  __device__ __forceinline__ void ask_pairs(const MmTile& t) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {        // 16 columns of every 32
      const int r = sorted_row(t, 32 * (2 * j + (lane >> 4)) + 16 * share, lane & 15);
      q[j] = r < 0 || !DX_BOUNDS(r < p.n_rows, p.dev_status) ? INT_MIN : p.b_index ? __ldg(p.b_index + r) : r;
    }
  }
  __device__ __forceinline__ void ask_weights() {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool in = q[j] >= 0 && q[j] < p.n_pairs;
      w4[j] = !in ? 0.0f : p.pair_w ? __ldg(p.pair_w + q[j]) : 1.0f;
      if (!in && q[j] != INT_MIN) atomicExch(p.dev_status, (int32_t)DX_DEV_BAD_ROW);
    }
  }
  __device__ __forceinline__ void begin(const MmTile& t, int lane0, int c0, const MmTile& next_, bool more_) {
    if (first) {
      ask_pairs(t);
      ask_weights();
      first = false;
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) sts4(at + 2 * kBuffer + (uint32_t)(32 * j + lane) * 4, w4[j]);
    __syncwarp();
    next = next_;
    more = more_;
    if (more) ask_pairs(next);
    if (!chunks(t, lane0, c0) && more) ask_weights();        // (the last chunk does it otherwise)
  }
  __device__ __forceinline__ void finish() {
    if (lane == 0) {               // (the loop over the tiles ended early: no box may still be landing)
      const uint32_t end = turn + (gone ? 1u : 0u) + (asked ? 1u : 0u);
      for (uint32_t n = turn; n < end; ++n)
        for (uint32_t spin = 0; spin < kDrainPolls; ++spin)
          if (mbar_try_wait(own.bar + (n & 1u) * 8u, (n >> 1) & 1u)) break;
    }
    FragmentEpilogue<16>::finish();
  }
  // the chunk behind (t, c0): into the buffer that the chunk in front of it went out from
  __device__ __forceinline__ void ask_next(const MmTile& t, int lane0, int c0) {
    const bool here = c0 + 2 * kCols < t.ncols;
    if (!here && more) ask_weights();
    const int next0 = next.m0 + lane0 - t.m0;
    asked = here || (more && chunks(next, next0, kCols * share));
    if (!asked) return;
    if (lane == 0) tma_store_read();
    if (here) fetch(turn + 1, t, lane0, c0 + 2 * kCols);
    else fetch(turn + 1, next, next0, kCols * share);
  }
  template <class Taken>
  __device__ __forceinline__ void chunk(const MmTile& t, int lane0, int c0, Values& x, Taken taken) {
    if (gone) {
      arrived(x);
      taken();
      return;
    }
    const uint32_t buf = at + (turn & 1u) * kBuffer;
    if (!asked) {
      if (lane == 0) tma_store_read();
      fetch(turn, t, lane0, c0);
    }
    ask_next(t, lane0, c0);
    // (a wait that runs out raises the abort flag, which ends the loop over the tiles.  No barrier is armed again while its box
    // may still be landing, so this warp asks for none from here on.)
    if (!mm_store_wait(own.bar + (turn & 1u) * 8u, (turn >> 1) & 1u, own.abort_flag, own.limit, lane)) {
      gone = true;
      arrived(x);
      taken();
      return;
    }
    uint32_t g4[2][4], u4[2][4], a4[2][4], mask[2];
    F2 w[2], dw2[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const uint32_t from = buf + piece2(8 * n + (lane & 7), 0, lane >> 3);
      ldmatrix_t(from, g4[n]);
      ldmatrix_t(from + 64, u4[n]);
      const uint32_t from_w = at + 2 * kBuffer + (uint32_t)((c0 >> 5) * 16 + 8 * n + 2 * (lane & 3)) * 4;
      float w0, w1;
      asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(w0), "=f"(w1) : "r"(from_w) : "memory");
      w[n] = f2(w0, w1);
      mask[n] = (w0 != 0.0f ? 0xffffu : 0u) | (w1 != 0.0f ? 0xffff0000u : 0u);
      dw2[n] = f2(0.0f, 0.0f);
    }
    arrived(x);
    taken();
    __syncwarp();
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {       // eight lanes from 8 j, two columns
        const float2 g = bf16_unpair(g4[n][j]), u = bf16_unpair(u4[n][j]);
        const F2 gg = f2(g.x, g.y), uu = f2(u.x, u.y);
        const F2 d1 = f2(x.v[j >> 1][4 * n + 2 * (j & 1)], x.v[j >> 1][4 * n + 2 * (j & 1) + 1]);
        const F2 one = f2(1.0f, 1.0f);
        float e0, e1;
        f2_get(f2_mul(gg, f2(-kLog2e, -kLog2e)), e0, e1);
        f2_get(f2_add(f2(ex2(e0), ex2(e1)), one), e0, e1);
        const F2 sg = f2(rcp(e0), rcp(e1)), gs = f2_mul(gg, sg);
        const F2 slope = f2_fma(gs, f2_fma(sg, f2(-1.0f, -1.0f), one), sg);      // of silu: s + gate s (1 - s)
        const F2 act = f2_mul(gs, uu), d = f2_mul(w[n], d1);
        g4[n][j] = bf16_pair(f2_mul(f2_mul(d, uu), slope)) & mask[n];
        u4[n][j] = bf16_pair(f2_mul(d, gs)) & mask[n];
        a4[n][j] = bf16_pair(f2_mul(w[n], act)) & mask[n];
        if (lane0 + 8 * j < p.lanes) dw2[n] = f2_fma(d1, act, dw2[n]);
      }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const uint32_t to = buf + piece2(8 * n + (lane & 7), 0, lane >> 3);
      stmatrix_t(to, g4[n][0], g4[n][1], g4[n][2], g4[n][3]);
      stmatrix_t(to + 64, u4[n][0], u4[n][1], u4[n][2], u4[n][3]);
      stage64(buf + 2 * kArea, lane, n, a4[n][0], a4[n][1], a4[n][2], a4[n][3]);
    }
    if (c0 + kCols <= t.ncols) {
      written();
      if (lane == 0) {
        tma_store3(&maps.out[0], lane0, 0, t.n0 + c0, buf);
        tma_store2(&maps.out[1], lane0, t.n0 + c0, buf + 2 * kArea);
        tma_store_commit();
      }
    } else {
      __syncwarp();
      const int x = lane0 + 8 * (lane & 3);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int column = 8 * i + (lane >> 2);
        const uint4 u0 = lds16(buf + piece2(column, 0, lane & 3)), u1 = lds16(buf + piece2(column, 1, lane & 3));
        if (c0 + column < t.ncols && x < p.lanes && DX_BOUNDS(t.n0 + c0 + column < p.n_rows, p.dev_status)) {
          __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(p.out) + (int64_t)(t.n0 + c0 + column) * p.ld + x;
          *reinterpret_cast<uint4*>(to) = u0;
          *reinterpret_cast<uint4*>(to + p.lanes) = u1;
        }
      }
      flush_bf16<16>(p, lane, buf + 2 * kArea, sorted_row(t, c0, lane), lane0, reinterpret_cast<__nv_bfloat16*>(p.act_w),
                     p.ld_act);
      written();            // (boxes of the chunk after the next come here)
    }
    if (p.partial) {
      // eight threads (t / 4) hold shares of the columns 8 n + 2 (t % 4) + i: folded so that two of them each end with one
      float dw[4];
#pragma unroll
      for (int n = 0; n < 2; ++n) f2_get(dw2[n], dw[2 * n], dw[2 * n + 1]);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int h = 2 >> b, bit = 16 >> b;
        const bool high = (lane & bit) != 0;
#pragma unroll
        for (int j = 0; j < h; ++j) {
          const float got = __shfl_xor_sync(0xffffffffu, high ? dw[j] : dw[j + h], bit);
          dw[j] = (high ? dw[j + h] : dw[j]) + got;
        }
      }
      dw[0] += __shfl_xor_sync(0xffffffffu, dw[0], 4);
      const int k = lane >> 3, column = c0 + 8 * (k >> 1) + 2 * (lane & 3) + (k & 1);
      if (!(lane & 4) && column < t.ncols && DX_BOUNDS(t.n0 + column < p.n_rows && lane0 < p.lanes, p.dev_status))
        p.partial[(int64_t)(lane0 >> 5) * p.n_rows + t.n0 + column] = dw[0];
    }
    ++turn;
  }
};

// d pair_w[q] = sum of the shares, in order.  The row of a pair of weight 0 was taken out and may hold anything: where that makes
// no finite number, 0.
__global__ void __launch_bounds__(256) dx_pair_weight_grad_kernel(const float* partial, int parts, int n_rows,
                                                                  const int32_t* offsets, int n_groups,
                                                                  const int32_t* index, const float* pair_w, int n_pairs,
                                                                  float* d_pair_w,
                                                                  int32_t* dev_status) {
  dx_pdl_wait();
  dx_pdl_trigger();
  const int r = blockIdx.x * 256 + threadIdx.x;
  const int lo = max(0, __ldg(offsets)), hi = min(n_rows, __ldg(offsets + n_groups));
  if (r < lo || r >= hi || !DX_BOUNDS(r < n_rows, dev_status)) return;
  const int q = index ? __ldg(index + r) : r;
  if (q < 0 || q >= n_pairs) return;
  float sum = 0.0f;
#pragma unroll 16
  for (int i = 0; i < parts; ++i) sum += __ldg(partial + (int64_t)i * n_rows + r);      // (16 on their way at a time)
  d_pair_w[q] = isfinite(sum) || !pair_w || __ldg(pair_w + q) != 0.0f ? sum : 0.0f;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return fn;
}

}  // namespace

bool dx_tensor_map(CUtensorMap* out, const void* base, int rank, const uint64_t* dims, const uint64_t* strides,
                   const uint32_t* box) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  cuuint64_t d[5], s[4];
  cuuint32_t b[5], one[5] = {1, 1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) {
    d[i] = dims[i];
    b[i] = box[i];
    if (i + 1 < rank) s[i] = strides[i] * 2;
  }
  return encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), d, s, b, one,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool dx_box_map(CUtensorMap* out, const void* base, bool fp32, int rank, const uint64_t* dims, const uint64_t* strides,
                const uint32_t* box) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  const uint64_t elem = fp32 ? 4 : 2;
  cuuint64_t d[3], s[2];
  cuuint32_t b[3], one[3] = {1, 1, 1};
  for (int i = 0; i < rank; ++i) {
    d[i] = dims[i];
    b[i] = box[i];
    if (i + 1 < rank) s[i] = strides[i] * elem;
  }
  const uint64_t width = box[0] * elem;
  return encode(out, fp32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank,
                const_cast<void*>(base), d, s, b, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                width == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : width == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {
// boxes of `width` x `height` of a matrix
bool box_map(CUtensorMap* out, const void* base, bool fp32, int64_t rows, int64_t cols, int64_t ld, int width, int height) {
  const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows}, strides[1] = {(uint64_t)ld};
  const uint32_t box[2] = {(uint32_t)width, (uint32_t)height};
  return dx_box_map(out, base, fp32, 2, dims, strides, box);
}
// boxes of 32 columns of both halves (of `cols` each) of sixteen rows
bool halves_map(CUtensorMap* out, const void* base, int64_t rows, int64_t cols, int64_t ld) {
  const uint64_t dims[3] = {(uint64_t)cols, 2, (uint64_t)rows}, strides[2] = {(uint64_t)cols, (uint64_t)ld};
  const uint32_t box[3] = {32, 2, 16};
  return dx_box_map(out, base, false, 3, dims, strides, box);
}
}  // namespace

bool dx_matrix_map(CUtensorMap* out, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows}, strides[1] = {(uint64_t)ld};
  const uint32_t box[2] = {64, (uint32_t)box_rows};
  return dx_tensor_map(out, base, 2, dims, strides, box);
}

namespace {

// Few rows per group: the weights' bytes are the time, so tiles are small (128 lanes: twice as many CTAs have one, and eight
// stages of 24 KB keep 128 KB of weights in flight per SM).  That pays up to 32 rows where the matrices' rows are the contraction
// (64 groups of 24 rows x 2048 x 1408: 61.8 us, in pairs 67.8; its SwiGLU gradient 77.5, in pairs 86.4), otherwise for a handful
// (SwiGLU of one row 116.5 us, in pairs 117.7, of eight 118.3 and 119.6, of 40 123.4 and 123.0; W x of 24 64.2 and 63.3).  Some
// rows, and matrices whose rows are the contraction: 128 lanes with 128 columns (96 rows 67 us, in pairs 73; SwiGLU gradient 95,
// in pairs 103.  128 rows in every group 71 and 76, but 128 in the mean, as routing deals them out, 82 and 78, its SwiGLU
// gradient 123 and 115: groups of 129 rows take two tiles.  The other forms lose with it at 40 rows already: SwiGLU 137 us, in
// pairs 133).  Otherwise pairs of CTAs with 256 lanes x 256 columns.
template <int FORM, bool GATHER, class Epilogue>
cudaError_t launch_rows(dx_ctx* ctx, const MmMaps& maps, const MmParams& p, cudaStream_t st) {
  const bool few = p.n_rows <= (FORM == kRowsT ? kFewRows : kFewestRows) * (int64_t)p.n_groups;
  const bool some = FORM == kRowsT && !few && p.n_rows <= kSomeRows * (int64_t)p.n_groups;
  const long long lanes = few || some ? 128 : 256, bn = few ? 64 : some ? 128 : 256;
  // (every group may end in a tile that is not full)
  const long long most = ((p.lanes + lanes - 1) / lanes) *
                         ((p.n_rows + bn - 1) / bn + (p.n_groups < p.n_rows ? p.n_groups : p.n_rows));
  // (stages: as many as the staging leaves room for)
  constexpr int kFew = Epilogue::kStaging > 4096 ? 6 : 8, kMany = Epilogue::kStaging > 4096 ? 5 : 6;
  if (few) return mm_launch<FORM, GATHER, 1, 64, kFew, Epilogue>(ctx, maps, p, most, st);
  if constexpr (FORM == kRowsT)
    if (some) return mm_launch<FORM, GATHER, 1, 128, kMany, Epilogue>(ctx, maps, p, most, st);
  return mm_launch<FORM, GATHER, 2, 256, kMany, Epilogue>(ctx, maps, p, most, st);
}
template <int FORM, class Epilogue>
cudaError_t launch_rows(dx_ctx* ctx, const MmMaps& maps, const MmParams& p, cudaStream_t st) {
  return p.b_index || p.b_div.factor != 0u ? launch_rows<FORM, true, Epilogue>(ctx, maps, p, st)
                                           : launch_rows<FORM, false, Epilogue>(ctx, maps, p, st);
}

// the rows (columns of D): a tensor map, or the matrix they are gathered from
bool rows_source(MmMaps* m, MmParams* p, const DxGroupedMm& a, int cols) {
  p->b_index = a.gather;
  p->b_div = mm_div(a.gather_div);
  p->b_rows = a.x_rows;
  p->b_src = a.x;
  p->b_ld = a.ldx;
  int64_t rows = a.x_rows;
  if (a.w_rows) {      // (panels)
    rows = (int64_t)((a.w_rows + kPanel - 1) / kPanel) * a.group_rows;
    cols = kPanel;
  }
  return a.gather || a.gather_div > 1 ||
         (dx_matrix_map(&m->b, a.x, rows, cols, a.ldx, 128) && dx_matrix_map(&m->b_few, a.x, rows, cols, a.ldx, 32));
}

MmParams base_params(const dx_ctx* ctx, const int32_t* offsets, int groups, int rows) {
  MmParams p = {};
  p.offsets = offsets;
  p.n_groups = groups;
  p.n_rows = rows;
  p.dev_status = ctx->dev_status;
  p.wait_limit = ctx->wait_limit;
  p.section = kSectionBf16;
  return p;
}

}  // namespace

cudaError_t dx_launch_grouped_mm(dx_ctx* ctx, const DxGroupedMm& a, cudaStream_t st) {
  MmMaps m = {};
  MmParams p = base_params(ctx, a.offsets, a.n_groups, a.n_rows);
  const int n_in = a.transposed ? a.n : a.k, n_out = a.transposed ? a.k : a.n;
  p.lanes = n_out;
  p.kdim = n_in;
  p.out = a.y;
  p.ld = a.ldy;
  p.scatter = a.scatter;
  p.out_rows = a.y_rows;
  p.addend = a.addend;
  if (a.y_fp32 && !a.w_rows) p.section = kSectionFp32;      // (shares of the loss's gradient end in bf16)
  if (a.w_rows) {
    p.n_live = a.n_live;
    p.group_rows = a.group_rows;
    p.shared_out = (a.w_rows + kMmK - 1) / kMmK;
    p.kdim = a.w_rows;
  }
  const uint64_t dims[3] = {(uint64_t)a.k, (uint64_t)(a.w_rows ? a.w_rows : a.n), (uint64_t)(a.w_rows ? 1 : a.n_groups)};
  const uint64_t strides[2] = {(uint64_t)a.ldw, (uint64_t)a.w_stride};
  const uint32_t box[3] = {64, a.transposed ? 64u : 128u, 1};
  if (!dx_tensor_map(&m.a, a.w, 3, dims, strides, box) || !rows_source(&m, &p, a, n_in) ||
      (!a.scatter && !a.addend && !box_map(&m.out[0], a.y, a.y_fp32, a.y_rows, n_out, a.ldy, 32, a.y_fp32 ? 16 : 32)))
    return cudaErrorInvalidValue;
  if (a.transposed) {
    if (a.addend)      // (rows in place: shares of the loss's gradient)
      return a.y_fp32 ? launch_rows<kRowsT, false, StoreRows<float, true>>(ctx, m, p, st)
                      : launch_rows<kRowsT, false, StoreRows<__nv_bfloat16, true>>(ctx, m, p, st);
    return a.y_fp32 ? launch_rows<kRowsT, StoreRows<float, false>>(ctx, m, p, st)
                    : launch_rows<kRowsT, StoreRows<__nv_bfloat16, false>>(ctx, m, p, st);
  }
  return a.y_fp32 ? launch_rows<kRows, StoreRows<float, false>>(ctx, m, p, st)
                  : launch_rows<kRows, StoreRows<__nv_bfloat16, false>>(ctx, m, p, st);
}

cudaError_t dx_launch_grouped_swiglu(dx_ctx* ctx, const DxGroupedMm& a, void* gate_up, int64_t ld_gate_up, cudaStream_t st) {
  MmMaps m = {};
  MmParams p = base_params(ctx, a.offsets, a.n_groups, a.n_rows);
  const int n_inter = a.n / 2;
  p.lanes = a.n;
  p.kdim = a.k;
  p.out = a.y;
  p.ld = a.ldy;
  p.save = gate_up;
  p.ld_save = ld_gate_up;
  // a tile's lanes: eight gate rows, the same eight up rows, the next eight ...
  const uint64_t dims[5] = {(uint64_t)a.k, 8, 2, (uint64_t)(n_inter / 8), (uint64_t)a.n_groups};
  const uint64_t strides[4] = {(uint64_t)a.ldw, (uint64_t)(n_inter * a.ldw), (uint64_t)(8 * a.ldw), (uint64_t)a.w_stride};
  const uint32_t box[5] = {64, 8, 2, 8, 1};
  const __nv_bfloat16* gu = reinterpret_cast<const __nv_bfloat16*>(gate_up);
  if (!dx_tensor_map(&m.a, a.w, 5, dims, strides, box) || !rows_source(&m, &p, a, a.k) ||
      !box_map(&m.out[0], a.y, false, a.n_rows, n_inter, a.ldy, 16, 32) ||
      (gu && !(box_map(&m.out[1], gu, false, a.n_rows, n_inter, ld_gate_up, 16, 32) &&
               box_map(&m.out[2], gu + n_inter, false, a.n_rows, n_inter, ld_gate_up, 16, 32))))
    return cudaErrorInvalidValue;
  return gate_up ? launch_rows<kSwiglu, StoreSwiglu<true>>(ctx, m, p, st)
                 : launch_rows<kSwiglu, StoreSwiglu<false>>(ctx, m, p, st);
}

int dx_swiglu_grad_parts(int n_inter) { return (int)(((int64_t)n_inter + 255) / 256 * 8); }

cudaError_t dx_launch_grouped_swiglu_grad(dx_ctx* ctx, const DxGroupedMm& a, const void* gate_up, int64_t ld_gate_up,
                                          const float* pair_w, int n_pairs, void* act_w, int64_t ld_act, float* partial,
                                          float* d_pair_w, cudaStream_t st, int* n_launches) {
  MmMaps m = {};
  MmParams p = base_params(ctx, a.offsets, a.n_groups, a.n_rows);
  p.lanes = a.k;
  p.kdim = a.n;
  p.out = a.y;
  p.ld = a.ldy;
  p.pair_w = pair_w;
  p.n_pairs = n_pairs;
  p.act_w = act_w;
  p.ld_act = ld_act;
  p.partial = d_pair_w ? partial : nullptr;
  if (d_pair_w) p.section = kSectionFp32;
  const uint64_t dims[3] = {(uint64_t)a.k, (uint64_t)a.n, (uint64_t)a.n_groups};
  const uint64_t strides[2] = {(uint64_t)a.ldw, (uint64_t)a.w_stride};
  const uint32_t box[3] = {64, 64, 1};
  if (!dx_tensor_map(&m.a, a.w, 3, dims, strides, box) || !rows_source(&m, &p, a, a.n) ||
      !halves_map(&m.in, gate_up, a.n_rows, a.k, ld_gate_up) || !halves_map(&m.out[0], a.y, a.n_rows, a.k, a.ldy) ||
      !box_map(&m.out[1], act_w, false, a.n_rows, a.k, ld_act, 32, 16))
    return cudaErrorInvalidValue;
  cudaError_t e = launch_rows<kRowsT, StoreSwigluGrad>(ctx, m, p, st);
  *n_launches = 1;
  if (e != cudaSuccess || !d_pair_w) return e;
  // (lanes of a tile behind the last are no shares: only warps with lanes that exist wrote theirs)
  const int parts = (a.k + 31) / 32;
  *n_launches = 2;
  return dx_launch_pdl((ctx->pdl_mask & DX_PDL_EXPERTS) != 0, dx_pair_weight_grad_kernel, dim3((a.n_rows + 255) / 256),
                       dim3(256), 0, st, 1, partial, parts, a.n_rows, a.offsets, a.n_groups, a.gather, pair_w, n_pairs, d_pair_w,
                       ctx->dev_status);
}

cudaError_t dx_launch_grouped_dw(dx_ctx* ctx, const DxGroupedDw& a, cudaStream_t st) {
  MmMaps m = {};
  MmParams p = base_params(ctx, a.offsets, a.n_groups, a.n_rows);
  p.lanes = a.k;
  p.columns = a.n;
  p.a_src = a.x;
  p.a_ld = a.ldx;
  p.a_rows = a.x_rows;
  p.b_src = a.dy;
  p.b_ld = a.ld_dy;
  p.b_rows = a.dy_rows;
  p.a_index = a.gather_x;
  p.a_div = mm_div(a.x_div);
  p.b_index = a.gather_dy;
  p.b_div = mm_div(a.dy_div);
  p.out = a.dw;
  p.ld = a.ld_dw;
  if (a.dw_fp32) p.section = kSectionFp32;
  if (a.dy_panels) p.b_panel = a.dy_rows;
  if (!dx_matrix_map(&m.a, a.x, a.x_rows, a.k, a.ldx, 64) ||
      !dx_matrix_map(&m.b, a.dy, (int64_t)(a.dy_panels ? (a.n + kPanel - 1) / kPanel : 1) * a.dy_rows,
                     a.dy_panels ? kPanel : a.n, a.ld_dy, 64))
    return cudaErrorInvalidValue;
  const uint64_t dims[3] = {(uint64_t)a.k, (uint64_t)a.n, (uint64_t)a.n_groups};
  const uint64_t strides[2] = {(uint64_t)a.ld_dw, (uint64_t)a.dw_stride};
  const uint32_t box[3] = {32, a.dw_fp32 ? 16u : 32u, 1};
  if (!dx_box_map(&m.out[0], a.dw, a.dw_fp32, 3, dims, strides, box)) return cudaErrorInvalidValue;
  // Few rows per group, and one, three or five times 128 lanes: pairs would spend a sixth or more of their tiles on lanes that
  // do not exist, so CTAs work by themselves (130 groups of five rows, 1000 x 520 bf16: 45 us, in pairs 52; 256 of two, 640 x
  // 384 fp32: 55, in pairs 64.  Where pairs have no such lanes they are faster: 64 of five, 1408 x 2048 bf16 86 us, by
  // themselves 105).
  const int blocks = (a.k + 127) / 128;
  if (a.n_rows <= 64 * (int64_t)a.n_groups && blocks % 2 && blocks <= 5) {
    const long long tiles = (long long)a.n_groups * blocks * ((a.n + 255) / 256);
    return a.dw_fp32 ? mm_launch<kOuter, true, 1, 256, 4, StoreOuter<float, 4>>(ctx, m, p, tiles, st)
                     : mm_launch<kOuter, true, 1, 256, 4, StoreOuter<__nv_bfloat16, 4>>(ctx, m, p, tiles, st);
  }
  const long long tiles = (long long)a.n_groups * ((a.k + 255) / 256) * ((a.n + 255) / 256);
  return a.dw_fp32 ? mm_launch<kOuter, true, 2, 256, 6, StoreOuter<float, 6>>(ctx, m, p, tiles, st)
                   : mm_launch<kOuter, true, 2, 256, 6, StoreOuter<__nv_bfloat16, 6>>(ctx, m, p, tiles, st);
}
