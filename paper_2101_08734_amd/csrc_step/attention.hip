// nopfs_packed_attention and its gradient: causal attention over packed
// samples of different lengths, query heads in groups that share a kv head.
//
//   S_ij = scale q_i.k_j (j <= i),  lse_i = log sum_j exp S_ij,
//   o_i = sum_j P_ij v_j with P_ij = exp(S_ij - lse_i)
//   dP_ij = do_i.v_j,  dS_ij = P_ij (dP_ij - do_i.o_i)
//   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij do_i
//
// All products are 32x32x16 matrix instructions with 32-bit sums. A wave owns
// 32 columns (queries in the forward and dq kernels, keys in the dk/dv
// kernels) and holds its own rows of the operands in registers for the whole
// pass; tiles of the other side (64 rows, or 128 keys) pass through LDS in two
// buffers, the next tile copied from global memory meanwhile.
//
// Where a call has few rows, the other side is split as well: over the waves
// of a workgroup (splits, joined through LDS) and over workgroups (parts,
// whose 32-bit sums a small kernel joins in order). Nothing is added to memory
// from two places, so results never depend on the order of the workgroups.
//
// S is computed transposed to its owner: tile[m][n] with n the owned column,
// so a lane holds 16 of a column's 32 values (its half of the wave the other
// 16) and a row statistic needs one exchange between the halves. Those
// registers, rounded to 16 bits, are at once the B operand of the second
// product: there the sum runs over m, whose order inside the product is free
// as long as A uses the same, and A (the transposed tile) is read from LDS
// with the transposing 64-bit read, four values of m per lane in that order.
//
// LDS rows are cut in 16-byte chunks, chunk c of row r at c ^ f(r) (low three
// bits) with f(r) = (r & 3) << 1 | (r >> 2 & 1): eight consecutive rows put
// one chunk on eight different bank groups (the row reads), and four
// consecutive rows put a 32-byte pair on four (the transposing reads).
//
// Softmax statistics, sums and the delta_i = do_i.o_i are held in 32 bits.
// P and dS are rounded to the inputs' type for the second products (they are
// matrix operands); everything else is rounded once, at the store. In fp16 the
// gradient's P and dS carry a power of two that its sums give back, since dS may
// be out of its range (beyond 65504, or subnormal for small do and long samples)
// where dq and dk are not: P 2^15; dS of a query in the dq kernel one that follows
// its largest, dS of a key in the dk/dv kernels one from the largest of all its
// queries, which the dq kernel leaves for every 32 rows (tops). 5,173 tokens of 41
// samples x 6 heads of 80: dq 24.5 -> 26.4 us, dk and dv 33.4 -> 35.
#include "step.hpp"

namespace nopfs {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct MBf16 {
  typedef __bf16 T;
  typedef __bf16 V8 __attribute__((ext_vector_type(8)));
  typedef __bf16 V4 __attribute__((ext_vector_type(4)));
  typedef __bf16 V2 __attribute__((ext_vector_type(2)));
  static constexpr bool kNarrow = false;  // has the exponents of 32-bit floats
  static __device__ __forceinline__ f32x16 mma(V8 a, V8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
struct MFp16 {
  typedef _Float16 T;
  typedef _Float16 V8 __attribute__((ext_vector_type(8)));
  typedef _Float16 V4 __attribute__((ext_vector_type(4)));
  typedef _Float16 V2 __attribute__((ext_vector_type(2)));
  static constexpr bool kNarrow = true;
  static __device__ __forceinline__ f32x16 mma(V8 a, V8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

struct Attention {
  int64_t T;
  int32_t n, heads, kv_heads, width;
  float scale;
  int64_t q_s[2], k_s[2], v_s[2], o_s[2], do_s[2], dq_s[2], dk_s[2], dv_s[2];
  const void *q, *k, *v, *d_o;
  void *o, *dq, *dk, *dv;  // o: output of the forward call, input of the gradient
  float* lse;
  float* delta;  // [heads][T] (scratch)
  // dk, dv: parts of a key tile's query tiles (of all heads of the group) that
  // workgroups of their own sum; with more than one, their sums
  // [part][dk, dv][T][kv_heads][width] in 32 bits (scratch), added in order
  // afterwards
  int32_t parts;
  float* partial;
  // the same of a query tile's keys, for o and dq: sums
  // [part][T][heads][width], and for o a row's maximum and sum of exponentials
  // [part][heads][T]
  int32_t q_parts;
  float* q_sums;
  f32x2* q_stats;
  // for dq also sum_j P_ij k_j, the row's statistics then eps_i and whether
  // that sum is there (not 0)
  float* q_bars;
  // fp16: the largest |dS| of 32 rows of a head, in the place of the first of
  // them, from every wave that had a share of it: [tops_of][heads][T]
  float* tops;
  int32_t tops_of;
  const int32_t* start;
  uint32_t tiles;  // an upper bound of the row tiles
  const int4* order;  // the tiles' (sample, first row, begin, length), costliest first, or NULL
};

constexpr float kLog2e = 1.4426950408889634f;
// The running maximum follows a row's scores only when they pass it by more
// than this (base 2): until then exponentials up to 2^8 are summed, exact to
// the same relative error, and the sums need no rescaling.
constexpr float kSlack = 8.0f;
// Exponentials are exp2(c s - c m) in one fused multiply-add as long as c m, which
// is rounded, is at most this: all of a row's then carry the same factor, within
// 2^-15 of 1. Beyond (large scores or scales) it would grow out of the floats'
// range, and they are exp2(c (s - m)).
constexpr float kFusedMost = 0x1p10f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// In fp16 P of the dk/dv kernels times 2^kLiftP. dS of a query is scaled again once
// it passes kMostS, to 2^(kTopS - 1) .. 2^kTopS, and dS of a key's queries to
// 2^(kTopK - 1) .. 2^kTopK by their bound (dS of tops has the delta from o, and
// its row's eps, the sum over all parts, comes on top: up to the parts + 1 times).
constexpr int kLiftP = 15, kTopS = 10, kTopK = 11;
constexpr float kMostS = 0x1p15f;

// The value of a lane combined with that of lane ^ 32.
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Row tiles of BM rows. Sample s's tiles are numbered from
// start[s] / BM + s: consecutive samples' numbers never overlap, since
// ceil((b - a) / BM) <= b / BM - a / BM + 1, and no pass over the lengths is
// needed before the launch. The rows behind the last sample count as one more
// sample.
struct Tile {
  int32_t sample;   // n: the rows of no sample
  int64_t begin;    // the sample's first row
  int32_t len, m0;  // its rows, and the tile's first row in it
};

// start[s], within the rows whatever the array holds; 0 before the first.
__device__ __forceinline__ int64_t sample_begin(const Attention& a, int32_t s) {
  const int64_t v = s <= 0 ? 0 : a.start[s];
  return v < 0 ? 0 : (v > a.T ? a.T : v);
}

// Completes a tile whose sample and first row are known; false where the row
// is none of the sample's.
__device__ __forceinline__ bool finish_tile(const Attention& a, Tile* t) {
  t->begin = sample_begin(a, t->sample);
  const int64_t end = t->sample < a.n ? sample_begin(a, t->sample + 1) : a.T;
  t->len = int32_t(end > t->begin ? end - t->begin : 0);
  return t->m0 >= 0 && t->m0 < t->len;
}

template <int BM>
__device__ inline bool find_tile(const Attention& a, uint32_t tile, Tile* t) {
  const int lane = __lane_id();
  // the last s in [lo, hi] whose number is <= tile, 64 candidates at a time
  int32_t lo = 0, hi = a.n;
  while (hi > lo) {
    const int32_t step = (hi - lo + 63) >> 6;  // candidates lo + step * (lane + 1)
    const int64_t cand = int64_t(lo) + int64_t(step) * (lane + 1);
    const bool le = cand <= hi && sample_begin(a, int32_t(cand)) / BM + cand <= int64_t(tile);
    const int k = __popcll(__ballot(le));  // monotone: the first k hold
    const int64_t top = int64_t(lo) + int64_t(step) * (k + 1) - 1;
    lo += step * k;
    hi = top < hi ? int32_t(top) : hi;
  }
  t->sample = lo;
  t->m0 = int32_t((int64_t(tile) - (sample_begin(a, lo) / BM + lo)) * BM);
  return finish_tile(a, t);
}

// The workgroup's tile: the rank-th of the order, or without one the tiles as
// packed, from the last (kLast) or from the first.
template <int BM, bool kLast>
__device__ __forceinline__ bool pick_tile(const Attention& a, uint32_t rank, Tile* t) {
  if (rank >= a.tiles) return false;
  if (a.order) {
    const int4 e = a.order[rank];
    *t = Tile{e.x, e.z, e.w, e.y};
    return e.x >= 0;
  }
  return find_tile<BM>(a, kLast ? a.tiles - 1 - rank : rank, t);
}

// Orders the tiles by what they cost, so that the longest work starts first:
// by their first row (a query tile sees the keys up to itself, by_row), or by
// the rows from there to the sample's end (a key tile). A counting sort by one
// workgroup; which of two tiles of one class comes first is left open (no
// result depends on it). Bound by the latency of its searches: the starts are
// in LDS where they fit (16,384 tokens of 32 samples: 9.2 -> 6.5 us,
// launch included). Beyond kHeldStarts samples they are read from global memory,
// and all tiles are one workgroup's work, however many.
constexpr int kClasses = 1024, kHeldStarts = 4096;
struct OrderJob {
  int4* order;
  uint32_t tiles;
  int32_t log_rows;  // of a tile
  bool by_row;
};
__global__ void __launch_bounds__(1024) at_order(const Attention a, const OrderJob j0, const OrderJob j1) {
  __shared__ uint32_t count[kClasses];
  __shared__ uint32_t tmp[65];
  __shared__ int32_t starts[kHeldStarts];
  const OrderJob& j = blockIdx.x == 0 ? j0 : j1;
  const bool held = a.n < kHeldStarts;
  if (held)
    for (int32_t s = threadIdx.x; s <= a.n; s += 1024) starts[s] = int32_t(sample_begin(a, s));
  int shift = 0;
  while (a.T >> j.log_rows >> shift >= kClasses) ++shift;
  count[threadIdx.x] = 0;
  __syncthreads();
  auto begin = [&](int32_t s) { return held ? starts[s] : int32_t(sample_begin(a, s)); };
  auto number = [&](int32_t s) { return (begin(s) >> j.log_rows) + s; };  // < 2^31
  auto tile = [&](uint32_t i, Tile* t) {
    int32_t lo = 0, hi = a.n;
    while (hi > lo) {
      const int32_t mid = lo + (hi - lo + 1) / 2;
      if (uint32_t(number(mid)) <= i) lo = mid;
      else hi = mid - 1;
    }
    t->sample = lo;
    t->begin = begin(lo);
    t->len = (lo < a.n ? begin(lo + 1) : int32_t(a.T)) - int32_t(t->begin);
    t->m0 = (int32_t(i) - number(lo)) << j.log_rows;
    if (t->m0 < 0 || t->m0 >= t->len) return -1;
    const int cost = (j.by_row ? t->m0 : t->len - t->m0 - 1) >> j.log_rows;
    return kClasses - 1 - min(lo == a.n ? 0 : cost >> shift, kClasses - 1);
  };
  for (uint32_t i = threadIdx.x; i < j.tiles; i += 1024) {
    Tile t;
    const int c = tile(i, &t);
    if (c >= 0) atomicAdd(&count[c], 1u);
  }
  __syncthreads();
  uint32_t total;
  const uint32_t first = block_exclusive_scan(count[threadIdx.x], tmp, &total);
  count[threadIdx.x] = first;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < j.tiles; i += 1024) {
    Tile t;
    const int c = tile(i, &t);
    if (c >= 0) j.order[atomicAdd(&count[c], 1u)] = int4{t.sample, t.m0, int32_t(t.begin), t.len};
  }
  for (uint32_t i = total + threadIdx.x; i < j.tiles; i += 1024) j.order[i] = int4{-1, 0, 0, 0};
}

// Workgroup -> (tile, head): all heads of a tile are neighbours, so every die
// (workgroup b runs on die b mod 8) gets the same share of each sample; where
// the heads divide by 8, a die has neighbouring heads, which share kv heads in
// its L2.
__device__ __forceinline__ void tile_and_head(uint32_t b, uint32_t heads, uint32_t* tile, uint32_t* head) {
  *tile = b / heads;
  const uint32_t h = b % heads;
  *head = heads % 8 == 0 ? (h % 8) * (heads / 8) + h / 8 : h;
}

__device__ __forceinline__ int row_swizzle(int r) { return ((r & 3) << 1) | ((r >> 2) & 1); }
// Byte offset of 16-byte chunk c of row r in an LDS tile of DP-element rows.
template <int DP>
__device__ __forceinline__ int lds_chunk(int r, int c) {
  return r * (DP * 2) + ((c ^ row_swizzle(r)) << 4);
}

// Copies of a tile of ROWS rows from global memory straight into LDS, by 256
// threads and 16 bytes a lane. A wave's copy fills 64 consecutive chunks of
// LDS, so a lane picks the chunk of the row that belongs in its place. Rows
// past the sample's end are its last row again (finite wherever the sample is;
// what they give is masked or not stored). Chunks past the width are not
// copied: zero_pad clears them once.
template <int DP, int ROWS>
struct TileCopy {
  static constexpr int kChunks = DP / 8;
  static constexpr int kStep = 256 / kChunks;  // rows of one round of copies: a multiple of 8, so
  static constexpr int kPer = ROWS / kStep;    // a lane's chunk is the same in every round
  uint32_t off;     // the lane's byte offset in the first round
  uint32_t stride;  // bytes from row to row
  int row;          // the lane's row in the first round
  bool in;
  __device__ __forceinline__ TileCopy(int64_t elems, int width) : stride(uint32_t(elems * 2)) {
    row = int(threadIdx.x) / kChunks;
    const int chunk = int(threadIdx.x) % kChunks ^ row_swizzle(row);
    in = chunk * 8 < width;
    off = uint32_t(row) * stride + uint32_t(chunk) * 16;
  }
  // base: the tile's first row; rows: the sample's rows from there on (>= 1)
  __device__ __forceinline__ void copy(const char* base, int rows, char* lds) const {
    if (!in) return;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      uint32_t o = off;
      if (rows < ROWS) o -= uint32_t(max(row + j * kStep - (rows - 1), 0)) * stride;
      // o wraps below 0 only together with the round's start: the sum is taken in 32 bits
      const uint32_t at = o + uint32_t(j * kStep) * stride;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + at),
                                       (__attribute__((address_space(3))) void*)(lds + j * 4096 + wave * 1024),
                                       16, 0, 0);
    }
  }
  __device__ __forceinline__ void zero_pad(char* lds) const {
    if (in) return;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      *reinterpret_cast<u32x4*>(lds + j * 4096 + threadIdx.x * 16) = u32x4{0, 0, 0, 0};
  }
};

// Every wave is here and has what it read from or wrote to LDS behind it, and
// its copies into LDS have landed, all but the last kBehind. (A __syncthreads
// would wait for all of them: the next tile's too.)
template <int kBehind>
__device__ __forceinline__ void meet() {
  static_assert(kBehind < 64, "vmcnt has 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (kBehind & 15) | (kBehind >> 4) << 14);  // vmcnt(kBehind) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A operand (32 rows x 16 elements): row `row0 + lane % 32` of an LDS tile.
template <class M, int DP>
__device__ __forceinline__ typename M::V8 frag_row(const char* lds, int row0, int chunk) {
  const int lane = threadIdx.x & 63;
  const int r = lane & 31;
  return *reinterpret_cast<const typename M::V8*>(lds + row0 * (DP * 2) + lds_chunk<DP>(r, chunk + (lane >> 5)));
}

// A operand of the transposed tile: element column `d0 + lane % 32` over 16
// tile rows from row0, in the order in which the first product's registers
// hold them: row0 + 4 half + 0..3, then row0 + 8 + 4 half + 0..3.
template <class M, int DP>
__device__ __forceinline__ typename M::V8 frag_col(const char* lds, int row0, int d0) {
  const int lane = threadIdx.x & 63;
  const int l = lane & 15;
  const int row = 4 * (lane >> 5) + (l >> 2);  // + row0, a multiple of 16: the swizzle is of `row`
  const int chunk = (d0 >> 3) + 2 * ((lane >> 4) & 1) + ((l >> 1) & 1);
  const char* p = lds + row0 * (DP * 2) + lds_chunk<DP>(row, chunk) + ((l & 1) << 3);
  typedef __attribute__((address_space(3))) s16x4 lds_v4;
  union {
    s16x4 h[2];
    typename M::V8 v;
  } u;
  u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4*)(p));
  u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4*)(p + 8 * (DP * 2)));
  return u.v;
}

// B operand from registers 8c..8c+7 of a first product's 32x32 tile.
template <class M>
__device__ __forceinline__ typename M::V8 pack8(const f32x16& x, int c) {
  union {
    typename M::V2 p[4];
    typename M::V8 v;
  } u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 y = {x[8 * c + 2 * i], x[8 * c + 2 * i + 1]};
    u.p[i] = __builtin_convertvector(y, typename M::V2);
  }
  return u.v;
}

// A row's value minus what a first product will add to it: the accumulator of
// a 32x32 tile, every column -x of its row, from one bf16 matrix product. The
// lanes of half `part` hold x of rows 0..31; x as a sum of three bf16 values is
// exact to 2^-24 of it, and the ones of the other operand pick them.
__device__ __forceinline__ f32x16 minus_rows(float x, int part) {
  const bool mine = ((threadIdx.x & 63) >> 5) == part;
  const float y = mine ? -x : 0.0f;
  const __bf16 one = __bf16(1.0f), zero = __bf16(0.0f);
  const __bf16 hi = __bf16(y);
  const float r = y - float(hi);
  const __bf16 mid = __bf16(r);
  const MBf16::V8 a = {hi, mid, __bf16(r - float(mid)), zero, zero, zero, zero, zero};
  const MBf16::V8 b = {one, one, one, zero, zero, zero, zero, zero};
  f32x16 c;
#pragma unroll
  for (int e = 0; e < 16; ++e) c[e] = 0.0f;
  return MBf16::mma(a, b, c);
}

// A column's operand chunk straight from global memory: 8 elements at
// 16 c + 8 half of the lane's own row, 0 past the width.
template <class M>
__device__ __forceinline__ typename M::V8 own_chunk(const typename M::T* row, int c, int width) {
  const int d = 16 * c + 8 * ((threadIdx.x & 63) >> 5);
  union {
    u32x4 u;
    typename M::V8 v;
  } x;
  x.u = *reinterpret_cast<const u32x4*>(row + (d < width ? d : 0));
  if (d >= width) x.u = u32x4{0, 0, 0, 0};
  return x.v;
}

// The tile row of accumulator register r (+ 4 per half of the wave).
__device__ __forceinline__ constexpr int acc_row(int r) { return 8 * (r >> 2) + (r & 3); }

// Stores the columns of an accumulator (element d of the lane's own row).
template <class M, int DT>
__device__ __forceinline__ void store_columns(typename M::T* row, const f32x16* acc, float f, int width) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 32 * t + 8 * i + 4 * half;
      if (d >= width) continue;
      typename M::V4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = typename M::T(acc[t][4 * i + e] * f);
      *reinterpret_cast<typename M::V4*>(row + d) = v;
    }
}
template <int DT>
__device__ __forceinline__ void store_sums(float* row, const f32x16* acc, int width) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 32 * t + 8 * i + 4 * half;
      if (d < width)
        *reinterpret_cast<f32x4*>(row + d) =
            f32x4{acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]};
    }
}

// dk and dv of the lane's key (row kr of all), elements d0 on: rounded where a
// workgroup has the whole group's sums, else its part of them.
template <class M, int DT>
__device__ __forceinline__ void store_dkv(const Attention& a, int64_t kr, int64_t kv, int part, int d0,
                                          const f32x16* dk, const f32x16* dv) {
  typedef typename M::T T;
  if (a.parts == 1) {
    store_columns<M, DT>(static_cast<T*>(a.dk) + kr * a.dk_s[0] + kv * a.dk_s[1] + d0, dk, a.scale, a.width - d0);
    store_columns<M, DT>(static_cast<T*>(a.dv) + kr * a.dv_s[0] + kv * a.dv_s[1] + d0, dv, 1.0f, a.width - d0);
    return;
  }
  const int64_t size = a.T * a.kv_heads * a.width;
  float* row = a.partial + 2 * part * size + (kr * a.kv_heads + kv) * a.width + d0;
  store_sums<DT>(row, dk, a.width - d0);
  store_sums<DT>(row + size, dv, a.width - d0);
}

template <int DT>
__device__ __forceinline__ void scale_sums(f32x16* acc, float f) {
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] *= f;
}

// The exponent that brings a key tile's dS of query tiles i0 .. i0 + n - 1 (of its
// sample's from j0 to j1 for all heads of the group) into range; the same in every
// thread. Infinities and NaN among them count for nothing. lds: free, and free again.
__device__ inline int ds_exponent(const Attention& a, const Tile& t, int64_t head0, int j0, int j1, int i0, int n,
                                  float* lds) {
  float top = 0.0f;
  for (int x = threadIdx.x; x < 2 * n; x += 256) {
    const int i = i0 + x / 2, row = (j0 + i % (j1 - j0)) * 64 + 32 * (x & 1);
    if (row >= t.len) continue;
    const float* p = a.tops + (head0 + i / (j1 - j0)) * a.T + t.begin + row;
    for (int c = 0; c < a.tops_of; ++c) top = fmaxf(top, p[c * (a.heads * a.T)]);
  }
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
  __syncthreads();
  const int e = top > 0.0f ? kTopK - __builtin_amdgcn_frexp_expf(top) : 0;
  return __builtin_amdgcn_readfirstlane(max(-100, min(100, e)));
}

// A wave's accumulators through LDS to the wave that owns the same columns,
// which adds them: acc = acc * f0 + theirs * f1.
template <int DT>
__device__ __forceinline__ void give_columns(char* lds, const f32x16* acc) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = {acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]};
      *reinterpret_cast<f32x4*>(lds + ((t * 4 + i) * 64 + lane) * 16) = v;
    }
}
template <int DT>
__device__ __forceinline__ void take_columns(const char* lds, f32x16* acc, float f0, float f1) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(lds + ((t * 4 + i) * 64 + lane) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[t][4 * i + e] = acc[t][4 * i + e] * f0 + v[e] * f1;
    }
}

template <class M>
__device__ inline void zero_rows(void* base, const int64_t* s, int64_t head, int64_t row0, int rows, int width) {
  const int per = width / 8;
  for (int i = threadIdx.x; i < rows * per; i += 256) {
    typename M::T* p = static_cast<typename M::T*>(base) + (row0 + i / per) * s[0] + head * s[1] + (i % per) * 8;
    *reinterpret_cast<u32x4*>(p) = u32x4{0, 0, 0, 0};
  }
}

// A workgroup's 4 waves are strips of 32 columns, times splits of the other
// side: with several splits, as many waves share a strip's columns, each takes
// its share of every tile's blocks, and their sums are joined through LDS at
// the end. Keys of a tile (forward, dq): a block of 32 for every split, or two.
template <int kSplits>
constexpr int kTileKeys = kSplits == 4 ? 128 : 64;

// ------------------------------------------------------------------ forward --
// One pass over the keys up to the diagonal with the running maximum and sum.
// 16,384 tokens of three samples, 16 heads of 128 on 2: 602 to 629 us on
// different cards, 0.97 PFLOP/s of the 1.38 of a large product; matrix units 46%
// busy, vector units (exponentials, maxima, roundings) 42%, LDS 46%: the phases of a
// SIMD's two waves overlap in part only. 8,192 x 16 heads of 64: 167 to 176 us, 0.80
// PFLOP/s, vector units 57%: half the products per exponential. 16,384 tokens of 32
// documents: 105 to 116 us, matrix units 28%; 228 MB read behind the L2s where the
// arrays hold 101: a sample's tiles on different dies read its keys again.
template <class M, int DP, int DW, int kSplits>
__global__ void __launch_bounds__(256, kSplits == 4 && DP == 128 ? 1 : 2) at_forward(const Attention a) {
  typedef typename M::T T;
  constexpr int DT = DW / 32, DC = DW / 16;
  constexpr int kKeys = kTileKeys<kSplits>, kStrips = 4 / kSplits, kRows = 32 * kStrips, NU = kKeys / 32 / kSplits;
  constexpr int kTileBytes = kKeys * DP * 2;
  // two buffers, apart by name so that a read waits for its own buffer's copies only
  __shared__ __align__(16) char lk0[kTileBytes], lv0[kTileBytes], lk1[kTileBytes], lv1[kTileBytes];
  uint32_t tile, head;
  tile_and_head(row_block(), uint32_t(a.heads * a.q_parts), &tile, &head);
  const int which = int(head) % a.q_parts;  // neighbours: the parts of a head
  head /= uint32_t(a.q_parts);
  Tile t;
  // the last tiles of the packed rows first: long samples' last rows see most keys
  if (!pick_tile<kRows, true>(a, tile, &t)) return;
  const int width = a.width;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, half = lane >> 5;
  const int strip = wave % kStrips, split = kSplits == 1 ? 0 : wave / kStrips;
  T* o = static_cast<T*>(a.o) + t.begin * a.o_s[0] + head * a.o_s[1];
  float* lse = a.lse + int64_t(head) * a.T + t.begin;
  if (t.sample == a.n) {
    if (a.q_parts > 1) return;  // the sum of the parts has these rows
    const int rows = min(kRows, t.len - t.m0);
    zero_rows<M>(a.o, a.o_s, head, t.begin + t.m0, rows, width);
    for (int i = threadIdx.x; i < rows; i += 256) lse[t.m0 + i] = -INFINITY;
    return;
  }
  const int64_t kv = head / (a.heads / a.kv_heads);
  const T* kb = static_cast<const T*>(a.k) + t.begin * a.k_s[0] + kv * a.k_s[1];
  const T* vb = static_cast<const T*>(a.v) + t.begin * a.v_s[0] + kv * a.v_s[1];
  const int q0 = t.m0 + 32 * strip;  // the wave's first query
  const int qi = q0 + (lane & 31);  // the lane's query
  const int qr = min(qi, t.len - 1);
  const T* qrow = static_cast<const T*>(a.q) + (t.begin + qr) * a.q_s[0] + head * a.q_s[1];
  typename M::V8 q[DC];
#pragma unroll
  for (int c = 0; c < DC; ++c) q[c] = own_chunk<M>(qrow, c, width);

  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;  // l: over the lane's own keys
  const float c2 = a.scale * kLog2e, slack = kSlack / c2;

  // this part's tiles of those up to the diagonal: j_first .. n_tiles - 1
  const int64_t all = (min(t.len, t.m0 + kRows) + kKeys - 1) / kKeys;
  const int j_first = int(all * which / a.q_parts), n_tiles = int(all * (which + 1) / a.q_parts);
  const TileCopy<DP, kKeys> ck(a.k_s[0], width), cv(a.v_s[0], width);
  const char* kt = reinterpret_cast<const char*>(kb) + int64_t(ck.stride) * (j_first * kKeys);
  const char* vt = reinterpret_cast<const char*>(vb) + int64_t(cv.stride) * (j_first * kKeys);
  if (width < DP) {
    ck.zero_pad(lk0);
    ck.zero_pad(lk1);
    cv.zero_pad(lv0);
    cv.zero_pad(lv1);
  }
  if (j_first < n_tiles) {
    ck.copy(kt, t.len - j_first * kKeys, lk0);
    cv.copy(vt, t.len - j_first * kKeys, lv0);
  }
  auto step = [&](int j, const char* lk, const char* lv, char* next_k, char* next_v) {
    meet<0>();  // tile j is in LDS, and tile j - 1 is done with
    const int k0 = j * kKeys;
    if (j + 1 < n_tiles) {
      kt += int64_t(ck.stride) * kKeys;
      vt += int64_t(cv.stride) * kKeys;
      ck.copy(kt, t.len - k0 - kKeys, next_k);
      cv.copy(vt, t.len - k0 - kKeys, next_v);
    }
    const int kb = k0 + 32 * NU * split;  // the wave's keys of the tile
    if (kb > q0 + 31) return;  // all later than this wave's queries
    // the other wave of the SIMD fills in with its exponentials (64 elements a head: no gain)
    if constexpr (DP == 128) __builtin_amdgcn_s_setprio(1);
    f32x16 s[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[u][e] = 0.0f;
#pragma unroll
      for (int c = 0; c < DC; ++c)
        s[u] = M::mma(frag_row<M, DP>(lk, 32 * (NU * split + u), 2 * c), q[c], s[u]);
    }
    if constexpr (DP == 128) __builtin_amdgcn_s_setprio(0);
    if (kb + 32 * NU - 1 > q0) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (kb + 32 * u + acc_row(e) + 4 * half > qi) s[u][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
    top = half_max(top);
    if (__any(top > m + slack)) {  // rare: see kSlack
      top = fmaxf(m, top);
      const float f = exp2_fast((m - top) * c2);
      m = top;
      l *= f;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] *= f;
    }
    const float mc = m * c2;
    if (__any(fabsf(mc) > kFusedMost)) {
      const float base = m == -INFINITY ? 0.0f : m;  // no score but -inf yet: exponentials of 0
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[u][e] = exp2_fast((s[u][e] - base) * c2);
          l += s[u][e];
        }
    } else {
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[u][e] = exp2_fast(fmaf(s[u][e], c2, -mc));
          l += s[u][e];
        }
    }
    if constexpr (DP == 128) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const typename M::V8 p = pack8<M>(s[u], c);
#pragma unroll
        for (int i = 0; i < DT; ++i)
          acc[i] = M::mma(frag_col<M, DP>(lv, 32 * (NU * split + u) + 16 * c, 32 * i), p, acc[i]);
      }
    if constexpr (DP == 128) __builtin_amdgcn_s_setprio(0);
  };
  for (int j = j_first; j < n_tiles; j += 2) {
    step(j, lk0, lv0, lk1, lv1);
    if (j + 1 < n_tiles) step(j + 1, lk1, lv1, lk0, lv0);
  }
  if constexpr (kSplits > 1) {
    // the other splits' sums join the first's, rescaled to the larger maximum
    auto place = [&](int i) -> char* { return i == 0 ? lk0 : i == 1 ? lv0 : lk1; };
    float* stats = reinterpret_cast<float*>(lv1) + lane;
    __syncthreads();
    const int slot = (split - 1) * kStrips + strip;
    if (split) {
      give_columns<DT>(place(slot), acc);
      stats[128 * slot] = m;
      stats[128 * slot + 64] = l;
    }
    __syncthreads();
    if (split) return;
#pragma unroll
    for (int x = 0; x < kSplits - 1; ++x) {
      const float* st = stats + 128 * (x * kStrips + strip);
      const float m1 = st[0], top = fmaxf(m, m1);
      const float base = top == -INFINITY ? 0.0f : top;  // neither has a key yet: factors of 0
      const float f0 = exp2_fast((m - base) * c2), f1 = exp2_fast((m1 - base) * c2);
      take_columns<DT>(place(x * kStrips + strip), acc, f0, f1);
      l = l * f0 + st[64] * f1;
      m = top;
    }
  }
  l = half_sum(l);
  if (qi >= t.len) return;
  if (a.q_parts == 1) {
    store_columns<M, DT>(o + int64_t(qi) * a.o_s[0], acc, 1.0f / l, width);
    if (half == 0) lse[qi] = m * a.scale + logf(l);
  } else {
    const int64_t row = which * a.T + t.begin + qi;
    store_sums<DT>(a.q_sums + (row * a.heads + head) * width, acc, width);
    if (half == 0) a.q_stats[(int64_t(which) * a.heads + head) * a.T + t.begin + qi] = f32x2{m, l};
  }
}

// o and lse from the parts' sums, four elements a thread.
template <class M>
__global__ void __launch_bounds__(256) at_join(const Attention a) {
  const int64_t size = a.T * a.heads * a.width;
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (i >= size) return;
  const int64_t rh = i / a.width;
  const int d = int(i - rh * a.width);
  const int64_t row = rh / a.heads, head = rh - row * a.heads;
  f32x4 o = {0, 0, 0, 0};
  float lse = -INFINITY;
  if (row < sample_begin(a, a.n)) {
    const f32x2* st = a.q_stats + head * a.T + row;
    const int64_t step = a.heads * a.T;
    float m = -INFINITY, l = 0.0f;
    for (int p = 0; p < a.q_parts; ++p) m = fmaxf(m, st[p * step][0]);
    for (int p = 0; p < a.q_parts; ++p) {
      const f32x2 x = st[p * step];
      const float f = exp2_fast((x[0] - m) * (a.scale * kLog2e));
      l += f * x[1];
      o += f * *reinterpret_cast<const f32x4*>(a.q_sums + p * size + i);
    }
    o *= 1.0f / l;
    lse = m * a.scale + logf(l);
  }
  typename M::V4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = typename M::T(o[e]);
  *reinterpret_cast<typename M::V4*>(static_cast<typename M::T*>(a.o) + row * a.o_s[0] + head * a.o_s[1] + d) = v;
  if (d == 0) a.lse[head * a.T + row] = lse;
}

// ----------------------------------------------------------------------- dq --
// P again from S and lse, whose subtraction (and delta's) is the accumulators'
// start, so no row statistic is needed; also writes delta_i for the dk/dv
// kernels. delta is do_i.o_i at first, off by eps_i for the roundings of o and of
// the P in it. That is not small beside dP - delta on keys that have most of a
// row's weight (scores of standard deviation 16: dq off by 3.4 roundings of its
// own). The pass sums eps_i = sum_j P_ij (dP_ij - delta_i), 0 for the true delta, in
// 32 bits; dq_i = scale (sum_j dS_ij k_j - eps_i sum_j P_ij k_j), and a second pass
// makes the latter sum over the key tiles where a query of the workgroup has more
// than kHeavy of its weight on a key (the rest of it is small beside what the
// rounding of dS leaves). 8,192 x 16 heads of 64: 216 to 230 us, 0.92 PFLOP/s of
// three products; matrix units 43%, vector units 54%. 16,384 tokens of 32 documents
// x 16 of 128: 162 to 172 us, matrix units 28%; 393 MB read behind the L2s, where
// the arrays hold 235. With standard normal scores and on one card eps and the
// second pass took 204 to 216 and 152 to 162 us; kHeavy 1/16 217 and 171, with no
// smaller errors; heads of 64 with two workgroups a compute unit instead of three 240.
constexpr float kHeavy = 1.0f / 8;
template <class M, int DP, int DW, int kSplits>
__global__ void __launch_bounds__(256, DP == 64 && kSplits < 4 ? 3 : kSplits == 4 && DP == 128 ? 1 : 2) at_dq(const Attention a) {
  typedef typename M::T T;
  constexpr int DT = DW / 32, DC = DW / 16;
  constexpr int kKeys = kTileKeys<kSplits>, kStrips = 4 / kSplits, kRows = 32 * kStrips, NU = kKeys / 32 / kSplits;
  constexpr int kTileBytes = kKeys * DP * 2;
  __shared__ __align__(16) char lk0[kTileBytes], lv0[kTileBytes], lk1[kTileBytes], lv1[kTileBytes];
  uint32_t tile, head;
  tile_and_head(row_block(), uint32_t(a.heads * a.q_parts), &tile, &head);
  const int which = int(head) % a.q_parts;  // neighbours: the parts of a head
  head /= uint32_t(a.q_parts);
  Tile t;
  if (!pick_tile<kRows, true>(a, tile, &t)) return;
  const int width = a.width;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, half = lane >> 5;
  const int strip = wave % kStrips, split = kSplits == 1 ? 0 : wave / kStrips;
  if (t.sample == a.n) {
    if (a.q_parts == 1) zero_rows<M>(a.dq, a.dq_s, head, t.begin + t.m0, min(kRows, t.len - t.m0), width);
    return;
  }
  const int64_t kv = head / (a.heads / a.kv_heads);
  const T* kb = static_cast<const T*>(a.k) + t.begin * a.k_s[0] + kv * a.k_s[1];
  const T* vb = static_cast<const T*>(a.v) + t.begin * a.v_s[0] + kv * a.v_s[1];
  const int q0 = t.m0 + 32 * strip;
  const int qi = q0 + (lane & 31);
  const int64_t qr = t.begin + min(qi, t.len - 1);
  const T* qrow = static_cast<const T*>(a.q) + qr * a.q_s[0] + head * a.q_s[1];
  const T* drow = static_cast<const T*>(a.d_o) + qr * a.do_s[0] + head * a.do_s[1];
  const T* orow = static_cast<const T*>(a.o) + qr * a.o_s[0] + head * a.o_s[1];
  typename M::V8 q[DC], d[DC];
  float delta = 0.0f;
#pragma unroll
  for (int c = 0; c < DC; ++c) {
    q[c] = own_chunk<M>(qrow, c, width);
    d[c] = own_chunk<M>(drow, c, width);
    const typename M::V8 ov = own_chunk<M>(orow, c, width);
#pragma unroll
    for (int e = 0; e < 8; ++e) delta += float(d[c][e]) * float(ov[e]);
  }
  delta = half_sum(delta);
  const int64_t stat = int64_t(head) * a.T + qr;
  const float c2 = a.scale * kLog2e, minus_lse = -a.lse[stat] / a.scale;

  // this part's tiles of those up to the diagonal: j_first .. n_tiles - 1
  const int64_t all = (min(t.len, t.m0 + kRows) + kKeys - 1) / kKeys;
  const int j_first = int(all * which / a.q_parts), n_tiles = int(all * (which + 1) / a.q_parts);
  const TileCopy<DP, kKeys> ck(a.k_s[0], width), cv(a.v_s[0], width);
  const char* kt = reinterpret_cast<const char*>(kb) + int64_t(ck.stride) * (j_first * kKeys);
  const char* vt = reinterpret_cast<const char*>(vb) + int64_t(cv.stride) * (j_first * kKeys);
  if (width < DP) {
    ck.zero_pad(lk0);
    ck.zero_pad(lk1);
    cv.zero_pad(lv0);
    cv.zero_pad(lv1);
  }
  if (j_first < n_tiles) {
    ck.copy(kt, t.len - j_first * kKeys, lk0);
    cv.copy(vt, t.len - j_first * kKeys, lv0);
  }

  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
  float eps = 0.0f;
  int group = 0;  // 2^group tiles share a bit of the tiles to go through again
  while ((n_tiles - 1 - j_first) >> group >= 64) ++group;
  uint64_t heavy = 0;  // such tiles of this wave
  // fp16: P, dS, eps and acc of the lane's query are 2^lift times what they are
  // (dS is below 2^40: products of 128 elements), most the largest |dS|
  float lift = 60.0f, most = 0.0f;

  auto step = [&](int j, const char* lk, const char* lv, char* next_k, char* next_v) {
    meet<0>();
    const int k0 = j * kKeys;
    if (j + 1 < n_tiles) {
      kt += int64_t(ck.stride) * kKeys;
      vt += int64_t(cv.stride) * kKeys;
      ck.copy(kt, t.len - k0 - kKeys, next_k);
      cv.copy(vt, t.len - k0 - kKeys, next_v);
    }
#pragma unroll
    for (int x = 0; x < NU; ++x) {
      const int u = NU * split + x, kb = k0 + 32 * u;
      if (kb > q0) break;  // all later than this wave's queries
      f32x16 s, dp;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = minus_lse;
        dp[e] = -delta;
      }
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        s = M::mma(frag_row<M, DP>(lk, 32 * u, 2 * c), q[c], s);
        dp = M::mma(frag_row<M, DP>(lv, 32 * u, 2 * c), d[c], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = exp2_fast(M::kNarrow ? fmaf(s[e], c2, lift) : s[e] * c2);
      if (kb == q0) {  // the diagonal: both are multiples of 32
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (acc_row(e) + 4 * half > (lane & 31)) s[e] = dp[e] = 0.0f;
      }
      float top = s[0];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        top = fmaxf(top, s[e]);
        s[e] *= dp[e];
        eps += s[e];
      }
      if (__any(top > (M::kNarrow ? kHeavy * exp2_fast(lift) : kHeavy))) heavy |= uint64_t(1) << ((j - j_first) >> group);
      if constexpr (M::kNarrow) {
        top = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(s[e]));
        top = half_max(top);
        most = fmaxf(most, top);
        if (__any(top > kMostS)) {
          const int d = top > kMostS ? kTopS - __builtin_amdgcn_frexp_expf(top) : 0;
          const float f = __builtin_ldexpf(1.0f, d);
          lift += float(d);
          most *= f;
          eps *= f;
          scale_sums<DT>(acc, f);
          scale_sums<1>(&s, f);
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const typename M::V8 p = pack8<M>(s, c);
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[i] = M::mma(frag_col<M, DP>(lk, 32 * u + 16 * c, 32 * i), p, acc[i]);
      }
    }
  };
  for (int j = j_first; j < n_tiles; j += 2) {
    step(j, lk0, lv0, lk1, lv1);
    if (j + 1 < n_tiles) step(j + 1, lk1, lv1, lk0, lv0);
  }
  auto join_splits = [&](f32x16* x) {  // into the first split's
    auto place = [&](int i) -> char* { return i == 0 ? lk0 : i == 1 ? lv0 : lk1; };
    __syncthreads();
    if (split) give_columns<DT>(place((split - 1) * kStrips + strip), x);
    __syncthreads();
    if (split) return;
#pragma unroll
    for (int y = 0; y < kSplits - 1; ++y) take_columns<DT>(place(y * kStrips + strip), x, 1.0f, 1.0f);
  };
  if constexpr (M::kNarrow) {
    const float f = exp2_fast(-lift);
    eps *= f;
    scale_sums<DT>(acc, f);
    float top = fmaf(most, f, fabsf(half_sum(eps)));
    top = top < INFINITY ? top : 0.0f;
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0 && q0 < t.len)
      a.tops[(int64_t(which * kSplits + split) * a.heads + head) * a.T + t.begin + q0] = top;
  }
  // eps of a row from the waves that share it, and the workgroup's heavy tiles
  __syncthreads();
  uint64_t* masks = reinterpret_cast<uint64_t*>(lv0);
  float* others = reinterpret_cast<float*>(lv0 + 64);
  eps = half_sum(eps);
  if (lane == 0) masks[wave] = heavy;
  if constexpr (kSplits > 1) others[wave * 64 + lane] = eps;
  __syncthreads();
  if constexpr (kSplits > 1) {
    eps = 0.0f;
#pragma unroll
    for (int x = 0; x < kSplits; ++x) eps += others[(x * kStrips + strip) * 64 + lane];
  }
  uint64_t todo = masks[0] | masks[1] | masks[2] | masks[3];
  todo = uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(todo >> 32)))) << 32 |
         uint32_t(__builtin_amdgcn_readfirstlane(int(todo)));
  const int64_t part_row = which * a.T + qr;
  if (a.q_parts == 1) {
    if (half == 0 && split == 0 && qi < t.len) a.delta[stat] = delta + eps;
  } else if (half == 0 && split == 0 && qi < t.len) {  // joined by at_sum_dq
    if (which == 0) a.delta[stat] = delta;
    a.q_stats[(int64_t(which) * a.heads + head) * a.T + qr] = f32x2{eps, todo ? 1.0f : 0.0f};
  }
  if (todo) {
    f32x16 bar[DT];  // sum_j P_ij k_j
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) bar[i][e] = 0.0f;
    auto next = [&](int j) {  // the first tile to do from j on
      while (j < n_tiles && !(todo >> ((j - j_first) >> group) & 1)) ++j;
      return j;
    };
    auto copy = [&](int j, char* to) {
      ck.copy(reinterpret_cast<const char*>(kb) + int64_t(ck.stride) * (int64_t(j) * kKeys), t.len - j * kKeys, to);
    };
    int j = next(j_first);
    copy(j, lk0);
    auto again = [&](const char* lk, char* other) {
      meet<0>();  // tile j is in LDS, and the one before it is done with
      const int k0 = j * kKeys;
      const bool mine = heavy >> ((j - j_first) >> group) & 1;
      j = next(j + 1);
      if (j < n_tiles) copy(j, other);
      if (!mine) return;
#pragma unroll 1
      for (int x = 0; x < NU; ++x) {
        const int u = NU * split + x, kb = k0 + 32 * u;
        if (kb > q0) break;
        f32x16 s;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = minus_lse;
#pragma unroll
        for (int c = 0; c < DC; ++c) s = M::mma(frag_row<M, DP>(lk, 32 * u, 2 * c), q[c], s);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[e] = exp2_fast(s[e] * c2);
          if (kb == q0 && acc_row(e) + 4 * half > (lane & 31)) s[e] = 0.0f;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const typename M::V8 p = pack8<M>(s, c);
#pragma unroll
          for (int i = 0; i < DT; ++i) bar[i] = M::mma(frag_col<M, DP>(lk, 32 * u + 16 * c, 32 * i), p, bar[i]);
        }
      }
    };
    while (j < n_tiles) {
      again(lk0, lk1);
      if (j < n_tiles) again(lk1, lk0);
    }
    if (a.q_parts == 1) {
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] -= eps * bar[i][e];
    } else {
      if constexpr (kSplits > 1) join_splits(bar);
      if (split == 0 && qi < t.len) store_sums<DT>(a.q_bars + (part_row * a.heads + head) * width, bar, width);
    }
  }
  if constexpr (kSplits > 1) {
    join_splits(acc);
    if (split) return;
  }
  if (qi >= t.len) return;
  if (a.q_parts == 1)
    store_columns<M, DT>(static_cast<T*>(a.dq) + qr * a.dq_s[0] + head * a.dq_s[1], acc, a.scale, width);
  else
    store_sums<DT>(a.q_sums + (part_row * a.heads + head) * width, acc, width);
}

// -------------------------------------------------------------------- dk, dv --
// One workgroup: 128 keys (64 with two splits) of one kv head, over the query
// heads of its group in order and the query tiles from the diagonal on, or over
// one part of that list. Four products a block of 32 x 32: 8,192 x 16 heads of
// 64 295 to 313 us, 0.90 PFLOP/s; matrix units 43%, vector units 45%.
template <class M, int DP, int DW, int kSplits>
__global__ void __launch_bounds__(256, 2) at_dkv(const Attention a) {
  typedef typename M::T T;
  constexpr int DT = DW / 32, DC = DW / 16;
  constexpr int kStrips = 4 / kSplits, kRows = 32 * kStrips, kQs = 64;
  constexpr int kTileBytes = kQs * DP * 2;
  // buffers, apart by name so that a read waits for its own buffer's copies only
  __shared__ __align__(16) char lq0[kTileBytes], ld0[kTileBytes], lq1[kTileBytes], ld1[kTileBytes];
  uint32_t tile, kv;
  tile_and_head(row_block(), uint32_t(a.kv_heads * a.parts), &tile, &kv);
  const int which = int(kv) % a.parts;  // neighbours: the parts of a kv head
  kv /= uint32_t(a.parts);
  Tile t;
  if (!pick_tile<kRows, false>(a, tile, &t)) return;  // a sample's first keys are seen by most queries
  const int width = a.width;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, half = lane >> 5;
  const int strip = wave % kStrips, split = kSplits == 1 ? 0 : wave / kStrips;
  if (t.sample == a.n) {
    if (a.parts > 1) return;  // the sum of the parts has these rows
    const int rows = min(kRows, t.len - t.m0);
    zero_rows<M>(a.dk, a.dk_s, kv, t.begin + t.m0, rows, width);
    zero_rows<M>(a.dv, a.dv_s, kv, t.begin + t.m0, rows, width);
    return;
  }
  const int k0 = t.m0 + 32 * strip;
  const int ki = k0 + (lane & 31);  // the lane's key
  const int64_t kr = t.begin + min(ki, t.len - 1);
  const T* krow = static_cast<const T*>(a.k) + kr * a.k_s[0] + kv * a.k_s[1];
  const T* vrow = static_cast<const T*>(a.v) + kr * a.v_s[0] + kv * a.v_s[1];
  typename M::V8 k[DC], v[DC];
#pragma unroll
  for (int c = 0; c < DC; ++c) {
    k[c] = own_chunk<M>(krow, c, width);
    v[c] = own_chunk<M>(vrow, c, width);
  }
  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) dk[i][e] = dv[i][e] = 0.0f;
  const float c2 = a.scale * kLog2e, inv_scale = 1.0f / a.scale;

  // The key tile's query tiles: from the diagonal to the sample's end, for all
  // query heads of the group; this part has a run of them.
  const int group = a.heads / a.kv_heads;
  const int j0 = t.m0 / kQs, j1 = (t.len + kQs - 1) / kQs;
  const int64_t all = int64_t(j1 - j0) * group;
  const int i0 = int(all * which / a.parts), n_tiles = int(all * (which + 1) / a.parts) - i0;
  if (n_tiles == 0) {  // fewer tiles than parts: this one's sums are 0
    if (ki < t.len) store_dkv<M, DT>(a, kr, kv, which, 0, dk, dv);
    return;
  }
  const int lift =
      M::kNarrow ? ds_exponent(a, t, int64_t(kv) * group, j0, j1, i0, n_tiles, reinterpret_cast<float*>(lq0)) : 0;
  const float lift_ds = __builtin_ldexpf(1.0f, lift - kLiftP);  // of dS with P's
  const TileCopy<DP, kQs> cq(a.q_s[0], width), cd(a.do_s[0], width);
  // the tile copied next: query head and tile of the sample
  int64_t h_next = int64_t(kv) * group + i0 / (j1 - j0);
  int j_next = j0 + i0 % (j1 - j0);
  int q0 = j_next * kQs;
  auto copy = [&](char* lq, char* ld, f32x2& stat) {
    const int row0 = j_next * kQs;
    const int64_t at = h_next * a.T + t.begin + min(row0 + lane, t.len - 1);
    stat = f32x2{a.lse[at], a.delta[at]};  // of row `lane` of the tile
    cq.copy(reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (t.begin + row0) * a.q_s[0] + h_next * a.q_s[1]),
            t.len - row0, lq);
    cd.copy(reinterpret_cast<const char*>(static_cast<const T*>(a.d_o) + (t.begin + row0) * a.do_s[0] + h_next * a.do_s[1]),
            t.len - row0, ld);
    if (++j_next == j1) {
      j_next = j0;
      ++h_next;
    }
  };
  if (width < DP) {
    cq.zero_pad(lq0);
    cq.zero_pad(lq1);
    cd.zero_pad(ld0);
    cd.zero_pad(ld1);
  }
  f32x2 stat0, stat1;
  copy(lq0, ld0, stat0);
  auto step = [&](int i, const char* lq, const char* ld, const f32x2& stat, char* next_q, char* next_d,
                  f32x2& next_stat) {
    meet<0>();  // tile i is in LDS, and tile i - 1 is done with
    if (i + 1 < n_tiles) copy(next_q, next_d, next_stat);
    const int row0 = q0;
    q0 = q0 + kQs < t.len ? q0 + kQs : j0 * kQs;
#pragma unroll 1
    for (int u = split; u < kQs / 32; u += kSplits) {
      if (row0 + 32 * u < k0) continue;  // all earlier than this wave's keys
      __builtin_amdgcn_s_setprio(1);
      f32x16 s = minus_rows(stat[0] * inv_scale, u), dp = minus_rows(stat[1], u);
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        s = M::mma(frag_row<M, DP>(lq, 32 * u, 2 * c), k[c], s);
        dp = M::mma(frag_row<M, DP>(ld, 32 * u, 2 * c), v[c], dp);
      }
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = exp2_fast(M::kNarrow ? fmaf(s[r], c2, float(kLiftP)) : s[r] * c2);
        dp[r] *= M::kNarrow ? s[r] * lift_ds : s[r];
      }
      if (row0 + 32 * u == k0) {  // the diagonal: both are multiples of 32
  #pragma unroll
        for (int r = 0; r < 16; ++r)
          if (acc_row(r) + 4 * half < (lane & 31)) s[r] = dp[r] = 0.0f;
      }
      if (row0 + 32 * u + 32 > t.len) {  // rows past the end
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (row0 + 32 * u + acc_row(r) + 4 * half >= t.len) s[r] = dp[r] = 0.0f;
      }
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const typename M::V8 p = pack8<M>(s, c);
        const typename M::V8 g = pack8<M>(dp, c);
#pragma unroll
        for (int x = 0; x < DT; ++x) {
          dv[x] = M::mma(frag_col<M, DP>(ld, 32 * u + 16 * c, 32 * x), p, dv[x]);
          dk[x] = M::mma(frag_col<M, DP>(lq, 32 * u + 16 * c, 32 * x), g, dk[x]);
        }
      }
      __builtin_amdgcn_s_setprio(0);
    }
  };
  for (int i = 0; i < n_tiles; i += 2) {
    step(i, lq0, ld0, stat0, lq1, ld1, stat1);
    if (i + 1 < n_tiles) step(i + 1, lq1, ld1, stat1, lq0, ld0, stat0);
  }
  if constexpr (M::kNarrow) {
    scale_sums<DT>(dk, __builtin_ldexpf(1.0f, -lift));
    scale_sums<DT>(dv, __builtin_ldexpf(1.0f, -kLiftP));
  }
  if constexpr (kSplits == 2) {
    __syncthreads();
    char* pk = strip ? lq1 : lq0;
    char* pv = strip ? ld1 : ld0;
    if (split) {
      give_columns<DT>(pk, dk);
      give_columns<DT>(pv, dv);
    }
    __syncthreads();
    if (split) return;
    take_columns<DT>(pk, dk, 1.0f, 1.0f);
    take_columns<DT>(pv, dv, 1.0f, 1.0f);
  }
  if (ki < t.len) store_dkv<M, DT>(a, kr, kv, which, 0, dk, dv);
}

// The same for heads of more than 64 elements, where a wave's own rows and
// sums of 32 keys (K, V: 64 registers, dk, dv: 128) leave no room for a second
// wave on the SIMD. One workgroup: 64 keys, in two strips of 32; two waves
// share a strip. In a tile of 64 queries each makes P and dS of 32 of them,
// hands them to the other through LDS (as the operands they are, 16 bytes a
// lane), and then sums one half of the head's elements over all 64: half the
// sums per wave, and two workgroups share a compute unit. Their LDS is exactly
// half of it, so lse and delta stay in registers, one row per lane. 8,192 x 16
// heads of 128: 600 us, 0.92 PFLOP/s (876 with a strip per wave); the meeting
// of the waves between the two phases is what it waits for. 16,384 tokens of 32
// documents: 183 to 205 us, 534 MB read behind the L2s, where the arrays hold 168:
// each key tile of a sample goes through its queries from another one on.
template <class M, int DW>
__global__ void __launch_bounds__(256, 2) at_dkv_wide(const Attention a) {
  typedef typename M::T T;
  typedef typename M::V8 V8;
  constexpr int DP = 128, DC = DW / 16, kRows = 64, kQs = 64;
  constexpr int kTileBytes = kQs * DP * 2;
  __shared__ __align__(16) char lq0[kTileBytes], ld0[kTileBytes], lq1[kTileBytes], ld1[kTileBytes];
  __shared__ __align__(16) char lx[4 * 4096];  // P and dS: 4 operands of every wave
  uint32_t tile, kv;
  tile_and_head(row_block(), uint32_t(a.kv_heads * a.parts), &tile, &kv);
  const int which = int(kv) % a.parts;  // neighbours: the parts of a kv head
  kv /= uint32_t(a.parts);
  Tile t;
  if (!pick_tile<kRows, false>(a, tile, &t)) return;
  const int width = a.width;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, half = lane >> 5;
  const int strip = wave & 1, part = wave >> 1;
  if (t.sample == a.n) {
    if (a.parts > 1) return;  // the sum of the parts has these rows
    const int rows = min(kRows, t.len - t.m0);
    zero_rows<M>(a.dk, a.dk_s, kv, t.begin + t.m0, rows, width);
    zero_rows<M>(a.dv, a.dv_s, kv, t.begin + t.m0, rows, width);
    return;
  }
  const int k0 = t.m0 + 32 * strip;
  const int ki = k0 + (lane & 31);  // the lane's key
  const int64_t kr = t.begin + min(ki, t.len - 1);
  const T* krow = static_cast<const T*>(a.k) + kr * a.k_s[0] + kv * a.k_s[1];
  const T* vrow = static_cast<const T*>(a.v) + kr * a.v_s[0] + kv * a.v_s[1];
  V8 k[DC], v[DC];
#pragma unroll
  for (int c = 0; c < DC; ++c) {
    k[c] = own_chunk<M>(krow, c, width);
    v[c] = own_chunk<M>(vrow, c, width);
  }
  f32x16 dk[2], dv[2];  // elements 64 part .. 64 part + 63
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) dk[i][e] = dv[i][e] = 0.0f;
  const float c2 = a.scale * kLog2e, inv_scale = 1.0f / a.scale;

  const int group = a.heads / a.kv_heads;
  const int j0 = t.m0 / kQs, j1 = (t.len + kQs - 1) / kQs;
  const int64_t all = int64_t(j1 - j0) * group;
  const int i0 = int(all * which / a.parts), n_tiles = int(all * (which + 1) / a.parts) - i0;
  if (n_tiles == 0) {  // fewer tiles than parts: this one's sums are 0
    if (ki < t.len) store_dkv<M, 2>(a, kr, kv, which, 64 * part, dk, dv);
    return;
  }
  const int lift =
      M::kNarrow ? ds_exponent(a, t, int64_t(kv) * group, j0, j1, i0, n_tiles, reinterpret_cast<float*>(lq0)) : 0;
  const float lift_ds = __builtin_ldexpf(1.0f, lift - kLiftP);  // of dS with P's
  const TileCopy<DP, kQs> cq(a.q_s[0], width), cd(a.do_s[0], width);
  int64_t h_next = int64_t(kv) * group + i0 / (j1 - j0);
  int j_next = j0 + i0 % (j1 - j0);
  int q0 = j_next * kQs;
  auto copy = [&](char* lq, char* ld, f32x2& stat) {
    const int row0 = j_next * kQs;
    const int64_t at = h_next * a.T + t.begin + min(row0 + lane, t.len - 1);
    stat = f32x2{a.lse[at], a.delta[at]};  // of row `lane` of the tile
    cq.copy(reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (t.begin + row0) * a.q_s[0] + h_next * a.q_s[1]),
            t.len - row0, lq);
    cd.copy(reinterpret_cast<const char*>(static_cast<const T*>(a.d_o) + (t.begin + row0) * a.do_s[0] + h_next * a.do_s[1]),
            t.len - row0, ld);
    if (++j_next == j1) {
      j_next = j0;
      ++h_next;
    }
  };
  if (width < DP) {
    cq.zero_pad(lq0);
    cq.zero_pad(lq1);
    cd.zero_pad(ld0);
    cd.zero_pad(ld1);
  }
  f32x2 stat0, stat1;
  copy(lq0, ld0, stat0);
  V8* const own = reinterpret_cast<V8*>(lx + (2 * strip + part) * 4096) + lane;
  const V8* const others = reinterpret_cast<const V8*>(lx + (2 * strip + 1 - part) * 4096) + lane;
  auto step = [&](int i, const char* lq, const char* ld, const f32x2& stat, char* next_q, char* next_d,
                  f32x2& next_stat) {
    meet<0>();  // tile i is in LDS, and tile i - 1 is done with
    if (i + 1 < n_tiles) copy(next_q, next_d, next_stat);
    const int row0 = q0;
    q0 = q0 + kQs < t.len ? q0 + kQs : j0 * kQs;
    // a block of 32 queries counts unless all are earlier than the strip's keys or past the end
    const bool on[2] = {row0 >= k0 && row0 < t.len, row0 + 32 >= k0 && row0 + 32 < t.len};
    V8 p[2], g[2];
    if (part ? on[1] : on[0]) {
      __builtin_amdgcn_s_setprio(1);  // the other wave of the SIMD fills in with its exponentials
      f32x16 s = minus_rows(stat[0] * inv_scale, part), dp = minus_rows(stat[1], part);
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        s = M::mma(frag_row<M, DP>(lq, 32 * part, 2 * c), k[c], s);
        dp = M::mma(frag_row<M, DP>(ld, 32 * part, 2 * c), v[c], dp);
      }
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = exp2_fast(M::kNarrow ? fmaf(s[r], c2, float(kLiftP)) : s[r] * c2);
        dp[r] *= M::kNarrow ? s[r] * lift_ds : s[r];
      }
      const int b0 = row0 + 32 * part;
      if (b0 == k0 || b0 + 32 > t.len) {  // the diagonal, or rows past the end
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = b0 + acc_row(r) + 4 * half;
          if (row < ki || row >= t.len) s[r] = dp[r] = 0.0f;
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        p[c] = pack8<M>(s, c);
        g[c] = pack8<M>(dp, c);
        own[64 * c] = p[c];
        own[64 * (2 + c)] = g[c];
      }
    }
    meet<63>();  // P and dS are in LDS; the next tile is still on its way
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int w = 0; w < 2; ++w) {  // the wave's own block, then the other's
      const int u = w == 0 ? part : 1 - part;
      if (!(u ? on[1] : on[0])) continue;
      if (w == 1) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          p[c] = others[64 * c];
          g[c] = others[64 * (2 + c)];
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int d0 = 64 * part + 32 * x;
          if (d0 >= DW) continue;
          dv[x] = M::mma(frag_col<M, DP>(ld, 32 * u + 16 * c, d0), p[c], dv[x]);
          dk[x] = M::mma(frag_col<M, DP>(lq, 32 * u + 16 * c, d0), g[c], dk[x]);
        }
    }
    __builtin_amdgcn_s_setprio(0);
  };
  for (int i = 0; i < n_tiles; i += 2) {
    step(i, lq0, ld0, stat0, lq1, ld1, stat1);
    if (i + 1 < n_tiles) step(i + 1, lq1, ld1, stat1, lq0, ld0, stat0);
  }
  if constexpr (M::kNarrow) {
    scale_sums<2>(dk, __builtin_ldexpf(1.0f, -lift));
    scale_sums<2>(dv, __builtin_ldexpf(1.0f, -kLiftP));
  }
  if (ki < t.len) store_dkv<M, 2>(a, kr, kv, which, 64 * part, dk, dv);
}

// Gradients from their parts' sums, four elements a thread: element i of
// [T][heads][width], the parts `stride` apart.
template <class M>
__device__ __forceinline__ void sum_parts(const Attention& a, const float* sums, int64_t stride, int parts, int64_t i,
                                          int heads, void* to, const int64_t* s, float f) {
  const int64_t rh = i / a.width;
  const int d = int(i - rh * a.width);
  const int64_t row = rh / heads, head = rh - row * heads;
  f32x4 x = {0, 0, 0, 0};
  if (row < sample_begin(a, a.n))
    for (int p = 0; p < parts; ++p) x += *reinterpret_cast<const f32x4*>(sums + p * stride + i);
  typename M::V4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = typename M::T(x[e] * f);
  *reinterpret_cast<typename M::V4*>(static_cast<typename M::T*>(to) + row * s[0] + head * s[1] + d) = v;
}
template <class M>
__global__ void __launch_bounds__(256) at_sum(const Attention a) {
  const int64_t size = a.T * a.kv_heads * a.width;
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (i >= size) return;
  sum_parts<M>(a, a.partial, 2 * size, a.parts, i, a.kv_heads, a.dk, a.dk_s, a.scale);
  sum_parts<M>(a, a.partial + size, 2 * size, a.parts, i, a.kv_heads, a.dv, a.dv_s, 1.0f);
}
// dq and delta from their parts.
template <class M>
__global__ void __launch_bounds__(256) at_sum_dq(const Attention a) {
  const int64_t size = a.T * a.heads * a.width;
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (i >= size) return;
  const int64_t rh = i / a.width;
  const int d = int(i - rh * a.width);
  const int64_t row = rh / a.heads, head = rh - row * a.heads;
  f32x4 x = {0, 0, 0, 0};
  if (row < sample_begin(a, a.n)) {
    const f32x2* st = a.q_stats + head * a.T + row;
    const int64_t step = a.heads * a.T;
    float eps = 0.0f;
    f32x4 bar = {0, 0, 0, 0};
    for (int p = 0; p < a.q_parts; ++p) {
      const f32x2 y = st[p * step];
      eps += y[0];
      x += *reinterpret_cast<const f32x4*>(a.q_sums + p * size + i);
      if (y[1] != 0.0f) bar += *reinterpret_cast<const f32x4*>(a.q_bars + p * size + i);
    }
    x -= eps * bar;
    if (d == 0) a.delta[head * a.T + row] += eps;
  }
  typename M::V4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = typename M::T(x[e] * a.scale);
  *reinterpret_cast<typename M::V4*>(static_cast<typename M::T*>(a.dq) + row * a.dq_s[0] + head * a.dq_s[1] + d) = v;
}

// --------------------------------------------------------------------- host --
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int check_array(const char* name, const void* p, const int64_t* s, int64_t heads, int64_t width) {
  if (!p) return fail(NOPFS_EINVAL, std::string(name) + " must be non-NULL");
  if (!aligned16(p) || (s[0] & 7) || (s[1] & 7))
    return fail(NOPFS_EINVAL, std::string(name) + " and its strides must be multiples of 16 bytes");
  if (s[0] < width || (heads > 1 && s[1] < width))
    return fail(NOPFS_EINVAL, std::string(name) + ": strides smaller than a head");
  if (s[0] > (int64_t(1) << 23) || s[1] > (int64_t(1) << 40))
    return fail(NOPFS_ERANGE, std::string(name) + ": the token stride must be <= 2^23, the head stride <= 2^40");
  return NOPFS_OK;
}

// Row tiles of `rows` rows at most, and the grid over them and the heads.
dim3 tile_grid(Attention* a, int rows, int32_t heads) {
  a->tiles = uint32_t(a->T / rows + a->n + 1);
  return row_grid(int64_t(a->tiles) * heads);
}

// The grid over [T][heads][width], 4 elements a thread.
dim3 sum_grid(const Attention& a, int32_t heads) { return dim3(uint32_t(ceil_div(a.T * heads * a.width / 4, 256))); }

int make_attention(const nopfs_attention* p, Attention* a) {
  if (!p) return fail(NOPFS_EINVAL, "attention is NULL");
  if (p->T < 0 || p->n < 0) return fail(NOPFS_EINVAL, "T and n must be >= 0");
  if (p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads)
    return fail(NOPFS_EINVAL, "heads must be a positive multiple of kv_heads");
  if (p->dtype != NOPFS_BF16 && p->dtype != NOPFS_FP16)
    return fail(NOPFS_EINVAL, "dtype must be NOPFS_BF16 or NOPFS_FP16");
  if (p->width < 8 || (p->width & 7)) return fail(NOPFS_EINVAL, "width must be a positive multiple of 8");
  if (p->width > 128) return fail(NOPFS_ERANGE, "width must be <= 128");
  if (!(p->scale > 0.0f) || !isfinite(p->scale))
    return fail(NOPFS_EINVAL, "scale must be positive and finite");
  // 1 / scale and the rows' lse in units of it stay finite
  if (p->scale < 0x1p-60f || p->scale > 0x1p60f) return fail(NOPFS_ERANGE, "scale must be in 2^-60 .. 2^60");
  if (p->T >= (int64_t(1) << 31) - 128 || p->n > (1 << 30))
    return fail(NOPFS_ERANGE, "T must be < 2^31 - 128, n <= 2^30");
  if ((p->T / 32 + p->n + 1) * p->heads >= (int64_t(1) << 31))  // the largest grid
    return fail(NOPFS_ERANGE, "too many rows, samples and heads for one call");
  a->T = p->T;
  a->n = p->n;
  a->heads = p->heads;
  a->kv_heads = p->kv_heads;
  a->width = p->width;
  a->scale = p->scale;
  for (int i = 0; i < 2; ++i) {
    a->q_s[i] = p->q_stride[i];
    a->k_s[i] = p->k_stride[i];
    a->v_s[i] = p->v_stride[i];
    a->o_s[i] = p->o_stride[i];
    a->do_s[i] = p->do_stride[i];
    a->dq_s[i] = p->dq_stride[i];
    a->dk_s[i] = p->dk_stride[i];
    a->dv_s[i] = p->dv_stride[i];
  }
  return NOPFS_OK;
}

// Splits of the other side: one where that fills the chip with two workgroups
// a compute unit, else two (5,003 tokens x 6 heads of 80 forward 26.2 -> 20.6
// us, 16,384 x 16 of 128 99 -> 131), and four for few, long samples (2,048 x 8
// of 64 24.3 -> 19.1, 3,000 x 2 of 128 27.0 -> 24.4; 1,000 tokens of four
// samples x 8 of 128 14.2 -> 17.5), as long as their workgroups run at once:
// two a compute unit, or one where LDS rows hold 128 elements.
template <int DP>
int splits_of(const Attention& a, int32_t heads) {
  if ((a.T / 128 + 1) * heads >= 512) return 1;
  const bool few = (a.T / 32 + 1) * heads <= (DP == 64 ? 640 : 320);
  return few && a.n > 0 && a.T / a.n >= 512 ? 4 : 2;
}

// An order by cost is worth its launch (4 us) where samples of several tiles
// differ: 32 documents of 16,384 tokens, forward 127 -> 99 us. A single sample
// is in order by itself, and samples below a tile all cost the same.
bool needs_order(const Attention& a) { return a.n > 1 && a.T >= 4096 && a.T / a.n >= 64; }

// Parts of a query tile's keys for o and dq, where few rows and heads leave the
// longest sample's last tiles alone on the chip (its length guessed as in
// dkv_parts): 24 key tiles or more a part, since a launch that joins them
// follows (9 to 18 us). Forward and dq, joined: 7,825 tokens of three samples x
// 3 heads of 80 161 -> 110 us, 5,000 x 4 of 128 173 -> 134, 16,000 x 2 of 64
// 345 -> 255; like samples, for which the guess is too long, lose: three of 2,048 x
// 8 of 128 107 -> 142, four 122 -> 144. In parts of 12 tiles 4,096 tokens of 8
// samples x 8 of 128 took 78 for 46.
int32_t q_parts(const Attention& a) {
  const int64_t rows = a.T * a.heads;
  const int64_t longest = a.n > 4 ? 4 * a.T / a.n : a.T;
  const int64_t most = (longest / 64 + 1) / 24;
  return int32_t(std::max<int64_t>(1, std::min(ceil_div(81920, rows), most)));
}

template <class M, int DP, int DW>
int launch_forward(Attention a, hipStream_t st) {
  const int splits = splits_of<DP>(a, a.heads * a.q_parts);
  const dim3 grid = tile_grid(&a, 128 / splits, a.heads * a.q_parts);
  int rc;
  Scratch sc(st);
  if (a.q_parts > 1) {
    if ((rc = step_alloc(&sc, &a.q_sums, size_t(a.q_parts) * size_t(a.T) * size_t(a.heads) * size_t(a.width))))
      return rc;
    if ((rc = step_alloc(&sc, &a.q_stats, size_t(a.q_parts) * size_t(a.T) * size_t(a.heads)))) return rc;
  }
  if (needs_order(a)) {
    OrderJob j{nullptr, a.tiles, __builtin_ctz(128 / splits), true};
    if ((rc = step_alloc(&sc, &j.order, a.tiles))) return rc;
    if ((rc = launch("at_order", at_order, dim3(1), dim3(1024), 0, st, a, j, j))) return rc;
    a.order = j.order;
  }
  const auto kernel = splits == 1 ? at_forward<M, DP, DW, 1> : splits == 2 ? at_forward<M, DP, DW, 2> : at_forward<M, DP, DW, 4>;
  rc = launch("at_forward", kernel, grid, dim3(256), 0, st, a);
  if (rc || a.q_parts == 1) return rc;
  return launch("at_join", at_join<M>, sum_grid(a, a.heads), dim3(256), 0, st, a);
}

// Products run over the head's elements rounded up to 32; LDS rows hold 64 or
// 128 of them, the rest of a row is 0.
template <class M>
int launch_forward(const Attention& a, hipStream_t st) {
  if (a.width <= 32) return launch_forward<M, 64, 32>(a, st);
  if (a.width <= 64) return launch_forward<M, 64, 64>(a, st);
  if (a.width <= 96) return launch_forward<M, 128, 96>(a, st);
  return launch_forward<M, 128, 128>(a, st);
}

int attention_impl(const nopfs_attention* p, const void* q, const void* k, const void* v,
                   const int32_t* start, void* o, float* lse, hipStream_t st) {
  Attention a = {};
  int rc = make_attention(p, &a);
  if (rc) return rc;
  if (a.T == 0) return NOPFS_OK;
  if ((rc = check_array("q", q, a.q_s, a.heads, a.width))) return rc;
  if ((rc = check_array("k", k, a.k_s, a.kv_heads, a.width))) return rc;
  if ((rc = check_array("v", v, a.v_s, a.kv_heads, a.width))) return rc;
  if ((rc = check_array("o", o, a.o_s, a.heads, a.width))) return rc;
  if (!start || !lse) return fail(NOPFS_EINVAL, "start and lse must be non-NULL");
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.lse = lse;
  a.start = start;
  a.q_parts = q_parts(a);
  return p->dtype == NOPFS_BF16 ? launch_forward<MBf16>(a, st) : launch_forward<MFp16>(a, st);
}

// Parts of a key tile's queries for dk and dv. Its workgroup goes through its
// sample's later queries of all heads of the group, one tile after the other:
// with few key tiles, or long ones among short, the longest holds up the call.
// The lengths are not known here; the longest sample is taken for four times
// the mean. Parts of 8 tiles or more (the parts' sums cost 8 bytes an element
// and part, written and read), as many as keep the longest workgroup below the
// chip's average load, more of them where lengths differ and fewer where all
// samples are short. 7,825 tokens of three samples x 3 heads: 144 -> 80 us,
// 5,000 x 4 heads on 1: 151 -> 99, 16,384 tokens of 32 documents x 16 on 4:
// 311 -> 239; 4,096 tokens of 8 like samples x 8 stay whole (35 us, 55 in two).
int32_t dkv_parts(const Attention& a) {
  const int64_t group = a.heads / a.kv_heads, rows = a.T * a.kv_heads;
  const int64_t longest = a.n > 4 ? 4 * a.T / a.n : a.T;
  const int64_t load = longest * group < 4096 ? 32768 : a.n > 1 ? 81920 : 65536;
  const int64_t want = ceil_div(load, rows);
  const int64_t most = (longest / 64 + 1) * group / 8;
  return int32_t(std::max<int64_t>(1, std::min(want, most)));
}

template <class M, int DP, int DW>
int launch_grad(Attention a, hipStream_t st) {
  const int splits = splits_of<DP>(a, a.heads * a.q_parts);
  const bool two_k = DP == 128 || splits_of<DP>(a, a.kv_heads * a.parts) > 1;
  int rc;
  Scratch sc(st);
  if (M::kNarrow) {
    a.tops_of = splits * a.q_parts;
    if ((rc = step_alloc(&sc, &a.tops, size_t(a.tops_of) * size_t(a.heads) * size_t(a.T)))) return rc;
  }
  Attention ak = a;
  const dim3 gq = tile_grid(&a, 128 / splits, a.heads * a.q_parts);
  const dim3 gk = tile_grid(&ak, two_k ? 64 : 128, a.kv_heads * a.parts);
  if (needs_order(a)) {
    OrderJob jq{nullptr, a.tiles, __builtin_ctz(128 / splits), true}, jk{nullptr, ak.tiles, two_k ? 6 : 7, false};
    if ((rc = step_alloc(&sc, &jq.order, a.tiles))) return rc;
    if ((rc = step_alloc(&sc, &jk.order, ak.tiles))) return rc;
    if ((rc = launch("at_order", at_order, dim3(2), dim3(1024), 0, st, a, jq, jk))) return rc;
    a.order = jq.order;
    ak.order = jk.order;
  }
  const auto dq = splits == 1 ? at_dq<M, DP, DW, 1> : splits == 2 ? at_dq<M, DP, DW, 2> : at_dq<M, DP, DW, 4>;
  if ((rc = launch("at_dq", dq, gq, dim3(256), 0, st, a))) return rc;
  if (a.q_parts > 1 &&
      (rc = launch("at_sum_dq", at_sum_dq<M>, sum_grid(a, a.heads), dim3(256), 0, st, a)))
    return rc;
  if constexpr (DP == 128) {
    rc = launch("at_dkv", at_dkv_wide<M, DW>, gk, dim3(256), 0, st, ak);
  } else {
    rc = two_k ? launch("at_dkv", at_dkv<M, DP, DW, 2>, gk, dim3(256), 0, st, ak)
               : launch("at_dkv", at_dkv<M, DP, DW, 1>, gk, dim3(256), 0, st, ak);
  }
  if (rc || a.parts == 1) return rc;
  return launch("at_sum", at_sum<M>, sum_grid(a, a.kv_heads), dim3(256), 0, st, ak);
}

template <class M>
int launch_grad(const Attention& a, hipStream_t st) {
  if (a.width <= 32) return launch_grad<M, 64, 32>(a, st);
  if (a.width <= 64) return launch_grad<M, 64, 64>(a, st);
  if (a.width <= 96) return launch_grad<M, 128, 96>(a, st);
  return launch_grad<M, 128, 128>(a, st);
}

int attention_grad_impl(const nopfs_attention* p, const void* d_o, const void* q, const void* k,
                        const void* v, const void* o, const float* lse, const int32_t* start, void* dq,
                        void* dk, void* dv, hipStream_t st) {
  Attention a = {};
  int rc = make_attention(p, &a);
  if (rc) return rc;
  if (a.scale > 0x1p10f)  // lse in 32 bits says too little of the softmax
    return fail(NOPFS_ERANGE, "the gradient's scale must be <= 2^10");
  if (a.T == 0) return NOPFS_OK;
  if ((rc = check_array("q", q, a.q_s, a.heads, a.width))) return rc;
  if ((rc = check_array("k", k, a.k_s, a.kv_heads, a.width))) return rc;
  if ((rc = check_array("v", v, a.v_s, a.kv_heads, a.width))) return rc;
  if ((rc = check_array("o", o, a.o_s, a.heads, a.width))) return rc;
  if ((rc = check_array("do", d_o, a.do_s, a.heads, a.width))) return rc;
  if ((rc = check_array("dq", dq, a.dq_s, a.heads, a.width))) return rc;
  if ((rc = check_array("dk", dk, a.dk_s, a.kv_heads, a.width))) return rc;
  if ((rc = check_array("dv", dv, a.dv_s, a.kv_heads, a.width))) return rc;
  if (!start || !lse) return fail(NOPFS_EINVAL, "start and lse must be non-NULL");
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = const_cast<void*>(o);
  a.lse = const_cast<float*>(lse);
  a.d_o = d_o;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.start = start;
  Scratch sc(st);
  if ((rc = step_alloc(&sc, &a.delta, size_t(a.heads) * size_t(a.T)))) return rc;
  a.q_parts = q_parts(a);
  if (a.q_parts > 1) {
    const size_t rows = size_t(a.q_parts) * size_t(a.T) * size_t(a.heads);
    if ((rc = step_alloc(&sc, &a.q_sums, rows * size_t(a.width)))) return rc;
    if ((rc = step_alloc(&sc, &a.q_bars, rows * size_t(a.width)))) return rc;
    if ((rc = step_alloc(&sc, &a.q_stats, rows))) return rc;
  }
  a.parts = dkv_parts(a);
  if (a.parts > 1 &&
      (rc = step_alloc(&sc, &a.partial, size_t(2 * a.parts) * size_t(a.T) * size_t(a.kv_heads) * size_t(a.width))))
    return rc;
  return p->dtype == NOPFS_BF16 ? launch_grad<MBf16>(a, st) : launch_grad<MFp16>(a, st);
}

}  // namespace
}  // namespace nopfs

using namespace nopfs;

extern "C" int nopfs_packed_attention(const nopfs_attention* a, const void* q, const void* k, const void* v,
                                      const int32_t* start, void* o, float* lse, void* hip_stream) {
  try {
    auto call = [&]() { return attention_impl(a, q, k, v, start, o, lse, static_cast<hipStream_t>(hip_stream)); };
    return a ? run_with_scratch(a->scratch, a->scratch_bytes, call) : call();
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_packed_attention_grad(const nopfs_attention* a, const void* d_o, const void* q,
                                           const void* k, const void* v, const void* o, const float* lse,
                                           const int32_t* start, void* dq, void* dk, void* dv,
                                           void* hip_stream) {
  try {
    auto call = [&]() {
      return attention_grad_impl(a, d_o, q, k, v, o, lse, start, dq, dk, dv, static_cast<hipStream_t>(hip_stream));
    };
    return a ? run_with_scratch(a->scratch, a->scratch_bytes, call) : call();
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_packed_attention_scratch(const nopfs_attention* a, int32_t gradient, int64_t* bytes) {
  try {
    void* x = no_array();
    return scratch_size(bytes, [&]() {
      return gradient ? attention_grad_impl(a, x, x, x, x, x, static_cast<float*>(x), static_cast<int32_t*>(x), x, x, x,
                                            nullptr)
                      : attention_impl(a, x, x, x, static_cast<int32_t*>(x), x, static_cast<float*>(x), nullptr);
    });
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}
