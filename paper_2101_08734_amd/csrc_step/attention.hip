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
// kernel) and holds its own rows of the operands in registers for the whole
// pass; tiles of the other side (64 keys, or 32 queries) pass through LDS,
// double buffered, the next tile's global loads in flight meanwhile.
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
// matrix operands); everything else is rounded once, at the store.
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
  static __device__ __forceinline__ f32x16 mma(V8 a, V8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
struct MFp16 {
  typedef _Float16 T;
  typedef _Float16 V8 __attribute__((ext_vector_type(8)));
  typedef _Float16 V4 __attribute__((ext_vector_type(4)));
  typedef _Float16 V2 __attribute__((ext_vector_type(2)));
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
  const int32_t* start;
  uint32_t tiles;  // an upper bound of the row tiles
};

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

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
// sample. Returns false where the tile's number belongs to no row.
struct Tile {
  int32_t sample;   // n: the rows of no sample
  int64_t begin;    // the sample's first row
  int32_t len, m0;  // its rows, and the tile's first row in it
};
template <int BM>
__device__ inline bool find_tile(const Attention& a, uint32_t tile, Tile* t) {
  const int lane = __lane_id();
  auto at = [&](int32_t s) -> int64_t {
    int64_t v = s <= 0 ? 0 : a.start[s];
    return v < 0 ? 0 : (v > a.T ? a.T : v);
  };
  // the last s in [lo, hi] whose number is <= tile, 64 candidates at a time
  int32_t lo = 0, hi = a.n;
  while (hi > lo) {
    const int32_t step = (hi - lo + 63) >> 6;  // candidates lo + step * (lane + 1)
    const int64_t cand = int64_t(lo) + int64_t(step) * (lane + 1);
    const bool le = cand <= hi && at(int32_t(cand)) / BM + cand <= int64_t(tile);
    const int k = __popcll(__ballot(le));  // monotone: the first k hold
    const int64_t top = int64_t(lo) + int64_t(step) * (k + 1) - 1;
    lo += step * k;
    hi = top < hi ? int32_t(top) : hi;
  }
  t->sample = lo;
  t->begin = at(lo);
  const int64_t end = lo < a.n ? at(lo + 1) : a.T;
  t->len = int32_t(end > t->begin ? end - t->begin : 0);
  const int64_t m0 = (int64_t(tile) - (t->begin / BM + lo)) * BM;
  t->m0 = int32_t(m0);
  return m0 >= 0 && m0 < t->len;
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

// This wave's copies into LDS have landed; with the barrier, every wave's.
__device__ __forceinline__ void copies_landed() {
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  __syncthreads();
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

template <class M>
__device__ inline void zero_rows(void* base, const int64_t* s, int64_t head, int64_t row0, int rows, int width) {
  const int per = width / 8;
  for (int i = threadIdx.x; i < rows * per; i += 256) {
    typename M::T* p = static_cast<typename M::T*>(base) + (row0 + i / per) * s[0] + head * s[1] + (i % per) * 8;
    *reinterpret_cast<u32x4*>(p) = u32x4{0, 0, 0, 0};
  }
}

constexpr int kRows = 128;  // columns of a workgroup: 32 per wave
constexpr int kKeys = 64;   // keys of a tile (forward, dq)
constexpr int kQs = 64;     // queries of a tile (dk, dv)

// ------------------------------------------------------------------ forward --
template <class M, int DP>
__global__ void __launch_bounds__(256, 2) at_forward(const Attention a) {
  typedef typename M::T T;
  constexpr int DT = DP / 32, DC = DP / 16;
  constexpr int kTileBytes = kKeys * DP * 2;
  // two buffers, apart by name so that a read waits for its own buffer's copies only
  __shared__ __align__(16) char lk0[kTileBytes], lv0[kTileBytes], lk1[kTileBytes], lv1[kTileBytes];
  const uint32_t id = xcd_logical(blockIdx.x, gridDim.x);
  const uint32_t head = id / a.tiles;
  if (head >= uint32_t(a.heads)) return;
  Tile t;
  // the last tiles of the packed rows first: long samples' last rows see most keys
  if (!find_tile<kRows>(a, a.tiles - 1 - id % a.tiles, &t)) return;
  const int width = a.width;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, half = lane >> 5;
  T* o = static_cast<T*>(a.o) + t.begin * a.o_s[0] + head * a.o_s[1];
  float* lse = a.lse + int64_t(head) * a.T + t.begin;
  if (t.sample == a.n) {
    const int rows = min(kRows, t.len - t.m0);
    zero_rows<M>(a.o, a.o_s, head, t.begin + t.m0, rows, width);
    for (int i = threadIdx.x; i < rows; i += 256) lse[t.m0 + i] = -INFINITY;
    return;
  }
  const int64_t kv = head / (a.heads / a.kv_heads);
  const T* kb = static_cast<const T*>(a.k) + t.begin * a.k_s[0] + kv * a.k_s[1];
  const T* vb = static_cast<const T*>(a.v) + t.begin * a.v_s[0] + kv * a.v_s[1];
  const int q0 = t.m0 + 32 * wave;  // the wave's first query
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
  const float c2 = a.scale * kLog2e;

  const int n_tiles = (min(t.len, t.m0 + kRows) + kKeys - 1) / kKeys;
  const TileCopy<DP, kKeys> ck(a.k_s[0], width), cv(a.v_s[0], width);
  const char* kt = reinterpret_cast<const char*>(kb);
  const char* vt = reinterpret_cast<const char*>(vb);
  if (width < DP) {
    ck.zero_pad(lk0);
    ck.zero_pad(lk1);
    cv.zero_pad(lv0);
    cv.zero_pad(lv1);
  }
  ck.copy(kt, t.len, lk0);
  cv.copy(vt, t.len, lv0);
  auto step = [&](int j, const char* lk, const char* lv, char* next_k, char* next_v) {
    copies_landed();  // tile j is in LDS, and tile j - 1 is done with
    const int k0 = j * kKeys;
    if (j + 1 < n_tiles) {
      kt += int64_t(ck.stride) * kKeys;
      vt += int64_t(cv.stride) * kKeys;
      ck.copy(kt, t.len - k0 - kKeys, next_k);
      cv.copy(vt, t.len - k0 - kKeys, next_v);
    }
    if (k0 > q0 + 31) return;  // all later than this wave's queries
    f32x16 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[u][e] = 0.0f;
#pragma unroll
      for (int c = 0; c < DC; ++c) s[u] = M::mma(frag_row<M, DP>(lk, 32 * u, 2 * c), q[c], s[u]);
    }
    if (k0 + kKeys - 1 > q0) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (k0 + 32 * u + acc_row(e) + 4 * half > qi) s[u][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
    top = fmaxf(m, half_max(top));
    const float f = exp2_fast((m - top) * c2);
    m = top;
    l *= f;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][e] *= f;
    const float mc = m * c2;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[u][e] = exp2_fast(fmaf(s[u][e], c2, -mc));
        l += s[u][e];
      }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const typename M::V8 p = pack8<M>(s[u], c);
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[i] = M::mma(frag_col<M, DP>(lv, 32 * u + 16 * c, 32 * i), p, acc[i]);
      }
  };
  for (int j = 0; j < n_tiles; j += 2) {
    step(j, lk0, lv0, lk1, lv1);
    if (j + 1 < n_tiles) step(j + 1, lk1, lv1, lk0, lv0);
  }
  l = half_sum(l);
  if (qi < t.len) {
    store_columns<M, DT>(o + int64_t(qi) * a.o_s[0], acc, 1.0f / l, width);
    if (half == 0) lse[qi] = m * a.scale + logf(l);
  }
}

// ----------------------------------------------------------------------- dq --
// Also writes delta_i = do_i.o_i for the dk/dv kernel.
template <class M, int DP>
__global__ void __launch_bounds__(256, 2) at_dq(const Attention a) {
  typedef typename M::T T;
  constexpr int DT = DP / 32, DC = DP / 16;
  constexpr int kTileBytes = kKeys * DP * 2;
  __shared__ __align__(16) char lk0[kTileBytes], lv0[kTileBytes], lk1[kTileBytes], lv1[kTileBytes];
  const uint32_t id = xcd_logical(blockIdx.x, gridDim.x);
  const uint32_t head = id / a.tiles;
  if (head >= uint32_t(a.heads)) return;
  Tile t;
  if (!find_tile<kRows>(a, a.tiles - 1 - id % a.tiles, &t)) return;
  const int width = a.width;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, half = lane >> 5;
  if (t.sample == a.n) {
    zero_rows<M>(a.dq, a.dq_s, head, t.begin + t.m0, min(kRows, t.len - t.m0), width);
    return;
  }
  const int64_t kv = head / (a.heads / a.kv_heads);
  const T* kb = static_cast<const T*>(a.k) + t.begin * a.k_s[0] + kv * a.k_s[1];
  const T* vb = static_cast<const T*>(a.v) + t.begin * a.v_s[0] + kv * a.v_s[1];
  const int q0 = t.m0 + 32 * wave;
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
  const float c2 = a.scale * kLog2e, lc = a.lse[stat] * kLog2e;
  if (half == 0 && qi < t.len) a.delta[stat] = delta;

  f32x16 acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;

  const int n_tiles = (min(t.len, t.m0 + kRows) + kKeys - 1) / kKeys;
  const TileCopy<DP, kKeys> ck(a.k_s[0], width), cv(a.v_s[0], width);
  const char* kt = reinterpret_cast<const char*>(kb);
  const char* vt = reinterpret_cast<const char*>(vb);
  if (width < DP) {
    ck.zero_pad(lk0);
    ck.zero_pad(lk1);
    cv.zero_pad(lv0);
    cv.zero_pad(lv1);
  }
  ck.copy(kt, t.len, lk0);
  cv.copy(vt, t.len, lv0);
  auto step = [&](int j, const char* lk, const char* lv, char* next_k, char* next_v) {
    copies_landed();
    const int k0 = j * kKeys;
    if (j + 1 < n_tiles) {
      kt += int64_t(ck.stride) * kKeys;
      vt += int64_t(cv.stride) * kKeys;
      ck.copy(kt, t.len - k0 - kKeys, next_k);
      cv.copy(vt, t.len - k0 - kKeys, next_v);
    }
    if (k0 > q0 + 31) return;
    const bool edge = k0 + kKeys - 1 > q0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x16 s, dp;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = dp[e] = 0.0f;
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        s = M::mma(frag_row<M, DP>(lk, 32 * u, 2 * c), q[c], s);
        dp = M::mma(frag_row<M, DP>(lv, 32 * u, 2 * c), d[c], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = exp2_fast(fmaf(s[e], c2, -lc)) * (dp[e] - delta);
      if (edge) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (k0 + 32 * u + acc_row(e) + 4 * half > qi) s[e] = 0.0f;
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const typename M::V8 p = pack8<M>(s, c);
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[i] = M::mma(frag_col<M, DP>(lk, 32 * u + 16 * c, 32 * i), p, acc[i]);
      }
    }
  };
  for (int j = 0; j < n_tiles; j += 2) {
    step(j, lk0, lv0, lk1, lv1);
    if (j + 1 < n_tiles) step(j + 1, lk1, lv1, lk0, lv0);
  }
  if (qi < t.len)
    store_columns<M, DT>(static_cast<T*>(a.dq) + qr * a.dq_s[0] + head * a.dq_s[1], acc, a.scale, width);
}

// -------------------------------------------------------------------- dk, dv --
// One workgroup: 128 keys of one kv head, over the query heads of its group in
// order and over the query tiles from the diagonal on. Nothing is added to
// memory from two places, so the sums' order never changes.
template <class M, int DP>
__global__ void __launch_bounds__(256, 2) at_dkv(const Attention a) {
  typedef typename M::T T;
  constexpr int DT = DP / 32, DC = DP / 16;
  constexpr int kTileBytes = kQs * DP * 2;
  __shared__ __align__(16) char lq0[kTileBytes], ld0[kTileBytes], lq1[kTileBytes], ld1[kTileBytes];
  __shared__ __align__(16) float ls0[2 * kQs], ls1[2 * kQs];  // a tile's lse and delta
  const uint32_t id = xcd_logical(blockIdx.x, gridDim.x);
  const uint32_t kv = id / a.tiles;
  if (kv >= uint32_t(a.kv_heads)) return;
  Tile t;
  if (!find_tile<kRows>(a, id % a.tiles, &t)) return;  // a sample's first keys are seen by most queries
  const int width = a.width;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), lane = threadIdx.x & 63, half = lane >> 5;
  if (t.sample == a.n) {
    const int rows = min(kRows, t.len - t.m0);
    zero_rows<M>(a.dk, a.dk_s, kv, t.begin + t.m0, rows, width);
    zero_rows<M>(a.dv, a.dv_s, kv, t.begin + t.m0, rows, width);
    return;
  }
  const int k0 = t.m0 + 32 * wave;
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
  const float c2 = a.scale * kLog2e;

  const int group = a.heads / a.kv_heads;
  const int j0 = t.m0 / kQs;  // the first query tile that sees the tile's keys
  const int j1 = (t.len + kQs - 1) / kQs;
  const int n_tiles = (j1 - j0) * group;
  const TileCopy<DP, kQs> cq(a.q_s[0], width), cd(a.do_s[0], width);
  // the tile copied next: query head and tile of the sample
  int64_t h_next = int64_t(kv) * group;
  int j_next = j0;
  float stat = 0.0f;
  auto copy = [&](char* lq, char* ld) {
    const int row0 = j_next * kQs;
    cq.copy(reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (t.begin + row0) * a.q_s[0] + h_next * a.q_s[1]),
            t.len - row0, lq);
    cd.copy(reinterpret_cast<const char*>(static_cast<const T*>(a.d_o) + (t.begin + row0) * a.do_s[0] + h_next * a.do_s[1]),
            t.len - row0, ld);
    if (threadIdx.x < 2 * kQs) {
      const int row = row0 + int(threadIdx.x % kQs);
      const int64_t at = h_next * a.T + t.begin + min(row, t.len - 1);
      // past the end: an infinite lse makes P and dS exactly 0
      stat = threadIdx.x < kQs ? (row < t.len ? a.lse[at] * kLog2e : INFINITY) : a.delta[at];
    }
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
  copy(lq0, ld0);
  int q0 = t.m0;
  auto step = [&](int i, const char* lq, const char* ld, float* ls, char* next_q, char* next_d) {
    if (threadIdx.x < 2 * kQs) ls[threadIdx.x] = stat;
    copies_landed();
    if (i + 1 < n_tiles) copy(next_q, next_d);
    const int row0 = q0;
    q0 = q0 + kQs < t.len ? q0 + kQs : t.m0;
    if (row0 + kQs - 1 < k0) return;  // all earlier than this wave's keys
#pragma unroll 1
    for (int u = 0; u < kQs / 32; ++u) {
      f32x16 s, dp;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = dp[e] = 0.0f;
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        s = M::mma(frag_row<M, DP>(lq, 32 * u, 2 * c), k[c], s);
        dp = M::mma(frag_row<M, DP>(ld, 32 * u, 2 * c), v[c], dp);
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const f32x4 lc = *reinterpret_cast<const f32x4*>(ls + 32 * u + 8 * b + 4 * half);
        const f32x4 de = *reinterpret_cast<const f32x4*>(ls + kQs + 32 * u + 8 * b + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * b + e;
          s[r] = exp2_fast(fmaf(s[r], c2, -lc[e]));
          dp[r] = s[r] * (dp[r] - de[e]);
        }
      }
      if (row0 < k0 + 31) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (row0 + 32 * u + acc_row(r) + 4 * half < ki) s[r] = dp[r] = 0.0f;
      }
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
    }
  };
  for (int i = 0; i < n_tiles; i += 2) {
    step(i, lq0, ld0, ls0, lq1, ld1);
    if (i + 1 < n_tiles) step(i + 1, lq1, ld1, ls1, lq0, ld0);
  }
  if (ki < t.len) {
    store_columns<M, DT>(static_cast<T*>(a.dk) + kr * a.dk_s[0] + kv * a.dk_s[1], dk, a.scale, width);
    store_columns<M, DT>(static_cast<T*>(a.dv) + kr * a.dv_s[0] + kv * a.dv_s[1], dv, 1.0f, width);
  }
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
  if (p->T >= (int64_t(1) << 31) - kRows || p->n > (1 << 30))
    return fail(NOPFS_ERANGE, "T must be < 2^31 - 128, n <= 2^30");
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
  const int64_t tiles = p->T / kRows + p->n + 1;
  if (tiles * p->heads > (int64_t(1) << 31) - 16)
    return fail(NOPFS_ERANGE, "too many rows, samples and heads for one call");
  a->tiles = uint32_t(tiles);
  return NOPFS_OK;
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
  const dim3 grid(xcd_padded(a.tiles * uint32_t(a.heads)));
  const bool bf = p->dtype == NOPFS_BF16;
  if (a.width <= 64)
    return bf ? launch("at_forward", at_forward<MBf16, 64>, grid, dim3(256), 0, st, a)
              : launch("at_forward", at_forward<MFp16, 64>, grid, dim3(256), 0, st, a);
  return bf ? launch("at_forward", at_forward<MBf16, 128>, grid, dim3(256), 0, st, a)
            : launch("at_forward", at_forward<MFp16, 128>, grid, dim3(256), 0, st, a);
}

template <class M, int DP>
int launch_grad(const Attention& a, hipStream_t st) {
  int rc = launch("at_dq", at_dq<M, DP>, dim3(xcd_padded(a.tiles * uint32_t(a.heads))), dim3(256), 0, st, a);
  if (rc) return rc;
  return launch("at_dkv", at_dkv<M, DP>, dim3(xcd_padded(a.tiles * uint32_t(a.kv_heads))), dim3(256), 0, st, a);
}

int attention_grad_impl(const nopfs_attention* p, const void* d_o, const void* q, const void* k,
                        const void* v, const void* o, const float* lse, const int32_t* start, void* dq,
                        void* dk, void* dv, hipStream_t st) {
  Attention a = {};
  int rc = make_attention(p, &a);
  if (rc) return rc;
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
  if ((rc = sc.alloc_n(&a.delta, size_t(a.heads) * size_t(a.T)))) return rc;
  if (a.width <= 64)
    return p->dtype == NOPFS_BF16 ? launch_grad<MBf16, 64>(a, st) : launch_grad<MFp16, 64>(a, st);
  return p->dtype == NOPFS_BF16 ? launch_grad<MBf16, 128>(a, st) : launch_grad<MFp16, 128>(a, st);
}

}  // namespace
}  // namespace nopfs

using namespace nopfs;

extern "C" int nopfs_packed_attention(const nopfs_attention* a, const void* q, const void* k, const void* v,
                                      const int32_t* start, void* o, float* lse, void* hip_stream) {
  try {
    return attention_impl(a, q, k, v, start, o, lse, static_cast<hipStream_t>(hip_stream));
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_packed_attention_grad(const nopfs_attention* a, const void* d_o, const void* q,
                                           const void* k, const void* v, const void* o, const float* lse,
                                           const int32_t* start, void* dq, void* dk, void* dv,
                                           void* hip_stream) {
  try {
    return attention_grad_impl(a, d_o, q, k, v, o, lse, start, dq, dk, dv,
                               static_cast<hipStream_t>(hip_stream));
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}
