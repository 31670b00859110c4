// nopfs_token_embed and its gradient: the rows of an embedding that the packed
// tokens name, and the sums of their gradients by name.
//     out_t = scale W[id_t],   dW_v = scale sum_{t: id_t = v} dout_t
// Both are bound by memory (16,384 tokens by 2,048 from 32,768 rows, a twelfth of them
// the most frequent one, bf16: forward 26 us for 108 MB; the gradient's zeros and sums
// 41 us for 205). The gradient's sums must not depend on the order in which work
// finishes, so the tokens are sorted by id first (radix sort, stable; 16 us of four
// dependent launches there) and added in an order that the ids alone decide: as in the
// batch within a piece of the sorted tokens, then the pieces' parts of a name. Sums are
// in 32 bits, rounded once.
#include "rows.hpp"

namespace nopfs {
namespace {

struct Embed {
  int64_t T, V, n_ids, weight_stride, out_stride;
  int32_t width;
  float scale;
  const void* ids;
  const int64_t* slot;
  bool wide;
};

// The row of the embedding that token t names, -1 for padding.
__device__ __forceinline__ int64_t name_of(const Embed& d, int64_t t) {
  int64_t at = t;
  if (d.slot) {
    at = d.slot[t];
    if (at < 0 || at >= d.n_ids) return -1;
  }
  const int64_t id = d.wide ? static_cast<const int64_t*>(d.ids)[at] : static_cast<const int32_t*>(d.ids)[at];
  return id >= 0 && id < d.V ? id : -1;
}

constexpr int kVec = 8;  // elements per lane and step

// A lane's elements of a row begin at c, its last ones behind the row: they are then
// the row's last kVec (made and written by two lanes alike), so that rows of any width
// are read and written in whole vectors. Of less than kVec, `some`.
__device__ __forceinline__ int32_t in_row(int32_t c, int32_t width) {
  return c + kVec <= width ? c : width > kVec ? width - kVec : 0;
}

// Rows by groups of 2^lg lanes, kPer rows of a group at a time. `names`, if given, gets
// what each token names.
template <class W, class E, int kPer>
__global__ void __launch_bounds__(256) te_forward(const Embed d, const typename W::T* weight, typename E::T* out,
                                                  int32_t* names, int lg) {
  const int lanes = 1 << lg;
  const int64_t t0 = (int64_t(row_block()) * (256 >> lg) + (threadIdx.x >> lg)) * kPer;
  if (t0 >= d.T) return;
  int64_t id[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) id[j] = t0 + j < d.T ? name_of(d, t0 + j) : -1;
  if (names && (threadIdx.x & (lanes - 1)) == 0) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (t0 + j < d.T) names[t0 + j] = int32_t(id[j]);
  }
  const int some = d.width;
  for (int32_t c0 = int32_t(threadIdx.x & (lanes - 1)) * kVec; c0 < d.width; c0 += lanes * kVec) {
    const int32_t c = in_row(c0, d.width);
    Pack<W, kVec> w[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      w[j].zero();
      const typename W::T* p = weight + id[j] * d.weight_stride + c;
      if (id[j] >= 0) {
        if (some >= kVec) w[j].load(p);
        else w[j].load_some(p, some);
      }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (t0 + j >= d.T) break;
      float v[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = id[j] >= 0 ? w[j].get(e) * d.scale : 0.0f;
      Pack<E, kVec> o;
      o.set(v);
      typename E::T* p = out + (t0 + j) * d.out_stride + c;
      if (some >= kVec) o.store(p);
      else o.store_some(p, some);
    }
  }
}

// ---- the tokens in the order of their ids ------------------------------------
// Least significant digit first, at most 10 bits a pass: a tile's counts of each
// digit, then each tile's own place among them. The keys are the ids, V for
// padding, which so comes last.
constexpr int kMostBits = 10;
constexpr int kSortTile = 1024;

struct Sort {
  const uint32_t *key_in, *val_in;  // the pass before (not in the first)
  uint32_t *key, *val;
  uint32_t* hist;   // [tiles][1 << bits]
  uint8_t* named;   // [V]: some token names the row (cleared and set in the first pass)
  int32_t tiles, per_tile, shift, bits;
};

// `named`, 16 rows at a time (its memory ends at a multiple of 256 bytes).
__device__ __forceinline__ void clear_names(const Embed& d, const Sort& s, int64_t first, int64_t step) {
  for (int64_t v = first; v < (d.V + 15) >> 4; v += step) reinterpret_cast<u32x4*>(s.named)[v] = u32x4{0, 0, 0, 0};
}

template <bool kFirst>
__device__ __forceinline__ uint32_t sort_key(const Embed& d, const Sort& s, int64_t i) {
  if (!kFirst) return s.key_in[i];
  const int64_t id = name_of(d, i);
  return uint32_t(id >= 0 ? id : d.V);
}

template <bool kFirst>
__global__ void __launch_bounds__(256) te_count(const Embed d, const Sort s) {
  __shared__ uint32_t count[1 << kMostBits];
  const int bins = 1 << s.bits;
  if (kFirst) {
    clear_names(d, s, int64_t(blockIdx.x) * 256 + threadIdx.x, int64_t(gridDim.x) * 256);
    if (int64_t(blockIdx.x) >= s.tiles) return;  // is here for that alone
  }
  for (int b = threadIdx.x; b < bins; b += 256) count[b] = 0;
  __syncthreads();
  const int64_t i0 = int64_t(blockIdx.x) * s.per_tile;
  const int64_t i1 = i0 + s.per_tile < d.T ? i0 + s.per_tile : d.T;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += 256)
    atomicAdd(&count[sort_key<kFirst>(d, s, i) >> s.shift & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += 256) s.hist[int64_t(blockIdx.x) * bins + b] = count[b];
}

template <bool kFirst>
__device__ inline void scatter_tile(const Embed& d, const Sort& s, int32_t tile) {
  constexpr int kDeep = 16;  // counts in flight
  __shared__ uint32_t base[1 << kMostBits], cnt[4][1 << kMostBits], tmp[65];
  const int bins = 1 << s.bits, wave = threadIdx.x >> 6;
  uint32_t mine[(1 << kMostBits) / 256];  // of the digit, in the tiles before this one
#pragma unroll
  for (int j = 0; j < (1 << kMostBits) / 256; ++j) {
    const int b = j * 256 + threadIdx.x;
    if (b >= bins) break;
    uint32_t before = 0, all = 0;
    for (int32_t t = 0; t < s.tiles; t += kDeep) {
      uint32_t c[kDeep];
#pragma unroll
      for (int i = 0; i < kDeep; ++i) c[i] = t + i < s.tiles ? s.hist[int64_t(t + i) * bins + b] : 0;
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        before += t + i < tile ? c[i] : 0;
        all += c[i];
      }
    }
    mine[j] = before;
    base[b] = all;
#pragma unroll
    for (int w = 0; w < 4; ++w) cnt[w][b] = 0;
  }
  __syncthreads();
  block_scan_array(base, uint32_t(bins), tmp);
#pragma unroll
  for (int j = 0; j < (1 << kMostBits) / 256; ++j) {
    const int b = j * 256 + threadIdx.x;
    if (b < bins) base[b] += mine[j];
  }
  __syncthreads();
  const int64_t i0 = int64_t(tile) * s.per_tile;
  const int64_t i1 = i0 + s.per_tile < d.T ? i0 + s.per_tile : d.T;
  for (int64_t r = i0; r < i1; r += 256) {
    const int64_t i = r + threadIdx.x;
    const bool in = i < i1;
    const uint32_t key = in ? sort_key<kFirst>(d, s, i) : 0;
    const uint32_t digit = key >> s.shift & (bins - 1);
    uint64_t same = __ballot(in);  // the wave's lanes of the same digit
    for (int b = 0; b < s.bits; ++b) {
      const uint64_t ones = __ballot(digit >> b & 1);
      same &= digit >> b & 1 ? ones : ~ones;
    }
    const uint32_t rank = __popcll(same & lanemask_lt());
    const bool leads = in && rank == 0;
    if (leads) cnt[wave][digit] = __popcll(same);
    __syncthreads();
    if (in) {
      uint32_t at = base[digit] + rank;
      for (int w = 0; w < wave; ++w) at += cnt[w][digit];
      if (at < d.T) {  // ids that change under the call leave the counts behind, not the arrays
        s.key[at] = key;
        s.val[at] = kFirst ? uint32_t(i) : s.val_in[i];
      }
      if (kFirst && key < d.V) s.named[key] = 1;
    }
    __syncthreads();
    if (leads) {
      atomicAdd(&base[digit], cnt[wave][digit]);
      cnt[wave][digit] = 0;
    }
    __syncthreads();
  }
}

template <bool kFirst>
__global__ void __launch_bounds__(256) te_scatter(const Embed d, const Sort s) {
  scatter_tile<kFirst>(d, s, int32_t(blockIdx.x));
}

// All of it by one workgroup, for small batches: 8 bits a pass, a wave's keys one
// after the other in its own counts, so that the waves meet only between the passes.
// Bound by latency: 5,173 keys of 15 bits 17 us; forward and gradient of that batch
// (250 elements a row) took 33 us with it and 40 by the passes above.
constexpr int kSmallKeys = 6;  // of a thread
constexpr int64_t kSmallSort = 1024 * kSmallKeys, kSmallNames = 1 << 18;

__global__ void __launch_bounds__(1024) te_sort(const Embed d, const Sort s, int passes) {
  constexpr int kBins = 256, kWaves = 16;
  __shared__ uint32_t keys[kSmallSort], vals[kSmallSort], base[kBins], tmp[65];
  __shared__ uint16_t cnt[kWaves][kBins];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = int(d.T);
  const int rounds = (n + 1023) >> 10, first = wave * rounds * 64 + lane;  // the wave's keys: every 64th from here
  clear_names(d, s, tid, 1024);
  uint32_t key[kSmallKeys], val[kSmallKeys];
#pragma unroll
  for (int r = 0; r < kSmallKeys; ++r) {
    const int i = first + r * 64;
    key[r] = val[r] = 0;
    if (r < rounds && i < n) {
      const int64_t id = name_of(d, i);
      key[r] = uint32_t(id >= 0 ? id : d.V);
      val[r] = uint32_t(i);
    }
  }
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * 8;
    for (int i = tid; i < kWaves * kBins / 2; i += 1024) reinterpret_cast<uint32_t*>(cnt)[i] = 0;
    __syncthreads();
    uint32_t at[kSmallKeys];
#pragma unroll
    for (int r = 0; r < kSmallKeys; ++r) {
      if (r >= rounds) break;
      const bool in = first + r * 64 < n;
      const uint32_t digit = key[r] >> shift & (kBins - 1);
      uint64_t same = __ballot(in);
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const uint64_t ones = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? ones : ~ones;
      }
      const uint32_t rank = __popcll(same & lanemask_lt());
      at[r] = 0;
      if (in) at[r] = cnt[wave][digit] + rank;  // read by all of the digit before its first lane adds to it
      wave_step();
      if (in && rank == 0) cnt[wave][digit] = uint16_t(cnt[wave][digit] + __popcll(same));
      wave_step();
    }
    __syncthreads();
    if (tid < kBins) {  // a digit's counts before each wave, and in all
      uint32_t sum = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = cnt[w][tid];
        cnt[w][tid] = uint16_t(sum);
        sum += c;
      }
      base[tid] = sum;
    }
    __syncthreads();
    block_scan_array(base, kBins, tmp);
#pragma unroll
    for (int r = 0; r < kSmallKeys; ++r) {
      if (r < rounds && first + r * 64 < n) {
        const uint32_t digit = key[r] >> shift & (kBins - 1);
        const uint32_t to = base[digit] + cnt[wave][digit] + at[r];
        keys[to] = key[r];
        vals[to] = val[r];
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallKeys; ++r) {
      const int i = first + r * 64;
      if (r < rounds && i < n) key[r] = keys[i], val[r] = vals[i];
    }
  }
#pragma unroll
  for (int r = 0; r < kSmallKeys; ++r) {
    const int i = first + r * 64;
    if (r < rounds && i < n) {
      s.key[i] = key[r];
      s.val[i] = val[r];
      if (key[r] < d.V) s.named[key[r]] = 1;  // cleared before the barriers above
    }
  }
}

// Rows that no token names, kZeroRows by a group of 2^lg lanes.
constexpr int kZeroRows = 8;
template <class W>
__device__ inline void zero_rows(const Embed& d, const uint8_t* named, typename W::T* dw, int lg, int64_t block) {
  const int lanes = 1 << lg;
  const int64_t v0 = (block * (256 >> lg) + (threadIdx.x >> lg)) * kZeroRows;
  Pack<W, kVec> o;
  o.zero();
  for (int64_t v = v0; v < v0 + kZeroRows && v < d.V; ++v) {
    if (named[v]) continue;
    for (int32_t c = int32_t(threadIdx.x & (lanes - 1)) * kVec; c < d.width; c += lanes * kVec) {
      typename W::T* p = dw + v * d.weight_stride + in_row(c, d.width);
      if (d.width >= kVec) o.store(p);
      else o.store_some(p, d.width);
    }
  }
}
// The last of several passes has few workgroups, so the rows without a token go with
// it (`named` is whole since the first); after a single pass they go with te_pieces.
template <class W>
__global__ void __launch_bounds__(256) te_scatter_zero(const Embed d, const Sort s, typename W::T* dw, int lg) {
  const int64_t block = row_block();
  if (block < s.tiles) scatter_tile<false>(d, s, int32_t(block));
  else zero_rows<W>(d, s.named, dw, lg, block - s.tiles);
}

// ---- sums ------------------------------------------------------------------
// The sorted tokens are cut into pieces of equal size, however many of them share
// a name (a row of the embedding each: 1,114 us where this takes 100), by groups of
// 2^lg lanes. A name whose tokens lie in one piece has its row written from there; the
// others leave the sum of each piece's part, and te_join adds those up.
struct Pieces {
  const uint32_t *key, *val;
  float *head, *tail;  // [pieces][width]: of the name that goes on from the piece before; into the next
  int32_t per, n;      // tokens of a piece, pieces
};

template <class W>
__device__ __forceinline__ void store_row(const Embed& d, typename W::T* dw, uint32_t v, int32_t c, int some,
                                          float (&sum)[kVec]) {
#pragma unroll
  for (int e = 0; e < kVec; ++e) sum[e] *= d.scale;
  Pack<W, kVec> o;
  o.set(sum);
  typename W::T* p = dw + int64_t(v) * d.weight_stride + c;
  if (some >= kVec) o.store(p);
  else o.store_some(p, some);
}

template <class W, class E>
__global__ void __launch_bounds__(256) te_pieces(const Embed d, const Pieces s, const typename E::T* dout,
                                                 typename W::T* dw, int lg, uint32_t blocks, const uint8_t* named) {
  constexpr int kDeep = 8;  // rows in flight
  if (row_block() >= blocks) return zero_rows<W>(d, named, dw, lg, row_block() - blocks);
  const int lanes = 1 << lg;
  const int64_t piece = int64_t(row_block()) * (256 >> lg) + (threadIdx.x >> lg);
  if (piece >= s.n) return;
  const int64_t i0 = piece * s.per, i1 = i0 + s.per < d.T ? i0 + s.per : d.T;
  const uint32_t none = uint32_t(d.V);
  const uint32_t before = i0 > 0 ? s.key[i0 - 1] : none, behind = i1 < d.T ? s.key[i1] : none;
  const int some = d.width;
  for (int32_t c0 = int32_t(threadIdx.x & (lanes - 1)) * kVec; c0 < d.width; c0 += lanes * kVec) {
    const int32_t c = in_row(c0, d.width);
    float sum[kVec] = {};
    uint32_t name = s.key[i0];
    bool from_before = name == before;
    auto flush = [&](bool goes_on) {
      if (name >= none) return;
      if (!from_before && !goes_on) return store_row<W>(d, dw, name, c, some, sum);
      float* p = (from_before ? s.head : s.tail) + piece * d.width + c;
      if (some >= kVec) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) p[e] = sum[e];
      } else {
        for (int e = 0; e < some; ++e) p[e] = sum[e];
      }
    };
    for (int64_t i = i0; i < i1; i += kDeep) {
      uint32_t key[kDeep], val[kDeep];
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        key[j] = i + j < i1 ? s.key[i + j] : none;
        val[j] = i + j < i1 ? s.val[i + j] : 0;
        // ids that changed under the call have left places that no token was written to
        val[j] = val[j] < d.T ? val[j] : 0;
      }
      Pack<E, kVec> x[kDeep];
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        x[j].zero();
        const typename E::T* p = dout + int64_t(val[j]) * d.out_stride + c;
        if (key[j] < none) {
          if (some >= kVec) x[j].load(p);
          else x[j].load_some(p, some);
        }
      }
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        if (i + j >= i1) break;
        if (key[j] != name) {
          flush(false);
          name = key[j];
          from_before = false;
#pragma unroll
          for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum[e] += x[j].get(e);
      }
    }
    flush(name == behind);
  }
}

// Tokens of a piece: 32, fewer (8 at least) while that leaves the chip idle, more where
// te_join would go over very many pieces. 5,003 tokens by 250 with 32, 16, 8: 28, 16, 10 us;
// 65,536 by 1,024: 76, 80, 79, and te_join 14, 26, 47.
constexpr int64_t kMostPieces = 8192, kPieceThreads = 1 << 17;

// The names of several pieces: a workgroup adds up the parts of the one that begins
// in its piece, 4 columns a lane. Each of its 2^(8 - jg) groups of lanes adds every so
// manieth part, in order, so that narrow rows take as many loads at once as wide ones,
// and the first adds the groups' sums, in order.
template <class W>
__global__ void __launch_bounds__(256) te_join(const Embed d, const Pieces s, typename W::T* dw, int jg) {
  constexpr int kCols = 4, kDeep = 8;
  __shared__ float sums[256][kCols + 1];
  const uint32_t none = uint32_t(d.V);
  const int64_t piece = blockIdx.x, i0 = piece * s.per, i1 = i0 + s.per;
  if (i1 >= d.T) return;
  const uint32_t name = s.key[i1 - 1];
  if (name >= none || s.key[i1] != name) return;
  if (i0 > 0 && s.key[i0 - 1] == name) return;
  const int lane = threadIdx.x & 63, group = threadIdx.x >> jg, groups = 256 >> jg;
  int64_t n = 1;  // parts: this piece's and those of the pieces behind it that begin with the name
  for (;;) {
    const int64_t at = (piece + n + lane) * s.per;
    const int more = __popcll(__ballot(at < d.T && s.key[at < d.T ? at : 0] == name));
    n += more;
    if (more < 64) break;
  }
  const int32_t c = (int32_t(blockIdx.y << jg) + int32_t(threadIdx.x & ((1 << jg) - 1))) * kCols;
  const int some = d.width - c;
  float sum[kCols] = {};
  for (int64_t q = group; q < n; q += groups * kDeep) {
    float x[kDeep][kCols];
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      const int64_t part = q + groups * j;
      const float* p = (part ? s.head : s.tail) + (piece + part) * d.width + c;
#pragma unroll
      for (int e = 0; e < kCols; ++e) x[j][e] = part < n && e < some ? p[e] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kDeep; ++j)
#pragma unroll
      for (int e = 0; e < kCols; ++e) sum[e] += x[j][e];
  }
#pragma unroll
  for (int e = 0; e < kCols; ++e) sums[threadIdx.x][e] = sum[e];
  __syncthreads();
  if (group) return;
  for (int w = 1; w < groups; ++w) {
#pragma unroll
    for (int e = 0; e < kCols; ++e) sum[e] += sums[(w << jg) + threadIdx.x][e];
  }
#pragma unroll
  for (int e = 0; e < kCols; ++e)
    if (e < some) dw[int64_t(name) * d.weight_stride + c + e] = typename W::T(sum[e] * d.scale);
}

int check(const nopfs_embed* p) {
  if (!p) return fail(NOPFS_EINVAL, "embed is NULL");
  if (p->T < 0 || p->V < 1 || p->width < 1 || p->n_ids < 0)
    return fail(NOPFS_EINVAL, "T and n_ids must be >= 0, V and width >= 1");
  if (!is_dtype(p->dtype) || !is_dtype(p->weight_dtype)) return fail(NOPFS_EINVAL, "unknown dtype");
  if (p->id_bytes != 4 && p->id_bytes != 8) return fail(NOPFS_EINVAL, "id_bytes must be 4 or 8");
  if (!isfinite(p->scale)) return fail(NOPFS_EINVAL, "scale must be finite");
  if ((p->V > 1 && p->weight_stride < p->width) || (p->T > 1 && p->out_stride < p->width))
    return fail(NOPFS_EINVAL, "rows overlap");
  if (p->T > INT32_MAX || p->V > INT32_MAX - 1) return fail(NOPFS_ERANGE, "T must be < 2^31, V <= 2^31 - 2");
  if (p->width > 1 << 23) return fail(NOPFS_ERANGE, "width must be <= 2^23");
  if (p->weight_stride > 1 << 28 || p->out_stride > 1 << 28)  // byte offsets below 2^63
    return fail(NOPFS_ERANGE, "row strides must be <= 2^28");
  return NOPFS_OK;
}

Embed describe(const nopfs_embed* p, const void* ids, const int64_t* slot) {
  return {p->T, p->V, p->n_ids, p->weight_stride, p->out_stride, p->width, p->scale, ids, slot, p->id_bytes == 8};
}

// Lanes for a row: one vector each, a workgroup at most.
int row_lanes(int32_t width) { return std::min(8, log2_ceil(ceil_div(width, kVec))); }

// A group has four rows at a time where a row is one step of it and there are enough
// of them, for the loads in flight (16,384 rows of 2,048 in bf16 30 -> 26 us), else one
// (8,192 of 8,192: 42, with four 45; 32 of 2,048: 2.5 and 3.6).
constexpr int32_t kOneStep = 256 * kVec;
constexpr int64_t kManyRows = 1024;  // workgroups with a row per group

int embed_impl(const nopfs_embed* p, const void* weight, const void* ids, const int64_t* slot, void* out,
               int32_t* names, hipStream_t st) {
  const int rc = check(p);
  if (rc) return rc;
  if (p->T == 0) return NOPFS_OK;
  if (!slot && p->n_ids != p->T) return fail(NOPFS_EINVAL, "without slot, ids has an entry per token");
  if (!weight || !out || (!ids && p->n_ids > 0)) return fail(NOPFS_EINVAL, "weight, ids and out must be non-NULL");
  const Embed d = describe(p, ids, slot);
  const int lg = row_lanes(p->width);
  const int64_t blocks = ceil_div(p->T, 256 >> lg);
  const bool several = p->width <= kOneStep && blocks >= kManyRows;
  return by_dtype(p->weight_dtype, [&](auto w) {
    return by_dtype(p->dtype, [&](auto e) {
      typedef decltype(w) W;
      typedef decltype(e) E;
      return launch("te_forward", several ? te_forward<W, E, 4> : te_forward<W, E, 1>,
                    row_grid(several ? ceil_div(blocks, 4) : blocks), dim3(256), 0, st, d,
                    static_cast<const typename W::T*>(weight), static_cast<typename E::T*>(out), names, lg);
    });
  });
}

int embed_grad_impl(const nopfs_embed* p, const void* dout, const void* ids, const int64_t* slot, void* dw,
                    hipStream_t st) {
  int rc = check(p);
  if (rc) return rc;
  if (p->T > 0 && !slot && p->n_ids != p->T)
    return fail(NOPFS_EINVAL, "without slot, ids has an entry per token");
  if (!dw || (p->T > 0 && (!dout || (!ids && p->n_ids > 0))))
    return fail(NOPFS_EINVAL, "d_out, ids and d_weight must be non-NULL");
  const Embed d = describe(p, ids, slot);
  const int bits = log2_ceil(p->V + 1);  // keys 0 .. V
  const int passes = std::max(1, int(ceil_div(bits, kMostBits)));
  Sort s{};
  s.bits = std::max(1, int(ceil_div(bits, passes)));
  s.tiles = int32_t(std::min<int64_t>(128, ceil_div(p->T, kSortTile)));
  s.per_tile = s.tiles ? int32_t(ceil_div(p->T, s.tiles)) : 0;
  Pieces pc{};
  const int lg = row_lanes(p->width);
  pc.per = 32;
  while (pc.per > 8 && (ceil_div(p->T, pc.per) << lg) < kPieceThreads) pc.per /= 2;
  while (ceil_div(p->T, pc.per) > kMostPieces) pc.per *= 2;
  pc.n = int32_t(ceil_div(p->T, pc.per));
  Scratch sc(st);
  uint32_t *key[2], *val[2];
  const size_t n = size_t(std::max<int64_t>(p->T, 1)), parts = size_t(std::max(1, pc.n)) * size_t(p->width);
  for (int i = 0; i < 2; ++i) {
    if ((rc = step_alloc(&sc, &key[i], n)) || (rc = step_alloc(&sc, &val[i], n))) return rc;
  }
  if ((rc = step_alloc(&sc, &s.hist, size_t(std::max(1, s.tiles)) << s.bits)) ||
      (rc = step_alloc(&sc, &s.named, size_t(p->V))) || (rc = step_alloc(&sc, &pc.head, parts)) ||
      (rc = step_alloc(&sc, &pc.tail, parts)))
    return rc;
  const int64_t zeros = ceil_div(p->V, (256 >> lg) * kZeroRows);
  return by_dtype(p->weight_dtype, [&](auto w) {
    typedef decltype(w) W;
    typename W::T* to = static_cast<typename W::T*>(dw);
    const bool small = p->T <= kSmallSort && p->V <= kSmallNames;
    bool zeroed = false;
    const int32_t clears = int32_t(std::min<int64_t>(256, ceil_div(p->V, 16 * 256 * 4)));
    int r = NOPFS_OK, at = 0;
    if (small) {
      s.key = key[0], s.val = val[0];
      r = launch("te_sort", te_sort, dim3(1), dim3(1024), 0, st, d, s, std::max(1, int(ceil_div(bits, 8))));
      at = 1;
    }
    for (int pass = 0; !small && pass < passes && !r; ++pass, at ^= 1) {
      s.key_in = key[at ^ 1], s.val_in = val[at ^ 1], s.key = key[at], s.val = val[at];
      s.shift = pass * s.bits;
      const dim3 tiles(uint32_t(s.tiles));
      // the first count clears `named` as well, with workgroups of its own for many rows
      r = pass == 0 ? launch("te_count", te_count<true>, dim3(uint32_t(std::max(s.tiles, clears))), dim3(256), 0, st, d, s)
                    : launch("te_count", te_count<false>, tiles, dim3(256), 0, st, d, s);
      if (r) break;
      zeroed = pass > 0 && pass == passes - 1;
      if (zeroed)
        r = launch("te_scatter_zero", te_scatter_zero<W>, row_grid(s.tiles + zeros), dim3(256), 0, st, d, s, to, lg);
      else if (pass == 0)
        r = launch("te_scatter", te_scatter<true>, tiles, dim3(256), 0, st, d, s);
      else
        r = launch("te_scatter", te_scatter<false>, tiles, dim3(256), 0, st, d, s);
    }
    if (r) return r;
    pc.key = key[at ^ 1], pc.val = val[at ^ 1];
    const int64_t blocks = ceil_div(pc.n, 256 >> lg);
    r = by_dtype(p->dtype, [&](auto e) {
      typedef decltype(e) E;
      return launch("te_pieces", te_pieces<W, E>, row_grid(blocks + (zeroed ? 0 : zeros)), dim3(256), 0, st, d, pc,
                    static_cast<const typename E::T*>(dout), to, lg, uint32_t(blocks), s.named);
    });
    if (r || pc.n <= 1) return r;  // one piece: no name has parts
    const int jg = std::min(6, log2_ceil(ceil_div(p->width, 4)));
    return launch("te_join", te_join<W>, dim3(uint32_t(pc.n), uint32_t(ceil_div(p->width, 4 << jg))), dim3(256), 0, st,
                  d, pc, to, jg);
  });
}

}  // namespace
}  // namespace nopfs

using namespace nopfs;

extern "C" int nopfs_token_embed(const nopfs_embed* e, const void* weight, const void* ids, const int64_t* slot,
                                 void* out, void* hip_stream) {
  try {
    return embed_impl(e, weight, ids, slot, out, nullptr, static_cast<hipStream_t>(hip_stream));
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_token_embed_names(const nopfs_embed* e, const void* weight, const void* ids, const int64_t* slot,
                                       void* out, int32_t* names, void* hip_stream) {
  try {
    if (e && e->T > 0 && !names) return fail(NOPFS_EINVAL, "names must be non-NULL");
    return embed_impl(e, weight, ids, slot, out, names, static_cast<hipStream_t>(hip_stream));
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_token_embed_grad(const nopfs_embed* e, const void* d_out, const void* ids, const int64_t* slot,
                                      void* d_weight, void* hip_stream) {
  try {
    auto call = [&]() {
      return embed_grad_impl(e, d_out, ids, slot, d_weight, static_cast<hipStream_t>(hip_stream));
    };
    return e ? run_with_scratch(e->scratch, e->scratch_bytes, call) : call();
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_token_embed_scratch(const nopfs_embed* e, int64_t* bytes) {
  try {
    return scratch_size(bytes, [&]() {
      return embed_grad_impl(e, no_array(), no_array(), static_cast<const int64_t*>(no_array()), no_array(), nullptr);
    });
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}
