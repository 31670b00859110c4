// nopfs_batch_tables: where the tokens of each worker's next reads lie.
//
// A resident token buffer holds samples in blocks of `block` tokens. For each
// group (worker) the reads are taken in stream order and given blocks from
// the group's free list, up to the first read that does not fit: with len_r
// and nb_r = ceil(len_r / block),
//     ct_r = sum_{s <= r} len_s,   cb_r = sum_{s <= r} nb_s,
//     read r is admitted iff ct_s <= cap, cb_s <= blocks, nb_s <= width for
//     every s <= r.
//   1. bt_scan   -- one workgroup per group: lengths gathered, both running
//                   sums and the cut; packed starts and first free entries
//                   (1,024 reads a round, one round after the other: a single
//                   group of very many reads is one workgroup's work).
//   2. bt_expand -- one workgroup per 8,192 packed tokens or table entries,
//                   four adjacent ones per thread: the tile's starts go to
//                   LDS, a token's read is searched there.
// The outputs are the traffic (16 bytes a packed token): bound by stores, 256
// groups x 294,912 tokens (1.25 GB) in 248 us, 5.0 TB/s. A few short groups
// take bt_small instead, one launch: every tile repeats its group's sums in
// LDS.
#include "step.hpp"

namespace nopfs {
namespace {

struct Batch {
  int64_t F, ids_stride, free_stride;
  int32_t G, n, blocks, block, width, cap;
  const int32_t *ids, *tokens, *free_list;
  int32_t *start, *table;
  int64_t* slot;
  int32_t *row, *pos, *used;
  int32_t* first;  // [G][n + 1]: free-list entries taken before read r (scratch)
};

__device__ inline int32_t read_length(const Batch& b, int64_t g, int32_t r) {
  int32_t len;
  if (b.ids) {
    const int64_t id = b.ids[g * b.ids_stride + r];
    len = id >= 0 && id < b.F ? b.tokens[id] : 0;
  } else {
    len = b.tokens[g * b.ids_stride + r];
  }
  return len > 0 ? len : 0;
}

// x div d for 0 <= x < 2^31 and the d >= 1 it was made for: with s = ceil(log2
// d), m = floor(2^(31+s) / d) + 1 exceeds 2^(31+s) / d by at most 1, so x m /
// 2^(31+s) exceeds x / d by less than 1 / d.
struct Divider {
  uint32_t m, shift;
  explicit Divider(int32_t d) {
    uint32_t s = 0;
    while ((int64_t(1) << s) < d) ++s;
    m = uint32_t((uint64_t(1) << (31 + s)) / uint32_t(d) + 1);
    shift = 31 + s;
  }
  __device__ __forceinline__ int32_t div(int32_t x) const { return int32_t((uint64_t(uint32_t(x)) * m) >> shift); }
};

// Sums of reads r0 .. r0 + kThreads - 1 and the first of them that does not
// fit (INT32_MAX: none); et, eb: the sums before the thread's own read.
struct Sums {
  uint64_t et, eb, tt, tb;
  int32_t len, nb, cut;
};
struct SumsLds {
  uint64_t wave_t[16], wave_b[16];
  uint64_t cut_t, cut_b;
  int32_t cut;
};
template <int kThreads>
__device__ inline Sums sum_reads(const Batch& b, int64_t g, int32_t r0, uint64_t ct, uint64_t cb, const Divider& by_block,
                                 SumsLds* lds) {
  const int32_t r = r0 + int32_t(threadIdx.x);
  const int wave = threadIdx.x >> 6;
  Sums s;
  s.len = r < b.n ? read_length(b, g, r) : 0;
  s.nb = by_block.div(s.len);
  s.nb += s.len - s.nb * b.block > 0;
  const uint64_t it = wave_inclusive_scan64(uint64_t(s.len)), ib = wave_inclusive_scan64(uint64_t(s.nb));
  if ((threadIdx.x & 63) == 63) {
    lds->wave_t[wave] = it;
    lds->wave_b[wave] = ib;
  }
  if (threadIdx.x == 0) lds->cut = INT32_MAX;
  __syncthreads();
  s.et = ct + it - uint64_t(s.len);
  s.eb = cb + ib - uint64_t(s.nb);
  s.tt = s.tb = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) {
      s.et += lds->wave_t[w];
      s.eb += lds->wave_b[w];
    }
    s.tt += lds->wave_t[w];
    s.tb += lds->wave_b[w];
  }
  const bool fits = s.et + s.len <= uint64_t(b.cap) && s.eb + s.nb <= uint64_t(b.blocks) && s.nb <= b.width;
  if (r < b.n && !fits) atomicMin(&lds->cut, r);
  __syncthreads();
  s.cut = lds->cut;
  if (s.cut != INT32_MAX) {  // the sums up to the cut: known to the first read left out
    if (r == s.cut) {
      lds->cut_t = s.et;
      lds->cut_b = s.eb;
    }
    __syncthreads();
    s.tt = lds->cut_t - ct;
    s.tb = lds->cut_b - cb;
  }
  return s;
}

template <int kThreads>
__global__ void __launch_bounds__(kThreads) bt_scan(const Batch b, const Divider by_block) {
  __shared__ SumsLds lds;
  const int64_t g = blockIdx.x;
  int32_t* start = b.start + g * (int64_t(b.n) + 1);
  int32_t* first = b.first + g * (int64_t(b.n) + 1);
  uint64_t ct = 0, cb = 0;  // sums of the admitted reads so far
  int32_t admitted = b.n;
  if (threadIdx.x == 0) start[0] = first[0] = 0;
  for (int32_t r0 = 0; r0 < b.n; r0 += kThreads) {
    const int32_t r = r0 + int32_t(threadIdx.x);
    const Sums s = sum_reads<kThreads>(b, g, r0, ct, cb, by_block, &lds);
    ct += s.tt;
    cb += s.tb;
    if (r < b.n && r < s.cut) {
      start[r + 1] = int32_t(s.et + s.len);
      first[r + 1] = int32_t(s.eb + s.nb);
    }
    if (s.cut != INT32_MAX) {  // the same in every thread
      admitted = s.cut;
      for (int64_t q = int64_t(s.cut) + threadIdx.x; q < b.n; q += kThreads) {
        start[q + 1] = int32_t(ct);
        first[q + 1] = int32_t(cb);
      }
      break;
    }
    __syncthreads();  // the sums in LDS are read: the next round may write them
  }
  if (threadIdx.x == 0) {
    b.used[3 * g] = admitted;
    b.used[3 * g + 1] = int32_t(ct);
    b.used[3 * g + 2] = int32_t(cb);
  }
}

// Packed tokens or table entries of a workgroup: 256 groups x 294,912 tokens
// took bt_expand 241 us with 8,192, 258 with 4,096, 330 with 1,024, 261 with
// 16,384; where that leaves compute units idle, 1,024 (one group of 12,288
// tokens took bt_small 6.8 us with 1,024, 10 with 4,096).
constexpr int kTile = 8192, kSmallTile = 1024;
constexpr int kTileRows = 1024;  // starts of a tile kept in LDS

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_by4 __attribute__((aligned(4)));  // rows of any length: adjacent, not aligned
typedef int64_t i64x2 __attribute__((ext_vector_type(2)));
typedef i64x2 i64x2_by8 __attribute__((aligned(8)));

// Packed tokens [t0, t0 + kTile) of group g. start and first hold the group's
// reads from r0 on (in global memory or LDS), the tile's tokens belong to reads r0
// .. r1.
template <int kTile>
__device__ inline void token_tile(const Batch& b, int64_t g, int32_t t0, int32_t total, int32_t r0, int32_t r1,
                                  const int32_t* start, const int32_t* first, const Divider& by_block) {
  const int32_t* free_list = b.free_list + g * b.free_stride;
  for (int i = 0; i < kTile / 1024; ++i) {
    const int32_t t = t0 + i * 1024 + int32_t(threadIdx.x) * 4;
    if (t >= b.cap) return;
    int64_t slot[4];
    int32_t row[4], pos[4];
    int32_t r = r0;
    if (t < total) {  // the first read with start[r + 1] > t
      int32_t hi = r1;
      while (r < hi) {
        const int32_t mid = (r + hi) >> 1;
        if (start[mid + 1 - r0] > t) hi = mid;
        else r = mid + 1;
      }
    }
    int32_t begin = 0, end = 0, f0 = 0;
    if (t < total) {
      begin = start[r - r0];
      end = start[r + 1 - r0];
      f0 = first[r - r0];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      slot[e] = row[e] = pos[e] = -1;
      if (t + e < total) {
        while (t + e >= end) {  // reads of no token are passed over
          ++r;
          begin = end;
          end = start[r + 1 - r0];
          f0 = first[r - r0];
        }
        row[e] = r;
        pos[e] = t + e - begin;
        const int32_t j = by_block.div(pos[e]);
        slot[e] = int64_t(free_list[f0 + j]) * b.block + (pos[e] - j * b.block);
      }
    }
    const int64_t o = g * b.cap + t;
    if (t + 4 <= b.cap) {
      *reinterpret_cast<i64x2_by8*>(b.slot + o) = i64x2{slot[0], slot[1]};
      *reinterpret_cast<i64x2_by8*>(b.slot + o + 2) = i64x2{slot[2], slot[3]};
      *reinterpret_cast<i32x4_by4*>(b.row + o) = i32x4{row[0], row[1], row[2], row[3]};
      *reinterpret_cast<i32x4_by4*>(b.pos + o) = i32x4{pos[0], pos[1], pos[2], pos[3]};
    } else {
      for (int e = 0; t + e < b.cap; ++e) {
        b.slot[o + e] = slot[e];
        b.row[o + e] = row[e];
        b.pos[o + e] = pos[e];
      }
    }
  }
}

// Table entries [e0, e0 + kTile) of group g; first holds all of its reads.
template <int kTile>
__device__ inline void table_tile(const Batch& b, int64_t g, int64_t e0, const int32_t* first) {
  const int64_t n_entries = int64_t(b.n) * b.width;
  const int32_t* free_list = b.free_list + g * b.free_stride;
  int32_t* table = b.table + g * n_entries;
  for (int i = 0; i < kTile / 1024; ++i) {
    const int64_t e = e0 + i * 1024 + int64_t(threadIdx.x) * 4;
    if (e >= n_entries) return;
    int32_t r = int32_t(e / b.width), j = int32_t(e - int64_t(r) * b.width);
    int32_t v[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      v[x] = -1;
      if (e + x < n_entries) {
        const int32_t f0 = first[r];
        if (j < first[r + 1] - f0) v[x] = free_list[f0 + j];
        if (++j == b.width) {
          j = 0;
          ++r;
        }
      }
    }
    if (e + 4 <= n_entries) {
      *reinterpret_cast<i32x4_by4*>(table + e) = i32x4{v[0], v[1], v[2], v[3]};
    } else {
      for (int x = 0; e + x < n_entries; ++x) table[e + x] = v[x];
    }
  }
}

// The first read r in [lo, hi] with start[r + 1] > t (hi if none), 64 candidates
// at a time; by a whole wave.
__device__ inline int32_t find_read(const int32_t* start, int32_t lo, int32_t hi, int32_t t) {
  const int lane = __lane_id();
  while (lo < hi) {
    const int32_t step = (hi - lo + 63) >> 6;
    const int64_t cand = int64_t(lo) + int64_t(step) * (lane + 1) - 1;  // below hi + 64 step
    const bool before = cand < hi && start[cand + 1] <= t;              // the read is behind cand
    const int k = __popcll(__ballot(before));                           // monotone: the first k
    const int64_t top = int64_t(lo) + int64_t(step) * (k + 1) - 1;
    lo += step * k;
    hi = top < hi ? int32_t(top) : hi;
  }
  return lo;
}

template <int kTile>
__global__ void __launch_bounds__(256) bt_expand(const Batch b, uint32_t tok_tiles, uint32_t tab_tiles,
                                                 const Divider by_block) {
  __shared__ int32_t s_start[kTileRows + 2], s_first[kTileRows + 2];
  const uint32_t per = tok_tiles + tab_tiles;
  const int64_t g = blockIdx.x / per;
  const uint32_t t = blockIdx.x % per;
  const int32_t* start = b.start + g * (int64_t(b.n) + 1);
  const int32_t* first = b.first + g * (int64_t(b.n) + 1);
  if (t >= tok_tiles) {
    table_tile<kTile>(b, g, int64_t(t - tok_tiles) * kTile, first);
    return;
  }
  const int32_t t0 = int32_t(t) * kTile, total = start[b.n];
  int32_t r0 = 0, r1 = 0;
  if (t0 < total) {  // every wave searches for itself
    r0 = find_read(start, 0, b.n - 1, t0);
    r1 = find_read(start, r0, b.n - 1, min(t0 + kTile, total) - 1);
  }
  if (r1 - r0 < kTileRows) {
    for (int32_t i = threadIdx.x; i < r1 - r0 + 2; i += 256) {
      s_start[i] = start[r0 + i];
      s_first[i] = first[r0 + i];
    }
    __syncthreads();
    token_tile<kTile>(b, g, t0, total, r0, r1, s_start, s_first, by_block);
  } else {  // a tile of very many reads, most of them empty
    token_tile<kTile>(b, g, t0, total, r0, r1, start + r0, first + r0, by_block);
  }
}

// One launch for a few groups of at most 256 reads: every tile makes its
// group's sums itself; the group's first tile writes them out.
__global__ void __launch_bounds__(256) bt_small(const Batch b, uint32_t tok_tiles, uint32_t tab_tiles,
                                                const Divider by_block) {
  __shared__ SumsLds lds;
  __shared__ int32_t s_start[257], s_first[257];
  const uint32_t per = tok_tiles + tab_tiles;
  const int64_t g = blockIdx.x / per;
  const uint32_t t = blockIdx.x % per;
  const Sums s = sum_reads<256>(b, g, 0, 0, 0, by_block, &lds);
  const int32_t r = int32_t(threadIdx.x);
  const int32_t total = int32_t(s.tt), taken = int32_t(s.tb);
  if (r < b.n) {
    s_start[r + 1] = r < s.cut ? int32_t(s.et + s.len) : total;
    s_first[r + 1] = r < s.cut ? int32_t(s.eb + s.nb) : taken;
  }
  if (r == 0) s_start[0] = s_first[0] = 0;
  __syncthreads();
  if (t == 0) {
    for (int32_t i = r; i <= b.n; i += 256) b.start[g * (int64_t(b.n) + 1) + i] = s_start[i];
    if (r == 0) {
      b.used[3 * g] = min(s.cut, b.n);
      b.used[3 * g + 1] = total;
      b.used[3 * g + 2] = taken;
    }
  }
  if (t < tok_tiles)
    token_tile<kSmallTile>(b, g, int32_t(t) * kSmallTile, total, 0, b.n - 1, s_start, s_first, by_block);
  else
    table_tile<kSmallTile>(b, g, int64_t(t - tok_tiles) * kSmallTile, s_first);
}

// Tiles that the chip runs at once: up to so many small ones the sums are
// repeated rather than made in a launch of their own, and below so many large
// ones small ones are taken.
constexpr int64_t kSmallTiles = 2048;

int batch_tables_impl(const nopfs_batch* p, const int32_t* ids, const int32_t* tokens,
                      const int32_t* free_list, int32_t* start, int32_t* table, int64_t* slot,
                      int32_t* row, int32_t* pos, int32_t* used, hipStream_t st) {
  if (!p) return fail(NOPFS_EINVAL, "batch is NULL");
  if (p->G < 1 || p->n < 1 || p->block < 1 || p->width < 1 || p->blocks < 0 || p->cap < 0)
    return fail(NOPFS_EINVAL, "G, n, block and width must be >= 1, blocks and cap >= 0");
  if (ids && p->F < 1) return fail(NOPFS_EINVAL, "F must be >= 1");
  if (p->G > 1 && (p->ids_stride < p->n || p->free_stride < p->blocks))
    return fail(NOPFS_EINVAL, "rows of ids or of the free lists overlap");
  if (!tokens || !start || !table || !used || (p->blocks > 0 && !free_list) ||
      (p->cap > 0 && (!slot || !row || !pos)))
    return fail(NOPFS_EINVAL, "tokens, the free lists and every output must be non-NULL");
  if (p->cap > (1 << 30) || p->n > (1 << 30)) return fail(NOPFS_ERANGE, "cap and n must be <= 2^30");
  const int64_t entries = int64_t(p->n) * p->width;
  const int64_t small_tok = ceil_div(p->cap, kSmallTile), small_tab = ceil_div(entries, kSmallTile);
  int64_t tok_tiles = ceil_div(p->cap, kTile), tab_tiles = ceil_div(entries, kTile);
  const bool small = p->G * (tok_tiles + tab_tiles) < kSmallTiles;
  if (small) tok_tiles = small_tok, tab_tiles = small_tab;
  const int64_t tiles = int64_t(p->G) * (tok_tiles + tab_tiles);
  if (tiles >= int64_t(1) << 24 || p->G >= 1 << 22)  // a launch has fewer than 2^32 threads
    return fail(NOPFS_ERANGE, "too many workers, table entries and packed tokens for one call");
  Batch b{p->F, p->ids_stride, p->free_stride, p->G, p->n, p->blocks, p->block, p->width, p->cap,
          ids, tokens, free_list, start, table, slot, row, pos, used, nullptr};
  const Divider by_block(p->block);
  if (p->n <= 256 && p->G * (small_tok + small_tab) <= kSmallTiles)
    return launch("bt_small", bt_small, dim3(uint32_t(p->G * (small_tok + small_tab))), dim3(256), 0, st, b,
                  uint32_t(small_tok), uint32_t(small_tab), by_block);
  Scratch sc(st);
  int rc = step_alloc(&sc, &b.first, size_t(p->G) * (size_t(p->n) + 1));
  if (rc) return rc;
  rc = p->n <= 256 ? launch("bt_scan", bt_scan<256>, dim3(uint32_t(p->G)), dim3(256), 0, st, b, by_block)
                   : launch("bt_scan", bt_scan<1024>, dim3(uint32_t(p->G)), dim3(1024), 0, st, b, by_block);
  if (rc) return rc;
  return launch("bt_expand", small ? bt_expand<kSmallTile> : bt_expand<kTile>, dim3(uint32_t(tiles)), dim3(256), 0, st,
                b, uint32_t(tok_tiles), uint32_t(tab_tiles), by_block);
}

}  // namespace
}  // namespace nopfs

using namespace nopfs;

extern "C" int nopfs_batch_tables(const nopfs_batch* batch, const int32_t* ids, const int32_t* tokens,
                                  const int32_t* free_blocks, int32_t* start, int32_t* table,
                                  int64_t* slot, int32_t* row, int32_t* pos, int32_t* used,
                                  void* hip_stream) {
  try {
    auto call = [&]() {
      return batch_tables_impl(batch, ids, tokens, free_blocks, start, table, slot, row, pos, used,
                               static_cast<hipStream_t>(hip_stream));
    };
    return batch ? run_with_scratch(batch->scratch, batch->scratch_bytes, call) : call();
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_batch_tables_scratch(const nopfs_batch* batch, int64_t* bytes) {
  try {
    int32_t* x = static_cast<int32_t*>(no_array());
    return scratch_size(bytes, [&]() {
      return batch_tables_impl(batch, nullptr, x, x, x, x, static_cast<int64_t*>(no_array()), x, x, x, nullptr);
    });
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}
