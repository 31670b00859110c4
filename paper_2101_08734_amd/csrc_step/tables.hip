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
//                   sums and the cut; packed starts and first free entries.
//   2. bt_expand -- one workgroup per tile of packed tokens or of table
//                   entries: a token's read by search in the starts.
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

template <int kThreads>
__global__ void __launch_bounds__(kThreads) bt_scan(const Batch b) {
  __shared__ uint64_t tmp[65];
  __shared__ int32_t s_cut;
  const int64_t g = blockIdx.x;
  int32_t* start = b.start + g * (int64_t(b.n) + 1);
  int32_t* first = b.first + g * (int64_t(b.n) + 1);
  uint64_t ct = 0, cb = 0;  // sums of the admitted reads so far
  int32_t admitted = b.n;
  if (threadIdx.x == 0) start[0] = first[0] = 0;
  for (int32_t r0 = 0; r0 < b.n; r0 += kThreads) {
    const int32_t r = r0 + int32_t(threadIdx.x);
    const int32_t len = r < b.n ? read_length(b, g, r) : 0;
    const int32_t nb = int32_t((int64_t(len) + b.block - 1) / b.block);
    if (threadIdx.x == 0) s_cut = INT32_MAX;
    uint64_t tt, tb;
    const uint64_t et = block_exclusive_scan64(uint64_t(len), tmp, &tt) + ct;
    const uint64_t eb = block_exclusive_scan64(uint64_t(nb), tmp, &tb) + cb;
    const bool fits = et + len <= uint64_t(b.cap) && eb + nb <= uint64_t(b.blocks) && nb <= b.width;
    if (r < b.n && !fits) atomicMin(&s_cut, r);
    __syncthreads();
    const int32_t cut = s_cut;
    __syncthreads();
    if (r < b.n && r < cut) {
      start[r + 1] = int32_t(et + len);
      first[r + 1] = int32_t(eb + nb);
    }
    if (cut != INT32_MAX) {  // the same in every thread
      // the sums up to the cut: known to the thread of the first read left out
      if (r == cut) {
        tmp[0] = et;
        tmp[1] = eb;
      }
      __syncthreads();
      ct = tmp[0];
      cb = tmp[1];
      admitted = cut;
      for (int64_t q = int64_t(cut) + threadIdx.x; q < b.n; q += kThreads) {
        start[q + 1] = int32_t(ct);
        first[q + 1] = int32_t(cb);
      }
      break;
    }
    ct += tt;
    cb += tb;
  }
  if (threadIdx.x == 0) {
    b.used[3 * g] = admitted;
    b.used[3 * g + 1] = int32_t(ct);
    b.used[3 * g + 2] = int32_t(cb);
  }
}

constexpr int kTokTile = 4096;  // packed tokens of a workgroup
constexpr int kTabTile = 4096;  // table entries of a workgroup

__global__ void __launch_bounds__(256) bt_expand(const Batch b, uint32_t tok_tiles, uint32_t tab_tiles) {
  const uint32_t per = tok_tiles + tab_tiles;
  const int64_t g = blockIdx.x / per;
  const uint32_t t = blockIdx.x % per;
  const int32_t* start = b.start + g * (int64_t(b.n) + 1);
  const int32_t* first = b.first + g * (int64_t(b.n) + 1);
  const int32_t* free_list = b.free_list + g * b.free_stride;
  if (t < tok_tiles) {
    const int32_t total = start[b.n];
    for (int32_t i = threadIdx.x; i < kTokTile; i += 256) {
      const int64_t at = int64_t(t) * kTokTile + i;
      if (at >= b.cap) return;
      int64_t slot = -1;
      int32_t row = -1, pos = -1;
      if (at < total) {
        int32_t lo = 0, hi = b.n - 1;  // the first r with start[r + 1] > at
        while (lo < hi) {
          const int32_t mid = (lo + hi) >> 1;
          if (start[mid + 1] > at) hi = mid;
          else lo = mid + 1;
        }
        row = lo;
        pos = int32_t(at) - start[lo];
        const int32_t j = pos / b.block;
        slot = int64_t(free_list[first[lo] + j]) * b.block + (pos - j * b.block);
      }
      const int64_t o = g * b.cap + at;
      b.slot[o] = slot;
      b.row[o] = row;
      b.pos[o] = pos;
    }
  } else {
    const int64_t n_entries = int64_t(b.n) * b.width;
    for (int32_t i = threadIdx.x; i < kTabTile; i += 256) {
      const int64_t e = int64_t(t - tok_tiles) * kTabTile + i;
      if (e >= n_entries) return;
      const int32_t r = int32_t(e / b.width);
      const int32_t j = int32_t(e - int64_t(r) * b.width);
      const int32_t f0 = first[r];
      b.table[g * n_entries + e] = j < first[r + 1] - f0 ? free_list[f0 + j] : -1;
    }
  }
}

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
  const int64_t tok_tiles = ceil_div(p->cap, kTokTile);
  const int64_t tab_tiles = ceil_div(int64_t(p->n) * p->width, kTabTile);
  if (int64_t(p->G) * (tok_tiles + tab_tiles) >= int64_t(INT32_MAX))
    return fail(NOPFS_ERANGE, "too many table entries and packed tokens for one call");
  Scratch sc(st);
  Batch b{p->F, p->ids_stride, p->free_stride, p->G, p->n, p->blocks, p->block, p->width, p->cap,
          ids, tokens, free_list, start, table, slot, row, pos, used, nullptr};
  int rc = sc.alloc_n(&b.first, size_t(p->G) * (size_t(p->n) + 1));
  if (rc) return rc;
  rc = launch("bt_scan", bt_scan<256>, dim3(uint32_t(p->G)), dim3(256), 0, st, b);
  if (rc) return rc;
  return launch("bt_expand", bt_expand, dim3(uint32_t(p->G * (tok_tiles + tab_tiles))), dim3(256), 0, st, b,
                uint32_t(tok_tiles), uint32_t(tab_tiles));
}

}  // namespace
}  // namespace nopfs

using namespace nopfs;

extern "C" int nopfs_batch_tables(const nopfs_batch* batch, const int32_t* ids, const int32_t* tokens,
                                  const int32_t* free_blocks, int32_t* start, int32_t* table,
                                  int64_t* slot, int32_t* row, int32_t* pos, int32_t* used,
                                  void* hip_stream) {
  try {
    return batch_tables_impl(batch, ids, tokens, free_blocks, start, table, slot, row, pos, used,
                             static_cast<hipStream_t>(hip_stream));
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}
