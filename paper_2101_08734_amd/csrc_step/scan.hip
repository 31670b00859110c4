// nopfs_gated_scan and its gradient: a gated linear recurrence over packed
// samples. For each channel, with a = 1 / (1 + exp(-gate)) and k = 1 - a,
//     h_t = a_t h_{t-1} + k_t x_t
// from h0 at a sample's first token, and for the gradient, from the last token back,
//     G_t = dh_t + R_{t+1},  R_t = a_t G_t,  dx_t = k_t G_t,
//     dgate_t = a_t k_t (h_{t-1} - x_t) G_t.
// A stretch of tokens is a map h -> A h + B (A the product of the a), or a constant
// if a sample begins in it. A wave holds 16 tokens of its channels in registers, makes
// their map, gets the state before them through the maps of the stretches before, and
// goes through its tokens again from there. Everything is read once and written once.
// 16,384 tokens by 2,048 channels in bf16: forward 64 us for 215 MB, the gradient 102 for
// 364; a workgroup loads, makes maps, waits and stores in turn beside vector units at 49
// and 43%, and there are three of them on a compute unit (70 registers a lane), of the
// gradient two (128, and 6 more in memory). Workgroups of 64 or 256 tokens took 78 and 77
// us where these took 70, the gradient 114 and 132 to 108.
//
// The states and maps are in 32 bits. A step is taken from the larger share,
// h + k (x - h) or x + a (h - x), so that its rounding is half a unit of the result; a
// map likewise, by the smaller of A and 1 - A, each summed up from the steps' shares, so
// that a gate near 1 loses nothing to the rounding of a product of its a. What goes from
// chunk to chunk so has one rounding of the state per chunk of 128 tokens: 25,600 tokens
// of gate 12.2 (a = 1 - 5e-6) are off by 2e-7, token by token by 1e-6, by products of
// rounded a by 3e-4.
#include "rows.hpp"

namespace nopfs {
namespace {

constexpr int kRows = NOPFS_SCAN_CHUNK;  // tokens of a wave
constexpr int kWaves = 8;
constexpr int kTile = kRows * kWaves;    // tokens of a workgroup
constexpr int kGroup = 16;               // chunks from one known state to the next, a power of two
constexpr int kLine = 32;                // words of 128 bytes

struct Scan {
  int64_t T;
  int32_t n, channels;
  int32_t tiles, chunks;  // of channels; of tokens
  int64_t x_stride, gate_stride, h_stride, dh_stride, dx_stride, dgate_stride;
  const void *x, *gate, *dh;
  const int32_t* start;
  const float *h0, *dlast, *carry_in;
  void *h, *dx, *dgate;
  float *last, *carry, *dh0;
  uint32_t* drawn;  // [tiles]: chunks that workgroups have drawn, kLine words apart
  int32_t* sample;  // [chunks]: of the chunk's first token
  uint64_t* slots;  // [chunks][tiles][64 kN]: what a chunk has said, of its lanes' first channels, then second
};

// A lane's channels, one word of them.
template <class E>
constexpr int kChannels = sizeof(typename E::T) == 4 ? 1 : 2;

// What a wave shares goes through here, so that the compiler keeps it once and not
// for every lane, and branches on it instead of masking lanes.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int wave_id() { return uniform(int(threadIdx.x >> 6)); }

// A lane's first channel. Lanes behind the last channels stand for the last ones once
// more (they read, make and write the same), so that no row masks lanes.
template <class E>
struct Cols {
  static constexpr int kN = kChannels<E>;
  uint32_t c;
  bool one;  // there is one channel alone, where kN is 2
};
template <class E>
__device__ __forceinline__ Cols<E> make_cols(const Scan& d, uint32_t tile) {
  const uint32_t c = (tile * 64 + (threadIdx.x & 63)) * Cols<E>::kN;
  const int32_t most = d.channels - Cols<E>::kN;
  return {most < 0 ? 0 : c < uint32_t(most) ? c : uint32_t(most), most < 0};
}

template <class E>
__device__ __forceinline__ void load_row(const void* base, int64_t stride, int64_t t, const Cols<E>& col,
                                         Pack<E, kChannels<E>>* v) {
  const typename E::T* p = static_cast<const typename E::T*>(base) + t * stride + col.c;
  if (col.one) v->load_some(p, 1);
  else v->template load<true>(p);
}
// A wave's rows, `rows` of them.
template <class E>
__device__ __forceinline__ void load_rows(const void* base, int64_t stride, int64_t t, int rows, const Cols<E>& col,
                                          Pack<E, kChannels<E>> (&v)[kRows]) {
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    v[r].zero();
    if (r < rows) load_row<E>(base, stride, t + r, col, &v[r]);
  }
}
template <class E>
__device__ __forceinline__ void store_row(void* base, int64_t stride, int64_t t, const Cols<E>& col,
                                          const float (&v)[kChannels<E>]) {
  typename E::T* p = static_cast<typename E::T*>(base) + t * stride + col.c;
  Pack<E, kChannels<E>> o;
  o.set(v);
  if (col.one) o.store_some(p, 1);
  else o.template store<true>(p);
}
// A row of the 32-bit arrays, of samples or chunks.
template <class E>
__device__ __forceinline__ void load_state(const float* base, int64_t row, const Scan& d, const Cols<E>& col,
                                           float (&v)[kChannels<E>]) {
  const float* p = base + row * d.channels + col.c;
#pragma unroll
  for (int i = 0; i < Cols<E>::kN; ++i) v[i] = i == 0 || !col.one ? p[i] : 0.0f;
}
template <class E>
__device__ __forceinline__ void store_state(float* base, int64_t row, const Scan& d, const Cols<E>& col,
                                            const float (&v)[kChannels<E>]) {
  float* p = base + row * d.channels + col.c;
#pragma unroll
  for (int i = 0; i < Cols<E>::kN; ++i)
    if (i == 0 || !col.one) p[i] = v[i];
}

// The smaller of a and k = 1 - a, with the gate's sign (negative: it is a), of gates of
// any type within 6 units of 2^-24 (the exponential 3, the sum, the reciprocal and the
// product 1 each): the exponent's rounding is made up for, the reciprocal refined. From
// 88 on the share is 0; the exponent of a much larger gate in 32 bits, or of an infinite
// one, would have lost an infinity.
constexpr float kMostGate = 128.0f;
__device__ __forceinline__ float share_of(float gate) {
  constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kLn2Low = -1.9046543e-9f;
  float g = fabsf(gate);
  g = g > kMostGate ? kMostGate : g;  // NaN stays
  const float t = -g * kLog2e;
  float e = __builtin_amdgcn_exp2f(t);
  e = fmaf(e, fmaf(-t, kLn2Low, fmaf(-t, kLn2, -g)), e);  // by what t has lost
  const float sum = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(sum);
  r = fmaf(r, fmaf(-sum, r, 1.0f), r);
  return copysignf(e * r, gate);
}
__device__ __forceinline__ bool is_a(float share) { return __float_as_int(share) < 0; }
__device__ __forceinline__ float a_of(float share) { return is_a(share) ? -share : 1.0f - share; }
__device__ __forceinline__ float step(float share, float h, float x) {
  return fmaf(share, x - h, is_a(share) ? x : h);  // x + a (h - x), or h + k (x - h)
}
// A stretch's map: B + A h, with the smaller of A and K = 1 - A as its share. A is what
// the stretch's steps make of 1 among zeros, K the sum of what they take from it. K is
// so only where no step's share is an a; of others A is at most a half and its
// rounding, and K not used.
__device__ __forceinline__ void more(float share, float* A, float* K) {
  *K = fmaf(share, *A, *K);
  *A = step(share, *A, 0.0f);
}
__device__ __forceinline__ float map_share(float A, float K) { return A <= 0.5625f ? -A : K; }
__device__ __forceinline__ float apply(float share, float B, float h) {
  return fmaf(-share, h, B) + (is_a(share) ? 0.0f : h);  // B + A h, or h + (B - K h)
}
// G's two shares, a G and k G.
__device__ __forceinline__ void split(float share, float G, float* aG, float* kG) {
  const float small = fabsf(share) * G, large = G - small;
  *aG = is_a(share) ? small : large;
  *kG = is_a(share) ? large : small;
}

// Where samples begin and end among a workgroup's tokens.
struct Marks {
  int32_t first[kTile], end[kTile];  // sample + 1 whose first, whose last token this is
};
// The tokens that belong to samples.
__device__ __forceinline__ int64_t tokens_of(const Scan& d) {
  const int64_t total = d.n > 0 ? uniform(d.start[d.n]) : 0;
  return total < 0 ? 0 : total < d.T ? total : d.T;
}
// The first sample s in [lo, n) with start[s + 1] > t (n - 1 if none), 64 candidates at a time.
__device__ inline int32_t sample_of(const Scan& d, int64_t t) {
  int32_t lo = 0, hi = d.n - 1;
  while (lo < hi) {
    const int32_t jump = (hi - lo + 63) >> 6;
    const int64_t cand = int64_t(lo) + int64_t(jump) * (__lane_id() + 1) - 1;
    const bool before = cand < hi && d.start[cand + 1] <= t;
    const int k = __popcll(__ballot(before));
    const int64_t top = int64_t(lo) + int64_t(jump) * (k + 1) - 1;
    lo = int64_t(lo) + int64_t(jump) * k < hi ? lo + jump * k : hi;
    hi = top < hi ? int32_t(top) : hi;
  }
  return lo;
}
// Of tokens t0 .. t0 + kTile - 1, by one wave, 64 samples at a time from s0, the first
// that matters. The first of them are read before the wave's own rows, whose loads
// theirs would otherwise wait for, and written behind.
struct Samples {
  int64_t s;
  int32_t a, b;  // its tokens
};
__device__ __forceinline__ Samples read_samples(const Scan& d, int64_t s0) {
  const int64_t s = s0 + int64_t(__lane_id());
  Samples v{s, INT32_MAX, 0};
  if (s < d.n) v.a = d.start[s], v.b = d.start[s + 1];
  return v;
}
__device__ inline void write_marks(const Scan& d, int64_t t0, Samples v, Marks* m) {
  const int64_t t1 = t0 + kTile < d.T ? t0 + kTile : d.T;
  for (int i = __lane_id(); i < kTile; i += 64) m->first[i] = m->end[i] = 0;
  for (;;) {
    wave_step();
    if (v.a < v.b) {  // it has tokens
      if (v.a >= t0 && v.a < t1) m->first[v.a - t0] = int32_t(v.s) + 1;
      if (v.b > t0 && v.b <= t1) m->end[v.b - 1 - t0] = int32_t(v.s) + 1;
    }
    if (!(__ballot(v.a < t1) >> 63)) break;  // the last of them is behind the chunk, or there is none
    v = read_samples(d, v.s - __lane_id() + 64);
  }
}
// Bit r: row r of the wave.
__device__ __forceinline__ uint32_t wave_marks(const int32_t* m) {
  const int lane = __lane_id();
  return uint32_t(__ballot(lane < kRows && m[wave_id() * kRows + (lane & (kRows - 1))] != 0));
}

// ---- from chunk to chunk ------------------------------------------------------
// The state behind a chunk is B + A times the state before it. Every chunk says
// its map, which takes only its own tokens; the last of a group of kGroup
// chunks says, when it knows the state before it, the state behind it instead. A
// chunk applies the maps of its group before it to the state behind the group
// before. So the chain is one wait per group, and the order of all roundings is fixed.
// (Groups of 8, 16, 32 chunks: 70, 70, 70 us forward, one sample of 65,536 tokens by
// 1,024 channels 144, 130, 135. Reading the slots is uncached: where every chunk read
// those of the 16 before it, 81 and 167.)
//
// A slot is one 64-bit word, written and read whole, so it needs no order with
// others: the upper half is the map's share, or kAbsolute where the lower half is the
// state whatever came before, or kNothing yet (both infinities, which no share is).
// A workgroup draws its chunk from its tile's counter, so all chunks that it waits
// for have been drawn by workgroups that run or have run.
constexpr uint32_t kAbsolute = 0xFF800000u, kNothing = 0x7F800000u;

__device__ __forceinline__ uint64_t slot_map(float share, float B) {
  return uint64_t(__float_as_uint(share)) << 32 | __float_as_uint(B);
}
__device__ __forceinline__ uint64_t slot_state(float h) { return uint64_t(kAbsolute) << 32 | __float_as_uint(h); }
__device__ __forceinline__ float through(uint64_t slot, float h) {
  const uint32_t code = uint32_t(slot >> 32);
  const float B = __uint_as_float(uint32_t(slot));
  return code == kAbsolute ? B : apply(__uint_as_float(code), B, h);
}

// The maps of a workgroup's waves; of a wave with a reset, the share is not used.
template <int kN>
struct Maps {
  float share[kWaves][64 * kN], B[kWaves][64 * kN];
  uint32_t reset[kWaves];
};
template <int kN>
__device__ __forceinline__ void keep_map(Maps<kN>* m, bool reset, const float (&A)[kN], const float (&K)[kN],
                                         const float (&B)[kN]) {
  const int wave = wave_id(), lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    m->share[wave][i * 64 + lane] = map_share(A[i], K[i]);
    m->B[wave][i * 64 + lane] = B[i];
  }
  if (lane == 0) m->reset[wave] = reset;
}
// The state before each wave's rows from that before the workgroup's, in place of the
// maps' B; by wave i < kN for the i-th channels. kBack: from the last wave on.
template <bool kBack, int kN>
__device__ __forceinline__ void spread(Maps<kN>* m, float state) {
  const int mine = threadIdx.x;
#pragma unroll
  for (int j = 0; j < kWaves; ++j) {
    const int w = kBack ? kWaves - 1 - j : j;
    const bool cut = uniform(m->reset[w]);
    const float share = m->share[w][mine], b = m->B[w][mine];
    m->B[w][mine] = state;
    state = cut ? b : apply(share, b, state);
  }
}

// A workgroup's chunk of its tile of channels, in the order of the chain.
template <bool kChain>
__device__ __forceinline__ int32_t draw(const Scan& d, uint32_t tile) {
  if (!kChain) return 0;
  __shared__ uint32_t drawn;
  if (threadIdx.x == 0) drawn = atomicAdd(d.drawn + tile * kLine, 1u);
  __syncthreads();
  return uniform(int32_t(drawn));
}

// What a chunk has been told: the state before the group, then the maps up to its own.
template <int kN>
struct Chain {
  uint64_t said[kGroup][64 * kN];
};

// The state before chunk number `at` of the chain (kBack: chunk chunks - 1 - at);
// tells the others the chunk's map, or the state behind its group. After a barrier
// behind keep_map. Wave i < kN works on the i-th channels of all lanes and gets their
// state, the waves share the waiting.
template <bool kBack, int kN>
__device__ inline float chain(const Scan& d, int32_t at, uint32_t tile, const Maps<kN>& maps, Chain<kN>* lds) {
  const int wave = wave_id(), lane = threadIdx.x & 63, mine = wave * 64 + lane;
  const int pos = at & (kGroup - 1);
  uint64_t* slots = d.slots + (int64_t(at - pos) * d.tiles + tile) * 64 * kN;  // of the group's first chunk
  const int64_t next = int64_t(d.tiles) * 64 * kN;
  float A = 1.0f, K = 0.0f, B = 0.0f;
  bool reset = false;
  if (wave < kN) {
#pragma unroll
    for (int j = 0; j < kWaves; ++j) {
      const int w = kBack ? kWaves - 1 - j : j;
      const bool cut = uniform(maps.reset[w]);
      const float share = maps.share[w][mine], b = maps.B[w][mine];
      more(share, &A, &K);
      B = cut ? b : apply(share, b, B);
      reset |= cut;
    }
    if (pos < kGroup - 1 || reset)
      __hip_atomic_store(slots + pos * next + mine, reset ? slot_state(B) : slot_map(map_share(A, K), B),
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  for (int j = wave; j < (pos + 1) * kN; j += kWaves) {
    const int from = j / kN, i = j & (kN - 1);  // 0: the chunk before the group
    uint64_t v = slot_state(0.0f);
    if (from > 0 || at >= kGroup) {
      const uint64_t* p = slots + (from - 1) * next + i * 64 + lane;
      for (;;) {
        v = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const uint32_t code = uint32_t(v >> 32);
        if (__all(from ? code != kNothing : code == kAbsolute)) break;
        __builtin_amdgcn_s_sleep(1);
      }
    }
    lds->said[from][i * 64 + lane] = v;
  }
  __syncthreads();
  float state = 0.0f;
  if (wave < kN) {
#pragma unroll
    for (int j = 0; j < kGroup; ++j)
      if (j <= pos) state = through(lds->said[j][mine], state);
    if (pos == kGroup - 1 && !reset)
      __hip_atomic_store(slots + pos * next + mine, slot_state(apply(map_share(A, K), B, state)), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
  }
  return state;
}

// Nothing said, nothing drawn; and the sample of each chunk's first token.
__global__ void __launch_bounds__(256) gs_clear(const Scan d, int64_t n) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256)
    d.slots[i] = uint64_t(kNothing) << 32;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < d.tiles; i += int64_t(gridDim.x) * 256)
    d.drawn[i * kLine] = 0;
  for (int64_t c = int64_t(blockIdx.x) * 4 + wave_id(); c < d.chunks; c += int64_t(gridDim.x) * 4) {
    const int32_t s = d.n > 0 ? sample_of(d, c * kTile) : 0;
    if ((threadIdx.x & 63) == 0) d.sample[c] = s;
  }
}

// Samples without tokens: their states go through. Workgroups behind the last
// chunk's, 64 samples by a tile of 64 channels each.
__device__ inline void empty_samples(const Scan& d, int64_t block, const float* from, float* to) {
  const int32_t tiles64 = (d.channels + 63) / 64;
  const int32_t c = int32_t(block % tiles64) * 64 + int32_t(threadIdx.x & 63);
  const int64_t s0 = block / tiles64 * 64;
  if (c >= d.channels) return;
  for (int64_t s = s0 + (threadIdx.x >> 6); s < s0 + 64 && s < d.n; s += kWaves)
    if (d.start[s] >= d.start[s + 1]) to[s * d.channels + c] = from ? from[s * d.channels + c] : 0.0f;
}

template <class E, bool kChain>
__global__ void __launch_bounds__(64 * kWaves, 6) gs_forward(const Scan d, uint32_t blocks) {
  constexpr int kN = kChannels<E>;
  __shared__ Marks marks;
  __shared__ Maps<kN> maps;
  __shared__ std::conditional_t<kChain, Chain<kN>, int> lds;
  if (row_block() >= blocks) {
    if (d.last) empty_samples(d, row_block() - blocks, d.h0, d.last);
    return;
  }
  const uint32_t tile = row_block() % uint32_t(d.tiles);
  const int32_t chunk = draw<kChain>(d, tile);
  const int wave = wave_id();
  const Cols<E> col = make_cols<E>(d, tile);
  const int64_t t0 = int64_t(chunk) * kTile, t = t0 + wave * kRows;
  const bool marks_them = wave == kWaves - 1;
  Samples samples{};
  if (marks_them) samples = read_samples(d, kChain ? uniform(d.sample[chunk]) : d.n > 0 ? sample_of(d, t0) : 0);
  const int there = t >= d.T ? 0 : d.T - t < kRows ? int(d.T - t) : kRows;  // rows; `rows` of them in samples
  Pack<E, kN> x[kRows];
  float share[kRows][kN];
  {
    Pack<E, kN> g[kRows];
    load_rows<E>(d.gate, d.gate_stride, t, there, col, g);
    load_rows<E>(d.x, d.x_stride, t, there, col, x);
    if (marks_them) write_marks(d, t0, samples, &marks);
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int i = 0; i < kN; ++i) share[r][i] = share_of(g[r].get(i));
  }
  const int64_t total = tokens_of(d);
  const int rows = total <= t ? 0 : total - t < kRows ? int(total - t) : kRows;
  __syncthreads();
  const uint32_t first = wave_marks(marks.first), end = wave_marks(marks.end);
  const int32_t *starts = marks.first + wave * kRows, *ends = marks.end + wave * kRows;
  {
    float A[kN], K[kN], B[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) A[i] = 1.0f, K[i] = B[i] = 0.0f;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (r >= rows) continue;
      if (first >> r & 1) {
#pragma unroll
        for (int i = 0; i < kN; ++i) B[i] = 0.0f;
        if (d.h0) load_state<E>(d.h0, uniform(starts[r]) - 1, d, col, B);
      }
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        B[i] = step(share[r][i], B[i], x[r].get(i));
        more(share[r][i], &A[i], &K[i]);
      }
    }
    keep_map<kN>(&maps, first != 0, A, K, B);
  }
  __syncthreads();
  float before = 0.0f;
  if constexpr (kChain) before = chain<false, kN>(d, chunk, tile, maps, &lds);
  if (wave < kN) spread<false, kN>(&maps, before);
  __syncthreads();
  float h[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) h[i] = maps.B[wave][i * 64 + (threadIdx.x & 63)];
  const float none[kN] = {};
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (r >= there) continue;
    if (r >= rows) {
      if (r == 0 && d.carry) store_state<E>(d.carry, t / kRows, d, col, none);
      store_row<E>(d.h, d.h_stride, t + r, col, none);
      continue;
    }
    if (first >> r & 1) {
#pragma unroll
      for (int i = 0; i < kN; ++i) h[i] = 0.0f;
      if (d.h0) load_state<E>(d.h0, uniform(starts[r]) - 1, d, col, h);
    }
    if (r == 0 && d.carry) store_state<E>(d.carry, t / kRows, d, col, h);
#pragma unroll
    for (int i = 0; i < kN; ++i) h[i] = step(share[r][i], h[i], x[r].get(i));
    store_row<E>(d.h, d.h_stride, t + r, col, h);
    if ((end >> r & 1) && d.last) store_state<E>(d.last, uniform(ends[r]) - 1, d, col, h);
  }
}

// Short samples (the next token of a generation, above all): a wave goes through a
// sample by itself. Sample n stands for the rows behind the last one.
template <class E>
__global__ void __launch_bounds__(256) gs_step(const Scan d) {
  constexpr int kN = kChannels<E>;
  const int64_t work = int64_t(row_block()) * 4 + wave_id();
  const int64_t s = work / d.tiles;
  if (s > d.n) return;
  const Cols<E> col = make_cols<E>(d, uint32_t(work % d.tiles));
  const int64_t total = tokens_of(d);
  int64_t a = total, b = d.T;
  float h[kN] = {};
  if (s < d.n) {
    a = uniform(d.start[s]), b = uniform(d.start[s + 1]);
    a = a < 0 ? 0 : a, b = b < total ? b : total;
    if (d.h0) load_state<E>(d.h0, s, d, col, h);
  }
  auto token = [&](int64_t t, const Pack<E, kN>& x, const Pack<E, kN>& g) {
    if (d.carry && t % kRows == 0) store_state<E>(d.carry, t / kRows, d, col, h);
#pragma unroll
    for (int i = 0; i < kN; ++i) h[i] = step(share_of(g.get(i)), h[i], x.get(i));
    store_row<E>(d.h, d.h_stride, t, col, h);
  };
  if (s == d.n) {
    for (int64_t t = a; t < b; ++t) {
      if (d.carry && t % kRows == 0) store_state<E>(d.carry, t / kRows, d, col, h);
      store_row<E>(d.h, d.h_stride, t, col, h);
    }
    return;
  }
  int64_t t = a;
  auto tokens = [&](auto deep) {  // so many in flight, while there are
    constexpr int kDeep = decltype(deep)::value;
    for (; t + kDeep <= b; t += kDeep) {
      Pack<E, kN> x[kDeep], g[kDeep];
#pragma unroll
      for (int r = 0; r < kDeep; ++r) {
        load_row<E>(d.x, d.x_stride, t + r, col, &x[r]);
        load_row<E>(d.gate, d.gate_stride, t + r, col, &g[r]);
      }
#pragma unroll
      for (int r = 0; r < kDeep; ++r) token(t + r, x[r], g[r]);
    }
  };
  tokens(std::integral_constant<int, 16>());
  tokens(std::integral_constant<int, 4>());
  tokens(std::integral_constant<int, 1>());
  if (d.last) store_state<E>(d.last, s, d, col, h);
}

template <class E, bool kChain>
__global__ void __launch_bounds__(64 * kWaves, 4) gs_grad(const Scan d, uint32_t blocks) {
  constexpr int kN = kChannels<E>;
  __shared__ Marks marks;
  __shared__ Maps<kN> maps;
  __shared__ std::conditional_t<kChain, Chain<kN>, int> lds;
  if (row_block() >= blocks) {
    if (d.dh0) empty_samples(d, row_block() - blocks, d.dlast, d.dh0);
    return;
  }
  const uint32_t tile = row_block() % uint32_t(d.tiles);
  const int32_t at = draw<kChain>(d, tile);
  const int wave = wave_id();
  const Cols<E> col = make_cols<E>(d, tile);
  const int64_t t0 = int64_t(d.chunks - 1 - at) * kTile, t = t0 + wave * kRows;
  const bool marks_them = wave == kWaves - 1;
  Samples samples{};
  if (marks_them) samples = read_samples(d, kChain ? uniform(d.sample[d.chunks - 1 - at]) : d.n > 0 ? sample_of(d, t0) : 0);
  const int there = t >= d.T ? 0 : d.T - t < kRows ? int(d.T - t) : kRows;
  Pack<E, kN> dh[kRows];
  float share[kRows][kN], under[kRows][kN];  // under: h_{t-1} - x_t
  float h[kN] = {};
  if (there > 0) load_state<E>(d.carry_in, t / kRows, d, col, h);
  Pack<E, kN> x[kRows];
  {
    Pack<E, kN> g[kRows];
    load_rows<E>(d.gate, d.gate_stride, t, there, col, g);
    load_rows<E>(d.dh, d.dh_stride, t, there, col, dh);
    load_rows<E>(d.x, d.x_stride, t, there, col, x);
    if (marks_them) write_marks(d, t0, samples, &marks);
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int i = 0; i < kN; ++i) share[r][i] = share_of(g[r].get(i));
  }
  const int64_t total = tokens_of(d);
  const int rows = total <= t ? 0 : total - t < kRows ? int(total - t) : kRows;
  __syncthreads();
  const uint32_t first = wave_marks(marks.first), end = wave_marks(marks.end);
  const int32_t *starts = marks.first + wave * kRows, *ends = marks.end + wave * kRows;
  {
    float A[kN], K[kN], R[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) A[i] = 1.0f, K[i] = R[i] = 0.0f;
#pragma unroll
    for (int r = kRows - 1; r >= 0; --r) {
      if (r >= rows) continue;
      if (end >> r & 1) {
#pragma unroll
        for (int i = 0; i < kN; ++i) R[i] = 0.0f;
        if (d.dlast) load_state<E>(d.dlast, uniform(ends[r]) - 1, d, col, R);
      }
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        float kG;
        split(share[r][i], dh[r].get(i) + R[i], &R[i], &kG);
        more(share[r][i], &A[i], &K[i]);
      }
    }
    keep_map<kN>(&maps, end != 0, A, K, R);
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (r >= rows) continue;
    if (r > 0 && (first >> r & 1)) {
#pragma unroll
      for (int i = 0; i < kN; ++i) h[i] = 0.0f;
      if (d.h0) load_state<E>(d.h0, uniform(starts[r]) - 1, d, col, h);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      under[r][i] = h[i] - x[r].get(i);
      h[i] = step(share[r][i], h[i], x[r].get(i));
    }
  }
  __syncthreads();
  float behind = 0.0f;
  if constexpr (kChain) behind = chain<true, kN>(d, at, tile, maps, &lds);
  if (wave < kN) spread<true, kN>(&maps, behind);
  __syncthreads();
  float R[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) R[i] = maps.B[wave][i * 64 + (threadIdx.x & 63)];
#pragma unroll
  for (int r = kRows - 1; r >= 0; --r) {
    if (r >= there) continue;
    float dx[kN] = {}, dg[kN] = {};
    if (r < rows) {
      if (end >> r & 1) {
#pragma unroll
        for (int i = 0; i < kN; ++i) R[i] = 0.0f;
        if (d.dlast) load_state<E>(d.dlast, uniform(ends[r]) - 1, d, col, R);
      }
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const float G = dh[r].get(i) + R[i];
        split(share[r][i], G, &R[i], &dx[i]);
        dg[i] = under[r][i] * (a_of(share[r][i]) * dx[i]);
      }
      if ((first >> r & 1) && d.dh0) store_state<E>(d.dh0, uniform(starts[r]) - 1, d, col, R);
    }
    store_row<E>(d.dx, d.dx_stride, t + r, col, dx);
    store_row<E>(d.dgate, d.dgate_stride, t + r, col, dg);
  }
}

int check(const nopfs_scan* p, bool gradient) {
  if (!p) return fail(NOPFS_EINVAL, "scan is NULL");
  if (p->T < 0 || p->n < 0 || p->channels < 1) return fail(NOPFS_EINVAL, "T and n must be >= 0, channels >= 1");
  if (!is_dtype(p->dtype)) return fail(NOPFS_EINVAL, "unknown dtype");
  if (p->T > INT32_MAX || p->n > 1 << 30) return fail(NOPFS_ERANGE, "T must be < 2^31, n <= 2^30");
  const int64_t strides[] = {p->x_stride, p->gate_stride, gradient ? p->dh_stride : p->h_stride, p->dx_stride,
                             p->dgate_stride};
  for (int i = 0; i < (gradient ? 5 : 3); ++i) {
    if (p->T > 1 && strides[i] < p->channels) return fail(NOPFS_EINVAL, "rows overlap");
    if (strides[i] > 1 << 30) return fail(NOPFS_ERANGE, "strides must be <= 2^30");
  }
  if (p->channels > 1 << 28) return fail(NOPFS_ERANGE, "channels must be <= 2^28");
  return NOPFS_OK;
}

// Workgroups: chunks by tiles of channels, and behind them those of the samples
// without tokens, if a state is asked for.
int tile_channels(int32_t dtype) { return 64 * (dtype == NOPFS_FP32 ? 1 : 2); }
struct Grid {
  int64_t blocks, all;
};
int make_grid(const nopfs_scan* p, bool states, Scan* d, Grid* g) {
  const int per = tile_channels(p->dtype);
  d->T = p->T, d->n = p->n, d->channels = p->channels;
  d->x_stride = p->x_stride, d->gate_stride = p->gate_stride, d->h_stride = p->h_stride;
  d->dh_stride = p->dh_stride, d->dx_stride = p->dx_stride, d->dgate_stride = p->dgate_stride;
  d->tiles = int32_t(ceil_div(p->channels, per));
  d->chunks = int32_t(ceil_div(p->T, kTile));
  g->blocks = int64_t(d->chunks) * d->tiles;
  g->all = g->blocks + (states ? ceil_div(p->n, 64) * ceil_div(p->channels, 64) : 0);
  if (g->all > INT32_MAX) return fail(NOPFS_ERANGE, "too many tokens, samples and channels for one call");
  return NOPFS_OK;
}

// What the chunks say to each other, if there are several, with nothing said yet.
int make_chain(Scratch* sc, Scan* d, int per, hipStream_t st) {
  if (d->chunks <= 1) return NOPFS_OK;
  int rc;
  const size_t n = size_t(d->chunks) * size_t(d->tiles) * size_t(per);
  if ((rc = step_alloc(sc, &d->slots, n)) || (rc = step_alloc(sc, &d->drawn, size_t(d->tiles) * kLine)) ||
      (rc = step_alloc(sc, &d->sample, size_t(d->chunks)))) return rc;
  return launch("gs_clear", gs_clear, dim3(uint32_t(std::min<int64_t>(ceil_div(int64_t(n), 1024), 4096))), dim3(256),
                0, st, *d, int64_t(n));
}

// Up to so many tokens, and two a sample, samples go one by one. Of 2,048 channels (bf16)
// 32, 256, 1,024 samples of one token took 10.9, 10.9, 11.3 us, by chunks 13.0, 19.8, 21.9
// (4,096: 31.8 and 36.4); where one sample has all 1,024 tokens, 260 and 17, which is why
// there is no more of it.
constexpr int64_t kStepTokens = 1024;

int scan_impl(const nopfs_scan* p, const void* x, const void* gate, const int32_t* start, const float* h0, void* h,
              float* last, float* carry, hipStream_t st) {
  int rc = check(p, false);
  if (rc) return rc;
  if (!start || (p->T > 0 && (!x || !gate || !h))) return fail(NOPFS_EINVAL, "x, gate, start and h must be non-NULL");
  if (last && last == h0) return fail(NOPFS_EINVAL, "last must not be h0");
  Scan d{};
  d.x = x, d.gate = gate, d.start = start, d.h0 = h0, d.h = h, d.last = last, d.carry = carry;
  Grid g;
  if ((rc = make_grid(p, last != nullptr, &d, &g))) return rc;
  const int64_t waves = (int64_t(p->n) + 1) * d.tiles;
  if (p->T <= kStepTokens && p->T <= 2 * int64_t(p->n) && waves <= INT32_MAX)
    return by_dtype(p->dtype, [&](auto e) {
      return launch("gs_step", gs_step<decltype(e)>, row_grid(ceil_div(waves, 4)), dim3(256), 0, st, d);
    });
  Scratch sc(st);
  if ((rc = make_chain(&sc, &d, tile_channels(p->dtype), st))) return rc;
  return by_dtype(p->dtype, [&](auto e) {
    typedef decltype(e) E;
    return launch("gs_forward", d.chunks > 1 ? gs_forward<E, true> : gs_forward<E, false>, row_grid(g.all),
                  dim3(64 * kWaves), 0, st, d, uint32_t(g.blocks));
  });
}

int scan_grad_impl(const nopfs_scan* p, const void* dh, const float* dlast, const void* x, const void* gate,
                   const int32_t* start, const float* h0, const float* carry, void* dx, void* dgate, float* dh0,
                   hipStream_t st) {
  int rc = check(p, true);
  if (rc) return rc;
  if (!start || (p->T > 0 && (!dh || !x || !gate || !carry || !dx || !dgate)))
    return fail(NOPFS_EINVAL, "d_h, x, gate, start, carry, d_x and d_gate must be non-NULL");
  if (dh0 && dh0 == dlast) return fail(NOPFS_EINVAL, "d_h0 must not be d_last");
  Scan d{};
  d.dh = dh, d.dlast = dlast, d.x = x, d.gate = gate, d.start = start, d.h0 = h0, d.carry_in = carry;
  d.dx = dx, d.dgate = dgate, d.dh0 = dh0;
  Grid g;
  if ((rc = make_grid(p, dh0 != nullptr, &d, &g))) return rc;
  Scratch sc(st);
  if ((rc = make_chain(&sc, &d, tile_channels(p->dtype), st))) return rc;
  return by_dtype(p->dtype, [&](auto e) {
    typedef decltype(e) E;
    return launch("gs_grad", d.chunks > 1 ? gs_grad<E, true> : gs_grad<E, false>, row_grid(g.all), dim3(64 * kWaves),
                  0, st, d, uint32_t(g.blocks));
  });
}

}  // namespace
}  // namespace nopfs

using namespace nopfs;

extern "C" int nopfs_gated_scan(const nopfs_scan* s, const void* x, const void* gate, const int32_t* start,
                                const float* h0, void* h, float* last, float* carry, void* hip_stream) {
  try {
    auto call = [&]() {
      return scan_impl(s, x, gate, start, h0, h, last, carry, static_cast<hipStream_t>(hip_stream));
    };
    return s ? run_with_scratch(s->scratch, s->scratch_bytes, call) : call();
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_gated_scan_grad(const nopfs_scan* s, const void* d_h, const float* d_last, const void* x,
                                     const void* gate, const int32_t* start, const float* h0, const float* carry,
                                     void* d_x, void* d_gate, float* d_h0, void* hip_stream) {
  try {
    auto call = [&]() {
      return scan_grad_impl(s, d_h, d_last, x, gate, start, h0, carry, d_x, d_gate, d_h0,
                            static_cast<hipStream_t>(hip_stream));
    };
    return s ? run_with_scratch(s->scratch, s->scratch_bytes, call) : call();
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_gated_scan_scratch(const nopfs_scan* s, int32_t gradient, int64_t* bytes) {
  try {
    void* x = no_array();
    float* f = static_cast<float*>(x);
    const int32_t* start = static_cast<const int32_t*>(x);
    return scratch_size(bytes, [&]() {
      return gradient ? scan_grad_impl(s, x, nullptr, x, x, start, nullptr, f, x, x, nullptr, nullptr)
                      : scan_impl(s, x, x, start, nullptr, x, nullptr, nullptr, nullptr);
    });
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}
