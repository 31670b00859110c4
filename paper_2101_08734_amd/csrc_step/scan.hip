// nopfs_gated_scan and its gradient: a gated linear recurrence over packed
// samples. For each channel, with a = 1 / (1 + exp(-gate)) and k = 1 - a,
//     h_t = a_t h_{t-1} + k_t x_t
// from h0 at a sample's first token, and for the gradient, from the last token back,
//     G_t = dh_t + R_{t+1},  R_t = a_t G_t,  dx_t = k_t G_t,
//     dgate_t = a_t k_t (h_{t-1} - x_t) G_t.
// A stretch of tokens is a map h -> A h + B (A the product of the a, 0 from a
// sample's start on), so the stretches are summed up side by side, their maps are
// applied one after the other, and each stretch is gone through again from its own
// first state. Bound by memory.
//
// The states and maps are in 32 bits. A step is taken from the larger share,
// h + k (x - h) or x + a (h - x), so that its rounding is half a unit of the
// result and a gate near 1 costs no accuracy over many tokens.
#include "rows.hpp"

namespace nopfs {
namespace {

constexpr int kRows = NOPFS_SCAN_CHUNK;  // tokens of a wave
constexpr int kWaves = 8;
constexpr int kTile = kRows * kWaves;    // tokens of a workgroup
constexpr float kReset = -1.0f;          // a map that has lost its state: A where B is all

struct Scan {
  int64_t T;
  int32_t n, channels;
  int32_t tiles;  // of channels
  int64_t x_stride, gate_stride, h_stride, dh_stride, dx_stride, dgate_stride;
  const void *x, *gate, *dh;
  const int32_t* start;
  const float *h0, *dlast, *carry_in;
  void *h, *dx, *dgate;
  float *last, *carry, *dh0;
  float *A, *B, *state;  // [chunks][channels]: the chunks' maps, the states before them
};

// A lane's channels, one word of them.
template <class E>
constexpr int kChannels = sizeof(typename E::T) == 4 ? 1 : 2;

template <class E>
struct Cols {
  static constexpr int kN = kChannels<E>;
  int32_t c;  // the first
  int n;      // so many of them are there
};
template <class E>
__device__ __forceinline__ Cols<E> make_cols(const Scan& d, int32_t tile) {
  const int32_t c = (tile * 64 + int32_t(threadIdx.x & 63)) * Cols<E>::kN;
  const int32_t left = d.channels - c;
  return {c, left < 0 ? 0 : left < Cols<E>::kN ? int(left) : Cols<E>::kN};
}

// A wave's rows, `rows` of them.
template <class E>
__device__ __forceinline__ void load_rows(const void* base, int64_t stride, int64_t t, int rows, const Cols<E>& col,
                                          Pack<E, kChannels<E>> (&v)[kRows]) {
  const typename E::T* p = static_cast<const typename E::T*>(base) + t * stride + col.c;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    v[r].zero();
    if (r < rows) {
      if (col.n == Cols<E>::kN) v[r].load(p + r * stride);
      else if (col.n > 0) v[r].load_some(p + r * stride, col.n);
    }
  }
}
template <class E>
__device__ __forceinline__ void store_row(void* base, int64_t stride, int64_t t, const Cols<E>& col,
                                          const float (&v)[kChannels<E>]) {
  typename E::T* p = static_cast<typename E::T*>(base) + t * stride + col.c;
  Pack<E, kChannels<E>> o;
  o.set(v);
  if (col.n == Cols<E>::kN) o.store(p);
  else if (col.n > 0) o.store_some(p, col.n);
}
// A row of the 32-bit arrays of n or chunks rows.
template <int kN>
__device__ __forceinline__ void load_state(const float* base, int64_t row, const Scan& d, int32_t c, int n,
                                           float (&v)[kN]) {
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = i < n ? base[row * d.channels + c + i] : 0.0f;
}
template <int kN>
__device__ __forceinline__ void store_state(float* base, int64_t row, const Scan& d, int32_t c, int n,
                                            const float (&v)[kN]) {
#pragma unroll
  for (int i = 0; i < kN; ++i)
    if (i < n) base[row * d.channels + c + i] = v[i];
}

// The smaller of a and k = 1 - a, in 32 bits of its own, with the gate's sign
// (negative: it is a).
__device__ __forceinline__ float share_of(float gate) {
  const float g = fabsf(gate);
  constexpr float kLog2e = 1.4426950408889634f, kLog2eLow = 1.9259629911266175e-8f, kLn2 = 0.6931471805599453f;
  const float t = -g * kLog2e;
  const float low = fmaf(-g, kLog2e, -t) - g * kLog2eLow;  // what t has lost
  float e = __builtin_amdgcn_exp2f(t);
  e = fmaf(e * kLn2, low, e);
  const float s = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(s);
  r = fmaf(r, fmaf(-s, r, 1.0f), r);
  return copysignf(e * r, gate);
}
__device__ __forceinline__ bool is_a(float share) { return __float_as_uint(share) >> 31; }
__device__ __forceinline__ float a_of(float share) { return is_a(share) ? -share : 1.0f - share; }
__device__ __forceinline__ float k_of(float share) { return is_a(share) ? 1.0f + share : share; }
__device__ __forceinline__ float step(float share, float h, float x) {
  const float d = x - h;
  return is_a(share) ? fmaf(share, d, x) : fmaf(share, d, h);  // x + a (h - x), h + k (x - h)
}
__device__ __forceinline__ float decay(float share, float g) {  // a g
  return is_a(share) ? -share * g : fmaf(-share, g, g);
}
__device__ __forceinline__ float apply(float A, float B, float h) { return A < 0.0f ? B : fmaf(A, h, B); }

// Where samples begin and end among a workgroup's tokens.
struct Marks {
  int32_t first[kTile], end[kTile];  // sample + 1 whose first, whose last token this is
};
// The tokens that belong to samples.
__device__ __forceinline__ int64_t tokens_of(const Scan& d) {
  const int64_t total = d.n > 0 ? d.start[d.n] : 0;
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
// Of tokens t0 .. t0 + kTile - 1, by all threads; ends with a barrier.
__device__ inline void make_marks(const Scan& d, int64_t t0, int64_t total, Marks* m) {
  for (int i = threadIdx.x; i < kTile; i += 64 * kWaves) m->first[i] = m->end[i] = 0;
  __syncthreads();
  if (t0 < total) {
    const int64_t t1 = t0 + kTile < total ? t0 + kTile : total;
    const int32_t s0 = sample_of(d, t0), s1 = sample_of(d, t1 - 1);
    for (int64_t s = s0 + int64_t(threadIdx.x); s <= s1; s += 64 * kWaves) {
      const int64_t a = d.start[s], b = d.start[s + 1];
      if (a >= b) continue;  // no tokens
      if (a >= t0 && a < t1) m->first[a - t0] = int32_t(s) + 1;
      if (b > t0 && b <= t1) m->end[b - 1 - t0] = int32_t(s) + 1;
    }
  }
  __syncthreads();
}
// Bit r: row r of the wave.
__device__ __forceinline__ uint32_t wave_marks(const int32_t* m) {
  const int lane = __lane_id();
  return uint32_t(__ballot(lane < kRows && m[(threadIdx.x >> 6) * kRows + (lane & (kRows - 1))] != 0));
}

// A wave's map of its rows, forwards.
template <class E>
__device__ __forceinline__ void forward_map(const Scan& d, const Pack<E, kChannels<E>> (&x)[kRows],
                                            const Pack<E, kChannels<E>> (&g)[kRows], int rows, uint32_t first,
                                            const int32_t* samples, const Cols<E>& col, float (&A)[kChannels<E>],
                                            float (&B)[kChannels<E>]) {
  constexpr int kN = kChannels<E>;
#pragma unroll
  for (int i = 0; i < kN; ++i) A[i] = 1.0f, B[i] = 0.0f;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (r >= rows) continue;
    if (first >> r & 1) {
#pragma unroll
      for (int i = 0; i < kN; ++i) A[i] = kReset, B[i] = 0.0f;
      if (d.h0) load_state<kN>(d.h0, samples[r] - 1, d, col.c, col.n, B);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float share = share_of(g[r].get(i));
      B[i] = step(share, B[i], x[r].get(i));
      A[i] = A[i] < 0.0f ? A[i] : A[i] * a_of(share);
    }
  }
}

// Grid: chunks by tiles of channels. Each chunk's map.
template <class E>
__global__ void __launch_bounds__(64 * kWaves) gs_sums(const Scan d) {
  constexpr int kN = kChannels<E>;
  __shared__ Marks marks;
  __shared__ float As[kWaves][64 * kN], Bs[kWaves][64 * kN];
  const uint32_t chunk = row_block() / uint32_t(d.tiles), tile = row_block() % uint32_t(d.tiles);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t0 = int64_t(chunk) * kTile, total = tokens_of(d);
  if (t0 >= d.T) return;
  const Cols<E> col = make_cols<E>(d, tile);
  const int64_t t = t0 + wave * kRows;
  const int rows = total <= t ? 0 : total - t < kRows ? int(total - t) : kRows;
  Pack<E, kN> x[kRows], g[kRows];
  load_rows<E>(d.x, d.x_stride, t, rows, col, x);
  load_rows<E>(d.gate, d.gate_stride, t, rows, col, g);
  make_marks(d, t0, total, &marks);
  float A[kN], B[kN];
  forward_map<E>(d, x, g, rows, wave_marks(marks.first), marks.first + wave * kRows, col, A, B);
#pragma unroll
  for (int i = 0; i < kN; ++i) As[wave][lane * kN + i] = A[i], Bs[wave][lane * kN + i] = B[i];
  __syncthreads();
  if (wave) return;
  for (int w = 1; w < kWaves; ++w) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float a = As[w][lane * kN + i], b = Bs[w][lane * kN + i];
      B[i] = apply(a, b, B[i]);
      A[i] = a < 0.0f ? kReset : A[i] < 0.0f ? A[i] : A[i] * a;
    }
  }
  store_state<kN>(d.A, chunk, d, col.c, col.n, A);
  store_state<kN>(d.B, chunk, d, col.c, col.n, B);
}

// A thread per channel: the states before the chunks (kBack: behind them).
template <bool kBack>
__global__ void __launch_bounds__(64) gs_states(const Scan d, int32_t chunks) {
  const int64_t c = int64_t(blockIdx.x) * 64 + threadIdx.x;
  if (c >= d.channels) return;
  float h = 0.0f;
  for (int32_t j = 0; j < chunks; ++j) {
    const int64_t at = int64_t(kBack ? chunks - 1 - j : j) * d.channels + c;
    d.state[at] = h;
    h = apply(d.A[at], d.B[at], h);
  }
}

// Samples without tokens: their states go through. Workgroups behind the last
// chunk's, 64 samples by a tile of 64 channels each.
__device__ inline void empty_samples(const Scan& d, int64_t block, int32_t tiles64, const float* from, float* to) {
  const int32_t tile = int32_t(block % tiles64);
  const int32_t c = tile * 64 + int32_t(threadIdx.x & 63);
  const int64_t s0 = block / tiles64 * 64;
  if (c >= d.channels) return;
  for (int64_t s = s0 + (threadIdx.x >> 6); s < s0 + 64 && s < d.n; s += kWaves)
    if (d.start[s] >= d.start[s + 1]) to[s * d.channels + c] = from ? from[s * d.channels + c] : 0.0f;
}

template <class E>
__global__ void __launch_bounds__(64 * kWaves) gs_forward(const Scan d, uint32_t blocks) {
  constexpr int kN = kChannels<E>;
  __shared__ Marks marks;
  __shared__ float As[kWaves][64 * kN], Bs[kWaves][64 * kN];
  if (row_block() >= blocks) {
    const int32_t tiles64 = (d.channels + 63) / 64;
    if (d.last) empty_samples(d, row_block() - blocks, tiles64, d.h0, d.last);
    return;
  }
  const uint32_t chunk = row_block() / uint32_t(d.tiles), tile = row_block() % uint32_t(d.tiles);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t0 = int64_t(chunk) * kTile, total = tokens_of(d);
  const Cols<E> col = make_cols<E>(d, tile);
  const int64_t t = t0 + wave * kRows;
  const int rows = total <= t ? 0 : total - t < kRows ? int(total - t) : kRows;
  Pack<E, kN> x[kRows], g[kRows];
  load_rows<E>(d.x, d.x_stride, t, rows, col, x);
  load_rows<E>(d.gate, d.gate_stride, t, rows, col, g);
  float h[kN] = {};
  if (d.state) load_state<kN>(d.state, chunk, d, col.c, col.n, h);
  make_marks(d, t0, total, &marks);
  const uint32_t first = wave_marks(marks.first), end = wave_marks(marks.end);
  const int32_t* starts = marks.first + wave * kRows;
  {
    float A[kN], B[kN];
    forward_map<E>(d, x, g, rows, first, starts, col, A, B);
#pragma unroll
    for (int i = 0; i < kN; ++i) As[wave][lane * kN + i] = A[i], Bs[wave][lane * kN + i] = B[i];
  }
  __syncthreads();
  for (int w = 0; w < wave; ++w) {
#pragma unroll
    for (int i = 0; i < kN; ++i) h[i] = apply(As[w][lane * kN + i], Bs[w][lane * kN + i], h[i]);
  }
  const float none[kN] = {};
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (t + r >= d.T) break;
    if (r >= rows) {
      if (r == 0 && d.carry) store_state<kN>(d.carry, t / kRows, d, col.c, col.n, none);
      store_row<E>(d.h, d.h_stride, t + r, col, none);
      continue;
    }
    if (first >> r & 1) {
#pragma unroll
      for (int i = 0; i < kN; ++i) h[i] = 0.0f;
      if (d.h0) load_state<kN>(d.h0, starts[r] - 1, d, col.c, col.n, h);
    }
    if (r == 0 && d.carry) store_state<kN>(d.carry, t / kRows, d, col.c, col.n, h);
#pragma unroll
    for (int i = 0; i < kN; ++i) h[i] = step(share_of(g[r].get(i)), h[i], x[r].get(i));
    store_row<E>(d.h, d.h_stride, t + r, col, h);
    if ((end >> r & 1) && d.last)
      store_state<kN>(d.last, marks.end[wave * kRows + r] - 1, d, col.c, col.n, h);
  }
}

// The map of a wave's rows backwards: R behind its last row to R before its first.
template <class E>
__device__ __forceinline__ void backward_map(const Scan& d, const Pack<E, kChannels<E>> (&g)[kRows],
                                             const Pack<E, kChannels<E>> (&dh)[kRows], int rows, uint32_t end,
                                             const int32_t* samples, const Cols<E>& col, float (&A)[kChannels<E>],
                                             float (&B)[kChannels<E>]) {
  constexpr int kN = kChannels<E>;
#pragma unroll
  for (int i = 0; i < kN; ++i) A[i] = 1.0f, B[i] = 0.0f;
#pragma unroll
  for (int r = kRows - 1; r >= 0; --r) {
    if (r >= rows) continue;
    if (end >> r & 1) {
#pragma unroll
      for (int i = 0; i < kN; ++i) A[i] = kReset, B[i] = 0.0f;
      if (d.dlast) load_state<kN>(d.dlast, samples[r] - 1, d, col.c, col.n, B);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float share = share_of(g[r].get(i));
      B[i] = decay(share, dh[r].get(i) + B[i]);
      A[i] = A[i] < 0.0f ? A[i] : A[i] * a_of(share);
    }
  }
}

template <class E>
__global__ void __launch_bounds__(64 * kWaves) gs_grad_sums(const Scan d) {
  constexpr int kN = kChannels<E>;
  __shared__ Marks marks;
  __shared__ float As[kWaves][64 * kN], Bs[kWaves][64 * kN];
  const uint32_t chunk = row_block() / uint32_t(d.tiles), tile = row_block() % uint32_t(d.tiles);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t0 = int64_t(chunk) * kTile, total = tokens_of(d);
  if (t0 >= d.T) return;
  const Cols<E> col = make_cols<E>(d, tile);
  const int64_t t = t0 + wave * kRows;
  const int rows = total <= t ? 0 : total - t < kRows ? int(total - t) : kRows;
  Pack<E, kN> g[kRows], dh[kRows];
  load_rows<E>(d.gate, d.gate_stride, t, rows, col, g);
  load_rows<E>(d.dh, d.dh_stride, t, rows, col, dh);
  make_marks(d, t0, total, &marks);
  float A[kN], B[kN];
  backward_map<E>(d, g, dh, rows, wave_marks(marks.end), marks.end + wave * kRows, col, A, B);
#pragma unroll
  for (int i = 0; i < kN; ++i) As[wave][lane * kN + i] = A[i], Bs[wave][lane * kN + i] = B[i];
  __syncthreads();
  if (wave != kWaves - 1) return;
  for (int w = kWaves - 2; w >= 0; --w) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float a = As[w][lane * kN + i], b = Bs[w][lane * kN + i];
      B[i] = apply(a, b, B[i]);
      A[i] = a < 0.0f ? kReset : A[i] < 0.0f ? A[i] : A[i] * a;
    }
  }
  store_state<kN>(d.A, chunk, d, col.c, col.n, A);
  store_state<kN>(d.B, chunk, d, col.c, col.n, B);
}

template <class E>
__global__ void __launch_bounds__(64 * kWaves) gs_grad(const Scan d, uint32_t blocks) {
  constexpr int kN = kChannels<E>;
  __shared__ Marks marks;
  __shared__ float As[kWaves][64 * kN], Bs[kWaves][64 * kN];
  if (row_block() >= blocks) {
    const int32_t tiles64 = (d.channels + 63) / 64;
    if (d.dh0) empty_samples(d, row_block() - blocks, tiles64, d.dlast, d.dh0);
    return;
  }
  const uint32_t chunk = row_block() / uint32_t(d.tiles), tile = row_block() % uint32_t(d.tiles);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t0 = int64_t(chunk) * kTile, total = tokens_of(d);
  const Cols<E> col = make_cols<E>(d, tile);
  const int64_t t = t0 + wave * kRows;
  const int rows = total <= t ? 0 : total - t < kRows ? int(total - t) : kRows;
  Pack<E, kN> x[kRows], g[kRows], dh[kRows];
  load_rows<E>(d.x, d.x_stride, t, rows, col, x);
  load_rows<E>(d.gate, d.gate_stride, t, rows, col, g);
  load_rows<E>(d.dh, d.dh_stride, t, rows, col, dh);
  float h[kN] = {}, R[kN] = {};
  if (rows > 0) load_state<kN>(d.carry_in, t / kRows, d, col.c, col.n, h);
  if (d.state) load_state<kN>(d.state, chunk, d, col.c, col.n, R);
  make_marks(d, t0, total, &marks);
  const uint32_t first = wave_marks(marks.first), end = wave_marks(marks.end);
  const int32_t *starts = marks.first + wave * kRows, *ends = marks.end + wave * kRows;
  {
    float A[kN], B[kN];
    backward_map<E>(d, g, dh, rows, end, ends, col, A, B);
#pragma unroll
    for (int i = 0; i < kN; ++i) As[wave][lane * kN + i] = A[i], Bs[wave][lane * kN + i] = B[i];
  }
  float share[kRows][kN], under[kRows][kN];  // under: h_{t-1} - x_t
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (r >= rows) continue;
    if (r > 0 && (first >> r & 1)) {
#pragma unroll
      for (int i = 0; i < kN; ++i) h[i] = 0.0f;
      if (d.h0) load_state<kN>(d.h0, starts[r] - 1, d, col.c, col.n, h);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      share[r][i] = share_of(g[r].get(i));
      under[r][i] = h[i] - x[r].get(i);
      h[i] = step(share[r][i], h[i], x[r].get(i));
    }
  }
  __syncthreads();
  for (int w = kWaves - 1; w > wave; --w) {
#pragma unroll
    for (int i = 0; i < kN; ++i) R[i] = apply(As[w][lane * kN + i], Bs[w][lane * kN + i], R[i]);
  }
#pragma unroll
  for (int r = kRows - 1; r >= 0; --r) {
    if (t + r >= d.T) continue;
    float dx[kN] = {}, dg[kN] = {};
    if (r < rows) {
      if (end >> r & 1) {
#pragma unroll
        for (int i = 0; i < kN; ++i) R[i] = 0.0f;
        if (d.dlast) load_state<kN>(d.dlast, ends[r] - 1, d, col.c, col.n, R);
      }
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const float G = dh[r].get(i) + R[i];
        R[i] = decay(share[r][i], G);
        dx[i] = k_of(share[r][i]) * G;
        dg[i] = a_of(share[r][i]) * under[r][i] * dx[i];
      }
      if ((first >> r & 1) && d.dh0) store_state<kN>(d.dh0, starts[r] - 1, d, col.c, col.n, R);
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
struct Grid {
  int64_t chunks, blocks, all;
};
int make_grid(const nopfs_scan* p, bool states, Scan* d, Grid* g) {
  const int per = 64 * (p->dtype == NOPFS_FP32 ? 1 : 2);
  d->tiles = int32_t(ceil_div(p->channels, per));
  g->chunks = ceil_div(p->T, kTile);
  g->blocks = g->chunks * d->tiles;
  g->all = g->blocks + (states ? ceil_div(p->n, 64) * ceil_div(p->channels, 64) : 0);
  if (g->all > INT32_MAX) return fail(NOPFS_ERANGE, "too many tokens, samples and channels for one call");
  return NOPFS_OK;
}

int alloc_maps(Scratch* sc, const Grid& g, Scan* d) {
  if (g.chunks <= 1) return NOPFS_OK;
  const size_t n = size_t(g.chunks) * size_t(d->channels);
  int rc;
  if ((rc = step_alloc(sc, &d->A, n)) || (rc = step_alloc(sc, &d->B, n)) || (rc = step_alloc(sc, &d->state, n)))
    return rc;
  return NOPFS_OK;
}

Scan describe(const nopfs_scan* p) {
  Scan d{};
  d.T = p->T, d.n = p->n, d.channels = p->channels;
  d.x_stride = p->x_stride, d.gate_stride = p->gate_stride, d.h_stride = p->h_stride;
  d.dh_stride = p->dh_stride, d.dx_stride = p->dx_stride, d.dgate_stride = p->dgate_stride;
  return d;
}

int scan_impl(const nopfs_scan* p, const void* x, const void* gate, const int32_t* start, const float* h0, void* h,
              float* last, float* carry, hipStream_t st) {
  int rc = check(p, false);
  if (rc) return rc;
  if (!start || (p->T > 0 && (!x || !gate || !h))) return fail(NOPFS_EINVAL, "x, gate, start and h must be non-NULL");
  if (last && last == h0) return fail(NOPFS_EINVAL, "last must not be h0");
  Scan d = describe(p);
  d.x = x, d.gate = gate, d.start = start, d.h0 = h0, d.h = h, d.last = last, d.carry = carry;
  Grid g;
  if ((rc = make_grid(p, last != nullptr, &d, &g))) return rc;
  Scratch sc(st);
  if ((rc = alloc_maps(&sc, g, &d))) return rc;
  return by_dtype(p->dtype, [&](auto e) {
    typedef decltype(e) E;
    int r = NOPFS_OK;
    if (g.chunks > 1) {
      r = launch("gs_sums", gs_sums<E>, row_grid(g.blocks), dim3(64 * kWaves), 0, st, d);
      if (!r)
        r = launch("gs_states", gs_states<false>, dim3(uint32_t(ceil_div(d.channels, 64))), dim3(64), 0, st, d,
                   int32_t(g.chunks));
    }
    if (r) return r;
    return launch("gs_forward", gs_forward<E>, row_grid(g.all), dim3(64 * kWaves), 0, st, d, uint32_t(g.blocks));
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
  Scan d = describe(p);
  d.dh = dh, d.dlast = dlast, d.x = x, d.gate = gate, d.start = start, d.h0 = h0, d.carry_in = carry;
  d.dx = dx, d.dgate = dgate, d.dh0 = dh0;
  Grid g;
  if ((rc = make_grid(p, dh0 != nullptr, &d, &g))) return rc;
  Scratch sc(st);
  if ((rc = alloc_maps(&sc, g, &d))) return rc;
  return by_dtype(p->dtype, [&](auto e) {
    typedef decltype(e) E;
    int r = NOPFS_OK;
    if (g.chunks > 1) {
      r = launch("gs_grad_sums", gs_grad_sums<E>, row_grid(g.blocks), dim3(64 * kWaves), 0, st, d);
      if (!r)
        r = launch("gs_states", gs_states<true>, dim3(uint32_t(ceil_div(d.channels, 64))), dim3(64), 0, st, d,
                   int32_t(g.chunks));
    }
    if (r) return r;
    return launch("gs_grad", gs_grad<E>, row_grid(g.all), dim3(64 * kWaves), 0, st, d, uint32_t(g.blocks));
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
