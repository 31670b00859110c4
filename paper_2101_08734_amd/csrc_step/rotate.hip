// nopfs_norm_rotate and its gradient: root-mean-square norms of queries and keys
// per head, with the rotation by position in the same pass. Per head x of width W
// at position p, with r = (mean x_i^2 + eps)^(-1/2), z = x r, y = z w, and for
// each pair (a, b) of the rotated elements the angle p f:
//     out_a = y_a cos - y_b sin,   out_b = y_b cos + y_a sin
// and back, with g the gradient turned by the opposite angles:
//     dx = r (g w - z mean(g w z)),   dw = sum g z
// Bound by memory: a head is read once and written once (the gradient reads the
// input and the output's gradient): 65,536 tokens, 32 on 8 heads of 128 in bf16 258 us a
// call, 5.2 TB/s, the rate of a large copy (271 us, 4.95 TB/s, in a kernel trace); 16,384
// tokens, 16 on 4 heads 44 us, the gradient 59 and 5 for the weights, with vector units at
// 57-61%; the same in fp32 63 us, 5.3 TB/s, and 106, 4.7. Few or narrow heads leave lanes
// idle, as a wave has a token: 90,000 tokens of one query and one key head of 64 in bf16 67
// and 75 us, 0.7 and 0.9 TB/s. Statistics, angles and sums are in 32 bits or more; outputs
// are rounded once.
#include "rows.hpp"

namespace nopfs {
namespace {

constexpr int kVec = 4;            // elements of a head per lane
constexpr int kMostPairs = 128;    // of a head
constexpr int kWaves = 4;          // of a workgroup

struct Rotate {
  int64_t T;
  int32_t heads, kv_heads, width, rotated, interleaved;
  int32_t tok;  // tokens that a workgroup has at a time: kWaves, or 1 (its waves share the heads)
  float eps;
  const int32_t* pos;
  const double* freq;
  const void *q_weight, *k_weight;
  int32_t weight_dtype;
};
struct Side {  // q or k: pointers and strides by token and head
  const void *x, *d;  // the input; the output's gradient
  void* out;          // the output; the input's gradient
  int64_t x_stride[2], d_stride[2], out_stride[2];
};

__device__ inline float weight_at(const void* w, int32_t dtype, int i) {
  if (!w) return 1.0f;
  switch (dtype) {
    case NOPFS_BF16: return float(static_cast<const Bf16::T*>(w)[i]);
    case NOPFS_FP16: return float(static_cast<const Fp16::T*>(w)[i]);
    default: return static_cast<const float*>(w)[i];
  }
}

// Sine and cosine of the angles of `tok` tokens from t0, by all threads. An angle
// in turns is reduced in 64 bits, so that far positions keep 32 bits of theirs; what its
// rounding to 32 bits leaves, up to 2^-26 turns, turns them a little further.
__device__ inline void make_angles(const Rotate& d, int64_t t0, float2 (*cs)[kMostPairs]) {
  const int pairs = d.rotated >> 1;
  for (int i = threadIdx.x; i < d.tok * pairs; i += 64 * kWaves) {
    const int k = i / pairs, f = i - k * pairs;
    const int32_t p = t0 + k < d.T ? d.pos[t0 + k] : -1;
    if (p < 0) continue;
    double turns = double(p) * (d.freq[f] * 0.15915494309189533577);
    turns -= rint(turns);
    const float near = float(turns), rest = float((turns - double(near)) * 6.28318530717958647693);
    float s, c;
    sincospif(2.0f * near, &s, &c);
    cs[k][f] = make_float2(fmaf(-rest, s, c), fmaf(rest, c, s));
  }
}

// What a lane has to do with its elements e0 .. e0 + 3 of a head.
struct Lane {
  int e0, partner;  // the lane with the other halves of its pairs
  bool active, turned;
  float cos[kVec], sin[kVec];  // the sine with the sign of the partner's share
};

// kLanes lanes for a head, the least power of two that holds it.
template <int kLanes>
__device__ __forceinline__ Lane make_lane(const Rotate& d) {
  Lane l;
  const int lane = threadIdx.x & 63, j = lane & (kLanes - 1);
  l.e0 = j * kVec;
  l.active = l.e0 < d.width;
  l.turned = l.e0 < d.rotated;
  l.partner = lane;
  if (l.turned && !d.interleaved) {
    const int half = d.rotated / (2 * kVec);  // in lanes
    l.partner = j < half ? lane + half : lane - half;
  }
  return l;
}
// kBack: by the opposite angles
template <bool kBack>
__device__ __forceinline__ void set_angles(const Rotate& d, const float2* cs, Lane* l) {
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    l->cos[e] = 1.0f;
    l->sin[e] = 0.0f;
    if (!l->turned) continue;
    const int i = l->e0 + e, half = d.rotated >> 1;
    const bool first = d.interleaved ? !(e & 1) : i < half;
    const float2 a = cs[d.interleaved ? i >> 1 : first ? i : i - half];
    l->cos[e] = a.x;
    l->sin[e] = first != kBack ? -a.y : a.y;
  }
}
__device__ __forceinline__ void turn(const Rotate& d, const Lane& l, float (&y)[kVec]) {
  float other[kVec];
#pragma unroll
  for (int e = 0; e < kVec; ++e) other[e] = d.interleaved ? y[e ^ 1] : __shfl(y[e], l.partner);
  if (l.turned) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) y[e] = y[e] * l.cos[e] + other[e] * l.sin[e];
  }
}

// z = x r of a head by its lanes, and r as two factors. Squares that overflow are
// taken again of x 2^-70 (32 bits' exponents only).
template <class E, int kLanes>
__device__ __forceinline__ void normalize(const Rotate& d, const Pack<E, kVec>& x, float (&z)[kVec], float* r1,
                                          float* r2) {
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    z[e] = x.get(e);
    s += z[e] * z[e];
  }
  s = group_sum<kLanes>(s);
  const float by_width = 1.0f / float(d.width);
  float eps = d.eps, small = 1.0f;
  if (E::kBits != 11 && s > 0x1p120f) {
    small = 0x1p-70f;
    eps = eps * small * small;
    s = 0.0f;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      z[e] *= small;
      s += z[e] * z[e];
    }
    s = group_sum<kLanes>(s);
  }
  const float m = s * by_width + eps;
  float r = __builtin_amdgcn_rsqf(m);
  if (m != INFINITY) r = r * (1.5f - 0.5f * m * r * r);
#pragma unroll
  for (int e = 0; e < kVec; ++e) z[e] *= r;
  *r1 = r;
  *r2 = small;
}

template <class E, int kLanes>
__device__ __forceinline__ void forward_heads(const Rotate& d, const Side& side, int32_t heads, int64_t t, bool there,
                                              int part, int parts, const Lane& l, const float (&w)[kVec]) {
  constexpr int kSlots = 64 / kLanes, kDeep = 4;  // heads at a time, and so many times
  typedef typename E::T T;
  const int slot = (threadIdx.x & 63) / kLanes;
  const T* x = static_cast<const T*>(side.x) + t * side.x_stride[0] + l.e0;
  T* out = static_cast<T*>(side.out) + t * side.out_stride[0] + l.e0;
  for (int32_t h0 = part * kSlots; h0 < heads; h0 += parts * kSlots * kDeep) {
    Pack<E, kVec> v[kDeep];
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      const int32_t h = h0 + j * parts * kSlots + slot;
      v[j].zero();
      if (there && l.active && h < heads) v[j].load(x + h * side.x_stride[1]);
    }
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      if (h0 + j * parts * kSlots >= heads) break;
      const int32_t h = h0 + j * parts * kSlots + slot;
      float y[kVec] = {}, r1, r2;
      if (there) {
        normalize<E, kLanes>(d, v[j], y, &r1, &r2);
#pragma unroll
        for (int e = 0; e < kVec; ++e) y[e] *= w[e];
        turn(d, l, y);
      }
      Pack<E, kVec> o;
      o.set(y);
      if (l.active && h < heads) o.store(out + h * side.out_stride[1]);
    }
  }
}

template <class E, int kLanes>
__global__ void __launch_bounds__(64 * kWaves) nr_forward(const Rotate d, const Side q, const Side k) {
  __shared__ float2 cs[kWaves][kMostPairs];
  const int64_t t0 = int64_t(row_block()) * d.tok;
  if (t0 >= d.T) return;
  const int wave = threadIdx.x >> 6, mine = d.tok == 1 ? 0 : wave;
  make_angles(d, t0, cs);
  Lane l = make_lane<kLanes>(d);
  float wq[kVec], wk[kVec];
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    wq[e] = l.active ? weight_at(d.q_weight, d.weight_dtype, l.e0 + e) : 0.0f;
    wk[e] = l.active ? weight_at(d.k_weight, d.weight_dtype, l.e0 + e) : 0.0f;
  }
  __syncthreads();
  const int64_t t = t0 + mine;
  if (t >= d.T) return;
  const bool there = d.pos[t] >= 0;
  if (there) set_angles<false>(d, cs[mine], &l);
  const int part = d.tok == 1 ? wave : 0, parts = d.tok == 1 ? kWaves : 1;
  forward_heads<E, kLanes>(d, q, d.heads, t, there, part, parts, l, wq);
  forward_heads<E, kLanes>(d, k, d.kv_heads, t, there, part, parts, l, wk);
}

template <class E, int kLanes>
__device__ __forceinline__ void grad_heads(const Rotate& d, const Side& side, int32_t heads, int64_t t, bool there,
                                           int part, int parts, const Lane& l, const float (&w)[kVec],
                                           float (&dw)[kVec]) {
  constexpr int kSlots = 64 / kLanes, kDeep = 4;
  typedef typename E::T T;
  const int slot = (threadIdx.x & 63) / kLanes;
  const T* x = static_cast<const T*>(side.x) + t * side.x_stride[0] + l.e0;
  const T* g = static_cast<const T*>(side.d) + t * side.d_stride[0] + l.e0;
  T* out = static_cast<T*>(side.out) + t * side.out_stride[0] + l.e0;
  const float by_width = 1.0f / float(d.width);
  float sum[kVec] = {};  // of the token
  for (int32_t h0 = part * kSlots; h0 < heads; h0 += parts * kSlots * kDeep) {
    Pack<E, kVec> v[kDeep], u[kDeep];
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      const int32_t h = h0 + j * parts * kSlots + slot;
      v[j].zero();
      u[j].zero();
      if (there && l.active && h < heads) {
        v[j].load(x + h * side.x_stride[1]);
        u[j].load(g + h * side.d_stride[1]);
      }
    }
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      if (h0 + j * parts * kSlots >= heads) break;
      const int32_t h = h0 + j * parts * kSlots + slot;
      float y[kVec] = {};
      if (there) {
        float z[kVec], r1, r2;
        normalize<E, kLanes>(d, v[j], z, &r1, &r2);
#pragma unroll
        for (int e = 0; e < kVec; ++e) y[e] = u[j].get(e);
        turn(d, l, y);
        float dot = 0.0f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          sum[e] += y[e] * z[e];
          y[e] *= w[e];
          dot += y[e] * z[e];
        }
        dot = group_sum<kLanes>(dot) * by_width;
#pragma unroll
        for (int e = 0; e < kVec; ++e) y[e] = (y[e] - z[e] * dot) * r1 * r2;
      }
      Pack<E, kVec> o;
      o.set(y);
      if (l.active && h < heads) o.store(out + h * side.out_stride[1]);
    }
  }
#pragma unroll
  for (int e = 0; e < kVec; ++e) dw[e] += sum[e];
}

// A workgroup has every gridDim.x-th group of tokens; its sums of the weights'
// gradients go to part[workgroup][2][width]. A lane's are over a token's heads, of kRun
// tokens, and of those, so that no long chain of roundings goes through one sum.
constexpr int kRun = 64;
template <class E, int kLanes>
__global__ void __launch_bounds__(64 * kWaves) nr_grad(const Rotate d, const Side q, const Side k, float* part_sums) {
  __shared__ float2 cs[2][kWaves][kMostPairs];
  __shared__ float sums[2][kWaves][64][kVec];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, mine = d.tok == 1 ? 0 : wave;
  Lane l = make_lane<kLanes>(d);
  float wq[kVec], wk[kVec], dq[kVec] = {}, dk[kVec] = {}, all_q[kVec] = {}, all_k[kVec] = {};
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    wq[e] = l.active ? weight_at(d.q_weight, d.weight_dtype, l.e0 + e) : 0.0f;
    wk[e] = l.active ? weight_at(d.k_weight, d.weight_dtype, l.e0 + e) : 0.0f;
  }
  const int part = d.tok == 1 ? wave : 0, parts = d.tok == 1 ? kWaves : 1;
  int which = 0, run = 0;
  for (int64_t t0 = int64_t(blockIdx.x) * d.tok; t0 < d.T; t0 += int64_t(gridDim.x) * d.tok, which ^= 1) {
    if (run++ == kRun) {
      run = 1;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        all_q[e] += dq[e], all_k[e] += dk[e];
        dq[e] = dk[e] = 0.0f;
      }
    }
    make_angles(d, t0, cs[which]);  // the other half may still be read
    __syncthreads();
    const int64_t t = t0 + mine;
    if (t >= d.T) continue;
    const bool there = d.pos[t] >= 0;
    if (there) set_angles<true>(d, cs[which][mine], &l);
    grad_heads<E, kLanes>(d, q, d.heads, t, there, part, parts, l, wq, dq);
    grad_heads<E, kLanes>(d, k, d.kv_heads, t, there, part, parts, l, wk, dk);
  }
  if (!part_sums) return;
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    sums[0][wave][lane][e] = all_q[e] + dq[e];
    sums[1][wave][lane][e] = all_k[e] + dk[e];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * d.width; i += 64 * kWaves) {
    const int side = i >= d.width, e = i - side * d.width;
    float s = 0.0f;
    for (int w = 0; w < kWaves; ++w) {
      float of_wave = 0.0f;
      for (int slot = 0; slot < 64 / kLanes; ++slot)
        of_wave += sums[side][w][slot * kLanes + e / kVec][e & (kVec - 1)];
      s += of_wave;
    }
    part_sums[int64_t(blockIdx.x) * 2 * d.width + i] = s;
  }
}

// The workgroups' sums, in a fixed order: 16 columns by 64 rows of threads, then the
// four rows of a wave, and the waves four by four.
__global__ void __launch_bounds__(1024) nr_weights(const float* part_sums, int32_t n, int32_t width, int32_t dtype,
                                                   void* dq, void* dk) {
  constexpr int kDeep = 16;  // in flight
  __shared__ float sums[16][17];
  const int c = threadIdx.x & 15, row = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + c;  // 2 width is a multiple of 16
  float s = 0.0f;
  for (int32_t i = row; i < n; i += 64 * kDeep) {
    float x[kDeep];
#pragma unroll
    for (int j = 0; j < kDeep; ++j)
      x[j] = i + 64 * j < n ? part_sums[int64_t(i + 64 * j) * 2 * width + col] : 0.0f;
#pragma unroll
    for (int j = 0; j < kDeep; ++j) s += x[j];
  }
  s += __shfl_xor(s, 16);
  s += __shfl_xor(s, 32);
  if ((row & 3) == 0) sums[row >> 2][c] = s;
  __syncthreads();
  if (row) return;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; i += 4) s += (sums[i][c] + sums[i + 1][c]) + (sums[i + 2][c] + sums[i + 3][c]);
  void* to = col < width ? dq : dk;
  const int e = col < width ? col : col - width;
  if (!to) return;
  switch (dtype) {
    case NOPFS_BF16: static_cast<Bf16::T*>(to)[e] = Bf16::T(s); break;
    case NOPFS_FP16: static_cast<Fp16::T*>(to)[e] = Fp16::T(s); break;
    default: static_cast<float*>(to)[e] = s;
  }
}

int check_stride(const int64_t* s, int64_t T, int32_t heads, int32_t width) {
  if ((heads > 1 && s[1] < width) || (T > 1 && s[0] < width)) return fail(NOPFS_EINVAL, "tokens or heads overlap");
  // of token-major and head-major arrays alike, no two heads share an element
  if (T > 1 && heads > 1 && s[0] < s[1] * (heads - 1) + width && s[1] < s[0] * (T - 1) + width)
    return fail(NOPFS_EINVAL, "tokens and heads overlap");
  return NOPFS_OK;
}

int check(const nopfs_rotate* p, bool gradient) {
  if (!p) return fail(NOPFS_EINVAL, "rotate is NULL");
  if (p->T < 0 || p->heads < 1 || p->kv_heads < 1) return fail(NOPFS_EINVAL, "T must be >= 0, heads and kv_heads >= 1");
  if (p->width < 8 || p->width % 8) return fail(NOPFS_EINVAL, "width must be a positive multiple of 8");
  if (p->rotated < 0 || p->rotated % 8 || p->rotated > p->width)
    return fail(NOPFS_EINVAL, "rotated must be a multiple of 8 in 0 .. width");
  if (p->interleaved != 0 && p->interleaved != 1) return fail(NOPFS_EINVAL, "interleaved must be 0 or 1");
  if (!is_dtype(p->dtype) || !is_dtype(p->weight_dtype)) return fail(NOPFS_EINVAL, "unknown dtype");
  if (!(p->eps > 0.0f) || !isfinite(p->eps)) return fail(NOPFS_EINVAL, "eps must be positive and finite");
  if (p->eps < 0x1p-60f || p->eps > 0x1p60f) return fail(NOPFS_ERANGE, "eps must be in 2^-60 .. 2^60");
  if (p->width > 2 * kMostPairs) return fail(NOPFS_ERANGE, "width must be <= 256");
  if (p->T > INT32_MAX || p->heads > 1 << 16 || p->kv_heads > 1 << 16)
    return fail(NOPFS_ERANGE, "T must be < 2^31, heads and kv_heads <= 2^16");
  for (const int64_t* s : {p->q_stride, p->k_stride, p->q_out_stride, p->k_out_stride, p->dq_stride, p->dk_stride}) {
    if (!gradient && (s == p->dq_stride || s == p->dk_stride)) continue;
    for (int i = 0; i < 2; ++i) {
      if (s[i] < 0) return fail(NOPFS_EINVAL, "strides must not be negative");
      if (s[i] > int64_t(1) << 30) return fail(NOPFS_ERANGE, "strides must be <= 2^30");
    }
    const bool is_q = s == p->q_stride || s == p->q_out_stride || s == p->dq_stride;
    const int rc = check_stride(s, p->T, is_q ? p->heads : p->kv_heads, p->width);
    if (rc) return rc;
  }
  return NOPFS_OK;
}

// A workgroup's tokens: one per wave, so that an angle is made once and serves all
// heads (16,384 tokens, 16 on 4 heads of 128 in bf16: 42 us, gradient 56; one per workgroup
// 68 and 84), except for few tokens (32: 8.5 us, one per workgroup 5.6).
Rotate describe(const nopfs_rotate* p, const int32_t* pos, const double* freq, const void* qw, const void* kw) {
  return {p->T, p->heads, p->kv_heads, p->width, p->rotated, p->interleaved, p->T <= 1024 ? 1 : kWaves,
          p->eps, pos, freq, qw, kw, p->weight_dtype};
}

Side make_side(const void* x, const int64_t* xs, const void* d, const int64_t* ds, void* out, const int64_t* os) {
  return {x, d, out, {xs[0], xs[1]}, {ds[0], ds[1]}, {os[0], os[1]}};
}

template <class F>
int by_lanes(int32_t width, F f) {
  switch (log2_ceil(width / kVec)) {
    case 1: return f(std::integral_constant<int, 2>());
    case 2: return f(std::integral_constant<int, 4>());
    case 3: return f(std::integral_constant<int, 8>());
    case 4: return f(std::integral_constant<int, 16>());
    case 5: return f(std::integral_constant<int, 32>());
    default: return f(std::integral_constant<int, 64>());
  }
}

int rotate_impl(const nopfs_rotate* p, const void* q, const void* k, const int32_t* pos, const double* freq,
                const void* qw, const void* kw, void* q_out, void* k_out, hipStream_t st) {
  const int rc = check(p, false);
  if (rc) return rc;
  if (p->T == 0) return NOPFS_OK;
  if (!q || !k || !pos || !q_out || !k_out || (p->rotated > 0 && !freq))
    return fail(NOPFS_EINVAL, "q, k, pos, freq, q_out and k_out must be non-NULL");
  const Rotate d = describe(p, pos, freq, qw, kw);
  const Side sq = make_side(q, p->q_stride, nullptr, p->q_stride, q_out, p->q_out_stride);
  const Side sk = make_side(k, p->k_stride, nullptr, p->k_stride, k_out, p->k_out_stride);
  return by_dtype(p->dtype, [&](auto e) {
    return by_lanes(p->width, [&](auto lanes) {
      return launch("nr_forward", nr_forward<decltype(e), decltype(lanes)::value>, row_grid(ceil_div(p->T, d.tok)),
                    dim3(64 * kWaves), 0, st, d, sq, sk);
    });
  });
}

// Workgroups of the gradient, each with sums of its own to be added up.
constexpr int64_t kMostParts = 1024;

int rotate_grad_impl(const nopfs_rotate* p, const void* dqo, const void* dko, const void* q, const void* k,
                     const int32_t* pos, const double* freq, const void* qw, const void* kw, void* dq, void* dk,
                     void* dqw, void* dkw, hipStream_t st) {
  int rc = check(p, true);
  if (rc) return rc;
  if (p->T > 0 && (!dqo || !dko || !q || !k || !pos || !dq || !dk || (p->rotated > 0 && !freq)))
    return fail(NOPFS_EINVAL, "the gradients, q, k, pos and freq must be non-NULL");
  const Rotate d = describe(p, pos, freq, qw, kw);
  const Side sq = make_side(q, p->q_stride, dqo, p->q_out_stride, dq, p->dq_stride);
  const Side sk = make_side(k, p->k_stride, dko, p->k_out_stride, dk, p->dk_stride);
  const int64_t parts = std::min(kMostParts, ceil_div(p->T, d.tok));
  const bool weights = dqw || dkw;
  Scratch sc(st);
  float* sums = nullptr;
  if (weights && (rc = step_alloc(&sc, &sums, size_t(std::max<int64_t>(parts, 1)) * 2 * p->width))) return rc;
  rc = by_dtype(p->dtype, [&](auto e) {
    return by_lanes(p->width, [&](auto lanes) {
      return launch("nr_grad", nr_grad<decltype(e), decltype(lanes)::value>, dim3(uint32_t(parts)), dim3(64 * kWaves),
                    0, st, d, sq, sk, sums);
    });
  });
  if (rc || !weights) return rc;
  return launch("nr_weights", nr_weights, dim3(uint32_t(2 * p->width / 16)), dim3(1024), 0, st, sums, int32_t(parts),
                p->width, p->weight_dtype, dqw, dkw);
}

}  // namespace
}  // namespace nopfs

using namespace nopfs;

extern "C" int nopfs_norm_rotate(const nopfs_rotate* r, const void* q, const void* k, const int32_t* pos,
                                 const double* freq, const void* q_weight, const void* k_weight, void* q_out,
                                 void* k_out, void* hip_stream) {
  try {
    return rotate_impl(r, q, k, pos, freq, q_weight, k_weight, q_out, k_out, static_cast<hipStream_t>(hip_stream));
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_norm_rotate_grad(const nopfs_rotate* r, const void* d_q_out, const void* d_k_out, const void* q,
                                      const void* k, const int32_t* pos, const double* freq, const void* q_weight,
                                      const void* k_weight, void* d_q, void* d_k, void* d_q_weight, void* d_k_weight,
                                      void* hip_stream) {
  try {
    auto call = [&]() {
      return rotate_grad_impl(r, d_q_out, d_k_out, q, k, pos, freq, q_weight, k_weight, d_q, d_k, d_q_weight,
                              d_k_weight, static_cast<hipStream_t>(hip_stream));
    };
    return r ? run_with_scratch(r->scratch, r->scratch_bytes, call) : call();
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}

extern "C" int nopfs_norm_rotate_scratch(const nopfs_rotate* r, int64_t* bytes) {
  try {
    void* x = no_array();
    return scratch_size(bytes, [&]() {
      return rotate_grad_impl(r, x, x, x, x, static_cast<int32_t*>(x), static_cast<double*>(x), x, x, x, x, x, x,
                              nullptr);
    });
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}
