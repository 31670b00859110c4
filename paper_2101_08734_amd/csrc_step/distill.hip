// nopfs_topk_distill: loss and gradient against a teacher's top logits.
//
// Per row (token) with logits s[V], teacher logits y at classes x, temperature
// tau and weight w, over the valid teacher entries (0 <= x_k < V):
//     p = softmax(y / tau),  z = log sum_v exp(s_v / tau)
//     loss  = w tau^2 sum_k p_k (log p_k - s[x_k] / tau + z)
//     ds_v  = w tau (exp(s_v / tau - z) - sum_{k: x_k = v} p_k)
// One workgroup per row, bound by memory: a row is read once and its gradient
// written once (8,192 rows of 32,768 classes in bf16, a tenth of them masked: 1.02
// GB in 220 us, 4.6 TB/s; a large copy reaches 4.9 here), except that rows too
// long for one workgroup's registers are read twice, and that many teacher entries
// take longer than the row: a class named twice is looked for among all others, K^2
// comparisons (8,192 rows without a mask: of 32,768 classes 239 us with 64 entries, 261
// with 128, 506 with 512, 1,246 with 1,024; of 2,048 classes 26, 41, 468, 3,301).
// Maxima, sums, probabilities and the loss are held in 32 bits; the gradient is
// rounded once, at the store.
#include "step.hpp"

namespace nopfs {
namespace {

struct Distill {
  int64_t T, V, logits_stride, grad_stride, index_stride, teacher_stride;
  int32_t K;
  float tau;
  const void* logits;
  const int32_t* index;
  const void* teacher;
  const float* weight;
  float* loss;
  void* grad;
};

constexpr int32_t kMaxTop = 1024;  // teacher entries per row held in LDS
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -INFINITY;
constexpr float kFusedMost = 0x1p20f;

__device__ inline float wave_max(float v) {
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ inline float wave_sum(float v) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Over the workgroup, the same in every thread. `tmp`: a slot per wave, not
// used by the reduction before this one (no barrier closes it).
template <int kThreads, bool kMax>
__device__ inline float block_reduce(float v, float* tmp) {
  v = kMax ? wave_max(v) : wave_sum(v);
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  v = tmp[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) v = kMax ? fmaxf(v, tmp[i]) : v + tmp[i];
  return v;
}

// 16 bytes of a row. Rows begin anywhere (an odd number of classes), so the
// type in memory claims its elements' alignment only; the hardware takes such
// loads and stores whole.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_by2 __attribute__((aligned(2)));

template <class E>
struct Packed {
  static constexpr bool kWide = sizeof(typename E::T) == 4;
  static constexpr int kN = kWide ? 4 : 8;  // elements of 16 bytes
  typedef typename E::T V2 __attribute__((ext_vector_type(2)));
  static constexpr uint32_t kLowest = kWide ? 0xFF800000u : E::kBits == 8 ? 0xFF80FF80u : 0xFC00FC00u;  // -inf
  static __device__ __forceinline__ float get(const u32x4& v, int e) {
    const uint32_t word = v[kWide ? e : e >> 1];  // by value: a bit_cast of a vector's element reads element 0
    if constexpr (kWide) return __uint_as_float(word);
    else if constexpr (E::kBits == 8) return __uint_as_float(e & 1 ? word & 0xFFFF0000u : word << 16);
    else return float(__builtin_bit_cast(V2, word)[e & 1]);
  }
  // elements 2 i and 2 i + 1 (one word) from a function of the element's index
  template <class F>
  static __device__ __forceinline__ u32x4 make(F f) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kWide) {
        v[i] = __float_as_uint(f(i));
      } else {
        const f32x2 x = {f(2 * i), f(2 * i + 1)};
        v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, V2));
      }
    }
    return v;
  }
};

// Makes the compiler forget what it knows of the held vectors, so that it
// unpacks the elements again in the next pass instead of keeping them unpacked
// from the last one, in twice the registers.
template <int kHold>
__device__ __forceinline__ void forget(u32x4* hold) {
#pragma unroll
  for (int j = 0; j < kHold; ++j) asm volatile("" : "+v"(hold[j]));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A maximum of nothing but -inf counts as 0 in differences from it: the
// exponentials are then 0, not NaN.
__device__ inline float finite_max(float m) { return m == kNegInf ? 0.0f : m; }

// The teacher's entries of a row, by one wave: their classes (-1: no entry),
// p and log p, and the logits of their classes.
struct Entries {
  float *p, *logp, *x;
  int32_t* id;
};
// Returns false where no entry has any mass; a NaN among them reaches all.
template <class E, class Y>
__device__ inline bool teacher_entries(const Distill& d, int64_t t, const typename E::T* s, const Entries& en) {
  const int lane = threadIdx.x & 63;
  const typename Y::T* y = static_cast<const typename Y::T*>(d.teacher) + t * d.teacher_stride;
  const int32_t* x = d.index + t * d.index_stride;
  const float inv_tau = 1.0f / d.tau;
  float top = kNegInf;
  for (int k = lane; k < d.K; k += 64) {
    const int32_t id = x[k];
    const float v = id >= 0 && id < d.V ? float(y[k]) : kNegInf;
    en.id[k] = v != kNegInf ? id : -1;
    en.p[k] = v;
    if (v != kNegInf) en.x[k] = float(s[id]);
    top = v == v ? fmaxf(top, v) : INFINITY;
  }
  top = wave_max(top);
  if (top == kNegInf) return false;
  float sum = 0.0f;
  for (int k = lane; k < d.K; k += 64) {
    const float v = (en.p[k] - top) * inv_tau;
    en.logp[k] = v;
    sum += expf(v);
  }
  sum = wave_sum(sum);
  const float lsum = logf(sum);
  for (int k = lane; k < d.K; k += 64) {
    const float v = en.logp[k];
    en.p[k] = en.id[k] >= 0 ? expf(v) / sum : 0.0f;
    en.logp[k] = v - lsum;
  }
  return true;
}

// A row by kThreads threads. kHold > 0: the row's 16-byte vectors stay in
// registers (kHold of each thread), so it is read once, its maximum m taken
// first, then its sum, then the gradient. kHold = 0: one pass for the running
// maximum and sum, and the row is read again for the gradient, if any.
//
// With c = log2(e) / tau the exponentials are exp2(c a - c m) in one fused
// multiply-add: c m is rounded once, so all of them carry the same factor,
// which cancels in q = e / sum and in log q: 2^(half a unit of c m), no more than
// 2^(1/32) up to c m = kFusedMost. Beyond (small temperatures, large logits, a
// maximum of +-inf) that factor would grow out of the floats' range, and they are
// exp2(c (a - m)).
template <class E, class Y, int kThreads, int kHold>
__global__ void __launch_bounds__(kThreads) td_row(const Distill d) {
  typedef typename E::T T;
  typedef Packed<E> P;
  constexpr int VE = P::kN;
  __shared__ float tmp[2 * kThreads / 64];
  __shared__ int s_any;
  extern __shared__ float lds[];  // 4 K
  const Entries en{lds, lds + d.K, lds + 2 * d.K, reinterpret_cast<int32_t*>(lds + 3 * d.K)};
  const int64_t t = row_block();
  if (t >= d.T) return;
  const int tid = threadIdx.x;
  const T* s = static_cast<const T*>(d.logits) + t * d.logits_stride;
  T* ds = d.grad ? static_cast<T*>(d.grad) + t * d.grad_stride : nullptr;
  const float w = d.weight ? d.weight[t] : 1.0f;
  const int64_t nv = d.V / VE;
  const int64_t end = nv * VE + tid;  // the thread's element behind the vectors, if below V
  const u32x4_by2* sv = reinterpret_cast<const u32x4_by2*>(s);
  u32x4_by2* dv = reinterpret_cast<u32x4_by2*>(ds);
  auto zero_row = [&]() {
    if (tid == 0) d.loss[t] = 0.0f;
    if (!ds) return;
    for (int64_t i = tid; i < nv; i += kThreads) dv[i] = u32x4{0, 0, 0, 0};
    if (end < d.V) ds[end] = T(0.0f);
  };
  if (w == 0.0f) return zero_row();  // nothing is learned from this row, whatever it holds

  auto load_masked = [&](int64_t i) -> u32x4 {
    u32x4 v = {P::kLowest, P::kLowest, P::kLowest, P::kLowest};  // adds nothing
    if (i < nv) v = sv[i];
    return v;
  };
  u32x4 hold[kHold > 0 ? kHold : 1];
#pragma unroll
  for (int j = 0; j < kHold; ++j) hold[j] = load_masked(tid + j * kThreads);
  const float last = end < d.V ? float(s[end]) : kNegInf;
  if (tid < 64) {
    const bool any = teacher_entries<E, Y>(d, t, s, en);
    if (tid == 0) s_any = any;
  }

  const float c = kLog2e / d.tau;
  float m, sum, cm = INFINITY;
  if constexpr (kHold > 0) {
    m = last;
#pragma unroll
    for (int j = 0; j < kHold; ++j)
      if (j * kThreads < nv) {
#pragma unroll
        for (int e = 0; e < VE; ++e) m = fmaxf(m, P::get(hold[j], e));
      }
    m = block_reduce<kThreads, true>(m, tmp);
    cm = c * m;
    forget<kHold>(hold);
    if (fabsf(cm) < kFusedMost) {
      sum = exp2_fast(fmaf(last, c, -cm));
#pragma unroll
      for (int j = 0; j < kHold; ++j)
        if (j * kThreads < nv) {
#pragma unroll
          for (int e = 0; e < VE; ++e) sum += exp2_fast(fmaf(P::get(hold[j], e), c, -cm));
        }
    } else {  // rare: element by element
      const float f = finite_max(m);
      sum = 0.0f;
      for (int64_t v = tid; v < d.V; v += kThreads) sum += exp2_fast((float(s[v]) - f) * c);
    }
  } else {
    float rm = kNegInf, rs = 0.0f;
    for (int64_t i = tid; i < nv; i += 4 * kThreads) {  // four loads in flight
      u32x4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = load_masked(i + j * kThreads);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float top = rm;
#pragma unroll
        for (int e = 0; e < VE; ++e) top = fmaxf(top, P::get(v[j], e));
        const float f = finite_max(top);
        rs *= exp2_fast((rm - f) * c);
#pragma unroll
        for (int e = 0; e < VE; ++e) rs += exp2_fast((P::get(v[j], e) - f) * c);
        rm = top;
      }
    }
    m = block_reduce<kThreads, true>(fmaxf(rm, last), tmp);
    const float f = finite_max(m);
    sum = rs * exp2_fast((rm - f) * c) + exp2_fast((last - f) * c);
  }
  sum = block_reduce<kThreads, false>(sum, tmp + kThreads / 64);
  if (!s_any) return zero_row();
  forget<kHold>(hold);

  const bool fused = fabsf(cm) < kFusedMost;  // the same in every thread
  const float wt = w * d.tau;
  if (tid < 64) {
    const float z = logf(sum);
    float loss = 0.0f;
    for (int k = tid; k < d.K; k += 64) {
      if (en.id[k] < 0) continue;
      const float under = en.x[k] - m, a = fused ? fmaf(en.x[k], c, -cm) : under * c;
      const float p = en.p[k];
      en.x[k] = a;
      if (p == 0.0f) continue;
      // tau times a term; a itself overflows where the logits are 2^128 tau / log2(e) apart
      const float term =
          fused && a != kNegInf ? d.tau * (en.logp[k] - a * kLn2 + z) : d.tau * (en.logp[k] + z) - under;
      loss += p * wt * term;
    }
    loss = wave_sum(loss);
    if (tid == 0) d.loss[t] = loss;
  }
  if (!ds) return;

  const float scale = wt / sum;
  if (kHold > 0 && fused) {
    auto grad = [&](float a) { return exp2_fast(fmaf(a, c, -cm)) * scale; };
#pragma unroll
    for (int j = 0; j < kHold; ++j) {
      const int64_t i = tid + j * kThreads;
      if (i < nv) dv[i] = P::make([&](int e) { return grad(P::get(hold[j], e)); });
    }
    if (end < d.V) ds[end] = T(grad(last));
  } else {
    auto grad = [&](float a) { return exp2_fast((a - m) * c) * scale; };
    for (int64_t i = tid; i < nv; i += kThreads) {
      const u32x4 v = load_masked(i);
      dv[i] = P::make([&](int e) { return grad(P::get(v, e)); });
    }
    if (end < d.V) ds[end] = T(grad(last));
  }
  __syncthreads();  // the row is written: the teacher's classes over it
  for (int k = tid; k < d.K; k += kThreads) {
    const int32_t id = en.id[k];
    if (id < 0) continue;
    float p = 0.0f;
    for (int j = 0; j < d.K; ++j) p += en.id[j] == id ? en.p[j] : 0.0f;  // a class named twice
    ds[id] = T(exp2_fast(en.x[k]) * scale - wt * p);
  }
}

template <class E, class Y, int kThreads, int kHold>
int launch_row(const Distill& d, hipStream_t st) {
  return launch("td_row", td_row<E, Y, kThreads, kHold>, row_grid(d.T), dim3(kThreads), size_t(d.K) * 16, st,
                d);
}

// By the row's 16-byte vectors: held in registers as long as one workgroup can
// (131,072 classes in 16 bits), by the fewest threads that hold it in at most 8
// vectors each (12 for the step between 256 and 512 threads: 8,192 rows of 21,841
// classes in bf16 160 us and 84 without a gradient, with 512 x 8 167 and 94; of
// 24,500 168 and 76, with 512 x 8 159 and 81), then 16. 8,192 rows of 32,768 classes in bf16 took 211 us with 512 x 8, 226 with 256 x 16,
// 245 with 1024 x 4, and 255 to 426 when read twice; 4,096 rows of 131,072 in
// fp16 491 with 1024 x 16, 549 when read twice. The loss alone is summed in the
// same order, so that it has the same bits with a gradient and without (8,192
// rows of 21,841: 84 us; one pass with nothing held took 74).
template <class E, class Y>
int launch_rows(const Distill& d, hipStream_t st) {
  const int64_t nv = d.V / Packed<E>::kN;
  if (nv <= 64 * 4) return launch_row<E, Y, 64, 4>(d, st);
  if (nv <= 256 * 4) return launch_row<E, Y, 256, 4>(d, st);
  if (nv <= 256 * 8) return launch_row<E, Y, 256, 8>(d, st);
  if (nv <= 256 * 12) return launch_row<E, Y, 256, 12>(d, st);
  if (nv <= 512 * 8) return launch_row<E, Y, 512, 8>(d, st);
  if (nv <= 512 * 16) return launch_row<E, Y, 512, 16>(d, st);
  if (nv <= 1024 * 16) return launch_row<E, Y, 1024, 16>(d, st);
  return launch_row<E, Y, 1024, 0>(d, st);
}

template <class E>
int launch_teacher(const Distill& d, int32_t teacher, hipStream_t st) {
  switch (teacher) {
    case NOPFS_BF16: return launch_rows<E, Bf16>(d, st);
    case NOPFS_FP16: return launch_rows<E, Fp16>(d, st);
    default: return launch_rows<E, Fp32>(d, st);
  }
}

int distill_impl(const nopfs_distill* p, const void* logits, const int32_t* index, const void* teacher,
                 const float* weight, float* loss, void* grad, hipStream_t st) {
  if (!p) return fail(NOPFS_EINVAL, "distill is NULL");
  if (p->T < 0 || p->V < 1 || p->K < 1) return fail(NOPFS_EINVAL, "T must be >= 0, V and K >= 1");
  if (p->dtype < NOPFS_BF16 || p->dtype > NOPFS_FP32 || p->teacher_dtype < NOPFS_BF16 ||
      p->teacher_dtype > NOPFS_FP32)
    return fail(NOPFS_EINVAL, "unknown dtype");
  if (!(p->tau > 0.0f) || !isfinite(p->tau)) return fail(NOPFS_EINVAL, "tau must be positive and finite");
  if (p->tau < 0x1p-60f || p->tau > 0x1p60f)  // tau^2 and 1 / tau stay finite
    return fail(NOPFS_ERANGE, "tau must be in 2^-60 .. 2^60");
  if (p->T > 1 && (p->logits_stride < p->V || p->index_stride < p->K || p->teacher_stride < p->K ||
                   (grad && p->grad_stride < p->V)))
    return fail(NOPFS_EINVAL, "rows overlap");
  if (p->T == 0) return NOPFS_OK;
  if (!logits || !index || !teacher || !loss)
    return fail(NOPFS_EINVAL, "logits, index, teacher and loss must be non-NULL");
  if (p->K > kMaxTop) return fail(NOPFS_ERANGE, "K must be <= 1024");
  if (p->T > INT32_MAX || p->V > INT32_MAX) return fail(NOPFS_ERANGE, "T and V must be < 2^31");
  const Distill d{p->T, p->V, p->logits_stride, p->grad_stride, p->index_stride, p->teacher_stride,
                  p->K, p->tau, logits, index, teacher, weight, loss, grad};
  switch (p->dtype) {
    case NOPFS_BF16: return launch_teacher<Bf16>(d, p->teacher_dtype, st);
    case NOPFS_FP16: return launch_teacher<Fp16>(d, p->teacher_dtype, st);
    default: return launch_teacher<Fp32>(d, p->teacher_dtype, st);
  }
}

}  // namespace
}  // namespace nopfs

using namespace nopfs;

extern "C" int nopfs_topk_distill(const nopfs_distill* distill, const void* logits, const int32_t* index,
                                  const void* teacher, const float* weight, float* loss, void* grad,
                                  void* hip_stream) {
  try {
    return distill_impl(distill, logits, index, teacher, weight, loss, grad,
                        static_cast<hipStream_t>(hip_stream));
  } catch (...) {
    return fail(NOPFS_EDEVICE, "unexpected host exception");
  }
}
