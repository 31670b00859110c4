// nopfs_topk_distill: loss and gradient against a teacher's top logits.
//
// Per row (token) with logits s[V], teacher logits y at classes x, temperature
// tau and weight w, over the valid teacher entries (0 <= x_k < V):
//     p = softmax(y / tau),  z = log sum_v exp(s_v / tau)
//     loss  = w tau^2 sum_k p_k (log p_k - s[x_k] / tau + z)
//     ds_v  = w tau (exp(s_v / tau - z) - sum_{k: x_k = v} p_k)
// One workgroup per row. The row is read for its maximum and its sum of
// exponentials together (the running sum is rescaled when the maximum grows),
// and again for the gradient. All sums are in 32 bits.
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
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -INFINITY;

__device__ inline float wave_max(float v) {
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ inline float wave_sum(float v) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

template <int kThreads, bool kMax>
__device__ inline float block_reduce(float v, float* tmp) {
  v = kMax ? wave_max(v) : wave_sum(v);
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = tmp[0];
  for (int i = 1; i < kThreads / 64; ++i) r = kMax ? fmaxf(r, tmp[i]) : r + tmp[i];
  __syncthreads();
  return r;
}

// The running maximum and sum of exponentials, base 2 after scaling by c. An
// infinite maximum of the wrong sign (nothing but -inf so far) counts as 0 in
// the differences: the sum stays 0 instead of NaN.
struct Running {
  float m = kNegInf, sum = 0.0f;
};
__device__ inline float finite_max(float m) { return m == kNegInf ? 0.0f : m; }

template <class E, class Y, int kThreads>
__global__ void __launch_bounds__(kThreads) td_row(const Distill d) {
  typedef typename E::T T;
  __shared__ float tmp[kThreads / 64];
  __shared__ float s_p[kMaxTop], s_x[kMaxTop];
  __shared__ int32_t s_id[kMaxTop];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  const T* s = static_cast<const T*>(d.logits) + t * d.logits_stride;
  T* ds = d.grad ? static_cast<T*>(d.grad) + t * d.grad_stride : nullptr;
  const float w = d.weight ? d.weight[t] : 1.0f;

  // the teacher's distribution over its valid entries
  const typename Y::T* y = static_cast<const typename Y::T*>(d.teacher) + t * d.teacher_stride;
  const int32_t* x = d.index + t * d.index_stride;
  const float inv_tau = 1.0f / d.tau;
  float ymax = kNegInf;
  for (int k = tid; k < d.K; k += kThreads) {
    const int32_t id = x[k];
    const bool valid = id >= 0 && id < d.V && w != 0.0f;
    const float v = valid ? float(y[k]) : kNegInf;
    s_id[k] = valid && v != kNegInf ? id : -1;
    s_p[k] = v;
    ymax = v == v ? fmaxf(ymax, v) : INFINITY;  // a NaN reaches every result of the row
  }
  ymax = block_reduce<kThreads, true>(ymax, tmp);
  if (ymax == kNegInf) {  // weight 0, or no entry with any mass: nothing is learned from this row
    if (tid == 0) d.loss[t] = 0.0f;
    if (ds)
      for (int64_t v = tid; v < d.V; v += kThreads) ds[v] = T(0.0f);
    return;
  }
  float ysum = 0.0f;
  for (int k = tid; k < d.K; k += kThreads) ysum += expf((s_p[k] - ymax) * inv_tau);
  ysum = block_reduce<kThreads, false>(ysum, tmp);

  const float c = kLog2e / d.tau;
  Running r;
  for (int64_t v = tid; v < d.V; v += kThreads) {
    const float a = float(s[v]);
    const float m = fmaxf(r.m, a);
    const float f = finite_max(m);
    r.sum = r.sum * exp2f((r.m - f) * c) + exp2f((a - f) * c);
    r.m = m;
  }
  const float m = block_reduce<kThreads, true>(r.m, tmp);
  const float sum = block_reduce<kThreads, false>(r.sum * exp2f((r.m - finite_max(m)) * c), tmp);
  const float z = logf(sum);  // of exp((s - m) / tau)

  float loss = 0.0f;
  for (int k = tid; k < d.K; k += kThreads) {
    const int32_t id = s_id[k];
    const float v = (s_p[k] - ymax) * inv_tau;
    const float p = id >= 0 ? expf(v) / ysum : 0.0f;
    s_p[k] = p;
    if (id >= 0) {
      const float a = (float(s[id]) - m) * inv_tau;
      s_x[k] = a;
      if (p != 0.0f) loss += p * (v - logf(ysum) - a + z);
    }
  }
  loss = block_reduce<kThreads, false>(loss, tmp);
  if (tid == 0) d.loss[t] = w * d.tau * d.tau * loss;
  if (!ds) return;

  const float wt = w * d.tau, inv = 1.0f / sum;
  for (int64_t v = tid; v < d.V; v += kThreads) ds[v] = T(wt * (exp2f((float(s[v]) - m) * c) * inv));
  __syncthreads();  // the row is written: the teacher's classes over it
  for (int k = tid; k < d.K; k += kThreads) {
    const int32_t id = s_id[k];
    if (id < 0) continue;
    float p = 0.0f;
    for (int j = 0; j < d.K; ++j) p += s_id[j] == id ? s_p[j] : 0.0f;  // a class named twice
    ds[id] = T(wt * (exp2f(s_x[k] * kLog2e) * inv - p));
  }
}

template <class E, class Y>
int launch_rows(const Distill& d, hipStream_t st) {
  return launch("td_row", td_row<E, Y, 256>, dim3(uint32_t(d.T)), dim3(256), 0, st, d);
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
