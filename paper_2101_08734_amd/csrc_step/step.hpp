// Shared by the operators of a training step: 16-bit types and conversions.
#pragma once

#include <limits.h>
#include <algorithm>
#include <type_traits>
#include <math.h>

#include "common.hpp"

namespace nopfs {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Element types by their code in the C ABI; kBits: of the significand.
struct Bf16 {
  typedef __bf16 T;
  static constexpr int kBits = 8;
};
struct Fp16 {
  typedef _Float16 T;
  static constexpr int kBits = 11;
};
struct Fp32 {
  typedef float T;
  static constexpr int kBits = 24;
};

// Scratch of calls that run in every step, and so in graphs. A graph that held
// addresses in its stream's block would share them with that stream's calls and
// with other graphs captured there, in any order: a captured call takes its
// scratch from its caller, whose block lives and is ordered as the graph is.
template <typename T>
int step_alloc(Scratch* sc, T** p, size_t n) {
  if (sc->shared_in_capture())
    return fail(NOPFS_EINVAL, "a call on a stream that is being captured needs its caller's scratch");
  return sc->alloc_n(p, n);
}

// Runs `call` with the scratch given in its description, if any.
template <class F>
int run_with_scratch(void* block, int64_t bytes, F call) {
  if (!block || sizing_only()) return call();
  if ((reinterpret_cast<uintptr_t>(block) & 255) || bytes < 0)
    return fail(NOPFS_EINVAL, "scratch must be a multiple of 256 bytes, its size not negative");
  return run_in_caller_block(block, size_t(bytes), call);
}

// The scratch that `call` takes, 0 where it fails.
template <class F>
int scratch_size(int64_t* bytes, F call) {
  if (!bytes) return fail(NOPFS_EINVAL, "bytes must be non-NULL");
  size_t peak = 0;
  const int rc = run_sizing(call, &peak);
  *bytes = rc ? 0 : int64_t(peak);
  return rc;
}
// Stands for the arrays of such a call, which touches none.
inline void* no_array() { return reinterpret_cast<void*>(uintptr_t(256)); }

// A launch counts its threads in 32 bits per dimension (2^22 workgroups of 1024):
// `blocks` workgroups in rows of 2^20, and a workgroup's number among them (the
// last row's may pass `blocks`).
inline dim3 row_grid(int64_t blocks) {
  return dim3(uint32_t(std::min<int64_t>(blocks, 1 << 20)), uint32_t(ceil_div(blocks, 1 << 20)));
}
__device__ __forceinline__ uint32_t row_block() { return blockIdx.y << 20 | blockIdx.x; }

}  // namespace nopfs
