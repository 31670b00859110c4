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

// A launch counts its threads in 32 bits per dimension (2^22 workgroups of 1024):
// `blocks` workgroups in rows of 2^20, and a workgroup's number among them (the
// last row's may pass `blocks`).
inline dim3 row_grid(int64_t blocks) {
  return dim3(uint32_t(std::min<int64_t>(blocks, 1 << 20)), uint32_t(ceil_div(blocks, 1 << 20)));
}
__device__ __forceinline__ uint32_t row_block() { return blockIdx.y << 20 | blockIdx.x; }

}  // namespace nopfs
