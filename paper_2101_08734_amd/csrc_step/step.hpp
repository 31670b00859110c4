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

}  // namespace nopfs
