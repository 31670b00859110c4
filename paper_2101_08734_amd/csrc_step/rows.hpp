// Shared by the layers over packed samples: vectors of rows that begin at any
// element, reductions, and the sample of a token.
#pragma once

#include "step.hpp"

namespace nopfs {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Words in memory at any element: they claim 2 bytes' alignment only; the hardware
// takes such loads and stores whole.
typedef uint32_t word_by2 __attribute__((aligned(2)));
typedef u32x2 pair_by2 __attribute__((aligned(2)));
typedef u32x4 quad_by2 __attribute__((aligned(2)));

// kN elements as they lie in memory, in 32-bit words.
template <class E, int kN>
struct Pack {
  typedef typename E::T T;
  static constexpr bool kWide = sizeof(T) == 4;
  static constexpr int kWords = kN * int(sizeof(T)) / 4;
  static_assert(kWords >= 1, "a word at least");
  typedef T V2 __attribute__((ext_vector_type(2)));
  uint32_t w[kWords];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  // kOnce: of data that nothing reads again soon
  template <bool kOnce = false>
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kWords == 1) {
      if constexpr (kOnce) w[0] = __builtin_nontemporal_load(reinterpret_cast<const word_by2*>(p));
      else w[0] = *reinterpret_cast<const word_by2*>(p);
    } else if constexpr (kWords == 2) {
      const u32x2 v = *reinterpret_cast<const pair_by2*>(p);
      w[0] = v[0], w[1] = v[1];
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const u32x4 v = reinterpret_cast<const quad_by2*>(p)[i];
        w[4 * i] = v[0], w[4 * i + 1] = v[1], w[4 * i + 2] = v[2], w[4 * i + 3] = v[3];
      }
    }
  }
  // the first n < kN elements, then zeros
  __device__ __forceinline__ void load_some(const T* p, int n) {
    float v[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) v[e] = e < n ? float(p[e]) : 0.0f;
    set(v);
  }
  __device__ __forceinline__ float get(int e) const {
    const uint32_t word = w[kWide ? e : e >> 1];
    if constexpr (kWide) return __uint_as_float(word);
    else if constexpr (E::kBits == 8) return __uint_as_float(e & 1 ? word & 0xFFFF0000u : word << 16);
    else return float(__builtin_bit_cast(V2, word)[e & 1]);
  }
  // rounds kN floats (to nearest, ties to even)
  __device__ __forceinline__ void set(const float (&v)[kN]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (kWide) {
        w[i] = __float_as_uint(v[i]);
      } else {
        const f32x2 x = {v[2 * i], v[2 * i + 1]};
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, V2));
      }
    }
  }
  template <bool kOnce = false>
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kWords == 1) {
      if constexpr (kOnce) __builtin_nontemporal_store(w[0], reinterpret_cast<word_by2*>(p));
      else *reinterpret_cast<word_by2*>(p) = w[0];
    } else if constexpr (kWords == 2) {
      *reinterpret_cast<pair_by2*>(p) = u32x2{w[0], w[1]};
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i)
        reinterpret_cast<quad_by2*>(p)[i] = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    }
  }
  __device__ __forceinline__ void store_some(T* p, int n) const {
#pragma unroll
    for (int e = 0; e < kN; ++e)
      if (e < n) p[e] = T(get(e));
  }
};

// The sum over groups of kLanes lanes (a power of two), the same in all of them, in
// registers: lanes 1 and 2 apart by permutations of four, then mirrors of 8 and 16
// lanes (whose parts are equal by then), then rows of 16 and halves exchanged.
template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), kCtrl, 0xf, 0xf, true));
}
template <int kLanes>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (kLanes >= 2) v += dpp<0xB1>(v);    // quad_perm:[1,0,3,2]
  if constexpr (kLanes >= 4) v += dpp<0x4E>(v);    // quad_perm:[2,3,0,1]
  if constexpr (kLanes >= 8) v += dpp<0x141>(v);   // row_half_mirror
  if constexpr (kLanes >= 16) v += dpp<0x140>(v);  // row_mirror
  if constexpr (kLanes >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (kLanes >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// A wave's lanes go on together from here, behind what all of them have read and
// written in LDS.
__device__ __forceinline__ void wave_step() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// A type's code in the C ABI as a type: f(E()).
template <class F>
int by_dtype(int32_t code, F f) {
  switch (code) {
    case NOPFS_BF16: return f(Bf16());
    case NOPFS_FP16: return f(Fp16());
    default: return f(Fp32());
  }
}
inline bool is_dtype(int32_t code) { return code >= NOPFS_BF16 && code <= NOPFS_FP32; }

// The least power of two >= n, as an exponent.
inline int log2_ceil(int64_t n) {
  int b = 0;
  while ((int64_t(1) << b) < n) ++b;
  return b;
}

}  // namespace nopfs
