// Element types of the operators that take a caller's tensors, and their conversions.
#pragma once
#include "device_utils.h"

namespace rb {

// element types of callers' tensors (rnnt_type_t)
struct TypeF32 {
  typedef float T;
};
struct TypeF16 {
  typedef _Float16 T;
};
struct TypeBf16 {
  typedef uint16_t T;
};
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(_Float16 v) { return (float)v; }
__device__ __forceinline__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// 16 bytes from any address (rows of odd lengths start anywhere; the hardware takes such loads whole)
template <typename T>
__device__ __forceinline__ void load16(const T *p, T (&v)[16 / sizeof(T)]) {
  __builtin_memcpy(v, p, 16);
}

constexpr double kLog2E = 1.4426950408889634;

// What lanes of a wave have written to LDS before, its lanes read after (a wave's LDS accesses are carried out in order)
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

}  // namespace rb
