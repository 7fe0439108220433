// Device helpers shared by the operators' kernels: vectors, bf16, loads of eight values.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gecc {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4_t;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2_t;

__device__ __forceinline__ float bf16_of(uint16_t h) { return __uint_as_float((unsigned)h << 16); }
// round to nearest even; a NaN stays one
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// eight consecutive values of a row from column c on (0 beyond the matrix)
template <bool F32, bool VEC>
__device__ __forceinline__ void load8(const void* X, int64_t at, int c, int cols, bool row_ok, float (&v)[8]) {
  if (VEC && row_ok && c + 8 <= cols) {
    if (F32) {
      const f32x4_t* p = reinterpret_cast<const f32x4_t*>(static_cast<const float*>(X) + at);
      const f32x4_t a = p[0], b = p[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
      const u32x4_t a = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(X) + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(a[i] << 16); v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.f;
      if (row_ok && c + i < cols)
        v[i] = F32 ? static_cast<const float*>(X)[at + i] : bf16_of(static_cast<const uint16_t*>(X)[at + i]);
    }
  }
}

}  // namespace
}  // namespace gecc
