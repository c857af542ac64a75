// Query rows and cached numbers as operands of the bf16 matrix instructions.
#pragma once

#include "cache.hpp"

namespace trevs {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// bf16 values enter as they are, fp32 ones as three bf16 parts (24 bits).
template <class E>
constexpr int kParts = E::kBytes == 2 ? 1 : 3;

// Eight e4m3 numbers, times a power of two, as bf16.
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight fp32 values as bf16 parts that sum to them (one part: rounded).
template <int N>
__device__ __forceinline__ void split_parts(float (&x)[8], bf16x8 (&out)[N]) {
#pragma unroll
  for (int p = 0; p < N; ++p)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      out[p][j] = (__bf16)x[j];
      x[j] -= (float)out[p][j];
    }
}

__device__ __forceinline__ void load_row8(const void* q, size_t i, float (&x)[8], BF16) {
  const u32x4 w = ldg16(reinterpret_cast<const uint16_t*>(q) + i);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = bf16_lo(w[j]);
    x[2 * j + 1] = bf16_hi(w[j]);
  }
}
__device__ __forceinline__ void load_row8(const void* q, size_t i, float (&x)[8], F32) {
  const float* f = reinterpret_cast<const float*>(q) + i;
  const u32x4 a = ldg16(f), b = ldg16(f + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = __uint_as_float(a[j]);
    x[4 + j] = __uint_as_float(b[j]);
  }
}

}  // namespace trevs
