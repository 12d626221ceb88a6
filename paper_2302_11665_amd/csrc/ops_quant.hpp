// Rows in 8 bits (alpaserve_ops.h): how values are read, and the codes that a
// row's largest magnitude gives them.
#pragma once

#include "ops_common.hpp"

namespace as_ops {

template <int TYPE>
__device__ __forceinline__ float load_one(const void* x, int64_t i) {
  if (TYPE == AS_F32) return reinterpret_cast<const float*>(x)[i];
  return to_f32<TYPE>(reinterpret_cast<const uint16_t*>(x)[i]);
}

// 16 values from column c of a row; columns beyond n_cols are 0.  Rows may start
// anywhere: memory takes unaligned loads of 16 bytes.
template <int TYPE>
__device__ __forceinline__ void load16(const void* x, int64_t row, int64_t c, int64_t n_cols, float (&f)[16]) {
  if (c + 16 <= n_cols) {
    if (TYPE == AS_F32) {
      const float* p = reinterpret_cast<const float*>(x) + row + c;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v4f v;
        __builtin_memcpy(&v, p + 4 * i, 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[4 * i + j] = v[j];
      }
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(x) + row + c;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v4u v;
        __builtin_memcpy(&v, p + 8 * i, 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f[8 * i + 2 * j] = to_f32<TYPE>(v[j] & 0xffffu);
          f[8 * i + 2 * j + 1] = to_f32<TYPE>(v[j] >> 16);
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) f[i] = c + i < n_cols ? load_one<TYPE>(x, row + c + i) : 0.0f;
}

// Largest magnitude as ordered bits: infinities above every number, NaN above
// them, so that one integer maximum finds both.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// How a row is quantised, from its largest magnitude.  A power of two takes
// rows of very large or small numbers away from the ends of fp32's range.
template <int TYPE>
struct Quantiser {
  float by, top, inv;  // 127 and the largest magnitude, scaled; 1 / top
  bool none;           // all codes are 0
  __device__ __forceinline__ Quantiser(float a, bool finite) {
    none = !finite || a == 0.0f;
    const float scale = a > 0x1p100f ? 0x1p-64f : a < 0x1p-64f ? 0x1p64f : 1.0f;
    by = 127.0f * scale;
    top = none ? 1.0f : a * scale;
    inv = 1.0f / top;
  }
  // Codes of four values.  127 x is exact for 16-bit x.  Its quotient by top is
  // taken with the reciprocal and corrected once by the exact remainder: off by
  // 2^-46 of itself before the last rounding, so a quotient that ties between
  // two codes comes out exactly, and no other one can reach a tie (the nearest
  // is 2^-19 away).  The codes are therefore those of exact arithmetic.  fp32
  // values are corrected twice: the first time leaves the quotient less than a unit
  // in its last place off, and then a correction with a reciprocal that is rounded
  // to nearest gives the quotient rounded to nearest (Markstein's theorem), in half
  // the instructions of a division.  Adding 1.5 * 2^23 rounds to whole numbers,
  // ties to even, and leaves the code in the low byte.
  __device__ __forceinline__ uint32_t codes4(const float* f) const {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = f[i] * by;
      float q = x * inv;
      q = fmaf(fmaf(-q, top, x), inv, q);
      if (TYPE == AS_F32) q = fmaf(fmaf(-q, top, x), inv, q);
      u[i] = __float_as_uint(q + 12582912.0f);
    }
    const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu);
    return none ? 0u : lo | hi;
  }
};

}  // namespace as_ops
