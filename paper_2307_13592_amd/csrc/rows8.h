// Rows of fp32, bf16 or 8-bit columns, four columns a lane (gfx950 / CDNA4).
//
// 8-bit rows: the codes are e4m3 (4 exponent bits, 3 of mantissa, largest
// finite value 448, no infinity), one byte a column, and each block of 128
// columns of a row has one fp32 scale; a code stands for its e4m3 value times
// the scale.  The scale is the least power of two that brings the block's
// largest finite magnitude to 448 or less: dividing by it is exact, so a value
// is rounded once (to nearest, ties to even), storing rows that were read back
// gives the same bytes, and since e4m3 is a floating format a power of two
// costs no mantissa bit against amax / 448, only up to one bit of range below.
#pragma once
#include "device_common.h"
#include "../../include/mgn.h"

namespace mgn {

constexpr int ROWS8_BLOCK = MGN_ROWS8_BLOCK;
__host__ __device__ inline int rows8_blocks(int cols) { return (cols + ROWS8_BLOCK - 1) / ROWS8_BLOCK; }

typedef float floatx2 __attribute__((ext_vector_type(2)));

// v[k] = column c + k of the row that starts at element `base` (0 past its end).
template <int TYPE, bool VEC>
__device__ __forceinline__ void load_cols(const void* p, int64_t base, int c, int cols, float (&v)[4]) {
  if constexpr (VEC) {
    if (c >= cols) {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = 0.f;
    } else if constexpr (TYPE == MGN_BF16) {
      const uint2 u = *reinterpret_cast<const uint2*>((const uint16_t*)p + base + c);
      v[0] = __uint_as_float(u.x << 16);
      v[1] = __uint_as_float(u.x & 0xffff0000u);
      v[2] = __uint_as_float(u.y << 16);
      v[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
      const floatx4 u = *reinterpret_cast<const floatx4*>((const float*)p + base + c);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = u[k];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = 0.f;
      if (c + k < cols) {
        if constexpr (TYPE == MGN_BF16) v[k] = bf2f(((const uint16_t*)p)[base + c + k]);
        else v[k] = ((const float*)p)[base + c + k];
      }
    }
  }
}

template <int TYPE, bool VEC>
__device__ __forceinline__ void store_cols(void* p, int64_t base, int c, int cols, const float (&v)[4]) {
  if constexpr (VEC) {
    if (c >= cols) return;
    if constexpr (TYPE == MGN_BF16) {
      const uint2 u{(uint32_t)f2bf(v[0]) | (uint32_t)f2bf(v[1]) << 16, (uint32_t)f2bf(v[2]) | (uint32_t)f2bf(v[3]) << 16};
      *reinterpret_cast<uint2*>((uint16_t*)p + base + c) = u;
    } else {
      *reinterpret_cast<floatx4*>((float*)p + base + c) = floatx4{v[0], v[1], v[2], v[3]};
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < cols) {
        if constexpr (TYPE == MGN_BF16) ((uint16_t*)p)[base + c + k] = f2bf(v[k]);
        else ((float*)p)[base + c + k] = v[k];
      }
  }
}

// The scale for a block whose largest finite magnitude is a: from a's bits,
// 2^(E - 8) for a = m 2^E with m <= 1.75 (448 = 1.75 * 2^8), else 2^(E - 7);
// at least 2^-126, so that its reciprocal is finite, and 1 for a = 0.
__device__ __forceinline__ float scale8(float a) {
  int e = (int)((__float_as_uint(a) + 0x1fffffu) >> 23) - 8;
  if (e < 1) e = 1;
  return a > 0.f ? __uint_as_float((uint32_t)e << 23) : 1.f;
}

// Four codes of v / scale, inv = 1 / scale.  Infinities become +-448; a NaN
// stays one.
__device__ __forceinline__ uint32_t codes8(const float (&v)[4], float inv) {
  float u[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float s = v[k] * inv;
    u[k] = s == s ? fminf(fmaxf(s, -448.f), 448.f) : s;
  }
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(u[0], u[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(u[2], u[3], r, true);
}

__device__ __forceinline__ void values8(uint32_t q, float scale, float (&v)[4]) {
  const floatx2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
  v[0] = a[0] * scale;
  v[1] = a[1] * scale;
  v[2] = b[0] * scale;
  v[3] = b[1] * scale;
}

// Stores columns c .. c + 3 of a row in 8 bits; the row's lanes call it
// together (TPR of them, 32 or all TPR neighbouring lanes hold a block; values
// past the row's end are 0), and the first lane of a block writes its scale.
template <int TPR, bool VEC>
__device__ __forceinline__ void store_cols8(uint8_t* q, float* scale, int c, int cols, const float (&v)[4]) {
  float a = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float m = fabsf(v[k]);
    a = m < INFINITY && m > a ? m : a;
  }
#pragma unroll
  for (int d = 1; d < (TPR < 32 ? TPR : 32); d *= 2) a = fmaxf(a, __shfl_xor(a, d));
  const float s = scale8(a);
  const uint32_t u = codes8(v, 1.f / s);
  if (c >= cols) return;
  if (c % ROWS8_BLOCK == 0) scale[c / ROWS8_BLOCK] = s;
  if constexpr (VEC) {
    *reinterpret_cast<uint32_t*>(q + c) = u;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < cols) q[c + k] = (uint8_t)(u >> (8 * k));
  }
}

template <bool VEC>
__device__ __forceinline__ void load_cols8(const uint8_t* q, float scale, int c, int cols, float (&v)[4]) {
  uint32_t u = 0;
  if constexpr (VEC) {
    if (c < cols) u = *reinterpret_cast<const uint32_t*>(q + c);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k < cols) u |= (uint32_t)q[c + k] << (8 * k);
  }
  values8(u, scale, v);
}

}  // namespace mgn
