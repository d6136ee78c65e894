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

// Two floats as bf16, to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2{a, b}), bf16x2));
}

// How the columns of a row are dealt to TPR threads, NV times V columns each.
// VEC: a thread holds runs of V neighbouring columns and reads 16 bytes (fp32
// V = 4, bf16 V = 8 or 4) at once.  Otherwise (odd widths, arrays aligned to
// their type only) the V = 4 columns of a thread lie 32 apart, so that
// neighbouring lanes still read neighbouring columns.  Either way the 128
// columns of an 8-bit block lie with 128 / V neighbouring lanes.
template <int TPR, int V, bool VEC>
struct Cols {
  static constexpr int G = TPR < 32 ? TPR : 32;
  static constexpr int STRIDE = VEC ? 1 : G;
  static constexpr int BLOCK_LANES = TPR < ROWS8_BLOCK / V ? TPR : ROWS8_BLOCK / V;
  // first column of thread t's run j; column k of it is first + STRIDE k
  __device__ __forceinline__ static int first(int j, int t) {
    return VEC ? (j * TPR + t) * V : (j * TPR + (t & ~(G - 1))) * V + (t & (G - 1));
  }
};

// v[k] = column c + STRIDE k of the row at p + b + o (0 past its end); b is the
// same for the whole wave, o the lane's.
template <int TYPE, class D, int V>
__device__ __forceinline__ void load_cols(const void* p, int64_t b, uint32_t o, int c, int cols, float (&v)[V]) {
  if constexpr (D::STRIDE == 1) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = 0.f;
    if (c >= cols) return;
    if constexpr (TYPE == MGN_BF16) {
      const uint16_t* r = (const uint16_t*)p + b;
      uint32_t u[V / 2];
      if constexpr (V == 8) {
        const uint4 w = *reinterpret_cast<const uint4*>(r + (o + c));
        u[0] = w.x, u[1] = w.y, u[2] = w.z, u[3] = w.w;
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(r + (o + c));
        u[0] = w.x, u[1] = w.y;
      }
#pragma unroll
      for (int k = 0; k < V / 2; ++k) {
        v[2 * k] = __uint_as_float(u[k] << 16);
        v[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
      }
    } else {
      const float* r = (const float*)p + b;
#pragma unroll
      for (int q = 0; q < V / 4; ++q) {
        const floatx4 u = *reinterpret_cast<const floatx4*>(r + (o + c + 4 * q));
#pragma unroll
        for (int k = 0; k < 4; ++k) v[4 * q + k] = u[k];
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      v[k] = 0.f;
      if (c + D::STRIDE * k < cols) {
        if constexpr (TYPE == MGN_BF16) v[k] = bf2f(((const uint16_t*)p + b)[o + c + D::STRIDE * k]);
        else v[k] = ((const float*)p + b)[o + c + D::STRIDE * k];
      }
    }
  }
}

template <int TYPE, class D, int V>
__device__ __forceinline__ void store_cols(void* p, int64_t b, uint32_t o, int c, int cols, const float (&v)[V]) {
  if constexpr (D::STRIDE == 1) {
    if (c >= cols) return;
    if constexpr (TYPE == MGN_BF16) {
      uint16_t* r = (uint16_t*)p + b;
      if constexpr (V == 8)
        *reinterpret_cast<uint4*>(r + (o + c)) = uint4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]),
                                                       pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
      else
        *reinterpret_cast<uint2*>(r + (o + c)) = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
      float* r = (float*)p + b;
#pragma unroll
      for (int q = 0; q < V / 4; ++q)
        *reinterpret_cast<floatx4*>(r + (o + c + 4 * q)) = floatx4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    }
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (c + D::STRIDE * k < cols) {
        if constexpr (TYPE == MGN_BF16) ((uint16_t*)p + b)[o + c + D::STRIDE * k] = (uint16_t)pack_bf16(v[k], 0.f);
        else ((float*)p + b)[o + c + D::STRIDE * k] = v[k];
      }
  }
}

// v from lane ^ D of the wave, D = 1, 2, 4, 8, for values that are equal in
// groups of D lanes (a butterfly's next step): the lane's mirror image in its
// group of 2 D is one of the group it wants, and such mirrors are DPP operands.
template <int D>
__device__ __forceinline__ float mirror(float v) {
  if constexpr (D >= 16) {
    if constexpr (D == 16) return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), 0x401f));  // lane ^ 16
    else return __shfl_xor(v, D);
  } else {
    constexpr int ctrl = D == 1 ? 0xb1 : D == 2 ? 0x4e : D == 4 ? 0x141 : 0x140;  // quads 1032, 2301; mirrors of 8, 16
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, true));
  }
}
// Sum (largest) over groups of N neighbouring lanes; every lane gets the same bits.
template <int N, int D = 1>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (D < N) return group_sum<N, 2 * D>(v + mirror<D>(v));
  return v;
}
template <int N, int D = 1>
__device__ __forceinline__ float group_max(float v) {
  if constexpr (D < N) return group_max<N, 2 * D>(fmaxf(v, mirror<D>(v)));
  return v;
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
__device__ __forceinline__ uint32_t codes8(const float* v, float inv) {
  float u[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float s = v[k] * inv;
    u[k] = s == s ? fminf(fmaxf(s, -448.f), 448.f) : s;
  }
  const int r = __builtin_amdgcn_cvt_pk_fp8_f32(u[0], u[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(u[2], u[3], r, true);
}

__device__ __forceinline__ void values8(uint32_t q, float scale, float* v) {
  const floatx2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
  v[0] = a[0] * scale;
  v[1] = a[1] * scale;
  v[2] = b[0] * scale;
  v[3] = b[1] * scale;
}

// Stores a thread's run of a row in 8 bits; the row's lanes call it together
// (values past the row's end are 0), and the first lane of a block writes its
// scale.  write = false: takes part in the block's largest value only.
template <class D, int V>
__device__ __forceinline__ void store_cols8(uint8_t* q, float* scale, int c, int cols, const float (&v)[V], bool write) {
  float a = 0.f;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const float m = fabsf(v[k]);
    a = m < INFINITY && m > a ? m : a;
  }
  a = group_max<D::BLOCK_LANES>(a);
  const float s = scale8(a), inv = __uint_as_float((254u << 23) - __float_as_uint(s));  // 1 / s, a power of two
  uint32_t u[V / 4];
#pragma unroll
  for (int k = 0; k < V / 4; ++k) u[k] = codes8(v + 4 * k, inv);
  if (c >= cols || !write) return;
  if (c % ROWS8_BLOCK == 0) scale[c / ROWS8_BLOCK] = s;
  if constexpr (D::STRIDE == 1) {
    if constexpr (V == 8) *reinterpret_cast<uint2*>(q + c) = uint2{u[0], u[1]};
    else *reinterpret_cast<uint32_t*>(q + c) = u[0];
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (c + D::STRIDE * k < cols) q[c + D::STRIDE * k] = (uint8_t)(u[0] >> (8 * k));
  }
}

template <class D, int V>
__device__ __forceinline__ void load_cols8(const uint8_t* q, float scale, int c, int cols, float (&v)[V]) {
  uint32_t u[V / 4] = {};
  if constexpr (D::STRIDE == 1) {
    if constexpr (V == 8) {
      const uint2 w = *reinterpret_cast<const uint2*>(q + c);
      u[0] = w.x, u[1] = w.y;
    } else {
      u[0] = *reinterpret_cast<const uint32_t*>(q + c);
    }
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (c + D::STRIDE * k < cols) u[0] |= (uint32_t)q[c + D::STRIDE * k] << (8 * k);
  }
#pragma unroll
  for (int k = 0; k < V / 4; ++k) values8(u[k], scale, v + 4 * k);
}

}  // namespace mgn
