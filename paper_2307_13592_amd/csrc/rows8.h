// Rows of fp32, bf16 or 8-bit columns in registers (gfx950 / CDNA4).
//
// 8-bit rows: the codes are e4m3 (4 exponent bits, 3 of mantissa, largest
// finite value 448, no infinity), one byte a column, and each block of 128
// columns of a row has one fp32 scale; a code stands for its e4m3 value times
// the scale.  The scale is the least power of two that brings the block's
// largest finite magnitude to 448 or less: dividing by it is exact, so a value
// is rounded once (to nearest, ties to even), rows that were read back and stored
// again stand for the same values, and since e4m3 is a floating format a power of
// two costs no mantissa bit against amax / 448, only up to one bit of range below.
#pragma once
#include <type_traits>

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
// Mostly a thread holds runs of V neighbouring columns, read 16 bytes (fp32
// V = 4, bf16 V = 8) at once; rows of any width and alignment, since the card's
// vector memory accesses need none; the columns past the last whole run are
// written in pieces of 4, 2 and 1.  Otherwise (arrays of a few elements) the V =
// 4 columns of a thread lie TPR apart, and are read one by one.  Either way the
// 128 columns of an 8-bit block lie with 128 / V neighbouring lanes.
enum RowMode {
  APART,   // columns TPR apart
  RUNS,    // runs
  WHOLE,   // whole runs on 16-byte boundaries
  STREAM,  // the same, read past the caches (kernels that move more than these hold)
};
template <int TPR, int V, int MODE>
struct Cols {
  static constexpr int STRIDE = MODE == APART ? TPR : 1;
  static constexpr bool EVEN = MODE == WHOLE || MODE == STREAM, PAST = MODE == STREAM;
  static constexpr int BLOCK_LANES = TPR < ROWS8_BLOCK / V ? TPR : ROWS8_BLOCK / V;
  // first column of thread t's run j; column k of it is first + STRIDE k
  __device__ __forceinline__ static int first(int j, int t) {
    return MODE == APART ? j * TPR * V + t : (j * TPR + t) * V;
  }
};

// N neighbouring elements at p, in one access where N allows.  Whole runs are
// written past the caches (what reads the result next loses no more than it
// gains: 51 MB stored and read 28.4 us, so 29.4; 102 MB 69 and 60), and read so
// in STREAM kernels.
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
template <class U, int A>
struct Near {  // a vector on the boundary of its elements
  typedef U T __attribute__((aligned(A)));
};
template <int N, class E, bool PAST = false>
__device__ __forceinline__ void get(const E* p, float* v) {
  constexpr int S = sizeof(E);
  if constexpr (N * S == 16) {
    uintx4 w;
    if constexpr (PAST) w = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(p));
    else w = *reinterpret_cast<const typename Near<uintx4, S>::T*>(p);
#pragma unroll
    for (int k = 0; k < N; ++k)
      v[k] = S == 4 ? __uint_as_float(w[k * S / 4])
                    : __uint_as_float(k % 2 ? w[k * S / 4] & 0xffff0000u : w[k * S / 4] << 16);
  } else if constexpr (S == 4) {
    float u[N];
    __builtin_memcpy(u, p, S * N);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = u[k];
  } else {
    uint16_t u[N];
    __builtin_memcpy(u, p, S * N);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = bf2f(u[k]);
  }
}
template <int N, class E>
__device__ __forceinline__ void put(E* p, const float* v) {
  constexpr int S = sizeof(E);
  if constexpr (S == 4) {
    if constexpr (N % 4 == 0) {
#pragma unroll
      for (int k = 0; k < N; k += 4)
        __builtin_nontemporal_store((floatx4{v[k], v[k + 1], v[k + 2], v[k + 3]}),
                                    reinterpret_cast<typename Near<floatx4, S>::T*>(p + k));
    } else {
      __builtin_memcpy(p, v, S * N);
    }
  } else if constexpr (N == 8) {
    __builtin_nontemporal_store((uintx4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                                        pack_bf16(v[6], v[7])}),
                                reinterpret_cast<typename Near<uintx4, S>::T*>(p));
  } else if constexpr (N == 1) {
    *p = (uint16_t)pack_bf16(v[0], 0.f);
  } else {
    uint32_t u[N / 2];
#pragma unroll
    for (int k = 0; k < N / 2; ++k) u[k] = pack_bf16(v[2 * k], v[2 * k + 1]);
    __builtin_memcpy(p, u, S * N);
  }
}

// f(first element, count) over pieces of 4, 2 and 1 that make up n < V columns
// (n the same for the whole launch).
template <int V, class F>
__device__ __forceinline__ void pieces(int n, F f) {
  constexpr std::integral_constant<int, 1> one;
  constexpr std::integral_constant<int, 2> two;
  constexpr std::integral_constant<int, 4> four;
  const auto rest = [&](auto from) {
    constexpr int S = from();
    constexpr std::integral_constant<int, S + 2> behind;
    if (n & 2) {
      f(from, two);
      if (n & 1) f(behind, one);
    } else if (n & 1) {
      f(from, one);
    }
  };
  if constexpr (V == 8)
    if (n & 4) {
      f(std::integral_constant<int, 0>(), four);
      rest(four);
      return;
    }
  rest(std::integral_constant<int, 0>());
}

template <int TYPE>
using Elem = std::conditional_t<TYPE == MGN_BF16, uint16_t, float>;

// v[k] = w[c + STRIDE k] of `cols` values (0 past them): weights, read once.
template <class D, int V>
__device__ __forceinline__ void load_values(const float* w, int c, int cols, float (&v)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = 0.f;
  if constexpr (D::STRIDE == 1) {
    if (c + V <= cols) get<V>(w + c, v);
    else if (c < cols) pieces<V>(cols & (V - 1), [&](auto s, auto n) { get<n()>(w + (c + s()), v + s()); });
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (c + D::STRIDE * k < cols) get<1>(w + (c + D::STRIDE * k), v + k);
  }
}

// v[k] = column c + STRIDE k of the row at p + b + o (0 past its end); b is the
// same for the whole wave, o the lane's; `left` elements of the array lie from
// p + b on.  A run of 16 bytes that passes its row's end is read whole, into the
// next row, and cut; one that would pass the array's end is read from `left`
// back and shifted.  (An array of runs holds 16 elements or more.)
template <int TYPE, class D, int V>
__device__ __forceinline__ void load_cols(const void* p, int64_t b, uint32_t o, int c, int cols, int64_t left,
                                          float (&v)[V]) {
  using E = Elem<TYPE>;
  const E* r = (const E*)p + b;
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = 0.f;
  if constexpr (D::STRIDE == 1) {
    static_assert(V * sizeof(E) == 16);
    if (c >= cols) return;
    if constexpr (D::EVEN) {
      get<V, E, D::PAST>(r + (o + c), v);
    } else {
      const int64_t most = left - V;
      const int32_t e = (int32_t)(o + c), at = most < (int64_t)e ? (int32_t)most : e;
      const uint32_t back = e - at;
      uint64_t w[2];
      __builtin_memcpy(w, r + at, 16);
      if (back) {
        const uint32_t bits = back * sizeof(E) * 8;
        w[0] = bits < 64 ? w[0] >> bits | w[1] << (64 - bits) : w[1] >> (bits - 64);
        w[1] = bits < 64 ? w[1] >> bits : 0;
      }
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const uint32_t u = (uint32_t)(w[k * sizeof(E) / 8] >> (k * sizeof(E) % 8 / 4 * 32));
        const float x = __uint_as_float(sizeof(E) == 4 ? u : k % 2 ? u & 0xffff0000u : u << 16);
        v[k] = c + k < cols ? x : 0.f;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (c + D::STRIDE * k < cols) get<1>(r + (o + c + D::STRIDE * k), v + k);
  }
}

template <int TYPE, class D, int V>
__device__ __forceinline__ void store_cols(void* p, int64_t b, uint32_t o, int c, int cols, const float (&v)[V]) {
  Elem<TYPE>* r = (Elem<TYPE>*)p + b;
  if constexpr (D::STRIDE == 1) {
    if (c + V <= cols) put<V>(r + (o + c), v);
    else if (!D::EVEN && c < cols) pieces<V>(cols & (V - 1), [&](auto s, auto n) { put<n()>(r + (o + c + s()), v + s()); });
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (c + D::STRIDE * k < cols) put<1>(r + (o + c + D::STRIDE * k), v + k);
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
__device__ __forceinline__ float code8(float v, float inv) {
  const float s = v * inv;
  return s == s ? fminf(fmaxf(s, -448.f), 448.f) : s;
}
__device__ __forceinline__ uint32_t codes8(float a, float b, float c, float d, float inv) {
  const int r = __builtin_amdgcn_cvt_pk_fp8_f32(code8(a, inv), code8(b, inv), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(code8(c, inv), code8(d, inv), r, true);
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
  for (int k = 0; k < V / 4; ++k) u[k] = codes8(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3], inv);
  if (c >= cols || !write) return;
  if (c % ROWS8_BLOCK == 0) scale[c / ROWS8_BLOCK] = s;
  if constexpr (D::STRIDE == 1) {
    if (c + V <= cols)
      __builtin_memcpy(q + c, u, V);
    else if (!D::EVEN)
      pieces<V>(cols & (V - 1), [&](auto f, auto n) {
        const uint32_t w = u[f() / 4] >> (8 * (f() % 4));
        __builtin_memcpy(q + (c + f()), &w, n());
      });
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
    if (c + V <= cols)
      __builtin_memcpy(u, q + c, V);
    else if (!D::EVEN && c < cols)
      pieces<V>(cols & (V - 1), [&](auto f, auto n) {
        uint32_t w = 0;
        __builtin_memcpy(&w, q + (c + f()), n());
        u[f() / 4] |= w << (8 * (f() % 4));
      });
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (c + D::STRIDE * k < cols) u[0] |= (uint32_t)q[c + D::STRIDE * k] << (8 * k);
  }
#pragma unroll
  for (int k = 0; k < V / 4; ++k) values8(u[k], scale, v + 4 * k);
}

}  // namespace mgn
