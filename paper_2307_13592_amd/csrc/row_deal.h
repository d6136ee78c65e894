// How rows of fp32 or bf16 columns are dealt to waves and workgroups, for the
// kernels over node rows (gfx950).
#pragma once
#include <initializer_list>
#include <type_traits>

#include "kernels.h"
#include "rows8.h"

namespace mgn {

// Threads of a workgroup: a wide row's own, else 256.
constexpr int threads(int TPR) { return TPR > 256 ? TPR : 256; }

// Sums of N values over the TPR threads of a row; every one of them gets the
// same bits.  Rows of several waves add the waves' sums in order, through LDS:
// one barrier a row, with two buffers in turn.
template <int TPR, int N>
struct RowSum {
  static constexpr int WAVES = TPR / 64;
  struct Lds {
    float v[2][N][TPR > 64 ? WAVES : 1];
  };
  Lds& lds;
  int turn = 0;
  __device__ __forceinline__ explicit RowSum(Lds& l) : lds(l) {}
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = group_sum<(TPR < 64 ? TPR : 64)>(v[k]);
    if constexpr (TPR > 64) {
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) lds.v[turn][k][threadIdx.x >> 6] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < N; ++k) {
        v[k] = lds.v[turn][k][0];
#pragma unroll
        for (int e = 1; e < WAVES; ++e) v[k] += lds.v[turn][k][e];
      }
      turn ^= 1;
    }
  }
};

// The rows of a wave (of a workgroup for TPR > 64): RPW at a time from `row`
// on, the lane's own being row + sub.
template <int TPR>
struct Rows {
  static constexpr int RPW = TPR > 64 ? 1 : 64 / TPR;  // rows a wave (workgroup) holds
  static constexpr int NT = threads(TPR), RPB = TPR > 64 ? 1 : NT / TPR;  // threads, rows of a workgroup
  int64_t row, next;
  int sub, t;
  __device__ __forceinline__ Rows() {
    t = threadIdx.x % TPR;
    sub = TPR > 64 ? 0 : (threadIdx.x & 63) / TPR;
    row = (int64_t)blockIdx.x * RPB + (TPR > 64 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * RPW);
    next = (int64_t)gridDim.x * RPB;
  }
};

inline int row_grid(int64_t rows, int rpb, int64_t most) {
  const int64_t b = (rows + rpb - 1) / rpb;
  return (int)(b < most ? b : most);
}

template <int N>
using Int = std::integral_constant<int, N>;

// Calls f(TPR, NV, V, MODE) with the dealing of `cols` columns of the type as
// constants: 16 bytes a run, as few threads a row as hold it.
template <int TYPE, class F>
hipError_t by_cols(int cols, RowMode mode, F f) {
  if (mode == APART) return f(Int<4>(), Int<1>(), Int<4>(), Int<APART>());
  const auto runs = [&](auto m) {
    if constexpr (TYPE == MGN_BF16) {
      const Int<8> v;
      if (cols <= 16) return f(Int<2>(), Int<1>(), v, m);
      if (cols <= 32) return f(Int<4>(), Int<1>(), v, m);
      if (cols <= 64) return f(Int<8>(), Int<1>(), v, m);
      if (cols <= 128) return f(Int<16>(), Int<1>(), v, m);
      if (cols <= 256) return f(Int<32>(), Int<1>(), v, m);
      if (cols <= 512) return f(Int<64>(), Int<1>(), v, m);
      if (cols <= 1024) return f(Int<64>(), Int<2>(), v, m);
      if (cols <= 2048) return f(Int<256>(), Int<1>(), v, m);
      if (cols <= 8192) return f(Int<1024>(), Int<1>(), v, m);
    } else {
      const Int<4> v;
      if (cols <= 8) return f(Int<2>(), Int<1>(), v, m);
      if (cols <= 16) return f(Int<4>(), Int<1>(), v, m);
      if (cols <= 32) return f(Int<8>(), Int<1>(), v, m);
      if (cols <= 64) return f(Int<16>(), Int<1>(), v, m);
      if (cols <= 128) return f(Int<32>(), Int<1>(), v, m);
      if (cols <= 256) return f(Int<64>(), Int<1>(), v, m);
      if (cols <= 1024) return f(Int<64>(), Int<4>(), v, m);
      if (cols <= 2048) return f(Int<256>(), Int<2>(), v, m);
      if (cols <= 8192) return f(Int<1024>(), Int<2>(), v, m);
    }
    return hipErrorInvalidValue;
  };
  return mode == STREAM ? runs(Int<STREAM>()) : mode == WHOLE ? runs(Int<WHOLE>()) : runs(Int<RUNS>());
}

// Calls f(TYPE, TPR, NV, V, MODE) for rows of the type.
template <class F>
hipError_t by_rows(int type, int cols, RowMode mode, F f) {
  if (type == MGN_BF16)
    return by_cols<MGN_BF16>(cols, mode, [&](auto t, auto n, auto v, auto m) { return f(Int<MGN_BF16>(), t, n, v, m); });
  return by_cols<MGN_FP32>(cols, mode, [&](auto t, auto n, auto v, auto m) { return f(Int<MGN_FP32>(), t, n, v, m); });
}

// How a kernel that moves `bytes` reads its arrays of `rows` rows: as whole runs
// where they are that, on 16-byte boundaries, and past the caches where it moves
// more than the last-level cache holds (256 MB).  Above: 2M x 128 bf16 rows with a
// residual into 8-bit rows 313 us through the caches, 286 past them.  Below,
// where the rows may still be cached: 200k of 400k x 256 bf16 rows gathered 28.4
// and 34.2.
inline RowMode row_mode(int64_t bytes, int type, int64_t rows, int cols, std::initializer_list<const void*> arrays) {
  if (cols <= 16 && rows * cols < 16) return APART;
  bool even = cols % (type == MGN_FP32 ? 4 : 8) == 0;
  for (const void* p : arrays) even = even && (uintptr_t)p % 16 == 0;
  return !even ? RUNS : bytes > ((int64_t)256 << 20) ? STREAM : WHOLE;
}
inline int64_t type_bytes(int type) { return type == MGN_FP32 ? 4 : type == MGN_BF16 ? 2 : 1; }

}  // namespace mgn
