// Device parts that the selective scan and its backward share (gfx950).
//
// A wave holds 16 groups of 4 neighbouring columns, one to each 4 of its lanes.
// For what is done once a column (delta, the products with x, the gate, y) lane q
// of the four holds column q; the states of the group's 4 columns are dealt by
// their index, lane q taking states q NL .. q NL + NL - 1 of all four.  So a lane
// reads 4 NL numbers of A and only NL of B and of C, four columns use each of these,
// and the sums over the states end in the lane of their column after two exchanges
// between neighbouring lanes.
#pragma once
#include <type_traits>

#include "kernels.h"
#include "raw.h"

namespace mgn {

constexpr float LOG2E = 1.44269504f, LN2 = 0.693147181f;

// a b, 0 where a is 0 whatever b holds.
__device__ __forceinline__ float mul_or_0(float a, float b) { return a == 0.f ? 0.f : a * b; }
// Whether any lane of the wave says so.
__device__ __forceinline__ bool any(bool v) { return __builtin_amdgcn_ballot_w64(v) != 0; }

// How a wave takes a step: as it comes; or where a column's step has size 0, at which x
// and B may hold anything, or a factor may pass the fp32 range (100 steps of 4,000 x 64
// bf16, 16 states: 132 us; with sizes of 0 in three tenths of the rows' steps 170).
enum Way { PLAIN, CAREFUL };

// The state f h + b.  Zero states stay zero whatever f is.
__device__ __forceinline__ float carried(float f, float h, float b) { return h == 0.f ? b : fmaf(f, h, b); }
// A factor on the way back.  Past the fp32 range it is one of a zero state and passes no
// gradient on.
__device__ __forceinline__ float passed(float f) { return f == INFINITY ? 0.f : f; }

// log(1 + e^v): with e = e^-|v| the logarithm of 1 + e is 2 atanh(s), s = e / (2 + e),
// an odd series in s <= 1 / 3 (five terms, fitted in s^2 to 8e-9 of the sum).  Off by 4
// half-steps of itself around 0, by fewer above, and below by some 0.8 |v| of them, to
// which the rounded argument of the exponential grows (8 at -5, 16 at -20, 63 at -80).
__device__ __forceinline__ float softplus(float v) {
  const float e = __expf(-fabsf(v));
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), w = s * s;
  float p = fmaf(w, 0.28161454f, 0.27964345f);
  p = fmaf(w, p, 0.40024651f);
  p = fmaf(w, p, 0.6666632f);
  p = fmaf(w, p, 2.f);
  return fmaf(s, p, fmaxf(v, 0.f));  // (NaN: s is)
}

// v of lane J of each four.
template <int J>
__device__ __forceinline__ float quad(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), J * 0x55, 0xf, 0xf, true));
}
__device__ __forceinline__ void quads(float v, float (&u)[4]) {
  u[0] = quad<0>(v), u[1] = quad<1>(v), u[2] = quad<2>(v), u[3] = quad<3>(v);
}
// The largest rate of growth among the wave's states (A: times log2(e)), at least 0: a
// factor passes the range at a step of more than 128 / rate, or of less than 0.
template <int NL>
__device__ __forceinline__ float growth(const float (&A)[4][NL]) {
  float most = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int k = 0; k < NL; ++k) most = fmaxf(most, A[j][k]);
  if (!any(most > 0.f)) return 0.f;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
  return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(most)));
}
// Sum over the four lanes of v[q], in lane q.
__device__ __forceinline__ float quad_sums(const float (&v)[4]) {
  const bool b0 = threadIdx.x & 1, b1 = threadIdx.x & 2;
  const float r0 = (b0 ? v[1] : v[0]) + mirror<1>(b0 ? v[0] : v[1]);
  const float r1 = (b0 ? v[3] : v[2]) + mirror<1>(b0 ? v[2] : v[3]);
  return (b1 ? r1 : r0) + mirror<2>(b1 ? r0 : r1);
}

template <int TYPE>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
  float v[1];
  get<1>((const Elem<TYPE>*)p + i, v);
  return v[0];
}
template <int TYPE>
__device__ __forceinline__ void store1(void* p, int64_t i, float v) {
  put<1>((Elem<TYPE>*)p + i, &v);
}

// A lane's states: the NL from `s` on, of which the first `skip` are another lane's and
// count as zeros here.  Where n is no multiple of NL, the last lane's run ends with the
// last state, so that every lane reads a whole run, and none behind its row.
template <int NL, bool FULL>
struct Share {
  int s, skip;
  __device__ __forceinline__ Share(int q, int n) : s(q * NL), skip(0) {
    if constexpr (!FULL) {
      s = q * NL < n - NL ? q * NL : n - NL;
      skip = q * NL - s;
    }
  }
  __device__ __forceinline__ bool has(int k) const { return FULL || k >= skip; }
  __device__ __forceinline__ void mask(float (&v)[NL]) const {
    if constexpr (!FULL)
#pragma unroll
      for (int k = 0; k < NL; ++k) v[k] = has(k) ? v[k] : 0.f;
  }
};

// Those of the numbers that begin at p + i.
template <int TYPE, int NL, bool FULL>
__device__ __forceinline__ void load_n(const void* p, int64_t i, const Share<NL, FULL>& own, float (&v)[NL]) {
  const Elem<TYPE>* r = (const Elem<TYPE>*)p + i;
  constexpr int RUN = 16 / sizeof(Elem<TYPE>) < NL ? 16 / sizeof(Elem<TYPE>) : NL;
#pragma unroll
  for (int k = 0; k < NL; k += RUN) get<RUN>(r + k, v + k);
  own.mask(v);
}

// Where a lane's groups and columns lie: the wave's first ones (the same for all of
// its lanes, so that addresses are a scalar and a lane's 32-bit offset), and the
// lane's from there.
struct Spot {
  int64_t row0, i0, bn0, at0;  // first row; first column of [rows][cols], [rows][n], [rows][cols][n]
  uint32_t o, ob, oa;          // the lane's column, row of n numbers, states of its group's first column
  int64_t row;
  int g, col;  // the group's first column, the lane's
  bool in, ok; // the group, the lane's column is there
  __device__ __forceinline__ Spot(const SsmArgs& a, int64_t group, int q) {
    const int per_row = (a.cols + 3) / 4, ld = (threadIdx.x & 63) >> 2;
    row0 = group >> 32 ? group / per_row : (int64_t)((uint32_t)group / (uint32_t)per_row);
    const int g0 = (int)(group - row0 * per_row);
    const uint32_t down = (uint32_t)(g0 + ld) / (uint32_t)per_row;
    row = row0 + down;
    g = (g0 + ld - (int)down * per_row) * 4;
    col = g + q;
    in = row < a.rows;
    ok = in && col < a.cols;
    i0 = row0 * a.cols + g0 * 4;
    bn0 = row0 * a.n;
    at0 = i0 * a.n;
    // lanes without a column read the first one's
    o = ok ? down * a.cols + col - g0 * 4 : 0;
    ob = in ? down * a.n : 0;
    oa = in ? (down * a.cols + g - g0 * 4) * a.n : 0;
  }
};

template <int NL, bool FULL>
__device__ __forceinline__ void store_n(float* p, int64_t i, const Share<NL, FULL>& own, const float (&v)[NL]) {
  float* r = p + i;
  if constexpr (FULL) {
#pragma unroll
    for (int k = 0; k < NL; k += NL < 4 ? NL : 4) put<(NL < 4 ? NL : 4)>(r + k, v + k);
  } else {
#pragma unroll
    for (int k = 0; k < NL; ++k)
      if (own.has(k)) r[k] = v[k];
  }
}

// A chunk in which a trajectory starts: what enters it does not reach its end.
constexpr float CUT = -INFINITY;

}  // namespace mgn
