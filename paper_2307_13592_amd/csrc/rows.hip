// Node rows outside the network's MLPs: rows held in 8 bits (stored, read
// back) and the root-mean-square norm with the residual's addition, forward
// and backward.
//
// All are bound by memory: a row is read once and stays in registers between
// its sum (or its blocks' largest values) and its result.  Its columns are dealt
// to TPR threads, 4, 16, 32 or 64 lanes of one wave or a workgroup of 256 or 1024
// (rows8.h, Cols), NV runs of V columns each; a wave takes 64 / TPR rows at a
// time.
#include <initializer_list>
#include <type_traits>

#include "kernels.h"
#include "rows8.h"

namespace mgn {
namespace {

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

// --------------------------------------------------------- rows in 8 bits ---

template <int TPR, int NV, int V, bool VEC, int TI>
__global__ __launch_bounds__(threads(TPR)) void store8_kernel(Rows8Args a) {
  using D = Cols<TPR, V, VEC>;
  const int nb = rows8_blocks(a.cols);
  Rows<TPR> w;
  for (; w.row < a.n; w.row += w.next) {
    const int64_t i = w.row + w.sub;
    bool ok = i < a.n;
    const int64_t r = ok ? (a.rows ? a.rows[i] : i) : 0, s = ok ? (a.slots ? a.slots[i] : i) : 0;
    ok = ok && r >= 0 && r < a.n_rows && s >= 0 && s < a.n_slots;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = D::first(j, w.t);
      float v[V];
      load_cols<TI, D>(a.x, ok ? r * a.cols : 0, 0, c, ok ? a.cols : 0, v);
      store_cols8<D>(a.q + (ok ? s * a.cols : 0), a.scale + (ok ? s * nb : 0), c, a.cols, v, ok);
    }
  }
}

template <int TPR, int NV, int V, bool VEC, int TO>
__global__ __launch_bounds__(threads(TPR)) void load8_kernel(Rows8Args a) {
  using D = Cols<TPR, V, VEC>;
  const int nb = rows8_blocks(a.cols);
  Rows<TPR> w;
  for (; w.row < a.n; w.row += w.next) {
    const int64_t i = w.row + w.sub;
    if (i >= a.n) continue;
    const int64_t r = a.rows ? a.rows[i] : i, s = a.slots ? a.slots[i] : i;
    if (r < 0 || r >= a.n_rows || s < 0 || s >= a.n_slots) continue;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = D::first(j, w.t);
      if (c >= a.cols) continue;
      float v[V];
      load_cols8<D>(a.q + s * a.cols, a.scale[s * nb + c / ROWS8_BLOCK], c, a.cols, v);
      if (a.add) {
        float o[V];
        load_cols<TO, D>(a.out, r * a.cols, 0, c, a.cols, o);
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] += o[k];
      }
      store_cols<TO, D>(a.out, r * a.cols, 0, c, a.cols, v);
    }
  }
}

// --------------------------------------------------- root-mean-square norm ---

template <class D, int NV, int V>
__device__ __forceinline__ void load_weight(const RmsArgs& a, int t, float (&w)[NV][V]) {
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int c = D::first(j, t) + D::STRIDE * k;
      w[j][k] = a.w && c < a.cols ? a.w[c] : 1.f;
    }
}

// y = t / sqrt(mean(t^2) + eps) * w for t = x + res, in fp32; t is rounded
// once where it is stored, y once where it is stored (y is formed from the
// unrounded t).
template <int TPR, int NV, int V, bool VEC, int TI, int TO>
__global__ __launch_bounds__(threads(TPR)) void rms_norm_kernel(RmsArgs a) {
  using D = Cols<TPR, V, VEC>;
  __shared__ typename RowSum<TPR, 1>::Lds lds;
  RowSum<TPR, 1> sum(lds);
  const int nb = rows8_blocks(a.cols);
  Rows<TPR> q;
  float w[NV][V];
  load_weight<D>(a, q.t, w);
  const float mean = 1.f / (float)a.cols;
  for (; q.row < a.rows; q.row += q.next) {
    const int64_t base = q.row * a.cols;
    const uint32_t o = (uint32_t)(q.sub * a.cols);
    const int cols = q.row + q.sub < a.rows ? a.cols : 0;
    float v[NV][V], s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) load_cols<TI, D>(a.x, base, o, D::first(j, q.t), cols, v[j]);
    if (a.res) {
      float r[NV][V];
#pragma unroll
      for (int j = 0; j < NV; ++j) load_cols<TI, D>(a.res, base, o, D::first(j, q.t), cols, r[j]);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) v[j][k] += r[j][k];
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) s[0] += v[j][k] * v[j][k];
    sum(s);
    const float inv = rsqrtf(s[0] * mean + a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = D::first(j, q.t);
      if (a.total) store_cols<TI, D>(a.total, base, o, c, cols, v[j]);
      float y[V];
#pragma unroll
      for (int k = 0; k < V; ++k) y[k] = v[j][k] * inv * w[j][k];
      if constexpr (TO == MGN_E4M3)
        store_cols8<D>((uint8_t*)a.y + base + o, a.y_scale + (q.row + q.sub) * nb, c, a.cols, y, cols > 0);
      else
        store_cols<TO, D>(a.y, base, o, c, cols, y);
    }
  }
}

// Backward of one row, u = t inv (the normalised row):
//   dt = (w dy - u mean(u w dy)) inv + d_total;  dw += dy u.
// Each thread sums dw of its columns over its rows in fp32; the workgroup's
// row groups are added in order and leave one partial per column.
template <int TPR, int NV, int V, bool VEC, int TI>
__global__ __launch_bounds__(threads(TPR)) void rms_grad_kernel(RmsArgs a) {
  using D = Cols<TPR, V, VEC>;
  constexpr int NT = threads(TPR), GROUPS = NT / TPR, W = NV * TPR * V;  // row groups; columns dealt to one
  __shared__ typename RowSum<TPR, 2>::Lds lds;
  RowSum<TPR, 2> sums(lds);
  __shared__ float part[GROUPS > 1 ? GROUPS * W : 1];
  Rows<TPR> q;
  float w[NV][V], dw[NV][V];
  load_weight<D>(a, q.t, w);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k) dw[j][k] = 0.f;
  const float mean = 1.f / (float)a.cols;
  for (; q.row < a.rows; q.row += q.next) {
    const int64_t base = q.row * a.cols;
    const uint32_t o = (uint32_t)(q.sub * a.cols);
    const int cols = q.row + q.sub < a.rows ? a.cols : 0;
    float v[NV][V], g[NV][V], r[NV][V], s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      load_cols<TI, D>(a.x, base, o, D::first(j, q.t), cols, v[j]);
      load_cols<TI, D>(a.dy, base, o, D::first(j, q.t), cols, g[j]);
      if (a.res) load_cols<TI, D>(a.res, base, o, D::first(j, q.t), cols, r[j]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        s[0] += v[j][k] * v[j][k];
        s[1] += v[j][k] * (g[j][k] * w[j][k]);
      }
    sums(s);
    const float inv = rsqrtf(s[0] * mean + a.eps);
    const float m = s[1] * inv * mean;  // mean(u w dy)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float d[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float u = v[j][k] * inv;
        d[k] = (g[j][k] * w[j][k] - u * m) * inv;
        if (a.res) d[k] += r[j][k];
        dw[j][k] += g[j][k] * u;
      }
      store_cols<TI, D>(a.total, base, o, D::first(j, q.t), cols, d);
    }
  }
  if (!a.part) return;
  float* dst = a.part + (int64_t)blockIdx.x * a.cols;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int c = D::first(j, q.t) + D::STRIDE * k;
        if (c < a.cols) dst[c] = dw[j][k];
      }
  } else {
    const int grp = threadIdx.x / TPR;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) part[grp * W + D::first(j, q.t) + D::STRIDE * k] = dw[j][k];
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += NT) {
      float total = part[c];
      for (int e = 1; e < GROUPS; ++e) total += part[e * W + c];
      dst[c] = total;
    }
  }
}

// dw from the workgroups' partials, added in fp64 in a fixed order: a wave
// per column group of 16 columns, four partial rows at a time.
constexpr int DW_NT = 256;
__global__ __launch_bounds__(DW_NT) void rms_dw_kernel(const float* __restrict__ part, int parts, int cols, int accumulate,
                                                    float* __restrict__ dw) {
  __shared__ double lds[DW_NT];
  const int c = blockIdx.x * 16 + threadIdx.x % 16, g = threadIdx.x / 16;
  double s = 0;
  if (c < cols)
    for (int q = g; q < parts; q += 16) s += part[(int64_t)q * cols + c];
  lds[threadIdx.x] = s;
  __syncthreads();
  if (g == 0 && c < cols) {
    for (int q = 1; q < 16; ++q) s += lds[q * 16 + threadIdx.x];
    dw[c] = (float)(accumulate ? s + dw[c] : s);
  }
}

// Rows at a time are dealt to at most this many workgroups, which then go
// through them in turn.
constexpr int ROW_GRID = 8192;
int row_grid(int64_t rows, int rpb, int most) {
  const int64_t b = (rows + rpb - 1) / rpb;
  return (int)(b < most ? b : most);
}

template <int N>
using Int = std::integral_constant<int, N>;

// Calls f(TPR, NV, V, VEC) with the dealing of `cols` columns as constants.
// vec: how many columns every array allows to be read at once (8, 4 or 1).  8
// columns a thread (16 bytes of bf16) halve the instructions a row costs.
// VMAX: the most the operands' types make use of.
template <int VMAX, class F>
hipError_t by_cols(int cols, int vec, F f) {
  if (cols <= 16) return f(Int<4>(), Int<1>(), Int<4>(), std::false_type());
  if constexpr (VMAX == 8)
    if (vec == 8) {
      const Int<8> v;
      const std::true_type y;
      if (cols <= 128) return f(Int<16>(), Int<1>(), v, y);
      if (cols <= 256) return f(Int<32>(), Int<1>(), v, y);
      if (cols <= 1024) return f(Int<64>(), Int<2>(), v, y);
      if (cols <= 2048) return f(Int<256>(), Int<1>(), v, y);
      if (cols <= 8192) return f(Int<1024>(), Int<1>(), v, y);
      return hipErrorInvalidValue;
    }
  const Int<4> v;
  const auto four = [&](auto y) {
    if (cols <= 64) return f(Int<16>(), Int<1>(), v, y);
    if (cols <= 128) return f(Int<32>(), Int<1>(), v, y);
    if (cols <= 256) return f(Int<64>(), Int<1>(), v, y);
    if (cols <= 1024) return f(Int<64>(), Int<4>(), v, y);
    if (cols <= 2048) return f(Int<256>(), Int<2>(), v, y);
    if (cols <= 8192) return f(Int<1024>(), Int<2>(), v, y);
    return hipErrorInvalidValue;
  };
  return vec >= 4 ? four(std::true_type()) : four(std::false_type());
}

// Columns of the type that may be read at once: rows begin at multiples of
// `cols` elements from p (null: no array).
int vec_of(const void* p, int type, int cols) {
  if (!p) return 8;
  const int size = type == MGN_FP32 ? 4 : type == MGN_BF16 ? 2 : 1;
  for (int v = 8; v >= 4; v -= 4) {
    const int bytes = v * size < 16 ? v * size : 16;
    if (cols % v == 0 && (uintptr_t)p % bytes == 0) return v;
  }
  return 1;
}
int least(std::initializer_list<int> v) {
  int m = 8;
  for (int x : v) m = x < m ? x : m;
  return m;
}

// Calls f(TYPE, TPR, NV, V, VEC) for rows of the type.
template <class F>
hipError_t by_rows(int type, int cols, int vec, F f) {
  if (type == MGN_BF16)
    return by_cols<8>(cols, vec, [&](auto t, auto n, auto v, auto y) { return f(Int<MGN_BF16>(), t, n, v, y); });
  return by_cols<4>(cols, vec, [&](auto t, auto n, auto v, auto y) { return f(Int<MGN_FP32>(), t, n, v, y); });
}

}  // namespace

hipError_t launch_rows_store8(const Rows8Args& a, int type, hipStream_t st) {
  const int vec = least({vec_of(a.x, type, a.cols), vec_of(a.q, MGN_E4M3, a.cols)});
  return by_rows(type, a.cols, vec, [&](auto ti, auto tpr, auto nv, auto v, auto y) {
    hipLaunchKernelGGL((store8_kernel<tpr(), nv(), v(), y(), ti()>), dim3(row_grid(a.n, Rows<tpr()>::RPB, ROW_GRID)),
                       dim3(Rows<tpr()>::NT), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_rows_load8(const Rows8Args& a, int type, hipStream_t st) {
  const int vec = least({vec_of(a.out, type, a.cols), vec_of(a.q, MGN_E4M3, a.cols)});
  return by_rows(type, a.cols, vec, [&](auto to, auto tpr, auto nv, auto v, auto y) {
    hipLaunchKernelGGL((load8_kernel<tpr(), nv(), v(), y(), to()>), dim3(row_grid(a.n, Rows<tpr()>::RPB, ROW_GRID)),
                       dim3(Rows<tpr()>::NT), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_rms_norm(const RmsArgs& a, int type, int y_type, hipStream_t st) {
  const int vec = least({vec_of(a.x, type, a.cols), vec_of(a.res, type, a.cols), vec_of(a.total, type, a.cols),
                         vec_of(a.y, y_type, a.cols)});
  return by_rows(type, a.cols, vec, [&](auto ti, auto tpr, auto nv, auto v, auto y) {
    const dim3 grid(row_grid(a.rows, Rows<tpr()>::RPB, ROW_GRID));
    if (y_type == MGN_E4M3)
      hipLaunchKernelGGL((rms_norm_kernel<tpr(), nv(), v(), y(), ti(), MGN_E4M3>), grid, dim3(Rows<tpr()>::NT), 0, st, a);
    else if (y_type == MGN_BF16)
      hipLaunchKernelGGL((rms_norm_kernel<tpr(), nv(), v(), y(), ti(), MGN_BF16>), grid, dim3(Rows<tpr()>::NT), 0, st, a);
    else
      hipLaunchKernelGGL((rms_norm_kernel<tpr(), nv(), v(), y(), ti(), MGN_FP32>), grid, dim3(Rows<tpr()>::NT), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_rms_norm_grad(const RmsArgs& a, int type, float* dw, int accumulate, hipStream_t st) {
  int grid = 0;
  if (a.rows > 0) {
    const int vec = least({vec_of(a.x, type, a.cols), vec_of(a.res, type, a.cols), vec_of(a.total, type, a.cols),
                           vec_of(a.dy, type, a.cols)});
    const hipError_t e = by_rows(type, a.cols, vec, [&](auto ti, auto tpr, auto nv, auto v, auto y) {
      grid = row_grid(a.rows, Rows<tpr()>::RPB, MGN_RMS_WORK_PER_COL);
      hipLaunchKernelGGL((rms_grad_kernel<tpr(), nv(), v(), y(), ti()>), dim3(grid), dim3(Rows<tpr()>::NT), 0, st, a);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (!dw) return hipSuccess;
  hipLaunchKernelGGL(rms_dw_kernel, dim3((a.cols + 15) / 16), dim3(DW_NT), 0, st, a.part, grid, a.cols, accumulate, dw);
  return hipGetLastError();
}

}  // namespace mgn
