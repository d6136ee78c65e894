// Node rows outside the network's MLPs: rows held in 8 bits (stored, read
// back) and the root-mean-square norm with the residual's addition, forward
// and backward.
//
// All are bound by memory: a row is read once and stays in registers between
// its sum (or its blocks' largest values) and its result.  Its columns are dealt
// to TPR threads, 2 to 64 lanes of one wave or a workgroup of 256 or 1024
// (rows8.h, Cols), NV runs of V columns each; a wave takes 64 / TPR rows at a
// time.  As few threads as hold a row at 16 bytes each: of 1M x 128 bf16 rows the
// norm takes 80 us (6.4 TB/s) and its backward 140 (5.5), against 104 and 235
// with four columns a thread.
// Times here are of calls queued one behind the other on two to four sets of
// arrays; single launches under a kernel trace take some per cent longer.
#include <type_traits>

#include "row_deal.h"

namespace mgn {
namespace {

// --------------------------------------------------------- rows in 8 bits ---
// Storing takes each block's largest finite magnitude over its lanes (DPP), the
// scale from its bits and the codes from the card's conversion; reading back is
// that conversion and one product.  Bound by HBM: 2M x 128 fp32 rows stored in
// 236 us (5.5 TB/s) and read back in 175 - 208 (6.2 and more); 100k of 2M such
// rows gathered by an index list, 512 bytes at a random place each, 14 us (4.5
// TB/s), and read back into random rows 11 (5.8).

template <int TPR, int NV, int V, int MODE, int TI>
__global__ __launch_bounds__(threads(TPR)) void store8_kernel(Rows8Args a) {
  using D = Cols<TPR, V, MODE>;
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
      load_cols<TI, D>(a.x, ok ? r * a.cols : 0, 0, c, ok ? a.cols : 0, (a.n_rows - r) * a.cols, v);
      store_cols8<D>(a.q + (ok ? s * a.cols : 0), a.scale + (ok ? s * nb : 0), c, a.cols, v, ok);
    }
  }
}

template <int TPR, int NV, int V, int MODE, int TO>
__global__ __launch_bounds__(threads(TPR)) void load8_kernel(Rows8Args a) {
  using D = Cols<TPR, V, MODE>;
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
        load_cols<TO, D>(a.out, r * a.cols, 0, c, a.cols, (a.n_rows - r) * a.cols, o);
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
  for (int j = 0; j < NV; ++j) {
    if (a.w) {
      load_values<D>(a.w, D::first(j, t), a.cols, w[j]);
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) w[j][k] = 1.f;
    }
  }
}

// y = t / sqrt(mean(t^2) + eps) * w for t = x + res, in fp32; t is rounded
// once where it is stored, y once where it is stored (y is formed from the
// unrounded t).  1M x 128 fp32 rows with a residual: 357 us, 5.7 TB/s; 2M x 128
// bf16 rows with one into 8-bit rows: 286 us, 6.3 TB/s.
template <int TPR, int NV, int V, int MODE, int TI, int TO>
__global__ __launch_bounds__(threads(TPR)) void rms_norm_kernel(RmsArgs a) {
  using D = Cols<TPR, V, MODE>;
  __shared__ typename RowSum<TPR, 1>::Lds lds;
  RowSum<TPR, 1> sum(lds);
  const int nb = rows8_blocks(a.cols);
  Rows<TPR> q;
  float w[NV][V];
  load_weight<D>(a, q.t, w);
  const float mean = 1.f / (float)a.cols;
  for (; q.row < a.rows; q.row += q.next) {
    const int64_t base = q.row * a.cols;
    const int64_t left = a.rows * a.cols - base;
    const uint32_t o = (uint32_t)(q.sub * a.cols);
    const int cols = q.row + q.sub < a.rows ? a.cols : 0;
    float v[NV][V], s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) load_cols<TI, D>(a.x, base, o, D::first(j, q.t), cols, left, v[j]);
    if (a.res) {
      float r[NV][V];
#pragma unroll
      for (int j = 0; j < NV; ++j) load_cols<TI, D>(a.res, base, o, D::first(j, q.t), cols, left, r[j]);
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
// (Where w dy lies along t, as in a row of one column, the difference cancels to a
// share eps inv^2 of its terms, and carries their rounding.)
// dw is a long sum over rows: a thread adds its columns' products over DW_ROWS
// rows in fp32 and these in fp64, in LDS (rows of a whole workgroup in fp64 at
// once; fp64 registers for all cost 100,000 x 999 bf16 118 -> 160 us).  The
// workgroup's row groups are added in order, in fp64, and leave one partial per
// column, rounded to fp32 (at most half a step of it), of at most
// MGN_RMS_WORK_PER_COL workgroups.  Of 1M x 128 fp32 rows dw is off by 7.5e-8 of
// itself (its products alone 5.3e-8, groups of 16 and 4 rows 8.8e-8 and 6.8e-8,
// all of a thread's rows in fp32 2.0e-7); with d_total 357 us, 5.7 TB/s (twice as
// many workgroups 377 - 427; groups of 4 rows up to 2 % longer on bf16 rows).
// Unaligned rows (100,003 x 77 bf16) take 16 us, 2.9 TB/s: their stores share
// lines, so that 1.5 times the bytes are written, and six rounds of rows a wave
// leave the last one part empty.
constexpr int DW_ROWS = 8;
template <int TPR, int NV, int V, int MODE, int TI>
__global__ __launch_bounds__(threads(TPR)) void rms_grad_kernel(RmsArgs a) {
  using D = Cols<TPR, V, MODE>;
  constexpr int NT = threads(TPR), GROUPS = NT / TPR, W = NV * TPR * V;  // row groups; columns dealt to one
  __shared__ typename RowSum<TPR, 2>::Lds lds;
  RowSum<TPR, 2> sums(lds);
  // [row group][column]: each thread adds to its own places only
  __shared__ double part[GROUPS > 1 ? GROUPS * W : 1];
  double* const mine = part + threadIdx.x / TPR * W;
  Rows<TPR> q;
  float w[NV][V];
  std::conditional_t<(GROUPS > 1), float, double> dw[NV][V];
  int turn = 0;
  load_weight<D>(a, q.t, w);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      dw[j][k] = 0;
      if constexpr (GROUPS > 1) mine[D::first(j, q.t) + D::STRIDE * k] = 0;
    }
  const auto add = [&] {
    if constexpr (GROUPS > 1) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) mine[D::first(j, q.t) + D::STRIDE * k] += dw[j][k], dw[j][k] = 0;
    }
  };
  const float mean = 1.f / (float)a.cols;
  for (; q.row < a.rows; q.row += q.next) {
    const int64_t base = q.row * a.cols;
    const int64_t left = a.rows * a.cols - base;
    const uint32_t o = (uint32_t)(q.sub * a.cols);
    const int cols = q.row + q.sub < a.rows ? a.cols : 0;
    float v[NV][V], g[NV][V], r[NV][V], s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      load_cols<TI, D>(a.x, base, o, D::first(j, q.t), cols, left, v[j]);
      load_cols<TI, D>(a.dy, base, o, D::first(j, q.t), cols, left, g[j]);
      if (a.res) load_cols<TI, D>(a.res, base, o, D::first(j, q.t), cols, left, r[j]);
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
    float m = s[1] * inv * mean;  // mean(u w dy)
    if (inv == 0.f) {
      // squares past the fp32 range: no gradient through the norm.  The second
      // sum may have passed it too; m is 0 for a finite row, NaN for others.
      s[0] = s[1] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) s[0] += v[j][k] - v[j][k];
      sums(s);
      m = s[0];
    }
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
    if (++turn % DW_ROWS == 0) add();
  }
  if (!a.part) return;
  float* dst = a.part + (int64_t)blockIdx.x * a.cols;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int c = D::first(j, q.t) + D::STRIDE * k;
        if (c < a.cols) dst[c] = (float)dw[j][k];
      }
  } else {
    add();
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += NT) {
      double total = part[c];
      for (int e = 1; e < GROUPS; ++e) total += part[e * W + c];
      dst[c] = (float)total;
    }
  }
}

// dw from the workgroups' partials, added in fp64 in a fixed order: a workgroup
// per 16 columns, 64 of its threads to a column, each over every 64th partial
// (1024 partials of 128 columns: 4 us; 18 with 16 threads a column).
constexpr int DW_NT = 1024, DW_COLS = 16;
__global__ __launch_bounds__(DW_NT) void rms_dw_kernel(const float* __restrict__ part, int parts, int cols,
                                                       int accumulate, float* __restrict__ dw) {
  constexpr int G = DW_NT / DW_COLS;
  __shared__ double lds[DW_NT];
  const int c = blockIdx.x * DW_COLS + threadIdx.x % DW_COLS, g = threadIdx.x / DW_COLS;
  double s = 0;
  if (c < cols)
#pragma unroll 8
    for (int q = g; q < parts; q += G) s += part[(int64_t)q * cols + c];
  lds[threadIdx.x] = s;
  for (int n = G / 2; n; n /= 2) {
    __syncthreads();
    if (g < n) lds[threadIdx.x] += lds[threadIdx.x + n * DW_COLS];
  }
  if (g == 0 && c < cols) dw[c] = (float)(accumulate ? lds[threadIdx.x] + dw[c] : lds[threadIdx.x]);
}

// Rows at a time are dealt to at most this many workgroups, which then go
// through them in turn: each reads the weights once (1M x 128 fp32 rows with a
// residual 380 us with 8,192, 357 with 32,768, 332 with one turn each; 2M x 128
// bf16 into 8-bit rows 287, 286 and 293; 500k x 256 fp32 into 8-bit rows 117, 113
// and 140).  Rows that are no whole runs, whose weights cost more, prefer 8,192
// (500k x 77 bf16 44 us, 55 with 32,768; 300k x 300 bf16 77 and 86; 500k x 77 fp32
// with a residual 130 and 127).  Storing gathered rows prefers few (200k x 256
// bf16 28.4 us with 8,192, 30.8 with 32,768); reading 8-bit rows back needs no
// turns (2M x 128 to fp32 209 - 220 us with 32,768 workgroups, 175 - 208 with as
// many as there are rows to deal).
constexpr int64_t NORM_GRID = 32768, NORM_GRID_RUNS = 8192, STORE_GRID = 8192, LOAD_GRID = 1 << 20;

}  // namespace

hipError_t launch_rows_store8(const Rows8Args& a, int type, hipStream_t st) {
  const RowMode mode = row_mode(a.n * a.cols * (type_bytes(type) + 1), type, a.n_rows, a.cols, {a.x});
  return by_rows(type, a.cols, mode, [&](auto ti, auto tpr, auto nv, auto v, auto y) {
    hipLaunchKernelGGL((store8_kernel<tpr(), nv(), v(), y(), ti()>), dim3(row_grid(a.n, Rows<tpr()>::RPB, STORE_GRID)),
                       dim3(Rows<tpr()>::NT), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_rows_load8(const Rows8Args& a, int type, hipStream_t st) {
  const RowMode mode = row_mode(0, type, a.n_rows, a.cols, {a.add ? a.out : nullptr});
  return by_rows(type, a.cols, mode, [&](auto to, auto tpr, auto nv, auto v, auto y) {
    hipLaunchKernelGGL((load8_kernel<tpr(), nv(), v(), y(), to()>), dim3(row_grid(a.n, Rows<tpr()>::RPB, LOAD_GRID)),
                       dim3(Rows<tpr()>::NT), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_rms_norm(const RmsArgs& a, int type, int y_type, hipStream_t st) {
  const int64_t per = type_bytes(type) * (1 + (a.res != nullptr) + (a.total != nullptr)) + type_bytes(y_type);
  const RowMode mode = row_mode(a.rows * a.cols * per, type, a.rows, a.cols, {a.x, a.res});
  return by_rows(type, a.cols, mode, [&](auto ti, auto tpr, auto nv, auto v, auto y) {
    const dim3 grid(row_grid(a.rows, Rows<tpr()>::RPB, mode == RUNS ? NORM_GRID_RUNS : NORM_GRID));
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
    const RowMode mode = row_mode(a.rows * a.cols * type_bytes(type) * (3 + (a.res != nullptr)), type, a.rows, a.cols,
                                  {a.x, a.dy, a.res});
    const hipError_t e = by_rows(type, a.cols, mode, [&](auto ti, auto tpr, auto nv, auto v, auto y) {
      grid = row_grid(a.rows, Rows<tpr()>::RPB, MGN_RMS_WORK_PER_COL);
      hipLaunchKernelGGL((rms_grad_kernel<tpr(), nv(), v(), y(), ti()>), dim3(grid), dim3(Rows<tpr()>::NT), 0, st, a);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (!dw) return hipSuccess;
  hipLaunchKernelGGL(rms_dw_kernel, dim3((a.cols + DW_COLS - 1) / DW_COLS), dim3(DW_NT), 0, st, a.part, grid, a.cols, accumulate, dw);
  return hipGetLastError();
}

}  // namespace mgn
