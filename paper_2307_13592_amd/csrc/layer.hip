// Layer norm of node rows with the residual's addition, forward and backward,
// and the sums over columns of partials that the weight gradients end in.
//
//   t = x + res,  m = mean(t),  u = (t - m) / sqrt(mean((t - m)^2) + eps),
//   y = u w + b;
//   dt = (g - mean(g) - u mean(g u)) / sqrt(..) + d_total with g = w dy,
//   dw += dy u,  db += dy.
// Bound by memory, as the other row kernels (rows.hip): a row is read once and
// stays in registers through its two sums, dealt the same way.  The variance is
// of the deviations from the mean as it was rounded, so an offset costs no digits,
// and what that rounding left, the mean of the deviations, is taken off in the same
// pass: a row of equal values is its bias.  2M x 128 bf16 rows with a residual 336 us
// (6.1 TB/s), into 8-bit rows 286 (6.3); the backward of 1M x 128 fp32 rows 361 us (5.7),
// bf16 188 (5.4).
#include "row_deal.h"

namespace mgn {
namespace {

template <class D, int NV, int V>
__device__ __forceinline__ void load_vector(const float* p, float none, int t, int cols, float (&w)[NV][V]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (p) {
      load_values<D>(p, D::first(j, t), cols, w[j]);
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) w[j][k] = none;
    }
  }
}

// v <- v - mean, 0 past the row's end.
template <class D, int NV, int V>
__device__ __forceinline__ void deviations(float m, int t, int cols, float (&v)[NV][V]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = D::first(j, t);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if constexpr (D::EVEN) v[j][k] = c < cols ? v[j][k] - m : 0.f;
      else v[j][k] = c + D::STRIDE * k < cols ? v[j][k] - m : 0.f;
    }
  }
}

// NaN where a row's sum of squared deviations is infinite or NaN because a value
// is (v - v), 0 where finite values passed the fp32 range.
template <int TPR, int NV, int V>
__device__ __forceinline__ float lost(RowSum<TPR, 1>& sum, const float (&v)[NV][V]) {
  float s[1] = {0.f};
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k) s[0] += v[j][k] - v[j][k];
  sum(s);
  return s[0];
}

template <int TPR, int NV, int V, int MODE, int TI, int TO>
__global__ __launch_bounds__(threads(TPR)) void layer_norm_kernel(LayerArgs a) {
  using D = Cols<TPR, V, MODE>;
  __shared__ typename RowSum<TPR, 1>::Lds lds1;
  __shared__ typename RowSum<TPR, 2>::Lds lds2;
  RowSum<TPR, 1> sum(lds1);
  RowSum<TPR, 2> sums(lds2);
  const int nb = rows8_blocks(a.cols);
  Rows<TPR> q;
  float w[NV][V], b[NV][V];
  load_vector<D>(a.w, 1.f, q.t, a.cols, w);
  load_vector<D>(a.b, 0.f, q.t, a.cols, b);
  const float mean = 1.f / (float)a.cols;
  for (; q.row < a.rows; q.row += q.next) {
    const int64_t base = q.row * a.cols;
    const int64_t left = a.rows * a.cols - base;
    const uint32_t o = (uint32_t)(q.sub * a.cols);
    const int cols = q.row + q.sub < a.rows ? a.cols : 0;
    float v[NV][V], m[1] = {0.f}, s[2] = {0.f, 0.f};
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
    for (int j = 0; j < NV; ++j) {
      if (a.total) store_cols<TI, D>(a.total, base, o, D::first(j, q.t), cols, v[j]);
#pragma unroll
      for (int k = 0; k < V; ++k) m[0] = fmaf(v[j][k], mean, m[0]);  // (shares of the mean: no sum passes the range)
    }
    sum(m);
    float d[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) d[j][k] = v[j][k];
    deviations<D>(m[0], q.t, cols, d);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        s[0] += d[j][k];
        s[1] += d[j][k] * d[j][k];
      }
    sums(s);
    float off = s[0] * mean, inv = rsqrtf(fmaxf(s[1] * mean - off * off, 0.f) + a.eps);
    if (!(s[1] < INFINITY)) {
      const float z = lost<TPR>(sum, v);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) d[j][k] = z;
      off = 0.f;
      inv = 1.f;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = D::first(j, q.t);
      float y[V];
#pragma unroll
      for (int k = 0; k < V; ++k) y[k] = fmaf((d[j][k] - off) * inv, w[j][k], b[j][k]);
      if constexpr (TO == MGN_E4M3) {
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (c + D::STRIDE * k >= cols) y[k] = 0.f;  // no part of the block's largest value
        store_cols8<D>((uint8_t*)a.y + base + o, a.y_scale + (q.row + q.sub) * nb, c, a.cols, y, cols > 0);
      } else {
        store_cols<TO, D>(a.y, base, o, c, cols, y);
      }
    }
  }
}

// dw and db are long sums over rows: DW_ROWS rows in fp32, these in fp64 (in LDS,
// each thread its own places; rows of a whole workgroup in fp64 registers), one
// partial a column and workgroup, rounded to fp32 once.
constexpr int DW_ROWS = 8;
template <int TPR, int NV, int V, int MODE, int TI>
__global__ __launch_bounds__(threads(TPR)) void layer_grad_kernel(LayerArgs a) {
  using D = Cols<TPR, V, MODE>;
  constexpr int NT = threads(TPR), GROUPS = NT / TPR, W = NV * TPR * V;
  __shared__ typename RowSum<TPR, 1>::Lds lds1;
  __shared__ typename RowSum<TPR, 4>::Lds lds4;
  RowSum<TPR, 1> sum(lds1);
  RowSum<TPR, 4> sums(lds4);
  __shared__ double part[2][GROUPS > 1 ? GROUPS * W : 1];
  const int mine = threadIdx.x / TPR * W;
  Rows<TPR> q;
  float w[NV][V];
  std::conditional_t<(GROUPS > 1), float, double> dw[NV][V], db[NV][V];
  int turn = 0;
  load_vector<D>(a.w, 1.f, q.t, a.cols, w);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      dw[j][k] = db[j][k] = 0;
      if constexpr (GROUPS > 1) {
        const int at = mine + D::first(j, q.t) + D::STRIDE * k;
        part[0][at] = part[1][at] = 0;
      }
    }
  const auto add = [&] {
    if constexpr (GROUPS > 1) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const int at = mine + D::first(j, q.t) + D::STRIDE * k;
          part[0][at] += dw[j][k], part[1][at] += db[j][k];
          dw[j][k] = db[j][k] = 0;
        }
    }
  };
  const float mean = 1.f / (float)a.cols;
  for (; q.row < a.rows; q.row += q.next) {
    const int64_t base = q.row * a.cols;
    const int64_t left = a.rows * a.cols - base;
    const uint32_t o = (uint32_t)(q.sub * a.cols);
    const int cols = q.row + q.sub < a.rows ? a.cols : 0;
    float v[NV][V], g[NV][V], r[NV][V], m[1] = {0.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      load_cols<TI, D>(a.x, base, o, D::first(j, q.t), cols, left, v[j]);
      load_cols<TI, D>(a.dy, base, o, D::first(j, q.t), cols, left, g[j]);
      if (a.res) load_cols<TI, D>(a.res, base, o, D::first(j, q.t), cols, left, r[j]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) m[0] = fmaf(v[j][k], mean, m[0]);
    sum(m);
    float d[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) d[j][k] = v[j][k];
    deviations<D>(m[0], q.t, cols, d);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float wg = g[j][k] * w[j][k];
        s[0] += d[j][k];
        s[1] += d[j][k] * d[j][k];
        s[2] += wg;
        s[3] += wg * d[j][k];
      }
    sums(s);
    float off = s[0] * mean, inv = rsqrtf(fmaxf(s[1] * mean - off * off, 0.f) + a.eps);
    float mg = s[2] * mean, mu = (s[3] - off * s[2]) * inv * mean;  // mean(g), mean(g u)
    if (!(s[1] < INFINITY)) {
      // squares past the fp32 range: no gradient through the norm, and none of
      // w; for a row that is not finite NaNs
      const float z = lost<TPR>(sum, v);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) d[j][k] = 0.f;
      off = 0.f;
      inv = mg = mu = z;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float e[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float u = (d[j][k] - off) * inv;
        e[k] = (g[j][k] * w[j][k] - mg - u * mu) * inv;
        if (a.res) e[k] += r[j][k];
        dw[j][k] += g[j][k] * u;
        db[j][k] += g[j][k];
      }
      store_cols<TI, D>(a.total, base, o, D::first(j, q.t), cols, e);
    }
    if (++turn % DW_ROWS == 0) add();
  }
  if (!a.part) return;
  float* dst = a.part + (int64_t)blockIdx.x * 2 * a.cols;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int c = D::first(j, q.t) + D::STRIDE * k;
        if (c < a.cols) dst[c] = (float)dw[j][k], dst[a.cols + c] = (float)db[j][k];
      }
  } else {
    add();
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.cols; i += NT) {
      const int which = i >= a.cols, c = i - which * a.cols;
      double total = part[which][c];
      for (int e = 1; e < GROUPS; ++e) total += part[which][e * W + c];
      dst[i] = (float)total;
    }
  }
}

// Column sums of partials [parts][cols], in fp64 in a fixed order, into up to
// three arrays that share the columns: a workgroup per SUM_COLS columns, SUM_G of
// its threads to a column, each over every SUM_G-th partial.
constexpr int SUM_NT = 1024, SUM_COLS = 16, SUM_G = SUM_NT / SUM_COLS;
__global__ __launch_bounds__(SUM_NT) void col_sums_kernel(ColSums a) {
  __shared__ double lds[SUM_NT];
  const int64_t c = (int64_t)blockIdx.x * SUM_COLS + threadIdx.x % SUM_COLS;
  const int g = threadIdx.x / SUM_COLS;
  double s = 0;
  if (c < a.cols)
#pragma unroll 8
    for (int64_t q = g; q < a.parts; q += SUM_G) s += a.part[q * a.cols + c];
  lds[threadIdx.x] = s;
  for (int n = SUM_G / 2; n; n /= 2) {
    __syncthreads();
    if (g < n) lds[threadIdx.x] += lds[threadIdx.x + n * SUM_COLS];
  }
  if (g != 0 || c >= a.cols) return;
  int64_t at = c;
  int k = 0;
  while (k < 2 && at >= a.len[k]) at -= a.len[k++];
  float* const dst = a.dst[k];
  if (dst) dst[at] = (float)(a.accumulate ? lds[threadIdx.x] + dst[at] : lds[threadIdx.x]);
}

// Workgroups of a forward launch, as the root-mean-square norm's.
constexpr int64_t NORM_GRID = 32768, NORM_GRID_RUNS = 8192, PARTS = MGN_LAYER_WORK_PER_COL / 2;

}  // namespace

hipError_t launch_col_sums(const ColSums& a, hipStream_t st) {
  if (a.cols <= 0) return hipSuccess;
  hipLaunchKernelGGL(col_sums_kernel, dim3((unsigned)((a.cols + SUM_COLS - 1) / SUM_COLS)), dim3(SUM_NT), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_layer_norm(const LayerArgs& a, int type, int y_type, hipStream_t st) {
  const int64_t per = type_bytes(type) * (1 + (a.res != nullptr) + (a.total != nullptr)) + type_bytes(y_type);
  const RowMode mode = row_mode(a.rows * a.cols * per, type, a.rows, a.cols, {a.x, a.res});
  return by_rows(type, a.cols, mode, [&](auto ti, auto tpr, auto nv, auto v, auto y) {
    const dim3 grid(row_grid(a.rows, Rows<tpr()>::RPB, mode == RUNS ? NORM_GRID_RUNS : NORM_GRID));
    if (y_type == MGN_E4M3)
      hipLaunchKernelGGL((layer_norm_kernel<tpr(), nv(), v(), y(), ti(), MGN_E4M3>), grid, dim3(Rows<tpr()>::NT), 0, st, a);
    else if (y_type == MGN_BF16)
      hipLaunchKernelGGL((layer_norm_kernel<tpr(), nv(), v(), y(), ti(), MGN_BF16>), grid, dim3(Rows<tpr()>::NT), 0, st, a);
    else
      hipLaunchKernelGGL((layer_norm_kernel<tpr(), nv(), v(), y(), ti(), MGN_FP32>), grid, dim3(Rows<tpr()>::NT), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_layer_norm_grad(const LayerArgs& a, int type, float* dw, float* db, int accumulate, hipStream_t st) {
  int grid = 0;
  if (a.rows > 0) {
    const RowMode mode = row_mode(a.rows * a.cols * type_bytes(type) * (3 + (a.res != nullptr)), type, a.rows, a.cols,
                                  {a.x, a.dy, a.res});
    const hipError_t e = by_rows(type, a.cols, mode, [&](auto ti, auto tpr, auto nv, auto v, auto y) {
      grid = row_grid(a.rows, Rows<tpr()>::RPB, PARTS);
      hipLaunchKernelGGL((layer_grad_kernel<tpr(), nv(), v(), y(), ti()>), dim3(grid), dim3(Rows<tpr()>::NT), 0, st, a);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (!dw && !db) return hipSuccess;
  return launch_col_sums(ColSums{a.part, grid, 2 * (int64_t)a.cols, {dw, db, nullptr}, {a.cols, a.cols}, accumulate}, st);
}

}  // namespace mgn
