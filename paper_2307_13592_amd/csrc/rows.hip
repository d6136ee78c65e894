// Node rows outside the network's MLPs: rows held in 8 bits (stored, read
// back) and the root-mean-square norm with the residual's addition, forward
// and backward.  A row's columns are dealt to TPR threads (16, 32 or 64 lanes
// of one wave, or a workgroup of 256) in runs of four: thread t holds columns
// (j TPR + t) 4 .. + 3 for j < NV, so that a row is read once, stays in
// registers between its sum and its result, and the 128 columns that share an
// 8-bit scale are 32 neighbouring lanes.
#include "kernels.h"
#include "rows8.h"

namespace mgn {
namespace {

constexpr int NT = 256;

// Sum over the TPR threads of a row; every one of them gets the same value
// (a butterfly: the order of additions does not depend on the lane).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* lds) {
#pragma unroll
  for (int d = 1; d < (TPR < 64 ? TPR : 64); d *= 2) v += __shfl_xor(v, d);
  if constexpr (TPR > 64) {
    __syncthreads();  // the row before may still be reading lds
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (lds[0] + lds[1]) + (lds[2] + lds[3]);
  }
  return v;
}

// --------------------------------------------------------- rows in 8 bits ---

template <int TPR, int NV, bool VEC, int TI>
__global__ __launch_bounds__(NT) void store8_kernel(Rows8Args a) {
  const int t = threadIdx.x % TPR;
  constexpr int RPB = NT / TPR;
  const int nb = rows8_blocks(a.cols);
  for (int64_t i = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; i < a.n; i += (int64_t)gridDim.x * RPB) {
    const int64_t r = a.rows ? a.rows[i] : i, s = a.slots ? a.slots[i] : i;
    if (r < 0 || r >= a.n_rows || s < 0 || s >= a.n_slots) continue;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + t) * 4;
      float v[4];
      load_cols<TI, VEC>(a.x, r * a.cols, c, a.cols, v);
      store_cols8<TPR, VEC>(a.q + s * a.cols, a.scale + s * nb, c, a.cols, v);
    }
  }
}

template <int TPR, int NV, bool VEC, int TO>
__global__ __launch_bounds__(NT) void load8_kernel(Rows8Args a) {
  const int t = threadIdx.x % TPR;
  constexpr int RPB = NT / TPR;
  const int nb = rows8_blocks(a.cols);
  for (int64_t i = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; i < a.n; i += (int64_t)gridDim.x * RPB) {
    const int64_t r = a.rows ? a.rows[i] : i, s = a.slots ? a.slots[i] : i;
    if (r < 0 || r >= a.n_rows || s < 0 || s >= a.n_slots) continue;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + t) * 4;
      if (c >= a.cols) break;
      float v[4];
      load_cols8<VEC>(a.q + s * a.cols, a.scale[s * nb + c / ROWS8_BLOCK], c, a.cols, v);
      if (a.add) {
        float o[4];
        load_cols<TO, VEC>(a.out, r * a.cols, c, a.cols, o);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += o[k];
      }
      store_cols<TO, VEC>(a.out, r * a.cols, c, a.cols, v);
    }
  }
}

// --------------------------------------------------- root-mean-square norm ---

// y = t / sqrt(mean(t^2) + eps) * w for t = x + res, in fp32; t is rounded
// once where it is stored, y once where it is stored (y is formed from the
// unrounded t).
template <int TPR, int NV, bool VEC, int TI, int TO>
__global__ __launch_bounds__(NT) void rms_norm_kernel(RmsArgs a) {
  __shared__ float lds[4];
  const int t = threadIdx.x % TPR;
  constexpr int RPB = NT / TPR;
  const int nb = rows8_blocks(a.cols);
  float w[NV][4];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = (j * TPR + t) * 4 + k;
      w[j][k] = a.w && c < a.cols ? a.w[c] : 1.f;
    }
  const float mean = 1.f / (float)a.cols;
  for (int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; r < a.rows; r += (int64_t)gridDim.x * RPB) {
    const int64_t base = r * a.cols;
    float v[NV][4], s = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + t) * 4;
      load_cols<TI, VEC>(a.x, base, c, a.cols, v[j]);
      if (a.res) {
        float o[4];
        load_cols<TI, VEC>(a.res, base, c, a.cols, o);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[j][k] += o[k];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) s += v[j][k] * v[j][k];
    }
    s = row_sum<TPR>(s, lds);
    const float inv = 1.f / sqrtf(s * mean + a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + t) * 4;
      if (a.total) store_cols<TI, VEC>(a.total, base, c, a.cols, v[j]);
      float y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = v[j][k] * inv * w[j][k];
      if constexpr (TO == MGN_E4M3)
        store_cols8<TPR, VEC>((uint8_t*)a.y + base, a.y_scale + r * nb, c, a.cols, y);
      else
        store_cols<TO, VEC>(a.y, base, c, a.cols, y);
    }
  }
}

// Backward of one row, u = t inv (the normalised row):
//   dt = (w dy - u mean(u w dy)) inv + d_total;  dw += dy u.
// Each thread sums dw of its columns over its rows in fp32; the workgroup's
// row groups are added in order and leave one partial per column.
template <int TPR, int NV, bool VEC, int TI>
__global__ __launch_bounds__(NT) void rms_grad_kernel(RmsArgs a) {
  __shared__ float lds[4];
  __shared__ float part[NV * TPR * 4 <= 1024 ? NT * NV * 4 : 1];
  const int t = threadIdx.x % TPR;
  constexpr int RPB = NT / TPR;
  float w[NV][4], dw[NV][4];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = (j * TPR + t) * 4 + k;
      w[j][k] = a.w && c < a.cols ? a.w[c] : 1.f;
      dw[j][k] = 0.f;
    }
  const float mean = 1.f / (float)a.cols;
  for (int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; r < a.rows; r += (int64_t)gridDim.x * RPB) {
    const int64_t base = r * a.cols;
    float v[NV][4], g[NV][4], s = 0.f, p = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + t) * 4;
      load_cols<TI, VEC>(a.x, base, c, a.cols, v[j]);
      load_cols<TI, VEC>(a.dy, base, c, a.cols, g[j]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s += v[j][k] * v[j][k];
        p += v[j][k] * (g[j][k] * w[j][k]);
      }
    }
    s = row_sum<TPR>(s, lds);
    p = row_sum<TPR>(p, lds);
    const float inv = 1.f / sqrtf(s * mean + a.eps);
    const float m = p * inv * mean;  // mean(u w dy)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + t) * 4;
      float d[4], o[4] = {0.f, 0.f, 0.f, 0.f};
      if (a.res) load_cols<TI, VEC>(a.res, base, c, a.cols, o);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float u = v[j][k] * inv;
        d[k] = (g[j][k] * w[j][k] - u * m) * inv + o[k];
        dw[j][k] += g[j][k] * u;
      }
      store_cols<TI, VEC>(a.total, base, c, a.cols, d);
    }
  }
  if (!a.part) return;
  float* dst = a.part + (int64_t)blockIdx.x * a.cols;
  if constexpr (TPR == NT) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = (j * TPR + t) * 4 + k;
        if (c < a.cols) dst[c] = dw[j][k];
      }
  } else {
    constexpr int W = NV * TPR * 4;  // columns dealt to a row's threads
    const int grp = threadIdx.x / TPR;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) part[grp * W + (j * TPR + t) * 4 + k] = dw[j][k];
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += NT) {
      float sum = part[c];
      for (int q = 1; q < RPB; ++q) sum += part[q * W + c];
      dst[c] = sum;
    }
  }
}

// dw from the workgroups' partials, added in fp64 in a fixed order: a wave
// per column group of 16 columns, four partial rows at a time.
__global__ __launch_bounds__(NT) void rms_dw_kernel(const float* __restrict__ part, int parts, int cols, int accumulate,
                                                    float* __restrict__ dw) {
  __shared__ double lds[NT];
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

int row_grid(int64_t rows, int rpb, int most) {
  const int64_t b = (rows + rpb - 1) / rpb;
  return (int)(b < most ? b : most);
}

constexpr int ROW_GRID = 8192;

// Calls f(TPR, NV) with the dealing of `cols` columns as constants.
template <class F>
hipError_t by_cols(int cols, F f) {
  if (cols <= 64) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
  if (cols <= 128) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
  if (cols <= 256) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
  if (cols <= 1024) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
  if (cols <= 8192) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 8>());
  return hipErrorInvalidValue;
}

template <class F>
hipError_t by_flag(bool v, F f) {
  return v ? f(std::true_type()) : f(std::false_type());
}

template <class F>
hipError_t by_type(int type, F f) {
  return type == MGN_BF16 ? f(std::integral_constant<int, MGN_BF16>()) : f(std::integral_constant<int, MGN_FP32>());
}

// Whether rows of `cols` columns of the type may be read four columns at a time.
bool vec_ok(const void* p, int type, int cols) {
  return cols % 4 == 0 && (uintptr_t)p % (type == MGN_FP32 ? 16 : type == MGN_BF16 ? 8 : 4) == 0;
}

}  // namespace

hipError_t launch_rows_store8(const Rows8Args& a, int type, hipStream_t st) {
  const bool vec = vec_ok(a.x, type, a.cols) && vec_ok(a.q, MGN_E4M3, a.cols);
  return by_cols(a.cols, [&](auto tpr, auto nv) {
    return by_flag(vec, [&](auto v) {
      return by_type(type, [&](auto ti) {
        hipLaunchKernelGGL((store8_kernel<tpr(), nv(), v(), ti()>), dim3(row_grid(a.n, NT / tpr(), ROW_GRID)), dim3(NT), 0, st, a);
        return hipGetLastError();
      });
    });
  });
}

hipError_t launch_rows_load8(const Rows8Args& a, int type, hipStream_t st) {
  const bool vec = vec_ok(a.out, type, a.cols) && vec_ok(a.q, MGN_E4M3, a.cols);
  return by_cols(a.cols, [&](auto tpr, auto nv) {
    return by_flag(vec, [&](auto v) {
      return by_type(type, [&](auto to) {
        hipLaunchKernelGGL((load8_kernel<tpr(), nv(), v(), to()>), dim3(row_grid(a.n, NT / tpr(), ROW_GRID)), dim3(NT), 0, st, a);
        return hipGetLastError();
      });
    });
  });
}

hipError_t launch_rms_norm(const RmsArgs& a, int type, int y_type, hipStream_t st) {
  const bool vec = vec_ok(a.x, type, a.cols) && vec_ok(a.res, type, a.cols) && vec_ok(a.total, type, a.cols) &&
                   vec_ok(a.y, y_type, a.cols);
  return by_cols(a.cols, [&](auto tpr, auto nv) {
    return by_flag(vec, [&](auto v) {
      return by_type(type, [&](auto ti) {
        const dim3 grid(row_grid(a.rows, NT / tpr(), ROW_GRID));
        if (y_type == MGN_E4M3)
          hipLaunchKernelGGL((rms_norm_kernel<tpr(), nv(), v(), ti(), MGN_E4M3>), grid, dim3(NT), 0, st, a);
        else if (y_type == MGN_BF16)
          hipLaunchKernelGGL((rms_norm_kernel<tpr(), nv(), v(), ti(), MGN_BF16>), grid, dim3(NT), 0, st, a);
        else
          hipLaunchKernelGGL((rms_norm_kernel<tpr(), nv(), v(), ti(), MGN_FP32>), grid, dim3(NT), 0, st, a);
        return hipGetLastError();
      });
    });
  });
}

hipError_t launch_rms_norm_grad(const RmsArgs& a, int type, float* dw, int accumulate, hipStream_t st) {
  const bool vec = vec_ok(a.x, type, a.cols) && vec_ok(a.res, type, a.cols) && vec_ok(a.total, type, a.cols) &&
                   vec_ok(a.dy, type, a.cols);
  int grid = 0;
  if (a.rows > 0) {
    const hipError_t e = by_cols(a.cols, [&](auto tpr, auto nv) {
      grid = row_grid(a.rows, NT / tpr(), MGN_RMS_WORK_PER_COL);
      return by_flag(vec, [&](auto v) {
        return by_type(type, [&](auto ti) {
          hipLaunchKernelGGL((rms_grad_kernel<tpr(), nv(), v(), ti()>), dim3(grid), dim3(NT), 0, st, a);
          return hipGetLastError();
        });
      });
    });
    if (e != hipSuccess) return e;
  }
  if (!dw) return hipSuccess;
  hipLaunchKernelGGL(rms_dw_kernel, dim3((a.cols + 15) / 16), dim3(NT), 0, st, a.part, grid, a.cols, accumulate, dw);
  return hipGetLastError();
}

}  // namespace mgn
