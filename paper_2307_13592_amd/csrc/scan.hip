// Gated linear recurrence over the time steps of a trajectory (gfx950):
//   f = sigmoid(g), z = 1 - f = sigmoid(-g),  h_t = f_t h_{t-1} + z_t x_t,
// every column of every node row on its own, and its backward pass
//   D_t = dh_t + f_{t+1} D_{t+1},  dx = z D,  dg = f z (h_{t-1} - x) D.
#include "kernels.h"
#include "rows8.h"

namespace mgn {
namespace {

constexpr int NT = 256;

// f and z of a gate logit, both with a small relative error: e = exp(-|g|),
// 1 / (1 + e) and e / (1 + e).  A weight below the smallest normal number is 0,
// and a term with a weight of 0 is left out whatever it multiplies.
__device__ __forceinline__ void gates(float g, float& f, float& z) {
  const float e = __expf(-fabsf(g));
  const float big = __builtin_amdgcn_rcpf(1.f + e);
  float small = e * big;
  small = small < 1.17549435e-38f ? 0.f : small;
  f = g < 0.f ? small : big;
  z = g < 0.f ? big : small;
}

__device__ __forceinline__ float term(float weight, float v) { return weight == 0.f ? 0.f : weight * v; }

template <int TG>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
  if constexpr (TG == MGN_BF16) return bf2f(((const uint16_t*)p)[i]);
  else return ((const float*)p)[i];
}
template <int TG>
__device__ __forceinline__ void store1(void* p, int64_t i, float v) {
  if constexpr (TG == MGN_BF16) ((uint16_t*)p)[i] = f2bf(v);
  else ((float*)p)[i] = v;
}
template <int TX>
__device__ __forceinline__ float load_x(const ScanArgs& a, int64_t t, int64_t i, int64_t C) {
  if constexpr (TX == MGN_E4M3) {
    const int64_t row = i / a.cols;
    const int c = (int)(i - row * a.cols), nb = rows8_blocks(a.cols);
    float v[4];
    values8(((const uint8_t*)a.x)[t * C + i], a.x_scale[(t * a.rows + row) * nb + c / ROWS8_BLOCK], v);
    return v[0];
  } else {
    return load1<TX>(a.x, t * C + i);
  }
}

template <int TG, int TX>
__global__ __launch_bounds__(NT) void scan_kernel(ScanArgs a) {
  const int64_t C = a.rows * a.cols;
  for (int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x; i < C; i += (int64_t)gridDim.x * NT) {
    float h = a.h0 ? a.h0[i] : 0.f;
    for (int64_t t = 0; t < a.steps; ++t) {
      float f, z;
      gates(load1<TG>(a.g, t * C + i), f, z);
      if (a.starts && a.starts[t]) f = 0.f;
      h = term(f, h) + term(z, load_x<TX>(a, t, i, C));
      if (a.h) a.h[t * C + i] = h;
    }
    if (a.h_last) a.h_last[i] = h;
  }
}

template <int TG, int TX>
__global__ __launch_bounds__(NT) void scan_grad_kernel(ScanArgs a) {
  constexpr int TD = TX == MGN_E4M3 ? TG : TX;
  const int64_t C = a.rows * a.cols;
  for (int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x; i < C; i += (int64_t)gridDim.x * NT) {
    float D = a.dh_last ? a.dh_last[i] : 0.f;
    for (int64_t t = a.steps - 1; t >= 0; --t) {
      float f, z;
      gates(load1<TG>(a.g, t * C + i), f, z);
      const bool fresh = a.starts && a.starts[t];
      const float prev = fresh ? 0.f : t > 0 ? a.h[(t - 1) * C + i] : a.h0 ? a.h0[i] : 0.f;
      if (a.dh) D += a.dh[t * C + i];
      store1<TD>(a.dx, t * C + i, term(z, D));
      store1<TG>(a.dg, t * C + i, term(f * z, (prev - load_x<TX>(a, t, i, C)) * D));
      D = fresh ? 0.f : term(f, D);
    }
    if (a.dh0) a.dh0[i] = D;
  }
}

template <class F>
hipError_t by_types(int g, int x, F f) {
  using std::integral_constant;
  if (g == MGN_BF16) {
    if (x == MGN_E4M3) return f(integral_constant<int, MGN_BF16>(), integral_constant<int, MGN_E4M3>());
    return f(integral_constant<int, MGN_BF16>(), integral_constant<int, MGN_BF16>());
  }
  if (x == MGN_E4M3) return f(integral_constant<int, MGN_FP32>(), integral_constant<int, MGN_E4M3>());
  return f(integral_constant<int, MGN_FP32>(), integral_constant<int, MGN_FP32>());
}

}  // namespace

size_t scan_work_bytes(int64_t, int64_t, int) { return 0; }

hipError_t launch_scan(const ScanArgs& a, int g_type, int x_type, hipStream_t st) {
  const int64_t b = (a.rows * a.cols + NT - 1) / NT;
  return by_types(g_type, x_type, [&](auto tg, auto tx) {
    hipLaunchKernelGGL((scan_kernel<tg(), tx()>), dim3((unsigned)(b < 65536 ? b : 65536)), dim3(NT), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_scan_grad(const ScanArgs& a, int g_type, int x_type, hipStream_t st) {
  const int64_t b = (a.rows * a.cols + NT - 1) / NT;
  return by_types(g_type, x_type, [&](auto tg, auto tx) {
    hipLaunchKernelGGL((scan_grad_kernel<tg(), tx()>), dim3((unsigned)(b < 65536 ? b : 65536)), dim3(NT), 0, st, a);
    return hipGetLastError();
  });
}

}  // namespace mgn
