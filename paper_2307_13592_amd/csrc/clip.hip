// The global norm of many tensors, and their scaling to a largest one (gfx950):
//   norm = sqrt(sum over all tensors of g^2),  out = g min(1, max_norm / norm).
//
// The tensors are cut into tiles of GRAD_TILE elements and the tiles dealt in
// turn to the workgroups, so that many small tensors and few large ones fill the
// card alike; the tables come with the kernel arguments, which a HIP graph records.
// Squares are formed and added in fp64 (two fp64 instructions an element, less than
// its load takes): neither gradients of 1e-25 nor of 1e25 leave the range, and the
// order of the sums does not show in the fp32 norm.  Every workgroup leaves one
// partial; a scaling workgroup adds all of them itself, in a fixed order, rather than
// have one more launch do it.
//
// Bound by HBM (two reads and a write), by launches for few elements.
#include "kernels.h"
#include "rows8.h"

namespace mgn {
namespace {

constexpr int NT = 256;
constexpr int RUN = 16;                    // bytes of a thread's access
constexpr int64_t NORM_WGS = 1024;         // workgroups of a norm launch with one table
constexpr int64_t NORM_WGS_MANY = 256;     // with several
constexpr int64_t FOLD = 4096;             // partials above which a launch of their own adds them
constexpr int64_t CLIP_WGS = 4096;

// The tensor that holds a tile: how many of the tensors begin at or before it, each
// lane counting for its own ones.
__device__ __forceinline__ int tensor_of(const GradTable& t, uint32_t tile) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int k = 0; k < GRAD_TABLE; k += 64)
    n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k + lane < t.count && t.first[k + lane] <= tile));
  return n - 1;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}
// Sum over the workgroup, in a fixed order; every thread gets the same bits.
__device__ __forceinline__ double group_total(double v, double* lds) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int e = 1; e < NT / 64; ++e) v += lds[e];
  return v;
}

// f(elements [at, at + count) of the tile's tensor, E, count <= run) over a
// thread's part of a tile.
template <class E, class F>
__device__ __forceinline__ void over_tile(int64_t n, int64_t begin, F f) {
  constexpr int V = RUN / sizeof(E);
  const int64_t left = n - begin;
  if (left >= GRAD_TILE) {
#pragma unroll 8
    for (int64_t i = threadIdx.x * V; i < GRAD_TILE; i += NT * V) f(begin + i, std::integral_constant<int, V>());
  } else {
    int64_t i = threadIdx.x * V;
    for (; i + V <= left; i += NT * V) f(begin + i, std::integral_constant<int, V>());
    for (int k = 0; k < V; ++k)
      if (i + k < left) f(begin + i + k, std::integral_constant<int, 1>());
  }
}

__global__ __launch_bounds__(NT) void grad_squares_kernel(GradTable t, double* part) {
  __shared__ double lds[NT / 64];
  double s = 0;
  for (uint32_t tile = blockIdx.x; tile < t.first[t.count]; tile += gridDim.x) {
    const int k = tensor_of(t, tile);
    const int64_t begin = (int64_t)(tile - t.first[k]) * GRAD_TILE;
    const auto add = [&](auto* p) {
      over_tile<std::remove_const_t<std::remove_pointer_t<decltype(p)>>>(t.n[k], begin, [&](int64_t i, auto count) {
        float v[count()];
        get<count()>(p + i, v);
#pragma unroll
        for (int e = 0; e < count(); ++e) s = fma((double)v[e], (double)v[e], s);
      });
    };
    if (t.bf16[k / 32] >> (k % 32) & 1) add((const uint16_t*)t.g[k]);
    else add((const float*)t.g[k]);
  }
  s = group_total(s, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm from the partials; in place of them their sum (fold), or the fp32 norm.
__device__ __forceinline__ double all_squares(const double* part, int64_t parts, double* lds) {
  double s = 0;
  for (int64_t i = threadIdx.x; i < parts; i += NT) s += part[i];
  return group_total(s, lds);
}
__global__ __launch_bounds__(NT) void grad_norm_kernel(double* part, int64_t parts, float* norm) {
  __shared__ double lds[NT / 64];
  const double s = all_squares(part, parts, lds);
  if (threadIdx.x != 0) return;
  if (norm) *norm = (float)sqrt(s);
  else part[0] = s;
}

// out = g scale.  A norm that is not a number, or infinite, scales nothing.
__global__ __launch_bounds__(NT) void grad_clip_kernel(GradTable t, const double* part, int64_t parts, float max_norm,
                                                       bool given, bool write, float* norm) {
  __shared__ double lds[NT / 64];
  const float n = given ? *norm : (float)sqrt(all_squares(part, parts, lds));
  if (write && blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
  const float scale = n > max_norm && n < INFINITY ? max_norm / n : 1.f;
  const uint32_t tiles = t.first[t.count];
  for (uint32_t b = blockIdx.x; b < tiles; b += gridDim.x) {
    // from the last tile on: those are the likeliest to be in the caches still
    const uint32_t tile = tiles - 1 - b;
    const int k = tensor_of(t, tile);
    if (scale == 1.f && t.out[k] == t.g[k]) continue;
    const int64_t begin = (int64_t)(tile - t.first[k]) * GRAD_TILE;
    const auto scaled = [&](auto* p) {
      using E = std::remove_const_t<std::remove_pointer_t<decltype(p)>>;
      over_tile<E>(t.n[k], begin, [&](int64_t i, auto count) {
        float v[count()];
        get<count()>(p + i, v);
#pragma unroll
        for (int e = 0; e < count(); ++e) v[e] *= scale;
        put<count()>((E*)t.out[k] + i, v);
      });
    };
    if (t.bf16[k / 32] >> (k % 32) & 1) scaled((const uint16_t*)t.g[k]);
    else scaled((const float*)t.g[k]);
  }
}

int64_t norm_wgs(const GradTable& t, int64_t tables) {
  const int64_t most = tables > 1 ? NORM_WGS_MANY : NORM_WGS, tiles = t.first[t.count];
  return tiles < most ? tiles : most;
}

}  // namespace

int64_t grad_work_doubles(int64_t n) { return n > 1 ? n * NORM_WGS_MANY : NORM_WGS; }

hipError_t launch_grads(const GradTable* t, int64_t n, float max_norm, bool given, float* norm, double* work,
                        hipStream_t st) {
  hipError_t e = hipSuccess;
  int64_t parts = 0;
  bool write = !given;
  if (!given) {
    for (int64_t k = 0; k < n; ++k) {
      const int64_t wgs = norm_wgs(t[k], n);
      if (wgs == 0) continue;
      hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)wgs), dim3(NT), 0, st, t[k], work + parts);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      parts += wgs;
    }
    if (max_norm < 0 || parts > FOLD || parts == 0) {
      hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(NT), 0, st, work, parts, max_norm < 0 || parts == 0 ? norm : nullptr);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      if (parts > 1) parts = 1;
    }
  }
  if (max_norm < 0) return hipSuccess;
  for (int64_t k = 0; k < n; ++k) {
    const int64_t tiles = t[k].first[t[k].count];
    if (tiles == 0) continue;
    hipLaunchKernelGGL(grad_clip_kernel, dim3((unsigned)(tiles < CLIP_WGS ? tiles : CLIP_WGS)), dim3(NT), 0, st, t[k], work,
                       parts, max_norm, given, write, norm);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    write = false;  // once
  }
  return hipSuccess;
}

}  // namespace mgn
