// The global norm of many tensors, and their scaling to a largest one (gfx950):
//   norm = sqrt(sum over all tensors of g^2),  out = g min(1, max_norm / norm).
//
// The tensors are cut into tiles of GRAD_TILE elements and consecutive tiles dealt to
// the workgroups, so that many small tensors and few large ones fill the card alike; a
// workgroup looks its first tile's tensor up and goes on from there.  The tables come
// with the kernel arguments, which a HIP graph records.  Squares are formed and added
// in fp64 (two fp64 instructions an element, less than its load takes): neither
// gradients of 1e-25 nor of 1e25 leave the range, and the order of the sums does not
// show in the fp32 norm.  Every workgroup leaves one partial; a scaling workgroup adds
// all of them itself, in a fixed order, rather than have one more launch do it, and
// goes through its tiles from the last on, which are the likeliest to be in the caches.
//
// Bound by HBM (two reads and a write), by launches for few elements.
#include "kernels.h"
#include "rows8.h"

namespace mgn {
namespace {

constexpr int NT = 256;
constexpr int RUN = 16, AT_ONCE = 4;   // bytes of a thread's access, and accesses in flight together (norm)
constexpr int64_t WGS = 1536;           // workgroups of a norm launch with one table
constexpr int64_t WGS_MANY = 256;       // with several
// Partials, and tiles, above which a launch of its own adds the partials and a scaling
// workgroup takes one tile: 480M bf16 values in 24 tensors 507 us (515 when 16,384
// workgroups that take several in turn and add the partials themselves took 537, and
// 4,096 572).  A model's 190 tensors (1.8M values) 12 us without that launch.
constexpr int64_t FOLD = 4096, FOLD_TILES = 16384, CLIP_WGS = 1 << 22;

// The tensor that holds a tile: how many of the tensors begin at or before it, each
// lane counting for its own ones.
struct Lookup {
  uint32_t first[(GRAD_TABLE + 63) / 64];
  __device__ __forceinline__ explicit Lookup(const GradTable& t) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < GRAD_TABLE; k += 64) first[k / 64] = k + lane < t.count ? t.first[k + lane] : ~0u;
  }
  __device__ __forceinline__ int operator()(uint32_t tile) const {
    int n = 0;
#pragma unroll
    for (int k = 0; k < GRAD_TABLE; k += 64) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(first[k / 64] <= tile));
    return n - 1;
  }
};

static_assert(sizeof(GradTable) + 64 <= 4096);

// The workgroup's tiles.
struct Tiles {
  uint32_t begin, end;
  __device__ __forceinline__ explicit Tiles(const GradTable& t) {
    const uint64_t all = t.first[t.count];
    begin = (uint32_t)(all * blockIdx.x / gridDim.x), end = (uint32_t)(all * (blockIdx.x + 1) / gridDim.x);
  }
};

// f(first element, count, number of runs) over the elements [at, end) of a tensor, each
// thread for its own runs of `count`, `ONCE` of them NT runs apart or one.
template <class E, int ONCE, class F>
__device__ __forceinline__ void over(int64_t at, int64_t end, F f) {
  constexpr int V = RUN / sizeof(E);
  constexpr int64_t STEP = NT * V;
  int64_t i = at + threadIdx.x * V;
  for (; at + STEP * ONCE <= end; at += STEP * ONCE, i += STEP * ONCE)
    f(i, std::integral_constant<int, V>(), std::integral_constant<int, ONCE>());
  for (; i + V <= end; i += STEP) f(i, std::integral_constant<int, V>(), std::integral_constant<int, 1>());
  for (int k = 0; k < V; ++k)
    if (i + k < end) f(i + k, std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
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

__global__ __launch_bounds__(NT) void grad_squares_kernel(GradTable t, double* part) {
  __shared__ double lds[NT / 64];
  double s[4] = {0, 0, 0, 0};
  const Tiles w(t);
  if (w.begin < w.end) {
    uint32_t tile = w.begin;
    for (int k = Lookup(t)(tile); tile < w.end; ++k) {
      const uint32_t stop = t.first[k + 1] < w.end ? t.first[k + 1] : w.end;
      const int64_t n = t.n(k), at = (int64_t)(tile - t.first[k]) * GRAD_TILE, to = (int64_t)(stop - t.first[k]) * GRAD_TILE;
      const auto add = [&](auto* p) {
        using E = std::remove_const_t<std::remove_pointer_t<decltype(p)>>;
        over<E, AT_ONCE>(at, to < n ? to : n, [&](int64_t i, auto count, auto runs) {
          float v[runs()][count()];
#pragma unroll
          for (int r = 0; r < runs(); ++r) get<count()>(p + i + r * (int64_t)NT * count(), v[r]);
#pragma unroll
          for (int r = 0; r < runs(); ++r)
#pragma unroll
            for (int e = 0; e < count(); ++e) s[e % 4] = fma((double)v[r][e], (double)v[r][e], s[e % 4]);
        });
      };
      if (t.is_bf16(k)) add((const uint16_t*)t.g(k));
      else add((const float*)t.g(k));
      tile = stop;
    }
  }
  const double all = group_total((s[0] + s[1]) + (s[2] + s[3]), lds);
  if (threadIdx.x == 0) part[blockIdx.x] = all;
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

// out = g scale rest.  A norm that is not a number, or infinite in fp32 as it is stored,
// scales nothing.  The quotient goes in one fp32 number, or, below the normal ones (which
// would leave it few digits or none), 2^126 times it and the exact rest.
__global__ __launch_bounds__(NT) void grad_clip_kernel(GradTable t, const double* part, int64_t parts, float max_norm,
                                                       bool given, bool write, float* norm) {
  __shared__ double lds[NT / 64];
  const float n = given ? *norm : (float)sqrt(all_squares(part, parts, lds));
  if (write && blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
  float scale = n > max_norm && n < INFINITY ? max_norm / n : 1.f, rest = 1.f;
  if (scale < 0x1p-126f) scale = (float)((double)max_norm / (double)n * 0x1p126), rest = 0x1p-126f;
  const Lookup tensor(t);
  const uint32_t tiles = t.first[t.count];
  for (uint32_t b = blockIdx.x; b < tiles; b += gridDim.x) {
    const uint32_t tile = tiles - 1 - b;
    const int k = tensor(tile);
    if (scale == 1.f && rest == 1.f && t.out(k) == t.g(k)) continue;
    const int64_t n = t.n(k), at = (int64_t)(tile - t.first[k]) * GRAD_TILE, to = at + GRAD_TILE;
    const auto scaled = [&](auto* p) {
      using E = std::remove_const_t<std::remove_pointer_t<decltype(p)>>;
      E* const out = (E*)t.out(k);
      over<E, GRAD_TILE / (NT * RUN / (int)sizeof(E))>(at, to < n ? to : n, [&](int64_t i, auto count, auto runs) {
        float v[runs()][count()];
#pragma unroll
        for (int r = 0; r < runs(); ++r) get<count()>(p + i + r * (int64_t)NT * count(), v[r]);
#pragma unroll
        for (int r = 0; r < runs(); ++r) {
#pragma unroll
          for (int e = 0; e < count(); ++e) v[r][e] = v[r][e] * scale * rest;
          put<count()>(out + i + r * (int64_t)NT * count(), v[r]);
        }
      });
    };
    if (t.is_bf16(k)) scaled((const uint16_t*)t.g(k));
    else scaled((const float*)t.g(k));
  }
}

int64_t workgroups(const GradTable& t, int64_t tables) {
  const int64_t most = tables > 1 ? WGS_MANY : WGS, tiles = t.first[t.count];
  return tiles < most ? tiles : most;
}

}  // namespace

int64_t grad_work_doubles(int64_t n) { return n > 1 ? n * WGS_MANY : WGS; }

hipError_t launch_grads(const GradTable* t, int64_t n, float max_norm, bool given, float* norm, double* work,
                        hipStream_t st) {
  hipError_t e = hipSuccess;
  int64_t parts = 0, tiles = 0;
  bool write = !given;
  for (int64_t k = 0; k < n; ++k) tiles += t[k].first[t[k].count];
  if (!given) {
    for (int64_t k = 0; k < n; ++k) {
      const int64_t wgs = workgroups(t[k], n);
      if (wgs == 0) continue;
      hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)wgs), dim3(NT), 0, st, t[k], work + parts);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      parts += wgs;
    }
    if (max_norm < 0 || parts > FOLD || tiles > FOLD_TILES || parts == 0) {
      hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(NT), 0, st, work, parts, max_norm < 0 || parts == 0 ? norm : nullptr);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      if (parts > 1) parts = 1;
    }
  }
  if (max_norm < 0) return hipSuccess;
  for (int64_t k = 0; k < n; ++k) {
    const int64_t own = t[k].first[t[k].count];
    if (own == 0) continue;
    hipLaunchKernelGGL(grad_clip_kernel, dim3((unsigned)(own < CLIP_WGS ? own : CLIP_WGS)), dim3(NT), 0, st, t[k], work, parts, max_norm, given, write,
                       norm);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    write = false;  // once
  }
  return hipSuccess;
}

}  // namespace mgn
