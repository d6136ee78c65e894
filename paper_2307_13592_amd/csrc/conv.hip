// Short causal convolution along time, each column with its own taps (gfx950):
//   v_t = b + sum_k w[W - 1 - k] x_{t-k},  y_t = v_t or v_t sigmoid(v_t),
// over the W - 1 steps before t that belong to its trajectory, and its backward
//   d_t = dy_t act'(v_t),  dx_t = sum_k w[W - 1 - k] d_{t+k},
//   dw[W - 1 - k] = sum d_t x_{t-k},  db = sum d_t.
//
// A lane holds V columns of a row and goes through time with the last
// W - 1 inputs in registers, STEPS steps' loads in flight together, so that each
// input is read once.  A workgroup takes as many rows as it has lanes for and, with
// many rows, all steps of them; with fewer the time axis is cut into segments,
// which read the W - 1 steps around them again (the neighbours', from the caches).
// The backward adds w d_t to the gradients of the W inputs that step t saw, and
// passes on the oldest: it needs each d once, and the pre-activation is formed
// again from the inputs that it holds.
//
// Bound by memory.  20 steps of 100,003 x 64 bf16, 4 taps, 91 us (5.6 TB/s); the
// backward of 600 steps of 1,885 x 128 fp32 348 us (5.0 TB/s), bf16 222 (3.9: two waves a
// SIMD keep too few bytes in flight).  8 columns a lane took 129 us of then 117.
#include <type_traits>

#include "raw.h"

namespace mgn {
namespace {

constexpr int NT = 256, MAX_W = MGN_CONV_MAX_WIDTH;

constexpr int V = 4;  // columns of a lane

// A thread's place: its columns, and its row among the `per` rows of a workgroup.  NEAR:
// the columns are neighbours, read at once; otherwise (rows of any width and alignment)
// they lie `lanes` apart, so that the wave's accesses are of neighbours still.
template <int TYPE, bool NEAR>
struct Place {
  int c, r, per, lanes, left;  // first column; left: columns of it on
  bool ok;
  __device__ __forceinline__ explicit Place(const ConvArgs& a) {
    lanes = a.lanes;
    per = NT / lanes;
    r = threadIdx.x / lanes;
    const int l = threadIdx.x % lanes;
    c = (int)blockIdx.y * lanes * V + l * (NEAR ? V : 1);
    ok = r < per && c < a.cols;
    left = ok ? a.cols - c : 0;
    if (!ok) c = 0;
  }
  // whether column k of the thread's is there
  __device__ __forceinline__ bool has(int k) const { return NEAR ? ok : k * lanes < left; }
  __device__ __forceinline__ int column(int k) const { return NEAR ? c + k : c + k * lanes; }
  __device__ __forceinline__ int64_t at(int k) const { return NEAR ? k : has(k) ? (int64_t)k * lanes : 0; }
  template <int T>
  __device__ __forceinline__ void load(const void* p, int64_t i, float (&v)[V]) const {
    const Elem<T>* const r = (const Elem<T>*)p + i;
    if constexpr (NEAR) {
      get<V>(r, v);
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) get<1>(r + at(k), v + k);
    }
  }
  template <int T>
  __device__ __forceinline__ void store(void* p, int64_t i, const float (&v)[V]) const {
    Elem<T>* const r = (Elem<T>*)p + i;
    if constexpr (!NEAR) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (has(k)) put<1>(r + at(k), v + k);
    } else if constexpr (T == MGN_BF16) {
      __builtin_nontemporal_store((uint64_t)pack_bf16(v[0], v[1]) | (uint64_t)pack_bf16(v[2], v[3]) << 32, (uint64_t*)r);
    } else {
      put<V>(r, v);
    }
  }
};

// Steps since the last start at or before step t, at most W: how far back step t
// + 1's predecessors go.  A lane looks at one step.
template <int W>
__device__ __forceinline__ int age_at(const uint8_t* starts, int64_t t) {
  if (!starts || t < 0) return W;
  const int lane = threadIdx.x & 63, k = lane < W && lane <= t ? lane : 0;
  const uint64_t m = __builtin_amdgcn_ballot_w64(starts[t - k] != 0 && k == lane);
  return m ? __builtin_ctzll(m) : W;
}

template <int W, class P>
__device__ __forceinline__ void load_taps(const ConvArgs& a, const P& p, float (&w)[W][V], float (&b)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int c = p.has(k) ? p.column(k) : 0;
    b[k] = a.b ? a.b[c] : 0.f;
    float all[W];
    get<(W % 4 == 0 ? W : 1)>(a.w + (int64_t)c * W, all);
    if constexpr (W % 4 != 0)
#pragma unroll
      for (int j = 1; j < W; ++j) all[j] = a.w[(int64_t)c * W + j];
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][k] = all[j];
  }
}

// The weighted inputs of the step whose own input is xs[W - 1]; of those before it
// the last `age` count, the others are left out whatever they are.
template <int W>
__device__ __forceinline__ void taps(const float (*xs)[V], const float (&w)[W][V], const float (&b)[V], int age, float (&v)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = b[k];
  if (age >= W - 1) {
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = fmaf(w[j][k], xs[j][k], v[k]);
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (W - 1 - j <= age)
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = fmaf(w[j][k], xs[j][k], v[k]);
  }
}

// A thread's columns of a step, as they lie in memory.
template <int TYPE, bool NEAR, bool PAST>
__device__ __forceinline__ void load_raw(const Place<TYPE, NEAR>& p, const void* x, int64_t i, Raw<TYPE, V, NEAR>& r) {
  const Elem<TYPE>* const q = (const Elem<TYPE>*)x + i;
  if constexpr (!NEAR) {
#pragma unroll
    for (int k = 0; k < V; ++k) __builtin_memcpy(&r.w[k], q + p.at(k), sizeof(*q));
  } else if constexpr (PAST) {
    r.stream((const char*)q);
  } else {
    r.load((const char*)q, 0);
  }
}

// What some steps bring; N arrays.  PAST: read past the caches.  Loaded a unit ahead of
// its use, without a branch between the loads or around them: where its ways meet, the
// compiler waits as for the one with the fewest loads.
template <int TYPE, int STEPS, int N, bool NEAR, bool PAST>
struct Inputs {
  Raw<TYPE, V, NEAR> v[N][STEPS];
  // steps t .. of those before `end` (the last of them again for those that are not)
  __device__ __forceinline__ void load(const Place<TYPE, NEAR>& p, const void* x, const void* y, int64_t t, int64_t end,
                                       int64_t C, int64_t i) {
#pragma unroll
    for (int e = 0; e < STEPS; ++e) {
      const int64_t s = t + e < end ? t + e : end - 1;
      load_raw<TYPE, NEAR, PAST>(p, x, s * C + i, v[0][e]);
      if constexpr (N > 1) load_raw<TYPE, NEAR, PAST>(p, y, s * C + i, v[1][e]);
    }
  }
};

// unit(in, t, all) for the units of steps t0 .. t1, each one's inputs (the first's are
// there) loaded while the one before it runs; all: it has all of its STEPS steps.
template <int STEPS, class In, class Load, class Unit>
__device__ __forceinline__ void in_units(int64_t t0, int64_t t1, In (&in)[2], Load load, Unit unit) {
  int64_t t = t0;
  while (t + STEPS < t1) {
    load(in[1], t + STEPS);
    unit(in[0], t, std::true_type());
    t += STEPS;
    if (t + STEPS >= t1) {
      in[0] = in[1];
      break;
    }
    load(in[0], t + STEPS);
    unit(in[1], t, std::true_type());
    t += STEPS;
  }
  unit(in[0], t, std::false_type());
}

// The window BY steps on: a unit's, or (its indexes have to be constants) one after
// each step of a unit that may have fewer.
template <int BY, int N>
__device__ __forceinline__ void forward(float (&v)[N][V]) {
#pragma unroll
  for (int j = 0; j + BY < N; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k) v[j][k] = v[j + BY][k];
}

// Inputs t0 - (W - 1) .. t0 - 1 of a row, oldest first.
template <int TYPE, int W, bool NEAR>
struct Before {
  Raw<TYPE, V, NEAR> v[W > 1 ? W - 1 : 1];
  __device__ __forceinline__ void load(const ConvArgs& a, const Place<TYPE, NEAR>& p, int64_t t0, int64_t C, int64_t i) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int64_t t = t0 - (W - 1) + j;
      const void* const from = t >= 0 || !a.past ? a.x : a.past;  // (without past anything that is there)
      load_raw<TYPE, NEAR, false>(p, from, (t >= 0 ? t : a.past ? t + W - 1 : 0) * C + i, v[j]);
    }
  }
  __device__ __forceinline__ void get(const ConvArgs& a, int64_t t0, bool ok, float (*xs)[V]) const {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      v[j].get(xs[j]);
#pragma unroll
      for (int k = 0; k < V; ++k) xs[j][k] = ok && (t0 - (W - 1) + j >= 0 || a.past) ? xs[j][k] : 0.f;
    }
  }
};

template <int TYPE, int W, int STEPS, bool NEAR, bool PAST>
__global__ __launch_bounds__(NT) void conv_kernel(ConvArgs a) {
  const Place<TYPE, NEAR> p(a);
  const int64_t C = a.rows * a.cols;
  float w[W][V], b[V];
  load_taps<W>(a, p, w, b);
  for (int64_t item = blockIdx.x; item < a.groups * a.segs; item += gridDim.x) {
    const int64_t s = item / a.groups, r = (item - s * a.groups) * p.per + p.r;
    const int64_t t0 = s * a.seg, t1 = s + 1 == a.segs ? a.steps : t0 + a.seg;
    const bool ok = p.ok && r < a.rows;
    const int64_t i = ok ? r * a.cols + p.c : 0;
    float xs[W - 1 + STEPS][V];
    Starts starts(a.starts, t0, t1);
    Before<TYPE, W, NEAR> before;
    Inputs<TYPE, STEPS, 1, NEAR, PAST> in[2];
    before.load(a, p, t0, C, i);
    in[0].load(p, a.x, nullptr, t0, t1, C, i);
    int age = age_at<W>(a.starts, t0 - 1);
    before.get(a, t0, ok, xs);
    const auto unit = [&](const Inputs<TYPE, STEPS, 1, NEAR, PAST>& now, int64_t t, auto all) __attribute__((always_inline)) {
      const int n = all() || t1 - t >= STEPS ? STEPS : (int)(t1 - t);
      const uint32_t fresh = starts.at<STEPS>(t);
#pragma unroll
      for (int e = 0; e < STEPS; ++e) now.v[0][e].get(xs[W - 1 + e]);
#pragma unroll
      for (int e = 0; e < STEPS; ++e) {
        if (e >= n) break;
        age = fresh >> e & 1 ? 0 : age < W ? age + 1 : W;
        float v[V];
        taps<W>(xs + (all() ? e : 0), w, b, age, v);
        if (a.silu) {
#pragma unroll
          for (int k = 0; k < V; ++k) v[k] *= sigmoid(v[k]);
        }
        if (ok) p.template store<TYPE>(a.y, (t + e) * C + i, v);
        if (!all()) forward<1>(xs);
      }
      if (all()) forward<STEPS>(xs);
    };
    in_units<STEPS>(t0, t1, in, [&](auto& to, int64_t t) { to.load(p, a.x, nullptr, t, t1, C, i); }, unit);
    if (a.past_out && ok && s + 1 == a.segs) {
      // what the next window's steps see: nothing from before the last start
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        float v[V];
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = W - 2 - j <= age ? xs[j][k] : 0.f;
        p.template store<TYPE>(a.past_out, j * C + i, v);
      }
    }
  }
}

// The backward; a.y is dx.  A thread's sums of dw and db go over all its items, in
// fp32 over SUM_STEPS steps and in fp64 over these.
constexpr int SUM_STEPS = 8;
template <int TYPE, int W, int STEPS, bool NEAR>
__global__ __launch_bounds__(NT) void conv_grad_kernel(ConvArgs a) {
  static_assert(SUM_STEPS % STEPS == 0);
  const Place<TYPE, NEAR> p(a);
  const int64_t C = a.rows * a.cols;
  float w[W][V], b[V], sw[W][V], sb[V];
  load_taps<W>(a, p, w, b);
  // [tap, or W for db][column][thread]: each thread adds to its own places only
  __shared__ double sums[W + 1][V][NT];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    sums[W][k][threadIdx.x] = 0, sb[k] = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) sums[j][k][threadIdx.x] = 0, sw[j][k] = 0.f;
  }
  const auto add = [&] {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      sums[W][k][threadIdx.x] += sb[k], sb[k] = 0.f;
#pragma unroll
      for (int j = 0; j < W; ++j) sums[j][k][threadIdx.x] += sw[j][k], sw[j][k] = 0.f;
    }
  };
  int turn = 0;
  for (int64_t item = blockIdx.x; item < a.groups * a.segs; item += gridDim.x) {
    const int64_t s = item / a.groups, r = (item - s * a.groups) * p.per + p.r;
    const int64_t t0 = s * a.seg, t1 = s + 1 == a.segs ? a.steps : t0 + a.seg;
    const int64_t te = s + 1 == a.segs ? t1 : t1 + (W - 1);  // the next segment's steps that saw this one's inputs
    const bool ok = p.ok && r < a.rows;
    const int64_t i = ok ? r * a.cols + p.c : 0;
    float xs[W - 1 + STEPS][V], g[W - 1 + STEPS][V];  // g[j]: gradient of the input of xs[j]
    Starts starts(a.starts, t0, te);
    Before<TYPE, W, NEAR> before;
    Inputs<TYPE, STEPS, 2, NEAR, false> in[2];
    before.load(a, p, t0, C, i);
    in[0].load(p, a.x, a.dy, t0, te, C, i);
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) g[j][k] = 0.f;
    int age = age_at<W>(a.starts, t0 - 1);
    before.get(a, t0, ok, xs);
    // the gradient of input t, complete
    const auto out = [&](int64_t t, const float (&v)[V]) {
      if (!ok || t >= t1) return;
      if (t >= t0) p.template store<TYPE>(a.y, t * C + i, v);
      else if (t < 0 && a.d_past) p.template store<MGN_FP32>(a.d_past, (t + W - 1) * C + i, v);
    };
    const auto unit = [&](const Inputs<TYPE, STEPS, 2, NEAR, false>& now, int64_t t, auto all) __attribute__((always_inline)) {
      const uint32_t fresh = starts.at<STEPS>(t);
      const int n = all() || te - t >= STEPS ? STEPS : (int)(te - t);
      float d[STEPS][V];
#pragma unroll
      for (int e = 0; e < STEPS; ++e) {
        now.v[0][e].get(xs[W - 1 + e]);
        now.v[1][e].get(d[e]);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          g[W - 1 + e][k] = 0.f;
          if (!ok) xs[W - 1 + e][k] = d[e][k] = 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < STEPS; ++e) {
        if (e >= n) break;
        const int at = all() ? e : 0;
        age = fresh >> e & 1 ? 0 : age < W ? age + 1 : W;
        if (a.silu) {
          float v[V];
          taps<W>(xs + at, w, b, age, v);
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const float f = sigmoid(v[k]);
            d[e][k] *= f * fmaf(v[k], 1.f - f, 1.f);
          }
        }
        const bool mine = t + e < t1;
#pragma unroll
        for (int j = 0; j < W; ++j)
          if (W - 1 - j <= age)
#pragma unroll
            for (int k = 0; k < V; ++k) {
              g[at + j][k] = fmaf(w[j][k], d[e][k], g[at + j][k]);
              if (mine) sw[j][k] = fmaf(d[e][k], xs[at + j][k], sw[j][k]);
            }
        if (mine)
#pragma unroll
          for (int k = 0; k < V; ++k) sb[k] += d[e][k];
        out(t + e - (W - 1), g[at]);
        if (!all()) forward<1>(xs), forward<1>(g);
      }
      if (++turn % (SUM_STEPS / STEPS) == 0) add();
      if (all()) forward<STEPS>(xs), forward<STEPS>(g);
    };
    in_units<STEPS>(t0, te, in, [&](auto& to, int64_t t) { to.load(p, a.x, a.dy, t, te, C, i); }, unit);
    if (s + 1 == a.segs) {
      // the inputs that steps after the last one see
#pragma unroll
      for (int j = 0; j < W - 1; ++j) {
        if (a.d_past_out && ok && W - 2 - j <= age) {
          float v[V];
          p.template load<MGN_FP32>(a.d_past_out, j * C + i, v);
#pragma unroll
          for (int k = 0; k < V; ++k) g[j][k] += v[k];
        }
        out(t1 - (W - 1) + j, g[j]);
      }
    }
  }
  if (!a.part) return;
  add();
  // the workgroup's rows, the upper half to the lower
  for (int n = p.per; n > 1;) {
    __syncthreads();
    const int half = (n + 1) / 2;
    if (p.r + half < n)
#pragma unroll
      for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) sums[j][k][threadIdx.x] += sums[j][k][threadIdx.x + half * p.lanes];
    n = half;
  }
  if (!p.ok || p.r != 0) return;
  float* const dst = a.part + blockIdx.x * ((int64_t)a.cols * (W + 1));
#pragma unroll
  for (int k = 0; k < V; ++k) {
    if (!p.has(k)) continue;
#pragma unroll
    for (int j = 0; j < W; ++j) dst[(int64_t)p.column(k) * W + j] = (float)sums[j][k][threadIdx.x];
    dst[(int64_t)a.cols * W + p.column(k)] = (float)sums[W][k][threadIdx.x];
  }
}

// past_out where no steps come: past, or zeros.
__global__ __launch_bounds__(NT) void past_copy_kernel(const uint8_t* in, uint8_t* out, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x; i < n; i += (int64_t)gridDim.x * NT) out[i] = in ? in[i] : 0;
}
hipError_t copy_bytes(const void* in, void* out, int64_t n, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  const int64_t b = (n + NT - 1) / NT;
  hipLaunchKernelGGL(past_copy_kernel, dim3((unsigned)(b < 8192 ? b : 8192)), dim3(NT), 0, st, (const uint8_t*)in, (uint8_t*)out, n);
  return hipGetLastError();
}
// past_out from the last W - 1 of `steps` inputs, where it lies on the array that
// the first segment reads.
template <int TYPE>
__global__ __launch_bounds__(NT) void past_tail_kernel(ConvArgs a, int W) {
  const int64_t C = a.rows * a.cols, n = (W - 1) * C;
  int age = MAX_W;
  if (a.starts)
    for (int k = W - 2; k >= 0; --k)
      if (a.starts[a.steps - 1 - k]) age = k;
  for (int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x; i < n; i += (int64_t)gridDim.x * NT) {
    const int64_t j = i / C;
    Elem<TYPE> v = 0;
    if (W - 2 - j <= age) v = ((const Elem<TYPE>*)a.x)[(a.steps - (W - 1)) * C + i];
    ((Elem<TYPE>*)a.past_out)[i] = v;
  }
}

constexpr int64_t FWD_WGS = 4096;   // workgroups that a forward launch wants
constexpr int64_t MOST_WGS = 1 << 20;
// A forward that moves more than the last-level cache holds reads past it: 20 steps of
// 100,003 x 64 bf16 94 us through it, 91 past it (the backward of 600 steps of 1,885 x
// 128 fp32 gained nothing).
constexpr int64_t CACHE = (int64_t)256 << 20;
constexpr int64_t LEAST_SEG = 8;    // steps of a segment (a short one reads its neighbours' steps again, but only where the card has room)

int64_t type_size(int type) { return type == MGN_FP32 ? 4 : 2; }
bool at(const void* p, int64_t bytes) { return (uintptr_t)p % bytes == 0; }

// How the rows and steps are dealt to about `want` workgroups.
void deal(ConvArgs& a, int64_t want) {
  const int per_row = (a.cols + V - 1) / V;
  a.tiles = (per_row + NT - 1) / NT;
  a.lanes = (per_row + a.tiles - 1) / a.tiles;
  const int per = NT / a.lanes;
  a.groups = (a.rows + per - 1) / per;
  const int64_t have = a.groups * a.tiles, most = a.steps / LEAST_SEG;
  a.segs = want / have;
  a.segs = a.segs < most ? a.segs : most;
  if (a.segs < 1) a.segs = 1;
  a.seg = (a.steps + a.segs - 1) / a.segs;
  a.segs = (a.steps + a.seg - 1) / a.seg;
  if (a.segs > 1 && a.steps - (a.segs - 1) * a.seg < MAX_W) --a.segs;  // the last one takes its few steps too
}

template <class F>
hipError_t by_width(int width, F f) {
  switch (width) {
    case 1: return f(Int<1>());
    case 2: return f(Int<2>());
    case 3: return f(Int<3>());
    case 4: return f(Int<4>());
    case 5: return f(Int<5>());
    case 6: return f(Int<6>());
    case 7: return f(Int<7>());
    case 8: return f(Int<8>());
  }
  return hipErrorInvalidValue;
}

}  // namespace

int64_t conv_work_floats(int cols, int width) { return (int64_t)MGN_CONV_PARTS * cols * (width + 1); }

hipError_t launch_conv(ConvArgs a, int type, int width, hipStream_t st) {
  const int64_t C = a.rows * a.cols;
  if (C <= 0) return hipSuccess;
  const int64_t past_bytes = (width - 1) * C * type_size(type);
  if (a.steps <= 0)
    return a.past_out && a.past_out != a.past ? copy_bytes(a.past, a.past_out, past_bytes, st) : hipSuccess;
  const int64_t edge = V * type_size(type);
  const bool near = a.cols % V == 0 && at(a.x, edge) && at(a.y, edge) && at(a.past, edge) && at(a.past_out, edge);
  deal(a, FWD_WGS);
  const bool past = 2 * a.steps * C * type_size(type) > CACHE;
  const bool tail = a.past_out && a.past_out == a.past && a.segs > 1;
  ConvArgs m = a;
  if (tail) m.past_out = nullptr;
  const int64_t items = a.groups * a.segs;
  const dim3 grid((unsigned)(items < MOST_WGS ? items : MOST_WGS), (unsigned)a.tiles);
  const hipError_t e = by_width(width, [&](auto w) {
    const auto go = [&](auto ty) {
      // (columns apart take four times the loads: 6 steps of 120,113 x 61 bf16, 6 taps, 121
      // us with 2 steps a unit, 153 with 4)
      constexpr int STEPS = 4;
      if (near && past) hipLaunchKernelGGL((conv_kernel<ty(), w(), STEPS, true, true>), grid, dim3(NT), 0, st, m);
      else if (near) hipLaunchKernelGGL((conv_kernel<ty(), w(), STEPS, true, false>), grid, dim3(NT), 0, st, m);
      else hipLaunchKernelGGL((conv_kernel<ty(), w(), 2, false, false>), grid, dim3(NT), 0, st, m);
    };
    if (type == MGN_BF16) go(Int<MGN_BF16>());
    else go(Int<MGN_FP32>());
    return hipGetLastError();
  });
  if (e != hipSuccess || !tail || width < 2) return e;
  const int64_t b = ((width - 1) * C + NT - 1) / NT;
  const dim3 tg((unsigned)(b < 8192 ? b : 8192));
  if (type == MGN_BF16) hipLaunchKernelGGL((past_tail_kernel<MGN_BF16>), tg, dim3(NT), 0, st, a, width);
  else hipLaunchKernelGGL((past_tail_kernel<MGN_FP32>), tg, dim3(NT), 0, st, a, width);
  return hipGetLastError();
}

hipError_t launch_conv_grad(ConvArgs a, int type, int width, float* dw, float* db, int accumulate, hipStream_t st) {
  const int64_t C = a.rows * a.cols;
  int64_t parts = 0;
  if (C > 0 && a.steps <= 0 && a.d_past)
    if (const hipError_t e = copy_bytes(a.d_past_out, a.d_past, (width - 1) * C * 4, st); e != hipSuccess) return e;
  if (C > 0 && a.steps > 0) {
    const int64_t edge = V * type_size(type);
    const bool near = a.cols % V == 0 && at(a.x, edge) && at(a.y, edge) && at(a.dy, edge) && at(a.past, edge) &&
                      at(a.d_past, 16) && at(a.d_past_out, 16);
    deal(a, MGN_CONV_PARTS);
    const int64_t items = a.groups * a.segs;
    parts = items < MGN_CONV_PARTS ? items : MGN_CONV_PARTS;
    const dim3 grid((unsigned)parts, (unsigned)a.tiles);
    const hipError_t e = by_width(width, [&](auto w) {
      const auto go = [&](auto ty) {
        // (fp32, 4 taps, with 2 steps: 600 steps of 1,885 x 128 387 us, 348 with 4; 20 of
        // 100,003 x 64 330 and 314.  bf16 is of two minds: 222 and 222, 214 and 206, but 100
        // of 20,003 x 64 172 and 200, and 2 taps 150 and 182.  More taps than 4 leave no
        // registers for 4 steps.)
        constexpr int STEPS = w() > 4 ? 2 : 4;
        if (near) hipLaunchKernelGGL((conv_grad_kernel<ty(), w(), STEPS, true>), grid, dim3(NT), 0, st, a);
        else hipLaunchKernelGGL((conv_grad_kernel<ty(), w(), 2, false>), grid, dim3(NT), 0, st, a);
      };
      if (type == MGN_BF16) go(Int<MGN_BF16>());
      else go(Int<MGN_FP32>());
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (!dw && !db) return hipSuccess;
  return launch_col_sums(ColSums{a.part, parts, (int64_t)a.cols * (width + 1), {dw, db, nullptr},
                                 {(int64_t)a.cols * width, a.cols}, accumulate}, st);
}

}  // namespace mgn
