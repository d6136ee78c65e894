// Backward of the selective scan (gfx950).  With G_t the gradient of the state h_t,
//   G_t = C_t o_t + exp(delta_{t+1} A) G_{t+1}   (o = dy z sigmoid(z); 0 past a start),
//   dC_t = sum over columns o_t h_t,  dB_t = sum over columns G_t delta x,
//   w = G_t exp(delta A) h_{t-1},  dA += w delta,
//   d(delta) = sum_k w A + x sum_k G B,  dx = delta sum_k G B + D o,  dD += o x.
//
// The states are formed again from the marks that the forward left every
// MGN_MARK_STEPS steps: a wave goes forward through a block of that many steps with
// all its states in registers, then back through it with G.  The lanes are dealt as
// in the forward (ssm.h); dB and dC, which are sums over columns, are added over a
// lane's four columns first and then over the wave's groups by exchanges that halve
// the numbers with each level.  Rows of more than 64 columns (GP groups) are several
// tiles, whose sums a second launch adds.  More than 16 states are dealt to NW waves
// of a workgroup, which add what they have of dx and d(delta) in LDS.  A workgroup
// goes through its rows in turn, so that dA, dD and d_bias, long sums over steps and
// rows, leave one partial each of it; a block's products are added in fp32, the blocks
// in fp64.  With few columns the time axis is cut into chunks as in the forward.
//
// Bound by the vector units: 13 instructions and two exponentials a state and step.
#include "ssm.h"

namespace mgn {
namespace {

constexpr int K = MGN_MARK_STEPS;

// v of the lane D = 4 or 8 away.
template <int D>
__device__ __forceinline__ float across(float v) {
  if constexpr (D == 4) {
    // the mirror image in 8 lanes, mirrored again in 4
    const int m = __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true);
    return __int_as_float(__builtin_amdgcn_update_dpp(0, m, 0x1b, 0xf, 0xf, true));
  } else if constexpr (D == 8) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, true));  // rotated by 8 of 16
  } else {
    return __shfl_xor(v, D);
  }
}

// Sums of v[0 .. M - 1] over the wave's groups (lanes 4, 8, .. 2 LG apart): a level
// leaves each of two partners the sums of one half of the numbers, and a single
// number goes to both.  Lane l ends with numbers `first` .. of which there are
// M >> LG or one, and is the one to write them if `keeps`.
template <int M, int LG>
struct GroupSums {
  static constexpr int LEFT = (M >> LG) > 0 ? M >> LG : 1;
  int first;
  bool keeps;
  template <int N, int D>
  __device__ __forceinline__ void level(float (&v)[M]) {
    const bool hi = threadIdx.x & D;
    if constexpr (N > 1) {
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        if constexpr (D == 32) {
          const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[k]), __float_as_uint(v[k + N / 2]), false, false);
          v[k] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        } else if constexpr (D == 16) {
          const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[k]), __float_as_uint(v[k + N / 2]), false, false);
          v[k] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        } else {
          const float mine = hi ? v[k + N / 2] : v[k], other = hi ? v[k] : v[k + N / 2];
          v[k] = mine + across<D>(other);
        }
      }
      first += hi ? N / 2 : 0;
    } else {
      v[0] += across<D>(v[0]);
      keeps = keeps && !hi;
    }
    if constexpr (D > 4) level<(N > 1 ? N / 2 : 1), D / 2>(v);
  }
  __device__ __forceinline__ void operator()(float (&v)[M]) {
    first = 0;
    keeps = true;
    if constexpr (LG > 0) level<M, 2 << LG>(v);
  }
};

// G that leaves each chunk (through its first step), from zeros at its end, and
// its sum of delta; chunk blockIdx.y + 1.
template <int TYPE, int NL, bool FULL, bool GATE>
__global__ __launch_bounds__(256) void ssm_carry_kernel(SsmArgs a) {
  constexpr int STEPS = NL <= 4 ? 4 : NL == 8 ? 2 : 1;
  const int per_row = (a.cols + 3) / 4, q = threadIdx.x & 3;
  const int64_t gi = ((int64_t)blockIdx.x * 256 + threadIdx.x) / 4, row = gi / per_row;
  const int g = (int)(gi - row * per_row) * 4, col = g + q, s = q * NL;
  const bool in = row < a.rows, ok = in && col < a.cols;
  const int c = blockIdx.y + 1;
  const int64_t ts = c * a.chunk, te = ts + a.chunk < a.steps ? ts + a.chunk : a.steps;
  const int64_t C = a.rows * a.cols, i = row * a.cols + col, bn = row * a.n, at = (row * a.cols + g) * a.n;
  float G[4][NL], A[4][NL];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int k = 0; k < NL; ++k) G[j][k] = A[j][k] = 0.f;
    if (in && g + j < a.cols) load_n<MGN_FP32, NL, FULL>(a.A, (int64_t)(g + j) * a.n, s, a.n, A[j]);
#pragma unroll
    for (int k = 0; k < NL; ++k) A[j][k] *= LOG2E;
  }
  const float bias = a.bias && ok ? a.bias[col] : 0.f;
  float sum = 0.f;
  for (int64_t t = te - 1; t >= ts; t -= STEPS) {
    float dt[STEPS], o[STEPS], z[STEPS], Cn[STEPS][NL];
    bool fresh[STEPS];
#pragma unroll
    for (int e = 0; e < STEPS; ++e) {
      dt[e] = o[e] = z[e] = 0.f;
      fresh[e] = false;
#pragma unroll
      for (int k = 0; k < NL; ++k) Cn[e][k] = 0.f;
      if (t - e < ts) continue;
      if (a.starts) fresh[e] = a.starts[t - e];
      if (ok) {
        dt[e] = load1<TYPE>(a.dt, (t - e) * C + i);
        o[e] = load1<TYPE>(a.dy, (t - e) * C + i);
        if (GATE) z[e] = load1<TYPE>(a.z, (t - e) * C + i);
      }
      if (in) load_n<TYPE, NL, FULL>(a.C, (t - e) * a.rows * a.n + bn, s, a.n, Cn[e]);
    }
#pragma unroll
    for (int e = 0; e < STEPS; ++e) {
      if (t - e < ts) break;
      float delta = dt[e] + bias;
      if (a.softplus) delta = softplus(delta);
      delta = ok ? delta : 0.f;
      sum += delta;
      if (GATE) o[e] *= z[e] * sigmoid(z[e]);
      float d[4], ov[4];
      quads(delta, d);
      quads(o[e], ov);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < NL; ++k)
          G[j][k] = fmaf(Cn[e][k], ov[j], G[j][k]) * __builtin_amdgcn_exp2f(d[j] * A[j][k]);
      if (fresh[e]) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int k = 0; k < NL; ++k) G[j][k] = 0.f;
        sum = CUT;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (in && g + j < a.cols) store_n<NL, FULL>(a.state + c * C * a.n, at + j * a.n, s, a.n, G[j]);
  if (ok) a.sums[c * C + i] = sum;
}

template <int TYPE, int NL, int NW, int LG, bool FULL, bool GATE>
__global__ __launch_bounds__(64 * NW) void ssm_grad_kernel(SsmArgs a) {
  constexpr int GP = 1 << LG, RPW = 16 / GP;
  __shared__ double accs[4 * NL][64 * NW];
  __shared__ float red[NW > 1 ? 2 : 1][NW > 1 ? NW : 1][NW > 1 ? K : 1][3][64];
  const int lane = threadIdx.x & 63, w = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane & 3;
  const int tile = blockIdx.x % a.tiles, sub = (lane >> 2) >> LG;
  const int64_t slot = blockIdx.x / a.tiles;
  const int g = (tile * GP + ((lane >> 2) & (GP - 1))) * 4, col = g + q, s0 = (w * 4 + q) * NL;
  const int c = blockIdx.y;
  const int64_t ts = c * a.chunk, te = ts + a.chunk < a.steps ? ts + a.chunk : a.steps;
  const int64_t C = a.rows * a.cols;

  float A[4][NL];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int k = 0; k < NL; ++k) A[j][k] = 0.f, accs[j * NL + k][threadIdx.x] = 0;
    if (g + j < a.cols) load_n<MGN_FP32, NL, FULL>(a.A, (int64_t)(g + j) * a.n, s0, a.n, A[j]);
#pragma unroll
    for (int k = 0; k < NL; ++k) A[j][k] *= LOG2E;
  }
  const float bias = a.bias && col < a.cols ? a.bias[col] : 0.f, D = a.D && col < a.cols ? a.D[col] : 0.f;
  double dD = 0, d_bias = 0;
  int par = 0;

  for (int64_t r0 = slot * RPW; r0 < a.rows; r0 += a.slots * RPW) {
    const int64_t row = r0 + sub, i = row * a.cols + col, bn = row * a.n, at = (row * a.cols + g) * a.n;
    const bool in = row < a.rows && g < a.cols, ok = in && col < a.cols;
    float G[4][NL];
    const float* const from = a.chunks > 1 ? a.state + c * C * a.n : a.dh_last;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int k = 0; k < NL; ++k) G[j][k] = 0.f;
      if (from && in && g + j < a.cols) load_n<MGN_FP32, NL, FULL>(from, at + j * a.n, s0, a.n, G[j]);
    }
    for (int64_t t0 = (te - 1) / K * K; t0 >= ts; t0 -= K) {
      const int n = te - t0 < K ? (int)(te - t0) : K;
      float x[K], v[K], delta[K], dy[K], z[K], h[K + 1][4][NL];
      bool fresh[K];
#pragma unroll
      for (int e = 0; e < K; ++e) {
        x[e] = v[e] = delta[e] = dy[e] = z[e] = 0.f;
        fresh[e] = false;
        if (e >= n) continue;
        if (a.starts) fresh[e] = a.starts[t0 + e];
        if (ok) {
          x[e] = load1<TYPE>(a.x, (t0 + e) * C + i);
          v[e] = load1<TYPE>(a.dt, (t0 + e) * C + i) + bias;
          dy[e] = load1<TYPE>(a.dy, (t0 + e) * C + i);
          if (GATE) z[e] = load1<TYPE>(a.z, (t0 + e) * C + i);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int k = 0; k < NL; ++k) h[0][j][k] = 0.f;
        if (in && g + j < a.cols) load_n<MGN_FP32, NL, FULL>(a.marks + t0 / K * C * a.n, at + j * a.n, s0, a.n, h[0][j]);
      }
      // the block's states
#pragma unroll
      for (int e = 0; e < K; ++e) {
        if (e >= n) break;
        float B[NL];
#pragma unroll
        for (int k = 0; k < NL; ++k) B[k] = 0.f;
        if (in) load_n<TYPE, NL, FULL>(a.B, (t0 + e) * a.rows * a.n + bn, s0, a.n, B);
        delta[e] = ok ? a.softplus ? softplus(v[e]) : v[e] : 0.f;
        float d[4], u[4];
        quads(delta[e], d);
        quads(mul_or_0(delta[e], x[e]), u);
        // B may hold anything where a column's step has size 0
        const auto step = [&](auto first, auto held) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < NL; ++k) {
              const float b = held() ? mul_or_0(u[j], B[k]) : u[j] * B[k];
              h[e + 1][j][k] = first() ? b : fmaf(__builtin_amdgcn_exp2f(d[j] * A[j][k]), h[e][j][k], b);
            }
        };
        if (fresh[e]) step(std::true_type(), std::true_type());
        else if (any(ok && delta[e] == 0.f)) step(std::false_type(), std::true_type());
        else step(std::false_type(), std::false_type());
      }
      // and back
      float dA[4][NL], sD = 0.f, sb = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < NL; ++k) dA[j][k] = 0.f;
      // the gradients of one column and step, from the sums over all its states
      const auto finish = [&](int e, float sB, float sA, float y) {
        const float sg = GATE ? sigmoid(z[e]) : 0.f, o = GATE ? dy[e] * (z[e] * sg) : dy[e];
        float dx = mul_or_0(delta[e], sB), dd = fmaf(sA, LN2, sB * x[e]);
        if (a.D) dx = fmaf(D, o, dx), sD = fmaf(o, x[e], sD);
        if (a.softplus) dd = mul_or_0(sigmoid(v[e]), dd);
        sb += dd;
        if (!ok) return;
        store1<TYPE>(a.dx, (t0 + e) * C + i, dx);
        store1<TYPE>(a.ddt, (t0 + e) * C + i, dd);
        if (GATE) {
          if (a.D) y = fmaf(D, x[e], y);
          store1<TYPE>(a.dz, (t0 + e) * C + i, dy[e] * y * (sg * fmaf(z[e], 1.f - sg, 1.f)));
        }
      };
#pragma unroll
      for (int e = K - 1; e >= 0; --e) {
        if (e >= n) continue;
        float B[NL], Cn[NL];
#pragma unroll
        for (int k = 0; k < NL; ++k) B[k] = Cn[k] = 0.f;
        if (in) {
          load_n<TYPE, NL, FULL>(a.B, (t0 + e) * a.rows * a.n + bn, s0, a.n, B);
          load_n<TYPE, NL, FULL>(a.C, (t0 + e) * a.rows * a.n + bn, s0, a.n, Cn);
        }
        float d[4], u[4], o[4], sB[4], sA[4], y[4], p[2 * NL];
        quads(delta[e], d);
        quads(mul_or_0(delta[e], x[e]), u);
        quads(GATE ? dy[e] * (z[e] * sigmoid(z[e])) : dy[e], o);
#pragma unroll
        for (int k = 0; k < 2 * NL; ++k) p[k] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sB[j] = sA[j] = y[j] = 0.f;
#pragma unroll
          for (int k = 0; k < NL; ++k) {
            const float Gt = fmaf(Cn[k], o[j], G[j][k]);
            sB[j] = fmaf(Gt, B[k], sB[j]);
            p[k] = fmaf(Gt, u[j], p[k]);
            p[NL + k] = fmaf(o[j], h[e + 1][j][k], p[NL + k]);
            if (GATE) y[j] = fmaf(Cn[k], h[e + 1][j][k], y[j]);
            G[j][k] = Gt;
          }
        }
        if (fresh[e]) {  // nothing passes a start
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < NL; ++k) G[j][k] = 0.f;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < NL; ++k) {
              G[j][k] *= __builtin_amdgcn_exp2f(d[j] * A[j][k]);
              const float wk = G[j][k] * h[e][j][k];
              sA[j] = fmaf(wk, A[j][k], sA[j]);
              dA[j][k] = fmaf(wk, d[j], dA[j][k]);
            }
        }
        GroupSums<2 * NL, LG> sums;
        sums(p);
        if (row < a.rows && sums.keeps) {
          const int64_t at_t = (t0 + e) * a.rows + row;
#pragma unroll
          for (int k = 0; k < sums.LEFT; ++k) {
            const int f = sums.first + k, st = s0 + (f < NL ? f : f - NL);
            if (!FULL && st >= a.n) continue;
            if (a.tiles > 1) a.bc[(tile * a.steps * a.rows + at_t) * 2 * a.n + (f < NL ? 0 : a.n) + st] = p[k];
            else store1<TYPE>(f < NL ? a.dB : a.dC, at_t * a.n + st, p[k]);
          }
        }
        const float tB = quad_sums(sB), tA = quad_sums(sA), ty = GATE ? quad_sums(y) : 0.f;
        if constexpr (NW == 1) {
          finish(e, tB, tA, ty);
        } else {
          red[par][w][e][0][lane] = tB, red[par][w][e][1][lane] = tA;
          if (GATE) red[par][w][e][2][lane] = ty;
        }
      }
      if constexpr (NW > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < K; ++e) {
          if (e >= n || e % NW != w) continue;
          float t[3] = {0.f, 0.f, 0.f};
#pragma unroll
          for (int f = 0; f < NW; ++f)
#pragma unroll
            for (int k = 0; k < (GATE ? 3 : 2); ++k) t[k] += red[par][f][e][k][lane];
          finish(e, t[0], t[1], t[2]);
        }
        par ^= 1;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < NL; ++k) accs[j * NL + k][threadIdx.x] += dA[j][k];
      dD += sD;
      d_bias += sb;
    }
    if (ts == 0 && a.dh0)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (in && g + j < a.cols) store_n<NL, FULL>(a.dh0, at + j * a.n, s0, a.n, G[j]);
  }
  if (!a.part) return;
  const int64_t width = (int64_t)a.cols * (a.n + 2);
  float* const dst = a.part + ((slot * a.chunks + c) * RPW + sub) * width;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int k = 0; k < NL; ++k)
      if (g + j < a.cols && s0 + k < a.n) dst[(int64_t)(g + j) * a.n + s0 + k] = (float)accs[j * NL + k][threadIdx.x];
  if constexpr (NW > 1) {  // the waves' steps
    double* const t = &accs[0][0];
    __syncthreads();
    t[threadIdx.x] = dD;
    t[64 * NW + threadIdx.x] = d_bias;
    __syncthreads();
    dD = d_bias = 0;
    for (int f = 0; f < NW; ++f) dD += t[f * 64 + lane], d_bias += t[(NW + f) * 64 + lane];
  }
  if (w == 0 && col < a.cols) {
    dst[(int64_t)a.cols * a.n + col] = (float)dD;
    dst[(int64_t)a.cols * (a.n + 1) + col] = (float)d_bias;
  }
}

// dB and dC from the tiles' sums.
template <int TYPE>
__global__ __launch_bounds__(256) void ssm_tiles_kernel(SsmArgs a) {
  const int64_t S = a.steps * a.rows * 2 * a.n;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < S; i += (int64_t)gridDim.x * 256) {
    float v = a.bc[i];
    for (int k = 1; k < a.tiles; ++k) v += a.bc[k * S + i];
    const int64_t at = i / (2 * a.n);
    const int k = (int)(i - at * 2 * a.n);
    store1<TYPE>(k < a.n ? a.dB : a.dC, at * a.n + (k < a.n ? k : k - a.n), v);
  }
}

constexpr int64_t WAVES = 2048;   // waves that a launch wants
constexpr int64_t CHUNK_WAVES = 2048;

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// How a backward is dealt, and its scratch.
struct Deal {
  int lg, tiles, waves;  // groups of a tile (their logarithm), tiles of a row, waves of a workgroup
  int64_t chunk, chunks, slots, parts;
  size_t state, sums, bc, part, all;
};
Deal deal(int64_t steps, int64_t rows, int cols, int n) {
  Deal d{};
  const int per_row = (cols + 3) / 4;
  d.lg = per_row == 1 ? 0 : per_row <= 4 ? 2 : 4;
  d.tiles = (per_row + (1 << d.lg) - 1) >> d.lg;
  d.waves = n <= 16 ? 1 : n <= 32 ? 2 : 4;
  const int rpw = 16 >> d.lg;
  d.chunk = ssm_chunk(steps, rows, cols, CHUNK_WAVES);
  d.chunks = (steps + d.chunk - 1) / d.chunk;
  const int64_t most = (rows + rpw - 1) / rpw, want = (WAVES + d.tiles * d.chunks - 1) / (d.tiles * d.chunks);
  d.slots = most < want ? most : want;
  d.parts = d.slots * d.chunks * rpw;
  const int64_t C = rows * cols;
  d.state = d.chunks > 1 ? up(4 * d.chunks * C * n) : 0;
  d.sums = d.chunks > 1 ? up(4 * d.chunks * C) : 0;
  d.bc = d.tiles > 1 ? up(4 * (size_t)d.tiles * steps * rows * 2 * n) : 0;
  d.part = up(4 * (size_t)d.parts * cols * (n + 2));
  d.all = d.state + d.sums + d.bc + d.part;
  return d;
}

// Calls f(NL, NW, FULL): states of a lane, waves that share a column's, whether
// they are all there.
template <class F>
hipError_t by_states(int n, F f) {
  const std::false_type part;
  if (n <= 4) return f(Int<1>(), Int<1>(), part);
  if (n == 16) return f(Int<4>(), Int<1>(), std::true_type());
  if (n <= 16) return f(Int<4>(), Int<1>(), part);
  if (n <= 32) return f(Int<4>(), Int<2>(), part);
  return f(Int<4>(), Int<4>(), part);
}
template <class F>
hipError_t by_groups(int lg, F f) {
  return lg == 0 ? f(Int<0>()) : lg == 2 ? f(Int<2>()) : f(Int<4>());
}

template <int TYPE, bool GATE>
hipError_t launch_typed(SsmArgs& a, const Deal& d, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (a.chunks > 1) {
    const int64_t groups = a.rows * ((a.cols + 3) / 4);
    const dim3 grid((unsigned)((groups * 4 + 255) / 256), (unsigned)a.chunks - 1);
    const auto carry = [&](auto nl) {
      if (a.n == 4 * nl()) hipLaunchKernelGGL((ssm_carry_kernel<TYPE, nl(), true, GATE>), grid, dim3(256), 0, st, a);
      else hipLaunchKernelGGL((ssm_carry_kernel<TYPE, nl(), false, GATE>), grid, dim3(256), 0, st, a);
      return hipGetLastError();
    };
    e = a.n <= 4 ? carry(Int<1>()) : a.n <= 8 ? carry(Int<2>()) : a.n <= 16 ? carry(Int<4>()) : a.n <= 32 ? carry(Int<8>()) : carry(Int<16>());
    if (e == hipSuccess) e = launch_ssm_join(a, a.dh_last, true, st);
    if (e != hipSuccess) return e;
  }
  e = by_states(a.n, [&](auto nl, auto nw, auto full) {
    return by_groups(d.lg, [&](auto lg) {
      const dim3 grid((unsigned)(a.slots * a.tiles), (unsigned)a.chunks), block(64 * nw());
      hipLaunchKernelGGL((ssm_grad_kernel<TYPE, nl(), nw(), lg(), full(), GATE>), grid, block, 0, st, a);
      return hipGetLastError();
    });
  });
  if (e != hipSuccess || a.tiles == 1) return e;
  const int64_t n = a.steps * a.rows * 2 * a.n, b = (n + 255) / 256;
  hipLaunchKernelGGL((ssm_tiles_kernel<TYPE>), dim3((unsigned)(b < 65536 ? b : 65536)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t ssm_grad_work_bytes(int64_t steps, int64_t rows, int cols, int n) {
  return steps > 0 && rows > 0 ? deal(steps, rows, cols, n).all : 0;
}

hipError_t launch_ssm_grad(SsmArgs a, int type, float* dA, float* dD, float* d_bias, int accumulate, void* work,
                           hipStream_t st) {
  const int64_t C = a.rows * a.cols, cn = (int64_t)a.cols * a.n;
  int64_t parts = 0;
  if (C > 0 && a.steps <= 0 && a.dh0 && a.dh0 != a.dh_last)
    if (const hipError_t e = launch_state_copy(a.dh_last, a.dh0, C * a.n, st); e != hipSuccess) return e;
  if (C > 0 && a.steps > 0) {
    const Deal d = deal(a.steps, a.rows, a.cols, a.n);
    char* p = (char*)work;
    a.state = (float*)p, p += d.state;
    a.sums = (float*)p, p += d.sums;
    a.bc = (float*)p, p += d.bc;
    a.part = dA || dD || d_bias ? (float*)p : nullptr;
    a.chunk = d.chunk, a.chunks = d.chunks, a.slots = d.slots, a.tiles = d.tiles;
    parts = d.parts;
    const hipError_t e = type == MGN_BF16
        ? a.z ? launch_typed<MGN_BF16, true>(a, d, st) : launch_typed<MGN_BF16, false>(a, d, st)
        : a.z ? launch_typed<MGN_FP32, true>(a, d, st) : launch_typed<MGN_FP32, false>(a, d, st);
    if (e != hipSuccess) return e;
  }
  if (!dA && !dD && !d_bias) return hipSuccess;
  return launch_col_sums(ColSums{a.part, parts, cn + 2 * (int64_t)a.cols, {dA, dD, d_bias}, {cn, a.cols}, accumulate}, st);
}

}  // namespace mgn
