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
// Bound by the vector units: 15 instructions and two exponentials a state and step (the
// states before a unit are formed first, then its own again).  20 steps of 20,011 x 64
// bf16, 16 states, 482 - 495 us under the profiler, the units busy 77 % of them with the
// two waves a SIMD that 256 registers leave.  Most forms of more than 8 states spill some:
// 8 registers here, 18 in fp32, 41 at most (2 waves, tiles of 4 groups, fp32).  That is
// what the last unit's and the sweep's loads ahead cost, and still the faster way: 570 us
// without.  A unit of 4 steps spills much more (1.3 ms and more).
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
  __device__ __forceinline__ void level(float (&v)[M]) const {
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
          const bool hi = threadIdx.x & D;
          const float mine = hi ? v[k + N / 2] : v[k], other = hi ? v[k] : v[k + N / 2];
          v[k] = mine + across<D>(other);
        }
      }
    } else {
      v[0] += across<D>(v[0]);
    }
    if constexpr (D > 4) level<(N > 1 ? N / 2 : 1), D / 2>(v);
  }
  __device__ __forceinline__ void operator()(float (&v)[M]) const {
    if constexpr (LG > 0) level<M, 2 << LG>(v);
  }
  __device__ __forceinline__ void find() {
    first = 0;
    keeps = true;
    int left = M;
#pragma unroll
    for (int d = 2 << LG; d >= 4; d /= 2) {
      const bool hi = threadIdx.x & d;
      if (left > 1) left /= 2, first += hi ? left : 0;
      else keeps = keeps && !hi;
    }
  }
};

// G that leaves each chunk (through its first step), from zeros at its end, and
// its sum of delta; chunk blockIdx.y + 1.
template <int TYPE, int NL, bool FULL, bool GATE>
__global__ __launch_bounds__(256) void ssm_carry_kernel(SsmArgs a) {
  constexpr int STEPS = NL <= 4 ? 4 : NL == 8 ? 2 : 1;
  const int per_row = (a.cols + 3) / 4, q = threadIdx.x & 3;
  const int64_t gi = ((int64_t)blockIdx.x * 256 + threadIdx.x) / 4, row = gi / per_row;
  const int g = (int)(gi - row * per_row) * 4, col = g + q;
  const Share<NL, FULL> own(q, a.n);
  const bool in = row < a.rows, ok = in && col < a.cols;
  const int c = blockIdx.y + 1;
  const int64_t ts = c * a.chunk, te = ts + a.chunk < a.steps ? ts + a.chunk : a.steps;
  const int64_t C = a.rows * a.cols, i = row * a.cols + col, bn = row * a.n, at = (row * a.cols + g) * a.n;
  float G[4][NL], A[4][NL];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int k = 0; k < NL; ++k) G[j][k] = A[j][k] = 0.f;
    if (in && g + j < a.cols) load_n<MGN_FP32>(a.A, (int64_t)(g + j) * a.n + own.s, own, A[j]);
#pragma unroll
    for (int k = 0; k < NL; ++k) A[j][k] *= LOG2E;
  }
  const bool growing = !a.softplus || growth(A) > 0.f;
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
      if (in) load_n<TYPE>(a.C, (t - e) * a.rows * a.n + bn + own.s, own, Cn[e]);
    }
    const auto back = [&](auto growing) {
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
          for (int k = 0; k < NL; ++k) {
            const float f = __builtin_amdgcn_exp2f(d[j] * A[j][k]);
            G[j][k] = fmaf(Cn[e][k], ov[j], G[j][k]) * (growing() ? passed(f) : f);
          }
        if (fresh[e]) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < NL; ++k) G[j][k] = 0.f;
          sum = CUT;
        }
      }
    };
    if (growing) back(std::true_type());
    else back(std::false_type());
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (in && g + j < a.cols) store_n(a.state + c * C * a.n, at + j * a.n + own.s, own, G[j]);
  if (ok) a.sums[c * C + i] = sum;
}

// Steps of a unit: their states and factors stay in registers between the way forth
// and the way back.
constexpr int U = 2, UNITS = K / U;
static_assert(U == 2 && UNITS >= 2);

template <int TYPE, int NL, int NW, int LG, bool FULL, bool GATE>
__global__ __launch_bounds__(64 * NW, 2) void ssm_grad_kernel(SsmArgs a) {
  constexpr int GP = 1 << LG, RPW = 16 / GP, SIZE = sizeof(Elem<TYPE>);
  using Sums = GroupSums<2 * NL, LG>;
  __shared__ double accs[4 * NL][64 * NW];
  // the states before units 0 .. UNITS - 2 (with 4 waves unit 0's are read again: two
  // workgroups of a CU have no room for them)
  constexpr int KEPT = NW == 4 ? 1 : 0;
  __shared__ float subs[UNITS - 1 - KEPT][4 * NL][64 * NW];
  __shared__ float red[NW > 1 ? 2 : 1][NW > 1 ? NW : 1][NW > 1 ? U : 1][3][64];
  const int lane = threadIdx.x & 63, w = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane & 3;
  const int tile = blockIdx.x % a.tiles, sub = (lane >> 2) >> LG;
  const int64_t slot = blockIdx.x / a.tiles;
  const int g = (tile * GP + ((lane >> 2) & (GP - 1))) * 4, col = g + q;
  const Share<NL, FULL> own(w * 4 + q, a.n);
  const int c = blockIdx.y;
  const int64_t ts = c * a.chunk, te = ts + a.chunk < a.steps ? ts + a.chunk : a.steps;
  const int64_t C = a.rows * a.cols, cb = C * SIZE, rb = a.rows * a.n * SIZE;  // a step's bytes

  float A[4][NL];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int k = 0; k < NL; ++k) A[j][k] = 0.f, accs[j * NL + k][threadIdx.x] = 0;
    if (g + j < a.cols) load_n<MGN_FP32>(a.A, (int64_t)(g + j) * a.n + own.s, own, A[j]);
#pragma unroll
    for (int k = 0; k < NL; ++k) A[j][k] *= LOG2E;
  }
  const float rate = growth(A);
  const float bias = a.bias && col < a.cols ? a.bias[col] : 0.f, D = a.D && col < a.cols ? a.D[col] : 0.f;
  double dD = 0, d_bias = 0;
  int par = 0;
  const auto step_size = [&](Word<TYPE> raw, bool ok) {
    float delta = value1<TYPE>(raw) + bias;
    if (a.softplus) delta = softplus(delta);
    return ok ? delta : 0.f;
  };
  // What a unit's steps bring, as it lies in memory.
  struct In {
    Word<TYPE> x[U], dt[U], o[U], z[U];
    Raw<TYPE, NL, true> B[U], C[U];
  };
  struct Sweep {
    Word<TYPE> x[U], dt[U];
    Raw<TYPE, NL, true> B[U];
  };

  for (int64_t r0 = slot * RPW; r0 < a.rows; r0 += a.slots * RPW) {
    const bool row_in = r0 + sub < a.rows, in = row_in && g < a.cols, ok = in && col < a.cols;
    // the lane's column, states and n numbers from the wave's first row's on
    // (lanes without one read that row's first)
    const uint32_t o = ok ? (uint32_t)(sub * a.cols + col) * SIZE : 0, ob = ((row_in ? (uint32_t)(sub * a.n) : 0) + own.s) * SIZE;
    const uint32_t oh = in ? (uint32_t)((sub * a.cols + g) * a.n) : 0;
    float G[4][NL], h[U + 1][4][NL];
    const auto load_states = [&](const float* from, float (&v)[4][NL]) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int k = 0; k < NL; ++k) v[j][k] = 0.f;
        if (from && in && g + j < a.cols)
          load_n<MGN_FP32>(from + r0 * a.cols * a.n, here(oh + j * a.n + own.s), own, v[j]);
      }
    };
    const auto zero = [](float (&v)[4][NL]) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < NL; ++k) v[j][k] = 0.f;
    };
    load_states(a.chunks > 1 ? a.state + c * C * a.n : a.dh_last, G);
    // the starts of a block's steps, from the lanes' loads of one; those of the block
    // before are on their way.  (Without starts a byte of x stands in: no branch, where
    // its ways meet the compiler waits as for the one with the fewest loads.)
    const uint8_t* const starts = a.starts ? a.starts : (const uint8_t*)a.x;
    const auto look = [&](int64_t t) { return starts[t + (lane & (K - 1)) < te ? t + (lane & (K - 1)) : te - 1]; };
    uint8_t ahead = look((te - 1) / K * K);

    for (int64_t t0 = (te - 1) / K * K; t0 >= ts; t0 -= K) {
      const float* const mark = a.marks + t0 / K * C * a.n;
      const int n = te - t0 < K ? (int)(te - t0) : K, last = (n - 1) / U;  // steps of the block, its last unit
      const int64_t x0 = (t0 * C + r0 * a.cols) * SIZE, n0 = (t0 * a.rows + r0) * a.n * SIZE;
      const auto load_unit = [&](int v, In& r) {
        const int m = n - v * U;
        const int64_t xu = x0 + v * U * cb, nu = n0 + v * U * rb;
#pragma unroll
        for (int e = 0; e < U; ++e) {
          const int at = e < m ? e : 0;
          const int64_t i = xu + at * cb, b = nu + at * rb;
          r.x[e] = raw1<TYPE>((const char*)a.x + i, o);
          r.dt[e] = raw1<TYPE>((const char*)a.dt + i, o);
          r.o[e] = raw1<TYPE>((const char*)a.dy + i, o);
          if (GATE) r.z[e] = raw1<TYPE>((const char*)a.z + i, o);
          r.B[e].load((const char*)a.B + b, ob);
          r.C[e].load((const char*)a.C + b, ob);
        }
      };
      const auto load_sweep = [&](int v, Sweep& r) {
        const int64_t xu = x0 + v * U * cb, nu = n0 + v * U * rb;
#pragma unroll
        for (int e = 0; e < U; ++e) {
          const int at = v * U + e < n ? e : 0;
          r.x[e] = raw1<TYPE>((const char*)a.x + (xu + at * cb), o);
          r.dt[e] = raw1<TYPE>((const char*)a.dt + (xu + at * cb), o);
          r.B[e].load((const char*)a.B + (nu + at * rb), ob);
        }
      };
      const uint32_t begins =
          a.starts ? (uint32_t)__builtin_amdgcn_ballot_w64(ahead != 0 && t0 + (lane & (K - 1)) < te) & ((1 << K) - 1) : 0;
      ahead = look(t0 >= ts + K ? t0 - K : ts);
      // the states before each unit, its loads in flight while the one before it runs
      load_states(mark, h[0]);
      In units[2];
      Sweep sweeps[2];
      load_sweep(0, sweeps[0]);
      load_unit(last, units[0]);
#pragma unroll
      for (int v = 0; v < UNITS - 1; ++v) {
        if (v >= last) break;
        const Sweep& now = sweeps[v % 2];
        load_sweep(v + 1 < last ? v + 1 : v, sweeps[(v + 1) % 2]);
        if (v >= KEPT)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < NL; ++k) subs[v - KEPT][j * NL + k][threadIdx.x] = h[0][j][k];
        const uint32_t fresh = begins >> (v * U) & ((1 << U) - 1);
        float delta[U];
        bool careful = false;
#pragma unroll
        for (int e = 0; e < U; ++e) {
          delta[e] = step_size(now.dt[e], ok);
          careful = careful || (ok && !(delta[e] > 0.f));
        }
        if (__float_as_int(rate) > 0) careful = careful || delta[0] * rate > 127.f || delta[1] * rate > 127.f;
        careful = any(careful);
        const auto step = [&](int e, auto way) {
          float d[4], u[4], B[NL];
          now.B[e].get(B);
          own.mask(B);
          quads(delta[e], d);
          quads(way() == CAREFUL ? mul_or_0(delta[e], value1<TYPE>(now.x[e])) : delta[e] * value1<TYPE>(now.x[e]), u);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < NL; ++k) {
              const float keep = __builtin_amdgcn_exp2f(d[j] * A[j][k]), b = way() == CAREFUL ? mul_or_0(u[j], B[k]) : u[j] * B[k];
              h[0][j][k] = fmaf(way() == CAREFUL ? passed(keep) : keep, h[0][j][k], b);
            }
        };
        if (!fresh && !careful) {
#pragma unroll
          for (int e = 0; e < U; ++e) step(e, Int<PLAIN>());
        } else {
#pragma unroll
          for (int e = 0; e < U; ++e) {
            if (fresh >> e & 1) zero(h[0]);
            if (careful) step(e, Int<CAREFUL>());
            else step(e, Int<PLAIN>());
          }
        }
      }
      float dA[4][NL], sD = 0.f, sb = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < NL; ++k) dA[j][k] = 0.f;
      const auto unit = [&](int v, const In& r) {
        const int m = n - v * U < U ? n - v * U : U;  // the unit's steps
        const int64_t xu = x0 + v * U * cb, nu = n0 + v * U * rb, tu = t0 + v * U;
        const bool fresh[U] = {(begins >> (v * U) & 1) != 0, (begins >> (v * U + 1) & 1) != 0};
        if (v != last) {
          if (KEPT && v < KEPT) {
            load_states(mark, h[0]);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int k = 0; k < NL; ++k) h[0][j][k] = subs[v - KEPT][j * NL + k][threadIdx.x];
          }
        }
        float delta[U], ov[U], sz[U], f[U][4][NL], tB[U], tA[U], ty[U], p[U][2 * NL];
        bool careful = false;
#pragma unroll
        for (int e = 0; e < U; ++e) {
          delta[e] = step_size(r.dt[e], ok);
          careful = careful || (ok && !(delta[e] > 0.f));
          ov[e] = value1<TYPE>(r.o[e]);
          if (GATE) {
            const float z = value1<TYPE>(r.z[e]);
            sz[e] = sigmoid(z);
            ov[e] *= z * sz[e];
          }
          // a step that is not there changes nothing
          if (!ok || e >= m) delta[e] = ov[e] = 0.f;
        }
        if (__float_as_int(rate) > 0) careful = careful || delta[0] * rate > 127.f || delta[1] * rate > 127.f;
        careful = any(careful);
        const auto input = [&](int e) { return mul_or_0(delta[e], value1<TYPE>(r.x[e])); };
        const auto forth = [&](int e, auto first, auto way) {
          float d[4], u[4], B[NL];
          r.B[e].get(B);
          own.mask(B);
          quads(delta[e], d);
          quads(input(e), u);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < NL; ++k) {
              const float b = way() == CAREFUL ? mul_or_0(u[j], B[k]) : u[j] * B[k];
              const float keep = first() ? 0.f : __builtin_amdgcn_exp2f(d[j] * A[j][k]);
              f[e][j][k] = way() == CAREFUL ? passed(keep) : keep;
              h[e + 1][j][k] = first() ? b : fmaf(f[e][j][k], h[e][j][k], b);
            }
          __builtin_amdgcn_sched_barrier(0);
        };
        const auto forth_any = [&](int e) {
          if (fresh[e]) forth(e, std::true_type(), Int<CAREFUL>());
          else if (careful) forth(e, std::false_type(), Int<CAREFUL>());
          else forth(e, std::false_type(), Int<PLAIN>());
        };
        const auto back = [&](int e) {
          float B[NL], Cn[NL], d[4], u[4], ot[4], sB[4], sA[4], y[4];
          r.B[e].get(B);
          own.mask(B);
          r.C[e].get(Cn);
          own.mask(Cn);
          quads(delta[e], d);
          quads(input(e), u);
          quads(ov[e], ot);
#pragma unroll
          for (int k = 0; k < 2 * NL; ++k) p[e][k] = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            sB[j] = sA[j] = y[j] = 0.f;
#pragma unroll
            for (int k = 0; k < NL; ++k) {
              const float Gt = fmaf(Cn[k], ot[j], G[j][k]);
              sB[j] = fmaf(Gt, B[k], sB[j]);
              p[e][k] = fmaf(Gt, u[j], p[e][k]);
              p[e][NL + k] = fmaf(ot[j], h[e + 1][j][k], p[e][NL + k]);
              if (GATE) y[j] = fmaf(Cn[k], h[e + 1][j][k], y[j]);
              G[j][k] = Gt * f[e][j][k];
              const float wk = G[j][k] * h[e][j][k];
              sA[j] = fmaf(wk, A[j][k], sA[j]);
              dA[j][k] = fmaf(wk, d[j], dA[j][k]);
            }
          }
          tB[e] = quad_sums(sB), tA[e] = quad_sums(sA);
          if (GATE) ty[e] = quad_sums(y);
          Sums()(p[e]);
          __builtin_amdgcn_sched_barrier(0);
        };
        if (!careful && !fresh[0] && !fresh[1]) {
          forth(0, std::false_type(), Int<PLAIN>());
          forth(1, std::false_type(), Int<PLAIN>());
        } else {
          forth_any(0);
          forth_any(1);
        }
        // a first step (f = 0) sees no state, whatever the one before it left, and
        // passes no gradient on
        if (fresh[1]) zero(h[1]);
        back(1);
        if (fresh[1]) {
          zero(G);
          forth_any(0);
        }
        if (fresh[0]) zero(h[0]);
        back(0);
        if (fresh[0]) zero(G);
        // dB, dC: a number of a step and row in one lane of the wave
        Sums where;
        where.find();
        if (row_in && where.keeps)
#pragma unroll
          for (int k = 0; k < Sums::LEFT; ++k) {
            const int x = where.first + k, st = x < NL ? x : x - NL;
            if (!own.has(st)) continue;
#pragma unroll
            for (int e = 0; e < U; ++e) {
              if (e >= m) continue;
              if (a.tiles > 1)
                write1<MGN_FP32>((char*)a.bc + ((tile * a.steps + tu + e) * a.rows + r0) * 2 * a.n * 4,
                                 (uint32_t)(sub * 2 * a.n + (x < NL ? 0 : a.n) + own.s + st) * 4, p[e][k]);
              else if (x < NL)
                write1<TYPE>((char*)a.dB + (nu + e * rb), ob + (uint32_t)(st * SIZE), p[e][k]);
              else
                write1<TYPE>((char*)a.dC + (nu + e * rb), ob + (uint32_t)(st * SIZE), p[e][k]);
            }
          }
        if constexpr (NW > 1) {
#pragma unroll
          for (int e = 0; e < U; ++e) {
            red[par][w][e][0][lane] = tB[e], red[par][w][e][1][lane] = tA[e];
            if (GATE) red[par][w][e][2][lane] = ty[e];
          }
          __syncthreads();
        }
        // the gradients of one column and step, from the sums over all its states
        if (ok)
#pragma unroll
          for (int e = 0; e < U; ++e) {
            if (e >= m || (NW > 1 && e % NW != w)) continue;
            if constexpr (NW > 1) {
              tB[e] = tA[e] = ty[e] = 0.f;
#pragma unroll
              for (int x = 0; x < NW; ++x) {
                tB[e] += red[par][x][e][0][lane], tA[e] += red[par][x][e][1][lane];
                if (GATE) ty[e] += red[par][x][e][2][lane];
              }
            }
            const float x = value1<TYPE>(r.x[e]);
            float dx = mul_or_0(delta[e], tB[e]), dd = fmaf(tA[e], LN2, tB[e] * x);
            if (a.D) dx = fmaf(D, ov[e], dx);
            // (x may hold anything at a step of size 0 that no gradient reaches; a D that is
            // left out has a gradient too)
            sD += mul_or_0(ov[e], x);
            if (a.softplus) dd = mul_or_0(sigmoid(value1<TYPE>(r.dt[e]) + bias), dd);
            sb += dd;
            write1<TYPE>((char*)a.dx + (xu + e * cb), o, dx);
            write1<TYPE>((char*)a.ddt + (xu + e * cb), o, dd);
            if (GATE) {
              const float z = value1<TYPE>(r.z[e]), s = sz[e], y = a.D ? fmaf(D, x, ty[e]) : ty[e];
              write1<TYPE>((char*)a.dz + (xu + e * cb), o, mul_or_0(value1<TYPE>(r.o[e]), y) * (s * fmaf(z, 1.f - s, 1.f)));
            }
          }
        if constexpr (NW > 1) par ^= 1;
      };
      for (int v = last;; v -= 2) {
        load_unit(v > 0 ? v - 1 : 0, units[1]);  // while this one runs
        unit(v, units[0]);
        if (v == 0) break;
        load_unit(v > 1 ? v - 2 : 0, units[0]);
        unit(v - 1, units[1]);
        if (v == 1) break;
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
        if (in && g + j < a.cols) store_n(a.dh0 + r0 * a.cols * a.n, oh + j * a.n + own.s, own, G[j]);
  }
  if (!a.part) return;
  const int64_t width = (int64_t)a.cols * (a.n + 2);
  float* const dst = a.part + (slot * a.chunks + c) * width;
  // the wave's rows
  const auto rows = [&](double v) {
#pragma unroll
    for (int d = 4 * GP; d < 64; d *= 2) v += __shfl_xor(v, d);
    return v;
  };
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int k = 0; k < NL; ++k) {
      const double v = rows(accs[j * NL + k][threadIdx.x]);
      if (sub == 0 && g + j < a.cols && own.has(k)) dst[(int64_t)(g + j) * a.n + own.s + k] = (float)v;
    }
  if constexpr (NW > 1) {  // the waves' steps
    double* const t = &accs[0][0];
    __syncthreads();
    t[threadIdx.x] = dD;
    t[64 * NW + threadIdx.x] = d_bias;
    __syncthreads();
    dD = d_bias = 0;
    for (int m = 0; m < NW; ++m) dD += t[m * 64 + lane], d_bias += t[(NW + m) * 64 + lane];
  }
  dD = rows(dD), d_bias = rows(d_bias);
  if (w == 0 && sub == 0 && col < a.cols) {
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

// Waves that a launch wants: two a SIMD, as many as its registers hold.
constexpr int64_t WAVES = 2048;

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// How a backward is dealt, and its scratch.
struct Deal {
  int lg, tiles;  // groups of a tile (their logarithm), tiles of a row
  int64_t chunk, chunks, slots, parts;
  size_t state, sums, bc, part, all;
};
Deal deal(int64_t steps, int64_t rows, int cols, int n) {
  Deal d{};
  const int per_row = (cols + 3) / 4;
  d.lg = per_row <= 4 ? 2 : 4;
  d.tiles = (per_row + (1 << d.lg) - 1) >> d.lg;
  const int rpw = 16 >> d.lg;
  d.chunk = ssm_chunk(steps, rows, cols, WAVES);
  d.chunks = (steps + d.chunk - 1) / d.chunk;
  const int64_t most = (rows + rpw - 1) / rpw, want = (WAVES + d.tiles * d.chunks - 1) / (d.tiles * d.chunks);
  d.slots = most < want ? most : want;
  d.parts = d.slots * d.chunks;
  const int64_t C = rows * cols;
  d.state = d.chunks > 1 ? up(4 * d.chunks * C * n) : 0;
  d.sums = d.chunks > 1 ? up(4 * d.chunks * C) : 0;
  d.bc = d.tiles > 1 ? up(4 * (size_t)d.tiles * steps * rows * 2 * n) : 0;
  d.part = up(4 * (size_t)d.parts * cols * (n + 2));
  d.all = d.state + d.sums + d.bc + d.part;
  return d;
}

// Calls f(NL, NW, FULL): states of a lane, waves that share a column's, whether they are
// all there, so that no run is masked, which is faster though it spills more: forward and
// backward of 20 steps of 20,011 x 64, 16 states, bf16 611 us, 737 as if some were
// missing, fp32 651 and 754; 100 steps of 1,000 x 128, 32 states, 794, 931 and 907, 940;
// 64 1,289, 1,658 and 1,382, 1,677.  (4 and 8: 228, 230 and 248, 259; their backward has
// the general form only.)
template <class F>
hipError_t by_states(int n, F f) {
  const std::false_type part;
  const std::true_type whole;
  if (n <= 4) return f(Int<1>(), Int<1>(), part);
  if (n <= 8) return f(Int<2>(), Int<1>(), part);
  if (n == 16) return f(Int<4>(), Int<1>(), whole);
  if (n <= 16) return f(Int<4>(), Int<1>(), part);
  if (n == 32) return f(Int<4>(), Int<2>(), whole);
  if (n <= 32) return f(Int<4>(), Int<2>(), part);
  if (n == 64) return f(Int<4>(), Int<4>(), whole);
  return f(Int<4>(), Int<4>(), part);
}
template <class F>
hipError_t by_groups(int lg, F f) {
  return lg == 2 ? f(Int<2>()) : f(Int<4>());
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
