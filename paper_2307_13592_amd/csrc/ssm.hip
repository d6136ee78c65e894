// Selective state space scan along time (gfx950): every column of every row has n
// states, with a step size, an input and an output vector of each step's own:
//   delta = softplus(dt + bias) (or dt + bias),
//   h_t[k] = exp(delta A[k]) h_{t-1}[k] + delta x B_t[k],
//   y_t = (sum_k C_t[k] h_t[k] + D x) z sigmoid(z).
//
// The states stay in registers (ssm.h) from the first step to the last, and each
// input is read once.  With few columns the time axis is cut into chunks: a first
// launch takes each chunk from zero states to its end, a second joins these (all
// that a chunk does to what enters it is the factor exp(A sum of delta), of which the
// sum is one number a column), a third runs every chunk from the state that enters
// it.  A chunk's work is then done twice but for y.
//
// Bound by the vector units: 4 products and sums and an exponential, which takes two
// instructions' time, for a state and step, and some 60 instructions a step for what is
// done once a column and for the exchanges, against 6 - 16 bytes an element.  600 steps
// of 1,885 x 64 bf16, 16 states, 404 us (the units busy 75 %: some SIMDs have one wave,
// some two); 20 steps of 20,011 x 64 141 us (81 %).  With one step by the states' 8 n
// bytes: 1,885 x 128 fp32 7.0 us, 4.9 TB/s.
#include "ssm.h"

namespace mgn {
namespace {

constexpr int NT = 256;
enum Pass { WHOLE_AXIS, MANY_ROWS, LOCAL_ENDS, FROM_STATES, ONE_STEP };

// What some steps bring, as it lies in memory.
template <int TYPE, int NL, int STEPS>
struct Inputs {
  Word<TYPE> x[STEPS], dt[STEPS], z[STEPS];
  Raw<TYPE, NL, true> B[STEPS], C[STEPS];
};

template <int TYPE, int NL, bool FULL, int PASS>
__global__ __launch_bounds__(NT) void ssm_kernel(SsmArgs a) {
  // Steps whose loads are in flight together.  With many rows two of them and a third
  // wave in a SIMD's registers: 20 steps of 20,011 x 64 bf16 141 us, 163 with four (fp32
  // 140 and 163); otherwise four: 600 steps of 1,885 x 64 404 us, 424 with two (396, 441).
  constexpr int STEPS = PASS == ONE_STEP || NL == 16 ? 1 : NL == 8 || (NL == 4 && PASS == MANY_ROWS) ? 2 : 4;
  using E = Elem<TYPE>;
  using In = Inputs<TYPE, NL, STEPS>;
  constexpr int SIZE = sizeof(E);
  const int q = threadIdx.x & 3, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t group = a.group0 + ((int64_t)blockIdx.x * (NT / 64) + wave) * 16;
  const Spot p(a, group, q);
  const Share<NL, FULL> own(q, a.n);
  if (p.row0 >= a.rows) return;
  const int c = blockIdx.y;
  const int64_t ts = c * a.chunk, te = ts + a.chunk < a.steps ? ts + a.chunk : a.steps;
  const int64_t C = a.rows * a.cols, cb = C * SIZE, rb = a.rows * a.n * SIZE;  // a step's bytes

  // the next steps to load, and to store.  No branch stands between the loads or around
  // them: where its ways meet, the compiler waits as for the one with the fewest loads.
  // So a z that is not there is read from x's place, and behind the last step comes the
  // last one again.
  const int64_t x0 = (ts * C + p.i0) * SIZE, n0 = (ts * a.rows * a.n + p.bn0) * SIZE;
  const char *px = (const char*)a.x + x0, *pd = (const char*)a.dt + x0, *pz = (const char*)(a.z ? a.z : a.x) + x0;
  const char *pB = (const char*)a.B + n0, *pC = (const char*)a.C + n0;
  char* py = (char*)a.y + x0;
  const uint32_t o = p.o * SIZE, ob = (p.ob + own.s) * SIZE;
  const auto load = [&](In& v, int64_t left) {
    const int n = left < STEPS ? left < 1 ? 1 : (int)left : STEPS;
    int64_t xo = 0, no = 0;
#pragma unroll
    for (int e = 0; e < STEPS; ++e) {
      v.x[e] = raw1<TYPE>(px + xo, o);
      v.dt[e] = raw1<TYPE>(pd + xo, o);
      if constexpr (PASS != LOCAL_ENDS) v.z[e] = raw1<TYPE>(pz + xo, o);
      v.B[e].load(pB + no, ob);
      if constexpr (PASS != LOCAL_ENDS) v.C[e].load(pC + no, ob);
      if (e + 1 < n) xo += cb, no += rb;
    }
    if (left > STEPS) px += STEPS * cb, pd += STEPS * cb, pz += STEPS * cb, pB += STEPS * rb, pC += STEPS * rb;
  };
  In v[2];
  load(v[0], te - ts);

  float h[4][NL], A[4][NL];
  const float* const from = PASS == FROM_STATES ? a.state + c * C * a.n : PASS == LOCAL_ENDS ? nullptr : a.h0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int k = 0; k < NL; ++k) h[j][k] = A[j][k] = 0.f;
    if (p.in && p.g + j < a.cols) {
      load_n<MGN_FP32>(a.A, (int64_t)(p.g + j) * a.n + own.s, own, A[j]);
      if (from) load_n<MGN_FP32>(from + p.at0, p.oa + j * a.n + own.s, own, h[j]);
    }
  }
  const float bias = a.bias && p.ok ? a.bias[p.col] : 0.f, D = a.D && p.ok ? a.D[p.col] : 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int k = 0; k < NL; ++k) A[j][k] *= LOG2E;
  const float rate = growth(A);
  float sum = 0.f;
  Starts starts(a.starts, ts, te);

  const auto run = [&](const In& v, int64_t t) {
    const int n = te - t < STEPS ? (int)(te - t) : STEPS;
    if (PASS != LOCAL_ENDS && a.marks && t % MGN_MARK_STEPS == 0)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (p.in && p.g + j < a.cols)
          store_n(a.marks + (t / MGN_MARK_STEPS * C * a.n + p.at0), p.oa + j * a.n + own.s, own, h[j]);
    // what is done once a column
    float x[STEPS], delta[STEPS], y[STEPS], f[STEPS];
    bool careful = false;
    const uint32_t fresh = starts.at<STEPS>(t);
#pragma unroll
    for (int e = 0; e < STEPS; ++e) {
      x[e] = value1<TYPE>(v.x[e]);
      delta[e] = value1<TYPE>(v.dt[e]) + bias;
      y[e] = 0.f, f[e] = 1.f;
    }
    if (a.softplus)
#pragma unroll
      for (int e = 0; e < STEPS; ++e) delta[e] = softplus(delta[e]);
#pragma unroll
    for (int e = 0; e < STEPS; ++e) {
      careful = careful || (p.ok && !(delta[e] > 0.f));
      delta[e] = p.ok ? delta[e] : 0.f;
    }
    if (__float_as_int(rate) > 0)
#pragma unroll
      for (int e = 0; e < STEPS; ++e) careful = careful || delta[e] * rate > 127.f;
    if constexpr (PASS != LOCAL_ENDS) {
      if (a.D)
#pragma unroll
        for (int e = 0; e < STEPS; ++e) y[e] = D * x[e];
      if (a.z)
#pragma unroll
        for (int e = 0; e < STEPS; ++e) {
          const float z = value1<TYPE>(v.z[e]);
          f[e] = z * sigmoid(z);
        }
    }
    const auto step = [&](int e, auto way) {
      float d[4], w[4], r[4], B[NL], Cn[NL];
      quads(delta[e], d);
      quads(way() == CAREFUL ? mul_or_0(delta[e], x[e]) : delta[e] * x[e], w);
      v.B[e].get(B);
      own.mask(B);
      if constexpr (PASS != LOCAL_ENDS) v.C[e].get(Cn), own.mask(Cn);
      else sum += delta[e];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        r[j] = 0.f;
#pragma unroll
        for (int k = 0; k < NL; ++k) {
          const float keep = __builtin_amdgcn_exp2f(d[j] * A[j][k]), b = way() == CAREFUL ? mul_or_0(w[j], B[k]) : w[j] * B[k];
          h[j][k] = way() == CAREFUL ? carried(keep, h[j][k], b) : fmaf(keep, h[j][k], b);
          if constexpr (PASS != LOCAL_ENDS) r[j] = fmaf(Cn[k], h[j][k], r[j]);
        }
      }
      if constexpr (PASS != LOCAL_ENDS) y[e] = (quad_sums(r) + y[e]) * f[e];
    };
    careful = any(careful);
    if (n == STEPS && !fresh && !careful) {
#pragma unroll
      for (int e = 0; e < STEPS; ++e) step(e, Int<PLAIN>());
    } else {
#pragma unroll
      for (int e = 0; e < STEPS; ++e) {
        if (e >= n) break;
        if (fresh >> e & 1) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < NL; ++k) h[j][k] = 0.f;
          sum = CUT;
        }
        if (careful) step(e, Int<CAREFUL>());
        else step(e, Int<PLAIN>());
      }
    }
    if constexpr (PASS != LOCAL_ENDS) {
      if (p.ok)
#pragma unroll
        for (int e = 0; e < STEPS; ++e)
          if (e < n) store1<TYPE>(py + (e * cb + o), 0, y[e]);
      py += STEPS * cb;
    }
  };
  if constexpr (PASS == ONE_STEP) run(v[0], ts);
  else for (int64_t t = ts; t < te; t += 2 * STEPS) {
    load(v[1], te - (t + STEPS));  // while the steps before run
    run(v[0], t);
    if (t + STEPS >= te) break;
    load(v[0], te - (t + 2 * STEPS));
    run(v[1], t + STEPS);
  }
  float* const to = PASS == LOCAL_ENDS ? a.state + c * C * a.n : te == a.steps ? a.h_last : nullptr;
  if (to)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (p.in && p.g + j < a.cols) store_n(to + p.at0, p.oa + j * a.n + own.s, own, h[j]);
  if (PASS == LOCAL_ENDS && p.ok) a.sums[c * C + p.i0 + p.o] = sum;
}

// What enters each chunk, in the place of its own end.  G threads to a state, each of
// them AHEAD consecutive chunks at a time: it joins its chunks, the G join theirs in
// LDS, and each runs its chunks again from what enters them.  G = 1 for few chunks
// (18 of 96,256 states 29 us with 16, of which 14 idle); two latencies for 256 chunks
// with G = 16.
constexpr int AHEAD = 16;
template <int G>
__global__ __launch_bounds__(NT) void ssm_join_kernel(SsmArgs a, const float* first, bool reverse) {
  constexpr int STATES = NT / G;
  __shared__ float lds[2][G][G > 1 ? STATES : 1];
  const int64_t C = a.rows * a.cols, S = C * a.n, step = reverse ? -1 : 1;
  const int si = threadIdx.x % STATES, gr = threadIdx.x / STATES;
  for (int64_t i0 = (int64_t)blockIdx.x * STATES; i0 < S; i0 += (int64_t)gridDim.x * STATES) {
    const int64_t i = i0 + si < S ? i0 + si : S - 1, ch = i / a.n;
    const bool ok = i0 + si < S;
    const float A = a.A[ch % a.cols * a.n + (i - ch * a.n)] * LOG2E;
    float v = first ? first[i] : 0.f;
    for (int64_t k0 = 0; k0 < a.chunks; k0 += G * AHEAD) {
      const int64_t k = k0 + gr * AHEAD, c = reverse ? a.chunks - 1 - k : k;  // chunk k of the order
      float own[AHEAD], f[AHEAD];
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) {
        own[e] = 0.f, f[e] = 0.f;
        if (k + e < a.chunks - 1) own[e] = a.state[(c + step * e) * S + i], f[e] = a.sums[(c + step * e) * C + ch];
      }
      float p = 1.f, q = 0.f;
      uint32_t cuts = 0;  // chunks in which a trajectory starts
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) {
        const bool here = k + e < a.chunks - 1 && f[e] == CUT;
        f[e] = k + e < a.chunks - 1 ? __builtin_amdgcn_exp2f(A * f[e]) : 1.f;
        if (here) f[e] = 0.f;
        if (reverse) f[e] = passed(f[e]);
        cuts |= (uint32_t)here << e;
        if constexpr (G > 1) {
          q = here ? own[e] : carried(f[e], q, own[e]);
          p = mul_or_0(p, f[e]);
        }
      }
      float mine = v;
      if constexpr (G > 1) {
        lds[0][gr][si] = cuts ? CUT : p, lds[1][gr][si] = q;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < G; ++e) {
          if (e == gr) mine = v;
          const float pe = lds[0][e][si], qe = lds[1][e][si];
          v = pe == CUT ? qe : carried(pe, v, qe);
        }
        __syncthreads();
      }
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) {
        if (k + e >= a.chunks) break;
        if (ok) a.state[(c + step * e) * S + i] = mine;
        mine = cuts >> e & 1 ? own[e] : carried(f[e], mine, own[e]);
      }
      if constexpr (G == 1) v = mine;
    }
  }
}

constexpr int64_t LAUNCH = 1 << 28;  // groups of one launch (a grid holds less than 2^32 threads)
constexpr int64_t WAVES = 2048;  // waves that a launch wants before it leaves the time axis whole

size_t up(size_t n) { return (n + 255) / 256 * 256; }

template <int TYPE, int PASS>
hipError_t launch_pass(SsmArgs a, int64_t chunks, hipStream_t st) {
  const int64_t groups = a.rows * ((a.cols + 3) / 4);
  const auto go = [&](auto nl) {
    constexpr int NL = nl();
    hipError_t e = hipSuccess;
    for (a.group0 = 0; a.group0 < groups && e == hipSuccess; a.group0 += LAUNCH) {
      const int64_t n = groups - a.group0 < LAUNCH ? groups - a.group0 : LAUNCH;
      const dim3 grid((unsigned)((n * 4 + NT - 1) / NT), (unsigned)chunks);
      // All states there: no run is masked.  100 steps of 4,000 x 64, 16 states, bf16 133 us,
      // 148 as if some were missing, fp32 150 and 177; 32 bf16 222, 245, fp32 278, 234 (the
      // one slower here: over 256 registers, one wave a SIMD); 64 513, 545 and 538, 556; 4
      // 70, 71, 8 91, 95; one step of 1,885 x 128, 16 states, 10.5 and 14.4 with the call.
      if (a.n == 4 * NL) hipLaunchKernelGGL((ssm_kernel<TYPE, NL, true, PASS>), grid, dim3(NT), 0, st, a);
      else hipLaunchKernelGGL((ssm_kernel<TYPE, NL, false, PASS>), grid, dim3(NT), 0, st, a);
      e = hipGetLastError();
    }
    return e;
  };
  if constexpr (PASS == MANY_ROWS) {
    return go(Int<4>());
  } else {
    if (a.n <= 4) return go(Int<1>());
    if (a.n <= 8) return go(Int<2>());
    if (a.n <= 16) return go(Int<4>());
    if (a.n <= 32) return go(Int<8>());
    return go(Int<16>());
  }
}

template <int TYPE>
hipError_t launch_typed(SsmArgs& a, hipStream_t st) {
  if (a.steps == 1) return launch_pass<TYPE, ONE_STEP>(a, 1, st);
  if (a.chunks == 1) {
    const int64_t waves = (a.rows * ((a.cols + 3) / 4) + 15) / 16;
    if (a.n > 8 && a.n <= 16 && waves > WAVES) return launch_pass<TYPE, MANY_ROWS>(a, 1, st);
    return launch_pass<TYPE, WHOLE_AXIS>(a, 1, st);
  }
  hipError_t e = launch_pass<TYPE, LOCAL_ENDS>(a, a.chunks - 1, st);
  if (e == hipSuccess) e = launch_ssm_join(a, a.h0, false, st);
  return e == hipSuccess ? launch_pass<TYPE, FROM_STATES>(a, a.chunks, st) : e;
}

}  // namespace

int64_t ssm_chunk(int64_t steps, int64_t rows, int cols, int64_t want) {
  const int64_t waves = (rows * ((cols + 3) / 4) + 15) / 16, least = 2 * MGN_MARK_STEPS;
  int64_t n = want / (waves > 0 ? waves : 1);
  if (n > steps / least) n = steps / least;
  if (n < 2) return steps;
  const int64_t chunk = (steps + n - 1) / n;
  return (chunk + MGN_MARK_STEPS - 1) / MGN_MARK_STEPS * MGN_MARK_STEPS;
}

hipError_t launch_ssm_join(const SsmArgs& a, const float* first, bool reverse, hipStream_t st) {
  const int64_t n = a.rows * a.cols * a.n, per = a.chunks <= 2 * AHEAD ? NT : NT / 16, b = (n + per - 1) / per;
  const dim3 grid((unsigned)(b < 65536 ? b : 65536));
  if (per == NT) hipLaunchKernelGGL((ssm_join_kernel<1>), grid, dim3(NT), 0, st, a, first, reverse);
  else hipLaunchKernelGGL((ssm_join_kernel<16>), grid, dim3(NT), 0, st, a, first, reverse);
  return hipGetLastError();
}

size_t ssm_work_bytes(int64_t steps, int64_t rows, int cols, int n) {
  if (steps <= 0 || rows <= 0) return 0;
  const int64_t chunk = ssm_chunk(steps, rows, cols, WAVES), chunks = (steps + chunk - 1) / chunk;
  if (chunks < 2) return 0;
  return up(4 * chunks * rows * cols * n) + up(4 * chunks * rows * cols);
}

hipError_t launch_ssm(SsmArgs a, int type, void* work, hipStream_t st) {
  const int64_t C = a.rows * a.cols;
  if (C <= 0) return hipSuccess;
  if (a.steps <= 0)
    return a.h_last && a.h_last != a.h0 ? launch_state_copy(a.h0, a.h_last, C * a.n, st) : hipSuccess;
  a.chunk = ssm_chunk(a.steps, a.rows, a.cols, WAVES);
  a.chunks = (a.steps + a.chunk - 1) / a.chunk;
  a.state = (float*)work;
  a.sums = (float*)((char*)work + up(4 * a.chunks * C * a.n));
  return type == MGN_BF16 ? launch_typed<MGN_BF16>(a, st) : launch_typed<MGN_FP32>(a, st);
}

}  // namespace mgn
