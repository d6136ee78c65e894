// Gated linear recurrence over the time steps of a trajectory (gfx950):
//   f = sigmoid(g), z = 1 - f = sigmoid(-g),  h_t = f_t h_{t-1} + z_t x_t,
// every column of every node row on its own, and its backward pass
//   D_t = dh_t + c_t,  c_{t-1} = f_t D_t  (c_{T-1} = dh_last; 0 before a start)
//   dx = z D,  dg = f z (h_{t-1} - x) D,  dh0 = c_{-1}.
// Both are y <- p y + q per step (the backward in reversed time), so steps join:
// (p2, q2) after (p1, q1) is (p1 p2, p2 q1 + q2).
//
// A lane holds V neighbouring columns of the flattened [rows][cols] and a wave
// SEG steps of them in registers: all its loads are in flight together, each
// element is read once.  With many columns a wave goes through the whole time
// axis alone (W = 1).  With fewer, W waves of a workgroup take consecutive
// segments of the same columns, join their (p, q) in LDS (one barrier a tile of
// W SEG steps) and each runs its own steps from the state that enters it.  With
// too few columns for that to fill the card the time axis is cut into chunks of
// whole tiles: a first launch leaves each chunk's (p, q) in the scratch, a second
// one joins those before its chunk and runs as above.  The operands are then
// read twice (mostly from the caches: such arrays are small), but no workgroup
// waits for another.
//
// Bound by HBM with many columns: 16 steps of 250,000 x 128 bf16 734 - 760 us
// (5.7 TB/s), 20 of 100,003 x 64 backward from an 8-bit history 347 us (5.6), 600
// of 1,885 x 128 fp32 backward 664 us (5.2; 943 waves).  With few by the launches
// and a load's latency in each of them: 8,192 steps of 192 columns 15 us, backward
// 19.  Loading a wave's next segment ahead of the join was slower (registers:
// 400 steps of 10,240 columns backward 26 -> 36 us).
#include "kernels.h"
#include "rows8.h"

namespace mgn {
namespace {

// f and z of a gate logit: e = exp(-|g|), 1 / (1 + e) and e / (1 + e).  The
// exponent's product rounds once, so that the small weight is off by about |g|
// half-steps of itself (less than 90: no smaller weight is left), and the large
// one by a few; a more exact exponential would move a term that weighs e^-|g| of
// the others.  A weight below the smallest normal number is 0, and a term with a
// weight of 0 is left out whatever it multiplies.
__device__ __forceinline__ void gates(float g, float& f, float& z) {
  const float e = __expf(-fabsf(g));
  const float big = __builtin_amdgcn_rcpf(1.f + e);
  float small = e * big;
  small = small < 1.17549435e-38f ? 0.f : small;
  f = g < 0.f ? small : big;
  z = g < 0.f ? big : small;
}

__device__ __forceinline__ float term(float weight, float v) { return weight == 0.f ? 0.f : weight * v; }
// The factor p of a stretch of time: 0 where one of its gates is (cut), and
// nowhere else: a product that passes below fp32 stays at the smallest number,
// 2^-149, so that a NaN or infinite state lasts as it does step by step (a finite
// one y is then off by at most 2^-149 |y|, as by that number's rounding).  A NaN
// gate needs no trace in p: the stretch's q is NaN from it to the next cut.
constexpr float LEAST = 1.40129846e-45f;
__device__ __forceinline__ float factor(float p, bool cut) { return cut ? 0.f : fmaxf(p, LEAST); }
// That of two joined stretches.
__device__ __forceinline__ float joined(float p, float f) { return f == 0.f ? 0.f : fmaxf(p * f, fminf(p, LEAST)); }
// p y + q, without y where p is 0
__device__ __forceinline__ float step(float p, float y, float q) { return p == 0.f ? q : fmaf(p, y, q); }

// V neighbouring elements from element b + o on: b is the same for the whole
// wave (an address in scalar registers), o the lane's 32-bit offset.  PAST: past
// the caches.
template <bool PAST, class U>
__device__ __forceinline__ U read(const void* p) {
  if constexpr (PAST) return __builtin_nontemporal_load((const U*)p);
  else return *(const U*)p;
}
template <int T, int V, bool PAST = false>
__device__ __forceinline__ void loadv(const void* p, int64_t b, uint32_t o, float (&v)[V]) {
  if constexpr (T == MGN_BF16) {
    const uint16_t* r = (const uint16_t*)p + b;
    if constexpr (V == 4) {
      const uint64_t w = read<PAST, uint64_t>(r + o);
      const uint2 u{(uint32_t)w, (uint32_t)(w >> 32)};
      v[0] = __uint_as_float(u.x << 16);
      v[1] = __uint_as_float(u.x & 0xffff0000u);
      v[2] = __uint_as_float(u.y << 16);
      v[3] = __uint_as_float(u.y & 0xffff0000u);
    } else {
      v[0] = bf2f(r[o]);
    }
  } else {
    const float* r = (const float*)p + b;
    if constexpr (V == 4) {
      const floatx4 u = read<PAST, floatx4>(r + o);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = u[k];
    } else {
      v[0] = r[o];
    }
  }
}
template <int T, int V>
__device__ __forceinline__ void storev(void* p, int64_t b, uint32_t o, const float (&v)[V]) {
  if constexpr (T == MGN_BF16) {
    uint16_t* r = (uint16_t*)p + b;
    if constexpr (V == 4)
      __builtin_nontemporal_store((uint64_t)pack_bf16(v[0], v[1]) | (uint64_t)pack_bf16(v[2], v[3]) << 32,
                                  reinterpret_cast<uint64_t*>(r + o));
    else
      r[o] = (uint16_t)pack_bf16(v[0], 0.f);
  } else {
    float* r = (float*)p + b;
    if constexpr (V == 4) __builtin_nontemporal_store(floatx4{v[0], v[1], v[2], v[3]}, reinterpret_cast<floatx4*>(r + o));
    else r[o] = v[0];
  }
}

// Where a lane's columns lie (i + o, i the same for its wave), and its view of x.
template <int V, int TX, bool PAST>
struct Lane {
  int64_t i, C, s0, scn;  // 8-bit x: scale of column i, scales of a step
  uint32_t o, so;
  bool ok;
  __device__ __forceinline__ Lane(const ScanArgs& a, int64_t tile) {
    C = a.rows * a.cols;
    i = tile * 64 * V;
    o = (threadIdx.x & 63) * V;
    ok = i + o < C;
    if constexpr (TX == MGN_E4M3) {
      const int nb = rows8_blocks(a.cols);
      const int64_t row = i / a.cols;
      const uint32_t c = (uint32_t)(i - row * a.cols) + o, down = c / (uint32_t)a.cols;
      s0 = row * nb;
      so = down * nb + (c - down * (uint32_t)a.cols) / ROWS8_BLOCK;
      scn = a.rows * nb;
    }
  }
  __device__ __forceinline__ void x(const ScanArgs& a, int64_t t, float (&v)[V]) const {
    if constexpr (TX == MGN_E4M3) {
      const uint8_t* q = (const uint8_t*)a.x + (t * C + i);
      const float* s = a.x_scale + (t * scn + s0);
      float u[4];
      uint32_t codes;
      if constexpr (V == 4) codes = read<PAST, uint32_t>(q + o);
      else codes = q[o];
      values8(codes, s[so], u);
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = u[k];
    } else {
      loadv<TX, V, PAST>(a.x, t * C + i, o, v);
    }
  }
};

// The waves' joined steps in LDS: [parity][wave][p, q][lane][V].
template <int W, int V>
struct Joint {
  float v[2][W][2][64][V];
};

// y at the start of the chunk `c`: entries 0 .. c of the scratch joined in
// order, the waves taking shares of them.
template <int W, int V>
__device__ __forceinline__ void chunk_entry(const ScanArgs& a, int c, int64_t i, uint32_t o, int64_t C, bool ok, int w,
                                            Joint<W, V>& lds, float (&y)[V]) {
  const float* wp = (const float*)a.work;
  const int lane = threadIdx.x & 63, n = c + 1, e0 = n * w / W, e1 = n * (w + 1) / W;
  float p[V], q[V];
#pragma unroll
  for (int k = 0; k < V; ++k) p[k] = 1.f, q[k] = 0.f;
  if (ok)
#pragma unroll 4
    for (int e = e0; e < e1; ++e) {
      float pe[V], qe[V];
      loadv<MGN_FP32, V>(wp, (2 * (int64_t)e) * C + i, o, pe);
      loadv<MGN_FP32, V>(wp, (2 * (int64_t)e + 1) * C + i, o, qe);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        q[k] = step(pe[k], q[k], qe[k]);
        p[k] = joined(p[k], pe[k]);
      }
    }
#pragma unroll
  for (int k = 0; k < V; ++k) lds.v[0][w][0][lane][k] = p[k], lds.v[0][w][1][lane][k] = q[k], y[k] = 0.f;
  __syncthreads();
  for (int e = 0; e < W; ++e)
#pragma unroll
    for (int k = 0; k < V; ++k) y[k] = step(lds.v[0][e][0][lane][k], y[k], lds.v[0][e][1][lane][k]);
  __syncthreads();
}

// Joins a tile's segments: p, q are the wave's own; y becomes the state that
// enters the wave's segment, `end` the one that leaves the tile.
template <int W, int V>
__device__ __forceinline__ void join(Joint<W, V>& lds, int par, int w, const float (&p)[V], const float (&q)[V],
                                     float (&y)[V], float (&end)[V]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < V; ++k) lds.v[par][w][0][lane][k] = p[k], lds.v[par][w][1][lane][k] = q[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < V; ++k) end[k] = y[k];
#pragma unroll
  for (int e = 0; e < W; ++e) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (e == w) y[k] = end[k];
      end[k] = step(lds.v[par][e][0][lane][k], end[k], lds.v[par][e][1][lane][k]);
    }
  }
}

// Chunks of the time axis: 8 waves, one column a lane (few columns).
template <int W, int V>
__device__ __forceinline__ bool chunked() {
  return W == 8 && V == 1 && gridDim.y > 1;
}

constexpr int threads(int W) { return W == 1 ? 256 : 64 * W; }

// FIRST: the first launch of a chunked scan, (p, q) of the chunk blockIdx.y
// into entry blockIdx.y + 1 (and, with the first chunk, the state that enters
// the scan into entry 0).
template <int W, int V, int SEG, int TG, int TX, bool FIRST, bool PAST>
__global__ __launch_bounds__(threads(W)) void scan_kernel(ScanArgs a) {
  __shared__ Joint<W, W == 1 ? 1 : V> lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = W == 1 ? 0 : wave;
  const Lane<V, TX, PAST> l(a, a.tile0 + (W == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x));
  const int64_t C = l.C, i = l.i;
  const int c = blockIdx.y;
  const int64_t ts = c * a.chunk, te = ts + a.chunk < a.steps ? ts + a.chunk : a.steps;
  float y[V], pt[V];
#pragma unroll
  for (int k = 0; k < V; ++k) y[k] = 0.f, pt[k] = 1.f;
  if constexpr (FIRST) {
    if (c == 0 && w == 0 && l.ok) {
      float h0[V];
#pragma unroll
      for (int k = 0; k < V; ++k) h0[k] = 0.f;
      if (a.h0) loadv<MGN_FP32, V>(a.h0, i, l.o, h0);
      storev<MGN_FP32, V>(a.work, i, l.o, y);
      storev<MGN_FP32, V>(a.work, C + i, l.o, h0);
    }
  } else if (chunked<W, V>()) {
    if constexpr (W > 1) chunk_entry<W, V>(a, c, i, l.o, C, l.ok, w, lds, y);
  } else if (a.h0 && l.ok && w == 0) {
    loadv<MGN_FP32, V>(a.h0, i, l.o, y);
  }
  int par = 0;
  for (int64_t t = ts; t < te; t += W * SEG, par ^= 1) {
    const int64_t t0 = t + w * SEG;
    float f[SEG][V], q[SEG][V];
#pragma unroll
    for (int s = 0; s < SEG; ++s) {
#pragma unroll
      for (int k = 0; k < V; ++k) f[s][k] = INFINITY, q[s][k] = 0.f;
      if (l.ok && t0 + s < te) {
        loadv<TG, V, PAST>(a.g, (t0 + s) * C + i, l.o, f[s]);
        l.x(a, t0 + s, q[s]);
      }
    }
    // the first segment starts from the state itself (p = 0), so that only its
    // wave reads that array, which another wave's last step may write
    const bool head = !FIRST && w == 0 && t == ts && !chunked<W, V>();
    float p[V], r[V];
    bool cut[V];
#pragma unroll
    for (int k = 0; k < V; ++k) p[k] = 1.f, cut[k] = head, r[k] = head ? y[k] : 0.f;
#pragma unroll
    for (int s = 0; s < SEG; ++s) {
      const bool fresh = a.starts && t0 + s < te && a.starts[t0 + s];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float z;
        gates(f[s][k], f[s][k], z);
        q[s][k] = term(z, q[s][k]);
        if (fresh) f[s][k] = 0.f;
        if constexpr (W > 1 || FIRST) {
          r[k] = step(f[s][k], r[k], q[s][k]);
          p[k] *= f[s][k];
          cut[k] = cut[k] || f[s][k] == 0.f;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) p[k] = factor(p[k], cut[k]);
    float end[V];
    if constexpr (W > 1) join<W, V>(lds, par, w, p, r, y, end);
    if constexpr (FIRST) {
#pragma unroll
      for (int e = 0; e < W; ++e)
#pragma unroll
        for (int k = 0; k < V; ++k) pt[k] = joined(pt[k], lds.v[par][e][0][threadIdx.x & 63][k]);
    } else {
#pragma unroll
      for (int s = 0; s < SEG; ++s) {
        if (t0 + s < te) {
#pragma unroll
          for (int k = 0; k < V; ++k) y[k] = step(f[s][k], y[k], q[s][k]);
          if (a.h && l.ok) storev<MGN_FP32, V>(a.h, (t0 + s) * C + i, l.o, y);
          if (t0 + s == a.steps - 1 && a.h_last && l.ok) storev<MGN_FP32, V>(a.h_last, i, l.o, y);
        }
      }
    }
    if constexpr (W > 1) {
#pragma unroll
      for (int k = 0; k < V; ++k) y[k] = end[k];
    }
  }
  if constexpr (FIRST) {
    if (w == 0 && l.ok) {
      storev<MGN_FP32, V>(a.work, (2 * (int64_t)(c + 1)) * C + i, l.o, pt);
      storev<MGN_FP32, V>(a.work, (2 * (int64_t)(c + 1) + 1) * C + i, l.o, y);
    }
  }
}

// The same in reversed time: a wave's step s is time te - 1 - (its position).
template <int W, int V, int SEG, int TG, int TX, bool FIRST, bool PAST>
__global__ __launch_bounds__(threads(W)) void scan_grad_kernel(ScanArgs a) {
  constexpr int TD = TX == MGN_E4M3 ? TG : TX;
  __shared__ Joint<W, W == 1 ? 1 : V> lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = W == 1 ? 0 : wave;
  const Lane<V, TX, PAST> l(a, a.tile0 + (W == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x));
  const int64_t C = l.C, i = l.i;
  const int c = blockIdx.y;
  // reversed steps u = steps - 1 - t of this chunk
  const int64_t us = c * a.chunk, ue = us + a.chunk < a.steps ? us + a.chunk : a.steps;
  float y[V], pt[V];
#pragma unroll
  for (int k = 0; k < V; ++k) y[k] = 0.f, pt[k] = 1.f;
  if constexpr (FIRST) {
    if (c == 0 && w == 0 && l.ok) {
      float d[V];
#pragma unroll
      for (int k = 0; k < V; ++k) d[k] = 0.f;
      if (a.dh_last) loadv<MGN_FP32, V>(a.dh_last, i, l.o, d);
      storev<MGN_FP32, V>(a.work, i, l.o, y);
      storev<MGN_FP32, V>(a.work, C + i, l.o, d);
    }
  } else if (chunked<W, V>()) {
    if constexpr (W > 1) chunk_entry<W, V>(a, c, i, l.o, C, l.ok, w, lds, y);
  } else if (a.dh_last && l.ok && w == 0) {
    loadv<MGN_FP32, V>(a.dh_last, i, l.o, y);
  }
  int par = 0;
  for (int64_t u = us; u < ue; u += W * SEG, par ^= 1) {
    const int64_t u0 = u + w * SEG;
    float f[SEG][V], d[SEG][V], z[FIRST ? 1 : SEG][V], m[FIRST ? 1 : SEG][V];
#pragma unroll
    for (int s = 0; s < SEG; ++s) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        f[s][k] = INFINITY, d[s][k] = 0.f;
        if constexpr (!FIRST) z[s][k] = 0.f, m[s][k] = 0.f;
      }
      if (l.ok && u0 + s < ue) {
        const int64_t t = a.steps - 1 - (u0 + s);
        loadv<TG, V, PAST>(a.g, t * C + i, l.o, f[s]);
        if (a.dh) loadv<MGN_FP32, V, PAST>(a.dh, t * C + i, l.o, d[s]);
        if constexpr (!FIRST) {
          l.x(a, t, z[s]);
          if (t > 0) loadv<MGN_FP32, V, PAST>(a.h, (t - 1) * C + i, l.o, m[s]);
          else if (a.h0) loadv<MGN_FP32, V>(a.h0, i, l.o, m[s]);
        }
      }
    }
    // the first segment starts from the state itself (p = 0), so that only its
    // wave reads that array, which another wave's last step may write
    const bool head = !FIRST && w == 0 && u == us && !chunked<W, V>();
    float p[V], r[V];
    bool cut[V];
#pragma unroll
    for (int k = 0; k < V; ++k) p[k] = 1.f, cut[k] = head, r[k] = head ? y[k] : 0.f;
#pragma unroll
    for (int s = 0; s < SEG; ++s) {
      const bool fresh = a.starts && u0 + s < ue && a.starts[a.steps - 1 - (u0 + s)];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float zz;
        gates(f[s][k], f[s][k], zz);
        if constexpr (!FIRST) {
          // m: f z (h_{t-1} - x), what dg takes of D, -0 where f or z is 0 and
          // the term left out; z: what dx takes
          const float fz = f[s][k] * zz;
          m[s][k] = fz == 0.f ? -0.f : fmaf(fz, (fresh ? 0.f : m[s][k]) - z[s][k], 0.f);
          z[s][k] = zz;
        }
        if (fresh) f[s][k] = 0.f;
        if constexpr (W > 1 || FIRST) {
          r[k] = term(f[s][k], r[k] + d[s][k]);
          p[k] *= f[s][k];
          cut[k] = cut[k] || f[s][k] == 0.f;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) p[k] = factor(p[k], cut[k]);
    float end[V];
    if constexpr (W > 1) join<W, V>(lds, par, w, p, r, y, end);
    if constexpr (FIRST) {
#pragma unroll
      for (int e = 0; e < W; ++e)
#pragma unroll
        for (int k = 0; k < V; ++k) pt[k] = joined(pt[k], lds.v[par][e][0][threadIdx.x & 63][k]);
    } else {
#pragma unroll
      for (int s = 0; s < SEG; ++s) {
        if (u0 + s < ue) {
          const int64_t t = a.steps - 1 - (u0 + s);
          float dx[V], dg[V];
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const float D = d[s][k] + y[k];
            dx[k] = term(z[s][k], D);
            dg[k] = __float_as_uint(m[s][k]) == 0x80000000u ? 0.f : m[s][k] * D;
            y[k] = term(f[s][k], D);
          }
          if (l.ok) {
            storev<TD, V>(a.dx, t * C + i, l.o, dx);
            storev<TG, V>(a.dg, t * C + i, l.o, dg);
            if (t == 0 && a.dh0) storev<MGN_FP32, V>(a.dh0, i, l.o, y);
          }
        }
      }
    }
    if constexpr (W > 1) {
#pragma unroll
      for (int k = 0; k < V; ++k) y[k] = end[k];
    }
  }
  if constexpr (FIRST) {
    if (w == 0 && l.ok) {
      storev<MGN_FP32, V>(a.work, (2 * (int64_t)(c + 1)) * C + i, l.o, pt);
      storev<MGN_FP32, V>(a.work, (2 * (int64_t)(c + 1) + 1) * C + i, l.o, y);
    }
  }
}

// out = in (or zeros): a scan of no steps.
__global__ __launch_bounds__(256) void state_copy_kernel(const float* in, float* out, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) out[i] = in ? in[i] : 0.f;
}

hipError_t copy_state(const float* in, float* out, int64_t n, hipStream_t st) {
  const int64_t b = (n + 255) / 256;
  hipLaunchKernelGGL(state_copy_kernel, dim3((unsigned)(b < 8192 ? b : 8192)), dim3(256), 0, st, in, out, n);
  return hipGetLastError();
}

constexpr int SEG4 = 4, SEG1 = 8;    // steps a wave holds with 4 columns a lane, with 1
constexpr int64_t VEC_COLS = 65536;  // columns from which a lane takes four of them
constexpr int64_t ALONE4 = 800, ALONE1 = 2048;  // waves from which one goes through the time axis alone
constexpr int64_t FEW = 256;         // waves below which the time axis is cut into chunks
constexpr int64_t LAUNCH = 1 << 20;  // tiles of one launch (a grid holds less than 2^32 threads)
constexpr int64_t CHUNK_WGS = 512;   // workgroups of a chunked scan, at most about

// How a scan is dealt, by its columns C and steps (vec: the arrays allow four
// columns a lane), from device times of the scan / its backward in fp32, us:
//   four columns a lane or one: 16 x 250,000 x 128 (bf16) 734 / 1529 and 1425 /
//     1798, C = 38,400 x 200 steps 35 / 52 and 23 / 40;
//   a wave alone or four along time, four columns a lane: C = 241,280 x 600 steps
//     312 / 673 and 345 / 700, C = 128,000 x 64 steps 29 / 47 and 18 / 33;
//   four or eight, one column a lane: C = 40,960 x 400 steps 39 / 92 and 38 / 94,
//     C = 20,480 x 400 steps 32 / 57 and 26 / 53;
//   eight, or chunks: C = 20,480 x 400 steps 26 / 53 and 33 / 54, C = 10,240 x
//     2,000 steps 85 / 157 and 67 / 123, C = 192 x 8,000 steps 299 / 539 and 15 / 19.
// A wave takes all steps at once where they fit its segment.
struct Deal {
  int V, W;
  int64_t tiles, chunk, chunks;
};
Deal deal(int64_t steps, int64_t C, bool vec) {
  Deal d{};
  d.V = vec && C >= VEC_COLS ? 4 : 1;
  const int seg = d.V == 4 ? SEG4 : SEG1;
  d.tiles = (C + 64 * d.V - 1) / (64 * d.V);
  if (steps <= seg || d.tiles >= (d.V == 4 ? ALONE4 : ALONE1)) d.W = 1;
  else d.W = d.V == 4 || steps <= 4 * seg || d.tiles >= ALONE1 / 4 ? 4 : 8;
  d.chunk = steps;
  d.chunks = 1;
  const int64_t tile = (int64_t)d.W * seg;
  if (d.W == 8 && d.tiles < FEW && steps >= 2 * tile) {
    const int64_t want = (CHUNK_WGS + d.tiles - 1) / d.tiles, most = (steps + tile - 1) / tile;
    const int64_t n = want < most ? want : most;
    d.chunk = ((steps + n - 1) / n + tile - 1) / tile * tile;
    d.chunks = (steps + d.chunk - 1) / d.chunk;
  }
  return d;
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

// Calls f(W, V) as constants.
template <class F>
hipError_t by_deal(const Deal& d, F f) {
  using std::integral_constant;
  const integral_constant<int, 1> one;
  const integral_constant<int, 4> four;
  if (d.V == 4) return d.W == 1 ? f(one, four) : f(four, four);
  return d.W == 1 ? f(one, one) : d.W == 4 ? f(four, one) : f(integral_constant<int, 8>(), one);
}

bool at(const void* p, int bytes) { return (uintptr_t)p % bytes == 0; }
int bytes(int type) { return type == MGN_FP32 ? 4 : type == MGN_BF16 ? 2 : 1; }
int quad(int type) { return 4 * bytes(type); }
// A scan of four columns a lane that moves more than the last-level cache holds
// reads past it: 16 steps of 250,000 x 128 bf16 744 us through it, 728 past it, its
// backward 1558 and 1507; below, 20 steps of 5,000 x 64 bf16 19 and 27 us, its
// backward 25 and 33, both in turn on 16 x 10,000 x 128 fp32 115 and 136.  It
// writes past it at any size (16 x 10,000 x 128 fp32, both in turn: 119 us, 125
// otherwise; 20 x 5,000 x 64 bf16 46 and 42).
constexpr int64_t CACHE = (int64_t)256 << 20;

}  // namespace

hipError_t launch_state_copy(const float* in, float* out, int64_t n, hipStream_t st) { return copy_state(in, out, n, st); }

size_t scan_work_bytes(int64_t steps, int64_t rows, int cols) {
  const int64_t C = rows * cols;
  if (steps <= 0 || C <= 0) return 0;
  const Deal d = deal(steps, C, false);  // chunks come with one column a lane
  return d.chunks > 1 ? (size_t)(2 * d.chunks * C) * 4 : 0;
}

hipError_t launch_scan(ScanArgs a, int g_type, int x_type, hipStream_t st) {
  const int64_t C = a.rows * a.cols;
  if (C <= 0) return hipSuccess;
  if (a.steps <= 0) return a.h_last ? copy_state(a.h0, a.h_last, C, st) : hipSuccess;
  const bool vec = (x_type == MGN_E4M3 ? a.cols : C) % 4 == 0 && at(a.g, quad(g_type)) && at(a.x, quad(x_type)) &&
                   at(a.h0, 16) && at(a.h, 16) && at(a.h_last, 16);
  const Deal d = deal(a.steps, C, vec);
  const bool past = a.steps * C * (bytes(g_type) + bytes(x_type) + (a.h ? 4 : 0)) > CACHE;
  a.chunk = d.chunk;
  return by_types(g_type, x_type, [&](auto tg, auto tx) {
    return by_deal(d, [&](auto w, auto v) {
      constexpr int W = w(), V = v(), SEG = V == 4 ? SEG4 : SEG1;
      const dim3 block(threads(W));
      hipError_t e = hipSuccess;
      for (a.tile0 = 0; a.tile0 < d.tiles && e == hipSuccess; a.tile0 += LAUNCH) {
        const int64_t n = d.tiles - a.tile0 < LAUNCH ? d.tiles - a.tile0 : LAUNCH;
        const unsigned gx = (unsigned)(W == 1 ? (n + 3) / 4 : n);
        if constexpr (W == 8 && V == 1) {
          if (d.chunks > 1) {
            hipLaunchKernelGGL((scan_kernel<W, V, SEG, tg(), tx(), true, false>), dim3(gx, (unsigned)d.chunks - 1), block, 0, st, a);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
          }
        }
        const dim3 grid(gx, (unsigned)d.chunks);
        if constexpr (V == 4) {
          if (past)
            hipLaunchKernelGGL((scan_kernel<W, V, SEG, tg(), tx(), false, true>), grid, block, 0, st, a);
          else
            hipLaunchKernelGGL((scan_kernel<W, V, SEG, tg(), tx(), false, false>), grid, block, 0, st, a);
        } else {
          hipLaunchKernelGGL((scan_kernel<W, V, SEG, tg(), tx(), false, false>), grid, block, 0, st, a);
        }
        e = hipGetLastError();
      }
      return e;
    });
  });
}

hipError_t launch_scan_grad(ScanArgs a, int g_type, int x_type, hipStream_t st) {
  const int64_t C = a.rows * a.cols;
  if (C <= 0) return hipSuccess;
  if (a.steps <= 0) return a.dh0 ? copy_state(a.dh_last, a.dh0, C, st) : hipSuccess;
  const int d_type = x_type == MGN_E4M3 ? g_type : x_type;
  const bool vec = (x_type == MGN_E4M3 ? a.cols : C) % 4 == 0 && at(a.g, quad(g_type)) && at(a.x, quad(x_type)) &&
                   at(a.h0, 16) && at(a.h, 16) && at(a.dh, 16) && at(a.dh_last, 16) && at(a.dg, quad(g_type)) &&
                   at(a.dx, quad(d_type)) && at(a.dh0, 16);
  const Deal d = deal(a.steps, C, vec);
  const bool past = a.steps * C * (bytes(g_type) + bytes(x_type) + bytes(g_type) + bytes(d_type) + (a.dh ? 8 : 4)) > CACHE;
  a.chunk = d.chunk;
  return by_types(g_type, x_type, [&](auto tg, auto tx) {
    return by_deal(d, [&](auto w, auto v) {
      constexpr int W = w(), V = v(), SEG = V == 4 ? SEG4 : SEG1;
      const dim3 block(threads(W));
      hipError_t e = hipSuccess;
      for (a.tile0 = 0; a.tile0 < d.tiles && e == hipSuccess; a.tile0 += LAUNCH) {
        const int64_t n = d.tiles - a.tile0 < LAUNCH ? d.tiles - a.tile0 : LAUNCH;
        const unsigned gx = (unsigned)(W == 1 ? (n + 3) / 4 : n);
        if constexpr (W == 8 && V == 1) {
          if (d.chunks > 1) {
            hipLaunchKernelGGL((scan_grad_kernel<W, V, SEG, tg(), tx(), true, false>), dim3(gx, (unsigned)d.chunks - 1), block, 0, st, a);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
          }
        }
        const dim3 grid(gx, (unsigned)d.chunks);
        if constexpr (V == 4) {
          if (past)
            hipLaunchKernelGGL((scan_grad_kernel<W, V, SEG, tg(), tx(), false, true>), grid, block, 0, st, a);
          else
            hipLaunchKernelGGL((scan_grad_kernel<W, V, SEG, tg(), tx(), false, false>), grid, block, 0, st, a);
        } else {
          hipLaunchKernelGGL((scan_grad_kernel<W, V, SEG, tg(), tx(), false, false>), grid, block, 0, st, a);
        }
        e = hipGetLastError();
      }
      return e;
    });
  });
}

}  // namespace mgn
