// Loads held as they lie in memory while other steps run, and the accesses of a lane
// at a 32-bit offset from its wave's address (gfx950).
#pragma once
#include <type_traits>

#include "kernels.h"
#include "rows8.h"

namespace mgn {

template <int N>
using Int = std::integral_constant<int, N>;

__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

// A lane's offset as the compiler finds it here: it is then added by the access
// itself, to a scalar address, and not beforehand to every array's, which would take
// two registers for each of them.
__device__ __forceinline__ uint32_t here(uint32_t o) {
  asm volatile("" : "+v"(o));
  return o;
}
// An element as it lies in memory, of its own width: widened to 32 bits it would be
// waited for where it is loaded, since the compiler widens it there.
template <int TYPE>
using Word = std::conditional_t<TYPE == MGN_BF16, uint16_t, uint32_t>;
// The element at byte `o` from a wave's base: a scalar address and a 32-bit offset.
template <int TYPE>
__device__ __forceinline__ Word<TYPE> raw1(const char* base, uint32_t o) {
  return *(const Word<TYPE>*)(base + here(o));
}
template <int TYPE>
__device__ __forceinline__ float value1(Word<TYPE> w) {
  return __uint_as_float(TYPE == MGN_BF16 ? (uint32_t)w << 16 : (uint32_t)w);
}
template <int TYPE>
__device__ __forceinline__ void write1(char* base, uint32_t o, float v) {
  if constexpr (TYPE == MGN_BF16) *(uint16_t*)(base + here(o)) = (uint16_t)pack_bf16(v, 0.f);
  else *(float*)(base + here(o)) = v;
}
// The starts of trajectories, a bit a step, from the lanes' loads of one step each: 64
// steps at once, those of the next 64 on their way while these are used.
struct Starts {
  const uint8_t* starts;
  int64_t first, end;
  uint64_t bits = 0;
  uint8_t ahead = 0;
  __device__ __forceinline__ Starts(const uint8_t* s, int64_t t0, int64_t t1) : starts(s), first(t0), end(t1) {
    if (starts) look(t0);
  }
  __device__ __forceinline__ void look(int64_t t) {
    t += threadIdx.x & 63;
    ahead = 0;
    if (t < end) ahead = starts[t];
  }
  // Those of steps t .. t + STEPS - 1 in the lowest bits; asked for in order, from t0 on.
  template <int STEPS>
  __device__ __forceinline__ uint32_t at(int64_t t) {
    static_assert(64 % STEPS == 0);
    if (!starts) return 0;
    if ((t - first) % 64 == 0) {
      bits = __builtin_amdgcn_ballot_w64(ahead != 0);
      look(t + 64);
    } else {
      bits >>= STEPS;
    }
    return (uint32_t)bits & ((1u << STEPS) - 1);
  }
};
// NL numbers as they lie in memory, so that a load in flight is not waited for
// before its step comes.  NEAR: neighbours, which are read at once.
template <int TYPE, int NL, bool NEAR>
struct Raw {
  static constexpr int SIZE = sizeof(Elem<TYPE>), WORDS = NEAR ? (NL * SIZE + 3) / 4 : NL;
  std::conditional_t<NEAR, uint32_t, Word<TYPE>> w[WORDS];
  // Those from byte `o` from the base on.
  __device__ __forceinline__ void load(const char* base, uint32_t o) { __builtin_memcpy(w, base + here(o), NL * SIZE); }
  // All numbers at p, past the caches.
  __device__ __forceinline__ void stream(const char* p) {
    if constexpr (WORDS == 2) {
      const uint64_t u = __builtin_nontemporal_load((const uint64_t*)p);
      w[0] = (uint32_t)u, w[1] = (uint32_t)(u >> 32);
    } else {
      static_assert(WORDS == 4);
      const uintx4 u = __builtin_nontemporal_load((const uintx4*)p);
      w[0] = u[0], w[1] = u[1], w[2] = u[2], w[3] = u[3];
    }
  }
  __device__ __forceinline__ void get(float (&v)[NL]) const {
#pragma unroll
    for (int k = 0; k < NL; ++k) {
      if constexpr (!NEAR || TYPE != MGN_BF16) v[k] = value1<TYPE>((Word<TYPE>)w[k]);
      else v[k] = __uint_as_float(k % 2 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
    }
  }
};

}  // namespace mgn
