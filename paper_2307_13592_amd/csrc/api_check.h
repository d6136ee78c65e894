// Argument checks of the C ABI's operators on device arrays.
#pragma once
#include <hip/hip_runtime.h>

#include <initializer_list>
#include <string>

#include "kernels.h"
#include "mgn_internal.h"

namespace mgn {
namespace {

mgn_status bad(const char* fn, const char* what) { return set_error(nullptr, MGN_E_ARG, std::string(fn) + ": " + what); }

mgn_status launched(hipError_t e, const char* fn) {
  if (e == hipSuccess) return MGN_OK;
  return set_error(nullptr, MGN_E_HIP, std::string(fn) + ": " + hipGetErrorString(e));
}

bool float_type(int32_t t) { return t == MGN_FP32 || t == MGN_BF16; }
int64_t type_size(int32_t t) { return t == MGN_FP32 ? 4 : t == MGN_BF16 ? 2 : 1; }
bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
int64_t blocks(int32_t cols) { return (cols + MGN_ROWS8_BLOCK - 1) / MGN_ROWS8_BLOCK; }

// A range of device memory that a call reads (rd) or writes (to).
struct Span {
  const void* p;
  int64_t bytes;
  bool written;
};
bool touch(const Span& a, const Span& b) {
  return a.p && b.p && a.bytes > 0 && b.bytes > 0 && (uintptr_t)a.p < (uintptr_t)b.p + (uintptr_t)b.bytes &&
         (uintptr_t)b.p < (uintptr_t)a.p + (uintptr_t)a.bytes;
}
// Whether a written span overlaps another one.
bool clash(std::initializer_list<Span> spans) {
  for (const Span* a = spans.begin(); a != spans.end(); ++a)
    for (const Span* b = a + 1; b != spans.end(); ++b)
      if ((a->written || b->written) && touch(*a, *b)) return true;
  return false;
}
Span rd(const void* p, int64_t bytes) { return Span{p, bytes, false}; }
Span to(const void* p, int64_t bytes) { return Span{p, bytes, true}; }
// p, unless it is one of the arrays that it may stand on (element for element).
const void* apart(const void* p, std::initializer_list<const void*> same) {
  for (const void* q : same)
    if (p == q) return nullptr;
  return p;
}

constexpr int64_t MAX_ELEMENTS = (int64_t)1 << 46;  // byte offsets stay far from 64 bits

// rows * cols within what the offsets hold
bool size_ok(int64_t n, int64_t cols) { return n >= 0 && n <= MAX_ELEMENTS / cols; }

}  // namespace
}  // namespace mgn
