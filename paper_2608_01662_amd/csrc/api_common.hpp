// What the C-ABI front ends share: the thread's error message, argument checks and small arithmetic.
#pragma once
#include "../../include/lsa.h"

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

namespace lsa {

extern thread_local char g_err[512];  // message of the last failing call on this thread (lsa_api.cpp)

inline lsa_status fail(lsa_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}

inline lsa_status hip_fail(hipError_t e, const char* where) {
  return fail(LSA_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool pow2(int64_t x) { return x > 0 && (x & (x - 1)) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace lsa

#define LSA_REQUIRE(cond, st, ...) \
  do {                             \
    if (!(cond)) return lsa::fail(st, __VA_ARGS__); \
  } while (0)
