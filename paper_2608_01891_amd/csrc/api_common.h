// What the files of the C-ABI layer share: the thread's error message and the
// checks that return a status with it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "aflex.h"

namespace aflex {

// Sets this thread's message (aflex_last_error) and returns s.
aflex_status fail(aflex_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
aflex_status hip_status(hipError_t e, const char* who);
aflex_status check_ws(void* ws, size_t have, size_t need, const char* who);
aflex_status check_attn(const aflex_attn_args* a, bool need_out);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace aflex

#define REQUIRE(cond, status, ...) \
  do {                             \
    if (!(cond)) return aflex::fail(status, __VA_ARGS__); \
  } while (0)
