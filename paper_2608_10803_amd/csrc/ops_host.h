// Shared by the files of C entry points of the operators beside the products:
// statuses, argument checks, pieces of a workspace.
#pragma once
#include <algorithm>
#include <memory>
#include <mutex>
#include <new>
#include <string>

#include "ops.h"

namespace ac {
namespace host {

// No exception leaves a C entry point.
template <class F>
adaptcore_status guarded(F f) noexcept {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return AC_ERR_OUT_OF_MEMORY;
  } catch (...) {
    return AC_ERR_INTERNAL;
  }
}

inline adaptcore_status launched(hipError_t e, int n) {
  if (e != hipSuccess)
    return ac::op_fail(AC_ERR_LAUNCH, std::string("kernel launch failed: ") + hipGetErrorString(e));
  ac::op_count_launches(n);
  return AC_OK;
}

inline adaptcore_status invalid(const char* msg) { return ac::op_fail(AC_ERR_INVALID_VALUE, msg); }
inline adaptcore_status unsupported(const char* msg) { return ac::op_fail(AC_ERR_UNSUPPORTED, msg); }

inline int type_bytes(int32_t t) { return t == AC_TYPE_F32 ? 4 : 2; }
inline bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Hands out pieces of a workspace (256-byte aligned); without a base it only
// counts.
struct Scratch {
  char* base = nullptr;
  int64_t used = 0;
  template <class T>
  T* take(int64_t n) {
    char* p = base ? base + used : nullptr;
    used += (n * (int64_t)sizeof(T) + 255) / 256 * 256;
    return reinterpret_cast<T*>(p);
  }
};

inline adaptcore_status first_bad(std::initializer_list<adaptcore_status> all) {
  for (adaptcore_status s : all)
    if (s != AC_OK) return s;
  return AC_OK;
}

// Runs f twice: counting the workspace, then on it.
template <class F>
adaptcore_status with_scratch(hipStream_t st, F f) {
  Scratch s;
  int n = 0;
  adaptcore_status rc = f(&s, &n);
  if (rc != AC_OK) return rc;
  char none[1];
  s.base = none;  // (no workspace needed: any address, nothing is taken from it)
  std::unique_lock<std::mutex> hold;
  if (s.used > 0) rc = ac::op_workspace(st, s.used, &s.base, &hold);
  if (rc != AC_OK) return rc;
  s.used = 0;
  n = 0;
  rc = f(&s, &n);
  if (rc == AC_OK) ac::op_count_launches(n);
  return rc;
}

}  // namespace host
}  // namespace ac
