// Host-side argument checks shared by the entry points: the thread's error
// message, the status helpers and the REQUIRE / SUPPORT / ALIGNED checks.
#pragma once

#include <cstdarg>
#include <cstdio>
#include <string>

#include "dmoe_common.h"

namespace dmoe {
namespace host {

inline thread_local std::string g_last_error;

inline dmoe_status fail(dmoe_status st, const char* fn, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_last_error = std::string(fn) + ": " + buf;
  return st;
}

inline dmoe_status ok() {
  g_last_error.clear();
  return DMOE_OK;
}

inline dmoe_status hip_status(hipError_t err, const char* fn) {
  if (err == hipSuccess) return ok();
  return fail(DMOE_ERR_HIP, fn, "kernel launch failed: %s", hipGetErrorString(err));
}

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline bool valid_dtype(dmoe_dtype dt) { return dt == DMOE_F32 || dt == DMOE_BF16; }

constexpr long kIntLimit = 0x7fffffffL;

// Name of the entry point in error messages.
#define DMOE_FN __func__
#define REQUIRE(cond, ...)                                  \
  do {                                                      \
    if (!(cond)) return fail(DMOE_ERR_INVALID_ARG, DMOE_FN, __VA_ARGS__); \
  } while (0)
#define SUPPORT(cond, ...)                                  \
  do {                                                      \
    if (!(cond)) return fail(DMOE_ERR_UNSUPPORTED, DMOE_FN, __VA_ARGS__); \
  } while (0)
#define ALIGNED(p) REQUIRE(!misaligned(p), #p " is not 16-byte aligned")

}  // namespace host
}  // namespace dmoe
