// What the C ABI's argument checks are written with: a failing one returns its status and leaves a message.
#pragma once
#include "common.h"

#define MB_REQUIRE(cond, code, ...) \
  do {                              \
    if (!(cond)) return ::mb::fail(code, __VA_ARGS__); \
  } while (0)

namespace mb {
inline mb_status check_ptr(const void* p, const char* name) {
  MB_REQUIRE(p != nullptr, MB_ERR_INVALID_ARG, "%s is NULL", name);
  MB_REQUIRE(aligned16(p), MB_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return MB_OK;
}
}  // namespace mb

#define MB_CHECK_PTR(p)                              \
  do {                                               \
    const mb_status st_ = ::mb::check_ptr((p), #p);  \
    if (st_ != MB_OK) return st_;                    \
  } while (0)
