// What the entry points of the state space operators check their arguments with: each returns an error code, and leaves the reason behind.
#pragma once

#include "nugpr_internal.h"

namespace nugpr {

inline int invalid(const std::string& what) {
  set_error(what);
  return NUGPR_ERR_INVALID;
}

// An array of rows, of values of that many bytes.
inline int check_rows(const nugpr_rows* x, const char* name, size_t value) {
  if (!x || !x->data) return invalid(std::string(name) + " is null");
  if (x->row_stride < 0) return invalid(std::string(name) + ": negative stride");
  if (reinterpret_cast<uintptr_t>(x->data) % value) return invalid(std::string(name) + " misaligned");
  return NUGPR_OK;
}

inline bool overlap(const void* a, const void* b, size_t bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x && y && x < y + bytes && y < x + bytes;
}

}  // namespace nugpr

#define NUGPR_TRY(call)                 \
  do {                                  \
    const int c__ = (call);             \
    if (c__ != NUGPR_OK) return c__;    \
  } while (0)
