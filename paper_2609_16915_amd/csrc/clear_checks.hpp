// What the clear side's entry points (clear_abi.cpp, decode_abi.cpp) check their
// arguments with, before anything is enqueued.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "internal.hpp"

namespace rosetta {

constexpr size_t MAX_STRIDE = (size_t)1 << 32;

inline rosetta_status fail(rosetta_status st, const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_last_error(buf);
  return st;
}

inline rosetta_status done(hipError_t e, const char *what) {
  if (e == hipSuccess) {
    set_last_error("");
    return ROSETTA_OK;
  }
  (void)hipGetLastError();
  if (e == hipErrorOutOfMemory)
    return fail(ROSETTA_ERR_NOMEM, "%s: %s", what, hipGetErrorString(e));
  if (e == hipErrorInvalidConfiguration)
    return fail(ROSETTA_ERR_UNSUPPORTED, "%s: sizes that one launch does not hold", what);
  return fail(ROSETTA_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

inline bool is_type(int t) { return t == ROSETTA_F32 || t == ROSETTA_BF16 || t == ROSETTA_F16; }

// A named device array: rows of `len` elements of `elem` bytes, `stride` apart.
struct Array {
  const char *name;
  const void *p;
  size_t rows, len, stride, elem;
  bool out;
  // (past 64 bits where a caller's sizes are: 2^31 rows 2^32 elements apart)
  unsigned __int128 bytes() const {
    return rows && len ? ((unsigned __int128)(rows - 1) * stride + len) * elem : 0;
  }
};

// Whether two arrays share memory: by the whole ranges, or, rows as far apart in both
// (columns of one buffer), by where the second's rows lie between the first's.
inline bool overlap(const Array &a, const Array &b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  if (!(x < y + b.bytes() && y < x + a.bytes())) return false;
  const size_t pitch = a.stride * a.elem;
  if (a.rows < 2 || b.rows < 2 || pitch != b.stride * b.elem) return true;
  const size_t at = y >= x ? (y - x) % pitch : (pitch - (x - y) % pitch) % pitch;
  return at < a.len * a.elem || at + b.len * b.elem > pitch;
}

inline rosetta_status check_strides(std::initializer_list<Array> as) {
  for (const Array &a : as)
    if (a.p && (a.stride < a.len || a.stride > MAX_STRIDE))
      return fail(ROSETTA_ERR_PARAMS, "%s: a stride of %zu elements for rows of %zu", a.name,
                  a.stride, a.len);
  return ROSETTA_OK;
}

// Alignment to the element, and outputs apart from everything else; an output
// and an input named in `same` may be one array.
inline rosetta_status check_arrays(std::initializer_list<Array> as, const char *out = nullptr,
                            std::initializer_list<const char *> same = {}) {
  for (const Array &a : as)
    if (a.p && (uintptr_t)a.p % a.elem)
      return fail(ROSETTA_ERR_PARAMS, "%s is not aligned to its elements", a.name);
  for (const Array *a = as.begin(); a != as.end(); ++a)
    for (const Array *b = a + 1; b != as.end(); ++b) {
      if (!a->p || !b->p || (!a->out && !b->out)) continue;
      if (!overlap(*a, *b)) continue;
      bool fine = false;
      for (const char *s : same)
        fine |= a->name == s && b->name == out && a->p == b->p && a->stride == b->stride;
      if (!fine) return fail(ROSETTA_ERR_ALIAS, "%s overlaps %s", b->name, a->name);
    }
  return ROSETTA_OK;
}

#define TRY(x)                        \
  do {                                \
    const rosetta_status st_ = (x);   \
    if (st_ != ROSETTA_OK) return st_; \
  } while (0)
#define NEED(p)                                                          \
  do {                                                                   \
    if (!(p)) return fail(ROSETTA_ERR_NULL, #p " is NULL");              \
  } while (0)

}  // namespace rosetta
