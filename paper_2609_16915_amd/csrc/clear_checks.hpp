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

// A named device array: rows of `len` elements of `elem` bytes, `stride` apart.  A row may be
// runs with others' elements between them: inner[0].n runs of inner[0].len elements,
// inner[0].stride apart, and each of those inner[1].n of inner[1].len (n = 0: all its own).
struct Runs {
  size_t n, len, stride;
};
struct Array {
  const char *name;
  const void *p;
  size_t rows, len, stride, elem;
  bool out;
  Runs inner[2] = {};
  // (past 64 bits where a caller's sizes are: 2^31 rows 2^32 elements apart)
  unsigned __int128 bytes() const {
    return rows && len ? ((unsigned __int128)(rows - 1) * stride + len) * elem : 0;
  }
  // Level `at`, from the rows on: its parts, their length and distance in elements.
  static constexpr int LEVELS = 3;
  Runs level(int at) const {
    if (at == 0) return {rows, len, stride};
    return at < LEVELS && inner[at - 1].n ? inner[at - 1] : Runs{0, 0, 0};
  }
};

// Whether two arrays share memory, from level ia of a and ib of b on, which are ea and eb bytes
// long, b's `by` bytes behind a's: by the whole ranges, or, parts as far apart in both (columns
// of one buffer), by the parts themselves.  Parts lie within their distance, so that one of a
// meets two of b at most: those that start before it and behind.
inline bool overlap_from(const Array &a, int ia, __int128 ea, const Array &b, int ib, __int128 eb,
                         __int128 by) {
  if (by >= ea || -by >= eb) return false;
  const Runs x = a.level(ia), y = b.level(ib);
  const __int128 ex = (__int128)x.len * a.elem, ey = (__int128)y.len * b.elem;
  if (x.n == 1) return overlap_from(a, ia + 1, ex, b, ib, eb, by);
  if (y.n == 1) return overlap_from(a, ia, ea, b, ib + 1, ey, by);
  const __int128 pitch = (__int128)x.stride * a.elem;
  if (!x.n || !y.n || pitch != (__int128)y.stride * b.elem) return true;
  // part i of a and i + k of b
  __int128 k = -by / pitch;
  if (by + k * pitch > 0) --k;
  for (int two = 0; two < 2; ++two, ++k)
    if (k > -(__int128)x.n && k < (__int128)y.n &&
        overlap_from(a, ia + 1, ex, b, ib + 1, ey, by + k * pitch))
      return true;
  return false;
}
inline bool overlap(const Array &a, const Array &b) {
  return overlap_from(a, 0, a.bytes(), b, 0, b.bytes(),
                      (__int128)(uintptr_t)b.p - (__int128)(uintptr_t)a.p);
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
