// Status reporting and argument checks shared by the entry points' files.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <initializer_list>

#include "../../include/fq.h"

namespace fq {

inline thread_local char g_err[512] = "";

inline fq_status fail(fq_status s, const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return s;
}

inline fq_status ok() {
  g_err[0] = '\0';
  return FQ_OK;
}

inline fq_status hip_fail(hipError_t e, const char *where) {
  return fail(FQ_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool is_pow2(int64_t v) { return v >= 1 && (v & (v - 1)) == 0; }

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Byte range [p, p + n) of a caller buffer, for the no-overlap preconditions.
struct Span {
  uintptr_t lo, hi;
};
inline Span span(const void *p, size_t n) { return Span{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + n}; }
inline bool overlap(Span a, Span b) { return a.lo && b.lo && a.lo < b.hi && b.lo < a.hi; }
// True when an output range overlaps another output or any input (NULL ranges are empty).
inline bool outputs_alias(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (auto p = o + 1; p != outs.end(); ++p)
      if (overlap(*o, *p)) return true;
    for (const Span &i : ins)
      if (overlap(*o, i)) return true;
  }
  return false;
}
// Bytes spanned by `rows` rows of `row_bytes` bytes at a stride of `ld_bytes`.
inline size_t rows_span(int64_t rows, int64_t ld_bytes, int64_t row_bytes) {
  return rows <= 0 ? 0 : (size_t)(rows - 1) * (size_t)ld_bytes + (size_t)row_bytes;
}

}  // namespace fq
