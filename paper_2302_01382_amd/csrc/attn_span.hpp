// attn_span.hpp -- which tokens the attention's rows see, and the steps that a workgroup takes over them.  Needs no HIP, so
// that a plain C++ program can check it.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define MPQ_ANYWHERE __attribute__((host, device)) inline __attribute__((always_inline))
#else
#define MPQ_ANYWHERE inline
#endif

namespace mpq {

// Tokens [lo, hi); none where hi <= lo (hi may be negative).
struct Span {
  int64_t lo, hi;
};
// A window as seen() takes it: positions lie within 2^31 of 0, so that one of 2^32 reaches as far as any wider one, and p - window
// stays far from the ends of 64 bits.
MPQ_ANYWHERE int64_t cut_window(int64_t window) { return window < ((int64_t)1 << 32) ? window : (int64_t)1 << 32; }

// What a row at position p sees of len tokens.  len is cut to the table's places, p is not: with a window lo may lie far behind
// len.
MPQ_ANYWHERE Span seen(int64_t p, int64_t len, bool causal, int64_t window) {
  return {window > 0 && p - window + 1 > 0 ? p - window + 1 : 0, causal && p + 1 < len ? p + 1 : len};
}

// Steps t0 .. t1 - 1 of `tokens` tokens each that split `split` of `splits` takes over a span: whole steps, dealt out in one
// piece each.  Tokens of a step that lie below span.hi are below len and may be looked up.
struct Steps {
  int64_t t0, t1;
};
MPQ_ANYWHERE Steps steps_of(const Span& span, int tokens, int splits, int split) {
  if (span.hi <= span.lo) return {0, 0};
  const int64_t first = span.lo / tokens, steps = (span.hi + tokens - 1) / tokens - first;
  const int64_t per = (unsigned)(steps + splits - 1) / (unsigned)splits;
  return {first + split * per, first + ((split + 1) * per < steps ? (split + 1) * per : steps)};
}

}  // namespace mpq
