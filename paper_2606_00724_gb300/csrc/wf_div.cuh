// Division by numbers that a launch fixes.
#pragma once

#include <stdint.h>

namespace wf {

// Quotient and remainder by an invariant divisor with a multiply and a shift
// (Granlund and Montgomery, "Division by invariant integers using
// multiplication", 1994): for 0 <= x < 2^31 and d >= 1, with
// l = ceil(log2 d) and mul = floor(2^32 (2^l - d) / d) + 1,
// x / d = (umulhi(mul, x) + x) >> l.
struct FastDiv {
  uint32_t d, mul, shift;
};
inline FastDiv make_fastdiv(uint32_t d) {
  FastDiv f;
  f.d = d;
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  f.shift = l;
  f.mul = (uint32_t)((((1ull << l) - d) << 32) / d + 1);
  return f;
}
__device__ __forceinline__ uint32_t fastdiv(uint32_t x, const FastDiv& f) {
  return (__umulhi(f.mul, x) + x) >> f.shift;
}

}  // namespace wf
