// Division by launch constants in the kernels. Internal; included by the kernel sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fa {
namespace {

// Division by a divisor that is fixed for the launch, as a multiply-high and two shifts (Granlund and
// Montgomery, "Division by invariant integers using multiplication", PLDI 1994, the algorithm for
// unsigned 32-bit operands): with l = ceil(log2 d) and m = floor(2^32 (2^l - d) / d) + 1, every 32-bit
// n has n / d = (t + ((n - t) >> min(l, 1))) >> max(l - 1, 0), t = mulhi(m, n). The host computes m and
// the two shifts (6 bits: min(l, 1) | max(l - 1, 0) << 1); the kernel's work decomposition then needs
// no division sequence (a runtime division by a value the compiler cannot see is ~25 instructions).
struct FastDiv {
  uint32_t m, sh;
};
FastDiv make_fastdiv(uint32_t d) {
  uint32_t l = 0;
  while ((uint64_t{1} << l) < d) ++l;
  const uint64_t m = ((uint64_t{1} << 32) * ((uint64_t{1} << l) - d)) / d + 1;
  return {static_cast<uint32_t>(m), (l < 1 ? l : 1u) | ((l > 0 ? l - 1 : 0u) << 1)};
}
__device__ __forceinline__ uint32_t fast_div(uint32_t n, uint32_t m, uint32_t sh) {
  const uint32_t t = __umulhi(m, n);
  return (t + ((n - t) >> (sh & 1u))) >> (sh >> 1);
}

}  // namespace
}  // namespace fa
