// The key that parts the `need` largest of many from the others, by counting (sparse.hip).  Plain arithmetic, the same on host and device.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace covspec {

// Keys of blocks: those that are not there, and those that are taken whatever their score.
constexpr uint32_t kNone = 0u, kAlways = 0xFFFFFFFFu;

// Of parts that keys were counted in: the one that holds the `need`-th largest, how many keys are beyond it, how many in it.
struct Part { int bin, before, here; };
// All keys above `at` are taken, and the first `more` of those at it.
struct Parting { uint32_t at; int more; };

// Of more than `need` keys, the least lo and the largest hi, neither of them kNone or kAlways.  count(pass, lo, width, shift, need) counts the keys lo .. lo + width in parts
// of 2^shift from lo on, 2^BITS of them at most; every pass keeps one part, which ends at hi at the latest: behind the largest keys, NaN's, a whole part would pass 32 bits,
// and a range that has come round to zero holds all keys, those of neither kind among them.
template <int BITS, typename Count>
__host__ __device__ __forceinline__ Parting parting_key(uint32_t lo, uint32_t hi, int need, Count count) {
  for (int pass = 0; need > 0; ++pass) {
    const uint32_t width = hi - lo;
    if (width == 0) return Parting{lo, need};
    const int bits = 32 - __builtin_clz(width), shift = bits > BITS ? bits - BITS : 0;
    const Part p = count(pass, lo, width, shift, need);
    need -= p.before;
    lo += (uint32_t)p.bin << shift;
    const uint32_t part = (1u << shift) - 1;
    hi = hi - lo > part ? lo + part : hi;
    if (need == p.here) return Parting{lo - 1, 0};
  }
  return Parting{kAlways - 1, 0};
}

}  // namespace covspec
