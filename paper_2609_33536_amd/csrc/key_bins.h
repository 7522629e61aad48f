// Scores as integers, and the narrowing of a pick among them by histograms (internal header): the
// kernels of select.hip and the host test of the pick share these steps.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ekv {

// A score as an integer that orders as it does, above 1; what is not a number above all scores.
constexpr uint64_t kNotNumber = ~0ull;
__host__ __device__ __forceinline__ uint64_t score_key(double x) {
  if (x != x) return kNotNumber;
  const uint64_t w = __builtin_bit_cast(uint64_t, x + 0.0);   // (-0 is 0)
  return w >> 63 ? ~w : w | 1ull << 63;
}

// The keys [from, to] in question, in at most 1024 bins of 2^shift keys from `from` on.
struct KeyBins {
  uint64_t from, to;

  // (of more than one key)
  __host__ __device__ __forceinline__ int shift() const {
    const int s = 54 - __builtin_clzll(to - from);   // (to - from) >> s < 1024
    return s > 0 ? s : 0;
  }
  __host__ __device__ __forceinline__ bool holds(uint64_t key) const { return key >= from && key <= to; }
  __host__ __device__ __forceinline__ uint32_t bin(uint64_t key, int shift) const { return (uint32_t)((key - from) >> shift); }
  // Goes on with one bin, which holds a key.  Its end may lie beyond `to`, and beyond 2^64 too (what
  // is not a number has the key 2^64 - 1): `to` moves only where the bin ends below it.
  __host__ __device__ __forceinline__ void enter(int bin, int shift) {
    from += (uint64_t)bin << shift;
    if ((to - from) >> shift) to = from + ((1ull << shift) - 1);
  }
};

}  // namespace ekv
