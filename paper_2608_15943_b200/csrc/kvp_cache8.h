// The 8-bit cache: e4m3 numbers, and for each block of 16 tokens and KV head a power of two that they are multiples of, kept as
// its exponent + 127 in a byte (no CUDA dependency: the kernels and a host-only test use the same rules).
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define KVP_HD __host__ __device__
#else
#define KVP_HD
#endif

namespace kvp {

constexpr int CACHE_BLOCK = 16;            // tokens that share a scale
constexpr int LEAST_SCALE = -100, MOST_SCALE = 120;   // exponents: 448 * 2^-100 is far below any activation; bf16 ends below 448 * 2^120

// Smallest e >= LEAST_SCALE with amax <= 448 * 2^e, from the bits of a finite amax >= 0.  448 = 1.75 * 2^8: the exponent of amax
// less 8, and one more where its mantissa is above 1.75 (adding 0x1fffff carries exactly then).
KVP_HD inline int scale_exponent(uint32_t amax_bits) {
  const int e = int((amax_bits + 0x1fffffu) >> 23) - 127 - 8;
  return e < LEAST_SCALE ? LEAST_SCALE : e;
}
// A byte that no append wrote is taken as the nearest that one could have written.
KVP_HD inline uint32_t scale_byte(uint32_t byte) {
  const uint32_t least = uint32_t(LEAST_SCALE + 127), most = uint32_t(MOST_SCALE + 127), b = byte < least ? least : byte;
  return b > most ? most : b;
}
KVP_HD inline int exponent_of_byte(uint32_t byte) { return int(scale_byte(byte)) - 127; }
// Bits of 2^e as a float; e below the smallest normal number's is taken as that (used for factors below 2^-20, where a number
// of the cache becomes 0 either way).
KVP_HD inline uint32_t power_bits(int e) { return uint32_t((e < -126 ? -126 : e) + 127) << 23; }

}  // namespace kvp
