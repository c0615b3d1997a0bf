// Rows of attention of new tokens: the query heads of a token, in each of the layers that share its donor, one token behind the other
// (no CUDA dependency: the kernels, the host and a host-only test use the same rules).
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define KVP_HD __host__ __device__
#else
#define KVP_HD
#endif

namespace kvp {

constexpr int CHUNK_TILE = 128;           // rows of a tile; two are a unit
constexpr int CHUNK_MOST_TOKENS = (1 << 24) - 1;   // of a call; a tile's rows are those of a token at most, so that rows are counted in 31 bits

// Rows of a token, and what divides by them: row / n is the upper word of 2 row * mul, shifted (mul: 2^(31 + shift) / n rounded up, n <=
// 2^shift; exact below 2^31).  The set-up of every call walks through some dozen such quotients ahead of its first load.
struct Rows {
  int n, shift;
  uint32_t mul;
  KVP_HD int token(int row) const {
#ifdef __CUDA_ARCH__
    return int(__umulhi(uint32_t(row) * 2, mul) >> shift);
#else
    return int(uint32_t(uint64_t(uint32_t(row) * 2) * mul >> 32) >> shift);
#endif
  }
};
inline Rows rows_of_token(int n) {
  Rows r{n, 0, 0};
  while (1 << r.shift < n) ++r.shift;
  r.mul = uint32_t(((uint64_t(1) << (31 + r.shift)) + n - 1) / n);
  return r;
}
// Units of a sequence's rows.
KVP_HD inline int units_of_rows(int rows) { return rows / (2 * CHUNK_TILE) + (rows % (2 * CHUNK_TILE) != 0); }   // (the sum rounded up may pass 2^31)

}  // namespace kvp
