// Rounds of one long axis in equal shares (paged_attention4.hip).  The rounds are counted up to 2^31 - 1, and n shares can reach
// past them by almost n: sums of the two are unsigned.
#pragma once

#include <stdint.h>

namespace kv {

// Rounds of a share: with one, its first loads are most of it, and there are more to join (one cache of up to 6000 rows 10.6 us,
// with one round 11.5, with four 12.0; 8 of up to 2000 13.2, 13.2 and 14.3).
constexpr uint32_t kLeastRounds4 = 2;

// Rounds to a share, of T in n shares.
__host__ __device__ inline int share_of(int T, int n) {
  const uint32_t even = ((uint32_t)T + (uint32_t)n - 1u) / (uint32_t)n;
  return (int)(even > kLeastRounds4 ? even : kLeastRounds4);
}

// Where share number `share` of S rounds each begins, and where it ends; T: there is none.
__host__ __device__ inline int share_begin(int T, int S, int share) {
  const uint32_t at = (uint32_t)share * (uint32_t)S;
  return (int)(at < (uint32_t)T ? at : (uint32_t)T);
}
__host__ __device__ inline int share_end(int T, int S, int at) {
  const uint32_t end = (uint32_t)at + (uint32_t)S;
  return (int)(end < (uint32_t)T ? end : (uint32_t)T);
}

}  // namespace kv
