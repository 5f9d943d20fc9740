// Random numbers of the dropout calls: Philox4x32-10 (Salmon, Moraes, Dror,
// Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011), a counter
// through ten rounds of two 32 x 32 bit products.  No state and no stored mask:
// every number is a function of (seed, offset) and of what it belongs to.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace scope {

__device__ __forceinline__ uint4 philox(uint4 c, uint2 key) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t x = static_cast<uint64_t>(c.x) * 0xD2511F53u;
    const uint64_t y = static_cast<uint64_t>(c.z) * 0xCD9E8D57u;
    c = make_uint4(static_cast<uint32_t>(y >> 32) ^ c.y ^ key.x, static_cast<uint32_t>(y),
                   static_cast<uint32_t>(x >> 32) ^ c.w ^ key.y, static_cast<uint32_t>(x));
    key.x += 0x9E3779B9u;
    key.y += 0xBB67AE85u;
  }
  return c;
}

// The generator's key and the stream's place, from the caller's {seed, offset};
// where nothing is dropped the caller may have none (null).
struct Stream {
  uint2 key, at;
  __device__ explicit Stream(const uint64_t *rng) {
    const uint64_t seed = rng ? rng[0] : 0, offset = rng ? rng[1] : 0;
    key = make_uint2(static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32));
    at = make_uint2(static_cast<uint32_t>(offset), static_cast<uint32_t>(offset >> 32));
  }
};

// Attention dropout.  A kernel meets its (query, key) pairs in an order of its
// own (gathered keys here, gathered queries there), so neighbours cannot share
// a Philox call.  Instead every query and every key has two Philox words, and a
// pair's number is one 32 x 32 bit product of them, both halves folded: two
// queries (or two keys) agree in both words with probability 2^-64.  Means, row,
// column and pairwise correlations and the largest singular value of 4096 x 4096
// masks are those of independent bits.
__device__ __forceinline__ uint2 pair_word(const Stream &s, uint32_t token, uint32_t head, uint32_t side) {
  const uint4 w = philox(make_uint4(token, 0x80000000u + 2u * head + side, s.at.x, s.at.y), s.key);
  return make_uint2(w.x, w.y);
}
// `drop`: the threshold in the upper 16 bits.
__device__ __forceinline__ bool pair_kept(uint2 query, uint2 key, uint32_t drop) {
  const uint64_t z = static_cast<uint64_t>(query.x ^ key.x) * (query.y + key.y);
  return (static_cast<uint32_t>(z >> 32) ^ static_cast<uint32_t>(z)) >= drop;
}

}  // namespace scope
