// The counter-based generator of the dropout: Philox4x32 of ten rounds (Salmon,
// Moraes, Dror and Shaw 2011: each round multiplies two of the four counter words
// by odd constants and mixes the products' halves with the other two words and a
// key that grows by a Weyl sequence). Any block of 128 bits is a function of its
// counter alone, so a backward pass forms the mask again instead of reading it.
#pragma once

#include <stdint.h>

namespace lx {

// What a kernel is given: rng points to the seed and the offset on the device; a
// value is dropped where its 16 bits are below `below`; kept ones are multiplied by
// scale = 65536 / (65536 - below).
struct Dropout {
  const uint64_t* rng;
  uint32_t below;
  float scale;
};

struct DropoutKeys {
  uint32_t k0, k1, o0, o1;
};
__device__ __forceinline__ DropoutKeys dropout_keys(const Dropout& d) {
  const uint64_t seed = d.rng[0], offset = d.rng[1];
  return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)};
}

// Which of the 8 columns of group `group` of token `token` are kept, as bits. The
// group's counter is (group, token, offset); column c has bits 16 (c % 2) ... of
// word c / 2.
__device__ __forceinline__ uint32_t dropout_kept(const Dropout& d, DropoutKeys q, uint32_t group, uint32_t token) {
  uint32_t x0 = group, x1 = token, x2 = q.o0, x3 = q.o1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
    x0 = (uint32_t)(b >> 32) ^ x1 ^ q.k0;
    x1 = (uint32_t)b;
    x2 = (uint32_t)(a >> 32) ^ x3 ^ q.k1;
    x3 = (uint32_t)a;
    q.k0 += 0x9E3779B9u;
    q.k1 += 0xBB67AE85u;
  }
  const uint32_t x[4] = {x0, x1, x2, x3};
  uint32_t kept = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) kept |= (uint32_t)((x[j] & 0xFFFFu) >= d.below) << 2 * j | (uint32_t)((x[j] >> 16) >= d.below) << (2 * j + 1);
  return kept;
}

}  // namespace lx
