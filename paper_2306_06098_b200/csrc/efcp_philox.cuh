// The mask of a dropout, computed where it is needed and never stored.
//
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011) turns a
// counter and a key into four words.  The counter is (e / 8, offset) for element e of the logical order, the
// key the seed; the words' eight 16-bit halves, low half first, are the numbers of the elements 8 (e / 8) + 0..7.
// An element is dropped when its number is below T = round(65536 p); the others are multiplied by
// 65536 / (65536 - T), the exact inverse of the share that stays.  16 bits an element instead of 32 halve the
// arithmetic, which would bound the kernels otherwise.
#pragma once

#include <stdint.h>

namespace efcp {

struct Drop {
  uint32_t threshold;  // 0: nothing is dropped
  float scale;
  unsigned long long seed, offset;
  const unsigned long long* rng;  // (seed, offset) on the device, or null
};

struct DropKey {
  uint32_t k0, k1, o0, o1;
};

__device__ __forceinline__ DropKey drop_key(const Drop& d) {
  unsigned long long s = d.seed, o = d.offset;
  if (d.rng) {
    s = d.rng[0];
    o = d.rng[1];
  }
  return {uint32_t(s), uint32_t(s >> 32), uint32_t(o), uint32_t(o >> 32)};
}

// The four words of a group of eight elements.
__device__ __forceinline__ void drop_words(unsigned long long group, const DropKey& key,
                                           uint32_t (&word)[4]) {
  uint32_t a = uint32_t(group), b = uint32_t(group >> 32), c = key.o0, d = key.o1;
  uint32_t k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const unsigned long long p = 0xD2511F53ull * a, q = 0xCD9E8D57ull * c;
    a = uint32_t(q >> 32) ^ b ^ k0;
    b = uint32_t(q);
    c = uint32_t(p >> 32) ^ d ^ k1;
    d = uint32_t(p);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  word[0] = a; word[1] = b; word[2] = c; word[3] = d;
}

// Bit j: element 8 * group + j stays.
__device__ __forceinline__ uint32_t drop_keep8(unsigned long long group, const DropKey& key,
                                               uint32_t threshold) {
  uint32_t keep = 0, word[4];
  drop_words(group, key, word);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    keep |= uint32_t((word[i] & 0xFFFFu) >= threshold) << (2 * i);
    keep |= uint32_t((word[i] >> 16) >= threshold) << (2 * i + 1);
  }
  return keep;
}

// Dropout of the eight elements of a group.  (A half-word in the upper half of a register is compared there, next to
// whatever the lower half holds: one instruction less.)
__device__ __forceinline__ void drop_group(float (&v)[8], unsigned long long group, const DropKey& key,
                                           uint32_t threshold, float scale) {
  uint32_t word[4];
  drop_words(group, key, word);
  const uint32_t below = (threshold << 16) - 1;  // (threshold > 0; 65536 drops all)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = (word[i] << 16) > below ? v[2 * i] * scale : 0.f;
    v[2 * i + 1] = word[i] > below ? v[2 * i + 1] * scale : 0.f;
  }
}

}  // namespace efcp
