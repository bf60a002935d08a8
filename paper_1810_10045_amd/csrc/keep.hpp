// Dropout's mask: a function of the seed and a value's place, computed where it is used
// and stored nowhere, so a backward pass that is given the seed makes the same mask.
//
// Word w of a call is value_word(w, keys of the seed), 32 bits for two neighbouring
// columns: row i of D columns has ceil(D / 2) words, column j the low (j even) or high (j
// odd) half of word i * ceil(D / 2) + j / 2. A value is kept where its half is at least
// round(65536 p), and multiplied by 1 over the share that is kept: the expectation is
// exact for the p that is drawn, which is within 2^-17 of the caller's. Two values to a
// word: the hash's two 32-bit products take a quarter of the vector rate, and a word for
// each value would cost as much as a large call's memory. What is kept correlates by 0.001 with
// its neighbours, seeds that follow each other not at all. The hash has one product
// left in which high bits of a word's number can spread, so certain far words do correlate: most
// where numbers differ by powers of two and their sums and differences, by up to 0.02 within 2^16
// words, 0.04 within 2^20, 0.08 within 2^24, 0.2 within 2^28, 0.4 within 2^32 and 0.95 beyond,
// where the number's upper half only adds a constant to the word before that product.
#pragma once

#include <math.h>

#include "moments.hpp"

namespace lmz {

struct KeepArgs {
  uint64_t seed;
  const int64_t* seed_at;  // on the device: read instead of seed, or nullptr
  uint32_t least;          // 0 to 65536
  float scale;
};

static inline KeepArgs make_keep(float p, uint64_t seed, const int64_t* seed_at) {
  KeepArgs k{seed, seed_at, 0, 1.f};
  k.least = static_cast<uint32_t>(nearbyint(65536.0 * static_cast<double>(p)));
  if (k.least) k.scale = k.least < 65536 ? static_cast<float>(65536.0 / (65536 - k.least)) : 0.f;
  return k;
}

struct Keep {
  StepKeys keys;
  uint32_t least;
  float scale;
  __device__ __forceinline__ explicit Keep(const KeepArgs& a)
      : keys(step_keys(a.seed_at ? static_cast<uint64_t>(*a.seed_at) : a.seed)),
        least(a.least),
        scale(a.scale) {}
  // P values from an even column on, the first two of word `word`. A dropped value is 0
  // whatever it was (infinity, NaN).
  template <int P>
  __device__ __forceinline__ void apply(uint64_t word, float* x) const {
    const uint32_t low = static_cast<uint32_t>(word);
    if (ballot(low > ~0u - P / 2)) {  // words on both sides of a multiple of 2^32
#pragma unroll
      for (int e = 0; e < P; e += 2) choose(value_word(word + e / 2, keys), x + e);
      return;
    }
    // The upper half of a word's number is the same for all of them: one product.
    StepKeys k = keys;
    k.k1 += static_cast<uint32_t>(word >> 32) * kHighWord;
#pragma unroll
    for (int e = 0; e < P; e += 2) choose(value_word(low + e / 2, k), x + e);
  }

 private:
  __device__ __forceinline__ void choose(uint32_t h, float* x) const {
    x[0] = (h & 0xffffu) >= least ? x[0] * scale : 0.f;
    x[1] = (h >> 16) >= least ? x[1] * scale : 0.f;
  }
};

}  // namespace lmz
