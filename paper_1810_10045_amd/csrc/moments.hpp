// Adam moments in 8 bits and the AdamW step on them (device code shared by the
// steps over tensors and over table rows).
//
// Format. 32 consecutive values share a scale 2^k, k the smallest integer with
// max|x| <= 448 * 2^k (448: the largest e4m3 number), kept as the byte k + 127.
// A value is its e4m3 code times the scale. A power of two makes decoding exact and
// costs e4m3 no precision: its step is relative. A value that the step leaves as it
// is (its new second moment is not finite) is scaled by the exact power too, so it
// stays the same number when its block's scale shrinks (and, down to the grid's
// subnormals, when it grows); the others by a power that may be half a unit low
// (fill_scales), which is within their rounding. The second moment is kept as its square
// root: codes reach 2^-18 below a block's largest, which is 2^-36 in v. The last 3 bits
// of that are the grid's subnormals, too coarse to hold a v that follows its gradients
// (below).
//
// Rounding is stochastic. With beta2 = 0.999 a step moves sqrt(v) by 0.05% of
// itself while half a code step is 3 to 6%: rounded to nearest it would not
// move until a gradient reached about 8 times its root mean square, and would
// never decay. v_cvt_sr_fp8_f32 takes floor(x / step + R / 2^20) steps, R the
// high 20 bits of a word given to it, in the subnormal range as well. The word
// is a hash of the value's number and the caller's seed, so a call can be
// repeated bit for bit. A root above zero never gets the code zero: beside it
// a first moment of the grid's smallest size would be divided by eps alone.
//
// The root is rounded without bias, so the mean of r^2 is above v by the rounding's
// variance, and a step starts from r^2. A step moves the root by little, so its variance
// is about |r' - r| s, s the grid's step (s / r is 1/16 to 1/8), which adds c2 |g^2 - v| s /
// (2 r) to each step's c2 g^2. With normal gradients v settles 4 to 5% above E g^2 (12,000
// steps, beta2 0.999: 1.04 to 1.05; the root scatters by 15% around a mean 1% high, and 1
// / r is 1% high), down to 2^-12 of a block's largest root. In the subnormals s / r
// grows: v is 7, 14, 28% high at 2^-14, 2^-15, 2^-16 of it, 1.8 and 2.3 times at 2^-17 and
// 2^-17.4, where updates are 13 and 28% short.
#pragma once

#include "common.hpp"

namespace lmz {

constexpr int kMomentBlock = LM_MOMENT_BLOCK;  // values that share a scale
static_assert(kMomentBlock == 32, "block_max8 reduces 8 lanes of 4 values");

typedef uint32_t u32x2e __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32e __attribute__((aligned(1)));

struct StepKeys {
  uint32_t k0, k1;
};

// Two words from the caller's 64-bit seed (host).
static inline StepKeys step_keys(uint64_t seed) {
  uint64_t z = seed * 0x9E3779B97F4A7C15ull + 0x632BE59BD9B4E019ull;
  z = (z ^ (z >> 29)) * 0xD6E8FEB86659FD93ull;
  z ^= z >> 32;
  return {static_cast<uint32_t>(z), static_cast<uint32_t>(z >> 32)};
}

// The random word of value number e: two rounds of multiply and xor-shift. The
// multipliers here and above are published ones, known to mix well: three primes of Y.
// Collet's 32-bit hash (2012), 2^64 over the golden ratio (Knuth) and that of a published
// 64-bit mixer (0xD6E8FEB86659FD93); the rounds are this file's.
__device__ __forceinline__ uint32_t value_word(uint64_t e, const StepKeys& k) {
  uint32_t h = (static_cast<uint32_t>(e) ^ k.k0) * 0x9E3779B1u;
  h ^= h >> 15;
  h = (h + k.k1 + static_cast<uint32_t>(e >> 32) * 0x85EBCA77u) * 0xC2B2AE3Du;
  return h ^ (h >> 16);
}

// Maximum over the 8 lanes of a block, in all of them.
__device__ __forceinline__ uint32_t block_max8(uint32_t x) {
  auto up = [](uint32_t a, int b) {
    const uint32_t u = static_cast<uint32_t>(b);
    return a > u ? a : u;
  };
  x = up(x, __builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0xB1, 0xf, 0xf, true));   // lane ^ 1
  x = up(x, __builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x4E, 0xf, 0xf, true));   // lane ^ 2
  return up(x, __builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x141, 0xf, 0xf, true));  // 7 - lane
}

// The scale byte of a block whose largest magnitude has these bits.
__device__ __forceinline__ int scale_byte(uint32_t top) {
  // The exponent of the largest value, one more where its fraction is above
  // 448's (1.75), less 448's own 8; all zeros and values below 2^-119: 0.
  const int b = static_cast<int>((top + 0x1FFFFFu) >> 23) - 8;
  return b > 0 ? b : 0;
}

// 4 values of codes in one word.
__device__ __forceinline__ void decode4(uint32_t codes, int scale, float* x) {
  const int k = scale - 127;
  x[0] = __builtin_amdgcn_ldexpf(__builtin_amdgcn_cvt_f32_fp8(codes, 0), k);
  x[1] = __builtin_amdgcn_ldexpf(__builtin_amdgcn_cvt_f32_fp8(codes, 1), k);
  x[2] = __builtin_amdgcn_ldexpf(__builtin_amdgcn_cvt_f32_fp8(codes, 2), k);
  x[3] = __builtin_amdgcn_ldexpf(__builtin_amdgcn_cvt_f32_fp8(codes, 3), k);
}

// 2^-k by scale byte, in LDS: what a value is multiplied by before it is rounded.
// powf gives some of these powers half a unit in the last place low. They are
// taken as it gives them, since torch's ldexp multiplies by the same numbers: a
// program that computes codes with torch operations gets the kernels', bit for
// bit. A rounding's threshold moves by 2^-20 of a step at most, the resolution of
// its random part; none is high, so no value passes 448. A thread's one call of
// powf serves the 8 values of its vectors: 4% more of a step of 202M parameters than
// exact powers take.
constexpr int kScales = 256;

__device__ __forceinline__ void fill_scales(float* inverse, int threads) {
  for (int b = threadIdx.x; b < kScales; b += threads)
    inverse[b] = powf(2.f, static_cast<float>(127 - b));
  __syncthreads();
}

// The codes of 4 values of this lane's block (8 lanes) and the block's scale byte.
// FLOOR: values above zero round to no code below 1. kept: a bit for each value that
// the step did not change.
template <bool FLOOR>
__device__ __forceinline__ uint32_t encode4(const float* x, const uint32_t* word, uint32_t kept,
                                            const float* inverse, int& scale) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t a = __float_as_uint(x[e]) & 0x7fffffffu;
    top = a > top ? a : top;
  }
  scale = scale_byte(block_max8(top));
  const float by = inverse[scale];
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = x[e] * by;
  if (ballot(kept != 0)) {
    // A kept value is on the grid unless its block's scale grew past it, and stays there: a
    // power half a unit low would take it a whole step down where its random part is 0.
#pragma unroll
    for (int e = 0; e < 4; ++e)
      y[e] = kept >> e & 1 ? __builtin_amdgcn_ldexpf(x[e], 127 - scale) : y[e];
  }
  if (FLOOR) {
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = x[e] > 0.f ? fmaxf(y[e], 0x1p-9f) : 0.f;
  }
  int c = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], word[0], 0, 0);
  c = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], word[1], c, 1);
  c = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], word[2], c, 2);
  return __builtin_amdgcn_cvt_sr_fp8_f32(y[3], word[3], c, 3);
}

struct MomentParams {
  float b1, c1, b2, c2;  // the moments' weights, c = 1 - b
  float lr, eps, wd;
  float inv_c1, root_c2;  // the bias corrections 1 / (1 - b1^t), sqrt(1 / (1 - b2^t))
};

static inline MomentParams make_moment_params(const OptParams& o, float beta2, int64_t step) {
  MomentParams q;
  q.b1 = o.b1;
  q.c1 = 1.f - o.b1;
  q.b2 = o.b2;
  q.c2 = 1.f - o.b2;
  q.lr = o.lr;
  q.eps = o.eps;
  q.wd = o.wd;
  q.inv_c1 = o.inv_c1;
  q.root_c2 = static_cast<float>(__builtin_sqrt(
      1.0 / (1.0 - __builtin_pow(static_cast<double>(beta2), static_cast<double>(step)))));
  return q;
}

// The step on one value with its moments decoded (r: the second's root). Each
// product and sum of the moments is rounded by itself, so that codes and scales
// can be computed again with any IEEE arithmetic. A value whose new second
// moment is not finite is left as it was; returns false for it.
__device__ __forceinline__ bool adamw_value8(float& p, float& m, float& r, float g, float wd,
                                             const MomentParams& o) {
#pragma clang fp contract(off)
  const float m1 = m * o.b1 + g * o.c1;
  const float v1 = (r * r) * o.b2 + (g * o.c2) * g;
  const bool ok = v1 < __builtin_inff();  // false for NaN too
  const float r1 = sqrtf(v1);
  // v_rcp_f32 is within an ulp of the quotient, far below what the update's sum
  // keeps of it (a division makes a step of 202M parameters 3% longer).
  const float step = (m1 * o.inv_c1) * __builtin_amdgcn_rcpf(__builtin_fmaf(r1, o.root_c2, o.eps));
  const float p1 = __builtin_fmaf(-o.lr, __builtin_fmaf(wd, p, step), p);
  p = ok ? p1 : p;
  m = ok ? m1 : m;
  r = ok ? r1 : r;
  return ok;
}

}  // namespace lmz
