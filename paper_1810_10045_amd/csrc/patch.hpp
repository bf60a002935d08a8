// A lane's 16 bytes of a row, as fp32 values: what the kernels that work on whole
// rows and matrices load and store.
#pragma once

#include <type_traits>

#include "common.hpp"

namespace lmz {

// P values of a row: 16 bytes at the alignment of an element. Matrices are read
// once: past the caches.
template <typename T>
struct Patch;

template <>
struct Patch<float> {
  static constexpr int P = 4;
  using raw_t = f32x4;
  static __device__ __forceinline__ raw_t load(const float* p) {
    return stream_load_e(reinterpret_cast<const f32x4e*>(p));
  }
  static __device__ __forceinline__ void widen(const raw_t& r, float* x) {
    x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w;
  }
  // The values from number `by` (0 to 4) on, zeros behind them.
  static __device__ __forceinline__ raw_t shift(const raw_t& r, int by) {
    raw_t a = by & 2 ? raw_t{r.z, r.w, 0.f, 0.f} : r;
    a = by & 1 ? raw_t{a.y, a.z, a.w, 0.f} : a;
    return by & 4 ? raw_t{0.f, 0.f, 0.f, 0.f} : a;
  }
  static __device__ __forceinline__ raw_t pack(const float* x) {
    return raw_t{x[0], x[1], x[2], x[3]};
  }
  static __device__ __forceinline__ void store(float* p, const float* x) {
    __builtin_nontemporal_store(f32x4e{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4e*>(p));
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ void put(float* p, float x) { *p = x; }
};

template <>
struct Patch<bf16_t> {
  static constexpr int P = 8;
  using raw_t = u32x4;
  static __device__ __forceinline__ raw_t load(const bf16_t* p) {
    return stream_load_e(reinterpret_cast<const u32x4e*>(p));
  }
  static __device__ __forceinline__ void widen(const raw_t& r, float* x) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ raw_t shift(const raw_t& r, int by) {
    raw_t a = by & 4 ? raw_t{r.z, r.w, 0u, 0u} : r;
    a = by & 2 ? raw_t{a.y, a.z, a.w, 0u} : a;
    if (by & 1)
      a = raw_t{a.x >> 16 | a.y << 16, a.y >> 16 | a.z << 16, a.z >> 16 | a.w << 16, a.w >> 16};
    return by & 8 ? raw_t{0u, 0u, 0u, 0u} : a;
  }
  static __device__ __forceinline__ uint32_t bits(float x) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
  }
  static __device__ __forceinline__ raw_t pack(const float* x) {
    return raw_t{bits(x[0]) | bits(x[1]) << 16, bits(x[2]) | bits(x[3]) << 16,
                 bits(x[4]) | bits(x[5]) << 16, bits(x[6]) | bits(x[7]) << 16};
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float* x) {
    const raw_t w = pack(x);
    __builtin_nontemporal_store(u32x4e{w.x, w.y, w.z, w.w}, reinterpret_cast<u32x4e*>(p));
  }
  static __device__ __forceinline__ float one(const bf16_t* p) { return bf16_to_f32(p->bits); }
  static __device__ __forceinline__ void put(bf16_t* p, float x) {
    p->bits = static_cast<uint16_t>(bits(x));
  }
};

// How rows end: every one in whole vectors of P values, in a part of one, or they hold fewer
// than P (and are loaded one value at a time).
enum class Ends { WHOLE, PART, NARROW };

static inline Ends ends_of(int64_t D, int P) {
  return D < P ? Ends::NARROW : D % P ? Ends::PART : Ends::WHOLE;
}

// Where a lane's vector of P values at column `col` lies in a row of D. Every load (but of
// NARROW rows) is a whole vector inside the row, so that none stands under a condition: at
// the row's end it starts at D - P, and the values are moved `by` places down to their own;
// what else it read is not used, so a row may be written in place by others meanwhile.
// `have`: how many of the lane's values exist. OFF: what holds a column's distance from the
// row's start in bytes (with uint32_t and a row that the wave shares, an address is that
// distance in one register beside the row's in scalar ones).
template <typename T, Ends ENDS, typename OFF = int64_t>
struct Span {
  static constexpr int P = Patch<T>::P;
  static constexpr bool NARROW = ENDS == Ends::NARROW;
  using raw_t = typename Patch<T>::raw_t;
  using index_t = std::conditional_t<sizeof(OFF) == 4, int, int64_t>;
  index_t from;
  int by, have;
  __device__ __forceinline__ Span(index_t col, index_t D, bool use = true) {
    const index_t left = use ? D - col : 0;
    have = left >= P ? P : left > 0 ? static_cast<int>(left) : 0;
    by = NARROW ? 0 : P - have;
    from = NARROW ? 0 : left >= P ? col : D - P;
  }
  template <typename Q>  // T or const T
  static __device__ __forceinline__ Q* at(Q* row, index_t col) {
    using byte_t = std::conditional_t<std::is_const<Q>::value, const char, char>;
    return reinterpret_cast<Q*>(reinterpret_cast<byte_t*>(row) +
                                static_cast<OFF>(col * static_cast<index_t>(sizeof(T))));
  }
  __device__ __forceinline__ raw_t load(const T* row) const {
    if constexpr (!NARROW) return Patch<T>::load(at(row, from));
    float x[P];
#pragma unroll
    for (int e = 0; e < P; ++e) x[e] = e < have ? Patch<T>::one(row + e) : 0.f;
    return Patch<T>::pack(x);
  }
  // The values in their places, zeros behind them.
  __device__ __forceinline__ void widen(raw_t r, float* x) const {
    if (ENDS == Ends::WHOLE) {
      r = have ? r : raw_t{0, 0, 0, 0};
    } else if (ENDS == Ends::PART && by) {
      r = Patch<T>::shift(r, by);
    }
    Patch<T>::widen(r, x);
  }
  __device__ __forceinline__ void store(T* row, const float* x) const {
    if (have == P) {
      Patch<T>::store(at(row, from), x);
    } else if (ENDS != Ends::WHOLE) {
      T* p = at(row, NARROW ? 0 : from + by);
#pragma unroll
      for (int e = 0; e < P - 1; ++e)
        if (e < have) Patch<T>::put(p + e, x[e]);
    }
  }
};

__device__ __forceinline__ float read_lane(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// f over groups of LANES neighbouring lanes, in all of them, in an order that depends on
// LANES only.
template <int LANES, typename F>
__device__ __forceinline__ float lanes_fold(float x, F f) {
  auto from = [](float v, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value,
                                                      0xf, 0xf, true));
  };
  x = f(x, from(x, std::integral_constant<int, 0xB1>{}));  // lane ^ 1
  x = f(x, from(x, std::integral_constant<int, 0x4E>{}));  // lane ^ 2
  if constexpr (LANES >= 8) x = f(x, from(x, std::integral_constant<int, 0x141>{}));  // 4 of 8
  if constexpr (LANES >= 16) x = f(x, from(x, std::integral_constant<int, 0x140>{}));  // 8 of 16
  if constexpr (LANES == 32) x = f(x, __shfl_xor(x, 16, kWave));
  if constexpr (LANES == 64)
    x = f(f(read_lane(x, 0), read_lane(x, 16)), f(read_lane(x, 32), read_lane(x, 48)));
  return x;
}

template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  return lanes_fold<LANES>(x, [](float a, float b) { return a + b; });
}

}  // namespace lmz
