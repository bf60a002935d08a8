// Layer norm: how a row is shared out among lanes, for the forward and the backward pass.
//
// A row stays in the registers of its group: LANES lanes of a wave, or WAVES whole waves,
// NV vectors of 16 bytes a lane, vector v of lane l being number l + v * lanes (a wave's
// lanes load neighbouring vectors).
#pragma once

#include "keep.hpp"
#include "patch.hpp"

namespace lmz {

constexpr int kNormThreads = 256;  // of a workgroup, where a row's group is no larger

template <int LANES_, int WAVES_, int NV_>
struct NormShape {
  static constexpr int LANES = LANES_, WAVES = WAVES_, NV = NV_;
  static constexpr int kGroup = WAVES > 1 ? WAVES * kWave : LANES;  // lanes of a row
  static constexpr int kThreads = kGroup > kNormThreads ? kGroup : kNormThreads;
  static constexpr int kRows = kThreads / kGroup;  // rows of a workgroup at once
  static_assert(WAVES == 1 || LANES == kWave, "whole waves");
};

// Sums over a row's group: of the lanes by lanes_sum, of the waves in their order. A
// group of several waves meets in LDS, every wave of the workgroup with it; calls that follow
// each other take different halves of `lds`.
template <typename S, int N>
__device__ __forceinline__ void group_sums(float (&x)[N], float (*lds)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = lanes_sum<S::LANES>(x[i]);
  if constexpr (S::WAVES > 1) {
    const int wave = threadIdx.x / kWave;
    if (threadIdx.x % kWave == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) lds[wave][i] = x[i];
    }
    __syncthreads();
    const int first = wave / S::WAVES * S::WAVES;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = lds[first][i];
#pragma unroll
    for (int w = 1; w < S::WAVES; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += lds[first + w][i];
  }
}

// P fp32 parameters of columns `s` (a weight or bias), zeros behind a row's end.
template <typename T, bool NARROW>
__device__ __forceinline__ void load_params(const float* w, const Span<T, NARROW>& s, float* x) {
  constexpr int P = Patch<T>::P;
  if (NARROW || s.have < P) {
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const int at = e < s.have ? e : 0;
      const float y = w[s.have ? s.from + s.by + at : 0];
      x[e] = e < s.have ? y : 0.f;
    }
  } else {
    load_vec<P>(w + s.from, x);
  }
}

// Calls f with the shape for rows of D values of type T.
template <typename T, typename F>
static inline int norm_shape(int64_t D, F f) {
  const int64_t vectors = (D + Patch<T>::P - 1) / Patch<T>::P;
  if (vectors <= 8) return f(NormShape<8, 1, 1>{});
  if (vectors <= 16) return f(NormShape<16, 1, 1>{});
  if (vectors <= 32) return f(NormShape<32, 1, 1>{});
  if (vectors <= 64) return f(NormShape<64, 1, 1>{});
  if (vectors <= 128) return f(NormShape<64, 2, 1>{});
  if (vectors <= 256) return f(NormShape<64, 4, 1>{});
  if (vectors <= 512) return f(NormShape<64, 4, 2>{});
  if (vectors <= 1024) return f(NormShape<64, 8, 2>{});
  if (vectors <= 2048) return f(NormShape<64, 16, 2>{});
  return f(NormShape<64, 16, 4>{});
}
static_assert(LM_NORM_MAX_WIDTH <= 4 * 16 * kWave * Patch<float>::P, "the widest shape");

}  // namespace lmz
