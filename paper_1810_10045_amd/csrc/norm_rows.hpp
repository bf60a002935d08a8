// Layer norm: how a row is shared out among lanes, for the forward and the backward pass.
// A row stays in the registers of its group: LANES lanes of a wave, or WAVES whole waves,
// NV vectors of 16 bytes a lane, vector v of lane l being number l + v * lanes (a wave's
// lanes load neighbouring vectors). A group takes ROWS rows at once, all of their loads under way.
#pragma once

#include "keep.hpp"
#include "patch.hpp"

namespace lmz {

constexpr int kNormThreads = 256;  // of a workgroup, where a row's group is no larger

template <int LANES_, int WAVES_, int NV_, int ROWS_ = 1, int THREADS_ = kNormThreads>
struct NormShape {
  static constexpr int LANES = LANES_, WAVES = WAVES_, NV = NV_, ROWS = ROWS_, THREADS = THREADS_;
  static constexpr int kGroup = WAVES > 1 ? WAVES * kWave : LANES;  // lanes of a row
  static constexpr int kThreads = kGroup > THREADS_ ? kGroup : THREADS_;
  static constexpr int kGroups = kThreads / kGroup;  // of a workgroup
  static constexpr int kRows = kGroups * ROWS;       // of a workgroup at once
  static_assert(WAVES == 1 || LANES == kWave, "whole waves");
  // The thread's group in its workgroup, in a scalar register where a wave has but one.
  static __device__ __forceinline__ int group() {
    if constexpr (kGroups == 1) return 0;
    const int g = threadIdx.x / kGroup;
    return kGroup >= kWave ? first_lane(g) : g;
  }
};

template <typename T, Ends ENDS>
using NormSpan = Span<T, ENDS, uint32_t>;  // LM_NORM_MAX_WIDTH columns

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
template <typename T, Ends ENDS>
__device__ __forceinline__ void load_params(const float* w, const NormSpan<T, ENDS>& s, float* x) {
  constexpr int P = Patch<T>::P;
  if (ENDS == Ends::WHOLE) {
    load_vec<P>(Span<float, ENDS, uint32_t>::at(w, s.have ? s.from : 0), x);
  } else if (ENDS == Ends::NARROW || s.have < P) {
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const int at = e < s.have ? e : 0;
      const float y = w[s.have ? s.from + s.by + at : 0];
      x[e] = e < s.have ? y : 0.f;
    }
  } else {
    load_vec<P>(Span<float, ENDS, uint32_t>::at(w, s.from), x);
  }
}

// A kernel's forms by how rows end: pick(form) with the End as a constant. Rows of less than
// a vector have the smallest group.
template <typename S, typename F>
static inline auto norm_ends(Ends ends, F pick) {
  if constexpr (S::kGroup == 8)
    if (ends == Ends::NARROW) return pick(std::integral_constant<Ends, Ends::NARROW>{});
  return ends == Ends::WHOLE ? pick(std::integral_constant<Ends, Ends::WHOLE>{})
                             : pick(std::integral_constant<Ends, Ends::PART>{});
}

}  // namespace lmz
