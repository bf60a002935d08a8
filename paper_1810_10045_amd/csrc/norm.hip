// Layer norm, with dropout and the residual sum before it:
//     h = add + dropout(x),  y = (h - mean) rstd weight + bias,  rstd = 1 / sqrt(var + eps).
// One pass: a row is read once into its group's registers (norm_rows.hpp), its mean and
// then the mean square of what is left are summed in fp32 (two sums, so that rows far from
// zero lose nothing), and y and h are written. HBM bounds it: up to 4 elements for each.
#include "launch_parts.hpp"
#include "norm_rows.hpp"

namespace lmz {

struct NormArgs {
  const void *x, *add;
  const float *weight, *bias;
  void *y, *h;
  float *mean, *rstd;
  int64_t ld_x, ld_add, ld_y, ld_h, rows;
  int D;
  float eps, inv_d;
  KeepArgs keep;
};

template <typename T, typename S, bool ADD, bool NARROW>
__global__ __launch_bounds__(S::kThreads) void k_norm(NormArgs a, uint32_t first) {
  constexpr int P = Patch<T>::P, NV = S::NV;
  using raw_t = typename Patch<T>::raw_t;
  __shared__ float part[2][S::kThreads / kWave][1];
  const int64_t i = (first + static_cast<int64_t>(blockIdx.x)) * S::kRows +
                    threadIdx.x / S::kGroup;
  const bool live = i < a.rows;
  const int64_t row = live ? i : a.rows - 1;
  const int lane = threadIdx.x % S::kGroup;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  const T* add = static_cast<const T*>(a.add) + row * a.ld_add;
  raw_t rx[NV], ra[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Span<T, NARROW> s((lane + v * S::kGroup) * P, a.D);
    rx[v] = s.load(x);
    if constexpr (ADD) ra[v] = s.load(add);
  }
  float h[NV][P], sum[1] = {0.f};
  const bool drops = a.keep.least != 0;
  const Keep keep(a.keep);
  const uint64_t word = static_cast<uint64_t>(row) * ((a.D + 1) / 2);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Span<T, NARROW> s((lane + v * S::kGroup) * P, a.D);
    s.widen(rx[v], h[v]);
    if (drops) keep.apply<P>(word + (lane + v * S::kGroup) * (P / 2), h[v]);
    if constexpr (ADD) {
      float z[P];
      s.widen(ra[v], z);
#pragma unroll
      for (int e = 0; e < P; ++e) h[v][e] += z[e];
    }
#pragma unroll
    for (int e = 0; e < P; ++e) sum[0] += h[v][e];
    if (a.h && live) s.store(static_cast<T*>(a.h) + row * a.ld_h, h[v]);
  }
  group_sums<S>(sum, part[0]);
  const float mean = sum[0] * a.inv_d;
  float square[1] = {0.f};
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Span<T, NARROW> s((lane + v * S::kGroup) * P, a.D);
#pragma unroll
    for (int e = 0; e < P; ++e) {
      h[v][e] -= mean;
      square[0] = e < s.have ? __builtin_fmaf(h[v][e], h[v][e], square[0]) : square[0];
    }
  }
  group_sums<S>(square, part[1]);
  const float rstd = 1.f / sqrtf(__builtin_fmaf(square[0], a.inv_d, a.eps));
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Span<T, NARROW> s((lane + v * S::kGroup) * P, a.D);
    float w[P], b[P];
    if (a.weight) load_params(a.weight, s, w);
    if (a.bias) load_params(a.bias, s, b);
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const float n = h[v][e] * rstd;
      h[v][e] = __builtin_fmaf(n, a.weight ? w[e] : 1.f, a.bias ? b[e] : 0.f);
    }
    if (live) s.store(static_cast<T*>(a.y) + row * a.ld_y, h[v]);
  }
  if (live && lane == 0) {
    a.mean[row] = mean;
    a.rstd[row] = rstd;
  }
}

template <typename T>
static int norm_launch(const NormArgs& a, hipStream_t st) {
  return norm_shape<T>(a.D, [&](auto shape) {
    using S = decltype(shape);
    auto kernel = a.add ? k_norm<T, S, true, false> : k_norm<T, S, false, false>;
    if constexpr (S::kGroup == 8)
      if (a.D < Patch<T>::P) kernel = a.add ? k_norm<T, S, true, true> : k_norm<T, S, false, true>;
    return launch_parts((a.rows + S::kRows - 1) / S::kRows, S::kThreads,
                        [&](uint32_t first, uint32_t n) {
                          kernel<<<n, S::kThreads, 0, st>>>(a, first);
                          return launch_status(hipGetLastError());
                        });
  });
}

int norm_run(const void* x, int64_t ld_x, const void* add, int64_t ld_add, int64_t rows, int64_t D,
             int dtype, const float* weight, const float* bias, float eps, float p, uint64_t seed,
             const int64_t* seed_at, void* y, int64_t ld_y, void* h, int64_t ld_h, float* mean,
             float* rstd, hipStream_t st) {
  if (rows == 0) return LM_OK;
  const NormArgs a{x, add, weight, bias, y, h, mean, rstd, ld_x, ld_add, ld_y, ld_h, rows,
                   static_cast<int>(D), eps, static_cast<float>(1.0 / static_cast<double>(D)),
                   make_keep(p, seed, seed_at)};
  return dtype == LM_BF16 ? norm_launch<bf16_t>(a, st) : norm_launch<float>(a, st);
}

}  // namespace lmz
