// Layer norm, with dropout and the residual sum before it:
//     h = add + dropout(x),  y = (h - mean) rstd weight + bias,  rstd = 1 / sqrt(var + eps).
// One pass: a row is read once into its group's registers (norm_rows.hpp), its mean and
// then the mean square of what is left are summed in fp32 (two sums, so that rows far from
// zero lose nothing), and y and h are written. HBM bounds it: up to 4 elements for each.
// 65,536 x 2048 bf16, dropout and residual: 187 us, 5.7 TB/s of equal parts read and written
// (28 vector instructions a value).
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

template <typename T, typename S, bool ADD, Ends ENDS>
__global__ __launch_bounds__(S::kThreads) void k_norm(NormArgs a, uint32_t first) {
  constexpr int P = Patch<T>::P, NV = S::NV, R = S::ROWS;
  using raw_t = typename Patch<T>::raw_t;
  __shared__ float part[2][S::kThreads / kWave][R];
  const int64_t i0 = (first + static_cast<int64_t>(blockIdx.x)) * S::kRows + S::group() * R;
  const int lane = threadIdx.x % S::kGroup;
  raw_t rx[R][NV], ra[R][NV];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = i0 + r < a.rows ? i0 + r : a.rows - 1;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const NormSpan<T, ENDS> s((lane + v * S::kGroup) * P, a.D);
      rx[r][v] = s.load(static_cast<const T*>(a.x) + row * a.ld_x);
      if constexpr (ADD) ra[r][v] = s.load(static_cast<const T*>(a.add) + row * a.ld_add);
    }
  }
  float h[R][NV][P], sum[R], square[R];
  const bool drops = a.keep.least != 0;
  const Keep keep(a.keep);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = i0 + r;
    const bool live = row < a.rows;
    sum[r] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const NormSpan<T, ENDS> s((lane + v * S::kGroup) * P, a.D);
      s.widen(rx[r][v], h[r][v]);
      if (drops)
        keep.apply<P>(static_cast<uint64_t>(row) * (static_cast<uint32_t>(a.D + 1) / 2) +
                          (lane + v * S::kGroup) * (P / 2),
                      h[r][v]);
      if constexpr (ADD) {
        float z[P];
        s.widen(ra[r][v], z);
#pragma unroll
        for (int e = 0; e < P; ++e) h[r][v][e] += z[e];
      }
#pragma unroll
      for (int e = 0; e < P; ++e) sum[r] += h[r][v][e];
      if (a.h && live) s.store(static_cast<T*>(a.h) + row * a.ld_h, h[r][v]);
    }
  }
  group_sums<S>(sum, part[0]);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    sum[r] *= a.inv_d;
    square[r] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const NormSpan<T, ENDS> s((lane + v * S::kGroup) * P, a.D);
#pragma unroll
      for (int e = 0; e < P; ++e) {
        h[r][v][e] -= sum[r];
        if (ENDS == Ends::WHOLE ? s.have == 0 : e >= s.have) h[r][v][e] = 0.f;
        square[r] = __builtin_fmaf(h[r][v][e], h[r][v][e], square[r]);
      }
    }
  }
  group_sums<S>(square, part[1]);
#pragma unroll
  for (int r = 0; r < R; ++r)
    square[r] = 1.f / sqrtf(__builtin_fmaf(square[r], a.inv_d, a.eps));
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const NormSpan<T, ENDS> s((lane + v * S::kGroup) * P, a.D);
    float w[P], b[P];
    if (a.weight) load_params(a.weight, s, w);
    if (a.bias) load_params(a.bias, s, b);
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int e = 0; e < P; ++e)
        h[r][v][e] = __builtin_fmaf(h[r][v][e] * square[r], a.weight ? w[e] : 1.f,
                                    a.bias ? b[e] : 0.f);
      if (i0 + r < a.rows)
        s.store(static_cast<T*>(a.y) + (i0 + r) * a.ld_y, h[r][v]);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (lane != 0 || i0 + r >= a.rows) continue;
    a.mean[i0 + r] = sum[r];
    a.rstd[i0 + r] = square[r];
  }
}

// Calls f with the shape for rows of D values of type T. Waves of their own, which wait for
// no other, where there are rows enough to fill the device (65,536 x 2048 bf16: 190 us, 206
// with four waves a row; 4099 x 517 fp32 6.2 and 8.9), short rows two at a time (200,000 x 128
// bf16: 21 us, one at a time 24). Rows that are few are spread over more waves (1 x 2048 bf16:
// 2.3 us with four waves, 3.7 with one; 256 rows 2.9 and 4.3; at 2048 rows both take 8.5), one
// at a time (700 x 128 bf16: 2.6 us, two at a time 3.0; 1000 x 500 4.0 and 4.6).
template <typename T, typename F>
static inline int norm_shape(int64_t rows, int64_t D, F f) {
  constexpr int64_t most = LM_NORM_MAX_WIDTH / Patch<T>::P;
  const int64_t vectors = (D + Patch<T>::P - 1) / Patch<T>::P;
  if (rows <= 1024) {
    if (vectors <= 8) return f(NormShape<8, 1, 1>{});
    if (vectors <= 16) return f(NormShape<16, 1, 1>{});
    if (vectors <= 32) return f(NormShape<32, 1, 1>{});
    if (vectors <= 64) return f(NormShape<64, 1, 1>{});
    if (vectors <= 128) return f(NormShape<64, 2, 1>{});
    if (vectors <= 256) return f(NormShape<64, 4, 1>{});
    if (vectors <= 512) return f(NormShape<64, 8, 1>{});
    if (vectors <= 1024) return f(NormShape<64, 16, 1>{});
  }
  if (vectors <= 8) return f(NormShape<8, 1, 1, 2>{});
  if (vectors <= 16) return f(NormShape<16, 1, 1, 2>{});
  if (vectors <= 32) return f(NormShape<32, 1, 1, 2>{});
  if (vectors <= 64) return f(NormShape<64, 1, 1, 2>{});
  if (vectors <= 128) return f(NormShape<64, 1, 2>{});
  if (vectors <= 192) return f(NormShape<64, 1, 3>{});
  if (vectors <= 256) return f(NormShape<64, 1, 4>{});
  if (vectors <= 512) return f(NormShape<64, 2, 4>{});
  if (vectors <= 1024) return f(NormShape<64, 4, 4>{});
  if constexpr (most <= 2048) return f(NormShape<64, 8, 4>{});
  else return vectors <= 2048 ? f(NormShape<64, 8, 4>{}) : f(NormShape<64, 16, most / 1024>{});
}

template <typename T>
static int norm_launch(const NormArgs& a, hipStream_t st) {
  return norm_shape<T>(a.rows, a.D, [&](auto shape) {
    using S = decltype(shape);
    auto kernel = norm_ends<S>(ends_of(a.D, Patch<T>::P), [&](auto ends) {
      constexpr Ends kEnds = decltype(ends)::value;
      return a.add ? k_norm<T, S, true, kEnds> : k_norm<T, S, false, kEnds>;
    });
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
