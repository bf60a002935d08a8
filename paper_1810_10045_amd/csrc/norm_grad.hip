// Layer norm's backward pass. With n = (h - mean) rstd and g = dy weight:
//     dh = add + rstd (g - E g - n E(g n)),  dx = dropout(dh) (the forward's mask),
//     dweight = sum over rows of dy n,  dbias = sum over rows of dy,
// E the mean over a row. One pass over the rows: a workgroup keeps a row's share in
// registers as the forward pass does, goes through its rows and adds dy n and dy of its own
// columns on the way; its sums are one row of the workspace, and k_norm_join adds those.
// Both orders depend on the sizes only. HBM bounds the pass: 3 to 5 elements for each.
// 65,536 x 2048 bf16 with dropout and the residual's gradient: 236 us with the join's 5, 5.7
// TB/s (42 vector instructions a value); rows loaded a turn ahead, or a wave a row without
// barriers, take as long.
#include "launch_parts.hpp"
#include "norm_rows.hpp"

namespace lmz {

struct NormGradArgs {
  const void *dy, *h, *add;
  const float *mean, *rstd, *weight;
  void *dh, *dx;
  float* sums;  // [workgroups][2][D]: dweight, dbias; or nullptr
  float *dweight, *dbias;  // of a workgroup without others, which writes the results itself
  int accumulate;
  int64_t ld_dy, ld_h, ld_add, ld_dh, ld_dx, rows;
  int D;
  float inv_d;
  KeepArgs keep;
};

constexpr int kSmallThreads = 256;  // of a workgroup of few rows

// The value of an operand that is kept as it was loaded, and not widened, between its uses.
__device__ __forceinline__ f32x4 kept(f32x4 x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ u32x4 kept(u32x4 x) {
  asm volatile("" : "+v"(x));
  return x;
}

template <typename T, typename S, bool ADD, Ends ENDS>
__global__ __launch_bounds__(S::kThreads) void k_norm_grad(NormGradArgs a) {
  constexpr int P = Patch<T>::P, NV = S::NV, R = S::ROWS;
  constexpr int kWaves = S::kThreads / kWave;
  using raw_t = typename Patch<T>::raw_t;
  __shared__ float part[2][kWaves][2 * R];
  const int group = S::group(), lane = threadIdx.x % S::kGroup;
  const Keep keep(a.keep);
  const uint64_t pairs = static_cast<uint64_t>(a.D + 1) / 2;
  float w[NV][P], dw[NV][P], db[NV][P];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const NormSpan<T, ENDS> s((lane + v * S::kGroup) * P, a.D);
    if (a.weight) {
      load_params(a.weight, s, w[v]);  // under way until the first turn uses them
    } else {
#pragma unroll
      for (int e = 0; e < P; ++e) w[v][e] = 1.f;
    }
#pragma unroll
    for (int e = 0; e < P; ++e) dw[v][e] = db[v][e] = 0.f;
  }
  int turn = 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * S::kRows;
  for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * S::kRows; i0 < a.rows; i0 += step) {
    raw_t ry[R][NV], rh[R][NV], ra[R][NV];
    float mean[R], rstd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t i = i0 + group * R + r, row = i < a.rows ? i : a.rows - 1;
      mean[r] = a.mean[row];
      rstd[r] = a.rstd[row];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const NormSpan<T, ENDS> s((lane + v * S::kGroup) * P, a.D);
        ry[r][v] = s.load(static_cast<const T*>(a.dy) + row * a.ld_dy);
        rh[r][v] = s.load(static_cast<const T*>(a.h) + row * a.ld_h);
        if constexpr (ADD) ra[r][v] = s.load(static_cast<const T*>(a.add) + row * a.ld_add);
      }
    }
    // A row behind the last one has only zeros, so it adds nothing.
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (i0 + group * R + r < a.rows) continue;
      mean[r] = rstd[r] = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) ry[r][v] = rh[r][v] = raw_t{0, 0, 0, 0};
    }
    float sums[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float g0 = 0.f, g1 = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const NormSpan<T, ENDS> s((lane + v * S::kGroup) * P, a.D);
        float y[P], n[P];
        s.widen(ry[r][v], y);  // zeros behind the row's end
        s.widen(rh[r][v], n);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          n[e] = (n[e] - mean[r]) * rstd[r];
          const float g = y[e] * w[v][e];
          g0 += g;
          g1 = __builtin_fmaf(g, n[e], g1);
          dw[v][e] = __builtin_fmaf(y[e], n[e], dw[v][e]);
          db[v][e] += y[e];
          // added here, not at the turn's end with every row's y and n waiting for it
          asm volatile("" : "+v"(dw[v][e]), "+v"(db[v][e]));
        }
        ry[r][v] = kept(ry[r][v]);
        rh[r][v] = kept(rh[r][v]);
        __builtin_amdgcn_sched_barrier(0);
      }
      sums[2 * r] = g0;
      sums[2 * r + 1] = g1;
    }
    group_sums<S>(sums, part[turn]);
    turn ^= 1;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = i0 + group * R + r;
      if (row >= a.rows) continue;
      const float e0 = sums[2 * r] * a.inv_d, e1 = sums[2 * r + 1] * a.inv_d;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const NormSpan<T, ENDS> s((lane + v * S::kGroup) * P, a.D);
        float y[P], n[P], z[P];
        s.widen(ry[r][v], y);
        s.widen(rh[r][v], n);
        if constexpr (ADD) s.widen(ra[r][v], z);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          n[e] = (n[e] - mean[r]) * rstd[r];
          const float d = (y[e] * w[v][e] - e0) - n[e] * e1;
          y[e] = __builtin_fmaf(rstd[r], d, ADD ? z[e] : 0.f);
        }
        s.store(static_cast<T*>(a.dh) + row * a.ld_dh, y);
        if (a.dx) {
          keep.apply<P>(static_cast<uint64_t>(row) * pairs + (lane + v * S::kGroup) * (P / 2), y);
          s.store(static_cast<T*>(a.dx) + row * a.ld_dx, y);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  constexpr bool kAlone = S::THREADS == kSmallThreads;  // may have the call to itself
  if (!a.sums && (!kAlone || (!a.dweight && !a.dbias))) return;
  // The groups' sums, added in their order: of a wave by their lanes, of the waves in LDS.
  constexpr int kGroups = S::kThreads / (S::kGroup > kWave ? S::kGroup : kWave);
  constexpr int kCols = S::kGroup * NV * P;
  alignas(16) __shared__ float joined[kGroups > 1 ? kGroups : 1][kGroups > 1 ? kCols : 1];
  auto put = [&](int k, int col, float x) {
    if (!kAlone || a.sums) {
      a.sums[(static_cast<int64_t>(blockIdx.x) * 2 + k) * a.D + col] = x;
    } else if (float* out = k ? a.dbias : a.dweight) {
      out[col] = a.accumulate ? out[col] + x : x;
    }
  };
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k && kGroups > 1) __syncthreads();
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const NormSpan<T, ENDS> s((lane + v * S::kGroup) * P, a.D);
      const int col = (lane + v * S::kGroup) * P;
      float x[P];
#pragma unroll
      for (int e = 0; e < P; ++e) {
        x[e] = k ? db[v][e] : dw[v][e];
#pragma unroll
        for (int off = S::kGroup; off < kWave; off *= 2) x[e] += __shfl_xor(x[e], off, kWave);
      }
      if constexpr (kGroups > 1) {
#pragma unroll
        for (int e = 0; e < P; ++e)
          joined[threadIdx.x / (kGroups > 1 ? S::kThreads / kGroups : 1)][col + e] = x[e];
      } else if (a.sums && s.have == P) {
        // whole vectors: 100 x 16,384 bf16 15.9 us, 26.9 a value at a time
        float* out = a.sums + (static_cast<int64_t>(blockIdx.x) * 2 + k) * a.D + col;
#pragma unroll
        for (int e = 0; e < P; e += 4)
          *reinterpret_cast<f32x4e*>(out + e) = f32x4e{x[e], x[e + 1], x[e + 2], x[e + 3]};
      } else {
#pragma unroll
        for (int e = 0; e < P; ++e)
          if (e < s.have) put(k, col + e, x[e]);
      }
    }
    if constexpr (kGroups > 1) {
      __syncthreads();
      for (int c = threadIdx.x; c < kCols && c < a.D; c += S::kThreads) {
        float x = joined[0][c];
#pragma unroll
        for (int g = 1; g < kGroups; ++g) x += joined[g][c];
        put(k, c, x);
      }
    }
  }
}

// dweight and dbias (+)= the workgroups' sums, COLS columns of the two a workgroup:
// kJoinThreads / COLS threads share a column's parts, their sums are added in a fixed order.
constexpr int kJoinThreads = 1024, kJoinWaves = kJoinThreads / kWave;

template <int COLS>
__global__ __launch_bounds__(kJoinThreads) void k_norm_join(const float* sums, int parts, int D,
                                                            float* dweight, float* dbias,
                                                            int accumulate) {
  __shared__ float lds[kJoinWaves][COLS];
  const int col = threadIdx.x % COLS, wave = threadIdx.x / kWave;
  const int c = blockIdx.x * COLS + col;
  const float* at = sums + (c < 2 * D ? c : 0);
  float x = 0.f;
#pragma unroll 8
  for (int g = threadIdx.x / COLS; g < parts; g += kJoinThreads / COLS)
    x += at[static_cast<int64_t>(g) * 2 * D];
#pragma unroll
  for (int off = COLS; off < kWave; off *= 2) x += __shfl_xor(x, off, kWave);
  if (threadIdx.x % kWave < COLS) lds[wave][col] = x;
  __syncthreads();
  if (threadIdx.x >= COLS || c >= 2 * D) return;
  float y = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) y += lds[w][col];
  float* out = c < D ? dweight : dbias;
  if (!out) return;
  out += c < D ? c : c - D;
  *out = accumulate ? *out + y : y;
}

// Calls f with the shape for rows of D values of type T, in workgroups of THREADS that take up
// to MOST rows a group at once.
template <typename T, int THREADS, int MOST, typename F>
static inline int grad_shape(int64_t D, F f) {
  constexpr int P = Patch<T>::P;
  const int64_t vectors = (D + P - 1) / P;
  if (vectors <= 8) return f(NormShape<8, 1, 1, MOST, THREADS>{});
  if (vectors <= 16) return f(NormShape<16, 1, 1, MOST, THREADS>{});
  if (vectors <= 32) return f(NormShape<32, 1, 1, MOST, THREADS>{});
  if (vectors <= 64) return f(NormShape<64, 1, 1, MOST, THREADS>{});
  if (D <= 512) return f(NormShape<64, 1, 8 / P, MOST, THREADS>{});
  if (D <= 1024) return f(NormShape<64, 2, 8 / P, MOST, THREADS>{});
  if (D <= 2048) return f(NormShape<64, 4, 8 / P, MOST, THREADS>{});
  if (D <= 4096) return f(NormShape<64, 4, 16 / P, 1, THREADS>{});
  if (D <= 8192) return f(NormShape<64, 8, 16 / P, 1, THREADS>{});
  static_assert(LM_NORM_MAX_WIDTH == 16384, "the widest shape");
  return f(NormShape<64, 16, 16 / P, 1, THREADS>{});
}

// Workgroups of the pass, at most kGradBlocks. Each leaves 2 D sums behind, so that fewer and
// larger ones cost less where every one has but a turn or two: 1280 x 1792 fp32 takes 11.3 us
// with 160 of 1024 threads, 13.4 with 320 of 512 (2048 x 2048 bf16 14.5 and 16.3). Where every
// one has many turns the smaller ones do: 16,384 x 1000 fp32 40.3 us with them, 42.4 with 1024.
constexpr int64_t kGradBlocks = 512;

// Rows that kGradSmall workgroups of one wave a SIMD would hold, a row a group, go to such small
// ones, as the instructions of the four waves of a larger one follow each other: 700 x 480 bf16
// takes 6.2 us, 7.0 otherwise, 16,384 x 35 8.5 and 10.7, 200 x 650 fp32 7.1 and 9.7, 200 x 2048
// bf16 8.1 and 8.4. These too are kGradBlocks at most: twice as many rows have two turns, as each
// workgroup's sums cost the join more than a turn takes (30,000 x 35 bf16: 10.0 us, with up to
// kGradSmall workgroups 12.3, with larger ones 11.5; 22,882 x 35 9.3, 10.1 and 10.9). More sums
// than kGradSums cost what small workgroups save, or half as many where several rows' are added
// first (900 x 1000 bf16: 11.8 and 9.7).
constexpr int64_t kGradSmall = 1024, kGradSums = int64_t(1) << 20;
// Rows of one of the larger workgroups, at most eight times a small one's, always fit.
static_assert(kGradSums / 2 / (2 * LM_NORM_MAX_WIDTH) >= 8 && kSmallThreads * 8 == 1024 * 2, "");

template <typename T, typename F>
static inline int norm_grad_shape(int64_t rows, int64_t D, F f) {
  const auto fit = [rows](int64_t blocks) {
    return [rows, blocks](auto shape) { return rows <= blocks * decltype(shape)::kRows ? 1 : 0; };
  };
  const bool small = grad_shape<T, kSmallThreads, 1>(D, [&](auto shape) {
    const int64_t most = (decltype(shape)::kGroups > 1 ? kGradSums / 2 : kGradSums) / (2 * D);
    return fit(most < kGradSmall ? most : kGradSmall)(shape);
  });
  if (small) return grad_shape<T, kSmallThreads, 1>(D, f);
  return grad_shape<T, 512, 2>(D, fit(kGradBlocks)) ? grad_shape<T, 1024, 2>(D, f)
                                                    : grad_shape<T, 512, 2>(D, f);
}

template <typename T>
static int64_t grad_blocks(int64_t rows, int64_t D) {
  return norm_grad_shape<T>(rows, D, [&](auto shape) {
    using S = decltype(shape);
    const int64_t n = (rows + S::kRows - 1) / S::kRows;  // turns
    // Of 16 waves a compute unit has but one: 2000 x 16,384 bf16 66 us, with 512 of them 77.
    constexpr int64_t most = S::kGroup == 1024 ? kGradBlocks / 2 : kGradBlocks;
    return static_cast<int>(n < most ? n : most);
  });
}
static int64_t norm_grad_blocks(int64_t rows, int64_t D, int dtype) {
  return dtype == LM_BF16 ? grad_blocks<bf16_t>(rows, D) : grad_blocks<float>(rows, D);
}

size_t norm_grad_workspace_bytes(int64_t rows, int64_t D, int dtype) {
  const int64_t blocks = norm_grad_blocks(rows, D, dtype);
  return blocks <= 1 ? 0 : static_cast<size_t>(blocks) * 2 * D * sizeof(float);
}

template <typename T>
static int norm_grad_launch(const NormGradArgs& a, int blocks, hipStream_t st) {
  return norm_grad_shape<T>(a.rows, a.D, [&](auto shape) {
    using S = decltype(shape);
    auto kernel = norm_ends<S>(ends_of(a.D, Patch<T>::P), [&](auto ends) {
      constexpr Ends kEnds = decltype(ends)::value;
      return a.add ? k_norm_grad<T, S, true, kEnds> : k_norm_grad<T, S, false, kEnds>;
    });
    kernel<<<blocks, S::kThreads, 0, st>>>(a);
    return launch_status(hipGetLastError());
  });
}

int norm_grad_run(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, const void* add,
                  int64_t ld_add, int64_t rows, int64_t D, int dtype, const float* mean,
                  const float* rstd, const float* weight, float p, uint64_t seed,
                  const int64_t* seed_at, void* dh, int64_t ld_dh, void* dx, int64_t ld_dx,
                  float* dweight, float* dbias, int accumulate, void* ws, hipStream_t st) {
  const int blocks = static_cast<int>(norm_grad_blocks(rows, D, dtype));
  const bool join = (dweight || dbias) && blocks != 1;
  float* sums = static_cast<float*>(ws);
  if (rows > 0) {
    const NormGradArgs a{dy, h, add, mean, rstd, weight, dh, dx,
                         join ? sums : nullptr, dweight, dbias, accumulate, ld_dy, ld_h, ld_add,
                         ld_dh, ld_dx, rows, static_cast<int>(D),
                         static_cast<float>(1.0 / static_cast<double>(D)),
                         make_keep(p, seed, dx ? seed_at : nullptr)};
    const int rc = dtype == LM_BF16 ? norm_grad_launch<bf16_t>(a, blocks, st)
                                    : norm_grad_launch<float>(a, blocks, st);
    if (rc != LM_OK) return rc;
  }
  if (!join) return LM_OK;
  // Columns of a workgroup: few where there would be no workgroup for each compute unit (200 x
  // 650 fp32: 7.1 us with 16, 7.5 with 32; 900 x 1000 bf16 9.7 and 9.9), else whole cache lines
  // (2048 x 2048 14.5 with 32, 16.1 with 16; 100 x 16,384 15.8 with 64, 16.8 with 32, 21.9 with 16).
  const int cols = static_cast<int>(2 * D), each = D <= 1024 ? 16 : D <= 4096 ? 32 : 64;
  auto kernel = each == 16 ? k_norm_join<16> : each == 32 ? k_norm_join<32> : k_norm_join<64>;
  kernel<<<(cols + each - 1) / each, kJoinThreads, 0, st>>>(
      sums, blocks, static_cast<int>(D), dweight, dbias, accumulate);
  return launch_status(hipGetLastError());
}

}  // namespace lmz
