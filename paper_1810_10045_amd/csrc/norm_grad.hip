// Layer norm's backward pass. With n = (h - mean) rstd and g = dy weight:
//     dh = add + rstd (g - E g - n E(g n)),  dx = dropout(dh) (the forward's mask),
//     dweight = sum over rows of dy n,  dbias = sum over rows of dy,
// E the mean over a row. One pass over the rows: a workgroup keeps a row's share in
// registers as the forward pass does, goes through its rows and adds dy n and dy of its own
// columns on the way; its sums are one row of the workspace, and k_norm_join adds those.
// Both orders depend on the sizes only. HBM bounds the pass: 3 to 5 elements for each.
#include "launch_parts.hpp"
#include "norm_rows.hpp"

namespace lmz {

struct NormGradArgs {
  const void *dy, *h, *add;
  const float *mean, *rstd, *weight;
  void *dh, *dx;
  float* sums;  // [workgroups][2][D]: dweight, dbias; or nullptr
  int64_t ld_dy, ld_h, ld_add, ld_dh, ld_dx, rows;
  int D;
  float inv_d;
  KeepArgs keep;
};

// Rows of a group that are under way at once.
template <typename S>
constexpr int kBatch = S::NV >= 4 ? 1 : S::NV >= 2 ? 2 : 4;

template <typename T, typename S, bool ADD, bool NARROW>
__global__ __launch_bounds__(S::kThreads) void k_norm_grad(NormGradArgs a) {
  constexpr int P = Patch<T>::P, NV = S::NV, R = kBatch<S>;
  constexpr int kWaves = S::kThreads / kWave;
  using raw_t = typename Patch<T>::raw_t;
  __shared__ float part[2][kWaves][2 * R];
  const int group = threadIdx.x / S::kGroup, lane = threadIdx.x % S::kGroup;
  const Keep keep(a.keep);
  const uint64_t pairs = static_cast<uint64_t>(a.D + 1) / 2;
  float w[NV][P], dw[NV][P], db[NV][P];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Span<T, NARROW> s((lane + v * S::kGroup) * P, a.D);
    if (a.weight) load_params(a.weight, s, w[v]);
#pragma unroll
    for (int e = 0; e < P; ++e) {
      w[v][e] = a.weight ? w[v][e] : 1.f;
      dw[v][e] = db[v][e] = 0.f;
    }
  }
  int turn = 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * S::kRows * R;
  for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * S::kRows * R; i0 < a.rows; i0 += step) {
    raw_t ry[R][NV], rh[R][NV], ra[R][NV];
    float mean[R], rstd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t i = i0 + group * R + r, row = i < a.rows ? i : a.rows - 1;
      mean[r] = a.mean[row];
      rstd[r] = a.rstd[row];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Span<T, NARROW> s((lane + v * S::kGroup) * P, a.D);
        ry[r][v] = s.load(static_cast<const T*>(a.dy) + row * a.ld_dy);
        rh[r][v] = s.load(static_cast<const T*>(a.h) + row * a.ld_h);
        if constexpr (ADD) ra[r][v] = s.load(static_cast<const T*>(a.add) + row * a.ld_add);
      }
    }
    float sums[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool live = i0 + group * R + r < a.rows;
      float g0 = 0.f, g1 = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Span<T, NARROW> s((lane + v * S::kGroup) * P, a.D, live);
        const Span<T, NARROW> at((lane + v * S::kGroup) * P, a.D);
        float y[P], n[P];
        at.widen(ry[r][v], y);
        at.widen(rh[r][v], n);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          n[e] = (n[e] - mean[r]) * rstd[r];
          const float g = y[e] * w[v][e];
          const bool in = e < s.have;
          g0 += in ? g : 0.f;
          g1 = in ? __builtin_fmaf(g, n[e], g1) : g1;
          dw[v][e] = in ? __builtin_fmaf(y[e], n[e], dw[v][e]) : dw[v][e];
          db[v][e] += in ? y[e] : 0.f;
        }
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
        const Span<T, NARROW> s((lane + v * S::kGroup) * P, a.D);
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
      }
    }
  }
  if (!a.sums) return;
  // The groups' sums, added in their order: of a wave by their lanes, of the waves in LDS.
  constexpr int kGroups = S::kThreads / (S::kGroup > kWave ? S::kGroup : kWave);
  constexpr int kCols = S::kGroup * NV * P;
  __shared__ float joined[kGroups > 1 ? kGroups : 1][kGroups > 1 ? kCols : 1];
  float* mine = a.sums + static_cast<int64_t>(blockIdx.x) * 2 * a.D;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k && kGroups > 1) __syncthreads();
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Span<T, NARROW> s((lane + v * S::kGroup) * P, a.D);
#pragma unroll
      for (int e = 0; e < P; ++e) {
        float x = k ? db[v][e] : dw[v][e];
#pragma unroll
        for (int off = S::kGroup; off < kWave; off *= 2) x += __shfl_xor(x, off, kWave);
        const int col = (lane + v * S::kGroup) * P + e;
        if constexpr (kGroups > 1) {
          joined[threadIdx.x / (kGroups > 1 ? S::kThreads / kGroups : 1)][col] = x;
        } else if (e < s.have) {
          mine[k * a.D + col] = x;
        }
      }
    }
    if constexpr (kGroups > 1) {
      __syncthreads();
      for (int c = threadIdx.x; c < kCols && c < a.D; c += S::kThreads) {
        float x = joined[0][c];
#pragma unroll
        for (int g = 1; g < kGroups; ++g) x += joined[g][c];
        mine[k * a.D + c] = x;
      }
    }
  }
}

// dweight and dbias (+)= the workgroups' sums, 64 columns of the two a workgroup: a wave
// adds every kJoinWaves-th row, the waves are added in their order.
constexpr int kJoinWaves = 16;

__global__ __launch_bounds__(kJoinWaves* kWave) void k_norm_join(const float* sums, int parts,
                                                                 int D, float* dweight,
                                                                 float* dbias, int accumulate) {
  __shared__ float lds[kJoinWaves][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = blockIdx.x * kWave + lane;
  const float* at = sums + (c < 2 * D ? c : 0);
  float x = 0.f;
#pragma unroll 8
  for (int g = wave; g < parts; g += kJoinWaves) x += at[static_cast<int64_t>(g) * 2 * D];
  lds[wave][lane] = x;
  __syncthreads();
  if (wave || c >= 2 * D) return;
  float y = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) y += lds[w][lane];
  float* out = c < D ? dweight : dbias;
  if (!out) return;
  out += c < D ? c : c - D;
  *out = accumulate ? *out + y : y;
}

constexpr int kNormGradBlocks = 512;  // two on each compute unit

// Workgroups of the pass.
static int64_t norm_grad_blocks(int64_t rows, int64_t D, int dtype) {
  auto blocks = [&](auto shape) {
    using S = decltype(shape);
    const int64_t n = (rows + S::kRows * kBatch<S> - 1) / (S::kRows * kBatch<S>);
    return static_cast<int>(n < kNormGradBlocks ? n : kNormGradBlocks);
  };
  return dtype == LM_BF16 ? norm_shape<bf16_t>(D, blocks) : norm_shape<float>(D, blocks);
}

size_t norm_grad_workspace_bytes(int64_t rows, int64_t D, int dtype) {
  return static_cast<size_t>(norm_grad_blocks(rows, D, dtype)) * 2 * D * sizeof(float);
}

template <typename T>
static int norm_grad_launch(const NormGradArgs& a, int blocks, hipStream_t st) {
  return norm_shape<T>(a.D, [&](auto shape) {
    using S = decltype(shape);
    auto kernel = a.add ? k_norm_grad<T, S, true, false> : k_norm_grad<T, S, false, false>;
    if constexpr (S::kGroup == 8)
      if (a.D < Patch<T>::P)
        kernel = a.add ? k_norm_grad<T, S, true, true> : k_norm_grad<T, S, false, true>;
    kernel<<<blocks, S::kThreads, 0, st>>>(a);
    return launch_status(hipGetLastError());
  });
}

int norm_grad_run(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, const void* add,
                  int64_t ld_add, int64_t rows, int64_t D, int dtype, const float* mean,
                  const float* rstd, const float* weight, float p, uint64_t seed,
                  const int64_t* seed_at, void* dh, int64_t ld_dh, void* dx, int64_t ld_dx,
                  float* dweight, float* dbias, int accumulate, void* ws, hipStream_t st) {
  const bool sums = dweight || dbias;
  const int blocks = static_cast<int>(norm_grad_blocks(rows, D, dtype));
  if (rows > 0) {
    const NormGradArgs a{dy, h, add, mean, rstd, weight, dh, dx,
                         sums ? static_cast<float*>(ws) : nullptr, ld_dy, ld_h, ld_add, ld_dh,
                         ld_dx, rows, static_cast<int>(D),
                         static_cast<float>(1.0 / static_cast<double>(D)),
                         make_keep(p, seed, seed_at)};
    const int rc = dtype == LM_BF16 ? norm_grad_launch<bf16_t>(a, blocks, st)
                                    : norm_grad_launch<float>(a, blocks, st);
    if (rc != LM_OK) return rc;
  }
  if (!sums) return LM_OK;
  const int cols = static_cast<int>(2 * D);
  k_norm_join<<<(cols + kWave - 1) / kWave, kJoinWaves * kWave, 0, st>>>(
      static_cast<const float*>(ws), blocks, static_cast<int>(D), dweight, dbias, accumulate);
  return launch_status(hipGetLastError());
}

}  // namespace lmz
