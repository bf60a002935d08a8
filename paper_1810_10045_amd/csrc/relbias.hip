// A learned relative position bias and its gradient: out[b, h, i, j] is
// table[bucket(r), h] for the distance r = j - (q_start + i) of key j from query
// i. The buckets are segments of the distance axis: segment s covers the
// distances from starts[s] up to starts[s + 1], and ids[s] names its table row
// (-1: masked).
//
// A head's bias depends on j - i only. The kernels work on square patches of
// kP rows and columns (a column vector of 16 bytes): 2 kP - 1 diagonals, each
// one number. The bias of a patch is that many values in registers; the
// gradient adds a patch into that many sums, and the patch one step down and
// right has the same diagonals, so a wave that walks down the diagonal keeps its
// sums in registers through the whole matrix. Each element of the matrices is
// read or written once: HBM bounds both.
#include "common.hpp"

namespace lmz {

constexpr int kRelThreads = 256;
constexpr int kRelWaves = kRelThreads / kWave;

struct Segments {
  int32_t starts[LM_REL_MAX_SEGMENTS];
  int16_t ids[LM_REL_MAX_SEGMENTS];
  int32_t n;
};

// The last segment that starts at or before r (starts[0] is below every distance).
__device__ __forceinline__ int segment_of(const int32_t* starts, int n, int r) {
  int lo = 0, hi = n;  // starts[lo] <= r < starts[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid] <= r) lo = mid; else hi = mid;
  }
  return lo;
}

// kP values of a row: 16 bytes at the alignment of an element.
template <typename T>
struct Patch;

template <>
struct Patch<float> {
  static constexpr int P = 4;
  using raw_t = f32x4;
  static __device__ __forceinline__ raw_t load(const float* p) {
    return *reinterpret_cast<const f32x4e*>(p);
  }
  static __device__ __forceinline__ raw_t part(const float* p, int have) {
    return f32x4{have > 0 ? p[0] : 0.f, have > 1 ? p[1] : 0.f, have > 2 ? p[2] : 0.f, 0.f};
  }
  static __device__ __forceinline__ void widen(const raw_t& r, float* x) {
    x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w;
  }
  static __device__ __forceinline__ void store(float* p, int have, const float* x) {
    if (have >= P) {
      *reinterpret_cast<f32x4e*>(p) = f32x4e{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
      for (int e = 0; e < P; ++e)
        if (e < have) p[e] = x[e];
    }
  }
};

template <>
struct Patch<bf16_t> {
  static constexpr int P = 8;
  using raw_t = u32x4;
  static __device__ __forceinline__ raw_t load(const bf16_t* p) {
    return *reinterpret_cast<const u32x4e*>(p);
  }
  static __device__ __forceinline__ raw_t part(const bf16_t* p, int have) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = 2 * e < have ? p[2 * e].bits : 0u;
      w[e] |= (2 * e + 1 < have ? uint32_t(p[2 * e + 1].bits) : 0u) << 16;
    }
    return u32x4{w[0], w[1], w[2], w[3]};
  }
  static __device__ __forceinline__ void widen(const raw_t& r, float* x) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint32_t bits(float x) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
  }
  static __device__ __forceinline__ void store(bf16_t* p, int have, const float* x) {
    if (have >= P) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = bits(x[2 * e]) | bits(x[2 * e + 1]) << 16;
      *reinterpret_cast<u32x4e*>(p) = w;
    } else {
#pragma unroll
      for (int e = 0; e < P; ++e)
        if (e < have) p[e].bits = static_cast<uint16_t>(bits(x[e]));
    }
  }
};

struct Strides {
  int64_t b, h, q;
};

// ---------------------------------------------------------------------------
// The bias, written or added. A workgroup covers kRelRows rows and one wave's
// width of columns of one head, for every batch entry: it looks up the numbers
// of its diagonals once, in LDS, and each wave takes patches from there.
// ---------------------------------------------------------------------------
constexpr int kRelRows = 64;

template <typename T, bool ADD>
__global__ __launch_bounds__(kRelThreads) void k_rel_bias(
    const float* __restrict__ table, int64_t ld_table, Segments seg, int B, int Lq, int Lk,
    int q_start, const T* add, Strides sa, T* out, Strides so, int col_tiles, int row_tiles) {
  constexpr int P = Patch<T>::P;
  constexpr int kCols = kWave * P;
  constexpr int kLine = kRelRows + kCols;
  __shared__ __attribute__((aligned(16))) float line[kLine];
  __shared__ int32_t starts[LM_REL_MAX_SEGMENTS];
  for (int s = threadIdx.x; s < seg.n; s += kRelThreads) starts[s] = seg.starts[s];
  __syncthreads();
  const int ct = blockIdx.x % col_tiles, rest = blockIdx.x / col_tiles;
  const int rt = rest % row_tiles, h = rest / row_tiles;
  const int row0 = rt * kRelRows, col0 = ct * kCols;
  // line[x]: column c of row r has x = c - r + kRelRows - 1 (c, r from the tile's corner)
  const int base = col0 - row0 - q_start - (kRelRows - 1);
  for (int x = threadIdx.x; x < kLine; x += kRelThreads) {
    const int id = seg.ids[segment_of(starts, seg.n, base + x)];
    line[x] = id < 0 ? -__builtin_inff() : table[id * ld_table + h];
  }
  __syncthreads();
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const int col = col0 + lane * P, have = Lk - col;
  if (have <= 0) return;
  for (int r = wave * P; r < kRelRows; r += kRelWaves * P) {
    const int row = row0 + r;
    if (row >= Lq) break;
    const int nr = Lq - row < P ? Lq - row : P;
    float d[2 * P];  // d[k]: diagonal k - (P - 1) of the patch
    const int at = lane * P + kRelRows - P - r;
#pragma unroll
    for (int k = 0; k < 2 * P; k += 4) {
      const f32x4 t = *reinterpret_cast<const f32x4*>(&line[at + k]);
      d[k] = t.x; d[k + 1] = t.y; d[k + 2] = t.z; d[k + 3] = t.w;
    }
    bool masked = true;  // a patch that is masked as a whole is not read
#pragma unroll
    for (int k = 0; k < 2 * P - 1; ++k) masked &= d[k] == -__builtin_inff();
    for (int b = 0; b < B; ++b) {
      T* o = out + b * so.b + h * so.h + static_cast<int64_t>(row) * so.q + col;
      const T* a = ADD ? add + b * sa.b + h * sa.h + static_cast<int64_t>(row) * sa.q + col
                       : nullptr;
      // Every load of the patch before its first store: out may be add, so the
      // compiler keeps a load behind the stores before it.
      typename Patch<T>::raw_t raw[P];
      if (ADD && !masked) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const T* ai = a + (i < nr ? i : 0) * sa.q;
          raw[i] = have >= P ? Patch<T>::load(ai) : Patch<T>::part(ai, have);
        }
      }
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (i >= nr) break;
        float x[P];
        if (ADD && !masked) {
          Patch<T>::widen(raw[i], x);
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const float y = d[P - 1 - i + e];
            x[e] = y == -__builtin_inff() ? y : x[e] + y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < P; ++e) x[e] = d[P - 1 - i + e];
        }
        Patch<T>::store(o + i * so.q, have, x);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The gradient. Patches are numbered along a line: patch diagonal q has its
// column c = P * (t + q - (nt - 1)) at row group t (nt groups of P rows), so it
// starts at the matrix's lower left corner and ends at its upper right. A wave
// takes 64 neighbouring patch diagonals (a band), some row groups and some
// batch entries of one head. Its 2P - 1 sums of a lane are added by segment at
// the end and written to the workspace; k_rel_join adds the waves' sums in
// their order, so results are the same from run to run.
// ---------------------------------------------------------------------------
struct GradPlan {
  int bands, row_parts, batch_parts;  // waves of a head: their product
  int groups;                         // row groups of a part
  int batches;                        // batch entries of a part
};

template <typename T>
__global__ __launch_bounds__(kRelThreads) void k_rel_grad(
    const T* __restrict__ dout, Strides sd, Segments seg, int H, int B, int Lq, int Lk,
    int q_start, GradPlan g, int waves, float* __restrict__ ws) {
  constexpr int P = Patch<T>::P;
  __shared__ int32_t starts[LM_REL_MAX_SEGMENTS + 1];
  for (int s = threadIdx.x; s < seg.n; s += kRelThreads) starts[s] = seg.starts[s];
  if (threadIdx.x == 0) starts[seg.n] = INT32_MAX;
  __syncthreads();
  const int lane = lane_id();
  const int64_t all = first_lane(static_cast<int64_t>(blockIdx.x) * kRelWaves + (threadIdx.x >> 6));
  if (all >= static_cast<int64_t>(waves) * H) return;
  const int h = static_cast<int>(all / waves), w = static_cast<int>(all % waves);
  const int band = w % g.bands, rest = w / g.bands;
  const int rp = rest % g.row_parts, bp = rest / g.row_parts;
  const int nt = (Lq + P - 1) / P, nk = (Lk + P - 1) / P;
  const int q = band * kWave + lane;
  // the groups where this band meets the matrix
  int t0 = rp * g.groups, t1 = t0 + g.groups < nt ? t0 + g.groups : nt;
  const int first = nt - 1 - (band * kWave + kWave - 1), last = nt - 1 - band * kWave + nk;
  if (first > t0) t0 = first;
  if (last < t1) t1 = last;
  const int b0 = bp * g.batches, b1 = b0 + g.batches < B ? b0 + g.batches : B;
  // lane's diagonal k has distance r0 + k; the wave's distances are w0 to w1
  const int r0 = P * (q - (nt - 1)) - q_start - (P - 1);
  const int w0 = r0 - lane * P, w1 = w0 + (kWave - 1) * P + 2 * P - 2;
  // a patch whose distances are all masked is not read
  const int own = segment_of(starts, seg.n, r0);
  const bool masked = starts[own + 1] > r0 + 2 * P - 2 && seg.ids[own] < 0;
  float acc[2 * P - 1];
#pragma unroll
  for (int k = 0; k < 2 * P - 1; ++k) acc[k] = 0.f;
  for (int b = b0; b < b1; ++b) {
    for (int t = t0; t < t1; ++t) {
      const int col = P * (t + q - (nt - 1)), have = Lk - col;
      if (col < 0 || have <= 0 || masked) continue;
      const int nr = Lq - t * P < P ? Lq - t * P : P;
      const T* p = dout + b * sd.b + h * sd.h + static_cast<int64_t>(t) * P * sd.q + col;
      typename Patch<T>::raw_t raw[P];
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const T* pi = p + (i < nr ? i : 0) * sd.q;
        raw[i] = have >= P ? Patch<T>::load(pi) : Patch<T>::part(pi, have);
      }
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float x[P];
        Patch<T>::widen(raw[i], x);
#pragma unroll
        for (int e = 0; e < P; ++e) acc[P - 1 - i + e] += i < nr ? x[e] : 0.f;
      }
    }
  }
  // Segment sums of the wave's distances; most waves lie in one or two segments.
  float* mine = ws + (static_cast<int64_t>(h) * waves + w) * seg.n;
  const int s0 = segment_of(starts, seg.n, w0), s1 = segment_of(starts, seg.n, w1);
  for (int s = lane; s < seg.n; s += kWave)
    if (s < s0 || s > s1) mine[s] = 0.f;
  for (int s = s0; s <= s1; ++s) {
    const int lo = starts[s], hi = starts[s + 1];
    float x = 0.f;
#pragma unroll
    for (int k = 0; k < 2 * P - 1; ++k) x += r0 + k >= lo && r0 + k < hi ? acc[k] : 0.f;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, kWave);
    if (lane == 0) mine[s] = x;
  }
}

// dtable[n, h] (+)= the sums of the segments with id n over a head's waves. One
// workgroup per head: a thread adds one segment (a column of the workspace) over
// every kJoinThreads / width-th wave, so neighbouring threads read neighbouring
// words, and the threads of a segment are added in their order.
constexpr int kJoinThreads = 1024;

__global__ __launch_bounds__(kJoinThreads) void k_rel_join(
    const float* __restrict__ ws, Segments seg, int waves, int num_buckets,
    float* __restrict__ dtable, int64_t ld_table, int accumulate) {
  __shared__ float part[kJoinThreads];
  __shared__ float sums[LM_REL_MAX_SEGMENTS];
  const int h = blockIdx.x, n = seg.n;
  int width = 32;  // segments of one turn
  while (width < n && width < kJoinThreads) width *= 2;
  const int column = threadIdx.x % width, first = threadIdx.x / width, step = kJoinThreads / width;
  const float* mine = ws + static_cast<int64_t>(h) * waves * n;
  float x = 0.f;
  if (column < n) {
#pragma unroll 8
    for (int w = first; w < waves; w += step) x += mine[static_cast<int64_t>(w) * n + column];
  }
  part[threadIdx.x] = x;
  __syncthreads();
  if (threadIdx.x < n) {
    float y = 0.f;
    for (int g = 0; g < step; ++g) y += part[g * width + threadIdx.x];
    sums[threadIdx.x] = y;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < num_buckets; b += kJoinThreads) {
    float y = 0.f;
    for (int s = 0; s < n; ++s)
      if (seg.ids[s] == b) y += sums[s];
    float* d = dtable + b * ld_table + h;
    *d = accumulate ? *d + y : y;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
static Segments make_segments(const int32_t* starts, const int32_t* ids, int n) {
  Segments s{};
  s.n = n;
  for (int i = 0; i < n; ++i) {
    s.starts[i] = starts[i];
    s.ids[i] = static_cast<int16_t>(ids[i]);
  }
  return s;
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <typename T>
static void rel_bias_launch(const float* table, int64_t ld_table, const Segments& seg, int64_t B,
                            int64_t H, int64_t Lq, int64_t Lk, int64_t q_start, const void* add,
                            const Strides& sa, void* out, const Strides& so, hipStream_t st) {
  const int64_t ct = ceil_div(Lk, kWave * Patch<T>::P), rt = ceil_div(Lq, kRelRows);
  const dim3 grid(static_cast<uint32_t>(ct * rt * H));
  if (add)
    k_rel_bias<T, true><<<grid, kRelThreads, 0, st>>>(
        table, ld_table, seg, static_cast<int>(B), static_cast<int>(Lq), static_cast<int>(Lk),
        static_cast<int>(q_start), static_cast<const T*>(add), sa, static_cast<T*>(out), so,
        static_cast<int>(ct), static_cast<int>(rt));
  else
    k_rel_bias<T, false><<<grid, kRelThreads, 0, st>>>(
        table, ld_table, seg, static_cast<int>(B), static_cast<int>(Lq), static_cast<int>(Lk),
        static_cast<int>(q_start), nullptr, sa, static_cast<T*>(out), so, static_cast<int>(ct),
        static_cast<int>(rt));
}

// Workgroups of a call, for the check of the grid's size.
int64_t rel_bias_blocks(int64_t H, int64_t Lq, int64_t Lk, int dtype) {
  const int P = dtype == LM_BF16 ? Patch<bf16_t>::P : Patch<float>::P;
  return ceil_div(Lk, kWave * P) * ceil_div(Lq, kRelRows) * H;
}

int rel_bias_run(const float* table, int64_t ld_table, const int32_t* starts, const int32_t* ids,
                 int n_seg, int64_t B, int64_t H, int64_t Lq, int64_t Lk, int64_t q_start,
                 const void* add, const int64_t* sa, void* out, const int64_t* so, int dtype,
                 hipStream_t st) {
  if (B == 0 || H == 0 || Lq == 0 || Lk == 0) return LM_OK;
  const Segments seg = make_segments(starts, ids, n_seg);
  const Strides a = add ? Strides{sa[0], sa[1], sa[2]} : Strides{0, 0, 0};
  const Strides o{so[0], so[1], so[2]};
  if (dtype == LM_BF16)
    rel_bias_launch<bf16_t>(table, ld_table, seg, B, H, Lq, Lk, q_start, add, a, out, o, st);
  else
    rel_bias_launch<float>(table, ld_table, seg, B, H, Lq, Lk, q_start, add, a, out, o, st);
  return launch_status(hipGetLastError());
}

// How a head's matrices are shared out among waves: about 64 KB for each, and
// at least 16 waves for each compute unit of the device where there is that much.
static GradPlan grad_plan(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int dtype) {
  const int P = dtype == LM_BF16 ? Patch<bf16_t>::P : Patch<float>::P;
  const int64_t nt = ceil_div(Lq, P), nk = ceil_div(Lk, P);
  GradPlan g;
  g.bands = static_cast<int>(ceil_div(nt - 1 + nk, kWave));
  const int64_t steps = nt * B;                    // a band's steps of P rows, all batch entries
  int64_t per = steps * g.bands * H / 4096;        // for 4096 waves
  per = per < 1 ? 1 : per > 16 ? 16 : per;
  g.groups = static_cast<int>(per < nt ? per : nt);
  g.row_parts = static_cast<int>(ceil_div(nt, g.groups));
  const int64_t nb = per / g.groups;
  g.batches = static_cast<int>(nb < 1 ? 1 : nb < B ? nb : B);
  g.batch_parts = static_cast<int>(ceil_div(B, g.batches));
  return g;
}

// Waves of one head; 0 where there is nothing to add.
int64_t rel_grad_waves(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int dtype) {
  if (B == 0 || H == 0 || Lq == 0 || Lk == 0) return 0;
  const GradPlan g = grad_plan(B, H, Lq, Lk, dtype);
  return static_cast<int64_t>(g.bands) * g.row_parts * g.batch_parts;
}

int rel_grad_run(const void* dout, int dtype, int64_t B, int64_t H, int64_t Lq, int64_t Lk,
                 const int64_t* sd, int64_t q_start, const int32_t* starts, const int32_t* ids,
                 int n_seg, int num_buckets, float* dtable, int64_t ld_table, int accumulate,
                 void* ws, hipStream_t st) {
  if (H == 0) return LM_OK;
  const Segments seg = make_segments(starts, ids, n_seg);
  const int64_t waves = rel_grad_waves(B, H, Lq, Lk, dtype);
  if (waves) {
    const GradPlan g = grad_plan(B, H, Lq, Lk, dtype);
    const Strides s{sd[0], sd[1], sd[2]};
    const dim3 grid(static_cast<uint32_t>(ceil_div(waves * H, kRelWaves)));
    if (dtype == LM_BF16)
      k_rel_grad<bf16_t><<<grid, kRelThreads, 0, st>>>(
          static_cast<const bf16_t*>(dout), s, seg, static_cast<int>(H), static_cast<int>(B),
          static_cast<int>(Lq), static_cast<int>(Lk), static_cast<int>(q_start), g,
          static_cast<int>(waves), static_cast<float*>(ws));
    else
      k_rel_grad<float><<<grid, kRelThreads, 0, st>>>(
          static_cast<const float*>(dout), s, seg, static_cast<int>(H), static_cast<int>(B),
          static_cast<int>(Lq), static_cast<int>(Lk), static_cast<int>(q_start), g,
          static_cast<int>(waves), static_cast<float*>(ws));
    const int rc = launch_status(hipGetLastError());
    if (rc != LM_OK) return rc;
  }
  k_rel_join<<<static_cast<uint32_t>(H), kJoinThreads, 0, st>>>(
      static_cast<const float*>(ws), seg, static_cast<int>(waves), num_buckets, dtable, ld_table,
      accumulate);
  return launch_status(hipGetLastError());
}

// The segments of the logarithmic buckets. One side has n buckets: distance d
// below near = n / 2 is bucket d; above, bucket near + t starts at the smallest
// d with d^N >= near^(N - t) * far^t, N = n - near (a whole-number form of
// floor(N log(d / near) / log(far / near)) >= t, so borders are exact). The
// products have up to N * 24 bits and are kept in limbs of 32.
struct Product {
  // Up to LM_REL_MAX_SEGMENTS factors below 2^24: 24 bits each.
  uint32_t limb[LM_REL_MAX_SEGMENTS * 24 / 32 + 1];
  int used = 1;
  Product() { limb[0] = 1; }
  void times(uint32_t f) {
    uint64_t carry = 0;
    for (int i = 0; i < used; ++i) {
      carry += static_cast<uint64_t>(limb[i]) * f;
      limb[i] = static_cast<uint32_t>(carry);
      carry >>= 32;
    }
    if (carry) limb[used++] = static_cast<uint32_t>(carry);
  }
};

// Whether d^N >= near^(N - t) far^t (all factors at least 1, so the top limb is not zero).
static bool reaches(uint32_t d, int N, uint32_t near, uint32_t far, int t) {
  Product a, b;
  for (int i = 0; i < N; ++i) a.times(d);
  for (int i = 0; i < N - t; ++i) b.times(near);
  for (int i = 0; i < t; ++i) b.times(far);
  if (a.used != b.used) return a.used > b.used;
  for (int i = a.used - 1; i >= 0; --i)
    if (a.limb[i] != b.limb[i]) return a.limb[i] > b.limb[i];
  return true;
}

int rel_buckets(int num_buckets, int max_distance, int mode, int32_t* starts, int32_t* ids) {
  const bool both = mode == LM_REL_BOTH;
  const int n = both ? num_buckets / 2 : num_buckets;
  const int near = n / 2, N = n - near;
  int32_t from[LM_REL_MAX_SEGMENTS];  // a side's bucket borders
  for (int d = 0; d < near; ++d) from[d] = d;
  from[near] = near;
  for (int t = 1; t < N; ++t) {
    int lo = from[near + t - 1], hi = max_distance;  // the answer is in [lo, hi]: far reaches every t
    while (lo < hi) {
      const int mid = lo + (hi - lo) / 2;
      if (reaches(mid, N, near, max_distance, t)) hi = mid; else lo = mid + 1;
    }
    from[near + t] = lo;
  }
  int s = 0;
  auto put = [&](int32_t start, int id) {
    if (s && starts[s - 1] == start) --s;  // an empty bucket: no distance reaches it
    starts[s] = start;
    ids[s++] = id;
  };
  // keys before the query: distances -infinity .. 0; bucket b covers -(from[b + 1] - 1) .. -from[b]
  for (int b = n - 1; b >= 0; --b)
    put(b == n - 1 ? INT32_MIN : 1 - from[b + 1], b);
  if (both)
    for (int b = 1; b < n; ++b) put(from[b], n + b);
  else if (mode == LM_REL_CAUSAL)
    put(1, -1);
  return s;
}

}  // namespace lmz
