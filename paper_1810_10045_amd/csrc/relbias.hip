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

// Where a lane's patch lies in its rows: `have` of its P columns exist (0 or less:
// it is outside). It loads from column `from`, inside the row wherever it lies, and
// its values start at number `by` of what it loads; so no load stands under a
// condition and all of a patch's rows are under way at once. Rows of less than P
// values (NARROW) are loaded one value at a time.
template <typename T, bool NARROW>
struct Columns {
  static constexpr int P = Patch<T>::P;
  int from, by, have;
  __device__ __forceinline__ Columns(int col, int Lk, bool use) {
    have = col < 0 || !use ? 0 : Lk - col;
    const int last = Lk - P;  // the last whole patch
    from = have <= 0 || NARROW ? 0 : col < last ? col : last;
    by = have <= 0 ? P : have < P && !NARROW ? P - have : 0;
  }
  __device__ __forceinline__ bool whole() const { return have >= P; }
  // Row p's patch as it is loaded, and its values moved to their places.
  __device__ __forceinline__ typename Patch<T>::raw_t load(const T* p, int Lk) const {
    if constexpr (!NARROW) return Patch<T>::load(p + from);
    float x[P];  // a row's few values: the only patch in it starts at column 0
#pragma unroll
    for (int e = 0; e < P; ++e) x[e] = e < Lk ? Patch<T>::one(p + e) : 0.f;
    return Patch<T>::pack(x);
  }
  __device__ __forceinline__ typename Patch<T>::raw_t place(
      const typename Patch<T>::raw_t& r) const {
    return Patch<T>::shift(r, by);
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

template <typename T, bool ADD, bool NARROW>
__global__ __launch_bounds__(kRelThreads) void k_rel_bias(
    const float* __restrict__ table, int64_t ld_table, Segments seg, int B, int Lq, int Lk,
    int q_start, const T* add, Strides sa, T* out, Strides so, int col_tiles, int row_tiles) {
  constexpr int P = Patch<T>::P;
  constexpr int kCols = kWave * P;
  constexpr int kLine = kRelRows + kCols;
  using raw_t = typename Patch<T>::raw_t;
  __shared__ __attribute__((aligned(16))) float line[kLine];
  __shared__ int32_t starts[LM_REL_MAX_SEGMENTS];
  __shared__ float value[LM_REL_MAX_SEGMENTS];
  const int ct = blockIdx.x % col_tiles, rest = blockIdx.x / col_tiles;
  const int rt = rest % row_tiles, h = rest / row_tiles;
  const int lane = lane_id(), wave = first_lane(threadIdx.x >> 6);
  const int row0 = rt * kRelRows, col0 = ct * kCols, col = col0 + lane * P;
  const Columns<T, NARROW> cols(col, Lk, true);
  // The scores of a patch: P rows from row0 + r of batch entry b. Rows past the last
  // are loaded from the last.
  auto load = [&](int r, int b, raw_t* raw) {
    const T* a = add + b * sa.b + h * sa.h;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int row = row0 + r + i < Lq ? row0 + r + i : Lq - 1;
      raw[i] = cols.load(a + static_cast<int64_t>(row) * sa.q, Lk);
    }
  };
  // the smallest distance from which on everything is masked
  const int masked = seg.ids[seg.n - 1] < 0 ? seg.starts[seg.n - 1] : INT32_MAX;
  auto hidden = [&](int r) { return col0 - (row0 + r + P - 1) - q_start >= masked; };
  raw_t raw[P], next[P];
  int r = wave * P;
  const bool some = row0 + r < Lq;
  if (ADD && some && !hidden(r)) load(r, 0, next);
  for (int s = threadIdx.x; s < seg.n; s += kRelThreads) {
    const int id = seg.ids[s];
    starts[s] = seg.starts[s];
    value[s] = id < 0 ? -__builtin_inff() : table[id * ld_table + h];
  }
  __syncthreads();
  // line[x]: column c of row r has x = c - r + kRelRows - 1 (c, r from the tile's corner)
  const int base = col0 - row0 - q_start - (kRelRows - 1);
  for (int x = threadIdx.x; x < kLine; x += kRelThreads)
    line[x] = value[segment_of(starts, seg.n, base + x)];
  __syncthreads();
  if (!some) return;
  const int rows = Lq - row0 < kRelRows ? Lq - row0 : kRelRows;
  for (; r < rows; r += kRelWaves * P) {
    const int nr = rows - r < P ? rows - r : P;
    float d[2 * P];  // d[k]: diagonal k - (P - 1) of the patch
    const int at = lane * P + kRelRows - P - r;
#pragma unroll
    for (int k = 0; k < 2 * P; k += 4) {
      const f32x4 t = *reinterpret_cast<const f32x4*>(&line[at + k]);
      d[k] = t.x; d[k + 1] = t.y; d[k + 2] = t.z; d[k + 3] = t.w;
    }
    const bool plain = !ADD || hidden(r);  // the bias alone
    for (int b = 0; b < B; ++b) {
      if (!plain) {
#pragma unroll
        for (int i = 0; i < P; ++i) raw[i] = next[i];
      }
      // The next patch's loads go out before this one's stores: they would wait behind
      // them otherwise, since out may be add.
      if (ADD) {
        const bool more = b + 1 < B;
        const int r1 = more ? r : r + kRelWaves * P;
        if (r1 < rows && !hidden(r1)) load(r1, more ? b + 1 : 0, next);
      }
      T* o = out + b * so.b + h * so.h + static_cast<int64_t>(row0 + r) * so.q + col;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (i >= nr) break;
        float x[P];
        if (plain) {
#pragma unroll
          for (int e = 0; e < P; ++e) x[e] = d[P - 1 - i + e];
        } else {
          Patch<T>::widen(cols.whole() ? raw[i] : cols.place(raw[i]), x);
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const float y = d[P - 1 - i + e];
            x[e] = y == -__builtin_inff() ? y : x[e] + y;
          }
        }
        if (cols.whole()) {
          Patch<T>::store(o + i * so.q, x);
        } else {
#pragma unroll
          for (int e = 0; e < P; ++e)
            if (e < cols.have) Patch<T>::put(o + i * so.q + e, x[e]);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The gradient. Patches are numbered along a line: patch diagonal q has its
// column c = P * (t + q - (nt - 1)) at row group t (nt groups of P rows), so it
// starts at the matrix's lower left corner and ends at its upper right. A
// workgroup takes 64 neighbouring patch diagonals (a band) of one head; its waves
// take turns of `steps` patches down the band, through the batch. A lane's 2P - 1
// sums stay in registers for the whole turn; the waves' sums are then added by
// distance and by segment in LDS, and written to the workspace. k_rel_join adds
// the workgroups' sums in their order, so results are the same from run to run.
// ---------------------------------------------------------------------------
struct GradPlan {
  int bands, parts;  // workgroups of a head: their product
  int steps;         // patches of a wave's turn
};

template <typename T, bool NARROW>
__global__ __launch_bounds__(kRelThreads) void k_rel_grad(
    const T* __restrict__ dout, Strides sd, Segments seg, int B, int Lq, int Lk, int q_start,
    GradPlan g, float* __restrict__ ws) {
  constexpr int P = Patch<T>::P;
  constexpr int kLine = kWave * P + P;  // a band's distances (one more than there are)
  using raw_t = typename Patch<T>::raw_t;
  __shared__ int32_t starts[LM_REL_MAX_SEGMENTS + 1];
  __shared__ float sums[kRelWaves][kLine];
  const int lane = lane_id(), wave = first_lane(threadIdx.x >> 6);
  const int band = blockIdx.x % g.bands, rest = blockIdx.x / g.bands;
  const int part = rest % g.parts, h = rest / g.parts;
  const int nt = (Lq + P - 1) / P, nk = (Lk + P - 1) / P;
  const int q0 = band * kWave - (nt - 1), q = q0 + lane;  // column patch at row group 0
  // lane's diagonal k has distance r0 + k; the band's distances start at w0
  const int w0 = P * q0 - q_start - (P - 1), r0 = w0 + lane * P;
  const int masked = seg.ids[seg.n - 1] < 0 ? seg.starts[seg.n - 1] : INT32_MAX;
  // the row groups t0 to t1 where this band meets the matrix and is not masked as a whole
  const int t0 = -(q0 + kWave - 1) > 0 ? -(q0 + kWave - 1) : 0;
  const int t1 = w0 >= masked ? t0 : nk - q0 < nt ? nk - q0 : nt;
  const int64_t all = t1 > t0 ? static_cast<int64_t>(t1 - t0) * B : 0;
  const int64_t from = (static_cast<int64_t>(part) * kRelWaves + wave) * g.steps;
  const int64_t to = from + g.steps < all ? from + g.steps : all;
  float acc[2 * P - 1];
#pragma unroll
  for (int k = 0; k < 2 * P - 1; ++k) acc[k] = 0.f;
  if (from < to) {
    const bool use = r0 < masked;
    int t = t0 + static_cast<int>(from % (t1 - t0));
    const T* base = dout + from / (t1 - t0) * sd.b + h * sd.h;
    for (int64_t s = from; s < to; ++s) {
      const Columns<T, NARROW> cols(P * (t + q), Lk, use);
      const int nr = Lq - t * P < P ? Lq - t * P : P;
      const T* p = base + static_cast<int64_t>(t) * P * sd.q;
      raw_t raw[P];
#pragma unroll
      for (int i = 0; i < P; ++i) raw[i] = cols.load(p + (i < nr ? i : 0) * sd.q, Lk);
      if (nr < P || ballot(!cols.whole())) {
#pragma unroll
        for (int i = 0; i < P; ++i) raw[i] = Patch<T>::shift(raw[i], i < nr ? cols.by : P);
      }
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float x[P];
        Patch<T>::widen(raw[i], x);
#pragma unroll
        for (int e = 0; e < P; ++e) acc[P - 1 - i + e] += x[e];
      }
      if (++t == t1) {
        t = t0;
        base += sd.b;
      }
    }
  }
  for (int s = threadIdx.x; s < seg.n; s += kRelThreads) starts[s] = seg.starts[s];
  if (threadIdx.x == 0) starts[seg.n] = INT32_MAX;
  // Diagonal P + k of a lane is diagonal k of the next one.
#pragma unroll
  for (int k = 0; k < P; ++k) {
    float below = 0.f;
    if (k < P - 1) {
      below = __shfl_up(acc[P + k], 1, kWave);
      if (lane == 0) below = 0.f;
      if (lane == kWave - 1) sums[wave][kWave * P + k] = acc[P + k];
    }
    sums[wave][lane * P + k] = acc[k] + below;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < kLine - 1; x += kRelThreads) {
    float y = sums[0][x];
#pragma unroll
    for (int w = 1; w < kRelWaves; ++w) y += sums[w][x];
    sums[0][x] = y;
  }
  __syncthreads();
  // Segment sums: 8 lanes add the distances of one, each every eighth.
  float* mine = ws + static_cast<int64_t>(blockIdx.x) * seg.n;
  for (int s = threadIdx.x / 8; s < (seg.n + kRelThreads / 8 - 1) / (kRelThreads / 8) * (kRelThreads / 8);
       s += kRelThreads / 8) {
    float y = 0.f;
    if (s < seg.n) {
      const int64_t lo = static_cast<int64_t>(starts[s]) - w0, hi = static_cast<int64_t>(starts[s + 1]) - w0;
      const int x1 = hi < kLine - 1 ? static_cast<int>(hi) : kLine - 1;
      for (int x = (lo > 0 ? static_cast<int>(lo < kLine ? lo : kLine) : 0) + (threadIdx.x & 7); x < x1; x += 8)
        y += sums[0][x];
    }
#pragma unroll
    for (int off = 4; off > 0; off >>= 1) y += __shfl_xor(y, off, kWave);
    if (s < seg.n && (threadIdx.x & 7) == 0) mine[s] = y;
  }
}

// dtable[n, h] (+)= the sums of the segments with id n over a head's parts. One
// workgroup per head: a thread adds one segment (a column of the workspace) over
// every kJoinThreads / width-th part, so neighbouring threads read neighbouring
// words, and the threads of a segment are added in their order.
constexpr int kJoinThreads = 1024;

__global__ __launch_bounds__(kJoinThreads) void k_rel_join(
    const float* __restrict__ ws, Segments seg, int parts, int num_buckets,
    float* __restrict__ dtable, int64_t ld_table, int accumulate) {
  __shared__ float part[kJoinThreads];
  __shared__ float sums[LM_REL_MAX_SEGMENTS];
  const int h = blockIdx.x, n = seg.n;
  int width = 32;  // segments of one turn
  while (width < n && width < kJoinThreads) width *= 2;
  const int column = threadIdx.x % width, first = threadIdx.x / width, step = kJoinThreads / width;
  const float* mine = ws + static_cast<int64_t>(h) * parts * n;
  float x = 0.f;
  if (column < n) {
#pragma unroll 8
    for (int w = first; w < parts; w += step) x += mine[static_cast<int64_t>(w) * n + column];
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
  const bool narrow = Lk < Patch<T>::P;
  auto kernel = add ? (narrow ? k_rel_bias<T, true, true> : k_rel_bias<T, true, false>)
                    : k_rel_bias<T, false, false>;
  kernel<<<grid, kRelThreads, 0, st>>>(table, ld_table, seg, static_cast<int>(B),
                                       static_cast<int>(Lq), static_cast<int>(Lk),
                                       static_cast<int>(q_start), static_cast<const T*>(add), sa,
                                       static_cast<T*>(out), so, static_cast<int>(ct),
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

// How a head's matrices are shared out among waves.
static GradPlan grad_plan(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int dtype) {
  const int P = dtype == LM_BF16 ? Patch<bf16_t>::P : Patch<float>::P;
  const int64_t nt = ceil_div(Lq, P), nk = ceil_div(Lk, P);
  GradPlan g;
  g.bands = static_cast<int>(ceil_div(nt - 1 + nk, kWave));
  // patches of 64 lanes in all: each row group meets its columns' bands and one more
  const int64_t all = nt * (nk / kWave + 1) * B * H;
  const int64_t most = nt < nk + kWave ? nt : nk + kWave;  // row groups of the longest band
  int64_t steps = all / 8192;
  steps = steps < 1 ? 1 : steps > 32 ? 32 : steps;
  g.steps = static_cast<int>(steps);
  g.parts = static_cast<int>(ceil_div(most * B, steps * kRelWaves));
  return g;
}

// Workgroups of one head; 0 where there is nothing to add.
int64_t rel_grad_parts(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int dtype) {
  if (B == 0 || H == 0 || Lq == 0 || Lk == 0) return 0;
  const GradPlan g = grad_plan(B, H, Lq, Lk, dtype);
  return static_cast<int64_t>(g.bands) * g.parts;
}

int rel_grad_run(const void* dout, int dtype, int64_t B, int64_t H, int64_t Lq, int64_t Lk,
                 const int64_t* sd, int64_t q_start, const int32_t* starts, const int32_t* ids,
                 int n_seg, int num_buckets, float* dtable, int64_t ld_table, int accumulate,
                 void* ws, hipStream_t st) {
  if (H == 0) return LM_OK;
  const Segments seg = make_segments(starts, ids, n_seg);
  const int64_t parts = rel_grad_parts(B, H, Lq, Lk, dtype);
  if (parts) {
    const GradPlan g = grad_plan(B, H, Lq, Lk, dtype);
    const Strides s{sd[0], sd[1], sd[2]};
    const dim3 grid(static_cast<uint32_t>(parts * H));
    auto launch = [&](auto kernel, auto* matrix) {
      kernel<<<grid, kRelThreads, 0, st>>>(matrix, s, seg, static_cast<int>(B),
                                           static_cast<int>(Lq), static_cast<int>(Lk),
                                           static_cast<int>(q_start), g, static_cast<float*>(ws));
    };
    if (dtype == LM_BF16)
      launch(Lk < Patch<bf16_t>::P ? k_rel_grad<bf16_t, true> : k_rel_grad<bf16_t, false>,
             static_cast<const bf16_t*>(dout));
    else
      launch(Lk < Patch<float>::P ? k_rel_grad<float, true> : k_rel_grad<float, false>,
             static_cast<const float*>(dout));
    const int rc = launch_status(hipGetLastError());
    if (rc != LM_OK) return rc;
  }
  k_rel_join<<<static_cast<uint32_t>(H), kJoinThreads, 0, st>>>(
      static_cast<const float*>(ws), seg, static_cast<int>(parts), num_buckets, dtable, ld_table,
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
