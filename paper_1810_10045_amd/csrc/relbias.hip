// A learned relative position bias and its gradient: out[b, h, i, j] is
// table[bucket(r), h] for the distance r = j - (q_start + i) of key j from query
// i. The buckets are segments of the distance axis: segment s covers the
// distances from starts[s] up to starts[s + 1], and ids[s] names its table row
// (-1: masked).
//
// A head's bias depends on j - i only. The kernels work on square patches of P rows
// and columns (a lane's column vector of 16 bytes, P = 8 bf16 or 4 fp32), 64 of
// them side by side: 2P - 1 diagonals, each one number. The bias of a patch is that
// many values in registers; the gradient adds a patch into that many sums. Each
// element of the matrices is read or written once: HBM bounds both.
#include "common.hpp"
#include "launch_parts.hpp"

namespace lmz {

constexpr int kRelThreads = 256;
constexpr int kRelWaves = kRelThreads / kWave;

struct Segments {
  int32_t starts[LM_REL_MAX_SEGMENTS];
  int16_t ids[LM_REL_MAX_SEGMENTS];
  int32_t n;
  int32_t masked;  // from this distance on everything is masked (INT32_MAX: nothing)
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

// Where a lane's patch lies in its rows: `have` of its P columns exist and are used
// (0 or less: none). It loads from column `from`, inside the row wherever it lies
// (the wave's first patch, col0, where none is used: no further line of memory), and
// its values start at number `by` of what it loads; so no load stands under a
// condition and all of a patch's rows are under way at once. Rows of less than P
// values (NARROW) are loaded one value at a time.
template <typename T, bool NARROW>
struct Columns {
  static constexpr int P = Patch<T>::P;
  int from, by, have;
  __device__ __forceinline__ Columns(int col0, int col, int Lk, bool use) {
    have = use ? Lk - col : 0;
    const int last = Lk - P, at = have > 0 ? col : col0;
    from = NARROW ? 0 : at < last ? at : last;  // last: the last whole patch
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

__device__ __forceinline__ float read_lane(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// LDS instructions of a wave take effect in their order; where lanes meet each
// other's addresses, the compiler has to keep it too.
__device__ __forceinline__ void in_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The value of the lane below; 0 in lane 0.
__device__ __forceinline__ float from_lane_below(float v) {
  return __int_as_float(
      __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x138, 0xf, 0xf, true));  // wave_shr:1
}

// ---------------------------------------------------------------------------
// The bias, written or added. A workgroup covers a patch's width for each of its
// waves, one below the other, in one head of one batch entry: it looks up the
// numbers of its diagonals once, in LDS, and each lane takes its patch's from there.
// Tiles of one column come one after the other (row tiles first), a batch entry
// after the other: 8 x 16 x 2048 x 2048 causal bf16 scores take 275 us so (5.9 TB/s),
// 12% more where a workgroup keeps its diagonals for several batch entries, 18% with
// column tiles first, 31 to 46% with two and four patches of each wave.
// ---------------------------------------------------------------------------
template <typename T, bool ADD, bool NARROW>
__global__ __launch_bounds__(kRelThreads) void k_rel_bias(
    const float* __restrict__ table, int64_t ld_table, Segments seg, int H, int Lq, int Lk,
    int q_start, const T* add, Strides sa, T* out, Strides so, int col_tiles, int row_tiles,
    uint32_t first_block) {
  constexpr int P = Patch<T>::P;
  constexpr int kCols = kWave * P, kRows = kRelWaves * P;
  constexpr int kLine = kRows + kCols;
  using raw_t = typename Patch<T>::raw_t;
  __shared__ __attribute__((aligned(16))) float line[kLine];
  __shared__ int32_t starts[LM_REL_MAX_SEGMENTS];
  __shared__ float value[LM_REL_MAX_SEGMENTS];
  const uint32_t block = first_block + blockIdx.x;
  const int rt = block % row_tiles, rest = block / row_tiles;
  const int ct = rest % col_tiles, rest2 = rest / col_tiles;
  const int h = rest2 % H, b = rest2 / H;
  const int lane = lane_id(), r = first_lane(threadIdx.x >> 6) * P;  // this wave's rows
  const int row0 = rt * kRows, col0 = ct * kCols, row = row0 + r, col = col0 + lane * P;
  // the smallest distance of a patch: one that is masked as a whole is not read
  const int low = col - (row + P - 1) - q_start;
  const Columns<T, NARROW> cols(col0, col, Lk, low < seg.masked);
  const bool read = ADD && row < Lq && low - lane * P < seg.masked;
  raw_t raw[P];
  if (read) {  // on their way while the diagonals are looked up; rows past the last: the last
    const T* a = add + b * sa.b + h * sa.h;
#pragma unroll
    for (int i = 0; i < P; ++i)
      raw[i] = cols.load(a + static_cast<int64_t>(row + i < Lq ? row + i : Lq - 1) * sa.q, Lk);
  }
  for (int s = threadIdx.x; s < seg.n; s += kRelThreads) {
    const int id = seg.ids[s];
    starts[s] = seg.starts[s];
    value[s] = id < 0 ? -__builtin_inff() : table[id * ld_table + h];
  }
  __syncthreads();
  // line[x]: column c of row i has x = c - i + kRows - 1 (c, i from the tile's corner)
  const int base = col0 - row0 - q_start - (kRows - 1);
  for (int x = threadIdx.x; x < kLine; x += kRelThreads)
    line[x] = value[segment_of(starts, seg.n, base + x)];
  __syncthreads();
  if (row >= Lq) return;
  const int nr = Lq - row < P ? Lq - row : P;
  float d[2 * P];  // d[k]: diagonal k - (P - 1) of the patch
#pragma unroll
  for (int k = 0; k < 2 * P; k += 4) {
    const f32x4 t = *reinterpret_cast<const f32x4*>(&line[lane * P + kRows - P - r + k]);
    d[k] = t.x; d[k + 1] = t.y; d[k + 2] = t.z; d[k + 3] = t.w;
  }
  T* o = out + b * so.b + h * so.h + static_cast<int64_t>(row) * so.q + col;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (i >= nr) break;
    float x[P];
    if (read) {
      Patch<T>::widen(cols.whole() ? raw[i] : cols.place(raw[i]), x);
#pragma unroll
      for (int e = 0; e < P; ++e) {
        const float y = d[P - 1 - i + e];
        x[e] = y == -__builtin_inff() ? y : x[e] + y;
      }
    } else {
#pragma unroll
      for (int e = 0; e < P; ++e) x[e] = d[P - 1 - i + e];
    }
    if (Lk - col >= P) {
      Patch<T>::store(o + i * so.q, x);
    } else {
#pragma unroll
      for (int e = 0; e < P; ++e)
        if (e < Lk - col) Patch<T>::put(o + i * so.q + e, x[e]);
    }
  }
}

// ---------------------------------------------------------------------------
// The gradient. A wave goes down `groups` row groups of P rows in one column tile of
// one head and, at each, through `batches` batch entries: their patches have the
// same diagonals, so a lane's 2P - 1 sums stay in registers. After a row group they
// are added to the wave's sums by distance in LDS, by a load, an add and a store:
// each address belongs to one lane of an instruction (ds_add_f32, which needs no
// such care, took about 195 clocks for a wave). Column tiles, not diagonal bands: a
// wave that walked down the diagonal kept its sums in registers throughout, but its
// rows began between cache lines (16 x 16 x 2048 x 2048 bf16: 450 us, against 318 us
// or 6.8 TB/s so). Loading a patch ahead did not help. At the end a
// workgroup adds its waves' sums by distance, then by segment, into the workspace:
// 2 us of a short call's 10. k_rel_join (4 us) adds the workgroups' in their order,
// so results are the same from run to run.
// ---------------------------------------------------------------------------
constexpr int kMaxGroups = 16;

struct GradPlan {
  int groups, batches;                    // of a wave
  int row_parts, col_tiles, batch_parts;  // workgroups of a head: their product
  bool direct;                            // one, of kDirectWaves waves
  int64_t parts() const { return static_cast<int64_t>(row_parts) * col_tiles * batch_parts; }
};

// The gradient's table: row n of head h, or what is added to it.
struct GradTable {
  float* at;
  int64_t ld;
  int rows, accumulate;
};

// dt[., h] (+)= the sums of n segments, in LDS like their ids. A row may have several
// segments, or none.
__device__ __forceinline__ void write_table(const float* sums, const int* ids, int n,
                                            const GradTable& dt, int h) {
  for (int row = threadIdx.x; row < dt.rows; row += blockDim.x) {
    float y = 0.f;
#pragma unroll 8
    for (int s = 0; s < n; ++s) y += ids[s] == row ? sums[s] : 0.f;
    float* d = dt.at + row * dt.ld + h;
    *d = dt.accumulate ? *d + y : y;
  }
}

// WAVES waves a workgroup. kDirectWaves: a head's only workgroup, which writes the table
// itself.
constexpr int kDirectWaves = 16;

template <typename T, bool NARROW, int WAVES>
__global__ __launch_bounds__(WAVES * kWave) void k_rel_grad(
    const T* __restrict__ dout, Strides sd, Segments seg, int B, int Lq, int Lk, int q_start,
    GradPlan g, float* __restrict__ ws, GradTable dt, uint32_t first_block) {
  constexpr int P = Patch<T>::P;
  constexpr bool kDirect = WAVES == kDirectWaves;
  constexpr int kThreads = WAVES * kWave;
  // The sum of distance x of a wave is at plane x % P, place x / P: neighbouring
  // lanes' sums of one diagonal lie side by side.
  constexpr int kPlane = kWave + kMaxGroups + 1;
  constexpr int kLong = 32;  // distances of a segment that a whole wave adds
  using raw_t = typename Patch<T>::raw_t;
  __shared__ float sums[WAVES][P * kPlane];
  __shared__ float line[P * (kWave + WAVES * kMaxGroups)];
  __shared__ int32_t starts[LM_REL_MAX_SEGMENTS + 1];
  __shared__ float total[kDirect ? LM_REL_MAX_SEGMENTS : 1];
  __shared__ int ids[kDirect ? LM_REL_MAX_SEGMENTS : 1];
  const int lane = lane_id(), wave = first_lane(threadIdx.x >> 6);
  const uint32_t block = first_block + blockIdx.x;
  const int rp = block % g.row_parts, rest = block / g.row_parts;
  const int ct = rest % g.col_tiles, rest2 = rest / g.col_tiles;
  const int bp = rest2 % g.batch_parts, h = rest2 / g.batch_parts;
  const int nt = (Lq + P - 1) / P;
  const int t0 = (rp * WAVES + wave) * g.groups;
  const int t1 = t0 + g.groups < nt ? t0 + g.groups : nt;
  const int b0 = bp * g.batches, b1 = b0 + g.batches < B ? b0 + g.batches : B;
  const int col0 = ct * kWave * P, col = col0 + lane * P;
  // a patch's diagonal k has distance low + k
  auto low = [&](int column, int t) { return column - (t * P + P - 1) - q_start; };
  float* mine = kDirect ? total : ws + static_cast<int64_t>(block) * seg.n;
  const int first = low(col0, (rp + 1) * WAVES * g.groups - 1);  // the smallest distance
  if (!kDirect && first >= seg.masked) {  // all of this workgroup's patches are
    for (int s = threadIdx.x; s < seg.n; s += kThreads) mine[s] = 0.f;
    return;
  }
  for (int x = lane; x < P * kPlane; x += kWave) sums[wave][x] = 0.f;
  in_order();
  for (int t = t0; t < t1; ++t) {
    if (low(col0, t) >= seg.masked) continue;
    const Columns<T, NARROW> cols(col0, col, Lk, low(col, t) < seg.masked);
    const int nr = Lq - t * P < P ? Lq - t * P : P;
    const bool edge = nr < P || ballot(!cols.whole());
    const T* p = dout + b0 * sd.b + h * sd.h + static_cast<int64_t>(t) * P * sd.q;
    float acc[2 * P - 1];
#pragma unroll
    for (int k = 0; k < 2 * P - 1; ++k) acc[k] = 0.f;
    for (int b = b0; b < b1; ++b, p += sd.b) {
      raw_t raw[P];
#pragma unroll
      for (int i = 0; i < P; ++i) raw[i] = cols.load(p + (i < nr ? i : 0) * sd.q, Lk);
      if (edge) {
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
    }
    // Diagonal P + k of a lane is diagonal k of the next one; the last lane's go one
    // place further, each by a lane of its own.
    const int place = lane + (g.groups - 1 - (t - t0));
    float over = 0.f;
#pragma unroll
    for (int k = 0; k < P - 1; ++k) {
      over = lane == k ? read_lane(acc[P + k], kWave - 1) : over;
      acc[k] += from_lane_below(acc[P + k]);
    }
    float* at = &sums[wave][place];
#pragma unroll
    for (int k = 0; k < P; ++k) at[k * kPlane] += acc[k];
    if (lane < P - 1) sums[wave][lane * kPlane + place - lane + kWave] += over;
    in_order();  // the next group's places are its neighbour lanes' of this one
  }
  for (int s = threadIdx.x; s < seg.n; s += kThreads) {
    starts[s] = seg.starts[s];
    if constexpr (kDirect) ids[s] = seg.ids[s];
  }
  if (threadIdx.x == 0) starts[seg.n] = INT32_MAX;
  __syncthreads();
  // The waves' sums by distance: line[x] is that of distance first + x, sum x of wave
  // w that of first + (WAVES - 1 - w) * below + x.
  const int below = g.groups * P, length = P * kWave + WAVES * below - 1;
  for (int x = threadIdx.x; x < length; x += kThreads) {
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      // (a load under no condition: the waves' loads are under way at once)
      const unsigned at = x - (WAVES - 1 - w) * below, span = P * kWave + below - 1;
      const unsigned in = at < span ? at : 0;
      const float z = sums[w][in % P * kPlane + in / P];
      y += at < span ? z : 0.f;
    }
    line[x] = y;
  }
  __syncthreads();
  // Segment sums: a wave for each of the long ones, 8 lanes for each of the others (4 x 12
  // x 1024 x 1024 causal: 20.1 us, 21.4 with 8 lanes for all, 22.1 with waves for all).
  // (bounded before they are subtracted: starts may lie anywhere in 32 bits)
  auto place_of = [&](int start) {
    return (start < first ? first : start < first + length ? start : first + length) - first;
  };
  for (int s = wave; s < seg.n; s += WAVES) {
    const int x0 = place_of(starts[s]), x1 = place_of(starts[s + 1]);
    if (x1 - x0 <= kLong) continue;
    float y = 0.f;
#pragma unroll 4
    for (int x = x0 + lane; x < x1; x += kWave) y += line[x];
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) y += __shfl_xor(y, off, kWave);
    if (lane == 0) mine[s] = y;
  }
  for (int s0 = 0; s0 < seg.n; s0 += kThreads / 8) {
    const int s = s0 + static_cast<int>(threadIdx.x) / 8;
    const int x0 = s < seg.n ? place_of(starts[s]) : 0;
    const int x1 = s < seg.n ? place_of(starts[s + 1]) : 0;
    const bool brief = x1 - x0 <= kLong;
    float y = 0.f;
    for (int x = x0 + static_cast<int>(threadIdx.x) % 8; x < (brief ? x1 : x0); x += 8)
      y += line[x];
#pragma unroll
    for (int off = 4; off > 0; off >>= 1) y += __shfl_xor(y, off, kWave);
    if (s < seg.n && brief && threadIdx.x % 8 == 0) mine[s] = y;
  }
  if constexpr (kDirect) {
    __syncthreads();
    write_table(total, ids, seg.n, dt, h);
  }
}

// dtable[n, h] (+)= the sums of the segments with id n over a head's parts. One
// workgroup per head: a thread adds one segment (a column of the workspace) over
// every kJoinThreads / width-th part, so neighbouring threads read neighbouring
// words, and the threads of a segment are added in their order.
constexpr int kJoinThreads = 1024;

__global__ __launch_bounds__(kJoinThreads) void k_rel_join(
    const float* __restrict__ ws, Segments seg, int parts, GradTable dt, uint32_t first_head) {
  __shared__ float part[kJoinThreads];
  __shared__ float sums[LM_REL_MAX_SEGMENTS];
  __shared__ int ids[LM_REL_MAX_SEGMENTS];
  const int h = first_head + blockIdx.x, n = seg.n;
  int width = 32;  // segments of one turn
  while (width < n) width *= 2;
  const int column = threadIdx.x % width, first = threadIdx.x / width, step = kJoinThreads / width;
  const float* mine = ws + static_cast<int64_t>(h) * parts * n;
  float x = 0.f;
  if (column < n) {
    if (first == 0) ids[column] = seg.ids[column];
#pragma unroll 4
    for (int w = first; w < parts; w += step) x += mine[static_cast<int64_t>(w) * n + column];
  }
  part[threadIdx.x] = x;
  __syncthreads();
  if (threadIdx.x < n) {
    float y = 0.f;
#pragma unroll 4
    for (int g = 0; g < step; ++g) y += part[g * width + threadIdx.x];
    sums[threadIdx.x] = y;
  }
  __syncthreads();
  write_table(sums, ids, n, dt, h);
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
  s.masked = ids[n - 1] < 0 ? starts[n - 1] : INT32_MAX;
  return s;
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <typename T>
static int rel_bias_launch(const float* table, int64_t ld_table, const Segments& seg, int64_t B,
                           int64_t H, int64_t Lq, int64_t Lk, int64_t q_start, const void* add,
                           const Strides& sa, void* out, const Strides& so, hipStream_t st) {
  constexpr int P = Patch<T>::P;
  const int64_t ct = ceil_div(Lk, kWave * P), rt = ceil_div(Lq, kRelWaves * P);
  const bool narrow = Lk < Patch<T>::P;
  auto kernel = add ? (narrow ? k_rel_bias<T, true, true> : k_rel_bias<T, true, false>)
                    : k_rel_bias<T, false, false>;
  return launch_parts(ct * rt * H * B, kRelThreads, [&](uint32_t first, uint32_t n) {
    kernel<<<n, kRelThreads, 0, st>>>(table, ld_table, seg, static_cast<int>(H),
                                      static_cast<int>(Lq), static_cast<int>(Lk),
                                      static_cast<int>(q_start), static_cast<const T*>(add), sa,
                                      static_cast<T*>(out), so, static_cast<int>(ct),
                                      static_cast<int>(rt), first);
    return launch_status(hipGetLastError());
  });
}

// Workgroups of a call, for the check of the grid's size.
int64_t rel_bias_blocks(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int dtype) {
  const int P = dtype == LM_BF16 ? Patch<bf16_t>::P : Patch<float>::P;
  return ceil_div(Lk, kWave * P) * ceil_div(Lq, kRelWaves * P) * H * B;
}

int rel_bias_run(const float* table, int64_t ld_table, const int32_t* starts, const int32_t* ids,
                 int n_seg, int64_t B, int64_t H, int64_t Lq, int64_t Lk, int64_t q_start,
                 const void* add, const int64_t* sa, void* out, const int64_t* so, int dtype,
                 hipStream_t st) {
  if (B == 0 || H == 0 || Lq == 0 || Lk == 0) return LM_OK;
  const Segments seg = make_segments(starts, ids, n_seg);
  const Strides a = add ? Strides{sa[0], sa[1], sa[2]} : Strides{0, 0, 0};
  const Strides o{so[0], so[1], so[2]};
  auto launch = dtype == LM_BF16 ? rel_bias_launch<bf16_t> : rel_bias_launch<float>;
  return launch(table, ld_table, seg, B, H, Lq, Lk, q_start, add, a, out, o, st);
}

// How a head's matrices are shared out among waves.
static GradPlan grad_plan(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int dtype) {
  const int P = dtype == LM_BF16 ? Patch<bf16_t>::P : Patch<float>::P;
  const int64_t nt = ceil_div(Lq, P), ct = ceil_div(Lk, kWave * P);
  GradPlan g;
  // A head in one workgroup, one launch, where its waves have few patches, one after the
  // other: 2 x 8 x 151 x 151 fp32 (6 patches of 4 rows) takes a caller 11.0 us so and 14.5
  // with a second launch, 2 x 12 x 128 x 128 bf16 (2 of 8 rows) 12.2 and 13.7; in a graph,
  // where launches cost less, 10.0 and 9.0, 11.3 and 10.7. 4 patches of 8 rows (1 x 16 x
  // 512 x 512) would take 16.7 us in a graph, 10.8 with two launches.
  g.groups = static_cast<int>(ceil_div(nt, kDirectWaves));
  g.direct = ct == 1 && g.groups <= kMaxGroups && g.groups * B * P * P <= 128;
  if (g.direct) {
    g.batches = static_cast<int>(B);
    g.row_parts = g.col_tiles = g.batch_parts = 1;
    return g;
  }
  // Patches of a wave (64 lanes'): enough waves for 8 on each compute unit, and up to
  // kMaxGroups patches each beyond that. 4 x 12 x 1024 x 1024 causal takes 21 us so, 26
  // with a quarter as many patches each and 29 with twice as many.
  int64_t patches = nt * ct * B * H / 2048;
  patches = patches < 1 ? 1 : patches > kMaxGroups ? kMaxGroups : patches;
  // batch entries in even shares
  g.batches = static_cast<int>(B < patches ? B : ceil_div(B, ceil_div(B, patches)));
  g.groups = static_cast<int>(patches / g.batches);
  g.row_parts = static_cast<int>(ceil_div(nt, static_cast<int64_t>(g.groups) * kRelWaves));
  g.col_tiles = static_cast<int>(ct);
  g.batch_parts = static_cast<int>(ceil_div(B, g.batches));
  return g;
}

// Workgroups of one head that write to the workspace.
int64_t rel_grad_parts(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int dtype) {
  if (B == 0 || H == 0 || Lq == 0 || Lk == 0) return 0;
  const GradPlan g = grad_plan(B, H, Lq, Lk, dtype);
  return g.direct ? 0 : g.parts();
}

template <typename T>
static int rel_grad_launch(const void* dout, const Strides& s, const Segments& seg, int64_t B,
                           int64_t H, int64_t Lq, int64_t Lk, int64_t q_start, const GradPlan& g,
                           float* ws, const GradTable& dt, hipStream_t st) {
  const bool narrow = Lk < Patch<T>::P;
  auto kernel = g.direct ? (narrow ? k_rel_grad<T, true, kDirectWaves>
                                   : k_rel_grad<T, false, kDirectWaves>)
                         : (narrow ? k_rel_grad<T, true, kRelWaves>
                                   : k_rel_grad<T, false, kRelWaves>);
  const int threads = (g.direct ? kDirectWaves : kRelWaves) * kWave;
  return launch_parts(g.parts() * H, threads, [&](uint32_t first, uint32_t n) {
    kernel<<<n, threads, 0, st>>>(static_cast<const T*>(dout), s, seg, static_cast<int>(B),
                                  static_cast<int>(Lq), static_cast<int>(Lk),
                                  static_cast<int>(q_start), g, ws, dt, first);
    return launch_status(hipGetLastError());
  });
}

int rel_grad_run(const void* dout, int dtype, int64_t B, int64_t H, int64_t Lq, int64_t Lk,
                 const int64_t* sd, int64_t q_start, const int32_t* starts, const int32_t* ids,
                 int n_seg, int num_buckets, float* dtable, int64_t ld_table, int accumulate,
                 void* ws, hipStream_t st) {
  if (H == 0) return LM_OK;
  const Segments seg = make_segments(starts, ids, n_seg);
  float* sums = static_cast<float*>(ws);
  const GradTable dt{dtable, ld_table, num_buckets, accumulate};
  int64_t parts = 0;
  if (B > 0 && Lq > 0 && Lk > 0) {
    const GradPlan g = grad_plan(B, H, Lq, Lk, dtype);
    const Strides s{sd[0], sd[1], sd[2]};
    auto launch = dtype == LM_BF16 ? rel_grad_launch<bf16_t> : rel_grad_launch<float>;
    const int rc = launch(dout, s, seg, B, H, Lq, Lk, q_start, g, sums, dt, st);
    if (rc != LM_OK || g.direct) return rc;
    parts = g.parts();
  }
  return launch_parts(H, kJoinThreads, [&](uint32_t first, uint32_t n) {
    k_rel_join<<<n, kJoinThreads, 0, st>>>(sums, seg, static_cast<int>(parts), dt, first);
    return launch_status(hipGetLastError());
  });
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
