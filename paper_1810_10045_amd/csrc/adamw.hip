// The AdamW step over many tensors in one launch, moments in fp32 or in 8 bits,
// and the lazy step on table rows with 8-bit moments.
//
// The step reads and writes each parameter and its moments once: HBM bounds it
// (fp32 moments with bf16 gradients and copies: 28 bytes a value, 202M values 974 us
// or 5.8 TB/s; 8-bit moments: 16.1 bytes, 531 us or 6.1 TB/s, with its vector units
// busy for about 85% of that: 91 instructions a value).
//
// A list of tensors is cut into chunks of kChunk values; one workgroup steps one
// chunk, so a list of a thousand small tensors is one launch and a large tensor
// spreads over the whole device. Which chunk is whose comes from the plan, a table in
// device memory that the caller builds once.
//
// - Streaming (non-temporal) loads and stores: nothing here is read again before the
//   next step. Through the caches 202M values take 8% longer (fp32) and 129,362 rows of
//   1024 in 8 bits 15%.
// - A workgroup ends with its chunk instead of going on to another: loads and stores
//   are counted together, so a wave's next loads would wait for its last stores (8 bits:
//   21% longer).
// - Two vectors of each operand a lane. One or four were no faster at 202M values, and a
//   list of 20 small tensors took 3.7 us with two, 5.0 with four.
#include "launch_parts.hpp"
#include "moments.hpp"

namespace lmz {

constexpr int kAdamwThreads = 256;
constexpr int kVec = 4;       // values of a lane's vector (16 bytes of fp32)
constexpr int kVectors = 2;   // vectors a lane holds at once
constexpr int kChunk = kAdamwThreads * kVec * kVectors;
static_assert(kChunk % kMomentBlock == 0, "chunks start on whole blocks");

// The plan: one record per chunk, with everything its workgroup needs, so that
// the data's addresses are one load away from the launch.
struct PlanChunk {
  float* p;
  const void* g;
  void* m;
  void* v;
  uint8_t* m_scale;
  uint8_t* v_scale;
  uint16_t* copy;
  int64_t first;  // the number of the chunk's first value: whole blocks before it
  int32_t n;      // values, 1 to kChunk
  int32_t decay;  // 1 or 0: whether the weight decay applies
  uint64_t kind;  // of the list: plan_kind
};
static_assert(sizeof(PlanChunk) == 80);

static uint64_t plan_kind(int64_t chunks, int gtype, int states, bool copies) {
  return 0x6c6d5a41ull << 32 ^ static_cast<uint64_t>(chunks) << 8 ^ gtype << 7 ^ copies << 6 ^ states;
}

// ---------------------------------------------------------------------------
// A lane's vectors of n values, its own from number i on. Where a vector may pass
// the end (PART), the last 4 values are loaded in its place and, once every load is
// under way, moved down, zeros behind them: 100,000 rows of 91 values in a table of a
// million take 64 us so, 40% more where each vector is moved before the next is loaded, 36%
// more with a load for each value (129,362 rows of 1,001: 581 us, 12% and 40% more). Fewer than 4 values (FEW) are loaded one by one.
// ---------------------------------------------------------------------------
enum End { WHOLE, PART, FEW };

template <End END>
__device__ __forceinline__ int load_from(int i, int n) {
  return END == PART && i > n - 4 ? n - 4 : i;
}

template <End END>
__device__ __forceinline__ void load4(const float* p, int i, int n, float* x) {
  if constexpr (END != FEW) {
    const f32x4 t = stream_load_e(reinterpret_cast<const f32x4e*>(p + load_from<END>(i, n)));
    x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = i + e < n ? p[i + e] : 0.f;
  }
}

template <End END>
__device__ __forceinline__ void load4(const bf16_t* p, int i, int n, float* x) {
  if constexpr (END != FEW) {
    const u32x2e t =
        __builtin_nontemporal_load(reinterpret_cast<const u32x2e*>(p + load_from<END>(i, n)));
    x[0] = __uint_as_float(t.x << 16); x[1] = __uint_as_float(t.x & 0xffff0000u);
    x[2] = __uint_as_float(t.y << 16); x[3] = __uint_as_float(t.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = i + e < n ? bf16_to_f32(p[i + e].bits) : 0.f;
  }
}

template <End END>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int i, int n) {
  if constexpr (END != FEW)
    return __builtin_nontemporal_load(reinterpret_cast<const u32e*>(p + load_from<END>(i, n)));
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) w |= (i + e < n ? uint32_t(p[i + e]) : 0u) << (8 * e);
  return w;
}

// The values of a PART vector moved to their places.
template <End END>
__device__ __forceinline__ void settle(int i, int n, float* x) {
  const int by = i - load_from<END>(i, n);  // values too early; 4 and more: none is wanted
  if (END != PART || !ballot(by > 0)) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = by & 2 ? (e < 2 ? x[e + 2] : 0.f) : x[e];
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = by & 1 ? (e < 3 ? x[e + 1] : 0.f) : x[e];
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = by > 3 ? 0.f : x[e];
}

template <End END>
__device__ __forceinline__ uint32_t settle(int i, int n, uint32_t codes) {
  const int by = i - load_from<END>(i, n);
  return by > 3 ? 0u : codes >> (8 * by);
}

template <End END>
__device__ __forceinline__ void store4(float* p, int i, int n, const float* x) {
  if (END == WHOLE || i + 4 <= n) {
    __builtin_nontemporal_store(f32x4e{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4e*>(p + i));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[i + e] = x[e];
  }
}

__device__ __forceinline__ uint32_t bf16_bits(float x) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}

template <End END>
__device__ __forceinline__ void store4(uint16_t* p, int i, int n, const float* x) {
  if (END == WHOLE || i + 4 <= n) {
    const u32x2e w = {bf16_bits(x[0]) | bf16_bits(x[1]) << 16,
                      bf16_bits(x[2]) | bf16_bits(x[3]) << 16};
    __builtin_nontemporal_store(w, reinterpret_cast<u32x2e*>(p + i));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[i + e] = static_cast<uint16_t>(bf16_bits(x[e]));
  }
}

template <End END>
__device__ __forceinline__ void store_codes(uint8_t* p, int i, int n, uint32_t w) {
  if (END == WHOLE || i + 4 <= n) {
    __builtin_nontemporal_store(w, reinterpret_cast<u32e*>(p + i));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[i + e] = static_cast<uint8_t>(w >> (8 * e));
  }
}

// ---------------------------------------------------------------------------
// The step over a list of tensors. One workgroup, one chunk; a lane's vectors
// are a workgroup's width apart, so every load and store of a wave is one
// contiguous piece.
// ---------------------------------------------------------------------------
template <typename GT, bool EIGHT, bool COPY, End END, int NV>
__device__ __forceinline__ bool step_vectors(const PlanChunk& t, int i0, float gs,
                                             const OptParams& o, const MomentParams& q,
                                             const StepKeys& keys, const float* inverse) {
  const int n = t.n;
  float p[NV][kVec], g[NV][kVec], m[NV][kVec], v[NV][kVec];
  uint32_t mc[NV], vc[NV];
  int ms[NV], vs[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = i0 + j * kAdamwThreads * kVec;
    load4<END>(t.p, i, n, p[j]);
    load4<END>(static_cast<const GT*>(t.g), i, n, g[j]);
    if constexpr (EIGHT) {
      const int b = (END == WHOLE || i < n ? i : n - 1) / kMomentBlock;
      mc[j] = load_codes<END>(static_cast<const uint8_t*>(t.m), i, n);
      vc[j] = load_codes<END>(static_cast<const uint8_t*>(t.v), i, n);
      ms[j] = t.m_scale[b];
      vs[j] = t.v_scale[b];
    } else {
      load4<END>(static_cast<const float*>(t.m), i, n, m[j]);
      load4<END>(static_cast<const float*>(t.v), i, n, v[j]);
    }
  }
  const float wd = t.decay ? o.wd : 0.f;
  bool ok = true;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = i0 + j * kAdamwThreads * kVec;
    settle<END>(i, n, p[j]);
    settle<END>(i, n, g[j]);
    if constexpr (EIGHT) {
      decode4(settle<END>(i, n, mc[j]), ms[j], m[j]);
      decode4(settle<END>(i, n, vc[j]), vs[j], v[j]);
    } else {
      settle<END>(i, n, m[j]);
      settle<END>(i, n, v[j]);
    }
    uint32_t word[kVec], low[kVec], kept = 0;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float x = g[j][e] * gs;
      if constexpr (EIGHT) {
        kept |= adamw_value8(p[j][e], m[j][e], v[j][e], x, wd, q) ? 0u : 1u << e;
        word[e] = value_word(static_cast<uint64_t>(t.first + i + e), keys);
        low[e] = word[e] << 12;
      } else {
        float p1 = p[j][e], m1 = m[j][e], v1 = v[j][e];
        OptParams ot = o;
        ot.wd = wd;
        adam_value(p1, m1, v1, x, ot);
        const bool fine = v1 < __builtin_inff();
        p[j][e] = fine ? p1 : p[j][e];
        m[j][e] = fine ? m1 : m[j][e];
        v[j][e] = fine ? v1 : v[j][e];
        ok &= fine;
      }
    }
    if constexpr (EIGHT) {
      ok &= kept == 0;
      mc[j] = encode4<false>(m[j], word, kept, inverse, ms[j]);
      vc[j] = encode4<true>(v[j], low, kept, inverse, vs[j]);
    }
    store4<END>(t.p, i, n, p[j]);
    if constexpr (COPY) store4<END>(t.copy, i, n, p[j]);
    if constexpr (EIGHT) {
      store_codes<END>(static_cast<uint8_t*>(t.m), i, n, mc[j]);
      store_codes<END>(static_cast<uint8_t*>(t.v), i, n, vc[j]);
      if ((threadIdx.x & 7) == 0 && (END == WHOLE || i < n)) {
        t.m_scale[i / kMomentBlock] = static_cast<uint8_t>(ms[j]);
        t.v_scale[i / kMomentBlock] = static_cast<uint8_t>(vs[j]);
      }
    } else {
      store4<END>(static_cast<float*>(t.m), i, n, m[j]);
      store4<END>(static_cast<float*>(t.v), i, n, v[j]);
    }
  }
  return ok;
}

template <typename GT, bool EIGHT, bool COPY>
__global__ __launch_bounds__(kAdamwThreads) void k_adamw(
    const PlanChunk* __restrict__ plan, uint64_t kind, OptParams o, MomentParams q,
    StepKeys keys, const float* __restrict__ grad_scale, int32_t* __restrict__ dev_err) {
  __shared__ float inverse[EIGHT ? kScales : 1];
  const PlanChunk t = plan[blockIdx.x];
  const float gs = grad_scale ? *grad_scale : 1.f;
  if (t.kind != kind) {
    if (threadIdx.x == 0) raise_err(dev_err, LM_DEVERR_CAPACITY);
    return;
  }
  if constexpr (EIGHT) fill_scales(inverse, kAdamwThreads);
  const int i0 = threadIdx.x * kVec;
  bool ok = true;
  if (t.n == kChunk) {
    ok = step_vectors<GT, EIGHT, COPY, WHOLE, kVectors>(t, i0, gs, o, q, keys, inverse);
  } else if (t.n >= kVec) {
#pragma unroll 1  // a small copy of the code: a list of small tensors waits for it from memory
    for (int j = 0; j < t.n; j += kAdamwThreads * kVec)
      ok &= step_vectors<GT, EIGHT, COPY, PART, 1>(t, i0 + j, gs, o, q, keys, inverse);
  } else {
    ok = step_vectors<GT, EIGHT, COPY, FEW, 1>(t, i0, gs, o, q, keys, inverse);
  }
  if (ballot(!ok) && lane_id() == 0) raise_err(dev_err, LM_DEVERR_NONFINITE);
}

// ---------------------------------------------------------------------------
// The lazy step on the rows of a table. LANES lanes hold a row (all 64 of a wave
// where it has more than 128 columns, else as few as cover it, a block of 32
// values being 8 lanes), NV vectors of it at a time, and kSlots / NV rows, so that
// a wave has kSlots vectors of every operand under way. Rows of whole vectors
// (WHOLE) load past their end from their last vector.
// ---------------------------------------------------------------------------
constexpr int kSlots = 4;

template <typename KeyT, int LANES, int NV, End END>
__global__ __launch_bounds__(kAdamwThreads) void k_rows8(
    float* __restrict__ table, int64_t V, int D, int64_t ld_table, const KeyT* __restrict__ rows,
    const int64_t* __restrict__ n_rows, int64_t rows_cap, const float* __restrict__ vals,
    int64_t ld_vals, MomentParams q, StepKeys keys, uint8_t* __restrict__ m,
    uint8_t* __restrict__ v, int64_t ld_codes, uint8_t* __restrict__ m_scale,
    uint8_t* __restrict__ v_scale, int64_t ld_scale, int32_t* __restrict__ dev_err,
    uint32_t first_block) {
  constexpr int kRows = kSlots / NV;              // rows a lane holds at once
  constexpr int kPerWave = kWave / LANES * kRows;  // rows of a wave's turn
  __shared__ float inverse[kScales];
  const int lane = lane_id(), part = lane % LANES, group = lane / LANES;
  const int64_t block = first_block + blockIdx.x;
  const int64_t u0 = (block * (kAdamwThreads / kWave) + first_lane(threadIdx.x >> 6)) * kPerWave;
  // The ids come with the count, not after it (any entry below the capacity may be read).
  int64_t id[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int64_t u = u0 + r * (kWave / LANES) + group;
    id[r] = static_cast<int64_t>(rows[u < rows_cap ? u : rows_cap - 1]);
  }
  int64_t count = *n_rows;
  if (count > rows_cap) {
    if (u0 == 0 && lane == 0) raise_err(dev_err, LM_DEVERR_CAPACITY);
    count = rows_cap;
  }
  if (block * (kAdamwThreads / kWave) * kPerWave >= count) return;
  fill_scales(inverse, kAdamwThreads);
  bool ok = true, range = true, live[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    live[r] = u0 + r * (kWave / LANES) + group < count;
    const bool in = id[r] >= 0 && id[r] < V;
    range &= in || !live[r];
    live[r] = live[r] && in;
    id[r] = in ? id[r] : 0;  // any row of the table: loaded, not stored
    if constexpr (LANES == kWave) id[r] = first_lane(id[r]);
  }
  if (u0 < count) {
    for (int cb = 0; cb < D; cb += NV * LANES * kVec) {
      float p[kSlots][kVec], g[kSlots][kVec];
      uint32_t mc[kSlots], vc[kSlots];
      int ms[kSlots], vs[kSlots];
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = s / NV, c = cb + (s % NV * LANES + part) * kVec;
        const int64_t u = u0 + r * (kWave / LANES) + group;
        const int cl = END == WHOLE && c >= D ? D - kVec : c;
        const int b = (c < D ? c : D - 1) / kMomentBlock;
        load4<END>(table + id[r] * ld_table, cl, D, p[s]);
        load4<END>(vals + (u < rows_cap ? u : rows_cap - 1) * ld_vals, cl, D, g[s]);
        mc[s] = load_codes<END>(m + id[r] * ld_codes, cl, D);
        vc[s] = load_codes<END>(v + id[r] * ld_codes, cl, D);
        ms[s] = m_scale[id[r] * ld_scale + b];
        vs[s] = v_scale[id[r] * ld_scale + b];
      }
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = s / NV, c = cb + (s % NV * LANES + part) * kVec;
        float mx[kVec], vx[kVec];
        uint32_t word[kVec], low[kVec], kept = 0;
        settle<END>(c, D, p[s]);
        settle<END>(c, D, g[s]);
        decode4(settle<END>(c, D, mc[s]), ms[s], mx);
        decode4(settle<END>(c, D, vc[s]), vs[s], vx);
        const uint64_t number = static_cast<uint64_t>(id[r]) * D + c;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          kept |= adamw_value8(p[s][e], mx[e], vx[e], g[s][e], q.wd, q) ? 0u : 1u << e;
          word[e] = value_word(number + e, keys);
          low[e] = word[e] << 12;
        }
        mc[s] = encode4<false>(mx, word, kept, inverse, ms[s]);
        vc[s] = encode4<true>(vx, low, kept, inverse, vs[s]);
        if (!live[r] || c >= D) continue;
        ok &= kept == 0;
        store4<END>(table + id[r] * ld_table, c, D, p[s]);
        store_codes<END>(m + id[r] * ld_codes, c, D, mc[s]);
        store_codes<END>(v + id[r] * ld_codes, c, D, vc[s]);
        if ((lane & 7) == 0) {
          m_scale[id[r] * ld_scale + c / kMomentBlock] = static_cast<uint8_t>(ms[s]);
          v_scale[id[r] * ld_scale + c / kMomentBlock] = static_cast<uint8_t>(vs[s]);
        }
      }
    }
  }
  if (ballot(!range) && lane == 0) raise_err(dev_err, LM_DEVERR_ID_RANGE);
  if (ballot(!ok) && lane == 0) raise_err(dev_err, LM_DEVERR_NONFINITE);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
static int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }

int64_t adamw_plan_chunks(const int64_t* sizes, int64_t tensors) {
  int64_t c = 0;
  for (int64_t i = 0; i < tensors; ++i) c += chunks_of(sizes[i]);
  return c;
}

size_t adamw_plan_bytes(int64_t chunks) {
  return static_cast<size_t>(chunks > 0 ? chunks : 1) * sizeof(PlanChunk);
}

void adamw_plan_write(void* const* p, const void* const* g, void* const* m, void* const* v,
                      void* const* m_scale, void* const* v_scale, void* const* copies,
                      const int64_t* sizes, const int32_t* decay, int64_t tensors, int gtype,
                      int states, void* plan) {
  PlanChunk* c = static_cast<PlanChunk*>(plan);
  const int64_t chunks = adamw_plan_chunks(sizes, tensors);
  const uint64_t kind = plan_kind(chunks, gtype, states, copies != nullptr);
  const int64_t state = states == 8 ? 1 : 4, grad = gtype == LM_BF16 ? 2 : 4;
  auto at = [](const void* base, int64_t bytes) {
    return const_cast<char*>(static_cast<const char*>(base)) + bytes;
  };
  int64_t first = 0;
  for (int64_t i = 0; i < tensors; ++i) {
    for (int64_t k = 0; k < sizes[i]; k += kChunk) {
      PlanChunk x{};
      x.p = static_cast<float*>(p[i]) + k;
      x.g = at(g[i], k * grad);
      x.m = at(m[i], k * state);
      x.v = at(v[i], k * state);
      if (states == 8) {
        x.m_scale = static_cast<uint8_t*>(m_scale[i]) + k / kMomentBlock;
        x.v_scale = static_cast<uint8_t*>(v_scale[i]) + k / kMomentBlock;
      }
      if (copies) x.copy = static_cast<uint16_t*>(copies[i]) + k;
      x.first = first + k;
      x.n = static_cast<int32_t>(sizes[i] - k < kChunk ? sizes[i] - k : kChunk);
      x.decay = !decay || decay[i] ? 1 : 0;
      x.kind = kind;
      *c++ = x;
    }
    first += (sizes[i] + kMomentBlock - 1) / kMomentBlock * kMomentBlock;
  }
}

template <typename GT, bool EIGHT>
static int adamw_launch(const void* plan, int64_t chunks, uint64_t kind, bool copies,
                        const OptParams& o, const MomentParams& q, const StepKeys& keys,
                        const float* grad_scale, int32_t* dev_err, hipStream_t st) {
  auto kernel = copies ? k_adamw<GT, EIGHT, true> : k_adamw<GT, EIGHT, false>;
  return launch_parts(chunks, kAdamwThreads, [&](uint32_t first, uint32_t n) {
    kernel<<<n, kAdamwThreads, 0, st>>>(static_cast<const PlanChunk*>(plan) + first, kind, o, q,
                                        keys, grad_scale, dev_err);
    return launch_status(hipGetLastError());
  });
}

int adamw_run(const void* plan, int64_t chunks, int gtype, int states, bool copies, float lr,
              float beta1, float beta2, float eps, float weight_decay, int64_t step,
              const float* grad_scale, uint64_t seed, int32_t* dev_err, hipStream_t st) {
  if (chunks == 0) return LM_OK;
  const OptParams o = make_opt_params(true, lr, beta1, beta2, eps, weight_decay, step, 1.f);
  const MomentParams q = make_moment_params(o, beta2, step);
  const uint64_t kind = plan_kind(chunks, gtype, states, copies);
  const StepKeys keys = step_keys(seed);
  const bool eight = states == 8;
  auto launch = gtype == LM_BF16 ? (eight ? adamw_launch<bf16_t, true> : adamw_launch<bf16_t, false>)
                                 : (eight ? adamw_launch<float, true> : adamw_launch<float, false>);
  return launch(plan, chunks, kind, copies, o, q, keys, grad_scale, dev_err, st);
}

struct Rows8 {
  float* table;
  int64_t V;
  int D;
  int64_t ld_table;
  const void* rows;
  const int64_t* n_rows;
  int64_t rows_cap;
  const float* vals;
  int64_t ld_vals;
  MomentParams q;
  StepKeys keys;
  uint8_t *m, *v;
  int64_t ld_codes;
  uint8_t *m_scale, *v_scale;
  int64_t ld_scale;
  int32_t* dev_err;
};

template <typename KeyT, int LANES, int NV, End END>
static int rows8_launch(const Rows8& a, hipStream_t st) {
  constexpr int kPerBlock = kAdamwThreads / LANES * (kSlots / NV);
  const int64_t blocks = (a.rows_cap + kPerBlock - 1) / kPerBlock;
  return launch_parts(blocks, kAdamwThreads, [&](uint32_t first, uint32_t n) {
    k_rows8<KeyT, LANES, NV, END><<<n, kAdamwThreads, 0, st>>>(
        a.table, a.V, a.D, a.ld_table, static_cast<const KeyT*>(a.rows), a.n_rows, a.rows_cap,
        a.vals, a.ld_vals, a.q, a.keys, a.m, a.v, a.ld_codes, a.m_scale, a.v_scale, a.ld_scale,
        a.dev_err, first);
    return launch_status(hipGetLastError());
  });
}

// Lanes a row, vectors a lane. 100,000 rows of 32, 64, 128 values in a table of a million
// take 23, 30, 47 us so, with a wave for each 2.5, 1.8, 1.4 times as long; rows of 256 and
// 512 86 and 166 us, with 4 vectors a lane 1.8 and 1.1 times. Rows of whole vectors (WHOLE)
// of 128 values would take 11% longer as PART, of 512 1%.
template <typename KeyT, End END>
static int rows8_shape(const Rows8& a, hipStream_t st) {
  const int vectors = (a.D + kVec - 1) / kVec;
  if constexpr (END != FEW) {
    if (vectors > 128) return rows8_launch<KeyT, 64, 4, END>(a, st);
    if (vectors > 64) return rows8_launch<KeyT, 64, 2, END>(a, st);
    if (vectors > 32) return rows8_launch<KeyT, 64, 1, END>(a, st);
    if (vectors > 16) return rows8_launch<KeyT, 32, 1, END>(a, st);
    if (vectors > 8) return rows8_launch<KeyT, 16, 1, END>(a, st);
  }
  return rows8_launch<KeyT, 8, 1, END>(a, st);
}

template <typename KeyT>
static int rows8_ends(const Rows8& a, hipStream_t st) {
  if (a.D % kVec == 0) return rows8_shape<KeyT, WHOLE>(a, st);
  return a.D > kVec ? rows8_shape<KeyT, PART>(a, st) : rows8_shape<KeyT, FEW>(a, st);
}

int rows8_run(float* table, int64_t V, int64_t D, int64_t ld_table, const void* rows, int idtype,
              const int64_t* n_rows, int64_t rows_cap, const float* vals, int64_t ld_vals,
              float lr, float beta1, float beta2, float eps, float weight_decay, int64_t step,
              uint8_t* m, uint8_t* v, int64_t ld_codes, uint8_t* m_scale, uint8_t* v_scale,
              int64_t ld_scale, uint64_t seed, int32_t* dev_err, hipStream_t st) {
  if (D == 0 || rows_cap == 0 || V == 0) return LM_OK;
  const OptParams o = make_opt_params(true, lr, beta1, beta2, eps, weight_decay, step, 1.f);
  const Rows8 a{table, V, static_cast<int>(D), ld_table, rows, n_rows, rows_cap, vals, ld_vals,
                make_moment_params(o, beta2, step), step_keys(seed), m, v, ld_codes, m_scale,
                v_scale, ld_scale, dev_err};
  return idtype == LM_I64 ? rows8_ends<int64_t>(a, st) : rows8_ends<int32_t>(a, st);
}

}  // namespace lmz
