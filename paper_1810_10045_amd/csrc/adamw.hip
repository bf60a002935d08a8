// The AdamW step over many tensors in one launch, moments in fp32 or in 8 bits,
// and the lazy step on table rows with 8-bit moments.
//
// The step reads and writes each parameter and its moments once: HBM bounds it.
// A list of tensors is cut into chunks of kChunk values; one workgroup steps one
// chunk, so a list of a thousand small tensors is one launch and a large tensor
// spreads over the whole device. Which chunk belongs to which tensor comes from
// the plan, a table in device memory that the caller builds once.
#include "moments.hpp"

namespace lmz {

constexpr int kAdamwThreads = 256;
constexpr int kVec = 4;       // values of a lane's vector (16 bytes of fp32)
constexpr int kVectors = 4;   // vectors a lane holds at once
constexpr int kChunk = kAdamwThreads * kVec * kVectors;
static_assert(kChunk % kMomentBlock == 0, "chunks start on whole blocks");

// The plan: a header, one entry per tensor, one word pair per chunk.
struct PlanHead {
  uint64_t magic;
  int64_t tensors, chunks;
  int32_t gtype, states;
  int32_t copies, pad[7];
};
static_assert(sizeof(PlanHead) == 64);

struct PlanTensor {
  float* p;
  const void* g;
  void* m;
  void* v;
  uint8_t* m_scale;
  uint8_t* v_scale;
  uint16_t* copy;
  int64_t n;
  int64_t first;  // the number of the tensor's first value: whole blocks before it
  float decay;    // 1 or 0: whether the weight decay applies
  int32_t pad;
};
static_assert(sizeof(PlanTensor) == 80);

struct PlanChunk {
  uint32_t tensor, index;
};

constexpr uint64_t kPlanMagic = 0x6c6d5a61646d7731ull;

// VEC values at p of which `have` (1 to VEC) exist.
__device__ __forceinline__ void load4(const float* p, int have, float* x) {
  if (have >= 4) {
    const f32x4e t = *reinterpret_cast<const f32x4e*>(p);
    x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = e < have ? p[e] : 0.f;
  }
}

__device__ __forceinline__ void load4(const bf16_t* p, int have, float* x) {
  if (have >= 4) {
    const u32x2e t = *reinterpret_cast<const u32x2e*>(p);
    x[0] = __uint_as_float(t.x << 16); x[1] = __uint_as_float(t.x & 0xffff0000u);
    x[2] = __uint_as_float(t.y << 16); x[3] = __uint_as_float(t.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = e < have ? bf16_to_f32(p[e].bits) : 0.f;
  }
}

__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int have) {
  if (have >= 4) return *reinterpret_cast<const u32e*>(p);
  uint32_t w = 0;
  for (int e = 0; e < have; ++e) w |= uint32_t(p[e]) << (8 * e);
  return w;
}

__device__ __forceinline__ void store4(float* p, int have, const float* x) {
  if (have >= 4) {
    *reinterpret_cast<f32x4e*>(p) = f32x4e{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < have) p[e] = x[e];
  }
}

__device__ __forceinline__ uint32_t bf16_bits(float x) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}

__device__ __forceinline__ void store4(uint16_t* p, int have, const float* x) {
  if (have >= 4) {
    *reinterpret_cast<u32x2e*>(p) = u32x2e{bf16_bits(x[0]) | bf16_bits(x[1]) << 16,
                                           bf16_bits(x[2]) | bf16_bits(x[3]) << 16};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < have) p[e] = static_cast<uint16_t>(bf16_bits(x[e]));
  }
}

__device__ __forceinline__ void store_codes(uint8_t* p, int have, uint32_t w) {
  if (have >= 4) {
    *reinterpret_cast<u32e*>(p) = w;
  } else {
    for (int e = 0; e < have; ++e) p[e] = static_cast<uint8_t>(w >> (8 * e));
  }
}

// ---------------------------------------------------------------------------
// The step over a list of tensors. One workgroup, one chunk; a lane's vectors
// are a workgroup's width apart, so every load and store of a wave is one
// contiguous piece.
// ---------------------------------------------------------------------------
template <typename GT, bool EIGHT, bool COPY>
__global__ __launch_bounds__(kAdamwThreads) void k_adamw(
    const PlanHead* __restrict__ head, PlanHead want, OptParams o, MomentParams q, StepKeys keys,
    const float* __restrict__ grad_scale, int32_t* __restrict__ dev_err) {
  if (head->magic != want.magic || head->tensors != want.tensors || head->chunks != want.chunks ||
      head->gtype != want.gtype || head->states != want.states || head->copies != want.copies) {
    if (threadIdx.x == 0) raise_err(dev_err, LM_DEVERR_CAPACITY);
    return;
  }
  __shared__ float inverse[EIGHT ? kScales : 1];
  if constexpr (EIGHT) fill_scales(inverse, kAdamwThreads);
  const PlanTensor* tensors = reinterpret_cast<const PlanTensor*>(head + 1);
  const PlanChunk chunk = reinterpret_cast<const PlanChunk*>(tensors + want.tensors)[blockIdx.x];
  const PlanTensor t = tensors[chunk.tensor];
  const int64_t at = static_cast<int64_t>(chunk.index) * kChunk;
  const int n = t.n - at < kChunk ? static_cast<int>(t.n - at) : kChunk;
  const float gs = grad_scale ? *grad_scale : 1.f;
  const float wd = t.decay * o.wd;
  const int i0 = threadIdx.x * kVec;
  float p[kVectors][kVec], g[kVectors][kVec], m[kVectors][kVec], v[kVectors][kVec];
  uint32_t mc[kVectors], vc[kVectors];
  int ms[kVectors], vs[kVectors];
#pragma unroll
  for (int j = 0; j < kVectors; ++j) {
    const int i = i0 + j * kAdamwThreads * kVec, have = n - i;
    mc[j] = vc[j] = 0;
    ms[j] = vs[j] = 0;
    if (have <= 0) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) p[j][e] = g[j][e] = m[j][e] = v[j][e] = 0.f;
      continue;
    }
    load4(t.p + at + i, have, p[j]);
    load4(static_cast<const GT*>(t.g) + at + i, have, g[j]);
    if constexpr (EIGHT) {
      mc[j] = load_codes(static_cast<const uint8_t*>(t.m) + at + i, have);
      vc[j] = load_codes(static_cast<const uint8_t*>(t.v) + at + i, have);
      ms[j] = t.m_scale[(at + i) / kMomentBlock];
      vs[j] = t.v_scale[(at + i) / kMomentBlock];
    } else {
      load4(static_cast<const float*>(t.m) + at + i, have, m[j]);
      load4(static_cast<const float*>(t.v) + at + i, have, v[j]);
    }
  }
  bool ok = true;
#pragma unroll
  for (int j = 0; j < kVectors; ++j) {
    const int i = i0 + j * kAdamwThreads * kVec, have = n - i;
    if constexpr (EIGHT) {
      decode4(mc[j], ms[j], m[j]);
      decode4(vc[j], vs[j], v[j]);
    }
    uint32_t word[kVec], low[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float x = g[j][e] * gs;
      if constexpr (EIGHT) {
        ok &= adamw_value8(p[j][e], m[j][e], v[j][e], x, wd, q);
        word[e] = value_word(static_cast<uint64_t>(t.first + at + i + e), keys);
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
      mc[j] = encode4<false>(m[j], word, inverse, ms[j]);
      vc[j] = encode4<true>(v[j], low, inverse, vs[j]);
    }
    if (have <= 0) continue;
    store4(t.p + at + i, have, p[j]);
    if constexpr (COPY) store4(t.copy + at + i, have, p[j]);
    if constexpr (EIGHT) {
      store_codes(static_cast<uint8_t*>(t.m) + at + i, have, mc[j]);
      store_codes(static_cast<uint8_t*>(t.v) + at + i, have, vc[j]);
      if ((threadIdx.x & 7) == 0) {
        t.m_scale[(at + i) / kMomentBlock] = static_cast<uint8_t>(ms[j]);
        t.v_scale[(at + i) / kMomentBlock] = static_cast<uint8_t>(vs[j]);
      }
    } else {
      store4(static_cast<float*>(t.m) + at + i, have, m[j]);
      store4(static_cast<float*>(t.v) + at + i, have, v[j]);
    }
  }
  if (ballot(!ok) && lane_id() == 0) raise_err(dev_err, LM_DEVERR_NONFINITE);
}

// ---------------------------------------------------------------------------
// The lazy step on the rows of a table: one wave per row (grid-stride).
// ---------------------------------------------------------------------------
template <typename KeyT>
__global__ __launch_bounds__(kAdamwThreads) void k_rows8(
    float* __restrict__ table, int64_t V, int D, int64_t ld_table, const KeyT* __restrict__ rows,
    const int64_t* __restrict__ n_rows, int64_t rows_cap, const float* __restrict__ vals,
    int64_t ld_vals, MomentParams q, StepKeys keys, uint8_t* __restrict__ m,
    uint8_t* __restrict__ v, int64_t ld_codes, uint8_t* __restrict__ m_scale,
    uint8_t* __restrict__ v_scale, int64_t ld_scale, int64_t nwaves,
    int32_t* __restrict__ dev_err) {
  __shared__ float inverse[kScales];
  fill_scales(inverse, kAdamwThreads);
  const int lane = lane_id();
  const int64_t w = first_lane(static_cast<int64_t>(blockIdx.x) * (kAdamwThreads / kWave) +
                               (threadIdx.x >> 6));
  int64_t count = first_lane(*n_rows);
  if (count > rows_cap) {
    if (w == 0 && lane == 0) raise_err(dev_err, LM_DEVERR_CAPACITY);
    count = rows_cap;
  }
  bool ok = true;
  for (int64_t u = w; u < count; u += nwaves) {
    const int64_t id = first_lane(static_cast<int64_t>(rows[u]));
    if (!(id >= 0 && id < V)) {
      if (lane == 0) raise_err(dev_err, LM_DEVERR_ID_RANGE);
      continue;
    }
    float* prow = table + id * ld_table;
    const float* grow = vals + u * ld_vals;
    uint8_t *mrow = m + id * ld_codes, *vrow = v + id * ld_codes;
    uint8_t *msrow = m_scale + id * ld_scale, *vsrow = v_scale + id * ld_scale;
    for (int cb = 0; cb < D; cb += kVectors * kWave * kVec) {
      float p[kVectors][kVec], g[kVectors][kVec];
      uint32_t mc[kVectors], vc[kVectors];
      int ms[kVectors], vs[kVectors];
#pragma unroll
      for (int j = 0; j < kVectors; ++j) {
        const int c = cb + (j * kWave + lane) * kVec, have = D - c;
        mc[j] = vc[j] = 0;
        ms[j] = vs[j] = 0;
        if (have <= 0) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) p[j][e] = g[j][e] = 0.f;
          continue;
        }
        load4(prow + c, have, p[j]);
        load4(grow + c, have, g[j]);
        mc[j] = load_codes(mrow + c, have);
        vc[j] = load_codes(vrow + c, have);
        ms[j] = msrow[c / kMomentBlock];
        vs[j] = vsrow[c / kMomentBlock];
      }
#pragma unroll
      for (int j = 0; j < kVectors; ++j) {
        const int c = cb + (j * kWave + lane) * kVec, have = D - c;
        float mx[kVec], vx[kVec];
        uint32_t word[kVec], low[kVec];
        decode4(mc[j], ms[j], mx);
        decode4(vc[j], vs[j], vx);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          ok &= adamw_value8(p[j][e], mx[e], vx[e], g[j][e], q.wd, q);
          word[e] = value_word(static_cast<uint64_t>(id * D + c + e), keys);
          low[e] = word[e] << 12;
        }
        mc[j] = encode4<false>(mx, word, inverse, ms[j]);
        vc[j] = encode4<true>(vx, low, inverse, vs[j]);
        if (have <= 0) continue;
        store4(prow + c, have, p[j]);
        store_codes(mrow + c, have, mc[j]);
        store_codes(vrow + c, have, vc[j]);
        if ((lane & 7) == 0) {
          msrow[c / kMomentBlock] = static_cast<uint8_t>(ms[j]);
          vsrow[c / kMomentBlock] = static_cast<uint8_t>(vs[j]);
        }
      }
    }
  }
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

size_t adamw_plan_bytes(const int64_t* sizes, int64_t tensors) {
  return sizeof(PlanHead) + static_cast<size_t>(tensors) * sizeof(PlanTensor) +
         static_cast<size_t>(adamw_plan_chunks(sizes, tensors)) * sizeof(PlanChunk);
}

static PlanHead plan_head(int64_t tensors, int64_t chunks, int gtype, int states, bool copies) {
  PlanHead h{};
  h.magic = kPlanMagic;
  h.tensors = tensors;
  h.chunks = chunks;
  h.gtype = gtype;
  h.states = states;
  h.copies = copies ? 1 : 0;
  return h;
}

void adamw_plan_write(void* const* p, const void* const* g, void* const* m, void* const* v,
                      void* const* m_scale, void* const* v_scale, void* const* copies,
                      const int64_t* sizes, const int32_t* decay, int64_t tensors, int gtype,
                      int states, void* plan) {
  PlanHead* head = static_cast<PlanHead*>(plan);
  *head = plan_head(tensors, adamw_plan_chunks(sizes, tensors), gtype, states, copies != nullptr);
  PlanTensor* t = reinterpret_cast<PlanTensor*>(head + 1);
  PlanChunk* c = reinterpret_cast<PlanChunk*>(t + tensors);
  int64_t first = 0;
  for (int64_t i = 0; i < tensors; ++i) {
    t[i] = PlanTensor{static_cast<float*>(p[i]), g[i], m[i], v[i],
                      m_scale ? static_cast<uint8_t*>(m_scale[i]) : nullptr,
                      v_scale ? static_cast<uint8_t*>(v_scale[i]) : nullptr,
                      copies ? static_cast<uint16_t*>(copies[i]) : nullptr, sizes[i], first,
                      !decay || decay[i] ? 1.f : 0.f, 0};
    first += (sizes[i] + kMomentBlock - 1) / kMomentBlock * kMomentBlock;
    for (int64_t k = 0; k < chunks_of(sizes[i]); ++k)
      *c++ = PlanChunk{static_cast<uint32_t>(i), static_cast<uint32_t>(k)};
  }
}

template <typename GT, bool EIGHT>
static void adamw_launch(const PlanHead& want, const void* plan, const OptParams& o,
                         const MomentParams& q, const StepKeys& keys, const float* grad_scale,
                         int32_t* dev_err, hipStream_t st) {
  const PlanHead* head = static_cast<const PlanHead*>(plan);
  const dim3 grid(static_cast<uint32_t>(want.chunks));
  if (want.copies)
    k_adamw<GT, EIGHT, true><<<grid, kAdamwThreads, 0, st>>>(head, want, o, q, keys, grad_scale,
                                                             dev_err);
  else
    k_adamw<GT, EIGHT, false><<<grid, kAdamwThreads, 0, st>>>(head, want, o, q, keys, grad_scale,
                                                              dev_err);
}

int adamw_run(const void* plan, int64_t tensors, int64_t chunks, int gtype, int states,
              bool copies, float lr, float beta1, float beta2, float eps, float weight_decay,
              int64_t step, const float* grad_scale, uint64_t seed, int32_t* dev_err,
              hipStream_t st) {
  if (chunks == 0) return LM_OK;
  const OptParams o = make_opt_params(true, lr, beta1, beta2, eps, weight_decay, step, 1.f);
  const MomentParams q = make_moment_params(o, beta2, step);
  const PlanHead want = plan_head(tensors, chunks, gtype, states, copies);
  const StepKeys keys = step_keys(seed);
  const bool eight = states == 8;
  if (gtype == LM_BF16) {
    if (eight) adamw_launch<bf16_t, true>(want, plan, o, q, keys, grad_scale, dev_err, st);
    else adamw_launch<bf16_t, false>(want, plan, o, q, keys, grad_scale, dev_err, st);
  } else {
    if (eight) adamw_launch<float, true>(want, plan, o, q, keys, grad_scale, dev_err, st);
    else adamw_launch<float, false>(want, plan, o, q, keys, grad_scale, dev_err, st);
  }
  return launch_status(hipGetLastError());
}

int rows8_run(float* table, int64_t V, int64_t D, int64_t ld_table, const void* rows, int idtype,
              const int64_t* n_rows, int64_t rows_cap, const float* vals, int64_t ld_vals,
              float lr, float beta1, float beta2, float eps, float weight_decay, int64_t step,
              uint8_t* m, uint8_t* v, int64_t ld_codes, uint8_t* m_scale, uint8_t* v_scale,
              int64_t ld_scale, uint64_t seed, int32_t* dev_err, hipStream_t st) {
  if (D == 0 || rows_cap == 0) return LM_OK;
  const OptParams o = make_opt_params(true, lr, beta1, beta2, eps, weight_decay, step, 1.f);
  const MomentParams q = make_moment_params(o, beta2, step);
  const StepKeys keys = step_keys(seed);
  constexpr int kWaves = kAdamwThreads / kWave;
  const int64_t waves = rows_cap < (int64_t(1) << 20) ? rows_cap : int64_t(1) << 20;
  const uint32_t blocks = static_cast<uint32_t>((waves + kWaves - 1) / kWaves);
  if (idtype == LM_I64)
    k_rows8<int64_t><<<blocks, kAdamwThreads, 0, st>>>(
        table, V, static_cast<int>(D), ld_table, static_cast<const int64_t*>(rows), n_rows,
        rows_cap, vals, ld_vals, q, keys, m, v, ld_codes, m_scale, v_scale, ld_scale,
        int64_t(blocks) * kWaves, dev_err);
  else
    k_rows8<int32_t><<<blocks, kAdamwThreads, 0, st>>>(
        table, V, static_cast<int>(D), ld_table, static_cast<const int32_t*>(rows), n_rows,
        rows_cap, vals, ld_vals, q, keys, m, v, ld_codes, m_scale, v_scale, ld_scale,
        int64_t(blocks) * kWaves, dev_err);
  return launch_status(hipGetLastError());
}

}  // namespace lmz
