// Log probabilities of given tokens with entropy and top alternatives, and their
// gradient. Of a row of logits x, with c = scale and m = max x,
//     S = sum e^(c (x - m)),  E = sum e^(c (x - m)) c (x - m),  log_sum = log S,
//     logp = c (x_t - m) - log_sum,  entropy = log_sum - E / S,
// and, with l = c (x - m) - log_sum and q = e^l,
//     dx = c (dlogp (1 at t - q) - dentropy q (l + entropy)).
// The statistics are relative to m, not one number log sum e^(c x): l then keeps its
// digits however far from zero a row lies.
//
// Forward: one pass over the logits, each lane with a running m, S and E in base 2. HBM and the
// vector units bound it alike: a logit takes 7.5 instructions and a v_exp_f32, which has a
// quarter of their rate. Short rows stay in the registers of some lanes, others go to a
// workgroup, and where these are few to several, which k_logp_join puts together. 8192 x 100,000
// bf16: 255 us, 6.4 TB/s. Backward: one pass that reads and writes each element once, bound by
// HBM: the same in 535 us, 6.1 TB/s.
#include "launch_parts.hpp"
#include "patch.hpp"

namespace lmz {

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
constexpr float kFarBelow = -1000.f;  // 2^this is 0
constexpr float kInf = __builtin_inff();
constexpr int kTopKeys = 1024;  // candidates of a row's alternatives
static_assert(LM_TOP_MAX == kWave, "a wave ranks the groups' maxima");

// The larger number; NaN if one of them is (v_maximum3_f32).
__device__ __forceinline__ float larger(float a, float b) {
  return __builtin_elementwise_maximum(a, b);
}

// A row's sums so far: its maximum m (NaN for good once it met one) and, with c = scale log2 e,
//     s = sum 2^(c x - b),  e = sum 2^(c x - b) (c x - b)
// relative to b, the fp32 number next to c m: then each exponent is one fma, and b's rounding
// (slip, at most 2^-5) is known where the sums are used. From |c m| = 2^20 on (masks of the
// type's lowest value among them) that rounding may be as large as the exponents, and they are
// relative to c m itself: c (x - m). s and e are 0 while m is -infinity.
struct Sums {
  float m, s, e;
  static __device__ __forceinline__ bool plain(float b) { return __builtin_fabsf(b) < 0x1p20f; }
  // c m - b.
  static __device__ __forceinline__ float slip(float m, float c) {
    const float b = m * c;
    return plain(b) ? __builtin_fmaf(m, c, -b) : 0.f;
  }
  // The sums relative to `to`, which is no less than m.
  __device__ __forceinline__ void rebase(float to, float c) {
#pragma clang fp contract(off)  // the b of both are rounded numbers
    float by = m * c - to * c;
    const bool ok = plain(m * c) && plain(to * c);
    if (ballot(!ok && m > -kInf)) by = ok ? by : (m - to) * c - slip(m, c) + slip(to, c);
    by = __builtin_fmaxf(by, kFarBelow);  // (NaN, of infinity less itself, too)
    by = m == to || m == -kInf ? 0.f : by;
    const float f = __builtin_amdgcn_exp2f(by);
    e = f * __builtin_fmaf(s, by, e);
    s *= f;
    m = to;
  }
  __device__ __forceinline__ void add(Sums o, float c) {
    const float to = larger(m, o.m);
    rebase(to, c);
    o.rebase(to, c);
    s += o.s;
    e += o.e;
  }
};

// N logits (masked ones -infinity), none above t.m.
template <int N>
__device__ __forceinline__ void sum_logits(Sums& t, const float* x, float c) {
  const float m = t.m == -kInf ? 0.f : t.m, b = m * c;
  float s = 0.f, e = 0.f;
  auto add = [&](float d) {
    d = __builtin_fmaxf(d, kFarBelow);  // 0 times no infinity below
    const float p = __builtin_amdgcn_exp2f(d);
    s += p;
    e = __builtin_fmaf(p, d, e);
  };
  const bool ok = Sums::plain(b);
  if (!ballot(!ok)) {
#pragma unroll
    for (int i = 0; i < N; ++i) add(__builtin_fmaf(x[i], c, -b));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) add(ok ? __builtin_fmaf(x[i], c, -b) : (x[i] - m) * c);
  }
  t.s += s;
  t.e += e;
}

// N logits, any.
template <int N>
__device__ __forceinline__ void add_logits(Sums& t, const float* x, float c) {
  float top = t.m;
#pragma unroll
  for (int i = 0; i < N; ++i) top = larger(top, x[i]);
  t.rebase(top, c);
  sum_logits<N>(t, x, c);
}

// One number for a logit and its id: larger logits first, of equal ones the lowest id; 0 is
// below all of them.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t id) {
  const uint32_t b = __float_as_uint(x + 0.f);  // -0 is 0
  const uint32_t up = b & 0x80000000u ? ~b : b | 0x80000000u;
  return static_cast<uint64_t>(up) << 32 | ~id;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t up = static_cast<uint32_t>(k >> 32);
  return __uint_as_float(up & 0x80000000u ? up & 0x7fffffffu : ~up);
}
__device__ __forceinline__ uint32_t key_id(uint64_t k) { return ~static_cast<uint32_t>(k); }

template <int THREADS>
struct TopSpace {
  float best[THREADS];
  uint32_t list[kTopKeys];
  uint64_t keys[kTopKeys];
  uint64_t top[LM_TOP_MAX];
  uint64_t most[THREADS / kWave];
  int n, groups;
};

struct NoSpace {
  static constexpr const uint64_t* top = nullptr;
};

__device__ __forceinline__ uint64_t wave_max(uint64_t x) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) {
    const uint64_t y = __shfl_xor(x, off, kWave);
    x = y > x ? y : x;
  }
  return x;
}

// Of n different keys the k largest to their places in `top`, by THREADS threads. Eight keys
// under way at once: 300 x 50,000 bf16 with 64 alternatives takes 67 us, 74 with four; with 16,
// 63, but 65,536 x 1000 with 8 takes 78, 75 with eight.
template <int THREADS>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int k, uint64_t* top,
                                          int tid) {
  for (int i = tid; i < n; i += THREADS) {
    const uint64_t key = keys[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += keys[j] > key ? 1 : 0;
    if (rank < k) top[rank] = key;
  }
}

// The largest number of groups of LANES lanes, in all of them; NaN if one is.
template <int LANES>
__device__ __forceinline__ float lanes_larger(float x) {
  return lanes_fold<LANES>(x, [](float a, float b) { return larger(a, b); });
}

// The k-th largest of a wave's numbers (no NaN): fewer than k are above each of the k largest.
__device__ __forceinline__ float kth_largest(float x, int k) {
  int above = 0;
#pragma unroll
  for (int i = 0; i < kWave; ++i) above += read_lane(x, i) > x ? 1 : 0;
  return -lanes_larger<kWave>(above < k ? -x : -kInf);
}

// The k largest keys into t.top, 0 behind the last: `mine` is the largest of the thread's
// logits; pick(bound, want, f) calls f(logit, id) for those logits at least that may reach the
// bound (want: the thread's do), scan(f) for all of the thread's. Of the 64 maxima of groups of
// threads the k-th is a bound that k logits reach; only threads that reach it look through
// their logits again, and the few they find are ranked (64 x 800,000 bf16, 8 alternatives: 31 us
// with the parts' maxima alone, 37 with the k best of each part, found there). Where more than
// kTopKeys reach the bound (equal logits, or logits that few of the groups have), each key is
// found by a pass of its own. Near k = 64 the bound is the smallest of the maxima: about 300
// candidates in place of 24 at k = 20 (300 x 50,000 bf16: 67 us with 64 alternatives, 18 with 8).
template <int THREADS, typename Pick, typename Scan>
__device__ __forceinline__ void select_top(float mine, int k, TopSpace<THREADS>& t, Pick pick,
                                           Scan scan) {
  const int tid = threadIdx.x, lane = lane_id();
  mine = mine == mine ? mine : -kInf;  // (a NaN's row has no alternatives)
  t.best[tid] = mine;
  if (tid == 0) t.n = t.groups = 0;
  if (tid < LM_TOP_MAX) t.top[tid] = 0;
  __syncthreads();
  float group = t.best[lane];
#pragma unroll
  for (int i = 1; i < THREADS / kWave; ++i)
    group = __builtin_fmaxf(group, t.best[lane + i * kWave]);
  const float bound = kth_largest(group, k);
  pick(bound, mine >= bound && mine > -kInf, [&](float x, uint32_t id) {
    if (x >= bound && x > -kInf) {
      const int i = atomicAdd(&t.n, 1);
      if (i < kTopKeys) t.keys[i] = key_of(x, id);
    }
  });
  __syncthreads();
  const int n = t.n;
  if (n <= kTopKeys) {
    rank_keys<THREADS>(t.keys, n, k, t.top, tid);
    __syncthreads();
    return;
  }
  uint64_t last = ~uint64_t(0);
  for (int r = 0; r < k; ++r) {
    uint64_t best = 0;
    scan([&](float x, uint32_t id) {
      if (!(x > -kInf)) return;
      const uint64_t key = key_of(x, id);
      best = key < last && key > best ? key : best;
    });
    best = wave_max(best);
    if (lane == 0) t.most[tid / kWave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) best = t.most[w] > best ? t.most[w] : best;
    __syncthreads();
    if (best == 0) break;
    if (tid == 0) t.top[r] = best;
    last = best;
  }
  __syncthreads();
}

constexpr int kPartThreads = 256, kMaxima = kPartThreads / 4, kMostParts = 128;

struct LogpArgs {
  const void* logits;
  int64_t ld, N;
  int V, parts, part_vectors, k;
  const void* targets;
  int64_t ignore;
  int wide;  // targets are int64
  float scale, c;  // c: scale log2 e, and how far it is off that, relative to it
  float c_off;
  float *logp, *entropy, *peak, *log_sum, *top_logp;
  int32_t *top_ids, *dev_err;
  Sums* sums;     // [N][parts], where rows are cut
  float* maxima;  // [N][parts][kMaxima]: of kPartThreads / kMaxima neighbouring threads
};

// A row's target: whether it has one, its logit (NaN outside the vocabulary). The logit's
// load is under way until it is used.
struct Target {
  bool any, in;
  float x;
};

template <typename T>
__device__ __forceinline__ Target target_of(const LogpArgs& a, int64_t row) {
  if (!a.logp) return {false, false, 0.f};
  const int64_t id = a.wide ? static_cast<const int64_t*>(a.targets)[row]
                            : static_cast<const int32_t*>(a.targets)[row];
  const bool in = id >= 0 && id < a.V;
  return {id != a.ignore, in,
          Patch<T>::one(static_cast<const T*>(a.logits) + row * a.ld + (in ? id : 0))};
}

// What a row's sums and keys come to, by thread `tid` of `threads`.
__device__ __forceinline__ void finish_row(const LogpArgs& a, int64_t row, const Sums& t,
                                           const Target& target, const uint64_t* top, int tid,
                                           int threads) {
  const bool bad = !(t.m < kInf);  // a NaN or +infinity among the logits
  const float nan = __builtin_nanf("");
  const float slip = Sums::slip(t.m, a.c), mean = t.e / t.s;
  // s = 2^slip sum 2^(c (x - m)); c's own rounding moves its logarithm by the mean exponent.
  // The sum holds its maximum's own 1, so its logarithm is no less than 0: what comes out below is
  // the rounding of 2^slip (one word left at 6.0: -4.6e-8), and would be a probability above 1.
  const float log_sum =
      __builtin_fmaxf(logf(t.s) - kLn2 * (slip + a.c_off * (mean - slip)), 0.f);
  if (tid == 0) {
    if (a.logp) {
      const float x = target.in ? target.x : nan;
      if (target.any && !target.in) raise_err(a.dev_err, LM_DEVERR_ID_RANGE);
      const float y = x == -kInf ? x : (x - t.m) * a.scale - log_sum;
      a.logp[row] = target.any ? (bad ? nan : y) : 0.f;
    }
    const float h = logf(t.s) - kLn2 * mean;
    a.entropy[row] = bad ? nan : t.s == 0.f || h < 0.f ? 0.f : h;
    a.peak[row] = bad ? nan : t.m;
    a.log_sum[row] = bad ? nan : t.s == 0.f ? -kInf : log_sum;
  }
  for (int i = tid; i < a.k; i += threads) {
    const uint64_t key = top[i];
    const bool any = key != 0 && !bad;
    a.top_ids[row * a.k + i] = any ? static_cast<int32_t>(key_id(key)) : -1;
    a.top_logp[row * a.k + i] =
        bad ? nan : any ? (key_value(key) - t.m) * a.scale - log_sum : -kInf;
  }
}

// The sums of the workgroup's threads, added in a fixed order, in all of them.
template <int THREADS>
__device__ __forceinline__ Sums join_sums(Sums t, float c, Sums (&lds)[THREADS / kWave]) {
  t.rebase(lanes_larger<kWave>(t.m), c);
  t.s = lanes_sum<kWave>(t.s);
  t.e = lanes_sum<kWave>(t.e);
  if constexpr (THREADS > kWave) {
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = t;
    __syncthreads();
    t = lds[0];
#pragma unroll
    for (int w = 1; w < THREADS / kWave; ++w) t.add(lds[w], c);
  }
  return t;
}

// LDS instructions of a wave take effect in their order; the compiler has to keep it where
// lanes read what others wrote.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Rows that LANES lanes hold in registers, kRowVectors vectors each: no wave waits for another.
constexpr int kRowVectors = 4, kRowKeys = 256;

template <typename T, int LANES, bool TOP, Ends ENDS>
__global__ __launch_bounds__(kPartThreads) void k_logp_rows(LogpArgs a, uint32_t first) {
  static_assert(!TOP || LANES == kWave, "a wave ranks");
  constexpr int P = Patch<T>::P, U = kRowVectors, kRows = kPartThreads / LANES;
  constexpr int kWaves = kPartThreads / kWave;
  using raw_t = typename Patch<T>::raw_t;
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int64_t i = (first + static_cast<int64_t>(blockIdx.x)) * kRows +
                    (LANES == kWave ? first_lane(group) : group);
  const bool live = i < a.N;
  const int64_t row = live ? i : a.N - 1;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  const int vectors = (a.V + P - 1) / P;
  raw_t r[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u * LANES >= vectors) break;
    r[u] = Span<T, ENDS, uint32_t>((lane + u * LANES) * P, a.V).load(x);
  }
  const Target target = target_of<T>(a, row);
  float y[U * P];
  Sums t{-kInf, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u * LANES >= vectors) break;
    const Span<T, ENDS, uint32_t> s((lane + u * LANES) * P, a.V);
    s.widen(r[u], y + u * P);
#pragma unroll
    for (int e = 0; e < P; ++e) {
      y[u * P + e] = e < s.have ? y[u * P + e] : -kInf;
      t.m = larger(t.m, y[u * P + e]);
    }
  }
  float mine = t.m;
  t.m = lanes_larger<LANES>(t.m);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u * LANES >= vectors) break;
    sum_logits<P>(t, y + u * P, a.c);
  }
  t.s = lanes_sum<LANES>(t.s);
  t.e = lanes_sum<LANES>(t.e);
  if constexpr (!TOP) {
    if (live) finish_row(a, row, t, target, nullptr, lane, LANES);
  } else {
    // As select_top, with the logits at hand and every wave for itself. kRowKeys are passed by
    // half of the rows of random logits at k = 64, by few at 62 and by none at 60: 65,536 x 1000
    // bf16 takes 739 us with 64 alternatives, 384 with 62, 255 with 60, 86 with 20.
    __shared__ uint64_t keys[kWaves][kRowKeys], top[kWaves][LM_TOP_MAX];
    uint64_t *key = keys[group], *best = top[group];
    best[lane] = 0;
    mine = mine == mine ? mine : -kInf;
    const float bound = kth_largest(mine, a.k);
    int n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * LANES >= vectors) break;
#pragma unroll
      for (int e = 0; e < P; ++e) {
        const float z = y[u * P + e];
        const bool hit = z >= bound && z > -kInf;
        const uint64_t hits = ballot(hit);
        if (!hits) continue;
        const int at = n + popc_below(hits);
        if (hit && at < kRowKeys)
          key[at] = key_of(z, static_cast<uint32_t>((lane + u * LANES) * P + e));
        n += __popcll(hits);
      }
    }
    wave_order();
    if (n <= kRowKeys) {
      rank_keys<kWave>(key, n, a.k, best, lane);
    } else {
      uint64_t last = ~uint64_t(0);
      for (int rank = 0; rank < a.k; ++rank) {
        uint64_t k = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (u * LANES >= vectors) break;
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const uint64_t z = y[u * P + e] > -kInf
                                   ? key_of(y[u * P + e],
                                            static_cast<uint32_t>((lane + u * LANES) * P + e))
                                   : 0;
            k = z < last && z > k ? z : k;
          }
        }
        k = wave_max(k);
        if (k == 0) break;
        if (lane == 0) best[rank] = k;
        last = k;
      }
    }
    wave_order();
    if (live) finish_row(a, row, t, target, best, lane, LANES);
  }
}

// A row, or a part of one, by a workgroup.
template <typename T, bool TOP, bool PARTS>
__global__ __launch_bounds__(kPartThreads) void k_logp(LogpArgs a, uint32_t first) {
  constexpr int P = Patch<T>::P, U = 4, THREADS = kPartThreads;
  using raw_t = typename Patch<T>::raw_t;
  __shared__ Sums lds[THREADS / kWave];
  __shared__ std::conditional_t<TOP && !PARTS, TopSpace<THREADS>, NoSpace> space;
  const uint32_t b = first + blockIdx.x;
  const int64_t row = PARTS ? b / static_cast<uint32_t>(a.parts) : b;
  const int part = PARTS ? static_cast<int>(b - row * a.parts) : 0;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  const int vectors = (a.V + P - 1) / P, whole = a.V / P;
  const int v0 = part * a.part_vectors;
  const int v1 = a.part_vectors < vectors - v0 ? v0 + a.part_vectors : vectors;
  const int w1 = whole < v1 ? whole : v1;  // whole vectors
  Target target{};
  if constexpr (!PARTS) target = target_of<T>(a, row);
  // Vectors from number v1 on are loaded as the row's last one and count as masked.
  auto span = [&](int v) {
    return Span<T, Ends::PART>(static_cast<int64_t>(v) * P, a.V, v < v1);
  };
  auto place = [&](int v, const raw_t& r, float* y) {
    const auto s = span(v);
    s.widen(r, y);
#pragma unroll
    for (int e = 0; e < P; ++e) y[e] = e < s.have ? y[e] : -kInf;
  };
  Sums t{-kInf, 0.f, 0.f};
  int base = v0;
  for (; base + THREADS * U <= w1; base += THREADS * U) {
    const T* at = x + static_cast<int64_t>(base) * P;
    raw_t r[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      r[u] = Patch<T>::load(at + static_cast<uint32_t>(threadIdx.x + u * THREADS) * P);
    float y[U * P];
#pragma unroll
    for (int u = 0; u < U; ++u) Patch<T>::widen(r[u], y + u * P);
    add_logits<U * P>(t, y, a.c);
  }
  if (base < v1) {  // fewer than U vectors a thread
    raw_t r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = span(base + threadIdx.x + u * THREADS).load(x);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (base + u * THREADS >= v1) break;
      float y[P];
      place(base + threadIdx.x + u * THREADS, r[u], y);
      add_logits<P>(t, y, a.c);
    }
  }
  const float mine = t.m;
  t = join_sums<THREADS>(t, a.c, lds);
  if constexpr (PARTS) {
    const int64_t at = row * a.parts + part;
    if (threadIdx.x == 0) a.sums[at] = t;
    if constexpr (TOP) {
      static_assert(THREADS / kMaxima == 4, "a quad's maximum");
      const float quad = lanes_fold<4>(mine, [](float p, float q) { return larger(p, q); });
      if (threadIdx.x % 4 == 0) a.maxima[at * kMaxima + threadIdx.x / 4] = quad;
    }
  } else {
    if constexpr (TOP) {
      auto look = [&](int v, const raw_t& r, auto f) {
        float y[P];
        place(v, r, y);
#pragma unroll
        for (int e = 0; e < P; ++e) f(y[e], static_cast<uint32_t>(v * P + e));
      };
      select_top<THREADS>(
          mine, a.k, space,
          // Several lanes of the wave share out one thread's vectors.
          [&](float, bool want, auto f) {
            const int from = threadIdx.x & ~(kWave - 1), lane = lane_id();
            const int count = (v1 + THREADS - 1) / THREADS;  // vectors of a thread
            const int lanes = count <= 16 ? 16 : count <= 32 ? 32 : 64;
            for (int i0 = lane % lanes; i0 - lane % lanes < count; i0 += lanes) {
              for (uint64_t todo = ballot(want); todo;) {
                raw_t r[U];
                int v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                  v[u] = v1;
                  for (int l = 0; l < kWave; l += lanes) {
                    if (todo && lane / lanes == l / lanes)
                      v[u] = from + __builtin_ctzll(todo) + i0 * THREADS;
                    todo &= todo - 1;
                  }
                  r[u] = span(v[u]).load(x);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                  if (v[u] < v1) look(v[u], r[u], f);
              }
            }
          },
          [&](auto f) {
            for (int v = threadIdx.x; v < v1; v += THREADS) look(v, span(v).load(x), f);
          });
    }
    finish_row(a, row, t, target, space.top, threadIdx.x, THREADS);
  }
}

// One workgroup a row that is cut into parts: adds their sums, and looks through the logits
// of those groups of threads whose maxima reach the bound.
constexpr int kJoinThreads = 256;

template <typename T, bool TOP>
__global__ __launch_bounds__(kJoinThreads) void k_logp_join(LogpArgs a, uint32_t first) {
  constexpr int P = Patch<T>::P, U = 4;
  __shared__ Sums lds[kJoinThreads / kWave];
  __shared__ std::conditional_t<TOP, TopSpace<kJoinThreads>, NoSpace> space;
  const int64_t row = first + static_cast<int64_t>(blockIdx.x);
  // Everything is loaded at once: a thread's part, its share of the maxima.
  constexpr int kShare = kMostParts * kMaxima / kJoinThreads;
  static_assert(kMostParts <= kJoinThreads, "a part a thread");
  const int n = a.parts * kMaxima, mine_at = static_cast<int>(threadIdx.x);
  const Sums* sums = a.sums + row * a.parts;
  Sums t = sums[mine_at < a.parts ? mine_at : 0];
  float maxima[kShare], mine = -kInf;
  if constexpr (TOP) {
    const float* at = a.maxima + row * n;
#pragma unroll
    for (int j = 0; j < kShare; ++j) {
      if (j * kJoinThreads >= n) break;
      const int i = mine_at + j * kJoinThreads;
      maxima[j] = at[i < n ? i : 0];
    }
  }
  const Target target = target_of<T>(a, row);
  if (mine_at >= a.parts) t = Sums{-kInf, 0.f, 0.f};
  if constexpr (TOP) {
#pragma unroll
    for (int j = 0; j < kShare; ++j) {
      if (j * kJoinThreads >= n) break;
      maxima[j] = mine_at + j * kJoinThreads < n ? maxima[j] : -kInf;
      mine = larger(mine, maxima[j]);
    }
  }
  t = join_sums<kJoinThreads>(t, a.c, lds);
  if constexpr (TOP) {
    const T* x = static_cast<const T*>(a.logits) + row * a.ld;
    const int vectors = (a.V + P - 1) / P;
    auto span = [&](int v) {
      return Span<T, Ends::PART>(static_cast<int64_t>(v) * P, a.V, v < vectors);
    };
    auto look = [&](int v, const typename Patch<T>::raw_t& r, auto f) {
      const auto s = span(v);
      float y[P];
      s.widen(r, y);
#pragma unroll
      for (int e = 0; e < P; ++e)
        if (e < s.have) f(y[e], static_cast<uint32_t>(v * P + e));
    };
    select_top<kJoinThreads>(
        mine, a.k, space,
        [&](float bound, bool want, auto f) {
#pragma unroll
          for (int j = 0; j < kShare; ++j) {
            if (j * kJoinThreads >= n) break;
            if (!want || !(maxima[j] >= bound && maxima[j] > -kInf)) continue;
            const int at = atomicAdd(&space.groups, 1);
            if (at < kTopKeys) space.list[at] = mine_at + j * kJoinThreads;
          }
          __syncthreads();
          const int groups = space.groups;
          if (groups > kTopKeys) {
            if (threadIdx.x == 0) space.n = kTopKeys + 1;
            return;
          }
          const int turns = (a.part_vectors + kPartThreads - 1) / kPartThreads;
          const int each = turns * 4, all = groups * each;
          for (int i0 = threadIdx.x; i0 - mine_at < all; i0 += kJoinThreads * U) {
            typename Patch<T>::raw_t r[U];
            int v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const int i = i0 + u * kJoinThreads;
              const int at = i < all ? i / each : 0, j = i - at * each;
              const int g = space.list[at], part = g / kMaxima;
              const int in = g % kMaxima * 4 + j % 4 + j / 4 * kPartThreads;
              v[u] = i < all && in < a.part_vectors ? part * a.part_vectors + in : vectors;
              r[u] = span(v[u]).load(x);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (v[u] < vectors) look(v[u], r[u], f);
          }
        },
        [&](auto f) {
          for (int v = threadIdx.x; v < vectors; v += kJoinThreads) look(v, span(v).load(x), f);
        });
  }
  finish_row(a, row, t, target, space.top, threadIdx.x, kJoinThreads);
}

// ---------------------------------------------------------------------------
// Gradient
// ---------------------------------------------------------------------------
struct LogpGradArgs {
  const void* logits;
  int64_t ld, N;
  int V, tiles;
  const void* targets;
  int64_t ignore;
  int wide;
  float scale, c;  // c: scale log2 e
  const float *peak, *log_sum, *dlogp, *entropy, *dentropy;
  void* out;
  int64_t ld_out;
};

// A workgroup: kGradThreads / LANES rows, of each a tile of LANES * kGradVectors vectors.
// 8192 x 100,000 bf16: 535 us with 2 of these, 546 with 4, 557 with 1; 1 x 100,000 2.6, 3.3, 2.3;
// 262,144 x 98 fp32 54, 55, 91.
constexpr int kGradThreads = 256, kGradVectors = 2;

template <typename T, int LANES, bool ENTROPY, Ends ENDS>
__global__ __launch_bounds__(kGradThreads) void k_logp_grad(LogpGradArgs a, uint32_t first) {
  constexpr int P = Patch<T>::P, U = kGradVectors, kRows = kGradThreads / LANES;
  using raw_t = typename Patch<T>::raw_t;
  const uint32_t b = first + blockIdx.x;
  const uint32_t group = b / static_cast<uint32_t>(a.tiles);
  const int tile = static_cast<int>(b - group * a.tiles);
  int64_t row = static_cast<int64_t>(group) * kRows;
  if constexpr (kRows > 1) row += threadIdx.x / LANES;
  const bool live = row < a.N;
  row = live ? row : a.N - 1;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  T* out = static_cast<T*>(a.out) + row * a.ld_out;
  const int vectors = (a.V + P - 1) / P;
  const int v0 = tile * LANES * U + threadIdx.x % LANES;
  raw_t r[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int v = v0 + u * LANES;
    if ((tile * U + u) * LANES >= vectors) break;
    r[u] = Span<T, ENDS>(static_cast<int64_t>(v) * P, a.V, v < vectors).load(x);
  }
  float dlogp = 0.f;
  int target = -1;
  if (a.dlogp) {
    const int64_t id = a.wide ? static_cast<const int64_t*>(a.targets)[row]
                              : static_cast<const int32_t*>(a.targets)[row];
    if (id != a.ignore) {
      dlogp = id < 0 || id >= a.V ? __builtin_nanf("") : a.dlogp[row] * a.scale;
      target = id < 0 || id >= a.V ? -1 : static_cast<int>(id);
    }
  }
  const float peak = a.peak[row], log_sum = a.log_sum[row], log2_sum = log_sum * kLog2e;
  float entropy = 0.f, dentropy = 0.f;
  if constexpr (ENTROPY) {
    entropy = a.entropy[row];
    dentropy = a.dentropy[row] * a.scale;
  }
  // Nothing is left of the row, or nothing depends on it: zeros, whatever its logits are.
  const bool none = peak == -kInf || (dlogp == 0.f && dentropy == 0.f);
  if (!live) return;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int v = v0 + u * LANES;
    if (v >= vectors) break;
    const Span<T, ENDS> s(static_cast<int64_t>(v) * P, a.V);
    float y[P];
    s.widen(r[u], y);
#pragma unroll
    for (int e = 0; e < P; ++e) {
      float l, q;
      if constexpr (sizeof(T) == 4) {
        // fp32 gradients: the exponent's rounding and the rest of log2 e, to first order
        constexpr float kRest = 1.925963033e-8f;  // log2 e - kLog2e
        l = __builtin_fmaf(y[e] - peak, a.scale, -log_sum);
        const float z = l * kLog2e, rest = __builtin_fmaf(l, kLog2e, -z) + l * kRest;
        q = __builtin_amdgcn_exp2f(z);
        q = l > kFarBelow ? __builtin_fmaf(q, rest * kLn2, q) : q;
      } else {
        const float z = __builtin_fmaf(y[e] - peak, a.c, -log2_sum);
        q = __builtin_amdgcn_exp2f(z);
        l = z * kLn2;
      }
      float d = -dlogp * q;
      if constexpr (ENTROPY)
        d = __builtin_fmaf(-dentropy * q, __builtin_fmaxf(l, kFarBelow) + entropy, d);
      y[e] = d;
    }
    const int hit = target - v * P;
    if (hit >= 0 && hit < P) {
#pragma unroll
      for (int e = 0; e < P; ++e) y[e] += e == hit ? dlogp : 0.f;
    }
    if (none) {
#pragma unroll
      for (int e = 0; e < P; ++e) y[e] = 0.f;
    }
    s.store(out, y);
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct LogpPlan {
  int64_t parts, part_vectors;
};

// Rows go to a workgroup each where there are kFullGroups of them, or where they are short;
// others are cut into parts, at most kMostParts (each more costs the one workgroup that joins
// them), so that about that many workgroups have work. 64 rows of 800,000
// bf16, 8 alternatives: 31 us so, with half as many workgroups 38, with twice as many 31; 1 x
// 800,000, 20 alternatives: 14 us in 98 parts, 27 in 391.
constexpr int64_t kFullGroups = 1024, kWholeVectors = 1024;

static LogpPlan logp_plan(int64_t N, int64_t V, int dtype) {
  const int P = dtype == LM_BF16 ? Patch<bf16_t>::P : Patch<float>::P;
  const int64_t vectors = (V + P - 1) / P;
  if (N >= kFullGroups || vectors <= kWholeVectors) return {1, vectors};
  // Vectors of a thread.
  int64_t each = N * vectors / (kFullGroups * kPartThreads) + 1;
  const int64_t least = (vectors - 1) / (kMostParts * kPartThreads) + 1;
  each = each > least ? each : least;
  const int64_t parts = (vectors - 1) / (each * kPartThreads) + 1;
  each = (vectors - 1) / parts + 1;
  return {(vectors - 1) / each + 1, each};
}

static size_t sums_bytes(int64_t n) {
  return (static_cast<size_t>(n) * sizeof(Sums) + 15) / 16 * 16;
}

size_t logp_workspace_bytes(int64_t N, int64_t V, int dtype, int k) {
  const int64_t parts = logp_plan(N, V, dtype).parts;
  if (parts == 1) return 0;
  return sums_bytes(N * parts) + (k ? static_cast<size_t>(N * parts) * kMaxima * 4 : 0);
}

template <typename T>
static int logp_launch(const LogpArgs& a, hipStream_t st) {
  constexpr int P = Patch<T>::P;
  const bool top = a.k > 0;
  auto launch = [&](auto kernel, int64_t blocks, int threads) {
    return launch_parts(blocks, threads, [&](uint32_t first, uint32_t n) {
      kernel<<<n, threads, 0, st>>>(a, first);
      return launch_status(hipGetLastError());
    });
  };
  const int64_t vectors = (static_cast<int64_t>(a.V) + P - 1) / P;
  if (vectors <= kWave * kRowVectors) {
    const bool part = !top && vectors <= 16 * kRowVectors;  // 16 lanes a row
    const bool narrow = a.V < P;
    auto kernel = narrow ? (top ? k_logp_rows<T, kWave, true, Ends::NARROW>
                                : k_logp_rows<T, 16, false, Ends::NARROW>)
                  : top  ? k_logp_rows<T, kWave, true, Ends::PART>
                  : part ? k_logp_rows<T, 16, false, Ends::PART>
                         : k_logp_rows<T, kWave, false, Ends::PART>;
    const int rows = kPartThreads / (part ? 16 : kWave);
    return launch(kernel, (a.N + rows - 1) / rows, kPartThreads);
  }
  if (a.parts == 1)
    return launch(top ? k_logp<T, true, false> : k_logp<T, false, false>, a.N, kPartThreads);
  const int rc = launch(top ? k_logp<T, true, true> : k_logp<T, false, true>, a.N * a.parts,
                        kPartThreads);
  if (rc != LM_OK) return rc;
  return launch(top ? k_logp_join<T, true> : k_logp_join<T, false>, a.N, kJoinThreads);
}

int logp_run(const void* logits, int64_t ld, int64_t N, int64_t V, int dtype, const void* targets,
             int idtype, int64_t ignore, float scale, int k, float* logp, float* entropy,
             float* peak, float* log_sum, float* top_logp, int32_t* top_ids, int32_t* dev_err,
             void* ws, hipStream_t st) {
  if (N == 0) return LM_OK;
  const LogpPlan p = logp_plan(N, V, dtype);
  char* maxima = ws ? static_cast<char*>(ws) + sums_bytes(N * p.parts) : nullptr;
  const double log2e = 1.4426950408889634 * static_cast<double>(scale);
  const float c = static_cast<float>(log2e);
  const LogpArgs a{logits, ld, N, static_cast<int>(V), static_cast<int>(p.parts),
                   static_cast<int>(p.part_vectors), k, targets, ignore, idtype == LM_I64, scale, c,
                   static_cast<float>(c / log2e - 1.0),
                   targets ? logp : nullptr, entropy, peak, log_sum, top_logp, top_ids, dev_err,
                   static_cast<Sums*>(ws),
                   reinterpret_cast<float*>(maxima)};
  return dtype == LM_BF16 ? logp_launch<bf16_t>(a, st) : logp_launch<float>(a, st);
}

template <typename T, int LANES>
static int grad_launch(LogpGradArgs a, hipStream_t st) {
  constexpr int P = Patch<T>::P, kRows = kGradThreads / LANES;
  const int64_t vectors = (static_cast<int64_t>(a.V) + P - 1) / P;
  a.tiles = static_cast<int>((vectors + LANES * kGradVectors - 1) / (LANES * kGradVectors));
  auto kernel = a.dentropy ? k_logp_grad<T, LANES, true, Ends::PART>
                           : k_logp_grad<T, LANES, false, Ends::PART>;
  if constexpr (LANES == 16)
    if (a.V < P)
      kernel = a.dentropy ? k_logp_grad<T, LANES, true, Ends::NARROW>
                          : k_logp_grad<T, LANES, false, Ends::NARROW>;
  return launch_parts((a.N + kRows - 1) / kRows * a.tiles, kGradThreads,
                      [&](uint32_t first, uint32_t n) {
                        kernel<<<n, kGradThreads, 0, st>>>(a, first);
                        return launch_status(hipGetLastError());
                      });
}

template <typename T>
static int grad_lanes(const LogpGradArgs& a, hipStream_t st) {
  const int64_t vectors = (static_cast<int64_t>(a.V) + Patch<T>::P - 1) / Patch<T>::P;
  if (vectors <= 16 * kGradVectors) return grad_launch<T, 16>(a, st);
  if (vectors <= 64 * kGradVectors) return grad_launch<T, 64>(a, st);
  return grad_launch<T, 256>(a, st);
}

// Workgroups of a call, for the check of the grid's size.
int64_t logp_grad_blocks(int64_t N, int64_t V, int dtype) {
  const int P = dtype == LM_BF16 ? Patch<bf16_t>::P : Patch<float>::P;
  const int64_t vectors = (V + P - 1) / P;
  return (vectors + 256 * kGradVectors - 1) / (256 * kGradVectors) * N;
}

int logp_grad_run(const void* logits, int64_t ld, int64_t N, int64_t V, int dtype,
                  const void* targets, int idtype, int64_t ignore, float scale, const float* peak,
                  const float* log_sum, const float* dlogp, const float* entropy,
                  const float* dentropy, void* out, int64_t ld_out, hipStream_t st) {
  if (N == 0) return LM_OK;
  const LogpGradArgs a{logits, ld, N, static_cast<int>(V), 0, targets, ignore, idtype == LM_I64,
                       scale, static_cast<float>(1.4426950408889634 * static_cast<double>(scale)),
                       peak, log_sum, targets ? dlogp : nullptr, entropy, dentropy, out,
                       ld_out};
  return dtype == LM_BF16 ? grad_lanes<bf16_t>(a, st) : grad_lanes<float>(a, st);
}

}  // namespace lmz
