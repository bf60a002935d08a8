// Dropout: out = add + x kept / (1 - p), and its gradient (the same on dout). One pass,
// bound by HBM: 2 or 3 elements moved for each, the mask made in registers (keep.hpp).
//
// A thread takes one 16-byte vector of the rows as if these lay one behind the other; which row
// it is in comes from one product (Divide), so no shape leaves lanes idle. 65,536 x 2048 bf16
// with a residual: 124 us, 6.5 TB/s (four vectors a thread, their loads under way at once, 127;
// without the residual 86 and 89; 3,000,000 x 3 bf16 21 and 27); 700 x 650 fp32 2.8 us (3.5),
// of which a launch and two trips to memory take most.
#include "keep.hpp"
#include "patch.hpp"

namespace lmz {

constexpr int kDropThreads = 256;

// n / d for n below 2^31: with 2^(l-1) < d <= 2^l and m = floor(2^(31+l) / d) + 1,
// m d - 2^(31+l) is in (0, 2^l], so n m / 2^(31+l) is above n / d by less than 1 / d.
struct Divide {
  uint32_t d, m, shift;
  explicit Divide(uint32_t by) : d(by), shift(0) {
    while ((uint64_t(1) << shift) < by) ++shift;
    m = static_cast<uint32_t>((uint64_t(1) << (31 + shift)) / by + 1);
    shift += 31;
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const {
    return static_cast<uint32_t>((static_cast<uint64_t>(n) * m) >> shift);
  }
};

struct DropArgs {
  int64_t D, ld_x, ld_add, ld_out;
  uint64_t word;     // of the first row
  uint32_t vectors;  // of the launch
  Divide per_row;
};

template <typename T, bool ADD, Ends ENDS>
__global__ __launch_bounds__(kDropThreads) void k_dropout(const T* x, const T* add, T* out,
                                                         DropArgs a, KeepArgs ka) {
  constexpr int P = Patch<T>::P;
  const uint32_t v = blockIdx.x * kDropThreads + threadIdx.x;
  if (v >= a.vectors) return;
  const uint32_t row = a.per_row(v), vec = v - row * a.per_row.d;
  const Span<T, ENDS> s(static_cast<int64_t>(vec) * P, a.D);
  const auto rx = s.load(x + row * a.ld_x);
  typename Patch<T>::raw_t ra;
  if constexpr (ADD) ra = s.load(add + row * a.ld_add);
  const Keep keep(ka);
  const uint64_t pairs = static_cast<uint64_t>(a.D + 1) / 2;
  float y[P];
  s.widen(rx, y);
  keep.apply<P>(a.word + row * pairs + vec * (P / 2), y);
  if constexpr (ADD) {
    float z[P];
    s.widen(ra, z);
#pragma unroll
    for (int e = 0; e < P; ++e) y[e] += z[e];
  }
  s.store(out + row * a.ld_out, y);
}

template <typename T>
static int dropout_launch(const T* x, int64_t ld_x, const T* add, int64_t ld_add, T* out,
                          int64_t ld_out, int64_t rows, int64_t D, const KeepArgs& k,
                          hipStream_t st) {
  constexpr int P = Patch<T>::P;
  const int64_t per_row = (D + P - 1) / P, pairs = (D + 1) / 2;
  const bool narrow = D < P;
  auto kernel = add ? (narrow ? k_dropout<T, true, Ends::NARROW> : k_dropout<T, true, Ends::PART>)
                    : (narrow ? k_dropout<T, false, Ends::NARROW>
                              : k_dropout<T, false, Ends::PART>);
  // Rows of a launch: vectors are counted in 31 bits, the last workgroup's included.
  const int64_t most = ((int64_t(1) << 31) - kDropThreads) / per_row;
  for (int64_t r = 0; r < rows; r += most) {
    const int64_t n = rows - r < most ? rows - r : most;
    const DropArgs a{D, ld_x, ld_add, ld_out, static_cast<uint64_t>(r) * pairs,
                     static_cast<uint32_t>(n * per_row), Divide(static_cast<uint32_t>(per_row))};
    const uint32_t blocks = static_cast<uint32_t>((n * per_row + kDropThreads - 1) / kDropThreads);
    kernel<<<blocks, kDropThreads, 0, st>>>(x + r * ld_x, add ? add + r * ld_add : nullptr,
                                            out + r * ld_out, a, k);
    if (const int rc = launch_status(hipGetLastError())) return rc;
  }
  return LM_OK;
}

int dropout_run(const void* x, int64_t ld_x, const void* add, int64_t ld_add, void* out,
                int64_t ld_out, int64_t rows, int64_t D, int dtype, float p, uint64_t seed,
                const int64_t* seed_at, hipStream_t st) {
  if (rows == 0 || D == 0) return LM_OK;
  const KeepArgs k = make_keep(p, seed, seed_at);
  if (dtype == LM_BF16)
    return dropout_launch(static_cast<const bf16_t*>(x), ld_x, static_cast<const bf16_t*>(add),
                          ld_add, static_cast<bf16_t*>(out), ld_out, rows, D, k, st);
  return dropout_launch(static_cast<const float*>(x), ld_x, static_cast<const float*>(add), ld_add,
                        static_cast<float*>(out), ld_out, rows, D, k, st);
}

}  // namespace lmz
