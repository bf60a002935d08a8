// Whether the rows of two B x H x Lq x Lk operands meet in memory (host code).
#pragma once

#include <stdint.h>

#include <algorithm>

namespace lmz {

// A stride that is taken lo to hi times.
struct Steps {
  __int128 lo, hi, stride;
};

// Whether some sum of `k` steps is in [from, to]. Strides are above zero and descend, each of
// about the others' reach behind it, so that few counts of the first can be part of it.
static inline bool steps_reach(const Steps* s, int k, __int128 from, __int128 to) {
  if (k == 0) return from <= 0 && 0 <= to;
  __int128 low = 0, high = 0;  // what the others add
  for (int i = 1; i < k; ++i) low += s[i].lo * s[i].stride, high += s[i].hi * s[i].stride;
  auto floor_div = [](__int128 a, __int128 b) { return a >= 0 ? a / b : -((-a + b - 1) / b); };
  const __int128 first = std::max(s->lo, -floor_div(high - from, s->stride));
  const __int128 last = std::min(s->hi, floor_div(to - low, s->stride));
  for (__int128 n = first; n <= last; ++n)
    if (steps_reach(s + 1, k - 1, from - n * s->stride, to - n * s->stride)) return true;
  return false;
}

enum class Meet { NO, YES, MANY };  // MANY: too many rows to tell

constexpr int64_t kMeetRows = int64_t(1) << 22;

// n: B, H, Lq; strides in elements, none negative. The rows of `out` do not meet each other;
// those of `add` start `at` elements from out's. Equal strides: the operands meet where a
// difference of two places is within a row of `at`, of which few can be. Others, where their
// spans meet: each row of add is looked for in out.
static inline Meet rows_meet(const int64_t* n, int64_t Lk, const int64_t* out, const int64_t* add,
                             __int128 at) {
  const __int128 row = Lk - 1;
  Steps s[3];
  int k = 0;
  bool equal = true;
  __int128 out_span = row, add_span = row;
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    equal = equal && out[i] == add[i];
    out_span += static_cast<__int128>(n[i] - 1) * out[i];
    add_span += static_cast<__int128>(n[i] - 1) * add[i];
    s[k++] = {0, n[i] - 1, out[i]};
  }
  if (at > out_span || at + add_span < 0) return Meet::NO;
  std::sort(s, s + k, [](const Steps& x, const Steps& y) { return x.stride > y.stride; });
  if (equal) {
    for (int i = 0; i < k; ++i) s[i].lo = -s[i].hi;
    return steps_reach(s, k, at - row, at + row) ? Meet::YES : Meet::NO;
  }
  int64_t m[3];  // rows of add that differ
  for (int i = 0; i < 3; ++i) m[i] = add[i] == 0 ? 1 : n[i];
  if (static_cast<__int128>(m[0]) * m[1] * m[2] > kMeetRows) return Meet::MANY;
  for (int64_t b = 0; b < m[0]; ++b)
    for (int64_t h = 0; h < m[1]; ++h)
      for (int64_t i = 0; i < m[2]; ++i) {
        const __int128 x = at + static_cast<__int128>(b) * add[0] +
                           static_cast<__int128>(h) * add[1] + static_cast<__int128>(i) * add[2];
        if (steps_reach(s, k, x - row, x + row)) return Meet::YES;
      }
  return Meet::NO;
}

}  // namespace lmz
