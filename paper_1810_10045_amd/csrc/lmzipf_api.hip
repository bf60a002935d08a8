// The C ABI declared in include/lmzipf.h: argument validation (before any
// launch), dtype dispatch and stream plumbing. The kernels live in
// unique.hip, segsum.hip, fill.hip, adamw.hip, relbias.hip, dropout.hip, norm.hip,
// norm_grad.hip and logprobs.hip.
#include <algorithm>
#include <new>

#include "common.hpp"
#include "rows_meet.hpp"

namespace lmz {

size_t unique_workspace_bytes(int64_t K, int idtype, int64_t V);
int unique_run(const void* ids, int idtype, int64_t K, int64_t V, void* uniq, int32_t* counts,
               int32_t* offsets, int32_t* inverse, int32_t* perm, int64_t* num_unique,
               int32_t* dev_err, void* ws, size_t ws_bytes, hipStream_t st);
size_t segsum_workspace_bytes(int64_t K, int64_t D);
int segsum_run(const void* grad, int gtype, int64_t K, int64_t D, int64_t ld_grad,
               const int32_t* perm, const int32_t* inverse, const int32_t* offsets,
               const int64_t* num_unique, int64_t u_cap, float* out, int64_t ld_out,
               int32_t* dev_err, void* ws, size_t ws_bytes, hipStream_t st,
               const void* row_ids = nullptr, int row_ids64 = 0, int64_t out_rows = 0,
               int op = 0, const OptParams& opt = OptParams{}, float* m = nullptr,
               float* v = nullptr);
int map_run(const void* sub, const int64_t* n_sub, int64_t sub_cap, const void* sup,
            const int64_t* n_sup, int64_t sup_cap, int idtype, int32_t* map, int32_t* dev_err,
            hipStream_t st);
int fill_run(const float* src, int64_t ld_src, const void* src_ids, const int64_t* n_src,
             int64_t src_cap, const void* dst_ids, const int64_t* n_dst, int idtype, int64_t D,
             float* dst, int64_t dst_rows, int64_t ld_dst, int mode, int32_t* dev_err,
             hipStream_t st);
int apply_run(float* table, int64_t V, int64_t D, int64_t ld_table, const void* rows, int idtype,
              const int64_t* n_rows, int64_t rows_cap, const float* vals, int64_t ld_vals,
              int opt, float lr, float beta1, float beta2, float eps, float weight_decay,
              int64_t step, float* m, float* v, int32_t* dev_err, hipStream_t st);

int fill_run_f16(const float* src, int64_t ld_src, const void* src_ids, const int64_t* n_src,
                 int64_t src_cap, const void* dst_ids, const int64_t* n_dst, int idtype,
                 int64_t D, uint16_t* dst, int64_t dst_rows, int64_t ld_dst, int mode,
                 float scale, int32_t* dev_err, hipStream_t st);
int apply_run_f16(float* table, int64_t V, int64_t D, int64_t ld_table, const void* rows,
                  int idtype, const int64_t* n_rows, int64_t rows_cap, const uint16_t* vals,
                  int64_t ld_vals, float inv_scale, int opt, float lr, float beta1, float beta2,
                  float eps, float weight_decay, int64_t step, float* m, float* v,
                  int32_t* dev_err, hipStream_t st);

size_t adamw_plan_bytes(int64_t chunks);
int64_t adamw_plan_chunks(const int64_t* sizes, int64_t tensors);
void adamw_plan_write(void* const* p, const void* const* g, void* const* m, void* const* v,
                      void* const* m_scale, void* const* v_scale, void* const* copies,
                      const int64_t* sizes, const int32_t* decay, int64_t tensors, int gtype,
                      int states, void* plan);
int adamw_run(const void* plan, int64_t chunks, int gtype, int states, bool copies, float lr,
              float beta1, float beta2, float eps, float weight_decay, int64_t step,
              const float* grad_scale, uint64_t seed, int32_t* dev_err, hipStream_t st);
int rows8_run(float* table, int64_t V, int64_t D, int64_t ld_table, const void* rows, int idtype,
              const int64_t* n_rows, int64_t rows_cap, const float* vals, int64_t ld_vals,
              float lr, float beta1, float beta2, float eps, float weight_decay, int64_t step,
              uint8_t* m, uint8_t* v, int64_t ld_codes, uint8_t* m_scale, uint8_t* v_scale,
              int64_t ld_scale, uint64_t seed, int32_t* dev_err, hipStream_t st);
int rel_buckets(int num_buckets, int max_distance, int mode, int32_t* starts, int32_t* ids);
int64_t rel_bias_blocks(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int dtype);
int rel_bias_run(const float* table, int64_t ld_table, const int32_t* starts, const int32_t* ids,
                 int n_seg, int64_t B, int64_t H, int64_t Lq, int64_t Lk, int64_t q_start,
                 const void* add, const int64_t* sa, void* out, const int64_t* so, int dtype,
                 hipStream_t st);
int64_t rel_grad_parts(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int dtype);
int rel_grad_run(const void* dout, int dtype, int64_t B, int64_t H, int64_t Lq, int64_t Lk,
                 const int64_t* sd, int64_t q_start, const int32_t* starts, const int32_t* ids,
                 int n_seg, int num_buckets, float* dtable, int64_t ld_table, int accumulate,
                 void* ws, hipStream_t st);

int dropout_run(const void* x, int64_t ld_x, const void* add, int64_t ld_add, void* out,
                int64_t ld_out, int64_t rows, int64_t D, int dtype, float p, uint64_t seed,
                const int64_t* seed_at, hipStream_t st);
int norm_run(const void* x, int64_t ld_x, const void* add, int64_t ld_add, int64_t rows, int64_t D,
             int dtype, const float* weight, const float* bias, float eps, float p, uint64_t seed,
             const int64_t* seed_at, void* y, int64_t ld_y, void* h, int64_t ld_h, float* mean,
             float* rstd, hipStream_t st);
size_t norm_grad_workspace_bytes(int64_t rows, int64_t D, int dtype);
int norm_grad_run(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, const void* add,
                  int64_t ld_add, int64_t rows, int64_t D, int dtype, const float* mean,
                  const float* rstd, const float* weight, float p, uint64_t seed,
                  const int64_t* seed_at, void* dh, int64_t ld_dh, void* dx, int64_t ld_dx,
                  float* dweight, float* dbias, int accumulate, void* ws, hipStream_t st);
size_t logp_workspace_bytes(int64_t N, int64_t V, int dtype, int k);
int logp_run(const void* logits, int64_t ld, int64_t N, int64_t V, int dtype, const void* targets,
             int idtype, int64_t ignore, float scale, int k, float* logp, float* entropy,
             float* peak, float* log_sum, float* top_logp, int32_t* top_ids, int32_t* dev_err,
             void* ws, hipStream_t st);
int64_t logp_grad_blocks(int64_t N, int64_t V, int dtype);
int logp_grad_run(const void* logits, int64_t ld, int64_t N, int64_t V, int dtype,
                  const void* targets, int idtype, int64_t ignore, float scale, const float* peak,
                  const float* log_sum, const float* dlogp, const float* entropy,
                  const float* dentropy, void* out, int64_t ld_out, hipStream_t st);

int sample_run(const uint64_t* r, int64_t n, int64_t V, void* ids, int idtype, hipStream_t st);
void segsum_force_wait_failure(bool enable, uint32_t limit);
int segsum_set_two_launches(bool enable);
void unique_force_wait_failure(bool enable, uint32_t limit);

int launch_status(hipError_t e) { return e == hipSuccess ? LM_OK : LM_E_HIP; }

static bool finite_nonzero(float x) { return x == x && x != 0.f && x - x == 0.f; }

__global__ __launch_bounds__(256) void k_clear(uint32_t* p, int64_t words, uint8_t* tail,
                                               int tail_bytes) {
  for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < words;
       i += int64_t(gridDim.x) * 256)
    p[i] = 0u;
  if (blockIdx.x == 0 && static_cast<int>(threadIdx.x) < tail_bytes) tail[threadIdx.x] = 0;
}

static bool valid_idtype(int32_t t) { return t == LM_I32 || t == LM_I64; }

static bool valid_dtype(int32_t t) { return t == LM_F32 || t == LM_BF16; }

static bool valid_betas(float beta1, float beta2) {
  return beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f;
}

// A piece of memory that a step writes, or reads only.
struct Piece {
  uintptr_t begin, end;
  bool written;
};

// Whether a written piece meets another one (`n` pieces, put in order here).
static bool pieces_meet(Piece* a, int64_t n) {
  std::sort(a, a + n, [](const Piece& x, const Piece& y) { return x.begin < y.begin; });
  uintptr_t any = 0, written = 0;  // the furthest ends so far
  for (int64_t i = 0; i < n; ++i) {
    if (a[i].begin < written || (a[i].written && a[i].begin < any)) return true;
    any = std::max(any, a[i].end);
    if (a[i].written) written = std::max(written, a[i].end);
  }
  return false;
}

// The segments of a relative bias: ascending from INT32_MIN, ids below num_buckets.
static int check_segments(const int32_t* starts, const int32_t* ids, int32_t n,
                          int32_t num_buckets) {
  if (n < 1 || num_buckets < 1 || !starts || !ids) return LM_E_INVAL;
  if (n > LM_REL_MAX_SEGMENTS || num_buckets > LM_REL_MAX_BUCKETS) return LM_E_UNSUPPORTED;
  if (starts[0] != INT32_MIN) return LM_E_INVAL;
  for (int32_t i = 0; i < n; ++i)
    if (ids[i] < -1 || ids[i] >= num_buckets || (i && starts[i] <= starts[i - 1]))
      return LM_E_INVAL;
  return LM_OK;
}

static int check_rel_sizes(int64_t B, int64_t H, int64_t Lq, int64_t Lk, int64_t q_start) {
  if (B < 0 || H < 0 || Lq < 0 || Lk < 0) return LM_E_INVAL;
  if (B > LM_REL_MAX_LENGTH || H > LM_REL_MAX_LENGTH || Lq > LM_REL_MAX_LENGTH ||
      Lk > LM_REL_MAX_LENGTH || q_start > LM_REL_MAX_START || q_start < -LM_REL_MAX_START)
    return LM_E_UNSUPPORTED;
  if (B == 0 || H == 0 || Lq == 0 || Lk == 0) return LM_OK;
  constexpr int64_t most = int64_t(1) << 40;  // elements
  if (B > most / H || B * H > most / Lq || B * H * Lq > most / Lk) return LM_E_UNSUPPORTED;
  return LM_OK;
}

// Strides of a B x H x Lq x Lk operand: rows that do not meet (read only: any), within
// 2^60 elements.
static bool check_strides(const int64_t* s, int64_t B, int64_t H, int64_t Lq, int64_t Lk,
                          bool written) {
  if (!s) return false;
  if (s[0] < 0 || s[1] < 0 || s[2] < 0) return false;
  constexpr int64_t most = int64_t(1) << 40;
  if (s[0] > most || s[1] > most || s[2] > most) return false;
  // In the order of their strides, each dimension steps over all of the ones inside it.
  struct Dim {
    int64_t n, stride;
  } d[3] = {{B, s[0]}, {H, s[1]}, {Lq, s[2]}};
  std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  __int128 inside = Lk;  // elements that the inner dimensions span: three products below 2^64
  for (const Dim& x : d) {
    if (x.n <= 1) continue;
    if (written && x.stride < inside) return false;
    inside += static_cast<__int128>(x.n - 1) * x.stride;
  }
  return inside <= static_cast<__int128>(1) << 60;  // so the kernels' offsets fit in 63 bits
}

// The operands of a call on rows: which of them may meet in memory.
class Operands {
 public:
  // A rows x D matrix of elements of `size` bytes.
  void matrix(const void* at, int64_t rows, int64_t D, int64_t ld, int size, bool written) {
    if (!at || rows == 0 || D == 0) return;
    const uintptr_t a = reinterpret_cast<uintptr_t>(at);
    bad_ |= (a & (size - 1)) != 0 || ld < D || ld > (int64_t(1) << 40);
    all_[n_++] = {a, rows, D * size, rows > 1 ? ld * size : 0, written, true};
  }
  // n elements of `size` bytes.
  void vector(const void* at, int64_t n, int size, bool written) {
    if (!at || n == 0) return;
    const uintptr_t a = reinterpret_cast<uintptr_t>(at);
    bad_ |= (a & (size - 1)) != 0;
    all_[n_++] = {a, 1, n * size, 0, written, false};
  }
  // LM_E_INVAL where an operand that is written meets another one, but for a matrix that takes
  // the place of one that is read, row for row.
  int check() const {
    if (bad_) return LM_E_INVAL;
    for (int i = 0; i < n_; ++i)
      for (int k = 0; k < n_; ++k) {
        const Operand &w = all_[i], &o = all_[k];
        if (i == k || !w.written || (o.written && k < i)) continue;
        if (!o.written && w.matrix && o.matrix && w.at == o.at && w.ld == o.ld) continue;
        if (const int rc = meet(w, o)) return rc;
      }
    return LM_OK;
  }

 private:
  struct Operand {
    uintptr_t at;
    int64_t rows, row, ld;  // row, ld: bytes
    bool written, matrix;
  };
  static int meet(const Operand& w, const Operand& o) {
    auto end = [](const Operand& x) {
      return static_cast<__int128>(x.at) + static_cast<__int128>(x.rows - 1) * x.ld + x.row;
    };
    if (o.at >= end(w) || w.at >= end(o)) return LM_OK;
    // Spans that meet: matrices of the same rows may lie beside each other in wider ones.
    if (!w.matrix || !o.matrix) return LM_E_INVAL;
    const int64_t n[3] = {1, 1, w.rows}, sw[3] = {0, 0, w.ld}, so[3] = {0, 0, o.ld};
    const Meet m = rows_meet(n, w.row, sw, so,
                             static_cast<__int128>(o.at) - static_cast<__int128>(w.at));
    return m == Meet::NO ? LM_OK : m == Meet::YES ? LM_E_INVAL : LM_E_UNSUPPORTED;
  }
  Operand all_[12];
  int n_ = 0;
  bool bad_ = false;
};

static int element_size(int32_t dtype) { return dtype == LM_BF16 ? 2 : 4; }

static bool in_unit(float p) { return p >= 0.f && p <= 1.f; }

static bool finite_positive(float x) { return x > 0.f && x < 1e38f; }

}  // namespace lmz

using namespace lmz;

extern "C" {

const char* lm_status_string(int status) {
  switch (status) {
    case LM_OK: return "LM_OK";
    case LM_E_INVAL: return "LM_E_INVAL: invalid argument";
    case LM_E_WORKSPACE: return "LM_E_WORKSPACE: workspace too small";
    case LM_E_HIP: return "LM_E_HIP: HIP launch or runtime error";
    case LM_E_UNSUPPORTED: return "LM_E_UNSUPPORTED: unsupported dtype, mode or size";
    default: return "unknown lmzipf status";
  }
}

int lm_abi_version(void) { return 106; }

int lm_workspace_clear(void* ws, size_t bytes, void* stream) {
  if (bytes == 0) return LM_OK;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 3)) return LM_E_INVAL;
  const int64_t words = static_cast<int64_t>(bytes / 4);
  const int tail = static_cast<int>(bytes % 4);
  int64_t blocks = (words + 256 * 16 - 1) / (256 * 16);
  if (blocks < 1) blocks = 1;
  if (blocks > 4096) blocks = 4096;
  k_clear<<<static_cast<uint32_t>(blocks), 256, 0, static_cast<hipStream_t>(stream)>>>(
      static_cast<uint32_t*>(ws), words, static_cast<uint8_t*>(ws) + words * 4, tail);
  return launch_status(hipGetLastError());
}

size_t lm_unique_workspace_bytes(int64_t K, int32_t idtype, int64_t V) {
  if (K < 0 || K >= LM_MAX_K || V < 1 || !valid_idtype(idtype)) return 0;
  return unique_workspace_bytes(K, idtype, V);
}

int lm_unique(const void* ids, int32_t idtype, int64_t K, int64_t V, void* uniq, int32_t* counts,
              int32_t* offsets, int32_t* inverse, int32_t* perm, int64_t* num_unique,
              int32_t* dev_err, void* ws, size_t ws_bytes, void* stream) {
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (K < 0 || V < 1) return LM_E_INVAL;
  if (K >= LM_MAX_K) return LM_E_UNSUPPORTED;
  if (!offsets || !num_unique || !ws) return LM_E_INVAL;
  if (K > 0 && (!ids || !uniq || !counts || !inverse || !perm || !dev_err)) return LM_E_INVAL;
  if (reinterpret_cast<uintptr_t>(ws) & 255) return LM_E_INVAL;
  if (ws_bytes < unique_workspace_bytes(K, idtype, V)) return LM_E_WORKSPACE;
  return unique_run(ids, idtype, K, V, uniq, counts, offsets, inverse, perm, num_unique, dev_err,
                    ws, ws_bytes, static_cast<hipStream_t>(stream));
}

int lm_segsum_set_two_launches(int32_t enable) { return segsum_set_two_launches(enable != 0); }

int lm_test_force_wait_failure(int32_t enable, uint32_t spin_limit) {
  segsum_force_wait_failure(enable != 0, spin_limit);
  unique_force_wait_failure(enable != 0, spin_limit);
  return LM_OK;
}

size_t lm_segsum_workspace_bytes(int64_t K, int64_t D) {
  if (K < 0 || K >= LM_MAX_K || D < 0) return 0;
  return segsum_workspace_bytes(K, D);
}

int lm_segsum(const void* grad, int32_t gtype, int64_t K, int64_t D, int64_t ld_grad,
              const int32_t* perm, const int32_t* inverse, const int32_t* offsets,
              const int64_t* num_unique, int64_t u_cap, float* out, int64_t ld_out,
              int32_t* dev_err, void* ws, size_t ws_bytes, void* stream) {
  if (gtype != LM_F32 && gtype != LM_BF16) return LM_E_UNSUPPORTED;
  if (K < 0 || D < 0 || u_cap < 0 || ld_grad < D || ld_out < D) return LM_E_INVAL;
  if (K >= LM_MAX_K || D > (int64_t(1) << 24)) return LM_E_UNSUPPORTED;
  if (K > 0 && D > 0 && u_cap > 0 &&
      (!grad || !perm || !inverse || !offsets || !num_unique || !out || !dev_err || !ws))
    return LM_E_INVAL;
  if (ws && (reinterpret_cast<uintptr_t>(ws) & 255)) return LM_E_INVAL;
  if (ws_bytes < segsum_workspace_bytes(K, D)) return LM_E_WORKSPACE;
  return segsum_run(grad, gtype, K, D, ld_grad, perm, inverse, offsets, num_unique, u_cap, out,
                    ld_out, dev_err, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

int lm_segsum_rows(const void* grad, int32_t gtype, int64_t K, int64_t D, int64_t ld_grad,
                   const int32_t* perm, const int32_t* inverse, const int32_t* offsets,
                   const int64_t* num_unique, const void* row_ids, int32_t idtype,
                   int64_t rows_cap, float* out, int64_t out_rows, int64_t ld_out,
                   int32_t* dev_err, void* ws, size_t ws_bytes, void* stream) {
  if (gtype != LM_F32 && gtype != LM_BF16) return LM_E_UNSUPPORTED;
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (K < 0 || D < 0 || rows_cap < 0 || out_rows < 0 || ld_grad < D || ld_out < D)
    return LM_E_INVAL;
  if (K >= LM_MAX_K || D > (int64_t(1) << 24) || out_rows > INT32_MAX) return LM_E_UNSUPPORTED;
  if (K > 0 && D > 0 && rows_cap > 0 &&
      (!grad || !perm || !inverse || !offsets || !num_unique || !row_ids || !out || !dev_err ||
       !ws))
    return LM_E_INVAL;
  if (ws && (reinterpret_cast<uintptr_t>(ws) & 255)) return LM_E_INVAL;
  if (ws_bytes < segsum_workspace_bytes(K, D)) return LM_E_WORKSPACE;
  return segsum_run(grad, gtype, K, D, ld_grad, perm, inverse, offsets, num_unique, rows_cap,
                    out, ld_out, dev_err, ws, ws_bytes, static_cast<hipStream_t>(stream),
                    row_ids, idtype == LM_I64 ? 1 : 0, out_rows);
}

int lm_segsum_sgd(const void* grad, int32_t gtype, int64_t K, int64_t D, int64_t ld_grad,
                  const int32_t* perm, const int32_t* inverse, const int32_t* offsets,
                  const int64_t* num_unique, const void* row_ids, int32_t idtype,
                  int64_t rows_cap, float* table, int64_t V, int64_t ld_table, float lr,
                  int32_t* dev_err, void* ws, size_t ws_bytes, void* stream) {
  if (gtype != LM_F32 && gtype != LM_BF16) return LM_E_UNSUPPORTED;
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (K < 0 || D < 0 || rows_cap < 0 || V < 0 || ld_grad < D || ld_table < D) return LM_E_INVAL;
  if (K >= LM_MAX_K || D > (int64_t(1) << 24) || V > INT32_MAX) return LM_E_UNSUPPORTED;
  if (K > 0 && D > 0 && rows_cap > 0 &&
      (!grad || !perm || !inverse || !offsets || !num_unique || !row_ids || !table || !dev_err ||
       !ws))
    return LM_E_INVAL;
  if (ws && (reinterpret_cast<uintptr_t>(ws) & 255)) return LM_E_INVAL;
  if (ws_bytes < segsum_workspace_bytes(K, D)) return LM_E_WORKSPACE;
  return segsum_run(grad, gtype, K, D, ld_grad, perm, inverse, offsets, num_unique, rows_cap,
                    table, ld_table, dev_err, ws, ws_bytes, static_cast<hipStream_t>(stream),
                    row_ids, idtype == LM_I64 ? 1 : 0, V, 1,
                    make_opt_params(false, lr, 0.f, 0.f, 0.f, 0.f, 1, 1.f));
}

int lm_segsum_adam(const void* grad, int32_t gtype, int64_t K, int64_t D, int64_t ld_grad,
                   const int32_t* perm, const int32_t* inverse, const int32_t* offsets,
                   const int64_t* num_unique, const void* row_ids, int32_t idtype,
                   int64_t rows_cap, float* table, int64_t V, int64_t ld_table, float lr,
                   float beta1, float beta2, float eps, float weight_decay, int64_t step,
                   float* m, float* v, int32_t* dev_err, void* ws, size_t ws_bytes,
                   void* stream) {
  if (gtype != LM_F32 && gtype != LM_BF16) return LM_E_UNSUPPORTED;
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (K < 0 || D < 0 || rows_cap < 0 || V < 0 || ld_grad < D || ld_table < D) return LM_E_INVAL;
  if (K >= LM_MAX_K || D > (int64_t(1) << 24) || V > INT32_MAX) return LM_E_UNSUPPORTED;
  if (step < 1 || !(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f)) return LM_E_INVAL;
  if (K > 0 && D > 0 && rows_cap > 0 &&
      (!grad || !perm || !inverse || !offsets || !num_unique || !row_ids || !table || !m || !v ||
       !dev_err || !ws))
    return LM_E_INVAL;
  if (ws && (reinterpret_cast<uintptr_t>(ws) & 255)) return LM_E_INVAL;
  if (ws_bytes < segsum_workspace_bytes(K, D)) return LM_E_WORKSPACE;
  return segsum_run(grad, gtype, K, D, ld_grad, perm, inverse, offsets, num_unique, rows_cap,
                    table, ld_table, dev_err, ws, ws_bytes, static_cast<hipStream_t>(stream),
                    row_ids, idtype == LM_I64 ? 1 : 0, V, 2,
                    make_opt_params(true, lr, beta1, beta2, eps, weight_decay, step, 1.f), m, v);
}

int lm_map_ids(const void* sub_ids, const int64_t* n_sub, int64_t sub_cap, const void* sup_ids,
               const int64_t* n_sup, int64_t sup_cap, int32_t idtype, int32_t* map,
               int32_t* dev_err, void* stream) {
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (sub_cap < 0 || sup_cap < 0) return LM_E_INVAL;
  if (sub_cap > 0 && (!sub_ids || !n_sub || !sup_ids || !n_sup || !map || !dev_err))
    return LM_E_INVAL;
  if (sub_cap >= (int64_t(1) << 31) * kWave) return LM_E_UNSUPPORTED;
  return map_run(sub_ids, n_sub, sub_cap, sup_ids, n_sup, sup_cap, idtype, map, dev_err,
                 static_cast<hipStream_t>(stream));
}

int lm_fill_values(const float* src, int64_t ld_src, const void* src_ids, const int64_t* n_src,
                   int64_t src_cap, const void* dst_ids, const int64_t* n_dst, int32_t idtype,
                   int64_t D, float* dst, int64_t dst_rows, int64_t ld_dst, int32_t mode,
                   int32_t* dev_err, void* stream) {
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (mode != LM_FILL_EXPAND && mode != LM_FILL_SCATTER && mode != LM_FILL_SCATTER_ADD)
    return LM_E_UNSUPPORTED;
  if (D < 0 || src_cap < 0 || dst_rows < 0 || ld_src < D || ld_dst < D) return LM_E_INVAL;
  if (D > (int64_t(1) << 24)) return LM_E_UNSUPPORTED;
  if (mode == LM_FILL_EXPAND && (!dst_ids || !n_dst)) return LM_E_INVAL;
  if (dst_ids && !n_dst) return LM_E_INVAL;
  if ((src_cap > 0 || dst_rows > 0) && D > 0 && (!src_ids || !n_src || !dev_err)) return LM_E_INVAL;
  if (src_cap > 0 && D > 0 && !src) return LM_E_INVAL;
  if (dst_rows > 0 && D > 0 && !dst) return LM_E_INVAL;
  return fill_run(src, ld_src, src_ids, n_src, src_cap, dst_ids, n_dst, idtype, D, dst, dst_rows,
                  ld_dst, mode, dev_err, static_cast<hipStream_t>(stream));
}

int lm_sparse_apply(float* table, int64_t V, int64_t D, int64_t ld_table, const void* rows,
                    int32_t idtype, const int64_t* n_rows, int64_t rows_cap, const float* vals,
                    int64_t ld_vals, int32_t opt, float lr, float beta1, float beta2, float eps,
                    float weight_decay, int64_t step, float* m, float* v, int32_t* dev_err,
                    void* stream) {
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (opt != LM_OPT_SGD && opt != LM_OPT_ADAM) return LM_E_UNSUPPORTED;
  if (V < 0 || D < 0 || rows_cap < 0 || ld_table < D || ld_vals < D) return LM_E_INVAL;
  if (D > (int64_t(1) << 24)) return LM_E_UNSUPPORTED;
  if (rows_cap > 0 && D > 0 && (!table || !rows || !n_rows || !vals || !dev_err))
    return LM_E_INVAL;
  if (opt == LM_OPT_ADAM) {
    if (step < 1) return LM_E_INVAL;
    if (rows_cap > 0 && D > 0 && (!m || !v)) return LM_E_INVAL;
    if (!(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f)) return LM_E_INVAL;
  }
  return apply_run(table, V, D, ld_table, rows, idtype, n_rows, rows_cap, vals, ld_vals, opt, lr,
                   beta1, beta2, eps, weight_decay, step, m, v, dev_err,
                   static_cast<hipStream_t>(stream));
}

int lm_fill_values_f16(const float* src, int64_t ld_src, const void* src_ids,
                       const int64_t* n_src, int64_t src_cap, const void* dst_ids,
                       const int64_t* n_dst, int32_t idtype, int64_t D, uint16_t* dst,
                       int64_t dst_rows, int64_t ld_dst, int32_t mode, float scale,
                       int32_t* dev_err, void* stream) {
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (mode != LM_FILL_EXPAND && mode != LM_FILL_SCATTER) return LM_E_UNSUPPORTED;
  if (!finite_nonzero(scale)) return LM_E_INVAL;
  if (D < 0 || src_cap < 0 || dst_rows < 0 || ld_src < D || ld_dst < D) return LM_E_INVAL;
  if (D > (int64_t(1) << 24)) return LM_E_UNSUPPORTED;
  if (mode == LM_FILL_EXPAND && (!dst_ids || !n_dst)) return LM_E_INVAL;
  if (dst_ids && !n_dst) return LM_E_INVAL;
  if ((src_cap > 0 || dst_rows > 0) && D > 0 && (!src_ids || !n_src || !dev_err)) return LM_E_INVAL;
  if (src_cap > 0 && D > 0 && !src) return LM_E_INVAL;
  if (dst_rows > 0 && D > 0 && !dst) return LM_E_INVAL;
  return fill_run_f16(src, ld_src, src_ids, n_src, src_cap, dst_ids, n_dst, idtype, D, dst,
                      dst_rows, ld_dst, mode, scale, dev_err, static_cast<hipStream_t>(stream));
}

int lm_sparse_apply_f16(float* table, int64_t V, int64_t D, int64_t ld_table, const void* rows,
                        int32_t idtype, const int64_t* n_rows, int64_t rows_cap,
                        const uint16_t* vals, int64_t ld_vals, float inv_scale, int32_t opt,
                        float lr, float beta1, float beta2, float eps, float weight_decay,
                        int64_t step, float* m, float* v, int32_t* dev_err, void* stream) {
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (opt != LM_OPT_SGD && opt != LM_OPT_ADAM) return LM_E_UNSUPPORTED;
  if (!finite_nonzero(inv_scale)) return LM_E_INVAL;
  if (V < 0 || D < 0 || rows_cap < 0 || ld_table < D || ld_vals < D) return LM_E_INVAL;
  if (D > (int64_t(1) << 24)) return LM_E_UNSUPPORTED;
  if (rows_cap > 0 && D > 0 && (!table || !rows || !n_rows || !vals || !dev_err))
    return LM_E_INVAL;
  if (opt == LM_OPT_ADAM) {
    if (step < 1) return LM_E_INVAL;
    if (rows_cap > 0 && D > 0 && (!m || !v)) return LM_E_INVAL;
    if (!(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f)) return LM_E_INVAL;
  }
  return apply_run_f16(table, V, D, ld_table, rows, idtype, n_rows, rows_cap, vals, ld_vals,
                       inv_scale, opt, lr, beta1, beta2, eps, weight_decay, step, m, v, dev_err,
                       static_cast<hipStream_t>(stream));
}

size_t lm_adamw_plan_bytes(const int64_t* sizes, int64_t tensors) {
  if (tensors < 0 || (tensors > 0 && !sizes) || tensors > INT32_MAX) return 0;
  int64_t total = 0;
  for (int64_t i = 0; i < tensors; ++i) {
    if (sizes[i] < 0 || sizes[i] > LM_ADAMW_MAX_VALUES - total) return 0;
    total += sizes[i];
  }
  const int64_t chunks = adamw_plan_chunks(sizes, tensors);
  return chunks > INT32_MAX ? 0 : adamw_plan_bytes(chunks);
}

int lm_adamw_plan(void* const* p, const void* const* g, void* const* m, void* const* v,
                  void* const* m_scale, void* const* v_scale, void* const* copies,
                  const int64_t* sizes, const int32_t* decay, int64_t tensors, int32_t gtype,
                  int32_t states, void* plan, size_t plan_bytes, int64_t* chunks) {
  if (!valid_dtype(gtype) || (states != 32 && states != 8)) return LM_E_UNSUPPORTED;
  if (tensors < 0 || !plan || !chunks) return LM_E_INVAL;
  if (tensors > 0 && (!p || !g || !m || !v || !sizes)) return LM_E_INVAL;
  if (tensors > 0 && (states == 8) != (m_scale != nullptr)) return LM_E_INVAL;
  if (tensors > 0 && (states == 8) != (v_scale != nullptr)) return LM_E_INVAL;
  const size_t need = lm_adamw_plan_bytes(sizes, tensors);
  if (need == 0) return LM_E_UNSUPPORTED;
  if (plan_bytes < need) return LM_E_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(plan) & 7) return LM_E_INVAL;
  Piece* pieces = new (std::nothrow) Piece[static_cast<size_t>(tensors) * 7 + 1];
  if (!pieces) return LM_E_UNSUPPORTED;
  int64_t n = 0;
  bool bad = false;
  auto piece = [&](const void* at, int64_t bytes, int align, bool written) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(at);
    bad |= !at || (a & (align - 1));
    pieces[n++] = {a, a + static_cast<uintptr_t>(bytes), written};
  };
  for (int64_t i = 0; i < tensors; ++i) {
    const int64_t k = sizes[i], blocks = (k + LM_MOMENT_BLOCK - 1) / LM_MOMENT_BLOCK;
    if (k == 0) continue;
    const int state = states == 8 ? 1 : 4;
    piece(p[i], 4 * k, 4, true);
    piece(g[i], (gtype == LM_BF16 ? 2 : 4) * k, gtype == LM_BF16 ? 2 : 4, false);
    piece(m[i], state * k, state, true);
    piece(v[i], state * k, state, true);
    if (states == 8) {
      piece(m_scale[i], blocks, 1, true);
      piece(v_scale[i], blocks, 1, true);
    }
    if (copies) piece(copies[i], 2 * k, 2, true);
  }
  bad = bad || pieces_meet(pieces, n);
  delete[] pieces;
  if (bad) return LM_E_INVAL;
  adamw_plan_write(p, g, m, v, m_scale, v_scale, copies, sizes, decay, tensors, gtype, states,
                   plan);
  *chunks = adamw_plan_chunks(sizes, tensors);
  return LM_OK;
}

int lm_adamw(const void* plan, size_t plan_bytes, int64_t chunks, int32_t gtype, int32_t states,
             int32_t copies, float lr, float beta1, float beta2, float eps, float weight_decay,
             int64_t step, const float* grad_scale, uint64_t seed, int32_t* dev_err,
             void* stream) {
  if (!valid_dtype(gtype) || (states != 32 && states != 8)) return LM_E_UNSUPPORTED;
  if (chunks < 0 || chunks > INT32_MAX) return LM_E_INVAL;
  if (step < 1 || !valid_betas(beta1, beta2)) return LM_E_INVAL;
  if (chunks > 0 && (!plan || (reinterpret_cast<uintptr_t>(plan) & 7))) return LM_E_INVAL;
  if (plan_bytes < adamw_plan_bytes(chunks)) return LM_E_WORKSPACE;
  return adamw_run(plan, chunks, gtype, states, copies != 0, lr, beta1, beta2, eps,
                   weight_decay, step, grad_scale, seed, dev_err,
                   static_cast<hipStream_t>(stream));
}

int lm_sparse_apply_q8(float* table, int64_t V, int64_t D, int64_t ld_table, const void* rows,
                       int32_t idtype, const int64_t* n_rows, int64_t rows_cap, const float* vals,
                       int64_t ld_vals, float lr, float beta1, float beta2, float eps,
                       float weight_decay, int64_t step, uint8_t* m, uint8_t* v,
                       int64_t ld_codes, uint8_t* m_scale, uint8_t* v_scale, int64_t ld_scale,
                       uint64_t seed, int32_t* dev_err, void* stream) {
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (V < 0 || D < 0 || rows_cap < 0 || ld_table < D || ld_vals < D || ld_codes < D ||
      ld_scale < (D + LM_MOMENT_BLOCK - 1) / LM_MOMENT_BLOCK)
    return LM_E_INVAL;
  if (D > (int64_t(1) << 24) || rows_cap > INT32_MAX) return LM_E_UNSUPPORTED;
  if (step < 1 || !valid_betas(beta1, beta2)) return LM_E_INVAL;
  if (rows_cap > 0 && D > 0 &&
      (!table || !rows || !n_rows || !vals || !m || !v || !m_scale || !v_scale))
    return LM_E_INVAL;
  return rows8_run(table, V, D, ld_table, rows, idtype, n_rows, rows_cap, vals, ld_vals, lr, beta1,
                   beta2, eps, weight_decay, step, m, v, ld_codes, m_scale, v_scale, ld_scale,
                   seed, dev_err, static_cast<hipStream_t>(stream));
}

int lm_rel_buckets(int32_t num_buckets, int32_t max_distance, int32_t mode, int32_t* starts,
                   int32_t* ids, int32_t* n_seg) {
  if (mode != LM_REL_BOTH && mode != LM_REL_PAST && mode != LM_REL_CAUSAL) return LM_E_UNSUPPORTED;
  if (!starts || !ids || !n_seg) return LM_E_INVAL;
  if (num_buckets > LM_REL_MAX_BUCKETS || max_distance >= (1 << 24)) return LM_E_UNSUPPORTED;
  if (mode == LM_REL_BOTH && num_buckets % 2) return LM_E_INVAL;
  const int32_t side = mode == LM_REL_BOTH ? num_buckets / 2 : num_buckets;
  if (side < 2 || max_distance <= side / 2) return LM_E_INVAL;
  *n_seg = rel_buckets(num_buckets, max_distance, mode, starts, ids);
  return LM_OK;
}

int lm_rel_bias(const float* table, int64_t ld_table, int32_t num_buckets, const int32_t* starts,
                const int32_t* ids, int32_t n_seg, int64_t B, int64_t H, int64_t Lq, int64_t Lk,
                int64_t q_start, const void* add, const int64_t* add_strides, void* out,
                const int64_t* out_strides, int32_t dtype, void* stream) {
  if (!valid_dtype(dtype)) return LM_E_UNSUPPORTED;
  if (const int rc = check_segments(starts, ids, n_seg, num_buckets)) return rc;
  if (const int rc = check_rel_sizes(B, H, Lq, Lk, q_start)) return rc;
  if (ld_table < H) return LM_E_INVAL;
  if (B == 0 || H == 0 || Lq == 0 || Lk == 0) return LM_OK;
  if (!table || !out) return LM_E_INVAL;
  const uintptr_t mask = dtype == LM_BF16 ? 1 : 3;
  if ((reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(add)) & mask)
    return LM_E_INVAL;
  if (!check_strides(out_strides, B, H, Lq, Lk, true)) return LM_E_INVAL;
  if (add) {
    if (!check_strides(add_strides, B, H, Lq, Lk, false)) return LM_E_INVAL;
    // In place a workgroup reads before it writes, and no other uses its elements.
    const int64_t n[3] = {B, H, Lq};
    bool in_place = add == out;
    for (int i = 0; i < 3; ++i) in_place &= n[i] == 1 || add_strides[i] == out_strides[i];
    const __int128 at = (static_cast<__int128>(reinterpret_cast<uintptr_t>(add)) -
                         reinterpret_cast<uintptr_t>(out)) / (dtype == LM_BF16 ? 2 : 4);
    const Meet meet = in_place ? Meet::NO : rows_meet(n, Lk, out_strides, add_strides, at);
    if (meet != Meet::NO) return meet == Meet::YES ? LM_E_INVAL : LM_E_UNSUPPORTED;
  }
  if (rel_bias_blocks(B, H, Lq, Lk, dtype) > INT32_MAX) return LM_E_UNSUPPORTED;
  return rel_bias_run(table, ld_table, starts, ids, n_seg, B, H, Lq, Lk, q_start, add, add_strides,
                      out, out_strides, dtype, static_cast<hipStream_t>(stream));
}

size_t lm_rel_bias_grad_workspace_bytes(int64_t B, int64_t H, int64_t Lq, int64_t Lk,
                                        int32_t dtype, int32_t n_seg) {
  if (!valid_dtype(dtype) || check_rel_sizes(B, H, Lq, Lk, 0) != LM_OK || n_seg < 1 ||
      n_seg > LM_REL_MAX_SEGMENTS)
    return 0;
  return static_cast<size_t>(rel_grad_parts(B, H, Lq, Lk, dtype)) * H * n_seg * sizeof(float);
}

int lm_rel_bias_grad(const void* dout, int32_t dtype, int64_t B, int64_t H, int64_t Lq, int64_t Lk,
                     const int64_t* dout_strides, int64_t q_start, const int32_t* starts,
                     const int32_t* ids, int32_t n_seg, int32_t num_buckets, float* dtable,
                     int64_t ld_table, int32_t accumulate, void* ws, size_t ws_bytes,
                     void* stream) {
  if (!valid_dtype(dtype)) return LM_E_UNSUPPORTED;
  if (const int rc = check_segments(starts, ids, n_seg, num_buckets)) return rc;
  if (const int rc = check_rel_sizes(B, H, Lq, Lk, q_start)) return rc;
  if (ld_table < H) return LM_E_INVAL;
  if (H == 0) return LM_OK;
  if (!dtable) return LM_E_INVAL;
  if (B > 0 && Lq > 0 && Lk > 0) {
    if (!dout) return LM_E_INVAL;
    if (reinterpret_cast<uintptr_t>(dout) & (dtype == LM_BF16 ? 1 : 3)) return LM_E_INVAL;
    if (!check_strides(dout_strides, B, H, Lq, Lk, false)) return LM_E_INVAL;
    const int64_t parts = rel_grad_parts(B, H, Lq, Lk, dtype);
    if (parts > INT32_MAX / H) return LM_E_UNSUPPORTED;
    const size_t need = lm_rel_bias_grad_workspace_bytes(B, H, Lq, Lk, dtype, n_seg);
    if (need > 0 && (!ws || (reinterpret_cast<uintptr_t>(ws) & 3))) return LM_E_INVAL;
    if (ws_bytes < need) return LM_E_WORKSPACE;
  }
  return rel_grad_run(dout, dtype, B, H, Lq, Lk, dout_strides, q_start, starts, ids, n_seg,
                      num_buckets, dtable, ld_table, accumulate, ws,
                      static_cast<hipStream_t>(stream));
}

int lm_dropout(const void* x, int64_t ld_x, const void* add, int64_t ld_add, void* out,
               int64_t ld_out, int64_t rows, int64_t D, int32_t dtype, float p, uint64_t seed,
               const int64_t* seed_at, void* stream) {
  if (!valid_dtype(dtype)) return LM_E_UNSUPPORTED;
  if (rows < 0 || D < 0 || !in_unit(p)) return LM_E_INVAL;
  if (rows > INT32_MAX || D > INT32_MAX) return LM_E_UNSUPPORTED;
  if (rows == 0 || D == 0) return LM_OK;
  if (!x || !out || (reinterpret_cast<uintptr_t>(seed_at) & 7)) return LM_E_INVAL;
  Operands o;
  const int size = element_size(dtype);
  o.matrix(out, rows, D, ld_out, size, true);
  o.matrix(x, rows, D, ld_x, size, false);
  o.matrix(add, rows, D, ld_add, size, false);
  o.vector(seed_at, 1, 8, false);
  if (const int rc = o.check()) return rc;
  return dropout_run(x, ld_x, add, ld_add, out, ld_out, rows, D, dtype, p, seed, seed_at,
                     static_cast<hipStream_t>(stream));
}

int lm_layer_norm(const void* x, int64_t ld_x, const void* add, int64_t ld_add, int64_t rows,
                  int64_t D, int32_t dtype, const float* weight, const float* bias, float eps,
                  float p, uint64_t seed, const int64_t* seed_at, void* y, int64_t ld_y, void* h,
                  int64_t ld_h, float* mean, float* rstd, void* stream) {
  if (!valid_dtype(dtype)) return LM_E_UNSUPPORTED;
  if (rows < 0 || D < 1 || !in_unit(p) || !(eps >= 0.f && eps < 1e38f)) return LM_E_INVAL;
  if (rows > INT32_MAX || D > LM_NORM_MAX_WIDTH) return LM_E_UNSUPPORTED;
  if (rows == 0) return LM_OK;
  if (!x || !y || !mean || !rstd) return LM_E_INVAL;
  Operands o;
  const int size = element_size(dtype);
  o.matrix(y, rows, D, ld_y, size, true);
  o.matrix(h, rows, D, ld_h, size, true);
  o.vector(mean, rows, 4, true);
  o.vector(rstd, rows, 4, true);
  o.matrix(x, rows, D, ld_x, size, false);
  o.matrix(add, rows, D, ld_add, size, false);
  o.vector(weight, D, 4, false);
  o.vector(bias, D, 4, false);
  o.vector(seed_at, 1, 8, false);
  if (const int rc = o.check()) return rc;
  return norm_run(x, ld_x, add, ld_add, rows, D, dtype, weight, bias, eps, p, seed, seed_at, y,
                  ld_y, h, ld_h, mean, rstd, static_cast<hipStream_t>(stream));
}

size_t lm_layer_norm_grad_workspace_bytes(int64_t rows, int64_t D, int32_t dtype) {
  if (!valid_dtype(dtype) || rows < 0 || rows > INT32_MAX || D < 1 || D > LM_NORM_MAX_WIDTH)
    return 0;
  return norm_grad_workspace_bytes(rows, D, dtype);
}

int lm_layer_norm_grad(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, const void* add,
                       int64_t ld_add, int64_t rows, int64_t D, int32_t dtype, const float* mean,
                       const float* rstd, const float* weight, float p, uint64_t seed,
                       const int64_t* seed_at, void* dh, int64_t ld_dh, void* dx, int64_t ld_dx,
                       float* dweight, float* dbias, int32_t accumulate, void* ws, size_t ws_bytes,
                       void* stream) {
  if (!valid_dtype(dtype)) return LM_E_UNSUPPORTED;
  if (rows < 0 || D < 1 || !in_unit(p)) return LM_E_INVAL;
  if (rows > INT32_MAX || D > LM_NORM_MAX_WIDTH) return LM_E_UNSUPPORTED;
  if (rows > 0 && (!dy || !h || !mean || !rstd || !dh)) return LM_E_INVAL;
  const bool sums = dweight || dbias;
  const size_t need = sums ? norm_grad_workspace_bytes(rows, D, dtype) : 0;
  if (need > 0 && !ws) return LM_E_INVAL;
  if (ws_bytes < need) return LM_E_WORKSPACE;
  Operands o;
  const int size = element_size(dtype);
  o.matrix(dh, rows, D, ld_dh, size, true);
  o.matrix(dx, rows, D, ld_dx, size, true);
  o.vector(dweight, D, 4, true);
  o.vector(dbias, D, 4, true);
  o.vector(need ? ws : nullptr, static_cast<int64_t>(need / 4), 4, true);
  o.matrix(dy, rows, D, ld_dy, size, false);
  o.matrix(h, rows, D, ld_h, size, false);
  o.matrix(add, rows, D, ld_add, size, false);
  o.vector(mean, rows, 4, false);
  o.vector(rstd, rows, 4, false);
  o.vector(weight, D, 4, false);
  o.vector(seed_at, 1, 8, false);
  if (const int rc = o.check()) return rc;
  return norm_grad_run(dy, ld_dy, h, ld_h, add, ld_add, rows, D, dtype, mean, rstd, weight, p,
                       seed, seed_at, dh, ld_dh, dx, ld_dx, dweight, dbias, accumulate, ws,
                       static_cast<hipStream_t>(stream));
}

size_t lm_token_logprobs_workspace_bytes(int64_t N, int64_t V, int32_t dtype, int32_t top) {
  if (!valid_dtype(dtype) || N < 0 || N > INT32_MAX || V < 1 || V > LM_LOGP_MAX_V || top < 0 ||
      top > LM_TOP_MAX)
    return 0;
  return logp_workspace_bytes(N, V, dtype, top);
}

int lm_token_logprobs(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype,
                      const void* targets, int32_t idtype, int64_t ignore, float scale,
                      int32_t top, float* logp, float* entropy, float* peak, float* log_sum,
                      float* top_logp, int32_t* top_ids, int32_t* dev_err, void* ws,
                      size_t ws_bytes, void* stream) {
  if (!valid_dtype(dtype) || (targets && !valid_idtype(idtype))) return LM_E_UNSUPPORTED;
  if (N < 0 || V < 1 || top < 0 || !finite_positive(scale)) return LM_E_INVAL;
  if (N > INT32_MAX || V > LM_LOGP_MAX_V || top > LM_TOP_MAX) return LM_E_UNSUPPORTED;
  if (N == 0) return LM_OK;
  if (!logits || !entropy || !peak || !log_sum || (targets && !logp) ||
      (top > 0 && (!top_logp || !top_ids)))
    return LM_E_INVAL;
  const size_t need = logp_workspace_bytes(N, V, dtype, top);
  if (need > 0 && (!ws || (reinterpret_cast<uintptr_t>(ws) & 15))) return LM_E_INVAL;
  if (ws_bytes < need) return LM_E_WORKSPACE;
  Operands o;
  o.vector(targets ? logp : nullptr, N, 4, true);
  o.vector(entropy, N, 4, true);
  o.vector(peak, N, 4, true);
  o.vector(log_sum, N, 4, true);
  o.vector(top_logp, N * top, 4, true);
  o.vector(top_ids, N * top, 4, true);
  o.vector(dev_err, 1, 4, true);
  o.vector(need ? ws : nullptr, static_cast<int64_t>(need), 1, true);
  o.matrix(logits, N, V, ld, element_size(dtype), false);
  o.vector(targets, N, idtype == LM_I64 ? 8 : 4, false);
  if (const int rc = o.check()) return rc;
  return logp_run(logits, ld, N, V, dtype, targets, idtype, ignore, scale, top, logp, entropy,
                  peak, log_sum, top_logp, top_ids, dev_err, ws, static_cast<hipStream_t>(stream));
}

int lm_token_logprobs_grad(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype,
                           const void* targets, int32_t idtype, int64_t ignore, float scale,
                           const float* peak, const float* log_sum, const float* dlogp,
                           const float* entropy, const float* dentropy, void* out, int64_t ld_out,
                           void* stream) {
  if (!valid_dtype(dtype) || (targets && !valid_idtype(idtype))) return LM_E_UNSUPPORTED;
  if (N < 0 || V < 1 || !finite_positive(scale)) return LM_E_INVAL;
  if (N > INT32_MAX || V > LM_LOGP_MAX_V) return LM_E_UNSUPPORTED;
  if (N == 0) return LM_OK;
  if (!logits || !peak || !log_sum || !out || (dlogp && !targets) || (dentropy && !entropy))
    return LM_E_INVAL;
  if (logp_grad_blocks(N, V, dtype) > INT32_MAX) return LM_E_UNSUPPORTED;
  Operands o;
  const int size = element_size(dtype);
  o.matrix(out, N, V, ld_out, size, true);
  o.matrix(logits, N, V, ld, size, false);
  o.vector(dlogp ? targets : nullptr, N, idtype == LM_I64 ? 8 : 4, false);
  o.vector(peak, N, 4, false);
  o.vector(log_sum, N, 4, false);
  o.vector(dlogp, N, 4, false);
  o.vector(dentropy ? entropy : nullptr, N, 4, false);
  o.vector(dentropy, N, 4, false);
  if (const int rc = o.check()) return rc;
  return logp_grad_run(logits, ld, N, V, dtype, targets, idtype, ignore, scale, peak, log_sum,
                       dlogp, entropy, dentropy, out, ld_out, static_cast<hipStream_t>(stream));
}

int lm_sample_ids(const uint64_t* r, int64_t n, int64_t V, void* ids, int32_t idtype,
                  void* stream) {
  if (!valid_idtype(idtype)) return LM_E_UNSUPPORTED;
  if (n < 0 || V < 1) return LM_E_INVAL;
  if (idtype == LM_I32 && V > (int64_t(1) << 31)) return LM_E_INVAL;
  if (n > 0 && (!r || !ids)) return LM_E_INVAL;
  return sample_run(r, n, V, ids, idtype, static_cast<hipStream_t>(stream));
}

}  // extern "C"
