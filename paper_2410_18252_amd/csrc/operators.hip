// C entry points of the operators over a cache in pages and packed rows: what the host can check is checked here, then launched.
// A pass without rows has no tensors of rows, so their pointers may be null.
#include "../../include/rlgen.h"
#include "kernels.h"
#include "window.h"

#include <cmath>

#define HIPCHK(expr) do { if ((expr) != hipSuccess) return RLGEN_ERR_DEVICE; } while (0)

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
int page_shift(int page_size) {                        // -1: not a power of two from 8 to 1024
  for (int s = 3; s <= 10; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}
bool type16(int dtype) { return dtype == RLGEN_DTYPE_BF16 || dtype == RLGEN_DTYPE_F16; }
bool heads_ok(int rows, int Hq, int Hkv, int h) {
  return rows >= 0 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && h >= 16 && h <= 256 && h % 16 == 0 && (int64_t)rows * Hq <= INT32_MAX &&
         (int64_t)(Hq + 2ll * Hkv) * h <= INT32_MAX;
}
// rows of `heads` heads one behind the other, 16-byte loads
constexpr int64_t MAX_STRIDE = 1 << 23;      // (64 rows of a tile lie within 32-bit offsets)
bool rows_ok(const void* p, int64_t stride, int64_t heads, int h, int step = 8) {
  return aligned16(p) && stride >= heads * h && stride % step == 0 && stride <= MAX_STRIDE;
}
bool pages_ok(const void* pages, int n_pages, int shift, int Hkv, int h) {
  return aligned16(pages) && n_pages >= 1 && shift >= 0 && ((int64_t)n_pages << shift) <= INT32_MAX && ((int64_t)Hkv << shift) * h <= INT32_MAX;
}

int norm_rope_args(NormRopeArgs& a, const void* qkv, int64_t qkv_stride, int src_dtype, int rows, int Hq, int Hkv, int h, const float* q_gain,
                   const float* k_gain, float eps, const float* rope, int max_pos, int r, const int* positions, int dtype) {
  if (!q_gain || !k_gain || (rows > 0 && (!qkv || !positions)) || (r > 0 && !rope)) return RLGEN_ERR_NULL;
  if (!heads_ok(rows, Hq, Hkv, h) || !type16(dtype) || src_dtype < RLGEN_DTYPE_F32 || src_dtype > RLGEN_DTYPE_F16 || !std::isfinite(eps) || eps < 0.f ||
      r < 0 || r > h || r % 2 != 0 || max_pos < 1 || !rows_ok(qkv, qkv_stride, Hq + 2 * Hkv, h, src_dtype == RLGEN_DTYPE_F32 ? 4 : 8))
    return RLGEN_ERR_BAD_ARG;
  a.qkv = qkv; a.qkv_stride = qkv_stride; a.src_dtype = src_dtype; a.dtype = dtype;
  a.rows = rows; a.Hq = Hq; a.Hkv = Hkv; a.h = h;
  a.q_gain = q_gain; a.k_gain = k_gain; a.eps = eps;
  a.rope = (const float2*)rope; a.max_pos = max_pos; a.r = r; a.positions = positions;
  return RLGEN_OK;
}
bool window_ok(const WindowArgs& a) {
  return heads_ok(a.rows, a.Hq, a.Hkv, a.h) && type16(a.dtype) && a.S >= 1 && (int64_t)a.S * a.Hq <= INT32_MAX && a.max_new >= 1 &&
         a.window >= 0 && a.sinks >= 0 && std::isfinite(a.scale) && (int64_t)a.max_new * (a.Hq / a.Hkv) <= INT32_MAX - 256;
}
WindowArgs window_shape(int dtype, int rows, int Hq, int Hkv, int h, int S, int max_new, int window, int sinks, float scale) {
  WindowArgs a{};
  a.dtype = dtype; a.rows = rows; a.Hq = Hq; a.Hkv = Hkv; a.h = h; a.S = S; a.max_new = max_new;
  a.window = window; a.sinks = sinks; a.scale = scale;
  return a;
}

}  // namespace

extern "C" {

int rlgen_plan_pages(const int32_t* ctx_lens, const int32_t* new_lens, int32_t S, int32_t page_size, const int32_t* free_pages,
                     int32_t n_free, const int32_t* free_head, int32_t* page_table, int32_t table_stride, int32_t max_rows,
                     int32_t* total_lens, int32_t* row_starts, int32_t* slots, int32_t* positions, int32_t* counts, void* hip_stream) {
  if (!ctx_lens || !new_lens || !page_table || !total_lens || !row_starts || !counts || (n_free > 0 && !free_pages) ||
      (max_rows > 0 && (!slots || !positions)))
    return RLGEN_ERR_NULL;
  const int shift = page_shift(page_size);
  if (S < 1 || max_rows < 0 || n_free < 0 || table_stride < 1 || shift < 0) return RLGEN_ERR_BAD_ARG;
  PlanArgs a{};
  a.ctx_lens = ctx_lens; a.new_lens = new_lens; a.S = S; a.page_shift = shift;
  a.free_pages = free_pages; a.n_free = n_free; a.free_head = free_head;
  a.page_table = page_table; a.table_stride = table_stride; a.max_rows = max_rows;
  a.total_lens = total_lens; a.row_starts = row_starts; a.slots = slots; a.positions = positions; a.counts = counts;
  HIPCHK(rl_plan_pages(a, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

int rlgen_rope_table(float* table, int32_t max_pos, int32_t rotary_dim, float theta, void* hip_stream) {
  if (!table) return RLGEN_ERR_NULL;
  if (max_pos < 1 || rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > 256 || !std::isfinite(theta) || theta <= 0.f ||
      (int64_t)max_pos * rotary_dim > INT32_MAX)
    return RLGEN_ERR_BAD_ARG;
  HIPCHK(rl_rope_table((float2*)table, max_pos, rotary_dim, theta, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

int rlgen_qk_norm_rope(const void* qkv, int64_t qkv_stride, int32_t src_dtype, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads,
                       int32_t head_dim, const float* q_gain, const float* k_gain, float eps, const float* rope, int32_t max_pos,
                       int32_t rotary_dim, const int32_t* positions, int32_t dtype, void* q, int64_t q_stride, void* k, int64_t k_stride,
                       void* v, int64_t v_stride, void* pages, int32_t n_pages, int32_t page_size, const int32_t* slots, void* hip_stream) {
  NormRopeArgs a{};
  const int rc = norm_rope_args(a, qkv, qkv_stride, src_dtype, rows, n_q_heads, n_kv_heads, head_dim, q_gain, k_gain, eps, rope, max_pos,
                                rotary_dim, positions, dtype);
  if (rc != RLGEN_OK) return rc;
  if (rows > 0 && (!q || (!pages && !k) || (pages && !slots))) return RLGEN_ERR_NULL;
  const int shift = pages ? page_shift(page_size) : 0;
  if (!rows_ok(q, q_stride, n_q_heads, head_dim) || (k && !rows_ok(k, k_stride, n_kv_heads, head_dim)) ||
      (v && !rows_ok(v, v_stride, n_kv_heads, head_dim)) || (pages && !pages_ok(pages, n_pages, shift, n_kv_heads, head_dim)))
    return RLGEN_ERR_BAD_ARG;
  a.q = q; a.q_stride = q_stride; a.k = k; a.k_stride = k_stride; a.v = v; a.v_stride = v_stride;
  a.pages = pages; a.n_pages = n_pages; a.page_shift = shift; a.slots = slots;
  HIPCHK(rl_norm_rope(a, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

size_t rlgen_qk_norm_rope_backward_workspace(int32_t rows, int32_t head_dim) {
  return rows < 0 || head_dim < 1 || head_dim > 256 ? 0 : rl_norm_rope_backward_bytes(rows, head_dim);
}
int rlgen_qk_norm_rope_backward(const void* qkv, int64_t qkv_stride, int32_t src_dtype, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads,
                                int32_t head_dim, const float* q_gain, const float* k_gain, float eps, const float* rope, int32_t max_pos,
                                int32_t rotary_dim, const int32_t* positions, int32_t dtype, const void* dq, int64_t dq_stride,
                                const void* dk, int64_t dk_stride, const void* dv, int64_t dv_stride, void* dqkv, int64_t dqkv_stride,
                                float* dq_gain, float* dk_gain, void* workspace, size_t workspace_bytes, void* hip_stream) {
  NormRopeArgs a{};
  const int rc = norm_rope_args(a, qkv, qkv_stride, src_dtype, rows, n_q_heads, n_kv_heads, head_dim, q_gain, k_gain, eps, rope, max_pos,
                                rotary_dim, positions, dtype);
  if (rc != RLGEN_OK) return rc;
  if ((rows > 0 && (!dq || !dk || !dv || !dqkv)) || !dq_gain || !dk_gain || !workspace) return RLGEN_ERR_NULL;
  if (!rows_ok(dq, dq_stride, n_q_heads, head_dim) || !rows_ok(dk, dk_stride, n_kv_heads, head_dim) || !rows_ok(dv, dv_stride, n_kv_heads, head_dim) ||
      !rows_ok(dqkv, dqkv_stride, n_q_heads + 2 * n_kv_heads, head_dim, src_dtype == RLGEN_DTYPE_F32 ? 4 : 8))
    return RLGEN_ERR_BAD_ARG;
  if (!aligned16(workspace) || workspace_bytes < rl_norm_rope_backward_bytes(rows, head_dim)) return RLGEN_ERR_WORKSPACE;
  a.dq = dq; a.dq_stride = dq_stride; a.dk = dk; a.dk_stride = dk_stride; a.dv = dv; a.dv_stride = dv_stride;
  a.dqkv = dqkv; a.dqkv_stride = dqkv_stride; a.dq_gain = dq_gain; a.dk_gain = dk_gain; a.partial = (float*)workspace;
  HIPCHK(rl_norm_rope_backward(a, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

int rlgen_window_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int32_t dtype,
                           int32_t rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const int32_t* row_starts, int32_t S,
                           int32_t max_len, int32_t window, int32_t sinks, float scale, void* out, int64_t out_stride, float* lse,
                           void* hip_stream) {
  if ((rows > 0 && (!q || !k || !v || !out)) || !row_starts) return RLGEN_ERR_NULL;
  WindowArgs a = window_shape(dtype, rows, n_q_heads, n_kv_heads, head_dim, S, max_len, window, sinks, scale);
  if (!window_ok(a) || rl_window_rows_blocks(a) >= MOST_BLOCKS || !rows_ok(q, q_stride, n_q_heads, head_dim) ||
      !rows_ok(k, k_stride, n_kv_heads, head_dim) || !rows_ok(v, v_stride, n_kv_heads, head_dim) || !rows_ok(out, out_stride, n_q_heads, head_dim))
    return RLGEN_ERR_BAD_ARG;
  a.row_starts = row_starts;
  a.q = q; a.q_stride = q_stride; a.k = k; a.k_stride = k_stride; a.v = v; a.v_stride = v_stride;
  a.out = out; a.out_stride = out_stride; a.lse = lse;
  HIPCHK(rl_window_rows(a, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

size_t rlgen_window_attention_backward_workspace(int32_t rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t S,
                                                 int32_t max_len, int32_t window, int32_t sinks) {
  const WindowArgs a = window_shape(RLGEN_DTYPE_BF16, rows, n_q_heads, n_kv_heads, head_dim, S, max_len, window, sinks, 1.f);
  return window_ok(a) ? rl_window_backward_bytes(a) : 0;
}
int rlgen_window_attention_backward(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                    const void* out, int64_t out_stride, const float* lse, const void* dout, int64_t dout_stride,
                                    int32_t dtype, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    const int32_t* row_starts, int32_t S, int32_t max_len, int32_t window, int32_t sinks, float scale,
                                    void* dq, int64_t dq_stride, void* dk, int64_t dk_stride, void* dv, int64_t dv_stride, void* workspace,
                                    size_t workspace_bytes, void* hip_stream) {
  if ((rows > 0 && (!q || !k || !v || !out || !lse || !dout || !dq || !dk || !dv)) || !row_starts || !workspace) return RLGEN_ERR_NULL;
  WindowArgs a = window_shape(dtype, rows, n_q_heads, n_kv_heads, head_dim, S, max_len, window, sinks, scale);
  if (!window_ok(a) || rl_window_backward_blocks(a) >= MOST_BLOCKS || !rows_ok(q, q_stride, n_q_heads, head_dim) ||
      !rows_ok(k, k_stride, n_kv_heads, head_dim) || !rows_ok(v, v_stride, n_kv_heads, head_dim) || !rows_ok(out, out_stride, n_q_heads, head_dim) ||
      !rows_ok(dout, dout_stride, n_q_heads, head_dim) || !rows_ok(dq, dq_stride, n_q_heads, head_dim) ||
      !rows_ok(dk, dk_stride, n_kv_heads, head_dim) || !rows_ok(dv, dv_stride, n_kv_heads, head_dim))
    return RLGEN_ERR_BAD_ARG;
  if (!aligned16(workspace) || workspace_bytes < rl_window_backward_bytes(a)) return RLGEN_ERR_WORKSPACE;
  a.row_starts = row_starts;
  a.q = q; a.q_stride = q_stride; a.k = k; a.k_stride = k_stride; a.v = v; a.v_stride = v_stride;
  a.o = out; a.o_stride = out_stride; a.lse = (float*)lse; a.dout = dout; a.dout_stride = dout_stride;
  a.dq = dq; a.dq_stride = dq_stride; a.dk = dk; a.dk_stride = dk_stride; a.dv = dv; a.dv_stride = dv_stride;
  a.ws = workspace; a.ws_bytes = workspace_bytes;
  HIPCHK(rl_window_backward(a, (hipStream_t)hip_stream));
  return RLGEN_OK;
}

size_t rlgen_window_attention_paged_workspace(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t S, int32_t max_new,
                                              int32_t max_total, int32_t window, int32_t sinks) {
  WindowArgs a = window_shape(RLGEN_DTYPE_BF16, 1, n_q_heads, n_kv_heads, head_dim, S, max_new, window, sinks, 1.f);
  a.max_total = max_total;
  return window_ok(a) && max_new == 1 && max_total >= 1 ? rl_window_decode_bytes(a) : 0;
}
size_t rlgen_window_attention_chunk_workspace(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t S, int32_t max_new,
                                              int32_t max_total, int32_t window, int32_t sinks) {
  WindowArgs a = window_shape(RLGEN_DTYPE_BF16, 1, n_q_heads, n_kv_heads, head_dim, S, max_new, window, sinks, 1.f);
  a.max_total = max_total;
  return window_ok(a) && max_new > 1 && max_total >= 1 ? rl_window_rows_bytes(a) : 0;
}
int rlgen_window_attention_paged(const void* q, int64_t q_stride, int32_t dtype, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads,
                                 int32_t head_dim, const void* pages, int32_t n_pages, int32_t page_size, const int32_t* page_table,
                                 int32_t table_stride, const int32_t* row_starts, const int32_t* total_lens, int32_t S, int32_t max_new,
                                 int32_t max_total, int32_t window, int32_t sinks, float scale, void* out, int64_t out_stride, float* lse,
                                 void* workspace, size_t workspace_bytes, void* hip_stream) {
  if ((rows > 0 && (!q || !out)) || !pages || !page_table || !row_starts || !total_lens) return RLGEN_ERR_NULL;
  WindowArgs a = window_shape(dtype, rows, n_q_heads, n_kv_heads, head_dim, S, max_new, window, sinks, scale);
  const int shift = page_shift(page_size);
  if (!window_ok(a) || max_total < 1 || table_stride < 1 || !pages_ok(pages, n_pages, shift, n_kv_heads, head_dim) ||
      !rows_ok(q, q_stride, n_q_heads, head_dim) || !rows_ok(out, out_stride, n_q_heads, head_dim))
    return RLGEN_ERR_BAD_ARG;
  a.row_starts = row_starts; a.total_lens = total_lens; a.max_total = max_total;
  a.q = q; a.q_stride = q_stride; a.out = out; a.out_stride = out_stride; a.lse = lse;
  a.pages = pages; a.n_pages = n_pages; a.page_shift = shift; a.page_table = page_table; a.table_stride = table_stride;
  a.ws = workspace; a.ws_bytes = workspace_bytes;
  if ((max_new == 1 ? rl_window_decode_blocks(a) : rl_window_rows_blocks(a)) >= MOST_BLOCKS) return RLGEN_ERR_BAD_ARG;
  if (max_new == 1) {
    const size_t need = rl_window_decode_bytes(a);
    if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return RLGEN_ERR_WORKSPACE;
    HIPCHK(rl_window_decode(a, (hipStream_t)hip_stream));
  } else {
    if (workspace && !aligned16(workspace)) return RLGEN_ERR_WORKSPACE;
    HIPCHK(rl_window_rows(a, (hipStream_t)hip_stream));
  }
  return RLGEN_OK;
}

}  // extern "C"
