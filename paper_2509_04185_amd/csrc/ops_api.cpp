// C ABI of the operators without a context: the checks of their arguments.  Everything here
// runs on the host and touches no device memory; all arithmetic is in paged.hip,
// paged_attention.hip and scaled.hip.

#include <hip/hip_runtime.h>

#include <cmath>

#include "ops_internal.h"

using namespace sbd;

namespace {

constexpr int32_t kMaxOpBatch = 1 << 16;
constexpr int32_t kMaxOpRows = 1 << 24;
constexpr int32_t kMaxOpHeads = 1024;
constexpr int32_t kMaxOpDepth = 1 << 22;  // bytes of a row of codes: 256 rows lie within 32-bit offsets

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

bool page_size_ok(int32_t p) { return p >= 16 && p <= 256 && (p & (p - 1)) == 0; }

sbd_status check_table(const sbd_page_table* t) {
  if (!t) return op_fail(SBD_ERR_INVALID_ARG, "null page table");
  if (t->batch < 1 || t->batch > kMaxOpBatch) return op_fail(SBD_ERR_INVALID_ARG, "batch %d out of [1, %d]", t->batch, kMaxOpBatch);
  if (!page_size_ok(t->page_size))
    return op_fail(SBD_ERR_INVALID_ARG, "page_size %d is no power of two in [16, 256]", t->page_size);
  if (t->n_pages < 1 || (int64_t)t->n_pages * t->page_size > INT32_MAX)
    return op_fail(SBD_ERR_INVALID_ARG, "n_pages %d: need at least 1 and fewer than 2^31 tokens", t->n_pages);
  if (t->max_pages < 1 || (int64_t)t->max_pages * t->page_size > (1 << 30))
    return op_fail(SBD_ERR_INVALID_ARG, "max_pages %d: need at least 1 and at most 2^30 tokens", t->max_pages);
  if (!t->table || !t->held || !t->cached || !t->free_list || !t->free_count)
    return op_fail(SBD_ERR_INVALID_ARG, "null pointer in the page table");
  return SBD_OK;
}

sbd_status check_kv(const sbd_paged_kv* c, bool pointers) {
  if (!c) return op_fail(SBD_ERR_INVALID_ARG, "null paged cache");
  if (!page_size_ok(c->page_size))
    return op_fail(SBD_ERR_INVALID_ARG, "page_size %d is no power of two in [16, 256]", c->page_size);
  if (c->n_pages < 1 || (int64_t)c->n_pages * c->page_size > INT32_MAX)
    return op_fail(SBD_ERR_INVALID_ARG, "n_pages %d: need at least 1 and fewer than 2^31 tokens", c->n_pages);
  if (c->head_dim != 64 && c->head_dim != 128)
    return op_fail(SBD_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", c->head_dim);
  if (c->n_kv_heads < 1 || c->n_kv_heads > kMaxOpHeads)
    return op_fail(SBD_ERR_INVALID_ARG, "n_kv_heads %d out of [1, %d]", c->n_kv_heads, kMaxOpHeads);
  if (!pointers) return SBD_OK;
  if (!c->k_codes || !c->v_codes || !c->k_exp || !c->v_exp)
    return op_fail(SBD_ERR_INVALID_ARG, "null pointer in the paged cache");
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes)) return op_fail(SBD_ERR_INVALID_ARG, "codes must be 16-byte aligned");
  return SBD_OK;
}

sbd_status check_rows(int32_t batch, int32_t rows) {
  if (batch < 1 || batch > kMaxOpBatch) return op_fail(SBD_ERR_INVALID_ARG, "batch %d out of [1, %d]", batch, kMaxOpBatch);
  if (rows < 0 || rows > kMaxOpRows) return op_fail(SBD_ERR_INVALID_ARG, "rows %d out of [0, %d]", rows, kMaxOpRows);
  return SBD_OK;
}

// Rows of `width` elements of a 16-bit type, `stride` apart, that are read or written 16 bytes at a time.
sbd_status check_rows16(const char* what, const void* p, int64_t stride, int64_t width) {
  if (!p) return op_fail(SBD_ERR_INVALID_ARG, "%s is null", what);
  if (!aligned16(p)) return op_fail(SBD_ERR_INVALID_ARG, "%s must be 16-byte aligned", what);
  if (stride < width || stride % 8)
    return op_fail(SBD_ERR_INVALID_ARG, "%s: a row stride of %lld elements (need a multiple of 8 of at least %lld)", what,
                   (long long)stride, (long long)width);
  return SBD_OK;
}

sbd_status done(hipError_t e, const char* what) {
  if (e != hipSuccess) return op_fail(SBD_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
  return SBD_OK;
}

sbd_status check_attention(const sbd_paged_kv* c, bool pointers, int32_t batch, int32_t rows, int32_t n_q, int32_t max_kv) {
  if (sbd_status st = check_kv(c, pointers)) return st;
  if (sbd_status st = check_rows(batch, rows)) return st;
  if (n_q < 1 || n_q % c->n_kv_heads || n_q > kMaxOpHeads)
    return op_fail(SBD_ERR_INVALID_ARG, "n_q_heads %d is no multiple of n_kv_heads %d, or over %d", n_q, c->n_kv_heads, kMaxOpHeads);
  if (max_kv < 1 || max_kv > (1 << 30)) return op_fail(SBD_ERR_INVALID_ARG, "max_kv %d out of [1, 2^30]", max_kv);
  if ((int64_t)rows * n_q > INT32_MAX) return op_fail(SBD_ERR_INVALID_ARG, "rows * n_q_heads exceeds 2^31");
  return SBD_OK;
}

sbd_status check_matmul(int32_t m, int32_t n, int32_t k) {
  if (m < 0 || m > kMaxOpRows) return op_fail(SBD_ERR_INVALID_ARG, "m %d out of [0, %d]", m, kMaxOpRows);
  if (n < 1 || n > kMaxOpRows) return op_fail(SBD_ERR_INVALID_ARG, "n %d out of [1, %d]", n, kMaxOpRows);
  if (k < 16 || k % 16 || k > kMaxOpDepth)
    return op_fail(SBD_ERR_INVALID_ARG, "k %d is no multiple of 16 in [16, %d]", k, kMaxOpDepth);
  if ((int64_t)m * n > ((int64_t)1 << 36)) return op_fail(SBD_ERR_INVALID_ARG, "m * n exceeds 2^36");
  return SBD_OK;
}

}  // namespace

extern "C" {

sbd_status sbd_paged_plan(void* stream, const sbd_page_table* t, const int32_t* n_new, const uint8_t* release,
                          int32_t rows, int32_t* row_start, int32_t* kv_len, int32_t* slots, int32_t* scratch) {
  if (sbd_status st = check_table(t)) return st;
  if (sbd_status st = check_rows(t->batch, rows)) return st;
  if (!n_new || !row_start || !kv_len || (!slots && rows > 0) || !scratch) return op_fail(SBD_ERR_INVALID_ARG, "null argument");
  return done(launch_paged_plan(PlanArgs{*t, n_new, release, rows, row_start, kv_len, slots, scratch},
                                static_cast<hipStream_t>(stream)),
              "paged plan");
}

sbd_status sbd_paged_append(void* stream, const sbd_paged_kv* c, int32_t dtype, int32_t batch, int32_t rows,
                            const int32_t* row_start, const int32_t* slots, const void* k, int64_t k_stride,
                            const void* v, int64_t v_stride) {
  if (sbd_status st = check_kv(c, true)) return st;
  if (sbd_status st = check_rows(batch, rows)) return st;
  if (dtype != SBD_TYPE_BF16 && dtype != SBD_TYPE_FP16)
    return op_fail(SBD_ERR_INVALID_ARG, "keys and values must be SBD_TYPE_BF16 or SBD_TYPE_FP16 (got %d)", dtype);
  if (!row_start) return op_fail(SBD_ERR_INVALID_ARG, "null row_start");
  if (rows == 0) return SBD_OK;
  if (!slots) return op_fail(SBD_ERR_INVALID_ARG, "null slots");
  const int64_t width = (int64_t)c->n_kv_heads * c->head_dim;
  if (sbd_status st = check_rows16("k", k, k_stride, width)) return st;
  if (sbd_status st = check_rows16("v", v, v_stride, width)) return st;
  return done(launch_paged_append(AppendArgs{*c, batch, rows, row_start, slots, k, v, k_stride, v_stride}, dtype,
                                  static_cast<hipStream_t>(stream)),
              "paged append");
}

sbd_status sbd_paged_attention_workspace(const sbd_paged_kv* c, int32_t batch, int32_t rows, int32_t n_q_heads,
                                         int32_t max_kv, size_t* bytes) {
  if (sbd_status st = check_attention(c, false, batch, rows, n_q_heads, max_kv)) return st;
  if (!bytes) return op_fail(SBD_ERR_INVALID_ARG, "null bytes");
  *bytes = paged_attention_plan(*c, batch, rows, n_q_heads, max_kv).bytes;
  return SBD_OK;
}

sbd_status sbd_paged_attention(void* stream, const sbd_paged_kv* c, int32_t dtype, int32_t batch, int32_t rows,
                               int32_t n_q_heads, const int32_t* row_start, const int32_t* kv_len,
                               const int32_t* table, int32_t max_pages, const int32_t* n_causal, float scale,
                               int32_t max_kv, const void* q, int64_t q_stride, void* out, int64_t out_stride,
                               void* workspace, size_t workspace_bytes) {
  if (sbd_status st = check_attention(c, true, batch, rows, n_q_heads, max_kv)) return st;
  if (dtype != SBD_TYPE_BF16 && dtype != SBD_TYPE_FP16)
    return op_fail(SBD_ERR_INVALID_ARG, "queries must be SBD_TYPE_BF16 or SBD_TYPE_FP16 (got %d)", dtype);
  if (!row_start || !kv_len || !table) return op_fail(SBD_ERR_INVALID_ARG, "null argument");
  if (max_pages < 1 || (int64_t)max_pages * c->page_size > (1 << 30))
    return op_fail(SBD_ERR_INVALID_ARG, "max_pages %d: need at least 1 and at most 2^30 tokens", max_pages);
  if (max_kv > (int64_t)max_pages * c->page_size)
    return op_fail(SBD_ERR_INVALID_ARG, "max_kv %d exceeds the table's %lld tokens", max_kv,
                   (long long)max_pages * c->page_size);
  const float scale_log2 = scale * 1.44269504088896340736f;
  if (!std::isfinite(scale_log2)) return op_fail(SBD_ERR_INVALID_ARG, "scale must be finite (and below 2.3e38 in size)");
  if (rows == 0) return SBD_OK;
  const int64_t width = (int64_t)n_q_heads * c->head_dim;
  if (sbd_status st = check_rows16("q", q, q_stride, width)) return st;
  if (sbd_status st = check_rows16("out", out, out_stride, width)) return st;
  PagedAttnArgs a{};
  a.plan = paged_attention_plan(*c, batch, rows, n_q_heads, max_kv);
  if (a.plan.bytes > 0 && (!workspace || !aligned16(workspace)))
    return op_fail(SBD_ERR_INVALID_ARG, "workspace must be 16-byte aligned device memory");
  if (workspace_bytes < a.plan.bytes)
    return op_fail(SBD_ERR_OUT_OF_MEMORY, "workspace of %zu bytes, need %zu", workspace_bytes, a.plan.bytes);
  a.c = *c; a.batch = batch; a.rows = rows; a.n_q = n_q_heads; a.max_pages = max_pages;
  a.row_start = row_start; a.kv_len = kv_len; a.table = table; a.n_causal = n_causal;
  a.scale_log2 = scale_log2;
  a.q = q; a.out = out; a.q_stride = q_stride; a.out_stride = out_stride;
  if (a.plan.bytes > 0) {
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + a.plan.part_ml);
    a.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + a.plan.part_o);
  }
  return done(launch_paged_attention(a, dtype, static_cast<hipStream_t>(stream)), "paged attention");
}

sbd_status sbd_scaled_quantize(void* stream, int32_t dtype, int32_t rows, int32_t cols, const void* x,
                               int64_t x_stride, int32_t block_rows, uint8_t* codes, float* scales) {
  if (dtype != SBD_TYPE_BF16 && dtype != SBD_TYPE_FP16 && dtype != SBD_TYPE_FP32)
    return op_fail(SBD_ERR_INVALID_ARG, "unknown type %d", dtype);
  if (rows < 0 || rows > kMaxOpRows) return op_fail(SBD_ERR_INVALID_ARG, "rows %d out of [0, %d]", rows, kMaxOpRows);
  if (cols < 16 || cols % 16 || cols > kMaxOpRows)
    return op_fail(SBD_ERR_INVALID_ARG, "cols %d is no multiple of 16 in [16, %d]", cols, kMaxOpRows);
  if ((int64_t)rows * cols > ((int64_t)1 << 36)) return op_fail(SBD_ERR_INVALID_ARG, "rows * cols exceeds 2^36");
  if (block_rows != 1 && block_rows != 128) return op_fail(SBD_ERR_INVALID_ARG, "block_rows must be 1 or 128 (got %d)", block_rows);
  if (rows == 0) return SBD_OK;
  if (!x || !codes || !scales) return op_fail(SBD_ERR_INVALID_ARG, "null argument");
  const int64_t es = dtype == SBD_TYPE_FP32 ? 4 : 2;
  if (!aligned16(x) || !aligned16(codes)) return op_fail(SBD_ERR_INVALID_ARG, "x and codes must be 16-byte aligned");
  if (x_stride < cols || x_stride * es % 16)
    return op_fail(SBD_ERR_INVALID_ARG, "a row stride of %lld elements (need at least %d and rows 16-byte aligned)",
                   (long long)x_stride, cols);
  return done(launch_scaled_quantize(QuantizeArgs{rows, cols, block_rows, x, x_stride, codes, scales}, dtype,
                                     static_cast<hipStream_t>(stream)),
              "scaled quantize");
}

sbd_status sbd_scaled_matmul_workspace(int32_t m, int32_t n, int32_t k, size_t* bytes) {
  if (sbd_status st = check_matmul(m, n, k)) return st;
  if (!bytes) return op_fail(SBD_ERR_INVALID_ARG, "null bytes");
  *bytes = scaled_matmul_bytes(m, n, k);
  return SBD_OK;
}

sbd_status sbd_scaled_matmul(void* stream, int32_t m, int32_t n, int32_t k, const uint8_t* a, int64_t a_stride,
                             const float* a_scale, const uint8_t* b, const float* b_scale, int32_t out_type,
                             void* out, int64_t out_stride, void* workspace, size_t workspace_bytes) {
  if (sbd_status st = check_matmul(m, n, k)) return st;
  if (out_type != SBD_TYPE_BF16 && out_type != SBD_TYPE_FP16 && out_type != SBD_TYPE_FP32)
    return op_fail(SBD_ERR_INVALID_ARG, "unknown output type %d", out_type);
  if (m == 0) return SBD_OK;
  if (!a || !a_scale || !b || !b_scale || !out) return op_fail(SBD_ERR_INVALID_ARG, "null argument");
  if (!aligned16(a) || !aligned16(b)) return op_fail(SBD_ERR_INVALID_ARG, "a and b must be 16-byte aligned");
  if (a_stride < k || a_stride % 16 || a_stride > kMaxOpDepth)
    return op_fail(SBD_ERR_INVALID_ARG, "a row stride of %lld (need a multiple of 16 in [%d, %d])", (long long)a_stride, k,
                   kMaxOpDepth);
  if (out_stride < n) return op_fail(SBD_ERR_INVALID_ARG, "an output row stride of %lld, below n %d", (long long)out_stride, n);
  if (reinterpret_cast<uintptr_t>(out) % (out_type == SBD_TYPE_FP32 ? 4 : 2))
    return op_fail(SBD_ERR_INVALID_ARG, "out is not aligned to its type");
  const size_t need = scaled_matmul_bytes(m, n, k);
  if (need > 0 && (!workspace || !aligned16(workspace)))
    return op_fail(SBD_ERR_INVALID_ARG, "workspace must be 16-byte aligned device memory");
  if (workspace_bytes < need) return op_fail(SBD_ERR_OUT_OF_MEMORY, "workspace of %zu bytes, need %zu", workspace_bytes, need);
  return done(launch_scaled_matmul(MatmulArgs{m, n, k, a, b, a_stride, out_stride, a_scale, b_scale, out,
                                              static_cast<float*>(workspace)},
                                   out_type, static_cast<hipStream_t>(stream)),
              "scaled matmul");
}

}  // extern "C"
