// Internal declarations of the operators without a context (paged cache, block-scaled e4m3
// product): shared by their checks (ops_api.cpp) and their kernels (paged.hip,
// paged_attention.hip, scaled.hip).  Not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "sbd.h"

namespace sbd {

// Sets the calling thread's last error and returns st.
sbd_status op_fail(sbd_status st, const char* fmt, ...);

struct PlanArgs {
  sbd_page_table t;
  const int32_t* n_new;
  const uint8_t* release;
  int32_t rows;
  int32_t *row_start, *kv_len, *slots, *scratch;
};
hipError_t launch_paged_plan(const PlanArgs& a, hipStream_t s);

struct AppendArgs {
  sbd_paged_kv c;
  int32_t batch, rows;
  const int32_t *row_start, *slots;
  const void *k, *v;
  int64_t k_stride, v_stride;
};
hipError_t launch_paged_append(const AppendArgs& a, int dtype, hipStream_t s);

// How an attention call is cut: the shape of a workgroup (rows are (row, query head) pairs of a
// KV head), and every sequence's keys in n_splits parts.
struct PagedAttnPlan {
  int32_t shape, n_splits;
  int64_t rowblocks;  // workgroups of one KV head and key part, upper bound
  size_t part_ml, part_o, bytes;  // workspace: (max, sum) and outputs of the key parts
};
PagedAttnPlan paged_attention_plan(const sbd_paged_kv& c, int batch, int rows, int n_q, int max_kv);

struct PagedAttnArgs {
  sbd_paged_kv c;
  PagedAttnPlan plan;
  int32_t batch, rows, n_q, max_pages;
  const int32_t *row_start, *kv_len, *table, *n_causal;
  float scale_log2;  // scale * log2(e)
  const void* q;
  void* out;
  int64_t q_stride, out_stride;
  float *part_ml, *part_o;
};
hipError_t launch_paged_attention(const PagedAttnArgs& a, int dtype, hipStream_t s);

struct QuantizeArgs {
  int32_t rows, cols, block_rows;
  const void* x;
  int64_t x_stride;
  uint8_t* codes;
  float* scales;
};
hipError_t launch_scaled_quantize(const QuantizeArgs& a, int dtype, hipStream_t s);

struct MatmulArgs {
  int32_t m, n, k;
  const uint8_t *a, *b;
  int64_t a_stride, out_stride;
  const float *a_scale, *b_scale;
  void* out;
  float* part;
};
size_t scaled_matmul_bytes(int m, int n, int k);
hipError_t launch_scaled_matmul(const MatmulArgs& a, int out_type, hipStream_t s);

}  // namespace sbd
