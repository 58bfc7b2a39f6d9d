// The checks of the operators without a context (ops_api.cpp) on the CPU, built with
// AddressSanitizer and UndefinedBehaviorSanitizer: the sizes at the ends of their ranges reach
// the launchers (stand-ins that note the call) or are refused, with a reason.  Exit status 0
// when every check holds.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <limits>

#include "hip/hip_runtime.h"
#include "ops_internal.h"

static int g_failed = 0, g_launches = 0;
static hipError_t g_result = hipSuccess;

namespace sbd {
hipError_t launch_paged_plan(const PlanArgs&, hipStream_t) { ++g_launches; return g_result; }
hipError_t launch_paged_append(const AppendArgs&, int, hipStream_t) { ++g_launches; return g_result; }
PagedAttnPlan paged_attention_plan(const sbd_paged_kv&, int, int, int, int max_kv) {
  PagedAttnPlan p{};
  p.n_splits = max_kv > 1000 ? 2 : 1;
  p.bytes = p.n_splits > 1 ? 4096 : 0;
  p.part_o = p.n_splits > 1 ? 1024 : 0;
  return p;
}
hipError_t launch_paged_attention(const PagedAttnArgs& a, int, hipStream_t) {
  ++g_launches;
  if (a.plan.n_splits > 1 && (!a.part_ml || !a.part_o)) ++g_failed;
  return g_result;
}
hipError_t launch_scaled_quantize(const QuantizeArgs&, int, hipStream_t) { ++g_launches; return g_result; }
size_t scaled_matmul_bytes(int m, int, int) { return m == 7 ? 256 : 0; }
hipError_t launch_scaled_matmul(const MatmulArgs&, int, hipStream_t) { ++g_launches; return g_result; }
}  // namespace sbd

#define CHECK(cond)                                                  \
  do {                                                               \
    if (!(cond)) {                                                   \
      ++g_failed;                                                    \
      std::fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #cond); \
    }                                                                \
  } while (0)
#define RUNS(call)                   \
  do {                               \
    const int n_ = g_launches;       \
    CHECK((call) == SBD_OK);         \
    CHECK(g_launches == n_ + 1);     \
  } while (0)
#define REFUSES(want, call)                          \
  do {                                               \
    const int n_ = g_launches;                       \
    CHECK((call) == (want));                         \
    CHECK(g_launches == n_);                         \
    CHECK(std::strlen(sbd_last_error(nullptr)) > 0); \
  } while (0)

int main() {
  alignas(16) static unsigned char mem[64];
  int32_t* i = reinterpret_cast<int32_t*>(mem);
  float* f = reinterpret_cast<float*>(mem);
  uint8_t* u = mem;
  int8_t* e = reinterpret_cast<int8_t*>(mem);
  const int32_t big = std::numeric_limits<int32_t>::max(), low = std::numeric_limits<int32_t>::min();

  sbd_page_table t{1, 1, 1, 16, i, i, i, i, i};
  RUNS(sbd_paged_plan(nullptr, &t, i, nullptr, 0, i, i, nullptr, i));
  for (int32_t page : {16, 32, 64, 128, 256}) {
    t = sbd_page_table{1 << 16, (1 << 30) / page, big / page, page, i, i, i, i, i};
    RUNS(sbd_paged_plan(nullptr, &t, i, u, 1 << 24, i, i, i, i));
    t.n_pages = big / page + 1;
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_plan(nullptr, &t, i, u, 8, i, i, i, i));
  }
  for (int32_t bad : {big, low, -1, 0}) {
    t = sbd_page_table{bad, 1, 1, 16, i, i, i, i, i};
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_plan(nullptr, &t, i, u, 8, i, i, i, i));
    t = sbd_page_table{1, bad, 1, 16, i, i, i, i, i};
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_plan(nullptr, &t, i, u, 8, i, i, i, i));
    t = sbd_page_table{1, 1, bad, 16, i, i, i, i, i};
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_plan(nullptr, &t, i, u, 8, i, i, i, i));
    t = sbd_page_table{1, 1, 1, bad, i, i, i, i, i};
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_plan(nullptr, &t, i, u, 8, i, i, i, i));
  }

  sbd_paged_kv c{big / 256, 256, 1024, 128, u, u, e, e};
  RUNS(sbd_paged_append(nullptr, &c, SBD_TYPE_BF16, 1 << 16, 1 << 24, i, i, u, 1024 * 128, u, (int64_t)1 << 60));
  RUNS(sbd_paged_attention(nullptr, &c, SBD_TYPE_FP16, 1, 1 << 20, 1024, i, i, i, 1 << 22, nullptr, -1.f, 1000, u, 1024 * 128, u,
                           1024 * 128, nullptr, 0));
  RUNS(sbd_paged_attention(nullptr, &c, SBD_TYPE_FP16, 1, 1, 1024, i, i, i, 1 << 22, i, 0.f, 1 << 30, u, 1024 * 128, u, 1024 * 128,
                           u, 4096));
  REFUSES(SBD_ERR_OUT_OF_MEMORY, sbd_paged_attention(nullptr, &c, SBD_TYPE_FP16, 1, 1, 1024, i, i, i, 1 << 22, i, 0.f, 1 << 30, u,
                                                     1024 * 128, u, 1024 * 128, u, 4095));
  REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_attention(nullptr, &c, SBD_TYPE_FP16, 1, 1 << 22, 1024, i, i, i, 1 << 22, i, 0.f, 1000, u,
                                                   1024 * 128, u, 1024 * 128, u, 4096));
  for (int32_t bad : {big, low, -1, 0}) {
    sbd_paged_kv d = c;
    d.n_kv_heads = bad;
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_append(nullptr, &d, 0, 1, 1, i, i, u, 1024 * 128, u, 1024 * 128));
    d = c;
    d.n_pages = bad;
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_append(nullptr, &d, 0, 1, 1, i, i, u, 1024 * 128, u, 1024 * 128));
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_append(nullptr, &c, 0, bad, 1, i, i, u, 1024 * 128, u, 1024 * 128));
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_append(nullptr, &c, 0, 1, 1, i, i, u, bad, u, 1024 * 128));
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_attention(nullptr, &c, 0, 1, 1, bad, i, i, i, 1, i, 1.f, 1, u, 1 << 20, u, 1 << 20, u, 0));
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_attention(nullptr, &c, 0, 1, 1, 1024, i, i, i, bad, i, 1.f, 1, u, 1 << 20, u, 1 << 20, u, 0));
    REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_attention(nullptr, &c, 0, 1, 1, 1024, i, i, i, 1, i, 1.f, bad, u, 1 << 20, u, 1 << 20, u, 0));
    if (bad != 0) {
      REFUSES(SBD_ERR_INVALID_ARG, sbd_paged_append(nullptr, &c, 0, 1, bad, i, i, u, 1024 * 128, u, 1024 * 128));
      REFUSES(SBD_ERR_INVALID_ARG, sbd_scaled_quantize(nullptr, 0, bad, 128, u, 128, 1, u, f));
      REFUSES(SBD_ERR_INVALID_ARG, sbd_scaled_matmul(nullptr, bad, 128, 128, u, 128, f, u, f, 0, u, 128, nullptr, 0));
    }
    REFUSES(SBD_ERR_INVALID_ARG, sbd_scaled_quantize(nullptr, 0, 1, bad, u, 128, 1, u, f));
    REFUSES(SBD_ERR_INVALID_ARG, sbd_scaled_matmul(nullptr, 1, bad, 128, u, 128, f, u, f, 0, u, 128, nullptr, 0));
    REFUSES(SBD_ERR_INVALID_ARG, sbd_scaled_matmul(nullptr, 1, 128, bad, u, 128, f, u, f, 0, u, 128, nullptr, 0));
  }
  RUNS(sbd_scaled_quantize(nullptr, SBD_TYPE_FP32, 1 << 24, 1 << 12, u, (int64_t)1 << 50, 128, u, f));
  RUNS(sbd_scaled_quantize(nullptr, SBD_TYPE_FP32, 1 << 12, 1 << 24, u, (int64_t)1 << 50, 1, u, f));
  REFUSES(SBD_ERR_INVALID_ARG, sbd_scaled_quantize(nullptr, SBD_TYPE_FP32, 1 << 24, 1 << 13, u, 1 << 13, 1, u, f));
  RUNS(sbd_scaled_matmul(nullptr, 1 << 24, 1 << 12, 1 << 22, u, 1 << 22, f, u, f, SBD_TYPE_FP32, u, 1 << 24, nullptr, 0));
  REFUSES(SBD_ERR_INVALID_ARG, sbd_scaled_matmul(nullptr, 1 << 24, 1 << 24, 128, u, 128, f, u, f, 0, u, 1 << 24, nullptr, 0));
  RUNS(sbd_scaled_matmul(nullptr, 7, 1, 16, u, 16, f, u, f, SBD_TYPE_BF16, u + 2, 1, u, 256));
  REFUSES(SBD_ERR_OUT_OF_MEMORY, sbd_scaled_matmul(nullptr, 7, 1, 16, u, 16, f, u, f, SBD_TYPE_BF16, u, 1, u, 255));
  REFUSES(SBD_ERR_INVALID_ARG, sbd_scaled_matmul(nullptr, 7, 1, 16, u, 16, f, u, f, SBD_TYPE_BF16, u, 1, nullptr, 256));

  // a launch that fails is reported
  g_result = hipErrorInvalidValue;
  CHECK(sbd_scaled_quantize(nullptr, SBD_TYPE_FP32, 1, 128, u, 128, 1, u, f) == SBD_ERR_HIP);
  CHECK(std::strlen(sbd_last_error(nullptr)) > 0);

  if (g_failed) return 1;
  std::printf("operator checks passed\n");
  return 0;
}
