// Page tables of a serving batch (sbd_paged_plan) and the write into a paged e4m3 cache
// (sbd_paged_append).

#include "ops_device.h"

namespace sbd {

// ---- page tables ----------------------------------------------------------------------
//
// need_b = max(0, ceil((cached_b + new_b) / page) - held_b).  Everything else is three scans
// over the sequences: of the pages that released sequences give back, of the pages needed
// (sequence b's new pages are entries base + scan_b .. of the free list, base = pages left
// afterwards) and of the new rows.  One workgroup does the scans and the state (phase 1); the
// released pages are then copied to the free list (phase 2), and table entries and slots are
// written (phase 3), each by as many threads as there are items.  A row's slot is formed from
// the free list itself, not from the table entry another thread writes.
//
// scratch: [0, B) index of the first new page relative to base; [B, 2B) pages held before
// taking; [2B, 3B] scan of the pages given back; [3B + 1] free pages before the call.

constexpr int kPlanThreads = 1024;

// Exclusive scan over the workgroup; total gets the sum.
__device__ int64_t block_scan(int64_t v, int64_t* waves, int64_t& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(s, o);
    if (lane >= o) s += u;
  }
  __syncthreads();  // waves[] may still be read from the scan before
  if (lane == 63) waves[w] = s;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll 1
  for (int i = 0; i < kPlanThreads / 64; ++i) {
    if (i < w) before += waves[i];
    all += waves[i];
  }
  total = all;
  return before + s - v;
}

__device__ void plan_scans(const PlanArgs& a) {
  __shared__ int64_t waves[kPlanThreads / 64];
  const sbd_page_table& t = a.t;
  const int B = t.batch, W = t.max_pages;
  const int free0 = min(max(*t.free_count, 0), t.n_pages);
  int64_t back = 0, total;
  if (a.release) {
    for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
      const int b = b0 + threadIdx.x;
      const int v = (b < B && a.release[b]) ? min(max(t.held[b], 0), W) : 0;
      const int64_t at = back + block_scan(v, waves, total);
      if (b < B) a.scratch[2 * B + b] = (int)min(at, (int64_t)t.n_pages);
      back += total;
    }
  }
  const int given = (int)min(back, (int64_t)(t.n_pages - free0));
  const int avail = free0 + given;
  int64_t need_sum = 0, row_sum = 0, taken = 0;
  for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
    const int b = b0 + threadIdx.x;
    const bool in = b < B;
    const bool gone = in && a.release && a.release[b];
    const int held = (in && !gone) ? min(max(t.held[b], 0), W) : 0;
    const int cached = (in && !gone) ? t.cached[b] : 0;
    const int n = in ? a.n_new[b] : 0;
    const int64_t tokens = (int64_t)cached + n;
    const bool fits = in && cached >= 0 && n >= 0 && tokens <= (int64_t)W * t.page_size;
    const int need = fits ? max((int)((tokens + t.page_size - 1) / t.page_size) - held, 0) : 0;
    const int64_t at = need_sum + block_scan(need, waves, total);
    need_sum += total;
    const bool ok = fits && (need == 0 || at + need <= avail);
    const int got = ok ? need : 0;
    block_scan(got, waves, total);
    taken += total;
    const int64_t row = row_sum + block_scan(max(n, 0), waves, total);
    row_sum += total;
    if (in) {
      a.scratch[b] = (int)min(at, (int64_t)t.n_pages);
      a.scratch[B + b] = held;
      a.row_start[b] = (int)min(row, (int64_t)INT32_MAX);
      a.kv_len[b] = ok ? (int)tokens : 0;
      t.held[b] = held + got;
      if (gone) t.cached[b] = 0;
    }
  }
  if (threadIdx.x == 0) {
    a.row_start[B] = (int)min(row_sum, (int64_t)INT32_MAX);
    a.scratch[3 * B] = given;
    a.scratch[3 * B + 1] = free0;
    *t.free_count = avail - (int)taken;
  }
}

__device__ void plan_give_back(const PlanArgs& a, int64_t first, int64_t step) {
  const sbd_page_table& t = a.t;
  const int B = t.batch, n = a.scratch[3 * B], free0 = a.scratch[3 * B + 1];
  const int* start = a.scratch + 2 * B;
  for (int64_t i = first; i < n; i += step) {
    int lo = 0, hi = B;  // last sequence that starts at or before i (empty ones before it start there too)
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (start[mid] <= i) lo = mid; else hi = mid;
    }
    t.free_list[free0 + i] = t.table[(int64_t)lo * t.max_pages + min((int)i - start[lo], t.max_pages - 1)];
  }
}

__device__ void plan_tables(const PlanArgs& a, int64_t first, int64_t step) {
  const sbd_page_table& t = a.t;
  const int B = t.batch, W = t.max_pages, base = *t.free_count;
  auto free_page = [&](int b, int col, int held) {
    return t.free_list[min(max(base + a.scratch[b] + col - held, 0), t.n_pages - 1)];
  };
  for (int64_t i = first; i < (int64_t)B * W; i += step) {
    const int b = (int)(i / W), col = (int)(i % W);
    const int held = a.scratch[B + b], now = t.held[b];
    if (col >= held && col < now)
      t.table[i] = free_page(b, col, held);
    else if (col >= now && a.release && a.release[b])
      t.table[i] = -1;
  }
  const int rows = a.row_start[B];
  for (int64_t r = first; r < a.rows; r += step) {
    int slot = -1;
    if (r < rows) {
      int lo = 0, hi = B;  // last sequence that starts at or before r: it is not an empty one
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.row_start[mid] <= r) lo = mid; else hi = mid;
      }
      if (a.kv_len[lo] > 0) {
        const int p = t.cached[lo] + (int)r - a.row_start[lo], col = p / t.page_size, held = a.scratch[B + lo];
        const int page = col < held ? t.table[(int64_t)lo * W + col] : free_page(lo, col, held);
        if (page >= 0 && page < t.n_pages) slot = page * t.page_size + p % t.page_size;
      }
    }
    a.slots[r] = slot;
  }
}

__global__ __launch_bounds__(kPlanThreads) void plan_all_kernel(PlanArgs a) {
  plan_scans(a);
  __syncthreads();
  if (a.release) {
    plan_give_back(a, threadIdx.x, kPlanThreads);
    __syncthreads();
  }
  plan_tables(a, threadIdx.x, kPlanThreads);
}
__global__ __launch_bounds__(kPlanThreads) void plan_scans_kernel(PlanArgs a) { plan_scans(a); }
__global__ __launch_bounds__(256) void plan_give_back_kernel(PlanArgs a) {
  plan_give_back(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}
__global__ __launch_bounds__(256) void plan_tables_kernel(PlanArgs a) {
  plan_tables(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

hipError_t launch_paged_plan(const PlanArgs& a, hipStream_t s) {
  const int64_t items = std::max<int64_t>((int64_t)a.t.batch * a.t.max_pages, a.rows);
  if (items <= 16 * kPlanThreads) {
    hipLaunchKernelGGL(plan_all_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
    return hipGetLastError();
  }
  const unsigned grid = (unsigned)std::min<int64_t>((items + 255) / 256, 2048);
  hipLaunchKernelGGL(plan_scans_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  if (a.release) hipLaunchKernelGGL(plan_give_back_kernel, dim3(grid), dim3(256), 0, s, a);
  hipLaunchKernelGGL(plan_tables_kernel, dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}

// ---- write into the cache ---------------------------------------------------------------
//
// One workgroup per (page that the step writes, KV head, keys or values).  The pages are
// numbered without a list of them: a sequence whose n rows start at row r touches at most
// floor(n / page) + 2 pages, so numbers r / page + 2 b .. are its own and the workgroup finds
// its sequence by a search over row_start.

constexpr int kAppendThreads = 256;

// The workgroup's largest value, in every thread.
__device__ float block_max(float v) {
  __shared__ float waves[kAppendThreads / 64];
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  v = fmaxf(fmaxf(waves[0], waves[1]), fmaxf(waves[2], waves[3]));
  return v;
}

// A code at another scale: value * f, rounded again.
__device__ uint32_t rescale4(uint32_t w, float f) {
  return to_e4m3x4(e4m3_to_f32(w & 255, 1.f) * f, e4m3_to_f32((w >> 8) & 255, 1.f) * f,
                   e4m3_to_f32((w >> 16) & 255, 1.f) * f, e4m3_to_f32(w >> 24, 1.f) * f);
}

template <class T, int DH>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a) {
  extern __shared__ uint8_t tile[];  // [page_size][DH + 4] new codes of the values
  constexpr int kPieces = DH / 8, kLd = DH + 4;
  const int P = a.c.page_size, H = a.c.n_kv_heads;
  const int head = blockIdx.y >> 1;
  const bool values = blockIdx.y & 1;
  const int tid = threadIdx.x;
  auto start = [&](int b) { return (int64_t)(a.row_start[b] / P) + 2 * b; };
  const int b = find_sequence(a.batch, blockIdx.x, start);
  const int r0 = a.row_start[b], n = min(a.row_start[b + 1], a.rows) - r0;
  if (r0 < 0 || n <= 0) return;
  const int slot0 = a.slots[r0];
  if (slot0 < 0) return;
  // rows [j, j + m) of the sequence go to one page, from offset off
  const int64_t chunk = blockIdx.x - start(b);
  const int lead = P - slot0 % P;  // rows that the first page still takes
  const int64_t j64 = chunk == 0 ? 0 : lead + (chunk - 1) * P;
  if (chunk < 0 || j64 >= n) return;
  const int j = (int)j64, m = min(n - j, chunk == 0 ? lead : P);
  const int slot = a.slots[r0 + j];
  const int page = slot / P, off = slot % P;
  if (slot < 0 || page >= a.c.n_pages || off + m > P) return;

  const int64_t stride = values ? a.v_stride : a.k_stride;
  const uint16_t* x = static_cast<const uint16_t*>(values ? a.v : a.k) + (int64_t)(r0 + j) * stride + (int64_t)head * DH;
  float amax = 0.f;
  for (int i = tid; i < m * kPieces; i += kAppendThreads) {
    const i32x4 w = ld16(x + (int64_t)(i / kPieces) * stride + (i % kPieces) * 8);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const f32x2 f = unpack2<T>((uint32_t)w[u]);
      amax = fmaxf(amax, fmaxf(finite_abs(f[0]), finite_abs(f[1])));
    }
  }
  int8_t* exp = (values ? a.c.v_exp : a.c.k_exp) + (int64_t)page * H + head;
  const int old = *exp;
  int e = block_exponent(block_max(amax));  // its barrier: every thread has read the old exponent
  if (off > 0) e = max(e, old);
  const bool grown = off > 0 && e > old;
  const float again = ldexpf(1.f, old - e), inv = pow2i(-e);
  if (tid == 0) *exp = (int8_t)e;

  uint8_t* codes = (values ? a.c.v_codes : a.c.k_codes) + ((int64_t)page * H + head) * P * DH;
  if (!values && grown)
    for (int i = tid; i < off * DH / 8; i += kAppendThreads) {
      i32x2 w = *(const i32x2*)(codes + 8 * i);
      w[0] = (int)rescale4((uint32_t)w[0], again);
      w[1] = (int)rescale4((uint32_t)w[1], again);
      *(i32x2*)(codes + 8 * i) = w;
    }
  for (int i = tid; i < m * kPieces; i += kAppendThreads) {
    const int row = i / kPieces, c = (i % kPieces) * 8;
    const i32x4 w = ld16(x + (int64_t)row * stride + c);
    float f[8];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const f32x2 g = unpack2<T>((uint32_t)w[u]);
      f[2 * u] = g[0] * inv;
      f[2 * u + 1] = g[1] * inv;
    }
    const uint32_t lo = to_e4m3x4(f[0], f[1], f[2], f[3]), hi = to_e4m3x4(f[4], f[5], f[6], f[7]);
    if (values) {
      *(uint32_t*)(tile + row * kLd + c) = lo;
      *(uint32_t*)(tile + row * kLd + c + 4) = hi;
    } else {
      *(i32x2*)(codes + (int64_t)(off + row) * DH + c) = i32x2{(int)lo, (int)hi};
    }
  }
  if (!values) return;
  __syncthreads();
  // 16 tokens of one dimension at a time; a piece that also holds kept or later codes is read first
  const int first = grown ? 0 : off / 16, last = (off + m + 15) / 16;
  const int pieces = last - first;
  for (int i = tid; i < pieces * DH; i += kAppendThreads) {
    const int d = i / pieces, t0 = (first + i % pieces) * 16;
    uint8_t* at = codes + (int64_t)d * P + t0;
    uint32_t w[4] = {0, 0, 0, 0};
    if (t0 < off || t0 + 16 > off + m) {
      const i32x4 v = ld16(at);
#pragma unroll
      for (int u = 0; u < 4; ++u) w[u] = (uint32_t)v[u];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (grown && t0 + 4 * u < off) {
        const uint32_t r = rescale4(w[u], again);
        const int keep = min(off - t0 - 4 * u, 4);
        const uint32_t mask = keep == 4 ? ~0u : (1u << (8 * keep)) - 1;
        w[u] = (w[u] & ~mask) | (r & mask);
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int row = t0 + 4 * u + v - off;
        if (row >= 0 && row < m) w[u] = (w[u] & ~(255u << (8 * v))) | ((uint32_t)tile[row * kLd + d] << (8 * v));
      }
    }
    *(i32x4*)at = i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
  }
}

hipError_t launch_paged_append(const AppendArgs& a, int dtype, hipStream_t s) {
  const dim3 grid((unsigned)(a.rows / a.c.page_size + 2 * a.batch), (unsigned)(2 * a.c.n_kv_heads));
  const size_t lds = (size_t)a.c.page_size * (a.c.head_dim + 4);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kAppendThreads), lds, s, a); };
  if (a.c.head_dim == 128)
    dtype == SBD_TYPE_BF16 ? go(append_kernel<Bf16, 128>) : go(append_kernel<Fp16, 128>);
  else
    dtype == SBD_TYPE_BF16 ? go(append_kernel<Bf16, 64>) : go(append_kernel<Fp16, 64>);
  return hipGetLastError();
}

}  // namespace sbd
