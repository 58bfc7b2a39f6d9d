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
// A step of few items is one launch of one workgroup, which keeps what the scans found in LDS (a
// chain of loads is all its time); larger ones take a launch for each phase.

constexpr int kPlanThreads = 1024;
constexpr int kPlanItems = 16 * kPlanThreads;  // table entries or rows that one workgroup takes

// What phase 1 leaves for the others, per sequence, in scratch or in LDS.
struct PlanView {
  int *take;    // [B] first new page, relative to base
  int *before;  // [B] pages held before taking
  int *back;    // [B + 1] scan of the pages given back, their number
  int *free0;   // free pages before the call
  int *row, *kv, *now, *cached;  // row_start, kv_len, held, cached
  int *base;                     // free pages afterwards
};

// Exclusive scans of two values over the workgroup, whose first n threads have some; totals in t.
__device__ void block_scan2(int64_t (&v)[2], int64_t (&t)[2], int n, int64_t (*waves)[2]) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = (min(n, kPlanThreads) + 63) / 64;
  int64_t s[2] = {v[0], v[1]};
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t u = __shfl_up(s[i], o);
      if (lane >= o) s[i] += u;
    }
  __syncthreads();  // waves[] may still be read from the scan before
  if (lane == 63) {
    waves[w][0] = s[0];
    waves[w][1] = s[1];
  }
  __syncthreads();
  int64_t before[2] = {0, 0};
  t[0] = t[1] = 0;
#pragma unroll 1
  for (int i = 0; i < nw; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (i < w) before[j] += waves[i][j];
      t[j] += waves[i][j];
    }
#pragma unroll
  for (int j = 0; j < 2; ++j) v[j] = before[j] + s[j] - v[j];
}

template <bool LDS>
__device__ void plan_scans(const PlanArgs& a, const PlanView& o) {
  __shared__ int64_t waves[kPlanThreads / 64][2];
  __shared__ int64_t s_taken;
  const sbd_page_table& t = a.t;
  const int B = t.batch, W = t.max_pages;
  const int free0 = min(max(*t.free_count, 0), t.n_pages);
  int64_t back = 0, v[2], total[2];
  if (a.release) {
    for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
      const int b = b0 + threadIdx.x;
      v[0] = (b < B && a.release[b]) ? min(max(t.held[b], 0), W) : 0;
      v[1] = 0;
      block_scan2(v, total, B - b0, waves);
      if (b < B) o.back[b] = (int)min(back + v[0], (int64_t)t.n_pages);
      back += total[0];
    }
  }
  const int given = (int)min(back, (int64_t)(t.n_pages - free0));
  const int avail = free0 + given;
  if (threadIdx.x == 0) s_taken = 0;
  int64_t sums[2] = {0, 0};
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
    v[0] = need;
    v[1] = max(n, 0);
    block_scan2(v, total, B - b0, waves);  // its barriers: s_taken is 0 now
    const int64_t at = sums[0] + v[0], row = sums[1] + v[1];
    sums[0] += total[0];
    sums[1] += total[1];
    const bool ok = fits && (need == 0 || at + need <= avail);
    // those served that need pages come first, so the last of them ends where all that is taken does
    if (ok && need > 0) atomicMax((unsigned long long*)&s_taken, (unsigned long long)(at + need));
    if (in) {
      o.take[b] = (int)min(at, (int64_t)t.n_pages);
      o.before[b] = held;
      const int rs = (int)min(row, (int64_t)INT32_MAX), kv = ok ? (int)tokens : 0, now = held + (ok ? need : 0);
      a.row_start[b] = rs;
      a.kv_len[b] = kv;
      t.held[b] = now;
      if (gone) t.cached[b] = 0;
      if (LDS) {
        o.row[b] = rs;
        o.kv[b] = kv;
        o.now[b] = now;
        o.cached[b] = cached;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const int rows = (int)min(sums[1], (int64_t)INT32_MAX);
    a.row_start[B] = rows;
    o.back[B] = given;
    *o.free0 = free0;
    const int left = avail - (int)s_taken;
    *t.free_count = left;
    if (LDS) {
      o.row[B] = rows;
      *o.base = left;
    }
  }
}

__device__ void plan_give_back(const PlanArgs& a, const PlanView& o, int64_t first, int64_t step) {
  const sbd_page_table& t = a.t;
  const int B = t.batch, n = o.back[B], free0 = *o.free0;
  for (int64_t i = first; i < n; i += step) {
    int lo = 0, hi = B;  // last sequence that starts at or before i (empty ones before it start there too)
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (o.back[mid] <= i) lo = mid; else hi = mid;
    }
    t.free_list[free0 + i] = t.table[(int64_t)lo * t.max_pages + min((int)i - o.back[lo], t.max_pages - 1)];
  }
}

__device__ void plan_tables(const PlanArgs& a, const PlanView& o, int64_t first, int64_t step) {
  const sbd_page_table& t = a.t;
  const int B = t.batch, W = t.max_pages, base = *o.base;
  auto free_page = [&](int b, int col, int held) {
    return t.free_list[min(max(base + o.take[b] + col - held, 0), t.n_pages - 1)];
  };
  for (int64_t i = first; i < (int64_t)B * W; i += step) {
    const int b = (int)((uint64_t)i / (unsigned)W), col = (int)(i - (int64_t)b * W);
    const int held = o.before[b], now = o.now[b];
    if (col >= held && col < now)
      t.table[i] = free_page(b, col, held);
    else if (col >= now && a.release && a.release[b])
      t.table[i] = -1;
  }
  const int rows = o.row[B], pshift = 31 - __builtin_clz(t.page_size);
  for (int64_t r = first; r < a.rows; r += step) {
    int slot = -1;
    if (r < rows) {
      int lo = 0, hi = B;  // last sequence that starts at or before r: it is not an empty one
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (o.row[mid] <= r) lo = mid; else hi = mid;
      }
      if (o.kv[lo] > 0) {
        const int p = o.cached[lo] + (int)r - o.row[lo], col = p >> pshift, held = o.before[lo];
        const int page = col < held ? t.table[(int64_t)lo * W + col] : free_page(lo, col, held);
        if (page >= 0 && page < t.n_pages) slot = (page << pshift) + (p & (t.page_size - 1));
      }
    }
    a.slots[r] = slot;
  }
}

__global__ __launch_bounds__(kPlanThreads) void plan_all_kernel(PlanArgs a) {
  __shared__ int s[7 * kPlanThreads + 4];  // at most kPlanThreads sequences
  constexpr int N = kPlanThreads;
  const PlanView o{s, s + N, s + 2 * N, s + 7 * N + 2, s + 3 * N + 1, s + 4 * N + 2, s + 5 * N + 2, s + 6 * N + 2, s + 7 * N + 3};
  plan_scans<true>(a, o);
  __syncthreads();
  if (a.release) {
    plan_give_back(a, o, threadIdx.x, kPlanThreads);
    __syncthreads();
  }
  plan_tables(a, o, threadIdx.x, kPlanThreads);
}

__device__ PlanView scratch_view(const PlanArgs& a) {
  const int B = a.t.batch;
  return PlanView{a.scratch, a.scratch + B, a.scratch + 2 * B, a.scratch + 3 * B + 1,
                  a.row_start, a.kv_len, a.t.held, a.t.cached, a.t.free_count};
}
__global__ __launch_bounds__(kPlanThreads) void plan_scans_kernel(PlanArgs a) { plan_scans<false>(a, scratch_view(a)); }
__global__ __launch_bounds__(256) void plan_give_back_kernel(PlanArgs a) {
  plan_give_back(a, scratch_view(a), (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}
__global__ __launch_bounds__(256) void plan_tables_kernel(PlanArgs a) {
  plan_tables(a, scratch_view(a), (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

hipError_t launch_paged_plan(const PlanArgs& a, hipStream_t s) {
  const int64_t items = std::max<int64_t>((int64_t)a.t.batch * a.t.max_pages, a.rows);
  if (items <= kPlanItems && a.t.batch <= kPlanThreads) {
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
  // Few dependent reads, since they are most of a small step's time: what is known about up to 64
  // sequences is read before it is known which of them it is, and the rows before their page is.
  auto start = [&](int r0, int b) { return (int64_t)(r0 / P) + 2 * b; };
  int lo = 0, nb = a.batch;
  narrow_sequence(lo, nb, blockIdx.x, [&](int b) { return start(a.row_start[b], b); });
  const int lane = tid & 63, b = lo + min(lane, nb - 1);
  const int from = a.row_start[b], to = min(a.row_start[b + 1], a.rows);
  const int c = max(1, (int)__popcll(__ballot(lane < nb && start(from, b) <= (int64_t)blockIdx.x))) - 1;
  const int r0 = __builtin_amdgcn_readlane(from, c), n = __builtin_amdgcn_readlane(to, c) - r0;
  if (r0 < 0 || n <= 0) return;
  const int slot0 = a.slots[r0];
  if (slot0 < 0) return;
  // rows [j, j + m) of the sequence go to one page, from offset off
  const int64_t chunk = blockIdx.x - start(r0, lo + c);
  const int lead = P - slot0 % P;  // rows that the first page still takes
  const int64_t j64 = chunk == 0 ? 0 : lead + (chunk - 1) * P;
  if (chunk < 0 || j64 >= n) return;
  const int j = (int)j64, m = min(n - j, chunk == 0 ? lead : P);
  const int slot = chunk == 0 ? slot0 : a.slots[r0 + j];

  const int64_t stride = values ? a.v_stride : a.k_stride;
  const uint16_t* x = static_cast<const uint16_t*>(values ? a.v : a.k) + (int64_t)(r0 + j) * stride + (int64_t)head * DH;
  // A thread's first kHold pieces of 8 elements (all of them up to 64 rows of 128) stay in
  // registers between the exponent and the codes.
  constexpr int kHold = 4;
  i32x4 hold[kHold];
  float amax = 0.f;
  auto piece = [&](int i) { return ld16(x + (int64_t)(i / kPieces) * stride + (i % kPieces) * 8); };
#pragma unroll
  for (int h = 0; h < kHold; ++h)
    if (tid + h * kAppendThreads < m * kPieces) hold[h] = piece(tid + h * kAppendThreads);
  const int page = slot / P, off = slot % P;
  if (slot < 0 || page >= a.c.n_pages || off + m > P) return;
  int8_t* exp = (values ? a.c.v_exp : a.c.k_exp) + (int64_t)page * H + head;
  const int old = off > 0 ? *exp : 0;
  auto largest = [&](i32x4 w) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const f32x2 f = unpack2<T>((uint32_t)w[u]);
      amax = fmaxf(amax, fmaxf(finite_abs(f[0]), finite_abs(f[1])));
    }
  };
#pragma unroll
  for (int h = 0; h < kHold; ++h)
    if (tid + h * kAppendThreads < m * kPieces) largest(hold[h]);
  for (int i = tid + kHold * kAppendThreads; i < m * kPieces; i += kAppendThreads) largest(piece(i));
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
  auto encode = [&](int i, i32x4 w) {
    const int row = i / kPieces, c = (i % kPieces) * 8;
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
  };
#pragma unroll
  for (int h = 0; h < kHold; ++h)
    if (tid + h * kAppendThreads < m * kPieces) encode(tid + h * kAppendThreads, hold[h]);
  for (int i = tid + kHold * kAppendThreads; i < m * kPieces; i += kAppendThreads) encode(i, piece(i));
  if (!values) return;
  __syncthreads();
  // Pieces of 16 tokens that are all new: four dimensions at a time, turned around in registers.
  const int new0 = (off + 15) / 16, new1 = max(new0, (off + m) / 16), whole = new1 - new0;
  for (int i = tid; i < whole * (DH / 4); i += kAppendThreads) {
    const int d = i / whole * 4, t0 = (new0 + i % whole) * 16;
    const uint8_t* from = tile + (t0 - off) * kLd + d;
    i32x4 out[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint32_t r[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) r[v] = *(const uint32_t*)(from + (4 * u + v) * kLd);
      const uint32_t lo0 = __builtin_amdgcn_perm(r[1], r[0], 0x05010400), hi0 = __builtin_amdgcn_perm(r[1], r[0], 0x07030602);
      const uint32_t lo1 = __builtin_amdgcn_perm(r[3], r[2], 0x05010400), hi1 = __builtin_amdgcn_perm(r[3], r[2], 0x07030602);
      out[0][u] = (int)__builtin_amdgcn_perm(lo1, lo0, 0x05040100);
      out[1][u] = (int)__builtin_amdgcn_perm(lo1, lo0, 0x07060302);
      out[2][u] = (int)__builtin_amdgcn_perm(hi1, hi0, 0x05040100);
      out[3][u] = (int)__builtin_amdgcn_perm(hi1, hi0, 0x07060302);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) *(i32x4*)(codes + (int64_t)(d + v) * P + t0) = out[v];
  }
  // The others also hold kept or later codes (kept ones are all visited where their scale grew):
  // one dimension at a time, read first.
  const int first = grown ? 0 : off / 16, last = (off + m + 15) / 16, rest = last - first - whole;
  for (int i = tid; i < rest * DH; i += kAppendThreads) {
    const int d = i / rest, q = first + i % rest, t0 = (q < new0 ? q : q + whole) * 16;
    uint8_t* at = codes + (int64_t)d * P + t0;
    const i32x4 old = ld16(at);
    uint32_t w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      w[u] = (uint32_t)old[u];
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
