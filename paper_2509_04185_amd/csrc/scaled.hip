// Block-scaled e4m3: the quantiser (sbd_scaled_quantize) and the product (sbd_scaled_matmul).

#include "ops_device.h"

namespace sbd {

// ---- quantiser --------------------------------------------------------------------------

// Eight consecutive elements as floats.
template <class T>
__device__ __forceinline__ void load8(const void* x, int64_t at, float (&f)[8]) {
  if constexpr (std::is_same_v<T, float>) {
    const f32x4 a = *(const f32x4*)(static_cast<const float*>(x) + at), b = *(const f32x4*)(static_cast<const float*>(x) + at + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = a[i];
      f[4 + i] = b[i];
    }
  } else {
    const i32x4 w = ld16(static_cast<const uint16_t*>(x) + at);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const f32x2 g = unpack2<T>((uint32_t)w[u]);
      f[2 * u] = g[0];
      f[2 * u + 1] = g[1];
    }
  }
}

__device__ __forceinline__ float max8(const float (&f)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(f[i]));
  return m;
}
__device__ __forceinline__ i32x2 codes8(const float (&f)[8], float inv) {
  return i32x2{(int)to_e4m3x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv),
               (int)to_e4m3x4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv)};
}

// The codes are not read again by this kernel: stores that leave the caches to the reads (28672 x
// 4096 in tiles: 74 us without, 68 with; reads that do so too: 67).
__device__ __forceinline__ void store_codes(const QuantizeArgs& a, int row, int col, i32x2 v) {
  __builtin_nontemporal_store(v, (i32x2*)(a.codes + (int64_t)row * a.cols + col));
}

// A scale for each row and 128 columns: 16 lanes hold such a block, 8 elements each.  A workgroup
// has 16 rows, so that it stores 16 neighbouring scales of a block of columns, and U blocks.
template <class T, int U>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeArgs a, int across) {
  const int row = (int)(blockIdx.x / across) * 16 + (threadIdx.x >> 4), kb = (a.cols + 127) / 128;
  const int c0 = (int)(blockIdx.x % across) * U;
  if (row >= a.rows) return;  // whole groups of 16 lanes
  float f[U][8] = {};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int col = 128 * (c0 + u) + 8 * (threadIdx.x & 15);
    if (col < a.cols) load8<T>(a.x, row * a.x_stride + col, f[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u, col = 128 * c + 8 * (threadIdx.x & 15);
    float m = max8(f[u]);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    const int e = block_exponent(m);
    if (col < a.cols) store_codes(a, row, col, codes8(f[u], pow2i(-e)));
    if ((threadIdx.x & 15) == 0 && c < kb) a.scales[(int64_t)c * a.rows + row] = pow2i(e);
  }
}

// A scale for each 128 x 128 block: one workgroup each, 64 elements a thread.
template <class T>
__global__ __launch_bounds__(256) void quantize_tiles_kernel(QuantizeArgs a) {
  __shared__ float waves[4];
  const int kb = (a.cols + 127) / 128;
  const int rb = (int)(blockIdx.x / kb), c = (int)(blockIdx.x % kb), col = 128 * c + 8 * (threadIdx.x & 15);
  float f[8][8] = {};
  float m = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int row = 128 * rb + 16 * u + (threadIdx.x >> 4);
    if (row < a.rows && col < a.cols) load8<T>(a.x, row * a.x_stride + col, f[u]);
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) m = fmaxf(m, max8(f[u]));
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = m;
  __syncthreads();
  const int e = block_exponent(fmaxf(fmaxf(waves[0], waves[1]), fmaxf(waves[2], waves[3])));
  const float inv = pow2i(-e);
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int row = 128 * rb + 16 * u + (threadIdx.x >> 4);
    if (row < a.rows && col < a.cols) store_codes(a, row, col, codes8(f[u], inv));
  }
  if (threadIdx.x == 0) a.scales[blockIdx.x] = pow2i(e);
}

template <class T>
static hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t s) {
  const int kb = (a.cols + 127) / 128, tiles = (a.rows + 15) / 16;
  if (a.block_rows == 128) {
    const int64_t grid = (int64_t)(a.rows + 127) / 128 * kb;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(quantize_tiles_kernel<T>, dim3((unsigned)grid), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  // two blocks a workgroup where there are enough to fill the chip (28672 x 4096: 63 us, one block 73)
  const int u = (int64_t)tiles * kb >= 8192 ? 2 : 1, across = (kb + u - 1) / u;
  const int64_t grid = (int64_t)tiles * across;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (u == 2)
    hipLaunchKernelGGL((quantize_rows_kernel<T, 2>), dim3((unsigned)grid), dim3(256), 0, s, a, across);
  else
    hipLaunchKernelGGL((quantize_rows_kernel<T, 1>), dim3((unsigned)grid), dim3(256), 0, s, a, across);
  return hipGetLastError();
}

hipError_t launch_scaled_quantize(const QuantizeArgs& a, int dtype, hipStream_t s) {
  switch (dtype) {
    case SBD_TYPE_BF16: return launch_quantize<Bf16>(a, s);
    case SBD_TYPE_FP16: return launch_quantize<Fp16>(a, s);
    default: return launch_quantize<float>(a, s);
  }
}

// ---- product ----------------------------------------------------------------------------
//
// A block of 128 along K is summed by the matrix unit from zero, multiplied by the block's
// scales and added to fp32 sums in registers.  The weights (b) are the A operand, so lane
// (r, grp) of a result holds out row r and four neighbouring columns 4 grp + i: a_scale is one
// value a lane and b_scale one value a wave.  Both operands use the same order of k: lane group
// grp holds k = 64 p + 16 grp .. + 16, p = 0, 1, of a block.
//
// 16-bit outputs: one 16x16x128 e4m3 instruction a block.  It aligns groups of eight
// neighbouring products to the largest and keeps 14 bits of it (measured: 2^16 + 2^3 is exact,
// 2^16 + 2^2 gives 2^16; between groups the sums are fp32), far below the rounding of the
// result.  fp32 outputs: the codes are widened to bf16 (exact) for four 16x16x32 instructions,
// whose sums are fp32 throughout, at half the rate.

template <bool WIDE>
__device__ __forceinline__ f32x4 block_product(i32x8 a, i32x8 b) {
  if constexpr (!WIDE) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
  } else {
    f32x4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < 4; ++p)
      c = mfma16<Bf16>(e4m3x8_to_bf16(i32x2{a[2 * p], a[2 * p + 1]}, 1.f), e4m3x8_to_bf16(i32x2{b[2 * p], b[2 * p + 1]}, 1.f), c);
    return c;
  }
}

__device__ __forceinline__ i32x8 join8(i32x4 lo, i32x4 hi) {
  return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}
// This lane's fragment of block c of 16 rows of k codes (zeros behind their end), lane group grp
// holding k = 32 grp .. + 32 here.  The lanes of a pair first read 32 neighbouring bytes of the
// even row, then of the odd one, and swap halves: a lane that read its own row's pieces would have
// a neighbour in another row, and the vector cache would be asked for 16 bytes at a time.
struct RowPair {
  const uint8_t *even, *odd;  // this lane's pair of rows, its piece of block 0
};
__device__ __forceinline__ RowPair row_pair(const uint8_t* base, int64_t stride, int first, int rows) {
  const int lane = threadIdx.x & 63, r = lane & 15, grp = lane >> 4, piece = 32 * grp + 16 * (r & 1);
  return RowPair{base + min(first + (r & ~1), rows - 1) * stride + piece, base + min(first + (r | 1), rows - 1) * stride + piece};
}
__device__ __forceinline__ i32x8 load_frag(RowPair p, int c, int k) {
  const int lane = threadIdx.x & 63, k0 = 128 * c + 32 * (lane >> 4) + 16 * (lane & 1);
  i32x4 a{0, 0, 0, 0}, b = a, lo, hi;
  if (k0 < k) {
    a = ld16(p.even + 128 * c);
    b = ld16(p.odd + 128 * c);
  }
  const bool odd = lane & 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int sa = __builtin_amdgcn_mov_dpp(a[i], 0xb1, 0xf, 0xf, true), sb = __builtin_amdgcn_mov_dpp(b[i], 0xb1, 0xf, 0xf, true);
    lo[i] = odd ? sb : a[i];
    hi[i] = odd ? b[i] : sa;
  }
  return join8(lo, hi);
}

// Vectors at addresses that are aligned to their elements only (the memory unit takes them so).
typedef f32x4 __attribute__((aligned(4))) f32x4_any;
typedef i32x4 __attribute__((aligned(2))) i32x4_any;
typedef i32x2 __attribute__((aligned(2))) i32x2_any;

template <class T>
__device__ __forceinline__ void store4(void* out, int64_t at, int n_left, f32x4 v) {
  if constexpr (std::is_same_v<T, float>) {
    float* p = static_cast<float*>(out) + at;
    if (n_left >= 4) {
      *(f32x4_any*)p = v;
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < n_left) p[i] = v[i];
    }
  } else {
    uint16_t* p = static_cast<uint16_t*>(out) + at;
    const uint32_t lo = pack2<T>(v[0], v[1]), hi = pack2<T>(v[2], v[3]);
    if (n_left >= 4) {
      *(i32x2_any*)p = i32x2{(int)lo, (int)hi};
    } else {
      if (n_left > 0) p[0] = (uint16_t)lo;
      if (n_left > 1) p[1] = (uint16_t)(lo >> 16);
      if (n_left > 2) p[2] = (uint16_t)hi;
    }
  }
}

// At most 16 MT rows: the weights' bytes are all there is.  A workgroup makes 16 NT columns of
// all rows; its KW waves take the blocks of K in turn and are joined through LDS.  Other waves of
// the CU hide the latency: two blocks a wave in flight take registers from them and are slower
// (16 x 114688 x 4096: 94 us, 5.0 TB/s, with one, 107 us with two, 141 us with four).
template <class T, int MT, int NT, int KW>
__global__ __launch_bounds__(64 * KW) void skinny_kernel(MatmulArgs a) {
  constexpr bool WIDE = std::is_same_v<T, float>;
  __shared__ f32x4 s_acc[KW][MT * NT][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, grp = lane >> 4;
  const int kb = (a.k + 127) / 128, n0 = blockIdx.x * 16 * NT;
  RowPair xr[MT], wr[NT];
  int m[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    m[t] = min(16 * t + r, a.m - 1);
    xr[t] = row_pair(a.a, a.a_stride, 16 * t, a.m);
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) wr[t] = row_pair(a.b, a.k, n0 + 16 * t, a.n);
  const float* sb = a.b_scale + (int64_t)(n0 / 128) * kb;
  f32x4 acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int c = w; c < kb; c += KW) {
    i32x8 wf[NT], xf[MT];
    float sc[MT];
#pragma unroll
    for (int i = 0; i < NT; ++i) wf[i] = load_frag(wr[i], c, a.k);
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      xf[j] = load_frag(xr[j], c, a.k);
      sc[j] = a.a_scale[(int64_t)c * a.m + m[j]] * sb[c];
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < MT; ++j) acc[i][j] += block_product<WIDE>(wf[i], xf[j]) * sc[j];
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) s_acc[w][i * MT + j][lane] = acc[i][j];
  __syncthreads();
  // one wave a 16 x 16 tile, the others' sums added in order
  for (int t = w; t < MT * NT; t += KW) {
    f32x4 v = s_acc[0][t][lane];
#pragma unroll
    for (int u = 1; u < KW; ++u) v += s_acc[u][t][lane];
    const int row = 16 * (t % MT) + r, n = n0 + 16 * (t / MT) + 4 * grp;
    if (row < a.m) store4<T>(a.out, row * a.out_stride + n, a.n - n, v);
  }
}

// More rows: tiles of 16 MT MW rows x 16 NT NW columns, MW x NW waves.  The codes of both go
// through LDS, copied there straight from memory into one of two buffers while the other is
// multiplied.  (A wave's weights straight into its registers would save a third of the LDS
// reads, but a fragment's neighbouring lanes lie in different rows, so the vector cache is
// asked for 16 bytes at a time: 4096 x 28672 x 4096 took 700 us that way.)  LDS holds rows of
// 128 bytes whose 16-byte pieces are XOR-swizzled with the row, so that the 16 rows of a
// fragment read spread over all banks.
//
// The copies are written as assembly without results: the compiler would otherwise wait for
// every copy in flight before each read of LDS.  A wave waits for its copies once a block,
// before the barrier.
__device__ __forceinline__ void copy16_to_lds(__amdgpu_buffer_rsrc_t rsrc, uint32_t lds, uint32_t voff, uint32_t soff) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %1, %2, %3 offen lds"
      :
      : "s"(lds), "v"(voff), "s"(rsrc), "s"(soff)
      : "memory", "m0");
}

__device__ __forceinline__ void copy4_to_lds(__amdgpu_buffer_rsrc_t rsrc, uint32_t lds, uint32_t voff, uint32_t soff) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dword %1, %2, %3 offen lds"
      :
      : "s"(lds), "v"(voff), "s"(rsrc), "s"(soff)
      : "memory", "m0");
}

template <int MT, int NT, int MW, int NW>
struct TileShape {
  static constexpr int kWaves = MW * NW, kThreads = 64 * kWaves;
  static constexpr int BM = 16 * MT * MW, BN = 16 * NT * NW;
  static constexpr int kCopies = (BM + BN) / 8 / kWaves;  // 1 KB copies (8 rows) of a wave and block
  static_assert(kCopies * 8 * kWaves == BM + BN && BM % (8 * kWaves) == 0, "whole copies, of one operand each");
};

template <class T, int MT, int NT, int MW, int NW, bool SPLIT>
__global__ __launch_bounds__(64 * MW * NW, MW * NW >= 8 ? 1 : 2) void tile_kernel(MatmulArgs a, int tiles_m, int tiles_n,
                                                                                 int blocks_per_split) {
  using S = TileShape<MT, NT, MW, NW>;
  constexpr bool WIDE = std::is_same_v<T, float>;
  // 1 KB pieces of 8 rows, the two buffers' in turn; rows, then weights
  __shared__ __attribute__((aligned(1024))) uint8_t s_x[(S::BM + S::BN) * 256];
  __shared__ float s_s[2][S::BM], s_b[2][S::kWaves][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, grp = lane >> 4;
  const int mw = w % MW, nw = w / MW;
  const int kb = (a.k + 127) / 128;

  // Workgroup i runs on XCD i % 8: each XCD gets a run of neighbouring tiles, walked in groups
  // of 8 rows of tiles, so that what runs at once on an XCD shares rows and weights in its L2.
  const int tiles = tiles_m * tiles_n;
  int id = blockIdx.x;
  {
    const int per = tiles / 8, more = tiles % 8, x = id % 8;
    id = x * per + min(x, more) + id / 8;
  }
  const int group = id / (8 * tiles_n), first = group * 8, rows_in = min(8, tiles_m - first);
  const int tm = first + (id - group * 8 * tiles_n) % rows_in, tn = (id - group * 8 * tiles_n) / rows_in;
  const int m0 = tm * S::BM, n0 = tn * S::BN;
  const int c0 = SPLIT ? blockIdx.y * blocks_per_split : 0, c1 = SPLIT ? min(c0 + blocks_per_split, kb) : kb;

  // Copies: lane l brings piece (l % 8) ^ (l / 8) of row l / 8 of eight.  Rows behind the last
  // one are outside the buffer's range by the lane's own offset (row * stride is at least its
  // size): the hardware does not read them, and what stands for them is not stored.  Each wave also brings the scales of 64 rows (some waves the same ones) and the
  // weights' scale of its columns.
  constexpr int kRowCopies = S::BM / 8 / S::kWaves;
  auto rows_of = [](const uint8_t* p, int64_t rows, int64_t stride, int64_t width) {
    const int64_t bytes = min((rows - 1) * stride + width, (int64_t)0x7fffffff);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0, (int)bytes, 0x00020000);
  };
  const __amdgpu_buffer_rsrc_t rx = rows_of(a.a + m0 * a.a_stride, min(a.m - m0, S::BM), a.a_stride, a.k);
  const __amdgpu_buffer_rsrc_t rw = rows_of(a.b + (int64_t)n0 * a.k, min(a.n - n0, S::BN), a.k, a.k);
  const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
  const uint32_t off_x = (lane >> 3) * (uint32_t)a.a_stride + piece, off_w = (lane >> 3) * (uint32_t)a.k + piece;
  const int srow = w % (S::BM / 64) * 64;
  const uint32_t off_s = (uint32_t)min(m0 + srow + lane, a.m - 1) * 4;
  const __amdgpu_buffer_rsrc_t rb = buf_rsrc(a.b_scale + (int64_t)min((n0 + 16 * NT * nw) / 128, (a.n - 1) / 128) * kb);
  // Copies u0 .. u1 of a block (all of them: kCopies; the scales come with the first).
  auto copy_some = [&](int c, int buf, auto tail, int u0, int u1) {
    const uint32_t lds = lds_addr(s_x) + buf * 1024;
    // in the last block, pieces behind its end are read from inside the row (and not used)
    const uint32_t over = tail ? (uint32_t)max(0, 128 * c + piece - (a.k - 16)) : 0;
#pragma unroll
    for (int u = u0; u < u1; ++u) {
      const int q = w + S::kWaves * u, row = 8 * (u < kRowCopies ? q : q - S::BM / 8);
      const uint32_t at = (uint32_t)row * (uint32_t)(u < kRowCopies ? a.a_stride : a.k);
      copy16_to_lds(u < kRowCopies ? rx : rw, __builtin_amdgcn_readfirstlane(lds + q * 2048),
                    (u < kRowCopies ? off_x : off_w) - over + at, 128 * c);
    }
    if (u0 > 0) return;
    copy4_to_lds(buf_rsrc(a.a_scale + (int64_t)c * a.m), __builtin_amdgcn_readfirstlane(lds_addr(s_s[buf]) + srow * 4), off_s, 0);
    copy4_to_lds(rb, __builtin_amdgcn_readfirstlane(lds_addr(s_b[buf][w])), 0, 4 * c);
  };

  f32x4 acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const uint32_t lane_at = (r >> 3) * 2048 + (r & 7) * 128 + (grp ^ (r & 7)) * 16;
  const uint32_t frag_x = 2 * MT * mw * 2048 + lane_at, frag_w = (S::BM / 8 + 2 * NT * nw) * 2048 + lane_at;
  // A fragment piece of the last block is there if it is not behind its end; pieces are whole.
  const bool lo_in = 128 * (kb - 1) + 16 * grp < a.k, hi_in = 128 * (kb - 1) + 64 + 16 * grp < a.k;
  const i32x4 zero{0, 0, 0, 0};
  auto read_frag = [&](uint32_t at, uint32_t more, auto tail) {
    i32x4 lo = *(const i32x4*)(s_x + at + more), hi = *(const i32x4*)(s_x + (at ^ 64) + more);
    if (tail) {
      if (!lo_in) lo = zero;
      if (!hi_in) hi = zero;
    }
    return join8(lo, hi);
  };
  const std::integral_constant<bool, false> whole;
  const std::integral_constant<bool, true> part;
  auto wait_all = [] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(7 << 4);  // vmcnt(0), lgkmcnt(0): this wave's copies have landed, its reads are done
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // What a step begins with: the weights' fragments, the first row fragment and their scales.
  struct Begin {
    i32x8 f[NT], x;
    float sx, sb;
  };
  auto read_begin = [&](int buf, Begin& b, auto tail) {
    b.x = read_frag(frag_x, buf * 1024, tail);
    b.sx = s_s[buf][16 * MT * mw + r];
    b.sb = s_b[buf][w][0];
#pragma unroll
    for (int i = 0; i < NT; ++i) b.f[i] = read_frag(frag_w, buf * 1024 + 4096 * i, tail);
  };
  // One block.  The products of a fragment are issued one after the other; while one runs, the
  // sums take in the one before it and the next fragment is read.  When the last row fragment
  // is there (its own products are still to come) turn() passes the barrier at which every wave
  // is done with this buffer and the next block has landed in the other.
  auto step = [&](int buf, const Begin& b, auto tail, auto&& fill, auto&& turn) {
    i32x8 x = b.x, x_next = x;
    float scale = b.sx, scale_next = 0.f;
    f32x4 before;
    float before_scale = 0.f;
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      if (j + 1 < MT) {
        x_next = read_frag(frag_x, buf * 1024 + 4096 * (j + 1), tail);
        scale_next = s_s[buf][16 * (MT * mw + j + 1) + r];
      }
      if (j < MT / 2) fill(j);
      if (j == MT - 1) turn();
      const float f0 = scale * b.sb;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const f32x4 p = block_product<WIDE>(b.f[i], x);
        __builtin_amdgcn_sched_barrier(0);
        const int was = j * NT + i - 1;
        if (was >= 0) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            acc[was % NT][was / NT][q] = __builtin_fmaf(before[q], before_scale, acc[was % NT][was / NT][q]);
        }
        before = p;
        before_scale = f0;
        __builtin_amdgcn_sched_barrier(0);
      }
      x = x_next;
      scale = scale_next;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[NT - 1][MT - 1][q] = __builtin_fmaf(before[q], before_scale, acc[NT - 1][MT - 1][q]);
  };

  // Whole blocks (the last one is brought again where there is no next), then the last part.
  // A block's copies are spread over the first half of the step before it: issued at once they
  // fill the queue of the vector memory unit and every wave waits there.
  const int cf = min(c1, a.k / 128);
  if (c0 < cf) {
    Begin b0, b1;
    constexpr int kEach = (S::kCopies + MT / 2 - 1) / (MT / 2);
    auto fill = [&](int c, int buf, int j) {
      copy_some(min(c, cf - 1), buf, whole, min(kEach * j, S::kCopies), min(kEach * (j + 1), S::kCopies));
    };
    copy_some(c0, 0, whole, 0, S::kCopies);
    wait_all();
    read_begin(0, b0, whole);
    for (int c = c0;; c += 2) {
      step(0, b0, whole, [&](int j) { fill(c + 1, 1, j); }, [&] {
        wait_all();
        read_begin(1, b1, whole);
      });
      if (c + 1 >= cf) break;
      step(1, b1, whole, [&](int j) { fill(c + 2, 0, j); }, [&] {
        wait_all();
        read_begin(0, b0, whole);
      });
      if (c + 2 >= cf) break;
    }
    wait_all();
  }
  if (cf < c1) {
    Begin b;
    copy_some(cf, 0, part, 0, S::kCopies);
    wait_all();
    read_begin(0, b, part);
    step(0, b, part, [](int) {}, [] {});
  }

  // Each wave turns its sums around in a part of LDS of its own, so that it stores whole lines
  // (4096 x 28672 x 4096: 517 us when measured, 543 with 8-byte pieces straight from the registers).
  using E = std::conditional_t<SPLIT, float, T>;
  constexpr int ES = std::is_same_v<E, float> ? 4 : 2, kWidth = 16 * NT * ES, kPieces = kWidth / 16;
  static_assert(S::BM * S::BN * ES <= (int)sizeof(s_x), "the sums fit the buffers");
  __syncthreads();  // every wave is done with the buffers
  uint8_t* turn = s_x + w * 16 * MT * kWidth;
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int row = 16 * j + r;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int byte = (16 * i + 4 * grp) * ES, at = row * kWidth + (((byte / 16) ^ (row % kPieces)) * 16) + byte % 16;
      const f32x4 v = acc[i][j];
      if constexpr (ES == 4)
        *(f32x4*)(turn + at) = v;
      else
        *(i32x2*)(turn + at) = i32x2{(int)pack2<E>(v[0], v[1]), (int)pack2<E>(v[2], v[3])};
    }
  }
  __builtin_amdgcn_s_waitcnt((15 | (3 << 14)) | (7 << 4));  // lgkmcnt(0): only this wave reads what it wrote
  asm volatile("" ::: "memory");
  uint8_t* out = static_cast<uint8_t*>(SPLIT ? static_cast<void*>(a.part + (int64_t)blockIdx.y * a.m * a.n) : a.out);
  const int64_t stride = SPLIT ? a.n : a.out_stride;
  constexpr int kRows = 64 / kPieces, kEls = 16 / ES;
  const int p = lane % kPieces, n = n0 + 16 * NT * nw + p * kEls;
#pragma unroll
  for (int u = 0; u < 16 * MT / kRows; ++u) {
    const int row = u * kRows + lane / kPieces, m = m0 + 16 * MT * mw + row;
    const i32x4 v = *(const i32x4*)(turn + row * kWidth + ((p ^ (row % kPieces)) * 16));
    if (m >= a.m || n >= a.n) continue;
    uint8_t* at = out + (m * stride + n) * ES;
    if (n + kEls <= a.n) {
      *(i32x4_any*)at = v;
    } else {
#pragma unroll
      for (int e = 0; e < kEls - 1; ++e) {
        if (n + e >= a.n) break;
        if constexpr (ES == 4)
          *(int*)(at + 4 * e) = v[e];
        else
          *(uint16_t*)(at + 2 * e) = (uint16_t)((uint32_t)v[e / 2] >> (16 * (e % 2)));
      }
    }
  }
}

// Sum of the K parts, in order.
template <class T>
__global__ __launch_bounds__(256) void join_splits_kernel(MatmulArgs a, int splits) {
  const int64_t quads = (a.n + 3) / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= quads * a.m) return;
  const int row = (int)(i / quads), n = (int)(i % quads) * 4, left = a.n - n;
  const int64_t size = (int64_t)a.m * a.n;
  const float* p = a.part + (int64_t)row * a.n + n;
  f32x4 v{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s, p += size) {
    if (left >= 4) {
      v += *(const f32x4_any*)p;
    } else {
#pragma unroll
      for (int q = 0; q < 3; ++q)
        if (q < left) v[q] += p[q];
    }
  }
  store4<T>(a.out, row * a.out_stride + n, left, v);
}

// How a product is cut.  Fewer tiles than CUs are split along K to two workgroups a CU (203 x 4096 x
// 14336 in bf16, 128 tiles: 31 us with four parts, 44 with two, 35 with eight); from 256 tiles on the
// join costs more than it gives (1024 x 4096 x 4096: 29.5 us in one part, 34.5 in two).
struct MatmulPlan {
  enum { kSkinny, kSmall, kMedium, kLarge } kind;
  int tiles_m, tiles_n, splits, blocks_per_split;
};

static MatmulPlan matmul_plan(int m, int n, int k, bool wide) {
  MatmulPlan p{};
  const int kb = (k + 127) / 128;
  // The first kernel and tiles: 32 x 4096 x 4096 6.3 and 10.7 us, 32 x 28672 x 4096 35 and 23.5; 64 x
  // 4096 x 4096 10.2 and 13.0, 64 x 6144 x 4096 19 and 15, 40 x 4096 x 14336 30 and 20.
  if (m <= 16 || (m <= 32 && n <= 8192) || (m <= 64 && n <= 4096 && k <= 4096)) {
    p.kind = MatmulPlan::kSkinny;
    p.splits = 1;
    return p;
  }
  auto tiles = [&](int bm, int bn) { return (int64_t)((m + bm - 1) / bm) * ((n + bn - 1) / bn); };
  int bm, bn;
  // 256 x 256 where their rounds over the CUs are at least 5/8 full: 4096 x 6144 x 4096 (3/4) 124 us,
  // 149 with 128 x 128; 2560 x 7168 x 4096 (0.55) 113 and 114; 2529 x 6454 x 320 (0.49) 25.5 and 19.5.
  const int64_t round = (int64_t)256 * 256 * 256, rounds = (tiles(256, 256) + 255) / 256;
  if (!wide && (int64_t)m * n >= rounds * round / 8 * 5) {
    p.kind = MatmulPlan::kLarge;
    bm = bn = 256;
  } else if (m > 64 && tiles(128, 128) >= 128) {
    p.kind = MatmulPlan::kMedium;
    bm = bn = 128;
  } else {
    p.kind = MatmulPlan::kSmall;
    bm = 64;
    bn = 128;
  }
  p.tiles_m = (m + bm - 1) / bm;
  p.tiles_n = (n + bn - 1) / bn;
  const int64_t t = (int64_t)p.tiles_m * p.tiles_n;
  p.splits = t >= 256 || p.kind == MatmulPlan::kLarge ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({512 / t, kb / 4, 16}));
  p.blocks_per_split = (kb + p.splits - 1) / p.splits;
  p.splits = (kb + p.blocks_per_split - 1) / p.blocks_per_split;
  return p;
}

size_t scaled_matmul_bytes(int m, int n, int k) {
  const int s = std::max(matmul_plan(m, n, k, false).splits, matmul_plan(m, n, k, true).splits);
  return s > 1 ? (size_t)s * m * n * sizeof(float) : 0;
}

template <class T>
static hipError_t launch_skinny(const MatmulArgs& a, hipStream_t s) {
  auto go = [&](auto kernel, int nt, int kw) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.n + 16 * nt - 1) / (16 * nt))), dim3(64 * kw), 0, s, a);
  };
  // few columns: narrow tiles and more waves along K, so that more CUs bring weights (16 x 4096 x
  // 4096: 4.6 us with sixteen waves, 5.2 with eight, 7.1 with four; 16 x 6144 x 4096: 9.7, 9.0); many:
  // two tiles a wave halve the reads of the rows
  const bool few = a.n <= 4096;
  if (a.m > 32)
    go(skinny_kernel<T, 4, 1, 8>, 1, 8);
  else if (a.m > 16)
    few ? go(skinny_kernel<T, 2, 1, 16>, 1, 16) : go(skinny_kernel<T, 2, 1, 8>, 1, 8);
  else if (a.n >= 8192)
    go(skinny_kernel<T, 1, 2, 4>, 2, 4);
  else
    few ? go(skinny_kernel<T, 1, 1, 16>, 1, 16) : go(skinny_kernel<T, 1, 1, 8>, 1, 8);
  return hipGetLastError();
}

template <class T, int MT, int NT, int MW, int NW>
static hipError_t launch_tiles(const MatmulArgs& a, const MatmulPlan& p, hipStream_t s) {
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  if (tiles > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)tiles, (unsigned)p.splits), block(64 * MW * NW);
  if (p.splits == 1) {
    hipLaunchKernelGGL((tile_kernel<T, MT, NT, MW, NW, false>), grid, block, 0, s, a, p.tiles_m, p.tiles_n, p.blocks_per_split);
    return hipGetLastError();
  }
  if constexpr (MT < 8) {
    hipLaunchKernelGGL((tile_kernel<T, MT, NT, MW, NW, true>), grid, block, 0, s, a, p.tiles_m, p.tiles_n, p.blocks_per_split);
    const int64_t quads = (int64_t)((a.n + 3) / 4) * a.m;
    hipLaunchKernelGGL(join_splits_kernel<T>, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, a, p.splits);
  }
  return hipGetLastError();
}

template <class T>
static hipError_t launch_matmul(const MatmulArgs& a, hipStream_t s) {
  constexpr bool WIDE = std::is_same_v<T, float>;
  const MatmulPlan p = matmul_plan(a.m, a.n, a.k, WIDE);
  switch (p.kind) {
    case MatmulPlan::kSkinny: return launch_skinny<T>(a, s);
    case MatmulPlan::kSmall: return launch_tiles<T, 4, 2, 1, 4>(a, p, s);
    case MatmulPlan::kMedium: return launch_tiles<T, 4, 2, 2, 4>(a, p, s);
    default: break;
  }
  if constexpr (!WIDE) return launch_tiles<T, 8, 4, 2, 4>(a, p, s);
  return hipErrorInvalidValue;
}

hipError_t launch_scaled_matmul(const MatmulArgs& a, int out_type, hipStream_t s) {
  switch (out_type) {
    case SBD_TYPE_BF16: return launch_matmul<Bf16>(a, s);
    case SBD_TYPE_FP16: return launch_matmul<Fp16>(a, s);
    default: return launch_matmul<float>(a, s);
  }
}

}  // namespace sbd
