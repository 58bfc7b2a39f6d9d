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

// A scale for each row and 128 columns: 16 lanes hold such a block, 8 elements each.
template <class T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeArgs a) {
  const int kb = (a.cols + 127) / 128;
  const int64_t block = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (block >= (int64_t)a.rows * kb) return;  // whole groups of 16 lanes
  const int row = (int)(block / kb), c = (int)(block % kb), col = 128 * c + 8 * (threadIdx.x & 15);
  float f[8] = {};
  if (col < a.cols) load8<T>(a.x, row * a.x_stride + col, f);
  float m = max8(f);
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  const int e = block_exponent(m);
  if (col < a.cols) *(i32x2*)(a.codes + (int64_t)row * a.cols + col) = codes8(f, pow2i(-e));
  if ((threadIdx.x & 15) == 0) a.scales[(int64_t)c * a.rows + row] = pow2i(e);
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
    if (row < a.rows && col < a.cols) *(i32x2*)(a.codes + (int64_t)row * a.cols + col) = codes8(f[u], inv);
  }
  if (threadIdx.x == 0) a.scales[blockIdx.x] = pow2i(e);
}

template <class T>
static hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t s) {
  const int64_t kb = (a.cols + 127) / 128;
  const int64_t grid = a.block_rows == 1 ? ((int64_t)a.rows * kb + 15) / 16 : (int64_t)(a.rows + 127) / 128 * kb;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  if (a.block_rows == 1)
    hipLaunchKernelGGL(quantize_rows_kernel<T>, dim3((unsigned)grid), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(quantize_tiles_kernel<T>, dim3((unsigned)grid), dim3(256), 0, s, a);
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
// A block of 128 along K is summed by the matrix unit, multiplied by the block's scales and
// added to fp32 sums.  The weights are the A operand, so lane (r, grp) holds out row r and four
// neighbouring columns 4 grp + i, and a_scale is one value a lane.  Both operands use the same
// order of k: lane group grp holds k = 64 p + 16 grp .. + 16, p = 0, 1.
//
// The codes are widened to bf16 (exact) and multiplied by the bf16 instruction, whose sums are
// fp32.  The e4m3 instructions add groups of eight products aligned to the largest, of which
// they keep 14 bits (measured: 2^16 + 2^2 gives 2^16 within eight neighbours).

__device__ __forceinline__ f32x4 mfma_block(i32x8 a, i32x8 b) {
  f32x4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int p = 0; p < 4; ++p)
    c = mfma16<Bf16>(e4m3x8_to_bf16(i32x2{a[2 * p], a[2 * p + 1]}, 1.f), e4m3x8_to_bf16(i32x2{b[2 * p], b[2 * p + 1]}, 1.f), c);
  return c;
}

// This lane's fragment of block c of a row of k codes (zeros behind its end).
__device__ __forceinline__ i32x8 load_frag(const uint8_t* row, int c, int grp, int k) {
  const int k0 = 128 * c + 16 * grp;
  const i32x4 z{0, 0, 0, 0};
  const i32x4 lo = k0 < k ? ld16(row + k0) : z, hi = k0 + 64 < k ? ld16(row + k0 + 64) : z;
  return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

template <class T>
__device__ __forceinline__ void store4(void* out, int64_t at, int n_left, bool vec, f32x4 v) {
  if constexpr (std::is_same_v<T, float>) {
    float* p = static_cast<float*>(out) + at;
    if (vec && n_left >= 4) {
      *(f32x4*)p = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n_left) p[i] = v[i];
    }
  } else {
    uint16_t* p = static_cast<uint16_t*>(out) + at;
    const uint32_t lo = pack2<T>(v[0], v[1]), hi = pack2<T>(v[2], v[3]);
    if (vec && n_left >= 4) {
      *(i32x2*)p = i32x2{(int)lo, (int)hi};
    } else {
      if (n_left > 0) p[0] = (uint16_t)lo;
      if (n_left > 1) p[1] = (uint16_t)(lo >> 16);
      if (n_left > 2) p[2] = (uint16_t)hi;
      if (n_left > 3) p[3] = (uint16_t)(hi >> 16);
    }
  }
}

// Rows of out may be stored four elements at a time.
template <class T>
static __device__ __forceinline__ bool vec_ok(const MatmulArgs& a) {
  constexpr int ES = std::is_same_v<T, float> ? 4 : 2;
  return a.out_stride % 4 == 0 && (uintptr_t)a.out % (4 * ES) == 0;
}

// Each wave makes 16 rows x 64 columns from registers.
template <class T>
__global__ __launch_bounds__(256) void matmul_kernel(MatmulArgs a) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, grp = lane >> 4;
  const int kb = (a.k + 127) / 128;
  const int m0 = blockIdx.y * 64 + 16 * w, n0 = blockIdx.x * 64;
  if (m0 >= a.m) return;
  const int m = min(m0 + r, a.m - 1);
  f32x4 acc[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int c = 0; c < kb; ++c) {
    const i32x8 x = load_frag(a.a + m * a.a_stride, c, grp, a.k);
    const float sa = a.a_scale[(int64_t)c * a.m + m] * a.b_scale[(int64_t)(n0 / 128) * kb + c];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const i32x8 y = load_frag(a.b + (int64_t)min(n0 + 16 * t + r, a.n - 1) * a.k, c, grp, a.k);
      acc[t] += mfma_block(y, x) * sa;
    }
  }
  if (m0 + r >= a.m) return;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int n = n0 + 16 * t + 4 * grp;
    store4<T>(a.out, m * a.out_stride + n, a.n - n, vec_ok<T>(a), acc[t]);
  }
}

size_t scaled_matmul_bytes(int, int, int) { return 0; }

template <class T>
static hipError_t launch_matmul(const MatmulArgs& a, hipStream_t s) {
  const int64_t gx = (a.n + 63) / 64, gy = (a.m + 63) / 64;
  if (gy > 65535) return hipErrorInvalidValue;
  hipLaunchKernelGGL(matmul_kernel<T>, dim3((unsigned)gx, (unsigned)gy), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_scaled_matmul(const MatmulArgs& a, int out_type, hipStream_t s) {
  switch (out_type) {
    case SBD_TYPE_BF16: return launch_matmul<Bf16>(a, s);
    case SBD_TYPE_FP16: return launch_matmul<Fp16>(a, s);
    default: return launch_matmul<float>(a, s);
  }
}

}  // namespace sbd
