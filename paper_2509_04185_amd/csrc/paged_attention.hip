// Attention over a paged e4m3 cache with a power of two for each page and KV head
// (sbd_paged_attention).
//
// For one KV head the (row, query head) pairs of a sequence are its rows: row-major, so that
// the 16 * RT rows of a workgroup are neighbours and see nearly the same keys.  The four waves
// of a workgroup hold the same rows and take key stages of 64 in turn; each keeps its own
// softmax (maximum m, sum l, outputs O), and they are joined at the end.  A wave's fragments
// come straight from the cache into registers, 16 bytes a lane:
//   scores   S^T = K Q^T, K as the A operand.  The 16 keys of tile (h, t) are
//            16 (r / 4) + 8 h + 4 t + r % 4 for operand row r, so lane (r, grp) of the result
//            holds the 16 keys 16 grp + 8 h + 4 t + i of its query row r: one run of 16 keys,
//            which lies in one page and has one exponent for K and one for V;
//   outputs  O^T += V^T P^T: that lane's 8 weights of half h are the B operand as they are, and
//            16 bytes of row d of the transposed values are the A operands of both halves.
// Weights are p = 2^(s - m + 15) in fp16 (11 bits; the codes are exact in fp16 too): a weight
// below 2^-39 of the largest becomes 0, and the factor leaves through l.  The exponents of V
// enter as 2^(e - emax) in the widening (exact down to 2^-15) and 2^emax in the fp32 addition
// to O; where the exponents of a stage are further apart its four runs are added one by one.

#include "ops_device.h"

namespace sbd {

constexpr int kPAttnThreads = 256;
constexpr int kStage = 64;           // keys of a stage
constexpr int kRound = 4 * kStage;   // keys the four waves take at a time

namespace {

__device__ __forceinline__ float xor16_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

// Any byte of w an e4m3 NaN (0x7f or 0xff)
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// What a stage's keys need besides their codes, for this lane's run of 16 keys.
struct Run {
  int page;   // valid page id, or 0
  int off;    // offset of the run in it
  bool ok;    // the table names a page
};

// Where the keys of a sequence's part end, in stages of its own: see split_len.
__device__ __forceinline__ int split_len(int kv, const PagedAttnPlan& p) {
  const int even = (int)(((int64_t)kv + p.n_splits - 1) / p.n_splits);
  return max(p.split_keys, (even + kRound - 1) / kRound * kRound);
}

}  // namespace

template <class T, int DH, int RT>
__global__ __launch_bounds__(kPAttnThreads, RT == 4 ? 1 : 2) void paged_attn_kernel(PagedAttnArgs a) {
  constexpr int NDT = DH / 16, NJ = DH / 64, TR = 16 * RT;
  __shared__ f32x4 s_o[4][RT][NDT][64];
  __shared__ float s_m[4][TR], s_l[4][TR];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int r = lane & 15, grp = lane >> 4;
  const int H = a.c.n_kv_heads, G = a.n_q / H, P = a.c.page_size;
  const int pshift = 31 - __builtin_clz(P);

  const int g = blockIdx.x % H;
  const int item = blockIdx.x / H;
  const int split = item % a.plan.n_splits, rb_all = item / a.plan.n_splits;
  auto start = [&](int b) { return (int64_t)a.row_start[b] * G / TR + b; };
  const int b = find_sequence(a.batch, rb_all, start);
  const int r0 = a.row_start[b], n = a.row_start[b + 1] - r0;
  const int64_t rb = rb_all - start(b);
  if (r0 < 0 || n <= 0 || rb < 0 || rb * TR >= (int64_t)n * G) return;
  int kv = min(max(a.kv_len[b], 0), a.max_pages << pshift);
  const int nc = a.n_causal ? a.n_causal[b] : n;
  if (kv < n) kv = 0;  // not served: no row sees a key

  // this lane's rows (the same in every wave) and the keys that each sees
  int row[RT], head[RT], kend[RT];
  int kmax = 0, kmin = INT32_MAX;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t rho = rb * TR + 16 * t + r;
    const int j = (int)(rho / G);
    const bool ok = rho < (int64_t)n * G && r0 + j < a.rows;
    row[t] = ok ? r0 + j : -1;
    head[t] = g * G + (int)(rho % G);
    kend[t] = (ok && kv > 0) ? (j < nc ? kv - n + j + 1 : kv) : 0;
    kmax = max(kmax, kend[t]);
    if (ok) kmin = min(kmin, kend[t]);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    kmax = max(kmax, __shfl_xor(kmax, o));
    kmin = min(kmin, __shfl_xor(kmin, o));
  }
  const int len = split_len(kv, a.plan);
  const int k0 = (int)min((int64_t)split * len, (int64_t)kmax);
  const int k1 = (int)min((int64_t)k0 + len, (int64_t)kmax);

  // Query fragments (B operand): piece j, half h holds dims 64 j + 16 grp + 8 h .. + 8.
  i32x4 qf[RT][NJ][2];
  const uint16_t* q = static_cast<const uint16_t*>(a.q);
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        qf[t][j][h] = row[t] >= 0 ? ld16(q + row[t] * a.q_stride + head[t] * DH + 64 * j + 16 * grp + 8 * h)
                                  : i32x4{0, 0, 0, 0};

  const int* table = a.table + (int64_t)b * a.max_pages;
  auto find_run = [&](int key) {
    const int p = table[min(key >> pshift, a.max_pages - 1)];
    const bool ok = (unsigned)p < (unsigned)a.c.n_pages;
    return Run{ok ? p : 0, key & (P - 1), ok};
  };

  f32x4 o[RT][NDT];
  float m[RT], l[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < NDT; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int ks = k0 + kStage * w; ks < k1; ks += kRound) {
    const Run rk = find_run(ks + 16 * (r >> 2)), rv = find_run(ks + 16 * grp);
    i32x4 kf[4][NJ], vf[NDT];
    const uint8_t* kp = a.c.k_codes + (((int64_t)rk.page * H + g) * P + rk.off + (r & 3)) * DH + 16 * grp;
#pragma unroll
    for (int u = 0; u < 4; ++u)  // tile (h, t) = (u / 2, u % 2): keys 4 u + r % 4 of the run
#pragma unroll
      for (int j = 0; j < NJ; ++j) kf[u][j] = ld16(kp + 4 * u * DH + 64 * j);
    const uint8_t* vp = a.c.v_codes + (((int64_t)rv.page * H + g) * DH + r) * P + rv.off;
#pragma unroll
    for (int d = 0; d < NDT; ++d) vf[d] = ld16(vp + (int64_t)16 * d * P);
    const float ke = ldexpf(a.scale_log2, a.c.k_exp[(int64_t)rv.page * H + g]);
    int ve = rv.ok && ks + 16 * grp < kmax ? a.c.v_exp[(int64_t)rv.page * H + g] : -128;

    f32x4 s[RT][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int t = 0; t < RT; ++t) s[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const i32x4 kk = widen8<T>(i32x2{kf[u][j][2 * h], kf[u][j][2 * h + 1]}, 1.f);
#pragma unroll
          for (int t = 0; t < RT; ++t) s[t][u] = mfma16<T>(kk, qf[t][j][h], s[t][u]);
        }
    }

    // s[t][u][i]: key ks + 16 grp + 4 u + i of row r.  Keys that some row does not see need
    // care: their scores, and their values where they hold NaN.
    const bool edge = __any(ks + kStage > kmin || !rv.ok);
    bool nans = false;
    if (edge) {
      const int seen = rv.ok ? min(max(kmax - ks - 16 * grp, 0), 16) : 0;  // keys of the run that any row sees
      uint32_t found = 0;
#pragma unroll
      for (int d = 0; d < NDT; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int keep = min(max(seen - 4 * c, 0), 4);
          const uint32_t mask = keep == 4 ? ~0u : (1u << (8 * keep)) - 1;
          vf[d][c] &= (int)mask;
          found |= nan_bytes((uint32_t)vf[d][c]);
        }
      nans = __any(found != 0);
    }

    // weights, running maximum and sum (this lane's 16 keys; the sums are joined at the end)
    i32x4 pf[RT][2];
    float alpha[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v = s[t][u][i] * ke;
          if (edge && (!rv.ok || ks + 16 * grp + 4 * u + i >= kend[t])) v = -INFINITY;
          s[t][u][i] = v;
          top = fmaxf(top, v);
        }
      const float mn = fmaxf(m[t], xor16_max(top));
      const float base = mn == -INFINITY ? 0.f : mn - 15.f;
      alpha[t] = __builtin_amdgcn_exp2f(m[t] - (mn == -INFINITY ? 0.f : mn));
      m[t] = mn;
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = __builtin_amdgcn_exp2f(s[t][u][i] - base);
          sum += p[i];
        }
        pf[t][u >> 1][2 * (u & 1)] = (int)pack2<Fp16>(p[0], p[1]);
        pf[t][u >> 1][2 * (u & 1) + 1] = (int)pack2<Fp16>(p[2], p[3]);
      }
      l[t] = l[t] * alpha[t] + sum;
    }

    int vtop = max(max(__shfl(ve, 0), __shfl(ve, 16)), max(__shfl(ve, 32), __shfl(ve, 48)));
    vtop = max(vtop, -100);
    if (ve < -100) ve = vtop;  // a run that no row sees
    const int vlow = min(min(__shfl(ve, 0), __shfl(ve, 16)), min(__shfl(ve, 32), __shfl(ve, 48)));
    auto add = [&](float vs, float os, bool mine) {
#pragma unroll
      for (int d = 0; d < NDT; ++d) {
        i32x4 v0 = widen8<Fp16>(i32x2{vf[d][0], vf[d][1]}, vs), v1 = widen8<Fp16>(i32x2{vf[d][2], vf[d][3]}, vs);
        if (!mine) v0 = v1 = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
          x = mfma16<Fp16>(v0, pf[t][0], x);
          x = mfma16<Fp16>(v1, pf[t][1], x);
          o[t][d] = o[t][d] * alpha[t] + x * os;
        }
      }
    };
    if (__builtin_expect(nans, 0)) {
      // A NaN value reaches the rows that see its key and no other: count the NaN keys that
      // each row sees by a product of ones, then take the NaN codes out.
      i32x4 sf[RT][2];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = ks + 16 * grp + 4 * u + i < kend[t] ? 1.f : 0.f;
          sf[t][u >> 1][2 * (u & 1)] = (int)pack2<Fp16>(p[0], p[1]);
          sf[t][u >> 1][2 * (u & 1) + 1] = (int)pack2<Fp16>(p[2], p[3]);
        }
#pragma unroll
      for (int d = 0; d < NDT; ++d) {
        i32x4 ones[2];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t bad = nan_bytes((uint32_t)vf[d][c]) >> 7;  // 1 in the bytes of NaN codes
          ones[c >> 1][2 * (c & 1)] = (int)(((bad & 1) | ((bad >> 8 & 1) << 16)) * 0x3c00u);
          ones[c >> 1][2 * (c & 1) + 1] = (int)(((bad >> 16 & 1) | ((bad >> 24 & 1) << 16)) * 0x3c00u);
          vf[d][c] &= (int)~(bad * 255u);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
          x = mfma16<Fp16>(ones[0], sf[t][0], x);
          x = mfma16<Fp16>(ones[1], sf[t][1], x);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (x[i] > 0.f) o[t][d][i] = __builtin_nanf("");
        }
      }
    }
    if (__builtin_expect(vtop - vlow <= 15, 1)) {
      add(pow2i(ve - vtop), pow2i(vtop), true);
    } else {
      for (int u = 0; u < 4; ++u) {
        add(1.f, pow2i(__shfl(ve, 16 * u)), grp == u);
#pragma unroll
        for (int t = 0; t < RT; ++t) alpha[t] = 1.f;
      }
    }
  }

  // Join the waves: every wave brings its outputs to the common maximum and adds up a quarter
  // of the dimensions.
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] += __shfl_xor(l[t], 16);
    l[t] += __shfl_xor(l[t], 32);
    if (grp == 0) {
      s_m[w][16 * t + r] = m[t];
      s_l[w][16 * t + r] = l[t];
    }
  }
  __syncthreads();
  float lsum[RT], mall[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int i = 16 * t + r;
    const float mx = fmaxf(fmaxf(s_m[0][i], s_m[1][i]), fmaxf(s_m[2][i], s_m[3][i]));
    const float base = mx == -INFINITY ? 0.f : mx;
    lsum[t] = 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) lsum[t] += s_l[v][i] * __builtin_amdgcn_exp2f(s_m[v][i] - base);
    mall[t] = mx;
    const float f = __builtin_amdgcn_exp2f(m[t] - base);
#pragma unroll
    for (int d = 0; d < NDT; ++d) {
      o[t][d] = o[t][d] * f;
      if (d / (NDT / 4) != w) s_o[w][t][d][lane] = o[t][d];
    }
  }
  __syncthreads();
  const bool last = a.plan.n_splits == 1;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (row[t] < 0) continue;
    const int64_t pair = (int64_t)row[t] * a.n_q + head[t];
    const int64_t part = (int64_t)split * a.rows * a.n_q + pair;
    const float inv = lsum[t] == 0.f ? 0.f : 1.f / lsum[t];
    if (!last && w == 0 && grp == 0) {
      a.part_ml[2 * part] = mall[t];
      a.part_ml[2 * part + 1] = lsum[t];
    }
    if (!last && k0 >= k1) continue;  // the join leaves out parts whose sum is 0
#pragma unroll
    for (int d = 0; d < NDT; ++d) {
      if (d / (NDT / 4) != w) continue;
      f32x4 x = o[t][d];
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (v != w) x += s_o[v][t][d][lane];
      const int dim = 16 * d + 4 * grp;
      if (last) {
        x *= inv;
        uint16_t* out = static_cast<uint16_t*>(a.out) + row[t] * a.out_stride + head[t] * DH + dim;
        *(i32x2*)out = i32x2{(int)pack2<T>(x[0], x[1]), (int)pack2<T>(x[2], x[3])};
      } else {
        *(f32x4*)(a.part_o + part * DH + dim) = x;
      }
    }
  }
}

// Join the key parts of one (row, query head) pair: one wave each, in order of the parts.
template <class T, int DH>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PagedAttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t pairs = (int64_t)a.rows * a.n_q;
  const int64_t pair = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (pair >= pairs) return;
  const int row = (int)(pair / a.n_q), head = (int)(pair % a.n_q);
  if (row < a.row_start[0] || row >= a.row_start[a.batch]) return;
  const int ns = a.plan.n_splits;  // <= 64
  float ms = -INFINITY, ls = 0.f;
  if (lane < ns) {
    ms = a.part_ml[2 * (lane * pairs + pair)];
    ls = a.part_ml[2 * (lane * pairs + pair) + 1];
  }
  const float mx = wave_max(ms);
  const float wgt = __builtin_amdgcn_exp2f(ms - (mx == -INFINITY ? 0.f : mx));
  const float lsum = wave_sum(wgt * ls);
  constexpr int PER = DH / 64;
  float acc[PER] = {};
  uint64_t parts = __ballot(!(ls == 0.f));
  while (parts) {  // wave-uniform
    const int s = __ffsll((unsigned long long)parts) - 1;
    parts &= parts - 1;
    const float f = __shfl(wgt, s);
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] += f * a.part_o[(s * pairs + pair) * DH + PER * lane + e];
  }
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
  uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.out_stride + head * DH + PER * lane;
  if constexpr (PER == 2)
    *(uint32_t*)out = pack2<T>(acc[0] * inv, acc[1] * inv);
  else
    *out = (uint16_t)pack2<T>(acc[0] * inv, 0.f);
}

PagedAttnPlan paged_attention_plan(const sbd_paged_kv& c, int batch, int rows, int n_q, int max_kv) {
  PagedAttnPlan p{};
  const int64_t pairs = (int64_t)rows * (n_q / c.n_kv_heads);
  const int64_t each = (pairs + batch - 1) / batch;  // of a sequence, on average
  p.row_tiles = each <= 16 ? 1 : each <= 32 ? 2 : 4;
  const int tr = 16 * p.row_tiles;
  p.rowblocks = pairs / tr + batch;
  const int64_t groups = std::max<int64_t>(1, batch * ((each + tr - 1) / tr) * c.n_kv_heads);
  const int64_t want = (256 * (p.row_tiles == 4 ? 1 : 2) + groups - 1) / groups;
  p.n_splits = (int)std::max<int64_t>(1, std::min<int64_t>({want, 64, (max_kv + kRound - 1) / kRound}));
  p.split_keys = ((max_kv + p.n_splits - 1) / p.n_splits + kRound - 1) / kRound * kRound;
  if (p.n_splits > 1) {
    const size_t items = (size_t)p.n_splits * rows * n_q;
    p.part_ml = 0;
    p.part_o = (items * 2 * sizeof(float) + 255) / 256 * 256;
    p.bytes = p.part_o + items * c.head_dim * sizeof(float);
  }
  return p;
}

template <class T, int DH>
static hipError_t launch_dh(const PagedAttnArgs& a, hipStream_t s) {
  const int64_t grid = a.plan.rowblocks * a.plan.n_splits * a.c.n_kv_heads;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kPAttnThreads), 0, s, a); };
  switch (a.plan.row_tiles) {
    case 1: go(paged_attn_kernel<T, DH, 1>); break;
    case 2: go(paged_attn_kernel<T, DH, 2>); break;
    default: go(paged_attn_kernel<T, DH, 4>); break;
  }
  if (a.plan.n_splits > 1)
    hipLaunchKernelGGL((paged_attn_join_kernel<T, DH>), dim3((unsigned)(((int64_t)a.rows * a.n_q + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, int dtype, hipStream_t s) {
  if (a.c.head_dim == 128) return dtype == SBD_TYPE_BF16 ? launch_dh<Bf16, 128>(a, s) : launch_dh<Fp16, 128>(a, s);
  return dtype == SBD_TYPE_BF16 ? launch_dh<Bf16, 64>(a, s) : launch_dh<Fp16, 64>(a, s);
}

}  // namespace sbd
