// Attention over a paged e4m3 cache with a power of two for each page and KV head
// (sbd_paged_attention).
//
// For one KV head the (row, query head) pairs of a sequence are its rows: row-major, so that
// neighbours see nearly the same keys.  A wave holds 16 RT of them with their softmax (a
// reference m, the sum l, outputs O) and takes stages of 64 keys:
//   scores   S^T = K Q^T, K as the A operand.  The 16 keys of tile u are 16 (r / 4) + 4 u + r % 4
//            for operand row r, so lane (r, grp) of the result holds the 16 keys 16 grp + 4 u + i
//            of its query row r: one run of 16 keys, which lies in one page and has one exponent
//            for K and one for V;
//   outputs  O^T += V^T P^T: that lane's weights are the B operand as they are, and 16 bytes of
//            row d of the transposed values are the A operands; a row of ones makes l.
// The codes are exact in the 16-bit types; K is widened to the queries' type.
//
// Weights are p = 2^(s - m + 11) in fp16.  m follows the maximum only when it is exceeded by
// more than 4 (then O and l are scaled), so p stays below 2^15 and most stages scale nothing; a
// weight below 2^-36 of 2^m becomes 0, and the factor 2^11 leaves through l.  O is kept in units
// of 2^E, E the largest exponent of V seen so far: a run's exponent enters as 2^(e - E) in the
// widening (exact down to 2^-15); where it is further below, the stage's runs are added one by
// one in fp32.
//
// A stage's codes are copied from the cache straight into LDS (asm without results, as in
// scaled.hip), 16-byte pieces swizzled so that the fragment reads are free of bank conflicts.
// (Fragments loaded straight from the cache ask the vector cache for 16 bytes at a time:
// neighbouring lanes lie in different rows.)  Which pages the copies read and the exponents
// stand in LDS too, for up to kUnits runs at a time: the loop loads nothing else.

#include "ops_device.h"

namespace sbd {

constexpr int kStage = 64;           // keys of a stage
constexpr int kUnits = 1024;         // runs of 16 keys whose pages and exponents are in LDS at once
constexpr float kLift = 11.f, kSlack = 4.f;

namespace {

// Any byte of w an e4m3 NaN (0x7f or 0xff)
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

__device__ __forceinline__ void copy16(const uint8_t* p, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off"
      :
      : "s"(lds), "v"(p)
      : "memory", "m0");
}

// A run of 16 keys: its page (-1 where the table names none) and its exponents (K, then V).
struct Unit {
  int page;
  int16_t ke, ve;
};

// Keys of a part, at least split_keys.
__device__ __forceinline__ int split_len(int kv, const PagedAttnPlan& p) {
  const int even = (int)(((int64_t)kv + p.n_splits - 1) / p.n_splits);
  return max(p.split_keys, (even + kStage - 1) / kStage * kStage);
}

// One sequence and KV head as a workgroup sees it.
struct Seq {
  int b, r0, n, kv, nc;
  int g, G, pshift;
};
__device__ __forceinline__ Seq load_seq(const PagedAttnArgs& a, int b, int g) {
  Seq q;
  q.b = b;
  q.g = g;
  q.G = a.n_q / a.c.n_kv_heads;
  q.pshift = 31 - __builtin_clz(a.c.page_size);
  q.r0 = a.row_start[b];
  q.n = a.row_start[b + 1] - q.r0;
  q.kv = min(max(a.kv_len[b], 0), a.max_pages << q.pshift);
  q.nc = a.n_causal ? a.n_causal[b] : q.n;
  if (q.kv < q.n) q.kv = 0;  // not served: no row sees a key
  return q;
}

__device__ __forceinline__ void load_pages(const PagedAttnArgs& a, const Seq& q, int key0, int units, Unit* out) {
  const int* table = a.table + (int64_t)q.b * a.max_pages;
  for (int t = threadIdx.x; t < units; t += blockDim.x) {
    const int p = table[min((key0 + 16 * t) >> q.pshift, a.max_pages - 1)];
    out[t].page = (unsigned)p < (unsigned)a.c.n_pages ? p : -1;
  }
}
__device__ __forceinline__ void load_exponents(const PagedAttnArgs& a, const Seq& q, int units, Unit* out) {
  for (int t = threadIdx.x; t < units; t += blockDim.x) {
    const int64_t at = (int64_t)max(out[t].page, 0) * a.c.n_kv_heads + q.g;
    out[t].ke = a.c.k_exp[at];
    out[t].ve = a.c.v_exp[at];
  }
}

// Stages in LDS: K as [64 keys][DH], V as [DH][64 keys].
template <int DH>
struct Tiles {
  static constexpr int kBytes = 2 * kStage * DH, kCopies = kBytes / 1024;  // 1 KB copies: half K, half V
  __device__ static int ksw(int key) {
    return DH == 128 ? (key & 3) | ((key >> 4) & 1) << 2 : ((key >> 1) & 1) | ((key >> 4) & 1) << 1;
  }
  // LDS piece of K: 16 bytes `c` of a key; of V: the 16 keys of run `u` of a dimension
  __device__ static int k_at(int key, int c) { return key * DH + ((c ^ ksw(key)) * 16); }
  __device__ static int v_at(int dim, int u) { return kStage * DH + dim * kStage + ((u ^ ((dim >> 1) & 3)) * 16); }

  // Copy i of a stage (units: its four runs; key: its first key) into `lds`.
  __device__ static void copy(const PagedAttnArgs& a, const Seq& q, const Unit* units, int key, int i, uint32_t lds) {
    const int lane = threadIdx.x & 63, H = a.c.n_kv_heads, P = a.c.page_size;
    const uint8_t* p;
    if (i < kCopies / 2) {
      const int piece = 64 * i + lane, row = piece / (DH / 16), c = (piece % (DH / 16)) ^ ksw(row);
      const int u = 64 * i / (DH / 16) / 16;  // the copy's run
      const int page = max(units[u].page, 0), off = ((key + 16 * u) & (P - 1)) + (row & 15);
      p = a.c.k_codes + (((int64_t)page * H + q.g) * P + off) * DH + c * 16;
    } else {
      const int dim = 16 * (i - kCopies / 2) + (lane >> 2), u = (lane & 3) ^ ((lane >> 3) & 3);
      const int page = max(units[u].page, 0), off = (key + 16 * u) & (P - 1);
      p = a.c.v_codes + (((int64_t)page * H + q.g) * DH + dim) * P + off;
    }
    copy16(p, __builtin_amdgcn_readfirstlane(lds + i * 1024));
  }
};

// A wave's rows.
template <class T, int DH, int RT>
struct Rows {
  static constexpr int NDT = DH / 16, NJ = DH / 64;
  int row[RT], head[RT], kend[RT];  // of this lane's row of each tile; -1, 0 where there is none
  int kmax, kmin;                   // over all rows of the wave
  i32x4 qf[RT][NJ][2];              // B operand: piece j, half h holds dims 64 j + 16 grp + 8 h .. + 8
  f32x4 o[RT][NDT];                 // in units of 2^E
  f32x4 l[RT];                      // four times the same
  float m[RT];
  int E;

  __device__ __forceinline__ void init(const PagedAttnArgs& a, const Seq& s, int64_t first) {
    const int lane = threadIdx.x & 63, r = lane & 15, grp = lane >> 4;
    kmax = 0;
    kmin = INT32_MAX;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t rho = first + 16 * t + r;
      const int j = (int)(rho / s.G);
      const bool ok = rho < (int64_t)s.n * s.G && s.r0 + j < a.rows;
      row[t] = ok ? s.r0 + j : -1;
      head[t] = s.g * s.G + (int)(rho % s.G);
      kend[t] = (ok && s.kv > 0) ? (j < s.nc ? s.kv - s.n + j + 1 : s.kv) : 0;
      kmax = max(kmax, kend[t]);
      if (ok) kmin = min(kmin, kend[t]);
    }
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) {
      kmax = max(kmax, __shfl_xor(kmax, x));
      kmin = min(kmin, __shfl_xor(kmin, x));
    }
    kmax = __builtin_amdgcn_readfirstlane(kmax);
    kmin = __builtin_amdgcn_readfirstlane(kmin);
    const uint16_t* q = static_cast<const uint16_t*>(a.q);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          i32x4 v{0, 0, 0, 0};
          if (row[t] >= 0) v = ld16(q + row[t] * a.q_stride + head[t] * DH + 64 * j + 16 * grp + 8 * h);
          qf[t][j][h] = v;
        }
      m[t] = -INFINITY;
      l[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < NDT; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    E = -128;
  }

  // The scale's sign goes into the queries (stage() takes its size).
  __device__ __forceinline__ void flip() {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) qf[t][j][h][e] ^= (int)0x80008000;
  }

  // One stage: keys ks .. ks + 64 at `buf`, this lane's run `un` (of keys ks + 16 grp ..).
  __device__ __forceinline__ void stage(const uint8_t* buf, int ks, Unit un, float scale_log2) {
    const int lane = threadIdx.x & 63, r = lane & 15, grp = lane >> 4;
    using L = Tiles<DH>;
    const int run = ks + 16 * grp;
    const bool known = un.page >= 0;
    // never 0, so that a hidden score (-infinity) stays one
    const float ke = fmaxf(ldexpf(fabsf(scale_log2), un.ke), 1.17549435e-38f);
    int ve = known && run < kmax ? un.ve : -128;

    f32x4 s[RT][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int t = 0; t < RT; ++t) s[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const i32x4 kf = *(const i32x4*)(buf + L::k_at(16 * (r >> 2) + 4 * u + (r & 3), 4 * j + grp));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const i32x4 kk = widen8<T>(i32x2{kf[2 * h], kf[2 * h + 1]}, 1.f);
#pragma unroll
          for (int t = 0; t < RT; ++t) s[t][u] = mfma16<T>(kk, qf[t][j][h], s[t][u]);
        }
      }
    }

    // s[t][u][i]: key run + 4 u + i of row r.  Keys that some row does not see need care: their
    // scores here, and their values where those are NaN.
    const bool edge = __any(ks + kStage > kmin || !known);
    if (edge) {
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!known || run + 4 * u + i >= kend[t]) s[t][u][i] = -INFINITY;
    }
    float mn[RT];
    bool up = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < 4; ++u) top = fmaxf(fmaxf(top, fmaxf(s[t][u][0], s[t][u][1])), fmaxf(s[t][u][2], s[t][u][3]));
      top *= ke;
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      mn[t] = top > m[t] + kSlack || m[t] == -INFINITY ? fmaxf(top, m[t]) : m[t];
      up |= mn[t] != m[t];
    }
    int vtop = max(max(__shfl(ve, 0), __shfl(ve, 16)), max(__shfl(ve, 32), __shfl(ve, 48)));
    vtop = __builtin_amdgcn_readfirstlane(max(vtop, -100));
    if (__any(up) || vtop > E) {
      const int e = max(E, vtop);
      const float f = E < -100 ? 0.f : ldexpf(1.f, E - e);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const float alpha = m[t] == mn[t] ? 1.f : __builtin_amdgcn_exp2f(m[t] - mn[t]);
        m[t] = mn[t];
        l[t] *= alpha;
#pragma unroll
        for (int d = 0; d < NDT; ++d) o[t][d] *= alpha * f;
      }
      E = e;
    }

    i32x4 pf[RT][2];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const float base = m[t] == -INFINITY ? 0.f : kLift - m[t];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][u][i], ke, base));
        pf[t][u >> 1][2 * (u & 1)] = (int)pack2<Fp16>(p[0], p[1]);
        pf[t][u >> 1][2 * (u & 1) + 1] = (int)pack2<Fp16>(p[2], p[3]);
      }
      const int one = 0x3c003c00;
      const i32x4 ones{one, one, one, one};
      l[t] = mfma16<Fp16>(ones, pf[t][0], l[t]);
      l[t] = mfma16<Fp16>(ones, pf[t][1], l[t]);
    }

    if (ve < -100) ve = E;  // a run that no row sees
    const bool near = __all(ve >= E - 15);
    if (__builtin_expect(near && !edge, 1)) {
      const float vs = pow2i(ve - E);
#pragma unroll
      for (int d = 0; d < NDT; ++d) {
        const i32x4 v = *(const i32x4*)(buf + L::v_at(16 * d + r, grp));
        const i32x4 v0 = widen8<Fp16>(i32x2{v[0], v[1]}, vs), v1 = widen8<Fp16>(i32x2{v[2], v[3]}, vs);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          o[t][d] = mfma16<Fp16>(v0, pf[t][0], o[t][d]);
          o[t][d] = mfma16<Fp16>(v1, pf[t][1], o[t][d]);
        }
      }
      return;
    }
    careful(buf, run, known, ve, near, pf);
  }

  // The values of a stage at the end of what some row sees, or with exponents far apart.
  __device__ __forceinline__ void careful(const uint8_t* buf, int run, bool known, int ve, bool near, const i32x4 (&pf)[RT][2]) {
    const int lane = threadIdx.x & 63, r = lane & 15, grp = lane >> 4;
    const int seen = known ? min(max(kmax - run, 0), 16) : 0;  // keys of the run that any row sees
    uint32_t mask[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int keep = min(max(seen - 4 * c, 0), 4);
      mask[c] = keep == 4 ? ~0u : (1u << (8 * keep)) - 1;
    }
    // A NaN value reaches the rows that see its key and no other: count the NaN keys that each
    // row sees by a product of ones, and take the NaN codes out of the sums.
    i32x4 sf[RT][2];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = run + 4 * u + i < kend[t] ? 1.f : 0.f;
        sf[t][u >> 1][2 * (u & 1)] = (int)pack2<Fp16>(p[0], p[1]);
        sf[t][u >> 1][2 * (u & 1) + 1] = (int)pack2<Fp16>(p[2], p[3]);
      }
#pragma unroll
    for (int d = 0; d < NDT; ++d) {
      i32x4 v = *(const i32x4*)(buf + Tiles<DH>::v_at(16 * d + r, grp));
      uint32_t found = 0, bad[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        v[c] &= (int)mask[c];
        bad[c] = nan_bytes((uint32_t)v[c]) >> 7;  // 1 in the bytes of NaN codes
        found |= bad[c];
      }
      if (__any(found != 0)) {
        i32x4 ones[2];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          ones[c >> 1][2 * (c & 1)] = (int)(((bad[c] & 1) | ((bad[c] >> 8 & 1) << 16)) * 0x3c00u);
          ones[c >> 1][2 * (c & 1) + 1] = (int)(((bad[c] >> 16 & 1) | ((bad[c] >> 24 & 1) << 16)) * 0x3c00u);
          v[c] &= (int)~(bad[c] * 255u);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          f32x4 x{0.f, 0.f, 0.f, 0.f};
          x = mfma16<Fp16>(ones[0], sf[t][0], x);
          x = mfma16<Fp16>(ones[1], sf[t][1], x);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (x[i] > 0.f) o[t][d][i] = __builtin_nanf("");
        }
      }
      if (near) {
        const float vs = pow2i(ve - E);
        const i32x4 v0 = widen8<Fp16>(i32x2{v[0], v[1]}, vs), v1 = widen8<Fp16>(i32x2{v[2], v[3]}, vs);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          o[t][d] = mfma16<Fp16>(v0, pf[t][0], o[t][d]);
          o[t][d] = mfma16<Fp16>(v1, pf[t][1], o[t][d]);
        }
      } else {
        const i32x4 w0 = widen8<Fp16>(i32x2{v[0], v[1]}, 1.f), w1 = widen8<Fp16>(i32x2{v[2], v[3]}, 1.f);
        for (int u = 0; u < 4; ++u) {
          const float f = ldexpf(1.f, __shfl(ve, 16 * u) - E);
          const i32x4 v0 = grp == u ? w0 : i32x4{0, 0, 0, 0}, v1 = grp == u ? w1 : i32x4{0, 0, 0, 0};
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            f32x4 x{0.f, 0.f, 0.f, 0.f};
            x = mfma16<Fp16>(v0, pf[t][0], x);
            x = mfma16<Fp16>(v1, pf[t][1], x);
            o[t][d] += x * f;
          }
        }
      }
    }
  }
};

template <class T>
__device__ __forceinline__ void store_out(const PagedAttnArgs& a, int row, int at, f32x4 x) {
  uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.out_stride + at;
  *(i32x2*)out = i32x2{(int)pack2<T>(x[0], x[1]), (int)pack2<T>(x[2], x[3])};
}

}  // namespace

// A workgroup has RW x KW waves.  RW of them, with 16 RT rows each, share a ring of NB stage
// buffers; the KW groups hold the same rows and take the stages of a part of the keys in turn, and
// are joined at the end.  Measured at these shapes (see paged_attention_plan for the choice): a
// few rows need all waves to bring keys (KW = 4, 64 KB in flight on a CU); with 64 rows and more
// every wave has rows of its own and nothing is joined; many rows take two tiles a wave and two
// waves a SIMD, so that the products of one run beside the exponentials and conversions of the
// other.
template <class T, int DH, int RT, int RW, int KW, int NB>
__global__ __launch_bounds__(64 * RW * KW, RT == 1 ? 2 : 1) void paged_attn_kernel(PagedAttnArgs a) {
  using L = Tiles<DH>;
  constexpr int NDT = DH / 16, TR = 16 * RT * RW, kKeys = kStage * KW;  // rows of a workgroup, keys of a round
  constexpr int kEach = L::kCopies / RW;                              // copies of a wave and stage
  static_assert(kEach * RW == L::kCopies && NDT % KW == 0, "whole copies, whole tiles to join");
  constexpr int kRing = KW * NB * L::kBytes, kJoin = KW == 1 ? 0 : KW * RW * RT * NDT * 1024;
  __shared__ __attribute__((aligned(1024))) uint8_t s_buf[kRing > kJoin ? kRing : kJoin];
  __shared__ Unit s_unit[kUnits];
  __shared__ int s_kmax[RW];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, grp = lane >> 4;
  const int rw = w % RW, kw = w / RW;
  const int H = a.c.n_kv_heads, G = a.n_q / H;
  const int g = blockIdx.x % H, item = blockIdx.x / H;
  const int split = item % a.plan.n_splits;
  const int rb_all = (int)(a.plan.rowblocks - 1 - item / a.plan.n_splits);  // the last rows, which see most keys, first
  auto start = [&](int b) { return (int64_t)a.row_start[b] * G / TR + b; };
  const int b = find_sequence(a.batch, rb_all, start);
  const Seq sq = load_seq(a, b, g);
  const int64_t rb = rb_all - start(b);
  if (sq.r0 < 0 || sq.n <= 0 || rb < 0 || rb * TR >= (int64_t)sq.n * G) return;
  Rows<T, DH, RT> rows;
  rows.init(a, sq, rb * TR + 16 * RT * rw);
  if (lane == 0 && kw == 0) s_kmax[rw] = rows.kmax;
  __syncthreads();
  int kmax = 0;
#pragma unroll
  for (int i = 0; i < RW; ++i) kmax = max(kmax, s_kmax[i]);
  const int len = split_len(sq.kv, a.plan);
  const int k0 = (int)min((int64_t)split * len, (int64_t)kmax);
  const int k1 = (int)min((int64_t)k0 + len, (int64_t)kmax);

  bool flipped = a.scale_log2 >= 0.f;
  uint8_t* ring = s_buf + kw * NB * L::kBytes;
  for (int seg = k0; seg < k1; seg += 16 * kUnits) {
    const int end = min(seg + 16 * kUnits, k1), rounds = (end - seg + kKeys - 1) / kKeys;
    if (seg != k0) __syncthreads();
    load_pages(a, sq, seg, rounds * kKeys / 16, s_unit);
    __syncthreads();
    // this group's stage of round i goes to buffer i % NB; behind the last one it is brought again
    auto copy = [&](int i) {
      const int at = min(i, rounds - 1) * kKeys + kStage * kw;
#pragma unroll
      for (int u = 0; u < kEach; ++u)
        L::copy(a, sq, s_unit + at / 16, seg + at, u * RW + rw, lds_addr(ring) + i % NB * L::kBytes);
    };
#pragma unroll
    for (int i = 0; i < NB - 1; ++i) copy(i);
    load_exponents(a, sq, rounds * kKeys / 16, s_unit);
    if (!flipped) rows.flip();
    flipped = true;
    for (int i = 0; i < rounds; ++i) {
      vm_wait<(NB - 2) * kEach>();  // this wave's copies of round i have landed
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      copy(i + NB - 1);  // into the buffer of round i - 1, which every wave has read
      const int at = i * kKeys + kStage * kw, ks = seg + at;
      if (ks < rows.kmax && ks < k1) rows.stage(ring + i % NB * L::kBytes, ks, s_unit[at / 16 + grp], fabsf(a.scale_log2));
    }
    vm_wait<0>();
  }

  const bool last = a.plan.n_splits == 1;
  auto put = [&](int t, int d, f32x4 x) {
    const int dim = 16 * d + 4 * grp;
    if (last)
      store_out<T>(a, rows.row[t], rows.head[t] * DH + dim, x);
    else
      *(f32x4*)(a.part_o + (((int64_t)split * a.rows + rows.row[t]) * a.n_q + rows.head[t]) * DH + dim) = x;
  };
  auto put_ml = [&](int t, float m, float l) {
    if (last || grp != 0 || kw != 0) return;
    float* ml = a.part_ml + 2 * (((int64_t)split * a.rows + rows.row[t]) * a.n_q + rows.head[t]);
    ml[0] = m;
    ml[1] = l;
  };
  const bool none = !last && k0 >= k1;  // the join leaves out parts whose sum is 0
  if constexpr (KW == 1) {
    const float real = pow2i(max(rows.E, -100));
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (rows.row[t] < 0) continue;
      const float l = rows.l[t][0], inv = l == 0.f ? 0.f : real / l;
      put_ml(t, rows.m[t], l);
      if (none) continue;
#pragma unroll
      for (int d = 0; d < NDT; ++d) put(t, d, rows.o[t][d] * inv);
    }
  } else {
    // Every group brings its outputs to the common reference and unit; each adds up its share of
    // the dimensions.
    __shared__ float s_m[KW][TR], s_l[KW][TR];
    __shared__ int s_e[KW][RW];
#pragma unroll
    for (int t = 0; t < RT; ++t)
      if (grp == 0) {
        s_m[kw][16 * (RT * rw + t) + r] = rows.m[t];
        s_l[kw][16 * (RT * rw + t) + r] = rows.l[t][0];
      }
    if (lane == 0) s_e[kw][rw] = rows.E;
    __syncthreads();
    int E = -100;
#pragma unroll
    for (int v = 0; v < KW; ++v) E = max(E, s_e[v][rw]);
    const float unit = rows.E < -100 ? 0.f : ldexpf(1.f, rows.E - E), real = pow2i(E);
    f32x4* s_o = reinterpret_cast<f32x4*>(s_buf);
    auto slot = [&](int v, int t, int d) { return (((v * RW + rw) * RT + t) * NDT + d) * 64 + lane; };
    float lsum[RT], mall[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int i = 16 * (RT * rw + t) + r;
      float mx = -INFINITY;
#pragma unroll
      for (int v = 0; v < KW; ++v) mx = fmaxf(mx, s_m[v][i]);
      const float base = mx == -INFINITY ? 0.f : mx;
      lsum[t] = 0.f;
#pragma unroll
      for (int v = 0; v < KW; ++v) lsum[t] += s_l[v][i] * __builtin_amdgcn_exp2f(s_m[v][i] - base);
      mall[t] = mx;
      const float f = __builtin_amdgcn_exp2f(rows.m[t] - base) * unit;
#pragma unroll
      for (int d = 0; d < NDT; ++d) {
        rows.o[t][d] *= f;
        if (d / (NDT / KW) != kw) s_o[slot(kw, t, d)] = rows.o[t][d];
      }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (rows.row[t] < 0) continue;
      const float inv = lsum[t] == 0.f ? 0.f : real / lsum[t];
      put_ml(t, mall[t], lsum[t]);
      if (none) continue;
#pragma unroll
      for (int d = 0; d < NDT; ++d) {
        if (d / (NDT / KW) != kw) continue;
        f32x4 x = rows.o[t][d];
#pragma unroll
        for (int v = 0; v < KW; ++v)
          if (v != kw) x += s_o[slot(v, t, d)];
        put(t, d, x * inv);
      }
    }
  }
}

// Join the key parts of one (row, query head) pair, each normalised by itself: one wave each, in
// order of the parts.
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
  const float wgt = __builtin_amdgcn_exp2f(ms - (mx == -INFINITY ? 0.f : mx)) * ls;
  const float lsum = wave_sum(wgt);
  constexpr int PER = DH / 64;
  float acc[PER] = {};
  const uint64_t parts = __ballot(!(ls == 0.f));  // the others have no outputs
  constexpr int kBatch = 8;
  for (int s0 = 0; s0 < ns; s0 += kBatch) {
    float x[kBatch][PER];
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
#pragma unroll
      for (int e = 0; e < PER; ++e)
        x[u][e] = (parts >> (s0 + u) & 1) ? a.part_o[((s0 + u) * pairs + pair) * DH + PER * lane + e] : 0.f;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float f = __shfl(wgt, (s0 + u) & 63);
#pragma unroll
      for (int e = 0; e < PER; ++e) acc[e] += (parts >> (s0 + u) & 1) ? f * x[u][e] : 0.f;
    }
  }
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
  uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.out_stride + head * DH + PER * lane;
  if constexpr (PER == 2)
    *(uint32_t*)out = pack2<T>(acc[0] * inv, acc[1] * inv);
  else
    *out = (uint16_t)pack2<T>(acc[0] * inv, 0.f);
}

// The shapes: 0: 16 rows, four key groups; 1: 32 rows, two; 2: 64 rows, one; 3: 256 rows, one.
static constexpr int kShapeRows[] = {16, 32, 64, 256}, kShapeKeys[] = {256, 128, 64, 64};

PagedAttnPlan paged_attention_plan(const sbd_paged_kv& c, int batch, int rows, int n_q, int max_kv) {
  PagedAttnPlan p{};
  const int64_t pairs = (int64_t)rows * (n_q / c.n_kv_heads);
  const int64_t each = (pairs + batch - 1) / batch;  // of a sequence, on average
  p.shape = pairs / 256 * c.n_kv_heads >= 128 ? 3 : each <= 16 ? 0 : each <= 32 ? 1 : 2;
  const int tr = kShapeRows[p.shape], round = kShapeKeys[p.shape];
  p.rowblocks = pairs / tr + batch;
  const int64_t groups = std::max<int64_t>(1, batch * ((each + tr - 1) / tr) * c.n_kv_heads);
  const int64_t want = p.shape == 3 ? 1 : ((p.shape == 0 ? 256 : 512) + groups - 1) / groups;
  p.n_splits = (int)std::max<int64_t>(1, std::min<int64_t>({want, 64, (max_kv + round - 1) / round}));
  p.split_keys = ((max_kv + p.n_splits - 1) / p.n_splits + round - 1) / round * round;
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
  auto go = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3((unsigned)threads), 0, s, a);
  };
  switch (a.plan.shape) {
    case 0: go(paged_attn_kernel<T, DH, 1, 1, 4, 2>, 256); break;
    case 1: go(paged_attn_kernel<T, DH, 1, 2, 2, 2>, 256); break;
    case 2: go(paged_attn_kernel<T, DH, 1, 4, 1, 4>, 256); break;
    default: go(paged_attn_kernel<T, DH, 2, 8, 1, 4>, 512); break;
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
