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
constexpr int kUnits = 256;          // runs of 16 keys whose pages and exponents are in LDS at once
constexpr float kLift = 11.f, kSlack = 4.f;

namespace {

// Any byte of w an e4m3 NaN (0x7f or 0xff)
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// 16 bytes a lane from base + off, or from p, to 1 KB of LDS.
__device__ __forceinline__ void copy16(const uint8_t* base, uint32_t off, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(lds), "v"(off), "s"(base)
      : "memory", "m0");
}
__device__ __forceinline__ void copy16(const uint8_t* p, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off"
      :
      : "s"(lds), "v"(p)
      : "memory", "m0");
}

// Largest of the four lanes r, r + 16, r + 32, r + 48, in each of them.
__device__ __forceinline__ int max_of_groups(int v) {
  auto p = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
  v = max((int)p[0], (int)p[1]);
  p = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
  return max((int)p[0], (int)p[1]);
}
__device__ __forceinline__ float max_of_groups(float v) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// The larger of m and x, m where x is NaN (m is not).  fmaxf would first quiet x by an instruction of its own.
__device__ __forceinline__ float larger(float m, float x) { return __builtin_amdgcn_fmed3f(m, x, INFINITY); }

// A run of 16 keys: where its page's codes of this KV head begin (page 0's where the table names
// none: page is -1 then) and its exponents.
struct Unit {
  int64_t at;
  int page;
  int16_t ke, ve;
};

// Keys of a part: every sequence is split evenly, whatever lengths the call expected (parts of one
// length for all, as long as the longest sequence needs: 32 sequences of 512 to 4104 keys 62 us
// instead of 53, and twice that where the call did not know how long they are).  Two stages at
// least: 4 sequences x 16 rows x 2016 keys take 27 us in 32 parts, 19 in 8.
__device__ __forceinline__ int split_len(int kv, int n_splits) {
  const int even = (int)(((int64_t)kv + n_splits - 1) / n_splits);
  return max(2 * kStage, (even + kStage - 1) / kStage * kStage);
}

// One sequence and KV head as a workgroup sees it.
struct Seq {
  int b, r0, n, kv, nc;
  int g, G, pshift;
  int64_t block;  // the workgroup's among the sequence's row blocks
};
// The sequence of row block `block` of tr rows: every row_start[b] * G / tr + b begins one.  What
// is known about up to 64 sequences is read at once, before it is known which of them it is.
__device__ __forceinline__ Seq find_seq(const PagedAttnArgs& a, int64_t block, int tr, int g) {
  Seq q;
  q.g = g;
  q.G = a.n_q / a.c.n_kv_heads;
  q.pshift = 31 - __builtin_clz(a.c.page_size);
  auto start = [&](int r0, int b) { return (int64_t)r0 * q.G / tr + b; };
  int lo = 0, n = a.batch;
  narrow_sequence(lo, n, block, [&](int b) { return start(a.row_start[b], b); });
  const int lane = threadIdx.x & 63, mine = lo + min(lane, n - 1);
  const int r0 = a.row_start[mine], r1 = a.row_start[mine + 1], kv = a.kv_len[mine];
  const int nc = a.n_causal ? a.n_causal[mine] : INT32_MAX;
  const int c = max(1, (int)__popcll(__ballot(lane < n && start(r0, mine) <= block))) - 1;
  q.b = __builtin_amdgcn_readlane(mine, c);
  q.r0 = __builtin_amdgcn_readlane(r0, c);
  q.n = __builtin_amdgcn_readlane(r1, c) - q.r0;
  q.kv = min(max(__builtin_amdgcn_readlane(kv, c), 0), a.max_pages << q.pshift);
  q.nc = __builtin_amdgcn_readlane(nc, c);
  q.block = block - start(q.r0, q.b);
  if (q.kv < q.n) q.kv = 0;  // not served: no row sees a key
  return q;
}

__device__ __forceinline__ void load_pages(const PagedAttnArgs& a, const Seq& q, int key0, int units, Unit* out) {
  const int* table = a.table + (int64_t)q.b * a.max_pages;
  for (int t = threadIdx.x; t < units; t += blockDim.x) {
    const int p = table[min((key0 + 16 * t) >> q.pshift, a.max_pages - 1)];
    const bool known = (unsigned)p < (unsigned)a.c.n_pages;
    out[t].page = known ? p : -1;
    out[t].at = ((int64_t)(known ? p : 0) * a.c.n_kv_heads + q.g) * a.c.page_size * a.c.head_dim;
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

  // Copies w, w + RW, ... of a stage (units: its four runs; key: its first key) into `lds`.
  // A copy of K lies in one run; of V it holds 16 dimensions of all four.
  template <int RW>
  __device__ __forceinline__ static void copy(const PagedAttnArgs& a, const Unit* units, int key, int w, uint32_t lds) {
    constexpr int kHalf = kCopies / 2, kEach = RW <= kHalf ? kHalf / RW : 1;
    const int lane = threadIdx.x & 63, P = a.c.page_size;
    if (RW <= kHalf || w < kHalf) {
#pragma unroll
      for (int n = 0; n < kEach; ++n) {
        const int i = w + RW * n, piece = 64 * i + lane, row = piece / (DH / 16), c = (piece % (DH / 16)) ^ ksw(row);
        const int run = 64 * i / (DH / 16) / 16;
        const int64_t at = units[run].at + ((key + 16 * run) & (P - 1)) * DH;
        const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)at) |
                              (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32;
        copy16(a.c.k_codes + base, (uint32_t)((row & 15) * DH + c * 16), __builtin_amdgcn_readfirstlane(lds + i * 1024));
      }
    }
    if (RW <= kHalf || w >= kHalf) {
      const int u = (lane & 3) ^ ((lane >> 3) & 3), first = RW <= kHalf ? w : w - kHalf;
      const uint8_t* v = a.c.v_codes + units[u].at + (16 * first + (lane >> 2)) * P + ((key + 16 * u) & (P - 1));
#pragma unroll
      for (int n = 0; n < kEach; ++n)
        copy16(v + 16 * RW * n * P, __builtin_amdgcn_readfirstlane(lds + (kHalf + first + RW * n) * 1024));
    }
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
    if (__builtin_expect(edge, 0)) {
      asm volatile("");  // a branch, not selects in every stage
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
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = larger(top, s[t][u][i]);
      top = max_of_groups(top * ke);
      mn[t] = top > m[t] + kSlack || m[t] == -INFINITY ? fmaxf(top, m[t]) : m[t];
      up |= mn[t] != m[t];
    }
    const int vtop = __builtin_amdgcn_readfirstlane(max(max_of_groups(ve), -100));
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

// A workgroup has RW waves with 16 RT rows each that share two stage buffers, one barrier a stage:
// one stage is on its way while the other is used.  What hides the latency of both is the number
// of workgroups on a CU, so LDS is kept small (36 KB at head_dim 128): with rings of four buffers
// and half the workgroups 32 sequences x 8 rows x 2312 keys took 79 us instead of 48.  The keys
// are split over workgroups where the rows do not fill the chip.  Where there are many rows two
// tiles a wave share the conversion of the codes (3 prompts of 2500 rows: 230 us, one tile 244).  The
// bound of two waves a SIMD keeps the accumulators out of the other half of the registers (32 ragged
// sequences: 47.9 us, 49.6 without).
template <class T, int DH, int RT, int RW>
__global__ __launch_bounds__(64 * RW, 2) void paged_attn_kernel(PagedAttnArgs a) {
  using L = Tiles<DH>;
  constexpr int NDT = DH / 16, TR = 16 * RT * RW, NB = 2;
  constexpr int kEach = L::kCopies / RW;  // copies of a wave and stage
  static_assert(kEach * RW == L::kCopies, "whole copies");
  __shared__ __attribute__((aligned(1024))) uint8_t s_buf[NB * L::kBytes];
  __shared__ Unit s_unit[kUnits];
  __shared__ int s_kmax[RW];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4;
  const int H = a.c.n_kv_heads;
  const int g = blockIdx.x % H, item = blockIdx.x / H;
  const int split = item % a.plan.n_splits;
  const int rb_all = (int)(a.plan.rowblocks - 1 - item / a.plan.n_splits);  // the last rows, which see most keys, first
  const Seq sq = find_seq(a, rb_all, TR, g);
  if (sq.r0 < 0 || sq.n <= 0 || sq.block < 0 || sq.block * TR >= (int64_t)sq.n * sq.G) return;
  Rows<T, DH, RT> rows;
  rows.init(a, sq, sq.block * TR + 16 * RT * w);
  if (lane == 0) s_kmax[w] = rows.kmax;
  __syncthreads();
  int kmax = 0;
#pragma unroll
  for (int i = 0; i < RW; ++i) kmax = max(kmax, s_kmax[i]);
  const int len = split_len(sq.kv, a.plan.n_splits);
  const int k0 = (int)min((int64_t)split * len, (int64_t)kmax);
  const int k1 = (int)min((int64_t)k0 + len, (int64_t)kmax);

  bool flipped = a.scale_log2 >= 0.f;
  for (int seg = k0; seg < k1; seg += 16 * kUnits) {
    const int end = min(seg + 16 * kUnits, k1), stages = (end - seg + kStage - 1) / kStage;
    if (seg != k0) __syncthreads();
    load_pages(a, sq, seg, 4 * stages, s_unit);
    __syncthreads();
    // stage i goes to buffer i % NB; behind the last one it is brought again
    auto copy = [&](int i) {
      const int st = min(i, stages - 1);
      L::template copy<RW>(a, s_unit + 4 * st, seg + kStage * st, w, lds_addr(s_buf) + i % NB * L::kBytes);
    };
#pragma unroll
    for (int i = 0; i < NB - 1; ++i) copy(i);
    load_exponents(a, sq, 4 * stages, s_unit);
    if (!flipped) rows.flip();
    flipped = true;
    for (int i = 0; i < stages; ++i) {
      vm_wait<(NB - 2) * kEach>();  // this wave's copies of stage i have landed
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      copy(i + NB - 1);  // into the buffer of stage i - 1, which every wave has read
      const int ks = seg + kStage * i;
      if (ks < rows.kmax) rows.stage(s_buf + i % NB * L::kBytes, ks, s_unit[4 * i + grp], fabsf(a.scale_log2));
    }
    vm_wait<0>();
  }

  const bool last = a.plan.n_splits == 1;
  const float real = pow2i(max(rows.E, -100));
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (rows.row[t] < 0) continue;
    const int64_t part = ((int64_t)split * a.rows + rows.row[t]) * a.n_q + rows.head[t];
    const float l = rows.l[t][0], inv = l == 0.f ? 0.f : real / l;
    if (!last && grp == 0) {
      a.part_ml[2 * part] = rows.m[t];
      a.part_ml[2 * part + 1] = l;
    }
    if (!last && k0 >= k1) continue;  // the join leaves out parts whose sum is 0
#pragma unroll
    for (int d = 0; d < NDT; ++d) {
      const f32x4 x = rows.o[t][d] * inv;
      const int dim = 16 * d + 4 * grp;
      if (last)
        store_out<T>(a, rows.row[t], rows.head[t] * DH + dim, x);
      else
        *(f32x4*)(a.part_o + part * DH + dim) = x;
    }
  }
}

// Join the key parts of one (row, query head) pair, each normalised by itself: one wave each, in
// order of the parts.
template <class T, int DH, int kBatch>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PagedAttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t pairs = (int64_t)a.rows * a.n_q;
  const int64_t pair = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (pair >= pairs) return;
  const int row = (int)(pair / a.n_q), head = (int)(pair % a.n_q);
  const bool padding = row < a.row_start[0] || row >= a.row_start[a.batch];
  const int ns = a.plan.n_splits;  // <= 64
  // Outputs are requested before the sums that tell which parts have some are there.
  constexpr int PER = DH / 64;
  typedef float Part __attribute__((ext_vector_type(PER)));
  Part x[kBatch];
  auto load = [&](int s0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (s0 + u < ns) x[u] = *(const Part*)(a.part_o + ((s0 + u) * pairs + pair) * DH + PER * lane);
  };
  load(0);
  float ms = -INFINITY, ls = 0.f;
  if (lane < ns) {
    ms = a.part_ml[2 * (lane * pairs + pair)];
    ls = a.part_ml[2 * (lane * pairs + pair) + 1];
  }
  const float mx = wave_max(ms);
  const float wgt = __builtin_amdgcn_exp2f(ms - (mx == -INFINITY ? 0.f : mx)) * ls;
  const float lsum = wave_sum(wgt);
  float acc[PER] = {};
  const uint64_t parts = __ballot(!(ls == 0.f));  // the others have no outputs
  for (int s0 = 0; s0 < ns; s0 += kBatch) {
    if (s0 > 0) load(s0);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float f = __shfl(wgt, s0 + u);
#pragma unroll
      for (int e = 0; e < PER; ++e) acc[e] += (s0 + u < ns && (parts >> (s0 + u) & 1)) ? f * x[u][e] : 0.f;
    }
  }
  if (padding) return;
  const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
  uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.out_stride + head * DH + PER * lane;
  if constexpr (PER == 2)
    *(uint32_t*)out = pack2<T>(acc[0] * inv, acc[1] * inv);
  else
    *out = (uint16_t)pack2<T>(acc[0] * inv, 0.f);
}

// Workgroups that a call is split into where it has fewer: four a CU.  Half as many are as fast where
// lengths are equal (32 sequences x 8 rows x 2312 keys: 51 us, 50 with four a CU) and leave CUs
// idle behind ragged ones; twice as many write and read more partial outputs than they save (57 us).
constexpr int kWant = 1024;
// The same where a sequence has more than 64 (row, query head) pairs of a KV head: one a CU, and
// parts of 1024 keys at least (500 rows of a prompt: 16 us in one part, 22 in two; 1000: 28, 45).
constexpr int kWantMany = 256, kPartMany = 1024;
// Keys of a part at least elsewhere: 256, or 128 where that leaves CUs without work (16 rows over
// 8208 keys: 18 us in parts of 256, 23 of 128; over 2064 keys: 13.8 and 13.0).
constexpr int kPart = 256, kPartFew = 128;
// Rows of a workgroup of each shape.  The smallest shape that holds a sequence's rows is taken, so
// that its keys are read once; the last one from 512 workgroups on, two a CU (the third and the last:
// a prompt of 1000 rows, 250 workgroups, 27 and 36 us; of 2500, 625, 89 and 84; of 4000, 1000, 197
// and 182; 8 x 128 rows over 2128 keys, 256, 86 and 93; 16 x 128, 512, 118 and 100).
static constexpr int kShapeRows[] = {16, 32, 64, 128};

PagedAttnPlan paged_attention_plan(const sbd_paged_kv& c, int batch, int rows, int n_q, int max_kv) {
  PagedAttnPlan p{};
  const int64_t pairs = (int64_t)rows * (n_q / c.n_kv_heads);
  const int64_t each = (pairs + batch - 1) / batch;  // of a sequence, on average
  p.shape = pairs / 128 * c.n_kv_heads >= 512 && each > 64 ? 3 : each <= 16 ? 0 : each <= 32 ? 1 : 2;
  const int tr = kShapeRows[p.shape];
  p.rowblocks = pairs / tr + batch;
  const int64_t groups = std::max<int64_t>(1, batch * ((each + tr - 1) / tr) * c.n_kv_heads);
  const bool many = each > 64;
  const int64_t want = ((many ? kWantMany : kWant) + groups - 1) / groups;
  const int64_t part = many ? kPartMany : groups * ((max_kv + kPart - 1) / kPart) >= 256 ? kPart : kPartFew;
  p.n_splits = (int)std::max<int64_t>(1, std::min<int64_t>({want, 64, (max_kv + part - 1) / part}));
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
    case 0: go(paged_attn_kernel<T, DH, 1, 1>, 64); break;
    case 1: go(paged_attn_kernel<T, DH, 1, 2>, 128); break;
    case 2: go(paged_attn_kernel<T, DH, 1, 4>, 256); break;
    default: go(paged_attn_kernel<T, DH, 2, 4>, 256); break;
  }
  if (a.plan.n_splits > 1) {
    const dim3 join((unsigned)(((int64_t)a.rows * a.n_q + 3) / 4));
    if (a.plan.n_splits <= 4)
      hipLaunchKernelGGL((paged_attn_join_kernel<T, DH, 4>), join, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((paged_attn_join_kernel<T, DH, 16>), join, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, int dtype, hipStream_t s) {
  if (a.c.head_dim == 128) return dtype == SBD_TYPE_BF16 ? launch_dh<Bf16, 128>(a, s) : launch_dh<Fp16, 128>(a, s);
  return dtype == SBD_TYPE_BF16 ? launch_dh<Bf16, 64>(a, s) : launch_dh<Fp16, 64>(a, s);
}

}  // namespace sbd
