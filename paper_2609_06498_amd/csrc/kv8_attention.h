// Attention over the paged 8-bit cache (included by attention.hip).
//
// o = sum_t softmax_t(scale q . k_t) v_t over the keys t a row sees, with
// k_t = ks[t / 16] * code and v_t likewise.  Rows are (token row j, query head g of the
// kv head's group) pairs, 16 to a row group.  Two kernels:
//   one row group: four waves, each with every fourth page of the split; pages go from memory to registers, the next
//     one's while this one is worked on;
//   more rows: four waves, TW row tiles x PW pages at a time; the pages go by
//     load-to-LDS to a ring that the TW waves of a page share, each 16-byte run
//     where its lane reads it; one barrier per page.
// The PW states of a row tile are merged through LDS at the end.
//
// Per page a wave computes S^T = K Q^T and O^T += V^T P^T on the matrix cores.
// Scores of bf16 queries: the key codes as they are against the query in two e4m3
// parts (see Kv8Query); of fp32 queries: codes converted to bf16, exact, against
// three bf16 parts, which hold all 24 bits.  Outputs: value
// codes converted to fp16, exact, against probabilities rounded to fp16 (fp32
// rows: two fp16 parts).  Tile row m of key tile kt is key 16 (m / 4) + 4 kt + m % 4, so
// the lanes of group g = lane / 16 hold the scores of keys 16 g .. 16 g + 15:
// one scale group.  With t = s ks + log2 vs (log2 units) the probability the
// matrix cores take is 2^(t - M), the value scale included, and the row sum adds
// it divided by vs: the scales cost one fused multiply-add operand.  M is the
// row's reference: the largest t when it last moved, less HEAD; it moves when t
// passes it by HEAD + SLACK, so that fp16 neither overflows (2^15) nor loses
// small probabilities (normal down to 2^-22 of the largest), and the rescale of
// the output is hardly ever taken.
//
// Keys a row does not see: scores are set to -inf, and values of keys that no
// row of the tile sees are cleared, since memory behind a sequence's end may
// hold NaN codes.  On pages that only some rows see in full a NaN value (its
// product with a zero probability is NaN) is taken out of the product and
// given to the rows that see it by a product of its own.
//
// A row's arithmetic depends on its own keys and the fixed page, wave and split
// boundaries only.  A split's result goes straight to the output when it is the
// row's only one, else as (M, sum, O) to the workspace; the combine kernel merges
// in split order.
#pragma once
#include "common.h"
#include "kernels.h"
#include "kv8.h"

namespace dflow {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// eight e4m3 codes (two words) as bf16 / fp16 operand fragments, exact
__device__ __forceinline__ u32x4_t kv8_bf16(uint32_t a, uint32_t b) {
  return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true))};
}
__device__ __forceinline__ u32x4_t kv8_f16(uint32_t a, uint32_t b) {
  return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true))};
}
__device__ __forceinline__ f32x4_t mma_f16(const u32x4_t& a, const u32x4_t& b, f32x4_t acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), acc, 0,
                                                0, 0);
}
__device__ __forceinline__ uint32_t pk_f16(float a, float b) {   // round to nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, f16x2_t));
}

// Work split of a launch, from the host's arguments only.
struct Kv8Split {
  int rg, tw, pw;            // 16-row groups of a wave, row tiles and pages of a workgroup's waves
  int tiles;                 // workgroup tiles (rg tw row groups) of the longest sequence
  int split_pages, nsplit;
};

// Rows of a sequence and the keys they see.
struct Kv8Rows {
  int start, n;              // rows of the sequence (n: the ones computed)
  int klen;                  // keys that may be read
  int first;                 // limit of row 0 under the causal mask, before clamping
  __device__ __forceinline__ int limit(int j, int causal) const {   // row j sees keys below this
    return causal ? min(max(first + j, 0), klen) : klen;
  }
};
__device__ __forceinline__ bool kv8_rows(const Kv8AttnParams& p, int s, Kv8Rows& r, int& bits) {
  const int a = __builtin_amdgcn_readfirstlane(p.row_start[s]), b = __builtin_amdgcn_readfirstlane(p.row_start[s + 1]);
  const int len = __builtin_amdgcn_readfirstlane(p.kv_len[s]);
  bits = 0;
  if (a < 0 || b < a || b > p.rows) {
    bits = ST_CAPACITY;
    return false;
  }
  r.start = a;
  r.n = min(b - a, p.max_rows);
  r.klen = min(max(len, 0), p.key_cap);
  if (b - a > p.max_rows || len < 0 || len > p.key_cap) bits = ST_CAPACITY;
  r.first = min(len, 1 << 30) - (b - a) + 1;
  return true;
}
// splits of the row tile whose last row sees keys below lim (one at least: it writes the rows)
__device__ __forceinline__ int kv8_active(int lim, int split_pages) {
  return max(1, ((lim + PAGE - 1) / PAGE + split_pages - 1) / split_pages);
}

template <typename T>
__device__ __forceinline__ void kv8_store4(const Kv8AttnParams& p, int row, int c, const float* y) {
  if (p.out) Run4<T>::store(reinterpret_cast<T*>(p.out) + (size_t)row * p.ld_out + c, y);
  else frag_st4<T>(p.outf, row, c, y);
}

typedef int i32x8_t __attribute__((ext_vector_type(8)));

// A row group's queries (lane % 16's row, the channels that match the lane's key
// runs: 64 c + 16 g + 0..15 of run c) and its scores against a key tile.
//
// fp32: three bf16 parts against the codes in bf16, in k steps of 32 channels.
template <typename T, int DH>
struct Kv8Query {
  static constexpr int KI = DH / 64, NQ = 3;
  u32x4_t part[2 * KI][NQ];
  __device__ __forceinline__ float scale() const { return 1.f; }
  __device__ __forceinline__ uint32_t anchor() const {   // a value that needs all loads
    uint32_t a = 0;
#pragma unroll
    for (int k = 0; k < 2 * KI; ++k) a |= part[k][0][0] | part[k][0][2];
    return a;
  }
  __device__ __forceinline__ void load(const T* row) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int k = 0; k < 2 * KI; ++k) {
      float x[8];
      const T* src = row + (k >> 1) * 64 + g * 16 + (k & 1) * 8;
      Run4<T>::load(src, x);
      Run4<T>::load(src + 4, x + 4);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t u = f2bf2(x[2 * e], x[2 * e + 1]);
          part[k][n][e] = u;
          x[2 * e] -= bf2f(u & 0xFFFF);
          x[2 * e + 1] -= bf2f(u >> 16);
        }
    }
  }
  template <int RG>
  __device__ static __forceinline__ void scores(const Kv8Query (&q)[RG], const u32x4_t (&run)[KI], f32x4_t (&acc)[RG][4],
                                                int kt) {
#pragma unroll
    for (int c = 0; c < KI; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4_t kf = h ? kv8_bf16(run[c][2], run[c][3]) : kv8_bf16(run[c][0], run[c][1]);
#pragma unroll
        for (int x = 0; x < RG; ++x)
#pragma unroll
          for (int n = NQ - 1; n >= 0; --n) acc[x][kt] = mma_frag(bf16(), kf, q[x].part[2 * c + h][n], acc[x][kt]);
      }
  }
};

// bf16: q = 2^e (hi + lo) with hi, lo in e4m3 and the row's largest magnitude brought
// to 224..448.  Eight significant bits are four and, signed, four more: exact for
// elements down to 2^-10 of the row's largest, smaller ones are off by at most
// 2^-18 of it (the subnormal step).  The key codes then go to the 128-deep e4m3
// product as they were stored: no conversions (64 of 354 vector operations a page and
// wave with bf16 operands), at the same matrix time.
template <int DH>
struct Kv8Query<bf16, DH> {
  static constexpr int KI = DH / 64;
  u32x4_t hi[KI], lo[KI];
  float s;
  __device__ __forceinline__ float scale() const { return s; }
  __device__ __forceinline__ uint32_t anchor() const { return __float_as_uint(s); }   // (s needs all loads)
  __device__ __forceinline__ void load(const bf16* row) {
    const int g = (threadIdx.x & 63) >> 4;
    float x[KI][16], top = 0.f, a, b;
#pragma unroll
    for (int c = 0; c < KI; ++c) {
      Row16<bf16>::load(row + c * 64 + g * 16, x[c]);
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(x[c][e]));
    }
    pair16(top, a, b);
    pair32(fmaxf(a, b), a, b);
    top = fmaxf(a, b);
    int e = 0;                                 // top / 2^e in 224 .. 448 (exponents whose inverse is normal too)
    if (top > 0.f && top < INFINITY) {
      const float m = frexpf(top, &e);
      e = min(max(e - 9 + (m > 0.875f ? 1 : 0), -126), 126);
    }
    s = __uint_as_float((uint32_t)(e + 127) << 23);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
    for (int c = 0; c < KI; ++c)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = x[c][4 * w + i] * inv;
        int u = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        u = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], u, true);
        hi[c][w] = (uint32_t)u;
        y[0] -= __builtin_amdgcn_cvt_f32_fp8(u, 0);
        y[1] -= __builtin_amdgcn_cvt_f32_fp8(u, 1);
        y[2] -= __builtin_amdgcn_cvt_f32_fp8(u, 2);
        y[3] -= __builtin_amdgcn_cvt_f32_fp8(u, 3);
        u = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        lo[c][w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], u, true);
      }
  }
  __device__ static __forceinline__ i32x8_t join(const u32x4_t& a, const u32x4_t& b) {
    return i32x8_t{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
  }
  __device__ static __forceinline__ f32x4_t mma(const i32x8_t& a, const i32x8_t& b, f32x4_t acc) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 0, 0, 0, 0, 0, 0);   // (scales of 0: none)
  }
  template <int RG>
  __device__ static __forceinline__ void scores(const Kv8Query (&q)[RG], const u32x4_t (&run)[KI], f32x4_t (&acc)[RG][4],
                                                int kt) {
    if constexpr (KI == 1) {                   // 64 channels: both parts in one product
      const i32x8_t k = join(run[0], run[0]);
#pragma unroll
      for (int x = 0; x < RG; ++x) acc[x][kt] = mma(k, join(q[x].lo[0], q[x].hi[0]), acc[x][kt]);
    } else {
      const i32x8_t k = join(run[0], run[1]);
#pragma unroll
      for (int x = 0; x < RG; ++x) acc[x][kt] = mma(k, join(q[x].lo[0], q[x].lo[1]), acc[x][kt]);
#pragma unroll
      for (int x = 0; x < RG; ++x) acc[x][kt] = mma(k, join(q[x].hi[0], q[x].hi[1]), acc[x][kt]);
    }
  }
};

// clears the bytes of the keys at or past lim_key of a lane's 16 (first key: key16)
__device__ __forceinline__ u32x4_t kv8_clear_from(u32x4_t v, int key16, int lim_key) {
  const int nv = lim_key - key16;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int t = min(max(nv - 4 * e, 0), 4);
    v[e] &= t == 4 ? 0xFFFFFFFFu : (1u << (8 * t)) - 1u;
  }
  return v;
}

// bytes that hold a NaN code (all low bits set), as 0xFF
__device__ __forceinline__ uint32_t kv8_nan_bytes(uint32_t u) {
  return ((((u & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xFFu;
}

// One running-softmax step of a 16-row group over a page: scores sc (key tile,
// element) of the lane's 16 keys from key16 on, its key scale (times the softmax
// scale, log2 units) c, log2 vs and 1 / vs; leaves the fp16 operands of P.
template <int DT, int NP, bool EDGE>
__device__ __forceinline__ void kv8_softmax(const f32x4_t (&sc)[4], int key16, int lim, float c, float ev,
                                            float inv, float& M, float& l, f32x4_t (&o)[DT], u32x4_t (&pa)[2][NP]) {
  constexpr float HEAD = 8.f, SLACK = 7.f;
  float t[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) t[e] = sc[e >> 2][e & 3];
  if constexpr (EDGE) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (key16 + e >= lim) t[e] = -INFINITY;
  }
  float mx = t[0], a, b;
#pragma unroll
  for (int e = 1; e < 16; ++e) mx = fmaxf(mx, t[e]);
  mx = fmaf(mx, c, ev);
  pair16(mx, a, b);
  pair32(fmaxf(a, b), a, b);
  mx = fmaxf(a, b);
  const float mn = mx - HEAD > M + SLACK ? mx - HEAD : M;
  if (__builtin_amdgcn_ballot_w64(mn != M) != 0) {   // uniform
    const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
    l *= f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[d][r] *= f;
    M = mn;
  }
  const float ref = ev - (M == -INFINITY ? 0.f : M);
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    t[e] = __builtin_amdgcn_exp2f(fmaf(t[e], c, ref));
    if (NP > 1) sum += t[e];
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float& u0 = t[8 * h + 2 * e];
        float& u1 = t[8 * h + 2 * e + 1];
        const uint32_t u = pk_f16(u0, u1);
        const f16x2_t y = __builtin_bit_cast(f16x2_t, u);
        pa[h][n][e] = u;
        // one part: the sum of the rounded values, two an operation, fp32
        if (NP == 1) sum = __builtin_amdgcn_fdot2(y, f16x2_t{(_Float16)1.f, (_Float16)1.f}, sum, false);
        if (n + 1 < NP) {
          u0 -= (float)y[0];
          u1 -= (float)y[1];
        }
      }
  l = fmaf(sum, inv, l);
}

// NaN values of an edge page: an output channel becomes NaN in the rows that see
// such a key, found as a product of ones (a NaN; a key that the row sees).
template <int DT, int RG, typename V>
__device__ __forceinline__ void kv8_nan_values(V&& vrun, int key16, int lim_last, const int (&lim)[RG],
                                               f32x4_t (&o)[RG][DT]) {
  constexpr uint32_t ONE8 = 0x38383838u, ONE16 = 0x3C00u;   // 1.0 as e4m3, as fp16
#pragma unroll
  for (int x = 0; x < RG; ++x) {
    u32x4_t sees[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = lim[x] - (key16 + 8 * h + 2 * e);   // of the two keys, those the row sees (a lane mask
        sees[h][e] = min(max(n, 0), 1) * ONE16 + min(max(n - 1, 0), 1) * (ONE16 << 16);   // each would spill)
      }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      u32x4_t u = kv8_clear_from(vrun(d), key16, lim_last);
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] = kv8_nan_bytes(u[e]) & ONE8;
      f32x4_t n = mma_f16(kv8_f16(u[0], u[1]), sees[0], f32x4_t{0.f, 0.f, 0.f, 0.f});
      n = mma_f16(kv8_f16(u[2], u[3]), sees[1], n);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        o[x][d][r] = __uint_as_float(__float_as_uint(o[x][d][r]) | min(__float_as_uint(n[r]), 1u) * 0x7FC00000u);
    }
  }
}

// What a workgroup does: its rows and its pages.
struct Kv8Item {
  int s, kvh, split, tile, G, R, nact, p0, p1;
  Kv8Rows rows;
};

// two floats of a partial, past the XCD's cache
__device__ __forceinline__ void kv8_put2(float* p, float a, float b) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a),
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 kv8_get2(const float* p) {
  const uint64_t u = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)u), __uint_as_float((uint32_t)(u >> 32)));
}

// Merges the states of a row tile's PW page waves, halves at a time, through LDS
// (TW (PW / 2) RG (DH / 4 + 2) 256 bytes; every wave is done with what it held).
// Rows with one split are stored from there; else the workgroup leaves its
// partial in the workspace.  A single row group (PW = 4): the last of its nact
// workgroups to arrive (a counter each, zero between launches) merges all of them
// in split order; partials then are written and read at device scope, since these
// workgroups may run on different XCDs, whose caches are not coherent.  (4096 keys, one
// row: 14.3 -> 11.6 us against a launch for it when added.)  More rows: the combine kernel,
// since one workgroup would read all of a tile's partials (64 rows of 32 splits: 17.4
// against 40 us).
template <typename T, int DH, int RG, int TW, int PW>
__device__ __forceinline__ void kv8_finish(const Kv8AttnParams& p, const Kv8Split& sp, const Kv8Item& it, int r0, int tw,
                                           int pw, float* smem, float (&M)[RG], float (&l)[RG],
                                           f32x4_t (&o)[RG][DH / 16]) {
  constexpr int DT = DH / 16, REC = (DT * 4 + 2) * 64;   // floats of a row group's state, register by register
  constexpr int PREC = 16 * DH + 32;                     // of a partial: outputs, then (M, l) of 16 rows
  const int lane = threadIdx.x & 63, g = lane >> 4, m16 = lane & 15;
#pragma unroll
  for (int x = 0; x < RG; ++x) {               // the row's sum over the lane groups
    float a, b;
    pair16(l[x], a, b);
    pair32(a + b, a, b);
    l[x] = a + b;
  }
  if constexpr (PW > 1) __syncthreads();
#pragma unroll
  for (int half = PW / 2; half >= 1; half >>= 1) {
    float* st = smem + (size_t)(tw * (PW / 2) + pw % half) * RG * REC + lane;
    if (pw >= half && pw < 2 * half) {
#pragma unroll
      for (int x = 0; x < RG; ++x) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) st[x * REC + (d * 4 + r) * 64] = o[x][d][r];
        st[x * REC + DT * 4 * 64] = M[x];
        st[x * REC + (DT * 4 + 1) * 64] = l[x];
      }
    }
    __syncthreads();
    if (pw < half) {
#pragma unroll
      for (int x = 0; x < RG; ++x) {
        const float m2 = st[x * REC + DT * 4 * 64], l2 = st[x * REC + (DT * 4 + 1) * 64];
        const float mn = fmaxf(M[x], m2);
        const float f1 = M[x] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M[x] - mn);
        const float f2 = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m2 - mn);
        l[x] = l[x] * f1 + l2 * f2;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[x][d][r] = o[x][d][r] * f1 + st[x * REC + (d * 4 + r) * 64] * f2;
        M[x] = mn;
      }
    }
    __syncthreads();
  }
  auto store = [&](int r, int d, const float* y, float sum) {   // channels 16 d + 4 g .. of row r
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = sum == 0.f ? 0.f : y[e] / sum;
    const int j = r / it.G;
    kv8_store4<T>(p, it.rows.start + j, (it.kvh * it.G + r - j * it.G) * DH + 16 * d + 4 * g, v);
  };
  if (it.nact == 1) {                          // uniform
    if (pw != 0) return;
#pragma unroll
    for (int x = 0; x < RG; ++x) {
      const int r = r0 + x * 16 + m16;
      if (r >= it.R) continue;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const float y[4] = {o[x][d][0], o[x][d][1], o[x][d][2], o[x][d][3]};
        store(r, d, y, l[x]);
      }
    }
    return;
  }
  constexpr bool FUSED = TW * RG == 1;
  const size_t item = ((size_t)it.s * p.c.Hkv + it.kvh) * sp.tiles + it.tile;
  float* base = p.part + KV8_COUNTERS + item * TW * RG * sp.nsplit * PREC;   // [row group][split]
  if (pw == 0) {
#pragma unroll
    for (int x = 0; x < RG; ++x) {
      if (r0 + x * 16 >= it.R) break;          // uniform
      float* rec = base + ((size_t)(tw * RG + x) * sp.nsplit + it.split) * PREC;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        float* at = rec + (d * 64 + lane) * 4;
        if constexpr (FUSED) {
          kv8_put2(at, o[x][d][0], o[x][d][1]);
          kv8_put2(at + 2, o[x][d][2], o[x][d][3]);
        } else {
          *reinterpret_cast<float4*>(at) = make_float4(o[x][d][0], o[x][d][1], o[x][d][2], o[x][d][3]);
        }
      }
      if (lane < 16) {
        if constexpr (FUSED) kv8_put2(rec + 16 * DH + 2 * lane, M[x], l[x]);
        else *reinterpret_cast<float2*>(rec + 16 * DH + 2 * lane) = make_float2(M[x], l[x]);
      }
    }
  }
  if constexpr (!FUSED) return;
  unsigned* arrive = reinterpret_cast<unsigned*>(p.part) + item;   // nsplit > 1: at most KV8_COUNTERS items
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  unsigned* flag = reinterpret_cast<unsigned*>(smem);
  if (threadIdx.x == 0) *flag = __hip_atomic_fetch_add(arrive, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (*flag != (unsigned)it.nact - 1) return;  // uniform
  if (threadIdx.x == 0) __hip_atomic_store(arrive, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  constexpr int U = 8, DU = DT / PW;           // splits at a time, output tiles of a wave
  const int d0 = pw * DU, r = r0 + m16;
  const float* rec = base;
  {
    float m = -INFINITY, sum = 0.f, y[DU][4];
#pragma unroll
    for (int d = 0; d < DU; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) y[d][e] = 0.f;
    for (int i = 0; i < it.nact; i += U) {     // (past the last split: it again, unused)
      float2 ml[U], v[U][DU][2];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float* at = rec + (size_t)min(i + u, it.nact - 1) * PREC;
        ml[u] = kv8_get2(at + 16 * DH + 2 * m16);
#pragma unroll
        for (int d = 0; d < DU; ++d) {
          v[u][d][0] = kv8_get2(at + ((d0 + d) * 64 + lane) * 4);
          v[u][d][1] = kv8_get2(at + ((d0 + d) * 64 + lane) * 4 + 2);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float mi = i + u < it.nact ? ml[u].x : -INFINITY;
        const float mn = fmaxf(m, mi);
        const float f1 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
        const float f2 = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mi - mn);
        const bool on = i + u < it.nact;       // (NaN of a partial stays NaN, an unused one adds nothing)
        sum = sum * f1 + (on ? ml[u].y * f2 : 0.f);
#pragma unroll
        for (int d = 0; d < DU; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) y[d][e] = y[d][e] * f1 + (on ? (e & 1 ? v[u][d][e / 2].y : v[u][d][e / 2].x) * f2 : 0.f);
        m = mn;
      }
    }
    if (r >= it.R) return;
#pragma unroll
    for (int d = 0; d < DU; ++d) store(r, d0 + d, y[d], sum);
  }
}

// A wave's state, and one page against it: S^T = K Q^T, a softmax step, O^T += V^T P^T.
template <typename T, int DH, int RG>
struct Kv8Wave {
  static constexpr int NP = sizeof(T) == 2 ? 1 : 2;  // fp16 parts of a probability
  static constexpr int KI = DH / 64;                 // 16-byte runs per key row and lane
  static constexpr int DT = DH / 16;
  Kv8Query<T, DH> q[RG];
  int lim[RG], lim_last;                       // keys that lane % 16's row sees, that the wave's last row sees
  float sl2;                                   // softmax scale, log2 units
  float M[RG], l[RG];
  f32x4_t o[RG][DT];                           // channel 16 dt + 4 g + r of row lane % 16

  // rows from r0 on of the sequence's R (clamped rows are never stored)
  __device__ __forceinline__ void load(const Kv8AttnParams& p, const Kv8Rows& rows, int kvh, int G, int r0, int R) {
    const int m16 = threadIdx.x & 15;
#pragma unroll
    for (int i = 0; i < RG; ++i) {
      const int r = min(r0 + i * 16 + m16, R - 1), j = r / G;
      lim[i] = rows.limit(j, p.causal);
      q[i].load(reinterpret_cast<const T*>(p.q) + (size_t)(rows.start + j) * p.ld_q + (size_t)(kvh * G + r - j * G) * DH);
      M[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[i][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    lim_last = rows.limit((min(r0 + RG * 16, R) - 1) / G, p.causal);
    sl2 = p.scale * 1.4426950408889634f;
  }

  __device__ __forceinline__ void arrived() {  // (waits for the queries)
#pragma unroll
    for (int i = 0; i < RG; ++i) asm volatile("" ::"v"(M[i]), "v"(q[i].anchor()));
  }

  // Page with first key kp0.  kk, vrun(d): the lane's 16-byte runs; ksc, vsc: its
  // group's scales; mid(): called when kk and the scales are used up, to refill
  // them for the next page.  EDGE: some row sees a part of the page only, or (ok
  // false: invalid page id) none does.
  template <bool EDGE, typename V, typename F>
  __device__ __forceinline__ void page(int kp0, bool ok, u32x4_t (&kk)[4][KI], V&& vrun, float ksc, float vsc, F&& mid) {
    const int key16 = kp0 + 16 * ((threadIdx.x & 63) >> 4);
    f32x4_t sc[RG][4];
#pragma unroll
    for (int x = 0; x < RG; ++x)
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) sc[x][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) Kv8Query<T, DH>::template scores<RG>(q, kk[kt], sc, kt);
    __builtin_amdgcn_s_setprio(1);               // (the softmax of one wave beside the other's products: 1024-row chunk 127 -> 116 us)
    int lm[RG], ll = lim_last;
#pragma unroll
    for (int x = 0; x < RG; ++x) lm[x] = lim[x];
    if constexpr (EDGE) {
      if (!ok) {                               // uniform
        ll = 0;
#pragma unroll
        for (int x = 0; x < RG; ++x) lm[x] = 0;
      }
      if (key16 >= ll) ksc = vsc = 1.f;        // a group that no row sees may have any scale
    }
    const float c = sl2 * ksc, ev = __builtin_amdgcn_logf(vsc), inv = __builtin_amdgcn_rcpf(vsc);
    u32x4_t vv[DT];                            // asked for ahead of their use, under the softmax
#pragma unroll
    for (int d = 0; d < DT; ++d) vv[d] = vrun(d);
    mid();
    __builtin_amdgcn_sched_barrier(0);
    u32x4_t pa[RG][2][NP];
#pragma unroll
    for (int x = 0; x < RG; ++x) kv8_softmax<DT, NP, EDGE>(sc[x], key16, lm[x], c * q[x].scale(), ev, inv, M[x], l[x], o[x], pa[x]);
    __builtin_amdgcn_s_setprio(0);
    uint32_t nan = 0;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      u32x4_t u = vv[d];
      if constexpr (EDGE) {                    // NaN would pass a zero probability: taken out here, and seen to below
        u = kv8_clear_from(u, key16, ll);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t b = kv8_nan_bytes(u[e]);
          nan |= b;
          u[e] &= ~b;
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4_t vf = h ? kv8_f16(u[2], u[3]) : kv8_f16(u[0], u[1]);
#pragma unroll
        for (int x = 0; x < RG; ++x)
#pragma unroll
          for (int n = NP - 1; n >= 0; --n) o[x][d] = mma_f16(vf, pa[x][h][n], o[x][d]);
      }
    }
    if constexpr (EDGE)
      if (__builtin_amdgcn_ballot_w64(nan != 0) != 0) kv8_nan_values<DT, RG>(vrun, key16, ll, lm, o);
  }
};

// false: nothing to do (uniform).  pid: the table's id of page p0 + first + step lane
__device__ __forceinline__ bool kv8_item(const Kv8AttnParams& p, const Kv8Split& sp, int tile_rows, int first, int step,
                                         Kv8Item& it, int& pid) {
  const int Hkv = p.c.Hkv;
  // kv head fastest (a page's heads are neighbours in memory), then split, row tile (last rows first), sequence
  it.kvh = blockIdx.x % Hkv;
  int rest = blockIdx.x / Hkv;
  it.split = rest % sp.nsplit;
  rest /= sp.nsplit;
  it.tile = sp.tiles - 1 - rest % sp.tiles;
  it.s = rest / sp.tiles;
  it.p0 = it.split * sp.split_pages;
  // (issued beside the lengths, which decide whether it counts)
  pid = p.page_table[(size_t)it.s * p.max_pages + min(it.p0 + first + step * (int)(threadIdx.x & 63), p.max_pages - 1)];
  it.G = p.Hq / Hkv;
  int bits;
  const bool ok = kv8_rows(p, it.s, it.rows, bits);
  if (bits && it.tile == 0 && it.split == 0 && it.kvh == 0 && threadIdx.x == 0) set_status(p.status, bits);
  it.R = ok ? it.rows.n * it.G : 0;
  const int r0 = it.tile * tile_rows;
  if (r0 >= it.R) return false;
  const int lim = it.rows.limit((min(r0 + tile_rows, it.R) - 1) / it.G, p.causal);
  it.nact = kv8_active(lim, sp.split_pages);
  it.p1 = min(it.p0 + sp.split_pages, (lim + PAGE - 1) / PAGE);
  return it.split < it.nact;
}
// A wave's pages p0 + first + step i, i < np: their ids 64 at a time, a lane
// each, taken in order; page i's validity stays known until page i + 32 is taken.
struct Kv8Pages {
  int pid, np;
  uint32_t ok;
  bool any_bad;                                // some page has an invalid id
  __device__ __forceinline__ void load(const Kv8AttnParams& p, const Kv8Item& it, int i, int first, int step) {
    pid = p.page_table[(size_t)it.s * p.max_pages + min(it.p0 + first + step * (i + (int)(threadIdx.x & 63)), p.max_pages - 1)];
  }
  __device__ __forceinline__ bool check(const Kv8AttnParams& p, int i0) {   // invalid ids become -1
    const bool bad = i0 + (int)(threadIdx.x & 63) < np && (pid < 0 || pid >= p.c.num_pages);
    if (bad) pid = -1;
    return __builtin_amdgcn_ballot_w64(bad) != 0;
  }
  __device__ __forceinline__ Kv8Pages(const Kv8AttnParams& p, const Kv8Item& it, int pid0, int n, int first, int step)
      : pid(pid0), np(n), ok(0), any_bad(false) {
    if (np > 64) {                             // uniform
      for (int i = (np - 1) & ~63; i > 0; i -= 64) {
        load(p, it, i, first, step);
        any_bad |= check(p, i);
      }
      pid = pid0;
    }
    any_bad |= check(p, 0);
    if (any_bad && (threadIdx.x & 63) == 0) set_status(p.status, ST_BAD_PAGE);
  }
  // id of page i (0 for an invalid one: read, and not used)
  __device__ __forceinline__ int take(const Kv8AttnParams& p, const Kv8Item& it, int i, int first, int step) {
    if (i > 0 && (i & 63) == 0) {              // uniform
      load(p, it, i, first, step);
      (void)check(p, i);
    }
    const int v = __builtin_amdgcn_readlane(pid, i & 63);
    const uint32_t bit = 1u << (i & 31);
    ok = v >= 0 ? ok | bit : ok & ~bit;
    return max(v, 0);
  }
  __device__ __forceinline__ bool valid(int i) const { return ok >> (i & 31) & 1; }
};

template <typename T, int DH>
__global__ void __launch_bounds__(256, 2) kv8_direct_kernel(Kv8AttnParams p, Kv8Split sp) {
  constexpr int PW = 4, RG = 1;
  typedef Kv8Wave<T, DH, RG> W;
  extern __shared__ __align__(16) float kv8_smem[];
  const int lane = threadIdx.x & 63, g = lane >> 4, m16 = lane & 15;
  const int pw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Kv8Item it;
  int pid;
  if (!kv8_item(p, sp, RG * 16, pw, PW, it, pid)) return;
  const int Hkv = p.c.Hkv, r0 = it.tile * RG * 16, pbase = it.p0 + pw;
  const int np = it.p1 > pbase ? (it.p1 - pbase + PW - 1) / PW : 0;   // pages pbase + PW i
  Kv8Pages pages(p, it, pid, np, pw, PW);
  u32x4_t kr[4][W::KI], vr[W::DT];
  size_t ph = 0;                               // (page, head) block of the last page asked for
  float ksn, vsn;
  const uint32_t koff = (16 * (m16 >> 2) + (m16 & 3)) * DH + g * 16, voff = m16 * 64 + g * 16;
  auto issue_k = [&](int i) {
    ph = (size_t)pages.take(p, it, i, pw, PW) * Hkv + it.kvh;
    const uint8_t* kb = p.c.k + ph * PAGE * DH;
    ksn = *(const gf32*)(p.c.ks + ph * 4 + g);
    vsn = *(const gf32*)(p.c.vs + ph * 4 + g);
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int c = 0; c < W::KI; ++c) kr[kt][c] = *(const gu4*)(kb + 4 * kt * DH + c * 64 + koff);
  };
  auto issue_v = [&]() {
    const uint8_t* vb = p.c.v + ph * PAGE * DH;
#pragma unroll
    for (int d = 0; d < W::DT; ++d) vr[d] = *(const gu4*)(vb + d * 1024 + voff);
  };
  if (np > 0) {
    issue_k(0);
    issue_v();
  }
  W w;
  w.load(p, it.rows, it.kvh, it.G, r0, it.R);
  const int lim_first = it.rows.limit(r0 / it.G, p.causal);
  auto step = [&]<bool EDGE>(int i, std::integral_constant<bool, EDGE>) {
    w.template page<EDGE>((pbase + PW * i) * PAGE, pages.valid(i), kr, [&](int d) { return vr[d]; }, ksn, vsn, [&]() {
      if (i + 1 < np) issue_k(i + 1);
    });
    if (i + 1 < np) issue_v();
  };
  // whole pages first, then those that some row sees in part (all, if an id is invalid)
  const int full = pages.any_bad ? 0 : min(np, max(0, (lim_first / PAGE - pbase + PW - 1) / PW));
  int i = 0;
  for (; i < full; ++i) step(i, std::integral_constant<bool, false>());
  for (; i < np; ++i) step(i, std::integral_constant<bool, true>());
  kv8_finish<T, DH, RG, 1, PW>(p, sp, it, r0, 0, pw, kv8_smem, w.M, w.l, w.o);
}

// 64 lanes x 4 bytes from base + voff to LDS bytes lds .. lds + 255
__device__ __forceinline__ void load_to_lds4(uint32_t lds, const void* base, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(voff), "s"(base)
               : "memory", "m0");
}

// Four waves and up to 80 KB of LDS, so that two workgroups, at no fixed distance
// from each other, share a compute unit: one's matrix operations run beside the
// other's softmax.
// Ring slots of a page: with one page at a time four, and the next page's keys
// are read ahead; with two pages two.
constexpr int KV8_SHARED_WAVES = 4;
constexpr int kv8_slots(int pw) { return pw == 1 ? 4 : 2; }
template <int DH> constexpr uint32_t kv8_slot_bytes() { return DH / 8 * 1024 + 512; }   // keys, values, scales

template <typename T, int DH, int RG, int TW>
__global__ void __launch_bounds__(KV8_SHARED_WAVES * 64, 2) kv8_shared_kernel(Kv8AttnParams p, Kv8Split sp) {
  constexpr int PW = KV8_SHARED_WAVES / TW, NS = kv8_slots(PW);
  constexpr int AHEAD = PW == 1 ? 1 : 0;      // pages that are in beyond the present one
  static_assert(NS >= AHEAD + 2, "a slot to load while the resident ones are read");
  typedef Kv8Wave<T, DH, RG> W;
  constexpr int NR = 4 * W::KI + W::DT;       // 1 KB runs of a page: keys, then values
  constexpr int LPW = NR / TW + 2;            // loads of a wave and page (the scales by every wave)
  constexpr uint32_t SLOT = kv8_slot_bytes<DH>();
  static_assert(NR % TW == 0 && SLOT == NR * 1024 + 512, "runs split evenly over the tile waves");
  extern __shared__ __align__(16) float kv8_smem[];
  const int lane = threadIdx.x & 63, g = lane >> 4, m16 = lane & 15;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pw = wv % PW, tw = wv / PW;
  Kv8Item it;
  int pid;
  if (!kv8_item(p, sp, TW * RG * 16, pw, PW, it, pid)) return;
  const int Hkv = p.c.Hkv, r0 = (it.tile * TW + tw) * RG * 16, pbase = it.p0 + pw;
  const int np = it.p1 > pbase ? (it.p1 - pbase + PW - 1) / PW : 0;   // pages pbase + PW i
  const int steps = it.p1 > it.p0 ? (it.p1 - it.p0 + PW - 1) / PW : 0;   // of the workgroup
  Kv8Pages pages(p, it, pid, np, pw, PW);
  unsigned char* ring = reinterpret_cast<unsigned char*>(kv8_smem) + pw * NS * SLOT;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)kv8_smem + pw * NS * SLOT;
  const uint32_t koff = (16 * (m16 >> 2) + (m16 & 3)) * DH + g * 16, voff = m16 * 64 + g * 16, soff = g * 4;
  W w;
  const bool own = r0 < it.R;                  // uniform: the wave has rows (else it only helps to load)
  w.load(p, it.rows, it.kvh, it.G, r0, it.R);
  const int lim_first = it.rows.limit(min(r0, it.R - 1) / it.G, p.causal);
  w.arrived();                                 // the rows are in before the ring's loads are counted
  auto issue = [&](int i, uint32_t slot) {     // the wave's part of page i
    const size_t ph = (size_t)pages.take(p, it, i, pw, PW) * Hkv + it.kvh;
    const uint32_t l = lds0 + slot * SLOT;
    const uint8_t* kb = p.c.k + ph * PAGE * DH;
    const uint8_t* vb = p.c.v + ph * PAGE * DH;
    load_to_lds4(l + NR * 1024, p.c.ks + ph * 4, soff);
    load_to_lds4(l + NR * 1024 + 256, p.c.vs + ph * 4, soff);
    static_for<NR / TW>([&]<int N>(std::integral_constant<int, N>) {
      const int n = tw * (NR / TW) + N;        // uniform
      if (n < 4 * W::KI) load_to_lds<0>(l + n * 1024, kb + (n / W::KI) * 4 * DH + (n % W::KI) * 64, koff);
      else load_to_lds<0>(l + n * 1024, vb + (n - 4 * W::KI) * 1024, voff);
    });
  };
  for (int i = 0; i < NS - 1 && i < np; ++i) issue(i, i);
  int slot = 0;
  // Page i + AHEAD is in (its loads waited for by every wave that issued a part) and page i - 1 read by all: its slot
  // takes page i + NS - 1.
  auto begin = [&](int i) {
    if (i + NS - 1 <= np) wait_barrier<(NS - 2 - AHEAD) * LPW>();
    else wait_barrier<0>();
    if (i + NS - 1 < np) issue(i + NS - 1, slot == 0 ? NS - 1 : slot - 1);
  };
  u32x4_t kk[4][W::KI];
  float ksc, vsc;
  auto read_keys = [&](int sl) {
    const unsigned char* sb = ring + sl * SLOT;
    const u32x4_t* runs = reinterpret_cast<const u32x4_t*>(sb) + lane;
    const float* scl = reinterpret_cast<const float*>(sb + NR * 1024) + lane;
    ksc = scl[0];
    vsc = scl[64];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int c = 0; c < W::KI; ++c) kk[kt][c] = runs[(kt * W::KI + c) * 64];
  };
  auto step = [&]<bool EDGE>(int i, std::integral_constant<bool, EDGE>) {
    const u32x4_t* runs = reinterpret_cast<const u32x4_t*>(ring + slot * SLOT) + lane;
    if constexpr (!AHEAD) {
      read_keys(slot);
      __builtin_amdgcn_sched_barrier(0);
    }
    w.template page<EDGE>((pbase + PW * i) * PAGE, pages.valid(i), kk,
                          [&](int d) { return runs[(4 * W::KI + d) * 64]; }, ksc, vsc, [&]() {
                            if constexpr (AHEAD) read_keys(slot + 1 == NS ? 0 : slot + 1);   // (past the last page: unused)
                          });
  };
  auto next = [&]() { slot = slot + 1 == NS ? 0 : slot + 1; };
  // whole pages first, then those that some row sees in part (all, if an id is invalid)
  const int full = !own || pages.any_bad ? 0 : min(np, max(0, (lim_first / PAGE - pbase + PW - 1) / PW));
  int i = 0;
  if (AHEAD && steps > 0) {
    if (np >= NS - 1) wait_barrier<(NS - 2) * LPW>();
    else wait_barrier<0>();
    read_keys(0);
  }
  for (; i < full; ++i, next()) {
    begin(i);
    step(i, std::integral_constant<bool, false>());
  }
  for (; i < steps; ++i, next()) {
    begin(i);
    if (own && i < np && (pbase + PW * i) * PAGE < w.lim_last) step(i, std::integral_constant<bool, true>());   // uniform
  }
  kv8_finish<T, DH, RG, TW, PW>(p, sp, it, r0, tw, pw, kv8_smem, w.M, w.l, w.o);
}

// Merges the splits of one 16-row group in split order, U splits' loads in flight
// together: wave d the 16 channels of output tile d, in the accumulator order the
// partials were left in.  Two splits, as a prompt chunk may have, load no more than
// two (1024-row chunk: 15.6 us with eight loads, six of them the second split again,
// 10.6 with two; the whole call 116.5 -> 110).
template <typename T, int DH, int U>
__global__ void __launch_bounds__(DH / 16 * 64) kv8_combine_kernel(Kv8AttnParams p, Kv8Split sp) {
  constexpr int REC = 16 * DH + 32;
  const int lane = threadIdx.x & 63, d = threadIdx.x >> 6;
  const int Hkv = p.c.Hkv, G = p.Hq / Hkv, tile_rg = sp.tw * sp.rg, rgs = sp.tiles * tile_rg;
  const int kvh = blockIdx.x % Hkv, rest = blockIdx.x / Hkv, rg = rest % rgs, s = rest / rgs;
  const float* rec = p.part + KV8_COUNTERS + (((size_t)s * Hkv + kvh) * rgs + rg) * sp.nsplit * REC;
  const float* pv = rec + (d * 64 + lane) * 4;
  const float* pm = rec + 16 * DH + 2 * (lane & 15);
  float2 ml[U];
  float4 v[U];
  auto load = [&](int i, int last) {           // (past the last split: it again, unused)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t at = (size_t)min(i + u, last) * REC;
      ml[u] = *reinterpret_cast<const float2*>(pm + at);
      v[u] = *reinterpret_cast<const float4*>(pv + at);
    }
  };
  Kv8Rows rows;
  int bits;
  if (!kv8_rows(p, s, rows, bits)) return;
  const int R = rows.n * G;
  if (rg * 16 >= R) return;
  const int tile_end = min((rg / tile_rg + 1) * tile_rg * 16, R);
  const int nact = kv8_active(rows.limit((tile_end - 1) / G, p.causal), sp.split_pages);
  if (nact == 1) return;
  const int r = rg * 16 + (lane & 15);
  float M = -INFINITY, l = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < nact; i += U) {
    load(i, nact - 1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool on = i + u < nact;            // (NaN of a partial stays NaN, an unused one adds nothing)
      const float mi = on ? ml[u].x : -INFINITY;
      const float mn = fmaxf(M, mi);
      const float f1 = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
      const float f2 = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mi - mn);
      l = l * f1 + (on ? ml[u].y * f2 : 0.f);
      y[0] = y[0] * f1 + (on ? v[u].x * f2 : 0.f);
      y[1] = y[1] * f1 + (on ? v[u].y * f2 : 0.f);
      y[2] = y[2] * f1 + (on ? v[u].z * f2 : 0.f);
      y[3] = y[3] * f1 + (on ? v[u].w * f2 : 0.f);
      M = mn;
    }
  }
  if (r >= R) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = l == 0.f ? 0.f : y[e] / l;
  const int j = r / G;
  kv8_store4<T>(p, rows.start + j, (kvh * G + r - j * G) * DH + d * 16 + 4 * (lane >> 4), y);
}

// Work split, a function of the host's arguments only.  One row group: the direct
// kernel; more: as many row tiles of a workgroup's four waves as the rows fill,
// the other waves on pages.  Pages per split: so that the launch has about two
// workgroups per compute unit if every sequence reaches key_cap, at least two pages
// per page wave (one sequence at 4096 positions: 10.8 us a row, 15.8 a block; with
// one page 12.0 and 17.2, with four 13.1 and 17.0).  So a launch that splits has at
// most as many row tiles as compute units: KV8_COUNTERS bounds them.  A prompt's
// chunks all take the tiles of many rows and splits of KV8_PROMPT_PAGES pages.
constexpr int KV8_PROMPT_PAGES = 32;
inline Kv8Split kv8_split(bool bf16, int nseq, int max_rows, int key_cap, int Hq, int Hkv, int cus, bool prompt) {
  const long long R = (long long)max_rows * (Hq / Hkv);
  Kv8Split sp;
  sp.rg = bf16 && (R > 32 || prompt) ? 2 : 1;
  const int per = 16 * sp.rg;
  sp.tw = prompt ? 4 : (R <= per ? 1 : (R <= 2 * per ? 2 : 4));
  sp.pw = 4 / sp.tw;
  sp.tiles = (int)((R + per * sp.tw - 1) / (per * sp.tw));
  if (cus > KV8_COUNTERS) cus = KV8_COUNTERS;
  const long long items = (long long)nseq * Hkv * sp.tiles;
  const int pages = key_cap > 0 ? (key_cap + PAGE - 1) / PAGE : 1;
  const long long want = items < 2 * cus ? 2 * cus / items : 1;
  long long pp = (pages + want - 1) / want;
  if (pp < 2 * sp.pw) pp = 2 * sp.pw;
  if (prompt) pp = KV8_PROMPT_PAGES;
  sp.split_pages = (int)pp;
  sp.nsplit = (int)((pages + pp - 1) / pp);
  return sp;
}

inline size_t kv8_part_floats(const Kv8Split& sp, int nseq, int Hkv, int Dh) {
  return sp.nsplit == 1 ? 0 : KV8_COUNTERS + (size_t)nseq * Hkv * sp.tiles * sp.tw * sp.rg * sp.nsplit * (16 * Dh + 32);
}

template <auto KERNEL>
static hipError_t launch_kv8_kernel(const Kv8AttnParams& p, const Kv8Split& sp, int threads, size_t lds, hipStream_t st) {
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (attr != hipSuccess) return attr;
  const long long wgs = (long long)p.nseq * p.c.Hkv * sp.tiles * sp.nsplit;
  if (wgs > KV8_MAX_WGS) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(KERNEL, dim3((unsigned)wgs), dim3(threads), lds, st, p, sp);
  return hipGetLastError();
}
template <typename T, int DH, int U>
static hipError_t launch_kv8_combine(const Kv8AttnParams& p, const Kv8Split& sp, hipStream_t st) {
  hipLaunchKernelGGL((kv8_combine_kernel<T, DH, U>), dim3(p.nseq * p.c.Hkv * sp.tiles * sp.tw * sp.rg), dim3(DH * 4), 0, st,
                     p, sp);
  return hipGetLastError();
}

constexpr size_t kv8_merge_bytes(int DH, int RG, int TW, int PW) {
  return (size_t)TW * (PW / 2) * RG * (DH / 4 + 2) * 64 * sizeof(float);
}

template <typename T, int DH>
static hipError_t launch_kv8_direct(const Kv8AttnParams& p, const Kv8Split& sp, hipStream_t st) {
  return launch_kv8_kernel<&kv8_direct_kernel<T, DH>>(p, sp, 256, kv8_merge_bytes(DH, 1, 1, 4), st);
}
template <typename T, int DH, int RG, int TW>
static hipError_t launch_kv8_shared(const Kv8AttnParams& p, const Kv8Split& sp, hipStream_t st) {
  constexpr int PW = KV8_SHARED_WAVES / TW;
  constexpr size_t ring = (size_t)PW * kv8_slots(PW) * kv8_slot_bytes<DH>();
  constexpr size_t merge = kv8_merge_bytes(DH, RG, TW, PW);
  const hipError_t e =
      launch_kv8_kernel<&kv8_shared_kernel<T, DH, RG, TW>>(p, sp, KV8_SHARED_WAVES * 64, ring > merge ? ring : merge, st);
  if (e != hipSuccess || sp.nsplit == 1) return e;
  return sp.nsplit == 2 ? launch_kv8_combine<T, DH, 2>(p, sp, st) : launch_kv8_combine<T, DH, 8>(p, sp, st);
}

template <typename T, int DH>
static hipError_t launch_kv8_dh(const Kv8AttnParams& p, const Kv8Split& sp, hipStream_t st) {
  constexpr int RG = sizeof(T) == 2 ? 2 : 1;
  if (sp.tw == 4) return launch_kv8_shared<T, DH, RG, 4>(p, sp, st);
  if (sp.tw == 2 && sp.rg == RG) return launch_kv8_shared<T, DH, RG, 2>(p, sp, st);
  if (sp.tw == 2) return launch_kv8_shared<T, DH, 1, 2>(p, sp, st);
  return launch_kv8_direct<T, DH>(p, sp, st);
}

size_t kv8_attn_workspace(bool bf16, int nseq, int max_rows, int key_cap, int Hq, int Hkv, int Dh, int cus,
                          bool prompt) {
  return kv8_part_floats(kv8_split(bf16, nseq, max_rows, key_cap, Hq, Hkv, cus, prompt), nseq, Hkv, Dh) * sizeof(float);
}

hipError_t launch_kv8_attention(bool bf16, const Kv8AttnParams& p, hipStream_t st) {
  if (p.nseq < 1 || p.rows < 1 || p.max_rows < 1) return hipSuccess;
  const Kv8Split sp = kv8_split(bf16, p.plan_seq, p.max_rows, p.key_cap, p.Hq, p.c.Hkv, p.cus, p.prompt != 0);
  if (p.c.Dh == 128)
    return bf16 ? launch_kv8_dh<dflow::bf16, 128>(p, sp, st) : launch_kv8_dh<float, 128>(p, sp, st);
  if (p.c.Dh == 64)
    return bf16 ? launch_kv8_dh<dflow::bf16, 64>(p, sp, st) : launch_kv8_dh<float, 64>(p, sp, st);
  return hipErrorInvalidValue;
}

}  // namespace dflow
