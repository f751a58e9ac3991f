// Attention over the paged 8-bit cache (included by attention.hip).
//
// o = sum_t softmax_t(scale q . k_t) v_t over the keys t a row sees, with
// k_t = ks[t / 16] * code and v_t likewise.  A workgroup has TW x PW waves: wave
// (tw, pw) owns RG groups of 16 rows (row = (token row j, query head g of the kv
// head's group)) and every PW-th page of the split; the PW waves of a row tile
// merge their running softmax states through LDS at the end.  K and V bytes go
// from memory to registers without LDS, the next page's while this one is
// worked on.
//
// Per page a wave computes S^T = K Q^T (codes converted to bf16, exact; fp32
// queries as three bf16 parts, so their 24 bits are all there) and O^T += V^T P^T
// (codes converted to fp16, exact; probabilities rounded to fp16, fp32 rows as
// two fp16 parts).  Tile row m of key tile kt is key 16 (m / 4) + 4 kt + m % 4, so
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
  int rg;                    // 16-row groups of a workgroup's row tile
  int tiles;                 // row tiles of the longest sequence
  int split_pages, nsplit;
};
constexpr int KV8_WAVES = 4; // page waves of a workgroup

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
  const int a = p.row_start[s], b = p.row_start[s + 1], len = p.kv_len[s];
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

// a lane's eight query channels as bf16 parts (fp32: three, which hold its 24 bits)
template <typename T, int NQ>
__device__ __forceinline__ void kv8_query(const T* src, u32x4_t (&out)[NQ]) {
  if constexpr (sizeof(T) == 2) {
    out[0] = *(const gu4*)src;
  } else {
    float x[8];
    Run4<float>::load(src, x);
    Run4<float>::load(src + 4, x + 4);
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t u = f2bf2(x[2 * e], x[2 * e + 1]);
        out[n][e] = u;
        x[2 * e] -= bf2f(u & 0xFFFF);
        x[2 * e + 1] -= bf2f(u >> 16);
      }
  }
}

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
template <int DT, int NP>
__device__ __forceinline__ void kv8_softmax(const f32x4_t (&sc)[4], bool edge, int key16, int lim, float c, float ev,
                                            float inv, float& M, float& l, f32x4_t (&o)[DT], u32x4_t (&pa)[2][NP]) {
  constexpr float HEAD = 8.f, SLACK = 7.f;
  float t[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) t[e] = sc[e >> 2][e & 3];
  if (edge) {
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
    sum += t[e];
  }
  l = fmaf(sum, inv, l);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float& u0 = t[8 * h + 2 * e];
        float& u1 = t[8 * h + 2 * e + 1];
        const uint32_t u = pk_f16(u0, u1);
        pa[h][n][e] = u;
        if (n + 1 < NP) {
          const f16x2_t y = __builtin_bit_cast(f16x2_t, u);
          u0 -= (float)y[0];
          u1 -= (float)y[1];
        }
      }
}

// NaN values of an edge page: an output channel becomes NaN in the rows that see
// such a key, found as a product of ones (a NaN; a key that the row sees).
template <int DT, int RG>
__device__ __forceinline__ void kv8_nan_values(const u32x4_t* vl, int key16, int lim_last, const int (&lim)[RG],
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
      u32x4_t u = kv8_clear_from(vl[d * 64], key16, lim_last);
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

// Merges the states of the PW page waves, halves at a time, through LDS (kv8_smem,
// (PW / 2) RG (DH / 4 + 2) 256 bytes; every wave is done with what it held), and
// stores wave 0's: the output where the rows have one split, else a partial.
template <typename T, int DH, int RG, int PW>
__device__ __forceinline__ void kv8_finish(const Kv8AttnParams& p, const Kv8Split& sp, const Kv8Rows& rows, int s, int kvh,
                                           int split, int nact, int R, int r0, int pw, float* smem, float (&M)[RG],
                                           float (&l)[RG], f32x4_t (&o)[RG][DH / 16]) {
  constexpr int DT = DH / 16, REC = (DT * 4 + 2) * 64;   // floats of a row group's state, register by register
  const int lane = threadIdx.x & 63, g = lane >> 4, m16 = lane & 15;
  const int Hkv = p.c.Hkv, G = p.Hq / Hkv;
#pragma unroll
  for (int x = 0; x < RG; ++x) {               // the row's sum over the lane groups
    float a, b;
    pair16(l[x], a, b);
    pair32(a + b, a, b);
    l[x] = a + b;
  }
  __syncthreads();
#pragma unroll
  for (int half = PW / 2; half >= 1; half >>= 1) {
    float* st = smem + (size_t)(pw % half) * RG * REC + lane;
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
  if (pw != 0) return;
#pragma unroll
  for (int x = 0; x < RG; ++x) {
    const int r = r0 + x * 16 + m16;
    if (r - m16 >= R) break;                   // uniform
    if (nact == 1) {
      if (r >= R) continue;
      const int j = r / G, col = (kvh * G + r - j * G) * DH + 4 * g;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = l[x] == 0.f ? 0.f : o[x][d][e] / l[x];
        kv8_store4<T>(p, rows.start + j, col + d * 16, y);
      }
    } else {
      const size_t idx = (((size_t)s * Hkv + kvh) * sp.tiles * RG + r / 16) * sp.nsplit + split;
      float* rec = p.part + idx * (16 * DH + 32);
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<float4*>(rec + (d * 64 + lane) * 4) = make_float4(o[x][d][0], o[x][d][1], o[x][d][2], o[x][d][3]);
      if (lane < 16) *reinterpret_cast<float2*>(rec + 16 * DH + 2 * lane) = make_float2(M[x], l[x]);
    }
  }
}

// 64 lanes x 4 bytes from base + voff to LDS bytes lds .. lds + 255
__device__ __forceinline__ void load_to_lds4(uint32_t lds, const void* base, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(voff), "s"(base)
               : "memory", "m0");
}

template <typename T, int DH, int RG>
__global__ void __launch_bounds__(256, 1) kv8_ring_kernel(Kv8AttnParams p, Kv8Split sp) {
  constexpr int PW = 4;
  constexpr int NQ = sizeof(T) == 2 ? 1 : 3;  // bf16 parts of a query
  constexpr int NP = sizeof(T) == 2 ? 1 : 2;  // fp16 parts of a probability
  constexpr int KI = DH / 64, KS = 2 * KI;    // 16-byte runs per key row and lane, k steps
  constexpr int DT = DH / 16;
  constexpr int NL = 4 * KI + DT + 2;         // loads of a page
  constexpr uint32_t SLOT = (4 * KI + DT) * 1024 + 512;   // bytes of a ring slot: keys, values, scales
  extern __shared__ __align__(16) float kv8_smem[];
  const int lane = threadIdx.x & 63, g = lane >> 4, m16 = lane & 15;
  const int pw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hkv = p.c.Hkv, G = p.Hq / Hkv;
  // kv head fastest (a page's heads are neighbours in memory), then split, row tile (last rows first), sequence
  const int kvh = blockIdx.x % Hkv;
  int rest = blockIdx.x / Hkv;
  const int split = rest % sp.nsplit;
  rest /= sp.nsplit;
  const int tile = sp.tiles - 1 - rest % sp.tiles, s = rest / sp.tiles;
  Kv8Rows rows;
  int bits;
  const bool ok_rows = kv8_rows(p, s, rows, bits);
  if (bits && tile == 0 && split == 0 && kvh == 0 && threadIdx.x == 0) set_status(p.status, bits);
  const int R = ok_rows ? rows.n * G : 0, r0 = tile * RG * 16;
  if (r0 >= R) return;                         // uniform over the workgroup
  const int lim_first = rows.limit(r0 / G, p.causal);
  const int lim_last = rows.limit((min(r0 + RG * 16, R) - 1) / G, p.causal);
  const int nact = kv8_active(lim_last, sp.split_pages);
  if (split >= nact) return;
  const int p0 = split * sp.split_pages, p1 = min(p0 + sp.split_pages, (lim_last + PAGE - 1) / PAGE);

  // the wave's pages: p0 + pw + PW i, page id i in lane i (split_pages <= 64 PW)
  const int np = p1 > p0 + pw ? (p1 - p0 - pw + PW - 1) / PW : 0;
  int pid = 0;
  if (np > 0) pid = p.page_table[(size_t)s * p.max_pages + min(p0 + pw + PW * min(lane, np - 1), p.max_pages - 1)];
  const bool bad = np > 0 && (pid < 0 || pid >= p.c.num_pages);
  if (__builtin_amdgcn_ballot_w64(bad) != 0 && lane == 0) set_status(p.status, ST_BAD_PAGE);
  if (bad) pid = -1;

  int lim[RG];                                 // of lane % 16's row (clamped rows are never stored)
  u32x4_t qf[RG][KS][NQ];
#pragma unroll
  for (int i = 0; i < RG; ++i) {
    const int r = min(r0 + i * 16 + m16, R - 1), j = r / G;
    lim[i] = rows.limit(j, p.causal);
    const T* q = reinterpret_cast<const T*>(p.q) + (size_t)(rows.start + j) * p.ld_q + (size_t)(kvh * G + r - j * G) * DH;
#pragma unroll
    for (int k = 0; k < KS; ++k)               // k step 2 c + h: channels 64 c + 16 g + 8 h ..
      kv8_query<T, NQ>(q + (k >> 1) * 64 + g * 16 + (k & 1) * 8, qf[i][k]);
  }
#pragma unroll
  for (int i = 0; i < RG; ++i)
#pragma unroll
    for (int k = 0; k < KS; ++k) asm volatile("" ::"v"(qf[i][k][0]));   // the rows are in before the ring's loads are counted

  // the wave's ring of two pages, each fragment where its lane reads it
  unsigned char* ring = reinterpret_cast<unsigned char*>(kv8_smem) + pw * 2 * SLOT;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)kv8_smem + pw * 2 * SLOT;
  const uint32_t koff = (16 * (m16 >> 2) + (m16 & 3)) * DH + g * 16, voff = lane / 16 * 16 + m16 * 64, soff = g * 4;
  auto issue = [&](int i) {
    const size_t ph = (size_t)max(__builtin_amdgcn_readlane(pid, i), 0) * Hkv + kvh;   // an invalid id reads page 0, unused
    const uint32_t l = lds0 + (i & 1) * SLOT;
    const uint8_t* kb = p.c.k + ph * PAGE * DH;
    const uint8_t* vb = p.c.v + ph * PAGE * DH;
    load_to_lds4(l + (4 * KI + DT) * 1024, p.c.ks + ph * 4, soff);
    load_to_lds4(l + (4 * KI + DT) * 1024 + 256, p.c.vs + ph * 4, soff);
    static_for<4 * KI>([&]<int N>(std::integral_constant<int, N>) {
      load_to_lds<N * 1024>(l, kb + (N / KI) * 4 * DH + (N % KI) * 64, koff);
    });
    static_for<DT>([&]<int N>(std::integral_constant<int, N>) {
      load_to_lds<(4 * KI + N) * 1024>(l, vb + N * 1024, voff);
    });
  };

  const float sl2 = p.scale * 1.4426950408889634f;
  float M[RG], l[RG];
  f32x4_t o[RG][DT];                           // channel 16 dt + 4 g + r of row lane % 16
#pragma unroll
  for (int i = 0; i < RG; ++i) {
    M[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[i][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  if (np > 0) issue(0);
  if (np > 1) issue(1);
  for (int i = 0; i < np; ++i) {
    if (i + 1 < np) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const unsigned char* slot = ring + (i & 1) * SLOT;
    const u32x4_t* kl = reinterpret_cast<const u32x4_t*>(slot) + lane;
    const u32x4_t* vl = reinterpret_cast<const u32x4_t*>(slot + 4 * KI * 1024) + lane;
    const float* scl = reinterpret_cast<const float*>(slot + (4 * KI + DT) * 1024) + lane;
    const int kp0 = (p0 + pw + PW * i) * PAGE;
    if (__builtin_amdgcn_readlane(pid, i) >= 0) {             // uniform
      const bool edge = kp0 + PAGE > lim_first;               // uniform: some row sees a part only
      f32x4_t sc[RG][4];
#pragma unroll
      for (int x = 0; x < RG; ++x)
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) sc[x][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int c = 0; c < KI; ++c) {
          const u32x4_t u = kl[(kt * KI + c) * 64];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4_t kf = h ? kv8_bf16(u[2], u[3]) : kv8_bf16(u[0], u[1]);
#pragma unroll
            for (int x = 0; x < RG; ++x)
#pragma unroll
              for (int n = NQ - 1; n >= 0; --n) sc[x][kt] = mma_frag(bf16(), kf, qf[x][2 * c + h][n], sc[x][kt]);
          }
        }
      // a group that no row sees may have any scale
      const bool seen = kp0 + 16 * g < lim_last;
      const float ksc = seen ? scl[0] : 1.f, vsc = seen ? scl[64] : 1.f;
      const float c = sl2 * ksc, ev = __builtin_amdgcn_logf(vsc), inv = 1.f / vsc;
      u32x4_t pa[RG][2][NP];
#pragma unroll
      for (int x = 0; x < RG; ++x) {
        __builtin_amdgcn_sched_barrier(0);
        kv8_softmax<DT, NP>(sc[x], edge, kp0 + 16 * g, lim[x], c, ev, inv, M[x], l[x], o[x], pa[x]);
      }
      __builtin_amdgcn_sched_barrier(0);
      uint32_t nan = 0;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        u32x4_t u = vl[d * 64];
        if (edge) {                            // NaN would pass a zero probability: taken out here, and seen to below
          u = kv8_clear_from(u, kp0 + 16 * g, lim_last);
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
      if (__builtin_amdgcn_ballot_w64(nan != 0) != 0) kv8_nan_values<DT, RG>(vl, kp0 + 16 * g, lim_last, lim, o);
    }
    if (i + 2 < np) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the slot is read
      issue(i + 2);
    }
  }
  kv8_finish<T, DH, RG, PW>(p, sp, rows, s, kvh, split, nact, R, r0, pw, kv8_smem, M, l, o);
}

// Merges the splits of one 16-row group in split order: wave d the 16 channels
// of output tile d, in the accumulator order the partials were left in.
template <typename T, int DH>
__global__ void __launch_bounds__(DH / 16 * 64) kv8_combine_kernel(Kv8AttnParams p, Kv8Split sp) {
  const int lane = threadIdx.x & 63, d = threadIdx.x >> 6;
  const int Hkv = p.c.Hkv, G = p.Hq / Hkv, rgs = sp.tiles * sp.rg;
  const int kvh = blockIdx.x % Hkv, rest = blockIdx.x / Hkv, rg = rest % rgs, s = rest / rgs;
  Kv8Rows rows;
  int bits;
  if (!kv8_rows(p, s, rows, bits)) return;
  const int R = rows.n * G;
  if (rg * 16 >= R) return;
  const int tile_end = min((rg / sp.rg + 1) * sp.rg * 16, R);
  const int nact = kv8_active(rows.limit((tile_end - 1) / G, p.causal), sp.split_pages);
  if (nact == 1) return;
  const float* rec = p.part + (((size_t)s * Hkv + kvh) * rgs + rg) * sp.nsplit * (16 * DH + 32);
  const int r = rg * 16 + (lane & 15);
  float M = -INFINITY, l = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < nact; ++i) {
    const float* ml = rec + (size_t)i * (16 * DH + 32) + 16 * DH + 2 * (lane & 15);
    const float mi = ml[0], li = ml[1];
    const float4 v = *reinterpret_cast<const float4*>(rec + (size_t)i * (16 * DH + 32) + (d * 64 + lane) * 4);
    const float mn = fmaxf(M, mi);
    const float f1 = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn);
    const float f2 = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mi - mn);
    l = l * f1 + li * f2;
    y[0] = y[0] * f1 + v.x * f2;
    y[1] = y[1] * f1 + v.y * f2;
    y[2] = y[2] * f1 + v.z * f2;
    y[3] = y[3] * f1 + v.w * f2;
    M = mn;
  }
  if (r >= R) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = l == 0.f ? 0.f : y[e] / l;
  const int j = r / G;
  kv8_store4<T>(p, rows.start + j, (kvh * G + r - j * G) * DH + d * 16 + 4 * (lane >> 4), y);
}

// Work split: 16 rows a wave up to 16 rows per kv head, 32 beyond (bf16: the
// converted keys and values serve two row groups), and of a workgroup's waves as
// many on row tiles as the rows fill, the others on pages.  Pages per split: so
// that the launch has about two workgroups per compute unit if every sequence
// reaches key_cap, at least one page per page wave.  A function of the host's
// arguments only.
inline Kv8Split kv8_split(bool bf16, int nseq, int max_rows, int key_cap, int Hq, int Hkv, int cus) {
  const long long R = (long long)max_rows * (Hq / Hkv);
  Kv8Split sp;
  sp.rg = !bf16 || R <= 16 ? 1 : (R <= 32 ? 2 : 4);
  sp.tiles = (int)((R + 16 * sp.rg - 1) / (16 * sp.rg));
  const long long items = (long long)nseq * Hkv * sp.tiles;
  const int pages = key_cap > 0 ? (key_cap + PAGE - 1) / PAGE : 1;
  const long long want = items < 2 * cus ? 2 * cus / items : 1;
  long long pp = (pages + want - 1) / want;
  if (pp < KV8_WAVES) pp = KV8_WAVES;
  if (pp > 64 * KV8_WAVES) pp = 64 * KV8_WAVES;
  sp.split_pages = (int)pp;
  sp.nsplit = (int)((pages + pp - 1) / pp);
  return sp;
}

inline size_t kv8_part_floats(const Kv8Split& sp, int nseq, int Hkv, int Dh) {
  return sp.nsplit == 1 ? 0 : (size_t)nseq * Hkv * sp.tiles * sp.rg * sp.nsplit * (16 * Dh + 32);
}

template <typename T, int DH, int RG>
static hipError_t launch_kv8_shape(const Kv8AttnParams& p, const Kv8Split& sp, hipStream_t st) {
  constexpr size_t ring = KV8_WAVES * 2 * (size_t)(DH / 8 * 1024 + 512);
  constexpr size_t merge = (size_t)(KV8_WAVES / 2) * RG * (DH / 4 + 2) * 64 * sizeof(float);
  constexpr size_t lds = ring > merge ? ring : merge;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv8_ring_kernel<T, DH, RG>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (attr != hipSuccess) return attr;
  const long long wgs = (long long)p.nseq * p.c.Hkv * sp.tiles * sp.nsplit;
  if (wgs > 0x7FFFFFFFll) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((kv8_ring_kernel<T, DH, RG>), dim3((unsigned)wgs), dim3(KV8_WAVES * 64), lds, st, p, sp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sp.nsplit == 1) return e;
  hipLaunchKernelGGL((kv8_combine_kernel<T, DH>), dim3(p.nseq * p.c.Hkv * sp.tiles * sp.rg), dim3(DH * 4), 0, st, p, sp);
  return hipGetLastError();
}

template <typename T, int DH>
static hipError_t launch_kv8_dh(const Kv8AttnParams& p, const Kv8Split& sp, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (sp.rg == 4) return launch_kv8_shape<T, DH, 4>(p, sp, st);
    if (sp.rg == 2) return launch_kv8_shape<T, DH, 2>(p, sp, st);
  }
  return launch_kv8_shape<T, DH, 1>(p, sp, st);
}

size_t kv8_attn_workspace(bool bf16, int nseq, int max_rows, int key_cap, int Hq, int Hkv, int Dh, int cus) {
  return kv8_part_floats(kv8_split(bf16, nseq, max_rows, key_cap, Hq, Hkv, cus), nseq, Hkv, Dh) * sizeof(float);
}

hipError_t launch_kv8_attention(bool bf16, const Kv8AttnParams& p, hipStream_t st) {
  if (p.nseq < 1 || p.rows < 1 || p.max_rows < 1) return hipSuccess;
  const Kv8Split sp = kv8_split(bf16, p.nseq, p.max_rows, p.key_cap, p.Hq, p.c.Hkv, p.cus);
  if (p.c.Dh == 128)
    return bf16 ? launch_kv8_dh<dflow::bf16, 128>(p, sp, st) : launch_kv8_dh<float, 128>(p, sp, st);
  if (p.c.Dh == 64)
    return bf16 ? launch_kv8_dh<dflow::bf16, 64>(p, sp, st) : launch_kv8_dh<float, 64>(p, sp, st);
  return hipErrorInvalidValue;
}

}  // namespace dflow
