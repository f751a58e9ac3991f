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
// row of the wave sees are cleared, since memory behind a sequence's end may
// hold NaN codes.  A NaN value that some rows see and earlier ones do not (its
// product with a zero probability is NaN) takes a row by row path.
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
  int rg, tw, pw;            // row groups per wave, row-tile waves, page waves
  int tiles;                 // row tiles of the longest sequence
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

template <typename T, int DH, int RG, int TW, int PW>
__global__ void __launch_bounds__(TW * PW * 64, 2) kv8_attn_kernel(Kv8AttnParams p, Kv8Split sp) {
  constexpr int NQ = sizeof(T) == 2 ? 1 : 3;  // bf16 parts of a query
  constexpr int NP = sizeof(T) == 2 ? 1 : 2;  // fp16 parts of a probability
  constexpr int KI = DH / 64, KS = 2 * KI;    // 16-byte loads per key row and lane, k steps
  constexpr int DT = DH / 16;
  constexpr float HEAD = 8.f, SLACK = 7.f;
  extern __shared__ __align__(16) float kv8_smem[];
  const int lane = threadIdx.x & 63, g = lane >> 4, m16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pw = w % PW, tw = w / PW;
  const int Hkv = p.c.Hkv, G = p.Hq / Hkv;
  // kv head fastest (a page's heads are neighbours in memory), then split, row tile, sequence
  const int kvh = blockIdx.x % Hkv;
  int rest = blockIdx.x / Hkv;
  const int split = rest % sp.nsplit;
  rest /= sp.nsplit;
  const int tile = rest % sp.tiles, s = rest / sp.tiles;
  Kv8Rows rows;
  int bits;
  const bool ok_rows = kv8_rows(p, s, rows, bits);
  if (bits && tile == 0 && split == 0 && kvh == 0 && threadIdx.x == 0) set_status(p.status, bits);
  const int R = ok_rows ? rows.n * G : 0, r0 = tile * TW * RG * 16;
  if (r0 >= R) return;                         // uniform over the workgroup
  const int lim_wg = rows.limit((min(r0 + TW * RG * 16, R) - 1) / G, p.causal);
  const int nact = kv8_active(lim_wg, sp.split_pages);
  if (split >= nact) return;
  const int p0 = split * sp.split_pages, p1 = min(p0 + sp.split_pages, (lim_wg + PAGE - 1) / PAGE);

  // the wave's pages: p0 + pw + PW i, page id i in lane i (split_pages <= 64 PW)
  const int np = p1 > p0 + pw ? (p1 - p0 - pw + PW - 1) / PW : 0;
  int pid = 0;
  if (np > 0) pid = p.page_table[(size_t)s * p.max_pages + min(p0 + pw + PW * min(lane, np - 1), p.max_pages - 1)];
  const bool bad = np > 0 && (pid < 0 || pid >= p.c.num_pages);
  if (__builtin_amdgcn_ballot_w64(bad) != 0 && lane == 0) set_status(p.status, ST_BAD_PAGE);
  if (bad) pid = -1;

  const int wr0 = r0 + tw * RG * 16;
  const bool own = wr0 < R;                    // uniform: the wave has rows
  const int lim_first = rows.limit(min(wr0, R - 1) / G, p.causal);
  const int lim_last = rows.limit((min(wr0 + RG * 16, R) - 1) / G, p.causal);
  int lim[RG];                                 // of lane % 16's row (clamped rows are never stored)
  u32x4_t qf[RG][KS][NQ];
#pragma unroll
  for (int i = 0; i < RG; ++i) {
    const int r = min(wr0 + i * 16 + m16, R - 1), j = r / G;
    lim[i] = rows.limit(j, p.causal);
    const T* q = reinterpret_cast<const T*>(p.q) + (size_t)(rows.start + j) * p.ld_q + (size_t)(kvh * G + r - j * G) * DH;
#pragma unroll
    for (int k = 0; k < KS; ++k) {             // k step 2 i + h: channels 64 i + 16 g + 8 h ..
      const T* src = q + (k >> 1) * 64 + g * 16 + (k & 1) * 8;
      if constexpr (sizeof(T) == 2) {
        qf[i][k][0] = *(const gu4*)src;
      } else {
        float x[8];
        Run4<float>::load(src, x);
        Run4<float>::load(src + 4, x + 4);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t u = f2bf2(x[2 * e], x[2 * e + 1]);
            qf[i][k][n][e] = u;
            x[2 * e] -= bf2f(u & 0xFFFF);
            x[2 * e + 1] -= bf2f(u >> 16);
          }
        }
      }
    }
  }

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

  u32x4_t kr[4][KI], vr[DT];
  float ksc, vsc;
  auto page = [&](int i) { return max(__builtin_amdgcn_readlane(pid, i), 0); };   // an invalid one reads page 0, unused
  auto issue_k = [&](int i) {
    const size_t ph = (size_t)page(i) * Hkv + kvh;
    const uint8_t* kb = p.c.k + ph * PAGE * DH + (16 * (m16 >> 2) + (m16 & 3)) * DH + g * 16;
    ksc = p.c.ks[ph * 4 + g];
    vsc = p.c.vs[ph * 4 + g];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int c = 0; c < KI; ++c) kr[kt][c] = *(const gu4*)(kb + 4 * kt * DH + c * 64);
  };
  auto issue_v = [&](int i) {
    const size_t ph = (size_t)page(i) * Hkv + kvh;
    const uint8_t* vb = p.c.v + ph * PAGE * DH + m16 * 64 + g * 16;
#pragma unroll
    for (int d = 0; d < DT; ++d) vr[d] = *(const gu4*)(vb + d * 16 * 64);
  };
  // clears the bytes of the keys at or past lim_key of a lane's 16 (first key: key16)
  auto clear_from = [&](u32x4_t v, int key16, int lim_key) {
    const int nv = lim_key - key16;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = min(max(nv - 4 * e, 0), 4);
      v[e] &= t == 4 ? 0xFFFFFFFFu : (1u << (8 * t)) - 1u;
    }
    return v;
  };

  if (np > 0 && own) {
    issue_k(0);
    issue_v(0);
  }
  for (int i = 0; own && i < np; ++i) {
    const int kp0 = (p0 + pw + PW * i) * PAGE;
    const bool on = kp0 < lim_last && __builtin_amdgcn_readlane(pid, i) >= 0;   // uniform
    const bool edge = kp0 + PAGE > lim_first;                                   // uniform: some row sees a part only
    f32x4_t sc[RG][4];
    float c = 0.f, ev = 0.f, inv = 1.f;
    if (on) {
#pragma unroll
      for (int x = 0; x < RG; ++x)
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) sc[x][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const u32x4_t& u = kr[kt][k >> 1];
          const u32x4_t kf = (k & 1) ? kv8_bf16(u[2], u[3]) : kv8_bf16(u[0], u[1]);
#pragma unroll
          for (int x = 0; x < RG; ++x)
#pragma unroll
            for (int n = NQ - 1; n >= 0; --n) sc[x][kt] = mma_frag(bf16(), kf, qf[x][k][n], sc[x][kt]);
        }
      // a group that no row sees may have any scale
      const bool seen = kp0 + 16 * g < lim_last;
      c = sl2 * (seen ? ksc : 1.f);
      ev = seen ? __builtin_amdgcn_logf(vsc) : 0.f;
      inv = seen ? 1.f / vsc : 1.f;
    }
    if (i + 1 < np) issue_k(i + 1);
    if (on) {
      u32x4_t pa[RG][2][NP];
#pragma unroll
      for (int x = 0; x < RG; ++x) {
        float t[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) t[e] = sc[x][e >> 2][e & 3];
        if (edge) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (kp0 + 16 * g + e >= lim[x]) t[e] = -INFINITY;
        }
        float mx = t[0], a, b;
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, t[e]);
        mx = fmaf(mx, c, ev);
        pair16(mx, a, b);
        pair32(fmaxf(a, b), a, b);
        mx = fmaxf(a, b);
        const float mn = mx - HEAD > M[x] + SLACK ? mx - HEAD : M[x];
        if (__builtin_amdgcn_ballot_w64(mn != M[x]) != 0) {   // uniform
          const float f = M[x] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M[x] - mn);
          l[x] *= f;
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[x][d][r] *= f;
          M[x] = mn;
        }
        const float ref = ev - (M[x] == -INFINITY ? 0.f : M[x]);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          t[e] = __builtin_amdgcn_exp2f(fmaf(t[e], c, ref));
          sum += t[e];
        }
        l[x] = fmaf(sum, inv, l[x]);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int n = 0; n < NP; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float& u0 = t[8 * h + 2 * e];
              float& u1 = t[8 * h + 2 * e + 1];
              const uint32_t u = pk_f16(u0, u1);
              pa[x][h][n][e] = u;
              if (n + 1 < NP) {
                const f16x2_t y = __builtin_bit_cast(f16x2_t, u);
                u0 -= (float)y[0];
                u1 -= (float)y[1];
              }
            }
      }
      bool rowwise = false;
      if (edge) {
        const int key16 = kp0 + 16 * g;
        bool nan = false;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          vr[d] = clear_from(vr[d], key16, lim_last);
          // NaN codes (all low bits of a byte set) of keys that only some rows see
#pragma unroll
          for (int e = 0; e < 4; ++e) nan |= (((vr[d][e] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
        }
        rowwise = __builtin_amdgcn_ballot_w64(nan) != 0;
      }
      if (!rowwise) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4_t vf = h ? kv8_f16(vr[d][2], vr[d][3]) : kv8_f16(vr[d][0], vr[d][1]);
#pragma unroll
            for (int x = 0; x < RG; ++x)
#pragma unroll
              for (int n = NP - 1; n >= 0; --n) o[x][d] = mma_f16(vf, pa[x][h][n], o[x][d]);
          }
      } else {                                 // each row against the values it sees
#pragma unroll
        for (int x = 0; x < RG; ++x)
#pragma unroll 1
          for (int n0 = 0; n0 < 16; ++n0) {
            const int ln = __builtin_amdgcn_readlane(lim[x], n0);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              const u32x4_t u = clear_from(vr[d], kp0 + 16 * g, ln);
              f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const u32x4_t vf = h ? kv8_f16(u[2], u[3]) : kv8_f16(u[0], u[1]);
#pragma unroll
                for (int n = NP - 1; n >= 0; --n) acc = mma_f16(vf, pa[x][h][n], acc);
              }
#pragma unroll
              for (int r = 0; r < 4; ++r) o[x][d][r] += m16 == n0 ? acc[r] : 0.f;
            }
          }
      }
    }
    if (i + 1 < np) issue_v(i + 1);
  }
#pragma unroll
  for (int x = 0; x < RG; ++x) {               // the row's sum over the lane groups
    float a, b;
    pair16(l[x], a, b);
    pair32(a + b, a, b);
    l[x] = a + b;
  }

  // merge of the page waves, halves at a time
  constexpr int REC = (DT * 4 + 2) * 64;       // floats of a row group's state, register by register
  for (int half = PW / 2; half >= 1; half >>= 1) {
    float* st = kv8_smem + (size_t)(tw * (PW / 2) + (pw % half)) * RG * REC + lane;
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
    const int r = wr0 + x * 16 + m16;
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
      const size_t rgs = (size_t)sp.tiles * TW * RG;
      const size_t idx = (((size_t)s * Hkv + kvh) * rgs + r / 16) * sp.nsplit + split;
      float* rec = p.part + idx * (16 * DH + 32);
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<float4*>(rec + (d * 64 + lane) * 4) = make_float4(o[x][d][0], o[x][d][1], o[x][d][2], o[x][d][3]);
      if (lane < 16) *reinterpret_cast<float2*>(rec + 16 * DH + 2 * lane) = make_float2(M[x], l[x]);
    }
  }
}

// Merges the splits of one 16-row group in split order: wave d the 16 channels
// of output tile d, in the accumulator order the partials were left in.
template <typename T, int DH>
__global__ void __launch_bounds__(DH / 16 * 64) kv8_combine_kernel(Kv8AttnParams p, Kv8Split sp) {
  const int lane = threadIdx.x & 63, d = threadIdx.x >> 6;
  const int Hkv = p.c.Hkv, G = p.Hq / Hkv, tile_rg = sp.tw * sp.rg, rgs = sp.tiles * tile_rg;
  const int kvh = blockIdx.x % Hkv, rest = blockIdx.x / Hkv, rg = rest % rgs, s = rest / rgs;
  Kv8Rows rows;
  int bits;
  if (!kv8_rows(p, s, rows, bits)) return;
  const int R = rows.n * G;
  if (rg * 16 >= R) return;
  const int tile_end = min((rg / tile_rg + 1) * tile_rg * 16, R);
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
  sp.rg = bf16 && R > 16 ? 2 : 1;
  const int per = 16 * sp.rg;
  sp.tw = R > 2 * per ? 4 : (R > per ? 2 : 1);
  sp.pw = sp.tw == 4 ? 2 : 4;
  sp.tiles = (int)((R + sp.tw * per - 1) / (sp.tw * per));
  const long long items = (long long)nseq * Hkv * sp.tiles;
  const int pages = key_cap > 0 ? (key_cap + PAGE - 1) / PAGE : 1;
  const long long want = items < 2 * cus ? 2 * cus / items : 1;
  long long pp = (pages + want - 1) / want;
  if (pp < sp.pw) pp = sp.pw;
  if (pp > 64 * sp.pw) pp = 64 * sp.pw;
  sp.split_pages = (int)pp;
  sp.nsplit = (int)((pages + pp - 1) / pp);
  return sp;
}

inline size_t kv8_part_floats(const Kv8Split& sp, int nseq, int Hkv, int Dh) {
  return sp.nsplit == 1 ? 0 : (size_t)nseq * Hkv * sp.tiles * sp.tw * sp.rg * sp.nsplit * (16 * Dh + 32);
}

template <typename T, int DH, int RG, int TW, int PW>
static hipError_t launch_kv8_shape(const Kv8AttnParams& p, const Kv8Split& sp, hipStream_t st) {
  constexpr size_t lds = (size_t)TW * (PW / 2) * RG * (DH / 4 + 2) * 64 * sizeof(float);
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv8_attn_kernel<T, DH, RG, TW, PW>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (attr != hipSuccess) return attr;
  const long long wgs = (long long)p.nseq * p.c.Hkv * sp.tiles * sp.nsplit;
  if (wgs > 0x7FFFFFFFll) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((kv8_attn_kernel<T, DH, RG, TW, PW>), dim3((unsigned)wgs), dim3(TW * PW * 64), lds, st, p, sp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sp.nsplit == 1) return e;
  hipLaunchKernelGGL((kv8_combine_kernel<T, DH>), dim3(p.nseq * p.c.Hkv * sp.tiles * sp.tw * sp.rg), dim3(DH * 4), 0, st,
                     p, sp);
  return hipGetLastError();
}

template <typename T, int DH>
static hipError_t launch_kv8_dh(const Kv8AttnParams& p, const Kv8Split& sp, hipStream_t st) {
  constexpr int RG = sizeof(T) == 2 ? 2 : 1;
  if constexpr (RG == 2)
    if (sp.rg == 1) return launch_kv8_shape<T, DH, 1, 1, 4>(p, sp, st);
  if (sp.tw == 1) return launch_kv8_shape<T, DH, RG, 1, 4>(p, sp, st);
  if (sp.tw == 2) return launch_kv8_shape<T, DH, RG, 2, 4>(p, sp, st);
  return launch_kv8_shape<T, DH, RG, 4, 2>(p, sp, st);
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
