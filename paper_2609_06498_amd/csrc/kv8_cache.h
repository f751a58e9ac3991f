// Writes of the paged 8-bit cache and its page table (included by elementwise.hip).
#pragma once
#include <limits.h>

#include "common.h"
#include "kernels.h"
#include "kv8.h"

namespace dflow {

// ---------------------------------------------------------------- append
// Key and value rows go to their slots in e4m3 with one power-of-two scale per
// 16 tokens and head: s = the smallest power of two with max|x| / s <= 448 over
// the group's kept tokens (those below the first appended one: they belong to the
// sequence already) and the appended ones.  Dividing by a power of two is exact,
// so kept codes move to a new scale exactly (apart from values that become
// subnormal), and a group filled token by token ends as one filled at once.
// Tokens behind the appended ones are left as they were.
//
// The rows of a run (consecutive rows of one group, ascending) are one wave's
// work, keys and values apart, a kv head each.  A key wave holds a quarter of a
// token's channels per lane; a value wave DH / 64 channels of all 16 tokens, whose
// codes are one 16-byte store per channel (values lie channel by channel).  Bound
// by memory: rows read once, codes written once; for many rows a workgroup takes
// 4 RC consecutive rows of one head, so that the value stores of a page's four
// groups meet in one cache.

// 2^e of the scale rule for a maximum of finite magnitudes (0: scale 1)
__device__ inline int kv8_exponent(float amax) {
  if (!(amax > 0.f)) return 0;
  int e;
  const float m = frexpf(amax, &e);            // amax = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
  e = e - 9 + (m > 0.875f ? 1 : 0);
  return min(max(e, KV8_MIN_EXP), KV8_MAX_EXP);
}
__device__ inline float kv8_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
// largest finite magnitude of a wave's values (infinities and NaN do not set a scale); inf: there are infinities
template <int N>
__device__ inline float kv8_amax(const float* x, bool* inf) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(x[i]));       // (ignores NaN)
  m = wave_max(m);
  *inf = m == INFINITY;
  if (*inf) {                                  // uniform
    m = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(x[i]) < INFINITY ? fabsf(x[i]) : 0.f);
    m = wave_max(m);
  }
  return m;
}
// four values / 2^e as e4m3 codes, nearest even (finite ones are at most 448 there, NaN stays NaN)
__device__ inline uint32_t kv8_pack4(const float* x, float inv) {
  int u = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, u, true);
}
// infinities to the largest magnitude of scale sc
__device__ inline float kv8_saturate(float x, float sc) { return fabsf(x) == INFINITY ? copysignf(448.f * sc, x) : x; }
__device__ inline void kv8_unpack4(uint32_t u, float scale, float* x) {
  x[0] = __builtin_amdgcn_cvt_f32_fp8(u, 0) * scale;
  x[1] = __builtin_amdgcn_cvt_f32_fp8(u, 1) * scale;
  x[2] = __builtin_amdgcn_cvt_f32_fp8(u, 2) * scale;
  x[3] = __builtin_amdgcn_cvt_f32_fp8(u, 3) * scale;
}

// One group of one head, by a wave.  ph: its (page, head) block, part: the group
// in it; lane t of src: the row of token t, -1 where it is not appended; tokens
// below t0 are kept; row: the run's first.  FULL: all 16 tokens are appended.
template <typename T, int DH, bool FULL>
__device__ inline void append_keys(const Kv8AppendParams& p, size_t ph, int h, int part, int t0, int src, int row) {
  constexpr int CL = DH / 4;                   // a lane: a quarter of a token's channels
  const int lane = threadIdx.x & 63, t = lane >> 2, c0 = (lane & 3) * CL;
  const int sr = FULL ? row + t : __shfl(src, t, 64);
  uint4* dst = reinterpret_cast<uint4*>(p.c.k + (ph * PAGE + part * KV8_GROUP + t) * DH + c0);
  float* scale = p.c.ks + ph * 4 + part;
  // all loads in flight at once (a token that is not appended reads the run's first row, unused)
  const T* k = reinterpret_cast<const T*>(p.k) + (size_t)(sr >= 0 ? sr : row) * p.ld_k + (size_t)h * DH + c0;
  float x[CL], old = 1.f;
  uint4 was[CL / 16];
  if (!FULL && t0 > 0) {                       // uniform
    old = *scale;
#pragma unroll
    for (int i = 0; i < CL / 16; ++i) was[i] = dst[i];
  }
#pragma unroll
  for (int i = 0; i < CL; i += 16) Row16<T>::load(k + i, x + i);
  if (!FULL && sr < 0) {
#pragma unroll
    for (int i = 0; i < CL; ++i) x[i] = 0.f;
    if (t < t0) {
#pragma unroll
      for (int i = 0; i < CL; i += 16) {
        kv8_unpack4(was[i / 16].x, old, x + i);
        kv8_unpack4(was[i / 16].y, old, x + i + 4);
        kv8_unpack4(was[i / 16].z, old, x + i + 8);
        kv8_unpack4(was[i / 16].w, old, x + i + 12);
      }
    }
  }
  bool inf;
  const int e = kv8_exponent(kv8_amax<CL>(x, &inf));
  const float sc = kv8_pow2(e), inv = kv8_pow2(-e);
  if (inf) {
#pragma unroll
    for (int i = 0; i < CL; ++i) x[i] = kv8_saturate(x[i], sc);
  }
  if (FULL || sr >= 0 || (t < t0 && sc != old)) {
#pragma unroll
    for (int i = 0; i < CL; i += 16)
      dst[i / 16] = make_uint4(kv8_pack4(x + i, inv), kv8_pack4(x + i + 4, inv), kv8_pack4(x + i + 8, inv),
                               kv8_pack4(x + i + 12, inv));
  }
  if (lane == 0) *scale = sc;
}

template <typename T, int DH, bool FULL>
__device__ inline void append_values(const Kv8AppendParams& p, size_t ph, int h, int part, int t0, int src, int row,
                                     uint32_t fresh) {
  constexpr int CL = DH / 64;                  // a lane: CL channels of all 16 tokens
  const int c0 = (threadIdx.x & 63) * CL;
  uint8_t* dst = p.c.v + (ph * DH + c0) * PAGE + part * KV8_GROUP;
  float* scale = p.c.vs + ph * 4 + part;
  T raw[KV8_GROUP][CL];
  const T* v0 = reinterpret_cast<const T*>(p.v) + (size_t)h * DH + c0;
#pragma unroll
  for (int t = 0; t < KV8_GROUP; ++t) {
    const int sr = FULL ? row + t : __builtin_amdgcn_readlane(src, t);
    const T* v = v0 + (size_t)(sr >= 0 ? sr : row) * p.ld_v;
    __builtin_memcpy(raw[t], __builtin_assume_aligned(v, CL * sizeof(T)), CL * sizeof(T));
  }
  float x[CL][KV8_GROUP], old = 1.f;
  uint32_t was[CL][4];
  if (!FULL) {
    old = *scale;
#pragma unroll
    for (int c = 0; c < CL; ++c) {
      const uint4 u = *reinterpret_cast<const uint4*>(dst + c * PAGE);
      was[c][0] = u.x; was[c][1] = u.y; was[c][2] = u.z; was[c][3] = u.w;
    }
  }
#pragma unroll
  for (int c = 0; c < CL; ++c)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float y[4];
      if (!FULL) kv8_unpack4(was[c][q], old, y);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int t = 4 * q + b;
        x[c][t] = TT<T>::ld(raw[t], c);
        if (!FULL && !(fresh >> t & 1)) x[c][t] = t < t0 ? y[b] : 0.f;
      }
    }
  bool inf;
  const int e = kv8_exponent(kv8_amax<CL * KV8_GROUP>(&x[0][0], &inf));
  const float sc = kv8_pow2(e), inv = kv8_pow2(-e);
  if (inf) {
#pragma unroll
    for (int i = 0; i < CL * KV8_GROUP; ++i) x[i / KV8_GROUP][i % KV8_GROUP] = kv8_saturate(x[i / KV8_GROUP][i % KV8_GROUP], sc);
  }
  const uint32_t live = fresh | ((1u << t0) - 1u);
#pragma unroll
  for (int c = 0; c < CL; ++c) {
    uint32_t u[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      u[q] = kv8_pack4(&x[c][4 * q], inv);
      if (!FULL) {
        uint32_t keep = 0;                     // bytes of the tokens that stay as they were
#pragma unroll
        for (int b = 0; b < 4; ++b) keep |= (live >> (4 * q + b)) & 1u ? 0u : 0xFFu << (8 * b);
        u[q] = (u[q] & ~keep) | (was[c][q] & keep);
      }
    }
    *reinterpret_cast<uint4*>(dst + c * PAGE) = make_uint4(u[0], u[1], u[2], u[3]);
  }
  if ((threadIdx.x & 63) == 0) *scale = sc;
}

template <typename T, int DH, int RC>
__global__ void __launch_bounds__(256) kv8_append_kernel(Kv8AppendParams p) {
  static_assert(RC + 17 <= 64, "a lane per row of the window");
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned unit = blockIdx.x % (2u * p.c.Hkv);   // fastest: the heads of a row are read together
  const bool is_v = unit & 1;
  const int h = unit >> 1;
  const unsigned first = (blockIdx.x / (2u * p.c.Hkv) * 4 + w) * RC;
  if (first >= (unsigned)p.rows) return;       // uniform per wave
  const int r0 = first;
  // slots of rows r0 - 1 (lane 0) .. r0 + RC + 15
  const int row = r0 - 1 + lane;
  const int cap = p.c.num_pages * PAGE;
  int slot = row >= 0 && row < p.rows && lane < RC + 17 ? p.slot[row] : -1;
  bool fault = slot < -1 || slot >= cap;
  if (fault) slot = -1;
  const int group = slot < 0 ? -1 - lane : slot / KV8_GROUP;     // (no two invalid rows share a group)
  const int before = __shfl_up(group, 1, 64), sbefore = __shfl_up(slot, 1, 64);
  const bool mine = lane >= 1 && lane <= RC;
  const bool follows = lane >= 1 && slot >= 0 && group == before;
  fault |= follows && slot <= sbefore;
  if (unit == 0 && __builtin_amdgcn_ballot_w64(mine && fault) != 0 && lane == 0) set_status(p.status, ST_BAD_SLOT);
  uint64_t leads = __builtin_amdgcn_ballot_w64(mine && slot >= 0 && !follows);
  while (leads) {                              // uniform
    const int ld = __builtin_ctzll(leads);
    leads &= leads - 1;
    const int s0 = __builtin_amdgcn_readlane(slot, ld), gr = s0 / KV8_GROUP, t0 = s0 % KV8_GROUP;
    // source row of each token of the group: lane t of src, -1: not appended
    int src;
    const uint64_t line = __builtin_amdgcn_ballot_w64(slot == s0 + lane - ld && lane < ld + KV8_GROUP - t0) >> ld;
    const int n = __builtin_ctzll(~line);      // rows of the run without a gap
    if (ld + n < 64 && __builtin_amdgcn_readlane(group, (ld + n) & 63) == gr) {   // uniform: more of the group follow
      int top = -1;
      src = -1;
      for (int i = 0; i < KV8_GROUP && ld + i < 64; ++i) {
        const int sl = __builtin_amdgcn_readlane(slot, ld + i);
        if (__builtin_amdgcn_readlane(group, ld + i) != gr) break;
        const int t = sl % KV8_GROUP;
        if (t <= top) continue;                // not ascending: skipped (status set above)
        top = t;
        if ((lane & 15) == t) src = r0 - 1 + ld + i;
      }
    } else {
      const int t = lane & 15;
      src = t >= t0 && t < t0 + n ? r0 - 1 + ld + t - t0 : -1;
    }
    const uint32_t fresh = (uint32_t)__builtin_amdgcn_ballot_w64(lane < 16 && src >= 0);
    const int page = gr / 4, part = gr % 4;
    const size_t ph = (size_t)page * p.c.Hkv + h;
    if (is_v) {
      if (fresh == 0xFFFFu) append_values<T, DH, true>(p, ph, h, part, t0, src, r0 - 1 + ld, fresh);
      else append_values<T, DH, false>(p, ph, h, part, t0, src, r0 - 1 + ld, fresh);
    } else {
      if (fresh == 0xFFFFu) append_keys<T, DH, true>(p, ph, h, part, t0, src, r0 - 1 + ld);
      else append_keys<T, DH, false>(p, ph, h, part, t0, src, r0 - 1 + ld);
    }
  }
}

// Lanes find their rows' runs 16 to a wave where there are many (prompts: a run is
// 16 rows; 15253 rows 36 us with 32, 29 with 16, 32 with 8, before whole groups had a path of
// their own: now 24), else one.
constexpr int APPEND_RC = 16;

template <typename T, int DH, int RC>
static hipError_t launch_append_rc(const Kv8AppendParams& p, hipStream_t st) {
  const long long wgs = 2ll * p.c.Hkv * (((long long)p.rows + 4 * RC - 1) / (4 * RC));
  if (wgs > KV8_MAX_WGS) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((kv8_append_kernel<T, DH, RC>), dim3((unsigned)wgs), dim3(256), 0, st, p);
  return hipGetLastError();
}
template <typename T, int DH>
static hipError_t launch_append_dh(const Kv8AppendParams& p, hipStream_t st) {
  // A round's rows spread over as many waves as there are rows; from a few
  // thousand rows on they are prompts, whose runs are 16 rows.
  return p.rows <= 2048 ? launch_append_rc<T, DH, 1>(p, st) : launch_append_rc<T, DH, APPEND_RC>(p, st);
}

hipError_t launch_kv8_append(bool isbf, const Kv8AppendParams& p, hipStream_t st) {
  if (p.rows < 1) return hipSuccess;
  if (p.c.Dh == 128) return isbf ? launch_append_dh<bf16, 128>(p, st) : launch_append_dh<float, 128>(p, st);
  if (p.c.Dh == 64) return isbf ? launch_append_dh<bf16, 64>(p, st) : launch_append_dh<float, 64>(p, st);
  return hipErrorInvalidValue;
}

// ---------------------------------------------------------------- rows of a round
__global__ void __launch_bounds__(256) kv8_batch_kernel(Kv8BatchParams p) {
  const int i = blockIdx.x * 256 + threadIdx.x, rows = p.nseq * p.B;
  if (i <= p.nseq) {
    p.row_start[i] = p.row0 + i * p.B;
    if (i < p.nseq) p.kv_len[i] = p.start_pos[i] + p.B;
  }
  if (i >= rows) return;
  const int s = i / p.B, pos = p.start_pos[s] + i - s * p.B;
  int slot = -1;
  if (pos < 0 || pos / PAGE >= p.max_pages) {
    set_status(p.status, ST_CAPACITY);
  } else {
    const int page = p.page_table[(size_t)s * p.max_pages + pos / PAGE];
    if (page < 0 || page >= p.num_pages) set_status(p.status, ST_BAD_PAGE);
    else slot = page * PAGE + pos % PAGE;
  }
  p.slot[i] = slot;
}

hipError_t launch_kv8_batch(const Kv8BatchParams& p, hipStream_t st) {
  const int n = p.nseq * p.B > p.nseq ? p.nseq * p.B : p.nseq + 1;
  hipLaunchKernelGGL(kv8_batch_kernel, dim3((n + 255) / 256), dim3(256), 0, st, p);
  return hipGetLastError();
}

// ---------------------------------------------------------------- pages
// Rows of a page table resized to request lengths.  One workgroup, a thread per
// sequence: target = ceil((len + new) / 64) pages; the pages above it go back to
// the free stack, then rows take pages from its top, both placed by exclusive
// sums over the sequences.  A page's place depends on its rank (by sequence, then
// page): the lowest rank of the released ones ends on top, the lowest of the taken
// ones is popped first, so growing and shrinking again restores the stack.
// Slots are mapped here when they are few, else by a launch of their own that
// spreads them over the chip.  Bound by latency (a few dependent loads and two
// scans), or by the slot stores.
constexpr int PAGES_T = 1024;
constexpr int PAGES_INLINE_ROWS = 4096;

// exclusive sums of three values over the workgroup's threads, and their totals
struct Sum3 { long long v[3]; };
__device__ inline Sum3 block_scan(const Sum3& x, Sum3* sh /* [16] */, Sum3* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  Sum3 s = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const long long y = __shfl_up(s.v[i], o, 64);
      if (lane >= o) s.v[i] += y;
    }
  if (lane == 63) sh[w] = s;
  __syncthreads();
  Sum3 base{{0, 0, 0}}, all{{0, 0, 0}};
  for (int k = 0; k < nw; ++k)
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if (k < w) base.v[i] += sh[k].v[i];
      all.v[i] += sh[k].v[i];
    }
#pragma unroll
  for (int i = 0; i < 3; ++i) s.v[i] += base.v[i] - x.v[i];
  *total = all;
  return s;
}

// slot of row r of the call: sequence by binary search over the row starts.
// base(s): tokens the sequence had, -1 where it was refused.
template <typename F>
__device__ inline int map_slot(const PageResizeParams& p, const int* starts, F&& base, int r) {
  int lo = 0, hi = p.nseq;                     // starts[lo] <= r < starts[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid] <= r) lo = mid;
    else hi = mid;
  }
  const int len = base(lo);
  if (len < 0) return -1;
  const int pos = len + r - starts[lo];
  const int page = p.page_table[(size_t)lo * p.max_pages + pos / PAGE];
  return page < 0 || page >= p.num_pages ? -1 : page * PAGE + pos % PAGE;
}

__global__ void __launch_bounds__(PAGES_T) page_resize_kernel(PageResizeParams p, int inline_slots) {
  __shared__ Sum3 sh[PAGES_T / 64];
  __shared__ int s_held[PAGES_MAX_SEQ], s_drop[PAGES_MAX_SEQ], s_doff[PAGES_MAX_SEQ], s_take[PAGES_MAX_SEQ],
      s_toff[PAGES_MAX_SEQ], s_len[PAGES_MAX_SEQ], s_start[PAGES_MAX_SEQ + 1], s_taken;
  const int s = threadIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  const bool have = s < p.nseq;
  const int sc = min(s, p.nseq - 1);
  const long long len = p.seq_len[sc], more = p.new_len ? p.new_len[sc] : 0;
  const int held0 = p.n_held[sc], top0 = *p.n_free;
  if (s == 0) s_taken = 0;
  int bits = top0 < 0 || top0 > p.num_pages ? ST_CAPACITY : 0;
  const int top = min(max(top0, 0), p.num_pages);
  const int held = min(max(held0, 0), p.max_pages);
  const long long target = (len + more + PAGE - 1) / PAGE;
  const bool valid = have && len >= 0 && more >= 0 && target <= p.max_pages;
  if (have && (!valid || held != held0)) bits |= ST_CAPACITY;
  const int drop = valid && held > target ? held - (int)target : 0;
  const int want = valid && target > held ? (int)target - held : 0;
  Sum3 tot;
  const Sum3 at = block_scan(Sum3{{drop, want, have && more > 0 ? more : 0}}, sh, &tot);
  const long long dropped = tot.v[0], avail = min((long long)top + dropped, (long long)p.num_pages);
  const int take = want > 0 && at.v[1] + want <= avail ? want : 0;   // (sequences that take are the first that want)
  if (want > take) bits |= ST_CAPACITY;
  const int cap = p.slot ? p.slot_cap : INT_MAX;
  const bool fits = valid && want == take;
  if (have) {
    s_held[s] = held - drop;
    s_drop[s] = drop;
    s_doff[s] = (int)at.v[0];
    s_take[s] = take;
    s_toff[s] = (int)at.v[1];
    s_len[s] = fits ? (int)len : -1;
    s_start[s] = (int)min(at.v[2], (long long)cap);
    if (take > 0) atomicMax(&s_taken, (int)at.v[1] + take);
    if (held - drop + take != held0) p.n_held[s] = held - drop + take;
  }
  if (s == 0) s_start[p.nseq] = (int)min(tot.v[2], (long long)cap);
  if (p.slot && tot.v[2] > cap) bits |= ST_CAPACITY;
  __syncthreads();
  if (dropped > 0) {                           // uniform: give back
    for (int q = w; q < p.nseq; q += nw)
      for (int i = lane; i < s_drop[q]; i += 64) {
        int* e = p.page_table + (size_t)q * p.max_pages + s_held[q] + i;
        const long long to = top + dropped - 1 - (s_doff[q] + i);
        if (to < p.num_pages) p.free_pages[to] = *e;
        else bits |= ST_CAPACITY;              // more pages than the pool has: the caller's state is wrong
        *e = -1;
      }
    __threadfence_block();
    __syncthreads();
  }
  const int taken = s_taken;
  if (taken > 0) {                             // uniform: take
    for (int q = w; q < p.nseq; q += nw)
      for (int i = lane; i < s_take[q]; i += 64)
        p.page_table[(size_t)q * p.max_pages + s_held[q] + i] = p.free_pages[avail - 1 - (s_toff[q] + i)];
  }
  if (s == 0) *p.n_free = (int)(avail - taken);
  if (p.slot) {
    for (int i = s; i <= p.nseq; i += blockDim.x) p.row_start[i] = s_start[i];
    if (inline_slots) {
      if (taken > 0) {
        __threadfence_block();
        __syncthreads();
      }
      for (int i = s; i < s_start[p.nseq]; i += blockDim.x)
        p.slot[i] = map_slot(p, s_start, [&](int q) { return s_len[q]; }, i);
    }
  }
  if (bits) set_status(p.status, bits);
}

// Slots of many rows, after page_resize_kernel: a sequence whose row is too short was refused.
__global__ void __launch_bounds__(256) slot_map_kernel(PageResizeParams p) {
  __shared__ int starts[PAGES_MAX_SEQ + 1];
  for (int i = threadIdx.x; i <= p.nseq; i += 256) starts[i] = p.row_start[i];
  __syncthreads();
  const unsigned at = blockIdx.x * 256 + threadIdx.x;
  if (at >= (unsigned)starts[p.nseq]) return;
  const int r = at;
  p.slot[r] = map_slot(p, starts, [&](int q) {
    const long long len = p.seq_len[q], more = p.new_len[q];
    return len < 0 || (len + more + PAGE - 1) / PAGE > p.n_held[q] ? -1 : (int)len;
  }, r);
}

hipError_t launch_page_resize(const PageResizeParams& p, hipStream_t st) {
  // a thread per sequence; more only where there are many slots to map
  const int inl = p.slot_cap <= PAGES_INLINE_ROWS;
  int threads = (p.nseq + 255) / 256 * 256;
  if (p.slot && inl && p.slot_cap > 1024) threads = PAGES_T;
  hipLaunchKernelGGL(page_resize_kernel, dim3(1), dim3(threads), 0, st, p, inl);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.slot || inl) return e;
  hipLaunchKernelGGL(slot_map_kernel, dim3(((unsigned)p.slot_cap + 255u) / 256u), dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace dflow
