// Internal launch interface of the paged 8-bit KV cache: page resize with the
// slot map, append, attention.
//
// One layer's cache (e4m3 bytes; a value is code * scale):
//   keys    [page][kv_head][64 tokens][Dh]
//   values  [page][kv_head][Dh][64 tokens]   (channel by channel)
//   scales  [page][kv_head][4]               one per group of 16 tokens, keys and values apart
// Keys lie row by row and values channel by channel so that a lane's 16-byte
// load is an operand run of the matrix cores in both products (the key order
// within a page is chosen by the loads), and a lane's 16 keys are one group: one
// key and one value scale per lane and page.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm.h"

namespace dflow {

constexpr int KV8_GROUP = 16;
constexpr long long KV8_MAX_WGS = (1ll << 24) - 1;     // of 256 threads: a launch has less than 2^32
constexpr int KV8_MIN_EXP = -100, KV8_MAX_EXP = 120;   // exponents of the append's scales

struct Kv8Cache {
  uint8_t* k;
  uint8_t* v;
  float* ks;
  float* vs;
  int num_pages, Hkv, Dh;
};

struct Kv8AppendParams {
  Kv8Cache c;
  const void* k;             // [rows][Hkv][Dh], ld elements from row to row
  const void* v;
  size_t ld_k, ld_v;
  const int* slot;           // [rows] page * 64 + token, or -1: the row is skipped
  int rows;
  int* status;
};
hipError_t launch_kv8_append(bool bf16, const Kv8AppendParams& p, hipStream_t s);

struct Kv8AttnParams {
  Kv8Cache c;
  const int* page_table;     // [nseq][max_pages]
  const int* kv_len;         // [nseq] cached tokens, the rows' own among them
  const int* row_start;      // [nseq + 1] rows of sequence s: row_start[s] .. row_start[s + 1] - 1
  const void* q;             // [rows][Hq][Dh], ld_q elements from row to row
  void* out;                 // [rows][Hq][Dh], or null: outf
  FragOut outf;              // matrix-core-order output (the O projection's operand)
  size_t ld_q, ld_out;
  float scale;               // softmax scale
  int nseq, rows, max_rows;  // rows of q, largest row count of one sequence
  int Hq, max_pages;
  int key_cap;               // keys read at most: min(max_len, 64 max_pages)
  int causal;
  // Work split: planned for plan_seq sequences; prompt: in a prefill, whose splits
  // (32 pages) and tiles do not depend on the chunk, so neither does a row's result
  int plan_seq, prompt;
  int cus;
  float* part;               // arrival counters and split partials, kv8_attn_workspace bytes
  int* status;
};
constexpr int KV8_COUNTERS = 1024;   // 4-byte arrival counters at the start of the workspace, zero between calls
size_t kv8_attn_workspace(bool bf16, int nseq, int max_rows, int key_cap, int Hq, int Hkv, int Dh, int cus, bool prompt);
hipError_t launch_kv8_attention(bool bf16, const Kv8AttnParams& p, hipStream_t s);

// Slots, row starts and lengths of nseq sequences of B rows at start_pos[s] .. (rows
// without a page in the table: slot -1, status).  row_start [nseq + 1], kv_len [nseq].
struct Kv8BatchParams {
  int nseq, B;
  const int* start_pos;
  const int* page_table;
  int max_pages, num_pages;
  int row0;                  // first row of the call's rows
  int *slot, *row_start, *kv_len;
  int* status;
};
hipError_t launch_kv8_batch(const Kv8BatchParams& p, hipStream_t s);

constexpr int PAGES_MAX_SEQ = 1024;
struct PageResizeParams {
  int nseq;
  const int* seq_len;        // [nseq] tokens cached
  const int* new_len;        // [nseq] tokens to come, null: none
  int* page_table;           // [nseq][max_pages]
  int max_pages, num_pages;
  int* n_held;               // [nseq] pages in each row
  int* free_pages;           // [num_pages] stack of page ids
  int* n_free;               // [1]
  int* slot;                 // [slot_cap], null: no slot map
  int slot_cap;
  int* row_start;            // [nseq + 1], null without a slot map
  int* status;
};
hipError_t launch_page_resize(const PageResizeParams& p, hipStream_t s);

}  // namespace dflow
