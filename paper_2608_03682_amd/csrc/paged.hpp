// The paged key/value cache: argument blocks of its kernels, the checks that a
// kernel makes of values that only the device knows (lengths, page numbers),
// and the launchers.
//
// Token p of request b lives in row p % page_size of page table[b][p / page_size].
// Lengths and tables are device memory, so that a captured call serves every
// later length; the host checks what bounds them (page count, table width,
// largest length) and the kernels never follow a value outside those bounds.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace phyai {

// status bits that the kernels raise
enum PagedStatus { PAGED_BAD_PAGE = 1, PAGED_BAD_LENGTH = 2 };

// The angle of pair i at position p is p * base^(-2i/D).  freq[i] holds
// base^(-2i/D) / 2 pi turns as a 64-bit fraction of a turn, so p * freq[i] mod 2^64
// is the angle with the whole turns taken off, good to p * (2^-64 + 2^-55 of freq): a
// float32 product would be off by 0.06 rad at a position of 10^6.
constexpr int kMaxPairs = 128;
struct RopeFreq {
  uint64_t f[kMaxPairs];
};

struct HeadRows {
  void* p;
  int64_t b, t, h;          // strides in elements
  int n;
};

// Pages of one layer.  Strides in bytes, the same for keys and values.
struct PagePool {
  char* k;
  char* v;
  const float* k_scale;     // 8-bit pools: one factor per head
  const float* v_scale;
  const int32_t* table;
  int64_t page_bytes, head_bytes, layer_bytes;
  int token_bytes;
  int page_shift, n_pages, max_pages, table_stride;
};

// Whether a table entry may be followed: the only check between a table and memory.
__host__ __device__ inline bool page_ok(int32_t page, int n_pages) {
  return static_cast<uint32_t>(page) < static_cast<uint32_t>(n_pages);
}

// Byte offset of a token's row in its pool.
__host__ __device__ inline int64_t page_row_offset(const PagePool& p, int32_t page, int64_t token, int head) {
  const int64_t row = token & ((int64_t(1) << p.page_shift) - 1);
  return static_cast<int64_t>(page) * p.page_bytes + row * p.token_bytes + head * p.head_bytes;
}

// Lengths of one request as a kernel uses them.  `ok` is false where the device
// values lie outside what the host checked; n and past are then safe to use.
struct RowSpan {
  int n;                    // valid rows, 0 .. rows
  int past;                 // tokens before the first row
  bool ok;
};
__host__ __device__ inline RowSpan row_span(int n, int past, int rows, int64_t cap) {
  RowSpan s;
  s.ok = n >= 0 && n <= rows && past >= 0 && static_cast<int64_t>(past) + n <= cap;
  s.n = n < 0 ? 0 : (n > rows ? rows : n);
  s.past = s.ok ? past : 0;
  return s;
}

// The keys that row `tok` of a request sees, [lo, hi): row tok stands at position
// kv - n + tok; causal rows see no later position, a window the last `window`
// positions up to their own.
__host__ __device__ inline int seen_end(int tok, int n, int kv, int causal) {
  if (!causal) return kv;
  const int e = kv - n + tok + 1;
  return e < 0 ? 0 : e;
}
__host__ __device__ inline int seen_begin(int tok, int n, int kv, int window) {
  if (window <= 0) return 0;
  const int64_t s = static_cast<int64_t>(kv) - n + tok + 1 - window;
  return s < 0 ? 0 : static_cast<int>(s);
}

struct NormRopeArgs {
  HeadRows q, k, q_out, k_out;   // n = 0: absent
  const float* q_gain;
  const float* k_gain;
  const int32_t* past_len;  // or null: 0
  const int32_t* new_len;   // or null: every row
  int32_t* status;
  int B, M, norm, rope, tokens_per_block;
  float eps;
  RopeFreq freq;
};

struct PagedAppendArgs {
  PagePool pool;
  HeadRows k, v;
  const int32_t* past_len;
  const int32_t* new_len;
  int32_t* status;
  int B, M, rope, tokens_per_block;
  RopeFreq freq;
};

struct PagedGatherArgs {
  PagePool pool;
  const int32_t* kv_len;
  void* out;                // [layers][2][B][rows][nkv * D]
  int32_t* status;
  int layers, B, rows, nkv, D;
};

struct PagedAttnArgs {
  PagePool pool;
  HeadRows q, out;
  const int32_t* kv_len;
  const int32_t* new_len;
  int32_t* status;
  float* part;              // n_split > 1: [B][nkv][M * G][n_split][D], not normalised
  float2* ml;               // and each split's (maximum, sum): [B][nkv][M * G][n_split]
  int B, M, nkv, G, max_kv, causal, window, n_split, split_keys, n_tiles;
  int pairs;                // 1: chunks in blocks of which a CU holds two
  float scale;
};

// Element kinds of rows and pools.
enum PagedKind { PAGED_F32 = 0, PAGED_BF16 = 1, PAGED_FP8 = 2 };

void norm_rope(const NormRopeArgs& a, int D, int kind, hipStream_t s);
void paged_append(const PagedAppendArgs& a, int D, int pool_kind, hipStream_t s);
void paged_gather(const PagedGatherArgs& a, int pool_kind, hipStream_t s);
// Plans the launch (row tiles, key splits) for a.B, M, nkv, G, max_kv and window and
// gives the floats of workspace it needs, most without a window; paged_attention
// launches what was planned.
int64_t paged_attention_plan(PagedAttnArgs& a, int D, int pool_kind);
void paged_attention(const PagedAttnArgs& a, int D, int pool_kind, hipStream_t s);

}  // namespace phyai
