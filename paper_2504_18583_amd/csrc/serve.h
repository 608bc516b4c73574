// Serving operators (a paged cache of keys and values, attention over it,
// logits before tokens are picked): argument blocks of the kernels, and the
// cache's formats.
#pragma once

#include "train.h"

namespace pard {

constexpr int kKvBlock = 32;               // elements of a head that share a scale (PARD_E4M3, PARD_E2M1)

// Bytes of a head of the cache, and of its scales.
__host__ __device__ constexpr int kv_row_bytes(int dtype, int hd) {
  return dtype == PARD_E2M1 ? hd / 2 : dtype == PARD_E4M3 ? hd : 2 * hd;
}
__host__ __device__ constexpr int kv_scale_bytes(int dtype, int hd) {
  return dtype == PARD_E4M3 || dtype == PARD_E2M1 ? hd / kKvBlock : 0;
}

struct KvCacheView {
  char *k, *v;
  uint8_t *k_scale, *v_scale;              // null: elements as they are
  int n_pages, n_kv, page_log2;
};
struct KvBatchView {
  const int32_t *table, *row_start, *kv_len;
  int n_seqs, max_pages, rows;
  int cap;                                 // positions a table row can name
};

// Sequence of a row: the first whose rows end behind it (n_seqs: none).
// `start`: row_start or a copy of it.
__device__ __forceinline__ int kv_seq_of(const int32_t* start, int n_seqs, int row) {
  int lo = 0, hi = n_seqs;                 // start[lo + 1] > row is first true at the answer
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (start[mid + 1] > row) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// Page of a position, -1 where there is none.
__device__ __forceinline__ int kv_page(const KvCacheView& c, const KvBatchView& b, int seq, int pos) {
  const uint32_t at = (uint32_t)pos >> c.page_log2;
  if (at >= (uint32_t)b.max_pages) return -1;
  const int page = b.table[(int64_t)seq * b.max_pages + at];
  return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}

struct KvCopyArgs {
  KvCacheView cache;
  KvBatchView batch;
  Heads k, v;                              // rows
};
// rows -> cache (write) or cache -> rows; dtype: of the rows; vec: rows take 16-byte accesses
hipError_t launch_kv_copy(bool write, int head_dim, int dtype, int cache_dtype, bool vec, const KvCopyArgs& a,
                          hipStream_t st);

struct KvAttnArgs {
  KvCacheView cache;
  KvBatchView batch;
  int n_heads, group;
  FastDiv by_group;
  int window, sinks;                       // window 0: none
  float scale;
  Heads16 q, out;
  float* lse;                              // [n_heads][rows], may be null
  void* work;
  int slots;                               // records of partial sums in it
  int* plan;                               // running numbers of large batches in it, or null
};
size_t kv_attn_workspace(const KvAttnArgs& a, int head_dim, int max_seq_rows);
hipError_t launch_kv_attn(int head_dim, int dtype, int cache_dtype, const KvAttnArgs& a, int max_seq_rows, hipStream_t st);

struct LogitsArgs {
  int rows, vocab, n_seqs;
  const char* logits;
  int64_t stride;
  char* out;
  int64_t out_stride;
  const int32_t *tokens, *row_seq, *row_len, *prompt_len;
  int64_t tokens_stride;
  const float *repetition, *presence, *frequency;
  const int32_t *bias_start, *bias_ids;
  const float* bias_values;
  int n_bias;
  const uint32_t* mask;
  int64_t mask_stride;
  const int32_t* mask_row;
  int n_masks;
  int32_t* best;
  uint64_t* keys;                          // workspace: [rows][logits_keys]
  int row0;                                // first row of a launch
};
int logits_keys(int vocab);                // candidates of a row for best
hipError_t launch_logits_adjust(int dtype, const LogitsArgs& a, hipStream_t st);

}  // namespace pard
