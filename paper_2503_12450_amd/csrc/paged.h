// What the kernels of the paged cache share: the batch as they see it, the
// sequence of a row, and the place of a token.
#pragma once

#include "common.h"

namespace marcache {

struct PagedBatch {
  void* k;
  void* v;
  const int32_t* table;
  const int32_t* q_start;
  const int32_t* kv_len;
  int n_pages, n_heads, page_shift, d_head, n_seqs, max_pages, max_kv;
};

struct RotaryArgs {
  const double* freq;  // null: no rotation
  const int32_t* axis;
  const int32_t* pos;  // [m, n_axes]
  int n_pairs, n_axes, neighbours;
};

constexpr int kMaxTokens = 1 << 30;  // bound of every token number and of m * heads

// A sequence's rows and tokens, bounded: rows [row0, row0 + n) of the m rows,
// row i at token first + i (its last row, which may lie past m, at the last
// token), keys 0 .. len - 1 in the cache.  Whatever the
// device arrays hold, 0 <= row0, row0 + n <= m, 0 <= len <= max_kv and
// |first + i| <= 2^30.
struct SeqSpan {
  int row0, n, first, len;
};
__device__ __forceinline__ SeqSpan seq_span(int start, int end, int kv_len, int max_kv, int m) {
  SeqSpan r;
  r.row0 = min(max(start, 0), m);
  end = min(max(end, 0), kMaxTokens);
  r.n = max(min(end, m) - r.row0, 0);
  const int len = min(max(kv_len, 0), kMaxTokens);
  r.first = len - max(end - r.row0, 0);
  r.len = min(len, max_kv);
  return r;
}

hipError_t launch_rotary(int dtype, const RotaryArgs& rot, const void* x, long ld_x, int m, int heads, int d_head,
                         void* out, long ld_out, hipStream_t st);
hipError_t launch_paged_store(int dtype, const PagedBatch& b, const RotaryArgs& rot, int m, const void* k, long ld_k,
                              const void* v, long ld_v, int heads_q, const void* q, long ld_q, void* q_out,
                              long ld_q_out, hipStream_t st);
hipError_t launch_paged_attention(int dtype, const PagedBatch& b, int m, int heads_q, const void* q, long ld_q,
                                  bool causal, int window, int sinks, void* ws, size_t ws_bytes, void* out,
                                  long ld_out, hipStream_t st);
size_t paged_attention_workspace(int dtype, const PagedBatch& b, int m, int heads_q, int window, int sinks);

// Trees of drafted tokens: a sequence's first kMaxTree new rows.
constexpr int kMaxTree = 256;
hipError_t launch_tree_attention(int dtype, const PagedBatch& b, int m, int heads_q, const void* q, long ld_q,
                                 const int32_t* parent, int window, int sinks, void* ws, size_t ws_bytes, void* out,
                                 long ld_out, hipStream_t st);
size_t tree_attention_workspace(int dtype, const PagedBatch& b, int m, int heads_q, int window, int sinks);

hipError_t launch_paged_keep(int dtype, const PagedBatch& b, int m, const int32_t* path, const int32_t* kept,
                             int32_t* kv_out, hipStream_t st);
hipError_t launch_paged_fork(int dtype, const PagedBatch& b, int n_new, const int32_t* source, const int32_t* keep,
                             const int32_t* add, int32_t* table_out, int32_t* kv_out, int32_t* missing, void* ws,
                             hipStream_t st);
size_t paged_fork_workspace(const PagedBatch& b, int n_new);

}  // namespace marcache
