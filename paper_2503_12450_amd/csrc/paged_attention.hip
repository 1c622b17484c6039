// Attention of a ragged batch of rows over a paged cache, causal or not.
#include <algorithm>

#include "paged.h"

namespace marcache {

namespace {

constexpr bool kTree = false;
#include "paged_attention.h"

}  // namespace

size_t paged_attention_workspace(int dtype, const PagedBatch& b, int m, int heads_q, int window, int sinks) {
  return attention_workspace(dtype, b, m, heads_q, window, sinks);
}

hipError_t launch_paged_attention(int dtype, const PagedBatch& b, int m, int heads_q, const void* q, long ld_q,
                                  bool causal, int window, int sinks, void* ws, size_t ws_bytes, void* out,
                                  long ld_out, hipStream_t st) {
  return run_attention(dtype, b, m, heads_q, q, ld_q, nullptr, causal, window, sinks, ws, ws_bytes, out, ld_out, st);
}

}  // namespace marcache
