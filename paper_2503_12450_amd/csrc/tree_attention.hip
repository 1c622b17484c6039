// Attention of trees of drafted tokens over a paged cache.
#include <algorithm>

#include "paged.h"

namespace marcache {

namespace tree {
namespace {

constexpr bool kTree = true;
#include "paged_attention.h"

}  // namespace
}  // namespace tree

size_t tree_attention_workspace(int dtype, const PagedBatch& b, int m, int heads_q, int window, int sinks) {
  return tree::attention_workspace(dtype, b, m, heads_q, window, sinks);
}

hipError_t launch_tree_attention(int dtype, const PagedBatch& b, int m, int heads_q, const void* q, long ld_q,
                                 const int32_t* parent, int window, int sinks, void* ws, size_t ws_bytes, void* out,
                                 long ld_out, hipStream_t st) {
  return tree::run_attention(dtype, b, m, heads_q, q, ld_q, parent, true, window, sinks, ws, ws_bytes, out, ld_out, st);
}

}  // namespace marcache
