// C entry points of the rotary positions, the paged cache, its attention and what
// decides about drafted tokens: every argument is checked here, on the host,
// before anything is enqueued.
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <initializer_list>

#include "../../include/mar_kernels.h"
#include "draft.h"
#include "paged.h"

using namespace marcache;

namespace {

mar_status fail(mar_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  abi_fail_v(s, fmt, ap);
  va_end(ap);
  return s;
}

mar_status device_result(hipError_t e, const char* what) {
  return e == hipSuccess ? MAR_OK : fail(MAR_E_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

mar_status check_dtype(int32_t dtype) {
  if (dtype != MAR_F32 && dtype != MAR_BF16) return fail(MAR_E_ARG, "unknown dtype %d", dtype);
  return MAR_OK;
}

// m rows of `heads` heads of d_head columns at p, row stride ld
mar_status check_rows(const char* name, const void* p, int64_t ld, int32_t m, int32_t heads, int32_t d_head) {
  if (heads < 1 || m < 0 || static_cast<int64_t>(m) * heads >= kMaxTokens || heads > 65536)
    return fail(MAR_E_SHAPE, "%s: need heads >= 1, m >= 0 and m * heads < 2^30", name);
  if (ld % 8 || ld < static_cast<int64_t>(heads) * d_head || ld >= (int64_t{1} << 31))
    return fail(MAR_E_SHAPE, "%s: row stride %lld must be a multiple of 8 and cover %d heads of %d", name,
                static_cast<long long>(ld), heads, d_head);
  if (m > 0 && !p) return fail(MAR_E_ARG, "%s is NULL", name);
  if (!aligned16(p)) return fail(MAR_E_ARG, "%s must be 16-byte aligned", name);
  return MAR_OK;
}

mar_status check_head(int32_t d_head) {
  if (d_head % 16 || d_head < 16 || d_head > 128) return fail(MAR_E_SHAPE, "d_head must be 16..128, multiple of 16");
  return MAR_OK;
}

mar_status take_rotary(const mar_rotary* r, const int32_t* pos, int32_t m, int32_t d_head, RotaryArgs* out) {
  if (!r->freq || !r->axis || (m > 0 && !pos)) return fail(MAR_E_ARG, "rotary: NULL pointer");
  if (r->n_pairs < 8 || r->n_pairs % 8 || r->n_pairs > d_head / 2)
    return fail(MAR_E_SHAPE, "rotary: n_pairs %d must be a multiple of 8 in [8, d_head / 2]", r->n_pairs);
  if (r->n_axes < 1 || r->n_axes > 4) return fail(MAR_E_SHAPE, "rotary: n_axes must be 1..4");
  if (r->layout != MAR_ROTARY_HALVES && r->layout != MAR_ROTARY_NEIGHBOURS)
    return fail(MAR_E_ARG, "rotary: unknown layout %d", r->layout);
  *out = RotaryArgs{r->freq, r->axis, pos, r->n_pairs, r->n_axes, r->layout == MAR_ROTARY_NEIGHBOURS};
  return MAR_OK;
}

mar_status take_batch(const mar_paged_batch* b, PagedBatch* out) {
  if (!b) return fail(MAR_E_ARG, "batch is NULL");
  mar_status s = check_head(b->d_head);
  if (s != MAR_OK) return s;
  if (b->n_heads < 1 || b->n_heads > 4096) return fail(MAR_E_SHAPE, "batch: n_heads %d outside [1, 4096]", b->n_heads);
  if (b->n_seqs < 0 || b->n_seqs > 65536) return fail(MAR_E_SHAPE, "batch: n_seqs %d outside [0, 65536]", b->n_seqs);
  if (b->page < 16 || b->page > 4096 || (b->page & (b->page - 1)))
    return fail(MAR_E_SHAPE, "batch: page %d must be a power of two, 16..4096", b->page);
  if (b->n_pages < 1 || b->max_pages < 1) return fail(MAR_E_SHAPE, "batch: n_pages and max_pages must be >= 1");
  const int64_t most = static_cast<int64_t>(b->max_pages) * b->page;
  if (most > kMaxTokens) return fail(MAR_E_SHAPE, "batch: max_pages * page must be at most 2^30");
  if (b->max_kv < 1 || b->max_kv > most)
    return fail(MAR_E_SHAPE, "batch: max_kv %d outside [1, max_pages * page]", b->max_kv);
  if (!b->k || !b->v || !b->q_start || (b->n_seqs > 0 && (!b->table || !b->kv_len)))
    return fail(MAR_E_ARG, "batch: NULL pointer");
  if (!aligned16(b->k) || !aligned16(b->v)) return fail(MAR_E_ARG, "batch: k and v must be 16-byte aligned");
  *out = PagedBatch{b->k, b->v, b->table, b->q_start, b->kv_len, b->n_pages, b->n_heads,
                    __builtin_ctz(static_cast<unsigned>(b->page)), b->d_head, b->n_seqs, b->max_pages, b->max_kv};
  return MAR_OK;
}

mar_status take_attention(int32_t dtype, const mar_paged_batch* batch, int32_t m, int32_t n_heads_q, int32_t window,
                          int32_t sinks, PagedBatch* b) {
  mar_status s = check_dtype(dtype);
  if (s == MAR_OK) s = take_batch(batch, b);
  if (s != MAR_OK) return s;
  if (n_heads_q < 1 || n_heads_q % b->n_heads)
    return fail(MAR_E_SHAPE, "n_heads_q %d must be a positive multiple of the %d key/value heads", n_heads_q, b->n_heads);
  if (m < 0 || n_heads_q > 65536 || static_cast<int64_t>(m) * n_heads_q >= kMaxTokens)
    return fail(MAR_E_SHAPE, "need m >= 0 and m * n_heads_q < 2^30");
  if (window < 0 || sinks < 0) return fail(MAR_E_ARG, "window and sinks must not be negative");
  return MAR_OK;
}

// Rows of `vocab` elements of es bytes at p, row stride ld
mar_status check_vocab_rows(const char* name, const void* p, int64_t ld, int32_t m, int32_t vocab, unsigned es) {
  if (ld < vocab || ld >= (int64_t{1} << 31))
    return fail(MAR_E_SHAPE, "%s: row stride %lld must cover %d tokens", name, static_cast<long long>(ld), vocab);
  if (m > 0 && !p) return fail(MAR_E_ARG, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % es) return fail(MAR_E_ARG, "%s must be aligned to its elements", name);
  return MAR_OK;
}

mar_status check_vocab(int32_t m, int32_t vocab) {
  if (m < 0 || m >= kMaxTokens) return fail(MAR_E_SHAPE, "need 0 <= m < 2^30");
  if (vocab < 1 || vocab > kMaxVocab) return fail(MAR_E_SHAPE, "vocab %d outside [1, %d]", vocab, kMaxVocab);
  return MAR_OK;
}

mar_status check_verify(int32_t m, int32_t n_seqs, int32_t vocab) {
  if (n_seqs < 0 || n_seqs > 65536) return fail(MAR_E_SHAPE, "n_seqs %d outside [0, 65536]", n_seqs);
  return check_vocab(m, vocab);
}

mar_status check_workspace(const void* ws, size_t have, size_t need) {
  if (have < need) return fail(MAR_E_WORKSPACE, "workspace of %zu bytes, need %zu", have, need);
  if (need && !ws) return fail(MAR_E_WORKSPACE, "workspace is NULL");
  if (!aligned16(ws)) return fail(MAR_E_WORKSPACE, "workspace must be 16-byte aligned");
  return MAR_OK;
}

// Bytes that a call reads or writes throughout (NULL or 0: none).
struct Range {
  const char* name;
  const void* at;
  size_t bytes;
};
Range vector_of(const char* name, const void* p, int64_t n) {
  return {name, p, p ? static_cast<size_t>(n) * sizeof(int32_t) : 0};
}
// m rows of n elements of es bytes; none if gaps lie between the rows, where others may be.
Range rows_of(const char* name, const void* p, int64_t ld, int32_t m, int64_t n, unsigned es) {
  return {name, p, p && (ld == n || m <= 1) ? static_cast<size_t>(m) * n * es : 0};
}
Range pages_of(const char* name, const void* p, const PagedBatch& b, int32_t dtype) {
  return {name, p, (static_cast<size_t>(b.n_pages) * b.n_heads * b.d_head << b.page_shift) * (dtype == MAR_BF16 ? 2 : 4)};
}
bool meet(const Range& a, const Range& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  return a.bytes && b.bytes && (x <= y ? y - x < a.bytes : x - y < b.bytes);
}
// Outputs (the first `outs`) that overlap one another or what is read are refused: a
// workgroup would read what another one has written already.
mar_status check_apart(std::initializer_list<Range> all, size_t outs) {
  for (const Range* a = all.begin(); a != all.begin() + outs; ++a)
    for (const Range* b = a + 1; b != all.end(); ++b)
      if (meet(*a, *b)) return fail(MAR_E_ARG, "%s must not overlap %s", a->name, b->name);
  return MAR_OK;
}
// The same for out and in, m rows of n elements each: exact for dense rows and where the
// rows lie equally far apart (columns of one matrix are apart).
mar_status check_rows_apart(const char* out_name, const void* out, int64_t ld_out, unsigned es_out, const char* in_name,
                            const void* in, int64_t ld_in, unsigned es_in, int32_t m, int64_t n) {
  bool overlap = meet(rows_of("", out, ld_out, m, n, es_out), rows_of("", in, ld_in, m, n, es_in));
  const int64_t ld = ld_out * es_out;
  if (m > 0 && ld == ld_in * es_in) {
    const int64_t far = reinterpret_cast<intptr_t>(in) - reinterpret_cast<intptr_t>(out);
    const int64_t rows = far >= 0 ? far / ld : -((ld - 1 - far) / ld), columns = far - rows * ld;  // columns >= 0
    overlap |= columns < n * es_out && rows > -m && rows < m;
    overlap |= columns + n * es_in > ld && rows + 1 > -m && rows + 1 < m;
  }
  return overlap ? fail(MAR_E_ARG, "%s must not overlap %s", out_name, in_name) : MAR_OK;
}

mar_status take_fork(const mar_paged_batch* batch, int32_t n_new, PagedBatch* b) {
  const mar_status s = take_batch(batch, b);
  if (s != MAR_OK) return s;
  if (n_new < 0 || n_new > 65536) return fail(MAR_E_SHAPE, "n_new %d outside [0, 65536]", n_new);
  return MAR_OK;
}

}  // namespace

extern "C" {

mar_status mar_k_rotary(int32_t dtype, const mar_rotary* rotary, const void* x, int64_t ld_x, const int32_t* pos,
                        int32_t m, int32_t n_heads, int32_t d_head, void* out, int64_t ld_out, void* stream) {
  abi_clear_error();
  RotaryArgs r;
  mar_status s = check_dtype(dtype);
  if (s == MAR_OK) s = check_head(d_head);
  if (s == MAR_OK && !rotary) s = fail(MAR_E_ARG, "rotary is NULL");
  if (s == MAR_OK) s = take_rotary(rotary, pos, m, d_head, &r);
  if (s == MAR_OK) s = check_rows("x", x, ld_x, m, n_heads, d_head);
  if (s == MAR_OK) s = check_rows("out", out, ld_out, m, n_heads, d_head);
  if (s == MAR_OK && out == x && ld_out != ld_x) s = fail(MAR_E_ARG, "out may be x only with the same row stride");
  if (s != MAR_OK) return s;
  return device_result(launch_rotary(dtype, r, x, ld_x, m, n_heads, d_head, out, ld_out,
                                     static_cast<hipStream_t>(stream)),
                       "rotary");
}

mar_status mar_k_paged_store(int32_t dtype, const mar_paged_batch* batch, const mar_rotary* rotary,
                             const int32_t* pos, int32_t m, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                             int32_t n_heads_q, const void* q, int64_t ld_q, void* q_out, int64_t ld_q_out,
                             void* stream) {
  abi_clear_error();
  PagedBatch b;
  RotaryArgs r{};
  mar_status s = check_dtype(dtype);
  if (s == MAR_OK) s = take_batch(batch, &b);
  if (s == MAR_OK && rotary) s = take_rotary(rotary, pos, m, b.d_head, &r);
  if (s == MAR_OK) s = check_rows("k", k, ld_k, m, b.n_heads, b.d_head);
  if (s == MAR_OK) s = check_rows("v", v, ld_v, m, b.n_heads, b.d_head);
  if (s == MAR_OK && q) {
    s = check_rows("q", q, ld_q, m, n_heads_q, b.d_head);
    if (s == MAR_OK) s = check_rows("q_out", q_out, ld_q_out, m, n_heads_q, b.d_head);
    if (s == MAR_OK && q_out == q && ld_q_out != ld_q)
      s = fail(MAR_E_ARG, "q_out may be q only with the same row stride");
  }
  if (s != MAR_OK) return s;
  return device_result(launch_paged_store(dtype, b, r, m, k, ld_k, v, ld_v, q ? n_heads_q : 0, q, ld_q, q_out, ld_q_out,
                                          static_cast<hipStream_t>(stream)),
                       "paged store");
}

size_t mar_k_paged_attention_workspace_bytes(int32_t dtype, const mar_paged_batch* batch, int32_t m,
                                             int32_t n_heads_q, int32_t window, int32_t sinks) {
  abi_clear_error();
  PagedBatch b;
  if (take_attention(dtype, batch, m, n_heads_q, window, sinks, &b) != MAR_OK) return 0;
  return paged_attention_workspace(dtype, b, m, n_heads_q, window, sinks);
}

mar_status mar_k_paged_attention(int32_t dtype, const mar_paged_batch* batch, int32_t m, int32_t n_heads_q,
                                 const void* q, int64_t ld_q, int32_t causal, int32_t window, int32_t sinks,
                                 void* workspace, size_t workspace_bytes, void* out, int64_t ld_out, void* stream) {
  abi_clear_error();
  PagedBatch b;
  mar_status s = take_attention(dtype, batch, m, n_heads_q, window, sinks, &b);
  if (s == MAR_OK) s = check_rows("q", q, ld_q, m, n_heads_q, b.d_head);
  if (s == MAR_OK) s = check_rows("out", out, ld_out, m, n_heads_q, b.d_head);
  if (s == MAR_OK && m > 0 && out == q) s = fail(MAR_E_ARG, "out must not be q");
  if (s == MAR_OK && !workspace && workspace_bytes) s = fail(MAR_E_WORKSPACE, "workspace is NULL");
  if (s == MAR_OK && !aligned16(workspace)) s = fail(MAR_E_WORKSPACE, "workspace must be 16-byte aligned");
  if (s != MAR_OK) return s;
  return device_result(launch_paged_attention(dtype, b, m, n_heads_q, q, ld_q, causal != 0, window, sinks, workspace,
                                              workspace_bytes, out, ld_out, static_cast<hipStream_t>(stream)),
                       "paged attention");
}

size_t mar_k_paged_tree_attention_workspace_bytes(int32_t dtype, const mar_paged_batch* batch, int32_t m,
                                                  int32_t n_heads_q, int32_t window, int32_t sinks) {
  abi_clear_error();
  PagedBatch b;
  if (take_attention(dtype, batch, m, n_heads_q, window, sinks, &b) != MAR_OK) return 0;
  return tree_attention_workspace(dtype, b, m, n_heads_q, window, sinks);
}

mar_status mar_k_paged_tree_attention(int32_t dtype, const mar_paged_batch* batch, int32_t m, int32_t n_heads_q,
                                      const void* q, int64_t ld_q, const int32_t* parent, int32_t window,
                                      int32_t sinks, void* workspace, size_t workspace_bytes, void* out,
                                      int64_t ld_out, void* stream) {
  abi_clear_error();
  PagedBatch b;
  mar_status s = take_attention(dtype, batch, m, n_heads_q, window, sinks, &b);
  if (s == MAR_OK) s = check_rows("q", q, ld_q, m, n_heads_q, b.d_head);
  if (s == MAR_OK) s = check_rows("out", out, ld_out, m, n_heads_q, b.d_head);
  if (s == MAR_OK && m > 0 && !parent) s = fail(MAR_E_ARG, "parent is NULL");
  if (s == MAR_OK && m > 0 && out == q) s = fail(MAR_E_ARG, "out must not be q");
  if (s == MAR_OK && !workspace && workspace_bytes) s = fail(MAR_E_WORKSPACE, "workspace is NULL");
  if (s == MAR_OK && !aligned16(workspace)) s = fail(MAR_E_WORKSPACE, "workspace must be 16-byte aligned");
  const unsigned es = dtype == MAR_BF16 ? 2 : 4;
  const int64_t width = static_cast<int64_t>(n_heads_q) * b.d_head;
  if (s == MAR_OK && b.n_seqs > 0) s = check_rows_apart("out", out, ld_out, es, "q", q, ld_q, es, m, width);
  if (s == MAR_OK && b.n_seqs > 0)
    s = check_apart({rows_of("out", out, ld_out, m, width, es), vector_of("parent", parent, m)}, 1);
  if (s != MAR_OK) return s;
  return device_result(launch_tree_attention(dtype, b, m, n_heads_q, q, ld_q, parent, window, sinks, workspace,
                                             workspace_bytes, out, ld_out, static_cast<hipStream_t>(stream)),
                       "tree attention");
}

mar_status mar_k_probabilities(int32_t dtype, const void* logits, int64_t ld, const float* temperature, int32_t m,
                               int32_t vocab, float* out, int64_t ld_out, void* stream) {
  abi_clear_error();
  mar_status s = check_dtype(dtype);
  if (s == MAR_OK) s = check_vocab(m, vocab);
  if (s == MAR_OK) s = check_vocab_rows("logits", logits, ld, m, vocab, dtype == MAR_BF16 ? 2 : 4);
  if (s == MAR_OK) s = check_vocab_rows("out", out, ld_out, m, vocab, 4);
  if (s == MAR_OK && m > 0 && static_cast<const void*>(out) == logits && (dtype != MAR_F32 || ld != ld_out))
    s = fail(MAR_E_ARG, "out may be logits only in fp32 with the same row stride");
  if (s == MAR_OK && static_cast<const void*>(out) != logits)
    s = check_rows_apart("out", out, ld_out, 4, "logits", logits, ld, dtype == MAR_BF16 ? 2 : 4, m, vocab);
  if (s == MAR_OK)
    s = check_apart({rows_of("out", out, ld_out, m, vocab, 4), vector_of("temperature", temperature, m)}, 1);
  if (s != MAR_OK) return s;
  return device_result(launch_probabilities(dtype, logits, ld, temperature, m, vocab, out, ld_out,
                                            static_cast<hipStream_t>(stream)),
                       "probabilities");
}

size_t mar_k_draft_verify_workspace_bytes(int32_t m, int32_t n_seqs, int32_t vocab) {
  abi_clear_error();
  if (check_verify(m, n_seqs, vocab) != MAR_OK) return 0;
  return verify_workspace(m, n_seqs, vocab);
}

mar_status mar_k_draft_verify(int32_t dtype, int32_t n_seqs, const int32_t* q_start, int32_t m, int32_t vocab,
                              const void* p, int64_t ld_p, const void* draft, int64_t ld_draft, const int32_t* parent,
                              const int32_t* tokens, const float* random, int32_t* path, int32_t* kept, int32_t* next,
                              void* workspace, size_t workspace_bytes, void* stream) {
  abi_clear_error();
  const unsigned es = dtype == MAR_BF16 ? 2 : 4;
  mar_status s = check_dtype(dtype);
  if (s == MAR_OK) s = check_verify(m, n_seqs, vocab);
  if (s == MAR_OK) s = check_vocab_rows("p", p, ld_p, m, vocab, es);
  if (s == MAR_OK && draft) s = check_vocab_rows("draft", draft, ld_draft, m, vocab, es);
  if (s == MAR_OK && draft && !random) s = fail(MAR_E_ARG, "draft needs random numbers");
  if (s == MAR_OK && n_seqs > 0 && (!q_start || !kept || !next)) s = fail(MAR_E_ARG, "NULL pointer");
  if (s == MAR_OK && m > 0 && (!parent || !tokens || !path)) s = fail(MAR_E_ARG, "NULL pointer");
  const size_t need = s == MAR_OK ? verify_workspace(m, n_seqs, vocab) : 0;
  if (s == MAR_OK) s = check_workspace(workspace, workspace_bytes, need);
  if (s == MAR_OK && n_seqs > 0)
    s = check_apart({vector_of("path", path, m), vector_of("kept", kept, n_seqs), vector_of("next", next, n_seqs),
                     {"workspace", workspace, need}, vector_of("q_start", q_start, n_seqs + 1),
                     vector_of("parent", parent, m), vector_of("tokens", tokens, m), vector_of("random", random, m),
                     rows_of("p", p, ld_p, m, vocab, es), rows_of("draft", draft, ld_draft, m, vocab, es)},
                    4);
  if (s != MAR_OK) return s;
  const VerifyArgs a{p,    draft, q_start, parent, tokens,   random, path,   kept,
                     next, workspace, ld_p, ld_draft, m, n_seqs, vocab};
  return device_result(launch_verify(dtype, a, static_cast<hipStream_t>(stream)), "draft verify");
}

mar_status mar_k_paged_keep(int32_t dtype, const mar_paged_batch* batch, int32_t m, const int32_t* path,
                            const int32_t* kept, int32_t* kv_len_out, void* stream) {
  abi_clear_error();
  PagedBatch b;
  mar_status s = check_dtype(dtype);
  if (s == MAR_OK) s = take_batch(batch, &b);
  if (s == MAR_OK && (m < 0 || m >= kMaxTokens)) s = fail(MAR_E_SHAPE, "need 0 <= m < 2^30");
  if (s == MAR_OK && ((m > 0 && !path) || (b.n_seqs > 0 && (!kept || !kv_len_out)))) s = fail(MAR_E_ARG, "NULL pointer");
  const int64_t n = s == MAR_OK ? b.n_seqs : 0;
  if (n > 0)
    s = check_apart({vector_of("kv_len_out", kv_len_out, n), vector_of("kv_len", b.kv_len, n),
                     vector_of("q_start", b.q_start, n + 1), vector_of("table", b.table, n * b.max_pages),
                     vector_of("path", path, m), vector_of("kept", kept, n), pages_of("k", b.k, b, dtype),
                     pages_of("v", b.v, b, dtype)},
                    1);
  if (s != MAR_OK) return s;
  return device_result(launch_paged_keep(dtype, b, m, path, kept, kv_len_out, static_cast<hipStream_t>(stream)),
                       "paged keep");
}

size_t mar_k_paged_fork_workspace_bytes(const mar_paged_batch* batch, int32_t n_new) {
  abi_clear_error();
  PagedBatch b;
  if (take_fork(batch, n_new, &b) != MAR_OK) return 0;
  return paged_fork_workspace(b, n_new);
}

mar_status mar_k_paged_fork(int32_t dtype, const mar_paged_batch* batch, int32_t n_new, const int32_t* source,
                            const int32_t* keep, const int32_t* add, int32_t* table_out, int32_t* kv_len_out,
                            int32_t* missing, void* workspace, size_t workspace_bytes, void* stream) {
  abi_clear_error();
  PagedBatch b;
  mar_status s = check_dtype(dtype);
  if (s == MAR_OK) s = take_fork(batch, n_new, &b);
  if (s == MAR_OK && (!missing || (n_new > 0 && (!source || !table_out || !kv_len_out))))
    s = fail(MAR_E_ARG, "NULL pointer");
  const size_t need = s == MAR_OK ? paged_fork_workspace(b, n_new) : 0;
  if (s == MAR_OK) s = check_workspace(workspace, workspace_bytes, need);
  if (s == MAR_OK)
    s = check_apart({vector_of("table_out", table_out, static_cast<int64_t>(n_new) * b.max_pages),
                     vector_of("kv_len_out", kv_len_out, n_new), vector_of("missing", missing, 1),
                     {"workspace", workspace, need}, pages_of("k", b.k, b, dtype), pages_of("v", b.v, b, dtype),
                     vector_of("table", b.table, static_cast<int64_t>(b.n_seqs) * b.max_pages),
                     vector_of("kv_len", b.kv_len, b.n_seqs), vector_of("source", source, n_new),
                     vector_of("keep", keep, n_new), vector_of("add", add, n_new)},
                    4);
  if (s != MAR_OK) return s;
  return device_result(launch_paged_fork(dtype, b, n_new, source, keep, add, table_out, kv_len_out, missing, workspace,
                                         static_cast<hipStream_t>(stream)),
                       "paged fork");
}

}  // extern "C"
