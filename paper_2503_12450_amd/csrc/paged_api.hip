// C entry points of the rotary positions, the paged cache and its attention:
// every argument is checked here, on the host, before anything is enqueued.
#include <hip/hip_runtime.h>

#include <cstdarg>

#include "../../include/mar_kernels.h"
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

}  // extern "C"
