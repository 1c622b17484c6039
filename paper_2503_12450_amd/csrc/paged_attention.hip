// Attention of a ragged batch of rows over a paged cache.
//
// One workgroup per (row, query head): 256 keys at a time, one per thread,
// with an online softmax; then the threads share the values' columns.
#include <algorithm>

#include "paged.h"

namespace marcache {

namespace {

template <typename T>
__global__ __launch_bounds__(256) void paged_attn_kernel(const PagedBatch b, const T* __restrict__ q, long ld_q,
                                                         T* __restrict__ out, long ld_out, int m, int heads_q,
                                                         bool causal, int window, int sinks, float scale_log2, unsigned first) {
  constexpr int KB = 256;
  __shared__ float qs[128], ps[KB], part[256], red[8];
  __shared__ long off[KB];
  const unsigned block = first + blockIdx.x;
  const int row = block / heads_q, h = block - row * heads_q;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int dh = b.d_head, hk = h / (heads_q / b.n_heads);
  int s = 0, n = b.n_seqs;
  while (n > 1) {
    const int half = n >> 1;
    const bool right = b.q_start[s + half] <= row;
    s = right ? s + half : s;
    n = right ? n - half : half;
  }
  const SeqSpan sp = seq_span(b, s, m);
  if (row < sp.row0 || row >= sp.row0 + sp.n) return;
  const int p = sp.first + row - sp.row0;
  const int hi = causal ? min(sp.len, p + 1) : sp.len;
  const int lo = window > 0 ? max(0, p - min(window, kMaxTokens) + 1) : 0;
  if (tid < dh) qs[tid] = Elem<T>::to_f(q[row * ld_q + h * dh + tid]) * scale_log2;
  const T* kp = static_cast<const T*>(b.k);
  const T* vp = static_cast<const T*>(b.v);
  const int page_mask = (1 << b.page_shift) - 1;
  float m_run = -__builtin_huge_valf(), l_run = 0.f, acc = 0.f;
  const int lanes_d = 256 / dh;  // threads that share a column
  const int d = tid % dh, sub = tid / dh;
  for (int j0 = 0; j0 < hi; j0 += KB) {
    if (j0 + KB <= lo && j0 >= sinks) continue;
    __syncthreads();
    const int j = j0 + tid;
    long at = -1;
    if (j < hi && (j >= lo || j < sinks)) {
      const int page = b.table[static_cast<long>(s) * b.max_pages + (j >> b.page_shift)];
      if (page >= 0 && page < b.n_pages)
        at = (((static_cast<long>(page) * b.n_heads + hk) << b.page_shift) + (j & page_mask)) * dh;
    }
    float sc = -__builtin_huge_valf();
    if (at >= 0) {
      sc = 0.f;
      for (int e = 0; e < dh; ++e) sc = fmaf(qs[e], Elem<T>::to_f(kp[at + e]), sc);
    }
    off[tid] = at;
    float mx = sc;
    for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
    if (lane == 0) red[wave] = mx;
    __syncthreads();
    const float m_new = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m_run);
    const float ref = m_new == -__builtin_huge_valf() ? 0.f : m_new;
    const float alpha = exp2f(m_run - ref);
    const float e = at >= 0 ? exp2f(sc - ref) : 0.f;
    ps[tid] = e;
    const float sum = wave_sum(e);
    if (lane == 0) red[4 + wave] = sum;
    __syncthreads();
    m_run = m_new;
    l_run = l_run * alpha + ((red[4] + red[5]) + (red[6] + red[7]));
    acc *= alpha;
    if (sub < lanes_d)
      for (int t = sub; t < KB; t += lanes_d)
        if (off[t] >= 0) acc = fmaf(ps[t], Elem<T>::to_f(vp[off[t] + d]), acc);
  }
  part[tid] = acc;
  __syncthreads();
  if (tid < dh) {
    float o = 0.f;
    for (int t = 0; t < lanes_d; ++t) o += part[t * dh + tid];
    out[row * ld_out + h * dh + tid] = Elem<T>::from_f(l_run == 0.f ? 0.f : o / l_run);
  }
}

}  // namespace

size_t paged_attention_workspace(int, const PagedBatch&, int, int, int, int) { return 0; }

hipError_t launch_paged_attention(int dtype, const PagedBatch& b, int m, int heads_q, const void* q, long ld_q,
                                  bool causal, int window, int sinks, void*, size_t, void* out, long ld_out,
                                  hipStream_t st) {
  if (m == 0 || b.n_seqs == 0) return hipSuccess;
  const float scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(b.d_head));
  const long grid = static_cast<long>(m) * heads_q;
  for (long first = 0; first < grid; first += kMaxGrid) {
    const dim3 part(static_cast<unsigned>(std::min(kMaxGrid, grid - first)));
    if (dtype == DT_BF16)
      hipLaunchKernelGGL(paged_attn_kernel<bf16_t>, part, dim3(256), 0, st, b, static_cast<const bf16_t*>(q), ld_q,
                         static_cast<bf16_t*>(out), ld_out, m, heads_q, causal, window, sinks, scale_log2,
                         static_cast<unsigned>(first));
    else
      hipLaunchKernelGGL(paged_attn_kernel<float>, part, dim3(256), 0, st, b, static_cast<const float*>(q), ld_q,
                         static_cast<float*>(out), ld_out, m, heads_q, causal, window, sinks, scale_log2,
                         static_cast<unsigned>(first));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace marcache
