// Pages of a cache between steps: accepted rows moved together, and sequences
// that are continued by others.
#include <algorithm>

#include "paged.h"

namespace marcache {

namespace {

// Token t's first element of head 0 in the pages, -1 if it has no place.
__device__ __forceinline__ long token_place(const PagedBatch& b, int s, int t, int limit) {
  if (t < 0 || t >= limit) return -1;
  const int page = b.table[static_cast<long>(s) * b.max_pages + (t >> b.page_shift)];
  if (page < 0 || page >= b.n_pages) return -1;
  return ((static_cast<long>(page) * b.n_heads << b.page_shift) + (t & ((1 << b.page_shift) - 1))) * b.d_head;
}

// ---------------------------------------------------------------------------
// Row path[k] of a sequence goes to the place of row k.  A workgroup takes one
// head of the keys or the values of a sequence, as many rows at a time as it has
// threads for 16 bytes each: all are read before any is written, and as the path
// ascends, rows that come later lie behind every place written so far.
// ---------------------------------------------------------------------------
constexpr int kKeepThreads = 256;

struct KeepArgs {
  PagedBatch b;
  const int32_t* path;
  const int32_t* kept;
  int32_t* kv_out;
  int m, es;       // bytes of an element
  unsigned first;  // work item of workgroup 0
};

__global__ __launch_bounds__(kKeepThreads) void keep_rows(const KeepArgs a) {
  const unsigned w = a.first + blockIdx.x, parts = 2u * a.b.n_heads;
  const int s = w / parts, part = w % parts;
  const int head = part >> 1;
  const int len = a.b.kv_len[s];
  const SeqSpan sp = seq_span(a.b.q_start[s], a.b.q_start[s + 1], len, a.b.max_kv, a.m);
  const int kept = min(max(a.kept[s], 0), sp.n);
  if (part == 0 && threadIdx.x == 0) a.kv_out[s] = sp.n > 0 ? sp.first + kept : len;
  char* base = static_cast<char*>(part & 1 ? a.b.v : a.b.k) +
               (static_cast<long>(head) * a.b.d_head << a.b.page_shift) * a.es;
  const int chunks = a.b.d_head * a.es / 16;
  const int at_once = kKeepThreads / chunks;
  const int r = threadIdx.x / chunks, c = threadIdx.x % chunks;
  for (int k0 = 0; k0 < kept; k0 += at_once) {
    const int k = k0 + r;
    u32x4_t x;
    long to = -1;
    if (r < at_once && k < kept) {
      const int i = a.path[sp.row0 + k];
      if (i > k && i < sp.n) {
        const long of = token_place(a.b, s, sp.first + i, sp.len);
        to = token_place(a.b, s, sp.first + k, sp.len);
        if (of < 0) to = -1;
        if (to >= 0) x = *reinterpret_cast<const u32x4_t*>(base + of * a.es + 16 * c);
      }
    }
    __syncthreads();
    if (to >= 0) *reinterpret_cast<u32x4_t*>(base + to * a.es + 16 * c) = x;
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// New row i of the table continues sequence source[i] with its first keep[i]
// tokens and room for add[i] more.  A page is free if no sequence of the batch
// holds it within its length; what a step needs of them are the lowest, in the
// order of the new rows and their slots, so that equal calls give equal tables.
// A part-filled page that its new row will write to stays that row's if nobody
// else names it, or if all that name it will write to it and the row is the
// lowest of them; the others get a copy of its kept rows.
// ---------------------------------------------------------------------------
struct ForkArgs {
  PagedBatch b;
  const int32_t* source;
  const int32_t* keep;  // nullable: all
  const int32_t* add;   // nullable: none
  int32_t* table_out;
  int32_t* kv_out;
  int32_t* missing;
  // workspace
  int32_t* used;     // [n_pages] by the batch's sequences
  int32_t* names;    // [n_pages] new rows that hold the page
  int32_t* writers;  // [n_pages] new rows that will write to it
  int32_t* lowest;   // [n_pages] the lowest of those
  int32_t* fresh;    // [n_pages] free pages, ascending
  int64_t* begin;    // [n_new + 1] fresh pages given to the rows before; how many there are
  int32_t* copied;   // [n_new] the row's last kept page is copied
  int n_new, es;
  int width;         // fork_plan_small: slots of a sequence at most
  Divisor by_width;
};

struct NewRow {
  int seq, keep, length;  // tokens
  int held, slots;        // pages kept, pages in all
  bool writes;            // to its last kept page
};
__device__ __forceinline__ int slots_of(const PagedBatch& b, int tokens) {
  return (tokens + (1 << b.page_shift) - 1) >> b.page_shift;
}
__device__ __forceinline__ int old_length(const PagedBatch& b, int s) { return min(max(b.kv_len[s], 0), b.max_kv); }
__device__ __forceinline__ NewRow new_row(const ForkArgs& a, int i) {
  NewRow r;
  r.seq = a.source[i];
  const bool real = r.seq >= 0 && r.seq < a.b.n_seqs;
  r.seq = real ? r.seq : 0;
  const int len = real ? old_length(a.b, r.seq) : 0;
  r.keep = a.keep ? min(max(a.keep[i], 0), len) : len;
  const int add = a.add ? max(a.add[i], 0) : 0;
  r.length = r.keep + min(add, (a.b.max_pages << a.b.page_shift) - r.keep);
  r.held = slots_of(a.b, r.keep);
  r.slots = slots_of(a.b, r.length);
  r.writes = r.length > r.keep && (r.keep & ((1 << a.b.page_shift) - 1)) != 0;
  return r;
}
// Page of slot j of sequence s, -1: none.
__device__ __forceinline__ int page_at(const PagedBatch& b, int s, int j) {
  const int page = b.table[static_cast<long>(s) * b.max_pages + j];
  return page >= 0 && page < b.n_pages ? page : -1;
}
// Whether row i has to copy its last kept page, which `names` rows hold and
// `writers` rows write to, the lowest of them `lowest`.
__device__ __forceinline__ bool needs_copy(int i, int names, int writers, int lowest) {
  return names > 1 && !(names == writers && lowest == i);
}

__global__ __launch_bounds__(256) void fork_clear(const ForkArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.b.n_pages) return;
  a.used[i] = a.names[i] = a.writers[i] = 0;
  a.lowest[i] = a.n_new;
}

__global__ __launch_bounds__(256) void fork_mark(const ForkArgs a) {
  const int w = blockIdx.x;
  if (w < a.b.n_seqs) {
    const int n = slots_of(a.b, old_length(a.b, w));
    for (int j = threadIdx.x; j < n; j += 256) {
      const int page = page_at(a.b, w, j);
      if (page >= 0) a.used[page] = 1;
    }
    return;
  }
  const int i = w - a.b.n_seqs;
  const NewRow r = new_row(a, i);
  for (int j = threadIdx.x; j < r.held; j += 256) {
    const int page = page_at(a.b, r.seq, j);
    if (page < 0) continue;
    atomicAdd(a.names + page, 1);
    if (r.writes && j == r.held - 1) {
      atomicAdd(a.writers + page, 1);
      atomicMin(a.lowest + page, i);
    }
  }
}

constexpr int kPlanThreads = 1024;

// v summed over the threads before this one; *total: over all.
__device__ __forceinline__ int64_t sum_before(int64_t v, int64_t* waves, int64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t upto = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t x = __shfl_up(upto, o, 64);
    upto += lane >= o ? x : 0;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int k = 0; k < kPlanThreads / 64; ++k) {
    before += k < wave ? waves[k] : 0;
    all += waves[k];
  }
  *total = all;
  return before + upto - v;
}

__global__ __launch_bounds__(kPlanThreads) void fork_plan(const ForkArgs a) {
  __shared__ int64_t waves[kPlanThreads / 64];
  int64_t need = 0;
  for (int i0 = 0; i0 < a.n_new; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int64_t mine = 0, all;
    if (i < a.n_new) {
      const NewRow r = new_row(a, i);
      const int last = r.writes ? page_at(a.b, r.seq, r.held - 1) : -1;
      const bool copy = last >= 0 && needs_copy(i, a.names[last], a.writers[last], a.lowest[last]);
      a.copied[i] = copy;
      mine = r.slots - r.held + copy;
    }
    const int64_t before = sum_before(mine, waves, &all);
    if (i < a.n_new) a.begin[i] = need + before;
    need += all;
  }
  int64_t have = 0;
  for (int p0 = 0; p0 < a.b.n_pages && have < need; p0 += kPlanThreads) {
    const int p = p0 + threadIdx.x;
    int64_t all;
    const bool is_free = p < a.b.n_pages && a.used[p] == 0;
    const int64_t before = sum_before(is_free, waves, &all);
    if (is_free) a.fresh[have + before] = p;
    have += all;
  }
  if (threadIdx.x == 0) {
    a.begin[a.n_new] = have;
    *a.missing = static_cast<int32_t>(min(max(need - have, int64_t{0}), int64_t{0x7FFFFFFF}));
  }
}

// The same, with the clearing and the marking, where the pages' counts fit into LDS
// and a workgroup walks all slots in a few steps.  Bound by four dependent loads and
// the barriers between them: 144 rows of 16 sequences of 1000 to 8000 tokens in pages
// of 64 take 6.7 us, the three kernels above 1.7, 3.5 and 5.2 and two more launches.
constexpr int kSmallPages = 8192;
constexpr int kSmallSlots = 32 * kPlanThreads;

__global__ __launch_bounds__(kPlanThreads) void fork_plan_small(const ForkArgs a) {
  constexpr int PER = kSmallPages / kPlanThreads;
  __shared__ int names[kSmallPages], writers[kSmallPages], lowest[kSmallPages];
  __shared__ unsigned char used[kSmallPages];
  __shared__ int row_seq[kPlanThreads], row_held[kPlanThreads], old_slots[kPlanThreads], heirs[kPlanThreads];
  __shared__ int64_t waves[kPlanThreads / 64];
  const int tid = threadIdx.x;
  NewRow r{};
  if (tid < a.n_new) r = new_row(a, tid);
  const int slots = tid < a.b.n_seqs ? slots_of(a.b, old_length(a.b, tid)) : 0;
  const int last = tid < a.n_new && r.writes ? page_at(a.b, r.seq, r.held - 1) : -1;
  row_seq[tid] = r.seq;
  row_held[tid] = r.held;
  old_slots[tid] = slots;
  heirs[tid] = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int p = tid + k * kPlanThreads;
    if (p >= a.b.n_pages) break;
    names[p] = writers[p] = 0;
    lowest[p] = kPlanThreads;
    used[p] = 0;
  }
  __syncthreads();
  // rows that keep all of their sequence hold what it holds
  if (!a.keep && r.held > 0) atomicAdd(heirs + r.seq, 1);
  __syncthreads();
  // (a batch without sequences has no table, whose first entries are read below whatever
  // a slot is for; no new row holds a page then)
  const int total = a.b.n_seqs > 0 ? (a.b.n_seqs + (a.keep ? a.n_new : 0)) * a.width : 0;
  for (int k0 = tid; k0 < total; k0 += 4 * kPlanThreads) {
    int page[4], count[4];  // rows that name the page; -1: the sequence itself
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int k = min(k0 + u * kPlanThreads, total - 1);
      const int w = div_by(k, a.by_width.magic, a.by_width.shift), j = k - w * a.width;
      const bool old = w < a.b.n_seqs;
      const int i = old ? w : w - a.b.n_seqs;
      const bool in = k0 + u * kPlanThreads < total && j < (old ? old_slots[i] : row_held[i]);
      page[u] = page_at(a.b, old ? i : row_seq[i], min(j, a.b.max_pages - 1));
      if (!in) page[u] = -1;
      count[u] = old ? (a.keep ? -1 : -1 - heirs[i]) : 1;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (page[u] < 0) continue;
      if (count[u] < 0) used[page[u]] = 1;
      const int rows = count[u] < 0 ? -1 - count[u] : count[u];
      if (rows > 0) atomicAdd(names + page[u], rows);
    }
  }
  if (last >= 0) {
    atomicAdd(writers + last, 1);
    atomicMin(lowest + last, tid);
  }
  __syncthreads();
  const bool copy = last >= 0 && needs_copy(tid, names[last], writers[last], lowest[last]);
  int64_t need, have;
  const int64_t begin = sum_before(tid < a.n_new ? r.slots - r.held + copy : 0, waves, &need);
  if (tid < a.n_new) {
    a.begin[tid] = begin;
    a.copied[tid] = copy;
  }
  int mine = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) mine += PER * tid + k < a.b.n_pages && !used[PER * tid + k];
  int64_t rank = sum_before(mine, waves, &have);
#pragma unroll
  for (int k = 0; k < PER; ++k)
    if (PER * tid + k < a.b.n_pages && !used[PER * tid + k]) {
      if (rank < need) a.fresh[rank] = PER * tid + k;
      ++rank;
    }
  if (tid == 0) {
    a.begin[a.n_new] = have;
    *a.missing = static_cast<int32_t>(min(max(need - have, int64_t{0}), int64_t{0x7FFFFFFF}));
  }
}

__global__ __launch_bounds__(256) void fork_rows(const ForkArgs a, int shares) {
  const int i = blockIdx.x / shares, share = blockIdx.x % shares;
  const NewRow r = new_row(a, i);
  const bool copy = a.copied[i] != 0;
  const int last = copy ? page_at(a.b, r.seq, r.held - 1) : -1;
  const int own = r.held - copy;  // slots from here on are fresh
  const int64_t begin = a.begin[i], have = a.begin[a.n_new];
  auto fresh = [&](int j) { return begin + j - own < have ? a.fresh[begin + j - own] : -1; };
  if (share == 0) {
    int32_t* row = a.table_out + static_cast<long>(i) * a.b.max_pages;
    for (int j = threadIdx.x; j < a.b.max_pages; j += 256)
      row[j] = j < own ? page_at(a.b, r.seq, j) : (j < r.slots ? fresh(j) : -1);
    if (threadIdx.x == 0) a.kv_out[i] = r.length;
  }
  if (last < 0) return;
  const int to = fresh(own);
  if (to < 0) return;
  const int rows = r.keep & ((1 << a.b.page_shift) - 1);
  const int bytes = rows * a.b.d_head * a.es, chunks = bytes / 16;  // of a head
  const long head_bytes = (static_cast<long>(a.b.d_head) << a.b.page_shift) * a.es;
  for (int h = share; h < 2 * a.b.n_heads; h += shares) {
    char* pages = static_cast<char*>(h & 1 ? a.b.v : a.b.k);
    const char* src = pages + (static_cast<long>(last) * a.b.n_heads + (h >> 1)) * head_bytes;
    char* dst = pages + (static_cast<long>(to) * a.b.n_heads + (h >> 1)) * head_bytes;
    for (int c = threadIdx.x; c < chunks; c += 256)
      *reinterpret_cast<u32x4_t*>(dst + 16l * c) = *reinterpret_cast<const u32x4_t*>(src + 16l * c);
  }
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

}  // namespace

hipError_t launch_paged_keep(int dtype, const PagedBatch& b, int m, const int32_t* path, const int32_t* kept,
                             int32_t* kv_out, hipStream_t st) {
  if (b.n_seqs == 0) return hipSuccess;
  KeepArgs a{b, path, kept, kv_out, m, dtype == DT_BF16 ? 2 : 4, 0};
  const long grid = 2l * b.n_heads * b.n_seqs;
  for (long first = 0; first < grid; first += kMaxGrid) {
    a.first = static_cast<unsigned>(first);
    hipLaunchKernelGGL(keep_rows, dim3(static_cast<unsigned>(std::min(kMaxGrid, grid - first))), dim3(kKeepThreads), 0,
                       st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t paged_fork_workspace(const PagedBatch& b, int n_new) {
  return 5 * up16(sizeof(int32_t) * static_cast<size_t>(b.n_pages)) +
         up16(sizeof(int64_t) * (static_cast<size_t>(n_new) + 1)) + sizeof(int32_t) * static_cast<size_t>(n_new);
}

hipError_t launch_paged_fork(int dtype, const PagedBatch& b, int n_new, const int32_t* source, const int32_t* keep,
                             const int32_t* add, int32_t* table_out, int32_t* kv_out, int32_t* missing, void* ws,
                             hipStream_t st) {
  ForkArgs a{};
  a.b = b;
  a.source = source;
  a.keep = keep;
  a.add = add;
  a.table_out = table_out;
  a.kv_out = kv_out;
  a.missing = missing;
  char* at = static_cast<char*>(ws);
  for (int32_t** p : {&a.used, &a.names, &a.writers, &a.lowest, &a.fresh}) {
    *p = reinterpret_cast<int32_t*>(at);
    at += up16(sizeof(int32_t) * static_cast<size_t>(b.n_pages));
  }
  a.begin = reinterpret_cast<int64_t*>(at);
  a.copied = reinterpret_cast<int32_t*>(at + up16(sizeof(int64_t) * (static_cast<size_t>(n_new) + 1)));
  a.n_new = n_new;
  a.es = dtype == DT_BF16 ? 2 : 4;
  a.width = (b.max_kv + (1 << b.page_shift) - 1) >> b.page_shift;
  a.by_width = make_divisor(a.width);
  if (b.n_pages <= kSmallPages && b.n_seqs <= kPlanThreads && n_new <= kPlanThreads &&
      static_cast<long>(b.n_seqs + (keep ? n_new : 0)) * a.width <= kSmallSlots) {
    hipLaunchKernelGGL(fork_plan_small, dim3(1), dim3(kPlanThreads), 0, st, a);
  } else {
    hipLaunchKernelGGL(fork_clear, dim3((b.n_pages + 255u) / 256u), dim3(256), 0, st, a);
    if (b.n_seqs + n_new > 0) hipLaunchKernelGGL(fork_mark, dim3(b.n_seqs + n_new), dim3(256), 0, st, a);
    hipLaunchKernelGGL(fork_plan, dim3(1), dim3(kPlanThreads), 0, st, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (n_new > 0) {
    const int shares = 8;
    hipLaunchKernelGGL(fork_rows, dim3(static_cast<unsigned>(n_new) * shares), dim3(256), 0, st, a, shares);
  }
  return hipGetLastError();
}

}  // namespace marcache
