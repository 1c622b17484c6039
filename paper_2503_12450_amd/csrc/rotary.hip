// Rotary positions, and new tokens into the pages of the cache.
//
// Memory-bound: every element is read once and written once.  A workgroup
// takes a few consecutive rows: first the cosines and sines of their pairs
// (once per row, shared by all its heads) and the rows' places in the cache go
// to LDS, then its threads walk the heads in units of 16 elements.  A unit
// holds 8 whole pairs in either layout, so a thread reads all that it turns
// before it writes, and the result may overwrite the input.  40960 rows of 32
// heads of 64 in bf16 (336 MB) take 65 us, 5.2 TB/s; 17243 rows into pages, 16 + 2
// x 16 heads of 80 (265 MB), 66 us.  Two rows to a workgroup where there are
// enough: a page's rows of one head are then written side by side (one row: 73
// us; four: 68).
//
// Angles: pos * freq in fp64, in quarter turns, reduced to [-1/2, 1/2] there
// and only then rounded to fp32 (positions reach 2^30, where an fp32 angle
// would be off by whole turns); sine and cosine of the rest in fp32.
#include <algorithm>

#include "paged.h"

namespace marcache {

namespace {

constexpr int kThreads = 256;
constexpr int kRowShift = 1;  // log2 of the rows of a workgroup, where there are enough
constexpr int kMaxRows = 1 << kRowShift;
constexpr int kMaxPairs = 64;

struct RowArgs {
  RotaryArgs rot;
  PagedBatch b;  // STORE only
  const void *q, *k, *v;
  void* q_out;
  long ld_q, ld_k, ld_v, ld_q_out;
  int m, heads_q, d_head;
  int row_shift;                 // 0 or kRowShift
  int first;                     // row of workgroup 0
  Divisor by_units;              // d_head / 16 units of a head
};

__device__ __forceinline__ float2 turn(int pos, double freq) {
  const double t = static_cast<double>(pos) * (freq * 0.63661977236758134308);  // quarter turns
  const double n = __builtin_rint(t);
  const int quadrant = static_cast<int>(n - 4.0 * __builtin_floor(n * 0.25));
  float s, c;
  sincospif(0.5f * static_cast<float>(t - n), &s, &c);
  if (quadrant & 1) {
    const float w = c;
    c = -s;
    s = w;
  }
  return quadrant & 2 ? make_float2(-c, -s) : make_float2(c, s);
}

template <typename T> __device__ __forceinline__ void load8(const T* p, float* x) {
  unpack16(*reinterpret_cast<const u32x4_t*>(p), x, static_cast<const T*>(nullptr));
  if constexpr (sizeof(T) == 4)
    unpack16(*reinterpret_cast<const u32x4_t*>(p + 4), x + 4, static_cast<const T*>(nullptr));
}
__device__ __forceinline__ void store8(bf16_t* p, const float* x) {
  u32x4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack2bf(x[2 * i], x[2 * i + 1]);
  *reinterpret_cast<u32x4_t*>(p) = v;
}
__device__ __forceinline__ void store8(float* p, const float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    *reinterpret_cast<f32x4_t*>(p + 4 * i) = f32x4_t{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
}

template <typename T, bool STORE>
__global__ __launch_bounds__(kThreads) void rows_kernel(const RowArgs a) {
  __shared__ float2 cs[kMaxRows * kMaxPairs];
  __shared__ long place[kMaxRows];  // element of the row's first key in the pages, or -1
  __shared__ int owned[kMaxRows];   // the row belongs to a sequence
  const int row0 = a.first + (blockIdx.x << a.row_shift);
  const int rows = min(1 << a.row_shift, a.m - row0);
  const int P = a.rot.freq ? a.rot.n_pairs : 0;
  const int units = a.d_head / 16;
  const int heads = a.heads_q + (STORE ? 2 * a.b.n_heads : 0);
  const int total = heads * units << a.row_shift;

  // Unit i is piece u of head h of row r; rows run faster than heads, so that
  // the rows of a page's head are written side by side.
  struct Unit {
    int r, h, e0, e1, pair;  // pair < 0: not turned
    bool key, value;
  };
  auto unit_of = [&](int i) {
    Unit t;
    const int hr = div_by(i, a.by_units.magic, a.by_units.shift), u = i - hr * units;
    t.h = hr >> a.row_shift;
    t.r = hr & ((1 << a.row_shift) - 1);
    t.value = STORE && t.h >= a.heads_q + a.b.n_heads;
    t.key = STORE && t.h >= a.heads_q && !t.value;
    const bool turned = u < P / 8 && !t.value;
    const bool halves = turned && !a.rot.neighbours;
    t.pair = turned ? 8 * u : -1;
    t.e0 = halves ? 8 * u : 16 * u;
    t.e1 = halves ? P + 8 * u : 16 * u + 8;
    if (t.key) t.h -= a.heads_q;
    if (t.value) t.h -= a.heads_q + a.b.n_heads;
    return t;
  };
  auto fetch = [&](const Unit& t, float* x) {
    const long row = row0 + t.r;
    const T* src = t.value ? static_cast<const T*>(a.v) + row * a.ld_v
                           : (t.key ? static_cast<const T*>(a.k) + row * a.ld_k
                                    : static_cast<const T*>(a.q) + row * a.ld_q);
    src += t.h * a.d_head;
    load8(src + t.e0, x);
    load8(src + t.e1, x + 8);
  };
  auto finish = [&](const Unit& t, const float* x) {
    T* dst;
    if (!t.key && !t.value) {
      if (STORE && !owned[t.r]) return;
      dst = static_cast<T*>(a.q_out) + (row0 + t.r) * a.ld_q_out + t.h * a.d_head;
    } else {
      if (place[t.r] < 0) return;
      dst = static_cast<T*>(t.value ? a.b.v : a.b.k) + place[t.r] +
            (static_cast<long>(t.h) * a.d_head << a.b.page_shift);
    }
    float y[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) y[j] = x[j];
    if (t.pair >= 0) {
      const float2* c = cs + t.r * kMaxPairs + t.pair;
      if (!a.rot.neighbours) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          y[j] = fmaf(x[j], c[j].x, -x[8 + j] * c[j].y);
          y[8 + j] = fmaf(x[8 + j], c[j].x, x[j] * c[j].y);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          y[2 * j] = fmaf(x[2 * j], c[j].x, -x[2 * j + 1] * c[j].y);
          y[2 * j + 1] = fmaf(x[2 * j + 1], c[j].x, x[2 * j] * c[j].y);
        }
      }
    }
    store8(dst + t.e0, y);
    store8(dst + t.e1, y + 8);
  };

  for (int i = threadIdx.x; i < rows * P; i += kThreads) {
    const int r = i / P, p = i - r * P;
    const int ax = a.rot.axis[p];
    cs[r * kMaxPairs + p] = ax < 0 || ax >= a.rot.n_axes
                                ? make_float2(1.f, 0.f)
                                : turn(a.rot.pos[static_cast<long>(row0 + r) * a.rot.n_axes + ax], a.rot.freq[p]);
  }
  if constexpr (STORE) {
    // a wave per row finds the last sequence that starts at or before it
    const int lane = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < rows; r += kThreads / 64) {
      const int row = row0 + r;
      int lo = 0, n = a.b.n_seqs;
      while (n > 64) {
        const int step = (n + 63) >> 6;
        const bool in = lane * step < n && a.b.q_start[min(lo + lane * step, lo + n - 1)] <= row;
        const int k = max(__builtin_popcountll(__builtin_amdgcn_ballot_w64(in)) - 1, 0);
        lo += k * step;
        n = min(step, n - k * step);
      }
      const int i = lo + min(lane, n - 1);
      const int start = a.b.q_start[i], end = a.b.q_start[i + 1], len = a.b.kv_len[i];
      const int k = max(__builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < n && start <= row)) - 1, 0);
      const SeqSpan s = seq_span(__builtin_amdgcn_readlane(start, k), __builtin_amdgcn_readlane(end, k),
                                 __builtin_amdgcn_readlane(len, k), a.b.max_kv, a.m);
      const bool mine = row >= s.row0 && row < s.row0 + s.n;
      const int t = s.first + row - s.row0;
      long at = -1;
      if (mine && t >= 0 && t < s.len) {
        const int page = a.b.table[static_cast<long>(lo + k) * a.b.max_pages + (t >> a.b.page_shift)];
        if (page >= 0 && page < a.b.n_pages)
          at = ((static_cast<long>(page) * a.b.n_heads << a.b.page_shift) + (t & ((1 << a.b.page_shift) - 1))) *
               a.d_head;
      }
      if (lane == 0) {
        place[r] = at;
        owned[r] = mine;
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < total; i += kThreads) {
    const Unit t = unit_of(i);
    if (t.r >= rows) continue;
    float x[16];
    fetch(t, x);
    finish(t, x);
  }
}

template <bool STORE>
hipError_t launch_rows(int dtype, RowArgs& a, hipStream_t st) {
  const int heads = a.heads_q + (STORE ? 2 * a.b.n_heads : 0);
  if (a.m == 0 || heads == 0 || (STORE && a.b.n_seqs == 0)) return hipSuccess;
  a.row_shift = a.m >= 4096 ? kRowShift : 0;
  a.by_units = make_divisor(a.d_head / 16);
  const int rows = 1 << a.row_shift;
  const long grid = (static_cast<long>(a.m) + rows - 1) / rows;
  for (long first = 0; first < grid; first += kMaxGrid) {
    a.first = static_cast<int>(first * rows);
    const dim3 part(static_cast<unsigned>(std::min(kMaxGrid, grid - first)));
    if (dtype == DT_BF16)
      hipLaunchKernelGGL((rows_kernel<bf16_t, STORE>), part, dim3(kThreads), 0, st, a);
    else
      hipLaunchKernelGGL((rows_kernel<float, STORE>), part, dim3(kThreads), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(int dtype, const RotaryArgs& rot, const void* x, long ld_x, int m, int heads, int d_head,
                         void* out, long ld_out, hipStream_t st) {
  RowArgs a{};
  a.rot = rot;
  a.q = x;
  a.ld_q = ld_x;
  a.q_out = out;
  a.ld_q_out = ld_out;
  a.m = m;
  a.heads_q = heads;
  a.d_head = d_head;
  return launch_rows<false>(dtype, a, st);
}

hipError_t launch_paged_store(int dtype, const PagedBatch& b, const RotaryArgs& rot, int m, const void* k, long ld_k,
                              const void* v, long ld_v, int heads_q, const void* q, long ld_q, void* q_out,
                              long ld_q_out, hipStream_t st) {
  RowArgs a{};
  a.rot = rot;
  a.b = b;
  a.q = q;
  a.ld_q = ld_q;
  a.q_out = q_out;
  a.ld_q_out = ld_q_out;
  a.k = k;
  a.ld_k = ld_k;
  a.v = v;
  a.ld_v = ld_v;
  a.m = m;
  a.heads_q = heads_q;
  a.d_head = b.d_head;
  return launch_rows<true>(dtype, a, st);
}

}  // namespace marcache
