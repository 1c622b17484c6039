// Probabilities of logits, and the verification of drafted tokens.
#include <algorithm>

#include "draft.h"

namespace marcache {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_huge_valf();
constexpr float kLowest = -3.40282347e38f;
constexpr float kCold = 0x1p-100f;  // temperatures up to here count as 0: 1 / T stays finite

// Rows of any length start at any element: sixteen bytes from there.
typedef uint32_t any_f32x4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t any_bf16x8_t __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> struct Any;
template <> struct Any<float> { typedef any_f32x4_t type; };
template <> struct Any<bf16_t> { typedef any_bf16x8_t type; };
template <typename T> constexpr int kPer = 16 / sizeof(T);

template <typename T> __device__ __forceinline__ u32x4_t load_any(const T* p) {
  return *reinterpret_cast<const typename Any<T>::type*>(p);
}
template <typename T> __device__ __forceinline__ float load_one(const T* p) { return Elem<T>::to_f(*p); }

// (value, index): the larger value, of equals the lower index.
__device__ __forceinline__ void better(float& v, int& i, float v2, int i2) {
  const bool take = v2 > v || (v2 == v && i2 < i);
  v = take ? v2 : v;
  i = take ? i2 : i;
}

// ---------------------------------------------------------------------------
// p = exp((x - max) / T) / sum, a workgroup to a row; T 0: one at the first
// maximum.
// ---------------------------------------------------------------------------
constexpr int kProbThreads = 1024;

template <typename T>
__global__ __launch_bounds__(kProbThreads) void probabilities(const T* logits, long ld, const float* temperature,
                                                              int first, int vocab, float* out, long ld_out) {
  constexpr int N = kPer<T>, WAVES = kProbThreads / 64;
  __shared__ float sm[WAVES], ss[WAVES];
  __shared__ int si[WAVES];
  const long row = static_cast<long>(first) + blockIdx.x;
  const T* x = logits + row * ld;
  float* y = out + row * ld_out;
  const float temp = temperature ? temperature[row] : 1.f;
  const bool cold = !(temp > kCold);
  const float scale = cold ? 0.f : kLog2e / temp;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, whole = vocab / N;
  // a finite reference of no values: -infinity weighs 0 against it
  float top = cold ? -kInf : kLowest, sum = 0.f;
  int at = vocab;
  auto take = [&](const float* v, int n, int i0) {
    if (cold) {
      for (int e = 0; e < n; ++e) {
        at = v[e] > top ? i0 + e : at;
        top = fmaxf(top, v[e]);
      }
      return;
    }
    float m = top;
    for (int e = 0; e < n; ++e) m = fmaxf(m, v[e]);
    sum *= __builtin_amdgcn_exp2f((top - m) * scale);
    for (int e = 0; e < n; ++e) sum += __builtin_amdgcn_exp2f((v[e] - m) * scale);
    top = m;
  };
  for (int g = threadIdx.x; g < whole; g += kProbThreads) {
    float v[N];
    unpack16(load_any(x + N * g), v, static_cast<const T*>(nullptr));
    take(v, N, N * g);
  }
  if (N * whole + static_cast<int>(threadIdx.x) < vocab) {
    const int i = N * whole + threadIdx.x;
    const float v = load_one(x + i);
    take(&v, 1, i);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float m2 = __shfl_xor(top, o, 64), s2 = __shfl_xor(sum, o, 64);
    const int i2 = __shfl_xor(at, o, 64);
    const float m = fmaxf(top, m2);
    sum = sum * __builtin_amdgcn_exp2f((top - m) * scale) + s2 * __builtin_amdgcn_exp2f((m2 - m) * scale);
    better(top, at, m2, i2);
  }
  if (lane == 0) {
    sm[wave] = top;
    ss[wave] = sum;
    si[wave] = at;
  }
  __syncthreads();
  top = sm[0];
  at = si[0];
  for (int w = 1; w < WAVES; ++w) better(top, at, sm[w], si[w]);
  sum = 0.f;
  for (int w = 0; w < WAVES; ++w)
    sum += ss[w] * __builtin_amdgcn_exp2f((sm[w] - top) * scale);
  const float inv = 1.f / sum;
  auto p_of = [&](float v, int i) {
    return cold ? (i == at ? 1.f : 0.f) : __builtin_amdgcn_exp2f((v - top) * scale) * inv;
  };
  for (int g = threadIdx.x; g < whole; g += kProbThreads) {
    float v[N];
    unpack16(load_any(x + N * g), v, static_cast<const T*>(nullptr));
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      any_f32x4_t o;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = __float_as_uint(p_of(v[e + k], N * g + e + k));
      *reinterpret_cast<any_f32x4_t*>(y + N * g + e) = o;
    }
  }
  if (N * whole + static_cast<int>(threadIdx.x) < vocab) {
    const int i = N * whole + threadIdx.x;
    y[i] = p_of(load_one(x + i), i);
  }
}

// ---------------------------------------------------------------------------
// Greedy verification: the first maximum of every row.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void row_best(const T* p, long ld, int first, int vocab, int32_t* best) {
  constexpr int N = kPer<T>;
  __shared__ float sm[4];
  __shared__ int si[4];
  const long row = static_cast<long>(first) + blockIdx.x;
  const T* x = p + row * ld;
  float top = -kInf;
  int at = vocab;
  const int whole = vocab / N;
  for (int g = threadIdx.x; g < whole; g += 256) {
    float v[N];
    unpack16(load_any(x + N * g), v, static_cast<const T*>(nullptr));
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (v[e] > top) {
        top = v[e];
        at = N * g + e;
      }
  }
  if (N * whole + static_cast<int>(threadIdx.x) < vocab) {
    const int i = N * whole + threadIdx.x;
    const float v = load_one(x + i);
    if (v > top) {
      top = v;
      at = i;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) better(top, at, __shfl_xor(top, o, 64), __shfl_xor(at, o, 64));
  if ((threadIdx.x & 63) == 0) {
    sm[threadIdx.x >> 6] = top;
    si[threadIdx.x >> 6] = at;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 4; ++w) better(top, at, sm[w], si[w]);
    best[row] = at < vocab ? at : -1;
  }
}

// ---------------------------------------------------------------------------
// The walk down a tree, and the token after it: a workgroup to a sequence.
//
// cur starts at node 0, and the nodes are looked at in ascending order, those
// whose parent is cur; an accepted one becomes cur.  Without probabilities of
// the draft the weights of cur's tokens are p, without the tokens of the
// children that were rejected.  With them they are computed anew wherever they
// are read, from p, q and the sums W that cur's rejections left: w = p, then w =
// max(w / W - q, 0) for each of them (as the definition has it: the closed form
// max(alpha p - beta q, 0) loses what is left in the difference of two products
// that grow with every rejection).  All of it in fp64: the sums decide between
// tokens.
// ---------------------------------------------------------------------------
constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kTile = 1024;  // tokens of which a wave sums the weights
constexpr int kMaxTiles = kMaxVocab / kTile;
constexpr int kPart = kTile / 64;
constexpr int kMaxNodes = 256;

// Values that are no probabilities (negative, infinite, NaN) count as 0.
__device__ __forceinline__ float proper(float x) { return x > 0.f && x < kInf ? x : 0.f; }

// A sequence's tree: its first kMaxNodes rows [row0, row0 + n), bounded by the m rows.
struct Tree {
  int row0, n, rows;           // nodes; rows of the sequence in all
  const int32_t* parent;       // LDS [n], -1: none
  const int32_t* token;        // LDS [n]
};
__device__ __forceinline__ Tree tree_of(const VerifyArgs& a, int s, int32_t* parent, int32_t* token) {
  Tree t;
  t.row0 = min(max(a.q_start[s], 0), a.m);
  t.rows = max(min(max(a.q_start[s + 1], 0), a.m) - t.row0, 0);
  t.n = min(t.rows, kMaxNodes);
  t.parent = parent;
  t.token = token;
  for (int i = threadIdx.x; i < t.n; i += blockDim.x) {
    const int p = a.parent[t.row0 + i];
    parent[i] = p >= 0 && p < i ? p : -1;
    token[i] = a.tokens[t.row0 + i];
  }
  return t;
}

template <typename T>
struct Weights {
  const T* p;
  const T* q;         // null: none
  const double* sums; // LDS: W of every rejection so far
  int rejected;
  __device__ __forceinline__ double of(float pv, float qv) const {
    double v = proper(pv);
    if (q) {
      const double d = proper(qv);
      if (rejected > 0) v = fmax(v - d, 0.0);  // W of the first is 1
      for (int k = 1; k < rejected; ++k) v = fmax(v / sums[k] - d, 0.0);
    }
    return v;
  }
  __device__ __forceinline__ double at(int i) const { return of(load_one(p + i), q ? load_one(q + i) : 0.f); }
};

// The next child of `node` behind node `after` (t.n: none); all lanes of the wave.
__device__ __forceinline__ int next_child(const Tree& t, int node, int after) {
  for (int i0 = (after + 1) & ~63; i0 < t.n; i0 += 64) {
    const int i = i0 + static_cast<int>(threadIdx.x & 63);
    const uint64_t who = __builtin_amdgcn_ballot_w64(i > after && i < t.n && t.parent[min(i, t.n - 1)] == node);
    if (who) return i0 + __builtin_ctzll(who);
  }
  return t.n;
}
// Whether token x has hung on `node` before node i.
__device__ __forceinline__ bool had_child(const Tree& t, int node, int i, int x) {
  for (int j0 = 0; j0 < i; j0 += 64) {
    const int j = j0 + static_cast<int>(threadIdx.x & 63);
    if (__builtin_amdgcn_ballot_w64(j < i && t.parent[min(j, t.n - 1)] == node && t.token[min(j, t.n - 1)] == x))
      return true;
  }
  return false;
}

// The weights of a tile's tokens 16 to a lane, in order; tokens of node's children are 0
// where the weights have no q.
template <typename T>
__device__ __forceinline__ void tile_weights(const VerifyArgs& a, const Tree& t, int node, const Weights<T>& w,
                                             int tile, double (&v)[kPart]) {
  constexpr int N = kPer<T>;
  const int lane = threadIdx.x & 63, i0 = tile * kTile + lane * kPart;
  float pv[kPart], qv[kPart];
  if (i0 + kPart <= a.vocab) {
#pragma unroll
    for (int k = 0; k < kPart; k += N) {
      unpack16(load_any(w.p + i0 + k), pv + k, static_cast<const T*>(nullptr));
      if (w.q) unpack16(load_any(w.q + i0 + k), qv + k, static_cast<const T*>(nullptr));
    }
  } else {
#pragma unroll
    for (int k = 0; k < kPart; ++k) {
      pv[k] = i0 + k < a.vocab ? load_one(w.p + i0 + k) : 0.f;
      qv[k] = w.q && i0 + k < a.vocab ? load_one(w.q + i0 + k) : 0.f;
    }
  }
#pragma unroll
  for (int k = 0; k < kPart; ++k) v[k] = w.of(pv[k], w.q ? qv[k] : 0.f);
  if (w.q) return;
  for (int j0 = 1; j0 < t.n; j0 += 64) {
    const int j = j0 + lane;
    int x = -1;
    if (j < t.n && t.parent[j] == node) x = t.token[j];
    uint64_t who = __builtin_amdgcn_ballot_w64(x >= 0 && x / kTile == tile);
    for (; who; who &= who - 1) {
      const int out = __builtin_amdgcn_readlane(x, __builtin_ctzll(who)) - i0;
#pragma unroll
      for (int k = 0; k < kPart; ++k)
        if (k == out) v[k] = 0.0;
    }
  }
}

// Sums of every tile into LDS, and their total (in order) to all threads.
template <typename T>
__device__ __forceinline__ double sum_tiles(const VerifyArgs& a, const Tree& t, int node, const Weights<T>& w,
                                            double* sums, double* total) {
  const int tiles = (a.vocab + kTile - 1) / kTile;
  __syncthreads();
  for (int tile = threadIdx.x >> 6; tile < tiles; tile += kWaves) {
    double v[kPart], sum = 0.0;
    tile_weights(a, t, node, w, tile, v);
#pragma unroll
    for (int k = 0; k < kPart; ++k) sum += v[k];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) sums[tile] = sum;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    double mine = 0.0;
    const int per = (tiles + 63) / 64;
    for (int k = 0; k < per; ++k) {
      const int i = threadIdx.x * per + k;
      mine += i < tiles ? sums[i] : 0.0;
    }
    mine = wave_sum(mine);
    if (threadIdx.x == 0) *total = mine;
  }
  __syncthreads();
  return *total;
}

// v summed over the lanes up to and with this one.
__device__ __forceinline__ double scan_add(double v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double x = __shfl_up(v, o, 64);
    v += lane >= o ? x : 0.0;
  }
  return v;
}

// The first token at which the summed weights pass `goal`, given the tiles' sums; the
// last one with a weight if none does, -1 if none has any.  One wave.
template <typename T>
__device__ __forceinline__ int pick(const VerifyArgs& a, const Tree& t, int node, const Weights<T>& w,
                                    const double* sums, double goal) {
  const int tiles = (a.vocab + kTile - 1) / kTile, lane = threadIdx.x & 63;
  double before = 0.0;
  int tile = -1, last = -1;
  double last_before = 0.0;
  for (int i0 = 0; i0 < tiles && tile < 0; i0 += 64) {
    const double mine = i0 + lane < tiles ? sums[i0 + lane] : 0.0;
    const double upto = before + scan_add(mine);
    const uint64_t over = __builtin_amdgcn_ballot_w64(mine > 0.0 && upto > goal);
    const uint64_t some = __builtin_amdgcn_ballot_w64(mine > 0.0);
    if (over) {
      const int k = __builtin_ctzll(over);
      tile = i0 + k;
      before = __shfl(upto - mine, k, 64);
    } else {
      if (some) {
        const int k = 63 - __builtin_clzll(some);
        last = i0 + k;
        last_before = __shfl(upto - mine, k, 64);
      }
      before = __shfl(upto, 63, 64);
    }
  }
  if (tile < 0) {
    if (last < 0) return -1;
    tile = last;
    before = last_before;
  }
  double v[kPart], mine = 0.0;
  tile_weights(a, t, node, w, tile, v);
#pragma unroll
  for (int k = 0; k < kPart; ++k) mine += v[k];
  double upto = before + (scan_add(mine) - mine);
  int first = -1, end = -1;  // this lane's first token past the goal, and last with a weight
#pragma unroll
  for (int k = 0; k < kPart; ++k) {
    upto += v[k];
    if (v[k] > 0.0) {
      end = k;
      if (first < 0 && upto > goal) first = k;
    }
  }
  const uint64_t over = __builtin_amdgcn_ballot_w64(first >= 0), some = __builtin_amdgcn_ballot_w64(end >= 0);
  if (over) {
    const int k = __builtin_ctzll(over);
    return tile * kTile + k * kPart + __shfl(first, k, 64);
  }
  if (!some) return -1;
  const int k = 63 - __builtin_clzll(some);
  return tile * kTile + k * kPart + __shfl(end, k, 64);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify(const VerifyArgs a, int first) {
  __shared__ double sums[kMaxTiles];
  __shared__ double rejections[kMaxNodes];
  __shared__ double total;
  __shared__ int32_t parents[kMaxNodes], tokens[kMaxNodes];
  const int s = first + blockIdx.x;
  const Tree t = tree_of(a, s, parents, tokens);
  if (t.n == 0) {
    if (threadIdx.x == 0) {
      a.kept[s] = 0;
      a.next[s] = -1;
    }
    return;
  }
  int32_t* path = a.path + t.row0;
  for (int i = threadIdx.x; i < t.rows; i += kThreads) path[i] = i == 0 ? 0 : -1;
  __syncthreads();
  int node = 0, kept = 1;
  Weights<T> w;
  double W;
  bool summed;  // sums and W are those of w
  auto stand_on = [&](int i) {
    const long row = t.row0 + i;
    node = i;
    w.p = static_cast<const T*>(a.p) + row * a.ld_p;
    w.q = a.draft ? static_cast<const T*>(a.draft) + row * a.ld_draft : nullptr;
    w.sums = rejections;
    w.rejected = 0;
    W = 1.0;
    summed = false;
  };
  stand_on(0);
  for (int i = next_child(t, 0, 0); i < t.n; i = next_child(t, node, i)) {
    const int x = t.token[i];
    const double r = a.random[t.row0 + i];
    const bool real = x >= 0 && x < a.vocab;
    double wx = real ? w.at(x) : 0.0;
    double qx = 1.0;
    if (w.q)
      qx = real ? static_cast<double>(proper(load_one(w.q + x))) : 0.0;
    else if (had_child(t, node, i, x))
      wx = 0.0;
    if (r * qx * W < wx) {
      if (threadIdx.x == 0) path[kept] = i;
      ++kept;
      stand_on(i);
    } else if (w.q) {
      if (threadIdx.x == 0) rejections[w.rejected] = W;
      ++w.rejected;
      const double sum = sum_tiles(a, t, node, w, sums, &total);
      summed = sum > 0.0;
      if (summed)
        W = sum;
      else
        --w.rejected;
    } else {
      W -= wx;
    }
  }
  double sum = W;
  if (!summed) sum = sum_tiles(a, t, node, w, sums, &total);
  if (threadIdx.x < 64) {
    const int x = pick(a, t, node, w, sums, static_cast<double>(a.random[t.row0]) * sum);
    if (threadIdx.x == 0) {
      a.kept[s] = kept;
      a.next[s] = x;
    }
  }
}

// The walk where the first maximum of each row is known: a wave to a sequence.
__global__ __launch_bounds__(64) void verify_best(const VerifyArgs a, const int32_t* best, int first) {
  __shared__ int32_t parents[kMaxNodes], tokens[kMaxNodes];
  const int s = first + blockIdx.x;
  const Tree t = tree_of(a, s, parents, tokens);
  int node = 0, kept = t.n > 0;
  int32_t* path = a.path + t.row0;
  for (int i = threadIdx.x; i < t.rows; i += 64) path[i] = i == 0 ? 0 : -1;
  int x = t.n > 0 ? best[t.row0] : -1;
  for (int i0 = 0; i0 < t.n; i0 += 64) {
    const int i = i0 + static_cast<int>(threadIdx.x);
    const bool in = i < t.n;
    const int up = in ? t.parent[i] : -1, token = in ? t.token[i] : -1;
    const int mine = in ? best[t.row0 + i] : -1;
    for (int from = 0; from < 64;) {
      const uint64_t who = __builtin_amdgcn_ballot_w64(up == node && token == x && token >= 0) >> from << from;
      if (!who) break;
      const int k = __builtin_ctzll(who);
      node = i0 + k;
      x = __builtin_amdgcn_readlane(mine, k);
      if (threadIdx.x == 0) path[kept] = node;
      ++kept;
      from = k + 1;
    }
  }
  if (threadIdx.x == 0) {
    a.kept[s] = kept;
    a.next[s] = x;
  }
}

}  // namespace

size_t verify_workspace(int m, int n_seqs, int vocab) { return static_cast<size_t>(m) * sizeof(int32_t); }

hipError_t launch_probabilities(int dtype, const void* logits, long ld, const float* temperature, int m, int vocab,
                                float* out, long ld_out, hipStream_t st) {
  for (long first = 0; first < m; first += kMaxGrid) {
    const dim3 part(static_cast<unsigned>(std::min(kMaxGrid, m - first)));
    if (dtype == DT_BF16)
      hipLaunchKernelGGL(probabilities<bf16_t>, part, dim3(kProbThreads), 0, st, static_cast<const bf16_t*>(logits), ld,
                         temperature, static_cast<int>(first), vocab, out, ld_out);
    else
      hipLaunchKernelGGL(probabilities<float>, part, dim3(kProbThreads), 0, st, static_cast<const float*>(logits), ld,
                         temperature, static_cast<int>(first), vocab, out, ld_out);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_verify(int dtype, const VerifyArgs& a, hipStream_t st) {
  if (a.n_seqs == 0) return hipSuccess;
  if (a.random) {
    if (dtype == DT_BF16)
      hipLaunchKernelGGL(verify<bf16_t>, dim3(a.n_seqs), dim3(kThreads), 0, st, a, 0);
    else
      hipLaunchKernelGGL(verify<float>, dim3(a.n_seqs), dim3(kThreads), 0, st, a, 0);
    return hipGetLastError();
  }
  int32_t* best = static_cast<int32_t*>(a.ws);
  for (long first = 0; first < a.m; first += kMaxGrid) {
    const dim3 part(static_cast<unsigned>(std::min(kMaxGrid, a.m - first)));
    if (dtype == DT_BF16)
      hipLaunchKernelGGL(row_best<bf16_t>, part, dim3(256), 0, st, static_cast<const bf16_t*>(a.p), a.ld_p,
                         static_cast<int>(first), a.vocab, best);
    else
      hipLaunchKernelGGL(row_best<float>, part, dim3(256), 0, st, static_cast<const float*>(a.p), a.ld_p,
                         static_cast<int>(first), a.vocab, best);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(verify_best, dim3(a.n_seqs), dim3(64), 0, st, a, best, 0);
  return hipGetLastError();
}

}  // namespace marcache
