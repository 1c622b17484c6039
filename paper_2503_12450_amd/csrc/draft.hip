// Probabilities of logits, and the verification of drafted tokens.
#include <algorithm>

#include "draft.h"

namespace marcache {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_huge_valf();
constexpr float kLowest = -3.40282347e38f;
constexpr float kCold = 0x1p-100f;  // temperatures up to here count as 0: 1 / T stays finite
constexpr float kLeast = 0x1p-149f;  // 2 log2(e) / T at least, see probabilities

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
//
// Bound by reading the logits and writing fp32: the first HELD x THREADS sixteen-byte
// pieces of a row stay in registers between the passes, so that it is read once
// (600 rows of 65536 in bf16, 236 MB: 56 us, 4.2 TB/s; read twice 68; with streaming
// stores 80); what a longer row has beyond them is read again.
//
// The exponent is (x / 2 - max / 2) (2 log2(e) / T): x - max itself passes the largest
// fp32 number where logits lie further apart, which a temperature of 10^37 and more still
// weighs.  (One FMA in place of the difference, and as exact.)  The factor stays
// above 0, so that -infinity weighs 0 at an infinite temperature too; finite logits then
// weigh the same but for 2^-21 at the most.
//   Four roundings of the exponent (log2(e), the factor, the difference, the product)
// make a probability 2^-a off by up to 4 a ln2 2^-24 of itself, exp2 and the division by
// 2^-23 more: 0.7e-7 to 1.3e-7 of the whole on rows of 32000 and 65536 logits (every
// difference divided by T and then exp: half of that or less), as 1 / T once a row costs
// no division for every logit.
// ---------------------------------------------------------------------------
template <typename T, int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void probabilities(const T* logits, long ld, const float* temperature, int first,
                                                         int vocab, float* out, long ld_out) {
  constexpr int N = kPer<T>, WAVES = THREADS / 64;
  __shared__ float sm[WAVES], ss[WAVES];
  __shared__ int si[WAVES];
  const long row = static_cast<long>(first) + blockIdx.x;
  const T* x = logits + row * ld;
  float* y = out + row * ld_out;
  const float temp = temperature ? temperature[row] : 1.f;
  const bool cold = !(temp > kCold);
  const float scale = cold ? 0.f : fmaxf(2.f * kLog2e / temp, kLeast);
  const int wave = threadIdx.x >> 6, whole = vocab / N, tid = threadIdx.x;
  // the piece g of the row, v[0 .. n) its elements
  u32x4_t held[HELD];
#pragma unroll
  for (int k = 0; k < HELD; ++k)
    if (tid + k * THREADS < whole) held[k] = load_any(x + N * (tid + k * THREADS));
  const int odd = N * whole + tid;  // the row's last, single elements
  const float alone = odd < vocab ? load_one(x + odd) : 0.f;
  auto each = [&](auto&& take) {
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
      const int g = tid + k * THREADS;
      if (g >= whole) continue;
      float v[N];
      unpack16(held[k], v, static_cast<const T*>(nullptr));
      take(v, N * g);
    }
    for (int g = tid + HELD * THREADS; g < whole; g += THREADS) {
      float v[N];
      unpack16(load_any(x + N * g), v, static_cast<const T*>(nullptr));
      take(v, N * g);
    }
  };
  if (cold) {
    float top = -kInf;
    int at = vocab;
    auto take = [&](float v, int i) {
      at = v > top ? i : at;
      top = fmaxf(top, v);
    };
    each([&](const float* v, int i) {
#pragma unroll
      for (int e = 0; e < N; ++e) take(v[e], i + e);
    });
    if (odd < vocab) take(alone, odd);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) better(top, at, __shfl_xor(top, o, 64), __shfl_xor(at, o, 64));
    if ((tid & 63) == 0) {
      sm[wave] = top;
      si[wave] = at;
    }
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) better(top, at, sm[w], si[w]);
    for (int g = tid; g < vocab / 4; g += THREADS) {
      any_f32x4_t o;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = 4 * g + k == at ? 0x3F800000u : 0u;
      *reinterpret_cast<any_f32x4_t*>(y + 4 * g) = o;
    }
    if (vocab / 4 * 4 + tid < vocab) y[vocab / 4 * 4 + tid] = vocab / 4 * 4 + tid == at ? 1.f : 0.f;
    return;
  }
  float top = kLowest;  // finite, so that -infinity weighs 0 against it
  each([&](const float* v, int) {
#pragma unroll
    for (int e = 0; e < N; ++e) top = fmaxf(top, v[e]);
  });
  if (odd < vocab) top = fmaxf(top, alone);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if ((tid & 63) == 0) sm[wave] = top;
  __syncthreads();
  for (int w = 0; w < WAVES; ++w) top = fmaxf(top, sm[w]);
  const float half_top = .5f * top;
  auto weight = [&](float v) { return __builtin_amdgcn_exp2f(fmaf(v, .5f, -half_top) * scale); };
  float sum = 0.f;
  each([&](const float* v, int) {
#pragma unroll
    for (int e = 0; e < N; ++e) sum += weight(v[e]);
  });
  if (odd < vocab) sum += weight(alone);
  sum = wave_sum(sum);
  if ((tid & 63) == 0) ss[wave] = sum;
  __syncthreads();
  sum = 0.f;
  for (int w = 0; w < WAVES; ++w) sum += ss[w];
  const float inv = 1.f / sum;
  each([&](const float* v, int i) {
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      any_f32x4_t o;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = __float_as_uint(weight(v[e + k]) * inv);
      *reinterpret_cast<any_f32x4_t*>(y + i + e) = o;
    }
  });
  if (odd < vocab) y[odd] = weight(alone) * inv;
}

// ---------------------------------------------------------------------------
// Greedy verification: the first maximum of every row.  Bound by reading them.
// ---------------------------------------------------------------------------
constexpr int kBestThreads = 512;

template <typename T>
__global__ __launch_bounds__(kBestThreads) void row_best(const T* p, long ld, int first, int vocab, int32_t* best) {
  constexpr int N = kPer<T>, WAVES = kBestThreads / 64, AHEAD = 8;
  __shared__ float sm[WAVES];
  __shared__ int si[WAVES];
  const long row = static_cast<long>(first) + blockIdx.x;
  const T* x = p + row * ld;
  float top = -kInf;
  int at = vocab;
  const int whole = vocab / N;
  auto take = [&](float v, int i) {
    at = v > top ? i : at;
    top = fmaxf(top, v);
  };
  for (int base = 0; base < whole; base += AHEAD * kBestThreads) {
    u32x4_t x16[AHEAD];
    const int g0 = base + threadIdx.x;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (base + k * kBestThreads < whole)
        x16[k] = load_any(x + static_cast<long>(N) * min(g0 + k * kBestThreads, whole - 1));
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (base + k * kBestThreads >= whole) continue;
      const int g = min(g0 + k * kBestThreads, whole - 1);  // the last one again changes nothing
      float v[N];
      unpack16(x16[k], v, static_cast<const T*>(nullptr));
#pragma unroll
      for (int e = 0; e < N; ++e) take(v[e], N * g + e);
    }
  }
  if (N * whole + static_cast<int>(threadIdx.x) < vocab) {
    const int i = N * whole + threadIdx.x;
    take(load_one(x + i), i);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) better(top, at, __shfl_xor(top, o, 64), __shfl_xor(at, o, 64));
  if ((threadIdx.x & 63) == 0) {
    sm[threadIdx.x >> 6] = top;
    si[threadIdx.x >> 6] = at;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < WAVES; ++w) better(top, at, sm[w], si[w]);
    best[row] = at < vocab ? at : -1;
  }
}

// ---------------------------------------------------------------------------
// The walk down a tree, and the token after it.
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
//
// What the walk asks of p and q are single values, one to a node, which the lanes
// of a wave fetch for all nodes at once; it then runs in registers.  Only a
// rejection that leaves other children (drawn ones) needs a sum over the
// vocabulary on the way; the last one's, and the sum that the next token is drawn
// from, are taken by many workgroups:
//   verify_walk   drawn tokens: the walk, a workgroup to a sequence
//   verify_sums   sums of kTile weights each, a wave to a tile; without a draft
//                 each workgroup repeats the walk, which costs less than a launch
//   verify_pick   the tile that the random number falls into, and the token in it,
//                 a wave to a sequence
// Bound by the three or four dependent loads of each (48 chains of 5 to 9, 65536 tokens
// in fp32: 5.5, 5.2 and 4.8 us, of which reading p and q once would take 4.9; 32 trees
// of 16 to 64, 100003 tokens: 6.5 and 4.5).
//   verify_whole  all of it, a workgroup to a sequence: for few tokens, and for as many
//                 sequences as fill the chip
// ---------------------------------------------------------------------------
constexpr int kWalkThreads = 512;
constexpr int kSumThreads = 256;
constexpr int kTile = 1024;  // tokens of which a wave sums the weights
constexpr int kPart = kTile / 64;
constexpr int kMaxNodes = 256;
constexpr int kChunks = kMaxNodes / 64;

// Values that are no probabilities (negative, infinite, NaN) count as 0.
__device__ __forceinline__ float proper(float x) { return x > 0.f && x < kInf ? x : 0.f; }

// A sequence's rows [row0, row0 + rows), bounded by the m rows; the first kMaxNodes
// are nodes.
struct TreeRows {
  int row0, rows, n;
};
__device__ __forceinline__ TreeRows tree_rows(const VerifyArgs& a, int s) {
  TreeRows t;
  t.row0 = min(max(a.q_start[s], 0), a.m);
  t.rows = max(min(max(a.q_start[s + 1], 0), a.m) - t.row0, 0);
  t.n = min(t.rows, kMaxNodes);
  return t;
}

// Node 64 c + lane in element c: its parent (-1: none), token, random number, and p
// and q of the token in the parent's rows.
struct Nodes {
  int n;
  int parent[kChunks], token[kChunks];
  float r[kChunks], p[kChunks], q[kChunks];
};
__device__ __forceinline__ void load_parents(const VerifyArgs& a, const TreeRows& t, Nodes& d) {
  d.n = t.n;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    d.parent[c] = d.token[c] = -1;
    const int i = 64 * c + static_cast<int>(threadIdx.x & 63);
    if (i < t.n) {
      const int up = a.parent[t.row0 + i];
      d.parent[c] = up >= 0 && up < i ? up : -1;
      d.token[c] = a.tokens[t.row0 + i];
    }
  }
}
template <typename T, bool DRAWN>
__device__ __forceinline__ void load_nodes(const VerifyArgs& a, const TreeRows& t, Nodes& d) {
  load_parents(a, t, d);
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int i = 64 * c + static_cast<int>(threadIdx.x & 63);
    d.r[c] = d.p[c] = d.q[c] = 0.f;
    if (i >= t.n) continue;
    d.r[c] = a.random[t.row0 + i];
    if (d.parent[c] < 0 || d.token[c] < 0 || d.token[c] >= a.vocab) continue;
    const long row = t.row0 + d.parent[c];
    d.p[c] = proper(load_one(static_cast<const T*>(a.p) + row * a.ld_p + d.token[c]));
    if (DRAWN) d.q[c] = proper(load_one(static_cast<const T*>(a.draft) + row * a.ld_draft + d.token[c]));
  }
}
__device__ __forceinline__ int of_node(const int (&v)[kChunks], int i) {
  if (i < 64) return __builtin_amdgcn_readlane(v[0], i);
  int x = 0;
#pragma unroll
  for (int c = 1; c < kChunks; ++c)
    if (i >> 6 == c) x = __builtin_amdgcn_readlane(v[c], i & 63);
  return x;
}
__device__ __forceinline__ float of_node(const float (&v)[kChunks], int i) {
  int bits[kChunks];
#pragma unroll
  for (int c = 0; c < kChunks; ++c) bits[c] = __float_as_int(v[c]);
  return __int_as_float(of_node(bits, i));
}
// The next child of `node` behind node `after` (kMaxNodes: none).
__device__ __forceinline__ int next_child(const Nodes& d, int node, int after) {
  int found = kMaxNodes;
#pragma unroll
  for (int c = kChunks - 1; c >= 0; --c) {
    if (64 * c >= d.n) continue;
    const int i = 64 * c + static_cast<int>(threadIdx.x & 63);
    const uint64_t who = __builtin_amdgcn_ballot_w64(d.parent[c] == node && i > after);
    if (who) found = 64 * c + __builtin_ctzll(who);
  }
  return found;
}
// Whether token x has hung on `node` before node i.
__device__ __forceinline__ bool had_child(const Nodes& d, int node, int i, int x) {
  uint64_t who = 0;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    if (64 * c >= d.n) continue;
    const int j = 64 * c + static_cast<int>(threadIdx.x & 63);
    who |= __builtin_amdgcn_ballot_w64(d.parent[c] == node && j < i && d.token[c] == x);
  }
  return who != 0;
}

// Weights of the tokens after a node: p, and q (null: none) as `rejected` sums W (LDS;
// the first is 1) leave it.
template <typename T, bool DRAWN>
struct Weights {
  const T* p;
  const T* q;
  const double* sums;
  int rejected;
  __device__ __forceinline__ double of(float pv, float qv) const {
    double v = pv;
    if constexpr (DRAWN) {
      const double d = qv;
      if (rejected > 0) v = fmax(v - d, 0.0);
      for (int k = 1; k < rejected; ++k) v = fmax(v / sums[k] - d, 0.0);
    }
    return v;
  }
};
template <typename T, bool DRAWN>
__device__ __forceinline__ Weights<T, DRAWN> weights_of(const VerifyArgs& a, const TreeRows& t, int node, int rejected,
                                                        const double* sums) {
  const long row = t.row0 + node;
  return Weights<T, DRAWN>{static_cast<const T*>(a.p) + row * a.ld_p,
                           DRAWN ? static_cast<const T*>(a.draft) + row * a.ld_draft : nullptr, sums, rejected};
}

// Tokens without weight: those that the children of the final node proposed.
struct Out {
  int32_t* token;  // LDS [kMaxNodes]
  int n;
};
// `write`: this wave fills the list.
__device__ __forceinline__ Out list_children(const Nodes& d, int node, int32_t* token, bool write) {
  Out o{token, 0};
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    if (64 * c >= d.n) continue;
    const bool mine = d.parent[c] == node;
    const uint64_t who = __builtin_amdgcn_ballot_w64(mine);
    if (mine && write) token[o.n + __builtin_popcountll(who & ((uint64_t{1} << lane) - 1))] = d.token[c];
    o.n += __builtin_popcountll(who);
  }
  return o;
}

// A tile's values, 16 tokens to a lane, in order.
struct Values {
  float p[kPart], q[kPart];
};
template <typename T, bool DRAWN>
__device__ __forceinline__ Values load_tile(int vocab, const Weights<T, DRAWN>& w, int tile) {
  constexpr int N = kPer<T>;
  const int i0 = tile * kTile + static_cast<int>(threadIdx.x & 63) * kPart;
  Values x{};
  if (i0 + kPart <= vocab) {
#pragma unroll
    for (int k = 0; k < kPart; k += N) {
      unpack16(load_any(w.p + i0 + k), x.p + k, static_cast<const T*>(nullptr));
      if (DRAWN) unpack16(load_any(w.q + i0 + k), x.q + k, static_cast<const T*>(nullptr));
    }
  } else {
#pragma unroll
    for (int k = 0; k < kPart; ++k) {  // none behind a branch: they are on their way together
      x.p[k] = load_one(w.p + min(i0 + k, vocab - 1));
      if (DRAWN) x.q[k] = load_one(w.q + min(i0 + k, vocab - 1));
    }
#pragma unroll
    for (int k = 0; k < kPart; ++k) x.p[k] = i0 + k < vocab ? x.p[k] : 0.f;
  }
  return x;
}
// Their weights.
template <typename T, bool DRAWN>
__device__ __forceinline__ void tile_weights(const Values& x, const Weights<T, DRAWN>& w, const Out& out, int tile,
                                             double (&v)[kPart]) {
  const int lane = threadIdx.x & 63, i0 = tile * kTile + lane * kPart;
#pragma unroll
  for (int k = 0; k < kPart; ++k) v[k] = w.of(proper(x.p[k]), proper(x.q[k]));
  if (DRAWN) return;
  for (int j0 = 0; j0 < out.n; j0 += 64) {
    const int t = j0 + lane < out.n ? out.token[j0 + lane] : -1;
    for (uint64_t who = __builtin_amdgcn_ballot_w64(t >= 0 && t / kTile == tile); who; who &= who - 1) {
      const int at = __builtin_amdgcn_readlane(t, __builtin_ctzll(who)) - i0;
#pragma unroll
      for (int k = 0; k < kPart; ++k)
        if (k == at) v[k] = 0.0;
    }
  }
}

// Sums of the tiles from, from + step, ... by one wave, the next tile's values on
// their way meanwhile: take(tile, sum).
template <typename T, bool DRAWN, typename Take>
__device__ __forceinline__ void sum_tiles(int vocab, const Weights<T, DRAWN>& w, const Out& out, int from, int step,
                                          Take&& take) {
  const int tiles = (vocab + kTile - 1) / kTile;
  if (from >= tiles) return;
  Values x = load_tile(vocab, w, from);
  for (int tile = from; tile < tiles; tile += step) {
    Values next;
    if (tile + step < tiles) next = load_tile(vocab, w, tile + step);
    double v[kPart], sum = 0.0;
    tile_weights(x, w, out, tile, v);
#pragma unroll
    for (int k = 0; k < kPart; ++k) sum += v[k];
    take(tile, wave_sum(sum));
    if (tile + step < tiles) x = next;
  }
}

// How a walk ended.
struct End {
  int node, kept;
  int rejected;  // drawn: rejections of node's children, the last one's sum not taken
};

// The walk, by every wave of the workgroup; the kept nodes go to `line` (LDS) if `write`.
// sum_of(weights): their sum over the vocabulary.  sums: LDS, W of each rejection.
template <typename T, bool DRAWN, typename Sum>
__device__ __forceinline__ End walk(const VerifyArgs& a, const TreeRows& t, const Nodes& d, int32_t* line, bool write,
                                    double* sums, Sum&& sum_of) {
  End e{0, 1, 0};
  double W = 1.0;
  if (write) line[0] = 0;
  for (int i = next_child(d, 0, 0); i < kMaxNodes;) {
    const Weights<T, DRAWN> w = weights_of<T, DRAWN>(a, t, e.node, e.rejected, sums);
    const float qx = of_node(d.q, i);
    double wx = w.of(of_node(d.p, i), qx);
    if (!DRAWN && had_child(d, e.node, i, of_node(d.token, i))) wx = 0.0;
    const double r = of_node(d.r, i);
    // (W is above 0 as long as the random numbers are below 1)
    if (wx > 0.0 && (DRAWN ? r * static_cast<double>(qx) * W : r * W) < wx) {
      e.node = i;
      if (write) line[e.kept] = i;
      ++e.kept;
      e.rejected = 0;
      W = 1.0;
      i = next_child(d, e.node, i);
      continue;
    }
    i = next_child(d, e.node, i);
    if constexpr (DRAWN) {
      if (write) sums[e.rejected] = W;
      ++e.rejected;
      if (i < kMaxNodes) {
        const double sum = sum_of(weights_of<T, DRAWN>(a, t, e.node, e.rejected, sums));
        if (sum > 0.0)
          W = sum;
        else
          --e.rejected;
      }
    } else {
      W -= wx;
    }
  }
  return e;
}

__device__ __forceinline__ void store_path(const VerifyArgs& a, const TreeRows& t, int s, const End& e,
                                           const int32_t* line) {
  for (int i = threadIdx.x; i < t.rows; i += blockDim.x) a.path[t.row0 + i] = i < e.kept ? line[i] : -1;
  if (threadIdx.x == 0) a.kept[s] = t.n > 0 ? e.kept : 0;
}

// What the kernels leave for each other, one to a sequence.
struct Header {
  int node, rejected;
  double sums[kMaxNodes];
};

template <typename T>
__global__ __launch_bounds__(kWalkThreads) void verify_walk(const VerifyArgs a, Header* headers) {
  __shared__ double sums[kMaxNodes], part[kWalkThreads / 64];
  __shared__ int32_t line[kMaxNodes];
  const int s = blockIdx.x, wave = threadIdx.x >> 6;
  const TreeRows t = tree_rows(a, s);
  Nodes d;
  load_nodes<T, true>(a, t, d);
  const End e = walk<T, true>(a, t, d, line, threadIdx.x == 0, sums, [&](const Weights<T, true>& w) {
    __syncthreads();  // W of the rejection is there, the sums before are read
    double sum = 0.0;
    sum_tiles(a.vocab, w, Out{nullptr, 0}, wave, kWalkThreads / 64, [&](int, double x) { sum += x; });
    if ((threadIdx.x & 63) == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int k = 0; k < kWalkThreads / 64; ++k) sum += part[k];
    return sum;
  });
  __syncthreads();
  store_path(a, t, s, e, line);
  Header* h = headers + s;
  for (int k = threadIdx.x; k < e.rejected; k += kWalkThreads) h->sums[k] = sums[k];
  if (threadIdx.x == 0) {
    h->node = e.node;
    h->rejected = e.rejected;
  }
}

template <typename T, bool DRAWN>
__global__ __launch_bounds__(kSumThreads) void verify_sums(const VerifyArgs a, Header* headers, double* tile_sums,
                                                           int shares) {
  __shared__ double sums[DRAWN ? kMaxNodes : 1];
  __shared__ int32_t line[kMaxNodes], children[kMaxNodes];
  const int s = blockIdx.x / shares, share = blockIdx.x % shares;
  const TreeRows t = tree_rows(a, s);
  Header* h = headers + s;
  int node, rejected = 0;
  Out out{children, 0};
  if constexpr (DRAWN) {
    if (t.n == 0) return;
    node = h->node;
    rejected = h->rejected;
    if (rejected > 1) {  // the first is 1
      for (int k = threadIdx.x; k < rejected; k += kSumThreads) sums[k] = h->sums[k];
      __syncthreads();
    }
  } else {
    Nodes d;
    load_nodes<T, false>(a, t, d);
    const End e = walk<T, false>(a, t, d, line, threadIdx.x == 0, sums, [](const Weights<T, false>&) { return 0.0; });
    out = list_children(d, e.node, children, threadIdx.x < 64);
    node = e.node;
    __syncthreads();
    if (share == 0) {
      store_path(a, t, s, e, line);
      if (threadIdx.x == 0) h->node = node;
    }
    if (t.n == 0) return;
  }
  const Weights<T, DRAWN> w = weights_of<T, DRAWN>(a, t, node, rejected, sums);
  const int tiles = (a.vocab + kTile - 1) / kTile;
  constexpr int waves = kSumThreads / 64;
  sum_tiles(a.vocab, w, out, share * waves + (threadIdx.x >> 6), shares * waves, [&](int tile, double sum) {
    if ((threadIdx.x & 63) == 0) tile_sums[static_cast<long>(s) * tiles + tile] = sum;
  });
}

// The lane's share of the tiles' sums.
__device__ __forceinline__ double lane_total(const double* tile_sums, int tiles) {
  double total = 0.0;
  for (int i = threadIdx.x & 63; i < tiles; i += 64) total += tile_sums[i];
  return total;
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

// The first token at which the summed weights pass r times their sum, given the tiles'
// sums (total: the lanes' shares of them); the last one with a weight if none does.  -1
// if none has any.
template <typename T, bool DRAWN>
__device__ __forceinline__ int pick(int vocab, const Weights<T, DRAWN>& w, const Out& out, const double* tile_sums,
                                    double total, double r) {
  const int tiles = (vocab + kTile - 1) / kTile, lane = threadIdx.x & 63;
  const double goal = r * wave_sum(total);
  double before = 0.0, last_before = 0.0;
  int tile = -1, last = -1;
  for (int i0 = 0; i0 < tiles && tile < 0; i0 += 64) {
    const double mine = i0 + lane < tiles ? tile_sums[i0 + lane] : 0.0;
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
  tile_weights(load_tile(vocab, w, tile), w, out, tile, v);
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

template <typename T, bool DRAWN>
__global__ __launch_bounds__(64) void verify_pick(const VerifyArgs a, const Header* headers, double* tile_sums) {
  __shared__ double sums[DRAWN ? kMaxNodes : 1];
  __shared__ int32_t children[kMaxNodes];
  const int s = blockIdx.x, tiles = (a.vocab + kTile - 1) / kTile;
  // loads that wait for none (a sequence without rows left nothing to read, but room)
  const Header* h = headers + s;
  double* mine = tile_sums + static_cast<long>(s) * tiles;
  const int node = h->node;
  int rejected = DRAWN ? h->rejected : 0;
  double total = lane_total(mine, tiles);
  const TreeRows t = tree_rows(a, s);
  if (t.n == 0) {
    if (threadIdx.x == 0) a.next[s] = -1;
    return;
  }
  const double r = a.random[t.row0];
  Out out{children, 0};
  if constexpr (DRAWN) {
    if (rejected > 1)
      for (int k = threadIdx.x; k < rejected; k += 64) sums[k] = h->sums[k];
  } else {
    Nodes d;
    load_parents(a, t, d);
    out = list_children(d, node, children, true);
  }
  __syncthreads();
  Weights<T, DRAWN> w = weights_of<T, DRAWN>(a, t, node, rejected, sums);
  if constexpr (DRAWN) {
    const bool any = rejected == 0 || __builtin_amdgcn_ballot_w64(total > 0.0) != 0;
    if (!any) {
      // the last rejection left nothing: the weights before it stay
      --w.rejected;
      sum_tiles(a.vocab, w, out, 0, 1, [&](int tile, double sum) {
        if (threadIdx.x == 0) mine[tile] = sum;
      });
      __syncthreads();
      total = lane_total(mine, tiles);
    }
  }
  const int x = pick(a.vocab, w, out, mine, total, r);
  if (threadIdx.x == 0) a.next[s] = x;
}

// All of it by one workgroup to a sequence.
template <typename T, bool DRAWN>
__global__ __launch_bounds__(kWalkThreads) void verify_whole(const VerifyArgs a) {
  constexpr int WAVES = kWalkThreads / 64;
  __shared__ double tile_sums[kMaxVocab / kTile], sums[DRAWN ? kMaxNodes : 1], part[WAVES];
  __shared__ int32_t line[kMaxNodes], children[kMaxNodes];
  const int s = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const TreeRows t = tree_rows(a, s);
  if (t.n == 0) {
    if (threadIdx.x == 0) {
      a.kept[s] = 0;
      a.next[s] = -1;
    }
    return;
  }
  const double r = a.random[t.row0];
  Nodes d;
  load_nodes<T, DRAWN>(a, t, d);
  // the tiles' sums to LDS, their total (of the waves' in order) to all
  auto sum_all = [&](const Weights<T, DRAWN>& w, const Out& out) {
    __syncthreads();  // what w and out read in LDS is there, the sums before are read
    double sum = 0.0;
    sum_tiles(a.vocab, w, out, wave, WAVES, [&](int tile, double x) {
      sum += x;
      if (lane == 0) tile_sums[tile] = x;
    });
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int k = 0; k < WAVES; ++k) sum += part[k];
    return sum;
  };
  const End e = walk<T, DRAWN>(a, t, d, line, threadIdx.x == 0, sums,
                               [&](const Weights<T, DRAWN>& w) { return sum_all(w, Out{nullptr, 0}); });
  Out out{children, 0};
  if (!DRAWN) out = list_children(d, e.node, children, wave == 0);
  Weights<T, DRAWN> w = weights_of<T, DRAWN>(a, t, e.node, e.rejected, sums);
  if (!(sum_all(w, out) > 0.0) && DRAWN && w.rejected > 0) {
    // the last rejection left nothing: the weights before it stay
    --w.rejected;
    sum_all(w, out);
  }
  store_path(a, t, s, e, line);
  if (wave == 0) {
    const int x = pick(a.vocab, w, out, tile_sums, lane_total(tile_sums, (a.vocab + kTile - 1) / kTile), r);
    if (lane == 0) a.next[s] = x;
  }
}

// The walk where the first maximum of each row is known: a wave to a sequence.
__global__ __launch_bounds__(64) void verify_best(const VerifyArgs a, const int32_t* best) {
  __shared__ int32_t line[kMaxNodes];
  const int s = blockIdx.x;
  const TreeRows t = tree_rows(a, s);
  Nodes d;
  load_parents(a, t, d);
  int mine[kChunks];
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int i = 64 * c + static_cast<int>(threadIdx.x);
    mine[c] = i < t.n ? best[t.row0 + i] : -1;
  }
  End e{0, 1, 0};
  if (threadIdx.x == 0) line[0] = 0;
  int x = of_node(mine, 0);
  for (int i = 0; x >= 0;) {
    int found = kMaxNodes;
#pragma unroll
    for (int c = kChunks - 1; c >= 0; --c) {
      if (64 * c >= d.n) continue;
      const int j = 64 * c + static_cast<int>(threadIdx.x);
      const uint64_t who = __builtin_amdgcn_ballot_w64(d.parent[c] == e.node && j > i && d.token[c] == x);
      if (who) found = 64 * c + __builtin_ctzll(who);
    }
    if (found == kMaxNodes) break;
    i = e.node = found;
    if (threadIdx.x == 0) line[e.kept] = found;
    ++e.kept;
    x = of_node(mine, found);
  }
  __syncthreads();
  store_path(a, t, s, e, line);
  if (threadIdx.x == 0) a.next[s] = t.n > 0 ? x : -1;
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// One launch for up to 16384 tokens (a chain drawn from them: 10.6 us, divided 11.4; 48
// chains: 13.0 and 14.2; 65536 tokens: 23 and 18), and from 192 sequences on (200 of
// 65536 tokens: 30 and 35).  It leaves nothing in the workspace.
constexpr int kDividedVocab = 16 * kTile, kDividedSeqs = 191;  // above, up to
bool in_one_launch(int n_seqs, int vocab) { return vocab <= kDividedVocab || n_seqs > kDividedSeqs; }

template <typename T>
hipError_t launch_drawn(const VerifyArgs& a, hipStream_t st) {
  if (in_one_launch(a.n_seqs, a.vocab)) {
    if (a.draft)
      hipLaunchKernelGGL((verify_whole<T, true>), dim3(a.n_seqs), dim3(kWalkThreads), 0, st, a);
    else
      hipLaunchKernelGGL((verify_whole<T, false>), dim3(a.n_seqs), dim3(kWalkThreads), 0, st, a);
    return hipGetLastError();
  }
  Header* headers = static_cast<Header*>(a.ws);
  double* sums = reinterpret_cast<double*>(static_cast<char*>(a.ws) + up16(sizeof(Header) * a.n_seqs));
  // a tile to a wave, but no more workgroups than fill the chip a few times
  const int tiles = (a.vocab + kTile - 1) / kTile, each = kSumThreads / 64;
  const int shares = std::max(1, std::min((tiles + each - 1) / each, 2048 / a.n_seqs));
  const dim3 grid(static_cast<unsigned>(a.n_seqs) * shares);
  if (a.draft) {
    hipLaunchKernelGGL(verify_walk<T>, dim3(a.n_seqs), dim3(kWalkThreads), 0, st, a, headers);
    hipLaunchKernelGGL((verify_sums<T, true>), grid, dim3(kSumThreads), 0, st, a, headers, sums, shares);
    hipLaunchKernelGGL((verify_pick<T, true>), dim3(a.n_seqs), dim3(64), 0, st, a, headers, sums);
  } else {
    hipLaunchKernelGGL((verify_sums<T, false>), grid, dim3(kSumThreads), 0, st, a, headers, sums, shares);
    hipLaunchKernelGGL((verify_pick<T, false>), dim3(a.n_seqs), dim3(64), 0, st, a, headers, sums);
  }
  return hipGetLastError();
}

}  // namespace

// The rows' maxima (greedy), or what the divided form's kernels leave for each other: for
// as many of the sequences as it takes, so that room for many is room for few.
size_t verify_workspace(int m, int n_seqs, int vocab) {
  const size_t best = up16(sizeof(int32_t) * static_cast<size_t>(m));
  if (vocab <= kDividedVocab) return best;
  const size_t seqs = std::min(n_seqs, kDividedSeqs), tiles = (static_cast<size_t>(vocab) + kTile - 1) / kTile;
  return std::max(best, up16(sizeof(Header) * seqs) + sizeof(double) * seqs * tiles);
}

namespace {

template <typename T, int THREADS, int HELD>
hipError_t launch_rows(const void* logits, long ld, const float* temperature, int m, int vocab, float* out, long ld_out,
                       hipStream_t st) {
  constexpr long most = max_grid(THREADS);
  for (long first = 0; first < m; first += most) {
    const dim3 part(static_cast<unsigned>(std::min(most, m - first)));
    hipLaunchKernelGGL((probabilities<T, THREADS, HELD>), part, dim3(THREADS), 0, st, static_cast<const T*>(logits), ld,
                       temperature, static_cast<int>(first), vocab, out, ld_out);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t launch_probabilities_of(const void* logits, long ld, const float* temperature, int m, int vocab, float* out,
                                   long ld_out, hipStream_t st) {
  const long bytes = static_cast<long>(vocab) * sizeof(T);
  // Up to 64 KB of a row many threads hold little each (7 rows of 32000 in bf16: 6.4
  // us, 512 threads 6.9); above, two workgroups to a CU still hold 128 KB (600 rows of
  // 65536: 56 us, 1024 threads 60, 256 threads 61).
  const auto run = bytes <= 8l << 10    ? launch_rows<T, 256, 2>
                   : bytes <= 64l << 10 ? launch_rows<T, 1024, 4>
                                        : launch_rows<T, 512, 16>;
  return run(logits, ld, temperature, m, vocab, out, ld_out, st);
}

}  // namespace

hipError_t launch_probabilities(int dtype, const void* logits, long ld, const float* temperature, int m, int vocab,
                                float* out, long ld_out, hipStream_t st) {
  return dtype == DT_BF16 ? launch_probabilities_of<bf16_t>(logits, ld, temperature, m, vocab, out, ld_out, st)
                          : launch_probabilities_of<float>(logits, ld, temperature, m, vocab, out, ld_out, st);
}

hipError_t launch_verify(int dtype, const VerifyArgs& a, hipStream_t st) {
  if (a.n_seqs == 0) return hipSuccess;
  if (a.random) return dtype == DT_BF16 ? launch_drawn<bf16_t>(a, st) : launch_drawn<float>(a, st);
  int32_t* best = static_cast<int32_t*>(a.ws);
  for (long first = 0; first < a.m; first += kMaxGrid) {
    const dim3 part(static_cast<unsigned>(std::min(kMaxGrid, a.m - first)));
    if (dtype == DT_BF16)
      hipLaunchKernelGGL(row_best<bf16_t>, part, dim3(kBestThreads), 0, st, static_cast<const bf16_t*>(a.p), a.ld_p,
                         static_cast<int>(first), a.vocab, best);
    else
      hipLaunchKernelGGL(row_best<float>, part, dim3(kBestThreads), 0, st, static_cast<const float*>(a.p), a.ld_p,
                         static_cast<int>(first), a.vocab, best);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(verify_best, dim3(a.n_seqs), dim3(64), 0, st, a, best);
  return hipGetLastError();
}

}  // namespace marcache
