// Attention of a ragged batch of rows over a paged cache: causal or not
// (paged_attention.hip), and of trees of drafted tokens (tree_attention.hip).
//
// The rows of a sequence that read one key/value head (its n new tokens times
// the `group` query heads that share the head) are packed, row R = token R /
// group, head R % group, and cut into tiles; a workgroup takes a tile of one
// sequence and head and walks the keys that any of its rows sees: first the
// sinks, then the window, in blocks, with an online softmax.  The softmax
// state of a row stays in the lanes that own it; what a row does not see
// inside a block is masked there, and blocks that no row sees are not read.
//
//   attn_many  128 rows, 32 to each of four waves, which share the key blocks
//              (prompts, frames, chunks)
//   attn_few   32 rows, held by each of four waves, which divide the keys
//              (single tokens and few rows: bound by reading the cache once)
//   attn_f32   16 or 32 rows on the fp32 MFMAs, the keys divided over the waves
//
// Where there are too few tiles to fill the chip, the key blocks of a tile are
// further divided among workgroups, which leave their rows' reference, sum and
// output in the workspace for attn_join.
//
// The files that include this one do so inside a namespace of their own, behind
// paged.h, and set the constant kTree.  It makes the kernels of trees: a sequence's
// new rows are the nodes of trees that grow on its past.  A row
// sees the past as a causal row at its depth would, and of the new tokens itself
// and its ancestors: a bit mask of kMaxTree nodes, which its wave keeps in LDS and
// reads in the few blocks that hold new tokens.
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_huge_valf();
// Reference of no scores: finite, so that 2^(-inf - kNone) is 0, and below every
// finite score, so that the first one overflows against it.
constexpr float kNone = -3.40282347e38f;
// The same of a row that saw tokens, all with scores of -infinity: above kNone, so
// that it stays where waves and parts are joined by the larger reference.
constexpr float kOnlyInf = -3.40282326e38f;
constexpr float kRough = 4096.f;  // see softmax_step
constexpr int kWaves = 4;
constexpr int kGroup = 16;  // keys that always lie in one page
constexpr int kTreeWords = kMaxTree / 64;
constexpr int kXcds = 8;
constexpr int kTileRun = 4;

struct AttnArgs {
  PagedBatch b;
  const void* q;
  void* out;
  const int32_t* parent;  // kTree only: [m], node of the row's sequence
  long ld_q, ld_out;
  int m, heads_q, group;
  Divisor by_group;
  int causal, window, sinks;
  float scale_log2;
  int tile_rows;          // packed rows of a tile
  int tiles;              // bound of the tiles of all sequences
  int parts, part_blocks; // workgroups that share a tile, blocks of keys of each
  float* ws_ml;           // [m * heads_q][parts][2]: reference of the exponents, sum
  float* ws_o;            // [m * heads_q][parts][d_head]
  unsigned first;         // work item of workgroup 0
};

// A tile: rows [r0, r0 + n) of the packed rows of sequence s.
struct Tile {
  SeqSpan sp;
  int s, r0, n;
};

// Tiles are numbered so that sequence s starts at floor(its first packed row /
// tile_rows) + s: numbers ascend, no two sequences share one, and the few that
// name no rows end at once.  Needs no pass over the lengths.  A wave finds the
// sequence of a tile among 64 at a time; with up to 64 that is one round of
// loads, which brings its rows and length along.
__device__ __forceinline__ int first_tile(const AttnArgs& a, int s, int start) {
  return min(max(start, 0), a.m) * a.group / a.tile_rows + s;
}
__device__ __forceinline__ SeqSpan rows_span(const AttnArgs& a, int start, int end, int len) {
  SeqSpan sp = seq_span(start, end, len, a.b.max_kv, a.m);
  if constexpr (kTree) sp.n = min(sp.n, kMaxTree);
  return sp;
}
__device__ __forceinline__ Tile make_tile(const AttnArgs& a, int s, int start, int end, int len, int tile) {
  Tile r;
  r.s = s;
  r.sp = rows_span(a, start, end, len);
  r.r0 = tile * a.tile_rows;
  r.n = tile < 0 ? 0 : min(a.tile_rows, r.sp.n * a.group - r.r0);
  return r;
}
__device__ __forceinline__ Tile find_tile(const AttnArgs& a, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.b.n_seqs;
  while (n > 64) {
    const int step = (n + 63) >> 6;
    const int i = lo + lane * step;
    const bool in = lane * step < n && first_tile(a, i, a.b.q_start[min(i, lo + n - 1)]) <= t;
    const int k = max(__builtin_popcountll(__builtin_amdgcn_ballot_w64(in)) - 1, 0);
    lo += k * step;
    n = min(step, n - k * step);
  }
  const int i = lo + min(lane, n - 1);
  const int start = a.b.q_start[i], end = a.b.q_start[i + 1], len = a.b.kv_len[i];
  const bool in = lane < n && first_tile(a, i, start) <= t;
  const int k = max(__builtin_popcountll(__builtin_amdgcn_ballot_w64(in)) - 1, 0);
  const int s = __builtin_amdgcn_readfirstlane(lo + k);
  const int q0 = __builtin_amdgcn_readlane(start, k);
  return make_tile(a, s, q0, __builtin_amdgcn_readlane(end, k), __builtin_amdgcn_readlane(len, k),
                         __builtin_amdgcn_readfirstlane(t - first_tile(a, s, q0)));
}
// The same for tiles that are taken whole and in turn: of up to 64 sequences
// those with the most tokens come first, and the last tiles of a sequence, so
// that the longest work starts first and the CUs end together (32 sequences of
// 578 to 1553 tokens, d_head 80, 1024 tiles: 77 us; in the sequences' order it
// was 11 us more).
__device__ __forceinline__ Tile find_tile_longest_first(const AttnArgs& a, int t) {
  const int n = a.b.n_seqs;
  if (n > 64) return find_tile(a, a.tiles - 1 - t);
  const int lane = threadIdx.x & 63;
  const int i = min(lane, n - 1);
  const int start = a.b.q_start[i], end = a.b.q_start[i + 1], len = a.b.kv_len[i];
  const int tiles =
      lane < n ? (rows_span(a, start, end, len).n * a.group + a.tile_rows - 1) / a.tile_rows : 0;
  int before = 0;  // tiles of the sequences that come before this lane's
  for (int k = 0; k < n; ++k) {
    const int len_k = __builtin_amdgcn_readlane(len, k), tiles_k = __builtin_amdgcn_readlane(tiles, k);
    before += (len_k > len) | ((len_k == len) & (k < lane)) ? tiles_k : 0;
  }
  const uint64_t mine = __builtin_amdgcn_ballot_w64(t >= before && t < before + tiles);
  const int s = mine ? __builtin_ctzll(mine) : 0;
  const int tile = __builtin_amdgcn_readlane(before, s) + __builtin_amdgcn_readlane(tiles, s) - 1 - t;
  return make_tile(a, s, __builtin_amdgcn_readlane(start, s), __builtin_amdgcn_readlane(end, s),
                         __builtin_amdgcn_readlane(len, s), mine ? tile : -1);
}

// Keys that the row at token p sees: [lo, hi) and those below sinks (and hi).
__device__ __forceinline__ int row_hi(const AttnArgs& a, const SeqSpan& sp, int p) {
  return a.causal ? min(sp.len, p + 1) : sp.len;
}
__device__ __forceinline__ int row_lo(const AttnArgs& a, int p) {
  return a.window ? max(0, p - a.window + 1) : 0;
}

// The pages of 64 consecutive groups of 16 keys, one to a lane, from group 64 *
// batch on: one load per 1024 keys.  Groups past the table's row, and entries
// that name no page, are marked invalid and read page 0, whose keys are then
// masked.
struct PageWindow {
  int batch = -1, page = 0;
  uint64_t valid = 0;
  __device__ __forceinline__ void seek(const PagedBatch& b, int s, int group) {
    if (group >> 6 == batch) return;
    batch = group >> 6;
    const int slot = ((batch << 6) + static_cast<int>(threadIdx.x & 63)) >> (b.page_shift - 4);
    const bool in = slot < b.max_pages;
    page = b.table[static_cast<long>(s) * b.max_pages + (in ? slot : 0)];
    const bool ok = in && page >= 0 && page < b.n_pages;
    valid = __builtin_amdgcn_ballot_w64(ok);
    if (!ok) page = 0;
  }
  __device__ __forceinline__ int page_of(int group) const { return __builtin_amdgcn_readlane(page, group & 63); }
  // validity of the n groups from `group` on, a bit per key
  template <int N> __device__ __forceinline__ uint64_t keys(int group) const {
    const uint64_t bits = valid >> (group & 63);
    if ((bits & ((1u << N) - 1)) == (1u << N) - 1) return N == 4 ? ~uint64_t{0} : (uint64_t{1} << 16 * (N & 3)) - 1;
    uint64_t r = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) r |= (bits >> i & 1) ? uint64_t{0xFFFF} << (16 * i) : 0;
    return r;
  }
};

// First element of key `key` (a multiple of 16) of head hk on `page`.
__device__ __forceinline__ long key_offset(const PagedBatch& b, int page, int hk, int key, int dh) {
  return (((static_cast<long>(page) * b.n_heads + hk) << b.page_shift) + (key & ((1 << b.page_shift) - 1))) * dh;
}

// What a lane's row of a tile is.
struct Row {
  long q_at, out_at;  // element offsets in q and out
  long part;          // index in the workspace
  int hi, lo;         // kTree: of the past
  bool ok;
  const uint64_t* nodes;  // kTree: the new tokens that it sees, a bit each
  int first;              // kTree: token of bit 0
};
__device__ __forceinline__ Row make_row(const AttnArgs& a, const Tile& t, int hk, int i) {
  Row r;
  r.ok = i < t.n;
  const int R = t.r0 + min(i, t.n - 1);
  const int tok = div_by(R, a.by_group.magic, a.by_group.shift);
  const int h = hk * a.group + R - tok * a.group;
  const long row = t.sp.row0 + tok;
  r.q_at = row * a.ld_q + static_cast<long>(h) * a.b.d_head;
  r.out_at = row * a.ld_out + static_cast<long>(h) * a.b.d_head;
  r.part = row * a.heads_q + h;
  if constexpr (kTree) {
    r.hi = min(t.sp.first, t.sp.len);
    r.lo = 0;  // add_nodes knows its depth
    r.first = t.sp.first;
    r.nodes = nullptr;
  } else {
    const int p = t.sp.first + tok;
    r.hi = row_hi(a, t.sp, p);
    r.lo = row_lo(a, p);
  }
  return r;
}

// Parents of the tree's nodes, node 64 w + lane in up[w]; -1: none.
struct Parents {
  int up[kTreeWords];
};
__device__ __forceinline__ Parents load_parents(const AttnArgs& a, const Tile& t) {
  Parents r;
#pragma unroll
  for (int w = 0; w < kTreeWords; ++w) {
    const int k = 64 * w + static_cast<int>(threadIdx.x & 63);
    r.up[w] = -1;
    if (64 * w < t.sp.n) {
      const int p = a.parent[t.sp.row0 + min(k, t.sp.n - 1)];
      r.up[w] = k < t.sp.n && p >= 0 && p < k ? p : -1;
    }
  }
  return r;
}

// The new tokens that a lane's row (row i of the tile) sees go to `nodes`, kTreeWords
// words of LDS for it alone that its wave reads; its depth bounds what it sees of the
// past.  Every lane walks up from its node by lane permutes: as many steps as the
// deepest has ancestors (at most kMaxTree: a parent comes before its child).  All
// lanes take part.
__device__ __forceinline__ void add_nodes(const AttnArgs& a, const Tile& t, const Parents& parents, int i,
                                          uint64_t* nodes, Row& row) {
  const int node = div_by(t.r0 + min(i, t.n - 1), a.by_group.magic, a.by_group.shift);
  auto above = [&](int k) {  // parent of node k (of -1: -1)
    int p = -1;
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w)
      if (64 * w < t.sp.n) {
        const int x = __builtin_amdgcn_ds_bpermute(4 * (k & 63), parents.up[w]);
        p = k >> 6 == w ? x : p;
      }
    return p;
  };
  uint64_t set[kTreeWords] = {};
  int depth = -1;
  for (int k = node; __builtin_amdgcn_ballot_w64(k >= 0) != 0; k = above(k)) {
    const int token = t.sp.first + k;
    const uint64_t bit = k >= 0 && token >= 0 && token < t.sp.len ? uint64_t{1} << (k & 63) : 0;
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) set[w] |= k >> 6 == w ? bit : 0;
    depth += k >= 0;
  }
  if (a.window) {
    row.lo = row_lo(a, t.sp.first + depth);
    // where a tree is deeper than the window, again without the ancestors outside it
    if (__builtin_amdgcn_ballot_w64(depth >= a.window) != 0) {
      int back = 0;  // steps up from the row's own node
      for (int k = node; __builtin_amdgcn_ballot_w64(k >= 0) != 0; k = above(k), ++back) {
        const bool far = k >= 0 && back >= a.window && t.sp.first + depth - back >= a.sinks;
#pragma unroll
        for (int w = 0; w < kTreeWords; ++w) set[w] &= far && k >> 6 == w ? ~(uint64_t{1} << (k & 63)) : ~uint64_t{0};
      }
    }
  }
#pragma unroll
  for (int w = 0; w < kTreeWords; ++w) nodes[w] = set[w];
  row.nodes = nodes;
}
// Which of the 64 keys from key0 on are new tokens that the row sees.
__device__ __forceinline__ uint64_t seen_nodes(const Row& row, int key0) {
  const int from = key0 - row.first;  // node of bit 0
  if (from <= -64 || from >= kMaxTree) return 0;
  if (from < 0) return row.nodes[0] << -from;
  const int w = from >> 6, shift = from & 63;
  uint64_t r = row.nodes[w] >> shift;
  if (shift && w + 1 < kTreeWords) r |= row.nodes[w + 1] << (64 - shift);
  return r;
}

// What rows i .. i + n - 1 of a tile see together: their tokens ascend, so the
// first and the last row bound both ends.
struct Reach {
  int hi_min, hi_max, lo_min, lo_max;  // of no rows: hi_max 0
};
__device__ __forceinline__ Reach rows_reach(const AttnArgs& a, const Tile& t, int i, int n) {
  n = min(n, t.n - i);
  if (n <= 0) return Reach{0, 0, 0, 0};
  const int p0 = t.sp.first + div_by(t.r0 + i, a.by_group.magic, a.by_group.shift);
  const int p1 = t.sp.first + div_by(t.r0 + i + n - 1, a.by_group.magic, a.by_group.shift);
  // a node sees no token after its own, and lies at most as deep as its number
  if constexpr (kTree)
    return Reach{min(t.sp.first, t.sp.len), min(t.sp.len, p1 + 1), row_lo(a, t.sp.first), row_lo(a, p1)};
  return Reach{row_hi(a, t.sp, p0), row_hi(a, t.sp, p1), row_lo(a, p0), row_lo(a, p1)};
}

// The blocks of KB keys that a tile reads: blocks 0 .. sink_blocks - 1, then
// from block0 on, `count` together.
struct Blocks {
  int sink_blocks, block0, count;
  __device__ __forceinline__ int at(int i) const { return i < sink_blocks ? i : block0 + i - sink_blocks; }
};
__device__ __forceinline__ Blocks tile_blocks(const AttnArgs& a, const Tile& t, int kb) {
  const Reach reach = rows_reach(a, t, 0, t.n);
  const int hi = max(reach.hi_max, 0), lo = reach.lo_min;
  Blocks r;
  r.block0 = lo / kb;
  r.sink_blocks = min((min(a.sinks, hi) + kb - 1) / kb, r.block0);
  r.count = r.sink_blocks + max((hi + kb - 1) / kb - r.block0, 0);
  return r;
}

// ---------------------------------------------------------------------------
// bf16: 32 rows by 32 keys at a time on the 32x32x16 MFMAs, transposed so that
// a row stays in one column (lane % 32) of both products:
//   S^T (32 keys x 32 rows) = K Q^T,   O^T (32 d x 32 rows) += V^T P^T.
// Lane (c, h) = (lane % 32, lane / 32) owns row c: S^T leaves it keys
// 8 j + 4 h + i (register 4 j + i), which are the k-slots it feeds to the
// second product; V^T follows that order through transposed LDS reads.
// ---------------------------------------------------------------------------

template <int DH_>
struct Geo {
  static constexpr int DH = DH_;
  static constexpr int DS = DH / 16;         // k-steps of S^T
  static constexpr int DT = (DH + 31) / 32;  // 32-row tiles of O^T
  static constexpr int CH = DH / 8;          // 16-byte chunks of a row
};
// Rows of keys and values in LDS.  A row's chunk c lies at c ^ swizzle(row), so
// that the rows that one LDS access reads fall on different banks as far as the
// row length allows: the keys' 16 rows x 1 chunk, the values' 4 rows x 4 chunks
// (of 16 chunks, a row of banks).
template <int DH_>
struct Dense : Geo<DH_> {  // rows without gaps, as the copies leave them
  using Geo<DH_>::CH;
  static constexpr int ROW = DH_;
  static __device__ __forceinline__ int k_swizzle(int row) {
    return CH == 16 ? row & 15 : CH == 8 ? (row >> 1) & 7 : CH % 4 == 0 ? (row >> 2) & 3 : (row >> 3) & 1;
  }
  static __device__ __forceinline__ int v_swizzle(int row) {
    return CH == 16 ? (row & 3) << 2 : CH == 8 ? (row >> 1 & 1) << 2 : 0;
  }
};
template <int DH_>
struct Padded : Geo<DH_> {  // rows of 4, 8 or 16 chunks
  using Geo<DH_>::CH;
  static constexpr int CHP = CH <= 4 ? 4 : (CH <= 8 ? 8 : 16);
  static constexpr int ROW = 8 * CHP;
  static __device__ __forceinline__ int v_swizzle(int row) {
    return CHP == 16 ? (row & 3) << 2 : (CHP == 8 ? (row >> 1 & 1) << 2 : 0);
  }
};

template <int DH>
struct RowState {
  f32x16_t o[Geo<DH>::DT];
  float t = kNone;  // the score that the exponents refer to
  float l = 0.f;    // this lane's share of the row's sum
  __device__ __forceinline__ RowState() {
#pragma unroll
    for (int t = 0; t < Geo<DH>::DT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  }
};

__device__ __forceinline__ u32x2_t read_tr(const bf16_t* p) {
  typedef __attribute__((ext_vector_type(4))) short s16x4_t;
  return __builtin_bit_cast(
      u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p)));
}

// acc, or NaN if either of two bf16 is an infinity or NaN.
__device__ __forceinline__ float times_zero(uint32_t two, float acc) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, two), __builtin_bit_cast(bf16x2_t, 0u), acc, false);
}
__device__ __forceinline__ uint32_t finite_part(uint32_t two) {
  if ((two & 0x7F80u) == 0x7F80u) two &= 0xFFFF0000u;
  if ((two & 0x7F800000u) == 0x7F800000u) two &= 0xFFFFu;
  return two;
}

// The values' fragments of NSB x 32 keys: element [sb][s2][t] holds keys 32 sb
// + 16 s2 + {4 h + i, 8 + 4 h + i} of column 32 t + c.
template <class G, int NSB>
__device__ __forceinline__ void load_values(const bf16_t* vs, int lane, u32x4_t (&vf)[NSB][2][G::DT]) {
  const int row = 4 * (lane >> 5) + ((lane & 15) >> 2);
  const int col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  // row's swizzle does not change with the multiples of 8 added to it
  const int sw = G::v_swizzle(row);
#pragma unroll
  for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int t = 0; t < G::DT; ++t) {
        // columns past the row's end feed rows of O^T that are never stored
        const int chunk = 32 * t + 32 <= 8 * G::CH ? (32 * t + col) >> 3 : min((32 * t + col) >> 3, G::ROW / 8 - 1);
        const bf16_t* p = vs + (32 * sb + 16 * s2 + row) * G::ROW + 8 * (chunk ^ sw) + (col & 7);
        const u32x2_t lo = read_tr(p), hi = read_tr(p + 8 * G::ROW);
        vf[sb][s2][t] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
      }
}

// Which of the 64 keys from key0 on the row sees, of those that are alive.
__device__ __forceinline__ uint64_t first_bits(int n) {
  return n <= 0 ? 0 : (n >= 64 ? ~uint64_t{0} : (uint64_t{1} << n) - 1);
}
__device__ __forceinline__ uint64_t seen_keys(const Row& row, int key0, int sinks, uint64_t alive) {
  uint64_t seen = first_bits(row.hi - key0) & (~first_bits(row.lo - key0) | first_bits(sinks - key0));
  if constexpr (kTree) seen |= seen_nodes(row, key0);
  return seen & alive;
}

// One block of 32 NSB keys from key0 on, given its scores S^T: mask (unless
// the whole wave sees the whole block), softmax step, second product.
// `alive`: a bit per key whose page exists.
template <class G, int NSB>
__device__ __forceinline__ void softmax_step(RowState<G::DH>& st, f32x16_t (&sc)[NSB], u32x4_t (&vf)[NSB][2][G::DT],
                                             const bf16_t* vs, int key0, const Row& row, int sinks,
                                             uint64_t alive, float scale_log2, bool masked) {
  const int lane = threadIdx.x & 63, hg = lane >> 5;
  uint64_t odd = 0;  // keys whose value row is not finite throughout
  if (masked) {
    const uint64_t seen = seen_keys(row, key0, sinks, alive) >> (4 * hg);
    const uint32_t half[2] = {static_cast<uint32_t>(seen), static_cast<uint32_t>(seen >> 32)};
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t all = static_cast<uint32_t>(__builtin_amdgcn_sbfe(half[sb], 8 * (r >> 2) + (r & 3), 1));
        sc[sb][r] = __uint_as_float((__float_as_uint(sc[sb][r]) & all) | (0xFF800000u & ~all));  // -inf
      }
    // 0 times an unseen infinity or NaN would spoil the row: such values leave
    // the product here, and are added below to the rows that do see them.  Times
    // zero and summed, they show.
    float zero = 0.f;
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int t = 0; t < G::DT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) zero = times_zero(vf[sb][s2][t][i], zero);
    if (__builtin_amdgcn_ballot_w64(!(zero == 0.f)) != 0) {
      zero = 0.f;
      if (lane < 32 * NSB)
#pragma unroll 1
        for (int c = 0; c < G::CH; ++c) {
          const u32x4_t x = *reinterpret_cast<const u32x4_t*>(vs + lane * G::ROW + 8 * (c ^ G::v_swizzle(lane)));
#pragma unroll
          for (int i = 0; i < 4; ++i) zero = times_zero(x[i], zero);
        }
      odd = __builtin_amdgcn_ballot_w64(!(zero == 0.f));
#pragma unroll
      for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
          for (int t = 0; t < G::DT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) vf[sb][s2][t][i] = finite_part(vf[sb][s2][t][i]);
    }
  }
  // p = 2^((s - t) scale) gives the same softmax for any reference t of the row, as
  // long as nothing overflows: t stays until a lane's p of a block add up to more
  // than 2^13, and only then (in the first block, and seldom after it) the maximum
  // is looked for.  Which rows move is their own affair: the others of the wave
  // multiply by 1 and get the same p again.
  // One FMA gives s scale - m, m = t scale rounded.  What the rounding took, up to
  // 2^-24 |m|, is the same factor of every p of one t and falls out of their mean;
  // where references of blocks, waves or parts meet it counts, as little as 2^-13
  // up to |m| = 2^12.  Rows past that (`rough`) take it off in every block; they
  // move by their maximum, not by p that lack it.
  // The weights p are rounded to bf16, as the matrix units take both operands of the
  // second product in one type; two bf16 for each would double that product.  Rows of
  // 4000 normal keys: 1.6e-3 of the output, as much as the output's own rounding to
  // bf16 adds (1.7e-3; 2.3e-3 together).
  u32x4_t pf[NSB][2];
  float psum;
  auto weights = [&](auto arg) {
    psum = 0.f;
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t two = pack2bf(__builtin_amdgcn_exp2f(arg(sc[sb][8 * s2 + 2 * i])),
                                       __builtin_amdgcn_exp2f(arg(sc[sb][8 * s2 + 2 * i + 1])));
          pf[sb][s2][i] = two;
          // the sum of the weights as rounded: they are what the values are
          // multiplied by
          psum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, two),
                                                 __builtin_bit_cast(bf16x2_t, 0x3F803F80u), psum, false);
        }
  };
  const float m = st.t * scale_log2;
  const bool rough = fabsf(m) >= kRough && st.t != kNone;
  weights([&](float s) { return fmaf(s, scale_log2, -m); });
  if (__builtin_amdgcn_ballot_w64(rough || !(psum <= 8192.f)) != 0) {
    float top = kNone;
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, sc[sb][r]);
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float other = __shfl_xor(psum, 32, 64);
    const bool over = rough ? (top - st.t) * scale_log2 > 8.f : !(psum <= 8192.f) || !(other <= 8192.f);
    const bool move = over && top > st.t;
    const float alpha = move ? __builtin_amdgcn_exp2f((st.t - top) * scale_log2) : 1.f;
    st.t = move ? top : st.t;
    st.l *= alpha;
#pragma unroll
    for (int t = 0; t < G::DT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[t][r] *= alpha;
    const float m2 = st.t * scale_log2;
    const float rest = fabsf(m2) >= kRough && st.t != kNone ? fmaf(st.t, scale_log2, -m2) : 0.f;
    weights([&](float s) { return fmaf(s, scale_log2, -m2) - rest; });
  }
  st.l += psum;
#pragma unroll
  for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int t = 0; t < G::DT; ++t)
        st.o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf[sb][s2][t]),
                                                          __builtin_bit_cast(bf16x8_t, pf[sb][s2]), st.o[t], 0, 0, 0);
  for (odd &= alive; odd; odd &= odd - 1) {
    const int at = __builtin_ctzll(odd);
    if (!(seen_keys(row, key0, sinks, alive) >> at & 1)) continue;
#pragma unroll
    for (int t = 0; t < G::DT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (4 * t + j >= G::CH) continue;
        const u32x2_t x = *reinterpret_cast<const u32x2_t*>(vs + at * G::ROW + 8 * ((4 * t + j) ^ G::v_swizzle(at)) +
                                                            4 * hg);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t w = i & 1 ? x[i >> 1] & 0xFFFF0000u : x[i >> 1] << 16;
          if ((w & 0x7F800000u) == 0x7F800000u) st.o[t][4 * j + i] += __uint_as_float(w);
        }
      }
  }
}

// 1 / l.  A row without weights: zeros if it sees no token; 0 / 0 if it sees some
// and every score is -infinity.
__device__ __forceinline__ float inverse_sum(float l, float ref) {
  return l != 0.f ? 1.0f / l : (ref == kNone ? 0.f : __builtin_nanf(""));
}

// Reference `ref` of a row of which blocks from, from + step, ... < to left the sum
// l: tells apart whether one without weights saw a token.  Reads the table again,
// in the waves that have such rows.
template <int KB>
__device__ __forceinline__ float mark_seen(const AttnArgs& a, int s, const Blocks& blocks, int from, int to, int step,
                                           const Row& row, float l, PageWindow& pages, float ref) {
  const bool empty = row.ok && (kTree || row.hi > 0) && l == 0.f;
  if (__builtin_amdgcn_ballot_w64(empty) == 0) return ref;
  uint64_t seen = 0;
  for (int i = from; i < to; i += step) {
    const int group0 = blocks.at(i) * (KB / kGroup);
    pages.seek(a.b, s, group0);
    seen |= seen_keys(row, group0 * kGroup, a.sinks, pages.keys<KB / kGroup>(group0));
  }
  return empty && seen ? kOnlyInf : ref;
}

template <int DH>
__device__ __forceinline__ void load_q(const AttnArgs& a, const Row& row, int hg, u32x4_t (&qf)[Geo<DH>::DS]) {
  const bf16_t* q = static_cast<const bf16_t*>(a.q) + row.q_at;
#pragma unroll
  for (int st = 0; st < Geo<DH>::DS; ++st)
    qf[st] = row.ok ? *reinterpret_cast<const u32x4_t*>(q + 16 * st + 8 * hg) : u32x4_t{0u, 0u, 0u, 0u};
}

// Whether a tile of `count` blocks has one part, which then writes out itself.
__device__ __forceinline__ bool one_part(const AttnArgs& a, int count) {
  return a.parts == 1 || (kTree && count <= a.part_blocks);
}

// The lane's share of its row, finished or as a part: o[t][4 j + i] = O[32 t +
// 8 j + 4 h + i].
template <int DH>
__device__ __forceinline__ void store_row(const AttnArgs& a, const Row& row, const RowState<DH>& st, float l,
                                          int hg, int part, bool whole) {
  if (!row.ok) return;
  if (!whole) {
    const long at = row.part * a.parts + part;
    if (hg == 0) *reinterpret_cast<float2*>(a.ws_ml + 2 * at) = make_float2(st.t, l);
    float* o = a.ws_o + at * DH;
#pragma unroll
    for (int t = 0; t < Geo<DH>::DT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = 32 * t + 8 * j + 4 * hg;
        if (d < DH)
          *reinterpret_cast<f32x4_t*>(o + d) =
              f32x4_t{st.o[t][4 * j], st.o[t][4 * j + 1], st.o[t][4 * j + 2], st.o[t][4 * j + 3]};
      }
    return;
  }
  const float inv = inverse_sum(l, st.t);
  bf16_t* o = static_cast<bf16_t*>(a.out) + row.out_at;
#pragma unroll
  for (int t = 0; t < Geo<DH>::DT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = 32 * t + 8 * j + 4 * hg;
      if (d < DH)
        *reinterpret_cast<u32x2_t*>(o + d) = u32x2_t{pack2bf(st.o[t][4 * j] * inv, st.o[t][4 * j + 1] * inv),
                                                     pack2bf(st.o[t][4 * j + 2] * inv, st.o[t][4 * j + 3] * inv)};
    }
}

// Work item -> (tile, head, part).  Heads run fastest: workgroups are dealt to
// the eight XCDs in turn, so the tiles of one head meet in one L2.  Then the
// tiles, and the parts slowest: short sequences have the first parts only, which
// must not all fall to the same XCDs.
// kTree: the four tiles of a run go to one XCD one after the other, where they read
// the same keys (a tree's rows times the heads that share its keys are several
// tiles); then the heads, the parts, turned on by one with every run, and the runs.
// (64 nodes on 131000 keys, 16 heads of 128 on 2: 97 us, dealt out as above 151.)
__device__ __forceinline__ void work_item(const AttnArgs& a, int& tile, int& hk, int& part) {
  const unsigned w = a.first + blockIdx.x;
  if constexpr (kTree) {
    const unsigned unit = w % kXcds + w / (kXcds * kTileRun) * kXcds;
    const unsigned r = unit / a.b.n_heads, run = r / a.parts;
    hk = unit - r * a.b.n_heads;
    part = (r - run * a.parts + run) % a.parts;
    tile = run * kTileRun + w / kXcds % kTileRun;
    return;
  }
  hk = w % a.b.n_heads;
  const unsigned r = w / a.b.n_heads;
  part = r / a.tiles;
  tile = r - part * a.tiles;
}
// Parts of a tile of `count` blocks.
__device__ __forceinline__ int tile_parts(const AttnArgs& a, int count) {
  return max(1, min(a.parts, (count + a.part_blocks - 1) / a.part_blocks));
}
__device__ __forceinline__ void part_range(const AttnArgs& a, int part, int count, int& from, int& to) {
  from = part * a.part_blocks;
  to = part == a.parts - 1 ? count : min(count, from + a.part_blocks);
}

// Twice sixteen bytes per lane into LDS at k_lds (v_lds) + 16 * lane, each from a
// wave-uniform address and a lane's byte offset.  Issued from asm so that the
// compiler adds no waits of its own; lds_arrived() waits.  Nor does it add the
// wait states that the loads need: one after a write of m0, five after a vector
// instruction that wrote their scalar address (a spilled one comes back that way).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16(const void* k, int koff, unsigned k_lds, const void* v, int voff,
                                       unsigned v_lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2\n\t"
      "s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %5"
      :
      : "s"(k_lds), "v"(koff), "s"(k), "s"(v_lds), "v"(voff), "s"(v)
      : "memory", "m0");
}
#pragma clang diagnostic pop
// All but this wave's last N copies are in LDS and its LDS reads are done; then
// all waves'.
template <int N> __device__ __forceinline__ void lds_arrived() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// LDS operations of one wave execute in order; this keeps the compiler to it.
__device__ __forceinline__ void wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// 128 rows, 32 to a wave; the waves share blocks of 64 keys, which lie in a ring
// in LDS and are copied RING - 1 blocks ahead, a group of 16 keys (of one page)
// by each wave.  A barrier per block: behind it block i is there for all, and
// block i - 1's place is free.
// With two places the next copy is issued right behind that barrier, as it has to
// arrive by the next one.  With three it has two blocks' time and is issued behind
// the block's first product, whose LDS reads then do not wait for its addresses
// (77 against 83 us for 32 frames of 256 rows, 16 heads of 80; with two places
// that would be 567 against 541 us for the chunks below).
// Bound by the vector ALU's part of the softmax (a quarter-rate exp2 per score)
// and by LDS and memory latency that three waves a SIMD (two above d_head 64)
// hide in part: 4 chunks of about 1000 rows on 15000 keys, 16 heads of 128 on 4,
// take 525 us (913 TFLOP/s, matrix units 37 % busy; 105 scalars
// spilled to vector registers); 31605 rows with a window of 1024, 16 heads of 64:
// 199 us (684 TFLOP/s, vector ALUs 72 % busy).  Tiles of 256
// rows (eight waves, or 64 rows to a wave) halve the copies or the LDS reads, but
// leave fewer waves to hide them and are slower.
template <int DH, int RING>
__global__ __launch_bounds__(64 * kWaves, DH <= 64 ? 3 : 2) void attn_many(const AttnArgs a) {
  using G = Dense<DH>;
  constexpr int KB = kWaves * kGroup;
  constexpr int COPIES = (G::CH + 3) / 4;       // of 64 chunks that make a group of 16 rows
  constexpr int REST = 16 * G::CH - 64 * (COPIES - 1);  // chunks of the last one
  __shared__ __align__(256) bf16_t ring[RING][2][KB * G::ROW];
  __shared__ uint64_t nodes[kTree ? 32 * kWaves : 1][kTreeWords];
  int tile_no, hk, part;
  work_item(a, tile_no, hk, part);
  if (kTree && tile_no >= a.tiles) return;
  const Tile tile = find_tile_longest_first(a, tile_no);
  if (tile.n <= 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hg = lane >> 5;
  const Blocks blocks = tile_blocks(a, tile, KB);
  int from, to;
  part_range(a, part, blocks.count, from, to);
  if (from >= to && from > 0) return;  // attn_join knows which parts there are

  // Byte offsets in the group of the chunks that the lane copies.
  int koff[COPIES], voff[COPIES];
#pragma unroll
  for (int k = 0; k < COPIES; ++k) {
    const int piece = min(64 * k + lane, 16 * G::CH - 1), r = piece / G::CH, at = piece % G::CH;
    koff[k] = 2 * (r * DH + 8 * (at ^ G::k_swizzle(r)));
    voff[k] = 2 * (r * DH + 8 * (at ^ G::v_swizzle(r)));
  }
  const unsigned lds0 = static_cast<unsigned>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) bf16_t*)&ring[0][0][kGroup * wave * G::ROW]));
  PageWindow pages;
  uint64_t alive[RING];  // of blocks i, i + 1, ... as they are copied
  auto copy_block = [&](int i) {
    const int group0 = blocks.at(i) * kWaves, group = group0 + wave;
    pages.seek(a.b, tile.s, group0);
    const unsigned lds = lds0 + static_cast<unsigned>(i - from) % RING * (4u * KB * G::ROW);
    const long at = key_offset(a.b, pages.page_of(group), hk, group * kGroup, DH);
    const bf16_t* kp = static_cast<const bf16_t*>(a.b.k) + at;
    const bf16_t* vp = static_cast<const bf16_t*>(a.b.v) + at;
#pragma unroll
    for (int k = 0; k < COPIES; ++k)
      if (k + 1 < COPIES || REST == 64 || lane < REST)
        copy16(kp, koff[k], lds + 1024u * k, vp, voff[k], lds + 1024u * k + 2u * KB * G::ROW);
    return pages.keys<kWaves>(group0);
  };
#pragma unroll
  for (int k = 0; k < RING; ++k) alive[k] = k < RING - 1 && from + k < to ? copy_block(from + k) : 0;
  auto copy_ahead = [&](int i) {
    if (i + RING - 1 < to) alive[RING - 1] = copy_block(i + RING - 1);
#pragma unroll
    for (int k = 0; k + 1 < RING; ++k) alive[k] = alive[k + 1];
  };

  Row row = make_row(a, tile, hk, wave * 32 + c);
  if constexpr (kTree) add_nodes(a, tile, load_parents(a, tile), wave * 32 + c, nodes[wave * 32 + c], row);
  u32x4_t qf[G::DS];
  load_q<DH>(a, row, hg, qf);
  const Reach reach = rows_reach(a, tile, wave * 32, 32);
  RowState<DH> st;
  for (int i = from; i < to; ++i) {
    // of the blocks after i, RING - 2 may still be on their way
    if (i + RING - 2 < to)
      lds_arrived<(RING - 2) * 2 * COPIES>();
    else
      lds_arrived<0>();
    const uint64_t here = alive[0];
    if constexpr (RING == 2) copy_ahead(i);
    const int key0 = blocks.at(i) * KB;
    if (key0 >= reach.hi_max || (key0 + KB <= reach.lo_min && key0 >= a.sinks)) {  // not for this wave
      if constexpr (RING > 2) copy_ahead(i);
      continue;
    }
    const bf16_t* kb = ring[static_cast<unsigned>(i - from) % RING][0];
    const bf16_t* vb = kb + KB * G::ROW;
    f32x16_t sc[2];
#pragma unroll
    for (int sb = 0; sb < 2; ++sb) {
      u32x4_t kf[G::DS];
#pragma unroll
      for (int s = 0; s < G::DS; ++s)
        kf[s] = *reinterpret_cast<const u32x4_t*>(kb + (32 * sb + c) * G::ROW + 8 * ((2 * s + hg) ^ G::k_swizzle(c)));
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[sb][r] = 0.f;
#pragma unroll
      for (int s = 0; s < G::DS; ++s)
        sc[sb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[s]),
                                                         __builtin_bit_cast(bf16x8_t, qf[s]), sc[sb], 0, 0, 0);
    }
    u32x4_t vf[2][2][G::DT];
    load_values<G, 2>(vb, lane, vf);
    if constexpr (RING > 2) copy_ahead(i);
    const bool whole =
        key0 + KB <= reach.hi_min && (key0 >= reach.lo_max || key0 + KB <= a.sinks) && here == ~uint64_t{0};
    softmax_step<G, 2>(st, sc, vf, vb, key0, row, a.sinks, here, a.scale_log2, !whole);
  }
  const float l = st.l + __shfl_xor(st.l, 32, 64);
  st.t = mark_seen<KB>(a, tile.s, blocks, from, to, 1, row, l, pages, st.t);
  store_row<DH>(a, row, st, l, hg, part, one_part(a, blocks.count));
}

// 32 rows; wave w takes blocks w, w + 4, ... of 32 keys.  The keys go from
// memory to the registers that feed the first product, the values through a
// piece of LDS of the wave's own; both are loaded a block ahead.
// Bound by reading the cache once: 64 sequences of 521 to 15919 keys, 32 query
// heads of 128 on 4, 579 MB in 130 us (4.5 TB/s); one of 131001, 16 heads on 2,
// 134 MB in 28 us (4.8 TB/s).  The 32-row products cost nothing there, so single
// tokens share the form of a few rows.
template <int DH>
__global__ __launch_bounds__(64 * kWaves, 2) void attn_few(const AttnArgs a) {
  using G = Padded<DH>;
  constexpr int KB = 32;
  constexpr int RPI = 64 / G::CHP;     // value rows that a wave loads at once
  constexpr int LOADS = KB / RPI;
  constexpr int OROW = DH + 4;         // row stride of the outputs that waves exchange
  constexpr int VBYTES = kWaves * KB * G::ROW * 2, OBYTES = (kWaves / 2) * 32 * (OROW + 2) * 4;
  __shared__ __align__(16) unsigned char lds[VBYTES > OBYTES ? VBYTES : OBYTES];
  __shared__ uint64_t nodes[kTree ? 32 * kWaves : 1][kTreeWords];
  int tile_no, hk, part;
  work_item(a, tile_no, hk, part);
  if (kTree && tile_no >= a.tiles) return;
  const Tile tile = find_tile(a, tile_no);
  if (tile.n <= 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hg = lane >> 5;
  const Blocks blocks = tile_blocks(a, tile, KB);
  int from, to;
  part_range(a, part, blocks.count, from, to);
  if (from >= to && from > 0) return;
  Row row = make_row(a, tile, hk, c);
  u32x4_t qf[G::DS];
  load_q<DH>(a, row, hg, qf);
  const Reach reach = rows_reach(a, tile, 0, tile.n);
  bf16_t* vs = reinterpret_cast<bf16_t*>(lds) + wave * KB * G::ROW;

  PageWindow pages;
  u32x4_t kf[G::DS], vr[LOADS];
  uint64_t alive_next = 0;
  const int vrow = lane / G::CHP, vchunk = lane % G::CHP;
  auto load_block = [&](int i) {
    const int group0 = blocks.at(i) * (KB / kGroup);
    pages.seek(a.b, tile.s, group0);
    alive_next = pages.keys<KB / kGroup>(group0);
    const long at0 = key_offset(a.b, pages.page_of(group0), hk, group0 * kGroup, DH);
    const long at1 = key_offset(a.b, pages.page_of(group0 + 1), hk, (group0 + 1) * kGroup, DH);
    const bf16_t* kp = static_cast<const bf16_t*>(a.b.k) + (c < 16 ? at0 : at1) + (c & 15) * DH + 8 * hg;
#pragma unroll
    for (int s = 0; s < G::DS; ++s) kf[s] = *reinterpret_cast<const u32x4_t*>(kp + 16 * s);
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const int r = RPI * k;  // the rows of a load lie in one group
      const bf16_t* vp = static_cast<const bf16_t*>(a.b.v) + (r < 16 ? at0 : at1) + (r % 16 + vrow) * DH;
      vr[k] = *reinterpret_cast<const u32x4_t*>(vp + 8 * min(vchunk, G::CH - 1));
    }
  };
  RowState<DH> st;
  Parents parents;
  if constexpr (kTree) parents = load_parents(a, tile);
  if (from + wave < to) load_block(from + wave);
  if constexpr (kTree) add_nodes(a, tile, parents, c, nodes[wave * 32 + c], row);  // while they are on their way
  for (int i = from + wave; i < to; i += kWaves) {
    const uint64_t alive = alive_next;
    const int key0 = blocks.at(i) * KB;
#pragma unroll
    for (int k = 0; k < LOADS; ++k)
      *reinterpret_cast<u32x4_t*>(vs + (RPI * k + vrow) * G::ROW + 8 * (vchunk ^ G::v_swizzle(RPI * k + vrow))) = vr[k];
    f32x16_t sc[1];
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[0][r] = 0.f;
#pragma unroll
    for (int s = 0; s < G::DS; ++s)
      sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[s]),
                                                      __builtin_bit_cast(bf16x8_t, qf[s]), sc[0], 0, 0, 0);
    if (i + kWaves < to) load_block(i + kWaves);
    wave_order();
    u32x4_t vf[1][2][G::DT];
    load_values<G, 1>(vs, lane, vf);
    const bool whole =
        key0 + KB <= reach.hi_min && (key0 >= reach.lo_max || key0 + KB <= a.sinks) && (alive & 0xFFFFFFFFu) == 0xFFFFFFFFu;
    softmax_step<G, 1>(st, sc, vf, vs, key0, row, a.sinks, alive, a.scale_log2, !whole);
    wave_order();
  }
  // Join the waves' rows in pairs: the upper half of them leaves reference, sum
  // and output in LDS, the lower half takes them in.
  float l = st.l + __shfl_xor(st.l, 32, 64);
  st.t = mark_seen<KB>(a, tile.s, blocks, from + wave, to, kWaves, row, l, pages, st.t);
  float* ol = reinterpret_cast<float*>(lds);
  float* ml = ol + (kWaves / 2) * 32 * OROW;
#pragma unroll
  for (int half = kWaves / 2; half > 0; half >>= 1) {
    __syncthreads();
    if (wave >= half && wave < 2 * half) {
      float* o = ol + ((wave - half) * 32 + c) * OROW;
#pragma unroll
      for (int t = 0; t < G::DT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int d = 32 * t + 8 * j + 4 * hg;
          if (d < DH)
            *reinterpret_cast<f32x4_t*>(o + d) =
                f32x4_t{st.o[t][4 * j], st.o[t][4 * j + 1], st.o[t][4 * j + 2], st.o[t][4 * j + 3]};
        }
      if (hg == 0) {
        ml[2 * ((wave - half) * 32 + c)] = st.t;
        ml[2 * ((wave - half) * 32 + c) + 1] = l;
      }
    }
    __syncthreads();
    if (wave < half) {
      const float* o = ol + (wave * 32 + c) * OROW;
      const float t2 = ml[2 * (wave * 32 + c)], l2 = ml[2 * (wave * 32 + c) + 1];
      const float t_new = fmaxf(st.t, t2);
      const float f1 = __builtin_amdgcn_exp2f((st.t - t_new) * a.scale_log2);
      const float f2 = __builtin_amdgcn_exp2f((t2 - t_new) * a.scale_log2);
      st.t = t_new;
      l = fmaf(l, f1, l2 * f2);
#pragma unroll
      for (int t = 0; t < G::DT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int d = 32 * t + 8 * j + 4 * hg;
          if (d < DH) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(o + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) st.o[t][4 * j + e] = fmaf(st.o[t][4 * j + e], f1, x[e] * f2);
          }
        }
    }
  }
  if (wave == 0) store_row<DH>(a, row, st, l, hg, part, one_part(a, blocks.count));
}

// ---------------------------------------------------------------------------
// fp32: 16 QT rows; wave w takes blocks w, w + 4, ... of 16 keys, with the fp32
// 16x16x4 MFMAs: S^T (16 keys x 16 rows) = K Q^T, lane (c, g) = (lane % 16,
// lane / 16) feeding key (row) c at d = g DH/4 + step; O^T (16 d x 16 rows) +=
// V^T P^T, S^T leaving lane (c, g) with row c's keys 4 g + r.  Keys and values go
// from L2 to the registers that feed the products, so with many rows the L2
// bounds: 32 rows to a block of keys instead of 16 (500 rows in each of 4
// sequences of 3500 tokens, 16 heads of 64: 352 us, 76 TFLOP/s of 154).
// ---------------------------------------------------------------------------
template <int DH, int QT>
__global__ __launch_bounds__(64 * kWaves, 2) void attn_f32(const AttnArgs a) {
  constexpr int KB = 16;
  constexpr int DL = DH / 4;    // floats of a row per lane
  constexpr int DT = DH / 16;   // 16-row tiles of O^T
  constexpr int OROW = DH + 1;
  __shared__ float part_o[kWaves][16 * OROW];
  __shared__ float part_m[kWaves][16], part_l[kWaves][16];
  __shared__ uint64_t nodes[kTree ? kWaves : 1][kTree ? 16 * QT : 1][kTreeWords];
  int tile_no, hk, part;
  work_item(a, tile_no, hk, part);
  if (kTree && tile_no >= a.tiles) return;
  const Tile tile = find_tile(a, tile_no);
  if (tile.n <= 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const Blocks blocks = tile_blocks(a, tile, KB);
  int from, to;
  part_range(a, part, blocks.count, from, to);
  if (from >= to && from > 0) return;
  const Reach reach = rows_reach(a, tile, 0, tile.n);
  int key_hi[QT], key_lo[QT];
  f32x4_t q[QT][DL / 4], acc[QT][DT];
  float m_run[QT], l_run[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    Row row = make_row(a, tile, hk, 16 * qt + c);
    key_hi[qt] = row.hi;
    key_lo[qt] = row.lo;
    const float* qr = static_cast<const float*>(a.q) + row.q_at + g * DL;
#pragma unroll
    for (int i = 0; i < DL / 4; ++i) q[qt][i] = *reinterpret_cast<const f32x4_t*>(qr + 4 * i);
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[qt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m_run[qt] = kNone;
    l_run[qt] = 0.f;
  }
  // kTree: which of the 16 keys of a block from key0 on are nodes that it sees
  auto row_nodes = [&](int qt, int key0) -> uint32_t {
    if constexpr (kTree) {
      Row row;
      row.nodes = nodes[wave][16 * qt + c];
      row.first = tile.sp.first;
      return static_cast<uint32_t>(seen_nodes(row, key0)) & 0xFFFFu;
    }
    return 0;
  };
  PageWindow pages;
  f32x4_t k[DL / 4];
  float v[4][DT];  // V[key 4 g + r][16 t + c]
  bool alive_next = false;
  long at_next = 0;
  auto seek = [&](int i) {
    const int group = blocks.at(i);
    pages.seek(a.b, tile.s, group);
    alive_next = pages.keys<1>(group) != 0;
    at_next = key_offset(a.b, pages.page_of(group), hk, group * kGroup, DH);
  };
  auto load_keys = [&]() {
    const float* kr = static_cast<const float*>(a.b.k) + at_next + c * DH + g * DL;
#pragma unroll
    for (int i = 0; i < DL / 4; ++i) k[i] = *reinterpret_cast<const f32x4_t*>(kr + 4 * i);
  };
  auto load_values = [&]() {
    const float* vr = static_cast<const float*>(a.b.v) + at_next + 4 * g * DH + c;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < DT; ++t) v[r][t] = vr[r * DH + 16 * t];
  };
  Parents parents;
  if constexpr (kTree) parents = load_parents(a, tile);
  if (from + wave < to) {
    seek(from + wave);
    load_keys();
    load_values();
  }
  if constexpr (kTree)
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      Row row = make_row(a, tile, hk, 16 * qt + c);
      add_nodes(a, tile, parents, 16 * qt + c, nodes[wave][16 * qt + c], row);
      key_lo[qt] = row.lo;
    }
  for (int i = from + wave; i < to; i += kWaves) {
    const int key0 = blocks.at(i) * KB;
    const bool alive = alive_next, more = i + kWaves < to;
    const long at = at_next;
    f32x4_t sc[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      sc[qt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < DL / 4; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) sc[qt] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e][j], q[qt][e][j], sc[qt], 0, 0, 0);
    }
    if (more) {
      seek(i + kWaves);
      load_keys();
    }
    const bool whole = key0 + KB <= reach.hi_min && (key0 >= reach.lo_max || key0 + KB <= a.sinks) && alive;
    uint32_t odd[4] = {0, 0, 0, 0};  // [r] bit g: key 4 g + r holds a value that is not finite
    if (!whole) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        bool any = false;
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          const bool out = !(fabsf(v[r][t]) < kInf);
          any |= out;
          v[r][t] = out ? 0.f : v[r][t];
        }
        const uint64_t who = __builtin_amdgcn_ballot_w64(any);
#pragma unroll
        for (int g2 = 0; g2 < 4; ++g2) odd[r] |= (who >> (16 * g2) & 0xFFFF) ? 1u << g2 : 0u;
      }
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      float tmax = kNone;
      uint32_t tree = 0;
      if constexpr (kTree) tree = whole ? 0 : row_nodes(qt, key0) >> (4 * g);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = key0 + 4 * g + r;
        bool seen = whole || (alive && key < key_hi[qt] && (key >= key_lo[qt] || key < a.sinks));
        if constexpr (kTree) seen |= alive && (tree >> r & 1);
        sc[qt][r] = seen ? sc[qt][r] * a.scale_log2 : -kInf;
        tmax = fmaxf(tmax, sc[qt][r]);
      }
      tmax = fmaxf(tmax, __shfl_xor(tmax, 16, 64));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
      const float m_new = fmaxf(m_run[qt], tmax);
      const float alpha = exp2f(m_run[qt] - m_new);
      m_run[qt] = m_new;
      float psum = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sc[qt][r] = exp2f(sc[qt][r] - m_new);
        psum += sc[qt][r];
      }
      l_run[qt] = fmaf(l_run[qt], alpha, psum);
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[qt][t][r] *= alpha;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < DT; ++t)
          acc[qt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][t], sc[qt][r], acc[qt][t], 0, 0, 0);
    }
    if (!whole && alive) {
      // values that are not finite, for the rows that see their keys
#pragma unroll
      for (int r = 0; r < 4; ++r)
        for (uint32_t set = odd[r]; set; set &= set - 1) {
          const int in = 4 * __builtin_ctz(set) + r, key = key0 + in;
          const float* vr = static_cast<const float*>(a.b.v) + at + in * DH + 4 * g;
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) {
            bool seen = key < key_hi[qt] && (key >= key_lo[qt] || key < a.sinks);
            if constexpr (kTree) seen |= row_nodes(qt, key0) >> in & 1;
            if (!seen) continue;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float y = vr[16 * t + e];
                if (!(fabsf(y) < kInf)) acc[qt][t][e] += y;
              }
          }
        }
    }
    if (more) load_values();
  }
  // Join the waves, 16 rows at a time.
  for (int qt = 0; qt < QT; ++qt) {
    if (16 * qt >= tile.n) break;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < QT; ++u)
      if (u == qt) {
        const float l = l_run[u] + __shfl_xor(l_run[u], 16, 64);
        const float l4 = l + __shfl_xor(l, 32, 64);
        Row row;
        row.ok = 16 * u + c < tile.n;
        row.hi = key_hi[u];
        row.lo = key_lo[u];
        if constexpr (kTree) {
          row.nodes = nodes[wave][16 * u + c];
          row.first = tile.sp.first;
        }
        const float m = mark_seen<KB>(a, tile.s, blocks, from + wave, to, kWaves, row, l4, pages, m_run[u]);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) part_o[wave][c * OROW + 16 * t + 4 * g + r] = acc[u][t][r];
        if (g == 0) {
          part_m[wave][c] = m;
          part_l[wave][c] = l4;
        }
      }
    __syncthreads();
    const int i = threadIdx.x >> 4;
    if (16 * qt + i >= tile.n) continue;
    float m = part_m[0][i];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, part_m[w][i]);
    float f[kWaves], l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      f[w] = exp2f(part_m[w][i] - m);
      l = fmaf(part_l[w][i], f[w], l);
    }
    const Row mine = make_row(a, tile, hk, 16 * qt + i);
    const bool last = one_part(a, blocks.count);
    const float inv = last ? inverse_sum(l, m) : 1.f;
    const long slot = mine.part * a.parts + part;
    float* out = last ? static_cast<float*>(a.out) + mine.out_at : a.ws_o + slot * DH;
    if (!last && (threadIdx.x & 15) == 0) *reinterpret_cast<float2*>(a.ws_ml + 2 * slot) = make_float2(m, l);
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const int d = 16 * t + (threadIdx.x & 15);
      float o = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) o = fmaf(part_o[w][i * OROW + d], f[w], o);
      out[d] = o * inv;
    }
  }
}

// ---------------------------------------------------------------------------
// The parts of a tile's rows joined.  A workgroup takes 32 columns: 8 threads
// read a part's columns, and the 32 such octets divide `rows` rows at a time and
// their parts, each with a reference of its own (bf16: a score; fp32: its scaled
// maximum, log2 units), joined in LDS in order.  `shares`
// workgroups divide a tile's rows.  Bound by its launch and three dependent loads:
// 7 us for 16 rows of 128 parts, 8 us for 2048 rows of up to 15 (kTree, with the outputs
// read ahead of the references: 1024 rows of 64 parts, 34 MB, 12.2 us, 14.5 without).
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void attn_join(const AttnArgs a, int kb, int rows, int shares) {
  __shared__ f32x4_t so[256];
  __shared__ float sm[32], sl[32];
  const float unit = sizeof(T) == 2 ? a.scale_log2 : 1.f;
  const int dh = a.b.d_head, slices = (dh + 31) / 32;
  unsigned w = a.first + blockIdx.x;
  const int hk = w % a.b.n_heads;
  w /= a.b.n_heads;
  const int d = 32 * (w % slices) + 4 * (threadIdx.x & 7);
  w /= slices;
  const int share = w % shares;
  const Tile t = find_tile(a, w / shares);
  if (share * rows >= t.n) return;
  const int count = tile_blocks(a, t, kb).count;
  const int parts = tile_parts(a, count);
  if (kTree && parts == 1) return;
  const int octet = threadIdx.x >> 3, subs = 32 / rows;  // octets of a row
  const int sub = octet % subs;
  for (int row0 = share * rows; row0 < t.n; row0 += shares * rows) {
    const int i = row0 + octet / subs;
    const Row row = make_row(a, t, hk, i);
    const float* ml = a.ws_ml + 2 * row.part * a.parts;
    const float* o = a.ws_o + row.part * a.parts * dh + min(d, dh - 4);
    float m = kNone;
    float l = 0.f;
    f32x4_t x = {0.f, 0.f, 0.f, 0.f};
    int from = sub;
    if constexpr (kTree) {
      // the first parts' outputs are on their way before the reference is known
      constexpr int AHEAD = 4;  // all of them: the host gives a row as many octets as that takes
      f32x4_t y[AHEAD];
      float2 of[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int p = min(sub + k * subs, parts - 1);
        of[k] = *reinterpret_cast<const float2*>(ml + 2 * p);
        y[k] = *reinterpret_cast<const f32x4_t*>(o + static_cast<long>(p) * dh);
      }
      from = sub + AHEAD * subs;
      for (int p = from; p < parts; p += subs) m = fmaxf(m, ml[2 * p]);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) m = sub + k * subs < parts ? fmaxf(m, of[k].x) : m;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const float f = sub + k * subs < parts ? exp2f((of[k].x - m) * unit) : 0.f;
        l = fmaf(sub + k * subs < parts ? of[k].y : 0.f, f, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = sub + k * subs < parts ? fmaf(y[k][e], f, x[e]) : x[e];
      }
    } else {
      for (int p = sub; p < parts; p += subs) m = fmaxf(m, ml[2 * p]);
    }
#pragma unroll 8
    for (int p = from; p < parts; p += subs) {
      const f32x4_t y = *reinterpret_cast<const f32x4_t*>(o + static_cast<long>(p) * dh);
      const float f = exp2f((ml[2 * p] - m) * unit);
      l = fmaf(ml[2 * p + 1], f, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = fmaf(y[e], f, x[e]);
    }
    __syncthreads();  // the rows before are read
    so[threadIdx.x] = x;
    if ((threadIdx.x & 7) == 0) {
      sm[octet] = m;
      sl[octet] = l;
    }
    __syncthreads();
    if (sub != 0 || i >= t.n || d >= dh) continue;
    for (int k = 1; k < subs; ++k) m = fmaxf(m, sm[octet + k]);
    x = f32x4_t{0.f, 0.f, 0.f, 0.f};
    l = 0.f;
    for (int k = 0; k < subs; ++k) {
      const float f = exp2f((sm[octet + k] - m) * unit);
      l = fmaf(sl[octet + k], f, l);
      const f32x4_t y = so[threadIdx.x + 8 * k];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = fmaf(y[e], f, x[e]);
    }
    const float inv = inverse_sum(l, m);
    T* out = static_cast<T*>(a.out) + row.out_at + d;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<u32x2_t*>(out) = u32x2_t{pack2bf(x[0] * inv, x[1] * inv), pack2bf(x[2] * inv, x[3] * inv)};
    else
      *reinterpret_cast<f32x4_t*>(out) = f32x4_t{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

enum Kind { MANY, FEW, F32 };

struct Plan {
  Kind kind;
  int tile_rows, kb, tiles, parts, part_blocks;
};

Plan make_plan(int dtype, const PagedBatch& b, int m, int heads_q, int causal, int window, int sinks,
               size_t ws_bytes) {
  Plan p;
  const int group = heads_q / b.n_heads;
  const long packed = static_cast<long>(m) * group;
  // Tiles of 32 rows up to 48 rows a sequence, and up to 96 while there are no
  // more than 512 of them: they spread few rows over more CUs, but read the
  // keys four times as often as tiles of 128 (2000 keys, 16 heads of 64, 64 rows
  // in each of 16 sequences: 48 us, tiles of 128: 50; 128 rows: 74 and 55; 32
  // single tokens and 700 rows together, 4 heads: 40 and 47).
  const long few = (packed + 31) / 32 * b.n_heads;
  p.kind = dtype == DT_F32 ? F32
           : packed <= 48l * b.n_seqs || (packed <= 96l * b.n_seqs && few <= 512) ? FEW
                                                                                  : MANY;
  // Trees: tiles of 32 rows while what all of them read together, at max_kv keys
  // each, is at most 256 MB.  More of it costs more than the 128-row tiles' longer way
  // through a block (one tree of 128 nodes on 8000 keys, 16 heads of 64: 25 us, tiles
  // of 128: 40; 32 of 2 nodes on 500 to 8000, 32 heads of 128 on 4: 44 and 66; of 4: 69
  // and 66; one of 20 on 131000, 16 heads on 2: 112 and 91; 32 of 40 on 8000: 456 and
  // 285).  What a window leaves of the keys does not count here: on long contexts it
  // is read by tiles of 128, which few rows pay for (32 heads of 128 on 4, max_kv
  // 100000: one tree of 8 in a window of 1024 takes 25 us, at max_kv 1224, so with
  // tiles of 32, 15; 8 trees of 8 26 and 21, in a window of 4096 31 and 37).
  if (kTree && p.kind != F32) p.kind = few * b.max_kv * b.d_head <= 1l << 26 ? FEW : MANY;
  // fp32: 32 rows to a tile read the keys half as often, where that still makes
  // tiles enough (500 rows in each of 4 sequences, 3500 keys, 16 heads of 64: 365
  // us, tiles of 16: 440; 377 rows in 5 sequences, 12 heads: 25 and 17).
  const bool wide = packed > 16l * b.n_seqs && few >= 768;
  p.tile_rows = p.kind == MANY ? 128 : (p.kind == FEW || wide ? 32 : 16);
  p.kb = p.kind == MANY ? 64 : (p.kind == FEW ? 32 : 16);
  p.tiles = static_cast<int>(packed / p.tile_rows) + b.n_seqs;
  // keys that a tile reads at most
  long keys = b.max_kv;
  if (window > 0 && causal)
    keys = std::min(keys, static_cast<long>(window) + std::min(sinks, b.max_kv) +
                              (kTree ? std::min(m, kMaxTree) : p.tile_rows / group) + 3 * p.kb);
  const int blocks = static_cast<int>((keys + p.kb - 1) / p.kb);
  // tiles that there are in earnest, if the rows are spread evenly
  const long items = std::max<long>(b.n_seqs, (packed + p.tile_rows - 1) / p.tile_rows) * b.n_heads;
  // A workgroup for every CU, if each gets a few blocks; more of them, to even
  // out sequences of different lengths, as long as each has 1024 keys or more
  // and there are four or more of them to a tile: the join takes 6 us and more
  // (64 sequences of 500 to 16000 keys, 15 parts: 137 us, undivided 251; 32 single
  // tokens and 700 rows on 2100 keys, 2 parts: 33 us, undivided 28).
  // (fp32 single tokens: four for every CU; 16 sequences of 3000 tokens, 2 heads
  // of 128: 34 us, one for every CU: 44.)
  const long fill = p.kind == F32 && packed <= 16l * b.n_seqs ? 1024 : 256;
  long parts = std::min<long>((fill + items - 1) / items, blocks / (p.kind == MANY ? 4 : 8));
  const long even = std::min<long>((4096 + items - 1) / items, static_cast<long>(blocks) * p.kb / 1024);
  if (p.kind != MANY && even >= 4) parts = std::max(parts, even);
  // Trees, 128 rows to a tile: two workgroups for every CU, and parts of about 2560
  // keys of max_kv, where sequences may differ in length, while tiles times parts are
  // 4096 workgroups or fewer (32 trees of 16 to 59 nodes on 550 to 7850 keys, 32 heads
  // of 128 on 4: 101 us, undivided 218, with 1024 keys to a part 133; 4 trees of 64 on
  // 20000: 106, twice as many parts 122).
  if (kTree && p.kind == MANY)
    parts = std::min({std::max<long>(512 / items, (blocks + 39) / 40), static_cast<long>(blocks) / 8,
                      std::max(4096 / items, 1l)});
  // Trees, 32 rows to a tile: the join costs more than dividing a few blocks saves (6
  // trees of 20 nodes, 12 heads of 64: 600 keys 10 us, in two parts 14; 1500 keys 15, in
  // four 17.5; 16 of 6, 8 heads of 128 on 2, 1500 keys: 24, in four 20).
  if (kTree && p.kind == FEW && blocks <= (b.d_head <= 64 ? 48 : 24)) parts = 1;
  parts = std::max(parts, 1l);
  const size_t per_part = static_cast<size_t>(m) * heads_q * (b.d_head + 2) * sizeof(float);
  parts = std::max(1l, std::min<long>(parts, static_cast<long>(ws_bytes / per_part)));
  p.part_blocks = static_cast<int>((blocks + parts - 1) / parts);
  p.parts = (blocks + p.part_blocks - 1) / p.part_blocks;
  return p;
}

size_t plan_bytes(const PagedBatch& b, const Plan& p, int m, int heads_q) {
  return p.parts == 1 ? 0 : static_cast<size_t>(p.parts) * m * heads_q * (b.d_head + 2) * sizeof(float);
}

template <int DH>
void launch_tiles(Kind kind, const AttnArgs& a, dim3 grid, hipStream_t st) {
  if (kind == F32 && a.tile_rows == 16)
    hipLaunchKernelGGL((attn_f32<DH, 1>), grid, dim3(64 * kWaves), 0, st, a);
  else if (kind == F32)
    hipLaunchKernelGGL((attn_f32<DH, 2>), grid, dim3(64 * kWaves), 0, st, a);
  else if (kind == FEW)
    hipLaunchKernelGGL(attn_few<DH>, grid, dim3(64 * kWaves), 0, st, a);
  else
    hipLaunchKernelGGL((attn_many<DH, DH <= 96 ? 3 : 2>), grid, dim3(64 * kWaves), 0, st, a);
}

size_t attention_workspace(int dtype, const PagedBatch& b, int m, int heads_q, int window, int sinks) {
  if (m == 0 || b.n_seqs == 0) return 0;
  const size_t all = ~size_t{0};
  const size_t bytes = plan_bytes(b, make_plan(dtype, b, m, heads_q, 1, window, sinks, all), m, heads_q);
  if (kTree) return bytes;
  return std::max(plan_bytes(b, make_plan(dtype, b, m, heads_q, 0, window, sinks, all), m, heads_q), bytes);
}

hipError_t run_attention(int dtype, const PagedBatch& b, int m, int heads_q, const void* q, long ld_q,
                         const int32_t* parent, bool causal, int window, int sinks, void* ws, size_t ws_bytes,
                         void* out, long ld_out, hipStream_t st) {
  if (m == 0 || b.n_seqs == 0) return hipSuccess;
  window = std::min(window, kMaxTokens);
  sinks = std::min(sinks, kMaxTokens);
  const Plan p = make_plan(dtype, b, m, heads_q, causal, window, sinks, ws_bytes);
  AttnArgs a{};
  a.b = b;
  a.q = q;
  a.out = out;
  a.parent = parent;
  a.ld_q = ld_q;
  a.ld_out = ld_out;
  a.m = m;
  a.heads_q = heads_q;
  a.group = heads_q / b.n_heads;
  a.by_group = make_divisor(a.group);
  a.causal = causal;
  a.window = window;
  a.sinks = window ? sinks : 0;
  a.scale_log2 = kLog2e / sqrtf(static_cast<float>(b.d_head));
  a.tile_rows = p.tile_rows;
  a.tiles = p.tiles;
  a.parts = p.parts;
  a.part_blocks = p.part_blocks;
  if (p.parts > 1) {
    a.ws_o = static_cast<float*>(ws);
    a.ws_ml = a.ws_o + static_cast<size_t>(p.parts) * m * heads_q * b.d_head;
  }
  long grid = static_cast<long>(p.tiles) * p.parts * b.n_heads;
  if (kTree) {
    const long units = static_cast<long>((p.tiles + kTileRun - 1) / kTileRun) * p.parts * b.n_heads;
    grid = (units + kXcds - 1) / kXcds * kXcds * kTileRun;
  }
  for (long first = 0; first < grid; first += kMaxGrid) {
    a.first = static_cast<unsigned>(first);
    const dim3 part(static_cast<unsigned>(std::min(kMaxGrid, grid - first)));
    switch (b.d_head) {
      case 16: launch_tiles<16>(p.kind, a, part, st); break;
      case 32: launch_tiles<32>(p.kind, a, part, st); break;
      case 48: launch_tiles<48>(p.kind, a, part, st); break;
      case 64: launch_tiles<64>(p.kind, a, part, st); break;
      case 80: launch_tiles<80>(p.kind, a, part, st); break;
      case 96: launch_tiles<96>(p.kind, a, part, st); break;
      case 112: launch_tiles<112>(p.kind, a, part, st); break;
      case 128: launch_tiles<128>(p.kind, a, part, st); break;
      default: return hipErrorInvalidValue;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.parts == 1) return hipSuccess;
  // about four parts to an octet of threads; a tile's rows in turn if there are
  // enough tiles for every CU, or else a workgroup each
  int rows = 32;
  while (rows > 1 && rows * p.parts > 128) rows >>= 1;
  const long each = static_cast<long>(p.tiles) * ((b.d_head + 31) / 32) * b.n_heads;
  const int shares = each >= 512 ? 1 : std::max(1, p.tile_rows / rows);
  const long joins = each * shares;
  for (long first = 0; first < joins; first += kMaxGrid) {
    a.first = static_cast<unsigned>(first);
    const dim3 part(static_cast<unsigned>(std::min(kMaxGrid, joins - first)));
    if (dtype == DT_BF16)
      hipLaunchKernelGGL(attn_join<bf16_t>, part, dim3(256), 0, st, a, p.kb, rows, shares);
    else
      hipLaunchKernelGGL(attn_join<float>, part, dim3(256), 0, st, a, p.kb, rows, shares);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
