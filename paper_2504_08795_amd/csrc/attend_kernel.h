// Attention over the paged e4m3 cache with a running maximum and sum: one pass over the pages, scores and weights in registers only.
//
// Work. A tile is 16 (narrow) or 128 (wide: 32 a wave) columns; a column is one query head of one row, and all columns of a tile
// read the same key head, so that every page is fetched once for the whole group.  The tiles of all sequences times their visible
// pages are cut into units of equal numbers of pages -- the kernel reads the lengths itself, so the cut fits them whatever the table's
// width and however unequal they are -- and a workgroup takes one.  Units of one tile leave their unnormalised sums in the
// workspace; the workgroup that arrives last adds them in unit order, so the result does not depend on the order of arrival.
//
// Operands. Scores are S^T = K Q^T and outputs O^T = V^T P^T: a lane then holds sixteen scores of ONE column, namely of sixteen
// neighbouring tokens (the rows of the K tile are permuted so), which are the weights it has to supply to the second product: no
// exchange between lanes but for the maximum.  Sixteen tokens share a scale, so a lane needs one scale of K and one of V a page.
// Keys [token][channel] and values [channel][token] are loaded in the operands' own order, 16 bytes a lane, and spread from
// e4m3 to f16 two at a time (exact).  Queries are divided by a power of two that brings their largest number to 2^14, in one f16 part
// (bf16) or two (fp32).  The scale of V joins the exponent: w = 2^(s + log2(scale_v) - M + 10), M a running maximum
// of s + log2(scale_v) (at most 5 behind): w fits f16 whatever the scales are (its smallest step is 2^-34 of the largest w, what is less is lost), and
// the sum of weights takes 1 / scale_v back out.  What is nothing beside the largest s + log2(scale_v) may have the largest s (zeros beside large values), so
// the sum is scaled in steps that leave fp32's range no more than it does itself.
//
// Masks cost nothing on pages that all columns see, where these have a form of their own (kBoth).  On the others scores are selected away, and values that no column sees, as well as
// NaN codes, whose product with a zero weight would spoil other columns, are cleared; mark_nans finds the columns that see them.
//
// Narrow tiles are bound by the bytes of the cache: 64 streams, 8 key heads of 128, 368 MB in 81 to 83 us, 4.5 TB/s (a pure read reaches 6.2, a copy 5.1); one
// stream of 8001 tokens, 16 MB, takes 11.0 us, which is the chain lengths -> pages -> keys -> values -> the units' numbers -> the merge.
// Wide ones are bound by instruction issue: 2048 rows behind 4100 tokens (32 heads of 128), 172 GFLOP in 206 to 214 us a call, 800 to 835 TFLOP/s (a large
// matrix product: 1190); 1900 rows 199 us, 2049 279.  The matrix instructions take 41 % of a SIMD's cycles and the vector ones (a wave's page: 32 exponentials at a
// quarter of the rate and some 260 others) the rest; what one wave computes does not hide behind another's matrix instructions.
//
// Trees: every column sees the cached tokens (under a window the last of them and of its nodes) and the nodes of its mask, so only the pages that hold nodes
// (and, under a window, its first ones) are masked, by sixteen bits of the mask for a lane's sixteen scores.  32 trees of up to 64 nodes behind up to 4096 tokens (32 query and 8 key heads of
// 128, bf16), 37 GFLOP: 111 us a call, as long as the same rows following each other; wide tiles are two thirds full there, and cut ones leave 24 MB of sums.
#pragma once
#include "step_common.h"

namespace daris {

constexpr float kWeightBits = 10.f, kMaxLag = 5.f;  // a weight is at most 2^15
constexpr float kLeastWeight = 100.f;               // 2^-100: 26 bits above the smallest number, far below f16's

// What a workgroup has to do.
struct Unit {
  int s = 0, tile = 0, chunk = 0, chunks = 0, per = 0;  // per: pages of a unit
  int first = 0;                                        // number of the tile's first unit
  int row0 = 0, rows = 0, before = 0;
};

// Pages that any row of sequence s sees: [*lo, return value).  (A row of a tree may see one cached token more than its window: none of its nodes.)
template <bool TREE>
__device__ __forceinline__ int seen_pages(const AttendArgs& a, int rows, int before, int* lo) {
  const int end = before + rows;
  int from = a.window > 0 && before >= a.window ? before - a.window + (TREE ? 0 : 1) : 0;
  from /= kPage;
  *lo = from;
  if (end <= 0 || rows == 0) return from;
  int to = (end + kPage - 1) / kPage;
  if (to > a.c.pages_row) to = (int)a.c.pages_row;
  return to < from ? from : to;
}

// Every wave finds the workgroup's unit by itself, 64 * SETS sequences at a time (a token for 200 streams of 500, 8 query and 4 key heads of 128: 37 us a call, 44 when
// sets of 64 came one after the other).  False: nothing to do.
template <int TILE, int MOST, int SETS, bool TREE>
__device__ __forceinline__ bool find_among(const AttendArgs& a, int unit, Unit* u) {
  const int lane = threadIdx.x & 63, ns = a.c.n_seqs;
  int row0[SETS], rows[SETS], before[SETS], tiles[SETS], pages[SETS];
  auto look = [&](int s0) {  // (no branch around the fetches, so that those of all sets travel together)
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
      const int s = s0 + i * 64 + lane, in = s < ns ? s : ns - 1;
      row0[i] = first_row(a.c, in);
      rows[i] = s < ns ? rows_of(a.c, in) : 0;
      before[i] = tokens_before(a.c, in);
    }
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
      tiles[i] = (int)(((int64_t)rows[i] * a.group + TILE - 1) / TILE);
      int lo;
      pages[i] = seen_pages<TREE>(a, rows[i], before[i], &lo);
      pages[i] -= lo;
    }
  };
  float work = 0.f, most = 0.f;
  for (int s0 = 0; s0 < ns; s0 += 64 * SETS) {
    look(s0);
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
      work += (float)tiles[i] * (float)pages[i];
      most = fmaxf(most, (float)pages[i]);
    }
  }
  work = wave_sum<64>(work);
  most = wave_max<64>(most);
  // pages of a unit: what makes `target` of them, a little more so that rounding never makes too many; the merge holds MOST of a tile
  float per = a.target > 0 ? ceilf(work * 1.0001f / (float)a.target) : most;
  per = fmaxf(per, ceilf(most * (1.f / MOST)));
  int c = (int)fminf(per, 1.0e9f);
  c = c < 1 ? 1 : c;
  c = (c + 3) / 4 * 4;
  auto cut = [&](int i) { return tiles[i] == 0 ? 0 : pages[i] <= c ? 1 : (pages[i] + c - 1) / c; };
  // Tiles of little more pages than that would become twice as many units, which go in two rounds: they stay whole if all fit one.  (While the wave still holds
  // all lengths.  8 x 24 rows behind 2000 tokens, 384 tiles of 33 pages for 512 places: 49 us so, 37 in whole.)
  if (ns <= 64 * SETS && a.target > 0 && most > (float)c && most <= 2.f * (float)c) {
    float whole = 0.f, units = 0.f;
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
      whole += (float)tiles[i];
      units += (float)tiles[i] * (float)cut(i);
    }
    if (wave_sum<64>(units) > (float)a.target && wave_sum<64>(whole) <= (float)a.target) c = ((int)most + 3) / 4 * 4;
  }
  // Trees of a few tiles each, all as long as their sequence: to cut them pays where the longest takes clearly longer than a CU's even share, by what the sums of a cut tile
  // cost.  (us a call whole and cut, 32 query and 8 key heads of 128, bf16: 24 trees of up to 24 nodes behind up to 3000 tokens 43 and 57, 12 of 40 38 and 53, 8 of 64 behind 2000
  // 35 and 43, 8 of 32 behind 8000 65 and 55; wide 32 of 64 behind 4096 120 and 111, 6 of 256 behind 4000 130 and 92.  Fewer than six trees were not measured both ways.)
  if (TREE && a.target > 0 && most > (float)c && most <= work / (float)a.round + (TILE == kWideColumns ? 10.f : 30.f)) c = ((int)most + 3) / 4 * 4;
  int base = 0;
  for (int s0 = 0; s0 < ns; s0 += 64 * SETS) {
    if (ns > 64 * SETS) look(s0);
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
      const int chunks = cut(i), mine = tiles[i] * chunks;
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int o = __builtin_amdgcn_ds_bpermute((lane - d) * 4, upto);
        if (lane >= d) upto += o;
      }
      const int start = base + upto - mine;
      const uint64_t hit = __ballot(unit >= start && unit < start + mine);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        u->s = s0 + i * 64 + l;
        u->chunks = __builtin_amdgcn_readlane(chunks, l);
        const int in = unit - __builtin_amdgcn_readlane(start, l);
        u->tile = in / u->chunks;
        u->chunk = in - u->tile * u->chunks;
        u->first = unit - u->chunk;
        if (TILE == kWideColumns && u->chunks == 1) {
          // Later tiles see more pages, and the longest come first.  Of one sequence whose tiles go in two rounds of workgroups the second comes the other way round, so
          // that a CU gets a long and a short one.  (4 query heads to each of 8 key heads of 128, bf16, us a call in this order and in that of the rows: 1500 rows
          // behind 4100 tokens 175 and 193, 1900 199 and 217, 2047 208 and 226, 2 x 2048 rows 108 and 138, 1000 to 4000 rows 319 and 352.)
          const int all = __builtin_amdgcn_readlane(tiles[i], l);
          u->tile = ns > 1 || u->tile < a.round || all > 2 * a.round ? all - 1 - u->tile : u->tile - a.round;
        }
        u->per = c;
        u->row0 = __builtin_amdgcn_readlane(row0[i], l);
        u->rows = __builtin_amdgcn_readlane(rows[i], l);
        u->before = __builtin_amdgcn_readlane(before[i], l);
        // A row_start that decreases counts rows twice, and the last units are none that was launched: a tile that has such units is left out as a whole, lest
        // those that were launched wait at its counter for good.
        return u->chunks == 1 || u->first + u->chunks <= a.units;
      }
      base += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  return false;
}
template <int TILE, int MOST, bool TREE>
__device__ __forceinline__ bool find_unit(const AttendArgs& a, int unit, Unit* u) {
  return a.c.n_seqs <= 64 ? find_among<TILE, MOST, 1, TREE>(a, unit, u) : find_among<TILE, MOST, 4, TREE>(a, unit, u);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bool has_nan_code(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; }
// 0xff in the bytes that hold the NaN code
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t top = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return (top >> 7) * 0xffu;
}

// The lowest n bytes of a word.
__device__ __forceinline__ uint32_t bytes_below(int n) { return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u; }

// The lowest n halves of a word.
__device__ __forceinline__ uint32_t halves_below(int n) { return n >= 2 ? 0xffffffffu : n <= 0 ? 0u : 0xffffu; }
// A channel's codes of tokens t1 .. t1 + 15, those outside [lo, hi] cleared.
__device__ __forceinline__ uint4 seen(uint4 x, int t1, int lo, int hi) {
  const int a = lo - t1, b = hi + 1 - t1;
  return make_uint4(x.x & bytes_below(b) & ~bytes_below(a), x.y & bytes_below(b - 4) & ~bytes_below(a - 4), x.z & bytes_below(b - 8) & ~bytes_below(a - 8),
                    x.w & bytes_below(b - 12) & ~bytes_below(a - 12));
}

// The lowest n of sixteen bits.
__device__ __forceinline__ uint32_t bits_below(int n) { return n >= 16 ? 0xffffu : n <= 0 ? 0u : (1u << n) - 1u; }

// What the row of a column sees where the step's rows are nodes of a tree: cached tokens from `from` on, and the nodes of its mask from `least` on.
struct Sight {
  const uint64_t* mask;
  int before, nodes, words, from, least;
  // row: its number among all rows.  A window leaves the last tokens of those that it sees.
  __device__ __forceinline__ void start(const AttendArgs& a, const TreeMasks& tree, const Unit& u, int row) {
    mask = tree.mask + (int64_t)row * tree.words;
    before = u.before;
    words = tree.words;
    nodes = u.rows < 64 * words ? u.rows : 64 * words;
    from = least = 0;
    if (a.window <= 0) return;
    auto word = [&](int w) {
      const int left = nodes - 64 * w;
      return mask[w] & (left >= 64 ? ~0ull : left <= 0 ? 0ull : (1ull << left) - 1);
    };
    int over = -a.window;
    for (int w = 0; w < words; ++w) over += __popcll(word(w));
    from = before + over;
    for (int w = 0; w < words && over > 0; ++w) {
      uint64_t m = word(w);
      if (const int n = __popcll(m); over >= n) {
        over -= n;
        least = 64 * w + 64;
      } else {
        for (; over > 0; --over) m &= m - 1;
        least = 64 * w + __builtin_ctzll(m);
      }
    }
  }
  // ... of tokens t1 .. t1 + 15, a bit each
  __device__ __forceinline__ uint32_t bits(int t1) const {
    uint32_t seen = bits_below(before - t1) & ~bits_below(from - t1);
    const int node = t1 - before;  // the token t1 is this node
    if (node > -16 && node < nodes) {
      const int w = node < 0 ? 0 : node >> 6, shift = node & 63;
      uint64_t m = mask[w];
      if (node < 0) {
        m <<= -node;
      } else {
        m >>= shift;
        if (shift > 48 && w + 1 < words) m |= mask[w + 1] << (64 - shift);
      }
      seen |= (uint32_t)m & bits_below(nodes - node) & ~bits_below(least - node);
    }
    return seen;
  }
};

// One wave's columns, TILE = 16 or 32 of them, and its running sums.  TREE: the step's rows are nodes of trees.
template <bool BF16, int D, int TILE, bool TREE = false>
struct Columns {
  static constexpr int PARTS = BF16 ? 1 : 2;
  // Pages that all columns see have a form of their own where its registers leave two waves on a SIMD (64 streams, bf16, heads of 128: 83.0 us a call, 85.7
  // with the masked form for all; 8 x 32 rows behind 2000 tokens, heads of 64, 22.7 and 26.8; fp32 of 128 would have one wave, and 256 would spill).
  static constexpr bool kBoth = TILE == 32 || (BF16 && D < 256);
  // A page's keys are fetched while the values of the one before are used (200 streams of 500, bf16, heads of 128: 37.1 us a call in place of 38.2, 8 x 24
  // rows behind 2000 36.8 and 37.5, though 64 streams of 8192 83.0 and 82.3; fp32 heads of 128 and heads of 256, whose registers leave little room, were 3 % slower with it).
  static constexpr bool kKeysAhead = kBoth || D == 64;
  static constexpr int G = 64 / TILE;            // lanes of a column
  static constexpr int DEPTH = TILE == 16 ? 32 : 16;  // channels (tokens) of a matrix instruction
  static constexpr int KT = kPage / TILE;        // score tiles of a page
  static constexpr int KS = D / DEPTH;           // matrix instructions of a score tile
  static constexpr int VT = D / TILE;            // output tiles
  static constexpr int R = TILE * TILE / 64;     // numbers of a tile in a lane
  static constexpr int KV = D / G / 16;          // 16-byte pieces of a key in a lane
  static constexpr int HALVES = kPage / (16 * G);  // sixteenths of a page in a lane
  using Acc = typename std::conditional<TILE == 16, f32x4, f32x16>::type;
  static __device__ __forceinline__ Acc mma(const f16x8& x, const f16x8& y, const Acc& z) {
    if constexpr (TILE == 16) return mfma16(x, y, z);
    else return mfma32(x, y, z);
  }

  f16x8 q[PARTS][KS];
  Acc o[VT];
  float top, sum;   // M; the lane's share of the sum of weights
  float factor;     // of a score: scale * log2(e) / the queries' power of two
  int pos;          // position of the column's row
  Sight sight;      // (TREE: in its place)
  bool nans;        // there were NaN codes among the values of a masked page
  int lane;
  __device__ __forceinline__ int c() const { return lane & (TILE - 1); }  // column of the lane, and which of the column's lanes it is
  __device__ __forceinline__ int g() const { return lane / TILE; }

  // columns col0 .. of `rows` rows; those behind the last repeat it and are not stored
  __device__ __forceinline__ void start(const AttendArgs& a, const TreeMasks& tree, const Unit& u, int head, int col0) {
    lane = threadIdx.x & 63;
    const int c = this->c(), g = this->g();
    const int cols = u.rows * a.group;
    const int col = col0 + c < cols ? col0 + c : cols - 1;
    const int r = col / a.group;
    if constexpr (TREE) sight.start(a, tree, u, u.row0 + r);
    else pos = u.before + r;
    const int64_t at = (int64_t)(u.row0 + r) * a.q_row + (int64_t)(head * a.group + (col - r * a.group)) * a.q_head + g * (D / G);
    constexpr int W = BF16 ? 1 : 2;  // 16-byte vectors of eight channels
    uint4 raw[KS][W];
#pragma unroll
    for (int j = 0; j < KS; ++j)
#pragma unroll
      for (int i = 0; i < W; ++i) {
        if (a.q_vec) {
          raw[j][i] = *(const uint4*)((const char*)a.q + (at + 8 * j) * (BF16 ? 2 : 4) + 16 * i);
        } else if (BF16) {
          const uint16_t* x = (const uint16_t*)a.q + at + 8 * j;
          raw[j][i] = make_uint4(x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16, x[4] | (uint32_t)x[5] << 16, x[6] | (uint32_t)x[7] << 16);
        } else {
          const uint32_t* x = (const uint32_t*)a.q + at + 8 * j + 4 * i;
          raw[j][i] = make_uint4(x[0], x[1], x[2], x[3]);
        }
      }
    auto channels = [&](int j, float (&x)[8]) {
      if constexpr (BF16) {
        unpack<true>(raw[j][0], x);
      } else {
        float lo[4], hi[4];
        unpack<false>(raw[j][0], lo);
        unpack<false>(raw[j][W - 1], hi);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = lo[e];
          x[e + 4] = hi[e];
        }
      }
    };
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      float x[8];
      channels(j, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, size_of(x[e]));
    }
    most = lanes_max<TILE, 64>(most);
    int up = 141 - (int)(__float_as_uint(most) >> 23);
    up = up > 110 ? 110 : up;
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      __builtin_amdgcn_sched_barrier(0);
      float x[8];
      channels(j, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = __builtin_amdgcn_ldexpf(a.scale < 0.f ? -x[e] : x[e], up);
        q[0][j][e] = (_Float16)v;
        if (PARTS == 2) q[PARTS - 1][j][e] = is_finite(v) ? (_Float16)(v - (float)q[0][j][e]) : (_Float16)0.f;
      }
    }
    factor = fabsf(a.scale) * two_to(-up);
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int i = 0; i < R; ++i) o[t][i] = 0.f;
    top = -INFINITY;
    sum = 0.f;
    nans = false;
  }

  // token of a page that row r of score tile t is: a lane's numbers of the tiles are then neighbouring tokens
  static __device__ __forceinline__ int token_of(int t, int r) {
    if (TILE == 16) return (r >> 2) * 16 + t * 4 + (r & 3);
    return t * 32 + ((r >> 2) & 1) * 16 + (r >> 3) * 4 + (r & 3);
  }
  // first of the 16 tokens whose scores tile group `half` leaves in this lane, and the sixteenth they are
  __device__ __forceinline__ int sixteenth(int half) const { return TILE == 16 ? g() : half * 2 + g(); }

  // A page in registers, as its operands are: 16 bytes of a key's channels, of a channel's tokens.
  struct Page {
    static constexpr bool kShared = false;
    uint4 kr[KT][KV];
    uint4 vr[VT][HALVES];
    uint32_t ks, vs;  // four scale bytes each
    __device__ __forceinline__ f16x8 key(int t, int j) const {
      const uint4& w = kr[t][j >> 1];
      return j & 1 ? f16_of_codes(w.z, w.w) : f16_of_codes(w.x, w.y);
    }
    // The sixteen values of a channel; MASKED: those of tokens outside [lo, hi] and NaN codes as 0, *found: there were such codes.
    template <bool MASKED>
    __device__ __forceinline__ void values(int t, int h, int t1, int lo, int hi, uint32_t* found, f16x8 (&x)[2]) const {
      uint4 w = vr[t][h];
      if (MASKED) {
        w = seen(w, t1, lo, hi);
        const uint4 n = make_uint4(nan_bytes(w.x), nan_bytes(w.y), nan_bytes(w.z), nan_bytes(w.w));
        *found |= n.x | n.y | n.z | n.w;
        w = make_uint4(w.x & ~n.x, w.y & ~n.y, w.z & ~n.z, w.w & ~n.w);
      }
      x[0] = f16_of_codes(w.x, w.y);
      x[1] = f16_of_codes(w.z, w.w);
    }
  };
  __device__ __forceinline__ void fetch_keys(const AttendArgs& a, int head, int page, Page* p) const {
    const int64_t ph = (int64_t)page * a.c.kv_heads + head;
    p->ks = *(const uint32_t*)(a.c.k_scale + ph * 4);
    const uint8_t* k = a.c.k + ph * (kPage * D) + g() * (D / G);
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int i = 0; i < KV; ++i) p->kr[t][i] = *(const uint4*)(k + token_of(t, c()) * D + i * 16);
  }
  __device__ __forceinline__ void fetch_values(const AttendArgs& a, int head, int page, Page* p) const {
    const int64_t ph = (int64_t)page * a.c.kv_heads + head;
    p->vs = *(const uint32_t*)(a.c.v_scale + ph * 4);
    const uint8_t* v = a.c.v + ph * (kPage * D) + c() * kPage;
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int h = 0; h < HALVES; ++h) p->vr[t][h] = *(const uint4*)(v + t * TILE * kPage + sixteenth(h) * 16);
  }

  // The page that starts at token t0.  MASKED: some column does not see all of it; [see_lo, see_hi]: tokens that any column sees; over: what is done
  // once its keys are no longer needed.
  template <bool MASKED, typename P, typename F>
  __device__ __forceinline__ void take_page(const AttendArgs& a, const P& p, int t0, int see_lo, int see_hi, const F& over) {
    const uint32_t ks = p.ks, vs = p.vs;
    // tokens of its sixteenths that the column sees
    struct {
      int from[HALVES], to[HALVES];
      uint32_t bits[HALVES];
    } sees;
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      const int t1 = t0 + sixteenth(h) * 16;
      if constexpr (TREE) {
        sees.bits[h] = MASKED ? sight.bits(t1) : 0u;
      } else {
        sees.to[h] = pos + 1 - t1;
        sees.from[h] = a.window > 0 ? sees.to[h] - a.window : -(1 << 30);
      }
    }
    uint32_t found = 0;
    Acc s[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int i = 0; i < R; ++i) s[t][i] = 0.f;
    if constexpr (P::kShared) {
      // one pair of operands ahead of the instructions, in this order: left to itself the compiler reads all of them first, for which
      // there are no registers, or each when it is needed
      f16x8 k[KT], next[KT];
#pragma unroll
      for (int t = 0; t < KT; ++t) k[t] = p.key(t, 0);
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        if (j + 1 < KS) {
#pragma unroll
          for (int t = 0; t < KT; ++t) next[t] = p.key(t, j + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          if (PARTS == 2) s[t] = mma(k[t], q[PARTS - 1][j], s[t]);
          s[t] = mma(k[t], q[0][j], s[t]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < KT; ++t) k[t] = next[t];
      }
    } else {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          const f16x8 k = p.key(t, j);
          if (PARTS == 2) s[t] = mma(k, q[PARTS - 1][j], s[t]);
          s[t] = mma(k, q[0][j], s[t]);
        }
    }
    over();
    // A score is s * f + v in powers of two, v the values' scale; f > 0 and v are a sixteenth's, so its largest score is that of its largest s.
    constexpr int PER = 16 / R;  // score tiles of a sixteenth (16-column tiles: four; 32: one)
    float f[HALVES], v[HALVES], biggest[HALVES];
    float big = -INFINITY;
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      const int part = sixteenth(h);
      f[h] = fmaxf(factor * two_to((int)((ks >> (8 * part)) & 0xff) - 127), 1.0e-37f);  // (0 would make -inf a NaN)
      v[h] = (float)((int)((vs >> (8 * part)) & 0xff) - 127);
      float m = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x = s[h * PER + e / R][e % R];
        if (MASKED) {
          x = (TREE ? (sees.bits[h] >> e & 1) != 0 : e >= sees.from[h] && e < sees.to[h]) ? x : -INFINITY;
          s[h * PER + e / R][e % R] = x;
        }
        m = fmaxf(m, x);
      }
      biggest[h] = fmaf(m, f[h], v[h]);
      big = fmaxf(big, biggest[h]);
    }
    big = lanes_max<TILE, 64>(big);
    // M follows only when it has been passed by kMaxLag: up to there the weights have room, and most pages then leave the outputs alone
    const float now = big > top + kMaxLag ? big : top;
    if (__any(now != top)) {
      asm volatile("");  // (a branch: left to itself the compiler multiplies always)
      const float half = now == top ? 1.f : exp2_fast(0.5f * (top - now)), shrink = half * half;
#pragma unroll
      for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int i = 0; i < R; ++i) o[t][i] *= shrink;
      sum = sum * half * half;
      top = now;
    }
    const float base = (top == -INFINITY ? 0.f : top) - kWeightBits;
    // Weights below 2^-kLeastWeight are nothing among the outputs, but may be all of the sum, if their values are far smaller than others: they are
    // then taken times a power of two, which the sum takes out again with their scale.
    float least = INFINITY, from[HALVES];
    int back[HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      least = fminf(least, biggest[h]);
      from[h] = v[h] - base;
      back[h] = 127 - (int)((vs >> (8 * sixteenth(h))) & 0xff);
    }
    if (__any(least < base - kLeastWeight)) {
      asm volatile("");  // (a branch, as above)
#pragma unroll
      for (int h = 0; h < HALVES; ++h) {
        const int up = (int)fminf(fmaxf(base - kLeastWeight - biggest[h], 0.f), 300.f);
        from[h] += (float)up;
        back[h] -= up;
      }
    }
    f16x8 w[PARTS][2 * HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      float add = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = exp2_fast(fmaf(s[h * PER + e / R][e % R], f[h], from[h]));
        add += x;
        const _Float16 hi = (_Float16)x;
        w[0][h * 2 + (e >> 3)][e & 7] = hi;
        if (PARTS == 2) w[PARTS - 1][h * 2 + (e >> 3)][e & 7] = (_Float16)(x - (float)hi);
      }
      sum += __builtin_amdgcn_ldexpf(add, back[h]);
    }
    f16x8 x[2], next[2];  // (as above, sixteen values ahead)
    auto values = [&](int n, f16x8 (&to)[2]) { p.template values<MASKED>(n / HALVES, n % HALVES, t0 + sixteenth(n % HALVES) * 16, see_lo, see_hi, &found, to); };
    constexpr bool AHEAD = P::kShared && !MASKED;
    if (P::kShared) __builtin_amdgcn_sched_barrier(0);
    if (AHEAD) values(0, x);
#pragma unroll
    for (int n = 0; n < VT * HALVES; ++n) {
      const int t = n / HALVES, h = n % HALVES;
      if (!AHEAD) values(n, x);
      else if (n + 1 < VT * HALVES) values(n + 1, next);
      if (P::kShared) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (PARTS == 2) o[t] = mma(x[i], w[PARTS - 1][h * 2 + i], o[t]);
        o[t] = mma(x[i], w[0][h * 2 + i], o[t]);
      }
      if (P::kShared) __builtin_amdgcn_sched_barrier(0);
      if (AHEAD) {
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = next[i];
      }
    }
    if (MASKED && __any(found != 0)) nans = true;
  }

  // NaN codes among the values of a masked page count as 0 above, lest they spoil columns that do not see them.  If there were any, the columns that do
  // see them are found here, once the pages are through: the codes as numbers 1.0 (0x38) times 1 where the column sees the token are more than 0.
  __device__ __forceinline__ void mark_nans(const AttendArgs& a, const Unit& u, int head, int lo, int hi, int stride, int pos_lo, int pos_hi) {
    if (!nans) return;
    const int see_lo = a.window > 0 ? pos_lo - a.window + 1 : 0;
#pragma unroll 1
    for (int p = lo; p < hi; p += stride) {
      const int t0 = p * kPage, page = uniform(page_of(a.c, u.s, p));
      if (page < 0 || (kBoth && !is_masked(a, t0, pos_lo, pos_hi))) continue;
      const uint8_t* v = a.c.v + ((int64_t)page * a.c.kv_heads + head) * (kPage * D) + c() * kPage;
#pragma unroll
      for (int h = 0; h < HALVES; ++h) {
        const int t1 = t0 + sixteenth(h) * 16;
        f16x8 see[2];
        if constexpr (TREE) {
          const uint32_t bits = sight.bits(t1);
#pragma unroll
          for (int e = 0; e < 16; ++e) see[e >> 3][e & 7] = bits >> e & 1 ? (_Float16)1.f : (_Float16)0.f;
        } else {
          const int to = pos + 1 - t1, from = a.window > 0 ? to - a.window : -(1 << 30);
#pragma unroll
          for (int e = 0; e < 16; ++e) see[e >> 3][e & 7] = e >= from && e < to ? (_Float16)1.f : (_Float16)0.f;
        }
#pragma unroll
        for (int t = 0; t < VT; ++t) {
          __builtin_amdgcn_sched_barrier(0);
          const uint4 x = seen(*(const uint4*)(v + t * TILE * kPage + sixteenth(h) * 16), t1, see_lo, pos_hi);
          Acc count;
#pragma unroll
          for (int i = 0; i < R; ++i) count[i] = 0.f;
          count = mma(f16_of_codes(nan_bytes(x.x) & 0x38383838u, nan_bytes(x.y) & 0x38383838u), see[0], count);
          count = mma(f16_of_codes(nan_bytes(x.z) & 0x38383838u, nan_bytes(x.w) & 0x38383838u), see[1], count);
#pragma unroll
          for (int i = 0; i < R; ++i) o[t][i] = count[i] > 0.f ? __uint_as_float(0x7fc00000u) : o[t][i];
        }
      }
    }
  }

  // Whether some column does not see all of the page that starts at token t0.
  static __device__ __forceinline__ bool is_masked(const AttendArgs& a, int t0, int pos_lo, int pos_hi) { return t0 + kPage - 1 > pos_lo || (a.window > 0 && t0 <= pos_hi - a.window); }

  // The lanes of a column add their shares.
  __device__ __forceinline__ void finish() { sum = lanes_sum<TILE, 64>(sum); }

  // Pages [lo, hi) of the sequence, every `stride`-th; the page numbers of 64 of them are read at a time.
  __device__ __forceinline__ void run(const AttendArgs& a, const Unit& u, int head, int lo, int hi, int stride, int pos_lo, int pos_hi) {
    const int see_lo = a.window > 0 ? pos_lo - a.window + 1 : 0, see_hi = pos_hi;
    for (int base = lo; base < hi; base += 64 * stride) {
      const int at = base + lane * stride;
      const int mine = at < hi ? page_of(a.c, u.s, at) : -1;
      uint64_t left = __ballot(mine >= 0);
      if (left == 0) continue;
      int i = __builtin_ctzll(left);
      Page p;
      fetch_keys(a, head, __builtin_amdgcn_readlane(mine, i), &p);
      fetch_values(a, head, __builtin_amdgcn_readlane(mine, i), &p);
      for (;;) {
        // the next page's keys travel while this one's values are used, and its values while its keys are
        left &= left - 1;
        const int next = left ? __builtin_ctzll(left) : i, page = __builtin_amdgcn_readlane(mine, next);
        const int t0 = (base + i * stride) * kPage;
        auto over = [&] {
          if (kKeysAhead && left) fetch_keys(a, head, page, &p);
        };
        if (!kBoth || is_masked(a, t0, pos_lo, pos_hi)) take_page<true>(a, p, t0, see_lo, see_hi, over);
        else take_page<false>(a, p, t0, see_lo, see_hi, over);
        if (!left) break;
        if (!kKeysAhead) fetch_keys(a, head, page, &p);
        fetch_values(a, head, page, &p);
        i = next;
      }
    }
    mark_nans(a, u, head, lo, hi, stride, pos_lo, pos_hi);
    finish();
  }
  // first channel of the four (of neighbouring numbers r .. r + 3) that o[t][r] begins
  __device__ __forceinline__ int channel(int t, int r) const { return TILE == 16 ? t * 16 + g() * 4 : t * 32 + (r >> 2) * 8 + g() * 4; }
};

template <bool BF16>
__device__ __forceinline__ void put_out(const AttendArgs& a, int64_t at, const float4& v) {
  if (a.out_vec) {
    if (BF16) *(uint2*)((uint16_t*)a.out + at) = make_uint2(pack_bf16_rne(v.x, v.y), pack_bf16_rne(v.z, v.w));
    else *(float4*)((float*)a.out + at) = v;
  } else {
    const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (BF16) ((uint16_t*)a.out)[at + i] = (uint16_t)f32_to_bf16_bits(x[i]);
      else ((float*)a.out)[at + i] = x[i];
    }
  }
}

// Sums of a tile that several units share, in the workspace: [unit][COLS][D] numbers, then [unit][COLS] pairs (M, sum).
template <int COLS, int D>
__device__ __forceinline__ float* part_numbers(const AttendArgs& a, int head, int unit) {
  return a.part + (int64_t)(head * a.units + unit) * (COLS * (D + 2));
}

// N places of Q units at once: a fetch takes a microsecond, so as many as registers hold travel together (four at a time, 128 rows of 128 channels
// in nine units took 50 us to merge).
template <int COLS, int D, bool BF16, int N, int Q>
__device__ __forceinline__ void merge_numbers(const AttendArgs& a, int head, const Unit& u, int col0, int cols, const float* part, const float* weights, int tid) {
  constexpr int STEP = COLS * (D + 2);
  const int all = cols * (D / 4);
  for (int i0 = tid; i0 < all; i0 += 256 * N) {
    float4 s[N];
#pragma unroll
    for (int n = 0; n < N; ++n) s[n] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = 0; k0 < u.chunks; k0 += Q) {
      float4 v[N][Q];
#pragma unroll
      for (int e = 0; e < Q; ++e) {
        const float* from = part + (int64_t)(k0 + e < u.chunks ? k0 + e : k0) * STEP;
#pragma unroll
        for (int n = 0; n < N; ++n) v[n][e] = take_back(from + 4 * (i0 + 256 * n < all ? i0 + 256 * n : i0));
      }
#pragma unroll
      for (int e = 0; e < Q; ++e) {
        const bool on = k0 + e < u.chunks;  // (no branch: the fetches would be moved behind it, one after the other)
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const int c = (i0 + 256 * n) / (D / 4);
          const float w = weights[(on ? k0 + e : k0) * COLS + (c < COLS ? c : 0)];
          s[n].x = fmaf(w, on ? v[n][e].x : 0.f, s[n].x);
          s[n].y = fmaf(w, on ? v[n][e].y : 0.f, s[n].y);
          s[n].z = fmaf(w, on ? v[n][e].z : 0.f, s[n].z);
          s[n].w = fmaf(w, on ? v[n][e].w : 0.f, s[n].w);
        }
      }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = i0 + 256 * n, c = i / (D / 4), d = (i - c * (D / 4)) * 4;
      if (i >= all) break;
      const int col = col0 + c, r = col / a.group;
      put_out<BF16>(a, (int64_t)(u.row0 + r) * a.out_row + (int64_t)(head * a.group + (col - r * a.group)) * a.out_head + d, s[n]);
    }
  }
}

template <int COLS, int D, bool BF16>
__device__ __forceinline__ void merge(const AttendArgs& a, int head, const Unit& u, int col0, float* lds, int tid) {
  // lds [chunks][COLS]: M, then what each unit's numbers are multiplied with; behind it [chunks][COLS]: sums
  constexpr int STEP = COLS * (D + 2), EACH = 256 / COLS;  // EACH threads share a column
  const int cols = u.rows * a.group - col0 < COLS ? u.rows * a.group - col0 : COLS;
  const float* part = part_numbers<COLS, D>(a, head, u.first);
  {
    const int c = tid / EACH, j = tid % EACH;
    float* tops = lds + c;
    float* sums = lds + u.chunks * COLS + c;
    float top = -INFINITY, sum = 0.f;
    if (c < cols) {
#pragma unroll 4
      for (int k = j; k < u.chunks; k += EACH) {
        const float2 v = take_back2(part + (int64_t)k * STEP + COLS * D + 2 * c);
        tops[k * COLS] = v.x;
        sums[k * COLS] = v.y;
        top = fmaxf(top, v.x);
      }
    }
    top = wave_max<EACH>(top);
    const float base = top == -INFINITY ? 0.f : top;
    if (c < cols)
      for (int k = j; k < u.chunks; k += EACH) {
        const float half = exp2_fast(0.5f * (tops[k * COLS] - base));  // (of the weight, which may be 0 where its part of the sum is not)
        tops[k * COLS] = half * half;
        sum = fmaf(half * sums[k * COLS], half, sum);
      }
    sum = wave_sum<EACH>(sum);
    const float back = sum == 0.f ? 0.f : 1.f / sum;
    if (c < cols)
      for (int k = j; k < u.chunks; k += EACH) tops[k * COLS] *= back;
  }
  __syncthreads();
  if (u.chunks <= 4) merge_numbers<COLS, D, BF16, 4, 4>(a, head, u, col0, cols, part, lds, tid);
  else if (u.chunks <= 8) merge_numbers<COLS, D, BF16, 2, 8>(a, head, u, col0, cols, part, lds, tid);
  else if (u.chunks <= 16 || COLS > kNarrowColumns || D == 64) merge_numbers<COLS, D, BF16, 1, 16>(a, head, u, col0, cols, part, lds, tid);
  else if constexpr (COLS == kNarrowColumns && D > 64) merge_numbers<COLS, D, BF16, 1, 32>(a, head, u, col0, cols, part, lds, tid);  // (heads of 64 would lose half of their waves)
}

// Four waves on the pages of one 16-column tile, every fourth each.
template <bool BF16, int D, bool TREE = false>
__device__ __forceinline__ void attend_narrow_body(const AttendArgs& a, const TreeMasks& tree = {}) {
  constexpr int COLS = 16, MOST = kNarrowUnits, PITCH = D + 4;
  extern __shared__ float4 smem4[];
  float* lds = (float*)smem4;  // [4][16][PITCH] numbers, [4][16] M, [4][16] sums of weights, a flag; the merge takes the numbers' place
  float* tops = lds + narrow_numbers(D);
  float* sums = tops + 4 * COLS;
  int* flag = (int*)(sums + 4 * COLS);
  const int head = blockIdx.x % a.c.kv_heads, tid = threadIdx.x, wave = uniform(tid >> 6);
  Unit u;
  if (!find_unit<COLS, MOST, TREE>(a, blockIdx.x / a.c.kv_heads, &u)) return;
  const int col0 = u.tile * COLS, cols = u.rows * a.group - col0 < COLS ? u.rows * a.group - col0 : COLS;
  // (of a tree: all columns see the cached tokens, and each may see any of the nodes)
  const int pos_lo = TREE ? u.before - 1 : u.before + col0 / a.group, pos_hi = TREE ? u.before + u.rows - 1 : u.before + (col0 + cols - 1) / a.group;
  Columns<BF16, D, COLS, TREE> w;
  w.start(a, tree, u, head, col0);
  int lo, hi = seen_pages<TREE>(a, u.rows, u.before, &lo);
  lo += u.chunk * u.per;
  hi = hi < lo + u.per ? hi : lo + u.per;
  const int end = pos_hi < 0 ? 0 : pos_hi / kPage + 1;
  w.run(a, u, head, lo + wave, hi < end ? hi : end, 4, pos_lo, pos_hi);
  if (w.lane < COLS) {
    tops[wave * COLS + w.c()] = w.top;
    sums[wave * COLS + w.c()] = w.sum;
  }
#pragma unroll
  for (int t = 0; t < D / COLS; ++t) *(float4*)(lds + (wave * COLS + w.c()) * PITCH + w.channel(t, 0)) = make_float4(w.o[t][0], w.o[t][1], w.o[t][2], w.o[t][3]);
  __syncthreads();
  float* part = part_numbers<COLS, D>(a, head, u.first + u.chunk);
  for (int i = tid; i < cols * (D / 4); i += 256) {
    const int c = i / (D / 4), d = (i - c * (D / 4)) * 4;
    float top = tops[c], sum = 0.f;
#pragma unroll
    for (int k = 1; k < 4; ++k) top = fmaxf(top, tops[k * COLS + c]);
    const float base = top == -INFINITY ? 0.f : top;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float half = exp2_fast(0.5f * (tops[k * COLS + c] - base)), f = half * half;  // (as in merge)
      const float4 v = *(const float4*)(lds + (k * COLS + c) * PITCH + d);
      sum = fmaf(half * sums[k * COLS + c], half, sum);
      s.x = fmaf(f, v.x, s.x);
      s.y = fmaf(f, v.y, s.y);
      s.z = fmaf(f, v.z, s.z);
      s.w = fmaf(f, v.w, s.w);
    }
    if (u.chunks == 1) {
      const float back = sum == 0.f ? 0.f : 1.f / sum;
      s.x *= back;
      s.y *= back;
      s.z *= back;
      s.w *= back;
      const int col = col0 + c, r = col / a.group;
      put_out<BF16>(a, (int64_t)(u.row0 + r) * a.out_row + (int64_t)(head * a.group + (col - r * a.group)) * a.out_head + d, s);
    } else {
      put((void*)(part + c * D + d), s);
      if (d == 0) leave2(part + COLS * D + 2 * c, top, sum);
    }
  }
  if (u.chunks > 1 && arrive(a.count + (int64_t)head * a.units + u.first, u.chunks, flag, tid)) merge<COLS, D, BF16>(a, head, u, col0, lds, tid);
}

// A page in LDS as f16, shared by the waves of a workgroup.  Sixteen neighbouring lanes read sixteen keys (channels) at one place, so the
// 16-byte pieces of a row are exchanged by what tells these rows apart, and the lanes find them on different banks.
template <int D>
struct SharedPage {
  static constexpr bool kShared = true;
  static constexpr int ROW = D / 8;             // pieces of a key (of a channel: eight)
  static constexpr int PIECES = kPage * ROW;    // of K; as many of V behind them
  const u32x4* lds;
  uint32_t ks, vs;
  int lane;
  static __device__ __forceinline__ int key_place(int token, int piece) {
    const int by = (token & 7) | ((token >> 1) & 8);  // what tells the tokens of sixteen lanes apart
    return token * ROW + (piece ^ (ROW >= 16 ? by : by >> 1));
  }
  static __device__ __forceinline__ int value_place(int channel, int piece) { return PIECES + channel * 8 + (piece ^ ((channel >> 1) & 7)); }
  __device__ __forceinline__ f16x8 key(int t, int j) const {
    return __builtin_bit_cast(f16x8, lds[key_place(Columns<true, D, 32>::token_of(t, lane & 31), (lane >> 5) * (D / 16) + j)]);
  }
  template <bool MASKED>
  __device__ __forceinline__ void values(int t, int h, int t1, int lo, int hi, uint32_t* found, f16x8 (&x)[2]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u32x4 w = lds[value_place(t * 32 + (lane & 31), (h * 2 + (lane >> 5)) * 2 + i)];
      if (MASKED) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t2 = t1 + i * 8 + e * 2;
          w[e] &= halves_below(hi + 1 - t2) & ~halves_below(lo - t2);
          // a NaN has all bits of the exponent, which no finite code has as f16
          const uint32_t n = ((~(((w[e] & 0x7c007c00u) ^ 0x7c007c00u) + 0x7fff7fffu) & 0x80008000u) >> 15) * 0xffffu;
          *found |= n;
          w[e] &= ~n;
        }
      }
      x[i] = __builtin_bit_cast(f16x8, w);
    }
  }
};

// Four waves side by side on 32 columns each.  They share the pages: each fetches a quarter of the next one in whole cache lines while
// the present one is used from LDS, and spreads it to f16 once for all (a wave's operands straight from memory are 32 rows a load, 64 cycles of the CU's address
// unit: 4096 a page for the four, of 1024 for the matrix instructions).
template <bool BF16, int D, bool TREE = false>
__device__ __forceinline__ void attend_wide_body(const AttendArgs& a, const TreeMasks& tree = {}) {
  constexpr int COLS = 128, MOST = kWideUnits, PIECES = SharedPage<D>::PIECES, EACH = kPage * D / 16 / 256 * 2;  // 16-byte pieces of a page that a thread fetches
  extern __shared__ uint4 smem_pages[];
  float* lds = (float*)smem_pages;  // two pages; later for the merge [2][MOST][128]; a flag
  int* flag = (int*)(lds + wide_numbers(D));
  const int head = blockIdx.x % a.c.kv_heads, wave = uniform(threadIdx.x >> 6);
  Unit u;
  if (!find_unit<COLS, MOST, TREE>(a, blockIdx.x / a.c.kv_heads, &u)) return;
  const int all = u.rows * a.group, col0 = u.tile * COLS, mine0 = col0 + wave * 32;
  const int tile_cols = all - col0 < COLS ? all - col0 : COLS, cols = all - mine0 < 32 ? all - mine0 : 32;  // (cols may be none)
  // pages of the workgroup, and of the wave
  int lo, hi = seen_pages<TREE>(a, u.rows, u.before, &lo);
  lo += u.chunk * u.per;
  hi = hi < lo + u.per ? hi : lo + u.per;
  const int tile_lo = TREE ? u.before - 1 : u.before + col0 / a.group, tile_hi = TREE ? u.before + u.rows - 1 : u.before + (col0 + tile_cols - 1) / a.group;
  const int end = tile_hi < 0 ? 0 : tile_hi / kPage + 1, from = a.window > 0 && tile_lo >= a.window ? (tile_lo - a.window + 1) / kPage : 0;
  hi = hi < end ? hi : end;
  lo = lo > from ? lo : from;
  const int pos_lo = TREE ? tile_lo : u.before + mine0 / a.group, pos_hi = cols > 0 ? (TREE ? tile_hi : u.before + (mine0 + cols - 1) / a.group) : -1;
  const int see_lo = a.window > 0 ? pos_lo - a.window + 1 : 0;

  Columns<BF16, D, 32, TREE> w;
  w.start(a, tree, u, head, cols > 0 ? mine0 : col0);

  u32x4 next[EACH];
  uint32_t next_ks = 0, next_vs = 0;
  auto fetch = [&](int page) {
    const int tid = wave * 64 + w.lane;
    const int64_t ph = (int64_t)page * a.c.kv_heads + head;
    next_ks = *(const uint32_t*)(a.c.k_scale + ph * 4);
    next_vs = *(const uint32_t*)(a.c.v_scale + ph * 4);
    const u32x4* k = (const u32x4*)(a.c.k + ph * (kPage * D));
    const u32x4* v = (const u32x4*)(a.c.v + ph * (kPage * D));
#pragma unroll
    for (int i = 0; i < EACH / 2; ++i) {
      next[i] = k[i * 256 + tid];
      next[EACH / 2 + i] = v[i * 256 + tid];
    }
  };
  auto store = [&](int buf) {
    const int tid = wave * 64 + w.lane;
    u32x4* to = (u32x4*)smem_pages + buf * 2 * PIECES;
#pragma unroll
    for (int i = 0; i < EACH / 2; ++i) {
      const int n = i * 256 + tid;
      const u32x4 k = next[i], v = next[EACH / 2 + i];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        to[SharedPage<D>::key_place(n / (D / 16), n % (D / 16) * 2 + e)] = __builtin_bit_cast(u32x4, f16_of_codes(k[2 * e], k[2 * e + 1]));
        to[SharedPage<D>::value_place(n / 4, n % 4 * 2 + e)] = __builtin_bit_cast(u32x4, f16_of_codes(v[2 * e], v[2 * e + 1]));
      }
    }
  };
  // page numbers, 64 at a time (a wave has them all: the loop is the same for all four)
  int ids = -1, ids0 = 0;
  auto number = [&](int p) {
    if (p - ids0 >= 64) {
      ids0 = p;
      ids = p + w.lane < hi ? page_of(a.c, u.s, p + w.lane) : -1;
    }
    return __builtin_amdgcn_readlane(ids, p - ids0);
  };
  int page = -1;
  auto advance = [&](int p) {  // the first page from p on that is there
    for (; p < hi; ++p)
      if ((page = number(p)) >= 0) break;
    return p;
  };
  ids0 = lo;
  ids = lo + w.lane < hi ? page_of(a.c, u.s, lo + w.lane) : -1;
  int p = advance(lo), buf = 0;
  if (p < hi) {
    fetch(page);
    store(0);
  }
  while (p < hi) {
    __syncthreads();
    SharedPage<D> now;
    now.lds = (const u32x4*)smem_pages + buf * 2 * PIECES;
    now.ks = next_ks;
    now.vs = next_vs;
    now.lane = w.lane;
    const int after = advance(p + 1), t0 = p * kPage;
    if (after < hi) fetch(page);
    if (t0 <= pos_hi && (a.window == 0 || t0 + kPage > see_lo)) {
      if (w.is_masked(a, t0, pos_lo, pos_hi)) w.template take_page<true>(a, now, t0, see_lo, pos_hi, [] {});
      else w.template take_page<false>(a, now, t0, see_lo, pos_hi, [] {});
    }
    buf ^= 1;
    if (after < hi) store(buf);
    p = after;
  }
  w.mark_nans(a, u, head, lo, hi, 1, pos_lo, pos_hi);
  w.finish();
  if (cols > 0) {
    const bool on = w.c() < cols;
    const int col = mine0 + (on ? w.c() : 0), r = col / a.group;
    const int64_t at = (int64_t)(u.row0 + r) * a.out_row + (int64_t)(head * a.group + (col - r * a.group)) * a.out_head;
    float* part = part_numbers<COLS, D>(a, head, u.first + u.chunk);
    const float back = u.chunks > 1 ? 1.f : w.sum == 0.f ? 0.f : 1.f / w.sum;
    if (on) {
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 v = make_float4(w.o[t][i] * back, w.o[t][i + 1] * back, w.o[t][i + 2] * back, w.o[t][i + 3] * back);
          if (u.chunks == 1) put_out<BF16>(a, at + w.channel(t, i), v);
          else put((void*)(part + (wave * 32 + w.c()) * D + w.channel(t, i)), v);
        }
      if (u.chunks > 1 && w.g() == 0) leave2(part + COLS * D + 2 * (wave * 32 + w.c()), w.top, w.sum);
    }
  }
  const int tid = wave * 64 + w.lane;
  if (u.chunks > 1 && arrive(a.count + (int64_t)head * a.units + u.first, u.chunks, flag, tid)) merge<COLS, D, BF16>(a, head, u, col0, lds, tid);
}

}  // namespace daris
