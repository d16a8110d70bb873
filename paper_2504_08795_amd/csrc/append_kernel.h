// Appends the step's keys and values to the paged cache, turning keys (and queries) by their positions on the way.
//
// A wave owns one sixteenth (kScaleTokens tokens that share a scale) of one key head: it is the only one that reads or writes that
// sixteenth's codes and scale, whatever part of it the step fills, so nothing is atomic.  Keys lie with a token's channels
// side by side, lane l holds channels l * D / 64 and on; values lie with a channel's tokens side by side, lane l holds channels
// l, l + 64, ... and writes their sixteen bytes at once.  Single tokens are bound by the latency of length -> page -> codes, prompts by
// the bytes of k and v.  A token for each of 32 streams (32 + 8 heads of 128): 7.0 us, of which three dependent fetches are 3; nine prompts of
// 4800 tokens in all (16 + 4 heads of 64, fp32), 52 MB: 14.9 us, 3.5 TB/s.
// Where rows are nodes of trees a row's position is the number of bits of its mask, which sixteen lanes count for sixteen tokens at once, and a sixteenth's keys and values go in
// two waves: nodes fill sixteenths, whose rounding then is what takes the time (26 nodes of one stream 10.9 us in one wave, 8.6 in two; a call 14.5).
#pragma once
#include "step_common.h"

namespace daris {

// Which channel a channel is turned with, by which entry of the table, and whether it is the first of the two.
struct Turn {
  int with = 0, j = 0;
  bool on = false, first = false;
};
__device__ __forceinline__ Turn turn_of(int d, int rot, int pairs) {
  Turn t;
  t.on = d < rot;
  if (pairs) {
    t.with = d ^ 1;
    t.j = d >> 1;
    t.first = !(d & 1);
  } else {
    const int half = rot >> 1;
    t.first = d < half;
    t.with = t.first ? d + half : d - half;
    t.j = t.first ? d : d - half;
  }
  if (!t.on) {
    t.with = d;
    t.j = 0;
  }
  return t;
}
// Products and their difference are rounded one by one, as elementary operations on fp32 tensors round them.
__device__ __forceinline__ float turned(const Turn& t, float x, float other, float c, float s) {
#pragma clang fp contract(off)
  const float a = x * c, b = other * s;
  const float y = t.first ? a - b : a + b;
  return t.on ? y : x;
}
__device__ __forceinline__ void table_entry(const AppendArgs& a, const Turn& t, int pos, float* c, float* s) {
  const bool in = pos >= 0 && pos < a.turn_rows;
  const float* row = a.turn + (int64_t)(in ? pos : 0) * a.rot_dim + t.j;
  *c = *s = __uint_as_float(0x7fc00000u);
  if (in && t.on) {
    *c = row[0];
    *s = row[a.rot_dim >> 1];
  }
}

// Codes under a scale 1 / shrink times as large.
__device__ __forceinline__ uint32_t shrunk(uint32_t codes, float shrink) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  return codes4(lo.x * shrink, lo.y * shrink, hi.x * shrink, hi.y * shrink);
}

// Position of a row in its sequence: `at` where rows follow each other; of a node that of the first new token and the nodes above it.
template <bool TREE>
__device__ __forceinline__ int position_of(const TreeMasks& tree, int row, int before, int at) {
  if (!TREE) return at;
  const uint64_t* mask = tree.mask + (int64_t)row * tree.words;
  int n = -1;
  for (int w = 0; w < tree.words; ++w) n += __popcll(mask[w]);
  return before + n;
}

// KEYS, VALUES: what of the two this wave appends.
template <bool BF16, int D, bool TREE, bool KEYS = true, bool VALUES = true>
__device__ __forceinline__ void append_sixteenth(const AppendArgs& a, const TreeMasks& tree, int head, int row0, int page, int part, int lo, int hi, int pos0, int before) {
  // tokens lo .. hi - 1 of the sixteenth are rows row0 ... of the step, their places pos0 ... of the sequence
  constexpr int E = D / 64, Q = 4;  // channels of a lane; tokens that are read together
  const int lane = threadIdx.x & 63;
  const int64_t ph = (int64_t)page * a.c.kv_heads + head;
  const int had_k = lo > 0 ? a.c.k_scale[ph * 4 + part] : kLeastScale, had_v = lo > 0 ? a.c.v_scale[ph * 4 + part] : kLeastScale;

  const int mine = lane < lo ? lo : lane < hi ? lane : hi - 1;  // (TREE: lane i has the position of token i)
  const int position = KEYS ? position_of<TREE>(tree, row0 + mine - lo, before, 0) : 0;
  float xv[kScaleTokens][E];
  {  // ---- keys
    Turn t[E];
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] = turn_of(lane * E + e, a.rot_dim, a.pairs);
    float x[kScaleTokens][E];
    float most = 0.f, most_v = 0.f;
#pragma unroll
    for (int b = 0; b < kScaleTokens / Q; ++b) {
#pragma unroll
      for (int i = 0; i < Q; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) x[b * Q + i][e] = xv[b * Q + i][e] = 0.f;
      if (b * Q + Q <= lo || b * Q >= hi) continue;
      float own[Q][E], other[Q][E], c[Q][E], s[Q][E];
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        const int tok = b * Q + i, in = tok < lo ? lo : tok >= hi ? hi - 1 : tok;
        const int64_t kr = (int64_t)(row0 + in - lo) * a.k_row + head * a.k_head, vr = (int64_t)(row0 + in - lo) * a.v_row + head * a.v_head;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if constexpr (KEYS) own[i][e] = load_elem<BF16>(a.k, kr + lane * E + e);
          if constexpr (KEYS) other[i][e] = load_elem<BF16>(a.k, kr + t[e].with);
          if constexpr (VALUES) xv[tok][e] = load_elem<BF16>(a.v, vr + lane + 64 * e);
          c[i][e] = 1.f;
          s[i][e] = 0.f;
          if (KEYS && a.rot_dim) table_entry(a, t[e], TREE ? __builtin_amdgcn_readlane(position, in) : pos0 + in - lo, &c[i][e], &s[i][e]);
        }
      }
#pragma unroll
      for (int i = 0; i < Q; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int tok = b * Q + i;
          const bool on = tok >= lo && tok < hi;
          if constexpr (KEYS) x[tok][e] = on ? turned(t[e], own[i][e], other[i][e], c[i][e], s[i][e]) : 0.f;
          if (!on) xv[tok][e] = 0.f;
          most = fmaxf(most, size_of(x[tok][e]));
          most_v = fmaxf(most_v, size_of(xv[tok][e]));
        }
    }
    if constexpr (KEYS) {
    const int need = scale_byte(wave_max<64>(most)), now = need > had_k ? need : had_k;
    const float inv = two_to(127 - now), shrink = two_to(had_k - now);
    uint8_t* k = a.c.k + (ph * kPage + part * kScaleTokens) * D + lane * E;
#pragma unroll
    for (int tok = 0; tok < kScaleTokens; ++tok) {
      const bool fresh = tok >= lo && tok < hi;
      if (!fresh && !(tok < lo && now > had_k)) continue;
      uint8_t* p = k + tok * D;
      uint32_t w = 0;
      if (fresh) {
        w = codes4(x[tok][0] * inv, E > 1 ? x[tok][E > 1] * inv : 0.f, E > 2 ? x[tok][E > 2 ? 2 : 0] * inv : 0.f, E > 2 ? x[tok][E > 2 ? 3 : 0] * inv : 0.f);
      } else {
        w = E == 4 ? *(const uint32_t*)p : E == 2 ? *(const uint16_t*)p : *p;
        w = shrunk(w, shrink);
      }
      if (E == 4) *(uint32_t*)p = w;
      else if (E == 2) *(uint16_t*)p = (uint16_t)w;
      else *p = (uint8_t)w;
    }
    if (lane == 0) a.c.k_scale[ph * 4 + part] = (uint8_t)now;
    }
    if constexpr (!VALUES) return;
    // ---- values
    const int need_v = scale_byte(wave_max<64>(most_v)), now_v = need_v > had_v ? need_v : had_v;
    const float inv_v = two_to(127 - now_v), shrink_v = two_to(had_v - now_v);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      uint4* p = (uint4*)(a.c.v + (ph * D + lane + 64 * e) * kPage + part * kScaleTokens);
      uint4 was = make_uint4(0u, 0u, 0u, 0u);
      if (lo > 0 || hi < kScaleTokens) was = *p;
      uint32_t w[4] = {was.x, was.y, was.z, was.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t fresh = codes4(xv[4 * q][e] * inv_v, xv[4 * q + 1][e] * inv_v, xv[4 * q + 2][e] * inv_v, xv[4 * q + 3][e] * inv_v);
        uint32_t in_front = 0u, new_ones = 0u;  // bytes of earlier tokens, of the step's
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          in_front |= 4 * q + i < lo ? 0xffu << (8 * i) : 0u;
          new_ones |= 4 * q + i >= lo && 4 * q + i < hi ? 0xffu << (8 * i) : 0u;
        }
        if (now_v > had_v) w[q] = (shrunk(w[q], shrink_v) & in_front) | (w[q] & ~in_front);
        w[q] = (fresh & new_ones) | (w[q] & ~new_ones);
      }
      *p = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (lane == 0) a.c.v_scale[ph * 4 + part] = (uint8_t)now_v;
  }
}

// One of kTurnHeads neighbouring query heads of a row after the other, all of them read before the first is written (in place).
template <bool BF16, int D>
__device__ __forceinline__ void turn_queries(const AppendArgs& a, int row, int head0, int pos) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  float own[kTurnHeads][E], other[kTurnHeads][E], c[E], s[E];
  Turn t[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    t[e] = turn_of(lane * E + e, a.rot_dim, a.pairs);
    c[e] = 1.f;
    s[e] = 0.f;
    if (a.rot_dim) table_entry(a, t[e], pos, &c[e], &s[e]);
  }
#pragma unroll
  for (int h = 0; h < kTurnHeads; ++h) {
    const int head = head0 + h < a.q_heads ? head0 + h : a.q_heads - 1;
    const int64_t at = (int64_t)row * a.q_row + head * a.q_head;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      own[h][e] = load_elem<BF16>(a.q, at + lane * E + e);
      other[h][e] = load_elem<BF16>(a.q, at + t[e].with);
    }
  }
#pragma unroll
  for (int h = 0; h < kTurnHeads; ++h) {
    if (head0 + h >= a.q_heads) break;
    const int64_t at = (int64_t)row * a.qo_row + (head0 + h) * a.qo_head + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float y = turned(t[e], own[h][e], other[h][e], c[e], s[e]);
      if (BF16) ((uint16_t*)a.q_out)[at + e] = (uint16_t)f32_to_bf16_bits(y);
      else ((float*)a.q_out)[at + e] = y;
    }
  }
}

// The last sequence s whose first_row(s) / DIV + PER s is at most `at` (they grow with s), found by all lanes at once: a search by halves would wait
// for memory once for every halving.
template <int DIV, int PER>
__device__ __forceinline__ int sequence_at(const CacheArgs& c, int at) {
  int found = 0;
  for (int s0 = 0; s0 < c.n_seqs; s0 += 64) {
    const int s = s0 + (threadIdx.x & 63);
    const int n = __popcll(__ballot(s < c.n_seqs && first_row(c, s < c.n_seqs ? s : 0) / DIV + PER * s <= at));
    found += n;
    if (n < 64) break;
  }
  return found > 0 ? found - 1 : 0;
}

// Waves: first a.items sixteenths x key heads, then a.q_items groups of query heads.  TREE: rows are nodes of trees.
template <bool BF16, int D, bool TREE = false>
__device__ __forceinline__ void append_body(const AppendArgs& a, const TreeMasks& tree = {}) {
  const int wave = uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (wave < a.items) {
    const int both = TREE ? wave >> 1 : wave;  // (of a tree, whose nodes fill sixteenths, two waves share one: see kTreeAppendWaves)
    const int item = both / a.c.kv_heads, head = both - item * a.c.kv_heads;
    // Sequence s has the items from first_row(s) / 16 + 2 s on: n tokens lie in at most n / 16 + 2 sixteenths.
    int s = item, base = item;
    if (a.c.row_start) {
      s = sequence_at<kScaleTokens, 2>(a.c, item);
      base = first_row(a.c, s) / kScaleTokens + 2 * s;
    }
    if (s >= a.c.n_seqs) return;
    const int row0 = first_row(a.c, s), n = rows_of(a.c, s), before = tokens_before(a.c, s);
    if (n == 0 || item < base || before + n <= 0) return;
    const int start = before < 0 ? 0 : before;  // the first token that has a place
    const int64_t sixteenth = (int64_t)(start / kScaleTokens) + (item - base);
    const int64_t t0 = sixteenth * kScaleTokens;
    if (t0 >= before + n) return;
    const int lo = start > t0 ? (int)(start - t0) : 0, hi = before + n - t0 < kScaleTokens ? (int)(before + n - t0) : kScaleTokens;
    const int page = page_of(a.c, s, (int)(t0 / kPage));
    if (page < 0) return;
    const int tok = (int)t0 + lo;
    const int row = row0 + (tok - before), part = (int)(sixteenth % (kPage / kScaleTokens));
    if constexpr (TREE) {
      if (wave & 1) append_sixteenth<BF16, D, true, false, true>(a, tree, head, row, page, part, lo, hi, tok, before);
      else append_sixteenth<BF16, D, true, true, false>(a, tree, head, row, page, part, lo, hi, tok, before);
    } else {
      append_sixteenth<BF16, D, false>(a, tree, head, row, page, part, lo, hi, tok, before);
    }
  } else if (wave < a.items + a.q_items) {
    const int per_row = (a.q_heads + kTurnHeads - 1) / kTurnHeads;
    const int i = wave - a.items, row = i / per_row, head = (i - row * per_row) * kTurnHeads;
    int s = row;
    if (a.c.row_start) {
      s = sequence_at<1, 0>(a.c, row);
      if (row < first_row(a.c, s) || row >= first_row(a.c, s + 1)) return;
    }
    const int before = tokens_before(a.c, s);
    turn_queries<BF16, D>(a, row, head, position_of<TREE>(tree, row, before, before + (row - first_row(a.c, s))));
  }
}

}  // namespace daris
