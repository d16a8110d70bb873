// Tokens and pages that change their place in the cache: the kept nodes of a tree, and whole pages.
#pragma once
#include "append_kernel.h"

namespace daris {

// Keeps tokens before + path[j] as tokens before + j.  A wave owns the keys or the values of one head of a sequence and goes through the sixteenths that get
// tokens in order.  A token never moves forwards, and a token that a later sixteenth gets lies behind every place written before, so each sixteenth is read
// whole and then written.  Which slots move, from where and with which scale is found by sixteen lanes at once; a slot that does not move is read as well (from
// its own place), so that no branch stands between the fetches.  Bound by latency: row_start and path -> pages -> scales and codes ->
// stores.  Four tokens of one sequence (8 heads of 128) 5.4 us, up to eight of 64 sequences 10 (calls of 11.1 and 15.2).
template <int D>
__device__ __forceinline__ void keep_body(const KeepArgs& a) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, wave = uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int s = (wave >> 1) / a.c.kv_heads, head = (wave >> 1) - s * a.c.kv_heads;
  if (s >= a.c.n_seqs) return;
  const int row0 = first_row(a.c, s), rows = rows_of(a.c, s), before = tokens_before(a.c, s);
  int end = a.count[s];
  end = end < rows ? end : rows;
  const int32_t* path = a.path + row0;
  // The first entry that moves a token, and the first that names none (it is not behind the one in front of it, or no row of the step).
  int first = end, early = 0;  // (early: the lane's entry of the first 64)
  for (int j0 = 0; j0 < end; j0 += 64) {
    const int j = j0 + lane;
    const bool in = j < end;
    const int p = in ? path[j] : 0, q = in && j > 0 ? path[j - 1] : -1;
    if (j0 == 0) early = p;
    const uint64_t wrong = __ballot(in && (p <= q || p >= rows));
    if (wrong) end = j0 + __builtin_ctzll(wrong);
    const uint64_t moves = __ballot(in && p != j);
    if (moves && first > j0 + __builtin_ctzll(moves)) first = j0 + __builtin_ctzll(moves);
  }
  if (first >= end) return;
  const bool values = wave & 1;
  uint8_t* const scales = values ? a.c.v_scale : a.c.k_scale;
  uint8_t* const codes = values ? a.c.v : a.c.k;
  const int stay = before + first;  // tokens in front of this one stay
  for (int64_t t0 = stay < 0 ? 0 : stay / kScaleTokens * kScaleTokens; t0 < (int64_t)before + end; t0 += kScaleTokens) {
    const int page = uniform(page_of(a.c, s, (int)(t0 / kPage)));
    if (page < 0) continue;
    const int part = (int)(t0 % kPage) / kScaleTokens, slot = lane & 15;
    const int64_t t = t0 + slot, j = t - before;
    bool move = j >= first && j < end;
    const int entry = __shfl(early, (int)j & 63);
    const int64_t from = (int64_t)before + (!move ? 0 : j < 64 ? entry : path[j]);
    int from_page = move ? page_of(a.c, s, (int)(from / kPage)) : -1, from_slot = (int)(from % kPage);
    move = from_page >= 0;
    const int64_t to_head = (int64_t)page * a.c.kv_heads + head;
    const int had = scales[to_head * 4 + part];
    if (!move) {
      from_page = page;
      from_slot = part * kScaleTokens + slot;
    }
    const int came = scales[((int64_t)from_page * a.c.kv_heads + head) * 4 + (from_slot >> 4)];
    const uint32_t moves = (uint32_t)__ballot(move) & 0xffffu, stays = (uint32_t)__ballot(t < stay) & 0xffffu;
    if (!moves) continue;
    const int now = (int)lanes_max<1, 16>(move ? (float)came : t < stay ? (float)had : 0.f);
    const float times = two_to((move ? came : had) - now);  // (of the slot: what its codes are multiplied with)
    const bool rescale = uniform(now) > had && stays;
    if (!values) {
      uint32_t w[kScaleTokens];
#pragma unroll
      for (int i = 0; i < kScaleTokens; ++i) {
        const uint8_t* p = codes + (((int64_t)__builtin_amdgcn_readlane(from_page, i) * a.c.kv_heads + head) * kPage + __builtin_amdgcn_readlane(from_slot, i)) * D + lane * E;
        w[i] = E == 4 ? *(const uint32_t*)p : E == 2 ? *(const uint16_t*)p : *p;
      }
#pragma unroll
      for (int i = 0; i < kScaleTokens; ++i) {
        if (!((moves >> i & 1) || (rescale && (stays >> i & 1)))) continue;
        const uint32_t y = shrunk(w[i], __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, times), i)));
        uint8_t* p = codes + (to_head * kPage + part * kScaleTokens + i) * D + lane * E;
        if (E == 4) *(uint32_t*)p = y;
        else if (E == 2) *(uint16_t*)p = (uint16_t)y;
        else *p = (uint8_t)y;
      }
    } else {
      uint32_t w[E][kScaleTokens];
      uint4 was[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        was[e] = *(const uint4*)(codes + (to_head * D + lane + 64 * e) * kPage + part * kScaleTokens);
#pragma unroll
        for (int i = 0; i < kScaleTokens; ++i)
          w[e][i] = codes[(((int64_t)__builtin_amdgcn_readlane(from_page, i) * a.c.kv_heads + head) * D + lane + 64 * e) * kPage + __builtin_amdgcn_readlane(from_slot, i)];
      }
      const uint32_t fresh = rescale ? moves | stays : moves;
      float f[kScaleTokens];
#pragma unroll
      for (int i = 0; i < kScaleTokens; ++i) f[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, times), i));
#pragma unroll
      for (int e = 0; e < E; ++e) {
        uint32_t out[4] = {was[e].x, was[e].y, was[e].z, was[e].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t four = w[e][4 * q] | w[e][4 * q + 1] << 8 | w[e][4 * q + 2] << 16 | w[e][4 * q + 3] << 24;
          const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(four, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(four, true);
          const uint32_t y = codes4(lo.x * f[4 * q], lo.y * f[4 * q + 1], hi.x * f[4 * q + 2], hi.y * f[4 * q + 3]);
          uint32_t bytes = 0u;
#pragma unroll
          for (int i = 0; i < 4; ++i) bytes |= fresh >> (4 * q + i) & 1 ? 0xffu << (8 * i) : 0u;
          out[q] = (y & bytes) | (out[q] & ~bytes);
        }
        *(uint4*)(codes + (to_head * D + lane + 64 * e) * kPage + part * kScaleTokens) = make_uint4(out[0], out[1], out[2], out[3]);
      }
    }
    if (lane == 0) scales[to_head * 4 + part] = (uint8_t)now;
  }
}

// Pages pairs[2 i] copied over pages pairs[2 i + 1]: a workgroup a piece of the keys or of the values, which lie side by side for all heads.  Bound by bandwidth, past the caches:
// 1001 pages of 8 heads of 128, 262 MB, 51 us, 5.2 TB/s (a call 57; through the caches 61, and 46 where they hold the pages from the call before).
template <int D>
__device__ __forceinline__ void copy_body(const CopyArgs& a) {
  const int each = 2 * a.pieces, i = blockIdx.x / each, rest = blockIdx.x - i * each, piece = rest >> 1, tid = threadIdx.x;
  const int from = a.pairs[2 * i], to = a.pairs[2 * i + 1];
  if (from < 0 || from >= a.c.n_pages || to < 0 || to >= a.c.n_pages) return;
  const bool values = rest & 1;
  const int64_t bytes = (int64_t)a.c.kv_heads * kPage * D;  // a multiple of 4096
  const uint8_t* src = (values ? a.c.v : a.c.k) + from * bytes;
  uint8_t* dst = (values ? a.c.v : a.c.k) + to * bytes;
  constexpr int N = kCopyPiece / 4096;
  const int64_t at = (int64_t)piece * kCopyPiece + tid * 16;
  u32x4 x[N];
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = __builtin_nontemporal_load((const u32x4*)(src + (at + j * 4096 < bytes ? at + j * 4096 : tid * 16)));  // (no branch: they travel together)
  const uint32_t* s_src = (const uint32_t*)(values ? a.c.v_scale : a.c.k_scale) + (int64_t)from * a.c.kv_heads;
  uint32_t* s_dst = (uint32_t*)(values ? a.c.v_scale : a.c.k_scale) + (int64_t)to * a.c.kv_heads;
  if (piece == 0)
    for (int h = tid; h < a.c.kv_heads; h += 256) s_dst[h] = s_src[h];
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (at + j * 4096 < bytes) __builtin_nontemporal_store(x[j], (u32x4*)(dst + at + j * 4096));
}

}  // namespace daris
