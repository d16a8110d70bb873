// Products of a few rows with 4-bit weights and a scale for each group of channels.
//
// y^T is computed in tiles of 16 outputs: a wave reads 16 rows of weights, 128 channels (a step) at a time, 16 bytes a lane straight
// into registers, spreads the nibbles and multiplies them with the rows of x on the matrix instructions.  A group's sum is
// taken by them alone and multiplied by the weights' scale once, in fp32.  x lies in LDS in the order of the nibbles.
//   bf16 x: as it is.  0x3b80 | c is the bf16 number 2^-15 (128 + c); a second product with the constant -136 * 2^-15 takes the rest away.  Both sums are 17 times
//     as large as the result, which costs four of fp32's 24 bits; the power of two, which the end takes out again, keeps those of 128 of the largest numbers finite.
//   fp32 x: two f16 parts (22 bits), a group of a row divided by a power of two that makes its largest number 2^14 and more, so that
//     nothing overflows; 0x3c00 | c << 6 is the f16 number (16 + c) / 16.  The sum begins with -24 / 16 of that of x, which is taken in fp32 when x is
//     staged; it gets up to four times as large as the result, which costs two of fp32's 24 bits.  (c - 8 took three packed additions more for eight
//     nibbles, and one row's 4096 products with 25088 channels 26.7 us a call.  Nibbles as subnormal f16 numbers take three instructions less, but
//     the matrix instructions keep 20 bits of such a sum.)
//   e4m3 x: f16 holds every one of them, 16 times; the same.
// The waves of a workgroup share x, and neighbouring ones a tile: each takes neighbouring steps of it, and their sums are added in
// wave order.  A workgroup goes from group of tiles to group of tiles; x is staged once if all of K fits LDS, else in chunks: a wave fetches its part of the
// next one when it is done with the present one, and waits for it; only the weights' scales are fetched a chunk ahead.  Every wave has four steps of weights on
// their way, across chunks and tiles.  Where tiles are few, several workgroups share K.  The floor of few rows is the weights' bytes.  What they take is for two thirds the issue
// of vector instructions (16 rows in bf16 118 for each step of 1 KB in all, one row in fp32 141; the matrix instructions hold a SIMD for a sixth of its
// cycles), else what goes one after the other: x into LDS, a barrier, the first fetches, the last sums.  One row, 4096 outputs of 4096 channels (e4m3): 6.5 us (9 MB,
// 1.7 us at a copy's rate); 16 rows, 22016 of 4096, gated (bf16): 18.1 us (47 MB, 9.2); one row, 4096 of 25088 (fp32): 20.1 us (55 MB, 10.7); 2000 rows,
// 22016 of 4096 (bf16): 900 us a call, 400 TFLOP/s.
#pragma once
#include "step_common.h"

namespace daris {

enum { kRowsF32 = 0, kRowsBf16 = 1, kRowsF8 = 2 };

// What spreads nibbles: the constants stay in registers (an instruction that takes both as literals does not exist, and two take twice as long).
template <int XT>
struct Spread {
  uint32_t mask = XT == kRowsBf16 ? 0x000f000fu : 0x03c003c0u, high = XT == kRowsBf16 ? 0x3b803b80u : 0x3c003c00u;
  u32x4 minus = {0xbb88bb88u, 0xbb88bb88u, 0xbb88bb88u, 0xbb88bb88u};  // -136 * 2^-15 as bf16
  __device__ __forceinline__ Spread() {
    asm volatile("" : "+s"(mask));
    asm volatile("" : "+v"(high));
    if (XT == kRowsBf16) asm volatile("" : "+v"(minus));
  }
  // Eight nibbles in the order 0 4 1 5 2 6 3 7: 2^-15 (128 + c) as bf16, or 1 + c / 16 as f16.
  __device__ __forceinline__ uint4 operator()(uint32_t w) const {
    if (XT == kRowsBf16) return make_uint4((w & mask) | high, ((w >> 4) & mask) | high, ((w >> 8) & mask) | high, ((w >> 12) & mask) | high);
    return make_uint4(((w << 6) & mask) | high, ((w << 2) & mask) | high, ((w >> 2) & mask) | high, ((w >> 6) & mask) | high);
  }
};

// Eight channels of x in the nibbles' order.
__device__ __forceinline__ f16x8 f16_in_order(const float (&v)[8]) {
  f16x8 h;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[2 * i] = (_Float16)v[i];
    h[2 * i + 1] = (_Float16)v[i + 4];
  }
  return h;
}
// ... of 16-bit numbers, two to a word.
__device__ __forceinline__ uint4 in_order(const uint4& v) {
  return make_uint4(__builtin_amdgcn_perm(v.z, v.x, 0x05040100u), __builtin_amdgcn_perm(v.z, v.x, 0x07060302u), __builtin_amdgcn_perm(v.w, v.y, 0x05040100u),
                    __builtin_amdgcn_perm(v.w, v.y, 0x07060302u));
}

// Where lane group g has its eight channels for the j-th matrix instruction of a step of 128.  All of an instruction's channels belong
// to one group of G.
template <int G>
__device__ __forceinline__ constexpr int piece(int j, int g) {
  return G == 128 ? g * 32 + j * 8 : G == 64 ? (j >> 1) * 64 + (g & 1) * 32 + (g >> 1) * 16 + (j & 1) * 8 : j * 32 + g * 8;
}
// (j, g) of a piece, as j * 4 + g
template <int G>
__device__ __forceinline__ int place(int k) {
  const int p = k >> 3;
  if (G == 128) return (p & 3) * 4 + (p >> 2);
  if (G == 64) return ((p >> 3) * 2 + (p & 1)) * 4 + ((p >> 2) & 1) + (p & 2);
  return p;
}

// The 32 weights of a lane: 16 bytes of a row, lane group g the channels 32 g and on.  (Sixteen rows a load are as many cache lines,
// which take the CU's address unit 64 cycles however few bytes a lane wants.)  Groups of less than 128 are put together by
// exchanges between the lane groups.
template <int G>
__device__ __forceinline__ uint4 arranged(uint4 w) {
  if (G < 128) {
    const auto a = __builtin_amdgcn_permlane32_swap(w.x, w.z, false, false), b = __builtin_amdgcn_permlane32_swap(w.y, w.w, false, false);
    w = make_uint4(a[0], b[0], a[1], b[1]);
  }
  if (G == 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(w.x, w.y, false, false), b = __builtin_amdgcn_permlane16_swap(w.z, w.w, false, false);
    w = make_uint4(a[0], a[1], b[0], b[1]);
  }
  return w;
}

// Eight channels of a row of x on their way to LDS.
template <int XT>
struct RowPiece {
  uint4 v[XT == kRowsF32 ? 2 : 1];
  int scale;
};

// The same number, which the compiler does not know: addresses that come from it are computed where they are used, rather than held in
// registers from turn to turn.
__device__ __forceinline__ int afresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

template <int XT, int G, bool BF16_OUT>
__device__ __forceinline__ void matvec_body(const MatvecArgs& a) {
  // (short: with one row a wave has two or three steps to do, and what it computes around them takes longer than the steps)
  constexpr int PARTS = XT == kRowsF32 ? 2 : 1, GS = 128 / G, ROWS = kMatvecRows, T = kMatvecWaves * 64;
  constexpr int PIECES = matvec_pieces(PARTS), RING = 4, ES = XT == kRowsF32 ? 4 : XT == kRowsBf16 ? 2 : 1;
  extern __shared__ uint4 smem[];
  typedef char __attribute__((address_space(3))) * Lds;
  const Lds lds = (Lds)smem;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  const int split_log = 4 - a.across;  // tiles side by side: 1 << across; waves on one of them: 1 << split_log
  const int own_tile = wave >> split_log, part = wave & ((1 << split_log) - 1);
  int m0 = 0, tg = blockIdx.x, share = 0;  // share: of K, where several workgroups have one
  if (a.shares > 1) {
    tg = blockIdx.x / a.shares;
    share = blockIdx.x - tg * a.shares;
  }
  const int unit = tg;
  if (a.rows > ROWS) {
    const int mb = tg / a.wgs;
    m0 = mb * ROWS;
    tg -= mb * a.wgs;
  }
  const int rows = a.rows - m0 < ROWS ? a.rows - m0 : ROWS;
  const int cs = a.steps, all_steps = (a.k + 127) >> 7, step0 = share * a.share_steps, chunks = a.chunks;
  const int steps = all_steps - step0 < a.share_steps ? all_steps - step0 : a.share_steps;
  // LDS, in bytes: x [PARTS][step][row][instruction, lane group], the last exchanged by the row's number so that rows lie on different banks, and (of scaled
  // rows) their scales and what their sums begin with [step][four rows][group][2][4], twice if there is more than one chunk; the weights' scales [tiles * 16][pitch] twice if there is more to
  // come; sums [waves][ROWS][16]
  const int fours = (rows + 3) >> 2;
  const int part_size = cs * rows * 256, x_size = PARTS * part_size + (XT == kRowsBf16 ? 0 : cs * fours * GS * 32), pitch = a.pitch * 2;
  const int ws_at = (chunks > 1 ? 2 : 1) * x_size, ws_size = (16 << a.across) * pitch;
  float __attribute__((address_space(3)))* const red = (float __attribute__((address_space(3)))*)(lds + ws_at + (chunks > 1 || a.wgs < a.groups ? 2 : 1) * ws_size);

  // ---- weights: the wave's steps of a chunk are neighbouring ones, so that it reads whole cache lines
  const int own = (cs + (1 << split_log) - 1) >> split_log, first = part * own, turns = (own + RING - 1) & -RING;
  struct List {  // the wave's steps of a tile in a chunk: where the first is, how many there are, how much later the step comes that ends K
    const uint8_t* w;
    int n, to_last;
  };
  auto list = [&](int tg, int ch) {
    const int n = ((tg << a.across) + own_tile) * 16 + c, st = ch * cs + first;
    List l;
    l.n = tg < a.groups ? (cs < steps - ch * cs ? cs : steps - ch * cs) - first : 0;
    l.n = l.n < own ? l.n : own;
    l.to_last = all_steps - 1 - step0 - st;
    l.w = a.w + (int64_t)(n < a.n ? n : a.n - 1) * a.w_row + (step0 + st) * 64 + g * 16;
    return l;
  };
  // Channels past K: their x is 0, so any weights will do -- those of lane group 0.
  const int past = (a.k & 127) != 0 && g * 32 >= (a.k & 127) ? -g * 16 : 0;
  u32x4 ring[RING];
  // Steps i .. i + RING - 1 of a list.  A step that is none is fetched too, from one place for all lanes: a load that may or may not have been issued makes
  // the wave wait for all of them.
  auto fetch = [&](int slot, const List& l, int i) {
    const uint8_t* from = i < l.n ? l.w + i * 64 + (i == l.to_last ? past : 0) : a.w;
    ring[slot] = *(const u32x4*)from;
  };
  // ---- and their scales, eight neighbours a thread
  const int groups = a.k / G;
  u32x4 sc[kScalePieces];
  auto load_scales = [&](int tg, int ch) {
    const int tid = afresh(threadIdx.x);
#pragma unroll
    for (int i = 0; i < kScalePieces; ++i) {
      if ((i * T) >> a.eights >= 16 << a.across) break;
      const int p = i * T + tid, r = p >> a.eights, from = (step0 + ch * cs) * GS + (p & ((1 << a.eights) - 1)) * 8;
      if (r >= 16 << a.across || from >= groups) continue;
      const int n = (tg << a.across) * 16 + r;
      const uint16_t* s = a.w_scale + (int64_t)(n < a.n ? n : a.n - 1) * groups + from;
      if (from + 8 <= groups) {
        __builtin_memcpy(&sc[i], s, 16);
      } else {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          uint32_t lo = 0u, hi = 0u;
          if (from + e < groups) lo = s[e];
          if (from + e + 1 < groups) hi = s[e + 1];
          sc[i][e / 2] = lo | hi << 16;
        }
      }
    }
  };
  auto stage_scales = [&](int buf) {
    const int tid = afresh(threadIdx.x);
#pragma unroll
    for (int i = 0; i < kScalePieces; ++i) {
      if ((i * T) >> a.eights >= 16 << a.across) break;
      const int p = i * T + tid, r = p >> a.eights, at = (p & ((1 << a.eights) - 1)) * 16;
      if (r >= 16 << a.across || at >= pitch - 4) continue;
      uint32_t __attribute__((address_space(3)))* to = (uint32_t __attribute__((address_space(3)))*)(lds + ws_at + buf * ws_size + r * pitch + at);  // (the pitch is an odd number of words)
#pragma unroll
      for (int e = 0; e < 4; ++e) to[e] = sc[i][e];
    }
  };

  // ---- rows of x: neighbouring threads take neighbouring pieces of a row
  RowPiece<XT> raw[PIECES];
  const int row_log = a.chunk + 4, in_chunk = cs * 16;
  auto load = [&](int ch) {
    const int tid = afresh(threadIdx.x);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      if ((i * T) >> row_log >= rows) break;
      const int p = i * T + tid, m = p >> row_log, q = p & ((1 << row_log) - 1), k = (step0 + ch * cs) * 128 + q * 8;
#pragma unroll
      for (int e = 0; e < (XT == kRowsF32 ? 2 : 1); ++e) raw[i].v[e] = make_uint4(0u, 0u, 0u, 0u);
      raw[i].scale = 127;
      if (m >= rows || q >= in_chunk || k >= a.k) continue;
      const char* x = (const char*)a.x + ((int64_t)(m0 + m) * a.x_row + k) * ES;
      if (XT == kRowsF8) {
        raw[i].scale = a.x_scale[(int64_t)(m0 + m) * groups + k / G];
        if (a.x_vec) {
          const uint2 v = *(const uint2*)x;
          raw[i].v[0].x = v.x;
          raw[i].v[0].y = v.y;
        } else {
          const uint8_t* b = (const uint8_t*)x;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            raw[i].v[0].x |= (uint32_t)b[e] << (8 * e);
            raw[i].v[0].y |= (uint32_t)b[e + 4] << (8 * e);
          }
        }
      } else if (XT == kRowsBf16) {
        const uint16_t* h = (const uint16_t*)x;
        if (a.x_vec) raw[i].v[0] = *(const uint4*)x;
        else raw[i].v[0] = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
      } else {
        const uint32_t* f = (const uint32_t*)x;
#pragma unroll
        for (int e = 0; e < 2; ++e) raw[i].v[XT == kRowsF32 ? e : 0] = a.x_vec ? *(const uint4*)(f + 4 * e) : make_uint4(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3]);
      }
    }
  };
  auto stage = [&](int buf) {
    const Lds frag = lds + buf * x_size;
    const int tid = afresh(threadIdx.x);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      if ((i * T) >> row_log >= rows) break;
      const int p = i * T + tid, m = p >> row_log, q = p & ((1 << row_log) - 1), in_step = (q & 15) * 8;
      if (XT == kRowsF32) __builtin_amdgcn_sched_barrier(0);  // (piece by piece, or their parts do not fit the registers)
      uint4 high, low = make_uint4(0u, 0u, 0u, 0u);
      float back = 1.f, begin = 0.f;
      if (XT == kRowsBf16) {
        high = in_order(raw[i].v[0]);
      } else if (XT == kRowsF8) {
        const f16x8 h = __builtin_bit_cast(f16x8, in_order(__builtin_bit_cast(uint4, f16_of_codes(raw[i].v[0].x, raw[i].v[0].y, 16.f))));
#pragma unroll
        for (int e = 0; e < 8; ++e) begin += (float)h[e];
        high = __builtin_bit_cast(uint4, h);
        back = two_to(raw[i].scale - 127);
      } else {
        float v[8], rest[8];
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint4& r = raw[i].v[XT == kRowsF32 ? e >> 2 : 0];
          v[e] = __uint_as_float((e & 3) == 0 ? r.x : (e & 3) == 1 ? r.y : (e & 3) == 2 ? r.z : r.w);
          most = fmaxf(most, fabsf(v[e]));
        }
        most = wave_max<G / 8>(most);
        // to 2^14 and more, but no further than 2^110 times: what is smaller than 2^-96 loses bits
        int up = 141 - (int)(__float_as_uint(most) >> 23);
        up = up > 110 ? 110 : up;
        back = two_to(4 - up);  // (for (c - 8) / 16)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = __builtin_amdgcn_ldexpf(v[e], up);
          begin += v[e];
        }
        const f16x8 h = f16_in_order(v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          rest[e] = v[e] - (float)h[2 * e];
          rest[e + 4] = v[e + 4] - (float)h[2 * e + 1];
        }
        high = __builtin_bit_cast(uint4, h);
        low = __builtin_bit_cast(uint4, f16_in_order(rest));
      }
      if (XT != kRowsBf16) begin = wave_sum<G / 8>(begin) * -1.5f;
      if (m < rows && q < in_chunk) {
        const Lds to = frag + (((q >> 4) * rows + m) * 16 + (place<G>(in_step) ^ (m & 15))) * 16;
        *(u32x4 __attribute__((address_space(3)))*)to = __builtin_bit_cast(u32x4, high);
        if (PARTS == 2) *(u32x4 __attribute__((address_space(3)))*)(to + part_size) = __builtin_bit_cast(u32x4, low);
        if (XT != kRowsBf16 && (in_step & (G - 1)) == 0) {
          float __attribute__((address_space(3)))* const s = (float __attribute__((address_space(3)))*)(frag + PARTS * part_size) + (((q >> 4) * fours + (m >> 2)) * GS + in_step / G) * 8 + (m & 3);
          s[0] = back;
          s[4] = begin;
        }
      }
    }
  };

  f32x4 total = {0.f, 0.f, 0.f, 0.f};
  const Spread<XT> spread;

  // The outputs of a group of tiles, from the waves' sums or, where K is shared, from what the workgroups left.
  const int wide = a.across + 4;  // log2 of the outputs side by side
  auto of_waves = [&](int i) {
    const int m = i >> wide, o = i & ((1 << wide) - 1);
    const float __attribute__((address_space(3)))* r = red + (((o >> 4) << split_log) * ROWS + m) * 16 + (o & 15);
    float s = 0.f;
#pragma unroll 4
    for (int p = 0; p < 1 << split_log; ++p) s += r[p * ROWS * 16];
    return s;
  };
  auto write = [&](int tg, const float* left) {
    for (int i = afresh(threadIdx.x); i < rows << wide; i += T) {
      const int m = i >> wide;
      int out = (tg << wide) + (i & ((1 << wide) - 1));
      float s = 0.f;
      if (left) {
#pragma unroll 8
        for (int p = 0; p < a.shares; ++p) s += take_back1(left + (int64_t)p * (ROWS << wide) + i);  // (in order, whoever came last)
      } else {
        s = of_waves(i);
      }
      bool on = out < a.n;
      if (a.gate) {  // neighbouring lanes hold a pair (a row of the group is an even number of outputs, so pairs never part)
        float other, own;
        lane_pair<1>(s, &own, &other);
        s = s / (1.f + expf(-s)) * other;
        on = on && !(out & 1);
        out >>= 1;
      }
      if (!on) continue;
      const int64_t at = (int64_t)(m0 + m) * a.y_row + out;
      if (BF16_OUT) ((uint16_t*)a.y)[at] = (uint16_t)f32_to_bf16_bits(s);
      else ((float*)a.y)[at] = s;
    }
  };

  int ch = 0, buf = 0, last = -1;
  List now = list(tg, 0);
#pragma unroll
  for (int i = 0; i < RING; ++i) fetch(i, now, i);
  load(0);
  load_scales(tg, 0);
  stage(0);
  stage_scales(0);
  for (;;) {
    __syncthreads();
    if (ch == 0 && last >= 0) write(last, nullptr);
    const bool over = ch + 1 == chunks;
    const int next_ch = over ? 0 : ch + 1, next = over ? tg + a.wgs : tg;
    const bool more = next < a.groups;
    List after = now;
    after.n = 0;
    if (more) {
      after = list(next, next_ch);
      load_scales(next, next_ch);
    }
    const int x_at = chunks > 1 ? buf * x_size : 0;
    const int xr = c < rows ? c : rows - 1;
    int f = x_at + ((first * rows + xr) * 16 + (g ^ xr)) * 16;  // where the wave's operands of its next step lie
    Lds xs = lds + x_at + PARTS * part_size + (first * fours + (g < fours ? g : fours - 1)) * GS * 32;  // (rows that are none: any numbers will do)
    Lds ws = lds + ws_at + buf * ws_size + (own_tile * 16 + c) * pitch + first * GS * 2;
#pragma unroll 1
    for (int i0 = 0; i0 < turns; i0 += RING, ws += RING * GS * 2) {
      const bool same = i0 + RING < turns;
      const List ahead = same ? now : after;
      const int from = same ? i0 + RING : 0;
#pragma unroll
      for (int e = 0; e < RING; ++e) {
        const u32x4 mine = ring[e];
        fetch(e, ahead, from + e);
        if (i0 + e >= now.n) continue;
        const uint4 own_w = arranged<G>(__builtin_bit_cast(uint4, mine));
        const uint4 b[4] = {spread(own_w.x), spread(own_w.y), spread(own_w.z), spread(own_w.w)};
        u32x4 x[PARTS][4];
        auto operand = [&](int j) {
          const Lds at = lds + (f ^ (j * 64));
          x[0][j] = *(const u32x4 __attribute__((address_space(3)))*)at;
          if (PARTS == 2) x[PARTS - 1][j] = *(const u32x4 __attribute__((address_space(3)))*)(at + part_size);
        };
        if (PARTS == 1) {  // (both parts of all four do not fit sixteen waves' registers)
#pragma unroll
          for (int j = 0; j < 4; ++j) operand(j);
        }
#pragma unroll
        for (int u = 0; u < GS; ++u) {
          const Lds of_x = xs + u * 32;
          f32x4 sum = {0.f, 0.f, 0.f, 0.f};
          if (XT != kRowsBf16) sum = *(const f32x4 __attribute__((address_space(3)))*)(of_x + 16);
          f32x4 less = {0.f, 0.f, 0.f, 0.f};  // two chains: an instruction waits for the one it adds to
#pragma unroll
          for (int j = u * (4 / GS); j < (u + 1) * (4 / GS); ++j) {
            if (PARTS == 2) operand(j);
            if (XT == kRowsBf16) {
              sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[0][j]), __builtin_bit_cast(bf16x8, b[j]), sum, 0, 0, 0);
              less = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[0][j]), __builtin_bit_cast(bf16x8, spread.minus), less, 0, 0, 0);
            } else {
              sum = mfma16(__builtin_bit_cast(f16x8, x[0][j]), __builtin_bit_cast(f16x8, b[j]), sum);
              if (PARTS == 2) less = mfma16(__builtin_bit_cast(f16x8, x[PARTS - 1][j]), __builtin_bit_cast(f16x8, b[j]), less);
            }
          }
          if (XT == kRowsBf16 || PARTS == 2) {
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[q] += less[q];
          }
          const float by = bf16_bits_to_f32(*(const uint16_t __attribute__((address_space(3)))*)(ws + (e * GS + u) * 2));
          f32x4 x4 = {1.f, 1.f, 1.f, 1.f};
          if (XT != kRowsBf16) x4 = *(const f32x4 __attribute__((address_space(3)))*)of_x;
#pragma unroll
          for (int q = 0; q < 4; ++q) total[q] = fmaf(sum[q], by * x4[q], total[q]);
        }
        f += rows * 256;
        xs += fours * GS * 32;
      }
    }
    if (over) {
      if (last >= 0 && chunks == 1) __syncthreads();  // (the group before has been written; with chunks a barrier lies between)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[(wave * ROWS + g * 4 + i) * 16 + c] = XT == kRowsBf16 ? total[i] * 32768.f : total[i];
      total = f32x4{0.f, 0.f, 0.f, 0.f};
      last = tg;
    }
    if (!more) break;
    buf ^= 1;
    if (chunks > 1) {
      load(next_ch);
      stage(buf);
    }
    stage_scales(buf);
    tg = next;
    ch = next_ch;
    now = after;
  }
  __syncthreads();
  const float* left = nullptr;
  if (a.shares > 1) {
    float* all = a.part + (int64_t)unit * a.shares * (ROWS << wide);
    for (int i = threadIdx.x; i < rows << wide; i += T) put(all + share * (ROWS << wide) + i, of_waves(i));
    if (!arrive(a.count + unit, a.shares, (int*)smem, threadIdx.x)) return;
    left = all;
  }
  write(last, left);
}

}  // namespace daris
