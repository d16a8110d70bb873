// Products of a few rows with 4-bit weights and a scale for each group of channels.
//
// y^T is computed in tiles of 16 outputs: a wave reads 16 rows of weights, 128 channels (a step) at a time, 16 bytes a lane straight
// into registers, spreads the nibbles and multiplies them with the rows of x on the matrix instructions.  A group's sum is
// taken by them alone and multiplied by the weights' scale once, in fp32.  x lies in LDS in the order of the nibbles.
//   bf16 x: as it is.  0x4300 | c is the bf16 number 128 + c; a second product with the constant -136 takes the rest away in the same
//     accumulator.  Sums are 17 times as large as the result on the way, which costs four of fp32's 24 bits.
//   fp32 x: two f16 parts (22 bits), a group of a row divided by a power of two that makes its largest number 2^14 and more, so that
//     nothing overflows; 0x6400 | c is the f16 number 1024 + c, one packed addition makes it c - 8.
//   e4m3 x: f16 holds every one of them.
// The waves of a workgroup share x, and neighbouring ones a tile: each takes neighbouring steps of it, and their sums are added in
// wave order.  A workgroup goes from group of tiles to group of tiles; x is staged once if all of K fits LDS, else in chunks,
// the next one while the present one is computed, as are the weights' scales.  Every wave has four steps of weights on their way, across
// chunks and tiles.  Bound by the bytes of the weights while there are few rows.
#pragma once
#include "step_common.h"

namespace daris {

enum { kRowsF32 = 0, kRowsBf16 = 1, kRowsF8 = 2 };

// Eight nibbles as f16 in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ f16x8 f16_of_nibbles(uint32_t w) {
  const f16x2 minus = {(_Float16)-1032.0f, (_Float16)-1032.0f};
  f16x2 p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = __builtin_bit_cast(f16x2, ((w >> (4 * i)) & 0x000f000fu) | 0x64006400u) + minus;
  return halves(p[0], p[1], p[2], p[3]);
}

// ... plus 128 as bf16.
__device__ __forceinline__ bf16x8 bf16_of_nibbles(uint32_t w) {
  const uint4 v = make_uint4((w & 0x000f000fu) | 0x43004300u, ((w >> 4) & 0x000f000fu) | 0x43004300u, ((w >> 8) & 0x000f000fu) | 0x43004300u, ((w >> 12) & 0x000f000fu) | 0x43004300u);
  return __builtin_bit_cast(bf16x8, v);
}

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

template <int XT, int G, int MT, bool BF16_OUT>
__device__ __forceinline__ void matvec_body(const MatvecArgs& a) {
  constexpr int PARTS = XT == kRowsF32 ? 2 : 1, GS = 128 / G, ROWS = 16 * MT, WAVES = matvec_waves(MT), T = WAVES * 64;
  constexpr int PIECES = matvec_pieces(PARTS), RING = 4;
  constexpr bool AHEAD = MT > 1;  // a chunk of x travels while the one before is computed (sixteen waves have no registers for that)
  extern __shared__ uint4 smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, c = lane & 15;
  const int across = a.across, split = WAVES / across;  // tiles side by side, waves on one of them
  const int mb = blockIdx.x / a.wgs, m0 = mb * ROWS, rows = a.rows - m0 < ROWS ? a.rows - m0 : ROWS;
  const int own_tile = wave / split, part = wave - own_tile * split;
  const int groups = a.k / G, steps = (a.k + 127) / 128, cs = a.steps, chunks = (steps + cs - 1) / cs;
  // LDS: x [PARTS][step][row][instruction, lane group], the last exchanged by the row's number so that rows lie on different banks, and (of scaled rows) their scales [step][group][ROWS], twice if there is more than
  // one chunk; the weights' scales [across * 16][pitch] twice if there is more to come; sums [WAVES][ROWS][16]
  const int pieces = cs * 16 * rows, x_size = PARTS * pieces + (XT == kRowsBf16 ? 0 : cs * GS * ROWS / 4), pitch = matvec_pitch(cs * GS);
  uint16_t* const ws_lds = (uint16_t*)(smem + (chunks > 1 ? 2 : 1) * x_size);
  const int ws_size = across * 16 * pitch;
  const bool again = chunks > 1 || a.wgs < a.groups;
  float* const red = (float*)(ws_lds + (again ? 2 : 1) * ws_size);

  // ---- weights: the wave's steps of a chunk are neighbouring ones, so that it reads whole cache lines
  const int own = (cs + split - 1) / split, first = part * own, turns = (own + RING - 1) / RING * RING;
  uint4 ring[RING];
  auto fetch = [&](int slot, int tg, int ch, int i) {
    const int st = first + i, k = (ch * cs + st) * 128 + g * 32;
    const int n = (tg * across + own_tile) * 16 + c;
    ring[slot] = make_uint4(0u, 0u, 0u, 0u);
    if (tg < a.groups && i < own && st < cs && k < a.k) ring[slot] = *(const uint4*)(a.w + (int64_t)(n < a.n ? n : a.n - 1) * a.w_row + k / 2);
  };
  // ---- and their scales, eight neighbours a thread
  uint32_t sc[kScalePieces][4];
  const int eights = (cs * GS + 7) / 8;
  auto load_scales = [&](int tg, int ch) {
    const int tid = afresh(threadIdx.x);
#pragma unroll
    for (int i = 0; i < kScalePieces; ++i) {
      const int p = i * T + tid, r = p / eights, at = (p - r * eights) * 8, from = ch * cs * GS + at;
      if (r >= across * 16 || from >= groups) continue;
      const int n = tg * across * 16 + r;
      const uint16_t* s = a.w_scale + (int64_t)(n < a.n ? n : a.n - 1) * groups + from;
      if (from + 8 <= groups) {
        __builtin_memcpy(sc[i], s, 16);
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
      const int p = i * T + tid, r = p / eights, at = (p - r * eights) * 8;
      if (r >= across * 16) continue;
      uint32_t* to = (uint32_t*)(ws_lds + buf * ws_size + r * pitch + at);  // (the pitch is an odd number of words)
#pragma unroll
      for (int e = 0; e < 4; ++e) to[e] = sc[i][e];
    }
  };

  // ---- rows of x: neighbouring threads take neighbouring pieces of a row
  RowPiece<XT> raw[PIECES];
  auto load = [&](int ch) {
    const int tid = afresh(threadIdx.x);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int p = i * T + tid, m = p >> (a.chunk + 4), q = p & ((16 << a.chunk) - 1), k = ch * cs * 128 + q * 8;
#pragma unroll
      for (int e = 0; e < (XT == kRowsF32 ? 2 : 1); ++e) raw[i].v[e] = make_uint4(0u, 0u, 0u, 0u);
      raw[i].scale = 127;
      if (m >= rows || q >= cs * 16 || k >= a.k) continue;
      const int64_t at = (int64_t)(m0 + m) * a.x_row + k;
      if (XT == kRowsF8) {
        raw[i].scale = a.x_scale[(int64_t)(m0 + m) * groups + k / G];
        const uint8_t* x = (const uint8_t*)a.x + at;
        if (a.x_vec) {
          const uint2 v = *(const uint2*)x;
          raw[i].v[0].x = v.x;
          raw[i].v[0].y = v.y;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            raw[i].v[0].x |= (uint32_t)x[e] << (8 * e);
            raw[i].v[0].y |= (uint32_t)x[e + 4] << (8 * e);
          }
        }
      } else if (XT == kRowsBf16) {
        const uint16_t* x = (const uint16_t*)a.x + at;
        if (a.x_vec) raw[i].v[0] = *(const uint4*)x;
        else raw[i].v[0] = make_uint4(x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16, x[4] | (uint32_t)x[5] << 16, x[6] | (uint32_t)x[7] << 16);
      } else {
        const uint32_t* x = (const uint32_t*)a.x + at;
#pragma unroll
        for (int e = 0; e < 2; ++e) raw[i].v[XT == kRowsF32 ? e : 0] = a.x_vec ? *(const uint4*)(x + 4 * e) : make_uint4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
      }
    }
  };
  auto stage = [&](int buf) {
    uint4* frag = smem + buf * x_size;
    float* xs = (float*)(frag + PARTS * pieces);
    const int tid = afresh(threadIdx.x);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int p = i * T + tid, m = p >> (a.chunk + 4), q = p & ((16 << a.chunk) - 1), in_step = (q & 15) * 8;
      if ((i * T) >> (a.chunk + 4) >= rows) break;
      if (XT == kRowsF32) __builtin_amdgcn_sched_barrier(0);  // (piece by piece, or their parts do not fit the registers)
      const int to = ((q >> 4) * rows + m) * 16 + (place<G>(in_step) ^ (m & 15));
      uint4 high, low = make_uint4(0u, 0u, 0u, 0u);
      float back = 1.f;
      if (XT == kRowsBf16) {
        high = in_order(raw[i].v[0]);
      } else if (XT == kRowsF8) {
        high = in_order(__builtin_bit_cast(uint4, f16_of_codes(raw[i].v[0].x, raw[i].v[0].y)));
        back = two_to(raw[i].scale - 127);
      } else {
        float v[8], rest[8];
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint4& r = raw[i].v[XT == kRowsF32 ? e >> 2 : 0];
          v[e] = __uint_as_float((e & 3) == 0 ? r.x : (e & 3) == 1 ? r.y : (e & 3) == 2 ? r.z : r.w);
          most = fmaxf(most, size_of(v[e]));
        }
        most = wave_max<G / 8>(most);
        // to 2^14 and more, but no further than 2^110 times: what is smaller than 2^-96 loses bits
        int up = 141 - (int)(__float_as_uint(most) >> 23);
        up = up > 110 ? 110 : up;
        back = two_to(-up);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __builtin_amdgcn_ldexpf(v[e], up);
        const f16x8 h = f16_in_order(v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          rest[e] = is_finite(v[e]) ? v[e] - (float)h[2 * e] : 0.f;
          rest[e + 4] = is_finite(v[e + 4]) ? v[e + 4] - (float)h[2 * e + 1] : 0.f;
        }
        high = __builtin_bit_cast(uint4, h);
        low = __builtin_bit_cast(uint4, f16_in_order(rest));
      }
      if (m < rows && q < cs * 16) {
        frag[to] = high;
        if (PARTS == 2) frag[pieces + to] = low;
        if (XT != kRowsBf16 && (in_step & (G - 1)) == 0) xs[((q >> 4) * GS + in_step / G) * ROWS + m] = back;
      }
    }
  };

  f32x4 total[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) total[m] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bf16x8 minus = __builtin_bit_cast(bf16x8, make_uint4(0xc308c308u, 0xc308c308u, 0xc308c308u, 0xc308c308u));  // -136

  // the outputs of a group of tiles from the waves' sums
  auto write = [&](int tg) {
    for (int i = afresh(threadIdx.x); i < rows * across * 16; i += T) {
      const int m = i / (across * 16), o = i - m * across * 16, t = o >> 4, col = o & 15;
      float s = 0.f;
      for (int p = 0; p < split; ++p) s += red[((t * split + p) * ROWS + m) * 16 + col];
      int out = tg * across * 16 + o;
      bool on = out < a.n;
      if (a.gate) {
        // neighbouring lanes hold a pair: a row of the group is an even number of outputs, so pairs never part
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

  int tg = blockIdx.x - mb * a.wgs, ch = 0, buf = 0, last = -1;
  load(0);
  load_scales(tg, 0);
#pragma unroll
  for (int i = 0; i < RING; ++i) fetch(i, tg, 0, i);
  stage(0);
  stage_scales(0);
  for (;;) {
    __syncthreads();
    if (ch == 0 && last >= 0) write(last);
    const bool over = ch + 1 == chunks;
    const int next_ch = over ? 0 : ch + 1, next = over ? tg + a.wgs : tg;
    const bool more = next < a.groups;
    if (more) {
      if (AHEAD && chunks > 1) load(next_ch);
      load_scales(next, next_ch);
    }
    const uint4* frag = smem + (chunks > 1 ? buf * x_size : 0);
    const float* xs = (const float*)(frag + PARTS * pieces);
    const uint16_t* ws = ws_lds + buf * ws_size + (own_tile * 16 + c) * pitch;
#pragma unroll 1
    for (int i0 = 0; i0 < turns; i0 += RING) {
#pragma unroll
      for (int e = 0; e < RING; ++e) {
        const int i = i0 + e, st = first + i;  // of the chunk
        const uint4 now = arranged<G>(ring[e]);
        if (i + RING < turns) fetch(e, tg, ch, i + RING);
        else fetch(e, next, next_ch, i + RING - turns);
        if (i >= own || st >= cs || ch * cs + st >= steps) continue;
        const uint32_t wd[4] = {now.x, now.y, now.z, now.w};
        uint4 b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = XT == kRowsBf16 ? __builtin_bit_cast(uint4, bf16_of_nibbles(wd[j])) : __builtin_bit_cast(uint4, f16_of_nibbles(wd[j]));
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const int xr = m * 16 + c < rows ? m * 16 + c : rows - 1;
          const int f = (st * rows + xr) * 16 + (g ^ (xr & 15));
#pragma unroll
          for (int u = 0; u < GS; ++u) {
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = u * (4 / GS); j < (u + 1) * (4 / GS); ++j) {
              const uint4 x = frag[f ^ (j * 4)];
              if (XT == kRowsBf16) {
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, b[j]), sum, 0, 0, 0);
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), minus, sum, 0, 0, 0);
              } else {
                if (PARTS == 2) sum = mfma16(__builtin_bit_cast(f16x8, frag[pieces + (f ^ (j * 4))]), __builtin_bit_cast(f16x8, b[j]), sum);
                sum = mfma16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, b[j]), sum);
              }
            }
            const float by = bf16_bits_to_f32(ws[st * GS + u]);
            float4 x4 = make_float4(1.f, 1.f, 1.f, 1.f);
            if (XT != kRowsBf16) x4 = *(const float4*)(xs + (st * GS + u) * ROWS + m * 16 + g * 4);
            total[m][0] = fmaf(sum[0], by * x4.x, total[m][0]);
            total[m][1] = fmaf(sum[1], by * x4.y, total[m][1]);
            total[m][2] = fmaf(sum[2], by * x4.z, total[m][2]);
            total[m][3] = fmaf(sum[3], by * x4.w, total[m][3]);
          }
        }
      }
    }
    if (over) {
      if (last >= 0 && chunks == 1) __syncthreads();  // (the group before has been written; with chunks a barrier lies between)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int i = 0; i < 4; ++i) red[(wave * ROWS + m * 16 + g * 4 + i) * 16 + c] = total[m][i];
        total[m] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      last = tg;
    }
    if (!more) break;
    buf ^= 1;
    if (!AHEAD && chunks > 1) load(next_ch);
    if (chunks > 1) stage(buf);
    stage_scales(buf);
    tg = next;
    ch = next_ch;
  }
  __syncthreads();
  write(last);
}

}  // namespace daris
