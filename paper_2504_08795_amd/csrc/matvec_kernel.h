// Products of a few rows with 4-bit weights and a scale for each group of channels.
//
// y^T is computed in tiles of 16 outputs: a wave reads 16 rows of weights, 128 channels at a time, 16 bytes a lane straight into
// registers, spreads the nibbles into f16 (0x6400 | c is 1024 + c, one packed addition takes 1032 away) and multiplies them
// with the rows of x on v_mfma_f32_16x16x32_f16.  Weights are whole numbers from -8 to 7 and stay exact; a group's sum is taken
// by the matrix instructions alone and multiplied by the weights' scale once, in fp32.  x lies in LDS as f16 in the order of the
// nibbles, each group of a row divided by a power of two that makes its largest number 2^14 and more, so that nothing
// overflows; fp32 rows are two f16 parts (22 bits), e4m3 rows are exact.  The waves of a workgroup share x; they take either
// neighbouring tiles or, where n is short, every so many steps of one tile, whose sums are added in wave order.  Bound by the
// bytes of the weights while a workgroup has few rows.
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

// Where lane group g finds its eight channels for the j-th matrix instruction of a step of 128: all of an instruction's
// channels belong to one group of G, and a lane's pieces of memory are as wide as that allows.
template <int G>
__device__ __forceinline__ constexpr int piece(int j, int g) {
  return G == 128 ? g * 32 + j * 8 : G == 64 ? (j >> 1) * 64 + g * 16 + (j & 1) * 8 : j * 32 + g * 8;
}

// A lane's 32 weights of a step; channels past k count as absent (their x is 0).
template <int G>
__device__ __forceinline__ uint4 step_weights(const uint8_t* row, int k0, int g, int k) {
  uint4 w = make_uint4(0u, 0u, 0u, 0u);
  if (G == 128) {
    w = *(const uint4*)(row + (k0 + g * 32) / 2);
  } else if (G == 64) {
    const uint2 a = *(const uint2*)(row + (k0 + g * 16) / 2);
    w.x = a.x;
    w.y = a.y;
    if (k0 + 64 < k) {
      const uint2 b = *(const uint2*)(row + (k0 + 64 + g * 16) / 2);
      w.z = b.x;
      w.w = b.y;
    }
  } else {
    w.x = *(const uint32_t*)(row + (k0 + g * 8) / 2);
    if (k0 + 32 < k) w.y = *(const uint32_t*)(row + (k0 + 32 + g * 8) / 2);
    if (k0 + 64 < k) w.z = *(const uint32_t*)(row + (k0 + 64 + g * 8) / 2);
    if (k0 + 96 < k) w.w = *(const uint32_t*)(row + (k0 + 96 + g * 8) / 2);
  }
  return w;
}

template <int XT, int G, int MT, bool BF16_OUT>
__device__ __forceinline__ void matvec_body(const MatvecArgs& a) {
  constexpr int PARTS = XT == kRowsF32 ? 2 : 1, GS = 128 / G, AHEAD = 4, ROWS = 16 * MT;
  extern __shared__ uint4 smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, c = lane & 15;
  const int across = a.split & 0xff, split = kMatvecWaves / across;  // tiles side by side, waves on one of them
  const int mb = blockIdx.x / a.tiles, m0 = mb * ROWS, rows = a.rows - m0 < ROWS ? a.rows - m0 : ROWS;
  const int tile = (blockIdx.x - mb * a.tiles) * across + wave / split, part = wave % split;
  const int n = tile * 16 + c, row = n < a.n ? n : a.n - 1;
  const uint8_t* w = a.w + (int64_t)row * a.w_row;
  const int groups = a.k / G;
  const uint16_t* ws = a.w_scale + (int64_t)row * groups;
  const int units = a.chunk / 8;  // pieces of eight channels of a staged row
  uint4* frag = smem;             // [PARTS][units][rows]
  float* xs = (float*)(smem + PARTS * units * rows);  // [chunk / G][ROWS]

  f32x4 total[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) total[m] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int k0 = 0; k0 < a.k; k0 += a.chunk) {
    const int kn = a.k - k0 < a.chunk ? a.k - k0 : a.chunk, steps = (kn + 127) / 128;
    // the first steps' weights travel while x is staged
    uint4 ahead[AHEAD];
    float scale[AHEAD][GS];
    auto fetch = [&](int slot, int st) {
      ahead[slot] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int u = 0; u < GS; ++u) scale[slot][u] = 0.f;
      if (st < steps) {
        const int k = k0 + st * 128;
        ahead[slot] = step_weights<G>(w, k, g, a.k);
#pragma unroll
        for (int u = 0; u < GS; ++u)
          if (k + u * G < a.k) scale[slot][u] = bf16_bits_to_f32(ws[k / G + u]);
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(i, part + i * split);

    if (k0 > 0) __syncthreads();
    const int padded = steps * 16;  // pieces of a row that the steps read
    for (int i = tid; i < padded * rows; i += kMatvecWaves * 64) {
      const int m = i / padded, q = i - m * padded, k = k0 + q * 8;
      const bool in = q * 8 < kn;
      const int64_t at = (int64_t)(m0 + m) * a.x_row + k;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
      float back = 0.f;
      if (XT == kRowsF8) {
        uint32_t lo = 0, hi = 0;
        if (in) {
          const uint8_t* p = (const uint8_t*)a.x + at;
          if (a.x_vec) {
            const uint2 u = *(const uint2*)p;
            lo = u.x;
            hi = u.y;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              lo |= (uint32_t)p[e] << (8 * e);
              hi |= (uint32_t)p[e + 4] << (8 * e);
            }
          }
          back = two_to((int)a.x_scale[(int64_t)(m0 + m) * groups + k / G] - 127);
        }
        const f16x8 h = f16_of_codes(lo, hi);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
      } else {
        if (in) {
          if (a.x_vec) {
            if (XT == kRowsBf16) {
              unpack<true>(*(const uint4*)((const uint16_t*)a.x + at), v);
            } else {
              float lo[4], hi[4];
              unpack<false>(*(const uint4*)((const float*)a.x + at), lo);
              unpack<false>(*(const uint4*)((const float*)a.x + at + 4), hi);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                v[e] = lo[e];
                v[e + 4] = hi[e];
              }
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = load_elem<XT == kRowsBf16>(a.x, at + e);
          }
        }
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, size_of(v[e]));
        most = wave_max<G / 8>(most);
        // to 2^14 and more, but no further than 2^110 times: what is smaller than 2^-96 loses bits
        int up = 141 - (int)(__float_as_uint(most) >> 23);
        up = up > 110 ? 110 : up;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __builtin_amdgcn_ldexpf(v[e], up);
        back = two_to(-up);
      }
      const int st = q >> 4, in_step = (q & 15) * 8;
      // the piece whose first channel this is (the inverse of piece<G>)
      const int j = G == 128 ? (in_step >> 3) & 3 : G == 64 ? (in_step >> 6) * 2 + ((in_step >> 3) & 1) : in_step >> 5;
      const int lg = G == 128 ? in_step >> 5 : G == 64 ? (in_step >> 4) & 3 : (in_step >> 3) & 3;
      const int to = ((st * 4 + j) * 4 + lg) * rows + m;
      f16x8 h = f16_in_order(v);
      frag[to] = __builtin_bit_cast(uint4, h);
      if (PARTS == 2) {
        float rest[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          rest[e] = is_finite(v[e]) ? v[e] - (float)h[2 * e] : 0.f;
          rest[e + 4] = is_finite(v[e + 4]) ? v[e + 4] - (float)h[2 * e + 1] : 0.f;
        }
        frag[units * rows + to] = __builtin_bit_cast(uint4, f16_in_order(rest));
      }
      if ((in_step & (G - 1)) == 0) xs[(st * GS + in_step / G) * ROWS + m] = back;
    }
    __syncthreads();

    for (int st0 = part; st0 < steps; st0 += AHEAD * split) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int st = st0 + i * split;
        if (st >= steps) break;
        const uint32_t wd[4] = {ahead[i].x, ahead[i].y, ahead[i].z, ahead[i].w};
        float sc[GS];
#pragma unroll
        for (int u = 0; u < GS; ++u) sc[u] = scale[i][u];
        fetch(i, st + AHEAD * split);
        f16x8 b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = f16_of_nibbles(wd[j]);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const int xr = m * 16 + c < rows ? m * 16 + c : rows - 1;
          const uint4* f = frag + (st * 16 + g) * rows + xr;
#pragma unroll
          for (int u = 0; u < GS; ++u) {
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = u * (4 / GS); j < (u + 1) * (4 / GS); ++j) {
              if (PARTS == 2) sum = mfma16(__builtin_bit_cast(f16x8, f[units * rows + j * 4 * rows]), b[j], sum);
              sum = mfma16(__builtin_bit_cast(f16x8, f[j * 4 * rows]), b[j], sum);
            }
            const float4 x4 = *(const float4*)(xs + (st * GS + u) * ROWS + m * 16 + g * 4);
            total[m][0] = fmaf(sum[0], sc[u] * x4.x, total[m][0]);
            total[m][1] = fmaf(sum[1], sc[u] * x4.y, total[m][1]);
            total[m][2] = fmaf(sum[2], sc[u] * x4.z, total[m][2]);
            total[m][3] = fmaf(sum[3], sc[u] * x4.w, total[m][3]);
          }
        }
      }
    }
  }

  // the waves' sums, [wave][ROWS][16], added in wave order
  __syncthreads();
  float* red = (float*)smem;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) red[(wave * ROWS + m * 16 + g * 4 + i) * 16 + c] = total[m][i];
  __syncthreads();
  const int first = (blockIdx.x - mb * a.tiles) * across * 16;  // first output of the workgroup
  for (int i = tid; i < rows * across * 16; i += kMatvecWaves * 64) {
    const int m = i / (across * 16), o = i - m * across * 16, t = o >> 4, col = o & 15;
    float s = 0.f;
    for (int p = 0; p < split; ++p) s += red[((t * split + p) * ROWS + m) * 16 + col];
    int out = first + o;
    bool on = out < a.n;
    if (a.gate) {
      // neighbouring lanes hold a pair: across * 16 is even, so pairs never part, and a whole pair is in range or neither
      const float other = __shfl_xor(s, 1);
      s = s / (1.f + expf(-s)) * other;
      on = on && !(out & 1);
      out >>= 1;
    }
    if (!on) continue;
    const int64_t at = (int64_t)(m0 + m) * a.y_row + out;
    if (BF16_OUT) ((uint16_t*)a.y)[at] = (uint16_t)f32_to_bf16_bits(s);
    else ((float*)a.y)[at] = s;
  }
}

}  // namespace daris
