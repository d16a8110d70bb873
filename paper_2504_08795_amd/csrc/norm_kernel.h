// Root-mean-square norm of a row with the residual's addition in front and, if wanted, e4m3 codes behind.
//
// One workgroup a row, one pass over memory: the row stays in registers (NV 16-byte vectors a thread) between the sum of its
// squares and its outputs, and the weights arrive while the sum is taken.  Rows beyond that are read twice (NV = 0).  Nothing is
// computed that memory would wait for: bound by bandwidth for many rows and by latency for one.  8192 rows of 4096 (bf16, residual, codes):
// 235 MB in 38 us with what the last-level cache holds of them, 47 us without (5.0 TB/s; a large copy reaches 5.1); one row 3.3 us.  Rows that are not aligned to 16
// bytes travel element by element and take two to three times as long (8192 rows, fp32, us a call: 4096 wide 56, 4095 wide 114; bf16 with residual, 4095 wide, 184).
#pragma once
#include "step_common.h"

namespace daris {

// VEC elements from e on as floats; what lies past the row is 0.
template <bool BF16, bool ALIGNED>
__device__ __forceinline__ void row_vector(const void* p, int64_t e, int left, float* o) {
  constexpr int VEC = BF16 ? 8 : 4;
  if (ALIGNED) {
    const uint4 v = BF16 ? *(const uint4*)((const uint16_t*)p + e) : *(const uint4*)((const float*)p + e);
    unpack<BF16>(v, o);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) o[i] = i < left ? load_elem<BF16>(p, e + i) : 0.f;
  }
}
template <bool BF16, bool ALIGNED>
__device__ __forceinline__ void put_vector(void* p, int64_t e, int left, const float* o) {
  constexpr int VEC = BF16 ? 8 : 4;
  if (ALIGNED) {
    *(uint4*)(BF16 ? (void*)((uint16_t*)p + e) : (void*)((float*)p + e)) = pack<BF16>(o);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (i < left) {
        if (BF16) ((uint16_t*)p)[e + i] = (uint16_t)f32_to_bf16_bits(o[i]);
        else ((float*)p)[e + i] = o[i];
      }
  }
}

template <int T>
__device__ __forceinline__ float block_sum(float v, float* lds) {
  v = wave_sum<64>(v);
  if (T == 64) return v;
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) s += lds[i];
  return s;
}

// One vector's outputs: codes and scale, or dtype.
template <bool BF16, bool F8, bool ALIGNED>
__device__ __forceinline__ void norm_out(const NormArgs& a, int row, int vec, bool on, float (&h)[BF16 ? 8 : 4], const float* w, float r) {
  constexpr int VEC = BF16 ? 8 : 4;
  const int e = vec * VEC, left = on ? a.width - e : 0;
#pragma unroll
  for (int i = 0; i < VEC; ++i) h[i] = h[i] * r * w[i];
  if (!F8) {
    if (on) put_vector<BF16, ALIGNED>(a.y, row * a.y_row + e, left, h);
    return;
  }
  // (every lane takes part in the exchange; a group's vectors are all there or none of them is)
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < VEC; ++i) most = fmaxf(most, size_of(h[i]));
  const int lanes = a.group / VEC;
  for (int m = 1; m < lanes; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
  const int byte = scale_byte(most);
  const float inv = two_to(127 - byte);
#pragma unroll
  for (int i = 0; i < VEC; ++i) h[i] *= inv;
  if (!on) return;
  uint32_t* y = (uint32_t*)((uint8_t*)a.y + row * a.y_row + e);
  const uint32_t lo = codes4(h[0], h[1], h[2], h[3]), hi = BF16 ? codes4(h[VEC - 4], h[VEC - 3], h[VEC - 2], h[VEC - 1]) : 0u;
  if (ALIGNED) {
    if (BF16) *(uint2*)y = make_uint2(lo, hi);
    else *y = lo;
  } else {
    uint8_t* b = (uint8_t*)y;
#pragma unroll
    for (int i = 0; i < VEC; ++i) b[i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
  }
  if ((vec & (lanes - 1)) == 0) a.scale[(int64_t)row * (a.width / a.group) + vec / lanes] = (uint8_t)byte;
}

template <bool BF16, bool F8, bool ALIGNED, int NV, int T>
__device__ __forceinline__ void norm_body(const NormArgs& a) {
  constexpr int VEC = BF16 ? 8 : 4;
  __shared__ float lds[16];
  const int row = blockIdx.x, tid = threadIdx.x;
  const int64_t x0 = row * a.x_row, r0 = row * a.res_row, s0 = row * a.sum_row;
  if constexpr (NV > 0) {
    float h[NV][VEC], w[NV][VEC];
    float sq = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int vec = tid + j * T, e = vec * VEC, left = a.width - e;
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[j][i] = w[j][i] = 0.f;
      if (vec < a.vectors) {
        row_vector<BF16, ALIGNED>(a.x, x0 + e, left, h[j]);
        row_vector<BF16, ALIGNED>(a.weight, e, left, w[j]);
        if (a.res) {
          float q[VEC];
          row_vector<BF16, ALIGNED>(a.res, r0 + e, left, q);
#pragma unroll
          for (int i = 0; i < VEC; ++i) h[j][i] += q[i];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) sq = fmaf(h[j][i], h[j][i], sq);
    if (a.sum) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int vec = tid + j * T;
        if (vec < a.vectors) put_vector<BF16, ALIGNED>(a.sum, s0 + vec * VEC, a.width - vec * VEC, h[j]);
      }
    }
    const float r = rsqrtf(block_sum<T>(sq, lds) * a.inv_width + a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) norm_out<BF16, F8, ALIGNED>(a, row, tid + j * T, tid + j * T < a.vectors, h[j], w[j], r);
  } else {
    float sq = 0.f;
    for (int vec = tid; vec < a.vectors; vec += T) {
      const int e = vec * VEC, left = a.width - e;
      float h[VEC], q[VEC];
      row_vector<BF16, ALIGNED>(a.x, x0 + e, left, h);
      if (a.res) {
        row_vector<BF16, ALIGNED>(a.res, r0 + e, left, q);
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[i] += q[i];
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) sq = fmaf(h[i], h[i], sq);
    }
    const float r = rsqrtf(block_sum<T>(sq, lds) * a.inv_width + a.eps);
    for (int base = 0; base < a.vectors; base += T) {
      const int vec = base + tid, e = vec * VEC, left = a.width - e;
      const bool on = vec < a.vectors;
      float h[VEC], q[VEC], w[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[i] = w[i] = 0.f;
      if (on) {
        row_vector<BF16, ALIGNED>(a.x, x0 + e, left, h);
        row_vector<BF16, ALIGNED>(a.weight, e, left, w);
        if (a.res) {
          row_vector<BF16, ALIGNED>(a.res, r0 + e, left, q);
#pragma unroll
          for (int i = 0; i < VEC; ++i) h[i] += q[i];
        }
        // (x and res of this vector are read for the last time here, so that sum may lie on either)
        if (a.sum) put_vector<BF16, ALIGNED>(a.sum, s0 + e, left, h);
      }
      norm_out<BF16, F8, ALIGNED>(a, row, vec, on, h, w, r);
    }
  }
}

}  // namespace daris
