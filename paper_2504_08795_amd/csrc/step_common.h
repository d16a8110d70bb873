// Device helpers that the operators of a generation step share: e4m3 numbers under power-of-two scales, f16 operands of the matrix
// instructions, and where a step's rows belong.
#pragma once
#include "device_common.h"
#include "step_args.h"

namespace daris {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma16(const f16x8& a, const f16x8& b, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(const f16x8& a, const f16x8& b, const f32x16& c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ f16x8 halves(f16x2 a, f16x2 b, f16x2 c, f16x2 d) {
  f16x8 v;
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1]; v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
  return v;
}

// Eight e4m3 codes as f16, which holds every one of them.
__device__ __forceinline__ f16x8 f16_of_codes(uint32_t lo, uint32_t hi, float times = 1.0f) {
  return halves(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, times, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, times, true),
                __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, times, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, times, true));
}

__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u; }
// |x| for the largest of a group: what is not finite has no part in it.
__device__ __forceinline__ float size_of(float x) { return is_finite(x) ? fabsf(x) : 0.f; }

// Exponent byte of the smallest power of two s, 2^-100 at least, with most <= 448 s.  448 = 1.75 * 2^8: a mantissa above .75 carries.
constexpr int kLeastScale = 27;
__device__ __forceinline__ int scale_byte(float most) {
  const int e = (int)((__float_as_uint(most) + 0x1fffffu) >> 23) - 8;
  return e < kLeastScale ? kLeastScale : e;
}
__device__ __forceinline__ float two_to(int e) { return __builtin_amdgcn_ldexpf(1.0f, e); }

// x (already divided by its scale) as e4m3 codes, round to nearest even; what is not finite becomes the NaN code.
__device__ __forceinline__ float code_input(float x) { return is_finite(x) ? x : __uint_as_float(0x7fc00000u); }
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(code_input(a), code_input(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(code_input(c), code_input(d), r, true);
}

// v of this lane and of the lane whose number differs by M (in either order).
template <int M>
__device__ __forceinline__ void lane_pair(float v, float* a, float* b) {
  static_assert(M == 1 || M == 2 || M == 4 || M == 8 || M == 16 || M == 32, "a bit of the lane's number");
  const int x = __builtin_bit_cast(int, v);
  if constexpr (M == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    *a = __builtin_bit_cast(float, (int)r[0]);
    *b = __builtin_bit_cast(float, (int)r[1]);
  } else if constexpr (M == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    *a = __builtin_bit_cast(float, (int)r[0]);
    *b = __builtin_bit_cast(float, (int)r[1]);
  } else {
    *a = v;
    *b = __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(x, (M << 10) | 0x1f));
  }
}
// ... over lanes whose numbers differ in the bits FROM .. TO / 2: the result in all of them
template <int FROM, int TO>
__device__ __forceinline__ float lanes_max(float v) {
  if constexpr (FROM < TO) {
    float a, b;
    lane_pair<FROM>(v, &a, &b);
    return lanes_max<FROM * 2, TO>(fmaxf(a, b));
  }
  return v;
}
template <int FROM, int TO>
__device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (FROM < TO) {
    float a, b;
    lane_pair<FROM>(v, &a, &b);
    return lanes_sum<FROM * 2, TO>(a + b);
  }
  return v;
}
template <int N>
__device__ __forceinline__ float wave_max(float v) { return lanes_max<1, N>(v); }  // over N neighbouring lanes
template <int N>
__device__ __forceinline__ float wave_sum(float v) { return lanes_sum<1, N>(v); }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// ---- workgroups that share a result ----------------------------------------------------------------------------------------

// Whether this workgroup is the last of `all` that arrive at *count (which is 0 before and after).  What they leave for each other is written
// through to where all XCDs see it (put, leave2) and read from there (take_back), so neither side needs a fence: a release or an acquire of the
// device writes back or drops a whole L2, and with one for every workgroup attention for 64 streams took 300 us instead of 88.
__device__ __forceinline__ bool arrive(uint32_t* count, int all, int* lds, int tid) {
  puts_done();
  __syncthreads();
  if (tid == 0) {
    const uint32_t before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const bool last = before == (uint32_t)all - 1;
    if (last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *lds = last;
  }
  __syncthreads();
  return *lds != 0;
}
__device__ __forceinline__ float4 take_back(const float* p) {
  return __builtin_bit_cast(float4, __builtin_amdgcn_global_load_b128((u32x4 __attribute__((address_space(1)))*)p, "agent"));
}
__device__ __forceinline__ float2 take_back2(const float* p) {
  return __builtin_bit_cast(float2, __hip_atomic_load((const uint64_t __attribute__((address_space(1)))*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ float take_back1(const float* p) {
  return __hip_atomic_load((const float __attribute__((address_space(1)))*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void leave2(float* p, float x, float y) { put((void*)p, make_uint2(__float_as_uint(x), __float_as_uint(y))); }

// ---- where rows belong ---------------------------------------------------------------------------------------------------

// First row of sequence s (s <= n_seqs); whatever the caller's numbers are, one of the buffers' rows.
__device__ __forceinline__ int first_row(const CacheArgs& c, int s) {
  if (!c.row_start) return s < c.n_rows ? s : c.n_rows;
  const int r = c.row_start[s];
  return r < 0 ? 0 : r > c.n_rows ? c.n_rows : r;
}
__device__ __forceinline__ int rows_of(const CacheArgs& c, int s) {
  const int n = first_row(c, s + 1) - first_row(c, s);
  return n < 0 ? 0 : n;
}
// Tokens in front of the step's, kept away from what would overflow when rows are added.
__device__ __forceinline__ int tokens_before(const CacheArgs& c, int s) {
  const int b = c.before[s];
  return b < -(1 << 30) ? -(1 << 30) : b > (1 << 30) ? (1 << 30) : b;
}
// Page of token t >= 0 of sequence s, or -1.
__device__ __forceinline__ int page_of(const CacheArgs& c, int s, int page) {
  if (page >= c.pages_row) return -1;
  const int p = c.pages[(int64_t)s * c.pages_row + page];
  return p < 0 || p >= c.n_pages ? -1 : p;
}

}  // namespace daris
