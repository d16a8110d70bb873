// Draws a word for each row of logits: weights exp((x - M) / T) cut to the top_k largest, to the shortest front with top_p of their sum, to those of min_p,
// and the first word, by number, at which the sum of the kept weights passes random x total.
//
// Weights and their sums are held in 64 bits: a word is a whole number, and it changes where a sum passes the random number by a last bit.  Nothing is sorted:
// what is kept is everything above a threshold, (logit, number) of one word.  It is found by a histogram of 4096 equal steps of the exponent (counts, and weights as whole numbers, whose
// sums no order changes), and among the words of the one step that the threshold lies in by comparing each with each, or, where they are
// many (equal logits), by their bits.  A workgroup a row; a row's numbers are read in chunks of 512, a wave each, and chunks whose largest is below what a pass looks for are left out.
#pragma once
#include "step_common.h"

namespace daris {

constexpr int kSampleThreads = kSampleWaves * 64;
constexpr int kSampleChunks = kSampleMost / kSampleChunk;
constexpr float kSampleBits = 64.f;  // a weight below 2^-64 of the largest is nothing

struct SampleLds {
  float top[kSampleChunks];     // a chunk's largest
  double sum[kSampleChunks];    // ... kept weights, or how many of its numbers are the threshold's
  uint32_t count[kSampleSteps];
  uint64_t mass[kSampleSteps];
  uint32_t few_key[kSampleFew];
  int few_at[kSampleFew];
  double wave_d[kSampleWaves];
  uint64_t wave_m[kSampleWaves];
  uint32_t wave_c[kSampleWaves];
  uint64_t found_mass;
  uint32_t found_count, found_key;
  int found, found_at;
};

// Order of floats as order of whole numbers.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

// The least whole number that is p x all or more, 1 at least (p < 1; all < 2^63): exact, so that equal weights are cut where their number says.
__device__ __forceinline__ uint64_t part_of(float p, uint64_t all) {
  if (!(p > 0x1p-62f)) return 1;
  int e;
  const uint64_t m = (uint64_t)ldexpf(frexpf(p, &e), 24);  // p = m 2^(e - 24), e <= 0
  const uint64_t hi = __umul64hi(all, m), lo = all * m;
  const int down = 24 - e;  // 24 to 85
  if (down >= 64) return (down == 64 ? hi : hi >> (down - 64)) + ((lo | (down == 64 ? 0ull : hi & ((1ull << (down - 64)) - 1))) != 0);
  return (hi << (64 - down) | lo >> down) + ((lo & ((1ull << down) - 1)) != 0);
}

template <typename T>
__device__ __forceinline__ T wave_upto(T v) {  // of this lane and those in front
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const T o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

template <bool BF16>
struct Sampler {
  static constexpr int kPer = kSampleChunk / 64;  // numbers of a lane in a chunk, side by side
  static constexpr float kLowest = -3.4028235e38f;
  const SampleArgs& a;
  SampleLds& m;
  const char* row;
  int tid, lane, wave;
  float most;
  double step;  // log2(e) / T
  float bins;   // steps of the histogram for a unit of the logits
  double least_weight;
  uint32_t key;  // the threshold: kept is what is above it, or it with a number up to `upto`
  int upto;
  int shift;  // weights as whole numbers: times 2^shift

  __device__ __forceinline__ void load(int chunk, float (&x)[kPer]) const {
    const int e = chunk * kSampleChunk + lane * kPer;
    if (a.vec && e + kPer <= a.n) {
      if (BF16) {
        unpack<true>(*(const uint4*)(row + 2 * (int64_t)e), x);
      } else {
        float lo[4], hi[4];
        unpack<false>(*(const uint4*)(row + 4 * (int64_t)e), lo);
        unpack<false>(*(const uint4*)(row + 4 * (int64_t)e + 16), hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = lo[i];
          x[i + 4] = hi[i];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[i] = e + i < a.n ? load_elem<BF16>(row, e + i) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = x[i] != x[i] ? -INFINITY : x[i] + 0.f;  // (-0 and 0 are equal)
  }
  // In powers of two, 0 for the largest; NaN or below -64 for what is nothing.
  __device__ __forceinline__ double bits(float x) const { return x == most ? 0.0 : ((double)x - (double)most) * step; }
  __device__ __forceinline__ bool live(double y) const { return y >= -(double)kSampleBits; }
  // Whether the number has a weight and is on the threshold's side.
  __device__ __forceinline__ bool counted(float x, int at) const {
    const uint32_t k = order_key(x);
    return x > -INFINITY && live(bits(x)) && (k > key || (k == key && at <= upto));
  }
  __device__ __forceinline__ int bin(float x) const { return x == most ? 0 : (int)fminf((most - x) * bins, (float)(kSampleSteps - 1)); }
  __device__ __forceinline__ uint64_t whole(double w) const { return (uint64_t)(ldexp(w, shift) + 0.5); }

  // f(chunk, first number of the lane, its numbers) for the chunks whose largest is `from` or more
  template <typename F>
  __device__ __forceinline__ void each(float from, const F& f) const {
    for (int c = wave; c < a.chunks; c += kSampleWaves) {
      if (m.top[c] < from) continue;
      float x[kPer];
      load(c, x);
      f(c, c * kSampleChunk + lane * kPer, x);
    }
  }

  // The chunk at which the sum of m.sum passes (or, REACHES, reaches) `target` and target_of_all of the whole sum, the last that has any if none does; *front: the
  // sum in front of it, *all: of all.
  template <bool REACHES>
  __device__ __forceinline__ int chunk_at(double target_of_all, double target, double* front, double* all) {
    constexpr int EACH = kSampleChunks / kSampleThreads;
    double v[EACH], mine = 0;
    int last = -1;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int c = tid * EACH + i;
      v[i] = c < a.chunks ? m.sum[c] : 0;
      mine += v[i];
      if (v[i] > 0) last = c;
    }
    const double upto_me = wave_upto(mine);
    if (lane == 63) m.wave_d[wave] = upto_me;
    if (tid == 0) {
      m.found = kSampleChunks;
      m.found_at = -1;
    }
    __syncthreads();
    double base = 0, total = 0;
    for (int w = 0; w < kSampleWaves; ++w) {
      if (w == wave) base = total;
      total += m.wave_d[w];
    }
    target += target_of_all * total;
    double sum = base + upto_me - mine;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const double next = sum + v[i];
      if (v[i] > 0 && (REACHES ? next >= target : next > target)) atomicMin(&m.found, tid * EACH + i);
      sum = next;
    }
    if (last >= 0) atomicMax(&m.found_at, last);
    __syncthreads();
    int c = m.found < kSampleChunks ? m.found : m.found_at;
    c = c < 0 ? 0 : c;
    sum = base + upto_me - mine;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (tid * EACH + i == c) m.wave_d[0] = sum;  // (read by all above, before the last barrier)
      sum += v[i];
    }
    __syncthreads();
    *front = m.wave_d[0];
    *all = total;
    __syncthreads();
    return c;
  }

  // Threshold of the words in front (largest first) until their number reaches `want_count`, or (BY_MASS) their weight `want_mass`.
  template <bool BY_MASS>
  __device__ __forceinline__ void front(uint32_t want_count, uint64_t want_mass) {
    // ---- which step
    uint32_t above = 0;
    uint64_t above_mass = 0;
    uint32_t in = 0;
    const int b = step_at<BY_MASS, kSampleSteps>(want_count, want_mass, &above, &above_mass, &in);
    if (tid == 0) m.found_count = 0;
    __syncthreads();
    float edge = most - (float)(b + 1) / bins;  // nothing of the step is below it, but for roundings
    edge -= fabsf(edge) * 1e-5f + fabsf(most) * 1e-5f;
    if (!(edge > -INFINITY)) edge = kLowest;
    if (in <= kSampleFew) {
      each(edge, [&](int, int at, const float(&x)[kPer]) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (counted(x[i], at + i) && bin(x[i]) == b) {
            const uint32_t n = atomicAdd(&m.found_count, 1u);
            m.few_key[n] = order_key(x[i]);
            m.few_at[n] = at + i;
          }
      });
      __syncthreads();
      if (tid < (int)in) {
        const uint32_t k = m.few_key[tid];
        const int at = m.few_at[tid];
        uint32_t n = above;
        uint64_t w = above_mass;
        for (uint32_t o = 0; o < in; ++o) {
          const uint32_t ok = m.few_key[o];
          if (ok > k || (ok == k && m.few_at[o] < at)) {
            ++n;
            if (BY_MASS) w += whole(exp2(bits(of_key(ok))));
          }
        }
        const uint64_t own = BY_MASS ? whole(exp2(bits(of_key(k)))) : 0;
        if (BY_MASS ? w < want_mass && want_mass <= w + own : n + 1 == want_count) {
          m.found_key = k;
          m.found_at = at;
        }
      }
      __syncthreads();
      key = m.found_key;
      upto = m.found_at;
      __syncthreads();
      return;
    }
    // ---- many: by their bits, 11, 11 and 10 of them
    uint32_t prefix = 0;
    uint32_t ties = 0;
#pragma unroll 1
    for (int level = 0; level < 3; ++level) {
      const int low = level == 0 ? 21 : level == 1 ? 10 : 0, width = level == 2 ? 10 : 11;
      for (int i = tid; i < 2048; i += kSampleThreads) {
        m.count[i] = 0;
        m.mass[i] = 0;
      }
      __syncthreads();
      each(edge, [&](int, int at, const float(&x)[kPer]) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const uint32_t k = order_key(x[i]);
          if (counted(x[i], at + i) && bin(x[i]) == b && (level == 0 || k >> (low + width) == prefix)) {
            const uint32_t d = ((1u << width) - 1) & ~(k >> low);  // the largest first
            atomicAdd(&m.count[d], 1u);
            if (BY_MASS) atomicAdd((unsigned long long*)&m.mass[d], (unsigned long long)whole(exp2(bits(x[i]))));
          }
        }
      });
      __syncthreads();
      const uint32_t d = step_at<BY_MASS, 2048>(want_count - above, want_mass - above_mass, &above, &above_mass, &ties);
      prefix = prefix << width | (((1u << width) - 1) & ~d);
    }
    const uint32_t was = key;
    key = prefix;
    const uint64_t own = whole(exp2(bits(of_key(key))));
    const uint32_t take = BY_MASS ? (uint32_t)((want_mass - above_mass + own - 1) / own) : want_count - above;
    if (take < ties) upto = nth_equal(take);
    else if (key != was) upto = 0x7fffffff;
  }

  // The step (of N) in which the sums over m.count or m.mass reach what is wanted; *count, *mass: added to by what lies above it; *in: what it holds.
  template <bool BY_MASS, int N>
  __device__ __forceinline__ int step_at(uint32_t want_count, uint64_t want_mass, uint32_t* count, uint64_t* mass, uint32_t* in) {
    constexpr int EACH = N / kSampleThreads;
    uint32_t c = 0;
    uint64_t w = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      c += m.count[tid * EACH + i];
      w += m.mass[tid * EACH + i];
    }
    const uint32_t c_upto = wave_upto(c);
    const uint64_t w_upto = wave_upto((unsigned long long)w);
    if (lane == 63) {
      m.wave_c[wave] = c_upto;
      m.wave_m[wave] = w_upto;
    }
    if (tid == 0) m.found = N - 1;
    __syncthreads();
    uint32_t c_base = c_upto - c;
    uint64_t w_base = w_upto - w;
    for (int v = 0; v < wave; ++v) {
      c_base += m.wave_c[v];
      w_base += m.wave_m[v];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const uint32_t cc = m.count[tid * EACH + i];
      const uint64_t ww = m.mass[tid * EACH + i];
      if (BY_MASS ? w_base < want_mass && want_mass <= w_base + ww : c_base < want_count && want_count <= c_base + cc) {
        m.found = tid * EACH + i;
        m.found_count = c_base;
        m.found_mass = w_base;
      }
      c_base += cc;
      w_base += ww;
    }
    __syncthreads();
    const int b = m.found;
    *count += m.found_count;
    *mass += m.found_mass;
    *in = m.count[b];
    __syncthreads();
    return b;
  }

  // Number of the n-th word whose logit is the threshold's.
  __device__ __forceinline__ int nth_equal(uint32_t n) {
    const float value = of_key(key);
    for (int c = tid; c < kSampleChunks; c += kSampleThreads) m.sum[c] = 0;
    __syncthreads();
    each(value, [&](int c, int, const float(&x)[kPer]) {
      int k = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) k += __popcll(__ballot(x[i] == value));
      if (lane == 0) m.sum[c] = k;
    });
    __syncthreads();
    double front, all;
    const int c = chunk_at<true>(0, (double)n, &front, &all);
    if (wave == 0) {
      float x[kPer];
      load(c, x);
      int k = 0, left = (int)n - (int)front;
#pragma unroll
      for (int i = 0; i < kPer; ++i) k += x[i] == value;
      int base = wave_upto(k) - k;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (x[i] == value && ++base == left) m.found_at = c * kSampleChunk + lane * kPer + i;
    }
    __syncthreads();
    const int at = m.found_at;
    __syncthreads();
    return at;
  }

  __device__ __forceinline__ double kept(float x, int at) const {
    if (!counted(x, at)) return 0;
    const double w = exp2(bits(x));
    return w >= least_weight ? w : 0;
  }

  __device__ __forceinline__ void run(int r) {
    row = (const char*)a.logits + (int64_t)r * a.row * (BF16 ? 2 : 4);
    // ---- the largest
    float top = -INFINITY;
    for (int c = wave; c < a.chunks; c += kSampleWaves) {
      float x[kPer];
      load(c, x);
      float t = x[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) t = fmaxf(t, x[i]);
      t = wave_max<64>(t);
      if (lane == 0) m.top[c] = t;
      top = fmaxf(top, t);
    }
    if (lane == 0) m.wave_d[wave] = top;
    __syncthreads();
    most = -INFINITY;
    for (int w = 0; w < kSampleWaves; ++w) most = fmaxf(most, (float)m.wave_d[w]);
    __syncthreads();
    if (!(most > -INFINITY)) {
      if (tid == 0) {
        a.word[r] = -1;
        if (a.chance) a.chance[r] = 0.f;
      }
      return;
    }
    const float temperature = a.temperature ? a.temperature[r] : 1.f;
    const float mp = a.min_p ? a.min_p[r] : 0.f;
    const bool greedy = !a.random || !(temperature > 0.f) || mp > 1.f;  // (nothing weighs more than the largest)
    key = 0;
    upto = 0x7fffffff;
    least_weight = 0;
    step = 1.4426950408889634074 / (double)temperature;
    bins = fminf((float)(step * ((kSampleSteps - 1) / kSampleBits)), -kLowest);
    if (greedy) {
      key = order_key(most);
      step = 1;
      bins = 1.f;
      upto = nth_equal(1);
    } else {
      const int k = a.top_k ? a.top_k[r] : 0;
      const float p = a.top_p ? a.top_p[r] : 1.f;
      if (mp > 0.f) least_weight = (double)mp;
      const bool by_count = k > 0 && k < a.n, by_mass = p < 1.f;
      shift = 62 - (32 - __builtin_clz(a.n));
      if (by_count || by_mass) {
        for (int i = tid; i < kSampleSteps; i += kSampleThreads) {
          m.count[i] = 0;
          m.mass[i] = 0;
        }
        __syncthreads();
        uint32_t n = 0;
        uint64_t all = 0;
        each(kLowest, [&](int, int at, const float(&x)[kPer]) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            const double y = bits(x[i]);
            if (counted(x[i], at + i)) {
              const int b = bin(x[i]);
              ++n;
              atomicAdd(&m.count[b], 1u);
              if (by_mass) {
                const uint64_t w = whole(exp2(y));
                all += w;
                atomicAdd((unsigned long long*)&m.mass[b], (unsigned long long)w);
              }
            }
          }
        });
        n = wave_upto(n);
        all = wave_upto((unsigned long long)all);
        if (lane == 63) {
          m.wave_c[wave] = n;
          m.wave_m[wave] = all;
        }
        __syncthreads();
        n = 0;
        all = 0;
        for (int w = 0; w < kSampleWaves; ++w) {
          n += m.wave_c[w];
          all += m.wave_m[w];
        }
        __syncthreads();
        const bool fewer = by_count && k < (int)n;
        if (fewer) front<false>(k, 0);
        if (by_mass) {
          if (fewer) {
            // the k largest by themselves (the search by bits may have taken the histogram's place, too)
            all = 0;
            for (int i = tid; i < kSampleSteps; i += kSampleThreads) {
              m.count[i] = 0;
              m.mass[i] = 0;
            }
            __syncthreads();
            each(of_key(key), [&](int, int at, const float(&x)[kPer]) {
#pragma unroll
              for (int i = 0; i < kPer; ++i) {
                if (counted(x[i], at + i)) {
                  const uint64_t w = whole(exp2(bits(x[i])));
                  all += w;
                  atomicAdd(&m.count[bin(x[i])], 1u);
                  atomicAdd((unsigned long long*)&m.mass[bin(x[i])], (unsigned long long)w);
                }
              }
            });
            all = wave_upto((unsigned long long)all);
            if (lane == 63) m.wave_m[wave] = all;
            __syncthreads();
            all = 0;
            for (int w = 0; w < kSampleWaves; ++w) all += m.wave_m[w];
            __syncthreads();
          }
          front<true>(0, part_of(p, all));
        }
      }
    }
    // ---- the kept weights, and where their sum passes the random number
    for (int c = tid; c < kSampleChunks; c += kSampleThreads) m.sum[c] = 0;
    __syncthreads();
    each(key ? of_key(key) : kLowest, [&](int c, int at, const float(&x)[kPer]) {
      double s = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) s += kept(x[i], at + i);
      s = __shfl(wave_upto(s), 63);
      if (lane == 0) m.sum[c] = s;
    });
    __syncthreads();
    float u = a.random ? a.random[r] : 0.f;
    u = u >= 0.f ? u : 0.f;
    double before, total;
    const int c = chunk_at<false>((double)u, 0, &before, &total);
    if (wave == 0) {
      float x[kPer];
      load(c, x);
      double w[kPer], mine = 0;
      int last = -1;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        w[i] = kept(x[i], c * kSampleChunk + lane * kPer + i);
        mine += w[i];
        if (w[i] > 0) last = i;
      }
      double sum = before + (wave_upto(mine) - mine);
      int hit = -1;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        sum += w[i];
        if (hit < 0 && w[i] > 0 && sum > (double)u * total) hit = i;
      }
      uint64_t lanes = __ballot(hit >= 0);
      // (none, where roundings of the two sums differ, or the random number is 1: the last that is kept)
      const int l = lanes ? __builtin_ctzll(lanes) : 63 - __builtin_clzll(__ballot(last >= 0));
      if (lane == l) {
        const int i = lanes ? hit : last;
        a.word[r] = c * kSampleChunk + lane * kPer + i;
        double weight = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) weight = e == i ? w[e] : weight;
        if (a.chance) a.chance[r] = (float)(weight / total);
      }
    }
  }
};

static_assert(sizeof(SampleLds) == kSampleLds, "what the host asks for");
template <bool BF16>
__device__ __forceinline__ void sample_body(const SampleArgs& a) {
  extern __shared__ double smem_sample[];
  Sampler<BF16> s{a, *(SampleLds*)smem_sample};
  s.tid = threadIdx.x;
  s.lane = threadIdx.x & 63;
  s.wave = uniform(threadIdx.x >> 6);
  s.run(blockIdx.x);
}

}  // namespace daris
