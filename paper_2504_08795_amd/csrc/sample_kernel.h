// Draws a word for each row of logits: weights exp((x - M) / T) cut to the top_k largest, to the shortest front with top_p of their sum, to those of min_p,
// and the first word, by number, at which the sum of the weights that are left passes random x total.
//
// Weights and their sums are held in 64 bits: a word is a whole number, and it changes where a sum passes the random number by a last bit.  (A weight is within 2^-46 of itself, by
// the series that it comes of; as the whole numbers of top_p within 2^-39.  Random numbers are floats, 2^-24 apart where they are next to 1.)  Nothing is sorted:
// what is left is everything above a threshold, (logit, number) of one word.  It is found by a histogram of equal steps of the exponent (counts, and weights as whole
// numbers, whose sums no order changes), and among the words of the one step that the threshold lies in by finer steps and by comparing each with each, or, where they are
// too many (equal logits), by their bits.
//
// Work. A row is cut into parts of up to kSamplePart numbers, a workgroup each, which reads them once: the largest, and as the row's wishes ask the histogram, or the sums
// of weights, against its own largest (the steps are those of an absolute grid, so that histograms of parts are added by shifting them).  A second launch, a workgroup a row, adds them up and
// finishes the row, from chunks of 512 numbers (a wave each) whose largest is above what a pass looks for.  (In one launch, the row's last workgroup finishing it, the others' successors
// waited for its registers: 64 rows of 131072, bf16, top_p 0.5 to 0.95, 135 us a call and 85.)
//
// One row of 50001 (fp32, 40 likeliest): 28 us a call, the parts 6 of them and the end 16, which is a chain of barriers and fetches: histograms, the step, its words, their order.  64 rows
// of 131072 (bf16, wishes of every kind), 16.8 MB: 77 to 83 us, the parts 19 (75 % of the SIMDs' cycles are vector instructions), the end 54 on 64 CUs, of which the
// longest rows gather the words of their step from 256 chunks (18) and add up one part's weights (11).  Weights in 64 bits cost 20 instructions a number; a lane's numbers take
// turns in one loop of them (unrolled, the constants of eight weights leave half of the waves without registers).  Kept weights are taken again in one part only, as the
// histograms say what is left of the others (one row of 131072, flat: 48 us for all of it, 7 so).
#pragma once
#include "step_common.h"

namespace daris {

constexpr int kSampleThreads = kSampleWaves * 64, kSampleHeld = kSamplePart / kSampleChunk / kSampleWaves;
constexpr int kSampleChunks = kSampleMost / kSampleChunk;
constexpr double kSampleBits = 64.0;   // a weight below 2^-64 of the largest is nothing
constexpr double kSampleGrid = 15.9;   // steps of a power of two: all 64 of them in kSampleSteps
static_assert(kSampleSteps == kSampleThreads, "a step for each thread");

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef unsigned __int128 u128;

struct SampleLds {
  float top[kSampleChunks];         // a chunk's largest
  float part_top[kSampleParts];     // ... a part's
  int part_off[kSampleParts];       // steps of its histogram's first from the row's first; more than all: it has no part in it
  double part_weight[kSampleParts]; // weight of its largest
  uint64_t part_left[kSampleParts]; // ... of its words of the threshold's step that are left, in this step's numbers
  double sum[kSampleChunks];        // a chunk's weights that are left, or how many of its numbers are the threshold's
  uint32_t count[kSampleSteps];
  uint64_t mass[kSampleSteps];
  uint64_t few[kSampleFew];         // words of one step: (logit, number), the larger word the larger number
  double wave_d[kSampleWaves];
  u128 wave_w[kSampleWaves];
  uint64_t wave_m[kSampleWaves];
  uint32_t wave_c[kSampleWaves];
  u128 found_mass;
  uint64_t found_word;
  double found_sum;
  uint32_t found_count;
  int found, found_at;
};

// Order of floats as order of whole numbers.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

// Weights as whole numbers: those of step b of the histogram times 2^(b / 16), which leaves them between 0.37 and 1.05, and 2^SHIFT, which leaves the sum of a
// row's below 2^63.  Each is so rounded by 2^-40 of itself at most (2^-43 in rows of 131072), however little it weighs, and a part's step once more where parts are added up.  Sums over
// steps have them in their places.
__device__ __forceinline__ int up_of(int b) { return b >> 4; }
__device__ __forceinline__ u128 placed(uint64_t mass, int b) { return (u128)mass << (64 - up_of(b)); }
// What is to come of step b, in its own numbers: the least one that is v or more.
__device__ __forceinline__ uint64_t taken_from(u128 v, int b) {
  const int d = 64 - up_of(b);
  return (uint64_t)(v >> d) + ((v & (((u128)1 << d) - 1)) != 0);
}
// The least whole number that is p x all or more, 1 at least (p < 1; all < 2^127): exact, so that equal weights are cut where their number says.
__device__ __forceinline__ u128 part_of(float p, u128 all) {
  if (!(p > 0x1p-62f)) return 1;
  int e;
  const uint64_t m = (uint64_t)ldexpf(frexpf(p, &e), 24);  // p = m 2^(e - 24), e <= 0
  const u128 low = (u128)(uint64_t)all * m, hi = (u128)(uint64_t)(all >> 64) * m + (low >> 64);
  const uint64_t lo = (uint64_t)low;
  const int down = 24 - e;  // 24 to 85
  if (down >= 64) return (hi >> (down - 64)) + ((lo | ((uint64_t)hi & ((1ull << (down - 64)) - 1))) != 0);
  return (hi << (64 - down) | lo >> down) + ((lo & ((1ull << down) - 1)) != 0);
}

// v of other lanes of a wave, as CTRL says; 0 where there is none.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T from_lane(T v) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
  } else if constexpr (sizeof(T) == 16) {
    return (T)from_lane<CTRL, ROWS>((uint64_t)(v >> 64)) << 64 | from_lane<CTRL, ROWS>((uint64_t)v);
  } else {
    const u32x2 x = __builtin_bit_cast(u32x2, v);
    u32x2 y;
    y.x = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x.x, CTRL, ROWS, 0xf, false);
    y.y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x.y, CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(T, y);
  }
}
// The sum over this lane and those in front: in its row of sixteen, in the wave (a third of the time of an exchange through LDS).
template <typename T>
__device__ __forceinline__ T row_upto(T v) {
  v += from_lane<0x111, 0xf>(v);
  v += from_lane<0x112, 0xf>(v);
  v += from_lane<0x114, 0xf>(v);
  return v + from_lane<0x118, 0xf>(v);
}
template <typename T>
__device__ __forceinline__ T wave_upto(T v) {
  v = row_upto(v);
  v += from_lane<0x142, 0xa>(v);
  return v + from_lane<0x143, 0xc>(v);
}
template <typename T>
__device__ __forceinline__ T of_lane(T v, int lane) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
  } else if constexpr (sizeof(T) == 16) {
    return (T)of_lane((uint64_t)(v >> 64), lane) << 64 | of_lane((uint64_t)v, lane);
  } else {
    u32x2 x = __builtin_bit_cast(u32x2, v);
    x.x = (uint32_t)__builtin_amdgcn_readlane((int)x.x, lane);
    x.y = (uint32_t)__builtin_amdgcn_readlane((int)x.y, lane);
    return __builtin_bit_cast(T, x);
  }
}

// 2^(y + up) for -64 <= y <= 0, 2^up for 0: the series of e^f to the eleventh power, |f| <= ln 2 / 2, whose rest is below (ln 2 / 2)^12 / 12! = 2^-47.
__device__ __forceinline__ double weight(double y, int up = 0) {
  const double n = rint(y), f = (y - n) * 0.693147180559945309417;
  double p = 1.0 / 39916800;
  p = fma(p, f, 1.0 / 3628800);
  p = fma(p, f, 1.0 / 362880);
  p = fma(p, f, 1.0 / 40320);
  p = fma(p, f, 1.0 / 5040);
  p = fma(p, f, 1.0 / 720);
  p = fma(p, f, 1.0 / 120);
  p = fma(p, f, 1.0 / 24);
  p = fma(p, f, 1.0 / 6);
  p = fma(p, f, 0.5);
  p = fma(p, f, 1.0);
  p = fma(p, f, 1.0);
  return __builtin_amdgcn_ldexp(p, (int)n + up);
}

template <bool BF16>
struct Sampler {
  static constexpr int kPer = kSampleChunk / 64;  // numbers of a lane in a chunk, side by side
  static constexpr float kLowest = -3.4028235e38f;
  static constexpr int kAhead = BF16 ? 4 : 2;  // chunks of a wave that are on their way (registers for more there are not)
  const SampleArgs& a;
  SampleLds& m;
  const char* row;
  int tid, lane, wave;
  float most, temperature;
  double step;   // log2(e) / T
  double grid;   // steps of the histogram for a unit of the logits
  double place;  // the largest's place on the grid
  uint32_t key;  // the threshold: left is what is above it, or it with a number up to `upto`
  int upto;
  int listed;           // m.few has all words that are left (and others), so many
  int below;            // step of the histogram that the threshold is in, -1: the parts' sums are not known
  bool spent;           // the row's histogram has made room for a finer one
  int shift;            // of weights as whole numbers

  // A lane's numbers of a chunk as they are in memory.  They begin at `first` (the last ones of the row where it ends in front of them).
  struct Raw {
    uint32_t w[BF16 ? 4 : 8];
  };
  __device__ __forceinline__ int first_of(int chunk) const {
    const int e = chunk * kSampleChunk + lane * kPer, last = a.n - kPer;
    return e < last ? e : last > 0 ? last : 0;
  }
  __device__ __forceinline__ void fetch(int chunk, Raw* r) const {
    const int first = first_of(chunk);
    if (a.n >= kPer) {  // (rows need not be aligned to more than their numbers)
      const u32x4_a2* p = (const u32x4_a2*)(row + (BF16 ? 2 : 4) * (int64_t)first);
#pragma unroll
      for (int i = 0; i < (BF16 ? 1 : 2); ++i) {
        const u32x4 v = p[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) r->w[4 * i + j] = v[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int at = i < a.n ? i : a.n - 1;
        if (!BF16) r->w[i % (BF16 ? 4 : 8)] = ((const uint32_t*)row)[at];
        else if (i & 1) r->w[i / 2] |= (uint32_t)((const uint16_t*)row)[at] << 16;
        else r->w[i / 2] = ((const uint16_t*)row)[at];
      }
    }
  }
  // ... as numbers: -infinity for NaN, for what an earlier lane has and for what lies behind the row
  __device__ __forceinline__ void numbers(const Raw& r, int chunk, float (&x)[kPer]) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = fmaxf(__uint_as_float(BF16 ? (i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16) : r.w[i % (BF16 ? 4 : 8)]) + 0.f, -INFINITY);  // (-0 and 0 are equal)
    if ((chunk + 1) * kSampleChunk <= a.n) return;
    const int skip = chunk * kSampleChunk + lane * kPer - first_of(chunk), end = a.n < kPer ? a.n : kPer;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = i >= skip && i < end ? x[i] : -INFINITY;
  }
  __device__ __forceinline__ void load(int chunk, float (&x)[kPer]) const {
    Raw r;
    fetch(chunk, &r);
    numbers(r, chunk, x);
  }
  // f(x[i]) for all of them, in a loop that is one (the constants of eight weights at once leave half of the waves without registers)
  template <typename F>
  static __device__ __forceinline__ void in_turn(float (&x)[kPer], const F& f) {
#pragma unroll 1
    for (int i = 0; i < kPer; i += 2) {
      f(x[0]);
      f(x[1]);
#pragma unroll
      for (int e = 2; e < kPer; ++e) x[e - 2] = x[e];
    }
  }
  // f(i, x[i]) for the set bits of `on`, lowest first, a lane after its own
  template <typename F>
  static __device__ __forceinline__ void one_by_one(uint32_t on, const float (&x)[kPer], const F& f) {
    while (on) {
      const uint32_t least = on & -on;
      float v = -INFINITY;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        asm("" : "+v"(v));  // (a register each: left to itself the compiler makes an array in memory of them)
        v = least >> e & 1 ? x[e] : v;
      }
      f(__builtin_ctz(on), v);
      on &= on - 1;
    }
  }

  // In powers of two, 0 for the largest; NaN or below -64 for what is nothing.
  __device__ __forceinline__ double bits(float x) const { return x == most ? 0.0 : ((double)x - (double)most) * step; }
  // Its step of the histogram, from the largest's on.  (Where the grid is finer than 64 bits tell, what differs from the largest is nothing.)
  __device__ __forceinline__ int bin(float x) const {
    const double b = place - floor((double)x * grid);
    return x == most ? 0 : b < kSampleSteps ? (int)b : kSampleSteps - 1;
  }
  // The least number for which ok holds, as order_key has it: `guess` but for its rounding.  ok holds for the largest, and for what is above a number for which it does.
  template <typename F>
  __device__ __forceinline__ uint32_t least_key(double guess, const F& ok) const {
    uint32_t k = order_key(most == INFINITY ? most : fminf(fmaxf((float)guess, kLowest), most) + 0.f);
#pragma unroll 1
    for (int i = 0; i < 4 && k > order_key(kLowest) && ok(of_key(k - 1) + 0.f); ++i) --k;
#pragma unroll 1
    for (int i = 0; i < 4 && !ok(of_key(k)); ++i) ++k;
    return k;
  }
  // ... that is in step b or above
  __device__ __forceinline__ uint32_t least_of(int b) const {
    if (b >= kSampleSteps - 1) return order_key(kLowest);
    return least_key(grid > 0 ? (place - b) / grid : -INFINITY, [&](float x) { return bin(x) <= b; });
  }
  static __device__ __forceinline__ uint32_t between(const float (&x)[kPer], float lowest, float highest) {
    uint32_t on = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) on |= x[i] >= lowest && x[i] <= highest ? 1u << i : 0u;
    return on;
  }
  // A finer step of step b, the largest first.
  __device__ __forceinline__ int fine(float x, int b) const {
    const double t = (place - b + 1 - (double)x * grid) * kSampleSteps;
    return x == most ? 0 : (int)fmin(fmax(t, 0.0), kSampleSteps - 1.0);
  }
  // Whether the number is on the threshold's side (nothing that weighs nothing is).
  __device__ __forceinline__ bool counted(float x, int at) const {
    const uint32_t k = order_key(x);
    return k > key || (k == key && at <= upto);
  }
  // ... of a lane's numbers, a bit each
  __device__ __forceinline__ uint32_t counted(const float (&x)[kPer], int first) const {
    uint32_t on = 0;
    const float least = of_key(key);
    if (upto == 0x7fffffff) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) on |= x[i] >= least ? 1u << i : 0u;
      return on;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) on |= x[i] > least || (x[i] == least && first + i <= upto) ? 1u << i : 0u;
    return on;
  }
  // Moves the threshold up to the least number that weighs `least` or more (0: anything), which is most + far but for its rounding.
  __device__ __forceinline__ void leave(double far, double least) {
    const uint32_t k = least_key((double)most + far, [&](float x) {
      const double y = bits(x);
      return y >= -kSampleBits && (least == 0 || weight(y) >= least);
    });
    if (k > key) {
      key = k;
      upto = 0x7fffffff;
    }
  }
  // What follows is against this largest number; all that weighs anything beside it is left.
  __device__ __forceinline__ void against(float largest) {
    most = largest;
    place = floor((double)most * grid);
    key = 0;
    leave((double)temperature * (-kSampleBits * 0.693147180559945309417), 0);
  }
  __device__ __forceinline__ uint64_t whole(float x, int b) const { return (uint64_t)(weight(bits(x), up_of(b) + shift) + 0.5); }
  // One more in place `at`, of step b.
  __device__ __forceinline__ void add_to(int at, float x, bool mass, int b) {
    atomicAdd(&m.count[at], 1u);
    if (mass) atomicAdd((unsigned long long*)&m.mass[at], (unsigned long long)whole(x, b));
  }
  __device__ __forceinline__ void add_to(int b, float x, bool mass) { add_to(b, x, mass, b); }
  static __device__ __forceinline__ uint64_t scaled(uint64_t v, double f) { return f == 1.0 ? v : (uint64_t)((double)v * f + 0.5); }
  __device__ __forceinline__ void clear_steps() {
    m.count[tid] = 0;
    m.mass[tid] = 0;
  }
  // The sum of a lane's weights that are left, and of the wave's.
  __device__ __forceinline__ double sum_of(const float (&x)[kPer], int first) const {
    double s = 0;
    one_by_one(counted(x, first), x, [&](int, float v) { s += weight(bits(v)); });
    return s;
  }
  // Sums over the threads in front, and over all (v_wave: LDS for the waves' sums).  A barrier inside; another before v_wave is written again.
  template <typename T>
  __device__ __forceinline__ T in_front(T v, T* v_wave, T* all) const {
    const T upto_me = wave_upto(v);
    if (lane == 63) v_wave[wave] = upto_me;
    __syncthreads();
    return waves_in_front(upto_me - v, v_wave, all);
  }
  template <typename T>
  __device__ __forceinline__ T waves_in_front(T in_wave, const T* v_wave, T* all) const {
    const T waves = row_upto(v_wave[lane & (kSampleWaves - 1)]);
    *all = of_lane(waves, kSampleWaves - 1);
    const T before = of_lane(waves, wave > 0 ? wave - 1 : 0);
    return (wave > 0 ? before : T(0)) + in_wave;
  }

  // What the parts of a row leave: [row][chunks] floats, their largest, in front; [row][chunks] sums; [row][part] histograms.
  __device__ __forceinline__ float* tops_at(int r) const { return a.part + (int64_t)r * a.row_floats; }
  __device__ __forceinline__ double* sums_at(int r) const { return (double*)(tops_at(r) + (a.chunks + 1) / 2 * 2); }
  __device__ __forceinline__ uint64_t* mass_at(int r, int part) const { return (uint64_t*)(sums_at(r) + a.chunks) + (int64_t)part * (kSampleSteps + kSampleSteps / 2); }
  __device__ __forceinline__ uint32_t* counts_at(int r, int part) const { return (uint32_t*)(mass_at(r, part) + kSampleSteps); }

  // f(chunk, first, x) for the chunks whose largest is `from` or more: a lane's numbers x of them, from number `first` on.  kAhead chunks of a wave are on their way.
  template <typename F>
  __device__ __forceinline__ void each(float from, const F& f, int begin = 0, int end = kSampleChunks) const {
    end = end < a.chunks ? end : a.chunks;
#pragma unroll 1
    for (int base = begin; base < end; base += 64 * kSampleWaves) {
      const int mine = base + lane * kSampleWaves + wave;
      uint64_t left = __ballot(mine < end && m.top[mine < end ? mine : 0] >= from);
      if (!left) continue;
      Raw r[kAhead] = {};
      int c[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) c[i] = -1;
      bool more;
#pragma unroll 1
      do {
#pragma unroll
        for (int i = 0; i + 1 < kAhead; ++i) {
          r[i] = r[i + 1];
          c[i] = c[i + 1];
        }
        c[kAhead - 1] = left ? base + __builtin_ctzll(left) * kSampleWaves + wave : -1;
        left &= left - 1;
        if (c[kAhead - 1] >= 0) fetch(c[kAhead - 1], &r[kAhead - 1]);
        if (c[0] >= 0) {
          float x[kPer];
          numbers(r[0], c[0], x);
          f(c[0], first_of(c[0]), x);
        }
        more = false;
#pragma unroll
        for (int i = 1; i < kAhead; ++i) more = more || c[i] >= 0;
      } while (more);
    }
  }

  // The chunk at which the sum of m.sum passes (or, REACHES, reaches) `target` and target_of_all of the whole sum, the last that has any if none does; *front: the
  // sum in front of it, *all: of all.
  template <bool REACHES>
  __device__ __forceinline__ int chunk_at(double target_of_all, double target, double* front, double* all) {
    constexpr int EACH = kSampleChunks / kSampleThreads;
    double v[EACH], mine = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      v[i] = tid * EACH + i < a.chunks ? m.sum[tid * EACH + i] : 0;
      mine += v[i];
    }
    if (tid == 0) {
      m.found = kSampleChunks;
      m.found_at = 0;
    }
    double total, sum = in_front(mine, m.wave_d, &total);
    target += target_of_all * total;
    // (of a wave one lane says which is its first, and which its last: all at one address would come one after the other)
    double begins[EACH];
    int first = kSampleChunks, last = -1;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      begins[i] = sum;
      sum += v[i];
      if (v[i] > 0) {
        last = tid * EACH + i;
        if (first == kSampleChunks && (REACHES ? sum >= target : sum > target)) first = tid * EACH + i;
      }
    }
    const uint64_t any = __ballot(last >= 0), hit = __ballot(first < kSampleChunks);
    if (any && lane == 63 - __builtin_clzll(any)) atomicMax(&m.found_at, last);
    if (hit && lane == __builtin_ctzll(hit)) atomicMin(&m.found, first);
    __syncthreads();
    const int c = m.found < kSampleChunks ? m.found : m.found_at;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (tid * EACH + i == c) m.found_sum = begins[i];
    __syncthreads();
    *front = m.found_sum;
    *all = total;
    return c;
  }

  // The step in which the sums over m.count (or, by mass, m.mass) reach what is wanted (or all that there is, if that is less); *count, *mass: added to by what lies above it;
  // *in: what it holds.  M is u128 for the row's histogram: its masses in their places, and -1 if all of the count is wanted; uint64_t for one step's.
  template <typename M>
  __device__ __forceinline__ int step_at(bool by_mass, uint32_t want_count, M want_mass, uint32_t* count, M* mass, uint32_t* in) {
    constexpr bool whole_row = sizeof(M) == 16;
    M* wave_m;
    if constexpr (whole_row) wave_m = m.wave_w;
    else wave_m = m.wave_m;
    if (tid == 0) m.found = -1;
    const uint32_t c = m.count[tid];
    M w = m.mass[tid];
    if constexpr (whole_row) w = placed(m.mass[tid], tid);
    const uint32_t c_upto = wave_upto(c);
    const M w_upto = by_mass ? wave_upto(w) : 0;
    if (lane == 63) {
      m.wave_c[wave] = c_upto;
      wave_m[wave] = w_upto;
    }
    __syncthreads();
    uint32_t c_all;
    M w_all = 0, w_base = 0;
    const uint32_t c_base = waves_in_front(c_upto - c, m.wave_c, &c_all);
    if (by_mass) w_base = waves_in_front(w_upto - w, wave_m, &w_all);
    if (!by_mass && whole_row && want_count >= c_all) want_count = 0;
    want_count = want_count < c_all ? want_count : c_all;
    want_mass = want_mass < w_all ? want_mass : w_all;
    if (by_mass ? w_base < want_mass && want_mass <= w_base + w : c_base < want_count && want_count <= c_base + c) {
      m.found = tid;
      m.found_count = c_base;
      m.found_mass = w_base;
    }
    __syncthreads();
    const int b = m.found;
    if (b >= 0) {
      *count += m.found_count;
      *mass += (M)m.found_mass;
      *in = m.count[b];
    }
    __syncthreads();
    return b;
  }

  // Moves the threshold to the last word of those in front (largest first) whose number is `want_count`, or (by mass) whose weight reaches `want_mass`.
  // sums: what the step's words that are left weigh goes to m.part_left, which is zero.
  __device__ __forceinline__ void front(bool by_mass, uint32_t want_count, u128 want, bool sums) {
    uint32_t above = 0, in = 0;
    u128 in_front_of = 0;
    const int b = step_at(by_mass, want_count, want, &above, &in_front_of, &in);
    if (b < 0) return;  // fewer than that: none is cut
    const uint64_t want_mass = by_mass ? taken_from(want - in_front_of, b) : 0;
    uint64_t above_mass = 0;  // (of the step)
    below = -1;
    listed = 0;
    const uint32_t first_above = above;
    const uint32_t from = least_of(b);
    const float edge = of_key(from > key ? from : key);
    const float upper = b > 0 ? of_key(least_of(b - 1) - 1) : most;
    float highest = upper;
    bool few = in <= kSampleFew;
    if (few) {
      // ---- the step's words in LDS, with those above it where all are few
      const bool with_above = above + in <= kSampleRank / 2;
      if (with_above) {
        highest = most;
        above = 0;
      }
      if (tid == 0) m.found_count = 0;
      __syncthreads();
      each(edge, [&](int, int first, const float(&x)[kPer]) {
        uint32_t on = between(x, edge, highest);
        if (upto != 0x7fffffff) on &= counted(x, first);
        const int n = __popc(on), end = wave_upto(n), all = of_lane(end, 63);
        if (all == 0) return;
        int base = 0;
        if (lane == 0) base = (int)atomicAdd(&m.found_count, (uint32_t)all);
        base = uniform(base) + end - n;
        one_by_one(on, x, [&](int i, float v) {
          if (base < kSampleFew) m.few[base] = (uint64_t)order_key(v) << 32 | ~(uint32_t)(first + i);
          ++base;
        });
      });
      __syncthreads();
      in = m.found_count < kSampleFew ? m.found_count : kSampleFew;
      listed = with_above ? (int)in : 0;
      // (a thread keeps its words of the step: in the end those that are left are weighed for their parts)
      constexpr int N = kSampleFew / kSampleThreads;
      uint64_t mine[N];
#pragma unroll
      for (int i = 0; i < N; ++i) mine[i] = tid + i * kSampleThreads < (int)in ? m.few[tid + i * kSampleThreads] : 0;
      if (in == 0) return;  // (counted against parts whose largest is smaller: nothing here weighs 2^-64, and all that does is in front)
      if (in > kSampleRank / 4 && !with_above) {
        // ---- those of one of its finer steps
        int step_of[N];
        spent = true;
        clear_steps();
        if (tid == 0) m.found_at = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int n = tid + i * kSampleThreads;
          step_of[i] = -1;
          if (n < (int)in) {
            const float x = of_key((uint32_t)(mine[i] >> 32));
            step_of[i] = fine(x, b);
            add_to(step_of[i], x, by_mass, b);
          }
        }
        __syncthreads();
        const int d = step_at<uint64_t>(by_mass, want_count - above, want_mass - above_mass, &above, &above_mass, &in);
        if (d < 0) return;
        few = in <= kSampleRank;
        if (few) {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (step_of[i] == d) m.few[atomicAdd(&m.found_at, 1)] = mine[i];
          __syncthreads();
        }
      }
      if (few) {
        // ---- each with each, so many threads to a word that all have one
        int threads = 64;
        while (threads * (int)in > kSampleThreads) threads /= 2;
        const int word = tid / threads;
        const bool on = word < (int)in;
        const uint64_t own_word = on ? m.few[word] : 0;
        if (by_mass) {
          if (tid < (int)in) {  // (the histogram has done its work; what is above the step has been taken off what is wanted)
            const float x = of_key((uint32_t)(m.few[tid] >> 32));
            m.mass[tid] = x <= upper ? whole(x, b) : 0;
          }
          __syncthreads();
        }
        uint32_t n = 0;
        uint64_t w = 0;
#pragma unroll 4
        for (int o = tid & (threads - 1); o < (int)in; o += threads) {
          const bool before = m.few[o] > own_word;
          n += before;
          if (by_mass) w += before ? m.mass[o] : 0;
        }
#pragma unroll 1
        for (int d = 1; d < threads; d *= 2) {
          n += __shfl_xor(n, d);
          if (by_mass) w += __shfl_xor((unsigned long long)w, d);
        }
        n += above;
        w += above_mass;
        const uint64_t own = by_mass && on ? m.mass[word] : 0;
        // (the last, if they come to less: the histogram's sums are rounded otherwise)
        if (on && ((by_mass ? w < want_mass && want_mass <= w + own : n + 1 == want_count) || (n + 1 == above + in && (by_mass ? w + own < want_mass : n + 1 < want_count)))) m.found_word = own_word;
        __syncthreads();
        key = (uint32_t)(m.found_word >> 32);
        upto = (int)~(uint32_t)m.found_word;
        if (sums && !with_above) {
          below = b;
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (mine[i] >= m.found_word) atomicAdd((unsigned long long*)&m.part_left[(int)~(uint32_t)mine[i] / (a.part_chunks * kSampleChunk)], (unsigned long long)whole(of_key((uint32_t)(mine[i] >> 32)), b));
        }
        return;
      }
    }
    // ---- many: by their bits, 10, 10, 6 and 6 of them
    above = first_above;
    above_mass = 0;
    uint32_t prefix = 0, ties = 0;
    spent = true;
#pragma unroll 1
    for (int level = 0; level < 4; ++level) {
      const int low = level == 0 ? 22 : level == 1 ? 12 : level == 2 ? 6 : 0, width = level < 2 ? 10 : 6;
      clear_steps();
      __syncthreads();
      each(edge, [&](int, int first, const float(&x)[kPer]) {
        one_by_one(counted(x, first) & between(x, edge, highest), x, [&](int, float v) {
          const uint32_t k = order_key(v);
          if (level == 0 || k >> (low + width) == prefix) add_to(((1u << width) - 1) & ~(k >> low), v, by_mass, b);  // the largest first
        });
      });
      __syncthreads();
      const int d = step_at<uint64_t>(by_mass, want_count - above, want_mass - above_mass, &above, &above_mass, &ties);
      if (d < 0) return;  // (as above, of more words)
      prefix = prefix << width | (((1u << width) - 1) & ~(uint32_t)d);
    }
    const uint32_t was = key;
    key = prefix;
    const uint64_t own = whole(of_key(key), b);
    const uint32_t take = by_mass ? (uint32_t)((want_mass - above_mass + own - 1) / own) : want_count - above;
    if (take < ties) upto = nth_equal(take);
    else if (key != was) upto = 0x7fffffff;
  }

  // Number of the n-th word whose logit is the threshold's.
  __device__ __forceinline__ int nth_equal(uint32_t n) {
    const float value = of_key(key);
    for (int c = tid; c < a.chunks; c += kSampleThreads) m.sum[c] = 0;
    __syncthreads();
    each(value, [&](int c, int, const float(&x)[kPer]) {
      int k = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) k += __popcll(__ballot(x[i] == value));
      if (lane == 0) m.sum[c] = k;
    });
    __syncthreads();
    double in_chunks, all;
    const int c = chunk_at<true>(0, (double)n, &in_chunks, &all);
    if (wave == 0) {
      float x[kPer];
      load(c, x);
      int k = 0;
      const int left = (int)n - (int)in_chunks;
#pragma unroll
      for (int i = 0; i < kPer; ++i) k += x[i] == value;
      int base = wave_upto(k) - k;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (x[i] == value && ++base == left) m.found_at = first_of(c) + i;
    }
    __syncthreads();
    return m.found_at;
  }

  // Draws from the words of m.few that are left: in the order of their numbers, as each counts those in front of it.
  __device__ __forceinline__ void pick(int r, float u) {
    int threads = 64;
    while (threads * listed > kSampleThreads) threads /= 2;
    const int word = tid / threads;
    const uint64_t own = word < listed ? m.few[word] : 0;
    const bool on = word < listed && counted(of_key((uint32_t)(own >> 32)), (int)~(uint32_t)own);
    if (tid == 0) {
      m.found = kSampleThreads;
      m.found_at = 0;
    }
    int n = 0;
#pragma unroll 4
    for (int o = tid & (threads - 1); o < listed; o += threads) {
      const uint64_t w = m.few[o];
      n += (uint32_t)w > (uint32_t)own && counted(of_key((uint32_t)(w >> 32)), (int)~(uint32_t)w);
    }
#pragma unroll 1
    for (int d = 1; d < threads; d *= 2) n += __shfl_xor(n, d);
    __syncthreads();
    if (on && (tid & (threads - 1)) == 0) {
      m.sum[n] = weight(bits(of_key((uint32_t)(own >> 32))));
      m.count[n] = ~(uint32_t)own;
      atomicMax(&m.found_at, n);
    }
    __syncthreads();
    const int last = m.found_at;
    const double v = tid <= last ? m.sum[tid] : 0;
    double total;
    const double front = in_front(v, m.wave_d, &total);
    const uint64_t hit = __ballot(tid <= last && front + v > (double)u * total);
    if (hit && lane == __builtin_ctzll(hit)) atomicMin(&m.found, tid);
    __syncthreads();
    if (tid == (m.found <= last ? m.found : last)) {
      a.word[r] = (int)m.count[tid];
      if (a.chance) a.chance[r] = (float)(v / total);
    }
  }

  // What row r asks for.
  int k;
  float p, mp;
  bool greedy, by_count, by_mass, steps, all, weighed;
  __device__ __forceinline__ void wishes(int r) {
    row = (const char*)a.logits + (int64_t)r * a.row * (BF16 ? 2 : 4);
    temperature = a.temperature ? a.temperature[r] : 1.f;
    p = a.top_p ? a.top_p[r] : 1.f;
    mp = a.min_p ? a.min_p[r] : 0.f;
    k = a.top_k ? a.top_k[r] : 0;
    greedy = !a.random || !(temperature > 0.f) || mp > 1.f;  // (nothing weighs more than the largest)
    by_count = !greedy && k > 0 && k < a.n;
    by_mass = !greedy && p < 1.f;
    steps = by_count || by_mass;
    all = !greedy && !steps && !(mp > 0.f);  // of them are left
    // The histogram has weights where they are asked for, and where many words may be left, whose parts' sums then need not be taken again.
    weighed = by_mass || (by_count && k > kSampleChunk);
    step = 1.4426950408889634074 / (double)temperature;
    grid = step * kSampleGrid;
    shift = 62 - (32 - __builtin_clz(a.n));
  }

  // One part of row r: its chunks' largest, and as the row asks its histogram or its chunks' sums, in LDS and (where there are others) in a.part.
  __device__ __forceinline__ void part(int r, int part) {
    // ---- the part's largest
    const int c0 = part * a.part_chunks, c1 = c0 + a.part_chunks < a.chunks ? c0 + a.part_chunks : a.chunks;
    Raw raw[kSampleHeld];
#pragma unroll
    for (int h = 0; h < kSampleHeld; ++h) {
      const int c = c0 + h * kSampleWaves + wave;
      fetch(c < c1 ? c : c0, &raw[h]);  // (no branch: they travel together)
    }
    clear_steps();
    float top = -INFINITY;
#pragma unroll
    for (int h = 0; h < kSampleHeld; ++h) {
      const int c = c0 + h * kSampleWaves + wave;
      if (c >= c1) break;
      float x[kPer];
      numbers(raw[h], c, x);
      float t = x[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) t = fmaxf(t, x[i]);
      t = wave_max<64>(t);
      if (lane == 0) {
        m.top[c] = t;
        if (a.parts > 1) tops_at(r)[c] = t;
      }
      top = fmaxf(top, t);
    }
    if (lane == 0) m.wave_d[wave] = top;
    __syncthreads();
    top = lanes_max<1, kSampleWaves>((float)m.wave_d[lane & (kSampleWaves - 1)]);
    // ---- its weights against its largest
    if (greedy) most = top;
    else against(top);
    if ((steps || all) && top > -INFINITY) {
      const float least = of_key(key);
#pragma unroll 1
      for (int h = 0; h < kSampleHeld; ++h) {
        const int c = c0 + h * kSampleWaves + wave;
        if (c >= c1) break;
        float x[kPer];
        numbers(raw[0], c, x);
#pragma unroll
        for (int i = 1; i < kSampleHeld; ++i) raw[i - 1] = raw[i];
        if (steps) {
          in_turn(x, [&](float v) {
            if (v >= least) add_to(bin(v), v, weighed);
          });
        } else {
          double s = 0;
          in_turn(x, [&](float v) { s += v >= least ? weight(bits(v)) : 0.0; });
          s = of_lane(wave_upto(s), 63);
          if (lane == 0) {
            m.sum[c] = s;
            if (a.parts > 1) sums_at(r)[c] = s;
          }
        }
      }
    }
    if (steps && a.parts > 1) {
      __syncthreads();
      if (weighed) mass_at(r, part)[tid] = m.mass[tid];
      counts_at(r, part)[tid] = m.count[tid];
    }
  }

  // Row r, whose parts are known.
  __device__ __forceinline__ void finish(int r) {
    if (a.parts > 1) {
      for (int c = tid; c < a.chunks; c += kSampleThreads) m.top[c] = tops_at(r)[c];
      if (tid < kSampleParts) {
        m.part_top[tid] = -INFINITY;
        m.part_left[tid] = 0;
      }
      __syncthreads();
      if (tid < a.parts) {
        float t = -INFINITY;
#pragma unroll 8
        for (int i = 0; i < a.part_chunks; ++i) t = fmaxf(t, tid * a.part_chunks + i < a.chunks ? m.top[tid * a.part_chunks + i] : -INFINITY);
        m.part_top[tid] = t;
      }
      __syncthreads();
      const float top = wave_max<64>(fmaxf(m.part_top[lane], m.part_top[lane + 64]));
      if (greedy) most = top;
      else against(top);
      if (tid < a.parts && !greedy) {
        const float t = m.part_top[tid];
        const double off = t == top ? 0.0 : place - floor((double)t * grid), y = bits(t);  // (NaN beside an infinity: none of it)
        m.part_off[tid] = t > -INFINITY && off < kSampleSteps ? (int)off : kSampleSteps;
        m.part_weight[tid] = t > -INFINITY && y >= -kSampleBits ? weight(y) : 0.0;
      }
      __syncthreads();
      if (steps) {
        uint32_t n = 0;
        uint64_t w = 0;
        constexpr int TOGETHER = 8;  // (parts whose numbers travel together, those behind the last repeating it)
        for (int q0 = 0; q0 < a.parts; q0 += TOGETHER) {
          uint32_t c[TOGETHER];
          uint64_t v[TOGETHER];
#pragma unroll
          for (int i = 0; i < TOGETHER; ++i) {
            const int q = q0 + i < a.parts ? q0 + i : a.parts - 1, at = tid - m.part_off[q];
            c[i] = counts_at(r, q)[at > 0 ? at : 0];
            v[i] = weighed ? mass_at(r, q)[at > 0 ? at : 0] : 0;
          }
#pragma unroll
          for (int i = 0; i < TOGETHER; ++i) {
            const int q = q0 + i < a.parts ? q0 + i : a.parts - 1;
            const bool in = q0 + i < a.parts && tid >= m.part_off[q];
            n += in ? c[i] : 0;
            if (weighed) w += in ? scaled(v[i], __builtin_amdgcn_ldexp(m.part_weight[q], up_of(tid) - up_of(tid - m.part_off[q]))) : 0;
          }
        }
        m.count[tid] = n;
        m.mass[tid] = w;
      } else if (all) {
        for (int c = tid; c < a.chunks; c += kSampleThreads) {
          // (a chunk whose largest is nothing beside the row's has no part in it, nor is its sum weighed)
          const double s = sums_at(r)[c];
          m.sum[c] = counted(m.top[c], 0) ? s * m.part_weight[c / a.part_chunks] : 0.0;
        }
      }
    }
    __syncthreads();
    if (!(most > -INFINITY)) {
      if (tid == 0) {
        a.word[r] = -1;
        if (a.chance) a.chance[r] = 0.f;
      }
      return;
    }
    if (greedy) {
      if (tid == 0) m.found = kSampleChunks;
      __syncthreads();
      for (int c = tid; c < a.chunks; c += kSampleThreads)
        if (m.top[c] == most) atomicMin(&m.found, c);
      __syncthreads();
      if (wave != 0) return;
      const int c = m.found;
      float y[kPer];
      load(c, y);
      int at = kPer;
#pragma unroll
      for (int i = kPer - 1; i >= 0; --i) at = y[i] == most ? i : at;
      const uint64_t lanes = __ballot(at < kPer);
      if (lane == __builtin_ctzll(lanes)) {
        a.word[r] = first_of(c) + at;
        if (a.chance) a.chance[r] = 1.f;
      }
      return;
    }
    // ---- the threshold: of the count, then of the weight
    const uint32_t lowest = key;
    below = kSampleSteps;
    listed = 0;
    spent = false;
#pragma unroll 1
    for (int turn = 0; turn < 2; ++turn) {
      if (!(turn ? by_mass : by_count)) continue;
      u128 want = 0;
      if (turn) {
        if (key != lowest || upto != 0x7fffffff || spent) {
          // the k largest by themselves (or all, where the k-th weighs nothing)
          __syncthreads();
          clear_steps();
          __syncthreads();
          each(of_key(key), [&](int, int first, const float(&x)[kPer]) { one_by_one(counted(x, first), x, [&](int, float v) { add_to(bin(v), v, true); }); });
          __syncthreads();
        }
        u128 sum;
        (void)in_front(placed(m.mass[tid], tid), m.wave_w, &sum);
        __syncthreads();
        want = part_of(p, sum);
      }
      front(turn, k, want, weighed && a.parts > 1 && (turn || !by_mass));
    }
    if (mp > 0.f) leave((double)temperature * (mp < 1.f ? log((double)mp) : -0x1p-54), (double)mp);  // (what is nearer than that weighs 1 in 64 bits)
    float u = a.random[r];
    u = u >= 1.f ? INFINITY : u >= 0.f ? u : 0.f;  // (no sum passes it: 1 x the whole sum, added up another way, may be passed by less than all)
    // ---- the weights that are left, and where their sum passes the random number
    if (listed) {
      pick(r, u);
      return;
    }
    double skipped = 0, more = 0;  // weights of the parts in front of the one that is looked at, and of all others
    int c0_left = 0, c1_left = a.chunks;
    // (What the parts leave may have words of no weight in it where none is cut, lighter than 2^-64 of the row's largest but not of their part's: 2^-44 in all, which is at most half of the
    // distance to the next random number from 2^-20 on.  For smaller ones all weights are taken again.)
    const bool by_parts = u >= 0x1p-20f;
    if (weighed && a.parts > 1 && below >= 0 && !(mp > 0.f) && by_parts) {
      // The histograms say what is left of each part, and so in which part the sum passes.
      for (int q = wave; q < a.parts; q += kSampleWaves) {
        const int end = below - m.part_off[q];
        double w = 0;
#pragma unroll 8
        for (int i = 0; i < kSampleSteps / 64; ++i) {
          const uint64_t v = mass_at(r, q)[i * 64 + lane];
          w += i * 64 + lane < end ? __builtin_amdgcn_ldexp((double)v, -up_of(i * 64 + lane)) : 0;
        }
        w = of_lane(wave_upto(w), 63) * m.part_weight[q];
        if (lane == 0) m.sum[q] = w;
      }
      __syncthreads();
      const double per = __builtin_amdgcn_ldexp(1.0, -shift);
      auto left = [&](int q) { return q < a.parts ? m.sum[q] + __builtin_amdgcn_ldexp((double)m.part_left[q], -up_of(below)) : 0.0; };
      const double left0 = left(lane), left1 = left(lane + 64);
      const double upto0 = wave_upto(left0), all0 = of_lane(upto0, 63), upto1 = all0 + wave_upto(left1), sum = of_lane(upto1, 63);
      const double target = (double)u * sum;
      const uint64_t hit0 = __ballot(upto0 > target && left0 > 0), hit1 = __ballot(upto1 > target && left1 > 0);
      const int q = hit0 ? __builtin_ctzll(hit0) : hit1 ? 64 + __builtin_ctzll(hit1) : -1;
      if (q >= 0) {
        const double upto_q = q < 64 ? of_lane(upto0, q) : of_lane(upto1, q - 64), left_q = q < 64 ? of_lane(left0, q) : of_lane(left1, q - 64);
        skipped = (upto_q - left_q) * per;
        more = (sum - left_q) * per;
        c0_left = q * a.part_chunks;
        c1_left = c0_left + a.part_chunks < a.chunks ? c0_left + a.part_chunks : a.chunks;
      }
    }
    if (!all || (a.parts > 1 && !by_parts)) {
      __syncthreads();
      for (int c = tid; c < a.chunks; c += kSampleThreads) m.sum[c] = 0;
      __syncthreads();
      each(of_key(key), [&](int c, int first, const float(&x)[kPer]) {
        const double s = of_lane(wave_upto(sum_of(x, first)), 63);
        if (lane == 0) m.sum[c] = s;
      }, c0_left, c1_left);
      __syncthreads();
    }
    double before, total;
    const int c = chunk_at<false>((double)u, (double)u * more - skipped, &before, &total);
    total += more;
    if (wave == 0) {
      float x[kPer];
      load(c, x);
      const int first = first_of(c);
      const double mine = sum_of(x, first), target = (double)u * total;
      double sum = skipped + before + (wave_upto(mine) - mine), hit_weight = 0, last_weight = 0;
      int hit = -1, last = -1;
      one_by_one(counted(x, first), x, [&](int i, float v) {
        last = i;
        last_weight = weight(bits(v));
        sum += last_weight;
        if (hit < 0 && sum > target) {
          hit = i;
          hit_weight = last_weight;
        }
      });
      // (none, where roundings of the two sums differ, or the random number is 1 or more: the last that is left)
      const uint64_t lanes = __ballot(hit >= 0);
      const int l = lanes ? __builtin_ctzll(lanes) : 63 - __builtin_clzll(__ballot(last >= 0));
      if (lane == l) {
        a.word[r] = first + (lanes ? hit : last);
        if (a.chance) a.chance[r] = (float)((lanes ? hit_weight : last_weight) / total);
      }
    }
  }
};

static_assert(sizeof(SampleLds) == kSampleLds, "what the host asks for");
// FINISH: a workgroup a row, whose parts other workgroups have looked at (or which is its only part itself); else a workgroup a part.
template <bool BF16, bool FINISH>
__device__ __forceinline__ void sample_body(const SampleArgs& a) {
  extern __shared__ double smem_sample[];
  Sampler<BF16> s{a, *(SampleLds*)smem_sample};
  s.tid = threadIdx.x;
  s.lane = threadIdx.x & 63;
  s.wave = uniform(threadIdx.x >> 6);
  const int r = FINISH ? blockIdx.x : blockIdx.x / a.parts;
  s.wishes(r);
  if (!FINISH) s.part(r, blockIdx.x - r * a.parts);
  else if (a.parts == 1) s.part(r, 0);
  if (FINISH) s.finish(r);
}

}  // namespace daris
