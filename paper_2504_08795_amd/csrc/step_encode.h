// The operators of a generation step as launches: checks of their descriptors, which kernel each runs and with which arguments (host
// logic, no GPU needed; in a header because only daris_api.cpp uses it).
#pragma once
#include <cstdarg>
#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

#include "../../include/daris_ops.h"
#include "aql.h"
#include "step_args.h"

namespace daris {

struct StepLaunch {
  AqlKernel k;  // with the LDS that this launch takes
  uint32_t groups = 0, threads = 0, nbytes = 0;
  // what it needs of the partition's workspace, filled in by place_step: bytes of partial results, counters that are zero
  size_t part_bytes = 0, counters = 0;
  uint32_t part_at = 0, count_at = 0;  // where its arguments name them
  alignas(8) unsigned char args[336];
};

// The step kernels of the code objects, looked up once.
struct StepTable {
  const AqlKernel* norm[2][2][2][6] = {};  // [bf16][8 bits][aligned][kNormShapes]
  const AqlKernel* append[2][3] = {};      // [bf16][dim 64, 128, 256]
  const AqlKernel* narrow[2][3] = {};
  const AqlKernel* wide[2][3] = {};        // (none of 256)
  const AqlKernel* matvec[4][3] = {};      // [kMatvecTypes][group 32, 64, 128]
  std::string resolve(const AqlRuntime& rt);
};

// 16-byte vectors of a row that a thread holds, and threads.  The first that holds the row; bf16, us a call of one row and of 4096, beside the next ones:
// 512 wide 6.9 / 9.8 (7.1 / 10.3, 7.1 / 10.9, 7.3 / 11.9); 2048 7.2 / 17.9 (7.3 / 18.0, 7.5 / 18.2, 1024 threads 7.4 / 33.6); 8192 8.4 / 59.8 (8.0 / 65.0); read
// twice, 16384 9.2 / 116.6 and not 8.5 / 106.4.
constexpr struct { int vectors, threads; } kNormShapes[6] = {{1, 64}, {1, 256}, {2, 256}, {4, 256}, {4, 1024}, {0, 1024}};
constexpr struct { int rows, bf16; } kMatvecTypes[4] = {{0, 0}, {1, 1}, {2, 0}, {2, 1}};

inline std::string StepTable::resolve(const AqlRuntime& rt) {
  std::string missing;
  auto find = [&](const char* fmt, auto... v) {
    char name[96];
    snprintf(name, sizeof name, fmt, v...);
    const AqlKernel* k = rt.kernel(name);
    if (!k && missing.empty()) missing = std::string(name) + " is missing from the code objects";
    return k;
  };
  const char* tf[2] = {"false", "true"};
  for (int b = 0; b < 2; ++b) {
    for (int f = 0; f < 2; ++f)
      for (int al = 0; al < 2; ++al)
        for (int i = 0; i < 6; ++i)
          norm[b][f][al][i] = find("daris::step_norm<%s, %s, %s, %d, %d>", tf[b], tf[f], tf[al], kNormShapes[i].vectors, kNormShapes[i].threads);
    for (int d = 0; d < 3; ++d) {
      append[b][d] = find("daris::step_append<%s, %d>", tf[b], 64 << d);
      narrow[b][d] = find("daris::step_attend_narrow<%s, %d>", tf[b], 64 << d);
      if (d < 2) wide[b][d] = find("daris::step_attend_wide<%s, %d>", tf[b], 64 << d);
    }
  }
  for (int t = 0; t < 4; ++t)
    for (int g = 0; g < 3; ++g) matvec[t][g] = find("daris::step_matvec<%d, %d, %s>", kMatvecTypes[t].rows, 32 << g, tf[kMatvecTypes[t].bf16]);
  return missing;
}

// ---- checks -----------------------------------------------------------------------------------------------------------------

inline std::string text(const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return buf;
}
constexpr int kMostRows = 1 << 30;  // of any count that 32-bit sums of the kernels and of this file start from
inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

inline std::string check_dtype(int dtype) { return dtype == DARIS_FP32 || dtype == DARIS_BF16 ? "" : text("dtype %d is neither DARIS_FP32 nor DARIS_BF16", dtype); }

inline std::string check_norm(const daris_norm& o) {
  std::string e = check_dtype(o.dtype);
  if (!e.empty()) return e;
  const size_t es = o.dtype == DARIS_BF16 ? 2 : 4;
  if (o.rows < 0 || o.width < 1) return text("rows %d, width %d", o.rows, o.width);
  if (o.rows > kMostRows || o.width > kMostRows) return text("more than 2^30 rows or channels (%d, %d)", o.rows, o.width);
  if (!(o.eps >= 0.f)) return "eps is negative or NaN";
  if (o.rows == 0) return "";
  if (!o.x || !o.weight || !o.y) return "NULL buffer";
  if (!aligned_to(o.x, es) || !aligned_to(o.weight, es) || !aligned_to(o.res, es) || !aligned_to(o.sum, es) || (!o.scale && !aligned_to(o.y, es))) return "a buffer is not aligned to its elements";
  if (o.scale) {
    if (o.group != 32 && o.group != 64 && o.group != 128) return text("group %d is not 32, 64 or 128", o.group);
    if (o.width % o.group) return text("width %d is no multiple of the group %d", o.width, o.group);
  } else if (o.group != 0) {
    return "a group without scales";
  }
  return "";
}

inline std::string check_cache(const daris_cache& c, int n_rows, const int32_t* row_start) {
  if (c.dim != 64 && c.dim != 128 && c.dim != 256) return text("dim %d is not 64, 128 or 256", c.dim);
  if (c.kv_heads < 1 || c.n_seqs < 0 || c.n_pages < 0 || c.pages_row < 0 || n_rows < 0) return "a negative count, or no key head";
  if (n_rows > kMostRows || c.n_seqs > kMostRows) return text("more than 2^30 rows or sequences (%d, %d)", n_rows, c.n_seqs);
  if (n_rows == 0 || c.n_seqs == 0) return "";
  if (c.pages_row > (1 << 24)) return "more than 2^30 tokens of a sequence";
  if (!c.before || !c.k || !c.v || !c.k_scale || !c.v_scale || !c.pages) return "NULL buffer of the cache";
  if (!aligned_to(c.k, 16) || !aligned_to(c.v, 16)) return "k and v of the cache are not aligned to 16 bytes";
  if (!aligned_to(c.k_scale, 4) || !aligned_to(c.v_scale, 4) || !aligned_to(c.pages, 4) || !aligned_to(c.before, 4) || !aligned_to(row_start, 4)) return "a buffer of the cache is not aligned to 4 bytes";
  if (!row_start && n_rows != c.n_seqs) return text("%d rows for %d sequences without row_start", n_rows, c.n_seqs);
  return "";
}

inline std::string check_append(const daris_append& o) {
  std::string e = check_dtype(o.dtype);
  if (e.empty()) e = check_cache(o.cache, o.n_rows, o.row_start);
  if (!e.empty()) return e;
  const size_t es = o.dtype == DARIS_BF16 ? 2 : 4;
  if (o.rot_dim < 0 || o.rot_dim > o.cache.dim || o.rot_dim % 2) return text("rot_dim %d of %d channels", o.rot_dim, o.cache.dim);
  if (o.rot_dim > 0 && o.turn_rows < 0) return "turn_rows is negative";
  if (o.n_rows == 0 || o.cache.n_seqs == 0) return "";
  if (!o.k || !o.v) return "NULL buffer";
  if (o.rot_dim > 0 && o.turn_rows > 0 && !o.turn) return "no table of angles";
  if ((o.q != nullptr) != (o.q_out != nullptr)) return "q and q_out go together";
  if (o.q && o.q_heads < 1) return "no query head";
  if (!aligned_to(o.k, es) || !aligned_to(o.v, es) || !aligned_to(o.q, es) || !aligned_to(o.q_out, es) || !aligned_to(o.turn, 4)) return "a buffer is not aligned to its elements";
  return "";
}

inline std::string check_attend(const daris_attend& o) {
  std::string e = check_dtype(o.dtype);
  if (e.empty()) e = check_cache(o.cache, o.n_rows, o.row_start);
  if (!e.empty()) return e;
  const size_t es = o.dtype == DARIS_BF16 ? 2 : 4;
  if (o.q_heads < 1 || o.q_heads % o.cache.kv_heads) return text("%d query heads on %d key heads", o.q_heads, o.cache.kv_heads);
  if (o.window < 0) return "window is negative";
  if (!(o.scale >= -1e38f && o.scale <= 1e38f)) return "scale is not finite, or above 1e38";
  if (o.n_rows == 0 || o.cache.n_seqs == 0) return "";
  if (!o.q || !o.out) return "NULL buffer";
  if (!aligned_to(o.q, es) || !aligned_to(o.out, es)) return "a buffer is not aligned to its elements";
  return "";
}

inline std::string check_matvec(const daris_matvec& o) {
  std::string e = check_dtype(o.dtype);
  if (!e.empty()) return e;
  const size_t es = o.dtype == DARIS_BF16 ? 2 : 4;
  if (o.rows < 0 || o.n < 1 || o.k < 1) return text("rows %d, n %d, k %d", o.rows, o.n, o.k);
  if (o.rows > kMostRows || o.n > kMostRows || o.k > kMostRows) return text("more than 2^30 rows, outputs or channels (%d, %d, %d)", o.rows, o.n, o.k);
  if (o.group != 32 && o.group != 64 && o.group != 128) return text("group %d is not 32, 64 or 128", o.group);
  if (o.k % o.group) return text("k %d is no multiple of the group %d", o.k, o.group);
  if (o.gate && o.n % 2) return text("a gate of %d outputs, which are no pairs", o.n);
  if (o.rows == 0) return "";
  if (!o.x || !o.w || !o.w_scale || !o.y) return "NULL buffer";
  if (!aligned_to(o.w, 16) || o.w_row % 16) return "rows of w are not aligned to 16 bytes";
  if ((!o.x_scale && !aligned_to(o.x, es)) || !aligned_to(o.w_scale, 2) || !aligned_to(o.y, es)) return "a buffer is not aligned to its elements";
  return "";
}

// ---- launches -----------------------------------------------------------------------------------------------------------------

template <typename A>
inline void set_args(StepLaunch* l, const A& a) {
  static_assert(sizeof(A) <= sizeof(StepLaunch::args), "the argument block is too large");
  std::memcpy(l->args, &a, sizeof(A));
  l->nbytes = sizeof(A);
}
// false: more workgroups than a packet counts
inline bool set_grid(StepLaunch* l, const AqlKernel* k, int64_t groups, uint32_t threads, uint32_t lds) {
  if (groups < 1 || groups * threads > 0xffffffffll) return false;
  l->k = *k;
  l->k.lds += lds;
  l->groups = (uint32_t)groups;
  l->threads = threads;
  return true;
}
constexpr const char* kTooMany = "too many workgroups for one launch";

inline std::string encode_norm(const StepTable& t, const daris_norm& o, StepLaunch* l) {
  const int bf16 = o.dtype == DARIS_BF16, f8 = o.scale != nullptr, vec = bf16 ? 8 : 4, es = 16 / vec;
  NormArgs a = {};
  a.x = o.x; a.res = o.res; a.weight = o.weight; a.sum = o.sum; a.y = o.y; a.scale = o.scale;
  a.x_row = o.x_row; a.res_row = o.res_row; a.sum_row = o.sum_row; a.y_row = o.y_row;
  a.rows = o.rows; a.width = o.width; a.group = o.group; a.vectors = (o.width + vec - 1) / vec;
  a.eps = o.eps; a.inv_width = 1.0f / (float)o.width;
  const bool strides = o.rows == 1 || ((o.x_row * es) % 16 == 0 && (!o.res || (o.res_row * es) % 16 == 0) && (!o.sum || (o.sum_row * es) % 16 == 0) && (f8 ? o.y_row % vec : (o.y_row * es) % 16) == 0);
  const bool al = o.width % vec == 0 && strides && aligned_to(o.x, 16) && aligned_to(o.res, 16) && aligned_to(o.weight, 16) && aligned_to(o.sum, 16) && aligned_to(o.y, f8 ? vec : 16);
  int i = 0;
  while (i < 5 && kNormShapes[i].vectors * kNormShapes[i].threads < a.vectors) ++i;
  set_args(l, a);
  return set_grid(l, t.norm[bf16][f8][al][i], o.rows, kNormShapes[i].threads, 0) ? "" : kTooMany;
}

inline CacheArgs cache_args(const daris_cache& c, const int32_t* row_start, int n_rows) {
  CacheArgs a = {};
  a.k = c.k; a.v = c.v; a.k_scale = c.k_scale; a.v_scale = c.v_scale;
  a.pages = c.pages; a.before = c.before; a.row_start = row_start; a.pages_row = c.pages_row;
  a.n_pages = c.n_pages; a.n_seqs = c.n_seqs; a.kv_heads = c.kv_heads; a.n_rows = n_rows;
  return a;
}
inline int dim_index(int dim) { return dim == 64 ? 0 : dim == 128 ? 1 : 2; }

inline std::string encode_append(const StepTable& t, const daris_append& o, StepLaunch* l) {
  AppendArgs a = {};
  a.c = cache_args(o.cache, o.row_start, o.n_rows);
  a.k = o.k; a.v = o.v; a.q = o.q; a.q_out = o.q_out; a.turn = o.turn;
  a.k_row = o.k_row; a.k_head = o.k_head; a.v_row = o.v_row; a.v_head = o.v_head;
  a.q_row = o.q_row; a.q_head = o.q_head; a.qo_row = o.qo_row; a.qo_head = o.qo_head;
  a.q_heads = o.q ? o.q_heads : 0; a.turn_rows = o.turn_rows; a.rot_dim = o.rot_dim; a.pairs = o.pairs;
  const int64_t items = (o.row_start ? (int64_t)o.n_rows / kScaleTokens + 2 * (int64_t)o.cache.n_seqs : o.n_rows) * o.cache.kv_heads;
  const int64_t q_items = (int64_t)o.n_rows * ((a.q_heads + kTurnHeads - 1) / kTurnHeads);
  if (items + q_items > 0x7fffffffll) return kTooMany;
  a.items = (int)items;
  a.q_items = (int)q_items;
  set_args(l, a);
  return set_grid(l, t.append[o.dtype == DARIS_BF16][dim_index(o.cache.dim)], (items + q_items + 3) / 4, 256, 0) ? "" : kTooMany;
}

inline std::string encode_attend(const StepTable& t, const daris_attend& o, int n_cu, StepLaunch* l) {
  const int bf16 = o.dtype == DARIS_BF16, d = dim_index(o.cache.dim), vec = bf16 ? 8 : 4;
  AttendArgs a = {};
  a.c = cache_args(o.cache, o.row_start, o.n_rows);
  a.q = o.q; a.out = o.out;
  a.q_row = o.q_row; a.q_head = o.q_head; a.out_row = o.out_row; a.out_head = o.out_head;
  a.group = o.q_heads / o.cache.kv_heads;
  a.window = o.window > (1 << 30) ? 0 : o.window;  // (no token lies further back; its distance to a position in front of the first would pass 32 bits)
  a.scale = o.scale * 1.44269504088896341f;
  a.q_vec = aligned_to(o.q, 16) && o.q_row % vec == 0 && o.q_head % vec == 0;
  a.out_vec = aligned_to(o.out, bf16 ? 8 : 16) && o.out_row % 4 == 0 && o.out_head % 4 == 0;
  const int64_t columns = (int64_t)o.n_rows * a.group;
  // Wide tiles need columns to fill them, and narrow ones are faster while a few a CU hold all columns.  Four heads to a key head, 8 key heads, 256 CUs, us a call
  // with narrow and with wide tiles, bf16 and fp32.  Heads of 64: 16 x 48 rows (1536 narrow tiles) 38 and 43, 53 and 59; 8 x 128 (2048) 53 and 49, 81 and 70.  Heads of
  // 128: 16 x 24 (768) 41 and 43, 47 and 75; 8 x 64 (1024) 61 and 53, 71 and 100; 1 x 1024 (2048) 208 and 117, 240 and 243; 1 x 2048 444 and 203, 510 and 457; fp32's wide tiles have a CU for
  // themselves.  64 x 4 rows, which fill an eighth of wide tiles: 33 and 42.
  const int full = o.cache.dim == 64 ? 6 : bf16 ? 3 : 8;
  const bool wide = columns * o.cache.dim >= 4096 * (int64_t)o.cache.n_seqs && columns * o.cache.kv_heads > (int64_t)full * kNarrowColumns * n_cu && t.wide[bf16][d];
  const int cols = wide ? kWideColumns : kNarrowColumns;
  const int64_t tiles = columns / cols + o.cache.n_seqs;  // at most: each sequence's last one may be part of a tile
  // Two workgroups for each CU; wide tiles that are that many by themselves are not cut.  With one, two and four a CU, us a call: a token for 8 streams of 2000
  // (32 heads of 128, 8 key heads) 19.1, 19.0, 19.3; for 64 of 2800 74, 74, 83; for one of 32000 24, 27, 36 (the merge grows with the units).
  const int64_t aim = 2 * (int64_t)n_cu / o.cache.kv_heads;
  // Nor are those of one sequence that are as many, whose pages are alike, and narrow ones that are 64 for each place: a workspace for every tile would grow with a
  // prompt's rows.  (us a call whole and cut, 8 query and 8 key heads of 256: 32 x 256 rows behind 0 to 3100 tokens, 64 a place, 3524 and 3519; 32 x 256 rows and a row
  // behind 32000, 1834 and 1621; 8 x 256 and such a row, 16 a place, 902 and 415.)
  const int64_t least = o.cache.n_seqs == 1 ? (columns + cols - 1) / cols : columns / cols;  // tiles that there are at least
  const bool whole = least >= (wide || o.cache.n_seqs == 1 ? 1 : 64) * aim;
  a.target = whole ? 0 : aim < 1 ? 1 : (int)aim;
  const int64_t units = tiles + a.target + 1;
  if (units * o.cache.kv_heads > 0x7fffffll) return kTooMany;
  a.units = (int)units;
  a.round = n_cu / o.cache.kv_heads;
  l->part_at = offsetof(AttendArgs, part);
  l->count_at = offsetof(AttendArgs, count);
  l->counters = a.target ? (size_t)units * o.cache.kv_heads : 0;
  l->part_bytes = a.target ? (size_t)(units * o.cache.kv_heads * unit_floats(cols, o.cache.dim)) * sizeof(float) : 0;
  set_args(l, a);
  return set_grid(l, wide ? t.wide[bf16][d] : t.narrow[bf16][d], units * o.cache.kv_heads, 256, wide ? wide_lds(o.cache.dim) : narrow_lds(o.cache.dim)) ? "" : kTooMany;
}

inline std::string encode_matvec(const StepTable& t, const daris_matvec& o, int n_cu, StepLaunch* l) {
  const int bf16 = o.dtype == DARIS_BF16, type = o.x_scale ? 2 + bf16 : bf16, parts = type == 0 ? 2 : 1, es = o.x_scale ? 1 : bf16 ? 2 : 4;
  // (blocks of 64 rows for more than 16 of them, on eight waves, were slower throughout: 64 rows, 22016 outputs of 4096 channels in bf16 61 us and 43, 17 rows 40
  // and 27, 2000 rows 1143 and 900)
  constexpr int block = kMatvecRows, waves = kMatvecWaves;
  const int blocks = (o.rows + block - 1) / block;
  MatvecArgs a = {};
  a.x = o.x; a.x_scale = o.x_scale; a.w = o.w; a.w_scale = o.w_scale; a.y = o.y;
  a.x_row = o.x_row; a.w_row = o.w_row; a.y_row = o.y_row;
  a.rows = o.rows; a.n = o.n; a.k = o.k; a.gate = o.gate;
  const int x_bytes = es == 1 ? 8 : 16;
  a.x_vec = aligned_to(o.x, x_bytes) && (o.rows == 1 || (o.x_row * es) % x_bytes == 0);
  const int rows = o.rows < block ? o.rows : block, steps = (int)(((int64_t)o.k + 127) / 128);
  const int64_t tiles = ((int64_t)o.n + 15) / 16, room = n_cu / blocks > 1 ? n_cu / blocks : 1;
  // x in LDS, of all of K if it fits (with the weights' scales and the waves' sums), else of the largest chunk that fits twice
  const int per_group = 128 / o.group, step_bytes = 128 * 2 * parts * rows + (type == 1 ? 0 : per_group * ((rows + 3) / 4 * 4) * 8);
  auto lds = [&](int cs, int across, int steps) {
    const bool again = cs < steps || (tiles + across - 1) / across > room;
    return (cs < steps ? 2 : 1) * cs * step_bytes + (again ? 2 : 1) * across * 16 * matvec_pitch(cs * per_group) * 2 + waves * block * 16 * 4;
  };
  auto log2_up = [](int v) {
    int log = 0;
    while ((1 << log) < v) ++log;
    return log;
  };
  auto fits = [&](int cs, int across, int steps) {
    return ((16ll << log2_up(cs)) * rows <= matvec_pieces(parts) * waves * 64) && (across * 16 << log2_up((cs * per_group + 7) / 8)) <= kScalePieces * waves * 64 && lds(cs, across, steps) <= 160 * 1024;
  };
  // Tiles side by side in a workgroup, and workgroups that share K: what makes the shortest sequence of steps for a wave.  A wave's part of a chunk
  // counts in fours (its steps travel four at a time), a barrier as two steps and a thread's piece of x as half a step.  K is shared only where that leaves CUs none without a workgroup
  // more than before and two steps for a wave; to meet takes four steps and the last workgroup two for every eight numbers that a thread fetches.
  int64_t best = -1;
  for (int across = 1; across <= waves; across *= 2) {
    const int64_t groups = (tiles + across - 1) / across, rounds = (groups + room - 1) / room;
    int64_t most = rounds == 1 ? n_cu / (groups * blocks) : 1;
    most = most < (int64_t)steps * across / (2 * waves) ? most : (int64_t)steps * across / (2 * waves);
    for (int64_t shares = 1; shares <= (most < 64 ? most : 64) || shares == 1; shares *= 2) {
      const int each = (int)((steps + shares - 1) / shares);
      if ((each + 0ll) * (shares - 1) >= steps) continue;  // (the last share would have nothing)
      int cs = each;
      if (!fits(cs, across, each)) {
        cs = 1 << log2_up(cs);
        while (cs > 1 && !fits(cs, across, each)) cs /= 2;
      }
      if (!fits(cs, across, each)) continue;
      const int64_t chunks = (each + cs - 1) / cs, own = ((int64_t)cs * across + waves - 1) / waves;
      const int64_t numbers = ((int64_t)rows * across * 16 + waves * 64 - 1) / (waves * 64);
      const int64_t pieces = ((int64_t)rows * cs * 16 + waves * 64 - 1) / (waves * 64) * parts * (chunks > 1 ? rounds * chunks : 1);
      const int64_t cost = 2 * rounds * chunks * ((own + 3) / 4 * 4 + 2) + pieces + (shares > 1 ? 8 + 4 * numbers * ((shares + 7) / 8) : 0);
      if (best >= 0 && cost >= best) continue;
      best = cost;
      a.across = log2_up(across);
      a.steps = cs;
      a.chunks = (int)chunks;
      a.groups = (int)groups;
      a.wgs = (int)(groups < room ? groups : room);
      a.shares = (int)shares;
      a.share_steps = each;
    }
  }
  if (best < 0) return "no chunk of K fits LDS";
  a.chunk = log2_up(a.steps);
  a.eights = log2_up((a.steps * per_group + 7) / 8);
  a.pitch = matvec_pitch(a.steps * per_group);
  if (a.shares > 1) {
    l->part_at = offsetof(MatvecArgs, part);
    l->count_at = offsetof(MatvecArgs, count);
    l->counters = (size_t)a.wgs * blocks;
    l->part_bytes = l->counters * a.shares * block * (16 << a.across) * sizeof(float);
  }
  set_args(l, a);
  const int g = o.group == 32 ? 0 : o.group == 64 ? 1 : 2;
  return set_grid(l, t.matvec[type][g], (int64_t)a.wgs * blocks * a.shares, waves * 64, lds(a.steps, 1 << a.across, a.share_steps)) ? "" : kTooMany;
}

// What is wrong with an operator, or "".
inline std::string check_step(const daris_op& op) {
  switch (op.kind) {
    case DARIS_STEP_NORM: return check_norm(op.u.norm);
    case DARIS_STEP_APPEND: return check_append(op.u.append);
    case DARIS_STEP_ATTEND: return check_attend(op.u.attend);
    case DARIS_STEP_MATVEC: return check_matvec(op.u.matvec);
  }
  return text("kind %d is no operator", op.kind);
}

// An operator that check_step takes, as a launch on a partition of n_cu CUs: "" (l->groups == 0: it has no rows) or why it cannot be.
inline std::string encode_step(const StepTable& t, const daris_op& op, int n_cu, StepLaunch* l) {
  l->groups = 0;
  l->part_bytes = l->counters = 0;
  switch (op.kind) {
    case DARIS_STEP_NORM: return op.u.norm.rows ? encode_norm(t, op.u.norm, l) : "";
    case DARIS_STEP_APPEND: return op.u.append.n_rows && op.u.append.cache.n_seqs ? encode_append(t, op.u.append, l) : "";
    case DARIS_STEP_ATTEND: return op.u.attend.n_rows && op.u.attend.cache.n_seqs ? encode_attend(t, op.u.attend, n_cu, l) : "";
    case DARIS_STEP_MATVEC: return op.u.matvec.rows ? encode_matvec(t, op.u.matvec, n_cu, l) : "";
  }
  return "";
}

// The launch's places in the workspace.
inline void place_step(StepLaunch* l, void* part, uint32_t* counters) {
  if (!l->counters) return;
  std::memcpy(l->args + l->part_at, &part, sizeof part);
  std::memcpy(l->args + l->count_at, &counters, sizeof counters);
}

}  // namespace daris
