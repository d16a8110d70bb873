// Encodes operators of a generation step without a GPU and prints their launches.
// Lines in: `matvec rows n k group dtype codes gate n_cu`, `attend n_rows n_seqs q_heads kv_heads dim dtype n_cu`, `append n_rows n_seqs ragged kv_heads q_heads dim`,
// `norm rows width group dtype x_offset x_row`.  Lines out: `error TEXT` or numbers, see the prints.
#include <cstdio>
#include <iostream>
#include <sstream>

#include "../../paper_2504_08795_amd/csrc/step_encode.h"

using namespace daris;
namespace daris {
const AqlKernel* AqlRuntime::kernel(const std::string&) const { return nullptr; }
}  // namespace daris

int main() {
  AqlKernel kernels[8];  // which one was chosen shows in its object
  for (int i = 0; i < 8; ++i) kernels[i].object = i;
  StepTable t;
  for (auto& a : t.norm)
    for (auto& b : a)
      for (int al = 0; al < 2; ++al)
        for (int i = 0; i < 6; ++i) b[al][i] = &kernels[i];
  for (auto& a : t.append)
    for (auto& k : a) k = &kernels[0];
  for (auto& a : t.narrow)
    for (auto& k : a) k = &kernels[1];
  for (auto& a : t.wide)
    for (int d = 0; d < 2; ++d) a[d] = &kernels[2];
  for (auto& a : t.matvec)
    for (auto& k : a) k = &kernels[3];
  char* const some = reinterpret_cast<char*>(uintptr_t(1) << 20);  // an address that nothing reads
  std::string line, what;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    in >> what;
    daris_op op = {};
    int n_cu = 256;
    if (what == "matvec") {
      op.kind = DARIS_STEP_MATVEC;
      daris_matvec& o = op.u.matvec;
      int codes;
      in >> o.rows >> o.n >> o.k >> o.group >> o.dtype >> codes >> o.gate >> n_cu;
      o.x = o.y = some;
      o.w = reinterpret_cast<uint8_t*>(some);
      o.w_scale = reinterpret_cast<uint16_t*>(some);
      o.x_scale = codes ? reinterpret_cast<uint8_t*>(some) : nullptr;
      o.x_row = o.k;
      o.w_row = (o.k / 2 + 15) / 16 * 16;
      o.y_row = o.n;
    } else if (what == "attend" || what == "append") {
      daris_cache c = {};
      c.k = c.v = c.k_scale = c.v_scale = reinterpret_cast<uint8_t*>(some);
      c.pages = c.before = reinterpret_cast<int32_t*>(some);
      c.n_pages = 10;
      c.pages_row = 10;
      if (what == "attend") {
        op.kind = DARIS_STEP_ATTEND;
        daris_attend& o = op.u.attend;
        in >> o.n_rows >> c.n_seqs >> o.q_heads >> c.kv_heads >> c.dim >> o.dtype >> n_cu;
        o.q = o.out = some;
        o.row_start = c.pages;
        o.cache = c;
      } else {
        op.kind = DARIS_STEP_APPEND;
        daris_append& o = op.u.append;
        int ragged;
        in >> o.n_rows >> c.n_seqs >> ragged >> c.kv_heads >> o.q_heads >> c.dim;
        o.k = o.v = some;
        o.q = o.q_out = o.q_heads ? some : nullptr;
        o.row_start = ragged ? c.pages : nullptr;
        o.cache = c;
      }
    } else {
      op.kind = DARIS_STEP_NORM;
      daris_norm& o = op.u.norm;
      int offset;
      in >> o.rows >> o.width >> o.group >> o.dtype >> offset >> o.x_row;
      o.x = some + offset;
      o.weight = o.y = some;
      o.scale = o.group ? reinterpret_cast<uint8_t*>(some) : nullptr;
      o.y_row = o.width;
    }
    std::string e = check_step(op);
    StepLaunch l;
    if (e.empty()) e = encode_step(t, op, n_cu, &l);
    if (!e.empty()) {
      printf("error %s\n", e.c_str());
      continue;
    }
    printf("%d %u %u %u %zu %zu", (int)l.k.object, l.groups, l.threads, l.k.lds, l.part_bytes, l.counters);
    if (!l.groups) {
    } else if (op.kind == DARIS_STEP_MATVEC) {
      MatvecArgs a;
      std::memcpy(&a, l.args, sizeof a);
      printf(" %d %d %d %d %d %d %d", a.steps, a.chunk, 1 << a.across, a.groups, a.wgs, a.shares, a.share_steps);
    } else if (op.kind == DARIS_STEP_ATTEND) {
      AttendArgs a;
      std::memcpy(&a, l.args, sizeof a);
      printf(" %d %d %d", a.group, a.target, a.units);
    } else if (op.kind == DARIS_STEP_APPEND) {
      AppendArgs a;
      std::memcpy(&a, l.args, sizeof a);
      printf(" %d %d", a.items, a.q_items);
    } else {
      NormArgs a;
      std::memcpy(&a, l.args, sizeof a);
      printf(" %d", a.vectors);
    }
    printf("\n");
  }
  return 0;
}
