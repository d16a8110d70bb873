// Encodes operators of a drafted step without a GPU and prints their launches, and the layout of their descriptors.
// Lines in: `sample rows n dtype offset row`, `accept n_rows n_seqs words`, `keep n_rows n_seqs kv_heads dim`, `copy n n_pages kv_heads dim`,
// `append n_rows n_seqs kv_heads q_heads dim words`, `attend n_rows n_seqs q_heads kv_heads dim dtype words n_cu`, `sizes`.  Lines out: `error TEXT` or numbers, see the prints.
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
  for (int b = 0; b < 2; ++b) {
    for (int d = 0; d < 3; ++d) {
      t.tree_append[b][d] = &kernels[1];
      t.tree_narrow[b][d] = &kernels[2];
      if (d == 0 || (b && d == 1)) t.tree_wide[b][d] = &kernels[3];
      t.keep[d] = &kernels[5];
      t.copy[d] = &kernels[6];
    }
    t.sample[b] = &kernels[4];
    t.sample_parts[b] = &kernels[0];
  }
  t.accept = &kernels[7];
  char* const some = reinterpret_cast<char*>(uintptr_t(1) << 20);  // an address that nothing reads
  std::string line, what;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    in >> what;
    if (what == "sizes") {
      printf("%zu %zu %zu %zu %zu %zu %zu %zu %zu %zu\n", sizeof(daris_op), sizeof(daris_tree_append), sizeof(daris_tree_attend), sizeof(daris_sample), sizeof(daris_accept), sizeof(daris_keep),
             sizeof(daris_copy), offsetof(daris_tree_append, tree_words), offsetof(daris_tree_attend, tree_words), offsetof(daris_sample, dtype));
      continue;
    }
    daris_op op = {};
    int n_cu = 256;
    daris_cache c = {};
    c.k = c.v = c.k_scale = c.v_scale = reinterpret_cast<uint8_t*>(some);
    c.pages = c.before = reinterpret_cast<int32_t*>(some);
    c.n_pages = 10;
    c.pages_row = 10;
    int32_t* const ints = reinterpret_cast<int32_t*>(some);
    if (what == "sample") {
      op.kind = DARIS_STEP_SAMPLE;
      daris_sample& o = op.u.sample;
      int offset;
      in >> o.rows >> o.n >> o.dtype >> offset >> o.logits_row;
      o.logits = some + offset;
      o.word = ints;
    } else if (what == "accept") {
      op.kind = DARIS_STEP_ACCEPT;
      daris_accept& o = op.u.accept;
      in >> o.n_rows >> o.n_seqs >> o.tree_words;
      o.tree = reinterpret_cast<uint64_t*>(some);
      o.words = o.answers = o.row_start = ints;
      o.path = o.count = o.word = ints;
    } else if (what == "keep") {
      op.kind = DARIS_STEP_KEEP;
      daris_keep& o = op.u.keep;
      in >> o.n_rows >> c.n_seqs >> c.kv_heads >> c.dim;
      o.path = o.count = o.row_start = ints;
      o.cache = c;
    } else if (what == "copy") {
      op.kind = DARIS_STEP_COPY;
      daris_copy& o = op.u.copy;
      in >> o.n >> c.n_pages >> c.kv_heads >> c.dim;
      o.pairs = ints;
      c.pages = c.before = nullptr;
      o.cache = c;
    } else if (what == "append") {
      op.kind = DARIS_STEP_TREE_APPEND;
      daris_tree_append& o = op.u.tree_append;
      in >> o.n_rows >> c.n_seqs >> c.kv_heads >> o.q_heads >> c.dim >> o.tree_words;
      o.k = o.v = some;
      o.q = o.q_out = o.q_heads ? some : nullptr;
      o.row_start = ints;
      o.tree = reinterpret_cast<uint64_t*>(some);
      o.cache = c;
    } else {
      op.kind = DARIS_STEP_TREE_ATTEND;
      daris_tree_attend& o = op.u.tree_attend;
      in >> o.attend.n_rows >> c.n_seqs >> o.attend.q_heads >> c.kv_heads >> c.dim >> o.attend.dtype >> o.tree_words >> n_cu;
      o.attend.q = o.attend.out = some;
      o.attend.row_start = ints;
      o.attend.cache = c;
      o.tree = reinterpret_cast<uint64_t*>(some);
    }
    std::string e = check_step(op);
    StepLaunch first, l;
    if (e.empty()) e = encode_step(t, op, n_cu, &first, &l);
    if (!e.empty()) {
      printf("error %s\n", e.c_str());
      continue;
    }
    printf("%d %u %u %u %zu %zu", (int)l.k.object, l.groups, l.threads, l.k.lds, l.part_bytes, l.counters);
    if (!l.groups) {
    } else if (what == "sample") {
      SampleArgs a;
      std::memcpy(&a, l.args, sizeof a);
      printf(" %u %d %d %d", first.groups, a.parts, a.part_chunks, a.chunks);
    } else if (what == "copy") {
      CopyArgs a;
      std::memcpy(&a, l.args, sizeof a);
      printf(" %d", a.pieces);
    } else if (what == "append") {
      TreeAppendArgs a;
      std::memcpy(&a, l.args, sizeof a);
      printf(" %d %d %d", a.append.items, a.append.q_items, a.tree.words);
    } else if (what == "attend") {
      TreeAttendArgs a;
      std::memcpy(&a, l.args, sizeof a);
      printf(" %d %d %d %d", a.attend.group, a.attend.target, a.attend.units, a.tree.words);
    }
    printf("\n");
  }
  return 0;
}
