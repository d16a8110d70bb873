// Argument blocks of the operators of a generation step (include/daris_ops.h), shared by the host and the kernels.
#pragma once
#include <cstdint>

namespace daris {

constexpr int kPage = 64;         // tokens of a page
constexpr int kScaleTokens = 16;  // tokens that share a scale

struct NormArgs {
  const void* x;
  const void* res;
  const void* weight;
  void* sum;
  void* y;
  uint8_t* scale;
  int64_t x_row, res_row, sum_row, y_row;
  int rows, width, group, vectors;  // vectors: 16-byte pieces of a row
  float eps, inv_width;
};

struct CacheArgs {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  const int32_t* pages;
  const int32_t* before;
  const int32_t* row_start;  // null: row s is sequence s's
  int64_t pages_row;
  int n_pages, n_seqs, kv_heads, n_rows;
};

// Masks of the step's rows, where these are nodes of trees: [n_rows][words].
struct TreeMasks {
  const uint64_t* mask;
  int words;
};

struct AppendArgs {
  CacheArgs c;
  const void* k;
  const void* v;
  const void* q;
  void* q_out;
  const float* turn;
  int64_t k_row, k_head, v_row, v_head, q_row, q_head, qo_row, qo_head;
  int q_heads, turn_rows, rot_dim, pairs;
  int items, q_items;  // sixteenths x key heads at most; (row, kTurnHeads query heads)
};
constexpr int kTurnHeads = 4;
// Waves to a sixteenth of a tree's nodes: one for the keys, one for the values.
constexpr int kTreeAppendWaves = 2;
struct TreeAppendArgs {
  AppendArgs append;  // (items: times kTreeAppendWaves)
  TreeMasks tree;
};

struct AttendArgs {
  CacheArgs c;
  const void* q;
  void* out;
  int64_t q_row, q_head, out_row, out_head;
  float* part;      // what units of one tile leave for each other: see part_numbers
  uint32_t* count;  // arrivals of a tile's units, zero between launches
  int group;        // query heads of a key head
  int window;
  int target;       // units to aim at for each key head, 0 = one a tile
  int units;        // launched units for each key head, at most
  int round;        // workgroups of a key head that have a CU each
  float scale;      // times log2(e)
  int q_vec, out_vec;  // rows of q are 16-byte vectors; four channels of out are one vector
};
struct TreeAttendArgs {
  AttendArgs attend;
  TreeMasks tree;
};

constexpr int kNarrowColumns = 16, kWideColumns = 128;  // columns (query heads of a row) of a unit
constexpr int kNarrowUnits = 256, kWideUnits = 16;      // units of a tile, at most
// bytes of LDS
constexpr int narrow_numbers(int dim) {
  return 4 * kNarrowColumns * (dim + 4) > 2 * kNarrowUnits * kNarrowColumns ? 4 * kNarrowColumns * (dim + 4) : 2 * kNarrowUnits * kNarrowColumns;
}
constexpr int narrow_lds(int dim) { return (narrow_numbers(dim) + 8 * kNarrowColumns + 4) * 4; }
constexpr int wide_numbers(int dim) { return 2 * 2 * kPage * dim / 2 > 2 * kWideUnits * kWideColumns ? 2 * 2 * kPage * dim / 2 : 2 * kWideUnits * kWideColumns; }
constexpr int wide_lds(int dim) { return (wide_numbers(dim) + 4) * 4; }
// numbers of a unit in AttendArgs::part
constexpr int64_t unit_floats(int columns, int dim) { return (int64_t)columns * (dim + 2); }

// Rows of a block, waves of a workgroup; pieces of x (8 channels) and of the weights' scales (8 of them) that a thread stages at
// a time; the distance of the scales' rows in LDS, an odd number of words.
constexpr int kMatvecRows = 16, kMatvecWaves = 16;
constexpr int matvec_pieces(int parts) { return parts == 2 ? 4 : 8; }
constexpr int kScalePieces = 2;
constexpr int matvec_pitch(int scales) { return (scales + 7) / 8 * 8 + 2; }
struct MatvecArgs {
  const void* x;
  const uint8_t* x_scale;
  const uint8_t* w;
  const uint16_t* w_scale;
  void* y;
  int64_t x_row, w_row, y_row;
  int rows, n, k, gate;
  int x_vec;   // rows of x are 16-byte vectors (8-byte ones of codes)
  int steps;   // of 128 channels, in a chunk of K that LDS holds
  int chunk;   // log2 of them, rounded up
  int chunks;
  int across;  // log2 of a workgroup's tiles (16 outputs) side by side; its other waves share them
  int groups;  // of so many tiles
  int wgs;     // units of a block of rows: workgroups, or sets of them that share K
  int shares, share_steps;  // workgroups that share K, where there are few tiles; steps of each
  float* part;              // what they add to the outputs: [unit][share][rows of a block][outputs of a group]
  uint32_t* count;          // arrivals of a unit's shares, zero between launches
  int eights;  // log2 of the pieces of scales that a tile's row has in a chunk, rounded up
  int pitch;   // matvec_pitch of a chunk
};

struct SampleArgs {
  const void* logits;
  const float* temperature;  // null: 1
  const float* top_p;        // null: all, as the next two
  const float* min_p;
  const int32_t* top_k;
  const float* random;       // null: the largest
  int32_t* word;
  float* chance;             // may be null
  int64_t row;
  int rows, n;
  int chunks;  // of kSampleChunk numbers
  int parts, part_chunks;  // workgroups of a row, chunks of each
  float* part;             // what they leave for the row
  int64_t row_floats;
};
constexpr int kSampleChunk = 512, kSampleMost = 1 << 20;  // numbers that a wave reads at once; of a row, at most
constexpr int kSampleWaves = 16, kSampleSteps = 1024, kSampleFew = 4096, kSampleRank = 512;
constexpr int kSamplePart = 16384, kSampleParts = kSampleMost / (kSamplePart / 2);  // numbers of a part, at most; parts of a row
constexpr int kSampleLds = kSampleMost / kSampleChunk * 12 + kSampleParts * 24 + kSampleSteps * 12 + kSampleFew * 8 + kSampleWaves * 36 + 48;
// numbers of a row in SampleArgs::part: the chunks' largest, their sums, the parts' histograms
constexpr int64_t sample_floats(int chunks, int parts) { return (chunks + 1) / 2 * 2 + 2 * (int64_t)chunks + (int64_t)parts * kSampleSteps * 3; }

struct AcceptArgs {
  const uint64_t* tree;
  const int32_t* words;
  const int32_t* answers;
  const int32_t* row_start;
  const int32_t* before;
  int32_t* path;
  int32_t* count;
  int32_t* word;
  int32_t* after;  // may be null
  int n_rows, n_seqs, tree_words;
};
constexpr int kTreeWords = 16, kTreeNodes = 64 * kTreeWords;  // of a row's mask, at most

struct KeepArgs {
  CacheArgs c;
  const int32_t* path;
  const int32_t* count;
};

struct CopyArgs {
  CacheArgs c;
  const int32_t* pairs;
  int n;
  int pieces;  // of kCopyPiece bytes in a page's keys; as many in its values
};
constexpr int kCopyPiece = 16384;

}  // namespace daris
