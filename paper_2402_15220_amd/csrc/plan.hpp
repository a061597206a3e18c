// Decode plan: the work of a decode call whose rows may see a sliding window
// and sinks of their paths instead of all of it, and of every decode call
// over a 4-bit cache.
//
// The tree is cut into runs (maximal chains of chunks that the same rows
// cover). Of each run the chunks that some row sees, at the time the plan is
// made, are cut into pieces of about the same number of tokens, and the run's
// rows into tiles of up to 16; an item is one piece and one tile. Of most
// items a block of the launch works on one head, its four wavefronts on the
// tokens in turn; where single rows are long and many enough, a wavefront
// takes a head of an item to itself and a block four heads (no fold, and what
// a wavefront does once is spread over four times the tokens). Sequences only grow while the
// plan stands, so their windows only move forward and what it lists stays a
// superset of what they see; the kernel masks by the lengths on the device.
//
// Every row covered by a run takes one partial from each of the run's pieces,
// so a piece has the same place (ord) in the partial lists of all its rows:
// row r's partials are pbase[r] .. pbase[r] + np[r] - 1. A row with one piece
// (np = 1) has no partial, its item writes o.
#pragma once

#include <cstdint>
#include <vector>

#include "tables.hpp"
#include "tree.hpp"

namespace ca {

constexpr int kPlanRows = 16;          // rows of an item at most
constexpr int kPlanChunks = 64;        // chunks of an item at most
constexpr int32_t kNoWindow = 0x3fffffff;
// Tokens of a chunk at most: a unit's number (64 tokens, below 2^24 of them in 30
// bits of positions) times the units of a chunk then stays below 2^32, as the
// kernels' divisions need.
constexpr int32_t kWindowChunk = 16384;
constexpr int32_t kOpenEnd = 0x3fffffff;  // end of a chunk that may still be filled

struct PlanItem {
  int32_t row_begin;
  int32_t n_rows;
  int32_t n_chunks;
  int32_t ord;
  int32_t lo;  // no row of the item sees a position below lo that is no sink
  // of an item of one row, the row's PlanRow (one load less in a row's chain)
  int32_t last_slot, last_start, pbase, np;
  int32_t pad[3];
};
struct PlanChunk {
  int32_t slot;
  int32_t start;  // position of its first token
  int32_t end;    // position after its last one, kOpenEnd for a row's last chunk
  int32_t pad;
};
struct PlanRow {
  int32_t last_slot;   // the row's length is last_start + slot_len[last_slot]
  int32_t last_start;
  int32_t pbase;       // -1: one piece only
  int32_t np;
};
static_assert(sizeof(PlanItem) == 48 && sizeof(PlanChunk) == 16 && sizeof(PlanRow) == 16, "plan layout");

struct Plan {
  std::vector<PlanItem> items;
  std::vector<PlanChunk> chunks;  // [items][stride]
  std::vector<PlanRow> rows;
  // per row the items of its own chunks, [first, last], the last one ending in
  // the row's last chunk; -1: none
  std::vector<int32_t> first_item, last_item;
  int32_t stride = 0;
  int32_t n_parts = 0;
  int32_t window = 0, sinks = 0;
  int32_t n_block_items = 0;  // items whose tokens a block's four wavefronts share
};

// heads x items is the launch; the pieces are sized for waves_per_cu wavefronts
// on each of num_cus compute units.
void build_plan(const ChunkTree& tree, const Tables& t, int32_t window, int32_t sinks, int32_t heads,
                int32_t num_cus, int32_t waves_per_cu, Plan* out);

// Append the chunks that decode growth added (tree.grown()) to their rows'
// last items; false (the plan is then to be rebuilt) where one has no room.
bool patch_plan(const ChunkTree& tree, const std::unordered_map<int64_t, int32_t>& row_of_seq, Plan* p);

}  // namespace ca
