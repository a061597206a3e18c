// Random trees through build_plan and patch_plan: every (row, position) that
// the row sees lies in exactly one chunk of one of the row's items, the places
// of a row's items in its partial list are 0 .. np - 1, and the patched plans
// of growing trees keep both properties.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>

#include "plan.hpp"

using namespace ca;

static int check(const ChunkTree& tree, const Plan& P, int window, int sinks, const char* what) {
  Tables t;
  build_tables(tree, &t);
  const int B = static_cast<int>(t.row_seq.size());
  if (static_cast<int>(P.rows.size()) != B) return std::printf("%s: rows\n", what), 1;
  std::vector<std::vector<int>> hits(B);
  std::vector<std::set<int>> ords(B);
  std::vector<long> len(B);
  std::set<int> bases;
  for (int r = 0; r < B; ++r) {
    len[r] = tree.seqs().at(t.row_seq[r]).length;
    hits[r].assign(len[r], 0);
    const int leaf = t.path_node[t.path_ptr[r + 1] - 1];
    if (P.rows[r].last_slot != t.node_slot[leaf] || P.rows[r].last_start != t.node_start_pos[leaf])
      return std::printf("%s: last chunk of row %d\n", what, r), 1;
  }
  for (size_t i = 0; i < P.items.size(); ++i) {
    const PlanItem& it = P.items[i];
    if (it.n_rows < 1 || it.n_rows > kPlanRows || it.n_chunks < 1 || it.n_chunks > P.stride ||
        P.stride > kPlanChunks || it.row_begin < 0 || it.row_begin + it.n_rows > B)
      return std::printf("%s: item %zu\n", what, i), 1;
    if (it.n_rows == 1 && !(P.first_item[it.row_begin] >= 0 && static_cast<int>(i) >= P.first_item[it.row_begin] &&
                            static_cast<int>(i) <= P.last_item[it.row_begin] &&
                            it.last_slot == P.rows[it.row_begin].last_slot &&
                            it.last_start == P.rows[it.row_begin].last_start && it.pbase == P.rows[it.row_begin].pbase &&
                            it.np == P.rows[it.row_begin].np))
      return std::printf("%s: row of item %zu\n", what, i), 1;
    for (int r = it.row_begin; r < it.row_begin + it.n_rows; ++r) {
      if (!ords[r].insert(it.ord).second) return std::printf("%s: ord twice\n", what), 1;
      const long lo = len[r] > window ? len[r] - window : 0;
      if (it.lo > lo) return std::printf("%s: lo\n", what), 1;
      for (int c = 0; c < it.n_chunks; ++c) {
        const PlanChunk& ch = P.chunks[i * P.stride + c];
        bool on = false;  // the chunk lies on the row's path at that place
        for (int k = t.path_ptr[r]; k < t.path_ptr[r + 1]; ++k)
          on |= t.node_slot[t.path_node[k]] == ch.slot && t.node_start_pos[t.path_node[k]] == ch.start;
        if (!on) return std::printf("%s: foreign chunk\n", what), 1;
        for (long j = ch.start; j < std::min<long>(ch.end, len[r]); ++j) ++hits[r][j];
      }
    }
  }
  for (int r = 0; r < B; ++r) {
    const long lo = len[r] > window ? len[r] - window : 0;
    for (long j = 0; j < len[r]; ++j) {
      const bool seen = j >= lo || j < sinks;
      if (hits[r][j] > 1 || (seen && hits[r][j] != 1)) return std::printf("%s: row %d position %ld\n", what, r, j), 1;
    }
    const int np = P.rows[r].np;
    if (static_cast<int>(ords[r].size()) != np || *ords[r].begin() != 0 || *ords[r].rbegin() != np - 1)
      return std::printf("%s: places\n", what), 1;
    if ((np == 1) != (P.rows[r].pbase < 0)) return std::printf("%s: base\n", what), 1;
    if (np > 1)
      for (int k = 0; k < np; ++k)
        if (P.rows[r].pbase + k >= P.n_parts || !bases.insert(P.rows[r].pbase + k).second)
          return std::printf("%s: partials overlap\n", what), 1;
  }
  return 0;
}

int main() {
  int patched = 0;
  for (int seed = 0; seed < 60; ++seed) {
    std::mt19937 rng(seed);
    auto in = [&](int a, int b) { return a + static_cast<int>(rng() % (b - a + 1)); };
    const int C = std::vector<int>{1, 3, 16, 20, 64, 100}[seed % 6];
    ChunkTree tree(C, 100000);
    std::vector<int> base(in(1, 500));
    for (int& x : base) x = in(0, 3);
    const int n = in(1, 40);
    for (int s = 0; s < n; ++s) {
      std::vector<int> t(base.begin(), base.begin() + in(0, static_cast<int>(base.size())));
      const int tail = in(t.empty() ? 1 : 0, seed % 4 == 0 ? 3000 : 150);
      for (int k = 0; k < tail; ++k) t.push_back(in(0, 5));
      std::vector<KvJob> jobs;
      int64_t m;
      if (tree.insert(s, t.data(), static_cast<int64_t>(t.size()), &jobs, &m) != Err::ok) return 2;
    }
    for (int round = 0; round < 3; ++round) {
      const int window = std::vector<int>{1, 7, 64, 300, kNoWindow}[in(0, 4)], sinks = in(0, 2) ? in(0, 90) : 0;
      Tables t;
      build_tables(tree, &t);
      Plan P;
      build_plan(tree, t, window, sinks, in(1, 32), 256, in(1, 16), &P);
      std::unordered_map<int64_t, int32_t> row_of;
      for (size_t r = 0; r < t.row_seq.size(); ++r) row_of[t.row_seq[r]] = static_cast<int32_t>(r);
      tree.clear_dirty();
      if (check(tree, P, window, sinks, "built")) return std::printf("seed %d\n", seed), 1;
      for (int step = 0; step < 2 * C + 5 && step < 80; ++step) {
        std::vector<int64_t> ids;
        std::vector<int32_t> tok;
        for (const auto& kv : tree.seqs())
          if (in(0, 2)) {
            ids.push_back(kv.first);
            tok.push_back(in(0, 9));
          }
        std::vector<KvJob> jobs;
        if (tree.append_batch(static_cast<int64_t>(ids.size()), ids.data(), tok.data(), &jobs) != Err::ok) return 2;
        if (!tree.dirty()) {
          if (check(tree, P, window, sinks, "filled")) return std::printf("seed %d\n", seed), 1;
          continue;
        }
        if (!tree.private_growth_only() || !patch_plan(tree, row_of, &P)) break;
        tree.clear_dirty();
        ++patched;
        if (check(tree, P, window, sinks, "patched")) return std::printf("seed %d\n", seed), 1;
      }
      if (tree.num_seqs() > 1 && tree.remove(tree.seqs().begin()->first) != Err::ok) return 2;
    }
  }
  std::printf("ok, %d patches\n", patched);
  return patched > 20 ? 0 : 3;
}
