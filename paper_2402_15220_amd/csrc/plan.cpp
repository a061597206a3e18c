// Decode plan of windowed calls and of 4-bit caches; see plan.hpp.
#include "plan.hpp"

#include <algorithm>
#include <numeric>

namespace ca {

// Rows of their own go to single wavefronts where those get at least
// kSoloTokens tokens on average, and where a row has no more than kSoloShort:
// a block's four wavefronts would mostly wait for each other.
constexpr int64_t kSoloTokens = 256, kSoloShort = 128;

void build_plan(const ChunkTree& tree, const Tables& tab, int32_t window, int32_t sinks, int32_t heads,
                int32_t num_cus, int32_t waves_per_cu, Plan* out) {
  Plan& P = *out;
  const int32_t B = static_cast<int32_t>(tab.row_seq.size());
  const int32_t nn = static_cast<int32_t>(tab.node_slot.size());
  const int32_t C = tree.chunk_size();
  P = Plan();
  P.window = window;
  P.sinks = sinks;

  std::vector<int32_t> lo(B);  // first position of each row's window
  for (int32_t r = 0; r < B; ++r) {
    const int64_t len = tree.seqs().at(tab.row_seq[r]).length;
    lo[r] = static_cast<int32_t>(std::max<int64_t>(0, len - window));
  }

  // Runs in level order, so a run's parent comes before it.
  struct Run {
    int32_t row_begin, row_end, lo, parent, ord = 0;
    std::vector<int32_t> seen;  // visible nodes, root -> leaf
    int64_t tokens = 0;
    int32_t pieces = 0;
    bool solo = false;
  };
  std::vector<Run> runs;
  std::vector<int32_t> run_of(nn);
  for (int32_t i = 0; i < nn; ++i) {
    const int32_t p = tab.node_parent[i], rb = tab.node_row_begin[i], re = tab.node_row_end[i];
    if (p >= 0 && tab.node_row_begin[p] == rb && tab.node_row_end[p] == re) {
      run_of[i] = run_of[p];
    } else {
      run_of[i] = static_cast<int32_t>(runs.size());
      Run r;
      r.row_begin = rb;
      r.row_end = re;
      r.lo = *std::min_element(lo.begin() + rb, lo.begin() + re);
      r.parent = p < 0 ? -1 : run_of[p];
      runs.push_back(std::move(r));
    }
    Run& r = runs[run_of[i]];
    const int32_t start = tab.node_start_pos[i], end = start + tab.node_len[i];
    if (start < sinks || end > r.lo) {
      r.seen.push_back(i);
      // tokens read: the part in the window and the sinks
      r.tokens += end - std::max(start, std::min(end, r.lo)) +
                  std::max(0, std::min({end, sinks, std::max(start, r.lo)}) - start);
    }
  }

  // Pieces: as many as the chip is to have at once, of at least 128 tokens.
  int64_t load = 0, own = 0;
  for (const Run& r : runs) {
    const int64_t tiles = (r.row_end - r.row_begin + kPlanRows - 1) / kPlanRows;
    load += tiles * r.tokens * heads;
    if (r.row_end - r.row_begin == 1) own += r.tokens * heads;
  }
  const int64_t waves = static_cast<int64_t>(waves_per_cu) * num_cus;
  const int64_t piece_tokens = std::max<int64_t>(128, 4 * load / waves);
  const int64_t solo_tokens = own / waves >= kSoloTokens ? own / waves * 5 / 2 : kSoloShort;
  auto chunks_of = [&](int64_t tokens) {
    return static_cast<int32_t>(std::min<int64_t>(kPlanChunks - 2, std::max<int64_t>(1, (tokens + C - 1) / C)));
  };
  int32_t longest = 0;
  for (Run& r : runs) {
    const int32_t n = static_cast<int32_t>(r.seen.size());
    r.solo = r.row_end - r.row_begin == 1 && r.tokens <= solo_tokens;
    const int32_t len = chunks_of(r.solo ? solo_tokens : piece_tokens);
    r.pieces = (n + len - 1) / len;
    if (r.parent >= 0) r.ord = runs[r.parent].ord + runs[r.parent].pieces;
    if (r.pieces) longest = std::max(longest, (n + r.pieces - 1) / r.pieces);
  }
  P.stride = longest + 2;  // room for growth

  P.rows.resize(B);
  P.first_item.assign(B, -1);
  P.last_item.assign(B, -1);
  for (int32_t r = 0; r < B; ++r) {
    const int32_t leaf = tab.path_node[tab.path_ptr[r + 1] - 1];
    const Run& run = runs[run_of[leaf]];
    const int32_t np = run.ord + run.pieces;
    P.rows[r] = {tab.node_slot[leaf], tab.node_start_pos[leaf], np > 1 ? P.n_parts : -1, np};
    if (np > 1) P.n_parts += np;
  }

  // Shared runs first: their blocks work on up to 16 rows each; then single
  // rows, those of a wavefront a head last; of each kind the longest items first,
  // so that the launch does not end on a long one (128 rows of 64 to 1,024 tokens
  // of their own behind 2,048 shared ones, 4 bits: in tree order 72.7 us, so 59.0).
  std::vector<int32_t> order(runs.size());
  std::iota(order.begin(), order.end(), 0);
  std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) {
    return runs[a].tokens * std::max(1, runs[b].pieces) > runs[b].tokens * std::max(1, runs[a].pieces);
  });
  for (int pass = 0; pass < 3; ++pass) {
    if (pass == 2) P.n_block_items = static_cast<int32_t>(P.items.size());
    for (const int32_t at_run : order) {
      const Run& r = runs[at_run];
      const bool shared = r.row_end - r.row_begin > 1;
      if (pass != (shared ? 0 : r.solo ? 2 : 1)) continue;
      const int32_t n = static_cast<int32_t>(r.seen.size());
      for (int32_t k = 0; k < r.pieces; ++k) {
        const int32_t c0 = static_cast<int32_t>(static_cast<int64_t>(n) * k / r.pieces);
        const int32_t c1 = static_cast<int32_t>(static_cast<int64_t>(n) * (k + 1) / r.pieces);
        // even tiles: a shared run's never have one row only
        const int32_t rows = r.row_end - r.row_begin, tiles = (rows + kPlanRows - 1) / kPlanRows;
        for (int32_t t = 0; t < tiles; ++t) {
          const int32_t rb = r.row_begin + rows * t / tiles, re = r.row_begin + rows * (t + 1) / tiles;
          const size_t at = P.chunks.size();
          P.chunks.resize(at + P.stride, PlanChunk{0, 0, 0, 0});
          for (int32_t c = c0; c < c1; ++c) {
            const int32_t i = r.seen[c], start = tab.node_start_pos[i];
            const bool open = !shared && c == n - 1;
            P.chunks[at + c - c0] = {tab.node_slot[i], start, open ? kOpenEnd : start + tab.node_len[i], 0};
          }
          if (!shared) {
            P.last_item[rb] = static_cast<int32_t>(P.items.size());
            if (k == 0) P.first_item[rb] = P.last_item[rb];
          }
          const int32_t ilo = *std::min_element(lo.begin() + rb, lo.begin() + re);
          PlanItem it{rb, re - rb, c1 - c0, r.ord + k, ilo, 0, 0, -1, 0, {0, 0, 0}};
          if (!shared) {
            const PlanRow& pr = P.rows[rb];
            it.last_slot = pr.last_slot;
            it.last_start = pr.last_start;
            it.pbase = pr.pbase;
            it.np = pr.np;
          }
          P.items.push_back(it);
        }
      }
    }
  }
}

bool patch_plan(const ChunkTree& tree, const std::unordered_map<int64_t, int32_t>& row_of_seq, Plan* p) {
  std::vector<int32_t> added(p->items.size(), 0);
  for (const auto& g : tree.grown()) {
    const auto it = row_of_seq.find(g.first);
    if (it == row_of_seq.end() || p->last_item[it->second] < 0) return false;
    const int32_t i = p->last_item[it->second];
    if (p->items[i].n_chunks + ++added[i] > p->stride) return false;
  }
  for (const auto& g : tree.grown()) {
    const int32_t row = row_of_seq.at(g.first), i = p->last_item[row];
    PlanRow& r = p->rows[row];
    PlanItem& item = p->items[i];
    PlanChunk* c = p->chunks.data() + static_cast<size_t>(i) * p->stride;
    const Node& nd = tree.node(g.second);
    // the chunk that was last is full now
    const int32_t start = r.last_start + static_cast<int32_t>(tree.node(nd.parent).tokens.size());
    c[item.n_chunks - 1].end = start;
    c[item.n_chunks] = {nd.slot, start, kOpenEnd, 0};
    ++item.n_chunks;
    r.last_slot = nd.slot;
    r.last_start = start;
    for (int32_t k = p->first_item[row]; k <= i; ++k) {
      p->items[k].last_slot = nd.slot;
      p->items[k].last_start = start;
    }
  }
  return true;
}

}  // namespace ca
