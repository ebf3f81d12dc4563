// Planner of the chunk attention (host, integers only).
#include "chunk_plan.hpp"

#include <algorithm>
#include <queue>

namespace libra {

namespace {

// Time of one block in nanoseconds, for comparing cuts with each other: a fixed part (start, first copies, end), and a part per
// step of 128 cached tokens for items of two row tiles and of one; what the merge of cut items adds; and what a tile of K and
// one of V take of the memory, which all blocks share (64 KB at 6.4 TB/s).  Fitted to the time of 20 batches of 1 to 64 sequences
// with 1 to 2000 new tokens: against 4000 / 1500 / 1300 / 4000 and no shared memory, 128 tokens on 16384 of one sequence
// 65.7 -> 46.9 us, three tokens on eight trajectories of 32K 182 -> 169 us, 10 - 30 tokens on twelve of 1 - 2K 54 -> 45 us.
// All over bf16 pools, and used for E4M3 ones too, whose steps measured 1830 and 1040 ns and whose tiles are half the bytes.
constexpr int64_t kUnitNs = 8500, kPairStepNs = 2100, kSoloStepNs = 1200, kMergeNs = 8000, kTileNs = 10;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Tile {
  ChunkItem item;    // kv range whole
  int64_t steps;     // of 128 cached tokens
};

int64_t unit_ns(const Tile& t, int64_t steps) {
  return kUnitNs + steps * (t.item.n_rows > kChunkTileRows ? kPairStepNs : kSoloStepNs);
}

int n_chunks_for(const Tile& t, int64_t chunk_steps) {
  return int(std::min<int64_t>(std::max<int64_t>(1, ceil_div(t.steps, chunk_steps)), kChunkMaxSplits));
}

// The end of the last block when blocks are handed out longest first to n_sm multiprocessors; -1: over the limits.
int64_t makespan(const std::vector<Tile>& tiles, int n_sm, int heads, int64_t chunk_steps, int64_t max_units,
                 int64_t max_rows) {
  std::vector<int64_t> units;
  int64_t rows = 0, memory = 0;
  bool merged = false;
  for (const Tile& t : tiles) memory += t.steps * heads * kTileNs;
  for (const Tile& t : tiles) {
    const int n = n_chunks_for(t, chunk_steps);
    if (n > 1) {
      rows += int64_t(n) * t.item.n_rows;
      merged = true;
    }
    if (int64_t(units.size()) + int64_t(n) * heads > max_units || rows * heads > max_rows) return -1;
    const int64_t per = ceil_div(t.steps, n), real = per ? ceil_div(t.steps, per) : 1;
    for (int64_t j = 0; j < real; ++j) {
      const int64_t ns = unit_ns(t, std::min(per, t.steps - j * per));
      for (int h = 0; h < heads; ++h) units.push_back(ns);
    }
  }
  std::sort(units.begin(), units.end(), std::greater<int64_t>());
  std::priority_queue<int64_t, std::vector<int64_t>, std::greater<int64_t>> free_at;
  for (int i = 0; i < n_sm; ++i) free_at.push(0);
  int64_t end = 0;
  for (int64_t u : units) {
    const int64_t at = free_at.top() + u;
    free_at.pop();
    free_at.push(at);
    end = std::max(end, at);
  }
  return std::max(end, memory) + (merged ? kMergeNs : 0);
}

}  // namespace

int64_t chunk_max_items(int n_sm, int group, int64_t max_tokens, int64_t max_batch) {
  // whole items and one remainder per sequence with new tokens; cut items are at most 4 n_sm more
  return max_tokens * group / kChunkItemRows + std::min(max_batch, max_tokens) + 4 * int64_t(n_sm) + 1;
}

bool make_chunk_plan(int n_sm, int num_q_heads, int num_kv_heads, const int32_t* q_lens, const int32_t* seq_lens, int32_t batch,
                     ChunkPlan* plan) {
  plan->items.clear();
  plan->merges.clear();
  plan->partial_rows = 0;
  const int group = num_q_heads / num_kv_heads;
  std::vector<Tile> tiles;
  int64_t q_start = 0;
  for (int32_t b = 0; b < batch; ++b) {
    if (q_lens[b] < 0 || seq_lens[b] < 0 || seq_lens[b] > kChunkMaxLen) return false;
    const int64_t rows = int64_t(q_lens[b]) * group;
    if (rows > 0x7fffffff || q_start + q_lens[b] > 0x7fffffff) return false;
    const int64_t ctx = int64_t(seq_lens[b]) - q_lens[b];
    for (int64_t r = 0; r < rows; r += kChunkItemRows) {
      Tile t;
      t.item.b = b;
      t.item.q_start = int32_t(q_start);
      t.item.row0 = int32_t(r);
      t.item.n_rows = int32_t(std::min<int64_t>(kChunkItemRows, rows - r));
      t.item.kv_begin = 0;
      const int64_t last_token = (r + t.item.n_rows - 1) / group;
      t.item.kv_end = int32_t(std::max<int64_t>(0, ctx + last_token + 1));
      t.item.ctx = int32_t(ctx);
      t.item.slot = -1;
      t.steps = ceil_div(t.item.kv_end, kChunkKvTile);
      tiles.push_back(t);
    }
    q_start += q_lens[b];
  }

  // Cut the KV ranges where there are too few blocks to fill the device.  Cut lengths (in steps) that could matter are tried: the
  // total work over half a block to four blocks per multiprocessor, and the longest range in two to twelve.
  int64_t total = 0, longest = 0;
  for (const Tile& t : tiles) {
    total += t.steps * num_kv_heads;
    longest = std::max(longest, t.steps);
  }
  const int64_t max_units = int64_t(4) * n_sm;
  int64_t best_steps = std::max<int64_t>(longest, 1);
  if (int64_t(tiles.size()) * num_kv_heads < max_units) {
    int64_t best = makespan(tiles, n_sm, num_kv_heads, best_steps, max_units, chunk_max_partial_rows(n_sm));
    std::vector<int64_t> lengths;
    for (int quarter = 2; quarter <= 16; ++quarter) {   // quarters of a block per multiprocessor
      lengths.push_back(std::max<int64_t>(1, ceil_div(total * 4, int64_t(n_sm) * quarter)));
    }
    for (int n = 2; n <= 12; ++n) lengths.push_back(ceil_div(longest, n));
    std::sort(lengths.begin(), lengths.end(), std::greater<int64_t>());
    lengths.erase(std::unique(lengths.begin(), lengths.end()), lengths.end());
    for (int64_t steps : lengths) {   // longest first: of ends within 1 % the one with the fewest blocks
      if (steps >= longest) continue;
      const int64_t ns = makespan(tiles, n_sm, num_kv_heads, steps, max_units, chunk_max_partial_rows(n_sm));
      if (ns >= 0 && (best < 0 || ns * 100 < best * 99)) {
        best = ns;
        best_steps = steps;
      }
    }
  }

  for (const Tile& t : tiles) {
    const int n = n_chunks_for(t, best_steps);
    const int64_t per = ceil_div(t.steps, n);
    const int real = per ? int(ceil_div(t.steps, per)) : 1;
    if (real <= 1) {
      plan->items.push_back(t.item);
      continue;
    }
    ChunkMerge m = {};
    m.q_start = t.item.q_start;
    m.row0 = t.item.row0;
    m.n_rows = t.item.n_rows;
    m.slot = int32_t(plan->partial_rows);
    m.n_chunks = real;
    plan->merges.push_back(m);
    for (int j = 0; j < real; ++j) {
      ChunkItem it = t.item;
      it.kv_begin = int32_t(j * per * kChunkKvTile);
      it.kv_end = int32_t(std::min<int64_t>(t.item.kv_end, (j + 1) * per * kChunkKvTile));
      it.slot = int32_t(plan->partial_rows);
      plan->partial_rows += it.n_rows;
      plan->items.push_back(it);
    }
  }
  // longest first; items of equal length stay in row order, so that neighbours share pages in L2
  std::stable_sort(plan->items.begin(), plan->items.end(), [](const ChunkItem& a, const ChunkItem& b) {
    return ceil_div(a.kv_end - a.kv_begin, kChunkKvTile) > ceil_div(b.kv_end - b.kv_begin, kChunkKvTile);
  });
  return true;
}

}  // namespace libra
