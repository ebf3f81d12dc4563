// Work list of the chunk attention: host code, integers only, shared with the kernels that read it.
#pragma once
#include <cstdint>
#include <vector>

namespace libra {

// A chunk's query rows are flattened per KV head: row r of a sequence is query token r / G, head r % G of the group, so
// that any group size fills the tiles without padding.
constexpr int kChunkTileRows = 128;                  // rows of one score tile (the M of a tensor-core instruction)
constexpr int kChunkItemRows = 2 * kChunkTileRows;   // rows of one item
constexpr int kChunkKvTile = 128;                    // cached tokens of one step
constexpr int kChunkMaxSplits = 64;                  // chunks of one item's KV range at most
// A sequence's cached tokens at most: the kernel's 32-bit token numbers run up to two steps past the end.
constexpr int32_t kChunkMaxLen = 0x7fffffff - 4 * kChunkKvTile + 1;

struct ChunkItem {   // one block's work, for one KV head: 32 bytes, read as two 16-byte vectors
  int32_t b;         // row of the block table
  int32_t q_start;   // first row of the sequence in the packed q
  int32_t row0;      // first flattened row
  int32_t n_rows;    // 1 .. kChunkItemRows
  int32_t kv_begin;  // cached tokens [kv_begin, kv_end); kv_begin is a multiple of kChunkKvTile
  int32_t kv_end;
  int32_t ctx;       // seq_len - q_len: query token i sees cached tokens 0 .. ctx + i (negative: the first ones see nothing)
  int32_t slot;      // first row of the partial results, or -1: the KV range is whole and the output is written
};

struct ChunkMerge {  // one split item, for the merge kernel
  int32_t q_start, row0, n_rows;
  int32_t slot;      // partial rows of chunk j: slot + j * n_rows
  int32_t n_chunks;
  int32_t pad[3];
};

struct ChunkPlan {
  std::vector<ChunkItem> items;    // longest first
  std::vector<ChunkMerge> merges;
  int64_t partial_rows = 0;        // per KV head
};

// Partial rows (times KV heads) a plan may use on a device of n_sm multiprocessors: sizes the workspace.
inline int64_t chunk_max_partial_rows(int n_sm) { return int64_t(2) * n_sm * kChunkItemRows; }
// Items of any plan for up to max_tokens new tokens of up to max_batch sequences.
int64_t chunk_max_items(int n_sm, int group, int64_t max_tokens, int64_t max_batch);

// false: a negative length, one beyond kChunkMaxLen, or more rows than 32 bits count.
bool make_chunk_plan(int n_sm, int num_q_heads, int num_kv_heads, const int32_t* q_lens, const int32_t* seq_lens, int32_t batch,
                     ChunkPlan* plan);

}  // namespace libra
