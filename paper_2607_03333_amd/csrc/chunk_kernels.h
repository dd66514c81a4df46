// Launch interface of the attention of a chunk of new tokens over the paged
// cache (chunk.hip).
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace spork {

constexpr int kChunkSlices = 256;    // workgroups of the attention launch: one per compute unit
constexpr int kChunkTileRows = 256;  // packed rows (query row x head of a KV head's group) of a tile

// A tile whose tokens are split over slices `first` .. `last`, as the slice
// that holds its first token notes it for the merge; n_rows 0: none.
struct ChunkSplit {
  int32_t row0;       // query row of the tile's first packed row
  int32_t head;       // first KV head
  int32_t n_rows;     // packed rows of a KV head
  int32_t row_tiles;  // row tiles of a KV head
  int32_t heads;      // KV heads
  int32_t last;
};

struct ChunkArgs {
  const void* q;
  int64_t q_stride;  // elements between query rows
  const void* k_cache;
  const void* v_cache;
  const int32_t* table;
  const int32_t* row_off;
  const int32_t* kv_len;
  void* out;
  float* lse;  // nullptr: not wanted
  int32_t num_blocks, max_blocks, n_seqs, n_rows;
  int32_t hq, hkv, head_dim, block_size, dtype;
  int32_t group, tile_rows;  // query heads per KV head, query rows of a tile (kChunkTileRows / group)
  int32_t most_heads;        // KV heads of a tile, at most (chunk_tile_heads)
  float scale_log2;          // sm_scale * log2(e)
  // workspace
  ChunkSplit* splits;   // [kChunkSlices]
  int32_t* continues;   // [kChunkSlices] 1: the slice holds a piece of a tile that began before it
  float* part_ml;       // [kChunkSlices][2][kChunkTileRows][2] running max (base 2) and sum
  float* part_o;        // [kChunkSlices][2][kChunkTileRows][D] unnormalised outputs
};

// KV heads that a tile of a sequence with few rows may take together: a power of
// two that leaves a tile for every compute unit.
int32_t chunk_tile_heads(int32_t n_seqs, int32_t hkv);
bool chunk_supported(int32_t dtype, int32_t head_dim, int32_t block_size);
size_t chunk_workspace_bytes(int32_t head_dim);
void chunk_workspace(ChunkArgs* a, void* workspace);
hipError_t launch_chunk_attn(const ChunkArgs& a, hipStream_t stream);
hipError_t launch_chunk_merge(const ChunkArgs& a, hipStream_t stream);

}  // namespace spork
