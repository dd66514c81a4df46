// Launch interface of the attention of a chunk of new tokens over the paged
// cache (chunk.hip).
#pragma once

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace spork {

constexpr int kChunkSlices = 256;    // workgroups of the attention launch: one per compute unit
constexpr int kChunkTileRows = 256;  // packed rows (query row x head of a KV head's group) of a tile
constexpr int kChunkWaves = 8;       // of a workgroup: a unit (a KV head and a row tile of 32 packed rows) each

// KV heads that a tile of so many row tiles takes together, `most` (a power of two) in its
// batch. Tiles of more than NARROW row tiles, whose waves share their stages, are of one head.
template <int NARROW>
constexpr int chunk_heads(int most, int row_tiles) {
  if constexpr (2 * (NARROW + 1) <= kChunkWaves) {  // (else the waves don't suffice for a second head)
    if (row_tiles > NARROW) return 1;
  }
  return std::min(most, kChunkWaves / row_tiles);
}

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
  // of a cache of 8-bit codes: [num_blocks][hkv]
  const uint8_t* k_scale;
  const uint8_t* v_scale;
};

// KV heads that a tile of a sequence with few rows may take together: a power of
// two that leaves a tile for every compute unit.
int32_t chunk_tile_heads(int32_t n_seqs, int32_t hkv);
bool chunk_supported(int32_t dtype, int32_t head_dim, int32_t block_size);
size_t chunk_workspace_bytes(int32_t head_dim);
void chunk_workspace(ChunkArgs* a, void* workspace);
hipError_t launch_chunk_attn(const ChunkArgs& a, hipStream_t stream);
// the same over a cache of 8-bit codes (chunk_kvq.hip)
hipError_t launch_kvq_attn(const ChunkArgs& a, hipStream_t stream);
hipError_t launch_chunk_merge(const ChunkArgs& a, hipStream_t stream);

}  // namespace spork
