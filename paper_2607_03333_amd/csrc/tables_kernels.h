// Launch interface of the kernels that build block tables and slots on the GPU
// from request lengths, and of the batched block copy that follows them.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace spork {

// What the launches of a step leave each other: row results in row order and
// the step's totals. All of it lies in the workspace, behind the block words.
struct TablesTotals {
  int32_t error;         // lowest status of the rows, 0 between steps
  int32_t pad0;
  int32_t status;        // the step's status
  int32_t front;         // the queue's front before the step
  int32_t frees, takes;  // of all rows
  int32_t pad1[2];
};

struct TablesArgs {
  int32_t num_blocks, block_size, n_seqs, max_blocks, max_tokens;
  int32_t* table;
  int32_t* held;
  int32_t* refcount;
  int32_t* free_queue;
  int32_t* queue;
  const int32_t* lens;
  const int32_t* n_new;
  const int32_t* parents;  // nullptr: no forks
  int64_t* slots;
  int32_t* positions;  // nullptr: not wanted
  int32_t* row_off;
  int32_t* kv_len;
  int32_t* copies;
  int32_t* n_copies;
  int32_t* status;
  // workspace: words per block that are zero between steps ...
  int32_t* last_release;  // 1 + the last place (row * max_blocks + column) that releases the block
  int32_t* sharers;       // rows that append inside the block
  int32_t* last_sharer;   // 1 + the last of them
  // ... and per row
  int32_t* frees;      // blocks that the row's releases put into the queue
  int32_t* takes;      // blocks that the row takes from it
  int32_t* copies_of;  // 1: the row makes a copy
  int32_t* free_off;   // sums of these over the rows before (free_off: where tables_sum makes them); copy_off: -1 where
                       // the row makes no copy
  int32_t* take_off;
  int32_t* copy_off;
  TablesTotals* totals;
};

size_t tables_workspace_bytes(int32_t num_blocks, int32_t n_seqs);
// the words that have to be zero between steps: all of the workspace's block words and totals
size_t tables_control_bytes(int32_t num_blocks);
void tables_workspace(TablesArgs* a, void* workspace);

hipError_t launch_tables_init(const TablesArgs& a, const int32_t* free_order, hipStream_t stream);
hipError_t launch_words_clear(int32_t* words, int64_t n, hipStream_t stream);
hipError_t launch_tables_step(const TablesArgs& a, hipStream_t stream);
hipError_t launch_kv_copy_batch(int32_t elem_bytes, int32_t hkv, int32_t head_dim, int32_t block_size, int32_t num_blocks,
                                void* k_cache, void* v_cache, const int32_t* copies, const int32_t* n_copies,
                                int32_t max_copies, hipStream_t stream);

}  // namespace spork
