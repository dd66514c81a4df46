// Launch interface of the kernels between a projection's rows and the cache:
// norms and rotations of queries and keys (rope.hip), and the writes into a
// cache of 8-bit codes (kvq.hip).
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

namespace spork {

// What happens to a head of queries or keys: its norm, then its rotation.
struct TurnArgs {
  const double* inv_freq;  // [rotary_dim / 2] radians per position
  int32_t rotary_dim;      // 0: no rotation
  int32_t interleaved;
  double magnitude;
  const void* q_weight;  // nullptr: no norms
  const void* k_weight;
  double eps;
};

struct RopeArgs {
  TurnArgs turn;
  const int32_t* positions;  // nullptr: no rotation, every row is one
  const void* q;
  const void* k;
  void* q_out;
  void* k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;  // elements between rows
  int32_t n_rows, hq, hkv, head_dim, dtype;                // hq or hkv 0: not given
};

// The cache's pools: codes, and a scale byte for each block and head.
struct KvqPools {
  uint8_t* k_codes;
  uint8_t* v_codes;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int32_t num_blocks;
};

struct KvqWriteArgs {
  TurnArgs turn;
  KvqPools pools;
  const int64_t* slots;
  const int32_t* positions;  // read where there is a rotation
  const void* q;             // nullptr: keys and values only
  const void* k;
  const void* v;
  void* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  int32_t* bad_slots;  // nullable
  int32_t n_rows, hq, hkv, head_dim, block_size, dtype;
  int32_t window;           // rows whose runs a workgroup takes (launch_kvq_write)
  int32_t phases, stretch;  // order of the windows: stretch of each phase
};

// Head and block sizes that there are kernels for.
bool rows_supported(int32_t dtype, int32_t head_dim);
bool kvq_supported(int32_t dtype, int32_t head_dim, int32_t block_size);
hipError_t launch_qk_rope(const RopeArgs& a, hipStream_t stream);
hipError_t launch_kvq_write(const KvqWriteArgs& a, hipStream_t stream);
hipError_t launch_kvq_copy_batch(const KvqPools& p, int32_t hkv, int32_t head_dim, int32_t block_size, const int32_t* copies,
                                 const int32_t* n_copies, int32_t max_copies, hipStream_t stream);

}  // namespace spork
