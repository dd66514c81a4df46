// Kernel launchers between a projection's rows and the cache, for the
// host-sanitizer build of their entry points (tests only): every launch fails.
#include "chunk_kernels.h"
#include "rows_kernels.h"

namespace spork {

bool rows_supported(int32_t dtype, int32_t d) { return (dtype == 0 || dtype == 1) && (d == 64 || d == 128); }
bool kvq_supported(int32_t dtype, int32_t d, int32_t bs) { return rows_supported(dtype, d) && (bs == 16 || bs == 32); }
hipError_t launch_qk_rope(const RopeArgs&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_kvq_write(const KvqWriteArgs&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_kvq_copy_batch(const KvqPools&, int32_t, int32_t, int32_t, const int32_t*, const int32_t*, int32_t, hipStream_t) {
  return hipErrorNoDevice;
}
int32_t chunk_tile_heads(int32_t, int32_t) { return 1; }
size_t chunk_workspace_bytes(int32_t) { return 1 << 20; }
void chunk_workspace(ChunkArgs*, void*) {}
hipError_t launch_kvq_attn(const ChunkArgs&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_chunk_merge(const ChunkArgs&, hipStream_t) { return hipErrorNoDevice; }

}  // namespace spork
