// Kernel launchers of the steps whose lengths live on the GPU, for the
// host-sanitizer build of their entry points (tests only): every launch fails.
#include "chunk_kernels.h"
#include "tables_kernels.h"

namespace spork {

size_t tables_control_bytes(int32_t n) { return 4096 + 12 * static_cast<size_t>(n); }
size_t tables_workspace_bytes(int32_t n, int32_t s) { return tables_control_bytes(n) + 12 * static_cast<size_t>(s); }
void tables_workspace(TablesArgs*, void*) {}
hipError_t launch_tables_init(const TablesArgs&, const int32_t*, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_words_clear(int32_t*, int64_t, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_tables_step(const TablesArgs&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_kv_copy_batch(int32_t, int32_t, int32_t, int32_t, int32_t, void*, void*, const int32_t*, const int32_t*, int32_t,
                                hipStream_t) {
  return hipErrorNoDevice;
}
int32_t chunk_tile_heads(int32_t, int32_t) { return 1; }
bool chunk_supported(int32_t dtype, int32_t d, int32_t bs) {
  return (dtype == 0 || dtype == 1) && (d == 64 || d == 128) && (bs == 16 || bs == 32);
}
size_t chunk_workspace_bytes(int32_t) { return 1 << 20; }
void chunk_workspace(ChunkArgs*, void*) {}
hipError_t launch_chunk_attn(const ChunkArgs&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_chunk_merge(const ChunkArgs&, hipStream_t) { return hipErrorNoDevice; }

}  // namespace spork
