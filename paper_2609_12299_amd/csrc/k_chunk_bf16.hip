// k_chunk_bf16.hip -- the kernels of attention of chunks for one pair of types (k_chunk.h).
#include "k_chunk.h"

namespace argus {
namespace prompt {
void launch_chunk_bf16(const ChunkArgs& a, uint32_t grid, hipStream_t st) { launch_chunk_type<0, false>(a, grid, st); }
}  // namespace prompt
}  // namespace argus
