// k_chunk_fp16_f8.hip -- the kernels of attention of chunks for one pair of types (k_chunk.h).
#include "k_chunk.h"

namespace argus {
namespace prompt {
void launch_chunk_fp16_f8(const ChunkArgs& a, uint32_t grid, hipStream_t st) { launch_chunk_type<1, true>(a, grid, st); }
}  // namespace prompt
}  // namespace argus
