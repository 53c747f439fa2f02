// k_attend_fp16_f8.hip -- the attention kernels of one pair of types (k_attend.h).
#include "k_attend.h"

namespace argus {
namespace decode {
void launch_attend_fp16_f8(const AttendArgs& a, uint32_t grid, hipStream_t st) { launch_attend_type<1, true>(a, grid, st); }
}  // namespace decode
}  // namespace argus
