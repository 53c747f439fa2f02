// prompt.h -- what the operators of a prompt's pass share.
#pragma once

#include "../../include/argus_prompt.h"
#include "decode.h"

namespace argus {
namespace prompt {

using namespace decode;

inline bool marks_bad_all(const argus_markers* m) {
  return m && m->d_records && (!aligned_to(m->d_records, 16) || m->region_base > 65536u - ARGUS_NUM_ALL_REGIONS);
}

// The rows of sequence s, within [0, rows) whatever the offsets hold.
ARGUS_DEV uint32_t row_at(const int32_t* offsets, uint32_t s, uint32_t rows) {
  const int32_t r = offsets[s];
  return r < 0 ? 0u : ((uint32_t)r < rows ? (uint32_t)r : rows);
}

}  // namespace prompt
}  // namespace argus
