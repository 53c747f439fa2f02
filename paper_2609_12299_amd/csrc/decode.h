// decode.h -- what the operators of a decode step share: argument checks, the
// markers that their kernels write, page arithmetic.
#pragma once

#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "../../include/argus_decode.h"
#include "internal.h"

namespace argus {
namespace decode {

constexpr int kThreads = 256;  // of a block, where nothing else is said
constexpr int kWaves = kThreads / 64;
constexpr uint32_t kMaxBlocks = (1u << 24) - 1;  // of kThreads: a launch has less than 2^32 threads

// ---------------------------------------------------------------- markers

// Where the waves of one launch write their markers: `per_wave` records each.
struct Marks {
  argus_record* rec;  // NULL: none
  uint32_t ctx, region, per_wave;
};

// A wave's markers.  Without a buffer each costs one scalar branch; with one 0.2 to 0.4 us
// of a short call, 1 to 2 of a long one (79376 of them in a call of 95 us: 97).
struct WaveMarks {
  argus_record* at = nullptr;
  uint32_t ctx = 0, region = 0;
  ARGUS_DEV WaveMarks(const Marks& m) {
    if (m.rec) {
      const uint32_t wave = __builtin_amdgcn_readfirstlane(((blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x) * (blockDim.x / 64) + threadIdx.x / 64);
      at = m.rec + (uint64_t)wave * m.per_wave;
      ctx = m.ctx + wave;
      region = m.region;
    }
  }
  ARGUS_DEV void put(uint32_t r, uint32_t kind) {
    if (at) {
      if (lane_id() == 0) {
        const uint64_t t = wall_clock64();
        *reinterpret_cast<uint4*>(at) = make_uint4((uint32_t)t, (uint32_t)(t >> 32), ctx, (region + r) | (kind << 16));
      }
      ++at;
    }
  }
  ARGUS_DEV void begin(uint32_t r) { put(r, ARGUS_KIND_BEGIN); }
  ARGUS_DEV void end(uint32_t r) { put(r, ARGUS_KIND_END); }
};

// ------------------------------------------------------------------- host

// Sets the message of argus_decode_last_error and returns the code.
int refuse(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void accepted();
int device_ok();

inline bool aligned_to(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline uint32_t type_bytes(uint32_t type) { return type == ARGUS_FP32 ? 4u : type == ARGUS_FP8 ? 1u : 2u; }
inline size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
inline bool power_of_two(uint32_t v) { return v && !(v & (v - 1)); }
inline uint32_t log2_of(uint32_t v) { return 31u - (uint32_t)__builtin_clz(v); }

// Room for a launch's markers: checked for all launches of a call before the
// first, taken by each.
inline bool marks_fit(const argus_markers* m, uint64_t records) {
  return !m || !m->d_records || (m->used <= m->capacity && records <= m->capacity - m->used);
}
inline bool marks_bad(const argus_markers* m) {
  return m && m->d_records && (!aligned_to(m->d_records, 16) || m->region_base > 65536u - ARGUS_NUM_REGIONS);
}
inline Marks take_marks(argus_markers* m, uint64_t blocks, uint32_t per_wave) {
  if (!m || !m->d_records) return Marks{nullptr, 0, 0, 0};
  Marks r{m->d_records + m->used, m->ctx_base, m->region_base, per_wave};
  m->used += blocks * kWaves * per_wave;
  return r;
}
inline int check_view(const argus_page_view& v, uint32_t type, const char* name) {
  if (!v.base) return refuse(ARGUS_E_INVAL, "%s: no cache", name);
  const int64_t e = 16 / type_bytes(type);
  if (!aligned_to(v.base, 16) || v.page_stride % e || v.head_stride % e || v.token_stride % e)
    return refuse(ARGUS_E_ALIGN, "%s: base and strides of a cache are multiples of 16 bytes", name);
  return ARGUS_OK;
}

// n / d for n < 2^31 by a multiplication: m = ceil(2^(31 + s) / d), s = bits of d - 1.
struct FastDiv {
  uint32_t d, m, s;
};
inline FastDiv fast_div(uint32_t d) {
  FastDiv f{d, 0, 0};
  while (f.s < 31 && (1u << f.s) < d) ++f.s;
  f.m = (uint32_t)((((uint64_t)1 << (31 + f.s)) + d - 1) / d);
  return f;
}
ARGUS_DEV uint32_t divide(uint32_t n, const FastDiv& f) { return (uint32_t)(((uint64_t)n * f.m) >> (31 + f.s)); }

}  // namespace decode
}  // namespace argus
