// k_select.hip -- beam search's selection over beams and vocabulary.
//
// k_select_rows reads the logits once: a block takes a chunk of one row into
// registers, and gives the sum of its exponentials relative to the largest and
// its k first candidates.  The bound below which nothing has to be looked at comes
// from the threads' own maxima: in `lists` >= k disjoint sets of threads, the
// least of the sets' maxima has at least k elements at or above it, and few more
// (about lists * ln(lists)).  Those are ranked by counting.  Where equal values
// make them too many, the block picks its k one after the other.
//
// k_select_beams, one block per group of beams, joins the chunks' sums to the
// rows' logarithms and picks among the rows' candidates in the same way.
//
// What bounds it: the reading of the logits, and the exponential of each.
#include "decode.h"

namespace argus {
namespace decode {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kItems = 32;                   // elements of a thread
constexpr uint32_t kChunkElems = kItems * kThreads;
constexpr uint32_t kCands = 512;                  // candidates that are ranked by counting
constexpr uint32_t kMaxK = 64, kMaxBeams = 64;

struct SelectArgs {
  const uint8_t* logits;
  int64_t group_stride, beam_stride;  // bytes
  const float* scores;
  const uint8_t* finished;
  float* new_scores;
  int32_t *parents, *tokens;
  uint8_t* new_finished;
  float2* sums;     // [rows][chunks] largest value m, sum of exp(x - m)
  uint64_t* cands;  // [rows][chunks][k] (value, token) as a key, 0: none
  uint32_t W, V, K, chunks, lists;
  int32_t eos;
  Marks marks;
};

// Larger key: larger value, then lower token.  -0 and +0 are one value.
ARGUS_DEV uint32_t order_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
ARGUS_DEV float value_of(uint32_t o) { return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
ARGUS_DEV uint64_t key_of(float x, uint32_t token) { return join64(~token, order_of(x)); }

template <int TYPE>
ARGUS_DEV float element(const uint8_t* p) {
  if constexpr (TYPE == ARGUS_FP32) return *reinterpret_cast<const float*>(p);
  const uint32_t w = *reinterpret_cast<const uint16_t*>(p);
  if constexpr (TYPE == ARGUS_BF16) return __builtin_bit_cast(float, w << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)w);
}
template <int TYPE>
ARGUS_DEV float of_word(uint32_t w, int half) {
  if constexpr (TYPE == ARGUS_FP32) return __builtin_bit_cast(float, w);
  if constexpr (TYPE == ARGUS_BF16) return __builtin_bit_cast(float, half ? w & 0xFFFF0000u : w << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(half ? w >> 16 : w));
}

ARGUS_DEV float wave_max(float v) {
  for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
ARGUS_DEV float wave_sum(float v) {
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void k_select_rows(SelectArgs a) {
  constexpr uint32_t kBytes = TYPE == ARGUS_FP32 ? 4 : 2, kPer = 16 / kBytes, kVecs = kItems / kPer;
  __shared__ uint32_t s_list[kMaxK];
  __shared__ float s_red[2 * kWaves];
  __shared__ uint64_t s_cand[kCands];
  __shared__ uint32_t s_n;
  __shared__ uint64_t s_best[kWaves];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_SELECT_ROWS);
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
  const uint32_t row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  if (a.finished && a.finished[row]) {  // stands for itself: nothing of the row is looked at
    mk.end(ARGUS_REGION_SELECT_ROWS);
    return;
  }
  const uint8_t* base = a.logits + (int64_t)(row / a.W) * a.group_stride + (int64_t)(row % a.W) * a.beam_stride;
  // Vectors lie on 16 bytes: element j of the row is at place j + lead.
  const uint32_t lead = (uint32_t)((uintptr_t)base & 15u) / kBytes;
  float x[kItems];
#pragma unroll
  for (uint32_t v = 0; v < kVecs; ++v) {
    const int64_t j = (int64_t)chunk * kChunkElems + (v * kThreads + tid) * kPer - lead;
    if (j >= 0 && j + kPer <= a.V) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(base + j * kBytes);
#pragma unroll
      for (uint32_t i = 0; i < kPer; ++i) x[v * kPer + i] = of_word<TYPE>(w[i * kBytes / 4], i % (4 / kBytes));
    } else {
#pragma unroll
      for (uint32_t i = 0; i < kPer; ++i)
        x[v * kPer + i] = j + i >= 0 && j + i < a.V ? element<TYPE>(base + (j + i) * kBytes) : -INFINITY;
    }
  }
  if (tid < a.lists) s_list[tid] = 0;
  if (tid == 0) s_n = 0;
  float top = x[0];
#pragma unroll
  for (uint32_t i = 1; i < kItems; ++i) top = fmaxf(top, x[i]);
  const float wtop = wave_max(top);
  if (lane == 0) s_red[wave] = wtop;
  __syncthreads();
  atomicMax(&s_list[tid & (a.lists - 1)], order_of(top));
  const float all = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
  const float shift = all == -INFINITY ? 0.0f : all;  // (values times log2 e could overflow: the difference first)
  float sum = 0.0f;
#pragma unroll
  for (uint32_t i = 0; i < kItems; ++i) sum += __builtin_amdgcn_exp2f((x[i] - shift) * kLog2e);
  sum = wave_sum(sum);
  if (lane == 0) s_red[kWaves + wave] = sum;
  __syncthreads();
  if (tid == 0)
    a.sums[blockIdx.x] = make_float2(all, s_red[kWaves] + s_red[kWaves + 1] + s_red[kWaves + 2] + s_red[kWaves + 3]);
  uint32_t lo = s_list[lane & (a.lists - 1)];
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_xor(lo, d);
    lo = o < lo ? o : lo;
  }
  const float bound = value_of(lo);
  // (a list without a value leaves 0: the order of a NaN, which nothing is below)
  const bool any = lo != 0;
#pragma unroll
  for (uint32_t i = 0; i < kItems; ++i) {
    if ((any ? x[i] >= bound : x[i] == x[i]) && x[i] > -INFINITY) {
      const uint32_t at = atomicAdd(&s_n, 1u);
      const uint32_t token = chunk * kChunkElems + ((i / kPer) * kThreads + tid) * kPer + i % kPer - lead;
      if (at < kCands) s_cand[at] = key_of(x[i], token);
    }
  }
  __syncthreads();
  const uint32_t n = s_n;
  uint64_t* out = a.cands + (uint64_t)blockIdx.x * a.K;
  if (n <= kCands) {
    for (uint32_t c = tid; c < n; c += kThreads) {
      const uint64_t k = s_cand[c];
      uint32_t rank = 0;
      for (uint32_t o = 0; o < n; ++o) rank += s_cand[o] > k;
      if (rank < a.K) out[rank] = k;
    }
    for (uint32_t r = n + tid; r < a.K; r += kThreads) out[r] = 0;
  } else {
    uint64_t last = ~0ull;  // the key picked before
    for (uint32_t r = 0; r < a.K; ++r) {
      uint64_t best = 0;
#pragma unroll
      for (uint32_t i = 0; i < kItems; ++i) {
        const uint32_t token = chunk * kChunkElems + ((i / kPer) * kThreads + tid) * kPer + i % kPer - lead;
        const uint64_t k = x[i] > -INFINITY ? key_of(x[i], token) : 0ull;
        best = k < last && k > best ? k : best;
      }
      for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_xor(best, d);
        best = o > best ? o : best;
      }
      if (lane == 0) s_best[wave] = best;
      __syncthreads();
      best = s_best[0];
      for (uint32_t w = 1; w < (uint32_t)kWaves; ++w) best = s_best[w] > best ? s_best[w] : best;
      if (tid == 0) out[r] = best;
      last = best;
      __syncthreads();
    }
  }
  mk.end(ARGUS_REGION_SELECT_ROWS);
}

struct Pick {
  uint32_t order, beam;  // of the score; ~beam
  uint64_t key;
};
ARGUS_DEV bool before(const Pick& x, const Pick& y) {
  const uint64_t a = join64(x.beam, x.order), b = join64(y.beam, y.order);
  return a > b || (a == b && x.key > y.key);
}

__global__ __launch_bounds__(kThreads) void k_select_beams(SelectArgs a) {
  __shared__ float s_lse[kMaxBeams], s_score[kMaxBeams];
  __shared__ uint8_t s_done[kMaxBeams];
  __shared__ uint32_t s_list[kMaxK];
  __shared__ uint32_t s_n;
  __shared__ Pick s_cand[kCands];
  __shared__ Pick s_best[kWaves];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_SELECT_BEAMS);
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, group = blockIdx.x;
  for (uint32_t w = wave; w < a.W; w += kWaves) {
    const uint32_t row = group * a.W + w;
    const bool done = a.finished && a.finished[row];
    float top = -INFINITY, sum = 0.0f;
    if (!done) {
      for (uint32_t c = lane; c < a.chunks; c += 64) top = fmaxf(top, a.sums[(uint64_t)row * a.chunks + c].x);
      top = wave_max(top);
      for (uint32_t c = lane; c < a.chunks; c += 64) {
        const float2 v = a.sums[(uint64_t)row * a.chunks + c];
        sum += v.x == -INFINITY ? v.y : v.y * exp2f((v.x - top) * kLog2e);
      }
      sum = wave_sum(sum);
    }
    if (lane == 0) {
      s_lse[w] = top + logf(sum);
      s_score[w] = a.scores[row];
      s_done[w] = done;
    }
  }
  if (tid < a.lists) s_list[tid] = 0;
  if (tid == 0) s_n = 0;
  __syncthreads();
  const uint32_t per_row = a.chunks * a.K, total = a.W * per_row;
  const uint64_t* cands = a.cands + (uint64_t)group * total;
  // Candidate i of the group; false: none.
  auto pick_of = [&](uint32_t i, Pick* p) {
    const uint32_t w = i / per_row, r = i % per_row;
    float score;
    if (s_done[w]) {
      if (r != 0) return false;
      p->key = 0;
      score = s_score[w];
    } else {
      p->key = cands[i];
      if (p->key == 0) return false;
      score = s_score[w] + (value_of((uint32_t)(p->key >> 32)) - s_lse[w]);
    }
    p->order = order_of(score);
    p->beam = ~w;
    return score > -INFINITY;
  };
  uint32_t top = 0;
  for (uint32_t i = tid; i < total; i += kThreads) {
    Pick p;
    if (pick_of(i, &p)) top = p.order > top ? p.order : top;
  }
  atomicMax(&s_list[tid & (a.lists - 1)], top);
  __syncthreads();
  uint32_t bound = s_list[lane & (a.lists - 1)];
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_xor(bound, d);
    bound = o < bound ? o : bound;
  }
  for (uint32_t i = tid; i < total; i += kThreads) {
    Pick p;
    if (pick_of(i, &p) && p.order >= bound) {
      const uint32_t at = atomicAdd(&s_n, 1u);
      if (at < kCands) s_cand[at] = p;
    }
  }
  __syncthreads();
  const uint32_t n = s_n;
  auto put = [&](uint32_t r, const Pick& p) {
    const uint32_t w = ~p.beam;
    const uint64_t at = (uint64_t)group * a.K + r;
    const int32_t token = s_done[w] ? a.eos : (int32_t)~(uint32_t)p.key;
    a.new_scores[at] = value_of(p.order);
    a.parents[at] = (int32_t)(group * a.W + w);
    a.tokens[at] = token;
    a.new_finished[at] = s_done[w] || (token == a.eos && a.eos >= 0);
  };
  auto put_none = [&](uint32_t r) {
    const uint64_t at = (uint64_t)group * a.K + r;
    a.new_scores[at] = -INFINITY;
    a.parents[at] = -1;
    a.tokens[at] = -1;
    a.new_finished[at] = 0;
  };
  if (n <= kCands) {
    for (uint32_t c = tid; c < n; c += kThreads) {
      const Pick p = s_cand[c];
      uint32_t rank = 0;
      for (uint32_t o = 0; o < n; ++o) rank += before(s_cand[o], p);
      if (rank < a.K) put(rank, p);
    }
    for (uint32_t r = n + tid; r < a.K; r += kThreads) put_none(r);
  } else {
    Pick last{0xFFFFFFFFu, 0xFFFFFFFFu, ~0ull};
    bool more = true;
    for (uint32_t r = 0; r < a.K; ++r) {
      Pick best{0, 0, 0};
      for (uint32_t i = tid; more && i < total; i += kThreads) {
        Pick p;
        if (pick_of(i, &p) && before(last, p) && before(p, best)) best = p;
      }
      for (int d = 1; d < 64; d <<= 1) {
        const Pick o{__shfl_xor(best.order, d), __shfl_xor(best.beam, d), __shfl_xor(best.key, d)};
        if (before(o, best)) best = o;
      }
      if (lane == 0) s_best[wave] = best;
      __syncthreads();
      best = s_best[0];
      for (uint32_t w = 1; w < (uint32_t)kWaves; ++w)
        if (before(s_best[w], best)) best = s_best[w];
      more = more && best.order != 0;
      if (tid == 0) {
        if (more) put(r, best);
        else put_none(r);
      }
      last = best;
      __syncthreads();
    }
  }
  mk.end(ARGUS_REGION_SELECT_BEAMS);
}

struct Plan {
  uint32_t chunks;
  size_t cands_at, bytes;
};

int make_plan(const argus_select_config* c, Plan* p) {
  if (!c) return refuse(ARGUS_E_INVAL, "no configuration");
  if (c->abi_version != ARGUS_ATTR_ABI_VERSION) return refuse(ARGUS_E_ABI, "abi_version %u", c->abi_version);
  if (c->type > ARGUS_FP32) return refuse(ARGUS_E_INVAL, "logits are bf16, fp16 or fp32");
  if (c->beams < 1 || c->beams > kMaxBeams || c->k < 1 || c->k > kMaxK)
    return refuse(ARGUS_E_INVAL, "beams %u, k %u (1..64)", c->beams, c->k);
  if (c->vocab < 1 || c->vocab > (1u << 24)) return refuse(ARGUS_E_INVAL, "vocab %u (1..2^24)", c->vocab);
  // a row may start anywhere on 16 bytes: up to 15 bytes before its chunks
  const uint32_t lead = c->type == ARGUS_FP32 ? 3u : 7u;
  p->chunks = (c->vocab + lead + kChunkElems - 1) / kChunkElems;
  const uint64_t parts = (uint64_t)c->groups * c->beams * p->chunks;
  if (c->groups > (1u << 20) || parts > 0x7FFFFFFFull || (uint64_t)c->beams * p->chunks * c->k > 0x7FFFFFFFull)
    return refuse(ARGUS_E_CAPACITY, "groups x beams x vocab");
  p->cands_at = up256(parts * sizeof(float2));
  p->bytes = p->cands_at + up256(parts * c->k * sizeof(uint64_t));
  return ARGUS_OK;
}

}  // namespace
}  // namespace decode
}  // namespace argus

using namespace argus;
using namespace argus::decode;

extern "C" size_t argus_decode_select_workspace_bytes(const argus_select_config* cfg) {
  accepted();
  Plan p;
  return make_plan(cfg, &p) == ARGUS_OK ? p.bytes : (size_t)-1;
}

extern "C" int argus_decode_select(const argus_select_config* cfg, const argus_select_io* io, void* d_workspace,
                                   size_t workspace_bytes, argus_markers* markers, void* stream_v) {
  accepted();
  Plan p;
  int rc = make_plan(cfg, &p);
  if (rc != ARGUS_OK) return rc;
  if (!io || (cfg->groups && (!io->d_logits || !io->d_scores || !io->d_new_scores || !io->d_parents || !io->d_tokens ||
                              !io->d_new_finished)))
    return refuse(ARGUS_E_INVAL, "a required pointer is NULL");
  const uint32_t e = type_bytes(cfg->type);
  if (!aligned_to(io->d_logits, e) || !aligned_to(io->d_scores, 4) || !aligned_to(io->d_new_scores, 4) ||
      !aligned_to(io->d_parents, 4) || !aligned_to(io->d_tokens, 4))
    return refuse(ARGUS_E_ALIGN, "buffers lie on their elements' size");
  if (io->d_new_finished && io->d_new_finished == io->d_finished)
    return refuse(ARGUS_E_INVAL, "the new finished flags are another buffer than the old");
  if (io->d_new_scores && io->d_new_scores == io->d_scores)
    return refuse(ARGUS_E_INVAL, "the new scores are another buffer than the old");
  if (marks_bad(markers)) return refuse(ARGUS_E_INVAL, "markers: alignment or region_base");
  if (!d_workspace && cfg->groups) return refuse(ARGUS_E_INVAL, "no workspace");
  if (!aligned_to(d_workspace, 256)) return refuse(ARGUS_E_ALIGN, "the workspace lies on 256 bytes");
  if (workspace_bytes < p.bytes) return refuse(ARGUS_E_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, p.bytes);
  const uint32_t grid = cfg->groups * cfg->beams * p.chunks;
  if (!marks_fit(markers, ((uint64_t)grid + cfg->groups) * kWaves * 2))
    return refuse(ARGUS_E_CAPACITY, "the marker records do not fit");
  if (cfg->groups == 0) return ARGUS_OK;
  if ((rc = device_ok()) != ARGUS_OK) return rc;
  SelectArgs a{};
  a.logits = (const uint8_t*)io->d_logits;
  a.group_stride = io->group_stride * e, a.beam_stride = io->beam_stride * e;
  a.scores = io->d_scores, a.finished = io->d_finished;
  a.new_scores = io->d_new_scores, a.parents = io->d_parents, a.tokens = io->d_tokens, a.new_finished = io->d_new_finished;
  a.sums = (float2*)d_workspace;
  a.cands = (uint64_t*)((char*)d_workspace + p.cands_at);
  a.W = cfg->beams, a.V = cfg->vocab, a.K = cfg->k, a.chunks = p.chunks, a.eos = cfg->eos;
  a.lists = 1;
  while (a.lists < a.K) a.lists <<= 1;
  hipStream_t st = (hipStream_t)stream_v;
  a.marks = take_marks(markers, grid, 2);
  if (cfg->type == ARGUS_BF16) hipLaunchKernelGGL(k_select_rows<ARGUS_BF16>, dim3(grid), dim3(kThreads), 0, st, a);
  else if (cfg->type == ARGUS_FP16) hipLaunchKernelGGL(k_select_rows<ARGUS_FP16>, dim3(grid), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(k_select_rows<ARGUS_FP32>, dim3(grid), dim3(kThreads), 0, st, a);
  a.marks = take_marks(markers, cfg->groups, 2);
  hipLaunchKernelGGL(k_select_beams, dim3(cfg->groups), dim3(kThreads), 0, st, a);
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}
