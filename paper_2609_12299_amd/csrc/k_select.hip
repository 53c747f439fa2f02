// k_select.hip -- beam search's selection over beams and vocabulary.
//
// k_select_rows reads the logits once.  A wave takes a part of one row, 64 lanes
// of 32 elements at a time, the next ones under way while it looks at them, and
// keeps the sum of their exponentials and a list of candidates in LDS.  The
// least that a candidate needs is known after the first step: the k-th largest of
// the lanes' maxima has k elements at or above it, and few more.  From then on a
// step costs a comparison of each lane's largest value; where some are above, the step's elements
// go to LDS and the wave looks through those of the lanes in question.  When the
// list may not hold 64 more, it is cut to its first k, and what the k-th has becomes the
// least: the list never overflows, however many values are equal.
//
// k_select_beams, one block per group of beams, joins the parts' sums to the
// rows' logarithms and picks among the rows' candidates in the same way: the k-th
// largest of the threads' maxima, and those at or above it ranked by counting.
//
// What bounds it: the reading of the logits, and the exponential of each (a
// quarter of the rate of other instructions): 96 x 8 rows of 128003 in bf16, 197 MB, k 8: 37 us
// for the rows, 5.3 TB/s with the vector units busy 0.55 of the time, and 7 us for the beams.
#include "rows.h"

namespace argus {
namespace decode {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kItems = 32;               // elements of a lane per step
constexpr uint32_t kStep = kItems * 64;
// Candidates of a wave.  A cut counts, for each, those above it: the more room there is beyond
// 64, the rarer it is for a large k (32 x 4 rows of 128003, k 64: 174 us with 128, 68 with 192,
// 71 with 256; 96 x 8 rows, k 8, 43.5, 43.1 and 43.2; finding the k-th key bit by bit
// instead 54 against 43).
constexpr uint32_t kList = 192;
// Beyond its k a list holds so many before it is cut at the end of a step: the
// sooner the least rises, the fewer lanes are looked through (0: 43.4 us, 8: 43.1,
// 16: 43.1, only when half full: 48.0; 96 x 8 rows of 128003 in bf16, k 8).
constexpr uint32_t kRoom = 8;
constexpr uint32_t kCands = 512;              // candidates of a group that are ranked by counting
constexpr uint32_t kMaxK = 64, kMaxBeams = 64;

struct SelectArgs {
  const uint8_t* logits;
  int64_t group_stride, beam_stride;  // bytes
  const float* scores;
  const uint8_t* finished;
  float* new_scores;
  int32_t *parents, *tokens;
  uint8_t* new_finished;
  float2* sums;     // [rows][parts] reference, sum of exp(x - reference)
  uint64_t* cands;  // [rows][parts][k] (value, token) as a key, 0: none; no order
  uint32_t W, V, K, parts;
  FastDiv by_group, by_row;  // by W * parts, by parts
  uint32_t steps;   // of a part
  uint32_t rows;
  int32_t eos;
  Marks marks;
};

// How far a value may rise above the reference of the exponentials.
constexpr float kSlack = 8.0f;
// An exponential is 2^(x log2 e - c1), one multiply-add; from references of this size
// on the rounding of c1 would show in that, and the difference comes first.
constexpr float kFar = 1e6f;
// What a sum of exp(x - p) is worth as one of exp(x - q), q >= p.
ARGUS_DEV float moved(float p, float q) { return __builtin_amdgcn_exp2f((p - q) * kLog2e); }

template <int TYPE>
__global__ __launch_bounds__(kThreads) void k_select_rows(SelectArgs a) {
  constexpr uint32_t kBytes = TYPE == ARGUS_FP32 ? 4 : 2, kPer = 16 / kBytes, kVecs = kItems / kPer;
  __shared__ uint64_t s_list[kWaves][kList];
  __shared__ u32x4 s_step[kWaves][kVecs * 64];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_SELECT_ROWS);
  const uint32_t lane = threadIdx.x & 63u;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t job = blockIdx.x * kWaves + wave, row = job / a.parts, part = job % a.parts;
  // (a finished beam stands for itself: nothing of its row is looked at)
  if (row < a.rows && !(a.finished && a.finished[row])) {
    uint64_t* list = s_list[wave];
    const uint8_t* base = a.logits + (int64_t)(row / a.W) * a.group_stride + (int64_t)(row % a.W) * a.beam_stride;
    // Vectors lie on 16 bytes: `head` elements come before the first of `vecs`
    // vectors, less than a vector behind the last.
    uint32_t head = (uint32_t)(0 - (uintptr_t)base & 15u) / kBytes;
    head = head < a.V ? head : a.V;
    const uint32_t vecs = (a.V - head) / kPer, tail = head + vecs * kPer;
    const u32x4* body = reinterpret_cast<const u32x4*>(base + head * kBytes);
    const uint32_t first = part * a.steps * kVecs * 64;  // vector
    const uint32_t left = first < vecs ? (vecs - first + kVecs * 64 - 1) / (kVecs * 64) : 0;
    const uint32_t steps = left < a.steps ? left : a.steps;
    // Behind the last vector it is read again, and not looked at: without branches the
    // loads stay under way (one that may or may not have been made is waited for).
    // Past the caches, as they are read once: 42.7 us against 44.8.
    auto load = [&](uint32_t step, u32x4 (&w)[kVecs]) {
      const uint32_t v0 = first + step * kVecs * 64 + lane;
#pragma unroll
      for (uint32_t v = 0; v < kVecs; ++v) w[v] = __builtin_nontemporal_load(&body[v0 + v * 64 < vecs ? v0 + v * 64 : vecs - 1]);
    };
    uint32_t n = 0;           // candidates in the list
    uint64_t least = 0;       // their keys are above it
    float least_value = -INFINITY;
    // The list cut to its first k, in order: each lane counts what is above its keys, C of them.
    auto rank = [&](auto keys) {
      constexpr uint32_t C = keys();
      uint64_t key[C];
      uint32_t above[C];
#pragma unroll
      for (uint32_t c = 0; c < C; ++c) {
        key[c] = lane + 64 * c < n ? list[lane + 64 * c] : 0;
        above[c] = 0;
      }
#pragma unroll 8
      for (uint32_t i = 0; i < n; ++i) {
        const uint64_t o = list[i];
#pragma unroll
        for (uint32_t c = 0; c < C; ++c) above[c] += o > key[c];
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (uint32_t c = 0; c < C; ++c)
        if (lane + 64 * c < n && above[c] < a.K) list[above[c]] = key[c];
    };
    auto cut = [&]() {
      __builtin_amdgcn_wave_barrier();
      if (n <= 64) rank([]() constexpr { return 1u; });
      else if (n <= 128) rank([]() constexpr { return 2u; });
      else rank([]() constexpr { return kList / 64; });
      __builtin_amdgcn_wave_barrier();
      n = n < a.K ? n : a.K;
      if (n == a.K) {
        least = list[a.K - 1];
        least_value = value_of((uint32_t)(least >> 32));
      }
    };
    auto append = [&](bool want, uint64_t key) {  // at most 64 at a time
      const uint64_t take = __ballot(want);
      if (want) list[n + (uint32_t)__popcll(take & lanemask_lt())] = key;
      n += (uint32_t)__popcll(take);
    };
    // The sum is of 2^(x log2 e - c1), about exp(x - ref); far ones of exp(x - ref).  Either way a
    // sum moves, near and far ones among each other too, with no rounding of c1 that shows.
    float ref = -INFINITY, c1 = 0.0f, sum = 0.0f;
    bool far = false;
    auto refer = [&](float to) {
      if (to == -INFINITY) return;
      const float was = ref, c1_was = c1;
      const bool far_was = far;
      ref = to;
      far = fabsf(ref) >= kFar;
      c1 = ref * kLog2e;
      if (was == -INFINITY) sum *= 0.0f;  // (a NaN stays)
      else if (far) sum *= far_was ? moved(was, ref) : __builtin_amdgcn_exp2f(fmaf(-ref, kLog2e, c1_was));
      else sum *= __builtin_amdgcn_exp2f(far_was ? fmaf(was, kLog2e, -c1) : c1_was - c1);
    };
    if (part == 0) {  // what lies before and behind the vectors: at most 2 * (kPer - 1) elements
      const uint32_t j = lane < kPer ? lane : tail + lane - kPer;
      const bool in = lane < kPer ? j < head : lane < 2 * kPer && j < a.V;
      float x = -INFINITY;
      if (in) {
        if constexpr (TYPE == ARGUS_FP32) x = *reinterpret_cast<const float*>(base + (uint64_t)j * kBytes);
        else x = of_word<TYPE>(*reinterpret_cast<const uint16_t*>(base + (uint64_t)j * kBytes), 0);
      }
      refer(wave_max(x));
      sum = __builtin_amdgcn_exp2f(far ? (x - ref) * kLog2e : fmaf(x, kLog2e, -c1));
      append(x > -INFINITY, key_of(x, j));
    }
    auto look = [&](uint32_t step, const u32x4 (&w)[kVecs]) {
      float x[kItems];
#pragma unroll
      for (uint32_t i = 0; i < kItems; ++i) x[i] = of_word<TYPE>(w[i / kPer][(i % kPer) * kBytes / 4], i % (4 / kBytes));
      if (first + (step + 1) * kVecs * 64 > vecs) {
        const uint32_t v0 = first + step * kVecs * 64 + lane;
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) x[i] = v0 + i / kPer * 64 < vecs ? x[i] : -INFINITY;
      }
      float top = x[0];
#pragma unroll
      for (uint32_t i = 1; i < kItems; ++i) top = fmaxf(top, x[i]);
      if (__any(top > ref + kSlack)) refer(fmaxf(ref, wave_max(top)));
      float part_sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (!far) {
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) part_sum[i % 4] += __builtin_amdgcn_exp2f(fmaf(x[i], kLog2e, -c1));
      } else {
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) part_sum[i % 4] += __builtin_amdgcn_exp2f((x[i] - ref) * kLog2e);
      }
      sum += (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
      if (step == 0) {
        // the k-th largest of the lanes' maxima: the least that fewer than k are above
        const uint32_t mine = order_of(top);
        uint32_t above = 0;
#pragma unroll 16
        for (int i = 0; i < 64; ++i) above += (uint32_t)__builtin_amdgcn_readlane((int)mine, i) > mine;
        const uint32_t lo = ~wave_max_u32(above < a.K ? ~mine : 0u);
        least_value = value_of(lo);
        least = join64(0u, lo);  // below every key of this value
      }
      uint64_t hot = __ballot(top >= least_value && top > -INFINITY);
      if (hot) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (uint32_t v = 0; v < kVecs; ++v) s_step[wave][v * 64 + lane] = w[v];
        __builtin_amdgcn_wave_barrier();
        // two lanes' 32 elements at a time
        while (hot) {
          if (n > kList - 64) cut();
          const uint32_t l0 = (uint32_t)__builtin_ctzll(hot);
          hot &= hot - 1;
          const uint32_t l1 = hot ? (uint32_t)__builtin_ctzll(hot) : l0;
          const bool in = lane < kItems || l1 != l0;
          hot &= hot - 1;
          const uint32_t i = lane % kItems, at = (i / kPer) * 64 + (lane < kItems ? l0 : l1);
          float y;
          if constexpr (TYPE == ARGUS_FP32) y = reinterpret_cast<const any_f32*>(&s_step[wave][at])[i % kPer];
          else y = of_word<TYPE>(reinterpret_cast<const any_u16*>(&s_step[wave][at])[i % kPer], 0);
          const uint32_t token = head + (first + step * kVecs * 64 + at) * kPer + i % kPer;
          const uint64_t key = key_of(y, token);
          const bool there = first + step * kVecs * 64 + at < vecs;
          append(in && there && y >= least_value && key > least && y > -INFINITY, key);
        }
        if (n > a.K + kRoom) cut();
      }
    };
    u32x4 w0[kVecs], w1[kVecs];
    if (steps) {
      load(0, w0);
      uint32_t step = 0;
      for (; step + 1 < steps; step += 2) {
        load(step + 1, w1);
        look(step, w0);
        load(step + 2 < steps ? step + 2 : step, w0);
        look(step + 1, w1);
      }
      if (step < steps) look(step, w0);
    }
    cut();
    sum = wave_sum(sum);
    if (!far && ref > -INFINITY) sum *= __builtin_amdgcn_exp2f(fmaf(-ref, kLog2e, c1));
    if (lane == 0) a.sums[job] = make_float2(ref, sum);
    if (lane < a.K) a.cands[(uint64_t)job * a.K + lane] = lane < n ? list[lane] : 0;
  }
  mk.end(ARGUS_REGION_SELECT_ROWS);
}

// A candidate's place in the order: score, then ~beam; then the logit and ~token.
struct Pick {
  uint64_t first, key;
};
ARGUS_DEV bool before(const Pick& x, const Pick& y) { return x.first > y.first || (x.first == y.first && x.key > y.key); }

__global__ __launch_bounds__(kThreads) void k_select_beams(SelectArgs a) {
  constexpr uint32_t kMine = 4;  // candidates that a thread holds at a time
  __shared__ float s_ref[kMaxBeams], s_log[kMaxBeams], s_score[kMaxBeams];
  __shared__ uint32_t s_done[kMaxBeams];
  __shared__ uint32_t s_n;
  __shared__ Pick s_cand[kCands];
  __shared__ Pick s_best[kWaves];
  __shared__ uint64_t s_top[kWaves][64], s_bound;
  __shared__ uint32_t s_tops[kWaves];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_SELECT_BEAMS);
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, group = blockIdx.x;
  // Candidate i: the i / parts-th of the list of part i % parts (of the whole
  // group), so that the first of all parts lie in threads of their own.
  const uint32_t parts = a.W * a.parts, total = parts * a.K;
  const uint64_t* cands = a.cands + (uint64_t)group * total;
  uint64_t key[kMine];
  uint32_t beam[kMine];  // and, from bit 8 on, whether it is its beam's first
  auto fetch = [&](uint32_t i0) {
#pragma unroll
    for (uint32_t c = 0; c < kMine; ++c) {
      const uint32_t i = i0 + c * kThreads + tid;
      const uint32_t r = divide(i, a.by_group), j = i - r * parts, w = divide(j, a.by_row);
      key[c] = i < total ? cands[(uint64_t)j * a.K + r] : 0;
      beam[c] = i < total ? w | (r == 0 && j == w * a.parts ? 256u : 0u) : 0xFFFFu;
    }
  };
  fetch(0);  // under way while the sums are joined
  for (uint32_t w = tid / 16; w < a.W; w += kThreads / 16) {  // 16 lanes a row
    const uint32_t row = group * a.W + w;
    const bool done = a.finished && a.finished[row];
    const float score = a.scores[row];
    float top = -INFINITY, sum = 0.0f;
    if (!done) {
      for (uint32_t c = tid % 16; c < a.parts; c += 16) {
        const float2 v = a.sums[(uint64_t)row * a.parts + c];
        const float most = fmaxf(top, v.x);
        // (a part without a value leaves 0, a NaN stays)
        sum = sum * (top == -INFINITY ? 1.0f : moved(top, most)) + v.y * (v.x == -INFINITY ? 1.0f : moved(v.x, most));
        top = most;
      }
    }
    for (int d = 1; d < 16; d <<= 1) {
      const float o = __shfl_xor(top, d), os = __shfl_xor(sum, d), most = fmaxf(top, o);
      sum = sum * (top == -INFINITY ? 1.0f : moved(top, most)) + os * (o == -INFINITY ? 1.0f : moved(o, most));
      top = most;
    }
    if (tid % 16 == 0) {
      // The logarithm is taken off a logit in two steps: of one number near 10^6 the rounding
      // would show, and 10^10 leaves no place for the sum's.
      s_ref[w] = top;
      s_log[w] = logf(sum);
      s_score[w] = score;
      s_done[w] = done;
    }
  }
  if (tid == 0) {
    s_n = 0;
    s_bound = ~0ull;
  }
  __syncthreads();
  // What fetch() has brought, as a place in the order; false: no candidate.
  auto pick_of = [&](uint32_t c, Pick* p) {
    if (beam[c] == 0xFFFFu) return false;
    const uint32_t w = beam[c] & 255u;
    float score;
    if (s_done[w]) {
      if (beam[c] < 256u) return false;
      p->key = 0;
      score = s_score[w];
    } else {
      p->key = key[c];
      if (p->key == 0) return false;
      score = s_score[w] + (value_of((uint32_t)(p->key >> 32)) - s_ref[w] - s_log[w]);
    }
    p->first = join64(~w, order_of(score));
    return score > -INFINITY;
  };
  // (The first of all lists are enough for a bound: 2 x 16 rows of 17365 in fp32, k 32: 28.4 us against
  // 31.0 with all of them.)
  uint64_t top = 0;
#pragma unroll
  for (uint32_t c = 0; c < kMine; ++c) {
    Pick p;
    if (pick_of(c, &p)) top = p.first > top ? p.first : top;
  }
  // The k-th largest of these: in each wave those that fewer than k are above, then
  // of all such.  (What one of a wave's others is above, k of that wave are above.)
  uint32_t above = 0;
#pragma unroll 16
  for (int i = 0; i < 64; ++i)
    above += join64((uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)top, i),
                    (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(top >> 32), i)) > top;
  const uint64_t mine = __ballot(above < a.K);
  if (above < a.K) s_top[wave][__popcll(mine & lanemask_lt())] = top;
  if (lane == 0) s_tops[wave] = (uint32_t)__popcll(mine);
  __syncthreads();
  if (above < a.K) {
    above = 0;
    for (uint32_t w = 0; w < (uint32_t)kWaves; ++w) {
#pragma unroll 4
      for (uint32_t o = 0; o < s_tops[w]; ++o) above += s_top[w][o] > top;
    }
    if (above < a.K) atomicMin((unsigned long long*)&s_bound, (unsigned long long)top);
  }
  __syncthreads();
  const uint64_t bound = s_bound;
  for (uint32_t i0 = 0; i0 < total; i0 += kMine * kThreads) {
    if (i0) fetch(i0);
#pragma unroll
    for (uint32_t c = 0; c < kMine; ++c) {
      Pick p;
      if (pick_of(c, &p) && p.first >= bound) {
        const uint32_t at = atomicAdd(&s_n, 1u);
        if (at < kCands) s_cand[at] = p;
      }
    }
  }
  __syncthreads();
  const uint32_t n = s_n;
  auto put = [&](uint32_t r, const Pick& p) {
    const uint32_t w = ~(uint32_t)p.first;
    const uint64_t at = (uint64_t)group * a.K + r;
    const int32_t token = s_done[w] ? a.eos : (int32_t)~(uint32_t)p.key;
    a.new_scores[at] = value_of((uint32_t)(p.first >> 32));
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
#pragma unroll 8
      for (uint32_t o = 0; o < n; ++o) rank += before(s_cand[o], p);
      if (rank < a.K) put(rank, p);
    }
    for (uint32_t r = n + tid; r < a.K; r += kThreads) put_none(r);
  } else {
    // Too many equal scores to be ranked: one after the other.
    Pick last{~0ull, ~0ull};
    bool more = true;
    for (uint32_t r = 0; r < a.K; ++r) {
      Pick best{0, 0};
      for (uint32_t i0 = 0; more && i0 < total; i0 += kMine * kThreads) {
        fetch(i0);
#pragma unroll
        for (uint32_t c = 0; c < kMine; ++c) {
          Pick p;
          if (pick_of(c, &p) && before(last, p) && before(p, best)) best = p;
        }
      }
      for (int d = 1; d < 64; d <<= 1) {
        const Pick o{__shfl_xor(best.first, d), __shfl_xor(best.key, d)};
        if (before(o, best)) best = o;
      }
      if (lane == 0) s_best[wave] = best;
      __syncthreads();
      best = s_best[0];
      for (uint32_t w = 1; w < (uint32_t)kWaves; ++w)
        if (before(s_best[w], best)) best = s_best[w];
      more = more && best.first != 0;
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
  uint32_t parts, steps;
  size_t cands_at, bytes;
};

// Waves that read the logits (4096 and 2048: 44.2 and 49.9 us against 43.1 for 96 x
// 8 rows of 128003 in bf16).
constexpr uint32_t kRowWaves = 3072;
// More parts make shorter work of the rows and longer work of the group's
// candidates: parts of one step where those stay below kGroupCands (2 x 8 rows of
// 18641 in fp16, k 16: 17.6 us against 20.8 with three steps), else longer ones (8 x 8
// rows of 128003 in fp32, k 8: 22.3 us with four steps against 28.8 with one), up to
// kLongPart.  The lists of a large k are what costs in a part: 128 k candidates there (4 x 16 rows of
// 128003, k 32: 49 us against 54; 32 x 4, k 64: 74 against 71; 1 x 4, k 64: 60 against 68; with a
// bound from the first of all lists since then 45, 68 and 51, with 256 k 43, 68 and 53).
constexpr uint32_t kGroupCands = 2048, kCandsOfK = 128, kLongPart = 16;

int make_plan(const argus_select_config* c, Plan* p) {
  if (!c) return refuse(ARGUS_E_INVAL, "no configuration");
  if (c->abi_version != ARGUS_ATTR_ABI_VERSION) return refuse(ARGUS_E_ABI, "abi_version %u", c->abi_version);
  if (c->type > ARGUS_FP32) return refuse(ARGUS_E_INVAL, "logits are bf16, fp16 or fp32");
  if (c->beams < 1 || c->beams > kMaxBeams || c->k < 1 || c->k > kMaxK)
    return refuse(ARGUS_E_INVAL, "beams %u, k %u (1..64)", c->beams, c->k);
  if (c->vocab < 1 || c->vocab > (1u << 24)) return refuse(ARGUS_E_INVAL, "vocab %u (1..2^24)", c->vocab);
  if (c->groups > (1u << 20)) return refuse(ARGUS_E_CAPACITY, "groups %u", c->groups);
  const uint64_t rows = (uint64_t)c->groups * c->beams;
  if (rows > (uint64_t)kMaxBlocks * kWaves) return refuse(ARGUS_E_CAPACITY, "groups %u x beams %u", c->groups, c->beams);
  const uint32_t steps = (c->vocab + kStep - 1) / kStep;
  const uint64_t parts = rows ? kRowWaves / rows : 1;
  uint32_t most = (kCandsOfK * c->k > kGroupCands ? kCandsOfK * c->k : kGroupCands) / (c->beams * c->k);
  most = most < steps ? most : steps;
  const uint32_t some = (steps + kLongPart - 1) / kLongPart;
  most = most < some ? some : most;
  p->parts = parts < 1 ? 1u : parts < most ? (uint32_t)parts : most;
  p->steps = (steps + p->parts - 1) / p->parts;
  p->parts = (steps + p->steps - 1) / p->steps;
  const uint64_t jobs = rows * p->parts;
  p->cands_at = up256(jobs * sizeof(float2));
  p->bytes = p->cands_at + up256(jobs * c->k * sizeof(uint64_t));
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
  const uint32_t grid = (cfg->groups * cfg->beams * p.parts + kWaves - 1) / kWaves;
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
  a.W = cfg->beams, a.V = cfg->vocab, a.K = cfg->k, a.parts = p.parts, a.eos = cfg->eos;
  a.steps = p.steps, a.rows = cfg->groups * cfg->beams;
  a.by_group = fast_div(a.W * a.parts), a.by_row = fast_div(a.parts);
  hipStream_t st = (hipStream_t)stream_v;
  a.marks = take_marks(markers, grid, 2);
  if (cfg->type == ARGUS_BF16) hipLaunchKernelGGL(k_select_rows<ARGUS_BF16>, dim3(grid), dim3(kThreads), 0, st, a);
  else if (cfg->type == ARGUS_FP16) hipLaunchKernelGGL(k_select_rows<ARGUS_FP16>, dim3(grid), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(k_select_rows<ARGUS_FP32>, dim3(grid), dim3(kThreads), 0, st, a);
  a.marks = take_marks(markers, cfg->groups, 2);
  hipLaunchKernelGGL(k_select_beams, dim3(cfg->groups), dim3(kThreads), 0, st, a);
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}
