// k_score.hip -- log probabilities of given tokens, with entropy, rank and the best alternatives.
//
// With d = x - max x, S = sum e^d and T = sum d e^d of a row:
//
//   ln p[t] = (x[t] - max x) - ln S        entropy = ln S - T / S
//
// Both are sums of numbers of one sign where the maximum is the row's own: T <= 0 <= ln S, so nothing
// cancels. A lane keeps the maximum of what it has seen, exactly, and moves its sums where it
// rises (S' = S e^m, T' = (T + m S) e^m, m <= 0 the old maximum less the new one); lanes, waves and parts
// are joined in the same way, in a fixed order.
//
// A block reads a part of a row, its four waves 64 lanes of 32 elements in turn. The next ones' loads go out once
// these are in 32 bits and looked through for the maximum; the rest is done while they are under way, four to six
// waves on a SIMD (two sets of registers for them, three or four waves: 137 us where this took 108). The rank is a
// count of what is above the given token's own logit, read first. The k best are among what is not below the k-th
// largest of the block's 256 lanes' maxima, whichever elements the lanes have seen: that bound is worked out after
// the first step of each wave and again when a wave has seen four times as much, from what the others have noted
// by then. What is not below it goes to a list of the wave in LDS, and the rest of the work is a few steps
// over some k candidates.
//
// What bounds it: reading the logits, and nearly as much the arithmetic, 7.5 instructions an element (the exponential
// counts twice). Where a clamp is needed for minus infinities it is an eighth: steps go without until a sum
// becomes NaN, and ranks are counted by the scalar unit. 2048 rows of 128003 in bf16 with 20 alternatives take 103 us,
// 5.1 TB/s (a list of its own bound for each wave, a rank in each lane and a clamp of two instructions 143); 500 rows of
// 65537 in 32 bits, some of it minus infinity, 23.5 us, 5.6 TB/s; one row of 32000, 5 alternatives, 10.0 us, the
// host's and the kernel's time alike. Of a kernel that short a step is all: its loads go out first, what few elements
// need (the token's own vector, the row's end) is done with the others' instructions, and lanes are joined without
// LDS (10.7 us with shuffles through it).
#include "prompt.h"
#include "rows.h"

namespace argus {
namespace prompt {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kItems = 32;       // elements of a lane per step
constexpr uint32_t kStep = kItems * 64;
constexpr uint32_t kList = 192;       // candidates of a wave
constexpr uint32_t kManyWaves = 16;   // of a block that reads a row by itself
constexpr uint32_t kMaxTop = 64;
constexpr uint32_t kCands = 512;      // of the parts of a row, ranked by counting

struct Sums {
  float top, s, t;  // maximum, sum of e^d, sum of d e^d
  uint32_t above;
};

struct ScoreArgs {
  const uint8_t* logits;
  int64_t row_stride;  // bytes
  const int32_t* tokens;
  float *logprobs, *entropy;
  int32_t* ranks;
  float* top_logprobs;
  int32_t* top_tokens;
  Sums* sums;       // [rows][parts]
  uint64_t* cands;  // [rows][parts][K] in order, 0: none
  uint32_t V, K, parts, steps, rows;  // steps of a part
  Marks marks;
};

ARGUS_DEV float power(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// Sums about a larger maximum. (None yet: nothing to move; -inf - -inf would be NaN.)
ARGUS_DEV void move(Sums& a, float to) {
  if (a.top == -INFINITY) {
    a.top = to;
    return;
  }
  const float m = a.top - to, f = power(m);
  a.t = m < -128.0f ? 0.0f * a.s : (a.t + m * a.s) * f;  // (a NaN stays)
  a.s *= f;
  a.top = to;
}
ARGUS_DEV void join(Sums& a, Sums b) {
  const float to = fmaxf(a.top, b.top);
  move(a, to);
  move(b, to);
  a.s += b.s, a.t += b.t, a.above += b.above;
}
// A wave's, in all lanes: rows of 16 lanes without LDS, then the four of them.
ARGUS_DEV float lanes_sum(float v) {
  auto with = [&](uint32_t o) { v += __builtin_bit_cast(float, o); };
  with(dpp32<kDppQuad1032>(__builtin_bit_cast(uint32_t, v)));
  with(dpp32<kDppQuad2301>(__builtin_bit_cast(uint32_t, v)));
  with(dpp32<kDppHalfMirror>(__builtin_bit_cast(uint32_t, v)));
  with(dpp32<kDppMirror>(__builtin_bit_cast(uint32_t, v)));
  auto row = [&](int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); };
  return (row(0) + row(16)) + (row(32) + row(48));
}
ARGUS_DEV void join_lanes(Sums& a) {
  move(a, wave_max(a.top));
  a.s = lanes_sum(a.s);
  a.t = lanes_sum(a.t);
  const uint32_t n = row_sum32(a.above);
  auto row = [&](int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)n, lane); };
  a.above = (row(0) + row(16)) + (row(32) + row(48));
}

// A row's numbers, once its sums are known.
struct Row {
  float top, log, entropy;
  bool fine;
};
ARGUS_DEV Row row_of(const Sums& a) {
  Row r;
  r.top = a.top;
  r.log = logf(a.s);
  r.entropy = r.log - a.t / a.s;
  r.fine = a.s > 0.0f && a.s < INFINITY;
  return r;
}
ARGUS_DEV void put_row(const ScoreArgs& a, uint32_t row, const Row& r, uint32_t above, int32_t token, float mine) {
  const bool known = (uint32_t)token < a.V;
  a.logprobs[row] = !r.fine ? NAN : known ? (mine - r.top) - r.log : -INFINITY;
  a.entropy[row] = r.fine ? r.entropy : NAN;
  a.ranks[row] = r.fine && known ? (int32_t)above : -1;
}
ARGUS_DEV void put_top(const ScoreArgs& a, uint32_t row, const Row& r, uint32_t i, uint64_t key) {
  const uint64_t at = (uint64_t)row * a.K + i;
  a.top_tokens[at] = r.fine && key ? (int32_t)~(uint32_t)key : -1;
  a.top_logprobs[at] = !r.fine ? NAN : key ? (value_of((uint32_t)(key >> 32)) - r.top) - r.log : -INFINITY;
}

template <int TYPE>
ARGUS_DEV float element(const uint8_t* base, uint32_t i) {
  if constexpr (TYPE == ARGUS_FP32) return *reinterpret_cast<const float*>(base + (uint64_t)i * 4);
  else return of_word<TYPE>(*reinterpret_cast<const uint16_t*>(base + (uint64_t)i * 2), 0);
}

// W waves.
template <int TYPE, bool TOP, int W>
__global__ __launch_bounds__(64 * W) void k_score_rows(ScoreArgs a) {
  constexpr uint32_t kBytes = TYPE == ARGUS_FP32 ? 4 : 2, kPer = 16 / kBytes, kVecs = kItems / kPer;
  __shared__ uint64_t s_list[TOP ? W : 1][TOP ? kList : 1];
  __shared__ u32x4 s_step[TOP ? W : 1][TOP ? kVecs * 64 : 1];
  __shared__ float s_tops[TOP ? 64 * W : 1];  // the lanes' maxima
  __shared__ Sums s_sums[W];
  __shared__ uint32_t s_n[W];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_SCORE_ROWS);
  const uint32_t tid = threadIdx.x, lane = tid & 63u;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const uint8_t* base = a.logits + (int64_t)row * a.row_stride;
  const int32_t token = a.tokens[row];
  // Vectors lie on 16 bytes: `head` elements come before the first of `vecs`
  // vectors, less than a vector behind the last.
  uint32_t head = (uint32_t)(0 - (uintptr_t)base & 15u) / kBytes;
  head = head < a.V ? head : a.V;
  const uint32_t vecs = (a.V - head) / kPer, tail = head + vecs * kPer;
  const u32x4* body = reinterpret_cast<const u32x4*>(base + head * kBytes);
  const uint32_t all = (vecs + kVecs * 64 - 1) / (kVecs * 64);
  const uint32_t end = (part + 1) * a.steps < all ? (part + 1) * a.steps : all;
  u32x4 w[kVecs];  // the step's that is looked at, then the next one's
  auto load = [&](uint32_t step) {
    const uint32_t v0 = step * kVecs * 64;
    if (__builtin_expect(v0 + kVecs * 64 <= vecs, 1)) {
      const u32x4* from = body + v0;
#pragma unroll
      for (uint32_t v = 0; v < kVecs; ++v) w[v] = __builtin_nontemporal_load(&from[lane + v * 64]);
    } else {
#pragma unroll
      for (uint32_t v = 0; v < kVecs; ++v)
        w[v] = __builtin_nontemporal_load(&body[v0 + lane + v * 64 < vecs ? v0 + lane + v * 64 : vecs - 1]);
    }
  };
  uint32_t step = part * a.steps + wave;
  if (step < end) load(step);
  const bool known = (uint32_t)token < a.V;
  const float mine = known ? element<TYPE>(base, (uint32_t)token) : INFINITY;
  // the least number above it (what is as large and comes behind the token is not above)
  const float beyond = value_of(order_of(mine) + 1);
  // the vector that has the token; none: -1 or vecs
  const int32_t its = token < (int32_t)head ? -1 : (uint32_t)token >= tail ? (int32_t)vecs : (int32_t)((token - head) / kPer);
  Sums my{-INFINITY, 0.0f, 0.0f, 0u};
  uint32_t above = 0;  // of the wave's elements
  auto add = [&](float x, float base) {  // (a NaN of x goes on in s, a d of -inf has no part)
    const float d = x - base, e = power(d);
    my.s += e;
    my.t += e * fmaxf(d, -128.0f);
  };
  // the wave's list
  uint64_t* list = s_list[TOP ? wave : 0];
  uint32_t n = 0;
  uint64_t least = 0;
  float least_value = -INFINITY;
  auto cut = [&]() {  // to its first, in order
    constexpr uint32_t C = kList / 64;
    uint64_t key[C];
    uint32_t place[C];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) {
      key[c] = lane + 64 * c < n ? list[lane + 64 * c] : 0;
      place[c] = 0;
    }
#pragma unroll 4
    for (uint32_t i = 0; i < n; ++i) {
      const uint64_t o = list[i];
#pragma unroll
      for (uint32_t c = 0; c < C; ++c) place[c] += o > key[c];
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (uint32_t c = 0; c < C; ++c)
      if (lane + 64 * c < n && place[c] < a.K) list[place[c]] = key[c];
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
  // The k-th largest of the lanes' maxima, for 16-bit logits in its upper 16 bits: the largest number that k of them
  // are not below. What other waves note meanwhile may count or not.
  auto raise = [&]() {
    // (of 16 waves: of the maxima of four lanes each)
    uint32_t its[4], v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float top = -INFINITY;
#pragma unroll
      for (int w = i; w < W; w += 4)
        top = fmaxf(top, __hip_atomic_load(&s_tops[w * 64 + lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
      its[i] = order_of(top);
    }
#pragma unroll 1
    for (uint32_t bit = 1u << 31; bit >= (kBytes == 4 ? 1u : 1u << 16); bit >>= 1) {
      uint32_t many = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) many += (uint32_t)__popcll(__ballot(its[i] >= (v | bit)));
      v = many >= a.K ? v | bit : v;
    }
    const uint64_t bound = join64(0u, v);  // below every key of this value
    if (v > order_of(-INFINITY) && bound > least) least = bound, least_value = value_of(v);
  };
  uint32_t seen = 0, next = 4;  // steps of the wave; when the bound is worked out again
  bool holes = false;  // minus infinities have been seen
  auto look = [&](uint32_t step) {
    float x[kItems];
#pragma unroll
    for (uint32_t i = 0; i < kItems; ++i) x[i] = of_word<TYPE>(w[i / kPer][(i % kPer) * kBytes / 4], i % (4 / kBytes));
    const uint32_t v0 = step * kVecs * 64 + lane;
    const bool last = (step + 1) * kVecs * 64 > vecs;
    if (last) {
#pragma unroll
      for (uint32_t i = 0; i < kItems; ++i) x[i] = v0 + i / kPer * 64 < vecs ? x[i] : -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (uint32_t i = 1; i < kItems; ++i) top = fmaxf(top, x[i]);
    if (__any(top > my.top)) {
      move(my, fmaxf(my.top, top));
      if constexpr (TOP) __hip_atomic_store(&s_tops[tid], my.top, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    uint64_t hot = 0;
    if constexpr (TOP) {
      if (++seen == next) {
        next *= 4;
        raise();
      }
      hot = __ballot(top >= least_value && top > -INFINITY);
      if (hot) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (uint32_t v = 0; v < kVecs; ++v) s_step[wave][v * 64 + lane] = w[v];
        __builtin_amdgcn_wave_barrier();
      }
    }
    if (step + W < end) load(step + W);
    float base = my.top == -INFINITY ? 0.0f : my.top;
    const float s0 = my.s, t0 = my.t;
    if (!holes) {
#pragma unroll
      for (uint32_t i = 0; i < kItems; ++i) {
        const float d = x[i] - base, e = power(d);
        my.s += e;
        my.t += e * d;
        if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
      }
      holes = __any(my.t != my.t);  // 0 times infinity
      if (holes) my.s = s0, my.t = t0;
    }
    if (holes) {
      asm volatile("" : "+v"(base));  // (worked out anew: kept from above, it would take 64 registers)
#pragma unroll
      for (uint32_t i = 0; i < kItems; ++i) {
        add(x[i], base);
        if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
      }
    }
    // those above the token's logit, up to the end of its vector also those as large
    const uint32_t first = step * kVecs * 64;
    if (((int32_t)first > its || (int32_t)(first + kVecs * 64) <= its) && !last) {
      const float from = (int32_t)first > its ? beyond : mine;
#pragma unroll
      for (uint32_t i = 0; i < kItems; ++i) above += (uint32_t)__popcll(__ballot(x[i] >= from));
    } else {
#pragma unroll
      for (uint32_t v = 0; v < kVecs; ++v) {
        const float from = v0 + v * 64 >= vecs ? NAN : (int32_t)(v0 + v * 64) > its ? beyond : mine;
#pragma unroll
        for (uint32_t i = v * kPer; i < (v + 1) * kPer; ++i) above += (uint32_t)__popcll(__ballot(x[i] >= from));
      }
    }
    if constexpr (TOP) {
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
        const uint32_t tok = head + (step * kVecs * 64 + at) * kPer + i % kPer;
        const uint64_t key = key_of(y, tok);
        const bool there = step * kVecs * 64 + at < vecs;
        append(in && there && y >= least_value && key > least && y > -INFINITY, key);
      }
    }
  };
  if (part == 0 && wave == 0) {  // what lies before and behind the vectors: at most 2 * (kPer - 1) elements
    const uint32_t j = lane < kPer ? lane : tail + lane - kPer;
    const bool in = lane < kPer ? j < head : lane < 2 * kPer && j < a.V;
    const float x = in ? element<TYPE>(base, j) : -INFINITY;
    if (x > -INFINITY) my.top = x;
    if (in) add(x, my.top == -INFINITY ? 0.0f : my.top);
    above += (uint32_t)__popcll(__ballot(in && (x > mine || (x == mine && j < (uint32_t)token))));
    // what is counted below of the token's own vector, and is as large but not before it
    if (its >= 0 && its < (int32_t)vecs) {
      const uint32_t k = head + (uint32_t)its * kPer + lane;
      above -= (uint32_t)__popcll(__ballot(lane < kPer && k >= (uint32_t)token && element<TYPE>(base, lane < kPer ? k : head) == mine));
    }
    if constexpr (TOP) append(x > -INFINITY, key_of(x, j));
  }
  if constexpr (TOP) {
    float top = my.top;
    if (step < end) {
      const bool last = (step + 1) * kVecs * 64 > vecs;
#pragma unroll
      for (uint32_t i = 0; i < kItems; ++i) {
        const float x = of_word<TYPE>(w[i / kPer][(i % kPer) * kBytes / 4], i % (4 / kBytes));
        top = !last || step * kVecs * 64 + lane + i / kPer * 64 < vecs ? fmaxf(top, x) : top;
      }
    }
    s_tops[tid] = top;
    __syncthreads();
    raise();
  }
  for (; step < end; step += W) look(step);
  join_lanes(my);
  if (lane == 0) s_sums[wave] = Sums{my.top, my.s, my.t, above};
  __syncthreads();
  Sums sum = lane < W ? s_sums[lane] : Sums{-INFINITY, 0.0f, 0.0f, 0u};
  join_lanes(sum);
  const Row r = row_of(sum);
  if (tid == 0) {
    if (a.parts == 1) put_row(a, row, r, sum.above, token, mine);
    else a.sums[blockIdx.x] = sum;
  }
  if constexpr (TOP) {
    // what the whole block's bound leaves, 64 of a wave at most; a candidate's place is the number of those above it
    if (seen > 1) raise();
    uint32_t kept = 0;
    for (uint32_t i = 0; i < n; i += 64) {
      const uint64_t key = i + lane < n ? list[i + lane] : 0;
      const bool keep = key && key >= least;  // (the k-th of a list that was cut is its least)
      const uint64_t take = __ballot(keep);
      __builtin_amdgcn_wave_barrier();
      if (keep) list[kept + (uint32_t)__popcll(take & lanemask_lt())] = key;
      kept += (uint32_t)__popcll(take);
    }
    n = kept;
    if (n > 64) cut();
    if (lane == 0) s_n[wave] = n;
    __syncthreads();
    uint32_t total = 0;
    for (int w = 0; w < W; ++w) total += s_n[w];
    uint64_t* to = a.cands + (uint64_t)blockIdx.x * a.K;
    if (lane < n) {
      const uint64_t key = list[lane];
      uint32_t place = 0;
      for (int w = 0; w < W; ++w) {
        const uint32_t many = s_n[w];
#pragma unroll 8
        for (uint32_t i = 0; i < many; ++i) place += s_list[w][i] > key;
      }
      if (place < a.K) {
        if (a.parts == 1) put_top(a, row, r, place, key);
        else to[place] = key;
      }
    }
    for (uint32_t i = total + tid; i < a.K; i += 64 * W) {
      if (a.parts == 1) put_top(a, row, r, i, 0);
      else to[i] = 0;
    }
  }
  mk.end(ARGUS_REGION_SCORE_ROWS);
}

// The parts of a row joined.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void k_score_join(ScoreArgs a) {
  __shared__ uint64_t s_cand[kCands];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_SCORE_JOIN);
  const uint32_t tid = threadIdx.x, row = blockIdx.x, lane = tid & 63u;
  const uint32_t total = a.parts * a.K;
  for (uint32_t i = tid; i < total; i += kThreads) s_cand[i] = a.cands[(uint64_t)row * total + i];
  Sums sum{-INFINITY, 0.0f, 0.0f, 0u};
  for (uint32_t i = lane; i < a.parts; i += 64) join(sum, a.sums[(uint64_t)row * a.parts + i]);
  join_lanes(sum);
  const Row r = row_of(sum);
  if (tid == 0) {
    const int32_t token = a.tokens[row];
    const float mine = (uint32_t)token < a.V ? element<TYPE>(a.logits + (int64_t)row * a.row_stride, (uint32_t)token) : 0.0f;
    put_row(a, row, r, sum.above, token, mine);
  }
  __syncthreads();
  for (uint32_t i = tid; i < total; i += kThreads) {
    const uint64_t key = s_cand[i];
    uint32_t above = 0, none = 0;
    // places without a candidate come last, in their order
    for (uint32_t o = 0; o < total; ++o) {
      above += s_cand[o] > key;
      none += s_cand[o] == key && o < i;
    }
    above += none;
    if (above < a.K) put_top(a, row, r, above, key);
  }
  mk.end(ARGUS_REGION_SCORE_JOIN);
}

template <int TYPE>
void launch_score(const ScoreArgs& a, uint32_t grid, uint32_t waves, hipStream_t st) {
  const dim3 g(grid), b(64 * waves);
  if (waves == kManyWaves) {
    if (a.K) hipLaunchKernelGGL((k_score_rows<TYPE, true, kManyWaves>), g, b, 0, st, a);
    else hipLaunchKernelGGL((k_score_rows<TYPE, false, kManyWaves>), g, b, 0, st, a);
  } else {
    if (a.K) hipLaunchKernelGGL((k_score_rows<TYPE, true, kWaves>), g, b, 0, st, a);
    else hipLaunchKernelGGL((k_score_rows<TYPE, false, kWaves>), g, b, 0, st, a);
  }
}

struct Plan {
  uint32_t parts, steps, grid, waves;
  size_t cands_at, bytes;
};

constexpr uint32_t kRowBlocks = 768;
// Rows of which each compute unit has one at most: a block of 16 waves reads one by itself, and nothing is joined, where
// its waves have one step each (one row of 32000, 5 alternatives, 10.0 us against 14.0 in parts; one of 128003 20.9 against 13.7), or there are so many
// rows that parts of them would not fill the card better (256 of 128003, 20 alternatives, 25.1 us against 30.3; 100 of
// 128003 24.4 against 24.3, with 5 alternatives 22.4 against 19.1). Beyond that, parts or rows of four waves (300 of 32000, 20
// alternatives, 19.6 us, with 16 waves 24.5; 512 19.3 against 25.1).
constexpr uint32_t kFewRows = 256, kFewSteps = 4;

int make_plan(const argus_score_config* c, Plan* p) {
  if (!c) return refuse(ARGUS_E_INVAL, "no configuration");
  if (c->abi_version != ARGUS_ATTR_ABI_VERSION) return refuse(ARGUS_E_ABI, "abi_version %u", c->abi_version);
  if (c->type > ARGUS_FP32) return refuse(ARGUS_E_INVAL, "logits are bf16, fp16 or fp32");
  if (c->vocab < 1 || c->vocab > (1u << 24)) return refuse(ARGUS_E_INVAL, "vocab %u (1..2^24)", c->vocab);
  if (c->top > kMaxTop) return refuse(ARGUS_E_INVAL, "top %u (0..64)", c->top);
  if (c->rows > (1u << 22)) return refuse(ARGUS_E_CAPACITY, "rows %u", c->rows);
  const uint32_t steps = (c->vocab + kStep - 1) / kStep;
  uint32_t parts = c->rows ? kRowBlocks / c->rows : 1;
  p->waves = steps > kWaves && c->rows <= kFewRows &&
                     (steps <= kManyWaves || (c->rows > kFewRows / 2 && steps <= kFewSteps * kManyWaves))
                 ? kManyWaves : kWaves;
  if (p->waves == kManyWaves) parts = 1;
  uint32_t most = (steps + kWaves - 1) / kWaves;
  if (c->top && kCands / c->top < most) most = kCands / c->top;
  parts = parts < most ? parts : most;
  parts = parts < 1 ? 1 : parts;
  p->steps = (steps + parts - 1) / parts;
  p->parts = (steps + p->steps - 1) / p->steps;
  p->grid = c->rows * p->parts;
  p->cands_at = up256((size_t)p->grid * sizeof(Sums));
  p->bytes = p->parts > 1 ? p->cands_at + up256((size_t)p->grid * c->top * sizeof(uint64_t)) : 0;
  return ARGUS_OK;
}

}  // namespace
}  // namespace prompt
}  // namespace argus

using namespace argus;
using namespace argus::prompt;

extern "C" size_t argus_prompt_score_workspace_bytes(const argus_score_config* cfg) {
  accepted();
  Plan p;
  return make_plan(cfg, &p) == ARGUS_OK ? p.bytes : (size_t)-1;
}

extern "C" int argus_prompt_score(const argus_score_config* cfg, const argus_score_io* io, void* d_workspace,
                                  size_t workspace_bytes, argus_markers* markers, void* stream_v) {
  accepted();
  Plan p;
  int rc = make_plan(cfg, &p);
  if (rc != ARGUS_OK) return rc;
  if (!io || (cfg->rows && (!io->d_logits || !io->d_tokens || !io->d_logprobs || !io->d_entropy || !io->d_ranks ||
                            (cfg->top && (!io->d_top_logprobs || !io->d_top_tokens)))))
    return refuse(ARGUS_E_INVAL, "a required pointer is NULL");
  const uint32_t e = type_bytes(cfg->type);
  if (!aligned_to(io->d_logits, e) || !aligned_to(io->d_tokens, 4) || !aligned_to(io->d_logprobs, 4) ||
      !aligned_to(io->d_entropy, 4) || !aligned_to(io->d_ranks, 4) ||
      (cfg->top && (!aligned_to(io->d_top_logprobs, 4) || !aligned_to(io->d_top_tokens, 4))))
    return refuse(ARGUS_E_ALIGN, "buffers lie on their elements' size");
  if (marks_bad_all(markers)) return refuse(ARGUS_E_INVAL, "markers: alignment or region_base");
  if (p.bytes && !d_workspace) return refuse(ARGUS_E_INVAL, "no workspace");
  if (p.bytes && !aligned_to(d_workspace, 256)) return refuse(ARGUS_E_ALIGN, "the workspace lies on 256 bytes");
  if (workspace_bytes < p.bytes) return refuse(ARGUS_E_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, p.bytes);
  const uint32_t joins = p.parts > 1 ? cfg->rows : 0;
  if (!marks_fit(markers, ((uint64_t)p.grid * p.waves + joins * kWaves) * 2))
    return refuse(ARGUS_E_CAPACITY, "the marker records do not fit");
  if (cfg->rows == 0) return ARGUS_OK;
  if ((rc = device_ok()) != ARGUS_OK) return rc;
  ScoreArgs a{};
  a.logits = (const uint8_t*)io->d_logits, a.row_stride = io->row_stride * e, a.tokens = io->d_tokens;
  a.logprobs = io->d_logprobs, a.entropy = io->d_entropy, a.ranks = io->d_ranks;
  a.top_logprobs = io->d_top_logprobs, a.top_tokens = io->d_top_tokens;
  a.sums = (Sums*)d_workspace;
  a.cands = (uint64_t*)((char*)d_workspace + p.cands_at);
  a.V = cfg->vocab, a.K = cfg->top, a.parts = p.parts, a.steps = p.steps, a.rows = cfg->rows;
  hipStream_t st = (hipStream_t)stream_v;
  a.marks = take_marks(markers, p.grid * (p.waves / kWaves), 2);
  if (cfg->type == ARGUS_BF16) launch_score<ARGUS_BF16>(a, p.grid, p.waves, st);
  else if (cfg->type == ARGUS_FP16) launch_score<ARGUS_FP16>(a, p.grid, p.waves, st);
  else launch_score<ARGUS_FP32>(a, p.grid, p.waves, st);
  if (joins) {
    a.marks = take_marks(markers, joins, 2);
    if (cfg->type == ARGUS_BF16) hipLaunchKernelGGL(k_score_join<ARGUS_BF16>, dim3(joins), dim3(kThreads), 0, st, a);
    else if (cfg->type == ARGUS_FP16) hipLaunchKernelGGL(k_score_join<ARGUS_FP16>, dim3(joins), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL(k_score_join<ARGUS_FP32>, dim3(joins), dim3(kThreads), 0, st, a);
  }
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}
