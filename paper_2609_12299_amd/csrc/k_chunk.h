// k_chunk.h -- attention of chunks of new tokens over a paged cache.
//
// The queries of one sequence that share a key/value head, `group` of them for each
// new token, are rows r = token * group + head of one matrix; a block takes a tile of
// them (32 rows a wave) and goes over the tokens that its rows see, KT at a time:
//
//   S^T[token][row] = K[token][d] Q^T[d][row]    mfma 32x32x16
//   P = exp(S^T * c - m)                         c = scale * k_scale, m per row
//   O^T[d][row] += V^T[d][token] P^T[token][row] mfma 32x32x16
//
// With rows as columns a lane holds 16 scores of one row, half a wave apart from the
// other 16, and what the first product leaves in its registers is what the second takes:
// which token stands at which place of a contraction is free. Keys and values go through
// LDS, read once for the block; queries and O stay in registers. Weights are rounded once, to the 16 bits that
// the second product takes (to the nearest; in fp16 times 2^7, so that small ones keep their bits: those below 2^-32 of
// the largest have none left, and count in the sums alone), their sums are
// of the unrounded ones in 32 bits: a row's answer is off by half a step of a value at most, in all by 1.2 to 1.4 times
// what the answer's own rounding is. (As two 16-bit numbers they would take half as many matrix instructions again.)
//
// What bounds it. Long chunks: the matrix cores and the exponentials, one after the other. One sequence of 16384 tokens,
// 8 x 8 heads of 128 in bf16 (4.4 TFLOP), takes 3.8 to 4.1 ms, 1070 to 1150 TFLOP/s; a library product of 8192^3 reaches 1220
// to 1270 on this card, at 2.0 to 2.1 GHz both. By the counters the matrix cores are busy 0.52 of the time and the vector units 0.46:
// the two waves of a SIMD, which the block's barrier lets go together, hide next to nothing of each
// other; half-blocks that take turns, and other priorities, measured the same. What gave time: eight
// waves a block instead of four (4.25 to 3.97 ms), fragments that are read from LDS four matrix instructions
// ahead (1 ahead 4.08, 4 3.97, 8 3.98), loads three steps ahead, straight into LDS.
// Few tokens over long contexts: the cache's bytes. 4 sequences of 131000 tokens with 6 new ones each read
// 2.1 GB in 340 us (6.3 TB/s, a plain read reaches 6.7). Prompts of a few hundred tokens: the steps of the longest row
// tile, one after the other.
#pragma once

#include "k_attend.h"
#include "prompt.h"

namespace argus {
namespace prompt {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// Tokens of a step: a buffer of keys and values is 32 KiB at head sizes of 128 and 256.
template <int DP>
constexpr int kStepTokens = DP == 256 ? 32 : 64;

// Buffers of a step's keys and values: four where a block has a compute unit's LDS to itself, so that loads are
// three steps ahead. In 8 bits the step under way lies in registers.
template <bool F8, int DP, int W>
constexpr int kBuffers = !F8 && (W == 8 || DP == 256) ? 4 : 2;

struct ChunkArgs {
  const uint16_t* q;
  int64_t q_row, q_head;
  const uint8_t *k, *v;
  int64_t k_head, v_head, k_page, v_page;  // bytes
  uint32_t k_tok, v_tok;                   // bytes
  const int32_t* table;
  int64_t table_stride;
  const int32_t *lens, *offsets;
  const float *k_scale, *v_scale;
  uint16_t* out;
  float* lse;
  // in pieces: what the plan leaves, and what the pieces do
  uint64_t* head;    // [0] pieces of a head, [1] items that are cut, [2] most steps of a piece, [3] pieces of those
  uint4* items;      // [slots] sequence, row tile, steps
  uint4* joins;      // items that are cut: sequence, row tile, first piece, steps
  uint4* pieces;     // sequence, row tile, steps from .. to; those of items that are cut first
  float* part_o;     // [pieces of items that are cut][H][TR][DP]
  float* part_ml;    // [...][H][TR][2]
  uint32_t S, rows, H, G, D;
  uint32_t slots, tile_shift;  // row tiles that there may be; rows of one
  uint32_t blocks;             // that run at once; 0: a row tile each
  uint32_t step_shift;                 // tokens of a step
  uint32_t shift, num_pages, columns, window, sinks;
  FastDiv by_group;
  float scale;
  Marks marks;
};

// The thread's number and the kernel's arguments as values that the compiler knows nothing of: what follows
// from them is worked out where it is used. Kept from one row tile to the next it would take
// the registers that the steps need.
ARGUS_DEV uint32_t fresh_thread() {
  uint32_t tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid;
}
ARGUS_DEV ChunkArgs fresh_args() {
  auto p = (const __attribute__((address_space(4))) void*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  ChunkArgs a;
  __builtin_memcpy(&a, (const void*)p, sizeof(a));
  return a;
}

// What of the cache a row tile looks at: steps [0, sink_steps), then steps from `first` on.
struct Reach {
  uint32_t s, row0, r0, rows;  // sequence, its first row, the tile's first row and how many it has
  int32_t pos0;                // position of the sequence's first row
  uint32_t len;                // tokens of the sequence
  uint32_t sink_steps, first, steps;
};

// Row tile x of the batch: sequence s owns the slots from slot_of(s) on, one at least for
// each of its row tiles, whatever lies before it: no sum over the sequences is needed.
ARGUS_DEV uint32_t slot_of(const ChunkArgs& a, uint32_t s) {
  return (uint32_t)(((uint64_t)row_at(a.offsets, s, a.rows) * a.G) >> a.tile_shift) + s;
}

ARGUS_DEV uint32_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
ARGUS_DEV const uint8_t* scalar(const uint8_t* p) {
  const uint64_t x = (uint64_t)(uintptr_t)p;
  return (const uint8_t*)(uintptr_t)join64(scalar((uint32_t)x), scalar((uint32_t)(x >> 32)));
}
// What all threads of a block have alike, as scalars.
ARGUS_DEV Reach scalar(const Reach& r) {
  Reach u;
  u.s = scalar(r.s), u.row0 = scalar(r.row0), u.r0 = scalar(r.r0), u.rows = scalar(r.rows);
  u.pos0 = (int32_t)scalar((uint32_t)r.pos0), u.len = scalar(r.len);
  u.sink_steps = scalar(r.sink_steps), u.first = scalar(r.first), u.steps = scalar(r.steps);
  return u;
}

// false: the slot has no rows.
ARGUS_DEV bool reach_of(const ChunkArgs& a, uint32_t s, uint32_t rt, Reach* r) {
  const uint32_t lo = row_at(a.offsets, s, a.rows), hi = row_at(a.offsets, s + 1, a.rows);
  const uint32_t n = hi > lo ? hi - lo : 0;
  const uint64_t r0 = (uint64_t)rt << a.tile_shift;
  if (r0 >= (uint64_t)n * a.G) return false;
  r->s = s, r->row0 = lo, r->r0 = (uint32_t)r0;
  const uint32_t left = n * a.G - r->r0, most = 1u << a.tile_shift;
  r->rows = left < most ? left : most;
  const int32_t l = a.lens[s];
  const uint32_t cap = a.columns << a.shift;
  r->len = l < 0 ? 0u : ((uint32_t)l < cap ? (uint32_t)l : cap);
  r->pos0 = (int32_t)r->len - (int32_t)n;
  const int32_t p0 = r->pos0 + (int32_t)divide(r->r0, a.by_group);
  const int32_t p1 = r->pos0 + (int32_t)divide(r->r0 + r->rows - 1, a.by_group);
  const uint32_t end = p1 < 0 ? 0u : (uint32_t)p1 + 1;
  const uint32_t low = a.window && p0 >= 0 && (uint32_t)p0 + 1 > a.window ? (uint32_t)p0 + 1 - a.window : 0u;
  const uint32_t ones = (1u << a.step_shift) - 1, sinks = low ? a.sinks : 0u;
  r->first = low >> a.step_shift;
  r->sink_steps = (sinks + ones) >> a.step_shift;
  if (r->sink_steps >= r->first) r->sink_steps = r->first = 0;
  r->steps = r->sink_steps + ((end + ones) >> a.step_shift) - r->first;
  if (r->steps == 0) r->steps = 1;  // rows that see nothing answer too
  return true;
}

template <int T>
ARGUS_DEV f32x16 mfma32(u32x4 x, u32x4 y, f32x16 c) {
  if constexpr (T == 0)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}

// A row of LDS has its chunks of 16 bytes in another order for each of 16 rows (8 at head
// size 64), so that the rows that are read together, 16 of keys or 4 of values (four chunks each),
// lie in different banks.
template <int DP>
ARGUS_DEV uint32_t swizzle(uint32_t row) {
  return DP == 64 ? (row >> 1 & 1u) << 2 | (row >> 2 & 3u) : (row & 3u) << 2 | (row >> 2 & 3u);
}

typedef __attribute__((address_space(3))) uint8_t lds_byte;
ARGUS_DEV u32x4 lds16(const lds_byte* p) { return *(const __attribute__((address_space(3))) u32x4*)p; }

// 16 bytes of each lane from base + at to LDS, one lane's after the other's from `to` on. It
// has no registers to write; who reads them waits for the loads' count first. (M0, which says where
// to, holds nothing of the compiler's from one of its own instructions to another.)
ARGUS_DEV void to_lds(const uint8_t* base, uint32_t at, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(at), "s"(base), "s"(to) : "memory");
}
// The same for some lanes of a wave all of whose lanes are active, without a branch.
ARGUS_DEV void to_lds(const uint8_t* base, uint32_t at, uint32_t to, uint64_t lanes) {
  asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1" ::"v"(at), "s"(base),
               "s"(to), "s"(lanes)
               : "memory");
}

// What is read once, past the caches.
ARGUS_DEV void to_lds_once(const uint8_t* base, uint32_t at, uint32_t to, uint64_t lanes) {
  asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %0, %1 nt\n\ts_mov_b64 exec, -1" ::"v"(at), "s"(base),
               "s"(to), "s"(lanes)
               : "memory");
}
// 4 bytes of each lane.
ARGUS_DEV void to_lds_word(const uint8_t* base, uint32_t at, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(at), "s"(base), "s"(to) : "memory");
}

// N matrix instructions that take a fragment each, read from LDS some ahead: barriers that only vector, scalar and
// exponential instructions may pass keep the reads from coming later. (Groups for the compiler's scheduler in their place
// were given up by it in some kernels, in others after any change, and reads came one ahead: one prompt of 2048 tokens
// 59.9 us against 53.8 so, head size 256 474 against 409. Barriers that nothing passes: 1330 us in 8 bits against 1310.)
constexpr int kFragsAhead = 4;
constexpr int kVector = 0x2, kScalar = 0x4, kExponential = 0x400;  // that a barrier lets pass
template <int N, class Read, class Take>
ARGUS_DEV void fragments(Read read, Take take) {
#pragma unroll
  for (int i = 0; i < kFragsAhead; ++i) read(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_barrier(kVector | kScalar | kExponential);
    take(i);
    if (i + kFragsAhead < N) read(i + kFragsAhead);
  }
}

// Bits of 16-bit numbers whose exponent is all ones: infinities and NaN.
template <int T>
ARGUS_DEV uint32_t not_finite(uint32_t w) {
  return T == 0 ? ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u : ((w & 0x7C007C00u) + 0x04000400u) & 0x80008000u;
}

template <int T>
constexpr uint32_t kFrac = T == 0 ? 7 : 10;  // bits of a fraction
template <int T>
constexpr uint32_t kFracs = ((1u << kFrac<T>) - 1) * 0x10001u;

// O, maxima and sums of steps [t0, t1) of a row tile for one head. Rows of LDS have room for DP elements, of which DC
// are multiplied (at head size 96, of 128, a quarter of the products less: a batch of single tokens and chunks 139 us
// against 150, 4 prompts of up to 6000 tokens 469 against 523).
template <int T, bool F8, int DP, int DC, int W>
ARGUS_DEV void chunk_steps(const ChunkArgs& a, const Reach& g, uint32_t h, uint32_t t0, uint32_t t1, lds_byte* lds,
                           f32x16 (&acc)[DC / 32], float& m, float& l) {
  constexpr int KT = kStepTokens<DP>, HT = KT / 32;      // halves of a step
  constexpr int KF = DC / 16, DB = DC / 32;              // fragments of a key row, 32-wide parts of O
  constexpr uint32_t kRuns = KT / 8;                     // of eight tokens, in a step
  constexpr int RUNS = kRuns / W;                        // that a wave loads
  constexpr int NB = kBuffers<F8, DP, W>, PD = NB - 1;   // buffers; steps that loads are ahead
  constexpr uint32_t kRow = DP * 2, kSide = KT * kRow;
  // a lane's part of a load: CE elements, NI loads a run, RI rows a load
  constexpr int CE = F8 && DP > 64 ? 16 : 8, LR = DP / CE, RI = 64 / LR, NI = 8 / RI;
  constexpr int CW = F8 ? CE / 4 : 4;
  using Hf = Half<T>;
  const uint32_t tid = fresh_thread(), lane = tid & 63u, c = lane & 31u, hk = lane >> 5;
  const uint32_t wave = scalar(tid >> 6);
  const float kc = a.scale * (a.k_scale ? a.k_scale[h] : 1.0f), kd = fabsf(kc), kd2 = kd * kLog2e;
  bool far = !(kd > 1e-30f && kd < 1e30f);  // scores so large, or a scale so odd, that the differences come first

  // queries: lane (row c, half hk) holds elements 16 f + 8 hk ... of its row
  u32x4 qf[KF];
  const uint32_t at0 = 32 * wave, mine = at0 + c;
  const bool in = mine < g.rows;
  const uint32_t r = g.r0 + (in ? mine : 0), row_tok = divide(r, a.by_group), head = h * a.G + r - row_tok * a.G;
  const uint16_t* qr = a.q + (int64_t)(g.row0 + row_tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
  for (int f = 0; f < KF; ++f) {
    const uint32_t d = 16 * f + 8 * hk;
    qf[f] = in && d < a.D ? *reinterpret_cast<const u32x4*>(qr + d) : (u32x4)(0u);
    if (kc < 0.0f) qf[f] ^= 0x80008000u;  // so that the largest product is the largest score
  }
  // the row sees tokens below `end`, from `low` on (and the sinks)
  const int32_t pos = g.pos0 + (int32_t)row_tok, end = in ? pos + 1 : 0, low = a.window ? pos + 1 - (int32_t)a.window : 0;
  // of the wave's rows, as scalars; none: nothing is seen
  const int32_t p_least = at0 < g.rows ? g.pos0 + (int32_t)divide(g.r0 + at0, a.by_group) : -1;
  const int32_t p_most = at0 < g.rows ? g.pos0 + (int32_t)divide(g.r0 + (at0 + 32 < g.rows ? at0 + 31 : g.rows - 1), a.by_group) : -1;
  m = -INFINITY;
  l = 0.0f;
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = (f32x16)(0.0f);
  float base = 0.0f;  // the maximum to base 2, less kRaise
  // infinite values that the row has seen, a bit for each of the lane's elements (both: NaN)
  constexpr int kBits = (DB + 3) / 4;
  uint64_t plus[kBits] = {}, minus[kBits] = {};

  auto token_of = [&](uint32_t t) { return (t < g.sink_steps ? t : t - g.sink_steps + g.first) * KT; };
  const uint32_t in_page = (1u << a.shift) - 1;

  // The pages: a lane looks after one run of eight tokens, 64 / kRuns steps in a row. The table's entries
  // come to LDS, where each wave has a place of its own for this group of steps and for the next,
  // so that no register waits for them.
  constexpr uint32_t kGroup = 64 / kRuns;
  const uint8_t* tab = (const uint8_t*)(a.table + (int64_t)g.s * a.table_stride);
  lds_byte* const ring = lds + 2 * NB * kSide + wave * 512;
  auto column = [&](uint32_t s0) {
    const uint32_t s = s0 + lane / kRuns;
    return (token_of(s < t1 ? s : t1 - 1) + 8 * (lane % kRuns)) >> a.shift;
  };
  auto fetch = [&](uint32_t s0) {  // entries of steps from s0 on
    const uint32_t col = column(s0);
    to_lds_word(scalar(tab), (col < a.columns ? col : 0) * 4, (uint32_t)(uintptr_t)ring + ((s0 - t0) / kGroup & 1u) * 256);
  };
  uint64_t place_k, place_v, held64;
  uint32_t tokens;  // of the lane's run that there are
  auto use = [&](uint32_t s0) {
    const int32_t entry = *(const __attribute__((address_space(3))) int32_t*)(ring + ((s0 - t0) / kGroup & 1u) * 256 + lane * 4);
    const bool held = column(s0) < a.columns && (uint32_t)entry < a.num_pages;
    const uint32_t s = s0 + lane / kRuns, first = token_of(s < t1 ? s : t1 - 1) + 8 * (lane % kRuns);
    const uint32_t page = held ? (uint32_t)entry : 0u, place = first & in_page;
    place_k = (uint64_t)page * (uint64_t)a.k_page + (uint64_t)place * a.k_tok;
    place_v = (uint64_t)page * (uint64_t)a.v_page + (uint64_t)place * a.v_tok;
    tokens = held && first < g.len ? g.len - first : 0u;
    held64 = __ballot(held);
  };

  // What a lane adds to the scalar base of a load, and whether it has anything to load.
  const uint8_t* kb = a.k + (int64_t)h * a.k_head;
  const uint8_t* vb = a.v + (int64_t)h * a.v_head;
  const uint32_t lr = lane / LR, lc = lane % LR;
  uint32_t k_at[RUNS][NI], v_at[RUNS][NI], loads = 0;
  uint64_t lanes[RUNS][NI];
#pragma unroll
  for (int j = 0; j < RUNS; ++j)
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const uint32_t row = 8 * (wave * RUNS + j) + i * RI + lr;
      const uint32_t chunk = F8 ? lc : lc ^ swizzle<DP>(row);
      const uint32_t b = chunk * (F8 ? CE : 16);
      const bool some = chunk * CE < a.D;
      // (in 8 bits, behind the head size: elements of the row once more, taken off where they land)
      k_at[j][i] = (i * RI + lr) * a.k_tok + (F8 && !some ? 0 : b);
      v_at[j][i] = (i * RI + lr) * a.v_tok + (F8 && !some ? 0 : b);
      loads |= some ? 1u << (j * NI + i) : 0u;
      lanes[j][i] = __ballot(some);
    }
  const bool padded = a.D != DP;
  uint32_t staged[F8 ? 2 : 1][RUNS][NI][F8 ? CW : 1];
  typedef uint32_t words __attribute__((ext_vector_type(CW)));
  // Step s's keys (side 0) and values on their way, into LDS or (8 bits) registers. What lies behind
  // the sequence's end or in no page is 0; where nothing does, without a look at that.
  // (Four waves: few rows of a sequence, which read most of it once, past the caches. 4 sequences of 131000
  // tokens with 6 new ones each 340 us against 382, 64 of up to 30000 with one 278 against 306, and batches in which
  // row tiles share what they read the same.)
  auto load = [&](uint32_t s, int buffer, auto all_of) {
    constexpr bool all = all_of(), once = W == 4;
    const uint32_t run0 = (s - t0) % kGroup * kRuns + wave * RUNS;
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
      for (int j = 0; j < RUNS; ++j) {
        const uint64_t place = side ? place_v : place_k;
        const uint8_t* from = scalar((side ? vb : kb) + join64(__builtin_amdgcn_readlane((uint32_t)place, run0 + j),
                                                               __builtin_amdgcn_readlane((uint32_t)(place >> 32), run0 + j)));
        const uint32_t have = all ? 8u : __builtin_amdgcn_readlane(tokens, run0 + j);
        lds_byte* to = lds + (side * NB + buffer) * kSide + 8 * (wave * RUNS + j) * kRow;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const uint32_t at = (side ? v_at : k_at)[j][i];
          if constexpr (F8) {
            words x = (words)(0u);
            if (all || i * RI + lr < have)
              x = once ? __builtin_nontemporal_load(reinterpret_cast<const words*>(from + at)) : *reinterpret_cast<const words*>(from + at);
#pragma unroll
            for (int w = 0; w < CW; ++w) staged[side][j][i][w] = x[w];
          } else if constexpr (all) {
            if constexpr (once) to_lds_once(from, at, (uint32_t)(uintptr_t)to + i * RI * kRow, lanes[j][i]);
            else to_lds(from, at, (uint32_t)(uintptr_t)to + i * RI * kRow, lanes[j][i]);
          } else {
            const bool there = i * RI + lr < have;
            if (there && (loads >> (j * NI + i) & 1u)) to_lds(from, at, (uint32_t)(uintptr_t)to + i * RI * kRow);
            if (!there) *(__attribute__((address_space(3))) u32x4*)(to + i * RI * kRow + lane * 16) = (u32x4)(0u);
          }
        }
      }
  };
  auto land = [&](int buffer) {
    if constexpr (F8) {
#pragma unroll
      for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int j = 0; j < RUNS; ++j)
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const uint32_t row = 8 * (wave * RUNS + j) + i * RI + lr;
            lds_byte* to = lds + (side * NB + buffer) * kSide + row * kRow;
            const uint32_t some = loads >> (j * NI + i) & 1u ? ~0u : 0u;
#pragma unroll
            for (int e = 0; e < CE / 8; ++e) {
              const uint32_t w0 = staged[side][j][i][2 * e] & some, w1 = staged[side][j][i][2 * e + 1] & some;
              const u32x4 x = (u32x4){widen<T>(w0, false), widen<T>(w0, true), widen<T>(w1, false), widen<T>(w1, true)};
              *(__attribute__((address_space(3))) u32x4*)(to + (((lc * (CE / 8) + e) ^ swizzle<DP>(row)) << 4)) = x;
            }
          }
    }
  };

  // Where a lane's fragments lie: their addresses stay in registers, what differs beside them is
  // in the instructions.
  const uint32_t i16 = lane & 15u, piece = i16 & 3u, v_row = 4 * hk + (i16 >> 2);
  uint32_t k_frag[KF], v_frag[DB][2];
#pragma unroll
  for (int f = 0; f < KF; ++f) {
    k_frag[f] = (uint32_t)(uintptr_t)lds + c * kRow + (((2 * f + hk) ^ swizzle<DP>(c)) << 4);
    asm volatile("" : "+v"(k_frag[f]));
  }
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t chunk = 4 * d + 2 * (piece & 1u) + (lane >> 4 & 1u), row = v_row + 8 * e;
      v_frag[d][e] = (uint32_t)(uintptr_t)lds + NB * kSide + row * kRow + ((chunk ^ swizzle<DP>(row)) << 4) + (piece >> 1) * 8;
      asm volatile("" : "+v"(v_frag[d][e]));
    }
  auto k_part = [&](int buffer, int th, int f) { return lds16((const lds_byte*)(uintptr_t)(k_frag[f] + (buffer * kSide + th * 32 * kRow))); };
  // Fragment (d, f) of V^T: lane (m, hk) has tokens 16 f + 8 e + 4 hk + 0..3, e = 0, 1, of
  // element 32 d + 16 (m / 4 % 2) + 4 (m / 8) + m % 4, so that a lane of O^T holds 16 elements in a row.
  auto v_part = [&](int buffer, int d, int f) {
    u32x4 x;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)(uintptr_t)(v_frag[d][e] + (buffer * kSide + 16 * f * kRow)));
      x[2 * e] = __builtin_bit_cast(u32x2, y).x, x[2 * e + 1] = __builtin_bit_cast(u32x2, y).y;
    }
    return x;
  };

  // Steps [from, to) behind the sinks' whose tokens rows of positions p0 to p1 all see.
  struct Range {
    uint32_t from, to;
  };
  auto all_seen = [&](int32_t p0, int32_t p1) {
    const uint32_t shift = g.first - g.sink_steps;  // of a step's number behind the sinks' and its tokens'
    const uint32_t lo = a.window && p1 >= 0 && (uint32_t)p1 + 1 > a.window ? (uint32_t)p1 + 1 - a.window : 0u;
    Range x{(lo + KT - 1) / KT - shift, p0 < 0 ? 0u : ((uint32_t)p0 + 1) / KT - shift};
    if ((lo + KT - 1) / KT < g.first || x.from < g.sink_steps) x.from = g.sink_steps;
    if (p0 < 0 || ((uint32_t)p0 + 1) / KT < g.first || x.to < x.from) x.to = x.from;
    return x;
  };
  const Range mine_all = all_seen(p_least, p_most);
  const Range block_all = all_seen(g.pos0 + (int32_t)divide(g.r0, a.by_group), g.pos0 + (int32_t)divide(g.r0 + g.rows - 1, a.by_group));
  constexpr uint32_t kHeld = (1u << kRuns) - 1;
  f32x16 sc[HT];  // scores, then weights
  auto score = [&](int buffer) {
#pragma unroll
    for (int th = 0; th < HT; ++th) sc[th] = (f32x16)(0.0f);
    u32x4 k[KF * HT];
    auto read = [&](int i) { k[i] = k_part(buffer, i % HT, i / HT); };
    fragments<KF * HT>(read, [&](int i) { sc[i % HT] = mfma32<T>(k[i], qf[i / HT], sc[i % HT]); });
  };
  auto weigh = [&](uint32_t tok, uint32_t held, bool whole) {
    if (__builtin_expect(!whole, 0)) {
      // of the lane's 16 HT tokens, tok + 4 hk + 0..3, + 8..11, ..., those below x
      auto below = [&](int32_t x) {
        const int32_t y = x - (int32_t)(tok + 4 * hk), k = y < 0 ? 0 : 4 * (y >> 3) + ((y & 7) < 4 ? y & 7 : 4);
        return k < 32 ? (1u << k) - 1 : ~0u;
      };
      uint32_t vis = below(end) & (~below(low) | below((int32_t)a.sinks));
      if (held != kHeld) {
        uint32_t by_four = 0;
#pragma unroll
        for (uint32_t i = 0; i < kRuns; ++i) by_four |= held >> i & 1u ? 15u << (4 * i) : 0u;
        vis &= by_four;
      }
#pragma unroll
      for (int th = 0; th < HT; ++th)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[th][i] = vis >> (16 * th + i) & 1u ? sc[th][i] : -INFINITY;
    }
    float top = sc[0][0];
#pragma unroll
    for (int th = 0; th < HT; ++th)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[th][i]);
    top = top == -INFINITY ? top : top * kd;  // (kd may be 0)
    if (__builtin_expect(__any(top > m + kSlack), 0)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top);
      const float scale = m == -INFINITY ? 0.0f : exp_of(m - mn);
      l *= scale;
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[d] *= scale;
      m = mn;
      base = mn == -INFINITY ? 0.0f : fmaf(mn, kLog2e, -Hf::kRaise);
      far = far || __any(fabsf(mn) > kFar && mn != -INFINITY);
    }
#pragma unroll
    for (int th = 0; th < HT; ++th) {
      if (__builtin_expect(!far, 1)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[th][i] = __builtin_amdgcn_exp2f(fmaf(sc[th][i], kd2, -base));
      } else {
        const float ms = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = sc[th][i], y = x == -INFINITY ? x : x * kd;
          sc[th][i] = __builtin_amdgcn_exp2f(fmaf(y - ms, kLog2e, Hf::kRaise));
        }
      }
    }
  };
  // The weights' sums, and their rounding for the next products, beside the matrix instructions.
  auto apply = [&](int buffer) {
    u32x4 v[2 * HT * DB], p[2 * HT];
    float sum[4];
    auto round = [&](int f) {
#pragma unroll
      for (int j = 0; j < 4; ++j) p[f][j] = Hf::pack(sc[f / 2][f % 2 * 8 + 2 * j], sc[f / 2][f % 2 * 8 + 2 * j + 1]);
    };
    round(0);
    fragments<2 * HT * DB>([&](int i) { v[i] = v_part(buffer, i % DB, i / DB); },
                           [&](int i) {
                             const int f = i / DB, d = i % DB;
                             acc[d] = mfma32<T>(v[i], p[f], acc[d]);
                             if (d == 0 && f + 1 < 2 * HT) round(f + 1);
#pragma unroll
                             for (int e = 8 * d / DB; e < 8 * (d + 1) / DB; ++e) {
                               const float w = sc[f / 2][f % 2 * 8 + e];
                               sum[e % 4] = f == 0 && e < 4 ? w : sum[e % 4] + w;
                             }
                           });
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };

  // Of a step that some of the block's rows do not see, the values that are not finite (0 times infinity
  // would be NaN): noted where they are seen, and 0 from then on.  All waves look at the same
  // values, so they come to the same answer.
  auto settle = [&](uint32_t t, uint32_t held, int buffer) {
    if (__builtin_expect(t >= block_all.from && t < block_all.to, 1)) return;
    lds_byte* const values = lds + (NB + buffer) * kSide;
    uint32_t odd = 0;
#pragma unroll 4
    for (uint32_t i = 0; i < kSide / 1024; ++i) {
      const u32x4 x = lds16(values + i * 1024 + lane * 16);
      odd |= not_finite<T>(x[0]) | not_finite<T>(x[1]) | not_finite<T>(x[2]) | not_finite<T>(x[3]);
    }
    if (__builtin_expect(!__any(odd), 1)) return;
    const uint32_t tok = token_of(t);
#pragma unroll 1
    for (uint32_t j = 0; j < (uint32_t)KT; ++j) {
      const int32_t at = (int32_t)(tok + j);
      const bool seen = at < end && (at >= low || at < (int32_t)a.sinks) && (held >> (j / 8) & 1u);
#pragma unroll 1
      for (uint32_t e = 0; e < 2 * DB; ++e) {  // eight of the lane's elements
        const u32x4 x = lds16(values + j * kRow + (((4 * (e / 2) + 2 * hk + e % 2) ^ swizzle<DP>(j)) << 4));
        uint32_t up = 0, down = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t bad = seen ? not_finite<T>(x[w]) >> 15 : 0u, sign = x[w] >> 15 & 0x10001u;
          const uint32_t nan = bad & ((x[w] & kFracs<T>) + kFracs<T>) >> kFrac<T>, u = nan | (bad & ~sign), v = nan | (bad & sign);
          up |= ((u | u >> 15) & 3u) << (2 * w), down |= ((v | v >> 15) & 3u) << (2 * w);
        }
#pragma unroll
        for (int k = 0; k < kBits; ++k)
          if (e / 8 == (uint32_t)k) plus[k] |= (uint64_t)up << (8 * (e % 8)), minus[k] |= (uint64_t)down << (8 * (e % 8));
      }
    }
    __syncthreads();
#pragma unroll 1
    for (uint32_t i = tid; i < kSide / 16; i += 64 * W) {
      u32x4 x = lds16(values + i * 16);
#pragma unroll
      for (int w = 0; w < 4; ++w) x[w] &= ~((not_finite<T>(x[w]) >> 15) * 0xFFFFu);
      *(__attribute__((address_space(3))) u32x4*)(values + i * 16) = x;
    }
    __syncthreads();
  };

  // All waves have come this far, and what they wrote to LDS is there; of their loads all but the
  // last N.
  auto meet = [&](auto last_of) {
    constexpr int N = last_of();
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
  };
  constexpr auto none = []() constexpr { return 0; };
  // loads of a wave that may still be under way when a step's own have to be there: those of the steps
  // behind it
  constexpr auto rest = []() constexpr { return (PD - 1) * 2 * RUNS * NI; };
  constexpr auto some = []() constexpr { return false; };
  constexpr auto every = []() constexpr { return true; };
  meet(none);  // (what came before is done with the buffers)
  fetch(t0);
  if (padded) {  // elements behind the head size stay 0
    for (uint32_t i = tid; i < 2 * NB * kSide / 16; i += 64 * W)
      *(__attribute__((address_space(3))) u32x4*)(lds + i * 16) = (u32x4)(0u);
  }
  meet(none);
  use(t0);
  fetch(t0 + kGroup);
  uint32_t held[NB], sure = 0;  // of the steps that are loaded; how many of the last were loaded whole
#pragma unroll
  for (int i = 0; i < PD; ++i) {
    held[i] = (uint32_t)(held64 >> (i * kRuns)) & kHeld;
    if (t0 + i < t1) load(t0 + i, i, some);
    land(i);
  }
  auto step = [&](uint32_t t, auto buffer_of) {
    constexpr int b = buffer_of(), nb = (b + PD) % NB;
    // step t is there, and nobody reads step t - 1 any more
    if (PD > 1 && __builtin_expect(sure >= PD - 1, 1)) meet(rest);
    else meet(none);
    const uint32_t s = t + PD;
    if ((s - t0) % kGroup == 0) {
      use(s);
      fetch(s + kGroup);
    }
    held[nb] = (uint32_t)(held64 >> ((s - t0) % kGroup * kRuns)) & kHeld;
    // (as a scalar: all lanes go into load, which sets the mask of those that do)
    if (__builtin_expect(scalar(s >= block_all.from && s < block_all.to && s < t1 && held[nb] == kHeld ? 1u : 0u), 1)) {
      load(s, nb, every);
      ++sure;
    } else {
      if (s < t1) load(s, nb, some);
      sure = 0;
    }
    settle(t, held[b], b);
    // what the wave's rows see of the step: all of it, some, nothing
    bool whole = true, live = true;
    const uint32_t tok = token_of(t);
    if (__builtin_expect(t < mine_all.from || t >= mine_all.to || held[b] != kHeld, 0)) {
      const int32_t first = (int32_t)tok, last = first + KT - 1;
      whole = last <= p_least && held[b] == kHeld &&
              (!a.window || first > p_most - (int32_t)a.window || last < (int32_t)a.sinks);
      live = first <= p_most && held[b] && !(a.window && last <= p_least - (int32_t)a.window && tok >= a.sinks);
    }
    if (__builtin_expect(live, 1)) {
      score(b);
      weigh(tok, held[b], whole);
      apply(b);
    }
    if (s < t1) land(nb);
  };
  for (uint32_t t = t0; t < t1; t += NB) {
    step(t, []() constexpr { return 0; });
    if (t + 1 < t1) step(t + 1, []() constexpr { return 1; });
    if constexpr (NB == 4) {
      if (t + 2 < t1) step(t + 2, []() constexpr { return 2; });
      if (t + 3 < t1) step(t + 3, []() constexpr { return 3; });
    }
  }
  // (entries for steps that there are not: LDS is given back when the block ends)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  l += __shfl_xor(l, 32);
  uint64_t seen = 0;
#pragma unroll
  for (int k = 0; k < kBits; ++k) seen |= plus[k] | minus[k];
  if (__any(seen != 0)) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        acc[d][i] += plus[d / 4] >> (16 * (d % 4) + i) & 1u ? INFINITY : 0.0f;
        acc[d][i] -= minus[d / 4] >> (16 * (d % 4) + i) & 1u ? INFINITY : 0.0f;
      }
  }
}

// Which of a lane's elements (16 in a row from 32 d + 16 hk on, for each d) have values above, and which below all finite ones
// among the tokens of steps [t0, t1) that its row sees (NaN: both). For a wave whose rows came to NaN in elements `odd`: no
// further than until these are known to be. (A prompt of 16384 tokens all of which see a NaN 4.8 ms, without one 4.5.)
template <int T, int DP, int DC>
ARGUS_DEV void odd_values(const ChunkArgs& a, const Reach& g, uint32_t h, uint32_t t0, uint32_t t1, const uint32_t (&odd)[DC / 32],
                          uint32_t (&plus)[DC / 32], uint32_t (&minus)[DC / 32]) {
  constexpr int DB = DC / 32, KT = kStepTokens<DP>;
  const uint32_t tid = fresh_thread(), lane = tid & 63u, c = lane & 31u, hk = lane >> 5, mine = 32 * (tid >> 6) + c;
  const int32_t* tab = a.table + (int64_t)g.s * a.table_stride;
  const uint8_t* vb = a.v + (int64_t)h * a.v_head;
  const int32_t p0 = g.pos0 + (int32_t)divide(g.r0, a.by_group), p1 = g.pos0 + (int32_t)divide(g.r0 + g.rows - 1, a.by_group);
  const int32_t pos = g.pos0 + (int32_t)divide(g.r0 + (mine < g.rows ? mine : 0), a.by_group), end = mine < g.rows ? pos + 1 : 0;
  const int32_t low = a.window ? pos + 1 - (int32_t)a.window : 0, sinks = (int32_t)a.sinks;
  auto add = [&](u32x4 x, uint32_t& up, uint32_t& down) {  // of eight values
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t bad = not_finite<T>(x[w]) >> 15, sign = x[w] >> 15 & 0x10001u;
      const uint32_t nan = bad & ((x[w] & kFracs<T>) + kFracs<T>) >> kFrac<T>, u = nan | (bad & ~sign), v = nan | (bad & sign);
      up |= ((u | u >> 15) & 3u) << (2 * w), down |= ((v | v >> 15) & 3u) << (2 * w);
    }
  };
  auto value = [&](uint32_t at) {  // token `at`'s values; NULL: its page is not held
    const int32_t page = at < g.len ? tab[at >> a.shift] : -1;
    const uint8_t* r = vb + (int64_t)page * a.v_page + (uint64_t)(at & ((1u << a.shift) - 1)) * a.v_tok;
    return (uint32_t)page < a.num_pages ? r : nullptr;
  };
  uint32_t up = 0, down = 0;  // of steps that all of the block's rows see: eight elements of a lane, some tokens
  const uint32_t chunk = lane % (DP / 8);
  uint32_t open = 0;  // of the chunk's elements, those that are NaN in a row
#pragma unroll
  for (int d = 0; d < DB; ++d) {
    plus[d] = minus[d] = 0;
    uint32_t x = odd[d];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) x |= __shfl_xor(x, o);
    x = __shfl(x, chunk / 2 % 2 * 32);
    if (chunk / 4 == (uint32_t)d) open = x >> (8 * (chunk % 2)) & 255u;
  }
  auto lanes_of_a_chunk = [&](uint32_t x) {
#pragma unroll
    for (int o = DP / 8; o < 64; o <<= 1) x |= __shfl_xor(x, o);
    return x;
  };
#pragma unroll 1
  for (uint32_t t = t0; t < t1; ++t) {
    const int32_t first = (int32_t)((t < g.sink_steps ? t : t - g.sink_steps + g.first) * KT), last = first + KT - 1;
    if (last <= p0 && (!a.window || first > p1 - (int32_t)a.window || last < sinks)) {
      const uint32_t at = first + lane / (DP / 8);
      constexpr int kDeep = 4, kOf = 512 / DP;  // tokens at a time
#pragma unroll 1
      for (int j = 0; j < KT; j += kDeep * kOf) {
        const uint8_t* r[kDeep];
        u32x4 x[kDeep];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) r[i] = value(at + j + i * kOf);
#pragma unroll
        for (int i = 0; i < kDeep; ++i) x[i] = r[i] && 8 * chunk < a.D ? *reinterpret_cast<const u32x4*>(r[i] + 16 * chunk) : (u32x4)(0u);
#pragma unroll
        for (int i = 0; i < kDeep; ++i) add(x[i], up, down);
      }
      if (__all((open & ~lanes_of_a_chunk(up & down)) == 0)) break;
    } else {
#pragma unroll 1
      for (int32_t at = first; at <= last; ++at) {
        const uint8_t* r = value((uint32_t)at);
        if (r && at < end && (at >= low || at < sinks))
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (32 * d + 16 * hk + 8 * e < a.D) {
                uint32_t u = 0, v = 0;
                add(*reinterpret_cast<const u32x4*>(r + 2 * (32 * d + 16 * hk + 8 * e)), u, v);
                plus[d] |= u << (8 * e), minus[d] |= v << (8 * e);
              }
      }
    }
  }
  up = lanes_of_a_chunk(up), down = lanes_of_a_chunk(down);
#pragma unroll
  for (int d = 0; d < DB; ++d) {
    const uint32_t from = 4 * d + 2 * hk;
    plus[d] |= __shfl(up, from) | __shfl(up, from + 1) << 8, minus[d] |= __shfl(down, from) | __shfl(down, from + 1) << 8;
  }
}

template <int T, bool F8, int DP, int DC, int W, bool PIECES>
__global__ __launch_bounds__(64 * W, DP == 256 || W == 8 ? 1 : DP == 128 ? 2 : 3) void k_chunk(ChunkArgs a) {
  constexpr int DB = DC / 32, KT = kStepTokens<DP>, TR = 32 * W;
  using Hf = Half<T>;
  __shared__ __align__(1024) uint8_t s_raw[2 * kBuffers<F8, DP, W> * KT * DP * 2 + 512 * W];
  lds_byte* lds = (lds_byte*)s_raw;
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_CHUNK);
  // O of the rows, or (slot: not done) a piece of it, of steps t0 to t1
  auto put = [&](const ChunkArgs& a, const Reach& g, uint32_t h, const f32x16 (&acc)[DB], float m, float l, bool done,
                 uint64_t slot, uint32_t t0, uint32_t t1) {
    const uint32_t tid = fresh_thread(), c = tid & 31u, hk = tid >> 5 & 1u;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float vs = a.v_scale ? a.v_scale[h] : 1.0f;
    const uint32_t mine = 32 * wave + c;
    const bool in = mine < g.rows;
    const uint32_t r = g.r0 + (in ? mine : 0), tok = divide(r, a.by_group);
    const uint64_t row = (uint64_t)(g.row0 + tok) * a.H * a.G + h * a.G + (r - tok * a.G);
    const float inv = l == 0.0f ? 0.0f : vs / l;
    uint16_t* const out = a.out + row * a.D;
    float* const part = a.part_o + (slot * TR + mine) * DP;
    uint32_t nan = 0;
    if (in) {
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const uint32_t e = 32 * d + 16 * hk;
        if (done) {
#pragma unroll
          for (int i = 0; i < 16; i += 8)
            if (e + i < a.D) {
              u32x4 x;
#pragma unroll
              for (int w = 0; w < 4; ++w) x[w] = Hf::pack(acc[d][i + 2 * w] * inv, acc[d][i + 2 * w + 1] * inv);
              if (l == 0.0f) x = (u32x4)(0u);  // (whatever the values are)
              *reinterpret_cast<u32x4*>(out + e + i) = x;
            }
        } else {
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<f32x4*>(part + e + i) = (f32x4){acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
        }
        if constexpr (!F8)
#pragma unroll
          for (int i = 0; i < 16; ++i) nan |= acc[d][i] == acc[d][i] ? 0u : 1u;
      }
      if (hk == 0) {
        if (!done)
          *reinterpret_cast<f32x2*>(a.part_ml + (slot * TR + mine) * 2) = (f32x2){m, l};
        else if (a.lse)
          a.lse[row] = l == 0.0f ? -INFINITY : (m == -INFINITY ? 0.0f : m - Hf::kRaise * kLn2) + logf(l);
      }
    }
    if constexpr (!F8) {  // (e4m3 has no infinities)
      // An infinite value that all rows of a step see is NaN times a weight that is none in 16 bits, and NaN once a maximum
      // lies so far above its own that what came before is none. So where an element is NaN, and not by
      // its row's scores, it is what the values that the row sees make of it: infinite, or NaN.
      if (__builtin_expect(__any(nan && l == l && !(done && l == 0.0f)), 0)) {
        uint32_t odd[DB], plus[DB], minus[DB];
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          odd[d] = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) odd[d] |= in && l == l && acc[d][i] != acc[d][i] ? 1u << i : 0u;
        }
        odd_values<T, DP, DC>(fresh_args(), g, h, t0, t1, odd, plus, minus);
        if (in && l == l && !(done && l == 0.0f)) {
#pragma unroll 1
          for (uint32_t i = 0; i < 16 * DB; ++i) {
            uint32_t u = 0, v = 0;
#pragma unroll
            for (int d = 0; d < DB; ++d)
              if (i / 16 == (uint32_t)d) u = plus[d] >> (i % 16) & 1u, v = minus[d] >> (i % 16) & 1u;
            const float x = u && v ? NAN : u ? INFINITY : -INFINITY;
            const uint32_t e = 32 * (i / 16) + 16 * hk + i % 16;
            if (!(u | v)) continue;
            if (done) out[e] = (uint16_t)Hf::pack(x * inv, 0.0f);
            else part[e] = x;
          }
        }
      }
    }
  };

  f32x16 acc[DB];
  float m, l;
  Reach g;
  const uint32_t h = blockIdx.x % a.H;
  if constexpr (!PIECES) {
    // A row tile for the block: those that see the most tokens first.
    const uint32_t lane = threadIdx.x & 63u, x = a.slots - 1 - blockIdx.x / a.H;
    uint32_t lo = 0, hi = a.S;
    while (hi - lo > 1) {  // the last sequence whose slots start at or before x
      const uint32_t step = (hi - lo + 63) / 64, s = lo + lane * step;
      const uint32_t n = (uint32_t)__popcll(__ballot(s < hi && slot_of(a, s < hi ? s : lo) <= x));
      if (n == 0) break;
      lo += (n - 1) * step;
      hi = hi < lo + step ? hi : lo + step;
    }
    lo = scalar(lo);
    const uint32_t first = slot_of(a, lo);
    if (first <= x && reach_of(a, lo, x - first, &g)) {
      g = scalar(g);
      chunk_steps<T, F8, DP, DC, W>(a, g, h, 0, g.steps, lds, acc, m, l);
      put(a, g, h, acc, m, l, true, 0, 0, g.steps);
    }
  } else {
    const uint32_t q = blockIdx.x / a.H;
    if (q < (uint32_t)a.head[0]) {
      const uint4 piece = a.pieces[q];
      if (reach_of(a, scalar(piece.x), scalar(piece.y), &g)) {
        g = scalar(g);
        chunk_steps<T, F8, DP, DC, W>(a, g, h, scalar(piece.z), scalar(piece.w), lds, acc, m, l);
        const ChunkArgs e = fresh_args();
        put(e, g, h, acc, m, l, q >= (uint32_t)e.head[3], (uint64_t)q * e.H + h, scalar(e.pieces[q].z), scalar(e.pieces[q].w));
      }
    }
  }
  mk.end(ARGUS_REGION_CHUNK);
}

template <int T, bool F8, int DP, int DC, int W>
void launch_chunk_as(const ChunkArgs& a, uint32_t grid, hipStream_t st) {
  if (a.blocks) hipLaunchKernelGGL((k_chunk<T, F8, DP, DC, W, true>), dim3(grid), dim3(64 * W), 0, st, a);
  else hipLaunchKernelGGL((k_chunk<T, F8, DP, DC, W, false>), dim3(grid), dim3(64 * W), 0, st, a);
}

template <int T, bool F8>
void launch_chunk_type(const ChunkArgs& a, uint32_t grid, hipStream_t st) {
  if (a.D <= 64) {
    launch_chunk_as<T, F8, 64, 64, 4>(a, grid, st);
  } else if (a.D > 128) {
    launch_chunk_as<T, F8, 256, 256, 4>(a, grid, st);
  } else if (a.D <= 96) {
    if (a.tile_shift == 8) launch_chunk_as<T, F8, 128, 96, 8>(a, grid, st);
    else launch_chunk_as<T, F8, 128, 96, 4>(a, grid, st);
  } else {
    if (a.tile_shift == 8) launch_chunk_as<T, F8, 128, 128, 8>(a, grid, st);
    else launch_chunk_as<T, F8, 128, 128, 4>(a, grid, st);
  }
}

// One source file each, so that they compile side by side.
void launch_chunk_bf16(const ChunkArgs& a, uint32_t grid, hipStream_t st);
void launch_chunk_fp16(const ChunkArgs& a, uint32_t grid, hipStream_t st);
void launch_chunk_bf16_f8(const ChunkArgs& a, uint32_t grid, hipStream_t st);
void launch_chunk_fp16_f8(const ChunkArgs& a, uint32_t grid, hipStream_t st);

}  // namespace prompt
}  // namespace argus
