// k_attend.h -- attention of one new token per sequence over a paged cache.
//
// For one key/value head the `group` query heads that share it form the
// columns of a 16-wide matrix tile, and 32 tokens are one step of a wave:
//
//   S^T[token][q] = K[token][d] Q^T[d][q]        mfma 16x16x32, two token halves
//   P = exp(S^T * c - m)                         c = scale * k_scale, m per column
//   O^T[d][q] += V^T[d][token] P^T[token][q]     mfma 16x16x32
//
// Which token stands in which row of a product is free, and so is the order of the
// contractions, as long as both operands agree.  Row m = 4 g + r of a half of 16
// tokens is token place(m) = 8 (r / 2) + 2 g + r % 2, which makes every load below
// fall into one run of eight tokens, that is one page: its address is a scalar
// base and an offset per lane that never changes.
//
// The first product leaves lane (q = l % 16, g = l / 16) with rows 4 g + r of its
// column, and the second takes these eight registers as they are; V is read to
// match: lane (c, g) loads of token place(4 g + r) the VW = DP / 16 elements from
// c * VW on (16 lanes read a whole row), and 16-bit halves are then exchanged between
// registers.  K is wanted with 16 rows by 4 lanes each, which would read a part of
// 16 lines at a time.  So eight lanes read a run of 128 bytes of a row, eight rows per
// load, and lanes l and l ^ 2 trade places (in registers) for the rows of the other
// eight.  Nothing goes through LDS but the joining of a block's waves.
//
// What bounds it: the reading of the cache.  A tile of 32 tokens by 128
// elements is 16 KiB of bf16 and takes 24 matrix instructions of 16 cycles (P is
// taken as the sum of two 16-bit numbers, so that its rounding is not seen in
// the result), a third of the time that its bytes take.  Every byte is read once,
// by loads of whole lines, past the caches.  Measured: four sequences of 262143
// tokens, 8 x 8 heads of 128 in bf16, 4.3 GB: 643 us, 6.7 TB/s (with keys read by
// 16 rows x 64 bytes the same; values through the caches 707); 48 sequences of up to 32768
// tokens in 8 bits 64 us, 5.3 TB/s (73 before the keys' rows were read whole), 62 us for
// the shares and 6 for the joins.
//
// Shares: the units of work are the tiles (groups of 2^unit_shift tiles, where
// there could be more than 2^31) of all (sequence, head) segments one after the
// other, kPieceCost tiles more for each segment, and wave w takes units
// [w * per, (w + 1) * per) whatever the lengths are (they are known on the device
// alone): a batch of one long and many short sequences loads all compute
// units alike, and the short ones' latencies lie side by side.  A segment that lies
// in one share is finished there; of the others each wave leaves its piece (m, l,
// O in 32 bits), and k_attend_join joins them in the order of the shares: results
// do not depend on timing.  Where the table allows short sequences only, a block
// takes a segment and joins its four waves through LDS: one launch.
#pragma once

#include "decode.h"

namespace argus {
namespace decode {

constexpr uint32_t kTile = 32;        // tokens per step of a wave
constexpr uint32_t kMinShare = 4;     // units of a share, at least
constexpr uint32_t kPieceCost = 4;    // what a segment costs beside its tiles, in tiles

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct AttendArgs {
  const uint16_t* q;
  int64_t q_seq, q_head;
  const uint8_t *k, *v;
  int64_t k_head, v_head;               // bytes
  int64_t k_page, v_page;               // bytes
  uint32_t k_tok, v_tok;                // bytes
  const int32_t* table;
  int64_t table_stride;
  const int32_t* lens;
  const float *k_scale, *v_scale;
  uint16_t* out;
  float* lse;
  float* part_o;    // [shares][2][16 NQ][DP]
  float* part_ml;   // [shares][2][16 NQ][2]
  uint4* open;      // [min(shares, segments)] segment in pieces, its first and last share; y > z: none
  uint32_t S, H, G, D, HS, row_tiles;
  uint32_t shift, num_pages, columns, window, sinks;
  uint32_t shares;  // waves that share the batch
  uint32_t unit_shift;
  uint32_t by_seg;  // `open` goes by segment, else by share
  float scale;
  Marks marks;
};

// The tokens of a sequence that are looked at: tiles [0, sink_tiles), then tiles
// from `first` on.
struct Span {
  uint32_t len, lo, sinks, sink_tiles, first, tiles;
};

ARGUS_DEV Span span_of(const AttendArgs& a, int32_t n) {
  Span p;
  const uint32_t most = a.columns << a.shift;
  p.len = n < 0 ? 0u : ((uint32_t)n < most ? (uint32_t)n : most);
  p.lo = a.window && p.len > a.window ? p.len - a.window : 0u;
  p.sinks = p.lo ? a.sinks : 0u;
  p.first = p.lo / kTile;
  p.sink_tiles = (p.sinks + kTile - 1) / kTile;
  if (p.sink_tiles >= p.first) p.sink_tiles = p.first = 0;
  p.tiles = p.sink_tiles + (p.len + kTile - 1) / kTile - p.first;
  if (p.tiles == 0) p.tiles = 1;  // an empty sequence answers too
  return p;
}

template <int T>  // 0: bf16, 1: fp16
struct Half;
template <>
struct Half<0> {
  static ARGUS_DEV f32x4 mfma(u32x4 x, u32x4 y, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  }
  static ARGUS_DEV uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, bf16x2));
  }
  static ARGUS_DEV f32x2 unpack(uint32_t w) {
    return (f32x2){__builtin_bit_cast(float, w << 16), __builtin_bit_cast(float, w & 0xFFFF0000u)};
  }
  // Two weights as the sum of two numbers each, none of them above the weight
  // and none 0 beside a weight that is not: times an infinite value, a
  // negative or zero rest would make a NaN of infinity.  (It does where a weight is
  // below what its type has: 2^-126 of the largest, in fp16 2^-31.)
  static ARGUS_DEV void split(float x, float y, uint32_t* hi, uint32_t* lo) {
    const uint32_t a = __builtin_bit_cast(uint32_t, x) | 1u, b = __builtin_bit_cast(uint32_t, y) | 1u;
    *hi = __builtin_amdgcn_perm(b, a, 0x07060302u);
    *lo = pack(__builtin_bit_cast(float, a) - __builtin_bit_cast(float, a & 0xFFFF0000u),
               __builtin_bit_cast(float, b) - __builtin_bit_cast(float, b & 0xFFFF0000u));
  }
  static constexpr float kRaise = 0.0f;
};
template <>
struct Half<1> {
  static ARGUS_DEV f32x4 mfma(u32x4 x, u32x4 y, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
  }
  static ARGUS_DEV uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, f16x2));
  }
  static ARGUS_DEV f32x2 unpack(uint32_t w) {
    return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2);
  }
  static ARGUS_DEV void split(float x, float y, uint32_t* hi, uint32_t* lo) {
    *hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x, y));  // towards zero
    const f32x2 h = unpack(*hi);
    *lo = pack(fmaxf(x - h.x, fminf(x, 0x1p-24f)), fmaxf(y - h.y, fminf(y, 0x1p-24f)));
  }
  // weights are taken times 2^7, so that those of 2^-20 still are normal
  // numbers; they stay below 2^(7 + 8)
  static constexpr float kRaise = 7.0f;
};

// Two bytes of e4m3 (every such number is one of bf16 and of fp16).
template <int T>
ARGUS_DEV uint32_t widen(uint32_t w, bool hi) {
  if constexpr (T == 0)
    return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)
                                           : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
  else
    return __builtin_bit_cast(uint32_t, hi ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true)
                                           : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
}

// How far a score may rise above the running maximum before the maximum moves:
// weights stay below 2^8, and the sums need no rescaling at most steps.
constexpr float kSlack = 5.5f;
// A weight is 2^(x kd2 - base), one multiply-add and the exponential.  The base, the
// maximum to base 2, is rounded: all weights of one maximum are off alike, but not
// those of another, before it moved or in another wave.  Up to kFar that is 2^-14.5 of
// a weight.  Beyond it (at 2^15 it would be 2^-10, at 2^19 2^-6), and where a scale is so odd that the
// product overflows, the difference of the scores comes first, and that to base 2.
constexpr float kFar = 1024.0f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
ARGUS_DEV float exp_of(float x) { return exp2f(x * kLog2e); }

// Whether the rows of the next tile are loaded while one is taken: where a tile is small
// and the registers hold two (8 bits, head size 128: 65 us against 73 for 48
// sequences of up to 32768 tokens; two column tiles of it 60 against 41 for 20 of up to 20000, 4
// x 24 heads; 16 bits 867 against 638 for four of 262143, 8 bits at head size 256 184
// against 170 for 8 of 30000).
template <bool F8, int DP, int NQ>
constexpr bool kAhead = DP == 64 || (F8 && DP == 128 && NQ == 1);

// One wave's part of a segment: O, maxima and sums of tiles t0, t0 + dt, ... < t1
// for the 16 NQ query rows from q0 on.  T: type of q, out and the products; F8:
// the cache holds e4m3; DP: head size rounded up to 64, 128 or 256; NQ: 16-wide
// column tiles; EXACT: head size = DP.
template <int T, bool F8, int DP, int NQ, bool EXACT>
ARGUS_DEV void attend_tiles(const AttendArgs& a, const Span& p, uint32_t s, uint32_t h, uint32_t q0, uint32_t rows,
                            uint32_t t0, uint32_t t1, uint32_t dt, f32x4 (&acc)[NQ][DP / 16], float (&m)[NQ],
                            float (&l)[NQ]) {
  constexpr int ES = F8 ? 1 : 2;             // bytes of an element of the cache
  constexpr int KF = DP / 32;                // fragments of a key row
  constexpr int CB = F8 && DP == 64 ? 8 : 16;  // bytes of a key row that a lane loads at a time
  constexpr int CE = CB / ES;                // elements
  constexpr int CW = CB / 4;                 // words
  constexpr int KL = DP * ES / (8 * CB);     // loads of a key row by the 8 lanes that share it
  constexpr int VW = DP / 16;                // elements of a value row per lane
  constexpr int VD = VW * ES / 4;            // in 32-bit words
  constexpr int VH = VW / 2;                 // 16-bit pairs per lane
  constexpr bool AHEAD = kAhead<F8, DP, NQ>;
  using Hf = Half<T>;
  const uint32_t lane = threadIdx.x & 63u, c = lane & 15u, g = lane >> 4;
  const float kc = a.scale * (a.k_scale ? a.k_scale[h] : 1.0f), kd = fabsf(kc);
  // the query rows as operands: lane (q, g) holds 8 elements of its row per fragment
  u32x4 qf[NQ][KF];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const uint32_t row = 16 * i + c;
    const uint16_t* qr = a.q + (int64_t)s * a.q_seq + (int64_t)(h * a.G + q0 + (row < rows ? row : 0)) * a.q_head;
#pragma unroll
    for (int f = 0; f < KF; ++f) {
      // fragment (n, h, e) holds, of load n, elements 8 e ... of the lane's chunk 2 g + h
      const uint32_t e = f % (CE / 8), hn = f / (CE / 8), d = (hn / 2 * 8 + 2 * g + hn % 2) * CE + 8 * e;
      qf[i][f] = row < rows && d < a.D ? *reinterpret_cast<const u32x4*>(qr + d) : (u32x4)(0u);
      if (kc < 0.0f) qf[i][f] ^= 0x80008000u;  // so that the largest product is the largest score
    }
  }
  const int32_t* tab = a.table + (int64_t)s * a.table_stride;
  const uint8_t* kb = a.k + (int64_t)h * a.k_head;
  const uint8_t* vb = a.v + (int64_t)h * a.v_head;
  const uint32_t in_page = (1u << a.shift) - 1;

#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.0f;
#pragma unroll
    for (int f = 0; f < VW; ++f) acc[i][f] = (f32x4)(0.0f);
  }

  float base[NQ];  // the maximum to base 2, less kRaise
#pragma unroll
  for (int i = 0; i < NQ; ++i) base[i] = 0.0f;
  const float kd2 = kd * kLog2e;
  bool far = !(kd > 1e-30f && kd < 1e30f);  // scores so large, or a scale so odd, that the differences come first

  // What a lane adds to the scalar base of a load: of the keys, token w of eight and
  // chunk 2 g + part of its row; of the values, token 2 g and its elements.
  const uint32_t part = c >> 1 & 1u, w8 = 2 * (c >> 2) + (c & 1u);
  uint32_t k_at[EXACT ? 1 : KL], v_at;
#pragma unroll
  for (int n = 0; n < (EXACT ? 1 : KL); ++n) {
    const uint32_t b = (8 * n + 2 * g + part) * CB;
    k_at[n] = w8 * a.k_tok + (EXACT || b < a.D * ES ? b : a.D * ES - CB);
  }
  v_at = c * (VD * 4);
  if (!EXACT && v_at >= a.D * ES) v_at = 0;  // rows of O beyond the head size: not written
  v_at += 2 * g * a.v_tok;

  // The pages of tile t's four runs of eight tokens (scalar loads).
  struct Ids {
    int32_t p[4];
  };
  typedef const __attribute__((address_space(4))) int32_t* scalar_ptr;
  const scalar_ptr tab_s = (scalar_ptr)(uintptr_t)tab;
  auto token_of = [&](uint32_t t) { return (t < p.sink_tiles ? t : t - p.sink_tiles + p.first) * kTile; };
  auto find = [&](uint32_t t, Ids& ids) {
    const uint32_t tok = token_of(t < t1 ? t : t1 - 1);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t col = (tok + 8 * j) >> a.shift;
      const int32_t page = tab_s[col < a.columns ? col : 0];
      ids.p[j] = col < a.columns && (uint32_t)page < a.num_pages ? page : -1;
    }
  };
  // Its rows, and which of the lane's eight tokens are visible.  (A page that is not
  // held: any row, what comes of it is not taken.)
  struct Rows {
    uint32_t k[2][2][KL][CW];
    uint32_t v[8][VD];
    uint32_t vis;
  };
  auto load = [&](uint32_t t, const Ids& ids, Rows& w) {
    const uint32_t tok = token_of(t);
    // All of it is read once, whole lines at a time: past the caches.
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t page = ids.p[j] < 0 ? 0 : ids.p[j];
      const uint8_t* base = kb + page * a.k_page + (uint64_t)((tok + 8 * j) & in_page) * a.k_tok;
#pragma unroll
      for (int n = 0; n < KL; ++n) {
        const uint8_t* r = base + k_at[EXACT ? 0 : n] + (EXACT ? n * 8 * CB : 0);
        uint32_t(&to)[CW] = w.k[j / 2][j % 2][n];
        if constexpr (CW == 2) {
          const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(r));
          to[0] = x.x, to[1] = x.y;
        } else {
          const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(r));
          to[0] = x.x, to[1] = x.y, to[2] = x.z, to[3] = x.w;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {  // half i / 4, r = i % 4
      const int j = i / 2;           // run of eight tokens
      const int64_t page = ids.p[j] < 0 ? 0 : ids.p[j];
      const uint8_t* r = vb + page * a.v_page + (uint64_t)(((tok + 8 * j) & in_page) + i % 2) * a.v_tok + v_at;
      if constexpr (VD == 1) {
        w.v[i][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(r));
      } else if constexpr (VD == 2) {
        const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(r));
        w.v[i][0] = x.x, w.v[i][1] = x.y;
      } else {
#pragma unroll
        for (int j4 = 0; j4 < VD / 4; ++j4) {
          const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(r + 16 * j4));
          w.v[i][4 * j4] = x.x, w.v[i][4 * j4 + 1] = x.y, w.v[i][4 * j4 + 2] = x.z, w.v[i][4 * j4 + 3] = x.w;
        }
      }
    }
    // which of the lane's eight tokens are visible
    w.vis = 0xFFu;
    if (tok < p.lo || tok + kTile > p.len || (ids.p[0] | ids.p[1] | ids.p[2] | ids.p[3]) < 0) {
      w.vis = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t at = tok + 8 * (i / 2) + 2 * g + i % 2;
        const bool in = at < p.len && (at >= p.lo || at < p.sinks) && ids.p[i / 2] >= 0;
        w.vis |= in ? 1u << i : 0u;
      }
    }
  };
  auto take = [&](Rows& w) {
    const bool whole = __all(w.vis == 0xFFu);
    if (!whole) {  // what is not visible may hold anything
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < VD; ++j) w.v[i][j] = w.vis >> i & 1u ? w.v[i][j] : 0u;
    }

    // scores
    f32x4 sc[NQ][2];
#pragma unroll
    for (int i = 0; i < NQ; ++i) sc[i][0] = sc[i][1] = (f32x4)(0.0f);
#pragma unroll
    for (int hn = 0; hn < 2 * KL; ++hn) {  // load n = hn / 2, chunk 2 g + hn % 2
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        // of the first eight tokens for the lanes of part 0, of the others for those of part 1
        uint32_t x[CW];
#pragma unroll
        for (int i = 0; i < CW; ++i) {
          const uint32_t lo = w.k[hh][0][hn / 2][i], hi = w.k[hh][1][hn / 2][i];
          // (moved before it is chosen: under a condition the lanes read would be off)
          const uint32_t moved = dpp32<kDppQuad2301>(hn % 2 == 0 ? hi : lo);
          x[i] = hn % 2 == 0 ? (part ? moved : lo) : (part ? hi : moved);
          if (!EXACT && (hn / 2 * 8 + 2 * g + hn % 2) * CE >= a.D) x[i] = 0;  // (what stood there may be NaN)
        }
#pragma unroll
        for (int e = 0; e < CE / 8; ++e) {
          u32x4 kf;
          if constexpr (F8) {
            kf = (u32x4){widen<T>(x[2 * e], false), widen<T>(x[2 * e], true), widen<T>(x[2 * e + 1], false),
                         widen<T>(x[2 * e + 1], true)};
          } else {
            kf = (u32x4){x[0], x[1], x[2], x[3]};
          }
#pragma unroll
          for (int i = 0; i < NQ; ++i) sc[i][hh] = Hf::mfma(kf, qf[i][hn * (CE / 8) + e], sc[i][hh]);
        }
      }
    }

    // weights
    u32x4 p_hi[NQ], p_lo[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = sc[i][j / 4][j % 4];
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = w.vis >> j & 1u ? x[j] : -INFINITY;
      }
      float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      top = top == -INFINITY ? top : top * kd;  // (kd may be 0)
      if (__any(top > m[i] + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m[i], top);
        const float scale = m[i] == -INFINITY ? 0.0f : exp_of(m[i] - mn);
        l[i] *= scale;
#pragma unroll
        for (int f = 0; f < VW; ++f) acc[i][f] *= scale;
        m[i] = mn;
        base[i] = mn == -INFINITY ? 0.0f : fmaf(mn, kLog2e, -Hf::kRaise);
        far = far || __any(fabsf(mn) > kFar && mn != -INFINITY);
      }
      float wt[8], sum = 0.0f;
      if (!far) {
#pragma unroll
        for (int j = 0; j < 8; ++j) wt[j] = __builtin_amdgcn_exp2f(fmaf(x[j], kd2, -base[i]));
      } else {
        const float ms = m[i] == -INFINITY ? 0.0f : m[i];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float y = x[j] == -INFINITY ? x[j] : x[j] * kd;
          wt[j] = __builtin_amdgcn_exp2f(fmaf(y - ms, kLog2e, Hf::kRaise));
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += wt[j];
      l[i] += sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t hi, lo;
        Hf::split(wt[2 * j], wt[2 * j + 1], &hi, &lo);
        p_hi[i][j] = hi;
        p_lo[i][j] = lo;
      }
    }

    // values
#pragma unroll
    for (int f = 0; f < VH; ++f) {  // elements 2 f and 2 f + 1 of the lane's piece of a row
      u32x4 even, odd;
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // tokens 2 j and 2 j + 1
        uint32_t x, y;
        if constexpr (F8) {
          x = widen<T>(w.v[2 * j][f / 2], f % 2), y = widen<T>(w.v[2 * j + 1][f / 2], f % 2);
        } else {
          x = w.v[2 * j][f], y = w.v[2 * j + 1][f];
        }
        even[j] = __builtin_amdgcn_perm(y, x, 0x05040100u);
        odd[j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
      }
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        acc[i][2 * f] = Hf::mfma(even, p_hi[i], acc[i][2 * f]);
        acc[i][2 * f + 1] = Hf::mfma(odd, p_hi[i], acc[i][2 * f + 1]);
        acc[i][2 * f] = Hf::mfma(even, p_lo[i], acc[i][2 * f]);
        acc[i][2 * f + 1] = Hf::mfma(odd, p_lo[i], acc[i][2 * f + 1]);
      }
    }
  };

  if (t0 < t1) {
    uint32_t t = t0;
    Ids i0, i1;
    Rows w0;
    find(t, i0);
    if constexpr (AHEAD) {
      // The next tile's rows, and the pages of the one after it, are under way while a
      // tile is taken.  (No load stands in a branch that is left again: one that may
      // or may not have been made would be waited for at once.)
      Rows w1;
      find(t + dt, i1);
      load(t, i0, w0);
      for (;;) {
        if (t + dt >= t1) {
          take(w0);
          break;
        }
        t += dt;
        find(t + dt, i0);
        load(t, i1, w1);
        take(w0);
        if (t + dt >= t1) {
          take(w1);
          break;
        }
        t += dt;
        find(t + dt, i1);
        load(t, i0, w0);
        take(w1);
      }
    } else {
      for (; t < t1; t += dt) {
        load(t, i0, w0);
        find(t + dt, i0);
        take(w0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    l[i] += __shfl_xor(l[i], 16);
    l[i] += __shfl_xor(l[i], 32);
  }
}

// A segment per block, the tiles dealt out to its waves.
template <int T, bool F8, int DP, int NQ, bool EXACT>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void k_attend_whole(AttendArgs a) {
  constexpr int VW = DP / 16, QP = DP + 4;  // QP: pitch of a row of O in LDS
  using Hf = Half<T>;
  __shared__ float s_ml[kWaves][16 * NQ][2];
  __shared__ __align__(16) float s_o[kWaves][16 * NQ][QP];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_ATTEND);
  mk.begin(ARGUS_REGION_ATTEND_PLACE);
  const uint32_t tid = threadIdx.x, c = tid & 15u, g = (tid & 63u) >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t s = blockIdx.x / a.HS, hs = blockIdx.x % a.HS;
  const uint32_t h = hs / a.row_tiles, q0 = (hs % a.row_tiles) * 16 * NQ;
  const uint32_t rows = a.G - q0 < 16u * NQ ? a.G - q0 : 16u * NQ;
  const Span p = span_of(a, a.lens[s]);
  mk.end(ARGUS_REGION_ATTEND_PLACE);
  mk.begin(ARGUS_REGION_ATTEND_TOKENS);
  f32x4 acc[NQ][VW];
  float m[NQ], l[NQ];
  attend_tiles<T, F8, DP, NQ, EXACT>(a, p, s, h, q0, rows, wave, p.tiles, kWaves, acc, m, l);
  // Lane (q, g) holds of its column the elements d = (4 g + r) VW + f.
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const uint32_t row = 16 * i + c;
    if (g == 0) {
      s_ml[wave][row][0] = m[i];
      s_ml[wave][row][1] = l[i];
    }
    if (row < rows) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int f = 0; f < VW; f += 4)
          *reinterpret_cast<f32x4*>(&s_o[wave][row][(4 * g + r) * VW + f]) =
              (f32x4){acc[i][f][r], acc[i][f + 1][r], acc[i][f + 2][r], acc[i][f + 3][r]};
    }
  }
  __syncthreads();
  const uint64_t seg_row = (uint64_t)s * a.H * a.G + (uint64_t)h * a.G + q0;
  const float vs = a.v_scale ? a.v_scale[h] : 1.0f;
  const uint32_t quads = a.D / 4;
  for (uint32_t e = tid; e < rows * quads; e += kThreads) {
    const uint32_t row = e / quads, d = (e % quads) * 4;
    float mw[kWaves], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      mw[w] = s_ml[w][row][0];
      top = fmaxf(top, mw[w]);
    }
    f32x4 o = (f32x4)(0.0f);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float x = mw[w] == -INFINITY ? (s_ml[w][row][1] != 0.0f ? 1.0f : 0.0f) : exp_of(mw[w] - top);
      sum += s_ml[w][row][1] * x;
      o += *reinterpret_cast<const f32x4*>(&s_o[w][row][d]) * x;
    }
    const float inv = sum == 0.0f ? 0.0f : vs / sum;
    *reinterpret_cast<u32x2*>(a.out + (seg_row + row) * a.D + d) = (u32x2){Hf::pack(o.x * inv, o.y * inv), Hf::pack(o.z * inv, o.w * inv)};
    if (d == 0 && a.lse)
      a.lse[seg_row + row] = sum == 0.0f ? -INFINITY : (top == -INFINITY ? 0.0f : top - Hf::kRaise * kLn2) + logf(sum);
  }
  mk.end(ARGUS_REGION_ATTEND_TOKENS);
  mk.end(ARGUS_REGION_ATTEND);
}

// The batch shared among the grid's waves.
template <int T, bool F8, int DP, int NQ, bool EXACT>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void k_attend_shared(AttendArgs a) {
  constexpr int VW = DP / 16;
  using Hf = Half<T>;
  __shared__ uint32_t s_base[kThreads];
  __shared__ uint32_t s_wave[kWaves];
  __shared__ int32_t s_len[kThreads];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_ATTEND);
  mk.begin(ARGUS_REGION_ATTEND_PLACE);
  const uint32_t tid = threadIdx.x, lane = tid & 63u, c = lane & 15u, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t ones = (1u << a.unit_shift) - 1;
  auto units_of = [&](const Span& p) { return (p.tiles + kPieceCost + ones) >> a.unit_shift; };
  // A thread looks after `run` sequences in a row.
  const uint32_t run = (a.S + kThreads - 1) / kThreads;
  uint32_t mine = 0;
  for (uint32_t i = 0; i < run; ++i) {
    const uint32_t x = tid * run + i;
    if (x < a.S) {
      const int32_t len = a.lens[x];
      s_len[tid] = len;
      mine += units_of(span_of(a, len));
    }
  }
  const uint32_t incl = (uint32_t)wave_incl_scan32((int32_t)mine);
  if (lane == 63) s_wave[wave] = incl;
  __syncthreads();
  uint32_t before = 0, total = 0;
#pragma unroll
  for (uint32_t w = 0; w < (uint32_t)kWaves; ++w) {
    before += w < wave ? s_wave[w] : 0u;
    total += s_wave[w];
  }
  s_base[tid] = (before + incl - mine) * a.HS;
  total *= a.HS;
  __syncthreads();
  // this wave's units [u, end), and the sequence that they start in
  const uint32_t share = blockIdx.x * kWaves + wave;
  uint32_t per = (total + a.shares - 1) / a.shares;
  per = per < kMinShare ? kMinShare : per;
  uint32_t u = share < total / per + 1 ? share * per : total, end = total - u < per ? total : u + per, off = 0, s = 0;
  if (u < end) {
    uint32_t n = 0;  // threads whose sequences start at or before u
#pragma unroll
    for (uint32_t i = 0; i < (uint32_t)kThreads / 64; ++i) n += (uint32_t)__popcll(__ballot(s_base[64 * i + lane] <= u));
    s = (n - 1) * run;
    off = u - s_base[n - 1];
    while (run > 1) {
      const uint32_t w = units_of(span_of(a, a.lens[s])) * a.HS;
      if (off < w) break;
      off -= w;
      ++s;
    }
  }
  s = __builtin_amdgcn_readfirstlane(s);
  off = __builtin_amdgcn_readfirstlane(off);
  u = __builtin_amdgcn_readfirstlane(u), end = __builtin_amdgcn_readfirstlane(end), per = __builtin_amdgcn_readfirstlane(per);
  mk.end(ARGUS_REGION_ATTEND_PLACE);
  mk.begin(ARGUS_REGION_ATTEND_TOKENS);

  bool open = false;  // a segment starts here and does not end
  while (u < end) {
    const Span p = span_of(a, __builtin_amdgcn_readfirstlane(run == 1 ? s_len[s] : a.lens[s]));
    const uint32_t units = units_of(p);
    const uint32_t hs = off / units, o0 = off - hs * units;
    const uint32_t n = end - u < units - o0 ? end - u : units - o0;
    // its cost comes before its tiles
    const uint32_t a0 = o0 << a.unit_shift, a1 = (o0 + n) << a.unit_shift;
    const uint32_t t0 = a0 < kPieceCost ? 0 : a0 - kPieceCost;
    uint32_t t1 = a1 < kPieceCost ? 0 : a1 - kPieceCost;
    t1 = t1 < p.tiles ? t1 : p.tiles;
    if (t0 < t1) {
      const uint32_t h = hs / a.row_tiles, q0 = (hs % a.row_tiles) * 16 * NQ;
      const uint32_t rows = a.G - q0 < 16u * NQ ? a.G - q0 : 16u * NQ;
      f32x4 acc[NQ][VW];
      float m[NQ], l[NQ];
      attend_tiles<T, F8, DP, NQ, EXACT>(a, p, s, h, q0, rows, t0, t1, 1, acc, m, l);
      const bool done = t0 == 0 && t1 == p.tiles;
      const uint32_t seg = s * a.HS + hs;
      if (t0 == 0) {
        const uint32_t last = (u - o0 + units - 1) / per;
        if (lane == 0 && (a.by_seg || !done))
          a.open[a.by_seg ? seg : share] = make_uint4(seg, done ? 1u : share, done ? 0u : last, 0u);
        open = !done;
      }
      const uint64_t seg_row = (uint64_t)s * a.H * a.G + (uint64_t)h * a.G + q0;
      const uint64_t slot = 2ull * share + (t0 == 0 ? 1u : 0u);
      const float vs = a.v_scale ? a.v_scale[h] : 1.0f;
      // Lane (q, g) holds of its column the elements d = (4 g + r) VW + f.
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const uint32_t row = 16 * i + c;
        if (row < rows) {
          const float inv = l[i] == 0.0f ? 0.0f : vs / l[i];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int f = 0; f < VW; f += 4) {
              const uint32_t d = (4 * g + r) * VW + f;
              const f32x4 o = (f32x4){acc[i][f][r], acc[i][f + 1][r], acc[i][f + 2][r], acc[i][f + 3][r]};
              if (!done)
                *reinterpret_cast<f32x4*>(a.part_o + (slot * 16 * NQ + row) * DP + d) = o;
              else if (EXACT || d < a.D)
                *reinterpret_cast<u32x2*>(a.out + (seg_row + row) * a.D + d) =
                    (u32x2){Hf::pack(o.x * inv, o.y * inv), Hf::pack(o.z * inv, o.w * inv)};
            }
          }
          if (g == 0) {
            if (!done)
              *reinterpret_cast<f32x2*>(a.part_ml + (slot * 16 * NQ + row) * 2) = (f32x2){m[i], l[i]};
            else if (a.lse)
              a.lse[seg_row + row] = l[i] == 0.0f ? -INFINITY : (m[i] == -INFINITY ? 0.0f : m[i] - Hf::kRaise * kLn2) + logf(l[i]);
          }
        }
      }
    }
    u += n;
    off += n;
    if (off == units * a.HS) {
      off = 0;
      ++s;
    }
  }
  if (!a.by_seg && !open && lane == 0) a.open[share] = make_uint4(0u, 1u, 0u, 0u);
  mk.end(ARGUS_REGION_ATTEND_TOKENS);
  mk.end(ARGUS_REGION_ATTEND);
}

// ROWS rows by COLS elements of a segment that was left in pieces: piece 0 is the second
// of its first share, piece i the first of share i further on.
template <int T, int DP, int NQ, int ROWS, int COLS>
__global__ __launch_bounds__(kThreads) void k_attend_join(AttendArgs a) {
  constexpr uint32_t kRows = ROWS, kQuads = COLS / 4, kParts = kThreads / (kQuads * kRows);
  using Hf = Half<T>;
  static_assert(ROWS == 1 || ROWS == kWaves, "a row for the block, or one for each wave");
  __shared__ float s_m[kWaves], s_l[kWaves];
  __shared__ __align__(16) float s_o[kWaves][COLS];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_ATTEND_JOIN);
  const uint4 open = a.open[blockIdx.x];
  if (open.y <= open.z) {
    const uint32_t s = open.x / a.HS, hs = open.x % a.HS, n = open.z - open.y + 1;
    const uint32_t h = hs / a.row_tiles, q0 = (hs % a.row_tiles) * 16 * NQ;
    const uint32_t rows = a.G - q0 < 16u * NQ ? a.G - q0 : 16u * NQ;
    const uint32_t tid = threadIdx.x, r4 = tid / (kQuads * kParts), part = tid / kQuads % kParts, q4 = (tid % kQuads) * 4;
    const uint32_t d = blockIdx.z * COLS + q4;
    const uint32_t row = blockIdx.y * kRows + r4, at = row < rows ? row : 0;
    float m = -INFINITY, l = 0.0f;
    f32x4 o = (f32x4)(0.0f);
    constexpr uint32_t kDeep = 8;
    for (uint32_t i0 = part; i0 < n; i0 += kParts * kDeep) {
      f32x2 ml[kDeep];
      f32x4 v[kDeep];
      float top = m;
#pragma unroll
      for (uint32_t j = 0; j < kDeep; ++j) {
        const uint32_t i = i0 + j * kParts;
        const uint64_t x = (2ull * (open.y + (i < n ? i : 0)) + (i == 0 || i >= n ? 1u : 0u)) * 16 * NQ + at;
        ml[j] = *reinterpret_cast<const f32x2*>(a.part_ml + 2 * x);
        v[j] = *reinterpret_cast<const f32x4*>(a.part_o + x * DP + d);
        if (i >= n) ml[j] = (f32x2){-INFINITY, 0.0f}, v[j] = (f32x4)(0.0f);
        top = fmaxf(top, ml[j].x);
      }
      const float keep = m == -INFINITY ? 1.0f : exp_of(m - top);  // (nothing yet, or NaN)
      l *= keep;
      o *= keep;
#pragma unroll
      for (uint32_t j = 0; j < kDeep; ++j) {
        const float w = ml[j].x == -INFINITY ? 1.0f : exp_of(ml[j].x - top);  // a maximum of -inf: zeros, or NaN
        l += ml[j].y * w;
        o += v[j] * w;
      }
      m = top;
    }
    // the parts of a wave, then the waves
#pragma unroll
    for (uint32_t x = kQuads; x < 64; x <<= 1) {
      const float m2 = __shfl_xor(m, x), l2 = __shfl_xor(l, x), top = fmaxf(m, m2);
      const float w = m == -INFINITY ? 1.0f : exp_of(m - top), w2 = m2 == -INFINITY ? 1.0f : exp_of(m2 - top);
      l = l * w + l2 * w2;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = o[j] * w + __shfl_xor(o[j], x) * w2;
      m = top;
    }
    float top = m, sum = l;
    if constexpr (ROWS == 1) {
      if ((tid & 63u) < kQuads) {
        if (q4 == 0) s_m[tid >> 6] = m, s_l[tid >> 6] = l;
        *reinterpret_cast<f32x4*>(&s_o[tid >> 6][q4]) = o;
      }
      __syncthreads();
      top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
      sum = 0.0f;
      o = (f32x4)(0.0f);
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float w = s_m[i] == -INFINITY ? 1.0f : exp_of(s_m[i] - top);
        sum += s_l[i] * w;
        o += *reinterpret_cast<const f32x4*>(&s_o[i][q4]) * w;
      }
    }
    if (part == 0 && row < rows && d < a.D) {
      const uint64_t out = (uint64_t)s * a.H * a.G + (uint64_t)h * a.G + q0 + row;
      const float inv = sum == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[h] : 1.0f) / sum;
      *reinterpret_cast<u32x2*>(a.out + out * a.D + d) = (u32x2){Hf::pack(o.x * inv, o.y * inv), Hf::pack(o.z * inv, o.w * inv)};
      if (d == 0 && a.lse)
        a.lse[out] = sum == 0.0f ? -INFINITY : (top == -INFINITY ? 0.0f : top - Hf::kRaise * kLn2) + logf(sum);
    }
  }
  mk.end(ARGUS_REGION_ATTEND_JOIN);
}

template <int T, bool F8, int DP, int NQ>
void launch_attend_as(const AttendArgs& a, uint32_t grid, hipStream_t st) {
  const dim3 g(grid), b(kThreads);
  if (a.shares) {
    if (a.D == DP) hipLaunchKernelGGL((k_attend_shared<T, F8, DP, NQ, true>), g, b, 0, st, a);
    else hipLaunchKernelGGL((k_attend_shared<T, F8, DP, NQ, false>), g, b, 0, st, a);
  } else {
    if (a.D == DP) hipLaunchKernelGGL((k_attend_whole<T, F8, DP, NQ, true>), g, b, 0, st, a);
    else hipLaunchKernelGGL((k_attend_whole<T, F8, DP, NQ, false>), g, b, 0, st, a);
  }
}

// The head size rounded up, and as many column tiles as the group needs: two
// read the cache once for up to 32 query heads; a group beyond 32 reads it again.
template <int T, bool F8>
void launch_attend_type(const AttendArgs& a, uint32_t grid, hipStream_t st) {
  if (a.D <= 64)
    a.G <= 16 ? launch_attend_as<T, F8, 64, 1>(a, grid, st) : launch_attend_as<T, F8, 64, 2>(a, grid, st);
  else if (a.D <= 128)
    a.G <= 16 ? launch_attend_as<T, F8, 128, 1>(a, grid, st) : launch_attend_as<T, F8, 128, 2>(a, grid, st);
  else
    a.G <= 16 ? launch_attend_as<T, F8, 256, 1>(a, grid, st) : launch_attend_as<T, F8, 256, 2>(a, grid, st);
}

// What a block joins: four rows, one row, or 32 elements of one, for up to 2, 8 and 32 pieces
// side by side at head size 128.
enum JoinForm : uint32_t { kJoinFourRows, kJoinRow, kJoinPart };
constexpr int kJoinCols = 32;

template <int T, int DP, int NQ>
void launch_join_as(const AttendArgs& a, JoinForm form, dim3 g, hipStream_t st) {
  const dim3 b(kThreads);
  if (form == kJoinPart) hipLaunchKernelGGL((k_attend_join<T, DP, NQ, 1, kJoinCols>), g, b, 0, st, a);
  else if (form == kJoinRow) hipLaunchKernelGGL((k_attend_join<T, DP, NQ, 1, DP>), g, b, 0, st, a);
  else hipLaunchKernelGGL((k_attend_join<T, DP, NQ, 4, DP>), g, b, 0, st, a);
}

template <int T>
void launch_join_type(const AttendArgs& a, JoinForm form, dim3 g, hipStream_t st) {
  if (a.D <= 64)
    a.G <= 16 ? launch_join_as<T, 64, 1>(a, form, g, st) : launch_join_as<T, 64, 2>(a, form, g, st);
  else if (a.D <= 128)
    a.G <= 16 ? launch_join_as<T, 128, 1>(a, form, g, st) : launch_join_as<T, 128, 2>(a, form, g, st);
  else
    a.G <= 16 ? launch_join_as<T, 256, 1>(a, form, g, st) : launch_join_as<T, 256, 2>(a, form, g, st);
}

// One source file each, so that they compile side by side.
void launch_attend_bf16(const AttendArgs& a, uint32_t grid, hipStream_t st);
void launch_attend_fp16(const AttendArgs& a, uint32_t grid, hipStream_t st);
void launch_attend_bf16_f8(const AttendArgs& a, uint32_t grid, hipStream_t st);
void launch_attend_fp16_f8(const AttendArgs& a, uint32_t grid, hipStream_t st);

}  // namespace decode
}  // namespace argus
