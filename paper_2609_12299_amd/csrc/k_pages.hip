// k_pages.hip -- the paged cache of a decode step: new tokens written into their
// pages, page tables moved from one step to the next, pools compacted.
#include "decode.h"

#include "chain.h"

namespace argus {
namespace decode {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- append

struct AppendArgs {
  const uint8_t *new_k, *new_v;  // strides in bytes
  int64_t k_row, k_hd, v_row, v_hd;
  uint8_t *k, *v;
  int64_t k_page, k_head, k_tok, v_page, v_head, v_tok;
  const int32_t* table;
  int64_t table_stride;
  const int32_t *starts, *offsets;
  const float *k_scale, *v_scale;
  uint32_t S, rows, shift, num_pages, columns, tokens;  // tokens of a block
  FastDiv per_token, per_side, per_head;                // chunks of a token, of its keys, of a head
  Marks marks;
};

constexpr uint32_t kMaxTokens = 16;

// x / s rounded to nearest, limited to the range of e4m3.  y = 1 / s correctly
// rounded; then fma(x - q s, y, q) with q = x y is the correctly rounded
// quotient (Markstein), save where q overflows, which the limit settles.
ARGUS_DEV float quotient(float x, float s, float y) {
  const float q = x * y;
  float r = fmaf(fmaf(-q, s, x), y, q);
  r = fabsf(q) > 1000.0f ? q : r;  // beyond the range; infinities have no remainder
  r = r > 448.0f ? 448.0f : r;     // NaN stays
  return r < -448.0f ? -448.0f : r;
}

// Scales that quotient() takes.  Outside (0, infinities and NaN among them) the reciprocal, or the
// remainder of a quotient that is not rounded to zero, would leave the normal numbers of 32 bits.
ARGUS_DEV bool ordinary(float s) { return fabsf(s) >= 0x1p-80f && fabsf(s) <= 0x1p80f; }

template <int T>  // 0: bf16, 1: fp16
ARGUS_DEV f32x2 pair(uint32_t w) {
  if constexpr (T == 0) {
    return (f32x2){__builtin_bit_cast(float, w << 16), __builtin_bit_cast(float, w & 0xFFFF0000u)};
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2);
  }
}

// A chunk is 16 bytes of the cache: 8 elements copied, or 16 in 8 bits.  A block
// finds the places of its tokens once, then its threads go over their chunks,
// which lie one after the other in the input; past the caches (79374
// tokens of 8 heads of 128 into 8 bits: 94.4 us against 96.6).  What bounds it: memory,
// 488 MB read and written at 5.2 TB/s (a copy of 2 GiB runs at 4.9); a token for each of
// 64 sequences takes 2.9 us, and the call 7 us of the host.
// MODE 0: copy; 1: bf16 to e4m3; 2: fp16 to e4m3.
template <int MODE>
__global__ __launch_bounds__(kThreads) void k_append(AppendArgs a) {
  __shared__ int64_t s_page[kMaxTokens];   // -1: left out
  __shared__ uint32_t s_place[kMaxTokens];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_APPEND);
  const uint32_t tid = threadIdx.x;
  const uint32_t row0 = blockIdx.x * a.tokens;
  const uint32_t tokens = a.rows - row0 < a.tokens ? a.rows - row0 : a.tokens;
  if (tid < tokens) {
    const int32_t row = (int32_t)(row0 + tid);
    uint32_t s = row0 + tid;
    int64_t pos;
    bool in = true;
    if (a.offsets) {
      uint32_t lo = 0, hi = a.S;  // the first sequence that ends behind the row
      while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (a.offsets[mid + 1] > row) hi = mid; else lo = mid + 1;
      }
      in = lo < a.S && a.offsets[0] <= row;
      s = in ? lo : 0;
      pos = in ? (int64_t)a.starts[s] + row - a.offsets[s] : -1;
    } else {
      pos = a.starts[s];
    }
    in = pos >= 0 && (uint64_t)pos >> a.shift < a.columns;
    const int32_t page = in ? a.table[(int64_t)s * a.table_stride + (pos >> a.shift)] : -1;
    s_page[tid] = (uint32_t)page < a.num_pages ? page : -1;
    s_place[tid] = (uint32_t)pos & ((1u << a.shift) - 1);
  }
  __syncthreads();
  const uint32_t n = tokens * a.per_token.d;
  for (uint32_t e = tid; e < n; e += kThreads) {
    const uint32_t t = divide(e, a.per_token);
    uint32_t x = e - t * a.per_token.d;
    const bool values = x >= a.per_side.d;
    if (values) x -= a.per_side.d;
    const uint32_t h = divide(x, a.per_head), at = (x - h * a.per_head.d) * 16;
    const int64_t page = s_page[t];
    if (page < 0) continue;
    const uint8_t* src = values ? a.new_v + (int64_t)(row0 + t) * a.v_row + (int64_t)h * a.v_hd
                                : a.new_k + (int64_t)(row0 + t) * a.k_row + (int64_t)h * a.k_hd;
    uint8_t* dst = values ? a.v + page * a.v_page + (int64_t)h * a.v_head + (int64_t)s_place[t] * a.v_tok
                          : a.k + page * a.k_page + (int64_t)h * a.k_head + (int64_t)s_place[t] * a.k_tok;
    u32x4 out;
    if constexpr (MODE == 0) {
      out = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + at));
    } else {
      const u32x4 lo = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + 2 * at));
      const u32x4 hi = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + 2 * at + 16));
      const float* scale = values ? a.v_scale : a.k_scale;
      float sc = scale ? scale[h] : 1.0f, inv = 1.0f / sc;
      f32x2 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = pair<MODE - 1>(i < 4 ? lo[i] : hi[i - 4]);
      if (!ordinary(sc)) {  // divided here, and by 1 below
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (f32x2){x[i].x / sc, x[i].y / sc};
        sc = inv = 1.0f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 p = x[2 * i], q = x[2 * i + 1];
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(p.x, sc, inv), quotient(p.y, sc, inv), 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(q.x, sc, inv), quotient(q.y, sc, inv), w, true);
        out[i] = (uint32_t)w;
      }
    }
    __builtin_nontemporal_store(out, reinterpret_cast<u32x4*>(dst + at));
  }
  mk.end(ARGUS_REGION_APPEND);
}

// ------------------------------------------------------------ page copies

struct Planes {
  uint8_t* base;
  int64_t plane_stride, page_stride;
  uint32_t planes, units;  // 16-byte units of a page
};
struct Caches {
  Planes c[ARGUS_MAX_CACHES];
  uint32_t n;
};

// Copies pages src(i) to dst(i), i < n, in every plane of every cache, by the
// waves first, first + step, ...: 4 KiB at a time, four loads in flight per lane,
// past the caches (a pool of 16384 pages, 1.07 GB read and written: 218 us against 228).
template <class Pair>
ARGUS_DEV void copy_pages(const Caches& all, uint32_t n, uint32_t first, uint32_t step, Pair pair_of) {
  const uint32_t lane = lane_id();
  for (uint32_t ci = 0; ci < all.n; ++ci) {
    const Planes c = all.c[ci];
    const uint32_t parts = (c.units + 255) / 256;
    const uint64_t total = (uint64_t)n * c.planes * parts;
    for (uint64_t w = first; w < total; w += step) {
      const uint32_t part = (uint32_t)(w % parts);
      const uint64_t r = w / parts;
      const uint32_t plane = (uint32_t)(r % c.planes), i = (uint32_t)(r / c.planes);
      uint32_t src, dst;
      if (!pair_of(i, &src, &dst)) continue;
      uint8_t* base = c.base + (int64_t)plane * c.plane_stride;
      const u32x4* from = reinterpret_cast<const u32x4*>(base + (int64_t)src * c.page_stride) + part * 256 + lane;
      u32x4* to = reinterpret_cast<u32x4*>(base + (int64_t)dst * c.page_stride) + part * 256 + lane;
      const uint32_t left = c.units - part * 256;
      u32x4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (lane + 64 * j < left) v[j] = __builtin_nontemporal_load(&from[64 * j]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (lane + 64 * j < left) __builtin_nontemporal_store(v[j], &to[64 * j]);
    }
  }
}

constexpr uint32_t kCopyBlocks = 2048;

// ------------------------------------------------------------------ step
//
// With e[s][c] the entry that new sequence s takes over (parent's, or -1) and held[p]:
//   refs[p] = held[p] + #{(s, c): e[s][c] = p}
//   s writes on in its last page p if it ends inside, held[p] = 0, all refs[p] sequences have p
//   last and inside, and (length, -s) is the largest of theirs; else it takes a copy
//   fresh page of rank r = the r-th p with refs[p] = 0; ranks by a prefix sum over s
// Counts and maxima are of whole numbers: the order of the atomics does not show.  What
// bounds it: dependent ways to memory (parent, length, entry, counts of its page), the
// launches, and for a batch the copies (512 sequences of 256 columns over 16384 pages, 39 MB:
// clear 2.7 us, claim 4.8, plan 6.1, place with its copies 11.9).

struct StepArgs {
  const int32_t* table;
  int64_t table_stride;
  const int32_t *lens, *parents, *grow, *held;
  int32_t *new_table, *new_lens, *refs, *counters;
  uint64_t* best;      // [pages] of the sequences that have the page last: (length + 1) << 32 | ~sequence
  uint32_t* lasts;     // [pages] how many they are
  int2* ends;          // [S] page that the sequence would write on (-1: none), pages that it grows by
  uint32_t* base;      // [S] fresh pages before the sequence's
  uint2* copies;       // [S] page, rank of the fresh page
  uint32_t* free_list; // [pages]
  uint64_t* words;     // look-back over the tiles of pages
  uint32_t* state;     // 0: ticket, 1: free pages, 2: needed pages, 3: copies
  uint32_t S0, S, P, N, shift, window, sinks;
  uint32_t row_lanes;  // claim, place: threads of a row (a power of two)
  uint32_t rows_blocks;
  Caches caches;
  Marks marks;
};

constexpr uint32_t kPageTile = 4096;
constexpr uint32_t kPageItems = 16;  // pages of a thread
static_assert(kPageItems * kThreads == kPageTile, "a tile per block");
// Calls of at most so many table entries and pages are planned by every block for
// itself, in LDS, in one launch: what a call costs is its launches (3.5 us of the
// host each) and the ways to memory one after the other.  Steps over 4096 pages,
// with keys and values of one layer: 4096 entries 15.1 us a call against 22.2 by four
// launches, 8192 18.9 against 21.8, 16384 28.3 against 22.0.  Compaction: 4096
// pages 15.5 us against 21.7 by three launches (4097); more do not fit 16 bits of a thread.
constexpr uint32_t kSmallEntries = 8192, kSmallRows = 2048, kSmallPages = 4096;
constexpr uint32_t kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64;
constexpr uint32_t kSmallBlocks = 256;  // one for each compute unit: their LDS is taken

// Bit i: page p0 + i is in the pool and has (LIVE) or has not any reference.
template <bool LIVE>
ARGUS_DEV uint32_t page_flags(const int32_t* refs, uint32_t p0, uint32_t N) {
  int32_t v[kPageItems];
  if (p0 + kPageItems <= N && ((uintptr_t)refs & 15u) == 0) {
#pragma unroll
    for (uint32_t i = 0; i < kPageItems; i += 4) {
      const int4 q = *reinterpret_cast<const int4*>(refs + p0 + i);
      v[i] = q.x, v[i + 1] = q.y, v[i + 2] = q.z, v[i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kPageItems; ++i) {
      const bool in = p0 + i < N;
      const int32_t x = refs[in ? p0 + i : 0];
      v[i] = in ? x : (LIVE ? 0 : 1);
    }
  }
  uint32_t flags = 0;
#pragma unroll
  for (uint32_t i = 0; i < kPageItems; ++i) flags |= (LIVE ? v[i] > 0 : v[i] == 0) ? 1u << i : 0u;
  return flags;
}

// Exclusive prefix of v over the block and, in *total, the block's sum.
template <uint32_t WAVES>
ARGUS_DEV uint32_t block_scan(uint32_t v, uint32_t* s_wave, uint32_t* total) {
  const uint32_t lane = lane_id(), wave = threadIdx.x >> 6;
  const uint32_t incl = (uint32_t)wave_incl_scan32((int32_t)v);
  __syncthreads();
  if (lane == 63) s_wave[wave] = incl;
  __syncthreads();
  uint32_t at = incl - v, all = 0;
#pragma unroll
  for (uint32_t w = 0; w < WAVES; ++w) {
    const uint32_t x = s_wave[w];
    at += w < wave ? x : 0u;
    all += x;
  }
  *total = all;
  return at;
}

struct Row {
  uint32_t src, len, grown, used, need;  // old sequence, old and new length, old pages, new pages
  bool kept, bad, cut;
};

ARGUS_DEV Row row_of(const StepArgs& a, uint32_t s) {
  Row r;
  const int32_t parent = a.parents ? a.parents[s] : (int32_t)s;
  r.bad = parent < -1 || parent >= (int64_t)a.S0;
  r.kept = parent >= 0 && !r.bad;
  r.src = r.kept ? (uint32_t)parent : 0u;
  const uint32_t most = a.P << a.shift, mask = (1u << a.shift) - 1;
  const int32_t n = r.kept ? a.lens[r.src] : 0;
  r.len = n < 0 ? 0u : ((uint32_t)n < most ? (uint32_t)n : most);
  const int32_t g = a.grow ? a.grow[s] : 0;
  const uint32_t more = g < 0 ? 0u : (uint32_t)g;
  r.cut = more > most - r.len;
  r.grown = r.cut ? most : r.len + more;
  r.used = (r.len >> a.shift) + ((r.len & mask) != 0);
  r.need = (r.grown >> a.shift) + ((r.grown & mask) != 0);
  return r;
}

// The entry that the row takes over in a column (-1: none).
ARGUS_DEV int32_t entry_of(const StepArgs& a, const Row& r, uint32_t col) {
  if (!r.kept || col >= r.used) return -1;
  const int32_t e = a.table[(int64_t)r.src * a.table_stride + col];
  if ((uint32_t)e >= a.N) return -1;
  if (a.window) {
    const int64_t first = (int64_t)r.len + (r.grown > r.len ? 1 : 0) - (int64_t)a.window;
    if ((((int64_t)col + 1) << a.shift) <= first && ((uint64_t)col << a.shift) >= a.sinks) return -1;
  }
  return e;
}

ARGUS_DEV bool ends_inside(const StepArgs& a, const Row& r) { return (r.len & ((1u << a.shift) - 1)) != 0; }

ARGUS_DEV void clear_page(const StepArgs& a, uint32_t p) {
  const int32_t h = a.held ? a.held[p] : 0;
  a.refs[p] = h < 0 ? 0 : h;
  a.best[p] = 0;
  a.lasts[p] = 0;
}

// The entries that sequence s takes over, by `lanes` threads from c0 on.
ARGUS_DEV void claim_row(const StepArgs& a, uint32_t s, uint32_t c0, uint32_t lanes) {
  const Row r = row_of(a, s);
  const bool inside = ends_inside(a, r);
  int32_t end = -1;
  for (uint32_t c = c0; c < a.P; c += lanes) {
    const int32_t e = entry_of(a, r, c);
    a.new_table[(int64_t)s * a.P + c] = e;
    const bool last = c + 1 == r.used && inside;
    if (e >= 0) {
      atomicAdd(&a.refs[e], 1);
      if (last) {
        atomicMax((unsigned long long*)&a.best[e], (unsigned long long)(r.len + 1) << 32 | (0xFFFFFFFFu - s));
        atomicAdd(&a.lasts[e], 1u);
      }
    }
    if (c + 1 == r.used) end = last && r.grown > r.len ? e : -1;
    if (c + 1 == r.used || (r.used == 0 && c == 0)) a.ends[s] = make_int2(end, (int32_t)(r.need - r.used));
  }
  if (c0 == 0) {
    a.new_lens[s] = (int32_t)r.grown;
    if (r.bad) atomicAdd(&a.counters[ARGUS_ST_BAD_PARENT], 1);
    if (r.cut) atomicAdd(&a.counters[ARGUS_ST_CUT], 1);
  }
}

// Whether sequence s may write on in page e, which it has last.
ARGUS_DEV bool writes_on(const StepArgs& a, uint32_t s, int32_t e) {
  const uint32_t refs = ld_agent((const uint32_t*)&a.refs[e]), lasts = ld_agent(&a.lasts[e]);
  const uint64_t best = ld_agent(&a.best[e]);
  return (a.held == nullptr || a.held[e] <= 0) && lasts == refs && (uint32_t)best == 0xFFFFFFFFu - s;
}

// Fresh pages that the sequences before each one take, by one block.
ARGUS_DEV void plan_rows(const StepArgs& a, uint32_t* s_wave) {
  constexpr uint32_t kRows = 4, THREADS = kThreads;
  uint32_t pages = 0, copies = 0;  // before
  for (uint32_t s0 = 0; s0 < a.S; s0 += THREADS * kRows) {
    int2 e[kRows];
    uint32_t need[kRows], n = 0, nc = 0;
#pragma unroll
    for (uint32_t i = 0; i < kRows; ++i) {
      const uint32_t s = s0 + threadIdx.x * kRows + i;
      e[i] = s < a.S ? a.ends[s] : make_int2(-1, 0);
    }
#pragma unroll
    for (uint32_t i = 0; i < kRows; ++i) {
      if (e[i].x >= 0 && writes_on(a, s0 + threadIdx.x * kRows + i, e[i].x)) e[i].x = -1;
      need[i] = (uint32_t)e[i].y + (e[i].x >= 0);
      n += need[i];
      nc += e[i].x >= 0;
    }
    uint32_t total, total_c;
    uint32_t at = pages + block_scan<THREADS / 64>(n, s_wave, &total);
    uint32_t at_c = copies + block_scan<THREADS / 64>(nc, s_wave, &total_c);
    pages += total;
    copies += total_c;
#pragma unroll
    for (uint32_t i = 0; i < kRows; ++i) {
      const uint32_t s = s0 + threadIdx.x * kRows + i;
      if (s < a.S) a.base[s] = at | (e[i].x >= 0 ? 0x80000000u : 0u);
      if (e[i].x >= 0) a.copies[at_c++] = make_uint2((uint32_t)e[i].x, at);
      at += need[i];
    }
  }
  if (threadIdx.x == 0) {
    a.state[2] = pages;
    a.state[3] = copies;
  }
}

// Fresh pages into the table of sequence s, by `lanes` threads from c0 on.
ARGUS_DEV void place_row(const StepArgs& a, uint32_t s, uint32_t c0, uint32_t lanes, uint32_t n_free) {
  const Row r = row_of(a, s);
  const uint32_t word = a.base[s], base = word & 0x7FFFFFFFu, copy = word >> 31;
  for (uint32_t c = r.used + c0; c < r.need; c += lanes) {
    const uint32_t rank = base + copy + c - r.used;
    const int32_t page = rank < n_free ? (int32_t)a.free_list[rank] : -1;
    a.new_table[(int64_t)s * a.P + c] = page;
    if (page >= 0) a.refs[page] = 1;
  }
  if (copy && c0 == 0) {
    int32_t* at = &a.new_table[(int64_t)s * a.P + r.used - 1];
    const int32_t page = base < n_free ? (int32_t)a.free_list[base] : -1;
    const int32_t old = a.ends[s].x;
    *at = page;
    if (page >= 0) {
      a.refs[page] = 1;
      atomicAdd(&a.counters[ARGUS_ST_COPIED], 1);
    }
    if (atomicSub(&a.refs[old], 1) == 1) atomicSub(&a.counters[ARGUS_ST_LIVE], 1);
  }
}

ARGUS_DEV void count_pages(const StepArgs& a, uint32_t n_free, uint32_t needed) {
  a.counters[ARGUS_ST_NEEDED] = (int32_t)needed;
  a.counters[ARGUS_ST_SHORT] = (int32_t)(needed > n_free ? needed - n_free : 0u);
  atomicAdd(&a.counters[ARGUS_ST_LIVE], (int32_t)(a.N - n_free + (needed < n_free ? needed : n_free)));
}

ARGUS_DEV void copy_step(const StepArgs& a, uint32_t wave, uint32_t waves) {
  const uint32_t n_free = a.state[1];
  copy_pages(a.caches, a.state[3], wave, waves, [&](uint32_t i, uint32_t* src, uint32_t* dst) {
    const uint2 c = a.copies[i];
    if (c.y >= n_free) return false;
    *src = c.x;
    *dst = a.free_list[c.y];
    return true;
  });
}

__global__ __launch_bounds__(kThreads) void k_step_clear(StepArgs a) {
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_STEP_CLEAR);
  const uint32_t i0 = blockIdx.x * kThreads + threadIdx.x, step = gridDim.x * kThreads;
  for (uint32_t p = i0; p < a.N; p += step) clear_page(a, p);
  for (uint32_t p = i0; p < (a.N + kPageTile - 1) / kPageTile; p += step) a.words[p] = 0;
  if (i0 < ARGUS_ST_NUM_COUNTERS) {
    a.state[i0] = 0;
    a.counters[i0] = 0;
  }
  mk.end(ARGUS_REGION_STEP_CLEAR);
}

// The entries that the new sequences take over, and who has which page.
__global__ __launch_bounds__(kThreads) void k_step_claim(StepArgs a) {
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_STEP_CLAIM);
  const uint32_t rows = kThreads / a.row_lanes;
  const uint32_t s = blockIdx.x * rows + threadIdx.x / a.row_lanes;
  if (s < a.S) claim_row(a, s, threadIdx.x % a.row_lanes, a.row_lanes);
  mk.end(ARGUS_REGION_STEP_CLAIM);
}

// Block 0: the sequences' fresh pages.  The others: the free pages in order, one
// tile of the pool after the other.
__global__ __launch_bounds__(kThreads) void k_step_plan(StepArgs a) {
  __shared__ uint32_t s_tile, s_before;
  __shared__ uint32_t s_wave[kWaves];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_STEP_PLAN);
  const uint32_t tid = threadIdx.x;
  if (blockIdx.x == 0) {
    plan_rows(a, s_wave);
  } else {
    // Tiles are taken in order, so a block waits for running blocks alone.
    if (tid == 0) s_tile = atomicAdd(&a.state[0], 1u);
    __syncthreads();
    const uint32_t tile = s_tile, p0 = tile * kPageTile + tid * kPageItems;
    const uint32_t free = page_flags<false>(a.refs, p0, a.N);
    uint32_t total;
    uint32_t at = block_scan<kWaves>((uint32_t)__popc(free), s_wave, &total);
    if (tid < 64) {
      uint64_t error = 0;
      const uint32_t before = (uint32_t)scan_lookback(a.words, tile, total, &error, 1);
      if (tid == 0) {
        if (error) a.counters[ARGUS_ST_INTERNAL] = 1;
        s_before = before;
        if ((uint64_t)(tile + 1) * kPageTile >= a.N) a.state[1] = before + total;
      }
    }
    __syncthreads();
    at += s_before;
    for (uint32_t f = free; f; f &= f - 1) a.free_list[at++] = p0 + (uint32_t)__builtin_ctz(f);
  }
  mk.end(ARGUS_REGION_STEP_PLAN);
}

// Fresh pages into the tables (the first rows_blocks blocks), pages copied (the others).
__global__ __launch_bounds__(kThreads) void k_step_place(StepArgs a) {
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_STEP_PLACE);
  if (blockIdx.x < a.rows_blocks) {
    const uint32_t n_free = a.state[1];
    const uint32_t rows = kThreads / a.row_lanes;
    const uint32_t s = blockIdx.x * rows + threadIdx.x / a.row_lanes;
    if (s < a.S) place_row(a, s, threadIdx.x % a.row_lanes, a.row_lanes, n_free);
    if (blockIdx.x == 0 && threadIdx.x == 0) count_pages(a, n_free, a.state[2]);
  } else {
    const uint32_t wave = (blockIdx.x - a.rows_blocks) * kWaves + threadIdx.x / 64;
    copy_step(a, __builtin_amdgcn_readfirstlane(wave), (gridDim.x - a.rows_blocks) * kWaves);
  }
  mk.end(ARGUS_REGION_STEP_PLACE);
}

// A small call: every block plans all of it for itself, in LDS, then the blocks share the
// copies.  Block 0 writes the tables.  One launch.
__global__ __launch_bounds__(kSmallThreads) void k_step_small(StepArgs a) {
  constexpr uint32_t kPages = kSmallPages / kSmallThreads;  // of a thread
  constexpr uint32_t kRows = kSmallRows / kSmallThreads;
  __shared__ uint32_t s_wave[kSmallWaves], s_count[ARGUS_ST_NUM_COUNTERS];
  __shared__ uint32_t s_refs[kSmallPages], s_lasts[kSmallPages];
  __shared__ unsigned long long s_best[kSmallPages];
  __shared__ uint16_t s_free[kSmallPages];
  __shared__ int2 s_ends[kSmallRows];      // as StepArgs::ends
  __shared__ uint2 s_copies[kSmallRows];   // as StepArgs::copies
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_STEP_PLAN);
  const uint32_t tid = threadIdx.x;
  const bool writes = blockIdx.x == 0;
#pragma unroll
  for (uint32_t i = 0; i < kPages; ++i) {
    const uint32_t p = tid + i * kSmallThreads;
    const int32_t h = a.held && p < a.N ? a.held[p] : 0;
    s_refs[p] = h < 0 ? 0u : (uint32_t)h;
    s_lasts[p] = 0;
    s_best[p] = 0;
  }
  if (tid < ARGUS_ST_NUM_COUNTERS) s_count[tid] = 0;
  __syncthreads();

  // the entries that the sequences take over, and who has which page
  const uint32_t rows = kSmallThreads / a.row_lanes, c0 = tid % a.row_lanes;
  for (uint32_t s = tid / a.row_lanes; s < a.S; s += rows) {
    const Row r = row_of(a, s);
    const bool inside = ends_inside(a, r);
    for (uint32_t c = c0; c < a.P; c += a.row_lanes) {
      const int32_t e = entry_of(a, r, c);
      if (writes && (c < r.used || c >= r.need)) a.new_table[(int64_t)s * a.P + c] = e;
      const bool last = c + 1 == r.used && inside;
      if (e >= 0) {
        atomicAdd(&s_refs[e], 1u);
        if (last) {
          atomicMax(&s_best[e], (unsigned long long)(r.len + 1) << 32 | (0xFFFFFFFFu - s));
          atomicAdd(&s_lasts[e], 1u);
        }
      }
      if (c + 1 == r.used || (r.used == 0 && c == 0))
        s_ends[s] = make_int2(last && r.grown > r.len ? e : -1, (int32_t)(r.need - r.used));
    }
    if (writes && c0 == 0) {
      a.new_lens[s] = (int32_t)r.grown;
      if (r.bad) atomicAdd(&s_count[ARGUS_ST_BAD_PARENT], 1u);
      if (r.cut) atomicAdd(&s_count[ARGUS_ST_CUT], 1u);
    }
  }
  __syncthreads();

  // the free pages in order
  uint32_t free = 0, n_free;
#pragma unroll
  for (uint32_t i = 0; i < kPages; ++i) {
    const uint32_t p = tid * kPages + i;
    free |= p < a.N && s_refs[p] == 0 ? 1u << i : 0u;
  }
  uint32_t at = block_scan<kSmallWaves>((uint32_t)__popc(free), s_wave, &n_free);
  for (uint32_t f = free; f; f &= f - 1) s_free[at++] = (uint16_t)(tid * kPages + (uint32_t)__builtin_ctz(f));
  // the fresh pages that the sequences before each one take; at most kSmallRows
  uint32_t need = 0, copies = 0, needed, copied;
  int2 e[kRows];
#pragma unroll
  for (uint32_t i = 0; i < kRows; ++i) {
    const uint32_t s = tid * kRows + i;
    e[i] = s < a.S ? s_ends[s] : make_int2(-1, 0);
    if (e[i].x >= 0) {
      const uint32_t p = (uint32_t)e[i].x;
      if ((a.held == nullptr || a.held[p] <= 0) && s_lasts[p] == s_refs[p] && (uint32_t)s_best[p] == 0xFFFFFFFFu - s) e[i].x = -1;
    }
    need += (uint32_t)e[i].y + (e[i].x >= 0);
    copies += e[i].x >= 0;
  }
  uint32_t base = block_scan<kSmallWaves>(need, s_wave, &needed);
  uint32_t at_c = block_scan<kSmallWaves>(copies, s_wave, &copied);
#pragma unroll
  for (uint32_t i = 0; i < kRows; ++i) {
    const uint32_t s = tid * kRows + i;
    if (s < a.S) s_ends[s] = make_int2((int32_t)base, e[i].x);
    if (e[i].x >= 0) s_copies[at_c++] = make_uint2((uint32_t)e[i].x, base);
    base += (uint32_t)e[i].y + (e[i].x >= 0);
  }
  __syncthreads();
  auto fresh = [&](uint32_t rank) { return rank < n_free ? (int32_t)s_free[rank] : -1; };

  if (writes) {  // fresh pages into the tables
    for (uint32_t s = tid / a.row_lanes; s < a.S; s += rows) {
      const Row r = row_of(a, s);
      const uint32_t first = (uint32_t)s_ends[s].x;
      const int32_t old = s_ends[s].y;
      const uint32_t copy = old >= 0;
      for (uint32_t c = r.used + c0; c < r.need; c += a.row_lanes) {
        const int32_t page = fresh(first + copy + c - r.used);
        a.new_table[(int64_t)s * a.P + c] = page;
        if (page >= 0) s_refs[page] = 1;
      }
      if (copy && c0 == 0) {
        const int32_t page = fresh(first);
        a.new_table[(int64_t)s * a.P + r.used - 1] = page;
        if (page >= 0) {
          s_refs[page] = 1;
          atomicAdd(&s_count[ARGUS_ST_COPIED], 1u);
        }
        if (atomicSub(&s_refs[old], 1u) == 1u) atomicSub(&s_count[ARGUS_ST_LIVE], 1u);
      }
    }
    __syncthreads();
    if (tid < ARGUS_ST_NUM_COUNTERS) {
      const uint32_t got = needed < n_free ? needed : n_free;
      a.counters[tid] = (int32_t)(tid == ARGUS_ST_NEEDED ? needed : tid == ARGUS_ST_SHORT ? needed - got
                                  : s_count[tid] + (tid == ARGUS_ST_LIVE ? a.N - n_free + got : 0u));
    }
    for (uint32_t p = tid; p < a.N; p += kSmallThreads) a.refs[p] = (int32_t)s_refs[p];
  }
  mk.end(ARGUS_REGION_STEP_PLAN);
  mk.begin(ARGUS_REGION_STEP_PLACE);
  copy_pages(a.caches, copied, __builtin_amdgcn_readfirstlane(blockIdx.x * kSmallWaves + tid / 64), gridDim.x * kSmallWaves,
             [&](uint32_t i, uint32_t* src, uint32_t* dst) {
               const uint2 c = s_copies[i];
               if (c.y >= n_free) return false;
               *src = c.x;
               *dst = s_free[c.y];
               return true;
             });
  mk.end(ARGUS_REGION_STEP_PLACE);
}

// --------------------------------------------------------------- compact
//
// n live pages: page p >= n of rank r (live pages below it) goes to the (r - stay)-th free page
// below n, stay = live pages below n: as many movers as holes, both in order, and no page is
// read that another one is written to.  What bounds it: the copies (8192 of 16384 pages live,
// 1.07 GB read and written in 211 us, 5.1 TB/s; ranks before them 9 us).

struct CompactArgs {
  const int32_t* table;
  int64_t table_stride;
  const int32_t* refs;
  int32_t *new_table, *new_refs, *map, *counters;
  uint32_t* tile_live;  // [tiles] live pages of each
  uint32_t* rank;       // [pages] live pages below
  uint32_t* holes;      // [pages] free pages below n, in order
  uint32_t* movers;     // [pages] the r-th live page, for those from n on
  uint32_t* state;      // 0: n, 1: live pages below n
  uint32_t S, P, N, tiles;
  uint32_t page_blocks, row_blocks;
  Caches caches;
  Marks marks;
};

__global__ __launch_bounds__(kThreads) void k_compact_count(CompactArgs a) {
  __shared__ uint32_t s_wave[kWaves];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_COMPACT_COUNT);
  uint32_t total;
  block_scan<kWaves>((uint32_t)__popc(page_flags<true>(a.refs, blockIdx.x * kPageTile + threadIdx.x * kPageItems, a.N)),
                     s_wave, &total);
  if (threadIdx.x == 0) a.tile_live[blockIdx.x] = total;
  mk.end(ARGUS_REGION_COMPACT_COUNT);
}

// Ranks, holes and movers of pages p0, ..., `rank` live pages before them and n in all.
ARGUS_DEV void rank_pages(const CompactArgs& a, uint32_t p0, uint32_t live, uint32_t rank, uint32_t n) {
  for (uint32_t i = 0; i < kPageItems; ++i) {
    const uint32_t p = p0 + i;
    if (p >= a.N) break;
    if (p == n) a.state[1] = rank;
    a.rank[p] = rank;
    if (live >> i & 1u) {
      if (p >= n) a.movers[rank] = p;
      ++rank;
    } else if (p < n) {
      a.holes[p - rank] = p;
    }
  }
}

__global__ __launch_bounds__(kThreads) void k_compact_plan(CompactArgs a) {
  __shared__ uint32_t s_wave[kWaves];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_COMPACT_PLAN);
  const uint32_t tid = threadIdx.x;
  uint32_t before = 0, n = 0;
  for (uint32_t t = tid; t < a.tiles; t += kThreads) {
    const uint32_t v = a.tile_live[t];
    n += v;
    before += t < blockIdx.x ? v : 0u;
  }
  const uint32_t p0 = blockIdx.x * kPageTile + tid * kPageItems;
  const uint32_t live = page_flags<true>(a.refs, p0, a.N);
  uint32_t total, all, all_before;
  block_scan<kWaves>(n, s_wave, &all);
  block_scan<kWaves>(before, s_wave, &all_before);
  const uint32_t rank = all_before + block_scan<kWaves>((uint32_t)__popc(live), s_wave, &total);
  rank_pages(a, p0, live, rank, all);
  if (blockIdx.x == 0 && tid == 0) {
    a.state[0] = all;
    if (all == a.N) a.state[1] = all;
  }
  mk.end(ARGUS_REGION_COMPACT_PLAN);
}

// A block's part of the move: pages, table entries or copies.  PLAN: live(p), rank(p), the
// live pages below p, and the i-th hole() and mover().
template <class Plan>
ARGUS_DEV void move_block(const CompactArgs& a, uint32_t n, uint32_t stay, const Plan& plan) {
  uint32_t b = blockIdx.x;
  if (b < a.page_blocks) {
    const uint32_t p = b * kThreads + threadIdx.x;
    if (p < a.N) {
      const int32_t refs = a.refs[p];
      const uint32_t rank = plan.rank(p);
      a.map[p] = refs <= 0 ? -1 : p < n ? (int32_t)p : (int32_t)plan.hole(rank - stay);
      a.new_refs[p] = p >= n ? 0 : refs > 0 ? refs : a.refs[plan.mover(p - rank)];
    }
    if (b == 0 && threadIdx.x < ARGUS_CO_NUM_COUNTERS)
      a.counters[threadIdx.x] = threadIdx.x == ARGUS_CO_LIVE ? (int32_t)n : threadIdx.x == ARGUS_CO_MOVED ? (int32_t)(n - stay) : 0;
  } else if ((b -= a.page_blocks) < a.row_blocks) {
    const uint64_t total = (uint64_t)a.S * a.P;
    for (uint64_t e = (uint64_t)b * kThreads + threadIdx.x; e < total; e += (uint64_t)a.row_blocks * kThreads) {
      const uint32_t s = (uint32_t)(e / a.P), c = (uint32_t)(e % a.P);
      const int32_t p = a.table[(int64_t)s * a.table_stride + c];
      int32_t to = -1;
      if ((uint32_t)p < a.N && plan.live((uint32_t)p)) to = (uint32_t)p < n ? p : (int32_t)plan.hole(plan.rank((uint32_t)p) - stay);
      a.new_table[e] = to;
    }
  } else {
    b -= a.row_blocks;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(b * kWaves + threadIdx.x / 64);
    copy_pages(a.caches, n - stay, wave, (gridDim.x - a.page_blocks - a.row_blocks) * kWaves,
               [&](uint32_t i, uint32_t* src, uint32_t* dst) {
                 *src = plan.mover(i);
                 *dst = plan.hole(i);
                 return true;
               });
  }
}

struct LargePlan {
  const CompactArgs& a;
  uint32_t stay;
  ARGUS_DEV bool live(uint32_t p) const { return a.refs[p] > 0; }
  ARGUS_DEV uint32_t rank(uint32_t p) const { return a.rank[p]; }
  ARGUS_DEV uint32_t hole(uint32_t i) const { return a.holes[i]; }
  ARGUS_DEV uint32_t mover(uint32_t i) const { return a.movers[stay + i]; }
};

__global__ __launch_bounds__(kThreads) void k_compact_move(CompactArgs a) {
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_COMPACT_MOVE);
  const uint32_t n = a.state[0], stay = a.state[1];
  move_block(a, n, stay, LargePlan{a, stay});
  mk.end(ARGUS_REGION_COMPACT_MOVE);
}

// A small pool is planned by every block for itself, in LDS: one launch.
struct SmallPlan {
  uint32_t n, stay;
  const uint16_t *flags, *base, *holes, *movers;  // of 16 pages: which live, how many before; lists, the movers' backwards
  ARGUS_DEV bool live(uint32_t p) const { return flags[p / kPageItems] >> (p % kPageItems) & 1u; }
  ARGUS_DEV uint32_t rank(uint32_t p) const {
    return base[p / kPageItems] + (uint32_t)__popc(flags[p / kPageItems] & ((1u << (p % kPageItems)) - 1u));
  }
  ARGUS_DEV uint32_t hole(uint32_t i) const { return holes[i]; }
  ARGUS_DEV uint32_t mover(uint32_t i) const { return movers[n - stay - 1 - i]; }
};
static_assert(kSmallPages == kPageTile && kPageItems == 16 && kSmallPages <= 65536, "a tile, flags and numbers in 16 bits");

__global__ __launch_bounds__(kThreads) void k_compact_small(CompactArgs a) {
  __shared__ uint32_t s_wave[kWaves];
  __shared__ uint16_t s_flags[kThreads], s_base[kThreads], s_holes[kSmallPages / 2], s_movers[kSmallPages / 2];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_COMPACT_PLAN);
  const uint32_t tid = threadIdx.x, p0 = tid * kPageItems;
  const uint32_t live = page_flags<true>(a.refs, p0, a.N);
  uint32_t n;
  const uint32_t first = block_scan<kWaves>((uint32_t)__popc(live), s_wave, &n);
  s_flags[tid] = (uint16_t)live;
  s_base[tid] = (uint16_t)first;
  // No more than half of the pages: as many holes below n as movers from n on.
  uint32_t rank = first;
#pragma unroll
  for (uint32_t i = 0; i < kPageItems; ++i) {
    const uint32_t p = p0 + i;
    if (live >> i & 1u) {
      if (p >= n) s_movers[n - 1 - rank] = (uint16_t)p;
      ++rank;
    } else if (p < n) {
      s_holes[p - rank] = (uint16_t)p;
    }
  }
  __syncthreads();
  SmallPlan plan{n, n, s_flags, s_base, s_holes, s_movers};
  if (n < a.N) plan.stay = plan.rank(n);
  mk.end(ARGUS_REGION_COMPACT_PLAN);
  mk.begin(ARGUS_REGION_COMPACT_MOVE);
  move_block(a, n, plan.stay, plan);
  mk.end(ARGUS_REGION_COMPACT_MOVE);
}

// ------------------------------------------------------------------ host

int take_caches(const argus_page_planes* in, uint32_t n, Caches* out) {
  if (n > ARGUS_MAX_CACHES) return refuse(ARGUS_E_INVAL, "num_caches %u (0..%d)", n, ARGUS_MAX_CACHES);
  out->n = n;
  for (uint32_t i = 0; i < n; ++i) {
    if (!in[i].base || in[i].planes < 1 || in[i].page_bytes < 16)
      return refuse(ARGUS_E_INVAL, "cache %u: no base, planes or page_bytes", i);
    if (!aligned_to(in[i].base, 16) || in[i].plane_stride % 16 || in[i].page_stride % 16 || in[i].page_bytes % 16)
      return refuse(ARGUS_E_ALIGN, "cache %u: base, strides and page_bytes are multiples of 16", i);
    out->c[i] = Planes{(uint8_t*)in[i].base, in[i].plane_stride, in[i].page_stride, in[i].planes, in[i].page_bytes / 16};
  }
  return ARGUS_OK;
}

// Blocks for the copies of at most n pages.
uint32_t copy_blocks_for(const Caches& all, uint32_t n) {
  uint64_t chunks = 0;
  for (uint32_t i = 0; i < all.n; ++i) chunks += (uint64_t)n * all.c[i].planes * ((all.c[i].units + 255) / 256);
  const uint64_t blocks = (chunks + kWaves - 1) / kWaves;
  return blocks < kCopyBlocks ? (uint32_t)blocks : kCopyBlocks;
}

struct StepLayout {
  size_t best, lasts, ends, base, copies, free_list, words, state, bytes;
};
StepLayout step_layout(uint32_t S, uint32_t N) {
  StepLayout l{};
  size_t o = 0;
  auto take = [&](size_t b) {
    const size_t at = o;
    o += up256(b ? b : 1);
    return at;
  };
  l.best = take(8ull * N);
  l.lasts = take(4ull * N);
  l.free_list = take(4ull * N);
  l.ends = take(8ull * S);
  l.base = take(4ull * S);
  l.copies = take(8ull * S);
  l.words = take(8ull * ((N + kPageTile - 1) / kPageTile));
  l.state = take(64);
  l.bytes = o;
  return l;
}

uint32_t row_lanes_for(uint32_t columns) {
  uint32_t l = 1;
  while (l < columns && l < (uint32_t)kThreads) l <<= 1;
  return l;
}

}  // namespace
}  // namespace decode
}  // namespace argus

using namespace argus;
using namespace argus::decode;

extern "C" int argus_decode_append(const argus_append_config* cfg, const argus_append_io* io, argus_markers* markers,
                                   void* stream_v) {
  accepted();
  if (!cfg || !io) return refuse(ARGUS_E_INVAL, "no configuration");
  if (cfg->abi_version != ARGUS_ATTR_ABI_VERSION) return refuse(ARGUS_E_ABI, "abi_version %u", cfg->abi_version);
  if (cfg->source_type > ARGUS_FP16) return refuse(ARGUS_E_INVAL, "new rows are bf16 or fp16");
  if (cfg->cache_type != cfg->source_type && cfg->cache_type != ARGUS_FP8)
    return refuse(ARGUS_E_INVAL, "the cache is of the rows' type or fp8 (e4m3)");
  const bool f8 = cfg->cache_type == ARGUS_FP8;
  const uint32_t unit = f8 ? 16u : 8u;
  if (cfg->seqs > (1u << 20)) return refuse(ARGUS_E_CAPACITY, "seqs %u", cfg->seqs);
  if (cfg->kv_heads < 1 || cfg->kv_heads > 1024) return refuse(ARGUS_E_INVAL, "kv_heads %u (1..1024)", cfg->kv_heads);
  if (cfg->head_dim < 8 || cfg->head_dim > 256 || cfg->head_dim % unit)
    return refuse(ARGUS_E_INVAL, "head_dim %u: a multiple of %u up to 256", cfg->head_dim, unit);
  if (!power_of_two(cfg->page_size) || cfg->page_size < 8 || cfg->page_size > 65536)
    return refuse(ARGUS_E_INVAL, "page_size %u: a power of two, 8..65536", cfg->page_size);
  if (cfg->num_pages < 1 || cfg->num_pages > 0x7FFFFFFFu || cfg->columns < 1 ||
      (uint64_t)cfg->columns * cfg->page_size > 0x7FFFFFFFull || cfg->rows > 0x7FFFFFFFu)
    return refuse(ARGUS_E_CAPACITY, "pages, columns or rows out of range");
  if (!io->d_offsets && cfg->rows && cfg->rows != cfg->seqs)
    return refuse(ARGUS_E_INVAL, "without offsets there is one row per sequence: %u rows, %u sequences", cfg->rows, cfg->seqs);
  if (cfg->rows && cfg->seqs && (!io->d_new_k || !io->d_new_v || !io->d_table || !io->d_starts))
    return refuse(ARGUS_E_INVAL, "a required pointer is NULL");
  int rc;
  if ((rc = check_view(io->k, cfg->cache_type, "k")) != ARGUS_OK || (rc = check_view(io->v, cfg->cache_type, "v")) != ARGUS_OK)
    return rc;
  if (!aligned_to(io->d_new_k, 16) || !aligned_to(io->d_new_v, 16) || io->k_row_stride % 8 || io->k_head_stride % 8 ||
      io->v_row_stride % 8 || io->v_head_stride % 8 || !aligned_to(io->d_table, 4) || !aligned_to(io->d_starts, 4) ||
      !aligned_to(io->d_offsets, 4) || !aligned_to(io->d_k_scale, 4) || !aligned_to(io->d_v_scale, 4))
    return refuse(ARGUS_E_ALIGN, "rows of the new keys and values lie on 16 bytes");
  if (io->table_stride < (int64_t)cfg->columns && cfg->seqs > 1)
    return refuse(ARGUS_E_INVAL, "table_stride %lld below columns", (long long)io->table_stride);
  if (marks_bad(markers)) return refuse(ARGUS_E_INVAL, "markers: alignment or region_base");
  AppendArgs a{};
  const uint32_t per_head = cfg->head_dim / unit, per_token = 2 * cfg->kv_heads * per_head;
  // Blocks of 1024 chunks where there are enough of them, else a token each.
  a.tokens = cfg->rows >= 4096 ? 1024 / per_token : 1;
  a.tokens = a.tokens < 1 ? 1 : a.tokens > kMaxTokens ? kMaxTokens : a.tokens;
  const uint32_t blocks = (cfg->rows + a.tokens - 1) / a.tokens;
  if (blocks > kMaxBlocks) return refuse(ARGUS_E_CAPACITY, "%u rows in one call", cfg->rows);
  if (!marks_fit(markers, (uint64_t)blocks * kWaves * 2)) return refuse(ARGUS_E_CAPACITY, "the marker records do not fit");
  if (cfg->rows == 0 || cfg->seqs == 0) return ARGUS_OK;
  if ((rc = device_ok()) != ARGUS_OK) return rc;
  const int64_t e = type_bytes(cfg->cache_type);
  a.new_k = (const uint8_t*)io->d_new_k, a.new_v = (const uint8_t*)io->d_new_v;
  a.k_row = io->k_row_stride * 2, a.k_hd = io->k_head_stride * 2;
  a.v_row = io->v_row_stride * 2, a.v_hd = io->v_head_stride * 2;
  a.k = (uint8_t*)io->k.base, a.v = (uint8_t*)io->v.base;
  a.k_page = io->k.page_stride * e, a.k_head = io->k.head_stride * e, a.k_tok = io->k.token_stride * e;
  a.v_page = io->v.page_stride * e, a.v_head = io->v.head_stride * e, a.v_tok = io->v.token_stride * e;
  a.table = io->d_table, a.table_stride = io->table_stride;
  a.starts = io->d_starts, a.offsets = io->d_offsets;
  a.k_scale = io->d_k_scale, a.v_scale = io->d_v_scale;
  a.S = cfg->seqs, a.rows = cfg->rows, a.shift = log2_of(cfg->page_size);
  a.num_pages = cfg->num_pages, a.columns = cfg->columns;
  a.per_token = fast_div(per_token);
  a.per_side = fast_div(per_token / 2);
  a.per_head = fast_div(per_head);
  a.marks = take_marks(markers, blocks, 2);
  hipStream_t st = (hipStream_t)stream_v;
  if (!f8) hipLaunchKernelGGL(k_append<0>, dim3(blocks), dim3(kThreads), 0, st, a);
  else if (cfg->source_type == ARGUS_BF16) hipLaunchKernelGGL(k_append<1>, dim3(blocks), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(k_append<2>, dim3(blocks), dim3(kThreads), 0, st, a);
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}

extern "C" size_t argus_decode_step_workspace_bytes(uint32_t new_seqs, uint32_t num_pages) {
  accepted();
  if (new_seqs > (1u << 20) || num_pages < 1 || num_pages > (1u << 28)) {
    refuse(ARGUS_E_CAPACITY, "new_seqs %u, num_pages %u", new_seqs, num_pages);
    return (size_t)-1;
  }
  return step_layout(new_seqs, num_pages).bytes;
}

extern "C" int argus_decode_step(const argus_step_config* cfg, const argus_step_io* io, void* d_workspace,
                                 size_t workspace_bytes, argus_markers* markers, void* stream_v) {
  accepted();
  if (!cfg || !io) return refuse(ARGUS_E_INVAL, "no configuration");
  if (cfg->abi_version != ARGUS_ATTR_ABI_VERSION) return refuse(ARGUS_E_ABI, "abi_version %u", cfg->abi_version);
  if (cfg->old_seqs > (1u << 20) || cfg->new_seqs > (1u << 20) || cfg->num_pages < 1 || cfg->num_pages > (1u << 28))
    return refuse(ARGUS_E_CAPACITY, "sequences or pages out of range");
  if (!power_of_two(cfg->page_size) || cfg->page_size > 65536)
    return refuse(ARGUS_E_INVAL, "page_size %u: a power of two up to 65536", cfg->page_size);
  if (cfg->columns < 1 || (uint64_t)cfg->columns * cfg->page_size > 0x7FFFFFFFull ||
      (uint64_t)cfg->columns * cfg->new_seqs > 0x7FFF0000ull || cfg->window > 0x7FFFFFFFu || cfg->sinks > 0x7FFFFFFFu)
    return refuse(ARGUS_E_CAPACITY, "columns, window or sinks out of range");
  if (!io->d_parents && cfg->new_seqs && cfg->old_seqs != cfg->new_seqs)
    return refuse(ARGUS_E_INVAL, "without parents the sequences stay: %u old, %u new", cfg->old_seqs, cfg->new_seqs);
  if ((cfg->old_seqs && (!io->d_table || !io->d_lens)) || (cfg->new_seqs && (!io->d_new_table || !io->d_new_lens)) ||
      !io->d_refs || !io->d_counters)
    return refuse(ARGUS_E_INVAL, "a required pointer is NULL");
  // (without sequences the tables may both be NULL)
  if ((io->d_new_table && io->d_new_table == io->d_table) || (io->d_new_lens && io->d_new_lens == io->d_lens) || io->d_refs == io->d_held)
    return refuse(ARGUS_E_INVAL, "the new table, lens and refs are other buffers than the old");
  if (!aligned_to(io->d_table, 4) || !aligned_to(io->d_lens, 4) || !aligned_to(io->d_parents, 4) || !aligned_to(io->d_grow, 4) ||
      !aligned_to(io->d_held, 4) || !aligned_to(io->d_new_table, 4) || !aligned_to(io->d_new_lens, 4) ||
      !aligned_to(io->d_refs, 4) || !aligned_to(io->d_counters, 4))
    return refuse(ARGUS_E_ALIGN, "tables lie on 4 bytes");
  if (cfg->old_seqs > 1 && io->table_stride < (int64_t)cfg->columns)
    return refuse(ARGUS_E_INVAL, "table_stride %lld below columns", (long long)io->table_stride);
  StepArgs a{};
  int rc = take_caches(io->caches, cfg->num_caches, &a.caches);
  if (rc != ARGUS_OK) return rc;
  if (marks_bad(markers)) return refuse(ARGUS_E_INVAL, "markers: alignment or region_base");
  const StepLayout l = step_layout(cfg->new_seqs, cfg->num_pages);
  if (!d_workspace) return refuse(ARGUS_E_INVAL, "no workspace");
  if (!aligned_to(d_workspace, 256)) return refuse(ARGUS_E_ALIGN, "the workspace lies on 256 bytes");
  if (workspace_bytes < l.bytes) return refuse(ARGUS_E_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, l.bytes);
  char* ws = (char*)d_workspace;
  a.table = io->d_table, a.table_stride = io->table_stride, a.lens = io->d_lens, a.parents = io->d_parents;
  a.grow = io->d_grow, a.held = io->d_held, a.new_table = io->d_new_table, a.new_lens = io->d_new_lens;
  a.refs = io->d_refs, a.counters = io->d_counters;
  a.best = (uint64_t*)(ws + l.best), a.lasts = (uint32_t*)(ws + l.lasts), a.ends = (int2*)(ws + l.ends), a.base = (uint32_t*)(ws + l.base);
  a.copies = (uint2*)(ws + l.copies), a.free_list = (uint32_t*)(ws + l.free_list), a.words = (uint64_t*)(ws + l.words);
  a.state = (uint32_t*)(ws + l.state);
  a.S0 = cfg->old_seqs, a.S = cfg->new_seqs, a.P = cfg->columns, a.N = cfg->num_pages;
  a.shift = log2_of(cfg->page_size), a.window = cfg->window, a.sinks = cfg->sinks;
  a.row_lanes = row_lanes_for(a.P);
  const uint32_t rows = kThreads / a.row_lanes;
  a.rows_blocks = (a.S + rows - 1) / rows;
  if (a.rows_blocks == 0) a.rows_blocks = 1;
  const uint32_t tiles = (a.N + kPageTile - 1) / kPageTile;
  uint32_t clear = (a.N + kThreads - 1) / kThreads;
  clear = clear > 1024 ? 1024 : clear;
  const uint32_t copy_blocks = copy_blocks_for(a.caches, a.S);
  hipStream_t st = (hipStream_t)stream_v;
  if ((uint64_t)a.S * a.P <= kSmallEntries && a.S <= kSmallRows && a.N <= kSmallPages) {
    // (a block's waves write their markers as those of four blocks)
    constexpr uint32_t kBlocks = kSmallWaves / kWaves;
    const uint32_t wanted = (copy_blocks + kBlocks - 1) / kBlocks;
    const uint32_t blocks = wanted < 1 ? 1 : wanted < kSmallBlocks ? wanted : kSmallBlocks;
    if (!marks_fit(markers, (uint64_t)blocks * kSmallWaves * 4)) return refuse(ARGUS_E_CAPACITY, "the marker records do not fit");
    if ((rc = device_ok()) != ARGUS_OK) return rc;
    a.marks = take_marks(markers, (uint64_t)blocks * kBlocks, 4);
    hipLaunchKernelGGL(k_step_small, dim3(blocks), dim3(kSmallThreads), 0, st, a);
    return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
  }
  const uint32_t grid[4] = {clear, a.rows_blocks, tiles + 1, a.rows_blocks + copy_blocks};
  if (!marks_fit(markers, ((uint64_t)grid[0] + grid[1] + grid[2] + grid[3]) * kWaves * 2))
    return refuse(ARGUS_E_CAPACITY, "the marker records do not fit");
  if ((rc = device_ok()) != ARGUS_OK) return rc;
  a.marks = take_marks(markers, grid[0], 2);
  hipLaunchKernelGGL(k_step_clear, dim3(grid[0]), dim3(kThreads), 0, st, a);
  a.marks = take_marks(markers, grid[1], 2);
  hipLaunchKernelGGL(k_step_claim, dim3(grid[1]), dim3(kThreads), 0, st, a);
  a.marks = take_marks(markers, grid[2], 2);
  hipLaunchKernelGGL(k_step_plan, dim3(grid[2]), dim3(kThreads), 0, st, a);
  a.marks = take_marks(markers, grid[3], 2);
  hipLaunchKernelGGL(k_step_place, dim3(grid[3]), dim3(kThreads), 0, st, a);
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}

namespace {
struct CompactLayout {
  size_t tile_live, rank, holes, movers, state, bytes;
};
CompactLayout compact_layout(uint32_t N) {
  CompactLayout l{};
  size_t o = 0;
  auto take = [&](size_t b) {
    const size_t at = o;
    o += up256(b);
    return at;
  };
  l.tile_live = take(4ull * ((N + kPageTile - 1) / kPageTile));
  l.rank = take(4ull * N);
  l.holes = take(4ull * N);
  l.movers = take(4ull * N);
  l.state = take(64);
  l.bytes = o;
  return l;
}
}  // namespace

extern "C" size_t argus_decode_compact_workspace_bytes(uint32_t num_pages) {
  accepted();
  if (num_pages < 1 || num_pages > (1u << 28)) {
    refuse(ARGUS_E_CAPACITY, "num_pages %u", num_pages);
    return (size_t)-1;
  }
  return compact_layout(num_pages).bytes;
}

extern "C" int argus_decode_compact(const argus_compact_config* cfg, const argus_compact_io* io, void* d_workspace,
                                    size_t workspace_bytes, argus_markers* markers, void* stream_v) {
  accepted();
  if (!cfg || !io) return refuse(ARGUS_E_INVAL, "no configuration");
  if (cfg->abi_version != ARGUS_ATTR_ABI_VERSION) return refuse(ARGUS_E_ABI, "abi_version %u", cfg->abi_version);
  if (cfg->seqs > (1u << 20) || cfg->columns < 1 || (uint64_t)cfg->columns * cfg->seqs > 0x7FFF0000ull ||
      cfg->num_pages < 1 || cfg->num_pages > (1u << 28))
    return refuse(ARGUS_E_CAPACITY, "sequences, columns or pages out of range");
  if ((cfg->seqs && (!io->d_table || !io->d_new_table)) || !io->d_refs || !io->d_new_refs || !io->d_map || !io->d_counters)
    return refuse(ARGUS_E_INVAL, "a required pointer is NULL");
  if ((cfg->seqs && io->d_new_table == io->d_table) || io->d_new_refs == io->d_refs || io->d_map == io->d_refs || io->d_map == io->d_new_refs)
    return refuse(ARGUS_E_INVAL, "the new table, refs and map are buffers of their own");
  if (!aligned_to(io->d_table, 4) || !aligned_to(io->d_refs, 4) || !aligned_to(io->d_new_table, 4) ||
      !aligned_to(io->d_new_refs, 4) || !aligned_to(io->d_map, 4) || !aligned_to(io->d_counters, 4))
    return refuse(ARGUS_E_ALIGN, "tables lie on 4 bytes");
  if (cfg->seqs > 1 && io->table_stride < (int64_t)cfg->columns)
    return refuse(ARGUS_E_INVAL, "table_stride %lld below columns", (long long)io->table_stride);
  CompactArgs a{};
  int rc = take_caches(io->caches, cfg->num_caches, &a.caches);
  if (rc != ARGUS_OK) return rc;
  if (marks_bad(markers)) return refuse(ARGUS_E_INVAL, "markers: alignment or region_base");
  const CompactLayout l = compact_layout(cfg->num_pages);
  if (!d_workspace) return refuse(ARGUS_E_INVAL, "no workspace");
  if (!aligned_to(d_workspace, 256)) return refuse(ARGUS_E_ALIGN, "the workspace lies on 256 bytes");
  if (workspace_bytes < l.bytes) return refuse(ARGUS_E_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, l.bytes);
  char* ws = (char*)d_workspace;
  a.table = io->d_table, a.table_stride = io->table_stride, a.refs = io->d_refs;
  a.new_table = io->d_new_table, a.new_refs = io->d_new_refs, a.map = io->d_map, a.counters = io->d_counters;
  a.tile_live = (uint32_t*)(ws + l.tile_live), a.rank = (uint32_t*)(ws + l.rank), a.holes = (uint32_t*)(ws + l.holes);
  a.movers = (uint32_t*)(ws + l.movers), a.state = (uint32_t*)(ws + l.state);
  a.S = cfg->seqs, a.P = cfg->columns, a.N = cfg->num_pages;
  a.tiles = (a.N + kPageTile - 1) / kPageTile;
  a.page_blocks = (a.N + kThreads - 1) / kThreads;
  const uint64_t entries = (uint64_t)a.S * a.P;
  a.row_blocks = (uint32_t)((entries + 4 * kThreads - 1) / (4 * kThreads));
  const uint32_t copy_blocks = copy_blocks_for(a.caches, a.N / 2);
  const uint32_t moves = a.page_blocks + a.row_blocks + copy_blocks;
  const bool small = a.N <= kSmallPages;
  const uint64_t blocks = 2ull * (small ? 0 : a.tiles) + moves;
  if (!marks_fit(markers, (blocks + (small ? moves : 0)) * kWaves * 2)) return refuse(ARGUS_E_CAPACITY, "the marker records do not fit");
  if ((rc = device_ok()) != ARGUS_OK) return rc;
  hipStream_t st = (hipStream_t)stream_v;
  if (small) {
    a.marks = take_marks(markers, moves, 4);
    hipLaunchKernelGGL(k_compact_small, dim3(moves), dim3(kThreads), 0, st, a);
  } else {
    a.marks = take_marks(markers, a.tiles, 2);
    hipLaunchKernelGGL(k_compact_count, dim3(a.tiles), dim3(kThreads), 0, st, a);
    a.marks = take_marks(markers, a.tiles, 2);
    hipLaunchKernelGGL(k_compact_plan, dim3(a.tiles), dim3(kThreads), 0, st, a);
    a.marks = take_marks(markers, moves, 2);
    hipLaunchKernelGGL(k_compact_move, dim3(moves), dim3(kThreads), 0, st, a);
  }
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}
