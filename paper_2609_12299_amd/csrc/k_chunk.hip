// k_chunk.hip -- attention of chunks of new tokens (k_chunk.h): the host's side, the batch shared out,
// and the pieces joined.
#include "k_chunk.h"

namespace argus {
namespace prompt {
namespace {

// The batch in pieces, by one block: the items (row tiles) of a head, and those of more than `most` steps in
// equal pieces, which are the first in the list: they take the longest. Heads come innermost, so
// that with eight of them each has an XCD, in whose L2 its keys and values are.
//
// With U steps of n items and C blocks at a time, pieces of U / C steps would end together; cut from
// items of any length they are up to n more. So some lengths for one and for two rounds of blocks are
// tried, none but those whose pieces are as few, and the shortest way is taken: rounds times (length + what
// a piece costs), and what joining costs, all in steps; or nothing is cut. Where there are more items than two
// rounds of blocks take, those of more than 2 U / C steps are cut. What is not cut comes in eight classes of length, the
// longest first, each in the order of its slots (a batch of single tokens and chunks 139 us against 171, 64 single tokens
// behind up to 30000 278 against 295, chunks over 8 bits 1295 against 1377).
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
constexpr uint32_t kPlanItems = 4096, kPlanSplit = 1024;
constexpr uint32_t kLeastPiece = 4, kItemCost = 2, kPieceCost = 8, kJoinCost = 8, kClasses = 8;
__global__ __launch_bounds__(kPlanThreads) void k_chunk_plan(ChunkArgs a) {
  __shared__ uint64_t s_units[kPlanWaves];
  __shared__ uint32_t s_items[kPlanWaves], s_most[kPlanWaves], s_pieces[kPlanWaves], s_split[kPlanWaves], s_length[kPlanWaves], s_cost[kPlanWaves];
  __shared__ uint32_t s_class[kClasses], s_in_class[kPlanWaves][kClasses];
  __shared__ uint32_t s_steps[kPlanItems];
  __shared__ uint4 s_join[kPlanSplit];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_CHUNK_PLAN);
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = scalar(tid >> 6);
  uint64_t units = 0;
  uint32_t items = 0, longest = 0;
  // items in the order of their slots, the last first
  for (uint32_t x0 = 0; x0 < a.slots; x0 += kPlanThreads) {
    const uint32_t x = a.slots - 1 - x0 - tid;
    Reach g;
    bool real = false;
    uint32_t s = 0, first = 0;
    if (x0 + tid < a.slots) {
      uint32_t hi = a.S;
      while (hi - s > 1) {  // the last sequence whose slots start at or before x
        const uint32_t mid = (s + hi) / 2;
        if (slot_of(a, mid) <= x) s = mid; else hi = mid;
      }
      first = slot_of(a, s);
      real = first <= x && reach_of(a, s, x - first, &g);
    }
    const uint32_t mine = real ? g.steps : 0;
    uint64_t sum = mine;
    uint32_t most = mine;
    for (int d = 1; d < 64; d <<= 1) {
      sum += __shfl_xor(sum, d);
      const uint32_t o = __shfl_xor(most, d);
      most = o > most ? o : most;
    }
    const uint64_t there = __ballot(real);
    if (lane == 0) s_units[wave] = sum, s_items[wave] = (uint32_t)__popcll(there), s_most[wave] = most;
    __syncthreads();
    uint32_t at = items;
    for (uint32_t w = 0; w < (uint32_t)kPlanWaves; ++w) {
      if (w < wave) at += s_items[w];
      units += s_units[w], items += s_items[w];
      longest = s_most[w] > longest ? s_most[w] : longest;
    }
    if (real) {
      at += (uint32_t)__popcll(there & lanemask_lt());
      a.items[at] = make_uint4(s, x - first, mine, 0u);
      if (at < kPlanItems) s_steps[at] = mine;
    }
    __syncthreads();
  }
  auto steps_of = [&](uint32_t i) { return items <= kPlanItems ? s_steps[i] : a.items[i].z; };
  // lengths of a piece: rounds 1 and 2, with room for none, half and all of the items' last pieces
  const uint64_t all = units * a.H, blocks = a.blocks, heads = (uint64_t)items * a.H;
  uint32_t length = longest, cost = ~0u;
  if (wave < 6) {
    const uint64_t rounds = wave / 3 + 1, room = rounds * blocks - (heads * (wave % 3)) / 2;
    bool fits = rounds * blocks > heads && items;
    if (fits) {
      const uint64_t l = (all + room - 1) / room;
      length = l < kLeastPiece ? kLeastPiece : l < longest ? (uint32_t)l : longest;
      uint32_t pieces = 0;
      for (uint32_t i = lane; i < items; i += 64) pieces += (steps_of(i) + length - 1) / length;
      for (int d = 1; d < 64; d <<= 1) pieces += __shfl_xor(pieces, d);
      fits = (uint64_t)pieces * a.H <= rounds * blocks;
      if (fits) cost = (uint32_t)rounds * (length + kPieceCost) + kJoinCost;
    }
    if (lane == 0) s_length[wave] = length, s_cost[wave] = cost;
  }
  __syncthreads();
  // nothing cut: no joining, and as many rounds as there are items for
  uint32_t limit;  // steps of an item that is not cut, at most
  length = longest, cost = ~0u;
  if (heads > 2 * blocks) {
    const uint64_t l = (all + blocks - 1) / blocks;
    length = l < kLeastPiece ? kLeastPiece : l < longest ? (uint32_t)l : longest;
    limit = 2 * length;
  } else {
    // (one round, or one after the other as blocks end)
    cost = (heads > blocks ? (uint32_t)(all / blocks) + longest / 2 : longest) + kItemCost;
    for (int w = 0; w < 6; ++w)
      if (s_cost[w] < cost) cost = s_cost[w], length = s_length[w];
    limit = length;
  }
  auto parts_of = [&](uint32_t steps) { return steps > limit ? (steps + length - 1) / length : 1u; };
  auto class_of = [&](uint32_t steps) { return kClasses - 1 - (uint32_t)((uint64_t)steps * kClasses / (longest + 1)); };
  // how many items are cut, in how many pieces all of them, and how many of a class are not
  if (tid < kClasses) s_class[tid] = 0;
  __syncthreads();
  uint32_t cut = 0, parts = 0;
  for (uint32_t i = tid; i < items; i += kPlanThreads) {
    const uint32_t n = steps_of(i), k = parts_of(n);
    if (k > 1) ++cut, parts += k;
    else atomicAdd(&s_class[class_of(n)], 1u);
  }
  for (int d = 1; d < 64; d <<= 1) cut += __shfl_xor(cut, d), parts += __shfl_xor(parts, d);
  if (lane == 0) s_split[wave] = cut, s_pieces[wave] = parts;
  __syncthreads();
  cut = parts = 0;
  for (int w = 0; w < kPlanWaves; ++w) cut += s_split[w], parts += s_pieces[w];
  if (tid == 0) a.head[0] = parts + items - cut, a.head[1] = cut;
  // the next place of each class, behind the pieces
  if (tid == 0)
    for (uint32_t c = 0, at = parts; c < kClasses; ++c) {
      const uint32_t many = s_class[c];
      s_class[c] = at, at += many;
    }
  uint32_t cuts = 0, cut_parts = 0;  // before
  for (uint32_t i0 = 0; i0 < items; i0 += kPlanThreads) {
    __syncthreads();
    const uint32_t i = i0 + tid;
    const uint4 item = i < items ? a.items[i] : make_uint4(0u, 0u, 0u, 0u);
    const uint32_t k = i < items ? parts_of(item.z) : 0, mine = k == 1 ? class_of(item.z) : kClasses;
    const uint64_t is_cut = __ballot(k > 1);
    uint32_t q = 0;
#pragma unroll
    for (uint32_t c = 0; c < kClasses; ++c) {
      const uint64_t in = __ballot(mine == c);
      if (mine == c) q = s_class[c] + (uint32_t)__popcll(in & lanemask_lt());
      if (lane == c) s_in_class[wave][c] = (uint32_t)__popcll(in);
    }
    uint32_t incl = k > 1 ? k : 0;
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(incl, d);
      if ((int)lane >= d) incl += o;
    }
    if (lane == 63) s_pieces[wave] = incl, s_split[wave] = (uint32_t)__popcll(is_cut);
    __syncthreads();
    uint32_t part = cut_parts, j = cuts;
    for (uint32_t w = 0; w < (uint32_t)kPlanWaves; ++w) {
      if (w < wave) {
        part += s_pieces[w], j += s_split[w];
        if (mine < kClasses) q += s_in_class[w][mine];
      }
      cut_parts += s_pieces[w], cuts += s_split[w];
    }
    if (tid < kClasses)
      for (int w = 0; w < kPlanWaves; ++w) s_class[tid] += s_in_class[w][tid];
    if (k > 1) {
      const uint4 join = make_uint4(item.x, item.y, part + incl - k, item.z);
      j += (uint32_t)__popcll(is_cut & lanemask_lt());
      a.joins[j] = join;
      s_join[j] = join;
    } else if (k == 1) {
      a.pieces[q] = make_uint4(item.x, item.y, 0u, item.z);
    }
  }
  __syncthreads();
  for (uint32_t q = tid; q < parts; q += kPlanThreads) {
    uint32_t lo = 0, hi = cut;
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (s_join[mid].z <= q) lo = mid; else hi = mid;
    }
    const uint4 join = s_join[lo];
    const uint32_t k = (join.w + length - 1) / length, len = (join.w + k - 1) / k, t0 = (q - join.z) * len;
    a.pieces[q] = make_uint4(join.x, join.y, t0, t0 + len < join.w ? t0 + len : join.w);
  }
  if (tid == 0) a.head[2] = length, a.head[3] = parts;
  mk.end(ARGUS_REGION_CHUNK_PLAN);
}

// Rows of an item that was left in pieces. A block takes kRows of them at a time.
template <int T, int DP, int W>
__global__ __launch_bounds__(kThreads) void k_chunk_join(ChunkArgs a) {
  constexpr uint32_t kQuads = DP / 4, kRows = kThreads / kQuads, TR = 32 * W;
  using Hf = Half<T>;
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_CHUNK_JOIN);
  const uint32_t j = blockIdx.x / a.H, h = blockIdx.x % a.H;
  Reach g;
  if (j < (uint32_t)a.head[1]) {
    const uint4 join = a.joins[j];
    const uint32_t length = (uint32_t)a.head[2], n = (join.w + length - 1) / length;
    const bool real = reach_of(a, join.x, join.y, &g);
    const uint32_t d = threadIdx.x % kQuads * 4;
    for (uint32_t mine = blockIdx.y * kRows + threadIdx.x / kQuads; real && mine < g.rows; mine += gridDim.y * kRows) {
      float m = -INFINITY, l = 0.0f;
      f32x4 o = (f32x4)(0.0f);
      constexpr uint32_t kDeep = 8;
      for (uint32_t i0 = 0; i0 < n; i0 += kDeep) {
        f32x2 ml[kDeep];
        f32x4 v[kDeep];
        float top = m;
#pragma unroll
        for (uint32_t i = 0; i < kDeep; ++i) {
          const uint64_t x = ((uint64_t)(join.z + (i0 + i < n ? i0 + i : 0)) * a.H + h) * TR + mine;
          ml[i] = *reinterpret_cast<const f32x2*>(a.part_ml + 2 * x);
          v[i] = *reinterpret_cast<const f32x4*>(a.part_o + x * DP + d);
          if (i0 + i >= n) ml[i] = (f32x2){-INFINITY, 0.0f}, v[i] = (f32x4)(0.0f);
          top = fmaxf(top, ml[i].x);
        }
        const float keep = m == -INFINITY ? 1.0f : exp_of(m - top);  // (nothing yet, or NaN)
        l *= keep;
        o *= keep;
#pragma unroll
        for (uint32_t i = 0; i < kDeep; ++i) {
          const float w = ml[i].x == -INFINITY ? 1.0f : exp_of(ml[i].x - top);  // a maximum of -inf: zeros, or NaN
          l += ml[i].y * w;
          o += v[i] * w;
        }
        m = top;
      }
      // (NaN, and not by the scores: a piece's infinite sum may have met a weight that is none in 32 bits)
      if (__builtin_expect(l == l && !(o.x == o.x && o.y == o.y && o.z == o.z && o.w == o.w), 0)) {
        f32x4 sum = (f32x4)(0.0f);  // of what is not finite
        for (uint32_t i = 0; i < n; ++i) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(a.part_o + (((uint64_t)(join.z + i) * a.H + h) * TR + mine) * DP + d);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e] += fabsf(v[e]) < INFINITY ? 0.0f : v[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] == o[e] ? o[e] : sum[e];
      }
      const uint32_t r = g.r0 + mine, tok = divide(r, a.by_group);
      const uint64_t row = (uint64_t)(g.row0 + tok) * a.H * a.G + h * a.G + (r - tok * a.G);
      const float inv = l == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[h] : 1.0f) / l;
      if (d < a.D)
        *reinterpret_cast<u32x2*>(a.out + row * a.D + d) =
            l == 0.0f ? (u32x2)(0u) : (u32x2){Hf::pack(o.x * inv, o.y * inv), Hf::pack(o.z * inv, o.w * inv)};
      if (d == 0 && a.lse)
        a.lse[row] = l == 0.0f ? -INFINITY : (m == -INFINITY ? 0.0f : m - Hf::kRaise * kLn2) + logf(l);
    }
  }
  mk.end(ARGUS_REGION_CHUNK_JOIN);
}

template <int T>
void launch_chunk_join(const ChunkArgs& a, dim3 g, hipStream_t st) {
  const dim3 b(kThreads);
  const bool eight = a.tile_shift == 8;
  if (a.D <= 64) {
    hipLaunchKernelGGL((k_chunk_join<T, 64, 4>), g, b, 0, st, a);
  } else if (a.D <= 128) {
    if (eight) hipLaunchKernelGGL((k_chunk_join<T, 128, 8>), g, b, 0, st, a);
    else hipLaunchKernelGGL((k_chunk_join<T, 128, 4>), g, b, 0, st, a);
  } else {
    hipLaunchKernelGGL((k_chunk_join<T, 256, 4>), g, b, 0, st, a);
  }
}

// Eight waves a block, that read the cache once for 256 rows, or four. Eight where sequences have so many
// rows on the average, and there are so many tiles of them (16 prompts in chunks over 8 bits 1295 us against 1415 with
// four, one of 16384 tokens 3.97 ms against 4.25, four of up to 6000 at head size 96 469 us against 498; 16 prompts of up to
// 2000 tokens, 8 x 4 heads, 100.2 against 101.4, at head size 80 89 against 86), else four (proposals over 131000 tokens 340 us
// against 388 with eight, 64 single tokens 278 against 526, a batch of single tokens and chunks 139 against 150,
// one prompt of 512 tokens 18.6 against 22.8, of 2048, 8 x 4 heads, 54.3 against 60.7, of 512 behind 8192 in the cache 182
// both), and at head size 64, whose blocks of four run three at a time on a compute unit (4 prompts of up to
// 4000 tokens 159 us against 193 with eight).
constexpr uint32_t kManyRows = 1024, kManyTiles = 512;
// Blocks that run at once.
uint32_t blocks_at_once(uint32_t tile_shift, uint32_t head_dim) {
  return 256u * (head_dim > 128 || tile_shift == 8 ? 1 : head_dim > 64 ? 2 : 3);
}
// Row tiles of at most so many steps are not cut, and are found by their blocks: no plan and no joining (a
// prompt of 2048 tokens 54.3 us against 65.5, 16 of up to 2000 100 against 111). A table of more steps means both, and a workspace of
// 52 to 68 MB, whatever the lengths are, which are on the GPU: one prompt of 45 tokens 16.9 us where it is 9.7.
constexpr uint32_t kWholeSteps = 32;
constexpr uint32_t kJoinBlocks = 8;  // of an item, for its rows

struct Plan {
  uint32_t tile_shift, slots, grid, blocks, joins;
  size_t ml_at, o_at, items_at, joins_at, pieces_at, bytes;
};

int make_plan(const argus_chunk_config* c, Plan* p) {
  if (!c) return refuse(ARGUS_E_INVAL, "no configuration");
  if (c->abi_version != ARGUS_ATTR_ABI_VERSION) return refuse(ARGUS_E_ABI, "abi_version %u", c->abi_version);
  if (c->q_type > ARGUS_FP16) return refuse(ARGUS_E_INVAL, "q is bf16 or fp16");
  if (c->cache_type != c->q_type && c->cache_type != ARGUS_FP8)
    return refuse(ARGUS_E_INVAL, "the cache is of q's type or fp8 (e4m3)");
  if (c->seqs > (1u << 20)) return refuse(ARGUS_E_CAPACITY, "seqs %u", c->seqs);
  if (c->kv_heads < 1 || c->kv_heads > 1024 || c->group < 1 || c->group > 256)
    return refuse(ARGUS_E_INVAL, "kv_heads %u (1..1024), group %u (1..256)", c->kv_heads, c->group);
  if ((uint64_t)c->rows * c->group >= (1ull << 30)) return refuse(ARGUS_E_CAPACITY, "rows %u x group %u", c->rows, c->group);
  const uint32_t unit = c->head_dim > 128 || c->cache_type == ARGUS_FP8 ? 16u : 8u;
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % unit)
    return refuse(ARGUS_E_INVAL, "head_dim %u: a multiple of %u up to 256", c->head_dim, unit);
  if (!power_of_two(c->page_size) || c->page_size < 8 || c->page_size > 65536)
    return refuse(ARGUS_E_INVAL, "page_size %u: a power of two, 8..65536", c->page_size);
  if (c->num_pages < 1 || c->num_pages > 0x7FFFFFFFu || c->columns < 1 ||
      (uint64_t)c->columns * c->page_size > 0x3FFFFFFFull || c->window > 0x3FFFFFFFu || c->sinks > 0x3FFFFFFFu)
    return refuse(ARGUS_E_CAPACITY, "pages, columns, window or sinks out of range");
  const uint64_t rows = (uint64_t)c->rows * c->group;
  p->tile_shift = c->head_dim > 64 && c->head_dim <= 128 && rows >= (uint64_t)kManyRows * c->seqs &&
                          rows / 256 * c->kv_heads >= kManyTiles
                      ? 8 : 7;
  const uint32_t kt = c->head_dim > 128 ? 32 : 64, dp = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
  // At most two pieces for each block that runs at once are of items that were cut, and so few more than
  // the items are all pieces.
  uint64_t most, grid;
  for (;; p->tile_shift = 7) {
    p->slots = c->seqs ? ((c->rows * c->group) >> p->tile_shift) + c->seqs : 0;
    const uint64_t tiles = (uint64_t)p->slots * c->kv_heads;
    // steps of a row tile, as far as the table (or the window) allows
    uint64_t steps = ((uint64_t)c->columns * c->page_size + kt - 1) / kt;
    if (c->window) {
      const uint64_t w = (c->window + (1u << p->tile_shift) / c->group + 2 * kt) / kt + 1 + (c->sinks + kt - 1) / kt;
      steps = w < steps ? w : steps;
    }
    p->blocks = tiles && c->rows && steps > kWholeSteps ? blocks_at_once(p->tile_shift, c->head_dim) : 0;
    most = p->slots + 2 * p->blocks / c->kv_heads + 1, grid = p->blocks ? most * c->kv_heads : tiles;
    // (blocks of eight waves have twice the threads, and a launch has less than 2^32)
    if (grid <= (p->tile_shift == 8 ? kMaxBlocks / 2 : kMaxBlocks)) break;
    if (p->tile_shift == 7) return refuse(ARGUS_E_CAPACITY, "rows %u x group %u, seqs %u, kv_heads %u", c->rows, c->group, c->seqs, c->kv_heads);
  }
  p->grid = (uint32_t)grid;
  const uint32_t cut = p->slots < p->blocks / c->kv_heads ? p->slots : p->blocks / c->kv_heads;
  p->joins = p->blocks ? cut * c->kv_heads : 0;
  const size_t part_rows = (size_t)2 * p->blocks << p->tile_shift;
  p->ml_at = 256;
  p->o_at = p->ml_at + up256(part_rows * 2 * sizeof(float));
  p->items_at = p->o_at + up256(part_rows * dp * sizeof(float));
  p->joins_at = p->items_at + up256((size_t)p->slots * 16);
  p->pieces_at = p->joins_at + up256((size_t)(cut + 1) * 16);
  p->bytes = p->blocks ? p->pieces_at + up256(most * 16) : 0;
  return ARGUS_OK;
}

}  // namespace
}  // namespace prompt
}  // namespace argus

using namespace argus;
using namespace argus::prompt;

extern "C" size_t argus_prompt_attend_workspace_bytes(const argus_chunk_config* cfg) {
  accepted();
  Plan p;
  return make_plan(cfg, &p) == ARGUS_OK ? p.bytes : (size_t)-1;
}

extern "C" int argus_prompt_attend(const argus_chunk_config* cfg, const argus_chunk_io* io, void* d_workspace,
                                   size_t workspace_bytes, argus_markers* markers, void* stream_v) {
  accepted();
  Plan p;
  int rc = make_plan(cfg, &p);
  if (rc != ARGUS_OK) return rc;
  if (!io || (cfg->seqs && (!io->d_table || !io->d_lens || !io->d_offsets)) || (cfg->seqs && cfg->rows && (!io->d_q || !io->d_out)))
    return refuse(ARGUS_E_INVAL, "a required pointer is NULL");
  if ((rc = check_view(io->k, cfg->cache_type, "k")) != ARGUS_OK || (rc = check_view(io->v, cfg->cache_type, "v")) != ARGUS_OK)
    return rc;
  for (const argus_page_view* w : {&io->k, &io->v})
    if (w->page_stride < 0 || w->page_stride > (int64_t)(1ll << 35) || w->token_stride < 0 ||
        w->token_stride * (int64_t)cfg->page_size > 0x3FFFFFFFll)
      return refuse(ARGUS_E_CAPACITY, "a page's stride, or its tokens' times page_size, is out of range");
  if (!aligned_to(io->d_q, 16) || io->q_row_stride % 8 || io->q_head_stride % 8 || !aligned_to(io->d_out, 16) ||
      !aligned_to(io->d_table, 4) || !aligned_to(io->d_lens, 4) || !aligned_to(io->d_offsets, 4) ||
      !aligned_to(io->d_k_scale, 4) || !aligned_to(io->d_v_scale, 4) || !aligned_to(io->d_lse, 4))
    return refuse(ARGUS_E_ALIGN, "rows of q and out lie on 16 bytes");
  if (io->table_stride < (int64_t)cfg->columns && cfg->seqs > 1)
    return refuse(ARGUS_E_INVAL, "table_stride %lld below columns", (long long)io->table_stride);
  if (marks_bad_all(markers)) return refuse(ARGUS_E_INVAL, "markers: alignment or region_base");
  if (p.bytes && !d_workspace) return refuse(ARGUS_E_INVAL, "no workspace");
  if (p.bytes && !aligned_to(d_workspace, 256)) return refuse(ARGUS_E_ALIGN, "the workspace lies on 256 bytes");
  if (workspace_bytes < p.bytes)
    return refuse(ARGUS_E_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, p.bytes);
  const uint64_t plans = p.blocks ? kPlanThreads / kThreads : 0, waves = p.tile_shift == 8 ? 2 : 1;
  const uint64_t records = (p.grid * waves + plans + (uint64_t)p.joins * kJoinBlocks) * 2 * kWaves;
  if (!marks_fit(markers, records)) return refuse(ARGUS_E_CAPACITY, "%llu marker records do not fit", (unsigned long long)records);
  if (cfg->seqs == 0 || cfg->rows == 0) return ARGUS_OK;
  if ((rc = device_ok()) != ARGUS_OK) return rc;

  ChunkArgs a{};
  const int64_t e = type_bytes(cfg->cache_type);
  a.q = (const uint16_t*)io->d_q;
  a.q_row = io->q_row_stride, a.q_head = io->q_head_stride;
  a.k = (const uint8_t*)io->k.base, a.v = (const uint8_t*)io->v.base;
  a.k_page = io->k.page_stride * e, a.k_head = io->k.head_stride * e, a.k_tok = (uint32_t)(io->k.token_stride * e);
  a.v_page = io->v.page_stride * e, a.v_head = io->v.head_stride * e, a.v_tok = (uint32_t)(io->v.token_stride * e);
  a.table = io->d_table, a.table_stride = io->table_stride, a.lens = io->d_lens, a.offsets = io->d_offsets;
  a.k_scale = io->d_k_scale, a.v_scale = io->d_v_scale;
  a.out = (uint16_t*)io->d_out, a.lse = io->d_lse;
  a.S = cfg->seqs, a.rows = cfg->rows, a.H = cfg->kv_heads, a.G = cfg->group, a.D = cfg->head_dim;
  a.slots = p.slots, a.tile_shift = p.tile_shift, a.step_shift = cfg->head_dim > 128 ? 5 : 6;
  a.shift = log2_of(cfg->page_size), a.num_pages = cfg->num_pages, a.columns = cfg->columns;
  a.window = cfg->window, a.sinks = cfg->sinks;
  a.by_group = fast_div(cfg->group);
  a.scale = cfg->scale;
  hipStream_t st = (hipStream_t)stream_v;
  a.blocks = p.blocks;
  if (p.blocks) {
    char* ws = (char*)d_workspace;
    a.head = (uint64_t*)ws;
    a.part_ml = (float*)(ws + p.ml_at), a.part_o = (float*)(ws + p.o_at);
    a.items = (uint4*)(ws + p.items_at), a.joins = (uint4*)(ws + p.joins_at), a.pieces = (uint4*)(ws + p.pieces_at);
    a.marks = take_marks(markers, plans, 2);
    hipLaunchKernelGGL(k_chunk_plan, dim3(1), dim3(kPlanThreads), 0, st, a);
  }
  a.marks = take_marks(markers, p.grid * waves, 2);
  const bool f8 = cfg->cache_type == ARGUS_FP8, bf = cfg->q_type == ARGUS_BF16;
  (f8 ? (bf ? launch_chunk_bf16_f8 : launch_chunk_fp16_f8) : (bf ? launch_chunk_bf16 : launch_chunk_fp16))(a, p.grid, st);
  if (p.joins) {
    a.marks = take_marks(markers, (uint64_t)p.joins * kJoinBlocks, 2);
    (bf ? launch_chunk_join<0> : launch_chunk_join<1>)(a, dim3(p.joins, kJoinBlocks), st);
  }
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}
