// k_chunk.hip -- attention of chunks of new tokens (k_chunk.h): the host's side, the batch shared out,
// and the pieces joined.
#include "k_chunk.h"

namespace argus {
namespace prompt {
namespace {

// The shares of a batch, by one block. Units are steps, and kPieceCost more for each row tile,
// of all row tiles one after the other, of one head after the other; share i has units i * per and on.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
__global__ __launch_bounds__(kPlanThreads) void k_chunk_plan(ChunkArgs a) {
  __shared__ uint64_t s_units[kPlanWaves];
  __shared__ uint32_t s_items[kPlanWaves];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_CHUNK_PLAN);
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
  uint64_t units = 0;  // of all slots before
  uint32_t items = 0;
  for (uint32_t x0 = 0; x0 < a.slots; x0 += kPlanThreads) {
    const uint32_t x = x0 + tid;
    Reach g;
    bool real = false;
    uint32_t s = 0, first = 0, mine = 0;
    if (x < a.slots) {
      uint32_t hi = a.S;
      while (hi - s > 1) {  // the last sequence whose slots start at or before x
        const uint32_t mid = (s + hi) / 2;
        if (slot_of(a, mid) <= x) s = mid; else hi = mid;
      }
      first = slot_of(a, s);
      real = first <= x && reach_of(a, s, x - first, &g);
      if (real) mine = g.steps + kPieceCost;
    }
    // (64 lanes of at most 2^26 units each)
    uint64_t incl = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const uint64_t o = __shfl_up(incl, d);
      if ((int)lane >= d) incl += o;
    }
    const uint64_t there = __ballot(real);
    if (lane == 63) s_units[wave] = incl, s_items[wave] = (uint32_t)__popcll(there);
    __syncthreads();
    uint64_t before = units;
    uint32_t at = items;
    for (uint32_t w = 0; w < (uint32_t)kPlanWaves; ++w) {
      if (w < wave) before += s_units[w], at += s_items[w];
      units += s_units[w], items += s_items[w];
    }
    if (real) {
      at += (uint32_t)__popcll(there & lanemask_lt());
      a.items[at] = make_uint2(s, x - first);
      a.cum[at] = before + incl - mine;
    }
    __syncthreads();
  }
  uint64_t per = (units * a.H + a.shares - 1) / a.shares;
  per = per < kMinShare ? kMinShare : per;
  if (tid == 0) {
    a.cum[items] = units;
    a.head[0] = units, a.head[1] = per, a.head[2] = items;
  }
  __syncthreads();
  for (uint32_t i = tid; i < a.shares; i += kPlanThreads) {
    const uint64_t u = i * per;
    if (u >= units * a.H) {
      a.start[i] = make_uint4(0u, 0u, 0u, 0u);
      continue;
    }
    const uint32_t h = (uint32_t)(u / units);
    const uint64_t r = u - h * units;
    uint32_t lo = 0, hi = items;
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (a.cum[mid] <= r) lo = mid; else hi = mid;
    }
    const uint64_t left = units * a.H - u;
    a.start[i] = make_uint4(lo, h, (uint32_t)(r - a.cum[lo]), (uint32_t)(left < per ? left : per));
  }
  mk.end(ARGUS_REGION_CHUNK_PLAN);
}

// Rows of a row tile that was left in pieces: piece 0 is the second of its first share, piece i the
// first of share i further on.
template <int T, int DP, int W>
__global__ __launch_bounds__(kThreads) void k_chunk_join(ChunkArgs a) {
  constexpr uint32_t kQuads = DP / 4, kRows = kThreads / kQuads, TR = 32 * W;
  using Hf = Half<T>;
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_CHUNK_JOIN);
  const uint4 open = a.open[blockIdx.x];
  Reach g;
  if (open.w && blockIdx.y * kRows < TR) {
    const uint2 item = a.items[open.x];
    const uint32_t h = open.y, n = open.z - blockIdx.x + 1;
    const uint32_t mine = blockIdx.y * kRows + threadIdx.x / kQuads, d = threadIdx.x % kQuads * 4;
    if (reach_of(a, item.x, item.y, &g) && mine < g.rows) {
      float m = -INFINITY, l = 0.0f;
      f32x4 o = (f32x4)(0.0f);
      constexpr uint32_t kDeep = 8;
      for (uint32_t i0 = 0; i0 < n; i0 += kDeep) {
        f32x2 ml[kDeep];
        f32x4 v[kDeep];
        float top = m;
#pragma unroll
        for (uint32_t j = 0; j < kDeep; ++j) {
          const uint32_t i = i0 + j < n ? i0 + j : 0;
          const uint64_t x = (2ull * (blockIdx.x + i) + (i == 0 ? 1u : 0u)) * TR + mine;
          ml[j] = *reinterpret_cast<const f32x2*>(a.part_ml + 2 * x);
          v[j] = *reinterpret_cast<const f32x4*>(a.part_o + x * DP + d);
          if (i0 + j >= n) ml[j] = (f32x2){-INFINITY, 0.0f}, v[j] = (f32x4)(0.0f);
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
      const uint32_t r = g.r0 + mine, tok = divide(r, a.by_group);
      const uint64_t row = (uint64_t)(g.row0 + tok) * a.H * a.G + h * a.G + (r - tok * a.G);
      const float inv = l == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[h] : 1.0f) / l;
      if (d < a.D)
        *reinterpret_cast<u32x2*>(a.out + row * a.D + d) = (u32x2){Hf::pack(o.x * inv, o.y * inv), Hf::pack(o.z * inv, o.w * inv)};
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
    if (eight) hipLaunchKernelGGL((k_chunk_join<T, 64, 8>), g, b, 0, st, a);
    else hipLaunchKernelGGL((k_chunk_join<T, 64, 4>), g, b, 0, st, a);
  } else if (a.D <= 128) {
    if (eight) hipLaunchKernelGGL((k_chunk_join<T, 128, 8>), g, b, 0, st, a);
    else hipLaunchKernelGGL((k_chunk_join<T, 128, 4>), g, b, 0, st, a);
  } else {
    hipLaunchKernelGGL((k_chunk_join<T, 256, 4>), g, b, 0, st, a);
  }
}


// Blocks that share a batch: as many as run at once, two on a compute unit (one at head sizes
// beyond 128).
uint32_t share_count(uint32_t tile_shift, uint32_t head_dim) { return head_dim > 128 || tile_shift == 8 ? 256u : 512u; }
constexpr uint32_t kWholeSteps = 8;

struct Plan {
  uint32_t tile_shift, slots, grid, shares, joins, join_rows;
  size_t ml_at, o_at, open_at, start_at, items_at, cum_at, bytes;
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
  p->tile_shift = c->head_dim > 128 ? 7 : 8;
  p->slots = c->seqs ? ((c->rows * c->group) >> p->tile_shift) + c->seqs : 0;
  const uint64_t tiles = (uint64_t)p->slots * c->kv_heads;
  const uint32_t kt = c->head_dim > 128 ? 32 : 64, dp = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
  // steps of a row tile, as far as the table (or the window) allows
  uint64_t steps = ((uint64_t)c->columns * c->page_size + kt - 1) / kt;
  if (c->window) {
    const uint64_t w = (c->window + (1u << p->tile_shift) / c->group + 2 * kt) / kt + 1 + (c->sinks + kt - 1) / kt;
    steps = w < steps ? w : steps;
  }
  p->shares = 0;
  if (tiles && c->rows && (steps > kWholeSteps || tiles > kMaxBlocks)) {
    // (units of a share are counted in 32 bits)
    if (tiles * (steps + kPieceCost) >= 1ull << 40) return refuse(ARGUS_E_CAPACITY, "rows x heads x tokens");
    const uint64_t useful = tiles * (steps + kPieceCost) / kMinShare + 1;
    p->shares = share_count(p->tile_shift, c->head_dim);
    p->shares = useful < p->shares ? (uint32_t)useful : p->shares;
  }
  p->grid = p->shares ? p->shares : (uint32_t)tiles;
  p->join_rows = (1u << p->tile_shift) * dp / 4 / kThreads;
  p->joins = p->shares * p->join_rows;
  const size_t rows = (size_t)p->shares * 2 << p->tile_shift;
  p->ml_at = 256;
  p->o_at = p->ml_at + up256(rows * 2 * sizeof(float));
  p->open_at = p->o_at + up256(rows * dp * sizeof(float));
  p->start_at = p->open_at + up256((size_t)p->shares * 16);
  p->items_at = p->start_at + up256((size_t)p->shares * 16);
  p->cum_at = p->items_at + up256((size_t)p->slots * 8);
  p->bytes = p->shares ? p->cum_at + up256(((size_t)p->slots + 1) * 8) : 0;
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
  const uint64_t plans = p.shares ? kPlanThreads / kThreads : 0;
  const uint64_t records = (p.grid + plans + p.joins) * 2 * kWaves;
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
  a.shares = p.shares;
  if (p.shares) {
    char* ws = (char*)d_workspace;
    a.head = (uint64_t*)ws;
    a.part_ml = (float*)(ws + p.ml_at), a.part_o = (float*)(ws + p.o_at);
    a.open = (uint4*)(ws + p.open_at), a.start = (uint4*)(ws + p.start_at);
    a.items = (uint2*)(ws + p.items_at), a.cum = (uint64_t*)(ws + p.cum_at);
    a.marks = take_marks(markers, plans, 2);
    hipLaunchKernelGGL(k_chunk_plan, dim3(1), dim3(kPlanThreads), 0, st, a);
  }
  a.marks = take_marks(markers, p.grid, 2);
  const bool f8 = cfg->cache_type == ARGUS_FP8, bf = cfg->q_type == ARGUS_BF16;
  (f8 ? (bf ? launch_chunk_bf16_f8 : launch_chunk_fp16_f8) : (bf ? launch_chunk_bf16 : launch_chunk_fp16))(a, p.grid, st);
  if (p.shares) {
    a.marks = take_marks(markers, p.joins, 2);
    (bf ? launch_chunk_join<0> : launch_chunk_join<1>)(a, dim3(p.shares, p.join_rows), st);
  }
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}
