// k_attend.hip -- host side of the attention of one new token over a paged
// cache (k_attend.h), and the error text and device check of all operators.
#include <atomic>

#include "k_attend.h"

namespace argus {
namespace decode {

namespace {
thread_local char g_why[256];
std::atomic<unsigned char> g_dev_ok[64];
}  // namespace

int refuse(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_why, sizeof(g_why), fmt, ap);
  va_end(ap);
  return code;
}
void accepted() { g_why[0] = 0; }

int device_ok() {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return refuse(ARGUS_E_HIP, "no device");
  if (dev < 0 || dev >= 64) return refuse(ARGUS_E_DEVICE, "device %d", dev);
  if (!g_dev_ok[dev].load(std::memory_order_relaxed)) {
    hipDeviceProp_t prop;
    if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return refuse(ARGUS_E_HIP, "no device properties");
    if (strncmp(prop.gcnArchName, "gfx950", 6) != 0) return refuse(ARGUS_E_DEVICE, "the device is no gfx950");
    g_dev_ok[dev].store(1, std::memory_order_relaxed);
  }
  return ARGUS_OK;
}

namespace {

// Waves that share a batch: one block of four for each of the 256 compute
// units (twice as many: 650 us against 640 for four sequences of 262143 tokens, 72
// against 68 for the 8-bit batch).  All of them may
// fall to one segment (one of 131072 tokens, 1 x 8 heads of 128: 24 us, with at most 512 27,
// with 256 34).  Two blocks where a tile's rows are so short
// that one wave for each SIMD has too few bytes under way: of 64 bytes (64 sequences of up to
// 16384 tokens in 8 bits: 36 us against 41; of 128 bytes 49.7 against 48.1).
constexpr uint32_t kShares = 256 * kWaves, kSharesOfSegment = 1024;
// A block of the join takes 32 elements of a row where segments may lie in so many pieces
// (the join of a sequence in 66 pieces, 1 x 8 heads of 128, takes 3.9 us by parts and by whole
// rows, in 98 pieces 4.0 against 5.1, in 258 3.9 against 7.0, in 1024 7.8 against 18.1); a
// row where there are so few of them (6 sequences of up to 3111, 8 x 4 heads: 15.8 us a call
// against 16.7 by four rows), else four (10 of 8502 with a window of 1060, 2 x 24 heads: 18.3
// us against 19.4 by one row).
constexpr uint32_t kManyPieces = 64, kFewRows = 256;
// Segments of at most this many tiles are not shared: a block each, and no joining
// (64 sequences of 512 tokens, 8 x 4 heads of 128: 24 us against 30 shared; of 1024 tokens 44
// against 50, and 4 of them 14.8 against 15.3; at head size 256, 4 of 512 18.7 against 23.1,
// 4 of 1024 33 against 25).
uint32_t whole_tiles(uint32_t dp) { return dp == 256 ? 16u : 32u; }

struct Plan {
  uint32_t dp, nq, row_tiles, hs, shares, segs, grid, opens, unit_shift;
  JoinForm join;
  uint32_t join_y, join_z;
  size_t o_at, open_at, bytes;
};

int make_plan(const argus_attend_config* c, Plan* p) {
  if (!c) return refuse(ARGUS_E_INVAL, "no configuration");
  if (c->abi_version != ARGUS_ATTR_ABI_VERSION) return refuse(ARGUS_E_ABI, "abi_version %u", c->abi_version);
  if (c->q_type > ARGUS_FP16) return refuse(ARGUS_E_INVAL, "q is bf16 or fp16");
  if (c->cache_type != c->q_type && c->cache_type != ARGUS_FP8)
    return refuse(ARGUS_E_INVAL, "the cache is of q's type or fp8 (e4m3)");
  if (c->seqs > (1u << 20)) return refuse(ARGUS_E_CAPACITY, "seqs %u", c->seqs);
  if (c->kv_heads < 1 || c->kv_heads > 1024 || c->group < 1 || c->group > 256)
    return refuse(ARGUS_E_INVAL, "kv_heads %u (1..1024), group %u (1..256)", c->kv_heads, c->group);
  const uint32_t unit = c->head_dim > 128 || c->cache_type == ARGUS_FP8 ? 16u : 8u;
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % unit)
    return refuse(ARGUS_E_INVAL, "head_dim %u: a multiple of %u up to 256", c->head_dim, unit);
  if (!power_of_two(c->page_size) || c->page_size < 8 || c->page_size > 65536)
    return refuse(ARGUS_E_INVAL, "page_size %u: a power of two, 8..65536", c->page_size);
  if (c->num_pages < 1 || c->num_pages > 0x7FFFFFFFu || c->columns < 1 ||
      (uint64_t)c->columns * c->page_size > 0x7FFFFFFFull || c->window > 0x7FFFFFFFu || c->sinks > 0x7FFFFFFFu)
    return refuse(ARGUS_E_CAPACITY, "pages, columns, window or sinks out of range");
  p->dp = c->head_dim <= 64 ? 64u : c->head_dim <= 128 ? 128u : 256u;
  p->nq = c->group > 16 ? 2u : 1u;
  p->row_tiles = (c->group + 16 * p->nq - 1) / (16 * p->nq);
  p->hs = c->kv_heads * p->row_tiles;
  const uint64_t segs = (uint64_t)c->seqs * p->hs;
  if (segs > (1u << 30)) return refuse(ARGUS_E_CAPACITY, "seqs x heads");
  // tiles of the longest sequence that the table (or the window) allows
  uint64_t tiles = ((uint64_t)c->columns * c->page_size + kTile - 1) / kTile;
  if (c->window) {
    const uint64_t w = (c->window + kTile - 1) / kTile + 1 + (uint64_t)(c->sinks + kTile - 1) / kTile;
    tiles = w < tiles ? w : tiles;
  }
  p->segs = (uint32_t)segs;
  p->unit_shift = 0;
  while (segs * (((tiles + kPieceCost) >> p->unit_shift) + 1) >= (1ull << 31)) ++p->unit_shift;
  uint64_t shares = 0;
  if ((tiles > whole_tiles(p->dp) || segs > kMaxBlocks) && segs) {
    shares = p->dp * type_bytes(c->cache_type) <= 64 ? 2 * kShares : kShares;
    shares = segs * kSharesOfSegment < shares ? segs * kSharesOfSegment : shares;
    const uint64_t useful = segs * (tiles + kPieceCost) / kMinShare + 1;
    shares = useful < shares ? useful : shares;
    shares = (shares + kWaves - 1) / kWaves * kWaves;
  }
  p->shares = (uint32_t)shares;
  p->grid = shares ? p->shares / kWaves : p->segs;
  p->opens = p->shares < p->segs ? p->shares : p->segs;
  const uint32_t join_rows = c->group < 16 * p->nq ? c->group : 16 * p->nq;
  p->join = p->shares >= (uint64_t)p->segs * kManyPieces ? kJoinPart : p->opens * join_rows <= kFewRows ? kJoinRow : kJoinFourRows;
  p->join_y = p->join == kJoinFourRows ? (join_rows + 3) / 4 : join_rows;
  p->join_z = p->join == kJoinPart ? (c->head_dim + kJoinCols - 1) / kJoinCols : 1;
  const size_t rows = (size_t)shares * 2 * 16 * p->nq;
  p->o_at = up256(rows * 2 * sizeof(float));
  p->open_at = p->o_at + up256(rows * p->dp * sizeof(float));
  p->bytes = shares ? p->open_at + up256((size_t)p->opens * 16) : 0;
  return ARGUS_OK;
}

}  // namespace
}  // namespace decode
}  // namespace argus

using namespace argus;
using namespace argus::decode;

extern "C" const char* argus_decode_last_error(void) { return g_why; }

extern "C" size_t argus_decode_attend_workspace_bytes(const argus_attend_config* cfg) {
  accepted();
  Plan p;
  return make_plan(cfg, &p) == ARGUS_OK ? p.bytes : (size_t)-1;
}

extern "C" int argus_decode_attend(const argus_attend_config* cfg, const argus_attend_io* io, void* d_workspace,
                                   size_t workspace_bytes, argus_markers* markers, void* stream_v) {
  accepted();
  Plan p;
  int rc = make_plan(cfg, &p);
  if (rc != ARGUS_OK) return rc;
  if (!io || (cfg->seqs && (!io->d_table || !io->d_q || !io->d_lens || !io->d_out)))
    return refuse(ARGUS_E_INVAL, "a required pointer is NULL");
  if ((rc = check_view(io->k, cfg->cache_type, "k")) != ARGUS_OK || (rc = check_view(io->v, cfg->cache_type, "v")) != ARGUS_OK)
    return rc;
  for (const argus_page_view* w : {&io->k, &io->v})
    if (w->page_stride < 0 || w->page_stride > (int64_t)(1ll << 35) || w->token_stride < 0 ||
        w->token_stride * (int64_t)cfg->page_size > 0x3FFFFFFFll)
      return refuse(ARGUS_E_CAPACITY, "a page's stride, or its tokens' times page_size, is out of range");
  if (!aligned_to(io->d_q, 16) || io->q_seq_stride % 8 || io->q_head_stride % 8 || !aligned_to(io->d_out, 16) ||
      !aligned_to(io->d_table, 4) || !aligned_to(io->d_lens, 4) || !aligned_to(io->d_k_scale, 4) ||
      !aligned_to(io->d_v_scale, 4) || !aligned_to(io->d_lse, 4))
    return refuse(ARGUS_E_ALIGN, "rows of q and out lie on 16 bytes");
  if (io->table_stride < (int64_t)cfg->columns && cfg->seqs > 1)
    return refuse(ARGUS_E_INVAL, "table_stride %lld below columns", (long long)io->table_stride);
  if (marks_bad(markers)) return refuse(ARGUS_E_INVAL, "markers: alignment or region_base");
  if (p.bytes && !d_workspace) return refuse(ARGUS_E_INVAL, "no workspace");
  if (p.bytes && !aligned_to(d_workspace, 256)) return refuse(ARGUS_E_ALIGN, "the workspace lies on 256 bytes");
  if (workspace_bytes < p.bytes)
    return refuse(ARGUS_E_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, p.bytes);
  const uint64_t joins = p.shares ? (uint64_t)p.opens * p.join_y * p.join_z : 0;
  const uint32_t per_wave = 6;  // its own region, and in it the place and the tokens
  const uint64_t records = ((uint64_t)p.grid * per_wave + joins * 2) * kWaves;
  if (!marks_fit(markers, records)) return refuse(ARGUS_E_CAPACITY, "%llu marker records do not fit", (unsigned long long)records);
  if (cfg->seqs == 0) return ARGUS_OK;
  if ((rc = device_ok()) != ARGUS_OK) return rc;

  AttendArgs a{};
  const int64_t e = type_bytes(cfg->cache_type);
  a.q = (const uint16_t*)io->d_q;
  a.q_seq = io->q_seq_stride, a.q_head = io->q_head_stride;
  a.k = (const uint8_t*)io->k.base, a.v = (const uint8_t*)io->v.base;
  a.k_page = io->k.page_stride * e, a.k_head = io->k.head_stride * e, a.k_tok = (uint32_t)(io->k.token_stride * e);
  a.v_page = io->v.page_stride * e, a.v_head = io->v.head_stride * e, a.v_tok = (uint32_t)(io->v.token_stride * e);
  a.table = io->d_table, a.table_stride = io->table_stride, a.lens = io->d_lens;
  a.k_scale = io->d_k_scale, a.v_scale = io->d_v_scale;
  a.out = (uint16_t*)io->d_out, a.lse = io->d_lse;
  a.part_ml = (float*)d_workspace;
  a.part_o = (float*)((char*)d_workspace + p.o_at);
  a.open = (uint4*)((char*)d_workspace + p.open_at);
  a.S = cfg->seqs, a.H = cfg->kv_heads, a.G = cfg->group, a.D = cfg->head_dim;
  a.HS = p.hs, a.row_tiles = p.row_tiles;
  a.shift = log2_of(cfg->page_size), a.num_pages = cfg->num_pages, a.columns = cfg->columns;
  a.window = cfg->window, a.sinks = cfg->sinks;
  a.unit_shift = p.unit_shift;
  a.shares = p.shares, a.by_seg = p.segs <= p.shares, a.scale = cfg->scale;
  a.marks = take_marks(markers, p.grid, per_wave);
  hipStream_t st = (hipStream_t)stream_v;
  const bool f8 = cfg->cache_type == ARGUS_FP8, bf = cfg->q_type == ARGUS_BF16;
  (f8 ? (bf ? launch_attend_bf16_f8 : launch_attend_fp16_f8) : (bf ? launch_attend_bf16 : launch_attend_fp16))(a, p.grid, st);
  if (p.shares) {
    a.marks = take_marks(markers, joins, 2);
    (bf ? launch_join_type<0> : launch_join_type<1>)(a, p.join, dim3(p.opens, p.join_y, p.join_z), st);
  }
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}
