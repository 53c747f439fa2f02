// k_chunk.hip -- host side of the attention of chunks of new tokens (k_chunk.h).
#include "k_chunk.h"

namespace argus {
namespace prompt {
namespace {

constexpr uint32_t kTileShift = 7;  // rows of a tile: 32 for each of a block's waves

struct Plan {
  uint32_t slots, grid;
  size_t bytes;
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
  p->slots = c->seqs ? ((c->rows * c->group) >> kTileShift) + c->seqs : 0;
  const uint64_t grid = (uint64_t)p->slots * c->kv_heads;
  if (grid > kMaxBlocks) return refuse(ARGUS_E_CAPACITY, "rows x heads");
  p->grid = (uint32_t)grid;
  p->bytes = 0;
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
  const uint64_t records = (uint64_t)p.grid * 2 * kWaves;
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
  a.slots = p.slots, a.tile_shift = kTileShift, a.step_shift = cfg->head_dim > 128 ? 5 : 6;
  a.shift = log2_of(cfg->page_size), a.num_pages = cfg->num_pages, a.columns = cfg->columns;
  a.window = cfg->window, a.sinks = cfg->sinks;
  a.by_group = fast_div(cfg->group);
  a.scale = cfg->scale;
  a.marks = take_marks(markers, p.grid, 2);
  hipStream_t st = (hipStream_t)stream_v;
  const bool f8 = cfg->cache_type == ARGUS_FP8, bf = cfg->q_type == ARGUS_BF16;
  (f8 ? (bf ? launch_chunk_bf16_f8 : launch_chunk_fp16_f8) : (bf ? launch_chunk_bf16 : launch_chunk_fp16))(a, p.grid, st);
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}
