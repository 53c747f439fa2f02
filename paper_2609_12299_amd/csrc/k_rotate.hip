// k_rotate.hip -- rotary positions: queries turned, keys turned on their way into the
// pages, values beside them.
//
// A block takes a few rows. It finds their places and their angles' cosines and sines once, in
// LDS: the angle p f in turns, in 64 bits, of which only the part after the point goes on
// (at position 10^6 an angle of 32 bits would be off by 0.06); all heads of a row use them. Then its threads
// go over the rows' units: a unit of queries or keys is eight pairs, whose 16 elements one thread reads,
// turns and writes (so q may be turned in place), or eight elements that stay; one of values
// is eight elements. (Four pairs a unit where their number is odd in fours: 32768 rows of 16 + 4 heads of 80,
// 20 pairs each, 72 us against 201 pair by pair.)
//
// What bounds it: the bytes, read and written once: 65537 rows of 24 + 8 heads of 96 in 209 us, 4.8 TB/s, as
// fast as a copy; a step of 64 single tokens, 32 + 8 heads of 128, 4.1 us, of a call's 10, which are the host's.
#include "pages.h"
#include "prompt.h"

namespace argus {
namespace prompt {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// How a head's pairs lie: neighbours, or eight and eight of them in whole vectors, four and four in halves of
// vectors, or anyhow.
enum Layout { kNeighbours, kHalves, kFours, kAnyHalves };

struct RotateArgs {
  const uint8_t* q;
  uint8_t* out;
  const uint8_t *new_k, *new_v;
  int64_t q_row, q_hd, out_row, out_hd, k_row, k_hd, v_row, v_hd;  // bytes
  uint8_t *k, *v;
  int64_t k_page, k_head, k_tok, v_page, v_head, v_tok;
  const int32_t* table;
  int64_t table_stride;
  const int32_t *starts, *offsets;
  const double* frequencies;
  const float *k_scale, *v_scale;
  uint32_t S, rows, shift, num_pages, columns, tokens;  // tokens of a block
  uint32_t D, pairs, heads, kv_heads;
  uint32_t turned;  // units of a head, pairs first, that are pairs
  FastDiv per_token, per_head, per_value, by_pairs;  // units of a token, of a turned head, of a head's values
  float amplitude;
  Marks marks;
};

constexpr uint32_t kMaxTokens = 4, kMaxPairs = 128;

template <int T>
ARGUS_DEV float of_half(uint16_t x) {
  if constexpr (T == 0) return __builtin_bit_cast(float, (uint32_t)x << 16);
  else return (float)__builtin_bit_cast(_Float16, x);
}
template <int T>
ARGUS_DEV uint32_t pack(float x, float y) {
  if constexpr (T == 0) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, bf16x2));
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, f16x2));
  }
}
// Eight numbers as they go into a cache of 8 bits.
ARGUS_DEV u32x2 narrow(const float (&x)[8], float sc) {
  float y[8], inv = 1.0f / sc;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i];
  if (!ordinary(sc)) {  // divided here, and by 1 below
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] / sc;
    sc = inv = 1.0f;
  }
  u32x2 out;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(y[4 * i], sc, inv), quotient(y[4 * i + 1], sc, inv), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(y[4 * i + 2], sc, inv), quotient(y[4 * i + 3], sc, inv), w, true);
    out[i] = (uint32_t)w;
  }
  return out;
}

template <int T>
ARGUS_DEV void spread(u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 p = pair<T>(w[i]);
    x[2 * i] = p.x, x[2 * i + 1] = p.y;
  }
}
template <int T>
ARGUS_DEV u32x4 gather(const float (&x)[8]) {
  return (u32x4){pack<T>(x[0], x[1]), pack<T>(x[2], x[3]), pack<T>(x[4], x[5]), pack<T>(x[6], x[7])};
}

template <int T, bool F8, int LAYOUT>
__global__ __launch_bounds__(kThreads) void k_rotate(RotateArgs a) {
  // Neighbours: what a wave reads and writes at once are whole lines of 128 bytes, which go past the caches (40 prompts
  // of up to 8192 tokens into 8 bits 186 us against 195). Halves: parts of lines, whose rest comes next
  // (65537 rows of 24 + 8 heads of 96 209 us against 226).
  constexpr bool kOnce = LAYOUT == kNeighbours;
  __shared__ int64_t s_page[kMaxTokens];  // -1: not held
  __shared__ uint32_t s_place[kMaxTokens];
  __shared__ int64_t s_pos[kMaxTokens];
  __shared__ uint32_t s_in[kMaxTokens];
  __shared__ float2 s_turn[kMaxTokens * kMaxPairs];
  WaveMarks mk(a.marks);
  mk.begin(ARGUS_REGION_ROTATE);
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
      // (an offset outside [0, rows] is the nearer end: the comparisons come to the same without a look at that)
      const int32_t first = a.offsets[s];
      pos = in ? (int64_t)a.starts[s] + row - (first < 0 ? 0 : first) : 0;
    } else {
      pos = a.starts[s];
    }
    s_in[tid] = in;
    s_pos[tid] = pos;
    int32_t page = -1;
    if (a.kv_heads && in && pos >= 0 && (uint64_t)pos >> a.shift < a.columns)
      page = a.table[(int64_t)s * a.table_stride + (pos >> a.shift)];
    s_page[tid] = (uint32_t)page < a.num_pages ? page : -1;
    s_place[tid] = (uint32_t)pos & ((1u << a.shift) - 1);
  }
  __syncthreads();
  for (uint32_t i = tid; i < tokens * a.pairs; i += kThreads) {
    const uint32_t t = divide(i, a.by_pairs);
    const double turns = (double)s_pos[t] * a.frequencies[i - t * a.pairs] * 0.15915494309189533577;
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    s_turn[i] = make_float2(c * a.amplitude, s * a.amplitude);
  }
  __syncthreads();
  const uint32_t n = tokens * a.per_token.d, turned_units = (a.heads + a.kv_heads) * a.per_head.d;
  for (uint32_t e = tid; e < n; e += kThreads) {
    const uint32_t t = divide(e, a.per_token);
    uint32_t x = e - t * a.per_token.d;
    if (!s_in[t]) continue;
    const int64_t page = s_page[t], row = row0 + t;
    if (x >= turned_units) {  // values
      x -= turned_units;
      const uint32_t h = divide(x, a.per_value), d = (x - h * a.per_value.d) * 8;
      if (page < 0) continue;
      const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.new_v + row * a.v_row + (int64_t)h * a.v_hd + 2 * d));
      uint8_t* to = a.v + page * a.v_page + (int64_t)h * a.v_head + (int64_t)s_place[t] * a.v_tok;
      if constexpr (F8) {
        float y[8];
        spread<T>(w, y);
        __builtin_nontemporal_store(narrow(y, a.v_scale ? a.v_scale[h] : 1.0f), reinterpret_cast<u32x2*>(to + d));
      } else {
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(to + 2 * d));
      }
      continue;
    }
    uint32_t h = divide(x, a.per_head);
    const uint32_t u = x - h * a.per_head.d;
    const bool query = h < a.heads;
    const uint8_t* from;
    uint8_t* to;
    float scale = 1.0f;
    if (query) {
      from = a.q + row * a.q_row + (int64_t)h * a.q_hd;
      to = a.out + row * a.out_row + (int64_t)h * a.out_hd;
    } else {
      h -= a.heads;
      if (page < 0) continue;
      from = a.new_k + row * a.k_row + (int64_t)h * a.k_hd;
      to = a.k + page * a.k_page + (int64_t)h * a.k_head + (int64_t)s_place[t] * a.k_tok;
      if (a.k_scale) scale = a.k_scale[h];
    }
    const bool f8 = F8 && !query;
    auto store = [&](uint32_t d, const float (&y)[8]) {
      if (f8) __builtin_nontemporal_store(narrow(y, scale), reinterpret_cast<u32x2*>(to + d));
      else if constexpr (kOnce) __builtin_nontemporal_store(gather<T>(y), reinterpret_cast<u32x4*>(to + 2 * d));
      else *reinterpret_cast<u32x4*>(to + 2 * d) = gather<T>(y);
    };
    auto load = [&](uint32_t d, float (&y)[8]) {
      const u32x4* at = reinterpret_cast<const u32x4*>(from + 2 * d);
      if constexpr (kOnce) spread<T>(__builtin_nontemporal_load(at), y);
      else spread<T>(*at, y);
    };
    const float2* turn = s_turn + t * a.pairs;
    if constexpr (LAYOUT == kNeighbours) {
      float y[8];
      load(8 * u, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t p = 4 * u + i;
        if (p < a.pairs) {
          const float2 w = turn[p];
          const float y0 = y[2 * i] * w.x - y[2 * i + 1] * w.y;
          y[2 * i + 1] = y[2 * i + 1] * w.x + y[2 * i] * w.y;
          y[2 * i] = y0;
        }
      }
      store(8 * u, y);
    } else if constexpr (LAYOUT == kHalves) {
      float y[8];
      if (u >= a.turned) {  // elements that stay
        const uint32_t d = 2 * a.pairs + 8 * (u - a.turned);
        load(d, y);
        store(d, y);
        continue;
      }
      float z[8];
      load(8 * u, y);
      load(a.pairs + 8 * u, z);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 w = turn[8 * u + i];
        const float y0 = y[i] * w.x - z[i] * w.y;
        z[i] = z[i] * w.x + y[i] * w.y;
        y[i] = y0;
      }
      store(8 * u, y);
      store(a.pairs + 8 * u, z);
    } else if constexpr (LAYOUT == kFours) {
      float y[8];
      if (u >= a.turned) {
        const uint32_t d = 2 * a.pairs + 8 * (u - a.turned);
        load(d, y);
        store(d, y);
        continue;
      }
      const u32x2 w0 = *reinterpret_cast<const u32x2*>(from + 8 * u), w1 = *reinterpret_cast<const u32x2*>(from + 2 * a.pairs + 8 * u);
      spread<T>((u32x4){w0.x, w0.y, w1.x, w1.y}, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 w = turn[4 * u + i];
        const float y0 = y[i] * w.x - y[4 + i] * w.y;
        y[4 + i] = y[4 + i] * w.x + y[i] * w.y;
        y[i] = y0;
      }
      if (f8) {
        const u32x2 out = narrow(y, scale);
        *reinterpret_cast<uint32_t*>(to + 4 * u) = out.x;
        *reinterpret_cast<uint32_t*>(to + a.pairs + 4 * u) = out.y;
      } else {
        const u32x4 out = gather<T>(y);
        *reinterpret_cast<u32x2*>(to + 8 * u) = (u32x2){out.x, out.y};
        *reinterpret_cast<u32x2*>(to + 2 * a.pairs + 8 * u) = (u32x2){out.z, out.w};
      }
    } else {  // element by element
      const uint32_t p0 = u < a.turned ? 8 * u : 2 * a.pairs + 8 * (u - a.turned);
      const uint32_t p1 = u < a.turned ? (p0 + 8 < a.pairs ? p0 + 8 : a.pairs) : (p0 + 8 < a.D ? p0 + 8 : a.D);
      auto get = [&](uint32_t d) { return of_half<T>(*reinterpret_cast<const uint16_t*>(from + 2 * d)); };
      auto set = [&](uint32_t d, float y) {
        if (f8) {
          const float one[8] = {y, y, y, y, y, y, y, y};
          to[d] = (uint8_t)narrow(one, scale).x;
        } else {
          *reinterpret_cast<uint16_t*>(to + 2 * d) = (uint16_t)pack<T>(y, y);
        }
      };
      for (uint32_t p = p0; p < p1; ++p) {
        if (u < a.turned) {
          const float y = get(p), z = get(a.pairs + p);
          const float2 w = turn[p];
          set(p, y * w.x - z * w.y);
          set(a.pairs + p, z * w.x + y * w.y);
        } else {
          set(p, get(p));
        }
      }
    }
  }
  mk.end(ARGUS_REGION_ROTATE);
}

template <int T, bool F8>
void launch_as(const RotateArgs& a, Layout layout, uint32_t grid, hipStream_t st) {
  const dim3 g(grid), b(kThreads);
  if (layout == kNeighbours) hipLaunchKernelGGL((k_rotate<T, F8, kNeighbours>), g, b, 0, st, a);
  else if (layout == kHalves) hipLaunchKernelGGL((k_rotate<T, F8, kHalves>), g, b, 0, st, a);
  else if (layout == kFours) hipLaunchKernelGGL((k_rotate<T, F8, kFours>), g, b, 0, st, a);
  else hipLaunchKernelGGL((k_rotate<T, F8, kAnyHalves>), g, b, 0, st, a);
}

}  // namespace
}  // namespace prompt
}  // namespace argus

using namespace argus;
using namespace argus::prompt;

extern "C" int argus_prompt_rotate(const argus_rotate_config* cfg, const argus_rotate_io* io, argus_markers* markers,
                                   void* stream_v) {
  accepted();
  if (!cfg) return refuse(ARGUS_E_INVAL, "no configuration");
  if (cfg->abi_version != ARGUS_ATTR_ABI_VERSION) return refuse(ARGUS_E_ABI, "abi_version %u", cfg->abi_version);
  if (cfg->source_type > ARGUS_FP16) return refuse(ARGUS_E_INVAL, "rows are bf16 or fp16");
  if (cfg->cache_type != cfg->source_type && cfg->cache_type != ARGUS_FP8)
    return refuse(ARGUS_E_INVAL, "the cache is of the rows' type or fp8 (e4m3)");
  if (cfg->seqs > (1u << 20) || cfg->rows > (1u << 24) - 1) return refuse(ARGUS_E_CAPACITY, "seqs %u, rows %u", cfg->seqs, cfg->rows);
  const bool keys = cfg->kv_heads != 0, f8 = cfg->cache_type == ARGUS_FP8;
  if (cfg->kv_heads > 1024 || cfg->heads > 65535 || (!keys && !cfg->heads))
    return refuse(ARGUS_E_INVAL, "heads %u (0..65535), kv_heads %u (0..1024), not both 0", cfg->heads, cfg->kv_heads);
  const uint32_t unit = f8 ? 16u : 8u;
  if (cfg->head_dim < 8 || cfg->head_dim > 256 || cfg->head_dim % unit)
    return refuse(ARGUS_E_INVAL, "head_dim %u: a multiple of %u up to 256", cfg->head_dim, unit);
  if (cfg->pairs < 1 || cfg->pairs > cfg->head_dim / 2) return refuse(ARGUS_E_INVAL, "pairs %u of head_dim %u", cfg->pairs, cfg->head_dim);
  if (cfg->interleaved > 1) return refuse(ARGUS_E_INVAL, "interleaved %u", cfg->interleaved);
  if (keys && (!power_of_two(cfg->page_size) || cfg->page_size < 8 || cfg->page_size > 65536))
    return refuse(ARGUS_E_INVAL, "page_size %u: a power of two, 8..65536", cfg->page_size);
  if (keys && (cfg->num_pages < 1 || cfg->num_pages > 0x7FFFFFFFu || cfg->columns < 1 ||
               (uint64_t)cfg->columns * cfg->page_size > 0x7FFFFFFFull))
    return refuse(ARGUS_E_CAPACITY, "pages or columns out of range");
  if (!io || !io->d_frequencies || (cfg->seqs && !io->d_starts) || (cfg->heads && cfg->rows && (!io->d_q || !io->d_out)) ||
      (keys && cfg->rows && (!io->d_new_k || !io->d_new_v)) || (keys && cfg->seqs && !io->d_table))
    return refuse(ARGUS_E_INVAL, "a required pointer is NULL");
  if (!io->d_offsets && cfg->rows != cfg->seqs) return refuse(ARGUS_E_INVAL, "%u rows, %u sequences and no offsets", cfg->rows, cfg->seqs);
  int rc;
  if (keys && ((rc = check_view(io->k, cfg->cache_type, "k")) != ARGUS_OK || (rc = check_view(io->v, cfg->cache_type, "v")) != ARGUS_OK))
    return rc;
  if (cfg->heads && (!aligned_to(io->d_q, 16) || !aligned_to(io->d_out, 16) ||
                     (io->q_row_stride | io->q_head_stride | io->out_row_stride | io->out_head_stride) % 8))
    return refuse(ARGUS_E_ALIGN, "rows of q and out lie on 16 bytes");
  if (keys && (!aligned_to(io->d_new_k, 16) || !aligned_to(io->d_new_v, 16) ||
               (io->k_row_stride | io->k_head_stride | io->v_row_stride | io->v_head_stride) % 8))
    return refuse(ARGUS_E_ALIGN, "rows of the new keys and values lie on 16 bytes");
  if (!aligned_to(io->d_starts, 4) || !aligned_to(io->d_offsets, 4) || !aligned_to(io->d_frequencies, 8) ||
      (keys && (!aligned_to(io->d_table, 4) || !aligned_to(io->d_k_scale, 4) || !aligned_to(io->d_v_scale, 4))))
    return refuse(ARGUS_E_ALIGN, "buffers lie on their elements' size");
  if (keys && io->table_stride < (int64_t)cfg->columns && cfg->seqs > 1)
    return refuse(ARGUS_E_INVAL, "table_stride %lld below columns", (long long)io->table_stride);
  if (marks_bad_all(markers)) return refuse(ARGUS_E_INVAL, "markers: alignment or region_base");

  RotateArgs a{};
  const Layout layout = cfg->interleaved ? kNeighbours : cfg->pairs % 8 == 0 ? kHalves : cfg->pairs % 4 == 0 ? kFours : kAnyHalves;
  const uint32_t whole = cfg->head_dim / 8, rest = cfg->head_dim - 2 * cfg->pairs;
  a.turned = layout == kFours ? cfg->pairs / 4 : (cfg->pairs + 7) / 8;
  const uint32_t per_head = layout == kNeighbours ? whole : a.turned + (rest + 7) / 8;
  const uint32_t per_token = (cfg->heads + cfg->kv_heads) * per_head + cfg->kv_heads * whole;
  // Of many rows four to a block, which finds their places and angles in one go (65537 rows of 24 + 8 heads of 96
  // 209 us; eight 219, two 206; 40 prompts of up to 8192
  // tokens, 32 + 8 heads of 128 into 8 bits, 187, 187, 196). Of fewer one, for the blocks.
  a.tokens = cfg->rows >= 4096 ? kMaxTokens : 1;
  const uint32_t grid = (cfg->rows + a.tokens - 1) / a.tokens;
  if (!marks_fit(markers, (uint64_t)grid * kWaves * 2)) return refuse(ARGUS_E_CAPACITY, "the marker records do not fit");
  if (cfg->rows == 0 || cfg->seqs == 0) return ARGUS_OK;
  if ((rc = device_ok()) != ARGUS_OK) return rc;
  const int64_t e = type_bytes(cfg->cache_type);
  a.q = (const uint8_t*)io->d_q, a.out = (uint8_t*)io->d_out;
  a.new_k = (const uint8_t*)io->d_new_k, a.new_v = (const uint8_t*)io->d_new_v;
  a.q_row = io->q_row_stride * 2, a.q_hd = io->q_head_stride * 2;
  a.out_row = io->out_row_stride * 2, a.out_hd = io->out_head_stride * 2;
  a.k_row = io->k_row_stride * 2, a.k_hd = io->k_head_stride * 2, a.v_row = io->v_row_stride * 2, a.v_hd = io->v_head_stride * 2;
  if (keys) {
    a.k = (uint8_t*)io->k.base, a.v = (uint8_t*)io->v.base;
    a.k_page = io->k.page_stride * e, a.k_head = io->k.head_stride * e, a.k_tok = io->k.token_stride * e;
    a.v_page = io->v.page_stride * e, a.v_head = io->v.head_stride * e, a.v_tok = io->v.token_stride * e;
    a.table = io->d_table, a.table_stride = io->table_stride;
    a.shift = log2_of(cfg->page_size), a.num_pages = cfg->num_pages, a.columns = cfg->columns;
    a.k_scale = f8 ? io->d_k_scale : nullptr, a.v_scale = f8 ? io->d_v_scale : nullptr;
  }
  a.starts = io->d_starts, a.offsets = io->d_offsets, a.frequencies = io->d_frequencies;
  a.S = cfg->seqs, a.rows = cfg->rows, a.D = cfg->head_dim, a.pairs = cfg->pairs, a.heads = cfg->heads, a.kv_heads = cfg->kv_heads;
  a.per_token = fast_div(per_token), a.per_head = fast_div(per_head), a.per_value = fast_div(whole), a.by_pairs = fast_div(cfg->pairs);
  a.amplitude = cfg->amplitude;
  a.marks = take_marks(markers, grid, 2);
  hipStream_t st = (hipStream_t)stream_v;
  const bool bf = cfg->source_type == ARGUS_BF16;
  (f8 ? (bf ? launch_as<0, true> : launch_as<1, true>) : (bf ? launch_as<0, false> : launch_as<1, false>))(a, layout, grid, st);
  return hipGetLastError() == hipSuccess ? ARGUS_OK : refuse(ARGUS_E_HIP, "launch failed");
}
