/*
 * argus_decode.h -- the operators of a decode step on one MI355X (gfx950) GPU,
 * as kernels that write begin/end marker records of their own regions: the
 * decode megakernel and its parts are what the paper measures (Section 4.2),
 * and argus_attr_run (argus_attr.h) takes the records as they are.  C ABI,
 * part of libargus_attr.so.
 *
 * The operators work on a paged key/value cache.  A sequence's token p lies in
 * page table[s][p / page_size] at place p % page_size; an entry outside
 * [0, num_pages) is a page that is not held.
 *
 *   attend   attention of one new token per sequence over its pages
 *   append   new tokens' keys and values into their pages
 *   step     page tables from one decode step to the next: reordering, copy on
 *            write, growth, release
 *   compact  held pages to the front of the pool
 *   select   beam search's selection over beams and vocabulary
 *
 * Every function enqueues its work on `stream` without synchronising,
 * allocates nothing, and checks its arguments before the first GPU call:
 * ARGUS_E_INVAL, ARGUS_E_ABI, ARGUS_E_ALIGN, ARGUS_E_CAPACITY;
 * ARGUS_E_DEVICE if the current device is not gfx950, ARGUS_E_HIP if a launch
 * fails.  What device memory holds never fails a call: lengths, entries and
 * parents out of their range are read as the text of each operator says.
 * Strides and sizes are in elements unless they are called bytes.
 */
#ifndef ARGUS_DECODE_H
#define ARGUS_DECODE_H

#include "argus_attr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- markers */
/* Regions of the operators' markers: region_base + one of these. */
enum {
  ARGUS_REGION_ATTEND = 0,        /* a wave's part of attend */
  ARGUS_REGION_ATTEND_PLACE = 1,  /*   finding its share of the batch */
  ARGUS_REGION_ATTEND_TOKENS = 2, /*   its keys and values, and the joining of the block's waves */
  ARGUS_REGION_ATTEND_JOIN = 3,   /* the pieces of a sequence joined */
  ARGUS_REGION_APPEND = 4,
  ARGUS_REGION_STEP_CLEAR = 5,
  ARGUS_REGION_STEP_CLAIM = 6,
  ARGUS_REGION_STEP_PLAN = 7,
  ARGUS_REGION_STEP_PLACE = 8,
  ARGUS_REGION_COMPACT_COUNT = 9,
  ARGUS_REGION_COMPACT_PLAN = 10,
  ARGUS_REGION_COMPACT_MOVE = 11,
  ARGUS_REGION_SELECT_ROWS = 12,
  ARGUS_REGION_SELECT_BEAMS = 13,
  ARGUS_NUM_REGIONS = 14
};

/* A buffer of marker records.  A call that is given one adds its records
 * behind the first `used` and moves `used` on (ARGUS_E_CAPACITY, and nothing is
 * enqueued, where they do not fit); how many is known at the call.  One
 * context per wave (ctx_base + block * waves + wave; four waves a block, sixteen
 * in a step that is one launch: ARGUS_REGION_STEP_PLAN and _PLACE without _CLEAR), time
 * in ticks of the device's constant 100 MHz clock.  An operator's answers are
 * the same with and without markers. */
typedef struct argus_markers {
  argus_record* d_records; /* 16-byte aligned */
  uint64_t capacity;       /* records */
  uint64_t used;           /* in, out (host) */
  uint32_t ctx_base;
  uint32_t region_base;    /* region_base + ARGUS_NUM_REGIONS <= 65536 */
} argus_markers;

/* ------------------------------------------------------------------ types */
enum { ARGUS_BF16 = 0, ARGUS_FP16 = 1, ARGUS_FP32 = 2, ARGUS_FP8 = 3 /* e4m3, no infinities */ };

/* One side (keys or values) of a paged cache of one layer: token t of page p,
 * head h, element d lies at base[p * page_stride + h * head_stride +
 * t * token_stride + d].  Base and strides are multiples of 16 bytes; for
 * attend page_stride is 0..2^35 and page_size * token_stride below 2^30. */
typedef struct argus_page_view {
  void* base;
  int64_t page_stride, head_stride, token_stride;
} argus_page_view;

/* ----------------------------------------------------------------- attend */
/* out[s][h] = sum_j p_j v_j / sum_j p_j, p_j = exp(x_j - max x),
 * x_j = scale * k_scale * (q[s][h] . k_j), v_j times v_scale, over the visible
 * tokens j of the sequence, of the key/value head h / group.  Token j is
 * visible when j < lens[s], its page is held, and (window > 0)
 * j >= lens[s] - window or j < sinks.  lse[s][h] = ln sum_j exp(x_j).  A row
 * that sees nothing (or only scores of minus infinity) answers zeros and an
 * lse of minus infinity.  A length below 0 counts as 0, one beyond
 * columns * page_size as that. */
typedef struct argus_attend_config {
  uint32_t abi_version;  /* ARGUS_ATTR_ABI_VERSION */
  uint32_t q_type;       /* ARGUS_BF16 or ARGUS_FP16: of q and out */
  uint32_t cache_type;   /* q_type, or ARGUS_FP8 */
  uint32_t seqs;         /* 0..2^20 */
  uint32_t kv_heads;     /* 1..1024 */
  uint32_t group;        /* query heads per key/value head, 1..256 */
  uint32_t head_dim;     /* a multiple of 8 (of 16 beyond 128 or with ARGUS_FP8), 8..256 */
  uint32_t page_size;    /* a power of two, 8..65536 */
  uint32_t num_pages;    /* 1..2^31 - 1 */
  uint32_t columns;      /* of the page table; columns * page_size < 2^31 */
  uint32_t window;       /* 0: everything; else the last `window` tokens ... */
  uint32_t sinks;        /* ... and the first `sinks`; < 2^31 both */
  float scale;
  uint32_t pad;
} argus_attend_config;

typedef struct argus_attend_io {
  const void* d_q;              /* [seqs][kv_heads * group][head_dim], 16-byte aligned rows */
  int64_t q_seq_stride, q_head_stride;
  argus_page_view k, v;
  const int32_t* d_table;       /* [seqs][columns] */
  int64_t table_stride;
  const int32_t* d_lens;        /* [seqs] */
  const float* d_k_scale;       /* [kv_heads] or NULL (1) */
  const float* d_v_scale;
  void* d_out;                  /* [seqs][kv_heads * group][head_dim], dense, 16-byte aligned */
  float* d_lse;                 /* [seqs][kv_heads * group] or NULL */
} argus_attend_io;

/* Device workspace attend needs (256-byte aligned; may be 0); SIZE_MAX for a
 * bad configuration. */
size_t argus_decode_attend_workspace_bytes(const argus_attend_config* cfg);
int argus_decode_attend(const argus_attend_config* cfg, const argus_attend_io* io, void* d_workspace,
                        size_t workspace_bytes, argus_markers* markers, void* stream);

/* ----------------------------------------------------------------- append */
/* Row r of the new keys and values, of sequence s (offsets[s] <= r <
 * offsets[s + 1]), goes to position starts[s] + r - offsets[s] of the sequence.
 * Without offsets there is one row per sequence.  Into an ARGUS_FP8 cache
 * goes x / scale[head], limited to +-448, rounded to the nearest (ties to
 * even); else the rows are copied.  A row whose position is negative or
 * beyond the table, or whose page is not held, is left out, and so is one
 * outside [offsets[0], offsets[seqs]). */
typedef struct argus_append_config {
  uint32_t abi_version;
  uint32_t source_type;  /* ARGUS_BF16, ARGUS_FP16 */
  uint32_t cache_type;   /* source_type, or ARGUS_FP8 */
  uint32_t seqs;
  uint32_t kv_heads;
  uint32_t head_dim;     /* a multiple of 8 (16 with ARGUS_FP8), 8..256 */
  uint32_t page_size;    /* a power of two, 8..65536 */
  uint32_t num_pages;
  uint32_t columns;
  uint32_t rows;         /* seqs where d_offsets is NULL; 0..2^24 - 1, and to 2^28 - 16 where a row's
                            keys and values take at most 1024 bytes of the cache */
} argus_append_config;

typedef struct argus_append_io {
  const void* d_new_k;         /* [rows][kv_heads][head_dim], 16-byte aligned rows */
  const void* d_new_v;
  int64_t k_row_stride, k_head_stride, v_row_stride, v_head_stride;
  argus_page_view k, v;
  const int32_t* d_table;
  int64_t table_stride;
  const int32_t* d_starts;     /* [seqs] */
  const int32_t* d_offsets;    /* [seqs + 1], never falling, or NULL */
  const float* d_k_scale;      /* [kv_heads]; NULL: 1 */
  const float* d_v_scale;
} argus_append_io;

int argus_decode_append(const argus_append_config* cfg, const argus_append_io* io,
                        argus_markers* markers, void* stream);

/* ------------------------------------------------------------------- step */
/* Page tables of one decode step from those of the last.  New sequence s goes
 * on from sequence parents[s] of the old tables (-1: it starts empty), and gets
 * room for grow[s] more tokens:
 *
 *   old length L = lens[parents[s]] (0 for -1), new length N = L + grow[s], at
 *   most columns * page_size; the pages that hold tokens [0, L) are the
 *   parent's.  Entries beyond ceil(N / page_size) are -1.
 *   window > 0: pages that no later query sees are let go (entry -1): page c
 *   with (c + 1) * page_size <= L - window (+ 1 where N > L) and
 *   c * page_size >= sinks.
 *   Copy on write: where L ends inside a held page and N > L, the sequence
 *   writes on in that page if nobody else can tell: no hold in `held`, every
 *   new sequence that has the page has it as its last, ending inside, and of
 *   those s is the longest (of equals the first).  Else it gets a copy.
 *   Pages for copies and growth are the free ones (in no new table, not
 *   held) by ascending number, handed to s = 0, 1, ...: the copy first, then
 *   the columns.  Where none is left the entry is -1 and counts as short.
 *   refs[p] = holds in `held` + entries of the new tables.
 *   The pages that are copied are copied in every cache: all of the page, in
 *   all of its planes (layers).
 *
 * A parent outside [-1, old_seqs) counts as bad and as -1; lens and grow
 * below 0 as 0, held below 0 as 0. */
enum {
  ARGUS_ST_NEEDED = 0,    /* pages that copies and growth ask for */
  ARGUS_ST_SHORT = 1,     /* of these, not to be had */
  ARGUS_ST_COPIED = 2,    /* pages copied */
  ARGUS_ST_LIVE = 3,      /* pages with refs > 0 */
  ARGUS_ST_BAD_PARENT = 4,
  ARGUS_ST_CUT = 5,       /* sequences that would outgrow the table */
  ARGUS_ST_INTERNAL = 7,  /* 0 unless a consistency check in the library fails */
  ARGUS_ST_NUM_COUNTERS = 8
};

/* A cache for page copies: plane l (a layer's keys, say), page p: page_bytes
 * bytes at base + l * plane_stride + p * page_stride (bytes); all multiples of 16. */
typedef struct argus_page_planes {
  void* base;
  int64_t plane_stride, page_stride;
  uint32_t planes;
  uint32_t page_bytes;
} argus_page_planes;

enum { ARGUS_MAX_CACHES = 4 };

typedef struct argus_step_config {
  uint32_t abi_version;
  uint32_t old_seqs, new_seqs; /* 0..2^20 */
  uint32_t columns;            /* 1.. ; columns * page_size < 2^31 */
  uint32_t num_pages;          /* 1..2^28 */
  uint32_t page_size;          /* a power of two, 1..65536 */
  uint32_t window, sinks;
  uint32_t num_caches;         /* 0..ARGUS_MAX_CACHES */
  uint32_t pad;
} argus_step_config;

typedef struct argus_step_io {
  const int32_t* d_table;    /* [old_seqs][columns] */
  int64_t table_stride;
  const int32_t* d_lens;     /* [old_seqs] */
  const int32_t* d_parents;  /* [new_seqs], or NULL: the sequences stay (new_seqs == old_seqs) */
  const int32_t* d_grow;     /* [new_seqs], or NULL: 0 */
  const int32_t* d_held;     /* [num_pages], or NULL: 0 */
  /* the outputs overlap none of the inputs */
  int32_t* d_new_table;      /* out [new_seqs][columns], dense */
  int32_t* d_new_lens;       /* out [new_seqs] */
  int32_t* d_refs;           /* out [num_pages] */
  int32_t* d_counters;       /* out [ARGUS_ST_NUM_COUNTERS] */
  argus_page_planes caches[ARGUS_MAX_CACHES];
} argus_step_io;

/* SIZE_MAX for sizes out of range. */
size_t argus_decode_step_workspace_bytes(uint32_t new_seqs, uint32_t num_pages);
int argus_decode_step(const argus_step_config* cfg, const argus_step_io* io, void* d_workspace,
                      size_t workspace_bytes, argus_markers* markers, void* stream);

/* ---------------------------------------------------------------- compact */
/* Moves the pages with refs > 0 to the numbers below their count n: a page
 * below n stays, and the pages from n on go, in ascending order, to the free
 * numbers below n, in ascending order.  map[p] = the new number of page p
 * (-1 for a free one); tables and refs follow, an entry of a free page or out of
 * range becomes -1. */
enum { ARGUS_CO_LIVE = 0, ARGUS_CO_MOVED = 1, ARGUS_CO_INTERNAL = 7, ARGUS_CO_NUM_COUNTERS = 8 };

typedef struct argus_compact_config {
  uint32_t abi_version;
  uint32_t seqs, columns;
  uint32_t num_pages;  /* 1..2^28 */
  uint32_t num_caches;
  uint32_t pad;
} argus_compact_config;

typedef struct argus_compact_io {
  const int32_t* d_table;  /* [seqs][columns] */
  int64_t table_stride;
  const int32_t* d_refs;   /* [num_pages] */
  int32_t* d_new_table;    /* out [seqs][columns], dense; not the old one */
  int32_t* d_new_refs;     /* out [num_pages]; not refs */
  int32_t* d_map;          /* out [num_pages] */
  int32_t* d_counters;     /* out [ARGUS_CO_NUM_COUNTERS]; 2..6 are zero */
  argus_page_planes caches[ARGUS_MAX_CACHES];
} argus_compact_io;

size_t argus_decode_compact_workspace_bytes(uint32_t num_pages);
int argus_decode_compact(const argus_compact_config* cfg, const argus_compact_io* io, void* d_workspace,
                         size_t workspace_bytes, argus_markers* markers, void* stream);

/* ----------------------------------------------------------------- select */
/* Of each group's beams and tokens the k of the highest score
 *   score[g][b] + logits[g][b][t] - ln sum_t' exp(logits[g][b][t']),
 * in falling order; equal scores: the lower beam first, within a beam the
 * larger logit, then the lower token.  A finished beam has one candidate:
 * token `eos` with the beam's own score.  A score of minus infinity or NaN is
 * no candidate (a row that holds a NaN or +inf thus has none); places
 * left over get score -inf, parent -1, token -1, finished 0.  parents number
 * the beams of the whole batch (g * beams + b), as argus_decode_step takes
 * them. */
typedef struct argus_select_config {
  uint32_t abi_version;
  uint32_t type;          /* ARGUS_BF16, ARGUS_FP16, ARGUS_FP32 */
  uint32_t groups, beams; /* 0..2^20; 1..64; below 2^26 rows in all */
  uint32_t vocab;         /* 1..2^24 */
  uint32_t k;             /* 1..64 */
  int32_t eos;            /* < 0: none (finished beams then have token eos as it is) */
  uint32_t pad;
} argus_select_config;

typedef struct argus_select_io {
  const void* d_logits;       /* rows of `vocab`, contiguous elements; any alignment of the type */
  int64_t group_stride, beam_stride;
  const float* d_scores;      /* [groups][beams] */
  const uint8_t* d_finished;  /* [groups][beams] or NULL */
  float* d_new_scores;        /* out [groups][k] */
  int32_t* d_parents;         /* out [groups][k] */
  int32_t* d_tokens;          /* out [groups][k] */
  uint8_t* d_new_finished;    /* out [groups][k]: the parent was finished, or the token is eos */
} argus_select_io;

size_t argus_decode_select_workspace_bytes(const argus_select_config* cfg);
int argus_decode_select(const argus_select_config* cfg, const argus_select_io* io, void* d_workspace,
                        size_t workspace_bytes, argus_markers* markers, void* stream);

/* Why the last argus_decode_* call of this thread was refused ("" if it was not). */
const char* argus_decode_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* ARGUS_DECODE_H */
