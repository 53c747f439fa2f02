/*
 * argus_prompt.h -- the operators of a prompt's pass on one MI355X (gfx950)
 * GPU, beside those of a decode step (argus_decode.h) and over the same paged
 * cache.  C ABI, part of libargus_attr.so.
 *
 *   attend   attention of chunks of new tokens over their sequences' pages
 *   rotate   rotary positions: queries turned, keys turned on their way into
 *            the pages, values beside them
 *   score    log probabilities of given tokens, with entropy, rank and the
 *            best alternatives
 *
 * What argus_decode.h says of its functions holds for these too: streams,
 * argument checks and their codes, argus_decode_last_error, markers, entries
 * and lengths out of their range.  Strides and sizes are in elements unless
 * they are called bytes.
 *
 * Rows are tokens of several sequences one after the other: sequence s has the
 * rows offsets[s] <= r < offsets[s + 1].  Offsets never fall, and lie in
 * [0, rows] (one that does not is taken as the nearer end; where they fall,
 * which sequence a row counts to is not defined, but only rows of the call are
 * read and written).  Rows of no sequence are left out: nothing of theirs is
 * read, and what the outputs hold there stays.
 */
#ifndef ARGUS_PROMPT_H
#define ARGUS_PROMPT_H

#include "argus_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Regions of these operators' markers, behind those of argus_decode.h; a call
 * needs region_base + ARGUS_NUM_ALL_REGIONS <= 65536.  A block has four waves and
 * so four contexts; eight where a row tile of attend is 256 rows; sixteen in
 * attend's plan, and in score where a block reads a row by itself. */
enum {
  ARGUS_REGION_CHUNK_PLAN = 14, /* attend: the batch shared out */
  ARGUS_REGION_CHUNK = 15,      /*   a wave's part of it */
  ARGUS_REGION_CHUNK_JOIN = 16, /*   the pieces of rows joined */
  ARGUS_REGION_ROTATE = 17,
  ARGUS_REGION_SCORE_ROWS = 18,
  ARGUS_REGION_SCORE_JOIN = 19,
  ARGUS_NUM_ALL_REGIONS = 20
};

/* ----------------------------------------------------------------- attend */
/* Sequence s has n = offsets[s + 1] - offsets[s] new tokens, the last n of its
 * lens[s] (their keys and values are in the pages already): row
 * offsets[s] + i is the query of position p = lens[s] - n + i.
 *
 *   out[row][h] = sum_j w_j v_j / sum_j w_j, w_j = exp(x_j - max x),
 *   x_j = scale * k_scale * (q[row][h] . k_j), v_j times v_scale,
 *   lse[row][h] = ln sum_j exp(x_j),
 *
 * over the tokens j <= p whose page is held and (window > 0) with
 * j > p - window or j < sinks, of the key/value head h / group.  A row that
 * sees nothing (one of a position below 0 too, or only scores of minus
 * infinity) answers zeros and an lse of minus infinity.  What a row does not
 * see has no part in it, NaN and infinities among that.  An infinite v_j that it
 * sees makes its element infinite however small w_j is, and NaN beside one of
 * the other sign.
 *
 * Scores, weights, their sums and the answer are held in 32 bits.  The weights
 * that multiply values are rounded once to q's type (in fp16 those below 2^-21
 * of the largest to multiples of 2^-31 of it, or finer), the sums are of the
 * unrounded ones.  So where n is 1 this is the answer of argus_decode_attend,
 * which keeps more of the weights, to within half a step of the values in q's
 * type.  Lengths as there. */
typedef struct argus_chunk_config {
  uint32_t abi_version;  /* ARGUS_ATTR_ABI_VERSION */
  uint32_t q_type;       /* ARGUS_BF16 or ARGUS_FP16: of q and out */
  uint32_t cache_type;   /* q_type, or ARGUS_FP8 */
  uint32_t seqs;         /* 0..2^20 */
  uint32_t rows;         /* rows * group below 2^30; (rows * group / 128 + seqs) * kv_heads up to 2^24 - 4096 */
  uint32_t kv_heads;     /* 1..1024 */
  uint32_t group;        /* query heads per key/value head, 1..256 */
  uint32_t head_dim;     /* a multiple of 8 (of 16 beyond 128 or with ARGUS_FP8), 8..256 */
  uint32_t page_size;    /* a power of two, 8..65536 */
  uint32_t num_pages;    /* 1..2^31 - 1 */
  uint32_t columns;      /* of the page table; columns * page_size < 2^30 */
  uint32_t window;       /* 0: everything before; else the last `window` tokens ... */
  uint32_t sinks;        /* ... and the first `sinks`; < 2^30 both */
  float scale;
} argus_chunk_config;

typedef struct argus_chunk_io {
  const void* d_q;              /* [rows][kv_heads * group][head_dim], 16-byte aligned rows */
  int64_t q_row_stride, q_head_stride;
  argus_page_view k, v;
  const int32_t* d_table;       /* [seqs][columns] */
  int64_t table_stride;
  const int32_t* d_lens;        /* [seqs] */
  const int32_t* d_offsets;     /* [seqs + 1] */
  const float* d_k_scale;       /* [kv_heads] or NULL (1) */
  const float* d_v_scale;
  void* d_out;                  /* [rows][kv_heads * group][head_dim], dense, 16-byte aligned */
  float* d_lse;                 /* [rows][kv_heads * group] or NULL */
} argus_chunk_io;

/* Device workspace attend needs (256-byte aligned; may be 0); SIZE_MAX for a
 * bad configuration. */
size_t argus_prompt_attend_workspace_bytes(const argus_chunk_config* cfg);
int argus_prompt_attend(const argus_chunk_config* cfg, const argus_chunk_io* io, void* d_workspace,
                        size_t workspace_bytes, argus_markers* markers, void* stream);

/* ----------------------------------------------------------------- rotate */
/* Row r of sequence s is the token of position p = starts[s] + r - offsets[s],
 * its offset taken as above (without offsets there is one row per sequence).
 * Of the first 2 * pairs elements of a head, elements (x, y) of pair i become
 *
 *   (amplitude (x cos a - y sin a), amplitude (y cos a + x sin a)), a = p * frequencies[i],
 *
 * the angle in 64 bits, cosine, sine and products in 32, rounded once; the
 * others stay.  Pair i is elements i and i + pairs, or (interleaved) 2 i and 2 i + 1.
 *
 * Queries go to d_out, keys and values to their places in the pages, as
 * argus_decode_append has it (the values as they are).  Without d_q, or
 * without d_new_k and d_new_v, that part is left out; a row whose place is not
 * held still has its query turned. */
typedef struct argus_rotate_config {
  uint32_t abi_version;
  uint32_t source_type;  /* ARGUS_BF16, ARGUS_FP16: of q, out and the new keys and values */
  uint32_t cache_type;   /* source_type, or ARGUS_FP8 */
  uint32_t seqs;         /* 0..2^20 */
  uint32_t rows;         /* seqs where d_offsets is NULL; 0..2^24 - 1 */
  uint32_t heads;        /* of q, 0..65535; 0 without q */
  uint32_t kv_heads;     /* 0..1024; 0 without new keys */
  uint32_t head_dim;     /* a multiple of 8 (16 with ARGUS_FP8), 8..256 */
  uint32_t pairs;        /* 1..head_dim / 2 */
  uint32_t interleaved;  /* 0 or 1 */
  uint32_t page_size;    /* a power of two, 8..65536; these three are not looked at without new keys */
  uint32_t num_pages;
  uint32_t columns;
  float amplitude;
} argus_rotate_config;

typedef struct argus_rotate_io {
  const void* d_q;             /* [rows][heads][head_dim], 16-byte aligned rows, or NULL */
  int64_t q_row_stride, q_head_stride;
  void* d_out;                 /* the same; q itself, or apart from it */
  int64_t out_row_stride, out_head_stride;
  const void* d_new_k;         /* [rows][kv_heads][head_dim], 16-byte aligned rows; both or none */
  const void* d_new_v;
  int64_t k_row_stride, k_head_stride, v_row_stride, v_head_stride;
  argus_page_view k, v;
  const int32_t* d_table;
  int64_t table_stride;
  const int32_t* d_starts;     /* [seqs] */
  const int32_t* d_offsets;    /* [seqs + 1], or NULL */
  const double* d_frequencies; /* [pairs] radians per token */
  const float* d_k_scale;      /* [kv_heads]; NULL: 1 */
  const float* d_v_scale;
} argus_rotate_io;

int argus_prompt_rotate(const argus_rotate_config* cfg, const argus_rotate_io* io, argus_markers* markers, void* stream);

/* ------------------------------------------------------------------ score */
/* Of each row of logits, with ln p[t] = logits[t] - ln sum_t' exp(logits[t']):
 *
 *   logprobs[row]  = ln p[tokens[row]]
 *   entropy[row]   = - sum_t p[t] ln p[t]
 *   ranks[row]     = how many tokens come before tokens[row]: a larger logit, or an equal one and a
 *                    lower token
 *   top_tokens[row][i], top_logprobs[row][i]: the `top` tokens that come first, in that order
 *
 * A logit of minus infinity has no part in the sums, and is no alternative: places
 * left over get token -1 and minus infinity.  A row that holds a NaN or plus
 * infinity, or nothing but minus infinity, has NaN for every number, rank -1
 * and tokens -1.  A token outside [0, vocab) has minus infinity and rank -1. */
typedef struct argus_score_config {
  uint32_t abi_version;
  uint32_t type;   /* ARGUS_BF16, ARGUS_FP16, ARGUS_FP32 */
  uint32_t rows;   /* 0..2^22 */
  uint32_t vocab;  /* 1..2^24 */
  uint32_t top;    /* 0..64 */
  uint32_t pad;
} argus_score_config;

typedef struct argus_score_io {
  const void* d_logits;    /* rows of `vocab`, contiguous elements; any alignment of the type */
  int64_t row_stride;
  const int32_t* d_tokens; /* [rows] */
  float* d_logprobs;       /* out [rows] */
  float* d_entropy;        /* out [rows] */
  int32_t* d_ranks;        /* out [rows] */
  float* d_top_logprobs;   /* out [rows][top]; not looked at where top is 0 */
  int32_t* d_top_tokens;   /* out [rows][top] */
} argus_score_io;

size_t argus_prompt_score_workspace_bytes(const argus_score_config* cfg);
int argus_prompt_score(const argus_score_config* cfg, const argus_score_io* io, void* d_workspace,
                       size_t workspace_bytes, argus_markers* markers, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ARGUS_PROMPT_H */
