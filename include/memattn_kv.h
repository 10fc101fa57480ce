/*
 * memattn_kv.h -- C ABI of the key/value calls of libmemattn.so: a paged cache
 * of keys and values in 16, 8 or 4 bits that lives in the page pool of
 * memattn.h, and the attention that reads it through the block directory.
 *
 *   mem_kv_page_bytes   bytes of one page of the cache
 *   mem_kv_write        quantise new tokens' keys and values into their pages
 *   mem_kv_read         tokens of the cache as dense rows
 *   mem_attend          attention of each request's new tokens over its chunks
 *
 * The conventions of memattn.h hold for every call here: device pointers
 * unless marked HOST, buffers and workspace owned by the caller, everything
 * enqueued on `stream`, arguments validated on the host before anything is
 * enqueued.  mem_last_error and mem_status_string serve these calls too.
 *
 * The cache is made of ordinary pages, so mem_gather_chunks,
 * mem_compact_blocks and mem_colocate move its chunks as they move others.
 */
#ifndef MEMATTN_KV_H
#define MEMATTN_KV_H

#include "memattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * How a row of head_dim elements is held.  A row is cut into blocks of 32
 * elements; the elements of a block share the scale 2^e, held as one byte
 * e + 127.  With a = the largest magnitude in the block:
 *   MEM_KV_BF16  the values in bf16, no scales;
 *   MEM_KV_FP8   4 exponent and 3 mantissa bits (largest value 448, no
 *                infinities, 0x7F = NaN): e is the smallest integer with
 *                a <= 464 * 2^e, clamped to [-110, 119];
 *   MEM_KV_FP4   a sign and 0, .5, 1, 1.5, 2, 3, 4 or 6, two elements to a
 *                byte, the even one in the low half: e is the smallest integer
 *                with a <= 7 * 2^e, clamped to [-110, 125].
 * x * 2^-e is rounded to the nearest representable value, ties to the even
 * code, and saturates; the limits 464 and 7 are the largest magnitudes that
 * saturation moves by no more than half a step.  The scale is a power of two,
 * so every step but that rounding is exact and a value has one right code.
 * In MEM_KV_FP8 and MEM_KV_FP4 an infinity counts as the largest finite
 * float, and a block that holds a NaN gets the scale byte 255, which makes
 * all its elements NaN.  Scale bytes that mem_kv_write does not give (below 17,
 * and above 246 in MEM_KV_FP8 or 252 in MEM_KV_FP4, but for 255) stand for
 * values that are not specified.
 */
typedef enum { MEM_KV_BF16 = 0, MEM_KV_FP8 = 1, MEM_KV_FP4 = 2 } mem_kv_format;

/*
 * A cache of one layer.  A page holds page_tokens tokens of every head: head
 * h's part starts at byte h * S of the page, S = 2 * page_tokens * (r + s),
 * with r bytes of codes (head_dim * 2, * 1 or / 2) and s bytes of scales
 * (head_dim / 32, or 0 in bf16) a row, and is
 *   [K codes: page_tokens rows of r][V codes][K scales: page_tokens rows of s][V scales].
 * Token t of chunk c is row t % page_tokens of page table[c, t / page_tokens].
 * pages.page_bytes is at least mem_kv_page_bytes() (the rest of a page is not
 * touched); pages.pool is 16-byte aligned, and writable for mem_kv_write.
 */
typedef struct {
  mem_pages pages;     /* pool and directory */
  int32_t page_tokens; /* tokens per page: a multiple of 32, 32..4096 */
  int32_t heads;       /* key/value heads, 1..1024 */
  int32_t head_dim;    /* 64, 128 or 256 (others: MEM_ERR_UNSUPPORTED) */
  int32_t format;      /* mem_kv_format */
} mem_kv;

/* Dense rows of keys or values: element (token, head, i) is at
 * data[token * token_stride + head * head_stride + i], in elements. */
typedef struct {
  void* data;
  int64_t token_stride;
  int64_t head_stride;
} mem_kv_rows;

/* Bytes of one page (a multiple of 16); 0 on invalid sizes. */
MEMATTN_API size_t mem_kv_page_bytes(int32_t page_tokens, int32_t heads, int32_t head_dim, int32_t format);

/*
 * Quantise n tokens into the cache: token i of `k` and `v` (dtype MEM_F32 or
 * MEM_BF16, only read) becomes token pos[i] of chunk chunk[i] (device int32
 * [n] each).  A token whose chunk is outside [0, n_chunks), whose position is
 * outside the chunk or whose page is outside the pool is skipped (-1 marks
 * padding).  No two tokens of a call may name the same place.  A call is one
 * launch: some 2^36 elements and more are refused (MEM_ERR_UNSUPPORTED).
 */
MEMATTN_API mem_status mem_kv_write(const mem_kv* kv, const mem_kv_rows* k, const mem_kv_rows* v, int32_t dtype,
                                    const int32_t* chunk, const int32_t* pos, int64_t n, void* stream);

/*
 * Read n tokens back: rows i of `k` and `v` (dtype MEM_F32 or MEM_BF16,
 * written) receive the values of token pos[i] of chunk chunk[i], exactly;
 * places that mem_kv_write would skip give zeros.  A place may be named any
 * number of times.  The rows must not overlap each other (those of k may lie
 * between those of v) or the pool.
 */
MEMATTN_API mem_status mem_kv_read(const mem_kv* kv, const mem_kv_rows* k, const mem_kv_rows* v, int32_t dtype,
                                   const int32_t* chunk, const int32_t* pos, int64_t n, void* stream);

/* The requests and masks of mem_attend.  Nullable arrays are marked. */
typedef struct {
  const int32_t* tok_len;   /* device [n_chunks]: tokens held by each chunk (clamped to [0, its capacity]) */
  const int32_t* ids;       /* device [m, k]: chunks of each request, in context order; ids outside
                               [0, n_chunks) (-1) are skipped */
  int64_t m;                /* requests */
  int32_t k;                /* list length, 1..4096 */
  int32_t heads_q;          /* query heads, a multiple of kv->heads, at most 1024: query head h reads
                               key/value head h / (heads_q / heads) */
  const int32_t* q_offsets; /* device [m + 1]: request i's new tokens are rows q_offsets[i] .. q_offsets[i + 1]
                               of q, non-decreasing within [0, total_q]; NULL: total_q / m each */
  const int32_t* q_pos;     /* device [total_q]: position of each new token in its request's context (any
                               int32; the context's own tokens have positions 0, 1, ...); NULL: the new tokens
                               are the last ones of their context */
  float scale;              /* > 0, finite */
  float softcap;            /* cap of the scores, >= 0, finite (large ones change nothing); 0 = none */
  const float* slopes;      /* device [heads_q]: distance bias of each head; NULL = none */
  int32_t causal;           /* != 0: a token sees positions up to its own */
  int32_t window;           /* > 0: a token sees positions above its own minus `window`; 0 = all */
  const int32_t* prefix_len;/* device [m]: positions below prefix_len[i] are seen whatever causal and window
                               say; NULL = none */
  const int32_t* chunk_ns;  /* device [n_chunks]: document (namespace) of each chunk, negative = deleted;
                               NULL = all the same */
  const int32_t* query_ns;  /* device [total_q]: document of each new token; required with chunk_ns */
} mem_attend_args;

/* Workspace for mem_attend with these sizes, whatever its masks (0 on invalid
 * sizes, and where none is needed). */
MEMATTN_API size_t mem_attend_workspace_bytes(const mem_kv* kv, int64_t m, int32_t k, int64_t total_q,
                                              int32_t heads_q);

/*
 * Attention over the cache.  The context of request i is the tokens of its
 * chunks in list order, at positions 0, 1, ..., n_i - 1 (a token whose page is
 * outside the pool keeps its position and is never seen).  For new token j of
 * request i at position P (q_pos[j], or n_i minus the request's new tokens plus
 * j's place among them) and query head h with key/value head g:
 *   a(p)  = (chunk_ns NULL, or query_ns[j] >= 0 equals the chunk's) and
 *           (p < prefix_len[i], or (not causal or p <= P) and (window = 0 or p > P - window))
 *   s(p)  = scale * <q_jh, K_pg>;  s = softcap * tanh(s / softcap);  s = s - slopes[h] * |P - p|
 *   lse   = log sum over a(p) of exp(s(p))
 *   out   = sum over a(p) of exp(s(p) - lse) * V_pg
 * A token that sees nothing gets out = 0 and lse = -inf, and so does every
 * token of an empty context.  Tokens that a query does not see have no
 * influence on it, whatever they hold; a value that is not finite among those
 * that it does see makes its output so, however small its weight (also behind a
 * key that makes the score -inf).
 * q (device bf16, [total_q, heads_q, head_dim] with the strides given) is only
 * read; out (device bf16) and lse (device fp32, nullable) are [total_q,
 * heads_q, head_dim] and [total_q, heads_q], contiguous; out is 16-byte
 * aligned.  Products are bf16 with fp32 sums; the softmax weights are rounded
 * to bf16 for the second product (heavy ones to 16 bits) and out is divided by
 * the unrounded weights' sum, which is also lse's.  A capped score is off by at
 * most 2^-19 of itself, or with a cap of up to 64 by 2^-21 of the cap.  Scores,
 * distances and the sums of weighted values are fp32 before the division by
 * the weights' sum: weights below some 2^-126 of the largest count as 0, and
 * weights are relative to a reference that may lag 2^8 behind the largest, so
 * that values from 2^120 / n on (of n tokens) may overflow.  Rows of q that no request
 * owns are not written.  The context lengths are read on the device: nothing
 * is synchronised, and the call can be captured into a HIP graph.  Calls whose
 * tiles (16, 32 or 128 rows of a key/value head and request) come to 2^24 or
 * more are refused (MEM_ERR_UNSUPPORTED).
 */
MEMATTN_API mem_status mem_attend(const mem_kv* kv, const mem_attend_args* args, const void* q, int64_t total_q,
                                  int64_t q_token_stride, int64_t q_head_stride, void* out, float* lse,
                                  void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MEMATTN_KV_H */
