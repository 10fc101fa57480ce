/*
 * memattn_latent.h -- C ABI of the latent calls of libmemattn.so: a paged cache
 * that holds one latent vector and one rotated key part per token, shared by all
 * heads, and the attention that reads it.
 *
 *   mem_latent_page_bytes  bytes of one page of the cache
 *   mem_latent_append      new tokens' latent vectors and rotated key parts into
 *                          their pages, with their queries' rotation
 *   mem_latent_read        tokens of the cache as dense rows
 *   mem_latent_attend      attention of each request's new tokens over its chunks
 *
 * The conventions of memattn.h hold for every call here, and the cache is made of
 * ordinary pages: mem_gather_chunks, mem_compact_blocks and mem_colocate move its
 * chunks as they move others.
 */
#ifndef MEMATTN_LATENT_H
#define MEMATTN_LATENT_H

#include "memattn_append.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A latent cache of one layer.  A page of page_tokens tokens is
 *   [codes: page_tokens rows of r][key parts: page_tokens rows of 2 * rope_dim]
 *   [scales: page_tokens rows of s]
 * with r bytes of codes (latent_dim * 2, * 1 or / 2) and s bytes of scales
 * (latent_dim / 32, or 0 in bf16) a row, held as mem_kv_format says; key parts are
 * bf16.  Token t of chunk c is row t % page_tokens of page table[c, t /
 * page_tokens].  pages.page_bytes is at least mem_latent_page_bytes() (the rest of
 * a page is not touched); pages.pool is 16-byte aligned, and writable for
 * mem_latent_append.
 */
typedef struct {
  mem_pages pages;     /* pool and directory */
  int32_t page_tokens; /* tokens per page: a multiple of 32, 32..4096 */
  int32_t latent_dim;  /* 256 or 512 (others: MEM_ERR_UNSUPPORTED) */
  int32_t rope_dim;    /* 64 (others: MEM_ERR_UNSUPPORTED) */
  int32_t format;      /* mem_kv_format of the latent vectors */
} mem_latent;

/* Bytes of one page (a multiple of 16); 0 on invalid sizes. */
MEMATTN_API size_t mem_latent_page_bytes(int32_t page_tokens, int32_t latent_dim, int32_t rope_dim, int32_t format);

/*
 * Append n tokens: row i of `c` (latent_dim elements) and of `r` (rope_dim
 * elements; `dtype`, head strides are not used, only read) becomes token pos[i] of
 * chunk chunk[i], r rotated by rot (rot->dim = rope_dim; NULL: r is rotated
 * already, and q is NULL).  Where q is not NULL, row (token, head) of q (`dtype`,
 * heads_q heads of rope_dim: the rotated part of the queries) is rotated and
 * written to q_out as bf16.  Skipped tokens, q_out and sizes as in mem_kv_append.
 */
MEMATTN_API mem_status mem_latent_append(const mem_latent* cache, const mem_kv_rows* c, const mem_kv_rows* r,
                                         const mem_kv_rows* q, const mem_kv_rows* q_out, int32_t heads_q,
                                         int32_t dtype, const mem_rotation* rot, const int32_t* chunk,
                                         const int32_t* pos, int64_t n, void* stream);

/*
 * Read n tokens back: rows i of `c` and `r` (dtype MEM_F32 or MEM_BF16, written)
 * receive the values of token pos[i] of chunk chunk[i], exactly; places that do not
 * exist give zeros, and a place may be named any number of times.  The rows must
 * not overlap each other or the pool; what cannot be seen to be apart (as in
 * mem_kv_append) is refused.
 */
MEMATTN_API mem_status mem_latent_read(const mem_latent* cache, const mem_kv_rows* c, const mem_kv_rows* r,
                                       int32_t dtype, const int32_t* chunk, const int32_t* pos, int64_t n,
                                       void* stream);

/* What takes latent vectors to keys and values: element (head, row, i) is at
 * data[head * head_stride + row * row_stride + i], bf16; rows 0 .. head_dim - 1 of a
 * head make its keys (W_h), rows head_dim .. 2 head_dim - 1 its values (V_h). */
typedef struct {
  const void* data;    /* device, 16-byte aligned */
  int64_t head_stride; /* in elements, multiples of 8 (>= 0) */
  int64_t row_stride;
  int32_t head_dim;    /* 64 or 128 (others: MEM_ERR_UNSUPPORTED) */
} mem_latent_weights;

/*
 * The two forms of latent attention.  With c the latent vector and r the rotated
 * key part of a token, the key of head h is [W_h c, r] and its value V_h c:
 *   MEM_LATENT_EXPANDED  makes keys and values of all heads of the context first:
 *                        less work per pair, for turns of many tokens;
 *   MEM_LATENT_ABSORBED  takes W_h to the query (W_h^T q) and V_h behind the sum:
 *                        all heads share the latent vectors as keys and values, and
 *                        nothing is made of the context: for few new tokens.
 * MEM_LATENT_AUTO chooses by the sizes on the host alone: expanded where total_q / m,
 * rounded down, is above head_dim * latent_dim / (latent_dim - head_dim), as costs less
 * where the requests have about as many new tokens each and see most of their contexts.
 * It does not know masks, lengths, or how new tokens are spread, and both forms are
 * planned for contexts at their capacity: with a short window, documents of which little
 * is seen, one long turn beside single tokens, or lists with room for much more than
 * they hold, the other form may cost many times less, and the caller names it.
 */
typedef enum { MEM_LATENT_AUTO = 0, MEM_LATENT_ABSORBED = 1, MEM_LATENT_EXPANDED = 2 } mem_latent_form;

/* Workspace for mem_latent_attend with these sizes, whatever its masks and
 * q_offsets (0 on invalid sizes).  The expanded form's holds keys and values of all m
 * contexts at their capacity, m * k * pages_per_chunk * page_tokens * (2 head_dim +
 * rope_dim) * 2 bytes a head, of as many heads as 1 GiB holds and of one at least; the
 * absorbed form's goes by total_q * heads. */
MEMATTN_API size_t mem_latent_attend_workspace_bytes(const mem_latent* cache, int64_t m, int32_t k, int64_t total_q,
                                                     int32_t heads, int32_t head_dim, int32_t form);

/*
 * Attention over a latent cache.  Requests, contexts, positions and masks are those
 * of mem_attend (args->heads_q heads; softcap and slopes are not supported: 0 and
 * NULL, else MEM_ERR_UNSUPPORTED).  For new token j, head h and the tokens p that it
 * sees, with q the rows of `q` (head_dim elements) and t those of `t` (rope_dim
 * elements, rotated):
 *   s(p)  = scale * (<q_jh, W_h c_p> + <t_jh, r_p>)
 *   lse   = log sum exp(s(p))
 *   out   = sum exp(s(p) - lse) * V_h c_p
 * A token that sees nothing gets out = 0 and lse = -inf.  Tokens that a query does
 * not see have no influence on it, whatever they hold; an element of a latent vector
 * that is not finite among those that it does see makes its outputs so, however small
 * its weight (one of a key part counts as its score says: nothing at -inf).  An
 * element of V_h that is not finite makes the outputs that take it so, of rows that see
 * something with a score above -inf, and may make the others of its head so; one of W_h
 * counts as the scores that it makes say.  q and t (device bf16, strides
 * in `q` and `t`, only read), out (device bf16 [total_q, heads, head_dim], contiguous,
 * 16-byte aligned) and lse (device fp32 [total_q, heads], nullable).  Rows that no
 * request owns are not written.  out, lse and the workspace must not overlap each
 * other, q, t, w or the pool.
 *
 * Products are bf16 with fp32 sums.  Rounded to bf16 on the way are, in the absorbed
 * form, W_h^T q and the softmax weights, in the expanded form keys, values and weights.
 * (The absorbed form takes the weighted sums of latent vectors through V_h as two bf16
 * numbers each, and so it takes the weights where a request has at most 32 rows on
 * average, new tokens times heads, and a list of at most 2,559 chunks.)  A score is off
 * by at most e = 2^-8 * scale * the sum of its products' magnitudes, besides fp32 sums;
 * an output by at most exp(2 e) - 1 times sum exp(s(p) - lse) |V_h c_p|, with the largest
 * e, and by 2^-7 times that sum for rounded weights, 2^-8 times it for rounded values, and
 * 2^-8 of itself.  The workspace is rewritten by each call, and calls that share one must
 * not overlap.  Nothing is synchronised; the call can be captured into a HIP graph.
 * Refused (MEM_ERR_UNSUPPORTED) are calls whose tiles come to 2^24 or more; expanded
 * ones whose contexts have room for 2^24 groups of 128 tokens; absorbed ones of more
 * than 2^21 - 32 new tokens, or of 2^29 rows.
 */
MEMATTN_API mem_status mem_latent_attend(const mem_latent* cache, const mem_attend_args* args, const mem_kv_rows* q,
                                         const mem_kv_rows* t, int64_t total_q, const mem_latent_weights* w,
                                         int32_t form, void* out, float* lse, void* workspace, size_t ws_bytes,
                                         void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MEMATTN_LATENT_H */
