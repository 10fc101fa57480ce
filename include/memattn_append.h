/*
 * memattn_append.h -- C ABI of appending tokens to the key/value cache of
 * memattn_kv.h with the position rotation applied on the way, to keys and queries:
 *
 *   mem_kv_append       mem_kv_write of rotated keys, and the queries' rotation
 *
 * The conventions of memattn.h hold.
 */
#ifndef MEMATTN_APPEND_H
#define MEMATTN_APPEND_H

#include "memattn_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Which two elements of a row of `dim` rotated elements are a pair. */
typedef enum {
  MEM_ROTATE_HALVES = 0, /* i and i + dim / 2 */
  MEM_ROTATE_PAIRS = 1   /* 2 i and 2 i + 1 */
} mem_rotation_style;

/*
 * The position rotation of n rows: pair i = (a, b) of a token at position p
 * becomes (a cos t - b sin t, a sin t + b cos t) with t = p * freq[i], for the
 * first `dim` elements of a row; the others stay.  Angles, sines and products are
 * computed in 64 bits from the fp32 (or bf16) inputs, and a rotated element is
 * rounded once, to what it is held in.
 */
typedef struct {
  const int32_t* pos; /* device [n]: position of each token, any int32 */
  const float* freq;  /* device [dim / 2]: angle per position of each pair, in radians */
  int32_t dim;        /* rotated elements of a row: a multiple of 16, 16..the row's length */
  int32_t style;      /* mem_rotation_style */
} mem_rotation;

/*
 * mem_kv_write with the keys rotated on the way (rot; values are not), and, where
 * q is not NULL, the same tokens' queries too: row (token, head) of q (`dtype`,
 * heads_q heads of head_dim, only read) is rotated and written to q_out as bf16,
 * which mem_attend takes.  Tokens that mem_kv_write would skip have their queries
 * rotated all the same.  q_out may be q itself (same data and strides, MEM_BF16);
 * other than that its rows must not overlap each other, the pool, or the rows of q,
 * k and v, and that has to be seen from their spans, or from equal token strides
 * within which they lie side by side (as parts of a fused array); what cannot be
 * seen to be apart is refused.  Without q, heads_q is 0 and q_out NULL.  A call of
 * some 2^24 tokens (more where a workgroup has several) is refused
 * (MEM_ERR_UNSUPPORTED).
 */
MEMATTN_API mem_status mem_kv_append(const mem_kv* kv, const mem_kv_rows* k, const mem_kv_rows* v,
                                     const mem_kv_rows* q, const mem_kv_rows* q_out, int32_t heads_q, int32_t dtype,
                                     const mem_rotation* rot, const int32_t* chunk, const int32_t* pos, int64_t n,
                                     void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MEMATTN_APPEND_H */
