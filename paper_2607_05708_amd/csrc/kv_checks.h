// Checks shared by the C entry points of the caches.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdlib>

#include "memattn_append.h"
#include "error.h"
#include "kv.h"

namespace memattn {

constexpr int kMaxHeads = 1024;
constexpr int kMaxPageTokens = 4096;
constexpr int kMaxList = 4096;

inline bool known_format(int32_t f) { return f == MEM_KV_BF16 || f == MEM_KV_FP8 || f == MEM_KV_FP4; }

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Format and tokens of a page.
inline mem_status check_page(int32_t format, int32_t page_tokens) {
  if (!known_format(format)) return fail(MEM_ERR_INVALID_ARG, "format %d is no mem_kv_format", format);
  if (page_tokens < 32 || page_tokens > kMaxPageTokens || page_tokens % 32 != 0)
    return fail(MEM_ERR_INVALID_ARG, "page_tokens = %d is not a multiple of 32 in [32, %d]", page_tokens,
                kMaxPageTokens);
  return MEM_OK;
}

// Sizes of a pool and directory whose pages hold `need` bytes.
inline mem_status check_pages(const mem_pages& p, size_t need) {
  if (p.pages_per_chunk < 1 || p.pages_per_chunk > 64)
    return fail(MEM_ERR_INVALID_ARG, "pages_per_chunk outside [1, 64]");
  if (p.n_pages < 0 || p.n_chunks < 0) return fail(MEM_ERR_INVALID_ARG, "negative pool or table size");
  if (p.n_pages > INT32_MAX || p.n_chunks > INT32_MAX)
    return fail(MEM_ERR_UNSUPPORTED, "more than 2^31 - 1 pages or chunks");
  if (p.page_bytes <= 0 || p.page_bytes % 16 != 0)
    return fail(MEM_ERR_INVALID_ARG, "page_bytes must be a positive multiple of 16");
  if (static_cast<size_t>(p.page_bytes) < need)
    return fail(MEM_ERR_INVALID_ARG, "page_bytes = %lld < the %zu bytes of a page",
                static_cast<long long>(p.page_bytes), need);
  return MEM_OK;
}

inline mem_status check_pool(const mem_pages& p) {
  if ((p.n_pages > 0 && !p.pool) || (p.n_chunks > 0 && !p.table))
    return fail(MEM_ERR_INVALID_ARG, "NULL pool or table");
  if (!aligned(p.pool, 16)) return fail(MEM_ERR_INVALID_ARG, "pool must be 16-byte aligned");
  if (!aligned(p.table, 4)) return fail(MEM_ERR_INVALID_ARG, "table must be 4-byte aligned");
  return MEM_OK;
}

inline KvView view_of(const mem_pages& p, int32_t page_tokens, int32_t heads) {
  KvView v;
  v.pool = static_cast<uint8_t*>(const_cast<void*>(p.pool));
  v.n_pages = p.n_pages;
  v.page_bytes = p.page_bytes;
  v.table = p.table;
  v.n_chunks = p.n_chunks;
  v.ppc = p.pages_per_chunk;
  v.page_tokens = page_tokens;
  v.heads = heads;
  return v;
}

// Units of 32 tokens that k chunks can hold.
inline int64_t units_of(const mem_pages& p, int32_t page_tokens, int32_t k) {
  return static_cast<int64_t>(k) * p.pages_per_chunk * page_tokens / 32;
}

inline mem_status check_rows(const mem_kv_rows* r, int heads, int elem, int64_t n, const char* name) {
  if (!r || !r->data) return fail(MEM_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned(r->data, elem)) return fail(MEM_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
  if (r->token_stride < 0 || r->head_stride < 0) return fail(MEM_ERR_INVALID_ARG, "%s has a negative stride", name);
  constexpr int64_t kReach = int64_t{1} << 56;  // elements; more than any address space
  int64_t tokens, across;
  if (__builtin_mul_overflow(n - 1, r->token_stride, &tokens) || tokens > kReach ||
      __builtin_mul_overflow(int64_t{heads - 1}, r->head_stride, &across) || across > kReach)
    return fail(MEM_ERR_INVALID_ARG, "the strides of %s lead out of memory", name);
  return MEM_OK;
}

// First and last byte + 1 that rows cover (their strides have been checked).
inline void span_of(const mem_kv_rows* r, int heads, int d, int elem, int64_t n, uintptr_t* lo, uintptr_t* hi) {
  *lo = reinterpret_cast<uintptr_t>(r->data);
  *hi = *lo + static_cast<uintptr_t>(((n - 1) * r->token_stride + (heads - 1) * r->head_stride + d) * elem);
}

// Whether some row of n tokens shares an element with a different row, or with any row of the same strides that start
// `apart` elements later: whether |apart + i token_stride + j head_stride| < head_dim for some |i| < n, |j| < heads
// (other than both 0 where apart is 0).  For each j only the two i around the zero of that sum can do it.
inline bool rows_meet(const mem_kv_rows* r, int heads, int head_dim, int64_t n, int64_t apart) {
  const int64_t ts = r->token_stride, hs = r->head_stride, d = head_dim, h = heads;
  if (apart == 0 && ((hs >= d && ts >= (h - 1) * hs + d) || (ts >= d && hs >= (n - 1) * ts + d))) return false;
  for (int64_t j = apart == 0 ? 0 : 1 - h; j < h; ++j) {
    const int64_t at = apart + j * hs;
    int64_t i0 = ts == 0 ? 0 : -at / ts - 1;
    if (apart == 0 && j == 0) i0 = 1;
    for (int64_t i = i0; i < i0 + 3; ++i) {
      const int64_t k = std::min(std::max(i, 1 - n), n - 1);
      if (apart == 0 && j == 0 && k == 0) continue;
      if (std::llabs(at + k * ts) < d) return true;
    }
  }
  return false;
}

// Whether rows of two arrays of n tokens have no byte in common for a reason that can be seen: one lies behind the
// other, or both have the same token stride and lie side by side within it, as parts of a fused array do.
inline bool rows_apart(const mem_kv_rows* a, int heads_a, int da, int elem_a, const mem_kv_rows* b, int heads_b, int db,
                       int elem_b, int64_t n) {
  uintptr_t a0, a1, b0, b1;
  span_of(a, heads_a, da, elem_a, n, &a0, &a1);
  span_of(b, heads_b, db, elem_b, n, &b0, &b1);
  if (a1 <= b0 || b1 <= a0) return true;
  if (n == 1 || elem_a != elem_b || a->token_stride != b->token_stride) return false;
  const int64_t ts = a->token_stride, by = static_cast<int64_t>(b0) - static_cast<int64_t>(a0);
  const int64_t wide_a = (heads_a - 1) * a->head_stride + da, wide_b = (heads_b - 1) * b->head_stride + db;
  if (ts <= 0 || by % elem_a != 0) return false;
  const int64_t at = ((by / elem_a) % ts + ts) % ts;  // where b's rows start behind a's
  return at >= wide_a && at + wide_b <= ts;
}

// The rules of an attention call's arguments: numbers first, then how the new tokens go to requests, then arrays.
inline mem_status check_numbers(const mem_attend_args* a) {
  if (!(std::isfinite(a->scale) && a->scale > 0.f)) return fail(MEM_ERR_INVALID_ARG, "scale must be finite and > 0");
  if (!(std::isfinite(a->softcap) && a->softcap >= 0.f))
    return fail(MEM_ERR_INVALID_ARG, "softcap must be finite and >= 0");
  if (a->window < 0) return fail(MEM_ERR_INVALID_ARG, "window < 0");
  return MEM_OK;
}
inline mem_status check_requests(const mem_attend_args* a, int64_t total_q) {
  if (a->m == 0) return fail(MEM_ERR_INVALID_ARG, "new tokens without requests");
  if (!a->q_offsets && total_q % a->m != 0)
    return fail(MEM_ERR_INVALID_ARG, "q_offsets is NULL and total_q = %lld is not a multiple of m = %lld",
                static_cast<long long>(total_q), static_cast<long long>(a->m));
  return MEM_OK;
}
inline mem_status check_arrays(const mem_attend_args* a, int64_t n_chunks) {
  if (!a->ids || (n_chunks > 0 && !a->tok_len)) return fail(MEM_ERR_INVALID_ARG, "ids or tok_len is NULL");
  if (a->chunk_ns && !a->query_ns) return fail(MEM_ERR_INVALID_ARG, "chunk_ns without query_ns");
  return MEM_OK;
}
inline mem_status check_alignment(const mem_attend_args* a, const float* lse) {
  if (!aligned(a->ids, 4) || !aligned(a->tok_len, 4) || !aligned(a->q_offsets, 4) || !aligned(a->q_pos, 4) ||
      !aligned(a->slopes, 4) || !aligned(a->prefix_len, 4) || !aligned(a->chunk_ns, 4) || !aligned(a->query_ns, 4) ||
      !aligned(lse, 4))
    return fail(MEM_ERR_INVALID_ARG, "an int32 or float array is not 4-byte aligned");
  return MEM_OK;
}

// The arguments as the kernels take them, without queries and outputs.
inline AttendArgs attend_args(const mem_attend_args* a, const KvView& kv, int64_t total_q) {
  AttendArgs d{};
  d.kv = kv;
  d.tok_len = a->tok_len;
  d.ids = a->ids;
  d.m = a->m;
  d.k = a->k;
  d.hq = a->heads_q;
  d.q_offsets = a->q_offsets;
  d.q_pos = a->q_pos;
  d.scale = a->scale;
  d.softcap = a->softcap;
  d.slopes = a->slopes;
  d.causal = a->causal != 0;
  d.window = a->window;
  d.prefix_len = a->prefix_len;
  d.chunk_ns = a->chunk_ns;
  d.query_ns = a->query_ns;
  d.total_q = total_q;
  return d;
}

// Rows to append: `a` and `b` go to the cache, q is rotated into q_out.  `half` pairs of its rows of dq elements.
inline mem_status check_append(const mem_pages& pages, const mem_kv_rows* a, int heads_a, int da, const char* name_a,
                               const mem_kv_rows* b, int heads_b, int db, const char* name_b, const mem_kv_rows* q,
                               const mem_kv_rows* q_out, int32_t heads_q, int dq, int32_t dtype,
                               const mem_rotation* rot, const int32_t* chunk, const int32_t* pos, int64_t n) {
  const int elem = dtype == MEM_F32 ? 4 : 2;
  if (mem_status st = check_rows(a, heads_a, elem, n, name_a); st != MEM_OK) return st;
  if (mem_status st = check_rows(b, heads_b, elem, n, name_b); st != MEM_OK) return st;
  if (!chunk || !pos) return fail(MEM_ERR_INVALID_ARG, "chunk or pos is NULL");
  if (!aligned(chunk, 4) || !aligned(pos, 4)) return fail(MEM_ERR_INVALID_ARG, "chunk and pos must be 4-byte aligned");
  if (rot) {
    if (!rot->pos || !rot->freq) return fail(MEM_ERR_INVALID_ARG, "the rotation's pos or freq is NULL");
    if (!aligned(rot->pos, 4) || !aligned(rot->freq, 4))
      return fail(MEM_ERR_INVALID_ARG, "the rotation's pos and freq must be 4-byte aligned");
  }
  if (heads_q == 0) return MEM_OK;
  if (mem_status st = check_rows(q, heads_q, elem, n, "q"); st != MEM_OK) return st;
  if (mem_status st = check_rows(q_out, heads_q, 2, n, "q_out"); st != MEM_OK) return st;
  if (rows_meet(q_out, heads_q, dq, n, 0)) return fail(MEM_ERR_INVALID_ARG, "rows of q_out overlap");
  uintptr_t o0, o1;
  span_of(q_out, heads_q, dq, 2, n, &o0, &o1);
  const uintptr_t p0 = reinterpret_cast<uintptr_t>(pages.pool);
  if (o0 < p0 + static_cast<uintptr_t>(pages.n_pages * pages.page_bytes) && p0 < o1)
    return fail(MEM_ERR_INVALID_ARG, "q_out overlaps the page pool");
  const bool in_place = elem == 2 && q_out->data == q->data && (n == 1 || q_out->token_stride == q->token_stride) &&
                        (heads_q == 1 || q_out->head_stride == q->head_stride);
  if (!in_place && !rows_apart(q_out, heads_q, dq, 2, q, heads_q, dq, elem, n))
    return fail(MEM_ERR_INVALID_ARG, "q_out is not q, and cannot be seen to be apart from it");
  if (!rows_apart(q_out, heads_q, dq, 2, a, heads_a, da, elem, n) ||
      !rows_apart(q_out, heads_q, dq, 2, b, heads_b, db, elem, n))
    return fail(MEM_ERR_INVALID_ARG, "q_out cannot be seen to be apart from %s and %s", name_a, name_b);
  return MEM_OK;
}

// What comes before that: the counts and the rotation's numbers.
inline mem_status check_append_sizes(const mem_kv_rows* q, const mem_kv_rows* q_out, int32_t heads_q, int32_t dtype,
                                     const mem_rotation* rot, int64_t n) {
  if (dtype != MEM_F32 && dtype != MEM_BF16)
    return fail(MEM_ERR_INVALID_ARG, "dtype %d is neither MEM_F32 nor MEM_BF16", dtype);
  if (n < 0) return fail(MEM_ERR_INVALID_ARG, "n < 0");
  if (heads_q < 0 || heads_q > kMaxHeads) return fail(MEM_ERR_INVALID_ARG, "heads_q = %d outside [0, %d]", heads_q, kMaxHeads);
  if ((heads_q > 0) != (q != nullptr) || (heads_q > 0) != (q_out != nullptr))
    return fail(MEM_ERR_INVALID_ARG, "q and q_out are given with heads_q > 0, and only then");
  if (rot && rot->style != MEM_ROTATE_HALVES && rot->style != MEM_ROTATE_PAIRS)
    return fail(MEM_ERR_INVALID_ARG, "style %d is no mem_rotation_style", rot->style);
  return MEM_OK;
}

inline RowsView rows_view(const mem_kv_rows* r) {
  return r ? RowsView{r->data, r->token_stride, r->head_stride} : RowsView{nullptr, 0, 0};
}

inline AppendArgs append_args(const KvView& kv, const mem_kv_rows* a, const mem_kv_rows* b, const mem_kv_rows* q,
                              const mem_kv_rows* q_out, int32_t heads_q, const mem_rotation* rot,
                              const int32_t* chunk, const int32_t* pos, int64_t n) {
  AppendArgs x{};
  x.kv = kv;
  x.k = rows_view(a);
  x.v = rows_view(b);
  x.q = rows_view(q);
  x.q_out = rows_view(q_out);
  x.hq = heads_q;
  x.chunk = chunk;
  x.pos = pos;
  if (rot) {
    x.at = rot->pos;
    x.freq = rot->freq;
    x.half = rot->dim / 2;
    x.pairs = rot->style == MEM_ROTATE_PAIRS;
  }
  x.n = n;
  return x;
}

}  // namespace memattn
