// C ABI of the key/value calls (declared in include/memattn_kv.h): host-side
// argument validation and launches.  Nothing is enqueued before all
// arguments have been checked.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdlib>

#include "memattn_kv.h"
#include "error.h"
#include "kv.h"

namespace memattn {

namespace {

constexpr int kMaxHeads = 1024;
constexpr int kMaxPageTokens = 4096;
constexpr int kMaxList = 4096;

bool known_format(int32_t f) { return f == MEM_KV_BF16 || f == MEM_KV_FP8 || f == MEM_KV_FP4; }
bool known_dim(int32_t d) { return d == 64 || d == 128 || d == 256; }

size_t page_bytes_of(int32_t t, int32_t heads, int32_t d, int32_t fmt) {
  return static_cast<size_t>(heads) * 2 * t * (kv_row_bytes(fmt, d) + kv_scale_bytes(fmt, d));
}

bool valid_shape(int32_t t, int32_t heads, int32_t d, int32_t fmt) {
  return t >= 32 && t <= kMaxPageTokens && t % 32 == 0 && heads >= 1 && heads <= kMaxHeads && known_dim(d) &&
         known_format(fmt);
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// The cache's description (its pointers are checked by check_pool).
mem_status check_shape(const mem_kv* kv) {
  if (!kv) return fail(MEM_ERR_INVALID_ARG, "kv is NULL");
  if (!known_format(kv->format)) return fail(MEM_ERR_INVALID_ARG, "format %d is no mem_kv_format", kv->format);
  if (kv->page_tokens < 32 || kv->page_tokens > kMaxPageTokens || kv->page_tokens % 32 != 0)
    return fail(MEM_ERR_INVALID_ARG, "page_tokens = %d is not a multiple of 32 in [32, %d]", kv->page_tokens,
                kMaxPageTokens);
  if (kv->heads < 1 || kv->heads > kMaxHeads)
    return fail(MEM_ERR_INVALID_ARG, "heads = %d outside [1, %d]", kv->heads, kMaxHeads);
  if (kv->head_dim < 1) return fail(MEM_ERR_INVALID_ARG, "head_dim = %d < 1", kv->head_dim);
  if (!known_dim(kv->head_dim)) return fail(MEM_ERR_UNSUPPORTED, "head_dim = %d is not 64, 128 or 256", kv->head_dim);
  const mem_pages& p = kv->pages;
  if (p.pages_per_chunk < 1 || p.pages_per_chunk > 64)
    return fail(MEM_ERR_INVALID_ARG, "pages_per_chunk outside [1, 64]");
  if (p.n_pages < 0 || p.n_chunks < 0) return fail(MEM_ERR_INVALID_ARG, "negative pool or table size");
  if (p.n_pages > INT32_MAX || p.n_chunks > INT32_MAX)
    return fail(MEM_ERR_UNSUPPORTED, "more than 2^31 - 1 pages or chunks");
  if (p.page_bytes <= 0 || p.page_bytes % 16 != 0)
    return fail(MEM_ERR_INVALID_ARG, "page_bytes must be a positive multiple of 16");
  if (static_cast<size_t>(p.page_bytes) < page_bytes_of(kv->page_tokens, kv->heads, kv->head_dim, kv->format))
    return fail(MEM_ERR_INVALID_ARG, "page_bytes = %lld < the %zu bytes of a page",
                static_cast<long long>(p.page_bytes),
                page_bytes_of(kv->page_tokens, kv->heads, kv->head_dim, kv->format));
  return MEM_OK;
}

mem_status check_pool(const mem_kv* kv) {
  if ((kv->pages.n_pages > 0 && !kv->pages.pool) || (kv->pages.n_chunks > 0 && !kv->pages.table))
    return fail(MEM_ERR_INVALID_ARG, "NULL pool or table");
  if (!aligned(kv->pages.pool, 16)) return fail(MEM_ERR_INVALID_ARG, "pool must be 16-byte aligned");
  if (!aligned(kv->pages.table, 4)) return fail(MEM_ERR_INVALID_ARG, "table must be 4-byte aligned");
  return MEM_OK;
}

KvView view_of(const mem_kv* kv) {
  KvView v;
  v.pool = static_cast<uint8_t*>(const_cast<void*>(kv->pages.pool));
  v.n_pages = kv->pages.n_pages;
  v.page_bytes = kv->pages.page_bytes;
  v.table = kv->pages.table;
  v.n_chunks = kv->pages.n_chunks;
  v.ppc = kv->pages.pages_per_chunk;
  v.page_tokens = kv->page_tokens;
  v.heads = kv->heads;
  return v;
}

mem_status check_rows(const mem_kv* kv, const mem_kv_rows* r, int elem, int64_t n, const char* name) {
  if (!r || !r->data) return fail(MEM_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned(r->data, elem)) return fail(MEM_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
  if (r->token_stride < 0 || r->head_stride < 0) return fail(MEM_ERR_INVALID_ARG, "%s has a negative stride", name);
  constexpr int64_t kReach = int64_t{1} << 56;  // elements; more than any address space
  int64_t tokens, heads;
  if (__builtin_mul_overflow(n - 1, r->token_stride, &tokens) || tokens > kReach ||
      __builtin_mul_overflow(int64_t{kv->heads - 1}, r->head_stride, &heads) || heads > kReach)
    return fail(MEM_ERR_INVALID_ARG, "the strides of %s lead out of memory", name);
  return MEM_OK;
}

// First and last byte + 1 that rows cover (their strides have been checked).
void span_of(const mem_kv* kv, const mem_kv_rows* r, int elem, int64_t n, uintptr_t* lo, uintptr_t* hi) {
  *lo = reinterpret_cast<uintptr_t>(r->data);
  *hi = *lo + static_cast<uintptr_t>(((n - 1) * r->token_stride + (kv->heads - 1) * r->head_stride + kv->head_dim) *
                                     elem);
}

// Whether some row of n tokens shares an element with a different row, or with any row of the same strides that start
// `apart` elements later: whether |apart + i token_stride + j head_stride| < head_dim for some |i| < n, |j| < heads
// (other than both 0 where apart is 0).  For each j only the two i around the zero of that sum can do it.
bool rows_meet(const mem_kv* kv, const mem_kv_rows* r, int64_t n, int64_t apart) {
  const int64_t ts = r->token_stride, hs = r->head_stride, d = kv->head_dim, h = kv->heads;
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

mem_status move_tokens(bool write, const mem_kv* kv, const mem_kv_rows* k, const mem_kv_rows* v, int32_t dtype,
                       const int32_t* chunk, const int32_t* pos, int64_t n, void* stream) {
  clear_error();
  if (mem_status st = check_shape(kv); st != MEM_OK) return st;
  if (dtype != MEM_F32 && dtype != MEM_BF16)
    return fail(MEM_ERR_INVALID_ARG, "dtype %d is neither MEM_F32 nor MEM_BF16", dtype);
  if (n < 0) return fail(MEM_ERR_INVALID_ARG, "n < 0");
  if (n == 0) return MEM_OK;
  if (mem_status st = check_pool(kv); st != MEM_OK) return st;
  if (n > (int64_t{1} << 40) / (kv->heads * kv->head_dim) || !kv_move_fits(write, kv->heads, kv->head_dim, dtype, n))
    return fail(MEM_ERR_UNSUPPORTED, "n too large for one launch");
  const int elem = dtype == MEM_F32 ? 4 : 2;
  if (mem_status st = check_rows(kv, k, elem, n, "k"); st != MEM_OK) return st;
  if (mem_status st = check_rows(kv, v, elem, n, "v"); st != MEM_OK) return st;
  if (!chunk || !pos) return fail(MEM_ERR_INVALID_ARG, "chunk or pos is NULL");
  if (!aligned(chunk, 4) || !aligned(pos, 4)) return fail(MEM_ERR_INVALID_ARG, "chunk and pos must be 4-byte aligned");
  if (!write) {
    if (rows_meet(kv, k, n, 0) || rows_meet(kv, v, n, 0)) return fail(MEM_ERR_INVALID_ARG, "rows of k or v overlap");
    uintptr_t k0, k1, v0, v1;
    span_of(kv, k, elem, n, &k0, &k1);
    span_of(kv, v, elem, n, &v0, &v1);
    const uintptr_t p0 = reinterpret_cast<uintptr_t>(kv->pages.pool);
    const uintptr_t p1 = p0 + static_cast<uintptr_t>(kv->pages.n_pages * kv->pages.page_bytes);
    if ((k0 < p1 && p0 < k1) || (v0 < p1 && p0 < v1))
      return fail(MEM_ERR_INVALID_ARG, "k or v overlaps the page pool");
    if (k0 < v1 && v0 < k1) {  // rows of keys may lie between rows of values, as in a fused array
      const int64_t apart = (static_cast<int64_t>(v0) - static_cast<int64_t>(k0)) / elem;
      const bool alike = (n == 1 || k->token_stride == v->token_stride) &&
                         (kv->heads == 1 || k->head_stride == v->head_stride);
      if (apart == 0 || (alike && rows_meet(kv, k, n, apart)))
        return fail(MEM_ERR_INVALID_ARG, "rows of k and v overlap");
    }
  }
  const RowsView kr{k->data, k->token_stride, k->head_stride}, vr{v->data, v->token_stride, v->head_stride};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return device_status(write ? launch_kv_write(view_of(kv), kv->format, kv->head_dim, kr, vr, dtype, chunk, pos, n, s)
                             : launch_kv_read(view_of(kv), kv->format, kv->head_dim, kr, vr, dtype, chunk, pos, n, s),
                       write ? "cache write launch" : "cache read launch");
}

// Sizes shared by mem_attend and its workspace.
mem_status check_sizes(const mem_kv* kv, int64_t m, int32_t k, int64_t total_q, int32_t heads_q) {
  if (mem_status st = check_shape(kv); st != MEM_OK) return st;
  if (m < 0 || total_q < 0) return fail(MEM_ERR_INVALID_ARG, "m or total_q < 0");
  if (k < 1 || k > kMaxList) return fail(MEM_ERR_INVALID_ARG, "k = %d outside [1, %d]", k, kMaxList);
  if (heads_q < 1 || heads_q > kMaxHeads || heads_q % kv->heads != 0)
    return fail(MEM_ERR_INVALID_ARG, "heads_q = %d is not a multiple of heads = %d in [1, %d]", heads_q, kv->heads,
                kMaxHeads);
  if (m > (1 << 24) || total_q > (int64_t{1} << 30) / heads_q)
    return fail(MEM_ERR_UNSUPPORTED, "more than 2^24 requests or 2^30 query rows");
  return MEM_OK;
}

}  // namespace

}  // namespace memattn

using namespace memattn;

extern "C" {

size_t mem_kv_page_bytes(int32_t page_tokens, int32_t heads, int32_t head_dim, int32_t format) {
  return valid_shape(page_tokens, heads, head_dim, format) ? page_bytes_of(page_tokens, heads, head_dim, format) : 0;
}

mem_status mem_kv_write(const mem_kv* kv, const mem_kv_rows* k, const mem_kv_rows* v, int32_t dtype,
                        const int32_t* chunk, const int32_t* pos, int64_t n, void* stream) {
  return move_tokens(true, kv, k, v, dtype, chunk, pos, n, stream);
}

mem_status mem_kv_read(const mem_kv* kv, const mem_kv_rows* k, const mem_kv_rows* v, int32_t dtype,
                       const int32_t* chunk, const int32_t* pos, int64_t n, void* stream) {
  return move_tokens(false, kv, k, v, dtype, chunk, pos, n, stream);
}

size_t mem_attend_workspace_bytes(const mem_kv* kv, int64_t m, int32_t k, int64_t total_q, int32_t heads_q) {
  clear_error();
  if (check_sizes(kv, m, k, total_q, heads_q) != MEM_OK || m == 0 || total_q == 0) return 0;
  const int64_t units = static_cast<int64_t>(k) * kv->pages.pages_per_chunk * kv->page_tokens / 32;
  return attend_workspace_bytes(kv->head_dim, m, k, units, total_q, kv->heads, heads_q);
}

mem_status mem_attend(const mem_kv* kv, const mem_attend_args* a, const void* q, int64_t total_q,
                      int64_t q_token_stride, int64_t q_head_stride, void* out, float* lse, void* workspace,
                      size_t ws_bytes, void* stream) {
  clear_error();
  if (!a) return fail(MEM_ERR_INVALID_ARG, "args is NULL");
  if (mem_status st = check_sizes(kv, a->m, a->k, total_q, a->heads_q); st != MEM_OK) return st;
  if (!(std::isfinite(a->scale) && a->scale > 0.f)) return fail(MEM_ERR_INVALID_ARG, "scale must be finite and > 0");
  if (!(std::isfinite(a->softcap) && a->softcap >= 0.f))
    return fail(MEM_ERR_INVALID_ARG, "softcap must be finite and >= 0");
  if (a->window < 0) return fail(MEM_ERR_INVALID_ARG, "window < 0");
  if (total_q == 0) return MEM_OK;
  if (a->m == 0) return fail(MEM_ERR_INVALID_ARG, "new tokens without requests");
  if (!a->q_offsets && total_q % a->m != 0)
    return fail(MEM_ERR_INVALID_ARG, "q_offsets is NULL and total_q = %lld is not a multiple of m = %lld",
                static_cast<long long>(total_q), static_cast<long long>(a->m));
  if (mem_status st = check_pool(kv); st != MEM_OK) return st;
  if (!a->ids || (kv->pages.n_chunks > 0 && !a->tok_len))
    return fail(MEM_ERR_INVALID_ARG, "ids or tok_len is NULL");
  if (a->chunk_ns && !a->query_ns) return fail(MEM_ERR_INVALID_ARG, "chunk_ns without query_ns");
  if (!q || !out) return fail(MEM_ERR_INVALID_ARG, "q or out is NULL");
  if (!aligned(q, 2)) return fail(MEM_ERR_INVALID_ARG, "q is not aligned to its elements");
  if (!aligned(out, 16)) return fail(MEM_ERR_INVALID_ARG, "out must be 16-byte aligned");
  if (!aligned(a->ids, 4) || !aligned(a->tok_len, 4) || !aligned(a->q_offsets, 4) || !aligned(a->q_pos, 4) ||
      !aligned(a->slopes, 4) || !aligned(a->prefix_len, 4) || !aligned(a->chunk_ns, 4) || !aligned(a->query_ns, 4) ||
      !aligned(lse, 4))
    return fail(MEM_ERR_INVALID_ARG, "an int32 or float array is not 4-byte aligned");
  if (q_token_stride < 0 || q_head_stride < 0) return fail(MEM_ERR_INVALID_ARG, "negative stride of q");
  const int64_t units = static_cast<int64_t>(a->k) * kv->pages.pages_per_chunk * kv->page_tokens / 32;
  if (!attend_fits(kv->head_dim, a->m, a->k, units, total_q, kv->heads, a->heads_q, a->q_offsets != nullptr))
    return fail(MEM_ERR_UNSUPPORTED, "too many requests and heads for one launch");
  const size_t need = attend_workspace_bytes(kv->head_dim, a->m, a->k, units, total_q, kv->heads, a->heads_q);
  if (need > 0 && !workspace) return fail(MEM_ERR_WORKSPACE, "workspace is NULL");
  if (need > 0 && !aligned(workspace, 16)) return fail(MEM_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  if (ws_bytes < need) return fail(MEM_ERR_WORKSPACE, "workspace of %zu bytes < %zu needed", ws_bytes, need);
  AttendArgs d;
  d.kv = view_of(kv);
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
  d.q = static_cast<const uint16_t*>(q);
  d.q_ts = q_token_stride;
  d.q_hs = q_head_stride;
  d.total_q = total_q;
  d.out = static_cast<uint16_t*>(out);
  d.lse = lse;
  d.ws = workspace;
  return device_status(launch_attend(d, kv->format, kv->head_dim, static_cast<hipStream_t>(stream)),
                       "attention launch");
}

}  // extern "C"
