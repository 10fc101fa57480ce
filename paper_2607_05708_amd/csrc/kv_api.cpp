// C ABI of the key/value calls (declared in include/memattn_kv.h and include/memattn_append.h): host-side
// argument validation and launches.  Nothing is enqueued before all
// arguments have been checked.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "memattn_append.h"
#include "error.h"
#include "kv.h"
#include "kv_checks.h"

namespace memattn {

namespace {

bool known_dim(int32_t d) { return d == 64 || d == 128 || d == 256; }

size_t page_bytes_of(int32_t t, int32_t heads, int32_t d, int32_t fmt) {
  return static_cast<size_t>(heads) * 2 * t * (kv_row_bytes(fmt, d) + kv_scale_bytes(fmt, d));
}

bool valid_shape(int32_t t, int32_t heads, int32_t d, int32_t fmt) {
  return t >= 32 && t <= kMaxPageTokens && t % 32 == 0 && heads >= 1 && heads <= kMaxHeads && known_dim(d) &&
         known_format(fmt);
}

// The cache's description (its pointers are checked by check_pool).
mem_status check_shape(const mem_kv* kv) {
  if (!kv) return fail(MEM_ERR_INVALID_ARG, "kv is NULL");
  if (mem_status st = check_page(kv->format, kv->page_tokens); st != MEM_OK) return st;
  if (kv->heads < 1 || kv->heads > kMaxHeads)
    return fail(MEM_ERR_INVALID_ARG, "heads = %d outside [1, %d]", kv->heads, kMaxHeads);
  if (kv->head_dim < 1) return fail(MEM_ERR_INVALID_ARG, "head_dim = %d < 1", kv->head_dim);
  if (!known_dim(kv->head_dim)) return fail(MEM_ERR_UNSUPPORTED, "head_dim = %d is not 64, 128 or 256", kv->head_dim);
  return check_pages(kv->pages, page_bytes_of(kv->page_tokens, kv->heads, kv->head_dim, kv->format));
}

KvView view_of(const mem_kv* kv) {
  return memattn::view_of(kv->pages, kv->page_tokens, kv->heads);
}

mem_status move_tokens(bool write, const mem_kv* kv, const mem_kv_rows* k, const mem_kv_rows* v, int32_t dtype,
                       const int32_t* chunk, const int32_t* pos, int64_t n, void* stream) {
  clear_error();
  if (mem_status st = check_shape(kv); st != MEM_OK) return st;
  if (dtype != MEM_F32 && dtype != MEM_BF16)
    return fail(MEM_ERR_INVALID_ARG, "dtype %d is neither MEM_F32 nor MEM_BF16", dtype);
  if (n < 0) return fail(MEM_ERR_INVALID_ARG, "n < 0");
  if (n == 0) return MEM_OK;
  if (mem_status st = check_pool(kv->pages); st != MEM_OK) return st;
  if (n > (int64_t{1} << 40) / (kv->heads * kv->head_dim) || !kv_move_fits(write, kv->heads, kv->head_dim, dtype, n))
    return fail(MEM_ERR_UNSUPPORTED, "n too large for one launch");
  const int elem = dtype == MEM_F32 ? 4 : 2;
  if (mem_status st = check_rows(k, kv->heads, elem, n, "k"); st != MEM_OK) return st;
  if (mem_status st = check_rows(v, kv->heads, elem, n, "v"); st != MEM_OK) return st;
  if (!chunk || !pos) return fail(MEM_ERR_INVALID_ARG, "chunk or pos is NULL");
  if (!aligned(chunk, 4) || !aligned(pos, 4)) return fail(MEM_ERR_INVALID_ARG, "chunk and pos must be 4-byte aligned");
  if (!write) {
    if (rows_meet(k, kv->heads, kv->head_dim, n, 0) || rows_meet(v, kv->heads, kv->head_dim, n, 0))
      return fail(MEM_ERR_INVALID_ARG, "rows of k or v overlap");
    uintptr_t k0, k1, v0, v1;
    span_of(k, kv->heads, kv->head_dim, elem, n, &k0, &k1);
    span_of(v, kv->heads, kv->head_dim, elem, n, &v0, &v1);
    const uintptr_t p0 = reinterpret_cast<uintptr_t>(kv->pages.pool);
    const uintptr_t p1 = p0 + static_cast<uintptr_t>(kv->pages.n_pages * kv->pages.page_bytes);
    if ((k0 < p1 && p0 < k1) || (v0 < p1 && p0 < v1))
      return fail(MEM_ERR_INVALID_ARG, "k or v overlaps the page pool");
    if (k0 < v1 && v0 < k1) {  // rows of keys may lie between rows of values, as in a fused array
      const int64_t apart = (static_cast<int64_t>(v0) - static_cast<int64_t>(k0)) / elem;
      const bool alike = (n == 1 || k->token_stride == v->token_stride) &&
                         (kv->heads == 1 || k->head_stride == v->head_stride);
      if (apart == 0 || (alike && rows_meet(k, kv->heads, kv->head_dim, n, apart)))
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

mem_status mem_kv_append(const mem_kv* kv, const mem_kv_rows* k, const mem_kv_rows* v, const mem_kv_rows* q,
                         const mem_kv_rows* q_out, int32_t heads_q, int32_t dtype, const mem_rotation* rot,
                         const int32_t* chunk, const int32_t* pos, int64_t n, void* stream) {
  clear_error();
  if (mem_status st = check_shape(kv); st != MEM_OK) return st;
  if (!rot) return fail(MEM_ERR_INVALID_ARG, "rot is NULL");
  if (mem_status st = check_append_sizes(q, q_out, heads_q, dtype, rot, n); st != MEM_OK) return st;
  if (rot->dim < 16 || rot->dim > kv->head_dim || rot->dim % 16 != 0)
    return fail(MEM_ERR_INVALID_ARG, "the rotation's dim = %d is not a multiple of 16 in [16, %d]", rot->dim,
                kv->head_dim);
  if (n == 0) return MEM_OK;
  if (mem_status st = check_pool(kv->pages); st != MEM_OK) return st;
  if (n > (int64_t{1} << 40) / ((kv->heads + heads_q) * kv->head_dim) || !append_fits(false, rot->dim / 2, n))
    return fail(MEM_ERR_UNSUPPORTED, "n too large for one launch");
  if (mem_status st = check_append(kv->pages, k, kv->heads, kv->head_dim, "k", v, kv->heads, kv->head_dim, "v", q,
                                   q_out, heads_q, kv->head_dim, dtype, rot, chunk, pos, n);
      st != MEM_OK)
    return st;
  return device_status(launch_kv_append(append_args(view_of(kv), k, v, q, q_out, heads_q, rot, chunk, pos, n),
                                        kv->format, kv->head_dim, dtype, static_cast<hipStream_t>(stream)),
                       "cache append launch");
}

size_t mem_attend_workspace_bytes(const mem_kv* kv, int64_t m, int32_t k, int64_t total_q, int32_t heads_q) {
  clear_error();
  if (check_sizes(kv, m, k, total_q, heads_q) != MEM_OK || m == 0 || total_q == 0) return 0;
  const int64_t units = units_of(kv->pages, kv->page_tokens, k);
  return attend_workspace_bytes(kv->head_dim, m, k, units, total_q, kv->heads, heads_q);
}

mem_status mem_attend(const mem_kv* kv, const mem_attend_args* a, const void* q, int64_t total_q,
                      int64_t q_token_stride, int64_t q_head_stride, void* out, float* lse, void* workspace,
                      size_t ws_bytes, void* stream) {
  clear_error();
  if (!a) return fail(MEM_ERR_INVALID_ARG, "args is NULL");
  if (mem_status st = check_sizes(kv, a->m, a->k, total_q, a->heads_q); st != MEM_OK) return st;
  if (mem_status st = check_numbers(a); st != MEM_OK) return st;
  if (total_q == 0) return MEM_OK;
  if (mem_status st = check_requests(a, total_q); st != MEM_OK) return st;
  if (mem_status st = check_pool(kv->pages); st != MEM_OK) return st;
  if (mem_status st = check_arrays(a, kv->pages.n_chunks); st != MEM_OK) return st;
  if (!q || !out) return fail(MEM_ERR_INVALID_ARG, "q or out is NULL");
  if (!aligned(q, 2)) return fail(MEM_ERR_INVALID_ARG, "q is not aligned to its elements");
  if (!aligned(out, 16)) return fail(MEM_ERR_INVALID_ARG, "out must be 16-byte aligned");
  if (mem_status st = check_alignment(a, lse); st != MEM_OK) return st;
  if (q_token_stride < 0 || q_head_stride < 0) return fail(MEM_ERR_INVALID_ARG, "negative stride of q");
  const int64_t units = units_of(kv->pages, kv->page_tokens, a->k);
  if (!attend_fits(kv->head_dim, a->m, a->k, units, total_q, kv->heads, a->heads_q, a->q_offsets != nullptr))
    return fail(MEM_ERR_UNSUPPORTED, "too many requests and heads for one launch");
  const size_t need = attend_workspace_bytes(kv->head_dim, a->m, a->k, units, total_q, kv->heads, a->heads_q);
  if (need > 0 && !workspace) return fail(MEM_ERR_WORKSPACE, "workspace is NULL");
  if (need > 0 && !aligned(workspace, 16)) return fail(MEM_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  if (ws_bytes < need) return fail(MEM_ERR_WORKSPACE, "workspace of %zu bytes < %zu needed", ws_bytes, need);
  AttendArgs d = attend_args(a, view_of(kv), total_q);
  d.q = static_cast<const uint16_t*>(q);
  d.q_ts = q_token_stride;
  d.q_hs = q_head_stride;
  d.out = static_cast<uint16_t*>(out);
  d.lse = lse;
  d.ws = workspace;
  return device_status(launch_attend(d, kv->format, kv->head_dim, static_cast<hipStream_t>(stream)),
                       "attention launch");
}

}  // extern "C"
