// C ABI of the latent calls (declared in include/memattn_latent.h): host-side
// argument validation and launches.  Nothing is enqueued before all arguments
// have been checked.
#include <hip/hip_runtime.h>

#include "memattn_latent.h"
#include "error.h"
#include "kv_checks.h"
#include "latent.h"

namespace memattn {

namespace {

constexpr int64_t kMaxStride = int64_t{1} << 44;  // elements: of heads and rows together, within a 64-bit address

bool known_latent(int32_t l) { return l == 256 || l == 512; }
bool known_head(int32_t d) { return d == 64 || d == 128; }

size_t page_bytes_of(int32_t t, int32_t l, int32_t fmt) {
  return static_cast<size_t>(t) * (kv_row_bytes(fmt, l) + 2 * kRopeDim + kv_scale_bytes(fmt, l));
}

mem_status check_shape(const mem_latent* c) {
  if (!c) return fail(MEM_ERR_INVALID_ARG, "cache is NULL");
  if (mem_status st = check_page(c->format, c->page_tokens); st != MEM_OK) return st;
  if (c->latent_dim < 1 || c->rope_dim < 1)
    return fail(MEM_ERR_INVALID_ARG, "latent_dim = %d, rope_dim = %d: below 1", c->latent_dim, c->rope_dim);
  if (!known_latent(c->latent_dim))
    return fail(MEM_ERR_UNSUPPORTED, "latent_dim = %d is neither 256 nor 512", c->latent_dim);
  if (c->rope_dim != kRopeDim) return fail(MEM_ERR_UNSUPPORTED, "rope_dim = %d is not %d", c->rope_dim, kRopeDim);
  return check_pages(c->pages, page_bytes_of(c->page_tokens, c->latent_dim, c->format));
}

KvView view_of(const mem_latent* c) { return memattn::view_of(c->pages, c->page_tokens, 1); }

mem_status check_sizes(const mem_latent* c, int64_t m, int32_t k, int64_t total_q, int32_t heads, int32_t head_dim,
                       int32_t form) {
  if (mem_status st = check_shape(c); st != MEM_OK) return st;
  if (m < 0 || total_q < 0) return fail(MEM_ERR_INVALID_ARG, "m or total_q < 0");
  if (k < 1 || k > kMaxList) return fail(MEM_ERR_INVALID_ARG, "k = %d outside [1, %d]", k, kMaxList);
  if (heads < 1 || heads > kMaxHeads) return fail(MEM_ERR_INVALID_ARG, "heads = %d outside [1, %d]", heads, kMaxHeads);
  if (head_dim < 1) return fail(MEM_ERR_INVALID_ARG, "head_dim = %d < 1", head_dim);
  if (!known_head(head_dim)) return fail(MEM_ERR_UNSUPPORTED, "head_dim = %d is neither 64 nor 128", head_dim);
  if (form != MEM_LATENT_AUTO && form != MEM_LATENT_ABSORBED && form != MEM_LATENT_EXPANDED)
    return fail(MEM_ERR_INVALID_ARG, "form %d is no mem_latent_form", form);
  if (m > (1 << 24) || total_q > (int64_t{1} << 30) / heads)
    return fail(MEM_ERR_UNSUPPORTED, "more than 2^24 requests or 2^30 query rows");
  return MEM_OK;
}

// What a call writes lies apart from the rest of it and from what it reads: tiles write their outputs while others read.
mem_status check_apart(const mem_latent* c, const mem_kv_rows* q, const mem_kv_rows* t, const mem_latent_weights* w,
                       const LatentSizes& s, const void* out, const float* lse, const void* workspace, size_t need) {
  struct {
    const char* name;
    uintptr_t lo, hi;
  } x[7] = {{"out"}, {"lse"}, {"workspace"}, {"q"}, {"t"}, {"w"}, {"the page pool"}};
  const uintptr_t rows = static_cast<uintptr_t>(s.total_q) * s.heads;
  auto set = [&](int i, const void* from, uintptr_t bytes) {
    x[i].lo = reinterpret_cast<uintptr_t>(from);
    x[i].hi = x[i].lo + bytes;
  };
  set(0, out, rows * s.head_dim * 2);
  set(1, lse, lse ? rows * sizeof(float) : 0);
  set(2, workspace, need);
  span_of(q, s.heads, s.head_dim, 2, s.total_q, &x[3].lo, &x[3].hi);
  span_of(t, s.heads, kRopeDim, 2, s.total_q, &x[4].lo, &x[4].hi);
  set(5, w->data, 2 * static_cast<uintptr_t>((s.heads - 1) * w->head_stride + (2 * s.head_dim - 1) * w->row_stride +
                                             s.latent));
  set(6, c->pages.pool, static_cast<uintptr_t>(c->pages.n_pages * c->pages.page_bytes));
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 7; ++j)
      if (x[i].lo < x[j].hi && x[j].lo < x[i].hi)
        return fail(MEM_ERR_INVALID_ARG, "%s overlaps %s", x[i].name, x[j].name);
  return MEM_OK;
}

LatentSizes sizes_of(const mem_latent* c, int64_t m, int32_t k, int64_t total_q, int32_t heads, int32_t head_dim) {
  return {c->format, c->latent_dim, head_dim, m, k, units_of(c->pages, c->page_tokens, k), total_q, heads};
}

}  // namespace

}  // namespace memattn

using namespace memattn;

extern "C" {

size_t mem_latent_page_bytes(int32_t page_tokens, int32_t latent_dim, int32_t rope_dim, int32_t format) {
  const bool ok = known_format(format) && page_tokens >= 32 && page_tokens <= kMaxPageTokens && page_tokens % 32 == 0 &&
                  known_latent(latent_dim) && rope_dim == kRopeDim;
  return ok ? page_bytes_of(page_tokens, latent_dim, format) : 0;
}

mem_status mem_latent_append(const mem_latent* cache, const mem_kv_rows* c, const mem_kv_rows* r, const mem_kv_rows* q,
                             const mem_kv_rows* q_out, int32_t heads_q, int32_t dtype, const mem_rotation* rot,
                             const int32_t* chunk, const int32_t* pos, int64_t n, void* stream) {
  clear_error();
  if (mem_status st = check_shape(cache); st != MEM_OK) return st;
  if (mem_status st = check_append_sizes(q, q_out, heads_q, dtype, rot, n); st != MEM_OK) return st;
  if (rot && rot->dim != kRopeDim)
    return fail(MEM_ERR_INVALID_ARG, "the rotation's dim = %d is not rope_dim = %d", rot->dim, kRopeDim);
  if (!rot && heads_q > 0) return fail(MEM_ERR_INVALID_ARG, "q without a rotation");
  if (n == 0) return MEM_OK;
  if (mem_status st = check_pool(cache->pages); st != MEM_OK) return st;
  if (n > (int64_t{1} << 40) / (cache->latent_dim + (1 + heads_q) * kRopeDim) ||
      !append_fits(true, rot ? kRopeDim / 2 : 0, n))
    return fail(MEM_ERR_UNSUPPORTED, "n too large for one launch");
  if (mem_status st = check_append(cache->pages, c, 1, cache->latent_dim, "c", r, 1, kRopeDim, "r", q, q_out, heads_q,
                                   kRopeDim, dtype, rot, chunk, pos, n);
      st != MEM_OK)
    return st;
  return device_status(launch_latent_append(append_args(view_of(cache), c, r, q, q_out, heads_q, rot, chunk, pos, n),
                                            cache->format, cache->latent_dim, dtype, static_cast<hipStream_t>(stream)),
                       "latent append launch");
}

mem_status mem_latent_read(const mem_latent* cache, const mem_kv_rows* c, const mem_kv_rows* r, int32_t dtype,
                           const int32_t* chunk, const int32_t* pos, int64_t n, void* stream) {
  clear_error();
  if (mem_status st = check_shape(cache); st != MEM_OK) return st;
  if (mem_status st = check_append_sizes(nullptr, nullptr, 0, dtype, nullptr, n); st != MEM_OK) return st;
  if (n == 0) return MEM_OK;
  if (mem_status st = check_pool(cache->pages); st != MEM_OK) return st;
  const int l = cache->latent_dim, elem = dtype == MEM_F32 ? 4 : 2;
  if (n > (int64_t{1} << 40) / l || !append_fits(true, 0, n))
    return fail(MEM_ERR_UNSUPPORTED, "n too large for one launch");
  if (mem_status st = check_rows(c, 1, elem, n, "c"); st != MEM_OK) return st;
  if (mem_status st = check_rows(r, 1, elem, n, "r"); st != MEM_OK) return st;
  if (!chunk || !pos) return fail(MEM_ERR_INVALID_ARG, "chunk or pos is NULL");
  if (!aligned(chunk, 4) || !aligned(pos, 4)) return fail(MEM_ERR_INVALID_ARG, "chunk and pos must be 4-byte aligned");
  if (rows_meet(c, 1, l, n, 0) || rows_meet(r, 1, kRopeDim, n, 0))
    return fail(MEM_ERR_INVALID_ARG, "rows of c or r overlap");
  if (!rows_apart(c, 1, l, elem, r, 1, kRopeDim, elem, n))
    return fail(MEM_ERR_INVALID_ARG, "c and r cannot be seen to be apart");
  const mem_kv_rows pool{const_cast<void*>(cache->pages.pool), 0, 0};
  const int64_t pool_bytes = cache->pages.n_pages * cache->pages.page_bytes;
  uintptr_t c0, c1, r0, r1;
  span_of(c, 1, l, elem, n, &c0, &c1);
  span_of(r, 1, kRopeDim, elem, n, &r0, &r1);
  const uintptr_t p0 = reinterpret_cast<uintptr_t>(pool.data), p1 = p0 + static_cast<uintptr_t>(pool_bytes);
  if ((c0 < p1 && p0 < c1) || (r0 < p1 && p0 < r1))
    return fail(MEM_ERR_INVALID_ARG, "c or r overlaps the page pool");
  return device_status(launch_latent_read(view_of(cache), cache->format, l, rows_view(c), rows_view(r), dtype, chunk,
                                          pos, n, static_cast<hipStream_t>(stream)),
                       "latent read launch");
}

size_t mem_latent_attend_workspace_bytes(const mem_latent* cache, int64_t m, int32_t k, int64_t total_q, int32_t heads,
                                         int32_t head_dim, int32_t form) {
  clear_error();
  if (check_sizes(cache, m, k, total_q, heads, head_dim, form) != MEM_OK || m == 0 || total_q == 0) return 0;
  const LatentSizes s = sizes_of(cache, m, k, total_q, heads, head_dim);
  return latent_workspace_bytes(s, choose_latent_form(s, form));
}

mem_status mem_latent_attend(const mem_latent* cache, const mem_attend_args* a, const mem_kv_rows* q,
                             const mem_kv_rows* t, int64_t total_q, const mem_latent_weights* w, int32_t form,
                             void* out, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  if (!a) return fail(MEM_ERR_INVALID_ARG, "args is NULL");
  if (!w) return fail(MEM_ERR_INVALID_ARG, "w is NULL");
  if (mem_status st = check_sizes(cache, a->m, a->k, total_q, a->heads_q, w->head_dim, form); st != MEM_OK) return st;
  if (mem_status st = check_numbers(a); st != MEM_OK) return st;
  if (a->softcap != 0.f || a->slopes) return fail(MEM_ERR_UNSUPPORTED, "softcap and slopes are not supported here");
  if (total_q == 0) return MEM_OK;
  if (mem_status st = check_requests(a, total_q); st != MEM_OK) return st;
  if (mem_status st = check_pool(cache->pages); st != MEM_OK) return st;
  if (mem_status st = check_arrays(a, cache->pages.n_chunks); st != MEM_OK) return st;
  if (mem_status st = check_rows(q, a->heads_q, 2, total_q, "q"); st != MEM_OK) return st;
  if (mem_status st = check_rows(t, a->heads_q, 2, total_q, "t"); st != MEM_OK) return st;
  if (!w->data || !out) return fail(MEM_ERR_INVALID_ARG, "w's data or out is NULL");
  if (!aligned(w->data, 16)) return fail(MEM_ERR_INVALID_ARG, "w's data must be 16-byte aligned");
  if (w->head_stride < 0 || w->row_stride < 0 || w->head_stride % 8 != 0 || w->row_stride % 8 != 0)
    return fail(MEM_ERR_INVALID_ARG, "w's strides must be multiples of 8, and not negative");
  if (w->head_stride > kMaxStride || w->row_stride > kMaxStride)
    return fail(MEM_ERR_INVALID_ARG, "the strides of w lead out of memory");
  if (!aligned(out, 16)) return fail(MEM_ERR_INVALID_ARG, "out must be 16-byte aligned");
  if (mem_status st = check_alignment(a, lse); st != MEM_OK) return st;
  const LatentSizes s = sizes_of(cache, a->m, a->k, total_q, a->heads_q, w->head_dim);
  const mem_latent_form f = choose_latent_form(s, form);
  if (!latent_fits(s, f, a->q_offsets != nullptr))
    return fail(MEM_ERR_UNSUPPORTED, "too many requests and heads for one launch");
  const size_t need = latent_workspace_bytes(s, f);
  if (!workspace) return fail(MEM_ERR_WORKSPACE, "workspace is NULL");
  if (!aligned(workspace, 16)) return fail(MEM_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  if (ws_bytes < need) return fail(MEM_ERR_WORKSPACE, "workspace of %zu bytes < %zu needed", ws_bytes, need);
  if (mem_status st = check_apart(cache, q, t, w, s, out, lse, workspace, need); st != MEM_OK) return st;
  LatentArgs x{};
  x.a = attend_args(a, view_of(cache), total_q);
  x.a.lse = lse;
  x.q = rows_view(q);
  x.t = rows_view(t);
  x.w = static_cast<const uint16_t*>(w->data);
  x.w_hs = w->head_stride;
  x.w_rs = w->row_stride;
  x.out = static_cast<uint16_t*>(out);
  x.ws = workspace;
  return device_status(launch_latent_attend(x, s, f, static_cast<hipStream_t>(stream)), "latent attention launch");
}

}  // extern "C"
