// Appending tokens to a cache with the position rotation applied on the way, and
// reading a latent cache back.
//
// An element of a rotated pair (a, b) becomes a cos - b sin or a sin + b cos,
// computed in 64 bits and rounded once, to what it is held in.  (32 bits would
// lose the angle of a far position, and a value between two steps would go by the
// cosine's last bit.  The products cost nothing here: the kernels move 8 bytes per
// cycle and CU, and 64-bit products keep up with 64 lanes a cycle.)  Sine and
// cosine are made once per token and pair, in LDS, for all heads of the token: a
// workgroup has whole tokens, keys, values and queries.  A row's items of eight
// elements are neighbouring lanes, so halves of pairs and the largest magnitudes of
// blocks meet through cross-lane steps, and every row is read once.
#include <type_traits>

#include "kv.h"
#include "kv_items.h"
#include "device_common.h"

namespace memattn {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxGroup = 16;    // tokens of a workgroup
constexpr int kMaxAngles = 512;  // pairs of a workgroup's tokens

struct Turn {
  double cos, sin;
};

// x as fp32, rounded to the neighbour with an odd last bit where it is none: rounding that to fewer bits gives what
// one rounding of x gives.
__device__ __forceinline__ float to_odd(double x) {
  const float f = static_cast<float>(x);
  const double d = f;
  if (d == x || x != x) return f;
  uint32_t u = __float_as_uint(f);
  if (__builtin_fabs(d) > __builtin_fabs(x)) --u;  // towards zero
  return __uint_as_float(u | 1u);
}

// N numbers rounded so.  Those that are normal in fp32 are cut off, with what that leaves as the last bit (a fifth of the
// operations, and no 64-bit ones); if some are not, all go the long way.
template <int N>
__device__ __forceinline__ void all_to_odd(const double (&x)[N], float* y) {
  bool other = false;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, x[j]);
    const uint32_t hi = static_cast<uint32_t>(bits >> 32), lo = static_cast<uint32_t>(bits);
    other |= (hi >> 20 & 0x7FFu) - 897u >= 254u;
    const uint32_t cut = static_cast<uint32_t>(bits >> 29) - (896u << 23) & 0x7FFFFFFFu;
    y[j] = __uint_as_float((hi & 0x80000000u) | cut | min(lo << 3, 1u));
  }
  if (other) {
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = to_odd(x[j]);
  }
}

// The places of the workgroup's tokens tok0 .. tok0 + group - 1 and the turns of their pairs; ends with a barrier.
__device__ __forceinline__ void open_tokens(const AppendArgs& a, int64_t tok0, int group, Place* places, Turn* turns) {
  const int tid = threadIdx.x;
  if (tid < group) {
    const int64_t tok = tok0 + tid;
    places[tid] = tok < a.n ? kv_place(a.kv, a.chunk[tok], a.pos[tok]) : Place{-1, 0};
  }
  for (int i = tid; i < group * a.half; i += kThreads) {
    const int t = i / a.half;
    const int64_t tok = tok0 + t;
    if (tok >= a.n) continue;
    const double angle = static_cast<double>(a.at[tok]) * static_cast<double>(a.freq[i - t * a.half]);
    Turn x;
    sincos(angle, &x.sin, &x.cos);
    turns[i] = x;
  }
  __syncthreads();
}

// Rotate item i (elements 8 i .. 8 i + 7) of a row, of which `turns` has the pairs.  Every lane of the wave takes part;
// `turned` says whether the row is one that rotates.
__device__ __forceinline__ void turn_item(float* x, int i, int half, bool pairs, const Turn* turns, bool turned) {
  const bool inside = turned && 8 * i < 2 * half;
  if (pairs) {
    if (!inside) return;
    double z[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const Turn t = turns[4 * i + j];
      const double p = x[2 * j], q = x[2 * j + 1];
      z[2 * j] = p * t.cos - q * t.sin;
      z[2 * j + 1] = p * t.sin + q * t.cos;
    }
    all_to_odd(z, x);
    return;
  }
  const bool low = 8 * i < half;
  const int lane = threadIdx.x & 63, other = inside ? lane + (low ? half / 8 : -half / 8) : lane;
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j)
    y[j] = __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(4 * other, __float_as_int(x[j]))));
  if (!inside) return;
  double z[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const Turn t = turns[8 * i + j - (low ? 0 : half)];
    const double p = x[j], q = low ? -static_cast<double>(y[j]) : y[j];
    z[j] = p * t.cos + q * t.sin;
  }
  all_to_odd(z, x);
}

// A workgroup's rows are numbered head by head (keys, values, queries), 1 << shift tokens each.
template <int FMT, int D, typename T, bool VEC, bool NT>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(AppendArgs a, int shift) {
  constexpr int kPieces = D / 8;
  __shared__ Place places[kMaxGroup];
  __shared__ Turn turns[kMaxAngles];
  const int group = 1 << shift;
  const int64_t tok0 = static_cast<int64_t>(blockIdx.x) << shift;
  open_tokens(a, tok0, group, places, turns);
  const int hk = a.kv.heads, items = ((2 * hk + a.hq) << shift) * kPieces;
  // (one item a thread: many waves keep more in flight than many items a wave; 32,768 tokens 194 us, with the next item
  // on its way 203, with four 227)
  struct Item {
    int i, t, head;  // piece of its row, token, and row: keys, values, queries
    bool is_q, is_v;
  };
  auto item = [&](int at) {
    const int row = at / kPieces, head = row >> shift;
    const bool is_q = head >= 2 * hk, is_v = !is_q && head >= hk;
    return Item{at % kPieces, row & (group - 1), is_q ? head - 2 * hk : is_v ? head - hk : head, is_q, is_v};
  };
  auto fetch = [&](int at, float (&x)[8]) {
    const Item m = item(at);
    const int64_t tok = tok0 + m.t;
    const RowsView& src = m.is_q ? a.q : m.is_v ? a.v : a.k;
    for (int j = 0; j < 8; ++j) x[j] = 0.f;
    if (at < items && tok < a.n && (m.is_q || places[m.t].page >= 0))
      load8<T, VEC, NT>(static_cast<const T*>(src.data) + tok * src.ts + m.head * src.hs + 8 * m.i, x);
  };
  for (int at0 = 0; at0 < items; at0 += kThreads) {
    const int at = at0 + static_cast<int>(threadIdx.x);
    float x[8];
    fetch(at, x);
    const Item m = item(at);
    const int64_t tok = tok0 + m.t;
    const bool live = at < items && tok < a.n;
    turn_item(x, m.i, a.half, a.pairs, turns + m.t * a.half, live && !m.is_v);
    if (live && m.is_q)
      store_item<uint16_t, VEC, NT>(
          static_cast<uint16_t*>(a.q_out.data) + tok * a.q_out.ts + m.head * a.q_out.hs + 8 * m.i, x);
    const Place p = places[m.t];
    const bool kept = live && !m.is_q && p.page >= 0;
    int64_t co, so;
    kv_offsets<FMT, D, 8>(a.kv, m.head, m.is_v, p.row, m.i, &co, &so);
    uint8_t* base = a.kv.pool + p.page * a.kv.page_bytes;
    encode_item<FMT>(x, kept ? base + co : nullptr, kept ? base + so : nullptr, threadIdx.x % 4 == 0, kept);
  }
}

// A token of a latent cache: first the items of the group's latent rows, then those of the key parts and of the
// queries, 8 of each.
template <int FMT, int L, typename T, bool VEC, bool NT>
__global__ __launch_bounds__(kThreads) void latent_append_kernel(AppendArgs a, int shift) {
  constexpr int kPieces = L / 8, kParts = kRopeDim / 8;
  constexpr int kRow = kv_row_bytes(FMT, L), kSc = kv_scale_bytes(FMT, L);
  __shared__ Place places[kMaxGroup];
  __shared__ Turn turns[kMaxAngles];
  const int group = 1 << shift;
  const int64_t tok0 = static_cast<int64_t>(blockIdx.x) << shift, tokens = a.kv.page_tokens;
  open_tokens(a, tok0, group, places, turns);
  const int latent = kPieces << shift, items = latent + ((1 + a.hq) << shift) * kParts;
  struct Item {
    int i, t, head;  // piece of its row, token, and row: -1 latent, 0 key part, 1 + query head
  };
  auto item = [&](int at) {
    if (at < latent) return Item{at % kPieces, at / kPieces, -1};
    const int row = (at - latent) / kParts;
    return Item{at % kParts, row & (group - 1), row >> shift};
  };
  auto fetch = [&](int at, float (&x)[8]) {
    const Item m = item(at);
    const int64_t tok = tok0 + m.t;
    const RowsView& src = m.head < 0 ? a.k : m.head == 0 ? a.v : a.q;
    for (int j = 0; j < 8; ++j) x[j] = 0.f;
    if (at < items && tok < a.n && (m.head > 0 || places[m.t].page >= 0))
      load8<T, VEC, NT>(static_cast<const T*>(src.data) + tok * src.ts + (m.head > 0 ? m.head - 1 : 0) * src.hs + 8 * m.i,
                        x);
  };
  for (int at0 = 0; at0 < items; at0 += kThreads) {
    const int at = at0 + static_cast<int>(threadIdx.x);
    float x[8];
    fetch(at, x);
    const Item m = item(at);
    const int64_t tok = tok0 + m.t;
    const bool live = at < items && tok < a.n;
    turn_item(x, m.i, a.half, a.pairs, turns + m.t * a.half, live && m.head >= 0);
    if (live && m.head > 0)
      store_item<uint16_t, VEC, NT>(
          static_cast<uint16_t*>(a.q_out.data) + tok * a.q_out.ts + (m.head - 1) * a.q_out.hs + 8 * m.i, x);
    const Place p = places[m.t];
    const bool kept = live && p.page >= 0;
    uint8_t* base = a.kv.pool + p.page * a.kv.page_bytes;
    if (kept && m.head == 0)
      store_item<uint16_t, true, false>(
          reinterpret_cast<uint16_t*>(base + tokens * kRow + static_cast<int64_t>(p.row) * 2 * kRopeDim) + 8 * m.i, x);
    const bool is_latent = kept && m.head < 0;
    encode_item<FMT>(x, is_latent ? base + static_cast<int64_t>(p.row) * kRow + m.i * (kRow / kPieces) : nullptr,
                     is_latent ? base + tokens * (kRow + 2 * kRopeDim) + static_cast<int64_t>(p.row) * kSc + m.i / 4
                               : nullptr,
                     threadIdx.x % 4 == 0, is_latent);
  }
}

// Latent rows and key parts as dense rows, 16 bytes an item; places that do not exist give zeros.
template <int FMT, int L, typename T, bool VEC, bool NT>
__global__ __launch_bounds__(kThreads) void latent_read_kernel(KvView kv, RowsView c, RowsView r,
                                                               const int32_t* __restrict__ chunk,
                                                               const int32_t* __restrict__ pos, int64_t n, int shift) {
  constexpr int kN = 16 / static_cast<int>(sizeof(T)), kPieces = L / kN, kParts = kRopeDim / kN;
  constexpr int kRow = kv_row_bytes(FMT, L), kSc = kv_scale_bytes(FMT, L);
  constexpr int U = 4;  // items in flight per thread
  constexpr int kBytes = kN * kRow / L;  // of an item's codes
  __shared__ Place places[kMaxGroup];
  const int group = 1 << shift;
  const int64_t tok0 = static_cast<int64_t>(blockIdx.x) << shift, tokens = kv.page_tokens;
  if (static_cast<int>(threadIdx.x) < group) {
    const int64_t tok = tok0 + threadIdx.x;
    places[threadIdx.x] = tok < n ? kv_place(kv, chunk[tok], pos[tok]) : Place{-1, 0};
  }
  __syncthreads();
  const int latent = kPieces << shift, items = latent + (kParts << shift);
  for (int at0 = 0; at0 < items; at0 += kThreads * U) {
    uint32_t w[U][4], byte[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = at0 + u * kThreads + static_cast<int>(threadIdx.x);
      const bool is_latent = at < latent;
      const int i = is_latent ? at % kPieces : at % kParts, t = is_latent ? at / kPieces : (at - latent) / kParts;
      byte[u] = 127;
      for (int j = 0; j < 4; ++j) w[u][j] = 0;
      if (at >= items) continue;
      const Place p = places[t];
      if (p.page < 0) continue;
      const uint8_t* base = kv.pool + p.page * kv.page_bytes;
      if (!is_latent) {
        const uint8_t* src = base + tokens * kRow + static_cast<int64_t>(p.row) * 2 * kRopeDim + 2 * kN * i;
        if constexpr (kN == 8) {
          const u32x4_t v = *reinterpret_cast<const u32x4_t*>(src);
          for (int j = 0; j < 4; ++j) w[u][j] = v[j];
        } else {
          const u32x2_t v = *reinterpret_cast<const u32x2_t*>(src);
          w[u][0] = v[0];
          w[u][1] = v[1];
        }
        continue;
      }
      const uint8_t* src = base + static_cast<int64_t>(p.row) * kRow + i * kBytes;
      if constexpr (kBytes == 16) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(src);
        for (int j = 0; j < 4; ++j) w[u][j] = v[j];
      } else if constexpr (kBytes == 8) {
        const u32x2_t v = *reinterpret_cast<const u32x2_t*>(src);
        w[u][0] = v[0];
        w[u][1] = v[1];
      } else if constexpr (kBytes == 4) {
        w[u][0] = *reinterpret_cast<const uint32_t*>(src);
      } else {
        w[u][0] = *reinterpret_cast<const uint16_t*>(src);
      }
      if constexpr (FMT != MEM_KV_BF16)
        byte[u] = base[tokens * (kRow + 2 * kRopeDim) + static_cast<int64_t>(p.row) * kSc + i * kN / kKvBlock];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = at0 + u * kThreads + static_cast<int>(threadIdx.x);
      const bool is_latent = at < latent;
      const int i = is_latent ? at % kPieces : at % kParts, t = is_latent ? at / kPieces : (at - latent) / kParts;
      if (at >= items || tok0 + t >= n) continue;
      float x[kN];
      if (FMT == MEM_KV_BF16 || !is_latent) {
#pragma unroll
        for (int j = 0; j < kN / 2; ++j) {
          x[2 * j] = __uint_as_float(w[u][j] << 16);
          x[2 * j + 1] = __uint_as_float(w[u][j] & 0xFFFF0000u);
        }
      } else if constexpr (FMT != MEM_KV_BF16) {
        decode_item<FMT, kN>(w[u], byte[u], x);
      }
      const RowsView& to = is_latent ? c : r;
      store_item<T, VEC, NT>(static_cast<T*>(to.data) + (tok0 + t) * to.ts + kN * i, x);
    }
  }
}

// Tokens of a workgroup, as a power of two: one until that alone fills the GPU's CUs several times over, then more, as
// far as the angles fit.
int group_shift(int64_t n, int half, int most) {
  int shift = 0;
  while ((2 << shift) <= most && (half << (shift + 1)) <= kMaxAngles && (n >> (shift + 1)) >= 4096) ++shift;
  return shift;
}

// Tokens of a workgroup of a cache of keys and values: stretches of a page's rows of a head; of a latent cache, whose
// tokens are smaller.
constexpr int kKvGroup = 8, kLatentGroup = kMaxGroup;

template <int FMT, int D, bool LATENT>
hipError_t launch_append(const AppendArgs& a, int dtype, hipStream_t stream) {
  const int shift = group_shift(a.n, a.half, LATENT ? kLatentGroup : kKvGroup);
  const unsigned grid = static_cast<unsigned>((a.n + (1 << shift) - 1) >> shift);
  const int elem = dtype == MEM_F32 ? 4 : 2;
  bool vec = rows_aligned({a.k.data, a.k.ts, LATENT ? 0 : a.k.hs}, elem) &&
             rows_aligned({a.v.data, a.v.ts, LATENT ? 0 : a.v.hs}, elem);
  if (a.hq > 0) vec = vec && rows_aligned(a.q, elem) && rows_aligned(a.q_out, 2);
  auto go = [&](auto t, auto v, auto nt) {
    using T = decltype(t);
    if constexpr (LATENT)
      latent_append_kernel<FMT, D, T, decltype(v)::value, decltype(nt)::value><<<grid, kThreads, 0, stream>>>(a, shift);
    else
      kv_append_kernel<FMT, D, T, decltype(v)::value, decltype(nt)::value><<<grid, kThreads, 0, stream>>>(a, shift);
  };
  auto pick = [&](auto t) {
    if (!vec) go(t, std::false_type{}, std::false_type{});
    else if (shift == 0) go(t, std::true_type{}, std::false_type{});
    else go(t, std::true_type{}, std::true_type{});
  };
  if (dtype == MEM_F32) pick(float{});
  else pick(uint16_t{});
  return hipGetLastError();
}

template <int FMT, int L>
hipError_t launch_read(const KvView& kv, const RowsView& c, const RowsView& r, int dtype, const int32_t* chunk,
                       const int32_t* pos, int64_t n, hipStream_t stream) {
  const int shift = group_shift(n, 0, kLatentGroup);
  const unsigned grid = static_cast<unsigned>((n + (1 << shift) - 1) >> shift);
  const int elem = dtype == MEM_F32 ? 4 : 2;
  const bool vec = rows_aligned({c.data, c.ts, 0}, elem) && rows_aligned({r.data, r.ts, 0}, elem);
  auto pick = [&](auto t) {
    using T = decltype(t);
    (!vec         ? latent_read_kernel<FMT, L, T, false, false>
     : shift == 0 ? latent_read_kernel<FMT, L, T, true, false>
                  : latent_read_kernel<FMT, L, T, true, true>)<<<grid, kThreads, 0, stream>>>(kv, c, r, chunk, pos, n,
                                                                                          shift);
  };
  if (dtype == MEM_F32) pick(float{});
  else pick(uint16_t{});
  return hipGetLastError();
}

template <bool LATENT, int FMT>
hipError_t launch_append_fmt(const AppendArgs& a, int d, int dtype, hipStream_t stream) {
  if constexpr (LATENT) {
    return d == 256 ? launch_append<FMT, 256, true>(a, dtype, stream) : launch_append<FMT, 512, true>(a, dtype, stream);
  } else {
    return d == 64    ? launch_append<FMT, 64, false>(a, dtype, stream)
           : d == 128 ? launch_append<FMT, 128, false>(a, dtype, stream)
                      : launch_append<FMT, 256, false>(a, dtype, stream);
  }
}

template <bool LATENT>
hipError_t launch_append_any(const AppendArgs& a, int fmt, int d, int dtype, hipStream_t stream) {
  switch (fmt) {
    case MEM_KV_BF16: return launch_append_fmt<LATENT, MEM_KV_BF16>(a, d, dtype, stream);
    case MEM_KV_FP8: return launch_append_fmt<LATENT, MEM_KV_FP8>(a, d, dtype, stream);
    default: return launch_append_fmt<LATENT, MEM_KV_FP4>(a, d, dtype, stream);
  }
}

template <int FMT>
hipError_t launch_read_fmt(const KvView& kv, int l, const RowsView& c, const RowsView& r, int dtype,
                           const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream) {
  return l == 256 ? launch_read<FMT, 256>(kv, c, r, dtype, chunk, pos, n, stream)
                  : launch_read<FMT, 512>(kv, c, r, dtype, chunk, pos, n, stream);
}

}  // namespace

// One token a workgroup at least.
bool append_fits(bool latent, int half, int64_t n) {
  const int shift = group_shift(n, half, latent ? kLatentGroup : kKvGroup);
  return ((n + (1 << shift) - 1) >> shift) <= kMaxGroups;
}

hipError_t launch_kv_append(const AppendArgs& a, int fmt, int d, int dtype, hipStream_t stream) {
  return launch_append_any<false>(a, fmt, d, dtype, stream);
}

hipError_t launch_latent_append(const AppendArgs& a, int fmt, int l, int dtype, hipStream_t stream) {
  return launch_append_any<true>(a, fmt, l, dtype, stream);
}

hipError_t launch_latent_read(const KvView& kv, int fmt, int l, const RowsView& c, const RowsView& r, int dtype,
                              const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream) {
  switch (fmt) {
    case MEM_KV_BF16: return launch_read_fmt<MEM_KV_BF16>(kv, l, c, r, dtype, chunk, pos, n, stream);
    case MEM_KV_FP8: return launch_read_fmt<MEM_KV_FP8>(kv, l, c, r, dtype, chunk, pos, n, stream);
    default: return launch_read_fmt<MEM_KV_FP4>(kv, l, c, r, dtype, chunk, pos, n, stream);
  }
}

}  // namespace memattn
