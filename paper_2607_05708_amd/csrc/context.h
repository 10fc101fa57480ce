// What the attention kernels share: a workgroup's request, rows and units of the
// context, what its rows see, pieces of rows in their formats, and the running
// softmax of rows whose scores lie in the lanes of one column.
#pragma once

#include "kv.h"
#include "device_common.h"

namespace memattn {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kUnit = 32;       // tokens per unit
constexpr int kFar = 1 << 30;   // above every position

// One unit of the context, resolved.
struct Unit {
  int64_t at;     // byte of the pool at which its first key's codes start (of the workgroup's head)
  int32_t where;  // first row in the page | tokens held << 16 | kMasked
  int32_t pos;    // position of its first token
  int32_t ns;     // document of its chunk

  static constexpr int kMasked = 1 << 24;  // some row does not see some of its 32 tokens
  __device__ __forceinline__ int row() const { return where & 0xFFFF; }
  __device__ __forceinline__ int held() const { return (where >> 16) & 63; }
  __device__ __forceinline__ bool masked() const { return (where & kMasked) != 0; }
};

// ---------------------------------------------------------------- a workgroup's request, rows and units

struct Tile {
  int req;
  int q0;         // first query token of the request
  int nq;         // its new tokens
  int r0;         // first row of the tile among the request's rows
  int rows;       // rows in the tile
};

// Sum over the lanes up to this one (row by row, then across rows: no trip through the LDS unit).
__device__ __forceinline__ int wave_prefix_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  const int lane = threadIdx.x & 63;
  const int r0 = __builtin_amdgcn_readlane(x, 15), r1 = __builtin_amdgcn_readlane(x, 31),
            r2 = __builtin_amdgcn_readlane(x, 47);
  return x + (lane >= 48 ? r0 + r1 + r2 : lane >= 32 ? r0 + r1 : lane >= 16 ? r0 : 0);
}

// Request and rows of tile t.  With ragged requests there are ceil(n G / R) tiles for each; every wave adds them up by
// itself, 64 requests at a time, as long as there are few (kCounted) requests.  With more, tile t of request i is tile
// floor(q_offsets[i] G / R) + i + t: these starts leave room for every request's tiles and can be searched without a
// sum, 64 probes at a time; some of the tiles are empty.  (Empty tiles between the others cost more than their start:
// workgroups go to the XCDs and their shader engines in turn, and with one empty tile for each that is not only half
// of them got work: 64 requests of 128 rows over 16,384 tokens 1.20 ms, added up 0.70 ms; 512 of 128 over 512 tokens
// 553 and 342 us.  The sum itself shows where there are many short requests: 512 of 2 rows 89 and 98 us.)
constexpr int kCounted = 512;
template <int R>
__device__ __forceinline__ bool find_tile(const AttendArgs& a, uint32_t t, int group, Tile* out) {
  const int m = static_cast<int>(a.m), total = static_cast<int>(a.total_q);
  if (a.q_offsets && m <= kCounted) {
    const int lane = threadIdx.x & 63;
    int at = -1, first = 0, o = 0, e = 0;  // request, its first tile, its tokens
    for (int i0 = 0; i0 < m && at < 0; i0 += 64) {
      const int i = i0 + lane;
      const int from = i < m ? a.q_offsets[i] : 0, to = i < m ? a.q_offsets[i + 1] : 0;
      const int64_t n = min(max(static_cast<int64_t>(to) - from, int64_t{0}), a.total_q);
      const int mine = static_cast<int>((n * group + R - 1) / R);
      const int upto = wave_prefix_sum(mine);
      const uint64_t after = __ballot(first + upto > static_cast<int64_t>(t));
      if (after) {
        const int l = __builtin_ctzll(after);
        at = i0 + l;
        o = __builtin_amdgcn_readlane(from, l);
        e = __builtin_amdgcn_readlane(to, l);
        first += __builtin_amdgcn_readlane(upto - mine, l);
      } else {
        first += __builtin_amdgcn_readlane(upto, 63);
      }
    }
    if (at < 0 || o < 0 || e > total || o > e) return false;
    out->req = at;
    out->q0 = o;
    out->nq = e - o;
    t -= static_cast<uint32_t>(first);
  } else if (a.q_offsets) {
    auto start = [&](int i) { return static_cast<int64_t>(a.q_offsets[i]) * group / R + i; };
    const int lane = threadIdx.x & 63;
    int lo = 0, n = m;
    while (n > 0) {
      const int step = (n + 63) >> 6, i = lane * step;
      const bool before = i < n && start(lo + i) <= t;
      const int last = max(__builtin_popcountll(__ballot(before)) - 1, 0);  // the starts never fall
      lo += last * step;
      if (step == 1) break;
      n = min(step, n - last * step);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const int o = a.q_offsets[lo], e = a.q_offsets[lo + 1];
    if (o < 0 || e > total || o > e || start(lo) > t) return false;
    out->req = lo;
    out->q0 = o;
    out->nq = e - o;
    t -= static_cast<uint32_t>(start(lo));
  } else {
    const uint32_t nq = static_cast<uint32_t>(total) / static_cast<uint32_t>(m);
    const uint32_t per = (nq * group + R - 1) / R;
    out->req = static_cast<int>(t / per);
    out->q0 = out->req * static_cast<int>(nq);
    out->nq = static_cast<int>(nq);
    t -= out->req * per;
  }
  const int rows = out->nq * group;
  if (t >= static_cast<uint32_t>((rows + R - 1) / R)) return false;
  out->r0 = static_cast<int>(t) * R;
  out->rows = min(R, rows - out->r0);
  return true;
}

// Smallest and largest over a fully active wave, in a scalar register.
template <int CTRL>
__device__ __forceinline__ int dpp_i32(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, false);
}
__device__ __forceinline__ int wave_min(int x) {
  x = min(x, dpp_i32<0xB1>(x));
  x = min(x, dpp_i32<0x4E>(x));
  x = min(x, dpp_i32<0x141>(x));
  x = min(x, dpp_i32<0x140>(x));
  return min(min(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16)),
             min(__builtin_amdgcn_readlane(x, 32), __builtin_amdgcn_readlane(x, 48)));
}
__device__ __forceinline__ int wave_max(int x) { return ~wave_min(~x); }

// The request's chunk list in LDS: cid[c] = chunk of entry c, ub[c] / tb[c] = units / tokens before it; index k of
// the latter two holds the totals.
struct ChunkList {
  int *cid, *ub, *tb;
  int k;
};

// (with KEEP false the chunks stay where they are in memory, and only the sums take LDS)
template <int THREADS = kThreads, bool KEEP = true>
__device__ __forceinline__ ChunkList scan_list(const AttendArgs& a, int req, int* lds, int* tmp) {
  const int k = a.k;
  const int32_t* ids = a.ids + static_cast<int64_t>(req) * k;
  const ChunkList L = KEEP ? ChunkList{lds, lds + k, lds + 2 * k + 1, k}
                           : ChunkList{const_cast<int32_t*>(ids), lds, lds + k + 1, k};
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int cap = a.kv.ppc * a.kv.page_tokens;
  const int per = (k + THREADS - 1) / THREADS;
  const int c0 = min(tid * per, k), c1 = min(c0 + per, k);
  int u = 0, t = 0;
  for (int c = c0; c < c1; ++c) {
    const int32_t id = ids[c];
    const int len = id >= 0 && id < a.kv.n_chunks ? min(max(a.tok_len[id], 0), cap) : 0;
    if (KEEP) L.cid[c] = id;
    L.ub[c] = u;
    L.tb[c] = t;
    u += (len + kUnit - 1) / kUnit;
    t += len;
  }
  const int su = wave_prefix_sum(u), st = wave_prefix_sum(t);
  if (lane == 63) {
    tmp[2 * wave] = su;
    tmp[2 * wave + 1] = st;
  }
  __syncthreads();
  int bu = su - u, bt = st - t, total_u = 0, total_t = 0;
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) { bu += tmp[2 * w]; bt += tmp[2 * w + 1]; }
    total_u += tmp[2 * w];
    total_t += tmp[2 * w + 1];
  }
  for (int c = c0; c < c1; ++c) {
    L.ub[c] += bu;
    L.tb[c] += bt;
  }
  if (tid == 0) {
    L.ub[k] = total_u;
    L.tb[k] = total_t;
  }
  __syncthreads();
  return L;
}

// Last entry c of b[0..k] with b[c] <= x, below k.
__device__ __forceinline__ int find_entry(const int* b, int k, int x) {
  int lo = 0, hi = k - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (b[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Units that some row of a tile can see: [0, a) and [b, e) of the request's units.
struct Span {
  int a, b, e;
  __device__ __forceinline__ int count() const { return a + (e - b); }
  __device__ __forceinline__ int unit(int i) const { return i < a ? i : i - a + b; }
};

// The span for rows whose visible positions lie in [0, prefix) and [lo, hi].
__device__ __forceinline__ Span visible_units(const ChunkList& L, int prefix, int lo, int hi) {
  const int total = L.tb[L.k], units = L.ub[L.k];
  auto unit_of = [&](int pos) {  // unit that holds position pos < total
    const int c = find_entry(L.tb, L.k, pos);
    return L.ub[c] + (pos - L.tb[c]) / kUnit;
  };
  Span s{0, 0, 0};
  hi = min(hi, total - 1);
  lo = max(lo, 0);
  if (lo <= hi) {
    s.b = lo > 0 ? unit_of(lo) : 0;
    s.e = hi == total - 1 ? units : unit_of(hi) + 1;
  }
  const int p = prefix <= 0 ? 0 : prefix >= total ? units : unit_of(prefix - 1) + 1;
  if (p >= s.b) {  // one range
    s.a = max(p, s.e);
    s.b = s.e = s.a;
  } else {
    s.a = p;
  }
  return s;
}

// What a row of the tile may see and how it is biased.
struct RowRule {
  int64_t pos;   // its position
  int lo, hi;    // visible positions besides the prefix (clamped to -1 .. kFar)
  int ns;        // its document (negative: none)
  float slope;   // log2(e) times the head's slope
};

__device__ __forceinline__ RowRule row_rule(const AttendArgs& a, const Tile& t, int ctx, int g, int group, int r) {
  RowRule x;
  const int j = r / group, h = g * group + r % group;
  const int at = t.q0 + j;
  x.pos = a.q_pos ? a.q_pos[at] : static_cast<int64_t>(ctx) - t.nq + j;
  x.hi = a.causal ? static_cast<int>(min(max(x.pos, int64_t{-1}), static_cast<int64_t>(kFar))) : kFar;
  x.lo = a.window ? static_cast<int>(min(max(x.pos - a.window + 1, int64_t{0}), static_cast<int64_t>(kFar))) : 0;
  x.ns = a.chunk_ns ? a.query_ns[at] : 0;
  x.slope = a.slopes ? a.slopes[h] * kLog2e : 0.f;
  return x;
}

// What the rows of a tile see: any of them, and all of them.
struct TileRule {
  int lo, hi, ns_lo, ns_hi;  // some row sees positions lo .. hi, of documents ns_lo .. ns_hi
  int lo_all, hi_all;        // every row sees positions lo_all .. hi_all
  bool mixed;                // rows differ in their documents

  // Whether every row sees 32 positions from p on.
  __device__ __forceinline__ bool all_see(int p, int prefix) const {
    return !mixed && (p + kUnit <= prefix || (p >= lo_all && p + kUnit - 1 <= hi_all));
  }
};

// The rule of a tile whose rows are spread over the lanes of each wave (one or two a lane, repeats allowed).
template <int R>
__device__ __forceinline__ TileRule tile_rule(const AttendArgs& a, const Tile& t, int ctx, int g, int group) {
  TileRule x{kFar, -1, INT32_MAX, -1, 0, kFar, false};
  if (!a.causal && !a.window && !a.chunk_ns) return TileRule{0, kFar, 0, 0, 0, kFar, false};
  const int lane = threadIdx.x & 63;
  bool none = false;
#pragma unroll
  for (int i = 0; i < (R + 63) / 64; ++i) {
    const RowRule r = row_rule(a, t, ctx, g, group, t.r0 + min(lane + 64 * i, t.rows - 1));
    x.lo = min(x.lo, r.lo);
    x.hi = max(x.hi, r.hi);
    x.lo_all = max(x.lo_all, r.lo);
    x.hi_all = min(x.hi_all, r.hi);
    none |= r.ns < 0;
    if (r.ns >= 0) {
      x.ns_lo = min(x.ns_lo, r.ns);
      x.ns_hi = max(x.ns_hi, r.ns);
    }
  }
  // the same in every lane: scalar registers, and branches that the whole wave takes
  x.lo = wave_min(x.lo);
  x.hi = wave_max(x.hi);
  x.lo_all = wave_max(x.lo_all);
  x.hi_all = wave_min(x.hi_all);
  x.ns_lo = wave_min(x.ns_lo);
  x.ns_hi = wave_max(x.ns_hi);
  x.mixed = __any(none) || x.ns_lo != x.ns_hi;
  return x;
}

// Resolve units last, last - 1, ... (n of them, at most MAX) of the span into `list`, leaving out those that hold
// nothing or are of no row's document.  Returns how many there are; ends with a barrier.  head_at: start of the
// workgroup's head in a page, `row_bytes`: of a row's codes.  With
// SLOTS a unit's `at` is its number among the request's units instead.
template <int MAX, int THREADS = kThreads, bool SLOTS = false>
__device__ __forceinline__ int resolve_units(const AttendArgs& a, const ChunkList& L, const Span& span,
                                             const TileRule& tr, int prefix, int64_t head_at, int row_bytes, int last,
                                             int n, Unit* list, int* counts) {
  constexpr int kPer = (MAX + THREADS - 1) / THREADS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  Unit x[kPer];
  uint64_t kept[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int i = j * THREADS + tid;
    x[j] = Unit{0, 0, 0, 0};
    bool ok = false;
    if (i < n) {
      const int u = span.unit(last - i);
      const int c = find_entry(L.ub, L.k, u);
      const int t = (u - L.ub[c]) * kUnit;
      const int32_t id = L.cid[c];
      const int p = t / a.kv.page_tokens;
      const int32_t pg = a.kv.table[static_cast<int64_t>(id) * a.kv.ppc + p];
      const int row = t - p * a.kv.page_tokens, held = min(kUnit, L.tb[c + 1] - L.tb[c] - t);
      x[j].ns = a.chunk_ns ? a.chunk_ns[id] : 0;
      x[j].pos = L.tb[c] + t;
      x[j].at = SLOTS ? u : pg * a.kv.page_bytes + head_at + row * row_bytes;
      x[j].where = row | held << 16 | (held < kUnit || !tr.all_see(x[j].pos, prefix) ? Unit::kMasked : 0);
      ok = pg >= 0 && pg < a.kv.n_pages && x[j].ns >= 0 && x[j].ns >= tr.ns_lo && x[j].ns <= tr.ns_hi;
    }
    kept[j] = __ballot(ok);
    if (lane == 0) counts[j * (THREADS / 64) + wave] = __builtin_popcountll(kept[j]);
  }
  __syncthreads();
  int total = 0, at[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    for (int w = 0; w < (THREADS / 64); ++w) {
      if (w == wave) at[j] = total;
      total += counts[j * (THREADS / 64) + w];
    }
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if ((kept[j] >> lane) & 1u) list[at[j] + __builtin_popcountll(kept[j] & ((uint64_t{1} << lane) - 1))] = x[j];
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(total);
}

// A unit of the list in scalar registers.
__device__ __forceinline__ Unit uniform_unit(const Unit& x) {
  Unit u;
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x.at));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x.at >> 32));
  u.at = static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
  u.where = __builtin_amdgcn_readfirstlane(x.where);
  u.pos = __builtin_amdgcn_readfirstlane(x.pos);
  u.ns = __builtin_amdgcn_readfirstlane(x.ns);
  return u;
}

// ---------------------------------------------------------------- pieces of rows

template <int FMT, int D>
struct Dim {
  static constexpr int kRow = kv_row_bytes(FMT, D);
  static constexpr int kSc = kv_scale_bytes(FMT, D);
  static constexpr int kElems = D / 4;         // elements of a quarter row
  static constexpr int kBytes = kRow / 4;      // bytes of a quarter row's codes
  static constexpr int kWords = kBytes / 4;
  static constexpr int kSteps = D / 32;        // 8-element steps of a quarter row
};

// A quarter of a token's row: its codes and the scale bytes of its blocks (low byte first).
template <int FMT, int D>
struct Piece {
  uint32_t w[Dim<FMT, D>::kWords];
  uint32_t sc;
};

template <int FMT, int D>
__device__ __forceinline__ void load_piece(Piece<FMT, D>& p, const uint8_t* codes, const uint8_t* scales) {
  using K = Dim<FMT, D>;
  if constexpr (K::kWords == 2) {
    const u32x2_t v = *reinterpret_cast<const u32x2_t*>(codes);
    p.w[0] = v[0];
    p.w[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < K::kWords / 4; ++i) {
      const u32x4_t v = reinterpret_cast<const u32x4_t*>(codes)[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) p.w[4 * i + j] = v[j];
    }
  }
  if constexpr (FMT == MEM_KV_BF16) {
    p.sc = 0;
  } else if constexpr (K::kElems > kKvBlock) {
    p.sc = *reinterpret_cast<const uint16_t*>(scales);
  } else {
    p.sc = *scales;
  }
}

__device__ __forceinline__ uint32_t bits_of(bf16x2 v) { return __builtin_bit_cast(uint32_t, v); }

// Elements 8 i .. 8 i + 7 of a piece as bf16.
template <int FMT, int D>
__device__ __forceinline__ u32x4_t piece_step(const Piece<FMT, D>& p, int i) {
  u32x4_t o;
  if constexpr (FMT == MEM_KV_BF16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = p.w[4 * i + j];
  } else {
    const float s = kv_scale(Dim<FMT, D>::kElems > kKvBlock ? (i >= 4 ? p.sc >> 8 : p.sc & 255u) : p.sc);
    if constexpr (FMT == MEM_KV_FP4) {
      const uint32_t c = p.w[i];
      o[0] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
      o[1] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
      o[2] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
      o[3] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        o[2 * j] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(p.w[2 * i + j], s, false));
        o[2 * j + 1] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(p.w[2 * i + j], s, true));
      }
    }
  }
  return o;
}

// Whether a piece holds a value that is not finite, or may: scales above those that mem_kv_write gives can take a code
// out of range.
template <int FMT, int D>
__device__ __forceinline__ bool piece_bad(const Piece<FMT, D>& p) {
  bool bad = false;
  if constexpr (FMT != MEM_KV_BF16) bad = max(p.sc & 255u, p.sc >> 8) > kMaxScaleByte<FMT>;
  if constexpr (FMT == MEM_KV_FP8) {
#pragma unroll
    for (int i = 0; i < Dim<FMT, D>::kWords; ++i)
      bad |= (((p.w[i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
  }
  if constexpr (FMT == MEM_KV_BF16) {
    u16x2 most = {0, 0};
#pragma unroll
    for (int i = 0; i < Dim<FMT, D>::kWords; ++i)
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, p.w[i] & 0x7FFF7FFFu));
    bad = most[0] >= 0x7F80u || most[1] >= 0x7F80u;
  }
  return bad;
}

template <int FMT, int D>
__device__ __forceinline__ void piece_clear(Piece<FMT, D>& p) {
#pragma unroll
  for (int i = 0; i < Dim<FMT, D>::kWords; ++i) p.w[i] = 0;
  p.sc = 0x7F7F;
}

// Four rows (4 lanes each, 8 bytes a lane) of a 16-column block of LDS, transposed: lane i of each 16 gets column i.
__device__ __forceinline__ u32x2_t lds_transpose4(const uint16_t* p) {
  typedef __attribute__((address_space(3))) s16x4* Lds;
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p)));
}

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4_t v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const bf16x2 p = {static_cast<__bf16>(x), static_cast<__bf16>(y)};
  return bits_of(p);
}

// What rounding x and y to the bf16 values of `pair` left, in bf16.
__device__ __forceinline__ uint32_t rest2(float x, float y, uint32_t pair) {
  return pack2(x - __uint_as_float(pair << 16), y - __uint_as_float(pair & 0xFFFF0000u));
}

// Maximum that keeps a NaN: a score that is not a number must not be passed over.
__device__ __forceinline__ float nan_max(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// Reductions over lanes l, l ^ 32, and with WIDTH 16 l ^ 16 and l ^ 48 too: the lanes that hold one row's scores.
template <int WIDTH>
__device__ __forceinline__ float max_column(float x) {
  if constexpr (WIDTH == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = nan_max(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return nan_max(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int WIDTH>
__device__ __forceinline__ float sum_column(float x) {
  if constexpr (WIDTH == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int WIDTH>
__device__ __forceinline__ bool any_column(bool x, int col) {
  uint64_t v = __ballot(x);
  v |= v >> 32;
  if constexpr (WIDTH == 16) v |= v >> 16;
  return (v >> col) & 1u;
}

// Offset in its unit of score j of a lane whose part (lane / WIDTH) is 0; part x adds 4 x.
template <int WIDTH>
__device__ constexpr int score_token(int j) {
  return WIDTH == 16 ? 16 * (j >> 2) + (j & 3) : 8 * (j >> 2) + (j & 3);
}

// Tokens of a unit that a row sees, as bits.
__device__ __forceinline__ uint32_t visible_tokens(const RowRule& rule, const Unit& u, int prefix) {
  auto below = [](int n) { return n <= 0 ? 0u : n >= kUnit ? ~0u : (1u << n) - 1; };
  const uint32_t near = below(rule.hi - u.pos + 1) & ~below(rule.lo - u.pos);
  return u.ns == rule.ns ? (near | below(prefix - u.pos)) & below(u.held()) : 0;
}

// Scores of the tokens that a row does not see become -inf.
template <int WIDTH, int N, typename V>
__device__ __forceinline__ void mask_scores(V& s, uint32_t seen, int part) {
  seen >>= 4 * part;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint32_t keep = static_cast<uint32_t>(static_cast<int32_t>(seen << (31 - score_token<WIDTH>(j))) >> 31);
    const float x = s[j];
    s[j] = __uint_as_float((__float_as_uint(x) & keep) | (0xFF800000u & ~keep));
  }
}

// Running softmax of a row, in every lane that holds its scores: maximum (it may lag by kLag: weights up to 2^kLag
// cost no precision and spare most rescalings) and the lane's part of the sum of weights.
struct RowState {
  float m;
  float l;
};
constexpr float kLag = 8.f;
// The weights are rounded to bf16 for the second product.  Where one weighs more than 1 / kHeavy of its lane's sum so
// far, rounding it would show in the output, and the product is made a second time with what the rounding left (16
// bits of weight in all); smaller weights' roundings average out.  The sum is that of the unrounded ones.
constexpr float kHeavy = 4.f;

__device__ __forceinline__ float inverse_sum(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN; }
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

// Output rows of a wave: O^T in the layout of the products, `col` = row, NACC registers.
template <int WIDTH, int D>
struct Rows {
  static constexpr int kBlocks = D / WIDTH;           // products along D
  static constexpr int kRegs = WIDTH == 16 ? 4 : 16;  // registers per product
  typedef float Acc __attribute__((ext_vector_type(kRegs)));
  Acc o[kBlocks];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < kBlocks; ++n)
#pragma unroll
      for (int j = 0; j < kRegs; ++j) o[n][j] = 0.f;
  }
  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) o[n] *= f;
  }
  // Four consecutive columns d = 4 part + (16 n, or 32 n + 8 y) at a time.
  template <typename F>
  __device__ __forceinline__ void each4(int part, F f) const {
#pragma unroll
    for (int n = 0; n < kBlocks; ++n)
#pragma unroll
      for (int y = 0; y < kRegs / 4; ++y)
        f(n * WIDTH + 8 * y + 4 * part, f32x4{o[n][4 * y], o[n][4 * y + 1], o[n][4 * y + 2], o[n][4 * y + 3]});
  }
};

// Whether a unit with this largest score has to be weighed: if it is masked, and its values that are not finite have
// been noted and cleared, only where some score of the wave is above -inf; else always (what weighs little or nothing
// is not left out: its values may be large, or no numbers).  Raises the running maximum if it has to.
template <int WIDTH, int D>
__device__ __forceinline__ bool raise(float top, bool masked, RowState& st, Rows<WIDTH, D>& rows) {
  if (!__any(!masked || top != -INFINITY)) return false;
  if (__any(top > st.m + kLag)) {
    const float mn = fmaxf(st.m, top);
    const float r = mn == -INFINITY ? 1.f : fast_exp2(st.m - mn);
    st.l *= r;
    rows.scale(r);
    st.m = mn;
  }
  return true;
}
__device__ __forceinline__ bool is_heavy(float top, const RowState& st) {
  return __any(fast_exp2(top - finite_max(st.m)) * kHeavy > st.l);
}

template <int N>
__device__ __forceinline__ float max_of(const float (&s)[N]) {
  float top = s[0];
#pragma unroll
  for (int j = 1; j < N; ++j) top = nan_max(top, s[j]);
  return top;
}

// The queries of a lane's row: kSteps operands of eight elements, `stride` elements apart.
template <int STEPS>
__device__ __forceinline__ void load_queries(const uint16_t* src, int stride, bf16x8 (&q)[STEPS]) {
  const bool vec = (reinterpret_cast<uintptr_t>(src) & 15u) == 0;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    union { u32x4_t v; uint16_t h[8]; } x;
    if (vec) {
      x.v = *reinterpret_cast<const u32x4_t*>(src + stride * i);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x.h[j] = src[stride * i + j];
    }
    q[i] = as_bf16x8(x.v);
  }
}

// What is written before this is issued before it.
__device__ __forceinline__ void issue_first() { __builtin_amdgcn_sched_barrier(0); }

// N weights as operands of the second product, and what their rounding left.
template <int N, typename V>
__device__ __forceinline__ void pack_weights(const V& s, u32x4_t (&w)[N / 8]) {
#pragma unroll
  for (int j = 0; j < N / 2; ++j) w[j >> 2][j & 3] = pack2(s[2 * j], s[2 * j + 1]);
}
template <int N, typename V>
__device__ __forceinline__ void pack_rests(const V& s, const u32x4_t (&w)[N / 8], u32x4_t (&rest)[N / 8]) {
#pragma unroll
  for (int j = 0; j < N / 2; ++j) rest[j >> 2][j & 3] = rest2(s[2 * j], s[2 * j + 1], w[j >> 2][j & 3]);
}

__device__ __forceinline__ float wave_sum_f32(float x) {
  x += __uint_as_float(dpp_u32<0xB1>(__float_as_uint(x)));
  x += __uint_as_float(dpp_u32<0x4E>(__float_as_uint(x)));
  x += __uint_as_float(dpp_u32<0x141>(__float_as_uint(x)));
  x += __uint_as_float(dpp_u32<0x140>(__float_as_uint(x)));
  return (lane_f32(x, 0) + lane_f32(x, 16)) + (lane_f32(x, 32) + lane_f32(x, 48));
}

// Values in LDS: bf16 rows whose pitch puts the four (WIDTH 32) or eight (16) rows that a transposing read takes
// together on different banks; the 16-byte chunks of a row are exchanged within the 64 (32) bytes that such a read
// takes of it, by the row's number shifted right by SHIFT, so that the writes meet different banks too.
template <int WIDTH, int D>
constexpr int kValuePitch = D + WIDTH;
template <int WIDTH, int SHIFT>
__device__ __forceinline__ int value_chunk(int row, int chunk) {
  return chunk ^ ((row >> SHIFT) & (WIDTH == 32 ? 3 : 1));
}

// Transposed operands of the values of 32 tokens in LDS rows at `rows`: operand n of WIDTH 16 is for the output columns
// 16 n .. + 15, of 32 for the columns 32 (n / 2) .. + 31 and every second 16 tokens.
template <int WIDTH, int D, int SHIFT>
struct ValueOps {
  static constexpr int kOps = D / WIDTH * (WIDTH == 16 ? 1 : 2);
  static constexpr int P = kValuePitch<WIDTH, D>;
  const uint16_t* src[WIDTH == 16 ? 1 : 4];

  __device__ __forceinline__ ValueOps(const uint16_t* rows, int lane) {
    static_assert(WIDTH != 16 || SHIFT <= 3, "rows 16 apart have the same exchange");
    const int i = lane & 15;
    if constexpr (WIDTH == 16) {
      const int r = 4 * (lane >> 4) + (i >> 2);  // rows r and r + 16, columns 16 n + 4 (i & 3)
      src[0] = rows + r * P + 8 * value_chunk<16, SHIFT>(r, (i & 3) >> 1) + 4 * (i & 1);
    } else {
      // rows r + 8 y, columns 32 n + 16 (lane >> 4 & 1) + 4 (i & 3)
      const int r = 4 * (lane >> 5) + (i >> 2), c = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
#pragma unroll
      for (int y = 0; y < 4; ++y)
        src[y] = rows + (r + 8 * y) * P + 8 * value_chunk<32, SHIFT>(r + 8 * y, c) + 4 * (i & 1);
    }
  }
  __device__ __forceinline__ bf16x8 operator[](int n) const {
    if constexpr (WIDTH == 16) return pair(src[0] + 16 * n, src[0] + 16 * P + 16 * n);
    else return pair(src[2 * (n & 1)] + 32 * (n >> 1), src[2 * (n & 1) + 1] + 32 * (n >> 1));
  }
  // O^T += V^T P^T for operand n, with the weights of the lane's row.
  static __device__ __forceinline__ void multiply(Rows<WIDTH, D>& out, int n, bf16x8 v, const u32x4_t* w) {
    if constexpr (WIDTH == 16) {
      out.o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, as_bf16x8(w[0]), out.o[n], 0, 0, 0);
    } else {
      auto& o = out.o[n >> 1];
      o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, as_bf16x8(w[n & 1]), o, 0, 0, 0);
    }
  }

 private:
  static __device__ __forceinline__ bf16x8 pair(const uint16_t* p0, const uint16_t* p1) {
    const u32x2_t v0 = lds_transpose4(p0), v1 = lds_transpose4(p1);
    return as_bf16x8(u32x4_t{v0[0], v0[1], v1[0], v1[1]});
  }
};

// Write a row's output, or its part of a split context.
template <int WIDTH, int D>
__device__ __forceinline__ void write_rows(const AttendArgs& a, const Rows<WIDTH, D>& rows, RowState st, bool poison,
                                           int64_t at, int part, int split, int splits, float* part_o,
                                           RowState* part_ml) {
  if (splits == 1) {
    const float inv = poison ? NAN : inverse_sum(st.l);
    uint16_t* dst = a.out + at * D;
    rows.each4(part, [&](int d, f32x4 v) {
      *reinterpret_cast<u32x2_t*>(dst + d) = u32x2_t{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
    });
    if (a.lse && part == 0) a.lse[at] = lse_of(st.m, st.l);
  } else {
    const int64_t slot = static_cast<int64_t>(split) * a.total_q * a.hq + at;
    float* dst = part_o + slot * D;
    rows.each4(part, [&](int d, f32x4 v) {
      if (poison) v = f32x4{NAN, NAN, NAN, NAN};
      *reinterpret_cast<f32x4*>(dst + d) = v;
    });
    if (part == 0) part_ml[slot] = st;
  }
}

// ---------------------------------------------------------------- joining splits

constexpr int kMaxSplits = 64;  // one lane of the join each

// A row's partial results, weighed and added by W waves (1: four rows a workgroup): lane s of every wave weighs split
// s, wave w adds splits w, w + W, ..., whose outputs are on their way before the weights are known; then the waves'
// sums are added in order.  One wave a row where there are few splits (kJoinSplits): 32 requests of 96 rows in a few
// splits 148 us, with four waves a row 162; bound by its two launches' worth of latency (3 to 5 us).
constexpr int kJoinSplits = 8;
template <int D, int W>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a, int splits,
                                                               const float* __restrict__ part_o,
                                                               const RowState* __restrict__ part_ml) {
  constexpr int kPer = D / 64, kBatch = 8;
  __shared__ float sums[W == 1 ? 1 : W][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = W == 1 ? 0 : wave;
  const int64_t rows = a.total_q * a.hq, at = W == 1 ? static_cast<int64_t>(blockIdx.x) * kWaves + wave : blockIdx.x;
  if (at >= rows) return;
  if (a.q_offsets) {  // rows that no request owns were not computed
    const int64_t j = at / a.hq;
    if (j < a.q_offsets[0] || j >= a.q_offsets[a.m]) return;
  }
  RowState st{-INFINITY, 0.f};
  if (lane < splits) st = part_ml[lane * rows + at];
  float v[kBatch][kPer];
  auto load = [&](int s0) {  // (past the last split: the last one again, so that loads stand behind no condition)
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float* src = part_o + (min(s0 + W * u, splits - 1) * rows + at) * D + lane * kPer;
#pragma unroll
      for (int x = 0; x < kPer; ++x) v[u][x] = src[x];
    }
  };
  load(first);
  const float m = wave_max_f32(st.m);
  const float f = fast_exp2(st.m - finite_max(m));
  const float l = wave_sum_f32(f * st.l);
  float o[kPer] = {};
  for (int s0 = first; s0 < splits; s0 += W * kBatch) {
    if (s0 != first) load(s0);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (s0 + W * u >= splits) continue;
      const float w = lane_f32(f, s0 + W * u);
#pragma unroll
      for (int x = 0; x < kPer; ++x) o[x] += w * v[u][x];
    }
  }
  const float inv = inverse_sum(l);
  if (W == 1) {
    __bf16* dst = reinterpret_cast<__bf16*>(a.out + at * D + lane * kPer);
#pragma unroll
    for (int x = 0; x < kPer; ++x) dst[x] = static_cast<__bf16>(o[x] * inv);
    if (a.lse && lane == 0) a.lse[at] = lse_of(m, l);
    return;
  }
#pragma unroll
  for (int x = 0; x < kPer; ++x) sums[wave][lane * kPer + x] = o[x];
  __syncthreads();
  const int d = 2 * threadIdx.x;
  if (d < D) {
    float y[2] = {0.f, 0.f};
    for (int w = 0; w < W; ++w) {
      y[0] += sums[w][d];
      y[1] += sums[w][d + 1];
    }
    *reinterpret_cast<uint32_t*>(a.out + at * D + d) = pack2(y[0] * inv, y[1] * inv);
  }
  if (a.lse && threadIdx.x == 0) a.lse[at] = lse_of(m, l);
}

inline int64_t join_groups(int64_t rows, int64_t splits) {
  return splits <= kJoinSplits ? (rows + kWaves - 1) / kWaves : rows;
}

}  // namespace

}  // namespace memattn
