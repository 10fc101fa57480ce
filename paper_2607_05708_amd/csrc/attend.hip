// Attention over the paged key/value cache.
//
// For each request and key/value head the rows are (new token, query head of
// the group); they share the head's keys and values, which are read once per
// tile of rows.  The context is walked in units of 32 tokens of one page, so
// every unit is one page lookup and ends inside a tile only at the end of a
// chunk.  A workgroup first turns its request's chunk list into units (a scan
// of the chunk lengths, then one lookup per unit), then streams them; the
// softmax keeps a running maximum and sum in the log2 domain, so keys and
// values are read once.  Long contexts with few rows are split over
// workgroups, whose partial results a second kernel joins in a fixed order.
//
// Both kernels compute S^T = K Q^T and O^T = V^T P^T: the products' columns
// are the rows, so the softmax of a row stays in the lanes that hold its
// column, and the weights leave the first product in the layout in which the
// second one reads them: P never moves between lanes.
//
//   attend_few_kernel   at most 16 rows a tile (single new tokens): 16x16x32
//     products; each wave streams its own units with no barrier.  A lane
//     loads a quarter of a token's row (16 bytes of 4-bit codes of 128
//     elements: exactly one block, so one scale) straight from the page into
//     the operand of the first product; values go through the wave's own LDS
//     rows once, as bf16, to be read back transposed.
//   attend_tile_kernel  tiles of 128 rows: 32x32x16 products; the workgroup
//     unpacks 64 tokens at a time into LDS for its four waves.
#include "kv.h"
#include "device_common.h"

namespace memattn {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kUnit = 32;        // tokens per unit
constexpr int kBatch = 512;      // units resolved at a time
constexpr int kFewRows = 16;     // rows per tile of the few-rows kernel
constexpr int kTileRows = 128;   // rows per tile of the tile kernel
constexpr int kTileTokens = 64;  // tokens per step of the tile kernel
constexpr int kFar = 1 << 30;    // above every position

// One unit of the context, resolved.
struct Unit {
  int32_t page;   // page of the pool (0 if `count` is 0)
  int32_t where;  // first row in the page | tokens held << 16
  int32_t pos;    // position of its first token
  int32_t ns;     // document of its chunk
};

// How a call is spread over the GPU (shared by the workspace size and the launch).
struct AttendPlan {
  bool few;
  int64_t tiles;  // row tiles (upper bound with ragged requests)
  int splits;
};

// ---------------------------------------------------------------- a workgroup's request, rows and units

struct Tile {
  int64_t req;
  int64_t q0;     // first query token of the request
  int nq;         // its new tokens
  int r0;         // first row of the tile among the request's rows
  int rows;       // rows in the tile
};

// Request and rows of tile t.  With ragged requests tile t of request i is tile floor(q_offsets[i] G / R) + i + t:
// these starts leave room for every request's ceil(n G / R) tiles without a scan; the tiles in between are empty.
__device__ __forceinline__ bool find_tile(const AttendArgs& a, int64_t t, int group, int R, Tile* out) {
  if (a.q_offsets) {
    int64_t lo = 0, hi = a.m - 1;
    while (lo < hi) {
      const int64_t mid = (lo + hi + 1) >> 1;
      const int64_t o = a.q_offsets[mid];
      if (o * group / R + mid <= t) lo = mid; else hi = mid - 1;
    }
    const int64_t o = a.q_offsets[lo], e = a.q_offsets[lo + 1];
    if (o < 0 || e > a.total_q || o > e) return false;
    out->req = lo;
    out->q0 = o;
    out->nq = static_cast<int>(e - o);
    t -= o * group / R + lo;
  } else {
    const int64_t nq = a.total_q / a.m;
    const int64_t per = (nq * group + R - 1) / R;
    out->req = t / per;
    out->q0 = out->req * nq;
    out->nq = static_cast<int>(nq);
    t -= out->req * per;
  }
  const int64_t r0 = t * R, rows = static_cast<int64_t>(out->nq) * group;
  if (t < 0 || r0 >= rows) return false;
  out->r0 = static_cast<int>(r0);
  out->rows = static_cast<int>(min(static_cast<int64_t>(R), rows - r0));
  return true;
}

// Scan of the request's chunk list: ub[c] / tb[c] = units / tokens before entry c; index k holds the totals.
__device__ __forceinline__ void scan_list(const AttendArgs& a, const int32_t* ids, int* ub, int* tb, int* tmp) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int cap = a.kv.ppc * a.kv.page_tokens;
  const int per = (a.k + kThreads - 1) / kThreads;
  const int c0 = min(tid * per, a.k), c1 = min(c0 + per, a.k);
  int u = 0, t = 0;
  for (int c = c0; c < c1; ++c) {
    const int32_t id = ids[c];
    const int len = id >= 0 && id < a.kv.n_chunks ? min(max(a.tok_len[id], 0), cap) : 0;
    ub[c] = u;
    tb[c] = t;
    u += (len + kUnit - 1) / kUnit;
    t += len;
  }
  int su = u, st = t;
  for (int off = 1; off < 64; off <<= 1) {
    const int pu = __shfl_up(su, off), pt = __shfl_up(st, off);
    if (lane >= off) { su += pu; st += pt; }
  }
  if (lane == 63) {
    tmp[2 * wave] = su;
    tmp[2 * wave + 1] = st;
  }
  __syncthreads();
  int bu = su - u, bt = st - t, total_u = 0, total_t = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) { bu += tmp[2 * w]; bt += tmp[2 * w + 1]; }
    total_u += tmp[2 * w];
    total_t += tmp[2 * w + 1];
  }
  for (int c = c0; c < c1; ++c) {
    ub[c] += bu;
    tb[c] += bt;
  }
  if (tid == 0) {
    ub[a.k] = total_u;
    tb[a.k] = total_t;
  }
  __syncthreads();
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
__device__ __forceinline__ Span visible_units(const int* ub, const int* tb, int k, int prefix, int lo, int hi) {
  const int total = tb[k];
  auto unit_of = [&](int pos) {  // unit that holds position pos < total
    const int c = find_entry(tb, k, pos);
    return ub[c] + (pos - tb[c]) / kUnit;
  };
  Span s{0, 0, 0};
  hi = min(hi, total - 1);
  lo = max(lo, 0);
  if (lo <= hi) {
    s.b = lo > 0 ? unit_of(lo) : 0;
    s.e = hi == total - 1 ? ub[k] : unit_of(hi) + 1;
  }
  const int p = prefix <= 0 ? 0 : prefix >= total ? ub[k] : unit_of(prefix - 1) + 1;
  if (p >= s.b) {  // one range
    s.a = max(p, s.e);
    s.b = s.e = s.a;
  } else {
    s.a = p;
  }
  return s;
}

// Resolve units [first, first + n) of the span into `list`.
__device__ __forceinline__ void resolve_units(const AttendArgs& a, const int32_t* ids, const int* ub, const int* tb,
                                              const Span& span, int first, int n, Unit* list) {
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int u = span.unit(first + i);
    const int c = find_entry(ub, a.k, u);
    const int t = (u - ub[c]) * kUnit;
    const int32_t id = ids[c];
    const int p = t / a.kv.page_tokens;
    const int32_t pg = a.kv.table[static_cast<int64_t>(id) * a.kv.ppc + p];
    const bool ok = pg >= 0 && pg < a.kv.n_pages;
    const int held = ok ? min(kUnit, tb[c + 1] - tb[c] - t) : 0;
    Unit x;
    x.page = ok ? pg : 0;
    x.where = (t - p * a.kv.page_tokens) | held << 16;
    x.pos = tb[c] + t;
    x.ns = a.chunk_ns ? a.chunk_ns[id] : 0;
    list[i] = x;
  }
}

// What a row of the tile may see and how it is biased.
struct RowRule {
  int64_t pos;   // its position
  int lo, hi;    // visible positions besides the prefix
  int ns;        // its document (negative: none)
  float slope;   // log2(e) times the head's slope
};

__device__ __forceinline__ RowRule row_rule(const AttendArgs& a, const Tile& t, int ctx, int g, int group, int r) {
  RowRule x;
  const int j = r / group, h = g * group + r % group;
  const int64_t at = t.q0 + j;
  x.pos = a.q_pos ? a.q_pos[at] : static_cast<int64_t>(ctx) - t.nq + j;
  x.hi = a.causal ? static_cast<int>(min(x.pos, static_cast<int64_t>(kFar))) : kFar;
  x.lo = a.window ? static_cast<int>(min(max(x.pos - a.window + 1, int64_t{0}), static_cast<int64_t>(kFar))) : 0;
  x.ns = a.chunk_ns ? a.query_ns[at] : 0;
  x.slope = a.slopes ? a.slopes[h] * kLog2e : 0.f;
  return x;
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

// Whether a piece holds a value that is not finite.
template <int FMT, int D>
__device__ __forceinline__ bool piece_bad(const Piece<FMT, D>& p) {
  bool bad = false;
  if constexpr (FMT != MEM_KV_BF16) bad = (p.sc & 255u) == 255u || (p.sc >> 8) == 255u;
  if constexpr (FMT == MEM_KV_FP8) {
#pragma unroll
    for (int i = 0; i < Dim<FMT, D>::kWords; ++i)
      bad |= (((p.w[i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
  }
  if constexpr (FMT == MEM_KV_BF16) {
#pragma unroll
    for (int i = 0; i < Dim<FMT, D>::kWords; ++i)
      bad |= (p.w[i] & 0x7F80u) == 0x7F80u || (p.w[i] & 0x7F800000u) == 0x7F800000u;
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

// c plus both bf16 values of a word.
__device__ __forceinline__ float add_pair(uint32_t pair, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u), c,
                                         false);
}

// What rounding x and y to the bf16 values of `pair` left, in bf16.
__device__ __forceinline__ uint32_t rest2(float x, float y, uint32_t pair) {
  return pack2(x - __uint_as_float(pair << 16), y - __uint_as_float(pair & 0xFFFF0000u));
}

// Reductions over lanes l, l ^ 16, l ^ 32, l ^ 48 (column l & 15) and over l, l ^ 32.
__device__ __forceinline__ float max_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_rows(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_half(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_rows(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return sum_half(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// log2-domain score of a raw product: scale, cap, without the bias.  tanh(x) = 1 - 2 / (1 + e^2x).
struct Scores {
  float c;     // scale * log2(e), or with a cap 2 * scale * log2(e) / cap
  float cap2;  // cap * log2(e); 0: none
  __device__ __forceinline__ float operator()(float s) const {
    if (cap2 == 0.f) return s * c;
    return cap2 - 2.f * cap2 * __builtin_amdgcn_rcpf(1.f + fast_exp2(s * c));
  }
};

__device__ __forceinline__ Scores scores_of(const AttendArgs& a) {
  if (a.softcap > 0.f) return {2.f * a.scale * kLog2e / a.softcap, a.softcap * kLog2e};
  return {a.scale * kLog2e, 0.f};
}

// The weights are rounded to bf16 for the second product.  Where one weighs more than 1 / kHeavy of its lane's sum so
// far, rounding it would show in the output, and the product is made a second time with what the rounding left (16
// bits of weight in all); smaller weights' roundings average out.  Outputs are divided by the sum `lr` of the weights
// as they were used, so that a common part of the rounding cancels; the lse takes the sum `l` of the unrounded ones.
constexpr float kHeavy = 16.f;

struct RowState {
  float m;   // maximum so far (may lag, below)
  float l;
  float lr;
};

__device__ __forceinline__ float inverse_sum(float lr) { return lr > 0.f ? 1.f / lr : lr == 0.f ? 0.f : NAN; }
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Running maxima may lag by this much (log2): weights up to 2^8 cost no precision and spare most rescalings.
constexpr float kLag = 8.f;

// ---------------------------------------------------------------- few rows

template <int FMT, int D>
struct FewShape {
  static constexpr int kPitch = D + 16;                                   // bf16 elements between LDS rows
  static constexpr int kWaveBytes = kUnit * kPitch * 2;                    // a wave's unpacked values
  static constexpr int kJoinBytes = kWaves * kFewRows * D * 4;             // the waves' outputs at the end
  static constexpr int kArea = kWaves * kWaveBytes > kJoinBytes ? kWaves * kWaveBytes : kJoinBytes;
};

template <int FMT, int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attend_few_kernel(AttendArgs a, int splits, float* __restrict__ part_o,
                                                              RowState* __restrict__ part_ml) {
  using K = Dim<FMT, D>;
  using S = FewShape<FMT, D>;
  constexpr int kBlocks = D / 16;
  extern __shared__ int dyn[];  // ub[k + 1], tb[k + 1]
  __shared__ __align__(16) uint8_t area[S::kArea];
  __shared__ Unit list[kBatch];
  __shared__ int tmp[2 * kWaves];
  __shared__ RowState wave_ml[kWaves][kFewRows];
  int* ub = dyn;
  int* tb = dyn + a.k + 1;

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, quad = lane >> 4;
  const int heads = a.kv.heads, group = a.hq / heads;
  int64_t b = blockIdx.x;
  const int g = static_cast<int>(b % heads);
  b /= heads;
  const int split = static_cast<int>(b % splits);
  Tile t;
  if (!find_tile(a, b / splits, group, kFewRows, &t)) return;
  const int32_t* ids = a.ids + t.req * a.k;
  scan_list(a, ids, ub, tb, tmp);
  const int ctx = tb[a.k];
  const int prefix = a.prefix_len ? a.prefix_len[t.req] : 0;
  const RowRule rule = row_rule(a, t, ctx, g, group, t.r0 + min(col, t.rows - 1));

  // what the tile's rows see at most
  int lo = rule.lo, hi = rule.hi;
  for (int off = 1; off < 16; off <<= 1) {
    lo = min(lo, __shfl_xor(lo, off));
    hi = max(hi, __shfl_xor(hi, off));
  }
  int lo_all = rule.lo, hi_all = rule.hi;  // what all of them see
  for (int off = 1; off < 16; off <<= 1) {
    lo_all = max(lo_all, __shfl_xor(lo_all, off));
    hi_all = min(hi_all, __shfl_xor(hi_all, off));
  }
  const Span span = visible_units(ub, tb, a.k, prefix, lo, hi);
  const int n_units = span.count();
  const int u0 = static_cast<int>(static_cast<int64_t>(n_units) * split / splits);
  const int u1 = static_cast<int>(static_cast<int64_t>(n_units) * (split + 1) / splits);

  // the tile's queries: lane (col, quad) holds quarter `quad` of row `col`
  bf16x8 q[K::kSteps];
  {
    const int r = t.r0 + min(col, t.rows - 1);
    const uint16_t* src = a.q + (t.q0 + r / group) * a.q_ts + (g * group + r % group) * a.q_hs + quad * K::kElems;
    const bool vec = (reinterpret_cast<uintptr_t>(src) & 15u) == 0;
#pragma unroll
    for (int i = 0; i < K::kSteps; ++i) {
      union { u32x4_t v; uint16_t h[8]; } x;
      if (vec) {
        x.v = *reinterpret_cast<const u32x4_t*>(src + 8 * i);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x.h[j] = src[8 * i + j];
      }
      q[i] = as_bf16x8(x.v);
    }
  }

  const Scores score = scores_of(a);
  const int64_t T = a.kv.page_tokens;
  const int64_t head_at = static_cast<int64_t>(g) * 2 * T * (K::kRow + K::kSc);
  const int my_codes = col * K::kRow + quad * K::kBytes;
  const int my_scale = col * K::kSc + quad * K::kElems / kKvBlock;
  uint16_t* vrows = reinterpret_cast<uint16_t*>(area + wave * S::kWaveBytes);

  f32x4 acc[kBlocks];
#pragma unroll
  for (int n = 0; n < kBlocks; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f, lr = 0.f;
  bool poison = false;

  struct Stage {
    Piece<FMT, D> k[2], v[2];
    Unit u;
  };
  auto load = [&](Stage& s, int i) {
    Unit u = list[i];
    u.page = __builtin_amdgcn_readfirstlane(u.page);
    u.where = __builtin_amdgcn_readfirstlane(u.where);
    u.pos = __builtin_amdgcn_readfirstlane(u.pos);
    u.ns = __builtin_amdgcn_readfirstlane(u.ns);
    s.u = u;
    const int row = u.where & 0xFFFF;
    const uint8_t* part = a.kv.pool + u.page * a.kv.page_bytes + head_at;
    const uint8_t* kc = part + row * K::kRow + my_codes;
    const uint8_t* ks = part + 2 * T * K::kRow + row * K::kSc + my_scale;
    if ((u.where >> 16) == 0) return;  // no page: nothing of the unit is used
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      load_piece<FMT, D>(s.k[h], kc + h * 16 * K::kRow, ks + h * 16 * K::kSc);
      load_piece<FMT, D>(s.v[h], kc + T * K::kRow + h * 16 * K::kRow, ks + T * K::kSc + h * 16 * K::kSc);
    }
  };

  for (int first = u0; first < u1; first += kBatch) {
    const int n = min(kBatch, u1 - first);
    __syncthreads();
    resolve_units(a, ids, ub, tb, span, first, n, list);
    __syncthreads();
    Stage cur, next;
    if (wave < n) load(cur, wave);
    for (int i = wave; i < n; i += kWaves) {
      if (i + kWaves < n) load(next, i + kWaves);
      const Unit u = cur.u;
      const int held = u.where >> 16;
      const int row_pos = u.pos + 4 * quad;  // position of the lane's first score
      // S^T of two blocks of 16 tokens: lane (col, quad) gets tokens 4 quad .. 4 quad + 3 of each
      f32x4 s[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < K::kSteps; ++x)
          s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(piece_step<FMT, D>(cur.k[h], x)), q[x], s[h], 0, 0, 0);
      }
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = score(s[j >> 2][j & 3]);
      if (a.slopes) {
        const float dist = static_cast<float>(rule.pos - row_pos);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] -= rule.slope * fabsf(dist - static_cast<float>(16 * (j >> 2) + (j & 3)));
      }
      // Masks: every token of the unit is seen by every row, or each score is looked at.
      const bool inside = u.pos + kUnit <= prefix || (u.pos >= lo_all && u.pos + kUnit - 1 <= hi_all);
      uint32_t bad = 0;  // tokens whose values are not finite
      bool dead[2] = {false, false};  // this lane's value rows that are not read
      uint32_t seen = 0xFFu;
      if (held < kUnit || a.chunk_ns || !inside) {
        seen = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int tok = 16 * (j >> 2) + 4 * quad + (j & 3), p = u.pos + tok;
          const bool see = tok < held && (p < prefix || (p >= rule.lo && p <= rule.hi)) && u.ns == rule.ns && u.ns >= 0;
          seen |= see ? 1u << j : 0u;
          x[j] = see ? x[j] : -INFINITY;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bool out = 16 * h + col >= held;
          const bool nf = !out && piece_bad<FMT, D>(cur.v[h]);
          const uint64_t vote = __ballot(nf);
          bad |= static_cast<uint32_t>((vote | vote >> 16 | vote >> 32 | vote >> 48) & 0xFFFFu) << (16 * h);
          dead[h] = out || nf;
        }
      }
      float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      top = max_rows(top);
      if (__any(top > m + kLag)) {
        const float mn = fmaxf(m, top);
        const float f = mn == -INFINITY ? 1.f : fast_exp2(m - mn);
        l *= f;
        lr *= f;
#pragma unroll
        for (int n2 = 0; n2 < kBlocks; ++n2) acc[n2] *= f;
        m = mn;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      u32x4_t pw;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = fast_exp2(x[j] - ref);
        l += x[j];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        pw[j] = pack2(x[2 * j], x[2 * j + 1]);
        lr = add_pair(pw[j], lr);
      }
      if (bad) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          poison |= ((seen >> j) & 1u) && ((bad >> (16 * (j >> 2) + 4 * quad + (j & 3))) & 1u);
      }
      // values: unpack into the wave's LDS rows, read back transposed
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (dead[h]) piece_clear<FMT, D>(cur.v[h]);
        uint16_t* dst = vrows + (16 * h + col) * S::kPitch + quad * K::kElems;
#pragma unroll
        for (int y = 0; y < K::kSteps; ++y) *reinterpret_cast<u32x4_t*>(dst + 8 * y) = piece_step<FMT, D>(cur.v[h], y);
      }
      __builtin_amdgcn_wave_barrier();
      const uint16_t* src = vrows + (4 * quad + (col >> 2)) * S::kPitch + (col & 3) * 4;
      auto add_values = [&](const u32x4_t& w) {
#pragma unroll
        for (int n2 = 0; n2 < kBlocks; ++n2) {
          const u32x2_t v0 = lds_transpose4(src + 16 * n2);
          const u32x2_t v1 = lds_transpose4(src + 16 * S::kPitch + 16 * n2);
          const u32x4_t v = {v0[0], v0[1], v1[0], v1[1]};
          acc[n2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v), as_bf16x8(w), acc[n2], 0, 0, 0);
        }
      };
      add_values(pw);
      if (__any(fast_exp2(top - ref) * kHeavy > l)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          pw[j] = rest2(x[2 * j], x[2 * j + 1], pw[j]);
          lr = add_pair(pw[j], lr);
        }
        add_values(pw);
      }
      __builtin_amdgcn_wave_barrier();
      cur = next;
    }
  }

  // join the waves in LDS, in wave order
  l = sum_rows(l);
  lr = sum_rows(lr);
  {
    const uint64_t v = __ballot(poison);
    poison = ((v | v >> 16 | v >> 32 | v >> 48) >> col) & 1u;
  }
  __syncthreads();  // every wave is done with its rows of `area`
  float* jo = reinterpret_cast<float*>(area);
  if (quad == 0) wave_ml[wave][col] = RowState{m, l, lr};
#pragma unroll
  for (int n = 0; n < kBlocks; ++n) {
    f32x4 o = acc[n];
    if (poison) o = f32x4{NAN, NAN, NAN, NAN};
    *reinterpret_cast<f32x4*>(jo + (wave * kFewRows + col) * D + 16 * n + 4 * quad) = o;
  }
  __syncthreads();
  constexpr int kPer = kFewRows * D / kThreads;  // outputs per thread, consecutive in a row
  const int r = tid / (D / kPer), c0 = (tid % (D / kPer)) * kPer;
  if (r >= t.rows) return;
  float mm = -INFINITY;
  for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, wave_ml[w][r].m);
  const float ref = mm == -INFINITY ? 0.f : mm;
  float ll = 0.f, llr = 0.f, o[kPer] = {};
  for (int w = 0; w < kWaves; ++w) {
    const RowState st = wave_ml[w][r];
    const float f = fast_exp2(st.m - ref);
    ll += f * st.l;
    llr += f * st.lr;
    for (int x = 0; x < kPer; ++x) o[x] += f * jo[(w * kFewRows + r) * D + c0 + x];
  }
  const int row = t.r0 + r;
  const int64_t at = (t.q0 + row / group) * a.hq + g * group + row % group;
  if (splits == 1) {
    const float inv = inverse_sum(llr);
    uint16_t* dst = a.out + at * D + c0;
    for (int x = 0; x < kPer; x += 4) {
      const u32x2_t v = {pack2(o[x] * inv, o[x + 1] * inv), pack2(o[x + 2] * inv, o[x + 3] * inv)};
      *reinterpret_cast<u32x2_t*>(dst + x) = v;
    }
    if (a.lse && c0 == 0) a.lse[at] = lse_of(mm, ll);
  } else {
    const int64_t slot = static_cast<int64_t>(split) * a.total_q * a.hq + at;
    for (int x = 0; x < kPer; x += 4)
      *reinterpret_cast<f32x4*>(part_o + slot * D + c0 + x) = f32x4{o[x], o[x + 1], o[x + 2], o[x + 3]};
    if (c0 == 0) part_ml[slot] = RowState{mm, ll, llr};
  }
}

// ---------------------------------------------------------------- joining splits

// One wave per row: the splits' sums, weighted by their maxima, in split order.
template <int D>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a, int splits,
                                                               const float* __restrict__ part_o,
                                                               const RowState* __restrict__ part_ml) {
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t rows = a.total_q * a.hq;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (at >= rows) return;
  if (a.q_offsets) {  // rows that no request owns were not computed
    const int64_t j = at / a.hq;
    if (j < a.q_offsets[0] || j >= a.q_offsets[a.m]) return;
  }
  float mm = -INFINITY;
  for (int s = 0; s < splits; ++s) mm = fmaxf(mm, part_ml[s * rows + at].m);
  const float ref = mm == -INFINITY ? 0.f : mm;
  float ll = 0.f, llr = 0.f, o[kPer] = {};
  for (int s = 0; s < splits; ++s) {
    const RowState st = part_ml[s * rows + at];
    const float f = fast_exp2(st.m - ref);
    ll += f * st.l;
    llr += f * st.lr;
    const float* src = part_o + (s * rows + at) * D + lane * kPer;
    for (int x = 0; x < kPer; ++x) o[x] += f * src[x];
  }
  const float inv = inverse_sum(llr);
  uint16_t* dst = a.out + at * D + lane * kPer;
  for (int x = 0; x < kPer; ++x) dst[x] = static_cast<uint16_t>(pack2(o[x] * inv, 0.f) & 0xFFFFu);
  if (a.lse && lane == 0) a.lse[at] = lse_of(mm, ll);
}

// ---------------------------------------------------------------- tiles of rows

template <int FMT, int D>
struct TileShape {
  static constexpr int kPitch = D + 8;                          // bf16 elements between LDS rows
  static constexpr int kPart = kTileTokens * kPitch * 2;        // bytes of a step's keys or values
  static constexpr int kLoads = kTileTokens * 4 / kThreads;     // quarter rows per thread, keys and values each
};

template <int FMT, int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attend_tile_kernel(AttendArgs a, int splits, int64_t tiles,
                                                               float* __restrict__ part_o,
                                                               RowState* __restrict__ part_ml) {
  using K = Dim<FMT, D>;
  using S = TileShape<FMT, D>;
  static_assert(S::kLoads == 1, "one quarter row of keys and one of values per thread and step");
  constexpr int kBlocks = D / 32, kQSteps = D / 16;
  extern __shared__ int dyn[];  // ub[k + 1], tb[k + 1]
  __shared__ __align__(16) uint8_t area[2 * S::kPart];
  __shared__ Unit list[kBatch];
  __shared__ int tmp[2 * kWaves];
  __shared__ uint32_t bad_tok[2][2];  // tokens whose values are not finite, of even and odd steps
  int* ub = dyn;
  int* tb = dyn + a.k + 1;
  uint16_t* krows = reinterpret_cast<uint16_t*>(area);
  uint16_t* vrows = reinterpret_cast<uint16_t*>(area + S::kPart);

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int heads = a.kv.heads, group = a.hq / heads;
  int64_t b = blockIdx.x;
  const int g = static_cast<int>(b % heads);
  b /= heads;
  const int split = static_cast<int>(b % splits);
  Tile t;
  if (!find_tile(a, tiles - 1 - b / splits, group, kTileRows, &t)) return;  // the latest rows see most: first
  const int32_t* ids = a.ids + t.req * a.k;
  scan_list(a, ids, ub, tb, tmp);
  const int ctx = tb[a.k];
  const int prefix = a.prefix_len ? a.prefix_len[t.req] : 0;
  const int my_row = min(32 * wave + col, t.rows - 1);
  const RowRule rule = row_rule(a, t, ctx, g, group, t.r0 + my_row);

  // what the tile's rows see at most, and what all of them see
  int lo = kFar, hi = -1, lo_all = 0, hi_all = kFar;
  for (int r = lane; r < t.rows; r += 64) {
    const RowRule x = row_rule(a, t, ctx, g, group, t.r0 + r);
    lo = min(lo, x.lo);
    hi = max(hi, x.hi);
    lo_all = max(lo_all, x.lo);
    hi_all = min(hi_all, x.hi);
  }
  for (int off = 1; off < 64; off <<= 1) {
    lo = min(lo, __shfl_xor(lo, off));
    hi = max(hi, __shfl_xor(hi, off));
    lo_all = max(lo_all, __shfl_xor(lo_all, off));
    hi_all = min(hi_all, __shfl_xor(hi_all, off));
  }
  const Span span = visible_units(ub, tb, a.k, prefix, lo, hi);
  const int n_units = span.count();
  const int u0 = static_cast<int>(static_cast<int64_t>(n_units) * split / splits);
  const int u1 = static_cast<int>(static_cast<int64_t>(n_units) * (split + 1) / splits);

  // queries: lane (col, half) holds elements 16 s + 8 half .. + 7 of row `col` of the wave
  bf16x8 q[kQSteps];
  {
    const int r = t.r0 + my_row;
    const uint16_t* src = a.q + (t.q0 + r / group) * a.q_ts + (g * group + r % group) * a.q_hs + 8 * half;
    const bool vec = (reinterpret_cast<uintptr_t>(src) & 15u) == 0;
#pragma unroll
    for (int i = 0; i < kQSteps; ++i) {
      union { u32x4_t v; uint16_t h[8]; } x;
      if (vec) {
        x.v = *reinterpret_cast<const u32x4_t*>(src + 16 * i);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x.h[j] = src[16 * i + j];
      }
      q[i] = as_bf16x8(x.v);
    }
  }

  const Scores score = scores_of(a);
  const int64_t T = a.kv.page_tokens;
  const int64_t head_at = static_cast<int64_t>(g) * 2 * T * (K::kRow + K::kSc);
  const int my_tok = tid >> 2, my_quarter = tid & 3;  // the quarter row this thread unpacks

  f32x16 acc[kBlocks];
#pragma unroll
  for (int n = 0; n < kBlocks; ++n)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[n][j] = 0.f;
  float m = -INFINITY, l = 0.f, lr = 0.f;
  bool poison = false;
  if (tid < 2) bad_tok[0][tid] = 0;
  int odd = 0;

  for (int first = u0; first < u1; first += kBatch) {
    const int n = min(kBatch, u1 - first);
    __syncthreads();
    resolve_units(a, ids, ub, tb, span, first, n, list);
    __syncthreads();
    Piece<FMT, D> pk, pv;
    bool out = true;
    auto load = [&](int i) {
      // the thread's token is in unit i + (my_tok >> 5); past the batch's end nothing is held
      const int x = i + (my_tok >> 5);
      const Unit u = list[min(x, n - 1)];
      const int row = (u.where & 0xFFFF) + (my_tok & 31);
      out = x >= n || (my_tok & 31) >= (u.where >> 16);
      if (out) {
        piece_clear<FMT, D>(pk);
        piece_clear<FMT, D>(pv);
        return;
      }
      const uint8_t* part = a.kv.pool + u.page * a.kv.page_bytes + head_at;
      const uint8_t* kc = part + row * K::kRow + my_quarter * K::kBytes;
      const uint8_t* ks = part + 2 * T * K::kRow + row * K::kSc + my_quarter * K::kElems / kKvBlock;
      load_piece<FMT, D>(pk, kc, ks);
      load_piece<FMT, D>(pv, kc + T * K::kRow, ks + T * K::kSc);
    };
    load(0);
    for (int i = 0; i < n; i += 2) {
      Unit u[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u[h] = list[min(i + h, n - 1)];
        u[h].where = __builtin_amdgcn_readfirstlane(u[h].where);
        u[h].pos = __builtin_amdgcn_readfirstlane(u[h].pos);
        u[h].ns = __builtin_amdgcn_readfirstlane(u[h].ns);
        if (i + h >= n) u[h].where = 0;
      }
      bool masked = a.chunk_ns != nullptr;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        masked |= (u[h].where >> 16) < kUnit ||
                  !(u[h].pos + kUnit <= prefix || (u[h].pos >= lo_all && u[h].pos + kUnit - 1 <= hi_all));
      __syncthreads();  // the last step's reads of the rows and of its bad_tok are done
      if (tid < 2) bad_tok[odd ^ 1][tid] = 0;
      if (masked && piece_bad<FMT, D>(pv)) {
        atomicOr(&bad_tok[odd][my_tok >> 5], 1u << (my_tok & 31));
        piece_clear<FMT, D>(pv);
      }
      uint16_t* kd = krows + my_tok * S::kPitch + my_quarter * K::kElems;
      uint16_t* vd = vrows + my_tok * S::kPitch + my_quarter * K::kElems;
#pragma unroll
      for (int y = 0; y < K::kSteps; ++y) {
        *reinterpret_cast<u32x4_t*>(kd + 8 * y) = piece_step<FMT, D>(pk, y);
        *reinterpret_cast<u32x4_t*>(vd + 8 * y) = piece_step<FMT, D>(pv, y);
      }
      __syncthreads();
      if (i + 2 < n) load(i + 2);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if ((u[h].where >> 16) == 0) continue;
        f32x16 s;
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = 0.f;
        const uint16_t* kr = krows + (32 * h + col) * S::kPitch + 8 * half;
#pragma unroll
        for (int x = 0; x < kQSteps; ++x)
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*reinterpret_cast<const u32x4_t*>(kr + 16 * x)), q[x],
                                                      s, 0, 0, 0);
        // lane (col, half) holds tokens 8 (j >> 2) + 4 half + (j & 3)
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = score(s[j]);
        if (a.slopes) {
          const float dist = static_cast<float>(rule.pos - u[h].pos - 4 * half);
#pragma unroll
          for (int j = 0; j < 16; ++j)
            s[j] -= rule.slope * fabsf(dist - static_cast<float>(8 * (j >> 2) + (j & 3)));
        }
        uint32_t seen = 0xFFFFu;
        if (masked) {
          const int held = u[h].where >> 16;
          seen = 0;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int tok = 8 * (j >> 2) + 4 * half + (j & 3), p = u[h].pos + tok;
            const bool see = tok < held && (p < prefix || (p >= rule.lo && p <= rule.hi)) && u[h].ns == rule.ns &&
                             u[h].ns >= 0;
            seen |= see ? 1u << j : 0u;
            s[j] = see ? s[j] : -INFINITY;
          }
        }
        float top = s[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) top = fmaxf(top, s[j]);
        top = max_half(top);
        if (__any(top > m + kLag)) {
          const float mn = fmaxf(m, top);
          const float f = mn == -INFINITY ? 1.f : fast_exp2(m - mn);
          l *= f;
          lr *= f;
#pragma unroll
          for (int n2 = 0; n2 < kBlocks; ++n2) acc[n2] *= f;
          m = mn;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        u32x4_t pw[2];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          s[j] = fast_exp2(s[j] - ref);
          l += s[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          pw[j >> 2][j & 3] = pack2(s[2 * j], s[2 * j + 1]);
          lr = add_pair(pw[j >> 2][j & 3], lr);
        }
        if (masked && bad_tok[odd][h]) {
          const uint32_t bad = bad_tok[odd][h];
#pragma unroll
          for (int j = 0; j < 16; ++j)
            poison |= ((seen >> j) & 1u) && ((bad >> (8 * (j >> 2) + 4 * half + (j & 3))) & 1u);
        }
        // lane (16 x + i, half): rows 4 half + (i >> 2) (+ 8) of each 16 tokens, columns 16 x ..
        const int i16 = lane & 15;
        const uint16_t* vr = vrows + (32 * h + 4 * half + (i16 >> 2)) * S::kPitch + ((lane >> 4) & 1) * 16 + (i16 & 3) * 4;
        auto add_values = [&]() {
#pragma unroll
          for (int n2 = 0; n2 < kBlocks; ++n2) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const u32x2_t v0 = lds_transpose4(vr + (16 * x) * S::kPitch + 32 * n2);
              const u32x2_t v1 = lds_transpose4(vr + (16 * x + 8) * S::kPitch + 32 * n2);
              const u32x4_t v = {v0[0], v0[1], v1[0], v1[1]};
              acc[n2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v), as_bf16x8(pw[x]), acc[n2], 0, 0, 0);
            }
          }
        };
        add_values();
        if (__any(fast_exp2(top - ref) * kHeavy > l)) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            pw[j >> 2][j & 3] = rest2(s[2 * j], s[2 * j + 1], pw[j >> 2][j & 3]);
            lr = add_pair(pw[j >> 2][j & 3], lr);
          }
          add_values();
        }
      }
      odd ^= 1;
    }
  }

  l = sum_half(l);
  lr = sum_half(lr);
  {
    const uint64_t v = __ballot(poison);
    poison = ((v | v >> 32) >> col) & 1u;
  }
  const int r = 32 * wave + col;
  if (r >= t.rows) return;
  const int row = t.r0 + r;
  const int64_t at = (t.q0 + row / group) * a.hq + g * group + row % group;
  float inv = inverse_sum(lr);
  if (poison) inv = NAN;
  if (splits == 1) {
    uint16_t* dst = a.out + at * D + 4 * half;
#pragma unroll
    for (int n = 0; n < kBlocks; ++n)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const u32x2_t v = {pack2(acc[n][4 * y] * inv, acc[n][4 * y + 1] * inv),
                           pack2(acc[n][4 * y + 2] * inv, acc[n][4 * y + 3] * inv)};
        *reinterpret_cast<u32x2_t*>(dst + 32 * n + 8 * y) = v;
      }
    if (a.lse && half == 0) a.lse[at] = lse_of(m, l);
  } else {
    const int64_t slot = static_cast<int64_t>(split) * a.total_q * a.hq + at;
    float* dst = part_o + slot * D + 4 * half;
#pragma unroll
    for (int n = 0; n < kBlocks; ++n)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        f32x4 v = {acc[n][4 * y], acc[n][4 * y + 1], acc[n][4 * y + 2], acc[n][4 * y + 3]};
        if (poison) v = f32x4{NAN, NAN, NAN, NAN};
        *reinterpret_cast<f32x4*>(dst + 32 * n + 8 * y) = v;
      }
    if (half == 0) part_ml[slot] = RowState{m, l, lr};
  }
}

// ---------------------------------------------------------------- launches

int64_t tile_count(const int32_t* q_offsets, int64_t m, int64_t total_q, int group, int R) {
  if (q_offsets) return total_q * group / R + m;
  return m * ((total_q / m * group + R - 1) / R);
}

// Rows per request decide the kernel: up to 16 (on average) the few-rows kernel.  A context is split when the tiles
// alone leave CUs idle, into parts of at least kMinPart tokens.
constexpr int64_t kWantFew = 2048, kWantTile = 512;
constexpr int64_t kMinPart = 512;

AttendPlan make_plan(int64_t m, int64_t capacity, int64_t total_q, int heads, int heads_q, bool ragged) {
  AttendPlan p;
  const int group = heads_q / heads;
  p.few = total_q * group <= kFewRows * m;
  const int32_t some = 0;
  p.tiles = tile_count(ragged ? &some : nullptr, m, total_q, group, p.few ? kFewRows : kTileRows);
  const int64_t have = p.tiles * heads, want = p.few ? kWantFew : kWantTile;
  int64_t s = (want + have - 1) / have;
  s = s < capacity / kMinPart ? s : capacity / kMinPart;
  p.splits = static_cast<int>(s < 1 ? 1 : s > 256 ? 256 : s);
  return p;
}

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

size_t partial_o_bytes(int d, int64_t total_q, int heads_q, int splits) {
  return align256(static_cast<size_t>(splits) * total_q * heads_q * d * sizeof(float));
}

template <int FMT, int D>
hipError_t launch_dim(const AttendArgs& a, const AttendPlan& p, hipStream_t stream) {
  float* po = static_cast<float*>(a.ws);
  RowState* pml = p.splits > 1 ? reinterpret_cast<RowState*>(static_cast<uint8_t*>(a.ws) +
                                                         partial_o_bytes(D, a.total_q, a.hq, p.splits))
                             : nullptr;
  const dim3 grid(static_cast<unsigned>(p.tiles * a.kv.heads * p.splits));
  const size_t lds = static_cast<size_t>(2) * (a.k + 1) * sizeof(int);
  if (p.few)
    attend_few_kernel<FMT, D><<<grid, kThreads, lds, stream>>>(a, p.splits, po, pml);
  else
    attend_tile_kernel<FMT, D><<<grid, kThreads, lds, stream>>>(a, p.splits, p.tiles, po, pml);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || p.splits == 1) return e;
  const int64_t rows = a.total_q * a.hq;
  attend_join_kernel<D><<<dim3(static_cast<unsigned>((rows + kWaves - 1) / kWaves)), kThreads, 0, stream>>>(
      a, p.splits, po, pml);
  return hipGetLastError();
}

template <int FMT>
hipError_t launch_fmt(const AttendArgs& a, const AttendPlan& p, int d, hipStream_t stream) {
  switch (d) {
    case 64: return launch_dim<FMT, 64>(a, p, stream);
    case 128: return launch_dim<FMT, 128>(a, p, stream);
    default: return launch_dim<FMT, 256>(a, p, stream);
  }
}

}  // namespace

// The larger of the two forms of a call (ragged or not), so that one size serves both.
size_t attend_workspace_bytes(int d, int64_t m, int64_t capacity, int64_t total_q, int heads, int heads_q) {
  size_t need = 0;
  for (int ragged = 0; ragged < 2; ++ragged) {
    if (!ragged && total_q % m != 0) continue;
    const int s = make_plan(m, capacity, total_q, heads, heads_q, ragged != 0).splits;
    if (s == 1) continue;
    const size_t b = partial_o_bytes(d, total_q, heads_q, s) +
                     align256(static_cast<size_t>(s) * total_q * heads_q * sizeof(RowState));
    need = b > need ? b : need;
  }
  return need;
}

bool attend_fits(int64_t m, int64_t capacity, int64_t total_q, int heads, int heads_q, bool ragged) {
  const AttendPlan p = make_plan(m, capacity, total_q, heads, heads_q, ragged);
  return p.tiles * p.splits <= INT32_MAX / heads;
}

hipError_t launch_attend(const AttendArgs& a, int fmt, int d, hipStream_t stream) {
  const int64_t capacity = static_cast<int64_t>(a.k) * a.kv.ppc * a.kv.page_tokens;
  const AttendPlan p = make_plan(a.m, capacity, a.total_q, a.kv.heads, a.hq, a.q_offsets != nullptr);
  switch (fmt) {
    case MEM_KV_BF16: return launch_fmt<MEM_KV_BF16>(a, p, d, stream);
    case MEM_KV_FP8: return launch_fmt<MEM_KV_FP8>(a, p, d, stream);
    default: return launch_fmt<MEM_KV_FP4>(a, p, d, stream);
  }
}

}  // namespace memattn
