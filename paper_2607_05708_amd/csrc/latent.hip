// Latent attention, absorbed form: W_h goes to the query, V_h behind the sum, and
// all heads share a token's latent vector as key and value.
//
//   latent_query_kernel   W_h^T q and the query's rotated part as one row, bf16
//   latent_few_kernel,    attention of those rows over the cache: tiles of 16
//   latent_attend_kernel  rows, of 64 or 128
//   latent_out_kernel     joins the parts of split contexts, and takes V_h to the
//                         weighted sums of latent vectors
#include <algorithm>

#include "context.h"
#include "kv.h"
#include "latent.h"
#include "latent_rows.h"
#include "device_common.h"

namespace memattn {

namespace {

// ---------------------------------------------------------------- queries

// Rows of queries in the workspace: W_h^T q (L elements), then the rotated part.
template <int L>
constexpr int kQueryRow = L + kRopeDim;

constexpr int kTokenBlock = 32;  // tokens of a product's columns

// Four consecutive bf16 elements.
__device__ __forceinline__ u32x2_t load4(const uint16_t* p, bool vec) {
  union { u32x2_t v; uint16_t h[4]; } x;
  if (vec) {
    x.v = *reinterpret_cast<const u32x2_t*>(p);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x.h[j] = p[j];
  }
  return x.v;
}

// Workgroup (head, 128 of the L columns, tokens): W_h's part goes to LDS once, then products of 32 columns a wave with
// blocks of 32 tokens.  (W is read once for eight blocks; 64 tokens of 32 heads of 128 by 512 take 8.4 us, 128 heads 16: half
// of it the start, and 32 MB.)  They are rounded to bf16 as the operands of the scores' products: as two bf16 numbers
// each, the attention would take 1.5 times the products.
template <int L, int D>
__global__ __launch_bounds__(kThreads) void latent_query_kernel(LatentArgs x, int blocks, uint16_t* __restrict__ rows) {
  constexpr int kCols = 128, kPitch = kCols + 32;
  __shared__ __align__(16) uint16_t wk[D * kPitch];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int h = blockIdx.x, n0 = blockIdx.y * kCols;
  const int64_t total = x.a.total_q, tok0 = static_cast<int64_t>(blockIdx.z) * blocks * kTokenBlock;
  const uint16_t* w = x.w + h * x.w_hs + n0;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const int r = 16 * i + (tid >> 4), c = tid & 15;
    *reinterpret_cast<u32x4_t*>(wk + r * kPitch + 8 * (c ^ exchange(r))) =
        *reinterpret_cast<const u32x4_t*>(w + r * x.w_rs + 8 * c);
  }
  __syncthreads();
  // transposed operands: columns 32 wave .. of W_h, rows 16 y + 4 half + 0..3 and + 8
  bf16x8 a[D / 16];
  {
    const Transposed<kPitch> columns(lane);
#pragma unroll
    for (int y = 0; y < D / 16; ++y) a[y] = columns(wk + 16 * y * kPitch + 32 * wave);
  }
  for (int b = 0; b < blocks; ++b) {
    const int64_t tok = tok0 + b * kTokenBlock + col;
    if (tok - col >= total) return;
    const uint16_t* q = static_cast<const uint16_t*>(x.q.data) + min(tok, total - 1) * x.q.ts + h * x.q.hs + 4 * half;
    const bool vec = (reinterpret_cast<uintptr_t>(q) & 7u) == 0;
    f32x16 o;
#pragma unroll
    for (int j = 0; j < 16; ++j) o[j] = 0.f;
#pragma unroll
    for (int y = 0; y < D / 16; ++y) {
      const u32x2_t v0 = load4(q + 16 * y, vec), v1 = load4(q + 16 * y + 8, vec);
      o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[y], as_bf16x8(u32x4_t{v0[0], v0[1], v1[0], v1[1]}), o, 0, 0, 0);
    }
    if (tok >= total) continue;
    uint16_t* dst = rows + (tok * x.a.hq + h) * kQueryRow<L>;
#pragma unroll
    for (int y = 0; y < 4; ++y)
      *reinterpret_cast<u32x2_t*>(dst + n0 + 32 * wave + 8 * y + 4 * half) =
          u32x2_t{pack2(o[4 * y], o[4 * y + 1]), pack2(o[4 * y + 2], o[4 * y + 3])};
    if (blockIdx.y == 0) {  // 16 elements of the rotated part a wave
      const uint16_t* t = static_cast<const uint16_t*>(x.t.data) + tok * x.t.ts + h * x.t.hs + 16 * wave + 8 * half;
      const bool tv = (reinterpret_cast<uintptr_t>(t) & 7u) == 0;
      const u32x2_t v0 = load4(t, tv), v1 = load4(t + 4, tv);
      *reinterpret_cast<u32x4_t*>(dst + L + 16 * wave + 8 * half) = u32x4_t{v0[0], v0[1], v1[0], v1[1]};
    }
  }
}

// ---------------------------------------------------------------- attention over latent vectors

constexpr int kXcds = 8;

// Which tile and split a workgroup has.  Workgroups go to the XCDs in turn, and each XCD has an L2 of its own: `side` tiles
// that read one context (the rows of a request are consecutive tiles) follow each other on one XCD.  Tiles that ragged
// requests leave empty come last: started first, they leave the others unevenly spread (one request of 128 tokens, 16 heads,
// in 16 parts: 122 us, now 75).
struct Job {
  int64_t tile;  // may be past the last one
  int split;
};
__device__ __forceinline__ Job job_of(uint32_t block, int side, int splits) {
  const uint32_t xcd = block % kXcds, at = block / kXcds, group = at / side * kXcds + xcd;
  return {static_cast<int64_t>(group / splits) * side + at % side, static_cast<int>(group % splits)};
}
inline int64_t job_blocks(int64_t tiles, int side, int splits) {
  return ((tiles + side - 1) / side * splits + kXcds - 1) / kXcds * kXcds * side;
}

template <int L, int RG>
struct LatentShape {
  static constexpr int kBatch = 64;                           // units resolved at a time
  static constexpr int kUnitElems = kUnit * kLatentPitch<L>;  // a unit's rows in LDS
  // Operands of a row's query that LDS holds: with 512 columns of 32 rows a wave's outputs take all 256 accumulation
  // registers, and what else it needs is more than the others with all 36 operands.  (Registers spilled to memory would
  // wait, at each reload, for the loads of the units ahead: 64 x 32,768 fp8 tokens, 128 heads, 991 us without, 764 with 10.)
  static constexpr int kParked = L == 512 && RG == 4 ? 10 : 0;
};

// S^T = K Q^T and O^T = K^T P^T over the same rows of LDS, K the latent vectors (with the key part in the first product):
// 2 (2 L + 64) operations a row and token for 2 bytes an element and less.  A unit is unpacked once for all rows of the tile,
// into the third of three buffers, while the scores of one unit and the second product of the one before are made.
// Bound by issue and the waits for LDS: 64 x 32,768 fp8 tokens, 128 heads of 512, 677 us (matrix cores busy 39 %); 16, 32
// and 64 heads, in tiles of 16 to 64 rows, 279, 390 and 540.  Tiles of 256 rows (a wave with 64): 871 against 710 then.
// Tiles of 32 RG rows: wave w has the 32 rows w / (4 / RG) of the tile and, of the second product, a share of the
// columns; waves with the same rows make their scores each for itself.
template <int FMT, int L, int RG>
__global__ __launch_bounds__(kThreads, 1) void latent_attend_kernel(LatentArgs x, int splits, int64_t tiles, int side,
                                                                 const uint16_t* __restrict__ query_rows,
                                                                 float* __restrict__ part_o,
                                                                 RowState* __restrict__ part_ml) {
  using P = Part<FMT, L>;
  using S = LatentShape<L, RG>;
  constexpr int kPitch = kLatentPitch<L>, kShare = 4 / RG, kColumns = L / kShare;
  constexpr int kSteps = (L + kRopeDim) / 16;
  constexpr int kBlocks = kColumns / 32;
  extern __shared__ int dyn[];  // of the chunk list: ub[k + 1], tb[k + 1]
  __shared__ __align__(16) uint16_t unit_rows[3][S::kUnitElems];
  __shared__ __align__(16) uint16_t parked[S::kParked > 0 ? kWaves * S::kParked * 64 * 8 : 8];
  __shared__ Unit list[S::kBatch];
  __shared__ int tmp[2 * kWaves];
  // Tokens of a masked unit whose values are not finite: of the unit at hand, of the next, and of the one after that,
  // which is cleared (so that a barrier stands between clearing and noting, and between noting and reading).
  __shared__ uint32_t bad_tok[3];

  const AttendArgs& a = x.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int rg = wave / kShare, cg = wave % kShare;
  const Job job = job_of(blockIdx.x, side, splits);
  const int split = job.split;
  Tile t;
  if (job.tile >= tiles || !find_tile<32 * RG>(a, static_cast<uint32_t>(job.tile), a.hq, &t)) return;
  const ChunkList list_of = scan_list<kThreads, false>(a, t.req, dyn, tmp);
  const int ctx = list_of.tb[a.k];
  const int prefix = a.prefix_len ? __builtin_amdgcn_readfirstlane(min(max(a.prefix_len[t.req], 0), kFar)) : 0;
  const int my_row = t.r0 + min(32 * rg + col, t.rows - 1);
  const RowRule rule = row_rule(a, t, ctx, 0, a.hq, my_row);
  const TileRule tr = tile_rule<32 * RG>(a, t, ctx, 0, a.hq);
  const Span span = visible_units(list_of, prefix, tr.lo, tr.hi);
  const int n_units = __builtin_amdgcn_readfirstlane(span.count());
  const int u0 = static_cast<int>(static_cast<int64_t>(n_units) * split / splits);
  const int u1 = static_cast<int>(static_cast<int64_t>(n_units) * (split + 1) / splits);

  // lane (col, half) holds elements 16 s + 8 half .. + 7 of row `col` of the wave
  constexpr int kKept = kSteps - S::kParked;
  bf16x8 q[kKept];
  const int64_t row_at = static_cast<int64_t>(t.q0) * a.hq + my_row;
  load_queries(query_rows + row_at * kQueryRow<L> + 8 * half, 16, q);
  const uint16_t* my_parked = parked + (wave * S::kParked * 64 + lane) * 8;
  if constexpr (S::kParked > 0) {
    bf16x8 more[S::kParked];
    load_queries(query_rows + row_at * kQueryRow<L> + 16 * kKept + 8 * half, 16, more);
#pragma unroll
    for (int y = 0; y < S::kParked; ++y)
      *reinterpret_cast<bf16x8*>(parked + ((wave * S::kParked + y) * 64 + lane) * 8) = more[y];
  }

  const float c = a.scale * kLog2e;
  const int64_t T = a.kv.page_tokens;
  Rows<32, kColumns> rows;
  rows.clear();
  RowState st{-INFINITY, 0.f};
  float rounded = 0.f;  // sum of the weights as the second product takes them, which the outputs are divided by
  bool poison = false;

  const int tok = tid >> 3, part = tid & 7, exchanged = exchange(tok);  // the part of a row that this thread unpacks
  const int key_at = col * kPitch, f = exchange(col);
  const int even = key_at + 8 * (half ^ f), odd = key_at + 8 * ((2 + half) ^ f);  // chunks 0 and 2 (+ half) of a row
  const Transposed<kPitch> columns(lane);
  P p;

  for (int last = u1 - 1; last >= u0; last -= S::kBatch) {
    __syncthreads();
    const int n = resolve_units<S::kBatch>(a, list_of, span, tr, prefix, 0, P::kRow, last, min(S::kBatch, last - u0 + 1),
                                           list, tmp);
    if (n == 0) continue;
    if (tid < 3) bad_tok[tid] = 0;
    // the first step's second product is of weights 0: its values have to be numbers
    for (int z = tid; z < S::kUnitElems / 8; z += kThreads)
      reinterpret_cast<u32x4_t*>(unit_rows[2])[z] = u32x4_t{0, 0, 0, 0};
    __syncthreads();
    // this thread's row of a unit (of those that it holds): the unit's page, and its bytes there
    struct Place {
      const uint8_t *page, *parts, *scales;  // the same in every lane
      uint32_t row;
    };
    auto place = [&](const Unit& u) {
      const uint8_t* page = a.kv.pool + (u.at - u.row() * P::kRow);
      return Place{page, page + T * P::kRow, page + T * (P::kRow + 2 * kRopeDim),
                   static_cast<uint32_t>(u.row() + min(tok, u.held() - 1))};
    };
    auto load_codes = [&](const Place& from, int y) {
      p.codes[y] = *reinterpret_cast<const u32x4_t*>(from.page + (from.row * P::kRow + 16 * part + 128 * y));
    };
    auto load_rope = [&](const Place& from) {
      p.rope = *reinterpret_cast<const u32x4_t*>(from.parts + (from.row * (2 * kRopeDim) + 16 * part));
    };
    auto load_scales = [&](const Place& from, uint32_t (&to)[P::kScaleWords]) {
      if constexpr (FMT != MEM_KV_BF16) {
#pragma unroll
        for (int i = 0; i < P::kScaleWords / 2; ++i) {
          const u32x2_t v = reinterpret_cast<const u32x2_t*>(from.scales + from.row * P::kSc)[i];
          to[2 * i] = v[0];
          to[2 * i + 1] = v[1];
        }
      } else {
        to[0] = 0;
      }
    };
    // tokens that a masked unit does not hold are cleared, values that are not finite are noted and left out
    auto check = [&](const Unit& u, int to) {
      if (tok >= u.held()) p.clear();
      const bool bad = p.bad();
      const uint64_t vote = __ballot(bad);
      if (bad) atomicOr(&bad_tok[to], 1u << tok);
      if ((vote >> (lane & 56)) & 255u) p.clear();
    };
    // Piece z of the next unit, and the load of the same piece of the one after it.
    auto advance = [&](uint16_t* to, const Place& from, int z) {
      p.store(to, exchanged, part, z);
      if (z == P::kPieces - 1) load_rope(from);
      else if (z % P::kChunks == P::kChunks - 1) load_codes(from, z / P::kChunks);
    };
    Unit u = uniform_unit(list[0]), next = uniform_unit(list[min(1, n - 1)]);
    {
      const Place from = place(u);
#pragma unroll
      for (int y = 0; y < P::kLoads; ++y) load_codes(from, y);
      load_rope(from);
      load_scales(from, p.sc);
    }
    if (u.masked()) check(u, 0);
    {
      uint16_t* to = unit_rows[0] + tok * kPitch;
      const Place from = place(next);
      // (in the order of the steps, so that the compiler can count what is in flight behind a load)
      uint32_t scales[P::kScaleWords];
      load_scales(from, scales);
      issue_first();
#pragma unroll
      for (int z = 0; z < P::kPieces; ++z) {
        advance(to, from, z);
        issue_first();
      }
#pragma unroll
      for (int j = 0; j < P::kScaleWords; ++j) p.sc[j] = scales[j];
    }
    __syncthreads();
    // A step makes the scores of unit i, then its weights beside the second product of unit i - 1.  They go by the
    // running maximum as it is; where a score turns out to be above it by more than the lag (rare), they are made again.
    constexpr int kOps = 2 * kBlocks;
    u32x4_t w[2] = {u32x4_t{0, 0, 0, 0}, u32x4_t{0, 0, 0, 0}};
    int slot = 0;  // i mod 3: the unit's buffer, and its word of bad_tok
    for (int i = 0; i <= n; ++i) {  // (step n only finishes the last unit)
      const Unit after = uniform_unit(list[min(i + 2, n - 1)]);
      const int slot1 = slot == 2 ? 0 : slot + 1, slot2 = slot == 0 ? 2 : slot - 1;
      if (tid == 0) bad_tok[slot2] = 0;
      if (i + 1 < n && next.masked()) check(next, slot1);
      uint16_t* to = unit_rows[slot1] + tok * kPitch;
      const Place from = place(after);
      // (the scale bytes of the unit after the next are the first loads of a step, and wait in registers of their own:
      // what unpacking begins with would otherwise be the youngest load, and wait for all)
      uint32_t scales[P::kScaleWords];
      load_scales(from, scales);
      issue_first();
      // (a wave without rows goes along with its tile's last row: with a path of its own the compiler copies the loads
      // of the units ahead from register to register, which waits for them)
      const uint16_t* keys = unit_rows[slot];
      const uint16_t* values = unit_rows[slot2] + cg * kColumns;
      f32x16 s;
#pragma unroll
      for (int j = 0; j < 16; ++j) s[j] = 0.f;
      {
        constexpr int kAhead = 3;
        auto key = [&](int y) {
          return *reinterpret_cast<const u32x4_t*>(keys + (y & 1 ? odd : even) + 32 * (y >> 1));
        };
        auto query = [&](int y) { return *reinterpret_cast<const bf16x8*>(my_parked + (y - kKept) * 512); };
        u32x4_t k[kSteps];
        bf16x8 pq[S::kParked + 1];
#pragma unroll
        for (int y = 0; y < kAhead; ++y) k[y] = key(y);
        issue_first();
#pragma unroll
        for (int y = 0; y < kSteps; ++y) {
          if (y + kAhead < kSteps) k[y + kAhead] = key(y + kAhead);
          if (y + kAhead < kSteps && y + kAhead >= kKept) pq[y + kAhead - kKept] = query(y + kAhead);
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[y]),
                                                      y < kKept ? q[y < kKept ? y : 0] : pq[y < kKept ? 0 : y - kKept],
                                                      s, 0, 0, 0);
          if (y * P::kPieces / kSteps != (y + 1) * P::kPieces / kSteps) advance(to, from, y * P::kPieces / kSteps);
          issue_first();
        }
      }
      if (i == n) {
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = -INFINITY;
      } else if (u.masked()) {
        const uint32_t seen = visible_tokens(rule, u, prefix);
        mask_scores<32, 16>(s, seen, half);
        poison |= (seen & bad_tok[slot]) != 0;
      }
      u32x4_t now[2];
      float ref = finite_max(st.m), l = 0.f, lr = 0.f, top = s[0], e[2];
      auto weigh = [&](int j) {  // scores 2 j and 2 j + 1
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          e[y] = fast_exp2(fmaf(s[2 * j + y], c, -ref));
          l += e[y];
        }
        const uint32_t pair = pack2(e[0], e[1]);
        now[j >> 2][j & 3] = pair;
        lr = add_pair(pair, lr);
      };
      {  // operand x: columns 32 (x / 2), tokens 16 (x % 2)
        constexpr int kAhead = 2;
        auto value = [&](int x) { return columns(values + 16 * (x & 1) * kPitch + 32 * (x >> 1)); };
        bf16x8 v[kOps];
#pragma unroll
        for (int x = 0; x < kAhead; ++x) v[x] = value(x);
        issue_first();
#pragma unroll
        for (int x = 0; x < kOps; ++x) {
          if (x + kAhead < kOps) v[x + kAhead] = value(x + kAhead);
          rows.o[x >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[x], as_bf16x8(w[x & 1]), rows.o[x >> 1], 0, 0, 0);
#pragma unroll
          for (int j = 8 * x / kOps; j < 8 * (x + 1) / kOps; ++j) {
            top = nan_max(top, nan_max(s[2 * j], s[2 * j + 1]));
            weigh(j);
          }
          issue_first();
        }
      }
      const float high = max_column<32>(top) * c;
      if (__any(high > st.m + kLag)) {
        const float mn = fmaxf(st.m, high);
        const float by = mn == -INFINITY ? 1.f : fast_exp2(st.m - mn);
        st.l *= by;
        rounded *= by;
        scale_rows(rows, by);
        st.m = mn;
        ref = finite_max(mn);
        l = lr = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) weigh(j);
      }
      st.l += l;
      rounded += lr;
      w[0] = now[0];
      w[1] = now[1];
#pragma unroll
      for (int j = 0; j < P::kScaleWords; ++j) p.sc[j] = scales[j];
      u = next;
      next = after;
      slot = slot1;
      __syncthreads();
    }
  }

  st.l = sum_column<32>(st.l);
  rounded = sum_column<32>(rounded);
  poison = any_column<32>(poison, col);
  if (32 * rg + col >= t.rows) return;
  write_part<32, kColumns, L>(a, rows, st, rounded, poison, row_at, half, split, cg * kColumns, part_o, part_ml);
}

// ---------------------------------------------------------------- few rows

// A lane's parts of two tokens' rows (16 apart): 16-byte loads 4 parts apart, the key part's two, and the scale bytes.
template <int FMT, int L>
struct Quarter {
  static constexpr int kRow = kv_row_bytes(FMT, L);
  static constexpr int kSc = kv_scale_bytes(FMT, L);
  static constexpr int kElems = 16 * L / kRow;   // elements of a load
  static constexpr int kLoads = L / (4 * kElems);
  static constexpr int kChunks = kElems / 8;     // operands of eight elements that a load becomes
  static constexpr int kScaleWords = FMT == MEM_KV_BF16 ? 1 : kSc / 4;
  u32x4_t codes[kLoads], rope[2];
  uint32_t sc[kScaleWords];

  __device__ __forceinline__ uint32_t scale_byte(int y, int part) const {
    if constexpr (FMT == MEM_KV_FP8) return sc[y >> 1] >> (16 * (y & 1) + 8 * (part >> 1)) & 255u;  // block 2 y + part / 2
    return sc[y] >> (8 * part) & 255u;                                                             // block 4 y + part
  }
  __device__ __forceinline__ u32x4_t chunk(int y, int c, float s) const {
    if constexpr (FMT == MEM_KV_BF16) return codes[y];
    u32x4_t o;
    if constexpr (FMT == MEM_KV_FP4) {
      const uint32_t x = codes[y][c];
      o[0] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 0));
      o[1] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 1));
      o[2] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 2));
      o[3] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s, 3));
    } else if constexpr (FMT == MEM_KV_FP8) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        o[2 * j] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[y][2 * c + j], s, false));
        o[2 * j + 1] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[y][2 * c + j], s, true));
      }
    }
    return o;
  }
  // Whether it holds a latent value that is not finite, or may.
  __device__ __forceinline__ bool bad() const {
    u16x2 most = {0, 0};
    bool x = false;
#pragma unroll
    for (int y = 0; y < kLoads; ++y)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (FMT == MEM_KV_BF16)
          most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, codes[y][j] & 0x7FFF7FFFu));
        if constexpr (FMT == MEM_KV_FP8) x |= (((codes[y][j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
      }
    if constexpr (FMT != MEM_KV_BF16) {
#pragma unroll
      for (int i = 0; i < kScaleWords; ++i)
#pragma unroll
        for (int b = 0; b < 4; ++b) x |= (sc[i] >> (8 * b) & 255u) > kMaxScaleByte<FMT>;
    }
    return x || most[0] >= 0x7F80u || most[1] >= 0x7F80u;
  }
  __device__ __forceinline__ void clear(bool parts) {
#pragma unroll
    for (int y = 0; y < kLoads; ++y) codes[y] = u32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kScaleWords; ++i) sc[i] = 0x7F7F7F7Fu;
    if (parts) rope[0] = rope[1] = u32x4_t{0, 0, 0, 0};
  }
};

template <int L>
struct FewShape {
  static constexpr int kRows = 16;
  static constexpr int kBatch = 128;                                    // units resolved at a time
  static constexpr int kWaveBytes = kUnit * kValuePitch<16, L> * 2;     // a wave's unit as bf16
  static constexpr int kJoinBytes = 2 * kRows * L * 4;                  // two waves' outputs at the end
  static constexpr int kArea = kWaves * kWaveBytes > kJoinBytes ? kWaves * kWaveBytes : kJoinBytes;
  static constexpr int kShift = 3;
};

// Workgroups that share a CU.
constexpr int few_per_cu(int fmt, int latent) { return latent == 256 && fmt != MEM_KV_BF16 ? 2 : 1; }

// Tiles of 16 rows: each wave streams its own units with no barrier.  A lane loads parts of two tokens' rows straight
// from the page; unpacked, they are operands of the first product, and go through the wave's own LDS rows once to be
// read back transposed for the second.  Each load is made again, for the wave's next unit, as soon as it has been used.
// Weights go into the second product as two bf16 numbers.  Bound by HBM where contexts are long (4 x 131,072 bf16 tokens,
// 16 heads: 116 us, 5.2 TB/s), else by its start and end: one token over 2,560, 4 units a workgroup, 16 us.
template <int FMT, int L>
__global__ __launch_bounds__(kThreads, few_per_cu(FMT, L)) void latent_few_kernel(LatentArgs x, int splits, int64_t tiles, int side,
                                                                             const uint16_t* __restrict__ query_rows,
                                                                                         float* __restrict__ part_o,
                                                                             RowState* __restrict__ part_ml) {
  using P = Quarter<FMT, L>;
  using S = FewShape<L>;
  constexpr int R = S::kRows, kSteps = L / 32, kOps = L / 16;
  extern __shared__ int dyn[];  // of the chunk list: ub[k + 1], tb[k + 1]
  __shared__ __align__(16) uint8_t area[S::kArea];
  __shared__ Unit list[S::kBatch];
  __shared__ int tmp[2 * kWaves];
  __shared__ RowState joint[2][64];
  __shared__ int joint_poison[2][64];

  const AttendArgs& a = x.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, part = lane >> 4;
  const Job job = job_of(blockIdx.x, side, splits);
  const int split = job.split;
  Tile t;
  if (job.tile >= tiles || !find_tile<R>(a, static_cast<uint32_t>(job.tile), a.hq, &t)) return;
  const ChunkList list_of = scan_list<kThreads, false>(a, t.req, dyn, tmp);
  const int ctx = list_of.tb[a.k];
  const int prefix = a.prefix_len ? __builtin_amdgcn_readfirstlane(min(max(a.prefix_len[t.req], 0), kFar)) : 0;
  const int my_row = t.r0 + min(col, t.rows - 1);
  const RowRule rule = row_rule(a, t, ctx, 0, a.hq, my_row);
  const TileRule tr = tile_rule<R>(a, t, ctx, 0, a.hq);
  const Span span = visible_units(list_of, prefix, tr.lo, tr.hi);
  const int n_units = __builtin_amdgcn_readfirstlane(span.count());
  const int u0 = static_cast<int>(static_cast<int64_t>(n_units) * split / splits);
  const int u1 = static_cast<int>(static_cast<int64_t>(n_units) * (split + 1) / splits);

  // queries in the order of the loads: operand (y, c) of a lane holds elements E (4 y + part) + 8 c .. + 7
  bf16x8 q[kSteps], qr[2];
  const int64_t row_at = static_cast<int64_t>(t.q0) * a.hq + my_row;
  {
    const uint16_t* src = query_rows + row_at * kQueryRow<L>;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int y = i / P::kChunks, cc = i % P::kChunks;
      q[i] = as_bf16x8(*reinterpret_cast<const u32x4_t*>(src + P::kElems * (4 * y + part) + 8 * cc));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) qr[i] = as_bf16x8(*reinterpret_cast<const u32x4_t*>(src + L + 32 * i + 8 * part));
  }

  const float c = a.scale * kLog2e;
  const int64_t T = a.kv.page_tokens;
  uint16_t* rows_of = reinterpret_cast<uint16_t*>(area + wave * S::kWaveBytes);
  const ValueOps<16, L, S::kShift> ops(rows_of, lane);
  Rows<16, L> rows;
  rows.clear();
  RowState st{-INFINITY, 0.f};
  bool poison = false;
  P p[2];

  struct Place {
    const uint8_t *page, *parts, *scales;  // the same in every lane
    uint32_t row[2];
  };
  auto place = [&](const Unit& u) {
    const uint8_t* page = a.kv.pool + (u.at - u.row() * P::kRow);
    Place w{page, page + T * P::kRow, page + T * (P::kRow + 2 * kRopeDim), {}};
#pragma unroll
    for (int h = 0; h < 2; ++h) w.row[h] = static_cast<uint32_t>(u.row() + min(16 * h + col, u.held() - 1));
    return w;
  };
  auto load_codes = [&](const Place& from, int h, int y) {
    p[h].codes[y] = *reinterpret_cast<const u32x4_t*>(from.page + (from.row[h] * P::kRow + 16 * part + 64 * y));
  };
  auto load_rope = [&](const Place& from, int h, int y) {
    p[h].rope[y] =
        *reinterpret_cast<const u32x4_t*>(from.parts + (from.row[h] * (2 * kRopeDim) + 16 * part + 64 * y));
  };
  auto load_scales = [&](const Place& from, int h, uint32_t (&to)[P::kScaleWords]) {
    if constexpr (FMT != MEM_KV_BF16) {
#pragma unroll
      for (int i = 0; i < P::kScaleWords / 2; ++i) {
        const u32x2_t v = reinterpret_cast<const u32x2_t*>(from.scales + from.row[h] * P::kSc)[i];
        to[2 * i] = v[0];
        to[2 * i + 1] = v[1];
      }
    } else {
      to[0] = 0;
    }
  };

  for (int last = u1 - 1; last >= u0; last -= S::kBatch) {
    __syncthreads();
    const int n = resolve_units<S::kBatch>(a, list_of, span, tr, prefix, 0, P::kRow, last, min(S::kBatch, last - u0 + 1),
                                           list, tmp);
    if (wave >= n) continue;
    Unit u = uniform_unit(list[wave]);
    {
      const Place from = place(u);
#pragma unroll
      for (int h = 0; h < 2; ++h) load_scales(from, h, p[h].sc);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int y = 0; y < P::kLoads; ++y) load_codes(from, h, y);
#pragma unroll
        for (int y = 0; y < 2; ++y) load_rope(from, h, y);
      }
    }
    for (int i = wave; i < n; i += kWaves) {
      const Unit next = uniform_unit(list[i + kWaves < n ? i + kWaves : i]);
      const Place from = place(next);
      uint32_t bad = 0;
      if (u.masked()) {  // tokens that are not held are cleared, values that are not finite are noted and left out
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int tok = 16 * h + col;
          if (tok >= u.held()) p[h].clear(true);
          uint64_t vote = __ballot(p[h].bad());
          vote |= vote >> 32;
          vote |= vote >> 16;
          if ((vote >> col) & 1u) p[h].clear(false);
          bad |= static_cast<uint32_t>(vote & 0xFFFFu) << (16 * h);
        }
      }
      uint32_t scales[2][P::kScaleWords];
#pragma unroll
      for (int h = 0; h < 2; ++h) load_scales(from, h, scales[h]);
      issue_first();
      f32x4 sum[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sum[h] = f32x4{0.f, 0.f, 0.f, 0.f};
        uint16_t* dst = rows_of + (16 * h + col) * kValuePitch<16, L>;
#pragma unroll
        for (int y = 0; y < P::kLoads; ++y) {
          const float s = FMT == MEM_KV_BF16 ? 1.f : kv_scale(p[h].scale_byte(y, part));
#pragma unroll
          for (int cc = 0; cc < P::kChunks; ++cc) {
            const u32x4_t k = p[h].chunk(y, cc, s);
            sum[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k), q[y * P::kChunks + cc], sum[h], 0, 0, 0);
            *reinterpret_cast<u32x4_t*>(
                dst + 8 * value_chunk<16, S::kShift>(16 * h + col, P::kChunks * (part + 4 * y) + cc)) = k;
          }
          load_codes(from, h, y);
          issue_first();
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          sum[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(p[h].rope[y]), qr[y], sum[h], 0, 0, 0);
          load_rope(from, h, y);
          issue_first();
        }
      }
      float s[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = sum[j >> 2][j & 3];
      if (u.masked()) {
        const uint32_t seen = visible_tokens(rule, u, prefix);
        mask_scores<16, 8>(s, seen, part);
        poison |= (seen & bad) != 0;
      }
      const float high = max_column<16>(max_of(s)) * c;
      const bool counts = __any(!u.masked() || high != -INFINITY);
      if (counts) {
        if (__any(high > st.m + kLag)) {
          const float mn = fmaxf(st.m, high);
          const float r = mn == -INFINITY ? 1.f : fast_exp2(st.m - mn);
          st.l *= r;
          if constexpr (L == 512) scale_rows(rows, r);
          else rows.scale(r);
          st.m = mn;
        }
        const float ref = finite_max(st.m);
        // weights as two bf16 numbers each: the product is a small part of what a unit costs here
        u32x4_t w, rest;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          s[j] = fast_exp2(fmaf(s[j], c, -ref));
          st.l += s[j];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j] = pack2(s[2 * j], s[2 * j + 1]);
          rest[j] = rest2(s[2 * j], s[2 * j + 1], w[j]);
        }
        __builtin_amdgcn_wave_barrier();
        constexpr int kTogether = 8;  // operands loaded ahead of their products
#pragma unroll
        for (int n0 = 0; n0 < kOps; n0 += kTogether) {
          bf16x8 v[kTogether];
#pragma unroll
          for (int y = 0; y < kTogether; ++y) v[y] = ops[n0 + y];
          issue_first();
#pragma unroll
          for (int y = 0; y < kTogether; ++y) ops.multiply(rows, n0 + y, v[y], &w);
#pragma unroll
          for (int y = 0; y < kTogether; ++y) ops.multiply(rows, n0 + y, v[y], &rest);
        }
        __builtin_amdgcn_wave_barrier();
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < P::kScaleWords; ++j) p[h].sc[j] = scales[h][j];
      u = next;
    }
  }

  // join the waves: 2 and 3 into 0 and 1, then 1 into 0 (a lane holds the same outputs in every wave)
  st.l = sum_column<16>(st.l);
  poison = any_column<16>(poison, col);
  float* store = reinterpret_cast<float*>(area);
#pragma unroll
  for (int from = 2; from >= 1; --from) {
    __syncthreads();  // what `area` held is done with
    if (wave >= from && wave < 2 * from) {
      float* dst = store + (wave - from) * R * L + lane * 4;
      int i = 0;
      rows.each4(part, [&](int, f32x4 v) { *reinterpret_cast<f32x4*>(dst + 256 * i++) = v; });
      joint[wave - from][lane] = st;
      joint_poison[wave - from][lane] = poison;
    }
    __syncthreads();
    if (wave < from) {
      const RowState other = joint[wave][lane];
      poison |= joint_poison[wave][lane] != 0;
      const float mn = fmaxf(st.m, other.m), ref = finite_max(mn);
      const float f0 = fast_exp2(st.m - ref), f1 = fast_exp2(other.m - ref);
      st.l = st.l * f0 + other.l * f1;
      st.m = mn;
      const float* src = store + wave * R * L + lane * 4;
#pragma unroll
      for (int i = 0; i < kOps; ++i) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(src + 256 * i);
        rows.o[i] = rows.o[i] * f0 + v * f1;
      }
    }
  }
  if (wave > 0 || col >= t.rows) return;
  write_part<16, L, L>(a, rows, st, st.l, poison, row_at, part, split, 0, part_o, part_ml);
}

// ---------------------------------------------------------------- outputs

// Workgroup (head, up to 32 tokens): joins the parts of its rows' sums (in a fixed order; a context that is not split has
// one part), and multiplies them by V_h.  The sums go into the product as two bf16 numbers each, so that only the output is
// rounded; V_h is on its way meanwhile.  A wave has 32 of the output's elements, with heads of 64 half of the sum's.
// T: parts that are loaded together, the first ones before their weights are known.
template <int L, int D, int T>
__global__ __launch_bounds__(kThreads) void latent_out_kernel(LatentArgs x, int splits, int tokens,
                                                           const float* __restrict__ part_o,
                                                           const RowState* __restrict__ part_ml) {
  constexpr int kAcross = D / 32, kShares = kWaves / kAcross, kSteps = L / 16 / kShares;
  constexpr int kPitch = L + 32, kPer = L / 64;
  __shared__ __align__(16) uint16_t high[kTokenBlock * kPitch], low[kTokenBlock * kPitch];
  __shared__ float halves[kShares == 2 ? kAcross * 64 * 16 : 1];
  __shared__ bool sees[kTokenBlock];  // rows that something counts for: the others are 0 whatever V_h holds
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5, j0 = 32 * (wave % kAcross), k0 = wave / kAcross * (L / kShares);
  const int h = blockIdx.x;
  const int64_t tok0 = static_cast<int64_t>(blockIdx.y) * tokens, total = x.a.total_q, rows = total * x.a.hq;
  const int64_t first = x.a.q_offsets ? max(x.a.q_offsets[0], 0) : 0;
  const int64_t last = x.a.q_offsets ? min(static_cast<int64_t>(x.a.q_offsets[x.a.m]), total) : total;
  const uint16_t* src = x.w + h * x.w_hs + (D + j0 + col) * x.w_rs + k0 + 8 * half;
  u32x4_t w[kSteps];
#pragma unroll
  for (int y = 0; y < kSteps; ++y) w[y] = *reinterpret_cast<const u32x4_t*>(src + 16 * y);

  for (int r = wave; r < kTokenBlock; r += kWaves) {
    const int64_t tok = tok0 + r, at = tok * x.a.hq + h;
    float o[kPer];
    bool seen = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] = 0.f;
    if (r < tokens && tok >= first && tok < last) {  // (rows that no request owns were not computed)
      RowState st[2] = {{-INFINITY, 0.f}, {-INFINITY, 0.f}};  // of parts `lane` and 64 + `lane`
      if (lane < splits) st[0] = part_ml[lane * rows + at];
      if (64 + lane < splits) st[1] = part_ml[(64 + lane) * rows + at];
      float v[T][kPer];
      auto load = [&](int s0) {  // (past the last part: the last one again, so that nothing is conditional)
#pragma unroll
        for (int u = 0; u < T; ++u) {
          const float* from = part_o + (min(s0 + u, splits - 1) * rows + at) * L + lane * kPer;
#pragma unroll
          for (int i = 0; i < kPer; ++i) v[u][i] = from[i];
        }
      };
      load(0);
      const float m = wave_max_f32(fmaxf(st[0].m, st[1].m));
      const float f[2] = {fast_exp2(st[0].m - finite_max(m)), fast_exp2(st[1].m - finite_max(m))};
      const float l = wave_sum_f32(f[0] * st[0].l + f[1] * st[1].l);
      for (int s0 = 0; s0 < splits; s0 += T) {
        if (s0 > 0) load(s0);
#pragma unroll
        for (int u = 0; u < T; ++u) {
          if (s0 + u >= splits) continue;
          const float g = lane_f32(s0 < 64 ? f[0] : f[1], (s0 + u) & 63);
#pragma unroll
          for (int i = 0; i < kPer; ++i) o[i] += g * v[u][i];
        }
      }
      const float inv = inverse_sum(l);
      bool odd = false;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        o[i] *= inv;
        odd |= o[i] != o[i];
      }
      // (values that are not finite count behind weights of 0 too: scores of minus infinity)
      seen = l != 0.f || __any(odd);
      if (x.a.lse && lane == 0) x.a.lse[at] = lse_of(m, l);
    }
    if (lane == 0) sees[r] = seen;
    const int place = r * kPitch + 8 * ((lane * kPer / 8) ^ exchange(r)) + lane * kPer % 8;
#pragma unroll
    for (int i = 0; i < kPer; i += 2) {
      const uint32_t pair = pack2(o[i], o[i + 1]);
      *reinterpret_cast<uint32_t*>(high + place + i) = pair;
      *reinterpret_cast<uint32_t*>(low + place + i) = rest2(o[i], o[i + 1], pair);
    }
  }
  __syncthreads();
  f32x16 o;
#pragma unroll
  for (int j = 0; j < 16; ++j) o[j] = 0.f;
#pragma unroll
  for (int y = 0; y < kSteps; ++y) {
    const int place = col * kPitch + 8 * ((k0 / 8 + 2 * y + half) ^ exchange(col));
    o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(w[y]),
                                                as_bf16x8(*reinterpret_cast<const u32x4_t*>(low + place)), o, 0, 0, 0);
    o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(w[y]),
                                                as_bf16x8(*reinterpret_cast<const u32x4_t*>(high + place)), o, 0, 0, 0);
  }
  if constexpr (kShares == 2) {
    float* mine = halves + (wave % kAcross) * 64 * 16 + lane;
    if (wave >= kAcross) {
#pragma unroll
      for (int j = 0; j < 16; ++j) mine[64 * j] = o[j];
    }
    __syncthreads();
    if (wave >= kAcross) return;
#pragma unroll
    for (int j = 0; j < 16; ++j) o[j] += mine[64 * j];
  }
  const int64_t tok = tok0 + col;
  if (col >= tokens || tok < first || tok >= last) return;
  uint16_t* dst = x.out + (tok * x.a.hq + h) * D + j0 + 4 * half;
  if (!sees[col]) {
#pragma unroll
    for (int j = 0; j < 16; ++j) o[j] = 0.f;
  }
#pragma unroll
  for (int y = 0; y < 4; ++y)
    *reinterpret_cast<u32x2_t*>(dst + 8 * y) =
        u32x2_t{pack2(o[4 * y], o[4 * y + 1]), pack2(o[4 * y + 2], o[4 * y + 3])};
}

// ---------------------------------------------------------------- launches

size_t align256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }
size_t list_bytes(int k) { return (2 * static_cast<size_t>(k) + 2) * sizeof(int); }

struct AbsorbedPlan {
  int rows;  // of a tile: 16 (few-rows kernel), 64 or 128
  int64_t tiles;
  int splits;
  int side;  // tiles that follow each other on an XCD
};

// Parts of a context, taken at its capacity (the units of shorter ones, or that a window leaves, go to as many), by what a
// call would take in units of a tile: the passes of the busiest XCD's CUs, each with its units and its start and end;
// then the join, of whose rows kJoinRows are written and read while a tile works on a unit.  (Both from timings of 14 shapes with 1 to 128 parts: one request of 48 tokens and 16 heads over 8,192, us: 1 part 555,
// 8 111, 16 84, 32 72, 40, which need a second pass, 104.)  Up to 128 parts, two states a lane of latent_out_kernel: one
// token over 131,072, 16 heads, 64 us, with 64 parts 74; of 4 tokens 103 and 137.
constexpr int64_t kStart = 16;
constexpr int64_t kJoinRows = 10'000;
constexpr int kMostParts = 128;
// Tiles that stay on one XCD: with all of a request's, an XCD has whole requests or none (4 requests of 96 tokens, 16 heads:
// 12 tiles each 317 us, 4 of them 209); to 16 of them no case was faster than with 4.
constexpr int kMaxSide = 4;

// Tiles of 128 rows of 512 elements leave 4 KB of a CU's 160 KB for the chunk list, tiles of 16 rows 20 KB: calls with
// longer lists (more than 511 and 2,559 chunks) take tiles of 64, which leave 40.
bool list_fits_tiles(int latent, int k) { return latent < 512 || list_bytes(k) <= 4096; }
bool list_fits_few(int latent, int k) { return latent < 512 || list_bytes(k) <= 20 * 1024; }
static_assert(FewShape<512>::kArea + FewShape<512>::kBatch * sizeof(Unit) + 2048 + 20 * 1024 <= 160 * 1024,
              "a workgroup's LDS");
static_assert(2 * 3 * LatentShape<512, 2>::kUnitElems + LatentShape<512, 2>::kBatch * sizeof(Unit) + 128 + 8 * 4097 <=
                  160 * 1024,
              "a workgroup's LDS");
static_assert(2 * (3 * LatentShape<512, 4>::kUnitElems + 4 * 64 * 8 * LatentShape<512, 4>::kParked) +
                      LatentShape<512, 4>::kBatch * sizeof(Unit) + 128 + 4096 <= 160 * 1024,
              "a workgroup's LDS");

AbsorbedPlan absorbed_plan(const LatentSizes& s, bool ragged) {
  AbsorbedPlan p;
  const int64_t rows = s.total_q * s.heads;
  p.rows = rows <= 32 * s.m && list_fits_few(s.latent, s.k) ? 16 : rows <= 64 * s.m || !list_fits_tiles(s.latent, s.k) ? 64 : 128;
  const int R = p.rows;
  p.tiles = ragged ? rows / R + s.m : s.m * ((s.total_q / s.m * s.heads + R - 1) / R);
  // How many tiles ragged requests have is for the kernel to find.  They are taken to be alike; where that means one tile
  // each, of several tokens, some may have two, and a count of parts that suits both is sought.
  const int64_t each = (std::max<int64_t>(rows / s.m, 1) + R - 1) / R, alike = s.m * each;
  const int64_t uneven = ragged && each == 1 && s.total_q > s.m ? std::max(alike, (rows + R - 1) / R + s.m / 2) : alike;
  const int64_t slots = 256 / kXcds * (R == 16 ? few_per_cu(s.fmt, s.latent) : 1);  // workgroups that run on an XCD
  p.side = static_cast<int>(std::min<int64_t>(each, kMaxSide));
  int64_t best = INT64_MAX;
  p.splits = 1;
  for (int64_t n = 1; n <= kMostParts && (n == 1 || s.units / n >= 4); ++n) {
    if (n > 1 && job_blocks(p.tiles, p.side, n) > kMaxGroups) break;
    auto passes = [&](int64_t work) {
      return (((work + p.side - 1) / p.side * n + kXcds - 1) / kXcds * p.side + slots - 1) / slots;
    };
    const int64_t cost = (2 * passes(alike) + passes(uneven)) * ((s.units + n - 1) / n + kStart) +
                         3 * (n / 16 + rows * (n - 1) / kJoinRows);
    if (cost < best) {
      best = cost;
      p.splits = static_cast<int>(n);
    }
  }
  return p;
}

// Workspace of the absorbed form: query rows, and the parts of their sums.
struct AbsorbedSpace {
  size_t queries, part_o, part_ml, end;
};

AbsorbedSpace absorbed_space(const LatentSizes& s, int splits) {
  const size_t rows = static_cast<size_t>(s.total_q) * s.heads;
  AbsorbedSpace w;
  w.queries = 0;
  w.part_o = align256(rows * (s.latent + kRopeDim) * 2);
  w.part_ml = w.part_o + align256(splits * rows * s.latent * sizeof(float));
  w.end = w.part_ml + align256(splits * rows * sizeof(RowState));
  return w;
}

constexpr int kQueryBlocks = 8;  // blocks of tokens of a workgroup of latent_query_kernel
int64_t query_groups(int64_t total_q) {
  return (total_q + kQueryBlocks * kTokenBlock - 1) / (kQueryBlocks * kTokenBlock);
}
// Tokens of a workgroup of latent_out_kernel: fewer where that lets more CUs join (64 tokens of 32 heads in 4 parts: 17 us
// with 32, 11.7 with 8; with 4, whose V_h is read twice as often, 14.4).
int out_tokens(int64_t total_q, int heads) {
  int t = kTokenBlock;
  while (t > 4 && (total_q + t - 1) / t * heads < 256) t /= 2;
  return t;
}
int64_t out_groups(int64_t total_q, int heads) {
  const int t = out_tokens(total_q, heads);
  return (total_q + t - 1) / t;
}

template <int FMT, int L, int D>
hipError_t launch_absorbed(const LatentArgs& x, const LatentSizes& s, hipStream_t stream) {
  const AbsorbedPlan p = absorbed_plan(s, x.a.q_offsets != nullptr);
  const AbsorbedSpace at = absorbed_space(s, p.splits);
  uint8_t* ws = static_cast<uint8_t*>(x.ws);
  uint16_t* queries = reinterpret_cast<uint16_t*>(ws + at.queries);
  float* part_o = reinterpret_cast<float*>(ws + at.part_o);
  RowState* part_ml = reinterpret_cast<RowState*>(ws + at.part_ml);
  latent_query_kernel<L, D><<<dim3(s.heads, L / 128, static_cast<unsigned>(query_groups(s.total_q))), kThreads, 0,
                              stream>>>(x, kQueryBlocks, queries);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const unsigned grid = static_cast<unsigned>(job_blocks(p.tiles, p.side, p.splits));
  if (p.rows == 16)
    latent_few_kernel<FMT, L><<<grid, kThreads, list_bytes(s.k), stream>>>(x, p.splits, p.tiles, p.side, queries, part_o,
                                                                          part_ml);
  else
    (p.rows == 64 ? latent_attend_kernel<FMT, L, 2> : latent_attend_kernel<FMT, L, 4>)<<<
        grid, kThreads, list_bytes(s.k), stream>>>(x, p.splits, p.tiles, p.side, queries, part_o, part_ml);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  (p.splits <= 4 ? latent_out_kernel<L, D, 4> : latent_out_kernel<L, D, 16>)<<<
      dim3(s.heads, static_cast<unsigned>(out_groups(s.total_q, s.heads))), kThreads, 0, stream>>>(
      x, p.splits, out_tokens(s.total_q, s.heads), part_o, part_ml);
  return hipGetLastError();
}

template <int FMT, int L>
hipError_t launch_head(const LatentArgs& x, const LatentSizes& s, hipStream_t stream) {
  return s.head_dim == 64 ? launch_absorbed<FMT, L, 64>(x, s, stream) : launch_absorbed<FMT, L, 128>(x, s, stream);
}

template <int FMT>
hipError_t launch_fmt(const LatentArgs& x, const LatentSizes& s, hipStream_t stream) {
  return s.latent == 256 ? launch_head<FMT, 256>(x, s, stream) : launch_head<FMT, 512>(x, s, stream);
}

}  // namespace

mem_latent_form choose_latent_form(const LatentSizes& s, int32_t asked) {
  if (asked != MEM_LATENT_AUTO) return static_cast<mem_latent_form>(asked);
  // Products of a head, in units of a pair's 2 elements each: rows (2 L + R) absorbed, rows (2 d + R) and 2 d L for each
  // token of the context expanded.  Measured, us, absorbed and expanded, 512 elements and heads of 128 (the rule changes
  // at 171 tokens): 8 requests over 8,192 tokens, 16 heads, 128 tokens 455 and 548, 256 764 and 584; one over 4,096, 128
  // heads, 128 tokens 218 and 286, 160 303 and 319; 256 elements, heads of 64 (86 tokens): 4 over 8,192, 64 tokens 100 and
  // 106, 128 156 and 126.  Single requests of few heads change over earlier (16 heads over 8,192: 64 tokens 79 and 89, 128
  // 103 and 95) and short contexts at once (1,024: 16 tokens 50 and 40), by less than 30 us.  Masks, lengths and how new
  // tokens are spread over the requests are not known here: the workspace is asked for without them.
  const int64_t rows = s.total_q / s.m, d = s.head_dim, l = s.latent;
  return rows * (l - d) > d * l ? MEM_LATENT_EXPANDED : MEM_LATENT_ABSORBED;
}

// The larger of the two cases of a call (ragged or not), so that one size serves both.
size_t latent_workspace_bytes(const LatentSizes& s, mem_latent_form form) {
  size_t need = 0;
  for (int ragged = 0; ragged < 2; ++ragged) {
    if (!ragged && s.total_q % s.m != 0) continue;
    const size_t b = form == MEM_LATENT_EXPANDED ? expanded_workspace_bytes(s, ragged != 0)
                                                 : absorbed_space(s, absorbed_plan(s, ragged != 0).splits).end;
    need = b > need ? b : need;
  }
  return need;
}

bool latent_fits(const LatentSizes& s, mem_latent_form form, bool ragged) {
  if (form == MEM_LATENT_EXPANDED) return expanded_fits(s, ragged);
  const AbsorbedPlan p = absorbed_plan(s, ragged);
  const int64_t q = query_groups(s.total_q), o = out_groups(s.total_q, s.heads);
  return job_blocks(p.tiles, p.side, p.splits) <= kMaxGroups && q < 65536 && o < 65536 &&
         q * (s.latent / 128) * s.heads <= kMaxGroups && o * s.heads <= kMaxGroups;
}

hipError_t launch_latent_attend(const LatentArgs& x, const LatentSizes& s, mem_latent_form form, hipStream_t stream) {
  if (form == MEM_LATENT_EXPANDED) return launch_expanded(x, s, stream);
  switch (s.fmt) {
    case MEM_KV_BF16: return launch_fmt<MEM_KV_BF16>(x, s, stream);
    case MEM_KV_FP8: return launch_fmt<MEM_KV_FP8>(x, s, stream);
    default: return launch_fmt<MEM_KV_FP4>(x, s, stream);
  }
}

}  // namespace memattn
