// Latent attention, absorbed form: W_h goes to the query, V_h behind the sum, and
// all heads share a token's latent vector as key and value.
//
//   latent_query_kernel   W_h^T q and the query's rotated part as one row, bf16
//   latent_attend_kernel  attention of those rows over the cache
//   attend_join_kernel    joins the parts of split contexts
//   latent_out_kernel     V_h times the weighted sum of latent vectors
#include "context.h"
#include "kv.h"
#include "latent.h"
#include "device_common.h"

namespace memattn {

namespace {

// Rows of L latent elements and the key part in LDS, bf16.  The pitch is an odd multiple of 64 bytes, and the 16-byte
// chunks of a row are exchanged within 64 bytes by bits 1 and 2 of the row's number: eight rows' chunks of one column
// (the first product reads them along a row) lie in different banks, and so do the pieces of four rows that a
// transposing read takes (the second product).
template <int L>
constexpr int kLatentPitch = L + kRopeDim + 32;
__device__ __forceinline__ int exchange(int row) { return (row & 2) | ((row >> 2) & 1); }

// A thread's part of a token's row, 1/8 of it: 16-byte loads 8 parts apart, the key part, and the row's scale bytes.
template <int FMT, int L>
struct Part {
  static constexpr int kRow = kv_row_bytes(FMT, L);
  static constexpr int kSc = kv_scale_bytes(FMT, L);
  static constexpr int kElems = 16 * L / kRow;          // elements of a load: 8, 16 or 32
  static constexpr int kLoads = L / (8 * kElems);
  static constexpr int kChunks = kElems / 8;            // 16-byte chunks of bf16 that a load becomes
  static constexpr int kScaleWords = FMT == MEM_KV_BF16 ? 1 : kSc / 4;
  u32x4_t codes[kLoads];
  u32x4_t rope;
  uint32_t sc[kScaleWords];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int y = 0; y < kLoads; ++y) codes[y] = u32x4_t{0, 0, 0, 0};
    rope = u32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kScaleWords; ++i) sc[i] = 0x7F7F7F7Fu;
  }
  // Scale byte of load y.
  __device__ __forceinline__ uint32_t scale_byte(int y, int part) const {
    if constexpr (FMT == MEM_KV_FP8) return sc[y] >> (8 * (part >> 1)) & 255u;  // block part / 2 + 4 y
    const uint32_t w = part & 4 ? sc[2 * y + 1] : sc[2 * y];                    // block part + 8 y
    return w >> (8 * (part & 3)) & 255u;
  }
  // Chunk c of load y as bf16.
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
  // Piece z of unpacking it into its LDS row: chunks, then the key part.
  static constexpr int kPieces = kLoads * kChunks + 1;
  __device__ __forceinline__ void store(uint16_t* dst, int exchanged, int part, int z) const {
    if (z == kPieces - 1) {
      *reinterpret_cast<u32x4_t*>(dst + L + 8 * (part ^ exchanged)) = rope;
    } else {
      const int y = z / kChunks, c = z % kChunks;
      const float s = FMT == MEM_KV_BF16 ? 1.f : kv_scale(scale_byte(y, part));
      *reinterpret_cast<u32x4_t*>(dst + 8 * ((kChunks * (part + 8 * y) + c) ^ exchanged)) = chunk(y, c, s);
    }
  }
  // Whether it holds a latent value that is not finite, or may (scales that no write gives).  The key part only goes into
  // scores.
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
};

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
// blocks of 32 tokens.
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
    const int i = lane & 15, r = 4 * half + (i >> 2), c = 4 * wave + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    const uint16_t* src = wk + r * kPitch + 8 * (c ^ exchange(r)) + 4 * (i & 1);
#pragma unroll
    for (int y = 0; y < D / 16; ++y) {
      const u32x2_t v0 = lds_transpose4(src + 16 * y * kPitch), v1 = lds_transpose4(src + (16 * y + 8) * kPitch);
      a[y] = as_bf16x8(u32x4_t{v0[0], v0[1], v1[0], v1[1]});
    }
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

template <int L>
struct LatentShape {
  static constexpr int kBatch = 128;                          // units resolved at a time
  static constexpr int kUnitElems = kUnit * kLatentPitch<L>;  // a unit's rows in LDS
};

// x + both halves of a pair of bf16.
__device__ __forceinline__ float add_pair(uint32_t pair, float x) {
  constexpr uint32_t kOnes = 0x3F803F80u;
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(s16x2, pair), __builtin_bit_cast(s16x2, kOnes), x, false);
}

// Scales rows whose registers are accumulators.  (The compiler would otherwise keep them, for the multiplications' sake,
// where the matrix products cannot: of 32 x 512 it spills most.)
template <int D>
__device__ __forceinline__ void scale_rows(Rows<32, D>& rows, float f) {
#pragma unroll
  for (int n = 0; n < D / 32; ++n) {
    f32x16 x = rows.o[n];
    asm volatile("" : "+a"(x));
    f32x16 y = x * f;
    asm volatile("" : "+a"(y));
    rows.o[n] = y;
    issue_first();
  }
}

// Tiles of 32 RG rows: wave w has the 32 rows w / (4 / RG) of the tile and, of the second product, a share of the
// columns; waves with the same rows make their scores each for itself.
template <int FMT, int L, int RG>
__global__ __launch_bounds__(kThreads, 1) void latent_attend_kernel(LatentArgs x, int splits, int64_t tiles,
                                                                 const uint16_t* __restrict__ query_rows,
                                                                 uint16_t* __restrict__ sums,
                                                                 float* __restrict__ part_o,
                                                                 RowState* __restrict__ part_ml) {
  using P = Part<FMT, L>;
  using S = LatentShape<L>;
  constexpr int kPitch = kLatentPitch<L>, kShare = 4 / RG, kColumns = L / kShare;
  constexpr int kSteps = (L + kRopeDim) / 16;
  constexpr int kBlocks = kColumns / 32;
  extern __shared__ int dyn[];  // of the chunk list: ub[k + 1], tb[k + 1]
  __shared__ __align__(16) uint16_t unit_rows[3][S::kUnitElems];
  __shared__ Unit list[S::kBatch];
  __shared__ int tmp[2 * kWaves];
  // Tokens of a masked unit whose values are not finite: of the unit at hand, of the next, and of the one after that,
  // which is cleared (so that a barrier stands between clearing and noting, and between noting and reading).
  __shared__ uint32_t bad_tok[3];

  const AttendArgs& a = x.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int rg = wave / kShare, cg = wave % kShare;
  const uint32_t tile = blockIdx.x / static_cast<uint32_t>(splits);
  const int split = static_cast<int>(blockIdx.x - tile * splits);
  Tile t;
  if (!find_tile<32 * RG>(a, static_cast<uint32_t>(tiles) - 1 - tile, a.hq, &t)) return;
  const ChunkList list_of = scan_list<kThreads, false>(a, t.req, dyn, tmp);
  const int ctx = list_of.tb[a.k];
  const int prefix = a.prefix_len ? __builtin_amdgcn_readfirstlane(min(max(a.prefix_len[t.req], 0), kFar)) : 0;
  const int my_row = t.r0 + min(32 * rg + col, t.rows - 1);
  const bool works = 32 * rg < t.rows;
  const RowRule rule = row_rule(a, t, ctx, 0, a.hq, my_row);
  const TileRule tr = tile_rule<32 * RG>(a, t, ctx, 0, a.hq);
  const Span span = visible_units(list_of, prefix, tr.lo, tr.hi);
  const int n_units = __builtin_amdgcn_readfirstlane(span.count());
  const int u0 = static_cast<int>(static_cast<int64_t>(n_units) * split / splits);
  const int u1 = static_cast<int>(static_cast<int64_t>(n_units) * (split + 1) / splits);

  // lane (col, half) holds elements 16 s + 8 half .. + 7 of row `col` of the wave
  bf16x8 q[kSteps];
  const int64_t row_at = static_cast<int64_t>(t.q0) * a.hq + my_row;
  load_queries(query_rows + row_at * kQueryRow<L> + 8 * half, 16, q);

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
  int value_at;  // transposed operands: rows 4 half + .. of the unit, 16 columns
  {
    const int i = lane & 15, r = 4 * half + (i >> 2), cc = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    value_at = r * kPitch + 8 * (cc ^ exchange(r)) + 4 * (i & 1) + cg * kColumns;
  }
  P p;

  for (int last = u1 - 1; last >= u0; last -= S::kBatch) {
    __syncthreads();
    const int n = resolve_units<S::kBatch>(a, list_of, span, tr, prefix, 0, P::kRow, last, min(S::kBatch, last - u0 + 1),
                                           list, tmp);
    if (n == 0) continue;
    if (tid < 2) bad_tok[tid] = 0;
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
    auto load_scales = [&](const Place& from) {
      if constexpr (FMT != MEM_KV_BF16) {
#pragma unroll
        for (int i = 0; i < P::kScaleWords / 2; ++i) {
          const u32x2_t v = reinterpret_cast<const u32x2_t*>(from.scales + from.row * P::kSc)[i];
          p.sc[2 * i] = v[0];
          p.sc[2 * i + 1] = v[1];
        }
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
      load_scales(from);
    }
    if (u.masked()) check(u, 0);
    {
      uint16_t* to = unit_rows[0] + tok * kPitch;
      const Place from = place(next);
#pragma unroll
      for (int z = 0; z < P::kPieces; ++z) advance(to, from, z);
      load_scales(from);
    }
    __syncthreads();
    // Weights of the unit before: its second product is made beside the exponentials of the unit at hand.
    u32x4_t w[2];
    bool pending = false;
    int slot = 0;  // i mod 3: the unit's buffer, and its word of bad_tok
    for (int i = 0; i <= n; ++i) {
      const Unit after = uniform_unit(list[min(i + 2, n - 1)]);
      const int slot1 = slot == 2 ? 0 : slot + 1, slot2 = slot == 0 ? 2 : slot - 1;
      const bool has = i < n;
      if (tid == 0) bad_tok[slot2] = 0;
      if (i + 1 < n && next.masked()) check(next, slot1);
      uint16_t* to = unit_rows[slot1] + tok * kPitch;
      const Place from = place(after);
      if (works) {
        const uint16_t* keys = unit_rows[slot];
        const uint16_t* values = unit_rows[slot2] + value_at;
        f32x16 s;
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = 0.f;
        constexpr int kFirst = (P::kPieces + 1) / 2;  // pieces beside the first product
        if (has) {
          constexpr int kAhead = 3;
          auto key = [&](int y) {
            return *reinterpret_cast<const u32x4_t*>(keys + (y & 1 ? odd : even) + 32 * (y >> 1));
          };
          u32x4_t k[kSteps];
#pragma unroll
          for (int y = 0; y < kAhead; ++y) k[y] = key(y);
          issue_first();
#pragma unroll
          for (int y = 0; y < kSteps; ++y) {
            if (y + kAhead < kSteps) k[y + kAhead] = key(y + kAhead);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[y]), q[y], s, 0, 0, 0);
            if (y * kFirst / kSteps != (y + 1) * kFirst / kSteps) advance(to, from, y * kFirst / kSteps);
            issue_first();
          }
        }
        bool counts = false;
        float high = -INFINITY;
        if (has) {
          if (u.masked()) {
            const uint32_t seen = visible_tokens(rule, u, prefix);
            mask_scores<32, 16>(s, seen, half);
            poison |= (seen & bad_tok[slot]) != 0;
          }
          float top = s[0];
#pragma unroll
          for (int j = 1; j < 16; ++j) top = nan_max(top, s[j]);
          high = max_column<32>(top) * c;
          counts = __any(!u.masked() || high != -INFINITY);
        }
        auto value = [&](int x) {  // operand x: columns 32 (x / 2), tokens 16 (x % 2)
          const uint16_t* src = values + 16 * (x & 1) * kPitch + 32 * (x >> 1);
          const u32x2_t v0 = lds_transpose4(src), v1 = lds_transpose4(src + 8 * kPitch);
          return as_bf16x8(u32x4_t{v0[0], v0[1], v1[0], v1[1]});
        };
        constexpr int kOps = 2 * kBlocks;
        auto add = [&](const u32x4_t (&by)[2], auto share) {
          constexpr int kAhead = 2;
          bf16x8 v[kOps];
#pragma unroll
          for (int x = 0; x < kAhead; ++x) v[x] = value(x);
          issue_first();
#pragma unroll
          for (int x = 0; x < kOps; ++x) {
            if (x + kAhead < kOps) v[x + kAhead] = value(x + kAhead);
            rows.o[x >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[x], as_bf16x8(by[x & 1]), rows.o[x >> 1], 0, 0, 0);
            share(x);
            issue_first();
          }
        };
        const bool up = counts && __any(high > st.m + kLag);
        u32x4_t now[2];
        auto weigh_score = [&](float ref, int j) {
          s[j] = fast_exp2(fmaf(s[j], c, -ref));
          st.l += s[j];
          if (j & 1) {
            const uint32_t pair = pack2(s[j - 1], s[j]);
            now[j >> 3][(j >> 1) & 3] = pair;
            rounded = add_pair(pair, rounded);
          }
        };
        // The usual way: both in one.  (Two flags that the compiler does not know to be one: with an if and an else
        // over the same accumulators it keeps them twice.)
        const bool usual = pending && counts && !up;
        int usual_too = __builtin_amdgcn_readfirstlane(usual);
        asm volatile("" : "+s"(usual_too));
        if (!usual) {
          if (pending) add(w, [](int) {});
          if (up) {
            const float mn = fmaxf(st.m, high);
            const float r = mn == -INFINITY ? 1.f : fast_exp2(st.m - mn);
            st.l *= r;
            rounded *= r;
            scale_rows(rows, r);
            st.m = mn;
          }
          if (counts) {
            const float ref = finite_max(st.m);
#pragma unroll
            for (int j = 0; j < 16; ++j) weigh_score(ref, j);
          }
#pragma unroll
          for (int z = kFirst; z < P::kPieces; ++z) advance(to, from, z);
        }
        if (usual_too) {
          const float ref = finite_max(st.m);
          add(w, [&](int x) {
            constexpr int kSecond = P::kPieces - kFirst;
#pragma unroll
            for (int j = 16 * x / kOps; j < 16 * (x + 1) / kOps; ++j) weigh_score(ref, j);
#pragma unroll
            for (int z = kSecond * x / kOps; z < kSecond * (x + 1) / kOps; ++z) advance(to, from, kFirst + z);
          });
        }
        if (!has) break;
        pending = counts;
        w[0] = now[0];
        w[1] = now[1];
      } else {
        if (!has) break;
#pragma unroll
        for (int z = 0; z < P::kPieces; ++z) advance(to, from, z);
      }
      load_scales(from);
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
  if (splits == 1) {
    const float inv = poison ? NAN : inverse_sum(rounded);
    uint16_t* dst = sums + row_at * L + cg * kColumns;
    rows.each4(half, [&](int d, f32x4 v) {
      *reinterpret_cast<u32x2_t*>(dst + d) = u32x2_t{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
    });
    if (a.lse && half == 0 && cg == 0) a.lse[row_at] = poison ? NAN : lse_of(st.m, st.l);
  } else {
    const int64_t at = static_cast<int64_t>(split) * a.total_q * a.hq + row_at;
    float* dst = part_o + at * L + cg * kColumns;
    const float even_out = poison ? NAN : st.l == 0.f ? 0.f : st.l * inverse_sum(rounded);  // the join divides by l
    rows.each4(half, [&](int d, f32x4 v) {
      *reinterpret_cast<f32x4*>(dst + d) = v * even_out;
    });
    if (half == 0 && cg == 0) part_ml[at] = poison ? RowState{st.m, NAN} : st;
  }
}

// ---------------------------------------------------------------- outputs

// Workgroup (head, 32 or 64 tokens): a wave has 32 of the output's elements for 32 tokens.
template <int L, int D>
__global__ __launch_bounds__(kThreads) void latent_out_kernel(LatentArgs x, const uint16_t* __restrict__ sums) {
  constexpr int kAcross = D / 32, kBlocks = kWaves / kAcross;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5, j0 = 32 * (wave % kAcross);
  const int h = blockIdx.x;
  const int64_t tok0 = (static_cast<int64_t>(blockIdx.y) * kBlocks + wave / kAcross) * kTokenBlock, tok = tok0 + col;
  if (tok0 >= x.a.total_q) return;
  const uint16_t* w = x.w + h * x.w_hs + (D + j0 + col) * x.w_rs + 8 * half;
  const uint16_t* s = sums + (min(tok, x.a.total_q - 1) * x.a.hq + h) * L + 8 * half;
  f32x16 o;
#pragma unroll
  for (int j = 0; j < 16; ++j) o[j] = 0.f;
#pragma unroll 8
  for (int y = 0; y < L / 16; ++y)
    o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*reinterpret_cast<const u32x4_t*>(w + 16 * y)),
                                                as_bf16x8(*reinterpret_cast<const u32x4_t*>(s + 16 * y)), o, 0, 0, 0);
  if (tok >= x.a.total_q) return;
  if (x.a.q_offsets && (tok < x.a.q_offsets[0] || tok >= x.a.q_offsets[x.a.m])) return;  // no request's
  uint16_t* dst = x.out + (tok * x.a.hq + h) * D + j0 + 4 * half;
#pragma unroll
  for (int y = 0; y < 4; ++y)
    *reinterpret_cast<u32x2_t*>(dst + 8 * y) =
        u32x2_t{pack2(o[4 * y], o[4 * y + 1]), pack2(o[4 * y + 2], o[4 * y + 3])};
}

// ---------------------------------------------------------------- launches

size_t align256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }
size_t list_bytes(int k) { return (2 * static_cast<size_t>(k) + 2) * sizeof(int); }

struct AbsorbedPlan {
  int rg;  // tiles of 32 rg rows
  int64_t tiles;
  int splits;
};

constexpr int64_t kStart = 16;  // a workgroup's start and end, in units

AbsorbedPlan absorbed_plan(const LatentSizes& s, bool ragged) {
  AbsorbedPlan p;
  const int64_t rows = s.total_q * s.heads;
  p.rg = rows <= 32 * s.m ? 1 : rows <= 64 * s.m ? 2 : 4;
  const int R = 32 * p.rg;
  p.tiles = ragged ? rows / R + s.m : s.m * ((s.total_q / s.m * s.heads + R - 1) / R);
  const int64_t work = ragged ? (rows + R - 1) / R + s.m / 2 : p.tiles, slots = 256;
  int64_t best = INT64_MAX;
  p.splits = 1;
  for (int64_t n = 1; n <= kMaxSplits && (n == 1 || s.units / n >= 4); ++n) {
    if (n > 1 && (p.tiles * n > kMaxGroups || join_groups(rows, n) > kMaxGroups)) break;
    const int64_t cost = (work * n + slots - 1) / slots * ((s.units + n - 1) / n + kStart) + (n > 1 ? n / 4 : 0);
    if (cost < best) {
      best = cost;
      p.splits = static_cast<int>(n);
    }
  }
  return p;
}

// Workspace of the absorbed form: query rows, sums, and the parts of split contexts.
struct AbsorbedSpace {
  size_t queries, sums, part_o, part_ml, end;
};

AbsorbedSpace absorbed_space(const LatentSizes& s, int splits) {
  const size_t rows = static_cast<size_t>(s.total_q) * s.heads;
  AbsorbedSpace w;
  w.queries = 0;
  w.sums = align256(rows * (s.latent + kRopeDim) * 2);
  w.part_o = w.sums + align256(rows * s.latent * 2);
  w.part_ml = w.part_o + (splits > 1 ? align256(splits * rows * s.latent * sizeof(float)) : 0);
  w.end = w.part_ml + (splits > 1 ? align256(splits * rows * sizeof(RowState)) : 0);
  return w;
}

constexpr int kQueryBlocks = 8;  // blocks of tokens of a workgroup of latent_query_kernel
int64_t query_groups(int64_t total_q) {
  return (total_q + kQueryBlocks * kTokenBlock - 1) / (kQueryBlocks * kTokenBlock);
}
int64_t out_groups(int64_t total_q, int d) {
  const int tokens = kTokenBlock * kWaves / (d / 32);
  return (total_q + tokens - 1) / tokens;
}

template <int FMT, int L, int D>
hipError_t launch_absorbed(const LatentArgs& x, const LatentSizes& s, hipStream_t stream) {
  const AbsorbedPlan p = absorbed_plan(s, x.a.q_offsets != nullptr);
  const AbsorbedSpace at = absorbed_space(s, p.splits);
  uint8_t* ws = static_cast<uint8_t*>(x.ws);
  uint16_t* queries = reinterpret_cast<uint16_t*>(ws + at.queries);
  uint16_t* sums = reinterpret_cast<uint16_t*>(ws + at.sums);
  float* part_o = reinterpret_cast<float*>(ws + at.part_o);
  RowState* part_ml = reinterpret_cast<RowState*>(ws + at.part_ml);
  latent_query_kernel<L, D><<<dim3(s.heads, L / 128, static_cast<unsigned>(query_groups(s.total_q))), kThreads, 0,
                              stream>>>(x, kQueryBlocks, queries);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const unsigned grid = static_cast<unsigned>(p.tiles * p.splits);
  (p.rg == 1   ? latent_attend_kernel<FMT, L, 1>
   : p.rg == 2 ? latent_attend_kernel<FMT, L, 2>
               : latent_attend_kernel<FMT, L, 4>)<<<grid, kThreads, list_bytes(s.k), stream>>>(
      x, p.splits, p.tiles, queries, sums, part_o, part_ml);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (p.splits > 1) {
    AttendArgs j = x.a;
    j.out = sums;
    const dim3 join(static_cast<unsigned>(join_groups(s.total_q * s.heads, p.splits)));
    if (p.splits <= kJoinSplits)
      attend_join_kernel<L, 1><<<join, kThreads, 0, stream>>>(j, p.splits, part_o, part_ml);
    else
      attend_join_kernel<L, kWaves><<<join, kThreads, 0, stream>>>(j, p.splits, part_o, part_ml);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  latent_out_kernel<L, D><<<dim3(s.heads, static_cast<unsigned>(out_groups(s.total_q, D))), kThreads, 0, stream>>>(x,
                                                                                                                sums);
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
  // products of a head, in units of a pair's 2 elements each: rows (2 L + R) absorbed, rows (2 d + R) and 2 d L for
  // each token of the context expanded
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
  return p.tiles * p.splits <= kMaxGroups && query_groups(s.total_q) < 65536 && out_groups(s.total_q, s.head_dim) < 65536;
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
