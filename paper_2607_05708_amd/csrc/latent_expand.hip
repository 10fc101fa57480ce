// Latent attention, expanded form: keys and values of the context are made of the
// latent vectors first, in the workspace, for as many heads at a time as fit it.
//
//   latent_units_kernel     where each request's units of 32 tokens lie
//   latent_expand_kernel    keys [W_h c, r] and values V_h c of all units, bf16
//   expanded_attend_kernel  attention over them, head by head
//   attend_join_kernel      joins the parts of split contexts
//
// Of a head, a unit's keys are one block [element / 8][token][element % 8], its values one of [token / 16][token / 4 % 2]
// [element][token / 8 % 2][token % 4]: in both, the 16 bytes that a lane of a matrix product has lie next to its
// neighbours'.  Blocks are written, copied into LDS and read there in whole lines, without bank conflicts, and the values
// come transposed as the second product takes them.
#include <algorithm>
#include <type_traits>

#include "context.h"
#include "kv.h"
#include "latent.h"
#include "latent_rows.h"
#include "device_common.h"

namespace memattn {

namespace {

// A unit of a request's context: byte of the pool at which its first latent row starts (-1: not in the pool), its first
// row in the page, its tokens.
struct Source {
  int64_t at;
  int32_t row;
  int32_t held;
};

// Rows of L elements in LDS: see kLatentPitch.
template <int L>
constexpr int kPitchOf = L + 32;

// ---------------------------------------------------------------- units

__global__ __launch_bounds__(kThreads) void latent_units_kernel(AttendArgs a, int row_bytes, int64_t units,
                                                              Source* __restrict__ sources, int* __restrict__ counts) {
  extern __shared__ int dyn[];
  __shared__ int tmp[2 * kWaves];
  const int req = blockIdx.x;
  const ChunkList L = scan_list<kThreads, false>(a, req, dyn, tmp);
  const int n = L.ub[a.k];
  if (threadIdx.x == 0) {
    counts[req] = n;
    counts[a.m + req] = 0;  // whether some value made of the context is not finite
  }
  for (int u = threadIdx.x; u < n; u += kThreads) {
    const int c = find_entry(L.ub, L.k, u);
    const int t = (u - L.ub[c]) * kUnit;
    const int p = t / a.kv.page_tokens, row = t - p * a.kv.page_tokens;
    const int32_t pg = a.kv.table[static_cast<int64_t>(L.cid[c]) * a.kv.ppc + p];
    const bool ok = pg >= 0 && pg < a.kv.n_pages;
    sources[req * units + u] = Source{ok ? pg * a.kv.page_bytes + static_cast<int64_t>(row) * row_bytes : -1, row,
                                      min(kUnit, L.tb[c + 1] - L.tb[c] - t)};
  }
}

// ---------------------------------------------------------------- keys and values

constexpr int kGroupUnits = 4;                     // units of a workgroup
constexpr int kGroupTokens = kGroupUnits * kUnit;  // 128

// Workgroup (four units of a request, a share of the heads): the tokens' latent vectors stay in LDS as bf16; for each
// head a wave makes a quarter of its keys' and values' elements for all 128 tokens, its rows of W and V straight from
// memory.  The order of a product's k is free as long as both operands have it: lane (row, half) takes 64 consecutive
// bytes of each 128 of its row.  Keys and values are rounded to bf16 as the attention's operands: as two numbers each they
// would take twice the memory and 1.7 to 1.8 times the attention's products.  Units that no row sees are made too.
// Bound by the waits for its loads and stores, which leave in order (matrix cores busy 31 to 35 %): 4 x 8,192 tokens of 8
// bits, 16 heads, 253 us with the latent vectors of a group loaded one after the other, 174 with all at once and W's and
// V's rows for the next head on their way.
template <int FMT, int L, int D>
__global__ __launch_bounds__(kThreads, 1) void latent_expand_kernel(LatentArgs x, int64_t units,
                                                                 const Source* __restrict__ sources,
                                                                 int* __restrict__ counts, int h0, int heads,
                                                                 int per, uint16_t* __restrict__ keys,
                                                                 uint16_t* __restrict__ values) {
  constexpr int kPitch = kPitchOf<L>, kKeyRow = D + kRopeDim, kMine = 2 * D / kWaves, kBlocks = kMine / 32;  // rows of W and V of a wave
  __shared__ __align__(16) uint16_t rows[kGroupTokens * kPitch];
  const AttendArgs& a = x.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int64_t groups = (units + kGroupUnits - 1) / kGroupUnits;
  const int req = static_cast<int>(blockIdx.x / groups);
  const int u0 = static_cast<int>(blockIdx.x - req * groups) * kGroupUnits;
  const int n = counts[req];
  if (u0 >= n) return;
  const int64_t T = a.kv.page_tokens, slots = a.m * units * kUnit;       // rows of a head
  const int64_t slot0 = (req * units + u0) * kUnit;

  // latent vectors into LDS, and the key parts into the heads' keys
  const int hb = blockIdx.y * per, he = min(hb + per, heads);
  {
    const int tok = tid >> 3, part = tid & 7;
    Part<FMT, L> p[kGroupUnits];
    bool held[kGroupUnits];
#pragma unroll
    for (int k = 0; k < kGroupUnits; ++k) {
      const Source s = sources[req * units + min(u0 + k, n - 1)];
      held[k] = u0 + k < n && s.at >= 0 && tok < s.held;
      const int64_t at = max(s.at, int64_t{0}) - (s.at >= 0 ? static_cast<int64_t>(s.row) * Part<FMT, L>::kRow : 0);
      p[k].clear();
      if (held[k]) p[k].load(a.kv.pool + at, T, s.row + tok, part);
    }
#pragma unroll
    for (int k = 0; k < kGroupUnits; ++k) {
      const int t = kUnit * k + tok;
#pragma unroll
      for (int z = 0; z < Part<FMT, L>::kPieces - 1; ++z) p[k].store(rows + t * kPitch, exchange(t), part, z);
      if (held[k])
        for (int h = hb; h < he; ++h)
          *reinterpret_cast<u32x4_t*>(keys + (h * slots + slot0 + kUnit * k) * kKeyRow +
                                      ((D / 8 + part) * kUnit + tok) * 8) = p[k].rope;
    }
  }
  __syncthreads();

  const int f = exchange(col);
  // W and V: a wave's rows, 128 elements a step, loaded again for the next step (maybe of the next head) as soon as a
  // line has been used.
  constexpr int kStep = 128, kHeadSteps = L / kStep;
  // Waves that make values have the product's other order, so that a lane gets tokens of an element.
  auto make = [&](auto which) {
    constexpr bool kValues = decltype(which)::value;
    u32x4_t w[kBlocks][8];
    auto load = [&](int h, int s, int b, int y) {
      const uint16_t* src = x.w + (h0 + h) * x.w_hs + (wave * kMine + 32 * b + col) * x.w_rs + 32 * half + kStep * s;
      w[b][y] = *reinterpret_cast<const u32x4_t*>(src + 64 * (y >> 2) + 8 * (y & 3));
    };
#pragma unroll
    for (int y = 0; y < 8; ++y)
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) load(hb, 0, b, y);
    for (int h = hb; h < he; ++h) {
      f32x16 o[kBlocks][kGroupUnits];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int u = 0; u < kGroupUnits; ++u)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[b][u][j] = 0.f;
#pragma unroll 1
      for (int s = 0; s < kHeadSteps; ++s) {
        const bool last = s + 1 == kHeadSteps;
        const int next_h = last ? min(h + 1, he - 1) : h, next_s = last ? 0 : s + 1;
        const uint16_t* src = rows + col * kPitch + kStep * s + 32 * half;
        auto token = [&](int i) {  // operand of y = i / 4 and unit i % 4
          const int y = i / kGroupUnits, u = i % kGroupUnits;
          return as_bf16x8(*reinterpret_cast<const u32x4_t*>(src + 32 * u * kPitch + 64 * (y >> 2) + 8 * ((y & 3) ^ f)));
        };
        constexpr int kAhead = 4, kAll = 8 * kGroupUnits;
        bf16x8 k[kAll];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) k[i] = token(i);
        issue_first();
#pragma unroll
        for (int i = 0; i < kAll; ++i) {
          const int y = i / kGroupUnits, u = i % kGroupUnits;
          if (i + kAhead < kAll) k[i + kAhead] = token(i + kAhead);
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
            o[b][u] = kValues ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[i], as_bf16x8(w[b][y]), o[b][u], 0, 0, 0)
                              : __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(w[b][y]), k[i], o[b][u], 0, 0, 0);
          if (u + 1 == kGroupUnits && y % 4 == 3) {  // the four loads of a line together, while it is in the cache
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
              for (int z = y - 3; z <= y; ++z) load(next_h, next_s, b, z);
          }
          issue_first();
        }
      }
      u16x2 most = {0, 0};
      uint16_t* dst = kValues ? values + (h * slots + slot0) * D + (wave * kMine - D + col + half * D) * 8
                              : keys + (h * slots + slot0) * kKeyRow + wave * kMine * kUnit + col * 8 + 4 * half;
#pragma unroll
      for (int u = 0; u < kGroupUnits; ++u) {
        if (u0 + u >= n) break;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
          u32x4_t v[2];
#pragma unroll
          for (int y = 0; y < 8; ++y) v[y >> 2][y & 3] = pack2(o[b][u][2 * y], o[b][u][2 * y + 1]);
          if constexpr (kValues) {  // a lane has an element's tokens
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              *reinterpret_cast<u32x4_t*>(dst + u * kUnit * D + (2 * y * D + 32 * b) * 8) = v[y];
#pragma unroll
              for (int j = 0; j < 4; ++j)
                most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, v[y][j] & 0x7FFF7FFFu));
            }
          } else {                  // a token's elements
#pragma unroll
            for (int y = 0; y < 4; ++y)
              *reinterpret_cast<u32x2_t*>(dst + u * kUnit * kKeyRow + (4 * b + y) * kUnit * 8) =
                  u32x2_t{v[y >> 1][2 * (y & 1)], v[y >> 1][2 * (y & 1) + 1]};
          }
        }
      }
      if (kValues && (most[0] >= 0x7F80u || most[1] >= 0x7F80u)) counts[a.m + req] = 1;
    }
  };
  if (wave * kMine >= D)
    make(std::true_type{});
  else
    make(std::false_type{});
}

// ---------------------------------------------------------------- attention

constexpr int kTileRows = 128;

template <int D>
struct ExpandedShape {
  static constexpr int kKey = D + kRopeDim;
  static constexpr int kBatch = 128;  // units resolved at a time
};

// 16 bytes from `base` + `from` of each lane to LDS, lane after lane from `to` on.  In assembly, as the compiler would wait
// for it at the next read of any LDS: wait_for_lds() and a barrier stand between it and what reads it.  M0 is the
// compiler's to save, whose code here does not use it (a host test looks); a wait state has to follow its write.
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t from, const uint16_t* to) {
  const uint32_t at = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) uint16_t*)to));
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(from), "s"(base), "s"(__builtin_amdgcn_readfirstlane(at))
               : "memory");
}
__device__ __forceinline__ void wait_for_lds() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Tiles of 128 rows (new tokens) of a head, 32 a wave.  A step t makes the scores of unit t, the weights of unit t - 1
// and the second product of unit t - 2, while unit t + 1 goes straight into LDS: a wave issues in order, so that only what
// stands between its matrix products overlaps with them, and the exponentials are shared out over all of a step's.  They go by the
// running maximum as it is; where a score turns out to be above it by more than the lag (rare: the largest score of a
// unit is known at the end of its step), that unit's are made again.
// Bound by issue and the waits at a step's end: 8,192 tokens behind 24,576, 32 heads of 128, 4,830 us (5,150 on another
// MI355X), the matrix cores busy in 45 % and the vector unit issuing in 42 % of the cycles.  5,320 with rows in a pitch and values transposed on their way
// out of LDS (a quarter of whose cycles were bank conflicts); 5,170 with blocks as they lie in the workspace, through
// registers, 13 of which were spilled.  Units loaded two steps ahead change nothing with heads of 64.
template <int D>
__global__ __launch_bounds__(kThreads, 2) void expanded_attend_kernel(LatentArgs x, int splits, int64_t tiles,
                                                                   int64_t units, int h0, int heads,
                                                                   const uint16_t* __restrict__ key_rows,
                                                                   const uint16_t* __restrict__ value_rows,
                                                                   const int* __restrict__ counts,
                                                                   float* __restrict__ part_o,
                                                                   RowState* __restrict__ part_ml) {
  using S = ExpandedShape<D>;
  constexpr int kSteps = S::kKey / 16, kBlocks = D / 32, kOps = 2 * kBlocks;
  constexpr int kKeyChunks = S::kKey / 8, kValueChunks = D / 8;              // 16-byte chunks of a row
  constexpr int kKeyLoads = kUnit * kKeyChunks / kThreads, kValueLoads = kUnit * kValueChunks / kThreads;
  constexpr int kPieces = kKeyLoads + kValueLoads;
  static_assert(kUnit * kKeyChunks % kThreads == 0 && kUnit * kValueChunks % kThreads == 0, "whole loads");
  extern __shared__ int dyn[];  // of the chunk list: ub[k + 1], tb[k + 1]
  __shared__ __align__(16) uint16_t keys[2][kUnit * S::kKey];
  __shared__ __align__(16) uint16_t values[4][kUnit * D];
  __shared__ Unit list[S::kBatch];
  __shared__ int tmp[2 * kWaves];
  __shared__ uint32_t bad_tok[4];  // tokens of a masked unit whose values are not finite

  const AttendArgs& a = x.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const uint32_t b = blockIdx.x / static_cast<uint32_t>(heads), tile = b / static_cast<uint32_t>(splits);
  const int g = static_cast<int>(blockIdx.x - b * heads), split = static_cast<int>(b - tile * splits);
  Tile t;
  if (!find_tile<kTileRows>(a, static_cast<uint32_t>(tiles) - 1 - tile, 1, &t)) return;  // the latest rows see most: first
  const ChunkList list_of = scan_list<kThreads, false>(a, t.req, dyn, tmp);
  const int ctx = list_of.tb[a.k];
  const int prefix = a.prefix_len ? __builtin_amdgcn_readfirstlane(min(max(a.prefix_len[t.req], 0), kFar)) : 0;
  const int my_row = t.r0 + min(32 * wave + col, t.rows - 1);
  const RowRule rule = row_rule(a, t, ctx, g, 1, my_row);
  const TileRule tr = tile_rule<kTileRows>(a, t, ctx, g, 1);
  const Span span = visible_units(list_of, prefix, tr.lo, tr.hi);
  const int n_units = __builtin_amdgcn_readfirstlane(span.count());
  const int u0 = static_cast<int>(static_cast<int64_t>(n_units) * split / splits);
  const int u1 = static_cast<int>(static_cast<int64_t>(n_units) * (split + 1) / splits);

  bf16x8 q[kSteps];
  const int64_t tok_at = t.q0 + my_row;
  {
    bf16x8 own[D / 16], turned[kRopeDim / 16];
    load_queries(static_cast<const uint16_t*>(x.q.data) + tok_at * x.q.ts + (h0 + g) * x.q.hs + 8 * half, 16, own);
    load_queries(static_cast<const uint16_t*>(x.t.data) + tok_at * x.t.ts + (h0 + g) * x.t.hs + 8 * half, 16, turned);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) q[i] = i < D / 16 ? own[i < D / 16 ? i : 0] : turned[i < D / 16 ? 0 : i - D / 16];
  }
  const bool odd = counts[a.m + __builtin_amdgcn_readfirstlane(t.req)] != 0;
  const float c = a.scale * kLog2e;
  const int64_t row0 = (g * a.m + __builtin_amdgcn_readfirstlane(t.req)) * units * kUnit;
  const uint8_t* my_keys = reinterpret_cast<const uint8_t*>(key_rows + row0 * S::kKey);
  const uint8_t* my_values = reinterpret_cast<const uint8_t*>(value_rows + row0 * D);
  Rows<32, D> rows;
  rows.clear();
  RowState st{-INFINITY, 0.f};
  float rounded = 0.f;  // sum of the weights as the second product takes them
  bool poison = false;

  const int key_at = 8 * (half * kUnit + col), value_at = 8 * (half * D + col);

  for (int last = u1 - 1; last >= u0; last -= S::kBatch) {
    __syncthreads();
    const int n = resolve_units<S::kBatch, kThreads, true>(a, list_of, span, tr, prefix, 0, 0, last,
                                                         min(S::kBatch, last - u0 + 1), list, tmp);
    if (n == 0) continue;
    if (tid < 4) bad_tok[tid] = 0;
    // the first two steps' second products are of weights 0: their values have to be numbers
    for (int z = tid; z < 2 * kUnit * D / 8; z += kThreads)
      reinterpret_cast<u32x4_t*>(values[2])[z] = u32x4_t{0, 0, 0, 0};
    __syncthreads();
    // Piece z of a unit straight into LDS, 16 bytes a thread: of its keys (of token tid % 32), then of its values.
    auto load = [&](const Unit& u, int to, int z) {
      const uint8_t* src = z < kKeyLoads ? my_keys + u.at * (kUnit * S::kKey * 2) + z * (16 * kThreads)
                                         : my_values + u.at * (kUnit * D * 2) + (z - kKeyLoads) * (16 * kThreads);
      const uint16_t* dst = z < kKeyLoads ? keys[to & 1] + 8 * z * kThreads : values[to & 3] + 8 * (z - kKeyLoads) * kThreads;
      load_to_lds(src, 16 * tid, dst + 8 * 64 * wave);
    };
    // Where some value of the request is not finite: those of a masked unit are noted and left out.  (A unit's values
    // behind its tokens are 0, or not finite; its scores there are masked.)
    auto check = [&](const Unit& u, int to) {
      u32x4_t* value = reinterpret_cast<u32x4_t*>(values[to & 3]) + tid;
#pragma unroll
      for (int z = 0; z < kValueLoads; ++z) {
        u32x4_t p = value[z * kThreads];
        u16x2 most = {0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, p[j] & 0x7FFF7FFFu));
        if (most[0] < 0x7F80u && most[1] < 0x7F80u) continue;
        const int block = (z * kThreads + tid) / D;
        uint32_t bad = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int t = 16 * (block >> 1) + 4 * (block & 1) + 8 * (j >> 2) + (j & 3);
          const bool wrong = (p[j >> 1] >> 16 * (j & 1) & 0x7FFFu) >= 0x7F80u;
          if (wrong) p[j >> 1] &= 0xFFFFu << 16 * (1 - (j & 1));
          if (t < u.held() && wrong) bad |= 1u << t;
        }
        value[z * kThreads] = p;
        if (bad) atomicOr(&bad_tok[to & 3], bad);
      }
    };
    Unit u = uniform_unit(list[0]), next = uniform_unit(list[min(1, n - 1)]), old = u;
#pragma unroll
    for (int z = 0; z < kPieces; ++z) load(u, 0, z);
    wait_for_lds();
    if (odd && u.masked()) check(u, 0);
    __syncthreads();
    // Scores of units t and t - 1, weights of units t - 1 and t - 2: [t & 1] is made in step t.
    f32x16 s[2];
    u32x4_t w[2][2];
#pragma unroll
    for (int j = 0; j < 16; ++j) s[1][j] = -INFINITY;
    w[1][0] = w[1][1] = u32x4_t{0, 0, 0, 0};

    auto step = [&](auto parity, int i) {
      constexpr int kNew = decltype(parity)::value, kOld = 1 - kNew;
      f32x16 &sn = s[kNew], &so = s[kOld];
      const u32x4_t(&wo)[2] = w[kOld];
      u32x4_t(&wn)[2] = w[kNew];
      const Unit after = uniform_unit(list[min(i + 2, n - 1)]);
      if (tid == 0) bad_tok[(i + 2) & 3] = 0;
#pragma unroll
      for (int z = 0; z < kPieces; ++z) load(next, i + 1, z);
      if (i > 0 && i <= n && old.masked()) {
        const uint32_t seen = visible_tokens(rule, old, prefix);
        mask_scores<32, 16>(so, seen, half);
        poison |= (seen & bad_tok[(i + 3) & 3]) != 0;
      }
      const uint16_t* kp = keys[i & 1];
      const uint16_t* vp = values[(i + 2) & 3];
      float ref = finite_max(st.m), l = 0.f, lr = 0.f, top = so[0], e[2];
      auto weigh = [&](int j) {  // scores 2 j and 2 j + 1 of unit t - 1
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          e[y] = fast_exp2(fmaf(so[2 * j + y], c, -ref));
          l += e[y];
        }
        const uint32_t pair = pack2(e[0], e[1]);
        wn[j >> 2][j & 3] = pair;
        lr = add_pair(pair, lr);
      };
      constexpr int kSlots = kSteps + kOps;
      auto share = [&](int slot) {
#pragma unroll
        for (int j = 8 * slot / kSlots; j < 8 * (slot + 1) / kSlots; ++j) weigh(j);
      };
#pragma unroll
      for (int j = 0; j < 16; ++j) sn[j] = 0.f;
      {
        constexpr int kAhead = 3;
        auto key = [&](int y) {
          return *reinterpret_cast<const u32x4_t*>(kp + key_at + 16 * kUnit * y);
        };
        u32x4_t k[kSteps];
#pragma unroll
        for (int y = 0; y < kAhead; ++y) k[y] = key(y);
        issue_first();
#pragma unroll
        for (int y = 0; y < kSteps; ++y) {
          if (y + kAhead < kSteps) k[y + kAhead] = key(y + kAhead);
          sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[y]), q[y], sn, 0, 0, 0);
#pragma unroll
          for (int j = 16 * y / kSteps; j < 16 * (y + 1) / kSteps; ++j) top = nan_max(top, so[j]);
          share(y);
          issue_first();
        }
      }
      {  // the second product of unit t - 2: operand o has columns 32 (o / 2), tokens 16 (o % 2)
        constexpr int kAhead = 3;
        auto value = [&](int o) {
          return as_bf16x8(*reinterpret_cast<const u32x4_t*>(vp + value_at + 8 * (2 * (o & 1) * D + 32 * (o >> 1))));
        };
        bf16x8 v[kOps];
#pragma unroll
        for (int o = 0; o < kAhead; ++o) v[o] = value(o);
        issue_first();
#pragma unroll
        for (int o = 0; o < kOps; ++o) {
          if (o + kAhead < kOps) v[o + kAhead] = value(o + kAhead);
          rows.o[o >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[o], as_bf16x8(wo[o & 1]), rows.o[o >> 1], 0, 0, 0);
          share(kSteps + o);
          issue_first();
        }
      }
      const float high = max_column<32>(top) * c;
      if (__any(high > st.m + kLag)) {
        const float mn = fmaxf(st.m, high);
        const float by = mn == -INFINITY ? 1.f : fast_exp2(st.m - mn);
        st.l *= by;
        rounded *= by;
        rows.scale(by);
        st.m = mn;
        ref = finite_max(mn);
        l = lr = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) weigh(j);
      }
      st.l += l;
      rounded += lr;
      if (i >= n) {  // what follows the last unit weighs nothing
#pragma unroll
        for (int j = 0; j < 16; ++j) sn[j] = -INFINITY;
      }
      wait_for_lds();
      if (odd && i + 1 < n && next.masked()) check(next, i + 1);
      old = u;
      u = next;
      next = after;
      __syncthreads();
    };
    // Steps n and n + 1 only finish the last units.
    for (int i = 0; i < n + 2; i += 2) {
      step(std::integral_constant<int, 0>{}, i);
      if (i + 1 < n + 2) step(std::integral_constant<int, 1>{}, i + 1);
    }
  }

  st.l = sum_column<32>(st.l);
  rounded = sum_column<32>(rounded);
  poison = any_column<32>(poison, col);
  if (32 * wave + col >= t.rows) return;
  write_sums<32, D>(a, rows, st, rounded, poison, tok_at * a.hq + h0 + g, half, split, splits, x.out, part_o, part_ml);
}

// ---------------------------------------------------------------- launches

size_t align256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }
size_t list_bytes(int k) { return (2 * static_cast<size_t>(k) + 2) * sizeof(int); }

struct ExpandedPlan {
  int64_t tiles;
  int splits;
  int heads;  // at a time
};

constexpr int64_t kStart = 16;                            // a workgroup's start and end, in units
constexpr size_t kExpandBytes = size_t{1} << 30;          // of keys and values, unless a single head takes more

size_t head_bytes(const LatentSizes& s) {
  return static_cast<size_t>(s.m) * s.units * kUnit * (2 * s.head_dim + kRopeDim) * 2;
}

ExpandedPlan expanded_plan(const LatentSizes& s, bool ragged) {
  ExpandedPlan p;
  const int R = kTileRows;
  p.tiles = ragged ? s.total_q / R + s.m : s.m * ((s.total_q / s.m + R - 1) / R);
  p.heads = static_cast<int>(std::min<size_t>(std::max<size_t>(kExpandBytes / head_bytes(s), 1), s.heads));
  const int64_t filled = ragged ? (s.total_q + R - 1) / R + s.m / 2 : p.tiles, work = filled * p.heads, slots = 512;
  int64_t best = INT64_MAX;
  p.splits = 1;
  const int64_t most = work >= slots ? 1 : kMaxSplits;
  for (int64_t n = 1; n <= most && (n == 1 || s.units / n >= 4); ++n) {
    if (n > 1 && (p.tiles * p.heads * n > kMaxGroups || join_groups(s.total_q * s.heads, n) > kMaxGroups)) break;
    const int64_t cost = (work * n + slots - 1) / slots * ((s.units + n - 1) / n + kStart) + (n > 1 ? n / 4 : 0);
    if (cost < best) {
      best = cost;
      p.splits = static_cast<int>(n);
    }
  }
  return p;
}

struct ExpandedSpace {
  size_t sources, counts, keys, values, part_o, part_ml, end;
};

ExpandedSpace expanded_space(const LatentSizes& s, const ExpandedPlan& p) {
  const size_t rows = static_cast<size_t>(s.total_q) * s.heads, slots = static_cast<size_t>(s.m) * s.units * kUnit;
  ExpandedSpace w;
  w.sources = 0;
  w.counts = align256(static_cast<size_t>(s.m) * s.units * sizeof(Source));
  w.keys = w.counts + align256(2 * s.m * sizeof(int));
  w.values = w.keys + align256(p.heads * slots * (s.head_dim + kRopeDim) * 2);
  w.part_o = w.values + align256(p.heads * slots * s.head_dim * 2);
  w.part_ml = w.part_o + (p.splits > 1 ? align256(p.splits * rows * s.head_dim * sizeof(float)) : 0);
  w.end = w.part_ml + (p.splits > 1 ? align256(p.splits * rows * sizeof(RowState)) : 0);
  return w;
}

int64_t expand_groups(const LatentSizes& s) { return s.m * ((s.units + kGroupUnits - 1) / kGroupUnits); }

template <int FMT, int L, int D>
hipError_t launch(const LatentArgs& x, const LatentSizes& s, hipStream_t stream) {
  const ExpandedPlan p = expanded_plan(s, x.a.q_offsets != nullptr);
  const ExpandedSpace at = expanded_space(s, p);
  uint8_t* ws = static_cast<uint8_t*>(x.ws);
  Source* sources = reinterpret_cast<Source*>(ws + at.sources);
  int* counts = reinterpret_cast<int*>(ws + at.counts);
  uint16_t* keys = reinterpret_cast<uint16_t*>(ws + at.keys);
  uint16_t* values = reinterpret_cast<uint16_t*>(ws + at.values);
  float* part_o = reinterpret_cast<float*>(ws + at.part_o);
  RowState* part_ml = reinterpret_cast<RowState*>(ws + at.part_ml);
  latent_units_kernel<<<static_cast<unsigned>(s.m), kThreads, list_bytes(s.k), stream>>>(
      x.a, kv_row_bytes(FMT, L), s.units, sources, counts);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  for (int h0 = 0; h0 < s.heads; h0 += p.heads) {
    const int heads = std::min(p.heads, s.heads - h0);
    const int64_t groups = expand_groups(s);
    // heads are shared out where the groups of units alone leave CUs idle
    const int shares = static_cast<int>(std::min<int64_t>(heads, std::max<int64_t>(1, 512 / groups)));
    const int per = (heads + shares - 1) / shares;
    latent_expand_kernel<FMT, L, D><<<dim3(static_cast<unsigned>(groups), (heads + per - 1) / per), kThreads, 0,
                                      stream>>>(x, s.units, sources, counts, h0, heads, per, keys, values);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    expanded_attend_kernel<D><<<static_cast<unsigned>(p.tiles * heads * p.splits), kThreads, list_bytes(s.k),
                                stream>>>(x, p.splits, p.tiles, s.units, h0, heads, keys, values, counts, part_o,
                                part_ml);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (p.splits > 1) {
    AttendArgs j = x.a;
    j.out = x.out;
    const dim3 join(static_cast<unsigned>(join_groups(s.total_q * s.heads, p.splits)));
    if (p.splits <= kJoinSplits)
      attend_join_kernel<D, 1><<<join, kThreads, 0, stream>>>(j, p.splits, part_o, part_ml);
    else
      attend_join_kernel<D, kWaves><<<join, kThreads, 0, stream>>>(j, p.splits, part_o, part_ml);
    return hipGetLastError();
  }
  return hipSuccess;
}

template <int FMT>
hipError_t launch_fmt(const LatentArgs& x, const LatentSizes& s, hipStream_t stream) {
  if (s.latent == 256) return s.head_dim == 64 ? launch<FMT, 256, 64>(x, s, stream) : launch<FMT, 256, 128>(x, s, stream);
  return s.head_dim == 64 ? launch<FMT, 512, 64>(x, s, stream) : launch<FMT, 512, 128>(x, s, stream);
}

}  // namespace

size_t expanded_workspace_bytes(const LatentSizes& s, bool ragged) {
  return expanded_space(s, expanded_plan(s, ragged)).end;
}

// (heads are shared out over more workgroups of latent_expand_kernel only where there are fewer than 512)
bool expanded_fits(const LatentSizes& s, bool ragged) {
  const ExpandedPlan p = expanded_plan(s, ragged);
  return p.tiles * p.splits * p.heads <= kMaxGroups && expand_groups(s) <= kMaxGroups && s.m <= kMaxGroups;
}

hipError_t launch_expanded(const LatentArgs& x, const LatentSizes& s, hipStream_t stream) {
  switch (s.fmt) {
    case MEM_KV_BF16: return launch_fmt<MEM_KV_BF16>(x, s, stream);
    case MEM_KV_FP8: return launch_fmt<MEM_KV_FP8>(x, s, stream);
    default: return launch_fmt<MEM_KV_FP4>(x, s, stream);
  }
}

}  // namespace memattn
