// Latent attention, expanded form: keys and values of the context are made of the
// latent vectors first, in the workspace, for as many heads at a time as fit it.
//
//   latent_units_kernel     where each request's units of 32 tokens lie
//   latent_expand_kernel    keys [W_h c, r] and values V_h c of all units, bf16
//   expanded_attend_kernel  attention over them, head by head
//   attend_join_kernel      joins the parts of split contexts
//
// Row 32 u + j of a head's keys and values is token j of the request's unit u.
#include <algorithm>

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
  if (threadIdx.x == 0) counts[req] = n;
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

// 16 bytes of a row's elements 8 i .. 8 i + 7 as bf16.
template <int FMT, int L>
__device__ __forceinline__ u32x4_t latent_chunk(const uint8_t* codes, const uint8_t* scales, int i) {
  if constexpr (FMT == MEM_KV_BF16) {
    return *reinterpret_cast<const u32x4_t*>(codes + 16 * i);
  } else {
    const float s = kv_scale(scales[i / 4]);
    u32x4_t o;
    if constexpr (FMT == MEM_KV_FP4) {
      const uint32_t c = *reinterpret_cast<const uint32_t*>(codes + 4 * i);
      o[0] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
      o[1] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
      o[2] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
      o[3] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
    } else {
      const u32x2_t c = *reinterpret_cast<const u32x2_t*>(codes + 8 * i);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        o[2 * j] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[j], s, false));
        o[2 * j + 1] = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[j], s, true));
      }
    }
    return o;
  }
}

// Workgroup (four units of a request, a share of the heads): the tokens' latent vectors stay in LDS as bf16; for each
// head a wave makes a quarter of its keys' and values' elements for all 128 tokens, its rows of W and V straight from
// memory.  The order of a product's k is free as long as both operands have it: lane (row, half) takes 64 consecutive
// bytes of each 128 of its row.
template <int FMT, int L, int D>
__global__ __launch_bounds__(kThreads, 1) void latent_expand_kernel(LatentArgs x, int64_t units,
                                                                 const Source* __restrict__ sources,
                                                                 const int* __restrict__ counts, int h0, int heads,
                                                                 int per, uint16_t* __restrict__ keys,
                                                                 uint16_t* __restrict__ values) {
  constexpr int kRow = kv_row_bytes(FMT, L), kSc = kv_scale_bytes(FMT, L), kPitch = kPitchOf<L>;
  constexpr int kKeyRow = D + kRopeDim, kMine = 2 * D / kWaves, kBlocks = kMine / 32;  // rows of W and V of a wave
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
  for (int i = tid; i < kGroupTokens * (L / 8); i += kThreads) {
    const int t = i / (L / 8), c = i % (L / 8), u = u0 + t / kUnit;
    u32x4_t v = {0, 0, 0, 0};
    if (u < n) {
      const Source s = sources[req * units + u];
      if (s.at >= 0 && t % kUnit < s.held) {
        const int row = s.row + t % kUnit;
        const uint8_t* page = a.kv.pool + (s.at - static_cast<int64_t>(s.row) * kRow);
        v = latent_chunk<FMT, L>(page + static_cast<int64_t>(row) * kRow,
                                 page + T * (kRow + 2 * kRopeDim) + static_cast<int64_t>(row) * kSc, c);
      }
    }
    *reinterpret_cast<u32x4_t*>(rows + t * kPitch + 8 * (c ^ exchange(t))) = v;
  }
  for (int i = tid; i < kGroupTokens * 8; i += kThreads) {
    const int t = i / 8, c = i % 8, u = u0 + t / kUnit;
    if (u >= n) break;
    const Source s = sources[req * units + u];
    if (s.at < 0 || t % kUnit >= s.held) continue;
    const int row = s.row + t % kUnit;
    const u32x4_t v = *reinterpret_cast<const u32x4_t*>(a.kv.pool + (s.at - static_cast<int64_t>(s.row) * kRow) +
                                                        T * kRow + static_cast<int64_t>(row) * 2 * kRopeDim + 16 * c);
    for (int h = hb; h < he; ++h)
      *reinterpret_cast<u32x4_t*>(keys + (h * slots + slot0 + t) * kKeyRow + D + 8 * c) = v;
  }
  __syncthreads();

  const int f = exchange(col);
  for (int h = hb; h < he; ++h) {
    const uint16_t* w = x.w + (h0 + h) * x.w_hs + (wave * kMine + col) * x.w_rs + 32 * half;
    f32x16 o[kBlocks][kGroupUnits];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int u = 0; u < kGroupUnits; ++u)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[b][u][j] = 0.f;
    u32x4_t next[kBlocks][4];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int y = 0; y < 4; ++y) next[b][y] = *reinterpret_cast<const u32x4_t*>(w + 32 * b * x.w_rs + 8 * y);
#pragma unroll 2
    for (int s = 0; s < L / 64; ++s) {
      u32x4_t cur[kBlocks][4];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          cur[b][y] = next[b][y];
          if (s + 1 < L / 64)
            next[b][y] = *reinterpret_cast<const u32x4_t*>(w + 32 * b * x.w_rs + 64 * (s + 1) + 8 * y);
        }
#pragma unroll
      for (int y = 0; y < 4; ++y) {
#pragma unroll
        for (int u = 0; u < kGroupUnits; ++u) {
          const bf16x8 k = as_bf16x8(*reinterpret_cast<const u32x4_t*>(
              rows + (32 * u + col) * kPitch + 64 * s + 32 * half + 8 * (y ^ f)));
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
            o[b][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(cur[b][y]), k, o[b][u], 0, 0, 0);
        }
      }
    }
    const bool is_v = wave * kMine >= D;
    uint16_t* dst = is_v ? values + (h * slots + slot0 + col) * D + wave * kMine - D
                         : keys + (h * slots + slot0 + col) * kKeyRow + wave * kMine;
    const int pitch = is_v ? D : kKeyRow;
#pragma unroll
    for (int u = 0; u < kGroupUnits; ++u) {
      if (u0 + u >= n) break;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          *reinterpret_cast<u32x2_t*>(dst + 32 * u * pitch + 32 * b + 8 * y + 4 * half) =
              u32x2_t{pack2(o[b][u][4 * y], o[b][u][4 * y + 1]), pack2(o[b][u][4 * y + 2], o[b][u][4 * y + 3])};
    }
  }
}

// ---------------------------------------------------------------- attention

template <int D>
struct ExpandedShape {
  static constexpr int kKey = D + kRopeDim;
  static constexpr int kBatch = 128;         // units resolved at a time
  static constexpr int kKeyPitch = kKey + 32, kValuePitch = D + 32;
};

// Tiles of 32 WAVES rows (new tokens) of a head.  Units go through a ring of three in LDS: while the waves make the
// scores of unit i, they unpack unit i + 1 and load unit i + 2; the second product of unit i - 1 is written in groups of
// one matrix instruction and a share of unit i's exponentials (a wave issues in order, so that only what stands between
// its matrix products overlaps with them).
template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void expanded_attend_kernel(
    LatentArgs x, int splits, int64_t tiles, int64_t units, int h0, int heads, const uint16_t* __restrict__ key_rows,
    const uint16_t* __restrict__ value_rows, float* __restrict__ part_o, RowState* __restrict__ part_ml) {
  using S = ExpandedShape<D>;
  constexpr int kThreadsHere = 64 * WAVES, kR = 32 * WAVES;
  constexpr int kSteps = S::kKey / 16, kBlocks = D / 32, kOps = 2 * kBlocks;
  constexpr int kKeyChunks = S::kKey / 8, kValueChunks = D / 8;              // 16-byte chunks of a row
  constexpr int kKeyLoads = kUnit * kKeyChunks / kThreadsHere, kValueLoads = kUnit * kValueChunks / kThreadsHere;
  constexpr int kPieces = kKeyLoads + kValueLoads;
  static_assert(kUnit * kKeyChunks % kThreadsHere == 0 && kUnit * kValueChunks % kThreadsHere == 0, "whole loads");
  extern __shared__ int dyn[];  // of the chunk list: ub[k + 1], tb[k + 1]
  __shared__ __align__(16) uint16_t keys[3][kUnit * S::kKeyPitch];
  __shared__ __align__(16) uint16_t values[3][kUnit * S::kValuePitch];
  __shared__ Unit list[S::kBatch];
  __shared__ int tmp[2 * WAVES];
  __shared__ uint32_t bad_tok[3];  // tokens of a masked unit whose values are not finite: at hand, next, cleared

  const AttendArgs& a = x.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const uint32_t b = blockIdx.x / static_cast<uint32_t>(heads), tile = b / static_cast<uint32_t>(splits);
  const int g = static_cast<int>(blockIdx.x - b * heads), split = static_cast<int>(b - tile * splits);
  Tile t;
  if (!find_tile<kR>(a, static_cast<uint32_t>(tiles) - 1 - tile, 1, &t)) return;  // the latest rows see most: first
  const ChunkList list_of = scan_list<kThreadsHere, false>(a, t.req, dyn, tmp);
  const int ctx = list_of.tb[a.k];
  const int prefix = a.prefix_len ? __builtin_amdgcn_readfirstlane(min(max(a.prefix_len[t.req], 0), kFar)) : 0;
  const int my_row = t.r0 + min(32 * wave + col, t.rows - 1);
  const RowRule rule = row_rule(a, t, ctx, g, 1, my_row);
  const TileRule tr = tile_rule<kR>(a, t, ctx, g, 1);
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
  const float c = a.scale * kLog2e;
  const int64_t slots = a.m * units * kUnit;
  const uint16_t* my_keys = key_rows + (g * slots + t.req * units * kUnit) * S::kKey;
  const uint16_t* my_values = value_rows + (g * slots + t.req * units * kUnit) * D;
  Rows<32, D> rows;
  rows.clear();
  RowState st{-INFINITY, 0.f};
  float rounded = 0.f;  // sum of the weights as the second product takes them
  bool poison = false;

  const int f = exchange(col);
  const int even = col * S::kKeyPitch + 8 * (half ^ f), odd = col * S::kKeyPitch + 8 * ((2 + half) ^ f);
  int value_at;
  {
    const int i = lane & 15, r = 4 * half + (i >> 2), cc = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    value_at = r * S::kValuePitch + 8 * (cc ^ exchange(r)) + 4 * (i & 1);
  }
  // a thread's 16-byte pieces of a unit: of the key rows, then of the value rows
  u32x4_t p[kPieces];
  int row_of[kPieces], place_of[kPieces];  // the piece's token, and where it goes in LDS
#pragma unroll
  for (int z = 0; z < kPieces; ++z) {
    const bool is_v = z >= kKeyLoads;
    const int at = tid + (is_v ? z - kKeyLoads : z) * kThreadsHere, chunks = is_v ? kValueChunks : kKeyChunks;
    row_of[z] = at / chunks;
    place_of[z] = row_of[z] * (is_v ? S::kValuePitch : S::kKeyPitch) + 8 * ((at % chunks) ^ exchange(row_of[z]));
  }

  for (int last = u1 - 1; last >= u0; last -= S::kBatch) {
    __syncthreads();
    const int n = resolve_units<S::kBatch, kThreadsHere, true>(a, list_of, span, tr, prefix, 0, 0, last,
                                                             min(S::kBatch, last - u0 + 1), list, tmp);
    if (n == 0) continue;
    if (tid < 2) bad_tok[tid] = 0;
    __syncthreads();
    auto load = [&](const Unit& u, int z) {  // (what lies behind the last held token is cleared before it is used)
      p[z] = z < kKeyLoads
                 ? *reinterpret_cast<const u32x4_t*>(my_keys + u.at * (kUnit * S::kKey) + 8 * (tid + z * kThreadsHere))
                 : *reinterpret_cast<const u32x4_t*>(my_values + u.at * (kUnit * D) +
                                                     8 * (tid + (z - kKeyLoads) * kThreadsHere));
    };
    // tokens that a masked unit does not hold are cleared, values that are not finite are noted and left out
    auto check = [&](const Unit& u, int to) {
#pragma unroll
      for (int z = 0; z < kPieces; ++z) {
        if (row_of[z] >= u.held()) p[z] = u32x4_t{0, 0, 0, 0};
        if (z < kKeyLoads) continue;
        u16x2 most = {0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, p[z][j] & 0x7FFF7FFFu));
        if (most[0] >= 0x7F80u || most[1] >= 0x7F80u) {
          atomicOr(&bad_tok[to], 1u << row_of[z]);
          p[z] = u32x4_t{0, 0, 0, 0};
        }
      }
    };
    // Piece z of the next unit, and the load of the same piece of the one after it.
    auto advance = [&](int to, const Unit& from, int z) {
      *reinterpret_cast<u32x4_t*>((z < kKeyLoads ? keys[to] : values[to]) + place_of[z]) = p[z];
      load(from, z);
    };
    Unit u = uniform_unit(list[0]), next = uniform_unit(list[min(1, n - 1)]);
#pragma unroll
    for (int z = 0; z < kPieces; ++z) load(u, z);
    if (u.masked()) check(u, 0);
#pragma unroll
    for (int z = 0; z < kPieces; ++z) {
      advance(0, next, z);
      issue_first();
    }
    __syncthreads();
    u32x4_t w[2];  // weights of the unit before
    bool pending = false;
    const uint16_t* value_src = nullptr;
    auto value = [&](int o) {  // operand o: columns 32 (o / 2), tokens 16 (o % 2)
      const uint16_t* src = value_src + 16 * (o & 1) * S::kValuePitch + 32 * (o >> 1);
      const u32x2_t v0 = lds_transpose4(src), v1 = lds_transpose4(src + 8 * S::kValuePitch);
      return as_bf16x8(u32x4_t{v0[0], v0[1], v1[0], v1[1]});
    };
    auto add_values = [&](auto share) {
      constexpr int kAhead = 3;
      bf16x8 v[kOps];
#pragma unroll
      for (int o = 0; o < kAhead; ++o) v[o] = value(o);
      issue_first();
#pragma unroll
      for (int o = 0; o < kOps; ++o) {
        if (o + kAhead < kOps) v[o + kAhead] = value(o + kAhead);
        rows.o[o >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[o], as_bf16x8(w[o & 1]), rows.o[o >> 1], 0, 0, 0);
        share(o);
        issue_first();
      }
    };
    int slot = 0;  // i mod 3: the unit's buffer, and its word of bad_tok
    for (int i = 0; i < n; ++i) {
      const Unit after = uniform_unit(list[min(i + 2, n - 1)]);
      const int slot1 = slot == 2 ? 0 : slot + 1, slot2 = slot == 0 ? 2 : slot - 1;
      if (tid == 0) bad_tok[slot2] = 0;
      if (i + 1 < n && next.masked()) check(next, slot1);
      const uint16_t* kp = keys[slot];
      value_src = values[slot2] + value_at;
      f32x16 s;
#pragma unroll
      for (int j = 0; j < 16; ++j) s[j] = 0.f;
      {
        constexpr int kAhead = 3;
        auto key = [&](int y) {
          return *reinterpret_cast<const u32x4_t*>(kp + (y & 1 ? odd : even) + 32 * (y >> 1));
        };
        u32x4_t k[kSteps];
#pragma unroll
        for (int y = 0; y < kAhead; ++y) k[y] = key(y);
        issue_first();
#pragma unroll
        for (int y = 0; y < kSteps; ++y) {
          if (y + kAhead < kSteps) k[y + kAhead] = key(y + kAhead);
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[y]), q[y], s, 0, 0, 0);
          if (y * kPieces / kSteps != (y + 1) * kPieces / kSteps) advance(slot1, after, y * kPieces / kSteps);
          issue_first();
        }
      }
      if (u.masked()) {
        const uint32_t seen = visible_tokens(rule, u, prefix);
        mask_scores<32, 16>(s, seen, half);
        poison |= (seen & bad_tok[slot]) != 0;
      }
      float top = s[0];
#pragma unroll
      for (int j = 1; j < 16; ++j) top = nan_max(top, s[j]);
      const float high = max_column<32>(top) * c;
      const bool counts = __any(!u.masked() || high != -INFINITY);
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
      // The usual way: both in one.  (Two flags that the compiler does not know to be one: with an if and an else over
      // the same accumulators it keeps them twice.)
      const bool usual = pending && counts && !up;
      int usual_too = __builtin_amdgcn_readfirstlane(usual);
      asm volatile("" : "+s"(usual_too));
      if (!usual) {
        if (pending) add_values([](int) {});
        if (up) {
          const float mn = fmaxf(st.m, high);
          const float r = mn == -INFINITY ? 1.f : fast_exp2(st.m - mn);
          st.l *= r;
          rounded *= r;
          rows.scale(r);
          st.m = mn;
        }
        if (counts) {
          const float ref = finite_max(st.m);
#pragma unroll
          for (int j = 0; j < 16; ++j) weigh_score(ref, j);
        }
      }
      if (usual_too) {
        const float ref = finite_max(st.m);
        add_values([&](int o) {
#pragma unroll
          for (int j = 16 * o / kOps; j < 16 * (o + 1) / kOps; ++j) weigh_score(ref, j);
        });
      }
      pending = counts;
      w[0] = now[0];
      w[1] = now[1];
      u = next;
      next = after;
      slot = slot1;
      __syncthreads();
    }
    if (pending) {
      value_src = values[slot == 0 ? 2 : slot - 1] + value_at;
      add_values([](int) {});
    }
  }

  st.l = sum_column<32>(st.l);
  rounded = sum_column<32>(rounded);
  poison = any_column<32>(poison, col);
  if (32 * wave + col >= t.rows) return;
  write_sums<32, D, D>(a, rows, st, rounded, poison, tok_at * a.hq + h0 + g, half, split, splits, 0, x.out, part_o,
                       part_ml);
}

// ---------------------------------------------------------------- launches

size_t align256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }
size_t list_bytes(int k) { return (2 * static_cast<size_t>(k) + 2) * sizeof(int); }

struct ExpandedPlan {
  int waves;
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
  p.waves = 4;
  const int R = 32 * p.waves;
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
  w.keys = w.counts + align256(s.m * sizeof(int));
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
    expanded_attend_kernel<D, 4><<<static_cast<unsigned>(p.tiles * heads * p.splits), 256, list_bytes(s.k), stream>>>(
        x, p.splits, p.tiles, s.units, h0, heads, keys, values, part_o, part_ml);
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

bool expanded_fits(const LatentSizes& s, bool ragged) {
  const ExpandedPlan p = expanded_plan(s, ragged);
  return p.tiles * p.splits * p.heads <= kMaxGroups && expand_groups(s) <= kMaxGroups / s.heads;
}

hipError_t launch_expanded(const LatentArgs& x, const LatentSizes& s, hipStream_t stream) {
  switch (s.fmt) {
    case MEM_KV_BF16: return launch_fmt<MEM_KV_BF16>(x, s, stream);
    case MEM_KV_FP8: return launch_fmt<MEM_KV_FP8>(x, s, stream);
    default: return launch_fmt<MEM_KV_FP4>(x, s, stream);
  }
}

}  // namespace memattn
