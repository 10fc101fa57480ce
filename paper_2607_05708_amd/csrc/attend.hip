// Attention over the paged key/value cache.
//
// For each request and key/value head the rows are (new token, query head of
// the group); they share the head's keys and values, which are read once per
// tile of rows.  The context is walked in units of 32 tokens of one page, so
// every unit is one page lookup and ends inside a tile only at the end of a
// chunk.  A workgroup first turns its request's chunk list into units (a scan
// of the chunk lengths, then one lookup per unit; units that no row can see
// are left out), then streams them from the last to the first: where the
// nearest tokens weigh most the running maximum of the softmax (log2 domain)
// is found early.  Keys and values are read once.  Long contexts with few
// rows are split over workgroups, whose partial results a second kernel joins
// in a fixed order.
//
// Both kernels compute S^T = K Q^T and O^T = V^T P^T: the products' columns
// are the rows, so the softmax of a row stays in the lanes that hold its
// column, and the weights leave the first product in the layout in which the
// second one reads them: P never moves between lanes.
//
//   attend_few_kernel   tiles of 16 rows (16x16x32 products) or 32 rows
//     (32x32x16): each wave streams its own units with no barrier.  A lane
//     loads quarters of a token's row (16 bytes of 4-bit codes of 128
//     elements: exactly one block, so one scale) straight from the page into
//     the operand of the first product; values go through the wave's own LDS
//     rows once, as bf16, to be read back transposed.  Bound by HBM where the
//     contexts are long (128 x 32,768 tokens in 4 bits 782 us, 5.8 TB/s; a plain
//     copy reaches 5.1), by the start of a workgroup -- four dependent loads and
//     the lookups, some 6 us -- where they are short (2,560 tokens 13 us).
//   attend_tile_kernel  tiles of 128 rows: the workgroup unpacks two units at
//     a time into LDS for its four waves, into one half of a double buffer
//     while they work on the other; a wave's matrix products are interleaved
//     with the exponentials and the unpacking.  4 x 2,048 tokens over 8,192,
//     capped, 1.13 ms (849 TFLOP/s); 8,192 tokens behind 24,576, with a distance
//     bias, 4.67 ms (824 TFLOP/s); a large library product reaches 1,360.
//     Counters of these two: the vector unit issues in 61 and 53 % of the cycles,
//     the matrix cores are busy in 37 and 33 %, LDS in 40 and 36 % (a quarter of
//     that bank conflicts); the clock is at 2.3 and 2.4 GHz once the passes
//     follow each other for some 40 ms, and 1.8 to 2.1 before.  So it is the
//     vector work between the products, and what does not overlap with it.
//     Registers are short: heads of 64 (three workgroups a CU) spill 19 to 80 of
//     them, bf16 with wider heads 20 to 108 (tiles of 32 rows 10 to 12, and 107
//     at 256), 8 and 4 bits with heads of 256 up to 22, 8 bits with capped scores
//     and heads of 128 up to 10.
#include <type_traits>

#include "context.h"
#include "kv.h"
#include "device_common.h"

namespace memattn {

namespace {

constexpr int kTileRows = 128;  // rows per tile of the tile kernel

// How a call is spread over the GPU (shared by the workspace size and the launch).
struct AttendPlan {
  int rows;       // rows per tile: 16, 32 (few-rows kernel) or 128 (tile kernel)
  int64_t tiles;  // row tiles (upper bound with ragged requests)
  int splits;
};

// ---------------------------------------------------------------- scores and their softmax

// Caps that a kernel is made for: none, up to kModestCap, above.
enum Caps { kNoCap, kModestCaps, kLargeCaps };
constexpr float kModestCap = 64.f;

// How raw products become scores in the log2 domain: scaled, capped, biased.  The cap is softcap * tanh(x), x the
// scaled product over the cap.  By its definition the tanh is 1 - 2 / (1 + e^2x), with two transcendental operations
// of twice to three times a product's cost each, and an error of 2^-21 whatever its size.  Where |x| is at most
// kSmall, tanh(x) / x as a polynomial of degree 2 in t = x^2 does as well: its series 1 - t / 3 + 2 t^2 / 15 - 17 t^3
// / 315 with t^3 replaced by the quadratic that is nearest to it on [0, kSmall^2], off by at most kSmall^6 / 32
// (Chebyshev).  With the series' next term that is 1.1e-7 of the score.  Units without a larger product take it for
// all of them.  In the others a modest cap takes the definition for all (off by at most 2^-15, where the weights are
// rounded by 2^-9 of themselves); of a larger cap that error would be a multiple, so each score goes by its own size,
// and is off by 2^-19 of itself at most.  (The choice for each costs 20 % of a prefill whose scores are of the cap's
// size, and registers: kernels of their own.)
struct Scores {
  float c;     // scale * log2(e)
  float k2;    // 2 * log2(e) * scale / softcap
  float cap2;  // softcap * log2(e); 0: none
  float limit; // raw products up to this magnitude are small
  float s0, s1, s2;  // the polynomial in squared raw products, times scale * log2(e)
  bool bias;
  bool causal;

  static constexpr float kSmall = 0.1875f, kT = kSmall * kSmall, kCubic = 17.f / 315.f;
  static constexpr float kP0 = 1.f - kCubic * kT * kT * kT / 32.f, kP1 = -1.f / 3.f + kCubic * kT * kT * (9.f / 16.f),
                         kP2 = 2.f / 15.f - kCubic * kT * 1.5f;

  __device__ __forceinline__ explicit Scores(const AttendArgs& a)
      : c(a.scale * kLog2e), cap2(a.softcap * kLog2e), bias(a.slopes != nullptr), causal(a.causal != 0) {
    const float x = a.softcap > 0.f ? fminf(a.scale / a.softcap, 1e38f) : 0.f;  // (finite: 0 * x is 0)
    k2 = 2.f * kLog2e * x;
    // (within these ranges no coefficient and no square of a small product leaves the normal numbers)
    const bool plain = x >= 0x1p-20f && x <= 0x1p20f && c >= 0x1p-40f && c <= 0x1p40f;
    limit = plain ? kSmall / x : -1.f;
    s0 = c * kP0;
    s1 = c * x * x * kP1;
    s2 = c * x * x * x * x * kP2;
  }

  __device__ __forceinline__ float series(float s) const {  // capped score / s
    const float t = s * s;
    return s0 + t * (s1 + t * s2);
  }
  __device__ __forceinline__ float fraction(float s) const { return __builtin_amdgcn_rcpf(1.f + fast_exp2(s * k2)); }

  // Capped score of any product by its own size: the polynomial in u^2 = (2 log2(e) x)^2, or the definition.
  __device__ __forceinline__ float capped(float s) const {
    constexpr float kA = 1.f / (4.f * kLog2e * kLog2e);
    const float u = s * k2, t = u * u;
    const float near = s * c * (kP0 + t * (kP1 * kA + t * (kP2 * kA * kA)));
    const float far = cap2 * fmaf(fraction(s), -2.f, 1.f);
    return t <= kT / kA ? near : far;
  }

  // Scores of one unit made explicit: what masks and biases need.
  template <int WIDTH, int N, Caps CAPS, typename V>
  __device__ __forceinline__ void apply(V& s, const RowRule& rule, const TileRule& tr, int pos, int part) const {
    if (CAPS != kNoCap && cap2 != 0.f) {
      if (CAPS == kModestCaps) {
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] = cap2 - 2.f * cap2 * fraction(s[j]);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] = capped(s[j]);
      }
    }
    const float f = cap2 == 0.f ? c : 1.f;
    if (!bias) {
#pragma unroll
      for (int j = 0; j < N; ++j) s[j] *= f;
      return;
    }
    const float dist = static_cast<float>(rule.pos - pos - 4 * part);
    if (causal && pos + kUnit - 1 <= tr.hi_all) {  // every token lies behind every row
      const float near = -rule.slope * dist;
#pragma unroll
      for (int j = 0; j < N; ++j)
        s[j] = fmaf(s[j], f, fmaf(rule.slope, static_cast<float>(score_token<WIDTH>(j)), near));
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        s[j] = s[j] * f - rule.slope * fabsf(dist - static_cast<float>(score_token<WIDTH>(j)));
    }
  }
};

// How a unit's scores become weights 2^(score - ref): from numbers that only want a factor (scores in the log2 domain,
// or raw products without a cap), or from raw products whose cap (by the polynomial, by the definition, or each by its
// size) goes into the exponential's argument.
enum Mode { kLinear, kSeries, kExact, kBySize };

template <Mode MODE>
__device__ __forceinline__ float weigh(float s, float f, const Scores& sc, float ref) {
  if constexpr (MODE == kLinear) return fast_exp2(fmaf(s, f, -ref));
  if constexpr (MODE == kSeries) return fast_exp2(fmaf(s, sc.series(s), -ref));
  if constexpr (MODE == kExact) return fast_exp2(fmaf(sc.fraction(s), -2.f * sc.cap2, sc.cap2 - ref));
  return fast_exp2(sc.capped(s) - ref);
}

// The largest score of a row from the largest number (the cap grows with the product).
__device__ __forceinline__ float top_score(float top, float f, const Scores& sc, Mode mode) {
  if (mode == kLinear) return top * f;
  if (mode == kSeries) return top * sc.series(top);
  return mode == kExact ? sc.cap2 - 2.f * sc.cap2 * sc.fraction(top) : sc.capped(top);
}

// Unpack a quarter row of values into its LDS row.
template <int WIDTH, int SHIFT, int FMT, int D>
__device__ __forceinline__ void store_values(const Piece<FMT, D>& p, uint16_t* v, int row, int quarter) {
  uint16_t* dst = v + row * kValuePitch<WIDTH, D>;
#pragma unroll
  for (int y = 0; y < Dim<FMT, D>::kSteps; ++y)
    *reinterpret_cast<u32x4_t*>(dst + 8 * value_chunk<WIDTH, SHIFT>(row, quarter * Dim<FMT, D>::kSteps + y)) =
        piece_step<FMT, D>(p, y);
}

// ---------------------------------------------------------------- few rows

template <int FMT, int D, int R>
struct FewShape {
  static constexpr int kBatch = 256;                        // units resolved at a time
  static constexpr int kShift = R == 16 ? 3 : 2;            // exchange of chunks: a wave writes 16 rows at a time
  static constexpr int kWaveBytes = kUnit * kValuePitch<R, D> * 2;  // a wave's unpacked values
  static constexpr int kJoinBytes = 2 * R * D * 4;          // two waves' outputs at the end
  static constexpr int kArea = kWaves * kWaveBytes > kJoinBytes ? kWaves * kWaveBytes : kJoinBytes;
};

// CAPS: kModestCaps stands for none too.
template <int FMT, int D, int R, Caps CAPS>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attend_few_kernel(AttendArgs a, int splits,
                                                                                float* __restrict__ part_o,
                                                                                RowState* __restrict__ part_ml) {
  using K = Dim<FMT, D>;
  using S = FewShape<FMT, D, R>;
  constexpr int kParts = 64 / R;              // lanes that share a row's scores
  constexpr int kScores = kUnit / kParts;     // scores per lane and unit
  constexpr int kQSteps = D / (8 * kParts);   // operands of a row's queries per lane
  constexpr Mode kLarge = CAPS == kLargeCaps ? kBySize : kExact;  // for units with large products
  extern __shared__ int dyn[];                // the chunk list: cid[k], ub[k + 1], tb[k + 1]
  __shared__ __align__(16) uint8_t area[S::kArea];
  __shared__ Unit list[S::kBatch];
  __shared__ int tmp[2 * kWaves];
  __shared__ RowState joint[2][64];
  __shared__ int joint_poison[2][64];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane % R, part = lane / R;
  const int heads = a.kv.heads, group = a.hq / heads;
  const uint32_t b = blockIdx.x / static_cast<uint32_t>(heads), tile = b / static_cast<uint32_t>(splits);
  const int g = static_cast<int>(blockIdx.x - b * heads), split = static_cast<int>(b - tile * splits);
  Tile t;
  if (!find_tile<R>(a, tile, group, &t)) return;
  const ChunkList L = scan_list(a, t.req, dyn, tmp);
  const int ctx = L.tb[a.k];
  const int prefix = a.prefix_len ? __builtin_amdgcn_readfirstlane(min(max(a.prefix_len[t.req], 0), kFar)) : 0;
  const int my_row = t.r0 + min(col, t.rows - 1);
  const RowRule rule = row_rule(a, t, ctx, g, group, my_row);
  const TileRule tr = tile_rule<R>(a, t, ctx, g, group);
  const Span span = visible_units(L, prefix, tr.lo, tr.hi);
  const int n_units = __builtin_amdgcn_readfirstlane(span.count());
  const int u0 = static_cast<int>(static_cast<int64_t>(n_units) * split / splits);
  const int u1 = static_cast<int>(static_cast<int64_t>(n_units) * (split + 1) / splits);

  // lane (col, part) holds elements part D / kParts .. of row `col`
  bf16x8 q[kQSteps];
  load_queries(a.q + static_cast<int64_t>(t.q0 + my_row / group) * a.q_ts + (g * group + my_row % group) * a.q_hs + part * (D / kParts), 8, q);

  const Scores scores(a);
  const int64_t T = a.kv.page_tokens;
  const int64_t head_at = static_cast<int64_t>(g) * 2 * T * (K::kRow + K::kSc);
  // piece h of a lane: quarter `part` of row 16 h + col, or quarter 2 part + h of row `col`
  const int row_step = R == 16 ? 16 : 0;
  const int quarter = R == 16 ? part : 2 * part, quarter_step = R == 16 ? 0 : 1;
  uint16_t* vrows = reinterpret_cast<uint16_t*>(area + wave * S::kWaveBytes);

  Rows<R, D> rows;
  rows.clear();
  RowState st{-INFINITY, 0.f};
  bool poison = false;

  // Keys and values of the unit at hand.  Each is loaded again, for the wave's next unit, as soon as it has been used:
  // a wave keeps nearly a whole unit in flight without a second set of registers.
  Piece<FMT, D> pk[2], pv[2];
  const int my_codes = col * K::kRow + quarter * K::kBytes;
  auto load = [&](Piece<FMT, D> (&p)[2], const Unit& u, bool is_v) {
    const uint8_t* codes = a.kv.pool + u.at + (is_v ? T * K::kRow : 0);
    const uint8_t* sc = a.kv.pool + u.at + (2 * T * K::kRow - u.row() * (K::kRow - K::kSc)) + (is_v ? T * K::kSc : 0);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      load_piece<FMT, D>(p[h], codes + (my_codes + h * (row_step * K::kRow + quarter_step * K::kBytes)),
                         sc + ((col + h * row_step) * K::kSc + (quarter + h * quarter_step) * K::kElems / kKvBlock));
  };

  for (int last = u1 - 1; last >= u0; last -= S::kBatch) {
    __syncthreads();
    const int n = resolve_units<S::kBatch>(a, L, span, tr, prefix, head_at, K::kRow, last,
                                             min(S::kBatch, last - u0 + 1), list, tmp);
    if (wave >= n) continue;
    Unit u = uniform_unit(list[wave]);
    load(pk, u, false);
    load(pv, u, true);
    for (int i = wave; i < n; i += kWaves) {
      // (loads are not behind a condition, so that the compiler knows how many are in flight behind the one that it
      // waits for: the last unit is loaded again instead)
      const Unit next = uniform_unit(list[i + kWaves < n ? i + kWaves : i]);
      float s[kScores];
      if constexpr (R == 16) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int y = 0; y < K::kSteps; ++y)
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(piece_step<FMT, D>(pk[h], y)), q[y], x, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < 4; ++j) s[4 * h + j] = x[j];
        }
      } else {
        f32x16 x;
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int y = 0; y < K::kSteps; ++y)
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(piece_step<FMT, D>(pk[h], y)), q[h * K::kSteps + y],
                                                        x, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = x[j];
      }
      load(pk, next, false);
      const bool ready = u.masked() || scores.bias;
      if (ready) scores.template apply<R, kScores, CAPS>(s, rule, tr, u.pos, part);
      if (u.masked()) {
        const int held = u.held();
        const uint32_t seen = visible_tokens(rule, u, prefix);
        mask_scores<R, kScores>(s, seen, part);
        uint32_t bad = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = h * row_step + col;
          const bool nf = row < held && piece_bad<FMT, D>(pv[h]);
          uint64_t vote = __ballot(nf);
          vote |= vote >> 32;
          if (R == 16) vote |= vote >> 16;
          bad |= static_cast<uint32_t>(R == 16 ? vote & 0xFFFFu : vote) << (h * row_step);
          if (nf || row >= held) piece_clear<FMT, D>(pv[h]);
        }
        poison |= (seen & bad) != 0;
      }
      bool small = false;
      if (!ready && scores.cap2 != 0.f) {
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < kScores; ++j) most = fmaxf(most, fabsf(s[j]));
        small = !__any(most > scores.limit);
      }
      const Mode mode = ready || scores.cap2 == 0.f ? kLinear : small ? kSeries : kLarge;
      const float f = ready ? 1.f : scores.c;
      const float top = top_score(max_column<R>(max_of(s)), f, scores, mode);
      const bool counts = raise<R, D>(top, u.masked(), st, rows);
      if (counts) {
        const float ref = finite_max(st.m);
        auto weigh_all = [&](auto m) {
#pragma unroll
          for (int j = 0; j < kScores; ++j) {
            s[j] = weigh<decltype(m)::value>(s[j], f, scores, ref);
            st.l += s[j];
          }
        };
        if (mode == kLinear) weigh_all(std::integral_constant<Mode, kLinear>{});
        else if (mode == kSeries) weigh_all(std::integral_constant<Mode, kSeries>{});
        else weigh_all(std::integral_constant<Mode, kLarge>{});
      }
      if (counts) {  // values: unpack into the wave's LDS rows, to be read back transposed
#pragma unroll
        for (int h = 0; h < 2; ++h)
          store_values<R, S::kShift>(pv[h], vrows, h * row_step + col, quarter + h * quarter_step);
      }
      load(pv, next, true);
      if (counts) {
        __builtin_amdgcn_wave_barrier();
        u32x4_t w[kScores / 8], rest[kScores / 8];
        const bool heavy = is_heavy(top, st);
        const ValueOps<R, D, S::kShift> ops(vrows, lane);
        constexpr int kOps = ValueOps<R, D, S::kShift>::kOps, kTogether = 8;  // operands loaded ahead of their products
#pragma unroll
        for (int n0 = 0; n0 < kOps; n0 += kTogether) {
          bf16x8 v[kTogether];
#pragma unroll
          for (int x = 0; x < kTogether && n0 + x < kOps; ++x) v[x] = ops[n0 + x];
          issue_first();
          if (n0 == 0) {
            pack_weights<kScores>(s, w);
            if (heavy) pack_rests<kScores>(s, w, rest);
          }
#pragma unroll
          for (int x = 0; x < kTogether && n0 + x < kOps; ++x) ops.multiply(rows, n0 + x, v[x], w);
          if (heavy) {
#pragma unroll
            for (int x = 0; x < kTogether && n0 + x < kOps; ++x) ops.multiply(rows, n0 + x, v[x], rest);
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
      u = next;
    }
  }

  // join the waves: 2 and 3 into 0 and 1, then 1 into 0 (a lane holds the same outputs in every wave)
  st.l = sum_column<R>(st.l);
  poison = any_column<R>(poison, col);
  float* store = reinterpret_cast<float*>(area);
#pragma unroll
  for (int from = 2; from >= 1; --from) {
    __syncthreads();  // what `area` held is done with
    if (wave >= from && wave < 2 * from) {
      float* dst = store + (wave - from) * R * D + lane * 4;
      int x = 0;
      rows.each4(part, [&](int, f32x4 v) { *reinterpret_cast<f32x4*>(dst + 256 * x++) = v; });
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
      const float* src = store + wave * R * D + lane * 4;
      constexpr int kQ = Rows<R, D>::kRegs / 4;
#pragma unroll
      for (int n = 0; n < Rows<R, D>::kBlocks; ++n)
#pragma unroll
        for (int y = 0; y < kQ; ++y) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(src + 256 * (n * kQ + y));
#pragma unroll
          for (int j = 0; j < 4; ++j) rows.o[n][4 * y + j] = rows.o[n][4 * y + j] * f0 + v[j] * f1;
        }
    }
  }
  if (wave > 0 || col >= t.rows) return;
  const int row = t.r0 + col;
  write_rows<R, D>(a, rows, st, poison, static_cast<int64_t>(t.q0 + row / group) * a.hq + g * group + row % group, part,
                   split, splits,
                   part_o, part_ml);
}

// ---------------------------------------------------------------- tiles of rows

template <int FMT, int D>
struct TileShape {
  static constexpr int kBatch = 128;                        // units resolved at a time
  static constexpr int kTokens = 2 * kUnit;                 // tokens of a step
  static constexpr int kKeyPitch = D + 8;                   // bf16 elements between LDS rows of keys
  static constexpr int kKeys = kTokens * kKeyPitch;         // elements of a step's keys
  static constexpr int kValues = kTokens * kValuePitch<32, D>;
  static constexpr int kShift = 0;                          // exchange of chunks: a wave writes 4 rows at a time
  static_assert(kThreads == 4 * kTokens, "a quarter row of keys and one of values per thread");
};

// A wave issues in order, so its matrix products only overlap with what stands between them: the second product of a
// step's first unit is written in groups of one matrix instruction and a share of the second unit's exponentials, the
// second unit's with a share of the unpacking.  (Two units a step: of one unit's 1.59 us, 0.65 went into the step
// itself -- barrier, list, maximum -- whatever it did.)  A kernel has one way to weigh
// scores in those groups, and takes the rare others apart from them.
template <int FMT, int D, Caps CAPS>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : D == 128 ? 2 : 3) void attend_tile_kernel(AttendArgs a, int splits,
                                                                                 int64_t tiles,
                                                                                 float* __restrict__ part_o,
                                                                                 RowState* __restrict__ part_ml) {
  using K = Dim<FMT, D>;
  using S = TileShape<FMT, D>;
  using Ops = ValueOps<32, D, S::kShift>;
  constexpr int kQSteps = D / 16;
  constexpr bool kCapped = CAPS != kNoCap;
  constexpr Mode kLarge = CAPS == kLargeCaps ? kBySize : kExact;  // for units with large products
  extern __shared__ int dyn[];  // the chunk list: cid[k], ub[k + 1], tb[k + 1]
  __shared__ __align__(16) uint16_t key_rows[2][S::kKeys];
  __shared__ __align__(16) uint16_t value_rows[2][S::kValues];
  __shared__ Unit list[S::kBatch + 6];  // (read some steps ahead)
  __shared__ int tmp[2 * kWaves];
  // Tokens of a masked step's units whose values are not finite: of the step at hand, of the next, and of the one
  // after that, which is cleared (so that a barrier stands between clearing and noting, and between noting and reading).
  __shared__ uint32_t bad_tok[3][2];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int heads = a.kv.heads, group = a.hq / heads;
  const uint32_t b = blockIdx.x / static_cast<uint32_t>(heads), tile = b / static_cast<uint32_t>(splits);
  const int g = static_cast<int>(blockIdx.x - b * heads), split = static_cast<int>(b - tile * splits);
  Tile t;
  if (!find_tile<kTileRows>(a, static_cast<uint32_t>(tiles) - 1 - tile, group, &t)) return;  // the latest rows see most: first
  const ChunkList L = scan_list(a, t.req, dyn, tmp);
  const int ctx = L.tb[a.k];
  const int prefix = a.prefix_len ? __builtin_amdgcn_readfirstlane(min(max(a.prefix_len[t.req], 0), kFar)) : 0;
  const int my_row = t.r0 + min(32 * wave + col, t.rows - 1);
  const bool works = 32 * wave < t.rows;  // this wave has rows
  const RowRule rule = row_rule(a, t, ctx, g, group, my_row);
  const TileRule tr = tile_rule<kTileRows>(a, t, ctx, g, group);
  const Span span = visible_units(L, prefix, tr.lo, tr.hi);
  const int n_units = __builtin_amdgcn_readfirstlane(span.count());
  const int u0 = static_cast<int>(static_cast<int64_t>(n_units) * split / splits);
  const int u1 = static_cast<int>(static_cast<int64_t>(n_units) * (split + 1) / splits);

  // lane (col, half) holds elements 16 s + 8 half .. + 7 of row `col` of the wave
  bf16x8 q[kQSteps];
  load_queries(a.q + static_cast<int64_t>(t.q0 + my_row / group) * a.q_ts + (g * group + my_row % group) * a.q_hs + 8 * half, 16, q);

  const Scores scores(a);
  const int64_t T = a.kv.page_tokens;
  const int64_t head_at = static_cast<int64_t>(g) * 2 * T * (K::kRow + K::kSc);

  Rows<32, D> rows;
  rows.clear();
  RowState st{-INFINITY, 0.f};
  bool poison = false;

  // the quarter row that this thread unpacks, keys and values, of every step (a wave's are of one unit)
  const int tok = tid >> 2, quarter = tid & 3, my_unit = wave >> 1;
  const uint32_t my_codes = tok % kUnit * K::kRow + quarter * K::kBytes;
  const uint32_t my_scale = tok % kUnit * K::kSc + quarter * K::kElems / kKvBlock;
  Piece<FMT, D> pk, pv;

  for (int last = u1 - 1; last >= u0; last -= S::kBatch) {
    __syncthreads();
    const int n = resolve_units<S::kBatch>(a, L, span, tr, prefix, head_at, K::kRow, last,
                                           min(S::kBatch, last - u0 + 1), list, tmp);
    if (n == 0) continue;
    if (tid == 0) list[n] = Unit{0, Unit::kMasked, 0, -1};  // fills up the last step: holds nothing
    if (tid < 4) bad_tok[tid >> 1][tid & 1] = 0;
    __syncthreads();
    const int steps = (n + 1) / 2;
    auto load = [&](const Unit& u) {
      if (tok % kUnit < u.held()) {
        const uint8_t* codes = a.kv.pool + u.at;
        const uint8_t* sc = codes + (2 * T * K::kRow - u.row() * (K::kRow - K::kSc));
        load_piece<FMT, D>(pk, codes + my_codes, sc + my_scale);
        load_piece<FMT, D>(pv, codes + T * K::kRow + my_codes, sc + T * K::kSc + my_scale);
      } else {
        piece_clear<FMT, D>(pk);
        piece_clear<FMT, D>(pv);
      }
    };
    // part y of unpacking into the buffers of step i: keys first, then values
    auto unpack = [&](int i, int y) {
      if (y < K::kSteps) {
        *reinterpret_cast<u32x4_t*>(key_rows[i & 1] + tok * S::kKeyPitch + quarter * K::kElems + 8 * y) =
            piece_step<FMT, D>(pk, y);
      } else {
        y -= K::kSteps;
        *reinterpret_cast<u32x4_t*>(value_rows[i & 1] + tok * kValuePitch<32, D> +
                                    8 * value_chunk<32, S::kShift>(tok, quarter * K::kSteps + y)) =
            piece_step<FMT, D>(pv, y);
      }
    };
    // values of a masked step that are not finite are noted and left out
    auto check_bad = [&](int to) {
      if (piece_bad<FMT, D>(pv)) {
        atomicOr(&bad_tok[to][my_unit], 1u << (tok % kUnit));
        piece_clear<FMT, D>(pv);
      }
    };

    // the first step's rows, and the loads of the second
    Unit ua = uniform_unit(list[0]), ub = uniform_unit(list[1]);  // units of the step at hand
    load(my_unit ? ub : ua);
    if (ua.masked() || ub.masked()) check_bad(0);
#pragma unroll
    for (int y = 0; y < 2 * K::kSteps; ++y) unpack(0, y);
    Unit na = uniform_unit(list[2]), nb = uniform_unit(list[3]);  // of the next
    if (n == 3) nb = uniform_unit(list[n]);
    if (steps > 1) load(my_unit ? nb : na);
    __syncthreads();

    const int key_at = col * S::kKeyPitch + 8 * half;
    int slot = 0;  // i mod 3
    for (int i = 0; i < steps; ++i) {
      // lists are read two steps ahead, for the end of this one
      const int at2 = 2 * i + 4;
      const Unit next_a = list[min(at2, n)], next_b = list[min(at2 + 1, n)];
      const bool more = i + 1 < steps;
      const bool next_masked = more && (na.masked() || nb.masked());
      const int slot1 = slot == 2 ? 0 : slot + 1;
      if (tid < 2) bad_tok[slot == 0 ? 2 : slot - 1][tid] = 0;
      if (works) {
        const uint16_t* keys = key_rows[i & 1] + key_at;
        const uint16_t* values = value_rows[i & 1];
        const bool masked = ua.masked() || ub.masked(), ready = masked || scores.bias;
        // S^T of both units; operands are read kAhead products ahead.  (The other parts of a step have priority over
        // the other workgroup's wave: it is then at its matrix products while this one is at its exponentials.)
        f32x16 s[2];
        float top = -INFINITY, most = 0.f;  // largest product or score, largest magnitude of a product
        {
          constexpr int kAhead = 2, kAll = 2 * kQSteps;
          auto key = [&](int y) {
            return *reinterpret_cast<const u32x4_t*>(keys + y / kQSteps * kUnit * S::kKeyPitch + 16 * (y % kQSteps));
          };
          u32x4_t k[kAll];
#pragma unroll
          for (int y = 0; y < kAhead; ++y) k[y] = key(y);
#pragma unroll
          for (int j = 0; j < 16; ++j) s[0][j] = s[1][j] = 0.f;
          __builtin_amdgcn_s_setprio(0);
          issue_first();
#pragma unroll
          for (int y = 0; y < kAll; ++y) {
            if (y + kAhead < kAll) k[y + kAhead] = key(y + kAhead);
            f32x16& acc = s[y / kQSteps];
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[y]), q[y % kQSteps], acc, 0, 0, 0);
            issue_first();
          }
          __builtin_amdgcn_s_setprio(1);
        }
        if (ready) {
          scores.template apply<32, 16, CAPS>(s[0], rule, tr, ua.pos, half);
          scores.template apply<32, 16, CAPS>(s[1], rule, tr, ub.pos, half);
          if (masked) {
            const uint32_t seen_a = visible_tokens(rule, ua, prefix), seen_b = visible_tokens(rule, ub, prefix);
            mask_scores<32, 16>(s[0], seen_a, half);
            mask_scores<32, 16>(s[1], seen_b, half);
            poison |= ((seen_a & bad_tok[slot][0]) | (seen_b & bad_tok[slot][1])) != 0;
          }
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          top = nan_max(top, s[j >> 4][j & 15]);
          if (kCapped) most = fmaxf(most, fabsf(s[j >> 4][j & 15]));
        }
        const Mode mode = !kCapped || ready ? kLinear : __any(most > scores.limit) ? kLarge : kSeries;
        const float f = ready ? 1.f : scores.c;
        const float high = top_score(max_column<32>(top), f, scores, mode);
        const bool counts = raise<32, D>(high, masked, st, rows);
        const float ref = finite_max(st.m);
        auto weigh_score = [&](auto m, int j) {  // score j of both units' 32
          const float x = weigh<decltype(m)::value>(s[j >> 4][j & 15], f, scores, ref);
          s[j >> 4][j & 15] = x;
          st.l += x;
        };
        // O^T += V^T P^T of one unit, a product at a time, each with its share of other work
        auto add_values = [&](int unit, const u32x4_t (&w)[2], auto share) {
          const Ops ops(values + unit * kUnit * kValuePitch<32, D>, lane);
          constexpr int kAhead = 2;
          bf16x8 v[Ops::kOps];
#pragma unroll
          for (int x = 0; x < kAhead; ++x) v[x] = ops[x];
          issue_first();
#pragma unroll
          for (int x = 0; x < Ops::kOps; ++x) {
            if (x + kAhead < Ops::kOps) v[x + kAhead] = ops[x + kAhead];
            ops.multiply(rows, x, v[x], w);
            share(x);
            issue_first();
          }
        };
        // The usual way is the second block; the first is for steps that weigh nothing and for those with a heavy
        // weight or, where scores are capped, with a mask, a bias or a large score.  (Two flags that the compiler does
        // not know to be one: with an if and an else over the same accumulators it keeps them twice.)
        if (next_masked) check_bad(slot1);
        constexpr Mode kUsual = kCapped ? kSeries : kLinear;
        const bool usual = counts && mode == kUsual && !is_heavy(high, st);
        int usual_too = __builtin_amdgcn_readfirstlane(usual);
        asm volatile("" : "+s"(usual_too));
        if (!usual) {
          if (counts) {
            if (mode == kLinear) {
#pragma unroll
              for (int j = 0; j < 32; ++j) weigh_score(std::integral_constant<Mode, kLinear>{}, j);
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j) weigh_score(std::integral_constant<Mode, kLarge>{}, j);
            }
            u32x4_t w[2], rest[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              pack_weights<16>(s[h], w);
              pack_rests<16>(s[h], w, rest);
              add_values(h, w, [](int) {});
              add_values(h, rest, [](int) {});
            }
          }
#pragma unroll
          for (int y = 0; y < 2 * K::kSteps; ++y) unpack(i + 1, y);
        }
        if (usual_too) {
          const std::integral_constant<Mode, kUsual> m;
          u32x4_t w[2][2];
#pragma unroll
          for (int j = 0; j < 16; ++j) weigh_score(m, j);
          pack_weights<16>(s[0], w[0]);
          add_values(0, w[0], [&](int x) {
            constexpr int kPer = 16 / Ops::kOps;
#pragma unroll
            for (int j = kPer * x; j < kPer * (x + 1); ++j) {
              weigh_score(m, 16 + j);
              if (j & 1) w[1][j >> 3][(j >> 1) & 3] = pack2(s[1][j - 1], s[1][j]);
            }
          });
          add_values(1, w[1], [&](int x) { unpack(i + 1, x); });
        }
      } else {
        if (next_masked) check_bad(slot1);
#pragma unroll
        for (int y = 0; y < 2 * K::kSteps; ++y) unpack(i + 1, y);
      }
      slot = slot1;
      ua = na;
      ub = nb;
      na = uniform_unit(next_a);
      nb = uniform_unit(next_b);
      if (i + 2 < steps) load(my_unit ? nb : na);
      __syncthreads();
    }
  }

  st.l = sum_column<32>(st.l);
  poison = any_column<32>(poison, col);
  if (32 * wave + col >= t.rows) return;
  write_rows<32, D>(a, rows, st, poison,
                    static_cast<int64_t>(t.q0 + my_row / group) * a.hq + g * group + my_row % group, half, split,
                    splits, part_o, part_ml);
}

// ---------------------------------------------------------------- launches

int64_t tile_count(bool ragged, int64_t m, int64_t total_q, int group, int R) {
  if (ragged) return total_q * group / R + m;
  return m * ((total_q / m * group + R - 1) / R);
}

// Workgroups that run together on the 256 CUs, by the registers of the 4-bit kernels.  Others differ: with 16 rows
// heads of 64 in 4 and 8 bits run four a CU, heads of 128 in 8 bits and bf16 two; with 32 rows heads of 64 in 4 and 8
// bits three, in bf16 two; tiles of 128 rows of heads of 128 one where the list has some 235 entries or more (LDS).
// Plans for these are right, but their rounds are not those that are counted here.
int64_t slots_of(int rows, int d) {
  const int per_cu = d == 256 ? 1 : d == 64 ? 3 : rows == 16 ? 3 : 2;
  return int64_t{256} * per_cu;
}

// Rows per request (on average, so that a call of prompts and single tokens has one height for both) decide the
// kernel.  4-bit keys, heads of 128, 8 heads, 4,096 tokens a request, us: 128 requests of 8 rows over 1,024 tokens in
// tiles of 16 rows 39, of 32 rows 52; 32 requests of 48 rows in tiles of 32 rows 82, of 128 102; of 64 rows 112 and
// 107, of 96 rows 132 and 148, of 128 rows 185 and 152.  The context is split so that the rounds of workgroups take
// least, a workgroup being taken to cost its units and kStart more: finding its units, its start and its end.  Tiles
// of 128 rows that fill the GPU are left whole: causal ones are of unequal length, and even out by themselves.
constexpr int64_t kStart = 16;

// Bytes of LDS that a workgroup's chunk list takes.
size_t list_bytes(int k) { return (3 * static_cast<size_t>(k) + 2) * sizeof(int); }

// Tiles of 128 rows of heads of 256 leave 18 KB of a CU's 160 KB for the chunk list: calls with longer lists (more than
// 1,535 chunks a request) take the tiles of 32 rows, whose values leave 77 KB (the longest list takes 48).
bool list_fits_tiles(int d, int k) { return d < 256 || list_bytes(k) <= 18 * 1024; }
static_assert(2 * sizeof(uint16_t) * (TileShape<MEM_KV_BF16, 256>::kKeys + TileShape<MEM_KV_BF16, 256>::kValues) +
                      (TileShape<MEM_KV_BF16, 256>::kBatch + 6) * sizeof(Unit) + 128 + 18 * 1024 <=
                  160 * 1024,
              "a workgroup's LDS");

AttendPlan make_plan(int d, int64_t m, int k, int64_t units, int64_t total_q, int heads, int heads_q, bool ragged) {
  AttendPlan p;
  const int group = heads_q / heads;
  p.rows = total_q * group <= 16 * m ? 16 : total_q * group <= 64 * m || !list_fits_tiles(d, k) ? 32 : kTileRows;
  p.tiles = tile_count(ragged, m, total_q, group, p.rows);
  const int64_t filled = ragged ? (total_q * group + p.rows - 1) / p.rows + m / 2 : p.tiles;  // about
  const int64_t work = filled * heads, slots = slots_of(p.rows, d);
  int64_t best = INT64_MAX;
  p.splits = 1;
  const int64_t most = p.rows == kTileRows && work >= slots ? 1 : kMaxSplits;
  for (int64_t s = 1; s <= most && (s == 1 || units / s >= kWaves); ++s) {
    if (s > 1 && (p.tiles * heads * s > kMaxGroups || join_groups(total_q * heads_q, s) > kMaxGroups)) break;
    const int64_t cost = (work * s + slots - 1) / slots * ((units + s - 1) / s + kStart) + (s > 1 ? s / 4 : 0);
    if (cost < best) {
      best = cost;
      p.splits = static_cast<int>(s);
    }
  }
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
  const size_t lds = list_bytes(a.k);
  const bool large = a.softcap > kModestCap;
  if (p.rows == 16)
    (large ? attend_few_kernel<FMT, D, 16, kLargeCaps> : attend_few_kernel<FMT, D, 16, kModestCaps>)<<<grid, kThreads,
                                                                                                     lds, stream>>>(
        a, p.splits, po, pml);
  else if (p.rows == 32)
    (large ? attend_few_kernel<FMT, D, 32, kLargeCaps> : attend_few_kernel<FMT, D, 32, kModestCaps>)<<<grid, kThreads,
                                                                                                     lds, stream>>>(
        a, p.splits, po, pml);
  else
    (a.softcap == 0.f ? attend_tile_kernel<FMT, D, kNoCap>
     : large          ? attend_tile_kernel<FMT, D, kLargeCaps>
                      : attend_tile_kernel<FMT, D, kModestCaps>)<<<grid, kThreads, lds, stream>>>(
        a, p.splits, p.tiles, po, pml);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || p.splits == 1) return e;
  const dim3 join(static_cast<unsigned>(join_groups(a.total_q * a.hq, p.splits)));
  if (p.splits <= kJoinSplits)
    attend_join_kernel<D, 1><<<join, kThreads, 0, stream>>>(a, p.splits, po, pml);
  else
    attend_join_kernel<D, kWaves><<<join, kThreads, 0, stream>>>(a, p.splits, po, pml);
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
size_t attend_workspace_bytes(int d, int64_t m, int k, int64_t units, int64_t total_q, int heads, int heads_q) {
  size_t need = 0;
  for (int ragged = 0; ragged < 2; ++ragged) {
    if (!ragged && total_q % m != 0) continue;
    const int s = make_plan(d, m, k, units, total_q, heads, heads_q, ragged != 0).splits;
    if (s == 1) continue;
    const size_t b = partial_o_bytes(d, total_q, heads_q, s) +
                     align256(static_cast<size_t>(s) * total_q * heads_q * sizeof(RowState));
    need = b > need ? b : need;
  }
  return need;
}

bool attend_fits(int d, int64_t m, int k, int64_t units, int64_t total_q, int heads, int heads_q, bool ragged) {
  const AttendPlan p = make_plan(d, m, k, units, total_q, heads, heads_q, ragged);
  return p.tiles * p.splits * heads <= kMaxGroups;
}

hipError_t launch_attend(const AttendArgs& a, int fmt, int d, hipStream_t stream) {
  const int64_t units = static_cast<int64_t>(a.k) * a.kv.ppc * a.kv.page_tokens / kUnit;
  const AttendPlan p = make_plan(d, a.m, a.k, units, a.total_q, a.kv.heads, a.hq, a.q_offsets != nullptr);
  switch (fmt) {
    case MEM_KV_BF16: return launch_fmt<MEM_KV_BF16>(a, p, d, stream);
    case MEM_KV_FP8: return launch_fmt<MEM_KV_FP8>(a, p, d, stream);
    default: return launch_fmt<MEM_KV_FP4>(a, p, d, stream);
  }
}

}  // namespace memattn
