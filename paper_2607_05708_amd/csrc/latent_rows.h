// What the kernels of both forms of latent attention share: rows in LDS, sums of
// weights and the rows that they end as.
#pragma once

#include "context.h"
#include "kv.h"
#include "latent.h"

namespace memattn {

namespace {

// Rows of L latent elements and the key part in LDS, bf16.  The pitch is an odd multiple of 64 bytes, so that four rows
// lie in different banks, and the 16-byte chunks of a row are exchanged within 64 bytes by bits 2 and 3 of the row's
// number: neither reads along a row (the first product's operands: one column of 32 rows) nor transposing reads (the
// second product's) conflict.  (By bits 1 and 2 36 % of the cycles of these reads were conflicts.)
template <int L>
constexpr int kLatentPitch = L + kRopeDim + 32;
__device__ __forceinline__ int exchange(int row) { return (row >> 2) & 3; }

// Where a lane reads transposed operands of 16 rows (of 32 columns from a multiple of 32 on): rows 0 .. 7 at [0], 8 .. 15
// at [1], elements from the first row's.  Both are the same again 16 rows on.
template <int PITCH>
struct Transposed {
  int at[2];

  __device__ __forceinline__ explicit Transposed(int lane) {
    const int i = lane & 15, c = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int r = 4 * (lane >> 5) + (i >> 2) + 8 * y;
      at[y] = r * PITCH + 8 * (c ^ exchange(r)) + 4 * (i & 1);
    }
  }
  __device__ __forceinline__ bf16x8 operator()(const uint16_t* rows) const {
    const u32x2_t v0 = lds_transpose4(rows + at[0]), v1 = lds_transpose4(rows + at[1]);
    return as_bf16x8(u32x4_t{v0[0], v0[1], v1[0], v1[1]});
  }
};

// x + both halves of a pair of bf16.
__device__ __forceinline__ float add_pair(uint32_t pair, float x) {
  constexpr uint32_t kOnes = 0x3F803F80u;
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(s16x2, pair), __builtin_bit_cast(s16x2, kOnes), x, false);
}

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

  // All of it, from row `row` of a page of T tokens.
  __device__ __forceinline__ void load(const uint8_t* page, int64_t T, uint32_t row, int part) {
#pragma unroll
    for (int y = 0; y < kLoads; ++y)
      codes[y] = *reinterpret_cast<const u32x4_t*>(page + (row * kRow + 16 * part + 128 * y));
    rope = *reinterpret_cast<const u32x4_t*>(page + T * kRow + (row * (2 * kRopeDim) + 16 * part));
    if constexpr (FMT != MEM_KV_BF16) {
#pragma unroll
      for (int i = 0; i < kScaleWords / 2; ++i) {
        const u32x2_t v = reinterpret_cast<const u32x2_t*>(page + T * (kRow + 2 * kRopeDim) + row * kSc)[i];
        sc[2 * i] = v[0];
        sc[2 * i + 1] = v[1];
      }
    }
  }
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

// Scales rows whose registers are accumulation registers.  (The compiler would otherwise keep them, for the
// multiplications' sake, where the matrix products cannot: of 32 x 512 it spills most.)
template <int WIDTH, int D>
__device__ __forceinline__ void scale_rows(Rows<WIDTH, D>& rows, float f) {
#pragma unroll
  for (int n = 0; n < D / WIDTH; ++n) {
    auto x = rows.o[n];
    asm volatile("" : "+a"(x));
    auto y = x * f;
    asm volatile("" : "+a"(y));
    rows.o[n] = y;
    if (WIDTH == 32 || n % 4 == 3) issue_first();
  }
}

// Write elements first .. + N - 1 of a row's weighted sum (of L) as part `split` of it.  `rounded` is the sum of the
// weights as the product took them: dividing by it lets their roundings cancel where a few weigh most; what joins the
// parts divides by l.
template <int WIDTH, int N, int L>
__device__ __forceinline__ void write_part(const AttendArgs& a, const Rows<WIDTH, N>& rows, RowState st, float rounded,
                                           bool poison, int64_t row_at, int part, int split, int first, float* part_o,
                                           RowState* part_ml) {
  if (poison) st.l = NAN;
  const int64_t at = static_cast<int64_t>(split) * a.total_q * a.hq + row_at;
  const float even = st.l == 0.f ? 0.f : st.l * inverse_sum(rounded);
  float* dst = part_o + at * L + first;
  rows.each4(part, [&](int d, f32x4 v) { *reinterpret_cast<f32x4*>(dst + d) = v * even; });
  if (part == 0 && first == 0) part_ml[at] = st;
}

// The same, but where the context is not split the row itself, as bf16.
template <int WIDTH, int L>
__device__ __forceinline__ void write_sums(const AttendArgs& a, const Rows<WIDTH, L>& rows, RowState st, float rounded,
                                           bool poison, int64_t row_at, int part, int split, int splits, uint16_t* out,
                                           float* part_o, RowState* part_ml) {
  if (splits > 1) {
    write_part<WIDTH, L, L>(a, rows, st, rounded, poison, row_at, part, split, 0, part_o, part_ml);
    return;
  }
  const float inv = poison ? NAN : inverse_sum(rounded);
  uint16_t* dst = out + row_at * L;
  rows.each4(part, [&](int d, f32x4 v) {
    *reinterpret_cast<u32x2_t*>(dst + d) = u32x2_t{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
  });
  if (a.lse && part == 0) a.lse[row_at] = poison ? NAN : lse_of(st.m, st.l);
}

}  // namespace

}  // namespace memattn
