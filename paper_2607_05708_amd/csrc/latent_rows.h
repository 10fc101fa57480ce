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

// Write elements first .. + N - 1 of a row's weighted sum (of L), or of its part of a split context.  `rounded`
// is the sum of the weights as the product took them, and what it is divided by, so that their roundings cancel where a
// few weigh most; the join divides by l.
template <int WIDTH, int N, int L>
__device__ __forceinline__ void write_sums(const AttendArgs& a, const Rows<WIDTH, N>& rows, RowState st, float rounded,
                                           bool poison, int64_t row_at, int part, int split, int splits, int first,
                                           uint16_t* sums, float* part_o, RowState* part_ml) {
  if (poison) st.l = NAN;
  if (splits == 1) {
    const float inv = poison ? NAN : inverse_sum(rounded);
    uint16_t* dst = sums + row_at * L + first;
    rows.each4(part, [&](int d, f32x4 v) {
      *reinterpret_cast<u32x2_t*>(dst + d) = u32x2_t{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
    });
    if (a.lse && part == 0 && first == 0) a.lse[row_at] = lse_of(st.m, st.l);
  } else {
    const int64_t at = static_cast<int64_t>(split) * a.total_q * a.hq + row_at;
    const float even = st.l == 0.f ? 0.f : st.l * inverse_sum(rounded);
    float* dst = part_o + at * L + first;
    rows.each4(part, [&](int d, f32x4 v) { *reinterpret_cast<f32x4*>(dst + d) = v * even; });
    if (part == 0 && first == 0) part_ml[at] = st;
  }
}

}  // namespace

}  // namespace memattn
