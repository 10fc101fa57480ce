// What the kernels that move tokens into a cache and out of it share: the place of
// a token, items of a dense row, and their codes.
#pragma once

#include "kv.h"
#include "device_common.h"

namespace memattn {

namespace {

// Page and row of a token; page -1: the place does not exist.
struct Place {
  int32_t page;
  int32_t row;
};

__device__ __forceinline__ Place kv_place(const KvView& kv, int32_t chunk, int32_t pos) {
  if (chunk < 0 || chunk >= kv.n_chunks || pos < 0) return {-1, 0};
  const int p = pos / kv.page_tokens;
  if (p >= kv.ppc) return {-1, 0};
  const int32_t pg = kv.table[static_cast<int64_t>(chunk) * kv.ppc + p];
  if (pg < 0 || pg >= kv.n_pages) return {-1, 0};
  return {pg, pos - p * kv.page_tokens};
}

// Where item `i` of a row lies: byte offsets of its codes and of its scale byte in the page.
template <int FMT, int D, int ITEM>
__device__ __forceinline__ void kv_offsets(const KvView& kv, int head, bool is_v, int row, int i, int64_t* codes,
                                           int64_t* scale) {
  constexpr int kRow = kv_row_bytes(FMT, D), kSc = kv_scale_bytes(FMT, D);
  const int64_t t = kv.page_tokens;
  const int64_t base = static_cast<int64_t>(head) * 2 * t * (kRow + kSc);
  *codes = base + (is_v ? t * kRow : 0) + static_cast<int64_t>(row) * kRow + i * (kRow / (D / ITEM));
  *scale = base + 2 * t * kRow + (is_v ? t * kSc : 0) + static_cast<int64_t>(row) * kSc + i * ITEM / kKvBlock;
}

// 16 bytes; with NT past the caches, for large calls' dense rows, which no later part of the call touches.
template <bool NT>
__device__ __forceinline__ u32x4_t load16(const void* p) {
  if constexpr (NT) return __builtin_nontemporal_load(static_cast<const u32x4_t*>(p));
  return *static_cast<const u32x4_t*>(p);
}
template <bool NT>
__device__ __forceinline__ void store16(void* p, u32x4_t v) {
  if constexpr (NT)
    __builtin_nontemporal_store(v, static_cast<u32x4_t*>(p));
  else
    *static_cast<u32x4_t*>(p) = v;
}

template <typename T, bool VEC, bool NT>
__device__ __forceinline__ void load8(const T* p, float* x) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (VEC) {
      for (int h = 0; h < 2; ++h) {
        const u32x4_t v = load16<NT>(p + 4 * h);
        for (int j = 0; j < 4; ++j) x[4 * h + j] = __uint_as_float(v[j]);
      }
    } else {
      for (int j = 0; j < 8; ++j) x[j] = p[j];
    }
  } else {
    union { u32x4_t v; uint16_t h[8]; } u;
    if constexpr (VEC) {
      u.v = load16<NT>(p);
    } else {
      for (int j = 0; j < 8; ++j) u.h[j] = p[j];
    }
    for (int j = 0; j < 8; ++j) x[j] = bf16_to_f32(u.h[j]);
  }
}

// Two floats as bf16, to nearest, ties to even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf16x2 p = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
  return __builtin_bit_cast(uint32_t, p);
}

// 16 bytes of a dense row: 4 floats, or 8 rounded to bf16.
template <typename T, bool VEC, bool NT>
__device__ __forceinline__ void store_item(T* p, const float* x) {
  union { u32x4_t v; T e[16 / sizeof(T)]; } u;
  for (int j = 0; j < 4; ++j) u.v[j] = sizeof(T) == 4 ? __float_as_uint(x[j]) : pack_bf16(x[2 * j], x[2 * j + 1]);
  if constexpr (VEC) {
    store16<NT>(p, u.v);
  } else {
    for (int j = 0; j < static_cast<int>(16 / sizeof(T)); ++j) p[j] = u.e[j];
  }
}

// Codes of the block of which this lane holds eight elements, written to `codes`, and the scale byte.  A row's items
// are consecutive and start at a multiple of 8, so the four items of a block are lanes of one quad.
template <int FMT>
__device__ __forceinline__ void encode_item(float* x, uint8_t* codes, uint8_t* scale, bool first, bool live) {
  if constexpr (FMT == MEM_KV_BF16) {
    if (live) store_item<uint16_t, true, false>(reinterpret_cast<uint16_t*>(codes), x);
  } else {
    uint32_t amax = 0;
    for (int j = 0; j < 8; ++j) amax = max(amax, __float_as_uint(x[j]) & 0x7FFFFFFFu);
    amax = max(amax, dpp_u32<0xB1>(amax));
    amax = max(amax, dpp_u32<0x4E>(amax));
    if (!live) return;
    const uint32_t byte = kv_scale_byte<FMT>(amax);
    const float inv = kv_inverse_scale(byte);
    constexpr float kTop = FMT == MEM_KV_FP4 ? 6.f : 448.f;
    for (int j = 0; j < 8; ++j) x[j] = __builtin_amdgcn_fmed3f(x[j] * inv, -kTop, kTop);
    if constexpr (FMT == MEM_KV_FP4) {
      uint32_t c = 0;
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], 1.f, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], 1.f, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], 1.f, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], 1.f, 3);
      *reinterpret_cast<uint32_t*>(codes) = c;
    } else {
      u32x2_t c;
      for (int w = 0; w < 2; ++w) {
        const int u = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w], x[4 * w + 1], 0, false);
        c[w] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w + 2], x[4 * w + 3], u, true));
      }
      *reinterpret_cast<u32x2_t*>(codes) = c;
    }
    if (first) *scale = static_cast<uint8_t>(byte);
  }
}

// N elements (4 or 8) of a block from their codes.
template <int FMT, int N>
__device__ __forceinline__ void decode_item(const uint32_t* c, uint32_t byte, float* x) {
  const float s = kv_scale(byte);
  f32x2 p[N / 2];
  if constexpr (FMT == MEM_KV_FP4) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], s, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], s, 1);
    if constexpr (N == 8) {
      p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], s, 2);
      p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], s, 3);
    }
  } else {
    for (int w = 0; w < N / 4; ++w) {
      p[2 * w] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[w], s, false);
      p[2 * w + 1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[w], s, true);
    }
  }
  for (int j = 0; j < N / 2; ++j) {
    x[2 * j] = byte == 255u ? __uint_as_float(0x7FC00000u) : p[j][0];
    x[2 * j + 1] = byte == 255u ? __uint_as_float(0x7FC00000u) : p[j][1];
  }
}

// 16-byte accesses of the dense rows need aligned rows.
inline bool rows_aligned(const RowsView& r, int elem) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(r.data) | static_cast<uintptr_t>(r.ts * elem) |
                      static_cast<uintptr_t>(r.hs * elem);
  return (a & 15u) == 0;
}

}  // namespace

}  // namespace memattn
