// Writing a quantised key/value cache and reading it back.
//
// Both move every byte once: a dense row in one direction, its codes and
// scales in the other, and are bound by HBM.  A thread handles eight
// consecutive elements (16 bytes of bf16, 4 bytes of 4-bit codes); the four
// threads of a block of 32 share its largest magnitude through two
// cross-lane steps, so a row is read once and nothing is staged.
#include "kv.h"
#include "device_common.h"

namespace memattn {

namespace {

constexpr int kThreads = 256;
constexpr int kPiece = 8;  // elements per thread

// First byte of token (chunk, pos) of head 0's part, and its row in the page; false if the place does not exist.
__device__ __forceinline__ bool kv_place(const KvView& kv, int32_t chunk, int32_t pos, int64_t* page, int* row) {
  if (chunk < 0 || chunk >= kv.n_chunks || pos < 0) return false;
  const int p = pos / kv.page_tokens;
  if (p >= kv.ppc) return false;
  const int32_t pg = kv.table[static_cast<int64_t>(chunk) * kv.ppc + p];
  if (pg < 0 || pg >= kv.n_pages) return false;
  *page = pg;
  *row = pos - p * kv.page_tokens;
  return true;
}

// Where piece `i` (elements 8 i ..) of a row lies: byte offsets of its codes and of its scale byte in the page.
template <int FMT, int D>
__device__ __forceinline__ void kv_offsets(const KvView& kv, int head, bool is_v, int row, int i, int64_t* codes,
                                           int64_t* scale) {
  constexpr int kRow = kv_row_bytes(FMT, D), kSc = kv_scale_bytes(FMT, D);
  const int64_t t = kv.page_tokens;
  const int64_t base = static_cast<int64_t>(head) * 2 * t * (kRow + kSc);
  *codes = base + (is_v ? t * kRow : 0) + static_cast<int64_t>(row) * kRow + i * (kRow / (D / kPiece));
  *scale = base + 2 * t * kRow + (is_v ? t * kSc : 0) + static_cast<int64_t>(row) * kSc + i * kPiece / kKvBlock;
}

template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, float* x) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (VEC) {
      *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(p);
      *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(p + 4);
    } else {
      for (int j = 0; j < 8; ++j) x[j] = p[j];
    }
  } else {
    union { u32x4_t v; uint16_t h[8]; } u;
    if constexpr (VEC) {
      u.v = *reinterpret_cast<const u32x4_t*>(p);
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

template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, const float* x) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (VEC) {
      *reinterpret_cast<float4*>(p) = *reinterpret_cast<const float4*>(x);
      *reinterpret_cast<float4*>(p + 4) = *reinterpret_cast<const float4*>(x + 4);
    } else {
      for (int j = 0; j < 8; ++j) p[j] = x[j];
    }
  } else {
    union { u32x4_t v; uint16_t h[8]; } u;
    for (int j = 0; j < 4; ++j) u.v[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
    if constexpr (VEC) {
      *reinterpret_cast<u32x4_t*>(p) = u.v;
    } else {
      for (int j = 0; j < 8; ++j) p[j] = u.h[j];
    }
  }
}

// Threads of a row stay together (D / 8 is a multiple of 8 and divides 64), so a block's four threads are lanes of
// one quad and take the same branches.
template <int FMT, int D, typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvView kv, RowsView k, RowsView v,
                                                            const int32_t* __restrict__ chunk,
                                                            const int32_t* __restrict__ pos, int64_t n) {
  constexpr int kPieces = D / kPiece;
  const int64_t per_token = 2 * static_cast<int64_t>(kv.heads) * kPieces;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t tok = at / per_token;
  if (tok >= n) return;
  const int rest = static_cast<int>(at - tok * per_token);
  const int i = rest % kPieces, hv = rest / kPieces;
  const bool is_v = hv >= kv.heads;
  const int head = is_v ? hv - kv.heads : hv;
  int64_t page;
  int row;
  if (!kv_place(kv, chunk[tok], pos[tok], &page, &row)) return;
  const RowsView& src = is_v ? v : k;
  float x[8];
  load8<T, VEC>(static_cast<const T*>(src.data) + tok * src.ts + head * src.hs + i * kPiece, x);
  int64_t co, so;
  kv_offsets<FMT, D>(kv, head, is_v, row, i, &co, &so);
  uint8_t* base = kv.pool + page * kv.page_bytes;
  if constexpr (FMT == MEM_KV_BF16) {
    store8<uint16_t, true>(reinterpret_cast<uint16_t*>(base + co), x);
  } else {
    uint32_t amax = 0;
    for (int j = 0; j < 8; ++j) amax = max(amax, __float_as_uint(x[j]) & 0x7FFFFFFFu);
    amax = max(amax, dpp_u32<0xB1>(amax));
    amax = max(amax, dpp_u32<0x4E>(amax));
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
      *reinterpret_cast<uint32_t*>(base + co) = c;
    } else {
      u32x2_t c;
      for (int w = 0; w < 2; ++w) {
        int u = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w], x[4 * w + 1], 0, false);
        c[w] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w + 2], x[4 * w + 3], u, true));
      }
      *reinterpret_cast<u32x2_t*>(base + co) = c;
    }
    if (i % 4 == 0) base[so] = static_cast<uint8_t>(byte);
  }
}

template <int FMT, int D, typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvView kv, RowsView k, RowsView v,
                                                           const int32_t* __restrict__ chunk,
                                                           const int32_t* __restrict__ pos, int64_t n) {
  constexpr int kPieces = D / kPiece;
  const int64_t per_token = 2 * static_cast<int64_t>(kv.heads) * kPieces;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t tok = at / per_token;
  if (tok >= n) return;
  const int rest = static_cast<int>(at - tok * per_token);
  const int i = rest % kPieces, hv = rest / kPieces;
  const bool is_v = hv >= kv.heads;
  const int head = is_v ? hv - kv.heads : hv;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  int64_t page;
  int row;
  if (kv_place(kv, chunk[tok], pos[tok], &page, &row)) {
    int64_t co, so;
    kv_offsets<FMT, D>(kv, head, is_v, row, i, &co, &so);
    const uint8_t* base = kv.pool + page * kv.page_bytes;
    if constexpr (FMT == MEM_KV_BF16) {
      load8<uint16_t, true>(reinterpret_cast<const uint16_t*>(base + co), x);
    } else {
      const uint32_t byte = base[so];
      const float s = kv_scale(byte);
      f32x2 p[4];
      if constexpr (FMT == MEM_KV_FP4) {
        const uint32_t c = *reinterpret_cast<const uint32_t*>(base + co);
        p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0);
        p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
        p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2);
        p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
      } else {
        const u32x2_t c = *reinterpret_cast<const u32x2_t*>(base + co);
        for (int w = 0; w < 2; ++w) {
          p[2 * w] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[w], s, false);
          p[2 * w + 1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[w], s, true);
        }
      }
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = byte == 255u ? __uint_as_float(0x7FC00000u) : p[j][0];
        x[2 * j + 1] = byte == 255u ? __uint_as_float(0x7FC00000u) : p[j][1];
      }
    }
  }
  const RowsView& dst = is_v ? v : k;
  store8<T, VEC>(static_cast<T*>(dst.data) + tok * dst.ts + head * dst.hs + i * kPiece, x);
}

// 16-byte accesses of the dense rows need aligned rows.
bool rows_aligned(const RowsView& r, int elem) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(r.data) | static_cast<uintptr_t>(r.ts * elem) |
                      static_cast<uintptr_t>(r.hs * elem);
  return (a & 15u) == 0;
}

template <bool WRITE, int FMT, int D, typename T>
hipError_t launch_typed(const KvView& kv, const RowsView& k, const RowsView& v, const int32_t* chunk,
                        const int32_t* pos, int64_t n, hipStream_t stream) {
  const int64_t threads = n * 2 * kv.heads * (D / kPiece);
  const dim3 grid(static_cast<unsigned>((threads + kThreads - 1) / kThreads));
  const bool vec = rows_aligned(k, sizeof(T)) && rows_aligned(v, sizeof(T));
  if (WRITE) {
    if (vec)
      kv_write_kernel<FMT, D, T, true><<<grid, kThreads, 0, stream>>>(kv, k, v, chunk, pos, n);
    else
      kv_write_kernel<FMT, D, T, false><<<grid, kThreads, 0, stream>>>(kv, k, v, chunk, pos, n);
  } else {
    if (vec)
      kv_read_kernel<FMT, D, T, true><<<grid, kThreads, 0, stream>>>(kv, k, v, chunk, pos, n);
    else
      kv_read_kernel<FMT, D, T, false><<<grid, kThreads, 0, stream>>>(kv, k, v, chunk, pos, n);
  }
  return hipGetLastError();
}

template <bool WRITE, int FMT, int D>
hipError_t launch_dim(const KvView& kv, const RowsView& k, const RowsView& v, int dtype, const int32_t* chunk,
                      const int32_t* pos, int64_t n, hipStream_t stream) {
  return dtype == MEM_F32 ? launch_typed<WRITE, FMT, D, float>(kv, k, v, chunk, pos, n, stream)
                          : launch_typed<WRITE, FMT, D, uint16_t>(kv, k, v, chunk, pos, n, stream);
}

template <bool WRITE, int FMT>
hipError_t launch_fmt(const KvView& kv, int d, const RowsView& k, const RowsView& v, int dtype, const int32_t* chunk,
                      const int32_t* pos, int64_t n, hipStream_t stream) {
  switch (d) {
    case 64: return launch_dim<WRITE, FMT, 64>(kv, k, v, dtype, chunk, pos, n, stream);
    case 128: return launch_dim<WRITE, FMT, 128>(kv, k, v, dtype, chunk, pos, n, stream);
    default: return launch_dim<WRITE, FMT, 256>(kv, k, v, dtype, chunk, pos, n, stream);
  }
}

template <bool WRITE>
hipError_t launch_any(const KvView& kv, int fmt, int d, const RowsView& k, const RowsView& v, int dtype,
                      const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream) {
  switch (fmt) {
    case MEM_KV_BF16: return launch_fmt<WRITE, MEM_KV_BF16>(kv, d, k, v, dtype, chunk, pos, n, stream);
    case MEM_KV_FP8: return launch_fmt<WRITE, MEM_KV_FP8>(kv, d, k, v, dtype, chunk, pos, n, stream);
    default: return launch_fmt<WRITE, MEM_KV_FP4>(kv, d, k, v, dtype, chunk, pos, n, stream);
  }
}

}  // namespace

hipError_t launch_kv_write(const KvView& kv, int fmt, int d, const RowsView& k, const RowsView& v, int dtype,
                           const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream) {
  return launch_any<true>(kv, fmt, d, k, v, dtype, chunk, pos, n, stream);
}

hipError_t launch_kv_read(const KvView& kv, int fmt, int d, const RowsView& k, const RowsView& v, int dtype,
                          const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream) {
  return launch_any<false>(kv, fmt, d, k, v, dtype, chunk, pos, n, stream);
}

}  // namespace memattn
