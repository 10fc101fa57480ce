// Writing a quantised key/value cache and reading it back.
//
// Both move every byte once: a dense row in one direction, its codes and
// scales in the other, and are bound by HBM (4.9 to 6.3 TB/s in large calls,
// where a plain copy reaches 5.1; one token of 64 sessions takes 3.2 us).  An
// item is eight consecutive elements (four to be read back as fp32); when
// writing, the four items of a block of 32 are neighbouring lanes, which share
// its largest magnitude through two cross-lane steps, so a row is read once
// and nothing is staged.  A workgroup first looks up the places of its tokens
// (chunk, position and page: three dependent loads, made once per token and
// not once per item), then keeps kInFlight items per thread in flight.
#include "kv.h"
#include "device_common.h"

namespace memattn {

namespace {

constexpr int kThreads = 256;
constexpr int kInFlight = 4;  // items per thread of large calls (small ones: 1, to use more CUs)
constexpr int kTokenGroup = 32;  // consecutive tokens of a head moved together in large calls
constexpr int kMinItems = 8;   // items of a row of 64

// Tokens whose rows a workgroup moves (at most): U items a thread, groups of GROUP tokens of a row or more each.
template <int U, int GROUP>
constexpr int kMaxTokens = (kThreads * U / kMinItems / GROUP + 2) * GROUP;

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

// A workgroup's share of the rows, of keys or of values: a call moves all keys, then all values.  (Dense keys and
// values are arrays of one size, often a power of two apart: written together, both streams meet the same channels and
// banks.  131,071 tokens read back from 4 bits: token by token with keys and values side by side 192 us, so 129 us,
// 5.3 TB/s.)  Within them rows go by groups of GROUP consecutive tokens, head by head: consecutive tokens are mostly
// neighbours in a page, where heads lie apart, so that a workgroup moves whole stretches of codes and scales (65,536
// fp32 tokens to 8 bits and back: 5 % less, 138 and 106 us).  GROUP is 1 in small calls, where a group would be mostly
// empty.
template <int GROUP>
struct Share {
  int64_t tok0;      // first token of its first group
  int skip;          // rows of that group that belong to the workgroups before
  int group_rows;    // heads * GROUP
  uint64_t magic;    // ceil(2^40 / heads): x / heads = x * magic >> 40 for x < 2^18
  bool is_v;

  // Token (from tok0) and head of the workgroup's row r.
  __device__ __forceinline__ int token(int r, int* head) const {
    r += skip;
    const int x = r / GROUP, g = static_cast<int>((static_cast<uint64_t>(x) * magic) >> 40);
    *head = x - g * (group_rows / GROUP);
    return g * GROUP + r % GROUP;
  }
};

// Look up the places of the workgroup's tokens (those past the last token count as missing).
template <int GROUP>
__device__ __forceinline__ Share<GROUP> open_share(const KvView& kv, uint64_t magic, int rows, const int32_t* chunk,
                                                   const int32_t* pos, int64_t n, Place* places) {
  Share<GROUP> s;
  s.group_rows = kv.heads * GROUP;
  const uint32_t half = gridDim.x / 2;
  s.is_v = blockIdx.x >= half;
  const int64_t at = static_cast<int64_t>(s.is_v ? blockIdx.x - half : blockIdx.x) * rows;
  const int64_t group = at / s.group_rows;
  s.tok0 = group * GROUP;
  s.skip = static_cast<int>(at - group * s.group_rows);
  s.magic = magic;
  const int count = ((s.skip + rows - 1) / s.group_rows + 1) * GROUP;
  for (int t = threadIdx.x; t < count; t += kThreads) {
    const int64_t tok = s.tok0 + t;
    places[t] = tok < n ? kv_place(kv, chunk[tok], pos[tok]) : Place{-1, 0};
  }
  __syncthreads();
  return s;
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

// Elements per item: 16 bytes of a dense row read back, so that a wave's stores cover whole lines (with 32 bytes of
// fp32 a lane, stored in two halves, non-temporal stores lose 11 %); 8 of a row to be written, which keeps a block in
// one quad of lanes.
template <bool WRITE, typename T>
constexpr int kItem = WRITE ? 8 : 16 / static_cast<int>(sizeof(T));

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

template <int FMT, int D, typename T, bool VEC, int U>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvView kv, RowsView k, RowsView v,
                                                            const int32_t* __restrict__ chunk,
                                                            const int32_t* __restrict__ pos, int64_t n,
                                                            uint64_t magic) {
  constexpr int kN = kItem<true, T>, kPieces = D / kN, kGroup = U > 1 ? kTokenGroup : 1;
  __shared__ Place places[kMaxTokens<U, kGroup>];
  const auto sh = open_share<kGroup>(kv, magic, kThreads * U / kPieces, chunk, pos, n, places);
  float x[U][8];
  uint8_t *codes[U], *scales[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = threadIdx.x + u * kThreads, i = at % kPieces;
    int head;
    const int t = sh.token(at / kPieces, &head);
    const Place p = places[t];
    codes[u] = nullptr;
    scales[u] = nullptr;
    for (int j = 0; j < 8; ++j) x[u][j] = 0.f;
    if (p.page < 0) continue;
    const RowsView& src = sh.is_v ? v : k;
    load8<T, VEC, (U > 1)>(static_cast<const T*>(src.data) + (sh.tok0 + t) * src.ts + head * src.hs + i * kN, x[u]);
    int64_t co, so;
    kv_offsets<FMT, D, kN>(kv, head, sh.is_v, p.row, i, &co, &so);
    uint8_t* base = kv.pool + p.page * kv.page_bytes;
    codes[u] = base + co;
    scales[u] = base + so;
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    encode_item<FMT>(x[u], codes[u], scales[u], threadIdx.x % 4 == 0, codes[u] != nullptr);
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

template <int FMT, int D, typename T, bool VEC, int U>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvView kv, RowsView k, RowsView v,
                                                           const int32_t* __restrict__ chunk,
                                                           const int32_t* __restrict__ pos, int64_t n,
                                                           uint64_t magic) {
  constexpr int kN = kItem<false, T>, kPieces = D / kN, kGroup = U > 1 ? kTokenGroup : 1;
  constexpr int kBytes = kN * kv_row_bytes(FMT, D) / D, kWords = (kBytes + 3) / 4;  // of an item's codes
  __shared__ Place places[kMaxTokens<U, kGroup>];
  const auto sh = open_share<kGroup>(kv, magic, kThreads * U / kPieces, chunk, pos, n, places);
  uint32_t c[U][kWords], byte[U];
  T* dst[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = threadIdx.x + u * kThreads, i = at % kPieces;
    int head;
    const int t = sh.token(at / kPieces, &head);
    const Place p = places[t];
    const RowsView& to = sh.is_v ? v : k;
    const int64_t tok = sh.tok0 + t;
    dst[u] = tok < n ? static_cast<T*>(to.data) + tok * to.ts + head * to.hs + i * kN : nullptr;
    byte[u] = 127;
    for (int w = 0; w < kWords; ++w) c[u][w] = 0;
    if (p.page < 0) continue;  // reads as zeros
    int64_t co, so;
    kv_offsets<FMT, D, kN>(kv, head, sh.is_v, p.row, i, &co, &so);
    const uint8_t* base = kv.pool + p.page * kv.page_bytes;
    const uint32_t* src = reinterpret_cast<const uint32_t*>(base + co);
    if constexpr (kWords == 4) {
      const u32x4_t w = *reinterpret_cast<const u32x4_t*>(src);
      for (int j = 0; j < 4; ++j) c[u][j] = w[j];
    } else if constexpr (kWords == 2) {
      const u32x2_t w = *reinterpret_cast<const u32x2_t*>(src);
      c[u][0] = w[0];
      c[u][1] = w[1];
    } else if constexpr (kBytes == 4) {
      c[u][0] = *src;
    } else {
      c[u][0] = *reinterpret_cast<const uint16_t*>(src);
    }
    if constexpr (FMT != MEM_KV_BF16) byte[u] = base[so];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!dst[u]) continue;
    float x[kN];
    if constexpr (FMT == MEM_KV_BF16) {
      for (int j = 0; j < kN / 2; ++j) {
        x[2 * j] = __uint_as_float(c[u][j] << 16);
        x[2 * j + 1] = __uint_as_float(c[u][j] & 0xFFFF0000u);
      }
    } else {
      decode_item<FMT, kN>(c[u], byte[u], x);
    }
    store_item<T, VEC, (U > 1)>(dst[u], x);
  }
}

// 16-byte accesses of the dense rows need aligned rows.
bool rows_aligned(const RowsView& r, int elem) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(r.data) | static_cast<uintptr_t>(r.ts * elem) |
                      static_cast<uintptr_t>(r.hs * elem);
  return (a & 15u) == 0;
}

// Items per thread and workgroups of a call whose rows are moved in `pieces` items each.
struct MoveGrid {
  int u;
  int64_t groups;
};

MoveGrid move_grid(int heads, int pieces, int64_t n) {
  const int64_t items = 2 * n * heads * pieces;
  // one item per thread until that alone fills the GPU (256 CUs of 2,048 threads)
  const int u = items >= int64_t{256} * 2048 * kInFlight ? kInFlight : 1;
  const int group = u == 1 ? 1 : kTokenGroup;
  const int64_t half = (n + group - 1) / group * group * heads * pieces;  // of keys, and of values
  return {u, 2 * ((half + kThreads * u - 1) / (kThreads * u))};
}

template <bool WRITE, int FMT, int D, typename T>
hipError_t launch_typed(const KvView& kv, const RowsView& k, const RowsView& v, const int32_t* chunk,
                        const int32_t* pos, int64_t n, hipStream_t stream) {
  const bool vec = rows_aligned(k, sizeof(T)) && rows_aligned(v, sizeof(T));
  const uint64_t magic = ((uint64_t{1} << 40) + kv.heads - 1) / kv.heads;
  const MoveGrid g = move_grid(kv.heads, D / kItem<WRITE, T>, n);
  const dim3 grid(static_cast<unsigned>(g.groups));
  auto go = [&](auto write, auto read) {
    (WRITE ? write : read)<<<grid, kThreads, 0, stream>>>(kv, k, v, chunk, pos, n, magic);
    return hipGetLastError();
  };
  if (g.u == 1)
    return vec ? go(kv_write_kernel<FMT, D, T, true, 1>, kv_read_kernel<FMT, D, T, true, 1>)
               : go(kv_write_kernel<FMT, D, T, false, 1>, kv_read_kernel<FMT, D, T, false, 1>);
  return vec ? go(kv_write_kernel<FMT, D, T, true, kInFlight>, kv_read_kernel<FMT, D, T, true, kInFlight>)
             : go(kv_write_kernel<FMT, D, T, false, kInFlight>, kv_read_kernel<FMT, D, T, false, kInFlight>);
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

bool kv_move_fits(bool write, int heads, int d, int dtype, int64_t n) {
  const int item = write ? kItem<true, float> : dtype == MEM_F32 ? kItem<false, float> : kItem<false, uint16_t>;
  return move_grid(heads, d / item, n).groups <= kMaxGroups;
}

hipError_t launch_kv_write(const KvView& kv, int fmt, int d, const RowsView& k, const RowsView& v, int dtype,
                           const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream) {
  return launch_any<true>(kv, fmt, d, k, v, dtype, chunk, pos, n, stream);
}

hipError_t launch_kv_read(const KvView& kv, int fmt, int d, const RowsView& k, const RowsView& v, int dtype,
                          const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream) {
  return launch_any<false>(kv, fmt, d, k, v, dtype, chunk, pos, n, stream);
}

}  // namespace memattn
