// The paged key/value cache as the kernels see it, and the conversions of its
// blocks.  Internal to the library: the public interface is
// include/memattn_kv.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "memattn_kv.h"

namespace memattn {

constexpr int kKvBlock = 32;  // elements that share a scale

// Workgroups of a launch: all kernels here have 256 threads each, and a launch has fewer than 2^32 threads.
constexpr int64_t kMaxGroups = (int64_t{1} << 24) - 1;

// Bytes of codes and of scales of a row of d elements.
__host__ __device__ constexpr int kv_row_bytes(int fmt, int d) {
  return fmt == MEM_KV_BF16 ? 2 * d : fmt == MEM_KV_FP8 ? d : d / 2;
}
__host__ __device__ constexpr int kv_scale_bytes(int fmt, int d) { return fmt == MEM_KV_BF16 ? 0 : d / kKvBlock; }

struct KvView {
  uint8_t* pool;
  int64_t n_pages;
  int64_t page_bytes;
  const int32_t* table;  // [n_chunks, ppc]
  int64_t n_chunks;
  int32_t ppc;
  int32_t page_tokens;
  int32_t heads;
};

// Dense rows: element (token, head, i) at data[token * ts + head * hs + i].
struct RowsView {
  void* data;
  int64_t ts;
  int64_t hs;
};

constexpr int kRopeDim = 64;  // elements of a latent cache's rotated key part

// Tokens to append.  Of a latent cache `k` are the latent rows and `v` the key parts.
struct AppendArgs {
  KvView kv;
  RowsView k, v, q, q_out;
  int32_t hq;  // rows of q per token; 0: none
  const int32_t* chunk;
  const int32_t* pos;
  const int32_t* at;  // positions by which rows are rotated
  const float* freq;
  int32_t half;       // pairs of a rotated row
  bool pairs;         // pair i is (2 i, 2 i + 1), not (i, i + half)
  int64_t n;
};

struct AttendArgs {
  KvView kv;
  const int32_t* tok_len;
  const int32_t* ids;
  int64_t m;
  int32_t k;
  int32_t hq;
  const int32_t* q_offsets;
  const int32_t* q_pos;
  float scale;
  float softcap;
  const float* slopes;
  int32_t causal;
  int32_t window;
  const int32_t* prefix_len;
  const int32_t* chunk_ns;
  const int32_t* query_ns;
  const uint16_t* q;
  int64_t q_ts;
  int64_t q_hs;
  int64_t total_q;
  uint16_t* out;
  float* lse;
  void* ws;
};

hipError_t launch_kv_write(const KvView& kv, int fmt, int d, const RowsView& k, const RowsView& v, int dtype,
                           const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream);
hipError_t launch_kv_read(const KvView& kv, int fmt, int d, const RowsView& k, const RowsView& v, int dtype,
                          const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream);
// Whether n tokens (of at most 2^40 elements) fit one launch.
bool kv_move_fits(bool write, int heads, int d, int dtype, int64_t n);
// Whether n tokens fit one launch.
bool append_fits(bool latent, int half, int64_t n);
hipError_t launch_kv_append(const AppendArgs& a, int fmt, int d, int dtype, hipStream_t stream);
hipError_t launch_latent_append(const AppendArgs& a, int fmt, int l, int dtype, hipStream_t stream);
hipError_t launch_latent_read(const KvView& kv, int fmt, int l, const RowsView& c, const RowsView& r, int dtype,
                              const int32_t* chunk, const int32_t* pos, int64_t n, hipStream_t stream);
// `units`: blocks of 32 tokens that a request's chunks can hold.
size_t attend_workspace_bytes(int d, int64_t m, int k, int64_t units, int64_t total_q, int heads, int heads_q);
// Whether the call's workgroups fit its launches.
bool attend_fits(int d, int64_t m, int k, int64_t units, int64_t total_q, int heads, int heads_q, bool ragged);
hipError_t launch_attend(const AttendArgs& a, int fmt, int d, hipStream_t stream);

#ifdef __HIPCC__

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// The largest scale byte that mem_kv_write gives a block without a NaN.
template <int FMT>
constexpr uint32_t kMaxScaleByte = 127 + (FMT == MEM_KV_FP4 ? 125 : 119);

// Scale byte of a block whose largest magnitude has the bit pattern `amax`
// (the maximum of the elements' patterns without sign, so that a NaN is above
// every number): 127 plus the smallest e with amax <= 1.75 * 2^(e + 2) (FP4)
// or 1.8125 * 2^(e + 8) (FP8), clamped; 255 marks a NaN.
template <int FMT>
__device__ __forceinline__ uint32_t kv_scale_byte(uint32_t amax) {
  constexpr int kTop = FMT == MEM_KV_FP4 ? 2 : 8;
  constexpr uint32_t kLimit = FMT == MEM_KV_FP4 ? 0x600000u : 0x680000u;
  if (amax > 0x7F800000u) return 255u;
  const uint32_t a = min(amax, 0x7F7FFFFFu);
  const int e = static_cast<int>(a >> 23) - 127 - kTop + ((a & 0x7FFFFFu) > kLimit ? 1 : 0);
  return min(static_cast<uint32_t>(max(e, -110) + 127), kMaxScaleByte<FMT>);
}

// 2^-e of a scale byte that kv_scale_byte returned (a NaN for 255).
__device__ __forceinline__ float kv_inverse_scale(uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float((254u - byte) << 23);
}

// The scale operand of the hardware conversions: only its exponent is used.
__device__ __forceinline__ float kv_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

#endif  // __HIPCC__

}  // namespace memattn
