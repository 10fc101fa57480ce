// Attention over the paged key/value cache: the plain form.  One wave per
// (new token, query head) walks the request's chunks 64 tokens at a time; each
// lane scores one token, the running maximum and sum of the softmax are kept
// in the log2 domain, and each lane then owns head_dim / 64 output columns.
#include "kv.h"
#include "device_common.h"

namespace memattn {

namespace {

template <int FMT>
__device__ __forceinline__ float kv_value(const uint8_t* codes, const uint8_t* scales, int i) {
  if constexpr (FMT == MEM_KV_BF16) {
    return bf16_to_f32(reinterpret_cast<const uint16_t*>(codes)[i]);
  } else {
    const uint32_t byte = scales[i / kKvBlock];
    if (byte == 255u) return __uint_as_float(0x7FC00000u);
    constexpr int kMan = FMT == MEM_KV_FP4 ? 1 : 3, kBias = FMT == MEM_KV_FP4 ? 1 : 7;
    uint32_t c = codes[FMT == MEM_KV_FP4 ? i / 2 : i];
    uint32_t sign;
    if constexpr (FMT == MEM_KV_FP4) {
      c = (i & 1) ? c >> 4 : c & 15u;
      sign = c >> 3;
      c &= 7u;
    } else {
      sign = c >> 7;
      c &= 127u;
      if (c == 127u) return __uint_as_float(0x7FC00000u);
    }
    const int ex = static_cast<int>(c >> kMan);
    const float man = static_cast<float>(c & ((1u << kMan) - 1)) / (1 << kMan);
    const float v = ldexpf(ex ? 1.f + man : man, (ex ? ex : 1) - kBias + static_cast<int>(byte) - 127);
    return sign ? -v : v;
  }
}

template <int FMT, int D>
__global__ __launch_bounds__(64) void attend_simple_kernel(AttendArgs a) {
  constexpr int kRow = kv_row_bytes(FMT, D), kSc = kv_scale_bytes(FMT, D), kCols = D / 64;
  __shared__ float qs[D];
  __shared__ float ps[64];
  __shared__ const uint8_t* vs[64];
  const int lane = threadIdx.x;
  const int h = static_cast<int>(blockIdx.x % a.hq);
  const int64_t j = blockIdx.x / a.hq;
  const int g = h / (a.hq / a.kv.heads);
  // the request that owns row j
  int64_t req;
  int q0, nq;
  if (a.q_offsets) {
    int64_t lo = 0, hi = a.m - 1;
    while (lo < hi) {
      const int64_t mid = (lo + hi + 1) / 2;
      if (a.q_offsets[mid] <= j) lo = mid; else hi = mid - 1;
    }
    req = lo;
    q0 = a.q_offsets[req];
    nq = a.q_offsets[req + 1] - q0;
    if (j < q0 || j >= q0 + nq) return;
  } else {
    nq = static_cast<int>(a.total_q / a.m);
    req = j / nq;
    q0 = static_cast<int>(req) * nq;
  }
  const int32_t* ids = a.ids + req * a.k;
  const int cap = a.kv.ppc * a.kv.page_tokens;
  auto length = [&](int32_t c) {
    return c >= 0 && c < a.kv.n_chunks ? min(max(a.tok_len[c], 0), cap) : 0;
  };
  int ctx = 0;
  for (int r = 0; r < a.k; ++r) ctx += length(ids[r]);
  const int P = a.q_pos ? a.q_pos[j] : ctx - nq + static_cast<int>(j - q0);
  const int prefix = a.prefix_len ? a.prefix_len[req] : 0;
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  for (int i = lane; i < D; i += 64) qs[i] = bf16_to_f32(a.q[j * a.q_ts + h * a.q_hs + i]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, acc[kCols] = {};
  int base = 0;
  for (int r = 0; r < a.k; ++r) {
    const int32_t c = ids[r];
    const int len = length(c);
    const bool doc = !a.chunk_ns || (len > 0 && a.query_ns[j] >= 0 && a.chunk_ns[c] == a.query_ns[j]);
    for (int t0 = 0; doc && t0 < len; t0 += 64) {
      const int t = t0 + lane, p = base + t;
      float s = -INFINITY;
      const uint8_t* vrow = nullptr;
      const bool rule = p < prefix || ((!a.causal || p <= P) && (!a.window || static_cast<int64_t>(p) > static_cast<int64_t>(P) - a.window));
      if (t < len && rule) {
        const int32_t pg = a.kv.table[static_cast<int64_t>(c) * a.kv.ppc + t / a.kv.page_tokens];
        if (pg >= 0 && pg < a.kv.n_pages) {
          const int64_t T = a.kv.page_tokens;
          const int row = t % a.kv.page_tokens;
          const uint8_t* part = a.kv.pool + pg * a.kv.page_bytes + g * 2 * T * (kRow + kSc);
          const uint8_t* kc = part + static_cast<int64_t>(row) * kRow;
          const uint8_t* ks = part + 2 * T * kRow + row * kSc;
          vrow = kc + T * kRow;
          float dot = 0.f;
          for (int i = 0; i < D; ++i) dot += qs[i] * kv_value<FMT>(kc, ks, i);
          s = dot * a.scale;
          if (a.softcap > 0.f) s = a.softcap * tanhf(s / a.softcap);
          s -= slope * fabsf(static_cast<float>(P) - static_cast<float>(p));
        }
      }
      float top = s;
      for (int off = 32; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
      const float mn = fmaxf(m, top);
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float w = vrow ? expf(s - ref) : 0.f;
      float tot = w;
      for (int off = 32; off; off >>= 1) tot += __shfl_xor(tot, off);
      const float old = expf(m - ref);
      l = l * old + tot;
      for (int x = 0; x < kCols; ++x) acc[x] *= old;
      m = mn;
      ps[lane] = w;
      vs[lane] = vrow;
      __syncthreads();
      for (int u = 0; u < 64; ++u) {
        const uint8_t* vc = vs[u];
        if (!vc) continue;
        const int row = (t0 + u) % a.kv.page_tokens;
        const int64_t T = a.kv.page_tokens;
        const uint8_t* sc = vc + (T - row) * kRow + T * kSc + static_cast<int64_t>(row) * kSc;
        for (int x = 0; x < kCols; ++x) acc[x] += ps[u] * kv_value<FMT>(vc, sc, x * 64 + lane);
      }
      __syncthreads();
    }
    base += len;
  }
  uint16_t* out = a.out + (j * a.hq + h) * D;
  for (int x = 0; x < kCols; ++x) {
    const __bf16 o = static_cast<__bf16>(l == 0.f ? 0.f : acc[x] / l);
    out[x * 64 + lane] = __builtin_bit_cast(uint16_t, o);
  }
  if (a.lse && lane == 0) a.lse[j * a.hq + h] = l == 0.f ? -INFINITY : m + logf(l);
}

template <int FMT>
hipError_t launch_fmt(const AttendArgs& a, int d, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.total_q * a.hq));
  switch (d) {
    case 64: attend_simple_kernel<FMT, 64><<<grid, 64, 0, stream>>>(a); break;
    case 128: attend_simple_kernel<FMT, 128><<<grid, 64, 0, stream>>>(a); break;
    default: attend_simple_kernel<FMT, 256><<<grid, 64, 0, stream>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace

size_t attend_workspace_bytes(int, int64_t, int64_t, int64_t, int, int) { return 0; }

hipError_t launch_attend(const AttendArgs& a, int fmt, int d, hipStream_t stream) {
  switch (fmt) {
    case MEM_KV_BF16: return launch_fmt<MEM_KV_BF16>(a, d, stream);
    case MEM_KV_FP8: return launch_fmt<MEM_KV_FP8>(a, d, stream);
    default: return launch_fmt<MEM_KV_FP4>(a, d, stream);
  }
}

}  // namespace memattn
