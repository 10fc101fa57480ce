// Latent attention as the kernels see it.  Internal to the library: the public
// interface is include/memattn_latent.h.
#pragma once

#include "kv.h"
#include "memattn_latent.h"

namespace memattn {

struct LatentArgs {
  AttendArgs a;        // requests and masks; kv.heads = 1, hq = heads
  RowsView q, t;       // queries and their rotated parts, bf16
  const uint16_t* w;
  int64_t w_hs, w_rs;  // strides of its heads and rows, in elements
  uint16_t* out;       // [total_q, heads, head_dim]
  void* ws;
};

// What a call takes (form: MEM_LATENT_ABSORBED or MEM_LATENT_EXPANDED once it is chosen).
struct LatentSizes {
  int fmt, latent, head_dim;
  int64_t m;
  int k;
  int64_t units;  // blocks of 32 tokens that a request's chunks can hold
  int64_t total_q;
  int heads;
};

mem_latent_form choose_latent_form(const LatentSizes& s, int32_t asked);
size_t latent_workspace_bytes(const LatentSizes& s, mem_latent_form form);
// Whether the call's workgroups fit its launches.
bool latent_fits(const LatentSizes& s, mem_latent_form form, bool ragged);
hipError_t launch_latent_attend(const LatentArgs& x, const LatentSizes& s, mem_latent_form form, hipStream_t stream);

// The expanded form's.
size_t expanded_workspace_bytes(const LatentSizes& s, bool ragged);
bool expanded_fits(const LatentSizes& s, bool ragged);
hipError_t launch_expanded(const LatentArgs& x, const LatentSizes& s, hipStream_t stream);

}  // namespace memattn
