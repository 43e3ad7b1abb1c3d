// Host side shared by the entry points of several sources: the device check,
// pointer alignment, the paged layout's checks and the kernel arguments.
// Defined in decode_attn.hip.
#pragma once

#include <stdint.h>

#include "decode_attn.h"
#include "plan.h"
#include "tile.h"

namespace da {

constexpr int kMaxDevices = 64;

inline bool aligned(const void* ptr, uintptr_t a) { return ((uintptr_t)ptr & (a - 1)) == 0; }

// DA_OK and the current device's CU count, or an error unless it is a gfx950.
int ensure_gfx950(int* cus);

// A block table of [B, max_pages] pages for sequences of up to L_K_max keys.
int check_page_table(int B, int page_size, int max_pages, int num_pages, int L_K_max);

}  // namespace da

namespace {

// Shape and plan fields of the kernel arguments (the K/V layout fields are
// set by the caller).
inline void fill_params(Params& p, int B, int H_Q, int H_KV, int L_K_max, float scale, const da_plan& pl) {
  p.B = B;
  p.H_Q = H_Q;
  p.H_KV = H_KV;
  p.L_K = L_K_max;
  p.g = H_Q / H_KV;
  p.hpt = pl.heads_per_tile;
  p.tiles_per_seq = H_Q / pl.heads_per_tile;
  p.tiles = pl.tiles;
  p.s = pl.num_splits;
  p.div_s = make_div((uint32_t)p.s);
  p.div_tps = make_div((uint32_t)p.tiles_per_seq);
  p.div_g = make_div((uint32_t)p.g);
  p.xcd_group = pl.heads_per_tile < p.g ? 1 : 0;  // several workgroups read each KV head
  const float sigma = scale > 0.f ? scale : 1.0f / sqrtf((float)D);
  p.scale_log2 = sigma * kLog2e;
}

}  // namespace
