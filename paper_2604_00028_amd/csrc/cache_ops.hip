// What a decode step does to its cache before it attends: block tables and
// slots from request lengths (extend_kernel), norms and rotation of q and k
// with the rows' way into the cache (append_kernel), and rows of the 4-bit
// cache read back (read_kv4_kernel).  Entry points at the end.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "decode_attn.h"
#include "host.h"
#include "kv4.h"
#include "plan.h"
#include "tile.h"

namespace {

using da::aligned;
using da::ensure_gfx950;

// ---------------------------------------------------------------- tables

constexpr int kMaxRequests = DA_MAX_REQUESTS;
constexpr int kTableThreads = 256;
static_assert(kMaxRequests == 16 * kTableThreads, "extend_kernel<16> takes them all");
constexpr uint32_t kMost = 1u << 30;  // lengths and their sums saturate here

struct TableParams {
  const int32_t* lens;
  const int32_t* new_lens;
  const int32_t* free_pages;
  const int32_t* taken;
  int32_t* block_table;
  int32_t* lens_out;
  int32_t* taken_out;
  int32_t* cu_new;     // nullable
  int32_t* slots;
  int32_t* positions;  // nullable
  int B, max_pages, page_size, num_pages, num_free, max_tokens;
  uint32_t capacity;   // keys a table row holds, at most kMost
  Div div_page;
  int state;           // write lens_out, taken_out and cu_new
  int rows;            // write table entries, slots and positions
};

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) {  // a, b <= kMost
  const uint32_t s = a + b;
  return s < kMost ? s : kMost;
}

// Saturating sum of `x` over the threads before this one; *total: over all.
// (min(a + b, most) is associative over non-negative numbers.)  One barrier:
// wave_sums is this call's own.
__device__ __forceinline__ uint32_t group_scan(uint32_t x, uint32_t* wave_sums, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto from = [&](auto ctrl, auto rows) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
  };
  using std::integral_constant;
  x = sat_add(x, from(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{}));  // row_shr:1
  x = sat_add(x, from(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{}));
  x = sat_add(x, from(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{}));
  x = sat_add(x, from(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{}));
  x = sat_add(x, from(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{}));  // row_bcast:15
  x = sat_add(x, from(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{}));  // row_bcast:31
  if (lane == 63) wave_sums[wave] = x;
  const uint32_t up = (uint32_t)__shfl_up((int)x, 1);
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kTableThreads / 64; ++w) {
    before = w < wave ? sat_add(before, wave_sums[w]) : before;
    all = sat_add(all, wave_sums[w]);
  }
  *total = all;
  return lane == 0 ? before : sat_add(before, up);
}

// The last i in [0, n) with at[i] <= x; at[0] = 0, non-decreasing.
__device__ __forceinline__ int last_at_most(const uint32_t* at, int n, uint32_t x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Request b holds l_b keys in ceil(l_b / P) pages of P rows and gets n_b more:
// its rows start at the exclusive sum of n, its pages at `taken` plus the
// exclusive sum of the pages needed, also of those by requests that the list
// could not serve: past it once, the sum stays past it, so none of the later
// ones gets a page (and places that are given have no gaps).  Every workgroup takes both sums over all
// requests for itself (PER of them a thread), so one launch needs no hand-over;
// then the workgroups share the rows, each thread looking its row's request up
// in LDS.  Bound by latency: two dependent loads, two scans, log2 B LDS reads a
// row; one row a thread (four in turn measured 9.4 us for 19600 rows of 500
// requests).
template <int PER>
__global__ void __launch_bounds__(kTableThreads) extend_kernel(TableParams p) {
  constexpr int kMaxB = PER * kTableThreads;
  __shared__ uint32_t cu[kMaxB + 1];   // first row of each request
  __shared__ uint32_t pg[kMaxB + 1];   // first place in the free list, from *taken
  __shared__ int32_t held[kMaxB];      // keys held; ~keys for a request that is not extended
  __shared__ uint32_t wave_sums[2][kTableThreads / 64];
  __shared__ uint32_t granted;         // places taken
  const int tid = threadIdx.x;
  const int b0 = tid * PER;
  if (tid == 0) granted = 0;

  const int taken_raw = *p.taken;
  uint32_t len[PER], add[PER];
  uint32_t sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    len[i] = add[i] = 0;
    if (b0 + i < p.B) {
      const int l = p.lens[b0 + i], n = p.new_lens[b0 + i];
      len[i] = l < 0 ? 0u : min((uint32_t)l, kMost);
      add[i] = n < 0 ? 0u : min((uint32_t)n, kMost);
    }
    sum = sat_add(sum, add[i]);
  }
  const uint32_t taken = taken_raw < 0 ? 0u : (uint32_t)taken_raw;
  const uint32_t avail = taken < (uint32_t)p.num_free ? (uint32_t)p.num_free - taken : 0u;
  uint32_t total;
  uint32_t at = group_scan(sum, wave_sums[0], &total);
  uint32_t need[PER];
  uint32_t pages = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    need[i] = 0;
    if (b0 + i < p.B) {
      cu[b0 + i] = at;
      at = sat_add(at, add[i]);
      const uint32_t end = len[i] + add[i];  // <= 2^31
      const bool fits = end <= p.capacity && at <= (uint32_t)p.max_tokens;
      if (fits)
        need[i] = (uint32_t)(div_by((int)(end + p.page_size - 1), p.div_page) -
                             div_by((int)(len[i] + p.page_size - 1), p.div_page));
      held[b0 + i] = fits ? (int32_t)len[i] : ~(int32_t)len[i];
      pages = sat_add(pages, need[i]);
    }
  }
  uint32_t all_pages;
  // pages asked for before (exact: at most max_tokens + B in all)
  uint32_t upto = group_scan(pages, wave_sums[1], &all_pages);
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (b0 + i < p.B) {
      upto = sat_add(upto, need[i]);
      if (need[i] > 0 && upto > avail) held[b0 + i] = ~(int32_t)len[i];
      if (need[i] > 0 && upto <= avail) most = upto;
      pg[b0 + i + 1] = upto;
    }
  }
  if (most) atomicMax(&granted, most);
  if (tid == 0) {
    cu[p.B] = total;
    pg[0] = 0;
  }
  __syncthreads();
  const uint32_t places = granted;

  if (p.state && blockIdx.x == 0) {
    for (int b = tid; b < p.B; b += kTableThreads) {
      const int32_t h = held[b];
      const uint32_t n = cu[b + 1] - cu[b];  // exact for a request that is extended
      p.lens_out[b] = h < 0 ? ~h : h + (int32_t)n;
    }
    if (tid == 0) *p.taken_out = (int32_t)(taken + places);
    if (p.cu_new)
      for (int b = tid; b <= p.B; b += kTableThreads) p.cu_new[b] = (int32_t)cu[b];
  }
  if (!p.rows) return;

  const uint32_t step = gridDim.x * kTableThreads;
  // table entries: place e of the list goes to the last request whose places start at or before e
  for (uint32_t e = blockIdx.x * kTableThreads + tid; e < places; e += step) {
    const int b = last_at_most(pg, p.B, e);
    const int page = div_by((int)((uint32_t)held[b] + p.page_size - 1), p.div_page) + (int)(e - pg[b]);
    p.block_table[(int64_t)b * p.max_pages + page] = p.free_pages[taken + e];
  }
  for (uint32_t r = blockIdx.x * kTableThreads + tid; r < (uint32_t)p.max_tokens; r += step) {
    int32_t slot = -1, pos = 0;
    if (r < total) {
      const int b = last_at_most(cu, p.B, r);
      const int32_t h = held[b];
      const uint32_t l = h < 0 ? (uint32_t)~h : (uint32_t)h;
      const uint32_t key = l + (r - cu[b]);
      pos = (int32_t)key;
      if (h >= 0) {
        const int j = div_by((int)key, p.div_page);
        const int mine = div_by((int)(l + p.page_size - 1), p.div_page);
        const int32_t page = j < mine ? p.block_table[(int64_t)b * p.max_pages + j]
                                      : p.free_pages[taken + pg[b] + (uint32_t)(j - mine)];
        if (page >= 0 && page < p.num_pages) slot = page * p.page_size + (int32_t)(key - (uint32_t)j * p.page_size);
      }
    }
    p.slots[r] = slot;
    if (p.positions) p.positions[r] = pos;
  }
}

// ---------------------------------------------------------------- append

constexpr int kAppendWaves = 4;
constexpr int kMaxAxes = DA_MAX_AXES;
static_assert(kMaxAxes == 4 && D / 2 <= 64, "the axis of a pair has two bits, the axes of all pairs four words");

struct AppendParams {
  const uint16_t* q;  // nullable
  const uint16_t* k;
  const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;  // elements between tokens
  const uint16_t* q_weight;              // nullable: that one is not normalised
  const uint16_t* k_weight;
  float eps;
  const float* rope;                     // nullable: no rotation
  int rope_rows, rope_dim, neighbours;
  const int32_t* positions;              // [num_axes, N]
  int num_axes;
  int by_four;                           // pairs 4 i to 4 i + 3 have one axis
  uint32_t axes[4];                      // axis of pair i: bits 2 (i mod 16) of word i / 16
  const int32_t* slots;
  uint16_t* q_out;
  uint16_t* k_cache;                     // bf16 rows [num_rows, H_KV, D]
  uint16_t* v_cache;
  unsigned char* cache;                  // 4-bit cache
  int64_t num_rows;
  int page_size, blocks;
  Div div_page;
  int N, H_Q, H_KV;
  int q_passes, kv_passes;               // passes of four heads
  int per_wave, segments;                // passes a wave takes, waves a token's passes take
  Div div_segments;
};

// A lane of 16 gets the value of the lane `by` further on (rotating).
template <int BY>
__device__ __forceinline__ uint32_t row_rotate(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + BY, 0xf, 0xf, false);
}

// Sum over the 16 lanes of a head, the same bits in each.
__device__ __forceinline__ float head_sum(float x) {
  x += __uint_as_float(row_rotate<8>(__float_as_uint(x)));
  x += __uint_as_float(row_rotate<4>(__float_as_uint(x)));
  x += __uint_as_float(row_rotate<2>(__float_as_uint(x)));
  x += __uint_as_float(row_rotate<1>(__float_as_uint(x)));
  return x;
}

__device__ __forceinline__ float bf16_low(uint32_t two) { return __uint_as_float(two << 16); }
__device__ __forceinline__ float bf16_high(uint32_t two) { return __uint_as_float(two & 0xffff0000u); }

// A token's head takes 16 lanes, eight dims (16 bytes) each; a wave takes four
// heads a pass, and per_wave passes of one token's q, k and v heads.  Per head
// of q and k: y = x / sqrt(mean x^2 + eps) * w, and the pair (a, b) of the
// rotation becomes (a c - b s, b c + a s); both are one product per element
// with the element itself and one with its partner, coefficients that hold for
// all heads of the token: y_i = r (x_i w_i c_i + x_j w_j (-+ s_i)).  Everything
// in 32 bits, rounded to bf16 once.  Partners of a pair of halves lie half / 8
// lanes apart, so the bf16 words change lanes, four a pass.
//
// Bound by HBM (each head row read and written once: 8192 tokens of 64/8 heads,
// 340 MB, 62.5 us a call among others, 5.4 TB/s, where a copy of 2 GiB reaches
// 4.9).  STREAM 1: rows are written with the streaming hint (more than L2 holds:
// 42 MB 11.4 -> 10.5 us in a graph); 2: read with it too (more than half the
// last-level cache: 340 MB 70.5 -> 66.9 us in a graph, but 85 MB, which a
// projection may just have left there, 16.7 -> 20.9).  KV4: keys are rounded to
// bf16 as the bf16 cache would hold them and then to 4 bits, values at once
// (quantise in kv4.h); stores of 4 bytes of codes and single bytes of scales, one
// token a wave: 3001 tokens of 8 heads 7 us, where their 16 MB would take 3.
//
// AXES: pair i of the rotation turns by the token's position on axis a(i) of up
// to four, so its coefficients come from row positions[a(i)] of the table: four
// pairs a load where four have one axis each (8192 tokens with three axes 63 us, as with one;
// a wide load for each axis and a choice by pair, which takes 20 more registers,
// 79), else one by one.
template <bool KV4, int STREAM, bool AXES>
__global__ void __launch_bounds__(64 * kAppendWaves) append_kernel(AppendParams p) {
  const int lane = threadIdx.x & 63;
  const int unit = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kAppendWaves + (int)(threadIdx.x >> 6));
  const int n = div_by(unit, p.div_segments);
  if (n >= p.N) return;
  const int passes = p.q_passes + 2 * p.kv_passes;
  int pass = (unit - n * p.segments) * p.per_wave;
  const int end = min(pass + p.per_wave, passes);
  const int l = lane & 15, group = lane >> 4;

  // ---- the token's row of the rotation table: this lane's eight cosines and signed sines
  float c[8], s[8];
  const int lanes = p.rope ? p.rope_dim / 8 : 0;  // lanes whose dims turn
  const int half = lanes / 2;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    c[e] = 1.f;
    s[e] = 0.f;
  }
  if constexpr (AXES) {
    const bool second = !p.neighbours && l >= half;  // the pairs' second dims
    const int pair0 = p.neighbours ? 4 * l : 8 * (second ? l - half : l);  // the lane's first pair
    const int word = (pair0 >> 4) & 3;
    const uint32_t mine =
        (word == 0 ? p.axes[0] : word == 1 ? p.axes[1] : word == 2 ? p.axes[2] : p.axes[3]) >> (2 * (pair0 & 15));
    const int pairs = p.neighbours ? 4 : 8;
    // the token's positions: one load for all axes, then the lane's pairs' rows of the table
    const int at = p.positions[(int64_t)min(lane & 3, p.num_axes - 1) * p.N + n];
    const int pos[kMaxAxes] = {__builtin_amdgcn_readlane(at, 0), __builtin_amdgcn_readlane(at, 1),
                               __builtin_amdgcn_readlane(at, 2), __builtin_amdgcn_readlane(at, 3)};
    auto row_of = [&](int i, bool& in) {  // of the lane's pair i; outside the table: row 0, and zeros in the end
      const uint32_t a = (mine >> (2 * i)) & 3u;
      const int r = a == 0 ? pos[0] : a == 1 ? pos[1] : a == 2 ? pos[2] : pos[3];
      in = r >= 0 && r < p.rope_rows;
      return p.rope + (int64_t)(in ? r : 0) * p.rope_dim + pair0 + i;
    };
    auto set = [&](int i, float cosine, float sine) {
      if (p.neighbours) {
        if (i >= 4) return;
        c[2 * i] = c[2 * i + 1] = cosine;
        s[2 * i] = -sine;
        s[2 * i + 1] = sine;
      } else {
        c[i] = cosine;
        s[i] = second ? sine : -sine;
      }
    };
    if (l < lanes && p.by_four) {
      f32x4 cosine[2], sine[2];
      bool in[2] = {false, false};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i == 1 && p.neighbours) break;
        const float* row = row_of(4 * i, in[i]);
        cosine[i] = *reinterpret_cast<const f32x4*>(row);
        sine[i] = *reinterpret_cast<const f32x4*>(row + p.rope_dim / 2);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < pairs) set(i, in[i / 4] ? cosine[i / 4][i % 4] : 0.f, in[i / 4] ? sine[i / 4][i % 4] : 0.f);
    } else if (l < lanes) {
      float cosine[8], sine[8];
      bool in[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i == 4 && p.neighbours) break;
        const float* row = row_of(i, in[i]);
        cosine[i] = row[0];
        sine[i] = row[p.rope_dim / 2];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < pairs) set(i, in[i] ? cosine[i] : 0.f, in[i] ? sine[i] : 0.f);
    }
  } else if (p.rope) {
    const int pos = __builtin_amdgcn_readfirstlane(p.positions[n]);
    const bool in = pos >= 0 && pos < p.rope_rows;  // a position outside the table: zeros
    const __amdgpu_buffer_rsrc_t rr =
        make_rsrc(p.rope + (int64_t)(in ? pos : 0) * p.rope_dim, in ? (uint32_t)p.rope_dim * 4u : 0u);
    if (p.neighbours) {
      // lane l turns pairs 4 l + [0, 4)
      const f32x4 cc = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, 16u * l, 0, 0));
      const f32x4 ss =
          __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, 16u * l + 2u * p.rope_dim, 0, 0));
      if (l < lanes) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          c[e] = cc[e / 2];
          s[e] = e % 2 ? ss[e / 2] : -ss[e / 2];
        }
      }
    } else {
      const uint32_t at = 32u * (uint32_t)(l < half ? l : l - half);
      f32x4 cc[2], ss[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        cc[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, at + 16u * i, 0, 0));
        ss[i] =
            __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, at + 16u * i + 2u * p.rope_dim, 0, 0));
      }
      if (l < lanes) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          c[e] = cc[e / 4][e % 4];
          s[e] = l < half ? -ss[e / 4][e % 4] : ss[e / 4][e % 4];
        }
      }
    }
  }
  const int partner = p.neighbours || l >= lanes ? l : l < half ? l + half : l - half;
  const int partner4 = 4 * ((lane & 48) + partner);

  const int64_t slot = p.slots ? (int64_t)__builtin_amdgcn_readfirstlane(p.slots[n]) : (int64_t)n;
  const bool kept = slot >= 0 && slot < p.num_rows;

  // the pass's rows: 0 q, 1 k, 2 v
  auto role_of = [&](int i) { return i < p.q_passes ? 0 : i < p.q_passes + p.kv_passes ? 1 : 2; };
  auto head_of = [&](int i, int role) {
    return 4 * (i - (role == 0 ? 0 : role == 1 ? p.q_passes : p.q_passes + p.kv_passes)) + group;
  };
  auto load = [&](int i) {
    const int role = role_of(i), h = head_of(i, role);
    const uint16_t* src = role == 0 ? p.q + n * p.q_stride : role == 1 ? p.k + n * p.k_stride : p.v + n * p.v_stride;
    u32x4 x = {0u, 0u, 0u, 0u};
    if (h < (role == 0 ? p.H_Q : p.H_KV)) {
      const u32x4* at = reinterpret_cast<const u32x4*>(src + h * D + 8 * l);
      x = STREAM == 2 ? __builtin_nontemporal_load(at) : *at;
    }
    return x;
  };

  auto store = [&](uint16_t* row, const u32x4& x) {
    u32x4* at = reinterpret_cast<u32x4*>(row + 8 * l);
    if constexpr (STREAM)
      __builtin_nontemporal_store(x, at);
    else
      *at = x;
  };

  float own[8], other[8];  // coefficients of the element and of its partner
  int set = -1;            // the role they are for
  bool norm = false;
  u32x4 x = load(pass);
  for (; pass < end; ++pass) {
    const int role = role_of(pass), h = head_of(pass, role);
    const bool live = h < (role == 0 ? p.H_Q : p.H_KV);
    u32x4 next = x;
    if (pass + 1 < end) next = load(pass + 1);
    if (role < 2) {
      if (set != role) {
        set = role;
        const uint16_t* w = role == 0 ? p.q_weight : p.k_weight;
        norm = w != nullptr;
        float wi[8], wj[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) wi[e] = wj[e] = 1.f;
        if (norm) {
          const u32x4 a = *reinterpret_cast<const u32x4*>(w + 8 * l);
          const u32x4 b = *reinterpret_cast<const u32x4*>(w + 8 * partner);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            wi[e] = e % 2 ? bf16_high(a[e / 2]) : bf16_low(a[e / 2]);
            const int f = p.neighbours ? e ^ 1 : e;
            wj[e] = f % 2 ? bf16_high(b[e / 2]) : bf16_low(b[e / 2]);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          own[e] = wi[e] * c[e];
          other[e] = wj[e] * s[e];
        }
      }
      float f[8], g[8], r = 1.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = e % 2 ? bf16_high(x[e / 2]) : bf16_low(x[e / 2]);
      if (norm) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sq = fmaf(f[e], f[e], sq);
        r = 1.0f / sqrtf(fmaf(head_sum(sq), 1.0f / D, p.eps));
      }
      if (p.neighbours) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = f[e ^ 1];
      } else {
        u32x4 y;
        if (half == 8) {
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = row_rotate<8>(x[e]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = (uint32_t)__builtin_amdgcn_ds_bpermute(partner4, (int)x[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = e % 2 ? bf16_high(y[e / 2]) : bf16_low(y[e / 2]);
      }
      // dims that do not turn have other == 0; their partner is the element itself, so an infinite one stays one
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float turned = fmaf(g[e], other[e], f[e] * own[e]);
        f[e] = r * (l < lanes ? turned : f[e] * own[e]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = pack_bf16x2(f[2 * e], f[2 * e + 1]);
    }
    if (role == 0) {
      if (live) store(p.q_out + ((int64_t)n * p.H_Q + h) * D, x);
    } else if constexpr (KV4) {
      // every lane takes part in its block's maximum
      uint32_t scale;
      const uint32_t codes = quantise(x, &scale);
      if (live && kept) {
        const int page = div_by((int)slot, p.div_page);
        const int row = (int)slot - page * p.page_size, key = row & (kKeysPerTile - 1);
        unsigned char* tile =
            p.cache + (((int64_t)page * p.H_KV + h) * p.blocks + row / kKeysPerTile) * DA_KV4_TILE_BYTES;
        *reinterpret_cast<uint32_t*>(tile + (role - 1) * kKv4V + key * 64 + 4 * l) = codes;
        if ((l & 3) == 0) tile[kv4_scale_at(key, l >> 2, role - 1)] = (unsigned char)scale;
      }
    } else if (live && kept) {
      store((role == 1 ? p.k_cache : p.v_cache) + (slot * p.H_KV + h) * D, x);
    }
    x = next;
  }
}

// Rows of the 4-bit cache as bf16 (exact): 16 lanes a head row, eight dims each.
__global__ void __launch_bounds__(256) read_kv4_kernel(const unsigned char* cache, const int32_t* slots, uint16_t* k_out,
                                                       uint16_t* v_out, int64_t items, int H_KV, Div div_heads,
                                                       int page_size, Div div_page, int64_t num_rows) {
  const int64_t item = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);  // (row, head, K or V), up to 2^27
  if (item >= items) return;
  const int l = threadIdx.x & 15;
  const int isv = (int)item & 1, rh = (int)(item >> 1);
  const int n = div_by(rh, div_heads), h = rh - n * H_KV;
  const int64_t slot = slots ? (int64_t)slots[n] : (int64_t)n;
  u32x4 y = {0u, 0u, 0u, 0u};
  if (slot >= 0 && slot < num_rows) {
    const int page = div_by((int)slot, div_page);
    const int row = (int)slot - page * page_size, key = row & (kKeysPerTile - 1);
    const unsigned char* tile =
        cache + (((int64_t)page * H_KV + h) * (page_size / kKeysPerTile) + row / kKeysPerTile) * DA_KV4_TILE_BYTES;
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(tile + isv * kKv4V + key * 64 + 4 * l);
    dequantise(codes, kv4_scale(tile[kv4_scale_at(key, l >> 2, isv)]), y);
  }
  *reinterpret_cast<u32x4*>((isv ? v_out : k_out) + (int64_t)rh * D + 8 * l) = y;
}

// ---------------------------------------------------------------- host side

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? (int)DA_OK : da::fail(DA_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

// Checks shared by the two append entry points; fills all but the cache's fields.
int append_params(AppendParams& p, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                  int64_t v_stride, const void* q_weight, const void* k_weight, float eps, const float* rope,
                  int rope_rows, int rope_dim, int neighbours, const int32_t* positions, const int32_t* slots,
                  void* q_out, int N, int H_Q, int H_KV, int d) {
  if (d != D) return da::fail(DA_ERR_UNSUPPORTED, "head dim %d unsupported (only %d)", d, D);
  if (N < 0 || H_KV <= 0 || H_Q < 0) return da::fail(DA_ERR_SHAPE, "N=%d H_Q=%d H_KV=%d", N, H_Q, H_KV);
  if (N > (1 << 24) || H_Q > (1 << 20) || H_KV > (1 << 20))
    return da::fail(DA_ERR_SHAPE, "N=%d tokens of %d + 2 x %d heads are too many for one call", N, H_Q, H_KV);
  if (N > 0 && (!k || !v)) return da::fail(DA_ERR_NULL, "k and v must be non-NULL");
  if ((q != nullptr) != (H_Q > 0) && N > 0) return da::fail(DA_ERR_NULL, "q must be given with H_Q > 0, and only then");
  if (q && !q_out) return da::fail(DA_ERR_NULL, "q_out must be non-NULL with q");
  if (rope && N > 0 && !positions) return da::fail(DA_ERR_NULL, "positions must be non-NULL with a rotation table");
  if (!(eps >= 0.f)) return da::fail(DA_ERR_ARG, "eps must not be negative");
  if (rope) {
    if (rope_dim < 16 || rope_dim > D || rope_dim % 16 != 0)
      return da::fail(DA_ERR_UNSUPPORTED, "rope_dim=%d must be a multiple of 16 up to %d", rope_dim, D);
    if (rope_rows < 1) return da::fail(DA_ERR_SHAPE, "rope_rows=%d must be positive", rope_rows);
    if (neighbours != 0 && neighbours != 1) return da::fail(DA_ERR_ARG, "neighbours=%d not in {0, 1}", neighbours);
  }
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(q_weight, 16) ||
      !aligned(k_weight, 16) || !aligned(rope, 16))
    return da::fail(DA_ERR_ALIGN, "q, k, v, q_out, the weights and the rotation table must be 16-byte aligned");
  if (!aligned(positions, 4) || !aligned(slots, 4))
    return da::fail(DA_ERR_ALIGN, "positions and slots must be 4-byte aligned");
  for (int64_t s : {q ? q_stride : 0, k_stride, v_stride})
    if (s % 8 != 0 || s < 0) return da::fail(DA_ERR_ALIGN, "token strides must be multiples of 8 elements");
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.q_weight = static_cast<const uint16_t*>(q_weight);
  p.k_weight = static_cast<const uint16_t*>(k_weight);
  p.eps = eps;
  p.rope = rope;
  p.rope_rows = rope_rows;
  p.rope_dim = rope_dim;
  p.neighbours = rope ? neighbours : 0;
  p.positions = positions;
  p.slots = slots;
  p.q_out = static_cast<uint16_t*>(q_out);
  p.N = N;
  p.H_Q = H_Q;
  p.H_KV = H_KV;
  p.q_passes = (H_Q + 3) / 4;
  p.kv_passes = (H_KV + 3) / 4;
  return DA_OK;
}

// The axis of each pair of the rotation, for the calls with positions on several.
int append_axes(AppendParams& p, const uint8_t* axes, int num_axes) {
  if (!p.rope || !axes) return da::fail(DA_ERR_NULL, "rope and axes must be non-NULL");
  if (num_axes < 1 || num_axes > kMaxAxes)
    return da::fail(DA_ERR_ARG, "num_axes=%d not in [1, %d]", num_axes, kMaxAxes);
  for (int i = 0; i < p.rope_dim / 2; ++i) {
    if (axes[i] >= num_axes) return da::fail(DA_ERR_ARG, "axes[%d]=%d of %d axes", i, axes[i], num_axes);
    p.axes[i / 16] |= (uint32_t)axes[i] << (2 * (i % 16));
  }
  p.num_axes = num_axes;
  p.by_four = 1;
  for (int i = 0; i < p.rope_dim / 2; ++i) p.by_four &= axes[i] == axes[i & ~3];
  return DA_OK;
}

template <bool KV4, bool AXES>
int launch_append(AppendParams& p, int cus, hipStream_t stream) {
  if (p.N == 0) return DA_OK;
  // A wave keeps a token's coefficients over its passes, so it takes as many as
  // leave the chip enough waves to hide the loads (16 a CU).  Where the tokens
  // are more waves than the chip holds (28 a CU), five passes a wave: the last
  // waves to start then hold the launch up less.  64/8 heads: 4096 tokens one
  // wave each 39.6 us, four 42.9; 8192 tokens 88.2 and 72.4.
  const int passes = p.q_passes + 2 * p.kv_passes;
  const int64_t waves = p.N > 28 * cus ? (passes + 4) / 5
                                       : std::min<int64_t>(passes, std::max<int64_t>(1, (16ll * cus + p.N - 1) / p.N));
  p.per_wave = (int)((passes + waves - 1) / waves);
  p.segments = (passes + p.per_wave - 1) / p.per_wave;
  if ((int64_t)p.N * p.segments > (1 << 25)) {  // a launch holds fewer than 2^26 waves
    p.per_wave = passes;
    p.segments = 1;
  }
  p.div_segments = make_div((uint32_t)p.segments);
  const int64_t units = (int64_t)p.N * p.segments;
  void* args[] = {&p};
  const void* fn;
  if constexpr (KV4) {
    fn = reinterpret_cast<const void*>(&append_kernel<true, 0, AXES>);
  } else {
    const int64_t moved = (int64_t)p.N * (p.H_Q + 2 * p.H_KV) * D * 4;
    fn = moved > (128ll << 20)       ? reinterpret_cast<const void*>(&append_kernel<false, 2, AXES>)
         : moved > da::kL2Bytes ? reinterpret_cast<const void*>(&append_kernel<false, 1, AXES>)
                                : reinterpret_cast<const void*>(&append_kernel<false, 0, AXES>);
  }
  return launched(hipLaunchKernel(fn, dim3((uint32_t)((units + kAppendWaves - 1) / kAppendWaves)),
                                  dim3(64 * kAppendWaves), args, 0, stream),
                  "append");
}

// The pages of a 4-bit cache; their rows are numbered with 32 bits.
int check_kv4_cache(const void* cache, int page_size, int num_pages, int H_KV) {
  if (!cache && num_pages > 0) return da::fail(DA_ERR_NULL, "cache must be non-NULL");
  if (!aligned(cache, 16)) return da::fail(DA_ERR_ALIGN, "cache must be 16-byte aligned");
  if (page_size < kKeysPerTile || page_size % kKeysPerTile != 0 || page_size > (1 << 20))
    return da::fail(DA_ERR_UNSUPPORTED, "page_size=%d must be a multiple of %d (at most 2^20)", page_size, kKeysPerTile);
  if (num_pages < 0 || H_KV <= 0 || (int64_t)num_pages * page_size >= ((int64_t)1 << 31))
    return da::fail(DA_ERR_SHAPE, "num_pages=%d pages of %d rows (H_KV=%d)", num_pages, page_size, H_KV);
  return DA_OK;
}

// The rest of an append call: the cache's checks and the launch.
template <bool AXES>
int append_rows(AppendParams& p, void* k_cache, void* v_cache, int64_t num_rows, void* stream) {
  if (num_rows < 0) return da::fail(DA_ERR_SHAPE, "num_rows=%lld is negative", (long long)num_rows);
  if (num_rows > 0 && (!k_cache || !v_cache)) return da::fail(DA_ERR_NULL, "k_cache and v_cache must be non-NULL");
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16))
    return da::fail(DA_ERR_ALIGN, "k_cache and v_cache must be 16-byte aligned");
  int cus = 0;
  const int rc = ensure_gfx950(&cus);
  if (rc) return rc;
  p.k_cache = static_cast<uint16_t*>(k_cache);
  p.v_cache = static_cast<uint16_t*>(v_cache);
  p.num_rows = num_rows;
  return launch_append<false, AXES>(p, cus, static_cast<hipStream_t>(stream));
}

template <bool AXES>
int append_rows4(AppendParams& p, void* cache, int page_size, int num_pages, void* stream) {
  int rc = check_kv4_cache(cache, page_size, num_pages, p.H_KV);
  if (rc) return rc;
  int cus = 0;
  rc = ensure_gfx950(&cus);
  if (rc) return rc;
  p.cache = static_cast<unsigned char*>(cache);
  p.page_size = page_size;
  p.blocks = page_size / kKeysPerTile;
  p.div_page = make_div((uint32_t)page_size);
  p.num_rows = (int64_t)num_pages * page_size;
  return launch_append<true, AXES>(p, cus, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

int da_extend_tables(const int32_t* lens, const int32_t* new_lens, const int32_t* free_pages, const int32_t* taken,
                     int32_t* block_table, int32_t* lens_out, int32_t* taken_out, int32_t* cu_new, int32_t* slots,
                     int32_t* positions, int B, int page_size, int max_pages, int num_pages, int num_free,
                     int max_tokens, void* stream) {
  da::clear_error();
  if (B <= 0 || B > kMaxRequests) return da::fail(DA_ERR_SHAPE, "B=%d must be in [1, %d]", B, kMaxRequests);
  if (page_size < 1 || page_size > (1 << 20))
    return da::fail(DA_ERR_SHAPE, "page_size=%d must be in [1, 2^20]", page_size);
  if (max_pages < 1 || num_pages < 0 || num_free < 0 || num_free >= (1 << 30) || max_tokens < 0 ||
      max_tokens > (1 << 28))
    return da::fail(DA_ERR_SHAPE, "max_pages=%d num_pages=%d num_free=%d max_tokens=%d", max_pages, num_pages, num_free,
                    max_tokens);
  if ((int64_t)num_pages * page_size >= ((int64_t)1 << 31))
    return da::fail(DA_ERR_SHAPE, "num_pages=%d pages of %d rows: slots have 32 bits", num_pages, page_size);
  if (!lens || !new_lens || !taken || !block_table || !lens_out || !taken_out || (!free_pages && num_free > 0) ||
      (!slots && max_tokens > 0))
    return da::fail(DA_ERR_NULL, "lens, new_lens, free_pages, taken, block_table, lens_out, taken_out and slots must "
                                 "be non-NULL");
  for (const void* q : {(const void*)lens, (const void*)new_lens, (const void*)free_pages, (const void*)taken,
                        (const void*)block_table, (const void*)lens_out, (const void*)taken_out, (const void*)cu_new,
                        (const void*)slots, (const void*)positions})
    if (!aligned(q, 4)) return da::fail(DA_ERR_ALIGN, "tables and lengths must be 4-byte aligned");
  int cus = 0;
  int rc = ensure_gfx950(&cus);
  if (rc) return rc;
  TableParams p{lens,      new_lens, free_pages, taken,     block_table, lens_out, taken_out,
                cu_new,    slots,    positions,  B,         max_pages,   page_size, num_pages,
                num_free,  max_tokens, (uint32_t)std::min<int64_t>(kMost, (int64_t)max_pages * page_size),
                make_div((uint32_t)page_size), 1, 1};
  // Where several workgroups read the lengths, outputs that take their place are
  // written by a launch after them; one workgroup for up to eight rows a thread is
  // faster than that launch.
  const bool in_place = lens_out == lens || lens_out == new_lens || taken_out == taken;
  const int groups = std::min(std::max(1, (max_tokens + kTableThreads - 1) / kTableThreads), 8 * cus);
  const int grid = in_place && groups <= 8 ? 1 : groups;
  const bool later = grid > 1 && in_place;
  p.state = later ? 0 : 1;
  void* args[] = {&p};
  const void* fn = B <= kTableThreads       ? reinterpret_cast<const void*>(&extend_kernel<1>)
                   : B <= 4 * kTableThreads ? reinterpret_cast<const void*>(&extend_kernel<4>)
                                            : reinterpret_cast<const void*>(&extend_kernel<16>);
  rc = launched(hipLaunchKernel(fn, dim3(grid), dim3(kTableThreads), args, 0, static_cast<hipStream_t>(stream)),
                "table");
  if (rc || !later) return rc;
  p.state = 1;
  p.rows = 0;
  return launched(hipLaunchKernel(fn, dim3(1), dim3(kTableThreads), args, 0, static_cast<hipStream_t>(stream)), "table");
}

int da_append_kv(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                 const void* q_weight, const void* k_weight, float eps, const float* rope, int rope_rows, int rope_dim,
                 int neighbours, const int32_t* positions, const int32_t* slots, void* q_out, void* k_cache,
                 void* v_cache, int64_t num_rows, int N, int H_Q, int H_KV, int d, void* stream) {
  da::clear_error();
  AppendParams p{};
  int rc = append_params(p, q, q_stride, k, k_stride, v, v_stride, q_weight, k_weight, eps, rope, rope_rows, rope_dim,
                         neighbours, positions, slots, q_out, N, H_Q, H_KV, d);
  return rc ? rc : append_rows<false>(p, k_cache, v_cache, num_rows, stream);
}

int da_append_kv4(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                  const void* q_weight, const void* k_weight, float eps, const float* rope, int rope_rows, int rope_dim,
                  int neighbours, const int32_t* positions, const int32_t* slots, void* q_out, void* cache,
                  int page_size, int num_pages, int N, int H_Q, int H_KV, int d, void* stream) {
  da::clear_error();
  AppendParams p{};
  int rc = append_params(p, q, q_stride, k, k_stride, v, v_stride, q_weight, k_weight, eps, rope, rope_rows, rope_dim,
                         neighbours, positions, slots, q_out, N, H_Q, H_KV, d);
  return rc ? rc : append_rows4<false>(p, cache, page_size, num_pages, stream);
}

int da_append_kv_axes(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                      const void* q_weight, const void* k_weight, float eps, const float* rope, int rope_rows,
                      int rope_dim, int neighbours, const uint8_t* axes, int num_axes, const int32_t* positions,
                      const int32_t* slots, void* q_out, void* k_cache, void* v_cache, int64_t num_rows, int N, int H_Q,
                      int H_KV, int d, void* stream) {
  da::clear_error();
  AppendParams p{};
  int rc = append_params(p, q, q_stride, k, k_stride, v, v_stride, q_weight, k_weight, eps, rope, rope_rows, rope_dim,
                         neighbours, positions, slots, q_out, N, H_Q, H_KV, d);
  if (!rc) rc = append_axes(p, axes, num_axes);
  return rc ? rc : append_rows<true>(p, k_cache, v_cache, num_rows, stream);
}

int da_append_kv4_axes(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                       int64_t v_stride, const void* q_weight, const void* k_weight, float eps, const float* rope,
                       int rope_rows, int rope_dim, int neighbours, const uint8_t* axes, int num_axes,
                       const int32_t* positions, const int32_t* slots, void* q_out, void* cache, int page_size,
                       int num_pages, int N, int H_Q, int H_KV, int d, void* stream) {
  da::clear_error();
  AppendParams p{};
  int rc = append_params(p, q, q_stride, k, k_stride, v, v_stride, q_weight, k_weight, eps, rope, rope_rows, rope_dim,
                         neighbours, positions, slots, q_out, N, H_Q, H_KV, d);
  if (!rc) rc = append_axes(p, axes, num_axes);
  return rc ? rc : append_rows4<true>(p, cache, page_size, num_pages, stream);
}

int da_read_kv4(const void* cache, const int32_t* slots, void* k_out, void* v_out, int N, int H_KV, int page_size,
                int num_pages, int d, void* stream) {
  da::clear_error();
  if (d != D) return da::fail(DA_ERR_UNSUPPORTED, "head dim %d unsupported (only %d)", d, D);
  int rc = check_kv4_cache(cache, page_size, num_pages, H_KV);
  if (rc) return rc;
  const int64_t items = (int64_t)N * H_KV * 2;
  if (N < 0 || items > ((int64_t)1 << 27)) return da::fail(DA_ERR_SHAPE, "N=%d rows of %d heads", N, H_KV);
  if (N > 0 && (!k_out || !v_out)) return da::fail(DA_ERR_NULL, "k_out and v_out must be non-NULL");
  if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(slots, 4))
    return da::fail(DA_ERR_ALIGN, "k_out and v_out must be 16-byte, slots 4-byte aligned");
  int cus = 0;
  rc = ensure_gfx950(&cus);
  if (rc || N == 0) return rc;
  const unsigned char* c = static_cast<const unsigned char*>(cache);
  uint16_t* ko = static_cast<uint16_t*>(k_out);
  uint16_t* vo = static_cast<uint16_t*>(v_out);
  int64_t count = items, num_rows = (int64_t)num_pages * page_size;
  Div div_heads = make_div((uint32_t)H_KV), div_page = make_div((uint32_t)page_size);
  void* args[] = {&c, &slots, &ko, &vo, &count, &H_KV, &div_heads, &page_size, &div_page, &num_rows};
  return launched(hipLaunchKernel(reinterpret_cast<const void*>(&read_kv4_kernel), dim3((uint32_t)((items + 15) / 16)),
                                  dim3(256), args, 0, static_cast<hipStream_t>(stream)),
                  "4-bit read");
}

}  // extern "C"
