// Device code shared by the decode-attention kernels: the 32-key tile
// reduction on the matrix cores (scores, online softmax, P.V), the merge of a
// workgroup's wave states, the log-sum-exp merges of chunk states, and the
// launch parameters.  What each kernel does with them stands beside the kernel
// (decode_attn.hip, kv4.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "decode_attn.h"
#include "plan.h"

namespace {

constexpr int D = DA_HEAD_DIM;
constexpr int kKeysPerTile = 32;
constexpr int kVPitch = 288;                 // bytes per staged V row (256 + 32 pad)
constexpr int kKPitch = 288;                 // bytes per staged K row (256 + 32 pad)
constexpr int kDeviceScope = 16;             // cache-policy field: sc1, device-scope coherent access
constexpr int kStateVals = 2 + 32;           // one wave's state per lane: m, l, 8 x 4 outputs

// How a tile's K and V reach the matrix cores.
enum Fetch : int {
  kFetchDirect = 0,  // K straight into the MFMA operand layout; V via registers to LDS
  kFetchStaged = 1,  // K and V row-contiguous into registers, then through LDS
  kFetchLds = 2,     // K and V row-contiguous straight into LDS (buffer_load ... lds), two stages
};

// Direct-to-LDS tiles: an instruction writes 64 lanes x 16 bytes = 4 rows
// contiguously, so a 32-key tile is 8 such blocks.  Blocks sit kBlockStride
// bytes apart and within a block the 16-byte chunks of row r are rotated
// by 2r positions, which places every chunk on the LDS banks a 288-byte row
// pitch would (the pitch the register-staged path uses): the operand reads
// below then measure no bank conflicts.
constexpr int kBlockStride = 4 * 288;
constexpr int kLdsTileBytes = 8 * kBlockStride;                 // one K or V tile
constexpr int kLdsStageBytes = 2 * kLdsTileBytes;                // K and V of one tile

// LDS of one workgroup of W waves with NT head tiles: the per-wave stages,
// reused after the tile loop for the wave-state merge (W slots, one wave
// state of NT x kStateVals x 64 floats each).
constexpr int merge_slot_bytes(int NT) { return NT * kStateVals * 64 * 4; }  // V slices use less
constexpr int stage_bytes(int FETCH) {
  return FETCH == kFetchLds ? 2 * kLdsStageBytes
                            : kKeysPerTile * (kVPitch + (FETCH == kFetchStaged ? kKPitch : 0));
}
constexpr int smem_bytes(int W, int NT, int FETCH) {
  return W * stage_bytes(FETCH) > W * merge_slot_bytes(NT) ? W * stage_bytes(FETCH) : W * merge_slot_bytes(NT);
}
static_assert(smem_bytes(4, 2, kFetchLds) <= 160 * 1024, "a workgroup must fit the LDS of one CU");
static_assert(smem_bytes(4, 1, kFetchDirect) >= (2 * (DA_MAX_SPLITS + 16) * 32 + 8 * 32) * 4,
              "the single-launch merge stages chunk maxima and sums in LDS");

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;

// kDirect: one chunk per sequence, the normalised output is written.
// kPartials: chunk states go to the workspace for a separate combine launch.
// kFused: chunk states go to the workspace with device-scope stores, and
// the last workgroup of a tile to finish merges them (single launch).
enum Mode : int { kDirect = 0, kPartials = 1, kFused = 2 };

// Division by a launch constant d >= 1 as a multiply and a shift
// (Granlund and Montgomery, PLDI 1994, Theorem 4.2 with N = 32): with
// l = ceil(log2 d) and m = ceil(2^(32+l) / d) - 2^32, x / d = (x +
// mulhi(x, m)) >> l for every x < 2^32; for x < 2^31, the only numerators
// here, the sum does not overflow.  The host computes (m, l) once per launch.
struct Div {
  uint32_t m, l;
};

inline Div make_div(uint32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  return Div{(uint32_t)((((1ull << (32 + l)) + d - 1) / d) - (1ull << 32)), l};
}

__device__ __forceinline__ int div_by(int x, Div d) {
  return (int)(((uint32_t)x + __umulhi((uint32_t)x, d.m)) >> d.l);
}

struct Params {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* cu;    // nullable: fixed layout
  uint16_t* out;        // bf16 [B, H_Q, D]        (kDirect)
  float* lse;           // nullable, [B, H_Q]      (kDirect)
  float* o_part;        // [s, B, H_Q, D]          (kPartials)
  float* m_part;        // [s, B, H_Q]
  float* l_part;        // [s, B, H_Q]
  uint32_t* arrivals;   // kFused: one arrival counter per tile, zero between calls
  const int32_t* block_table;  // paged layout: [B, max_pages] page ids
  const int32_t* seq_lens;     // paged layout: [B] sequence lengths
  int page_size, max_pages, num_pages;
  Div div_page;         // page_size
  const int32_t* work;  // nullable: per-sequence schedule, int32x4 {tile, first, end, state row} per workgroup
  const int32_t* seqs;  // schedule, kFused: int32x2 [B] {first chunk-state row or -1, chunk count}
  int state_rows;       // chunk-state rows of the schedule
  int B, H_Q, H_KV, L_K, g, hpt, tiles_per_seq, tiles, s, mode;
  int xcd_group;        // 1: consecutive tiles share an XCD (packing off)
  Div div_s, div_tps, div_g;  // s, tiles_per_seq, g
  float scale_log2;     // softmax scale * log2(e)
  int groups;           // dealt launch: workgroups per head tile
  int window, sinks;    // windowed launch: keys visible at the end and at the start (window 0: all keys)
};

// A sequence's visible keys under a sliding window of `window` keys that ends
// with the sequence, and `sinks` first keys that stay visible: key j where j <
// sinks or j >= from.  The tiles of 32 keys that hold none lie between them;
// without those, position i (whole tiles kept) is key i before `jump` and key i
// + skip from there on.
struct Window {
  int sinks, from, jump, skip;
  __device__ __forceinline__ int key(int i) const { return i + (i >= jump ? skip : 0); }
  // Whether row `row` of the tile that starts at key `first` is invisible.
  __device__ __forceinline__ bool hides(int first, int row) const {
    return (uint32_t)(first + row - sinks) < (uint32_t)(from - sinks);
  }
  // Whether some row of that tile is.
  __device__ __forceinline__ bool cuts(int first) const {
    return from > sinks && first < from && first + kKeysPerTile > sinks;
  }
};

__device__ __forceinline__ Window window_of(int L, int window, int sinks) {
  Window w;
  w.sinks = sinks < L ? sinks : L;
  w.from = window < L ? L - window : 0;
  w.from = w.from > w.sinks ? w.from : w.sinks;  // nothing hidden
  const int ts = (w.sinks + kKeysPerTile - 1) / kKeysPerTile, tw = w.from / kKeysPerTile;
  w.jump = ts * kKeysPerTile;
  w.skip = tw > ts ? (tw - ts) * kKeysPerTile : 0;
  return w;
}

// Max and sum over lanes {l, l^16, l^32, l^48}: the 4 row groups of one MFMA
// column.  permlane16_swap(x, x) hands every lane the pair (x[l], x[l^16])
// and permlane32_swap(x, x) the pair (x[l], x[l^32]), in the same order on
// both lanes of a pair, so every lane of a column ends with identical bits.
__device__ __forceinline__ float max_rows(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto c = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(c[0]), __uint_as_float(c[1]));
}

__device__ __forceinline__ float sum_rows(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto c = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(c[0]) + __uint_as_float(c[1]);
}

// Two floats to bf16 (round to nearest even), packed low/high in one dword:
// a single v_cvt_pk_bf16_f32.
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 x) { return __builtin_bit_cast(bf16x8, x); }

// Byte offset of a shared-memory pointer within the workgroup's LDS.
__device__ __forceinline__ uint32_t lds_offset(const void* ptr) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)ptr;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)bytes, 0x00020000);
}

// Maximum over the 64 lanes of a wave (exact: the order does not matter).
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

// Inclusive prefix sum and maximum over the 64 lanes of a wave (DPP row
// shifts, then row broadcasts), for non-negative values.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return x;
}

__device__ __forceinline__ int wave_top(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}

__device__ __forceinline__ float lane_value(float x, int i) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), i));
}

// Whether a chunk of probability sum `l` holds a key.  NANS: a sum that is NaN (a
// key or a query that is not finite) counts too, so that the NaN reaches the
// output and the log-sum-exp instead of leaving its chunk out.
template <bool NANS>
__device__ __forceinline__ bool holds(float l) {
  return NANS ? !(l == 0.f) : l > 0.f;
}

// The log-sum-exp merge of s <= 64 chunk states (the paper's final
// reduction, Sections 3.1 and 5.3) for up to NR rows, by one wave: the lane
// holds output dims 2*lane and 2*lane + 1 of each row, and lane i holds the
// max and sum of chunk i.  Chunk i of row r is state row base[r] + i * srow
// (Otilde at o_part[row * D], m and l at m_part[row], l_part[row]).  Per
// row: M = max m_i over chunks with l_i > 0, w_i = exp(m_i - M) (0 for an
// empty chunk), then L = sum_i w_i l_i and O = sum_i w_i Otilde_i, both
// accumulated in chunk order i = 0..s-1, O / L rounded to bf16 and lse = M +
// ln L.  Every output element takes the same operations in the same order
// whichever kernel runs this, so the separate combine launch and the
// single-launch merge give the same bits.  COH: the states were written in
// this launch by other workgroups with device-scope stores and are read with
// device-scope loads.  State offsets are below 2 GiB (checked on the host).
template <int NR, bool COH, bool NANS = false>
__device__ __forceinline__ void merge_rows(const float* o_part, const float* m_part, const float* l_part,
                                           const int64_t (&base)[NR], const int64_t (&orow)[NR], int nr,
                                           int64_t srow, int s, uint16_t* out, float* lse, int lane) {
  constexpr int aux = COH ? kDeviceScope : 0;
  constexpr int CB = NR == 1 ? 16 : (32 / NR > 0 ? 32 / NR : 1);  // chunks loaded at once per row
  const __amdgpu_buffer_rsrc_t ors = make_rsrc(o_part, 0x7fffffff);
  const __amdgpu_buffer_rsrc_t mrs = make_rsrc(m_part, 0x7fffffff);
  const __amdgpu_buffer_rsrc_t lrs = make_rsrc(l_part, 0x7fffffff);
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  float mi[NR], li[NR];
  f32x2 a[NR][CB];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    mi[r] = -INFINITY;
    li[r] = 0.f;
    if (r < nr && lane < s) {
      const uint32_t off = (uint32_t)(base[r] + (int64_t)lane * srow) * 4u;
      mi[r] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(mrs, off, 0, aux));
      li[r] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(lrs, off, 0, aux));
    }
#pragma unroll
    for (int u = 0; u < CB; ++u)
      if (r < nr && u < s)
        a[r][u] = __builtin_bit_cast(
            f32x2, __builtin_amdgcn_raw_buffer_load_b64(
                       ors, (uint32_t)((base[r] + (int64_t)u * srow) * D + 2 * lane) * 4u, 0, aux));
  }
  float wi[NR], M[NR], L[NR], o0[NR], o1[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const bool live = holds<NANS>(li[r]);
    M[r] = wave_max(live ? mi[r] : -INFINITY);
    wi[r] = live ? __builtin_amdgcn_exp2f((mi[r] - M[r]) * kLog2e) : 0.f;
    L[r] = 0.f;
    for (int i = 0; i < s; ++i) L[r] = fmaf(lane_value(wi[r], i), lane_value(li[r], i), L[r]);
    o0[r] = 0.f;
    o1[r] = 0.f;
  }
  for (int i0 = 0; i0 < s; i0 += CB) {
    if (i0 > 0) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int u = 0; u < CB; ++u)
          if (r < nr && i0 + u < s)
            a[r][u] = __builtin_bit_cast(
                f32x2, __builtin_amdgcn_raw_buffer_load_b64(
                           ors, (uint32_t)((base[r] + (int64_t)(i0 + u) * srow) * D + 2 * lane) * 4u, 0, aux));
    }
#pragma unroll
    for (int u = 0; u < CB; ++u)
      if (i0 + u < s) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          const float w = lane_value(wi[r], i0 + u);
          const bool live = holds<NANS>(lane_value(li[r], i0 + u));
          o0[r] = fmaf(w, live ? a[r][u].x : 0.f, o0[r]);
          o1[r] = fmaf(w, live ? a[r][u].y : 0.f, o1[r]);
        }
      }
  }
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    if (r >= nr) continue;
    const float inv = L[r] > 0.f ? 1.0f / L[r] : 0.f;
    *reinterpret_cast<uint32_t*>(out + orow[r] * D + 2 * lane) = pack_bf16x2(o0[r] * inv, o1[r] * inv);
    if (lse && lane == 0) lse[orow[r]] = holds<NANS>(L[r]) ? M[r] + logf(L[r]) : -INFINITY;
  }
}

// The single-launch merge: the last workgroup of a tile merges the tile's
// s chunk states for its hpt <= 32 rows (query heads), with every thread
// holding J float4 output columns, CB chunks of each at once: column item tid + T j is row item / 32,
// float4 column item % 32.  Chunk i of the tile's head h is state row srow0 +
// i * cstride + h; with FIRST, chunk 0 sits first_rows further on.  Its output
// row is orow0 + h.  The states were written in this launch by other
// workgroups with device-scope stores and are read with device-scope loads.
// Per output element the operations and their order are those of merge_rows
// (maximum over non-empty chunks, then the weights, L and O accumulated in
// chunk order), so both merges give the same bits.
//
// Bound by latency: one trip to memory for up to CB chunks (all loads in
// flight at once), and the code's own fetch, since it runs once per launch on
// cold instruction caches.  So the loads carry no per-lane guard: the buffer
// ranges start at the tile's first state row and end with chunk s - 1, what is
// read past either is never used, and rows past hpt read other heads' states,
// which are not stored.  s <= CB merges in registers; more chunks stage their
// maxima and sums in `lds` (at least 2 x (64 + 16) x 32 + 8 x 32 floats) and
// take the columns in batches of CB.
template <int W, int J, int CB, bool FIRST, bool NANS>
__device__ __forceinline__ void merge_columns(const Params& p, float* lds, int64_t srow0, int64_t cstride, int s,
                                              int64_t orow0, int tid, uint32_t first_rows) {
  constexpr int T = 64 * W;    // threads
  constexpr int R = T / 32;    // thread t stages row t % 32 of chunks t / 32 + R u
  const int hpt = p.hpt;
  // 32-bit offsets: the chunk states of a call stay below 2 GiB (checked on the host)
  const uint32_t rows = (uint32_t)cstride;  // state rows between two chunks of one head
  const uint32_t span = (uint32_t)(s - 1) * rows + (uint32_t)hpt + (FIRST && s == 1 ? first_rows : 0u);
  const __amdgpu_buffer_rsrc_t mrs = make_rsrc(p.m_part + srow0, span * 4u);
  const __amdgpu_buffer_rsrc_t lrs = make_rsrc(p.l_part + srow0, span * 4u);
  const __amdgpu_buffer_rsrc_t ors = make_rsrc(p.o_part + srow0 * D, span * (uint32_t)D * 4u);
  auto chunk_row = [&](int i) { return (uint32_t)i * rows + (FIRST && i == 0 ? first_rows : 0u); };
  auto load_cols = [&](f32x4 (&a)[J][CB], int i0) {
#pragma unroll
    for (int u = 0; u < CB; ++u)
#pragma unroll
      for (int j = 0; j < J; ++j)
        a[j][u] = __builtin_bit_cast(
            f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       ors, (uint32_t)(tid + T * j) * 16u + chunk_row(i0 + u) * (uint32_t)D * 4u, 0, kDeviceScope));
  };
  auto store_item = [&](int j, float M, float L, const f32x4& o) {
    const int item = tid + T * j, h = item >> 5, c = item & 31;
    if (h >= hpt) return;
    const int64_t row = orow0 + h;
    const float inv = L > 0.f ? 1.0f / L : 0.f;
    *reinterpret_cast<uint2*>(p.out + row * D + 4 * c) =
        make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    if (p.lse && c == 0) p.lse[row] = holds<NANS>(L) ? M + logf(L) : -INFINITY;
  };
  float M[J], L[J];
  f32x4 o[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    M[j] = -INFINITY;
    L[j] = 0.f;
    o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // chunks [i0, min(i0 + CB, s)) with maxima bm and sums bl
  auto add = [&](const f32x4 (&a)[J][CB], const float (&bm)[J][CB], const float (&bl)[J][CB], int i0) {
#pragma unroll
    for (int u = 0; u < CB; ++u) {
      if (i0 + u < s) {  // uniform
#pragma unroll
        for (int j = 0; j < J; ++j) {
          // an empty chunk's output is exactly zero here (w = 0 and O~ = 0 add nothing), as the
          // combine's guard on empty chunks makes it
          const float w = holds<NANS>(bl[j][u]) ? __builtin_amdgcn_exp2f((bm[j][u] - M[j]) * kLog2e) : 0.f;
          L[j] = fmaf(w, bl[j][u], L[j]);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[j][e] = fmaf(w, a[j][u][e], o[j][e]);
        }
      }
    }
  };
  f32x4 a[J][CB];
  float bm[J][CB], bl[J][CB];
  if (s <= CB) {
    // one batch: every thread loads its own rows' maxima and sums with its columns
#pragma unroll
    for (int u = 0; u < CB; ++u)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t off = ((uint32_t)((tid + T * j) >> 5) + chunk_row(u)) * 4u;
        bm[j][u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(mrs, off, 0, kDeviceScope));
        bl[j][u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(lrs, off, 0, kDeviceScope));
      }
    load_cols(a, 0);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int u = 0; u < CB; ++u) M[j] = u < s && holds<NANS>(bl[j][u]) ? fmaxf(M[j], bm[j][u]) : M[j];
    add(a, bm, bl, 0);
  } else {
    // chunk rows are padded to 64 + CB so that a batch reads them unconditionally
    float* lm = lds;                               // [64 + CB chunks][32 rows] maxima
    float* ll = lds + (DA_MAX_SPLITS + CB) * 32;   // [64 + CB][32] sums
    float* lp = ll + (DA_MAX_SPLITS + CB) * 32;    // [R][32] maxima over each thread's live chunks
    {
      const uint32_t h = (uint32_t)tid & 31u;
      const int i0 = tid >> 5;
      float mv[DA_MAX_SPLITS / R], lv[DA_MAX_SPLITS / R];
#pragma unroll
      for (int u = 0; u < DA_MAX_SPLITS / R; ++u) {
        if (R * u >= s) break;  // uniform
        const uint32_t off = (chunk_row(i0 + R * u) + h) * 4u;
        mv[u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(mrs, off, 0, kDeviceScope));
        lv[u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(lrs, off, 0, kDeviceScope));
      }
      load_cols(a, 0);  // in flight while the maxima are staged
      float pm = -INFINITY;
#pragma unroll
      for (int u = 0; u < DA_MAX_SPLITS / R; ++u) {
        if (R * u >= s) break;
        const int i = i0 + R * u;  // < 64; rows past s are never used
        lm[i * 32 + h] = mv[u];
        ll[i * 32 + h] = lv[u];
        pm = i < s && holds<NANS>(lv[u]) ? fmaxf(pm, mv[u]) : pm;
      }
      lp[i0 * 32 + h] = pm;
    }
    __syncthreads();
    int hh[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      hh[j] = ((tid + T * j) >> 5) & 31;
#pragma unroll
      for (int r = 0; r < R; ++r) M[j] = fmaxf(M[j], lp[r * 32 + hh[j]]);
    }
    for (int i0 = 0; i0 < s; i0 += CB) {
      if (i0 > 0) load_cols(a, i0);
      // the batch's maxima and sums, read at once (rows past s are read, never used)
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int u = 0; u < CB; ++u) {
          bm[j][u] = lm[(i0 + u) * 32 + hh[j]];
          bl[j][u] = ll[(i0 + u) * 32 + hh[j]];
        }
      add(a, bm, bl, i0);
    }
  }
#pragma unroll
  for (int j = 0; j < J; ++j) store_item(j, M[j], L[j], o[j]);
}

// merge_columns by the rows and chunks in use.
template <int NT, int W, bool FIRST = false, bool NANS = false>
__device__ __forceinline__ void merge_tile(const Params& p, float* lds, int64_t srow0, int64_t cstride, int s,
                                           int64_t orow0, int tid, uint32_t first_rows = 0) {
  constexpr int T = 64 * W;              // threads
  constexpr int R = T / 32;              // rows that the threads' first float4 columns cover
  constexpr int IPT = NT * 16 / R;       // float4 columns per thread where all NT x 16 rows are in use
  constexpr int CB = da::kFusedBatch[NT - 1];
  // Up to R rows need one column item per thread, which leaves registers for
  // 16 chunks at once: B=1, H_KV=8, L_K=8192 in 16 chunks 12.0 -> 11.4 us per
  // call against batches of 8.  Loads past the last chunk still take their
  // turn and their code (4 chunks in a batch of 16: 8% of the step of 80 layers
  // at L_K=512), so few chunks take a small batch, and more than 16, whose
  // batches follow each other, the middle one.  2-4 chunks of 9 to 16 heads in
  // a batch of 8 ran at 0.96-0.98x of a loop over the chunks there are, in a
  // batch of 4 at 1.04-1.07x (5-8 chunks of up to 8 heads in one of 8: 0.97-1.02x).
  if (p.hpt <= R && s <= 4)
    merge_columns<W, 1, 4, FIRST, NANS>(p, lds, srow0, cstride, s, orow0, tid, first_rows);
  else if (p.hpt <= R && (s <= 8 || s > 16))
    merge_columns<W, 1, 8, FIRST, NANS>(p, lds, srow0, cstride, s, orow0, tid, first_rows);
  else if (p.hpt <= R)
    merge_columns<W, 1, 16, FIRST, NANS>(p, lds, srow0, cstride, s, orow0, tid, first_rows);
  else if (IPT == 2 && s <= 4)
    merge_columns<W, 2, 4, FIRST, NANS>(p, lds, srow0, cstride, s, orow0, tid, first_rows);
  else if (IPT > 2 && p.hpt <= 2 * R)
    merge_columns<W, 2, 8, FIRST, NANS>(p, lds, srow0, cstride, s, orow0, tid, first_rows);
  else
    merge_columns<W, IPT, CB, FIRST, NANS>(p, lds, srow0, cstride, s, orow0, tid, first_rows);
}

constexpr float kNoScore = -3.402823466e38f;  // -FLT_MAX

// One wave's running state over the 32-key tiles of a chunk: the packed query
// heads as the MFMA B operand and, per 16-head column tile, the online
// softmax's max and row-summed l and NB 16-dim blocks of unnormalised output.
template <int NT, int NB>
struct TileReducer {
  bf16x8 q[NT][4];
  float m[NT], l[NT];
  f32x4 o[NT][NB];
  float scale_log2;
  int quad;

  // Q^T as the MFMA B operand.  The reduction index of the product may
  // map to head dims in any order as long as K and Q agree: k-step j,
  // lane group `quad` covers dims [32j + 8*quad, +8).  The lane holds those
  // dims of head column `col` of the hpt rows at qrow; rows past them are out
  // of the buffer's range and read as zeros.  (Loads under a lane guard made
  // the compiler wait for Q before the first K/V load: launches of many short
  // chunks up to 7% slower.)
  __device__ __forceinline__ void load_q(const uint16_t* qrow, int hpt, int col) {
    const __amdgpu_buffer_rsrc_t qr = make_rsrc(qrow, (uint32_t)hpt * (D * 2));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        q[nt][j] = as_bf16x8(__builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       qr, (uint32_t)(nt * 16 + col) * (D * 2) + 64u * j + 16u * quad, 0, 0)));
  }

  // The maximum of no scores is the lowest finite number: scores of -inf (masked
  // ones, infinite keys) then weigh 0 also before the first finite one, where
  // -inf - (-inf) would be NaN.
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt] = kNoScore;
      l[nt] = 0.f;
#pragma unroll
      for (int nn = 0; nn < NB; ++nn) o[nt][nn] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // l summed over the row groups, once the last tile is in.
  __device__ __forceinline__ void close() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) l[nt] = sum_rows(l[nt]);
  }

  // S^T[16 keys x 16 heads] per (mt, nt) from the tile's 8 K operands.
  __device__ __forceinline__ void scores(const bf16x8 (&kop)[2][4], f32x4 (&sc)[NT][2]) const {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[mt][j], q[nt][j], acc, 0, 0, 0);
        sc[nt][mt] = acc;
      }
  }

  // Online softmax per head column, in log2 units of the scaled score: the
  // max is taken on raw scores (the scale is positive) and each exponent is
  // one fma, raw * scale*log2(e) - running max.  `last`: only the final tile
  // can be shorter than 32 keys and needs its scores masked.
  // PARTS 2 keeps what rounding the probabilities to bf16 leaves over as a
  // second operand (pb[1]; the difference is exact in fp32).
  template <int PARTS, typename Last>
  __device__ __forceinline__ void softmax(const f32x4 (&sc)[NT][2], int nvalid, Last last,
                                          bf16x8 (&pb)[PARTS][NT]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[8];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float r = sc[nt][mt][i];
          if constexpr (Last::value) r = (mt * 16 + quad * 4 + i) < nvalid ? r : -INFINITY;
          x[mt * 4 + i] = r;
        }
      const float rmax = max_rows(fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                                        fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))));
      const float m_new = fmaxf(m[nt], rmax * scale_log2);
      const float alpha = __builtin_amdgcn_exp2f(m[nt] - m_new);
      float psum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], scale_log2, -m_new));
        psum += x[e];
      }
      l[nt] = l[nt] * alpha + psum;
      m[nt] = m_new;
      // alpha == 1 exactly when the column max did not move: skip the
      // multiply by one (a wave-uniform branch)
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int nn = 0; nn < NB; ++nn) o[nt][nn] *= alpha;
      }
      u32x4 pk;
      pk.x = pack_bf16x2(x[0], x[1]);
      pk.y = pack_bf16x2(x[2], x[3]);
      pk.z = pack_bf16x2(x[4], x[5]);
      pk.w = pack_bf16x2(x[6], x[7]);
      pb[0][nt] = as_bf16x8(pk);
      if constexpr (PARTS == 2) {
        auto low = [&](uint32_t two, int e) {  // bf16 pair `two` stands for x[e], x[e + 1]
          return pack_bf16x2(x[e] - __uint_as_float(two << 16), x[e + 1] - __uint_as_float(two & 0xffff0000u));
        };
        pk.x = low(pk.x, 0);
        pk.y = low(pk.y, 2);
        pk.z = low(pk.z, 4);
        pk.w = low(pk.w, 6);
        pb[1][nt] = as_bf16x8(pk);
      }
    }
  }

  // O^T[16 dims x 16 heads] += V^T[16 dims x 32 keys] . P^T[32 keys x 16 heads]
  // The k index 8*quad + 4*mt + i of the product stands for key
  // 16*mt + 4*quad + i, matching the score layout.  The V^T operand comes
  // from transposing LDS reads (ds_read_b64_tr_b16): within each 16-lane
  // group, output lane j receives element j%4 of the 8-byte chunks that
  // lanes 4k + j/4 point at, k = 0..3.  Lane (quad, 4k + m) therefore points
  // at dims [16nn + 4m, +4) of key 16mt + 4quad + k -- vaddr(mt, nn) gives
  // that address for the stage layout in use -- and lane (quad, col)
  // receives V[16mt + 4quad + k][16nn + col] for k = 0..3.  All 16 reads are
  // issued before the first product so their LDS latency is paid once per
  // tile rather than once per 16 output dims.
  // With direct-to-LDS loads in flight (`opaque`; vaddr then gives LDS byte
  // offsets), the reads are written as inline assembly followed by an
  // explicit wait: the compiler cannot tell that they touch the other stage
  // and would otherwise drain every outstanding load before them.
  template <int PARTS, typename Addr, typename Opaque>
  __device__ __forceinline__ void pv(const bf16x8 (&pb)[PARTS][NT], Addr vaddr, Opaque opaque) {
    s16x4 vlo[NB], vhi[NB];
    if constexpr (Opaque::value) {
#pragma unroll
      for (int nn = 0; nn < NB; ++nn) {
        asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(vlo[nn]) : "v"((uint32_t)vaddr(0, nn)) : "memory");
        asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(vhi[nn]) : "v"((uint32_t)vaddr(1, nn)) : "memory");
      }
      // The wait names every result as an operand it updates, so nothing
      // that reads them can be scheduled before it.
      if constexpr (NB == 8)
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(vlo[0]), "+v"(vlo[1]), "+v"(vlo[2]), "+v"(vlo[3]), "+v"(vlo[4]), "+v"(vlo[5]),
                       "+v"(vlo[6]), "+v"(vlo[7]), "+v"(vhi[0]), "+v"(vhi[1]), "+v"(vhi[2]), "+v"(vhi[3]),
                       "+v"(vhi[4]), "+v"(vhi[5]), "+v"(vhi[6]), "+v"(vhi[7])
                     :
                     : "memory");
      else if constexpr (NB == 4)
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(vlo[0]), "+v"(vlo[1]), "+v"(vlo[2]), "+v"(vlo[3]), "+v"(vhi[0]), "+v"(vhi[1]),
                       "+v"(vhi[2]), "+v"(vhi[3])
                     :
                     : "memory");
      else
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(vlo[0]), "+v"(vlo[1]), "+v"(vhi[0]), "+v"(vhi[1]) : : "memory");
    } else {
#pragma unroll
      for (int nn = 0; nn < NB; ++nn) {
        vlo[nn] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)vaddr(0, nn));
        vhi[nn] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)vaddr(1, nn));
      }
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * NB, 0);   // the DS reads first
    __builtin_amdgcn_sched_group_barrier(0x008, PARTS * NB * NT, 0);  // then the MFMAs
#pragma unroll
    for (int nn = 0; nn < NB; ++nn) {
      const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vlo[nn], vhi[nn], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int i = PARTS - 1; i >= 0; --i)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          o[nt][nn] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[i][nt], o[nt][nn], 0, 0, 0);
    }
  }
};

// A chunk's W wave states are merged in one step.  Every wave publishes its
// closed state (per head column: running max, row-summed l, NB x 4 output values;
// all waves share one lane layout) to its LDS slot, value-major
// ([value][lane], conflict-free).  After a barrier (the caller's), wave w
// merges the W states for its NB/W blocks of 16 output dims -- maximum,
// weights, then sums taken in wave order, so the result is the same on every
// run -- and writes that slice of the output (finish_chunk).
template <int NB>
constexpr int kSlotVals = 2 + 4 * NB;  // state values per lane and head tile: m, l, NB x 4 outputs

template <int NT, int NB>
__device__ __forceinline__ void publish_wave(const TileReducer<NT, NB>& red, float* slots, int wave, int lane) {
  constexpr int SV = kSlotVals<NB>;
  float* v0 = slots + (size_t)wave * (NT * SV * 64);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float* v = v0 + nt * SV * 64;
    v[lane] = red.m[nt];
    v[64 + lane] = red.l[nt];
#pragma unroll
    for (int nn = 0; nn < NB; ++nn)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[(2 + nn * 4 + i) * 64 + lane] = red.o[nt][nn][i];
  }
}

// direct: the chunk is the whole sequence and the normalised output is
// written (rows row0_tile + h); otherwise the chunk state (state rows srow0 +
// h), with device-scope stores where p.mode is kFused.  nb0: first 16-dim
// block of this workgroup's V slice.  With fewer blocks than waves (V slices)
// waves 0 .. NB - 1 merge one block each.
template <int NT, int NB, int W, bool NANS = false>
__device__ __forceinline__ void finish_chunk(const Params& p, const float* slots, bool direct, int64_t row0_tile,
                                             int64_t srow0, int nb0, int wave, int lane) {
  static_assert(NB % W == 0 || W % NB == 0, "blocks must divide among the waves");
  constexpr int NBW = NB >= W ? NB / W : 1;
  constexpr int SV = kSlotVals<NB>;
  const int col = lane & 15, quad = lane >> 4;
  const bool merges = NB >= W || wave < NB;
  auto slot = [&](int w) { return slots + (size_t)w * (NT * SV * 64); };
  const __amdgpu_buffer_rsrc_t ors = make_rsrc(p.o_part + srow0 * D, (uint32_t)p.hpt * D * 4);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float mk[W], wk[W];
    float M = -INFINITY;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      mk[k] = slot(k)[nt * SV * 64 + lane];
      M = fmaxf(M, mk[k]);
    }
    float Lw = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      wk[k] = __builtin_amdgcn_exp2f(mk[k] - M);  // all empty: sums of 0 stay 0
      Lw = fmaf(wk[k], slot(k)[(nt * SV + 1) * 64 + lane], Lw);
    }
    // lane (col, quad) owns dims 16(nb0 + nn) + 4quad + [0, 4) of head
    // 16nt + col, nn = wave * NBW + bb
    f32x4 o[NBW];
#pragma unroll
    for (int bb = 0; bb < NBW; ++bb) {
      const int nn = merges ? wave * NBW + bb : 0;
      o[bb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < W; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[bb][i] = fmaf(wk[k], slot(k)[(nt * SV + 2 + nn * 4 + i) * 64 + lane], o[bb][i]);
    }
    const int h = nt * 16 + col;
    if (h >= p.hpt || !merges) continue;
    const int64_t row = row0_tile + h;
    const float mval = Lw > 0.f ? M * kLn2 : -INFINITY;
    if (direct) {
      const float inv = Lw > 0.f ? 1.0f / Lw : 0.f;
#pragma unroll
      for (int bb = 0; bb < NBW; ++bb) {
        const int nn = nb0 + wave * NBW + bb;
        *reinterpret_cast<uint2*>(p.out + row * D + 16 * nn + 4 * quad) =
            make_uint2(pack_bf16x2(o[bb][0] * inv, o[bb][1] * inv), pack_bf16x2(o[bb][2] * inv, o[bb][3] * inv));
      }
      if (p.lse && wave == 0 && quad == 0 && nb0 == 0) p.lse[row] = holds<NANS>(Lw) ? mval + logf(Lw) : -INFINITY;
    } else if (p.mode == kPartials) {
#pragma unroll
      for (int bb = 0; bb < NBW; ++bb) {
        const int nn = nb0 + wave * NBW + bb;
        const u32x4 bits = {__float_as_uint(o[bb][0]), __float_as_uint(o[bb][1]), __float_as_uint(o[bb][2]),
                            __float_as_uint(o[bb][3])};
        __builtin_amdgcn_raw_buffer_store_b128(bits, ors, (uint32_t)(h * D + 16 * nn + 4 * quad) * 4u, 0, 0);
      }
      if (wave == 0 && quad == 0 && nb0 == 0) {
        p.m_part[srow0 + h] = mval;
        p.l_part[srow0 + h] = Lw;
      }
    } else {
      // kFused: device-scope stores write the chunk state through L2, so
      // it is visible to every XCD once the stores have completed
#pragma unroll
      for (int bb = 0; bb < NBW; ++bb) {
        const int nn = nb0 + wave * NBW + bb;
        const u32x4 bits = {__float_as_uint(o[bb][0]), __float_as_uint(o[bb][1]), __float_as_uint(o[bb][2]),
                            __float_as_uint(o[bb][3])};
        __builtin_amdgcn_raw_buffer_store_b128(bits, ors, (uint32_t)(h * D + 16 * nn + 4 * quad) * 4u, 0,
                                               kDeviceScope);
      }
      if (wave == 0 && quad == 0 && nb0 == 0) {
        __hip_atomic_store(p.m_part + srow0 + h, mval, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(p.l_part + srow0 + h, Lw, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
  }
}

}  // namespace
