// Decode attention over a paged cache of 4-bit values: the kernel, its plan and
// the entry points.
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

constexpr int W = 4;  // waves per workgroup
// Most chunks of a sequence where their length is chosen: more cost the merge more
// than they save (one sequence of 16000 keys, 32/4 heads, 63 chunks 13.0 us, 32 10.7;
// three of 1-30000, 32/2, 19.6 and 17.1; larger batches do not reach it).
constexpr int kChosenChunks = 32;
constexpr int kFp8 = 0, kFp4 = 4;  // operand formats of the scaled product: e4m3, e2m1

struct Kv4Params {
  Params p;  // q, out, lse, chunk states, counters, block table, lengths, shape, window
  const unsigned char* cache;
  int chunk_tiles;   // tiles of 32 keys a chunk holds (even)
  int blocks;        // tiles a page holds
  uint32_t page_bytes;
  Div div_blocks;
  Div div_tiles;     // p.tiles
  int groups;        // dealt: shares of the batch's tiles a head tile has
  Div div_groups;
  int halves;        // dealt: half shares where the lengths differ much
};

constexpr int kv4_smem_bytes(int NT) {
  return W * kKeysPerTile * kVPitch > W * merge_slot_bytes(NT) ? W * kKeysPerTile * kVPitch : W * merge_slot_bytes(NT);
}
static_assert(kv4_smem_bytes(1) >= (2 * (DA_MAX_SPLITS + 16) * 32 + 8 * 32) * 4,
              "the merge stages chunk maxima and sums in LDS");

typedef int i32x8 __attribute__((ext_vector_type(8)));

// A head's query as the 8-bit operand of the scaled product, in three parts:
// q = 2^e (hi + 2^-4 mid + 2^-14 lo), all e4m3, the head's largest magnitude in
// [2^e, 2^(e+1)).  The unit adds the products of eight neighbouring dims in a
// window that ends 13 bits below the largest one's power of two, and cuts what
// lies lower.  Codes span three powers (0.5 to 6 is 2^-1 to 2^2), so a part may
// span ten: e4m3 below 2 does, from 2^0 to its smallest step of 2^-9.  Each part
// is what the ones before leave, rounded to four bits and to that step; it is at
// most half a step of theirs, 2^-4 and then 2^-14.  So no product is cut, and q
// is exact for every element within 11 powers of two of the largest, off by at
// most 2^-19 of the largest's power below that.  (Two parts that reached further
// down, cut in the sum: the log-sum-exp of short sequences off by up to 8e-5, now
// 1e-6, and queries with one large element by more.)
struct Query {
  i32x8 hi, mid, lo;
  int hi_scale, mid_scale, lo_scale;
};

// x: the lane's 32 bf16 values (dims 16 quad + [0, 16) and 64 + 16 quad + [0,
// 16), the operand's order).
__device__ __forceinline__ Query split_query(const u32x4 (&x)[4]) {
  float top = 0.f;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t two = x[i / 4][i % 4];
    top = fmaxf(top, fmaxf(fabsf(__uint_as_float(two << 16)), fabsf(__uint_as_float(two & 0xffff0000u))));
    bad = bad || (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u;
  }
  top = max_rows(bad ? INFINITY : top);
  const int e = max((int)(__float_as_uint(top) >> 23), 16);  // biased exponent of the scale
  // four floats as e4m3 in a word; they become `up` times what that leaves
  auto part = [](float (&f)[4], float up) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    x = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], x, true);
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(x, true);
    f[0] = up * (f[0] - a[0]);
    f[1] = up * (f[1] - a[1]);
    f[2] = up * (f[2] - b[0]);
    f[3] = up * (f[3] - b[1]);
    return x;
  };
  Query q;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float f[4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t two = x[i / 2][(2 * i + j) % 4];
      f[2 * j] = __builtin_amdgcn_ldexpf(__uint_as_float(two << 16), 127 - e);
      f[2 * j + 1] = __builtin_amdgcn_ldexpf(__uint_as_float(two & 0xffff0000u), 127 - e);
    }
    q.hi[i] = part(f, 0x1p4f);
    q.mid[i] = part(f, 0x1p10f);
    q.lo[i] = part(f, 0.f);
  }
  // a query with an infinity or a NaN: scale NaN
  q.hi_scale = top < INFINITY ? e : 255;
  q.mid_scale = top < INFINITY ? e - 4 : 255;
  q.lo_scale = top < INFINITY ? e - 14 : 255;
  return q;
}

// Softmax of a pair of tiles (64 keys) per head column, as TileReducer::softmax
// does it for one: sc holds the raw scores, then the probabilities as bf16
// operands of the two tiles.  Each is rounded once for that, by 2^-8 of itself at
// most; their sum is taken in 32 bits before, so the output is off by at most
// 2^-8 of the weighted mean of |v|, the size of its own rounding to bf16, and lse
// not at all.
template <int NT>
__device__ __forceinline__ void softmax_pair(TileReducer<NT, 8>& red, f32x4 (&sc)[NT][4], bf16x8 (&pb)[2][1][NT]) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float top = fmaxf(sc[nt][0][0], sc[nt][0][1]);
#pragma unroll
    for (int e = 2; e < 16; ++e) top = fmaxf(top, sc[nt][e / 4][e % 4]);
    const float m_new = fmaxf(red.m[nt], max_rows(top) * red.scale_log2);
    const float alpha = __builtin_amdgcn_exp2f(red.m[nt] - m_new);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = __builtin_amdgcn_exp2f(fmaf(sc[nt][e / 4][e % 4], red.scale_log2, -m_new));
      sc[nt][e / 4][e % 4] = x;
      sum += x;
    }
    red.l[nt] = red.l[nt] * alpha + sum;
    red.m[nt] = m_new;
    if (__any(alpha != 1.0f)) {
#pragma unroll
      for (int nn = 0; nn < 8; ++nn) red.o[nt][nn] *= alpha;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 pk;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4& x = sc[nt][2 * h + i / 2];
        pk[i] = pack_bf16x2(x[2 * (i % 2)], x[2 * (i % 2) + 1]);
      }
      pb[h][0][nt] = as_bf16x8(pk);
    }
  }
}

// One workgroup: a head tile (the query heads of one KV head, up to 16 NT of
// them) of a sequence, and a chunk of its 32-key tiles.  A pair of tiles (64
// keys) is a wave's step, W pairs side by side.
//   * S^T[key, head] = K . Q^T on v_mfma_scale_f32_16x16x128_f8f6f4, whose first
//     operand is the cache as it lies there: lane (key, block of 32 dims) gives 16
//     bytes of e2m1 codes and one scale byte.  The query is the other operand, in
//     three 8-bit parts (Query): three products for 16 keys, and no instruction
//     that unpacks K.  (The step from K unpacked to bf16, with the waits for the loads
//     put in order at the same time: 74 -> 55 us for 32 sequences of 8192 keys,
//     64/8 heads, one workgroup a CU.)
//   * V has its scales per key, the index that the second product sums over, so
//     it is unpacked, 64 conversions a pair that are exact in bf16, and goes
//     through the transposing LDS reads of TileReducer::pv.
//   * One softmax for the pair: half the row reductions, rescalings and branches
//     (the same work resident in L2: 36 -> 33 us).
// Bound by HBM over long batches: 32 sequences of 8192 keys, 64/8 heads (286 MB)
// 46-53 us by the run, 44 from the first workgroup's start to the last one's end,
// 6.5 TB/s; resident in L2 the same work takes 34 us at three workgroups a CU.
// Bound by latency where a wave has few pairs (1.1 us each alone).
template <int NT, bool NTL, bool WIN, bool DEAL>
__global__ void __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(NT == 1 ? 3 : 2, 8)))
kv4_kernel(Kv4Params a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int kv_aux = NTL ? 2 : 0;
  const Params& p = a.p;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;

  // ---- this workgroup's sequence, head tile and chunk
  int b, ht, chunk, L, chunk_tiles, chunks = 0;
  int64_t srow0, cstride;  // state row of its first head; rows between two chunks of a head
  Window wn{};
  if constexpr (DEAL) {
    // The lengths decide: chunks of an even share of the batch's tiles for each of
    // a.groups places a head tile, or half of one (at least a pair of tiles a wave,
    // at most 32 chunks a sequence; three pairs a wave are as fast as a merge).
    // Sequences have as many workgroups as chunks, so none is launched for nothing
    // but those by which the chunks' roundings stay below their bound.  (One split
    // count for all: 128 MQA sequences of 16-32768 keys 29 us at the best count,
    // 20 so.  Runs of equal length over sequence ends, as dealt_kernel gives its
    // workgroups, balance the CUs better and pay for the ends: over 250 MB 4-12%
    // faster, below it up to 45% slower.)
    // Lengths and tiles of 256 sequences, loaded together (one after the other they
    // took 4 us of 80 sequences): lane i has b0 + 64 w + i, none past the batch.
    constexpr int kPasses = 4;
    const __amdgpu_buffer_rsrc_t lens = make_rsrc(p.seq_lens, 4u * (uint32_t)p.B);
    int len[kPasses], tl[kPasses];
    auto load_lengths = [&](int b0) {
#pragma unroll
      for (int w = 0; w < kPasses; ++w)
        len[w] = (int)__builtin_amdgcn_raw_buffer_load_b32(lens, 4u * (uint32_t)(b0 + 64 * w + lane), 0, 0);
#pragma unroll
      for (int w = 0; w < kPasses; ++w) {
        len[w] = len[w] < 0 ? 0 : (len[w] > p.L_K ? p.L_K : len[w]);
        const int vis = WIN ? len[w] - window_of(len[w], p.window, p.sinks).skip : len[w];
        tl[w] = (vis + kKeysPerTile - 1) / kKeysPerTile;
      }
    };
    int sum = 0, top = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64 * kPasses) {
      load_lengths(b0);
#pragma unroll
      for (int w = 0; w < kPasses; ++w) {
        sum += tl[w];  // at most 2^30 in all
        top = max(top, tl[w]);
      }
    }
    const int total = __builtin_amdgcn_readlane(wave_scan(sum), 63);
    top = wave_top(top);
    int share = div_by(total + a.groups - 1, a.div_groups);
    // a longest sequence of more than one and a half times the mean length, and of
    // more than a share by an eighth (80 sequences of 1-8192 keys, 64/8 heads, none
    // of which fills a share: halves 87 us, whole 81; 48 such: 49 and 53)
    if (a.halves && (int64_t)top * p.B * 2 > (int64_t)total * 3 && top > share + share / 8) share = (share + 1) / 2;
    int per = max(max(share, 2 * W), (top + kChosenChunks - 1) / kChosenChunks);
    if (top <= 6 * W) per = top;
    per = max(2, (per + 1) & ~1);
    chunk_tiles = per;
    const float inv = 1.0f / (float)per;
    auto lane_chunks = [&](int at, int tiles_of) {  // small: the quotient is off by one at most
      const int x = tiles_of + per - 1;
      int q = (int)((float)x * inv);
      q += (q + 1) * per <= x ? 1 : 0;
      q -= q * per > x ? 1 : 0;
      return at + lane < p.B ? max(q, 1) : 0;
    };
    // Items: a sequence's chunks, the head tiles of each next to one another.
    // Workgroup i starts on XCD i % 8, and patterns in the lengths (two chunks
    // each, one whole and one short) could give some XCDs all the long ones (80
    // sequences of 1-8192 keys, chunks of a head tile next to one another: twice
    // the tiles on every other XCD), so each eight items are given out one place
    // further on.
    const int item = (int)((blockIdx.x & ~7u) + ((blockIdx.x + (blockIdx.x >> 3)) & 7u));
    b = -1;
    int first = 0;
    L = 0;
    for (int b0 = 0, before = 0; b0 < p.B && b < 0; b0 += 64 * kPasses) {
      if (p.B > 64 * kPasses) load_lengths(b0);
#pragma unroll
      for (int w = 0; w < kPasses; ++w) {
        const int at = b0 + 64 * w;
        if (b >= 0 || at >= p.B) continue;
        const int c = lane_chunks(at, tl[w]);
        const int incl = wave_scan(c);
        const uint64_t past = __ballot((before + incl) * p.tiles_per_seq > item);
        if (past) {
          const int i = __ffsll((unsigned long long)past) - 1;
          b = at + i;
          first = (before + __builtin_amdgcn_readlane(incl - c, i)) * p.tiles_per_seq;
          chunks = __builtin_amdgcn_readlane(c, i);
          L = __builtin_amdgcn_readlane(len[w], i);
        }
        before += __builtin_amdgcn_readlane(incl, 63);
      }
    }
    if (b < 0) return;  // fewer chunks than the bound: the whole workgroup
    chunk = div_by(item - first, p.div_tps);
    ht = item - first - chunk * p.tiles_per_seq;
    srow0 = (int64_t)item * p.hpt;
    cstride = (int64_t)p.tiles_per_seq * p.hpt;
    if constexpr (WIN) wn = window_of(L, p.window, p.sinks);
  } else {
    // all first chunks, then all second ones, ...
    chunk = div_by((int)blockIdx.x, a.div_tiles);
    const int tile = (int)blockIdx.x - chunk * p.tiles;
    b = div_by(tile, p.div_tps);
    ht = tile - b * p.tiles_per_seq;
    chunk_tiles = a.chunk_tiles;
    cstride = (int64_t)p.B * p.H_Q;
    srow0 = (int64_t)chunk * cstride + (int64_t)b * p.H_Q + ht * p.hpt;
  }
  const int head0 = ht * p.hpt;
  const int kvh = div_by(head0, p.div_g);
  // Q first: dims 16 quad + [0, 16) and 64 + 16 quad + [0, 16) of head column
  // `col`; it is waited for while the first tiles are on their way
  u32x4 qx[NT][4];
  {
    const __amdgpu_buffer_rsrc_t qr = make_rsrc(p.q + ((int64_t)b * p.H_Q + head0) * D, (uint32_t)p.hpt * (D * 2));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        qx[nt][j] = __builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       qr, (uint32_t)(nt * 16 + col) * (D * 2) + 32u * quad + 16u * (j % 2) + 128u * (j / 2), 0, 0));
  }
  const int t0 = chunk * chunk_tiles;
  // this wave's pairs of tiles: 2 wave, 2 wave + 2 W, ... from t0 on
  const int first_tile = t0 + 2 * wave;
  auto tile_of = [&](int i, int h) { return first_tile + 2 * W * i + h; };
  auto key_of = [&](int t) {  // first key of tile t
    const int at = kKeysPerTile * t;
    return WIN ? wn.key(at) : at;
  };
  // Page ids come by scalar loads, one pair ahead of the tiles' own loads (the
  // table is not written while the kernel runs).
  typedef const __attribute__((address_space(4))) int32_t* Ints;
  const Ints table = (Ints)(uintptr_t)(p.block_table + (int64_t)b * p.max_pages);
  struct Place {
    int page[2], block[2];
  };
  // Past the wave's last tile it is some other place, which is not read.
  auto place = [&](int i) {
    Place pl;
    int j[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int kt = key_of(tile_of(i, h)) / kKeysPerTile;
      const int page = div_by(kt, a.div_blocks);
      pl.block[h] = kt - page * a.blocks;
      j[h] = min(page, p.max_pages - 1);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) pl.page[h] = table[j[h]];
    return pl;
  };
  // The length and, without a window, the first places come together.
  if constexpr (!DEAL) L = ((Ints)(uintptr_t)p.seq_lens)[b];
  Place first_place{}, next{};
  if constexpr (!WIN || DEAL) {
    first_place = place(0);
    next = place(1);
  }
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (!DEAL) {
    L = L < 0 ? 0 : (L > p.L_K ? p.L_K : L);
    if constexpr (WIN) {
      wn = window_of(L, p.window, p.sinks);
      first_place = place(0);
      next = place(1);
    }
  }
  const int vis = L - wn.skip;  // positions
  const int T = (vis + kKeysPerTile - 1) / kKeysPerTile;
  if constexpr (!DEAL) chunks = max(1, (T + chunk_tiles - 1) / chunk_tiles);
  const int t1 = min(t0 + chunk_tiles, T);
  const int n = t1 > first_tile ? (t1 - first_tile + 2 * W - 1) / (2 * W) : 0;
  const unsigned char* const heads = a.cache + (int64_t)kvh * a.blocks * DA_KV4_TILE_BYTES;
  struct Tile {
    u32x4 k[2], v[2];
    uint32_t scales;
    __amdgpu_buffer_rsrc_t at;
  } tiles[2];
  const uint32_t off = 64u * col + 16u * quad;
  // K codes and scales of pair i, at `pl`; a tile past the wave's last: reads
  // of no bytes (the number of loads in flight stays known).  V codes apart.
  auto load_k = [&](const Place& pl, int i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // a page id outside the cache reads as zeros
      const bool in = (int)((uint32_t)pl.page[h] < (uint32_t)p.num_pages) & (int)(tile_of(i, h) < t1);
      const unsigned char* at = heads + (uint64_t)(uint32_t)(in ? pl.page[h] : 0) * a.page_bytes +
                                (uint32_t)pl.block[h] * (uint32_t)DA_KV4_TILE_BYTES;
      Tile& t = tiles[h];
      t.at = make_rsrc(at, in ? DA_KV4_TILE_BYTES : 0u);
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) t.k[mt] = __builtin_amdgcn_raw_buffer_load_b128(t.at, off, 1024 * mt, kv_aux);
      t.scales = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(t.at, 16u * col + 4u * quad, kKv4Scales, kv_aux);
    }
  };
  auto load_v = [&](int h) {
    Tile& t = tiles[h];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
      t.v[mt] = __builtin_amdgcn_raw_buffer_load_b128(t.at, off, 1024 * mt + kKv4V, kv_aux);
  };

  TileReducer<NT, 8> red;
  red.scale_log2 = p.scale_log2;
  red.quad = quad;
  // The loads before the loop keep the order of those in it: what the loop may
  // leave in flight at its top is counted over both.
  __builtin_amdgcn_sched_barrier(0);
  load_k(first_place, 0);
  __builtin_amdgcn_sched_barrier(0);
  load_v(0);
  __builtin_amdgcn_sched_barrier(0);
  load_v(1);
  __builtin_amdgcn_sched_barrier(0);
  // a chunk past the sequence's end: the whole workgroup (its loads read nothing;
  // leaving before them would put them behind the wait for the length)
  if (!DEAL && t0 >= T && chunk > 0) return;
  Query query[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) query[nt] = split_query(qx[nt]);
  red.reset();
  // V as bf16 rows of kVPitch bytes.  The 16-byte pieces of rows with bit 2 set
  // change places in pairs: eight lanes that write one piece of eight rows then
  // meet eight bank groups (without, 16 cycles a write instead of 8), and the
  // transposing reads, which take both pieces of a pair, are as they were.
  unsigned char* vstage = smem + wave * kKeysPerTile * kVPitch;
  const int swap = 16 * ((col >> 2) & 1);
  unsigned char* const vput[2] = {vstage + col * kVPitch + 64 * quad + swap,
                                  vstage + col * kVPitch + 64 * quad + (swap ^ 16)};
  auto stage_v = [&](const Tile& t, uint32_t scales) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const float s = kv4_scale((scales >> (16 + 8 * mt)) & 0xffu);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 y;
        dequantise(t.v[mt][j], s, y);
        *reinterpret_cast<u32x4*>(vput[j & 1] + 16 * mt * kVPitch + 32 * (j >> 1)) = y;
      }
    }
  };
  const unsigned char* vrow = vstage + (quad * 4 + (col >> 2)) * kVPitch + ((8 * (col & 3)) ^ (16 * (quad & 1)));
  constexpr std::integral_constant<int, 0> m0{};
  constexpr std::integral_constant<int, 1> m1{};
  constexpr std::false_type no{};

  for (int i = 0; i < n; ++i) {
    // S^T[16 keys x 16 heads]: codes and scales go into the product as they are
    f32x4 sc[NT][4];
    auto product = [&](f32x4 c, const Tile& t, auto mt, const i32x8& q, int q_scale) {
      constexpr int M = decltype(mt)::value;
      const i32x8 k = {(int)t.k[M][0], (int)t.k[M][1], (int)t.k[M][2], (int)t.k[M][3], 0, 0, 0, 0};
      return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q, c, kFp4, kFp8, M, (int)t.scales, 0, q_scale);
    };
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const Query& q = query[nt];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sc[nt][2 * h] = product(zero, tiles[h], m0, q.lo, q.lo_scale);
        sc[nt][2 * h + 1] = product(zero, tiles[h], m1, q.lo, q.lo_scale);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sc[nt][2 * h] = product(sc[nt][2 * h], tiles[h], m0, q.mid, q.mid_scale);
        sc[nt][2 * h + 1] = product(sc[nt][2 * h + 1], tiles[h], m1, q.mid, q.mid_scale);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sc[nt][2 * h] = product(sc[nt][2 * h], tiles[h], m0, q.hi, q.hi_scale);
        sc[nt][2 * h + 1] = product(sc[nt][2 * h + 1], tiles[h], m1, q.hi, q.hi_scale);
      }
    }
    uint32_t scales[2] = {tiles[0].scales, tiles[1].scales};
    const int first[2] = {key_of(tile_of(i, 0)), key_of(tile_of(i, 1))};
    const bool cut = L - first[1] < kKeysPerTile || (WIN && (wn.cuts(first[0]) || wn.cuts(first[1])));
    if (cut) {
      // invisible keys and those past the sequence
      auto dead = [&](int h, int row) -> bool {
        return (int)(first[h] + row >= L) | (int)(WIN && wn.hides(first[h], row));
      };
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // whatever such a row holds, its values come out finite: a zero probability cancels them
        if (dead(h, col)) scales[h] = (scales[h] & 0xff00ffffu) | 0x007f0000u;
        if (dead(h, 16 + col)) scales[h] = (scales[h] & 0x00ffffffu) | 0x7f000000u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool d = dead(h, (e / 4) * 16 + quad * 4 + e % 4);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            sc[nt][2 * h + e / 4][e % 4] = d ? -INFINITY : sc[nt][2 * h + e / 4][e % 4];
        }
      }
    }
    stage_v(tiles[0], scales[0]);
    const Tile second = tiles[1];
    load_k(next, i + 1);
    load_v(0);
    next = place(i + 2);
    bf16x8 pb[2][1][NT];
    softmax_pair(red, sc, pb);
    __builtin_amdgcn_wave_barrier();
    red.pv(pb[0], [&](int mt, int nn) { return vrow + mt * 16 * kVPitch + 32 * nn; }, no);
    __builtin_amdgcn_wave_barrier();
    stage_v(second, scales[1]);
    load_v(1);
    __builtin_amdgcn_wave_barrier();
    red.pv(pb[1], [&](int mt, int nn) { return vrow + mt * 16 * kVPitch + 32 * nn; }, no);
    __builtin_amdgcn_wave_barrier();
  }

  const int64_t row0 = (int64_t)b * p.H_Q + head0;
  const bool direct = chunks == 1;
  red.close();
  __syncthreads();  // every wave is done with its stage
  publish_wave(red, reinterpret_cast<float*>(smem), wave, lane);
  __syncthreads();
  finish_chunk<NT, 8, W, true>(p, reinterpret_cast<const float*>(smem), direct, row0, direct ? 0 : srow0, 0, wave,
                               lane);
  if (direct) return;

  // The merge inside the launch: the hand-off of split_partial_kernel
  // (decode_attn.hip), with this sequence's chunk count.
  __shared__ int s_last;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) {
    uint32_t* counter = p.arrivals + ((size_t)b * p.tiles_per_seq + ht) * da::kArrivalStride;
    const bool last =
        __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u == (uint32_t)chunks;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = last ? 1 : 0;
  }
  __syncthreads();
  if (!s_last) return;
  merge_tile<NT, W, false, true>(p, reinterpret_cast<float*>(smem), srow0 - chunk * cstride, cstride, chunks, row0,
                                 tid);
}

// ---------------------------------------------------------------- host side

constexpr int kDealtSequences = 1024;      // most of a batch that is dealt
constexpr double kStreamBytes = 64 << 20;  // a quarter of the last-level cache

struct Kv4Plan {
  int heads_per_tile, tiles;
  int chunk_tiles;  // tiles of a chunk; 0: dealt
  int groups;       // dealt: shares of a head tile
  int halves;
  int grid;         // workgroups
  int rows, heads;  // chunk states: rows x heads (0: none)
};

// num_splits <= 0: chosen.  `pool`: keys the cache holds, a bound of the batch's.
Kv4Plan kv4_plan(int B, int H_Q, int H_KV, int keys, int64_t pool, int num_splits, int cus) {
  Kv4Plan pl{};
  pl.heads_per_tile = da::heads_per_tile(H_Q, H_KV, 1);
  const int tps = H_Q / pl.heads_per_tile;
  pl.tiles = B * tps;
  const int T = std::max(1, (keys + kKeysPerTile - 1) / kKeysPerTile);
  // a counter for every tile, and chunk states below 2 GiB
  const int64_t most = pl.tiles > da::kMaxArrivalTiles
                           ? 1
                           : std::max<int64_t>(1, std::min<int64_t>(DA_MAX_SPLITS, (((int64_t)1 << 31) - 1) /
                                                                                       ((int64_t)B * H_Q * D * 4)));
  // Lengths that differ decide the chunks on the device (dealt).  That costs
  // about 1 us before the first load, so one sequence, and batches whose longest
  // takes a few microseconds anyway, have chunks of a length chosen here; so do
  // batches of so many sequences that each workgroup's two passes over the lengths
  // cost more than even chunks give (8/1 heads, lognormal lengths up to 16384: 1024
  // sequences 78 us whole, 45 dealt; 4096 sequences 125 and 226).
  if (num_splits <= 0 && B > 1 && B <= kDealtSequences && T > 8 * 2 * W && most == DA_MAX_SPLITS &&
      (int64_t)B * T <= (1 << 30)) {
    pl.groups = std::max(1, cus / tps);
    // the shares, and a chunk's rounding for each sequence
    // Where lengths differ, whole and partial chunks meet on a CU, and half shares
    // even that out if there are head tiles enough for few chunks of each: 32
    // sequences of 1024-16384 keys (64/8 heads) 66.8 -> 63.1 us, 16 of which two
    // have 32768 and the rest 1024 27.1 -> 22.4, 24 of 1-16000 (16/16) 90.3 -> 81.5;
    // 32-column tiles (128/2) 23.6 -> 33.9, and equal lengths 0-19% slower.
    pl.halves = pl.heads_per_tile <= 16 && pl.tiles >= cus / 2;
    const int64_t chunks =
        std::min<int64_t>((int64_t)pl.groups * (1 + pl.halves) + B, (int64_t)B * kChosenChunks);
    pl.grid = (int)((chunks * tps + 7) / 8 * 8);
    pl.rows = pl.grid;
    pl.heads = pl.heads_per_tile;
    if ((int64_t)pl.rows * pl.heads * D * 4 < ((int64_t)1 << 31)) return pl;
  }
  int64_t chunk;
  if (num_splits > 0) {
    chunk = (T + num_splits - 1) / num_splits;
  } else {
    const int64_t mean = std::min<int64_t>(T, (pool / B + kKeysPerTile - 1) / kKeysPerTile);
    chunk = T <= 6 * W ? T : std::max<int64_t>({mean * pl.tiles / cus, 2 * W, (T + kChosenChunks - 1) / kChosenChunks});
  }
  chunk = std::max<int64_t>(chunk, (T + most - 1) / most);
  pl.chunk_tiles = 2 * (int)((std::min<int64_t>(chunk, T) + 1) / 2);  // whole pairs
  const int chunks = (T + pl.chunk_tiles - 1) / pl.chunk_tiles;
  pl.grid = (int)std::min<int64_t>((int64_t)pl.tiles * chunks, INT32_MAX);
  pl.groups = 0;
  pl.rows = chunks > 1 ? chunks * B : 0;
  pl.heads = H_Q;
  return pl;
}

// Shape checks (no HIP calls).  Heads as for the bf16 layouts; their limit on a
// sequence's bytes is one of 32-bit offsets into it, and this cache is addressed
// by page: positions of a few thousand keys past a sequence have to fit an int.
constexpr int kMostKeys = 1 << 30;

int check_kv4_shape(int B, int H_Q, int H_KV, int L_K_max, int d) {
  const int rc = da::check_shape(B, H_Q, H_KV, std::min(L_K_max, 0), d);
  if (rc) return rc;
  if (L_K_max > kMostKeys) return da::fail(DA_ERR_SHAPE, "L_K_max=%d exceeds %d keys", L_K_max, kMostKeys);
  return DA_OK;
}

int kv4_keys(int L_K_max, int window, int sinks) {
  return window > 0 ? da::window_keys(L_K_max, window, sinks) : L_K_max;
}

}  // namespace

extern "C" {

size_t da_kv4_workspace_bytes(int B, int H_Q, int H_KV, int L_K_max, int64_t pool_keys, int window, int sinks,
                              int num_splits, int num_cus) {
  if (check_kv4_shape(B, H_Q, H_KV, L_K_max, D) || window < 0 || sinks < 0 || num_splits > DA_MAX_SPLITS) return 0;
  if (num_cus <= 0 && ensure_gfx950(&num_cus)) return 0;
  const Kv4Plan pl = kv4_plan(B, H_Q, H_KV, kv4_keys(L_K_max, window, sinks),
                               pool_keys > 0 ? pool_keys : 1, num_splits, num_cus);
  return pl.rows ? da::workspace_layout(pl.rows, pl.heads, D, 1).total : 0;
}

int da_decode_attn_kv4(const void* q, const void* cache, const int32_t* block_table, const int32_t* seq_lens, void* out,
                       float* lse_out, int B, int H_Q, int H_KV, int page_size, int max_pages, int num_pages,
                       int L_K_max, int d, float softmax_scale, int window, int sinks, int num_splits, void* workspace,
                       size_t workspace_bytes, void* stream) {
  da::clear_error();
  int rc = check_kv4_shape(B, H_Q, H_KV, L_K_max, d);
  if (!q) return da::fail(DA_ERR_NULL, "q must be non-NULL");
  if (!block_table || !seq_lens) return da::fail(DA_ERR_NULL, "block_table and seq_lens must be non-NULL");
  if (!cache && !(rc == DA_OK && L_K_max == 0)) return da::fail(DA_ERR_NULL, "cache must be non-NULL");
  if (rc) return rc;
  rc = da::check_page_table(B, page_size, max_pages, num_pages, L_K_max);
  if (rc) return rc;
  if (!out) return da::fail(DA_ERR_NULL, "out must be non-NULL");
  if (!aligned(q, 16) || !aligned(cache, 16) || !aligned(out, 16))
    return da::fail(DA_ERR_ALIGN, "q, cache and out must be 16-byte aligned");
  if (!aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(lse_out, 4))
    return da::fail(DA_ERR_ALIGN, "block_table, seq_lens and lse_out must be 4-byte aligned");
  if (window < 0 || sinks < 0)
    return da::fail(DA_ERR_ARG, "window=%d and sinks=%d must not be negative", window, sinks);
  if (num_splits > DA_MAX_SPLITS)
    return da::fail(DA_ERR_SPLITS, "num_splits=%d exceeds %d", num_splits, DA_MAX_SPLITS);
  if (workspace && !aligned(workspace, 16)) return da::fail(DA_ERR_ALIGN, "workspace must be 16-byte aligned");
  const int64_t page_bytes = (int64_t)H_KV * (page_size / kKeysPerTile) * DA_KV4_TILE_BYTES;
  if (page_bytes >= ((int64_t)1 << 32))
    return da::fail(DA_ERR_SHAPE, "a page of %d keys of %d heads exceeds 4 GiB", page_size, H_KV);
  int cus = 0;
  rc = ensure_gfx950(&cus);
  if (rc) return rc;
  const int keys = kv4_keys(L_K_max, window, sinks);
  const int64_t pool = (int64_t)num_pages * page_size;
  const Kv4Plan pl = kv4_plan(B, H_Q, H_KV, keys, pool, num_splits, cus);
  if (pl.grid >= (1 << 24)) return da::fail(DA_ERR_SHAPE, "%d head tiles are too many workgroups", pl.tiles);
  Kv4Params a{};
  da_plan dp{};
  dp.num_splits = 1;
  dp.heads_per_tile = pl.heads_per_tile;
  dp.tiles = pl.tiles;
  fill_params(a.p, B, H_Q, H_KV, L_K_max, softmax_scale, dp);
  a.p.q = static_cast<const uint16_t*>(q);
  a.p.out = static_cast<uint16_t*>(out);
  a.p.lse = lse_out;
  a.p.mode = kFused;
  a.p.block_table = block_table;
  a.p.seq_lens = seq_lens;
  a.p.max_pages = max_pages;
  a.p.num_pages = num_pages;
  a.p.window = window;
  a.p.sinks = sinks;
  a.cache = static_cast<const unsigned char*>(cache);
  a.chunk_tiles = pl.chunk_tiles;
  a.blocks = page_size / kKeysPerTile;
  a.page_bytes = (uint32_t)page_bytes;
  a.div_blocks = make_div((uint32_t)a.blocks);
  a.div_tiles = make_div((uint32_t)pl.tiles);
  a.groups = pl.groups;
  a.div_groups = make_div((uint32_t)std::max(1, pl.groups));
  a.halves = pl.halves;
  if (pl.rows) {
    const da::WorkspaceLayout wl = da::workspace_layout(pl.rows, pl.heads, D, 1);
    if (!workspace || workspace_bytes < wl.total)
      return da::fail(DA_ERR_WORKSPACE, "the 4-bit launch needs %zu workspace bytes, got %zu", wl.total,
                      workspace ? workspace_bytes : (size_t)0);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    a.p.o_part = reinterpret_cast<float*>(ws + wl.o_off);
    a.p.m_part = reinterpret_cast<float*>(ws + wl.m_off);
    a.p.l_part = reinterpret_cast<float*>(ws + wl.l_off);
    a.p.arrivals = reinterpret_cast<uint32_t*>(ws + da::arrival_offset(workspace_bytes));
  }
  // The caches of a step's layers follow each other, so one call's keys are seldom
  // near when it reads them, and streaming loads read faster from HBM: with three
  // caches in turn 140 MB took 32.1 us and 28.8 streamed, 286 MB 57 and 51; one
  // cache again and again 27.5 and 27.9, 47.7 and 50.0 (up to 72 MB no difference).
  const double bytes = (double)std::min<int64_t>((int64_t)B * keys, pool) * H_KV * (DA_KV4_TILE_BYTES / kKeysPerTile);
  const bool ntl = bytes > kStreamBytes && pl.heads_per_tile == H_Q / H_KV;
  auto pick = [&](auto nt, auto deal) -> const void* {
    constexpr int N = decltype(nt)::value;
    constexpr bool DEAL = decltype(deal)::value;
    if (window > 0)
      return ntl ? reinterpret_cast<const void*>(&kv4_kernel<N, true, true, DEAL>)
                 : reinterpret_cast<const void*>(&kv4_kernel<N, false, true, DEAL>);
    return ntl ? reinterpret_cast<const void*>(&kv4_kernel<N, true, false, DEAL>)
               : reinterpret_cast<const void*>(&kv4_kernel<N, false, false, DEAL>);
  };
  auto pick_deal = [&](auto nt) { return pl.groups ? pick(nt, std::true_type{}) : pick(nt, std::false_type{}); };
  const bool narrow = pl.heads_per_tile <= 16;
  const void* fn = narrow ? pick_deal(std::integral_constant<int, 1>{}) : pick_deal(std::integral_constant<int, 2>{});
  const int smem = narrow ? kv4_smem_bytes(1) : kv4_smem_bytes(2);
  void* args[] = {&a};
  const hipError_t e =
      hipLaunchKernel(fn, dim3(pl.grid), dim3(64 * W), args, smem, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return da::fail(DA_ERR_HIP, "4-bit attention launch: %s", hipGetErrorString(e));
  return DA_OK;
}

}  // extern "C"
