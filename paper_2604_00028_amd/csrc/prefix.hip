// Decode attention of a batch whose sequences share prefixes, three launches:
// the batch's work cut into units on the device (plan_kernel), the chunk states
// of the units (unit_kernel), and their merge (merge_kernel).  Entry points at
// the end.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "decode_attn.h"
#include "host.h"
#include "plan.h"
#include "tile.h"

namespace {

using da::aligned;
using da::ensure_gfx950;

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kMostGroupChunks = 64;  // of a prefix, and of a sequence's own keys: one a lane in the merge
constexpr int kSharedRows = 128;      // query rows of the largest unit
constexpr int kUnitWaves = 4;

// A unit: `rows` query rows against the tiles [t0, t1) of one KV head.  Row r is
// query head kvh g + (row0 + r) mod g of sequence seq0 + (row0 + r) / g, its
// chunk state is state row state0 + (its sequence - seq0) H_Q + its head, and
// state0 < 0 writes the output.  Keys come from table row `table`, up to key
// `end`.
struct Unit {
  int32_t table, end, t0, t1, seq0, row0, rows_kvh, state0;  // rows | kvh << 8; rows 0: nothing to do
};
static_assert(sizeof(Unit) == 32, "two 16-byte loads");

// How a row's states are found: `chunks` of the shared keys from state row
// `shared` on, `stride` apart, then `own` ones from state row `own0` on, H_Q
// apart; heads follow each other.
struct SeqStates {
  int32_t shared, chunks, stride, own0, own;  // own < 0: the output is written already
};

struct PrefixParams {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* block_table;
  const int32_t* seq_lens;
  const int32_t* cu;
  const int32_t* prefix_lens;
  uint16_t* out;
  float* lse;
  int32_t* head;      // workspace: units there are
  Unit* units;
  SeqStates* seqs;
  float* o_part;
  float* m_part;
  float* l_part;
  int64_t most_rows;  // state rows there is room for
  int most_units;
  int B, G, H_Q, H_KV, g, hpt, L_K, page_size, max_pages, num_pages;
  int slots;          // workgroups that run at once
  int chunk_tiles;    // 0: chosen on the device
  Div div_page, div_g, div_heads, div_hq;
  float scale_log2;
};

// ---------------------------------------------------------------- plan

// Chunk lengths (in tiles) that the plan chooses among.
constexpr int kLengths[kPlanWaves] = {2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256, 512};

__device__ __forceinline__ int chunks_of(int tiles, int length) {
  const int most = tiles < kMostGroupChunks ? tiles : kMostGroupChunks;
  const int n = (tiles + length - 1) / length;
  return n < most ? n : most;
}

__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

// Sums of x and y over the threads before this one, and over all.
__device__ __forceinline__ void sum_before(int& x, int& y, int2* sums, int2* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sx = wave_scan(x), sy = wave_scan(y);
  __syncthreads();
  if (lane == 63) sums[wave] = make_int2(sx, sy);
  __syncthreads();
  x = sx - x;
  y = sy - y;
  int2 t = make_int2(0, 0);
  for (int w = 0; w < kPlanWaves; ++w) {
    const int2 s = sums[w];
    if (w < wave) {
      x += s.x;
      y += s.y;
    }
    t.x += s.x;
    t.y += s.y;
  }
  *all = t;
}

// One workgroup.  A group's shared keys are its prefix length, or its shortest
// sequence's that has keys if that is less, in whole tiles; a group of one such
// sequence shares none.  They are cut into chunks for tiles of up to 128 of the
// group's query rows, and what each sequence has behind them into chunks for
// the heads of each KV head, all of about one length: of 16 lengths, tried by a
// wave each, the one with the least rounds of the chip's workgroups, each
// priced at its tiles and a few more for its start and the merge of its states.
// Units stand in the order they run in: workgroup i, on XCD i mod 8, takes
// units i, i + grid, ...; the row tiles of a chunk (which read the same keys)
// stand 8 apart, next to each other on one XCD's L2.
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(PrefixParams p) {
  extern __shared__ int32_t lds[];
  __shared__ int2 sums[kPlanWaves];
  __shared__ uint32_t price[kPlanWaves];
  __shared__ int bad;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* tiles = lds;            // [B] tiles of the sequence's own keys
  int32_t* group = tiles + p.B;    // [B] its group, or -1
  int32_t* unit_b = group + p.B;   // [B] its first unit
  int32_t* state_b = unit_b + p.B; // [B] its first state row / H_Q
  int32_t* cu = state_b + p.B;     // [G + 1]
  int32_t* shared = cu + p.G + 1;  // [G] shared keys, then tiles
  int32_t* reader = shared + p.G;  // [G] its first sequence that has keys
  int32_t* unit_g = reader + p.G;  // [G] sequences that have keys, then its first unit
  int32_t* state_g = unit_g + p.G; // [G]

  if (tid == 0) bad = 0;
  for (int i = tid; i <= p.G; i += kPlanThreads) {
    cu[i] = p.G > 0 ? max(0, min(p.cu[i], p.B)) : 0;
    if (i < p.G) {
      shared[i] = max(0, min(p.prefix_lens[i], p.L_K));
      reader[i] = p.B;
      unit_g[i] = 0;
    }
  }
  __syncthreads();
  for (int i = tid; i < p.G; i += kPlanThreads)
    if (cu[i] > cu[i + 1]) bad = 1;
  __syncthreads();
  const int G = bad ? 0 : p.G;  // groups that run backwards share nothing
  for (int b = tid; b < p.B; b += kPlanThreads) {
    const int L = max(0, min(p.seq_lens[b], p.L_K));
    int at = -1;
    if (G > 0 && b >= cu[0] && b < cu[G]) {
      int lo = 0, hi = G;  // the last group that starts at or before b
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= b)
          lo = mid;
        else
          hi = mid;
      }
      at = lo;
    }
    group[b] = at;
    tiles[b] = L;
    if (at >= 0 && L > 0) {
      atomicMin(&shared[at], L);
      atomicMin(&reader[at], b);
      atomicAdd(&unit_g[at], 1);
    }
  }
  __syncthreads();
  for (int i = tid; i < G; i += kPlanThreads) shared[i] = unit_g[i] > 1 ? shared[i] / kKeysPerTile : 0;
  __syncthreads();
  for (int b = tid; b < p.B; b += kPlanThreads) {
    const int L = tiles[b], at = group[b];
    const int first = at >= 0 ? shared[at] : 0;
    tiles[b] = L > 0 ? (L + kKeysPerTile - 1) / kKeysPerTile - first : 0;
  }
  __syncthreads();

  const int own_tiles = p.g / p.hpt;  // head tiles of a KV head
  auto row_tiles = [&](int i) { return (int)(((int64_t)(cu[i + 1] - cu[i]) * p.g + kSharedRows - 1) / kSharedRows); };
  // streams of keys that `readers` units each read, in units
  auto units_of = [&](int64_t streams, int readers) {
    return readers == 1 ? streams : (streams + 7) / 8 * 8 * readers;
  };
  int length = p.chunk_tiles;
  {
    const int mine = length > 0 ? length : kLengths[wave];
    int64_t units = 0, rows = 0;
    for (int i = lane; i < G; i += 64) {
      const int n = chunks_of(shared[i], mine);
      units += units_of((int64_t)n * p.H_KV, row_tiles(i));
      rows += (int64_t)n * (cu[i + 1] - cu[i]);
    }
    for (int b = lane; b < p.B; b += 64) {
      const int n = chunks_of(tiles[b], mine);
      units += units_of((int64_t)n * p.H_KV, own_tiles);
      rows += n;
    }
    const int u = wave_total((int)min<int64_t>(units, 1 << 24)), r = wave_total((int)min<int64_t>(rows, 1 << 24));
    const bool fits = u <= p.most_units && (int64_t)r * p.H_Q <= p.most_rows;
    const uint32_t rounds = (uint32_t)(u + p.slots - 1) / (uint32_t)p.slots;
    if (lane == 0) price[wave] = fits ? min(rounds * (uint32_t)(mine + 4), 0x7ffffffeu) : 0x7fffffffu;
  }
  __syncthreads();
  if (length > 0) {
    if (price[0] == 0x7fffffffu) length = 1 << 26;  // whole prefixes and sequences always fit
  } else {
    uint32_t best = 0x7fffffffu;
    length = 1 << 26;
    for (int w = 0; w < kPlanWaves; ++w)
      if (price[w] < best) {
        best = price[w];
        length = kLengths[w];
      }
  }

  // first units and state rows: groups, then sequences, each thread some in a row
  int2 all_g, all_b;
  {
    const int per = (G + kPlanThreads - 1) / kPlanThreads, i0 = min(tid * per, G), i1 = min(i0 + per, G);
    int u = 0, r = 0;
    for (int i = i0; i < i1; ++i) {
      const int n = chunks_of(shared[i], length);
      unit_g[i] = u;
      state_g[i] = r;
      u += (int)units_of((int64_t)n * p.H_KV, row_tiles(i));
      r += n * (cu[i + 1] - cu[i]);
    }
    sum_before(u, r, sums, &all_g);
    for (int i = i0; i < i1; ++i) {
      unit_g[i] += u;
      state_g[i] += r;
    }
  }
  {
    const int per = (p.B + kPlanThreads - 1) / kPlanThreads, i0 = min(tid * per, p.B), i1 = min(i0 + per, p.B);
    int u = 0, r = 0;
    auto state_chunks = [&](int b, int n) { return n == 1 && (group[b] < 0 || shared[group[b]] == 0) ? 0 : n; };
    for (int b = i0; b < i1; ++b) {
      const int n = chunks_of(tiles[b], length);
      unit_b[b] = u;
      state_b[b] = r;
      u += (int)units_of((int64_t)n * p.H_KV, own_tiles);
      r += state_chunks(b, n);
    }
    sum_before(u, r, sums, &all_b);
    u += all_g.x;
    r += all_g.y;
    for (int b = i0; b < i1; ++b) {
      unit_b[b] += u;
      state_b[b] += r;
      const int n = chunks_of(tiles[b], length), at = group[b];
      const int shared_chunks = at >= 0 && p.seq_lens[b] > 0 ? chunks_of(shared[at], length) : 0;
      SeqStates s;
      s.shared = shared_chunks ? (state_g[at] + (b - cu[at])) * p.H_Q : 0;
      s.chunks = shared_chunks;
      s.stride = shared_chunks ? (cu[at + 1] - cu[at]) * p.H_Q : 0;
      s.own0 = state_b[b] * p.H_Q;
      s.own = n > 0 && state_chunks(b, n) == 0 ? -1 : n;
      p.seqs[b] = s;
    }
  }
  __syncthreads();
  const int total = all_g.x + all_b.x;
  if (tid == 0) p.head[0] = total;
  for (int w = tid; w < total; w += kPlanThreads) {
    const bool of_group = w < all_g.x;
    const int32_t* starts = of_group ? unit_g : unit_b;
    int lo = 0, hi = of_group ? G : p.B;  // the last that starts at or before w
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (starts[mid] <= w)
        lo = mid;
      else
        hi = mid;
    }
    const int at = w - starts[lo];
    const int T = of_group ? shared[lo] : tiles[lo];
    const int n = chunks_of(T, length);
    const int readers = of_group ? row_tiles(lo) : own_tiles;
    int stream = at, reader_at = 0;
    if (readers > 1) {
      const int bundle = at / (8 * readers), in = at - bundle * 8 * readers;
      reader_at = in / 8;
      stream = bundle * 8 + in % 8;
    }
    Unit u{};
    if (stream < n * p.H_KV) {
      const int kvh = stream / n, chunk = stream - kvh * n;
      const int first = of_group ? 0 : group[lo] >= 0 ? shared[group[lo]] : 0;
      u.t0 = first + (int)((int64_t)T * chunk / n);
      u.t1 = first + (int)((int64_t)T * (chunk + 1) / n);
      if (of_group) {
        const int rows = (cu[lo + 1] - cu[lo]) * p.g;
        u.table = reader[lo];
        u.end = T * kKeysPerTile;
        u.seq0 = cu[lo];
        u.row0 = reader_at * kSharedRows;
        u.rows_kvh = min(rows - u.row0, kSharedRows) | kvh << 8;
        u.state0 = (state_g[lo] + chunk * (cu[lo + 1] - cu[lo])) * p.H_Q;
      } else {
        const bool direct = n == 1 && first == 0;
        u.table = lo;
        u.end = max(0, min(p.seq_lens[lo], p.L_K));
        u.seq0 = lo;
        u.row0 = reader_at * p.hpt;
        u.rows_kvh = p.hpt | kvh << 8;
        u.state0 = direct ? -1 : (state_b[lo] + chunk) * p.H_Q;
      }
    }
    p.units[w] = u;
  }
}

// ---------------------------------------------------------------- units

constexpr int kStages = 4;
constexpr int kStageBytes = 2 * kLdsTileBytes;  // K and V of one tile
constexpr int unit_smem() {
  int most = kStages * kStageBytes;
  most = std::max(most, kUnitWaves * kKeysPerTile * kVPitch);
  return std::max(most, kUnitWaves * merge_slot_bytes(2));
}

// Where a unit's row lives.
struct RowPlace {
  int64_t out;    // row of q and of the output
  int64_t state;  // chunk-state row
};

__device__ __forceinline__ RowPlace place_of(const PrefixParams& p, const Unit& u, int kvh, int r) {
  const int rr = u.row0 + r;
  const int s = div_by(rr, p.div_g), h = kvh * p.g + (rr - s * p.g);
  return {(int64_t)(u.seq0 + s) * p.H_Q + h, (int64_t)u.state0 + (int64_t)s * p.H_Q + h};
}

// The page ids of a unit's tiles, 64 at a time, one a lane; a tile's first row.
struct Pages {
  const int32_t* row;
  int first, last, ids;
  __device__ __forceinline__ void start(const PrefixParams& p, const Unit& u, int lane) {
    row = p.block_table + (int64_t)u.table * p.max_pages;
    first = div_by(u.t0 * kKeysPerTile, p.div_page);
    last = div_by(u.t1 * kKeysPerTile - 1, p.div_page);
    ids = first + lane <= last ? row[first + lane] : 0;
  }
  // element offset of the tile's first row of the KV head; false: outside the pool
  __device__ __forceinline__ bool tile(const PrefixParams& p, int t, int kvh, int lane, int64_t& elems) {
    const int key = t * kKeysPerTile, j = div_by(key, p.div_page);
    if (j - first >= 64) {  // wave-uniform
      first = j;
      ids = j + lane <= last ? row[j + lane] : 0;
      asm volatile("" : "+v"(ids));  // waited for here, and not (with the tiles in flight) at every tile's use
    }
    const int page = __builtin_amdgcn_readlane(ids, (j - first) & 63);
    const bool in = page >= 0 && page < p.num_pages;
    elems = (((in ? (int64_t)page : 0) * p.page_size + (key - j * p.page_size)) * p.H_KV + kvh) * D;
    return in;
  }
};

template <int NT>
__device__ __forceinline__ void load_rows(TileReducer<NT, 8>& red, const PrefixParams& p, const Unit& u, int kvh,
                                          int rows, int first, int col, int quad) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    // rows past the unit's repeat its last one; nothing of theirs is stored
    const uint16_t* row = p.q + place_of(p, u, kvh, min(first + nt * 16 + col, rows - 1)).out * D + 8 * quad;
#pragma unroll
    for (int j = 0; j < 4; ++j) red.q[nt][j] = as_bf16x8(*reinterpret_cast<const u32x4*>(row + 32 * j));
  }
}

// 16 NT rows or fewer: the waves take one tile in four, K straight into the
// operand layout and V by way of LDS, the next tile's loads in flight; their
// states meet in LDS at the end (in wave order).
template <int NT>
__device__ __forceinline__ void stream_unit(const PrefixParams& p, const Unit& u, unsigned char* smem, int lane,
                                            int wave) {
  const int rows = u.rows_kvh & 255, kvh = u.rows_kvh >> 8;
  const int col = lane & 15, quad = lane >> 4;
  const uint32_t rs = (uint32_t)p.H_KV * (D * 2);
  TileReducer<NT, 8> red;
  red.scale_log2 = p.scale_log2;
  red.quad = quad;
  load_rows(red, p, u, kvh, rows, 0, col, quad);
  red.reset();
  unsigned char* vstage = smem + wave * kKeysPerTile * kVPitch;
  Pages pages;
  pages.start(p, u, lane);
  auto load = [&](u32x4 (&kreg)[2][4], u32x4 (&vreg)[8], int t) {
    int64_t elems;
    const bool in = pages.tile(p, t, kvh, lane, elems);
    const int n = min(u.end - t * kKeysPerTile, kKeysPerTile);
    const uint32_t bytes =
        (uint32_t)__builtin_amdgcn_readfirstlane(in && n > 0 ? (uint32_t)(n - 1) * rs + D * 2u : 0u);
    const __amdgpu_buffer_rsrc_t kt = make_rsrc(p.k + elems, bytes), vt = make_rsrc(p.v + elems, bytes);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        kreg[mt][j] = __builtin_amdgcn_raw_buffer_load_b128(kt, (uint32_t)(16 * mt + col) * rs + 64u * j + 16u * quad, 0, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      vreg[i] = __builtin_amdgcn_raw_buffer_load_b128(vt, (uint32_t)(4 * i + quad) * rs + 16u * col, 0, 0);
  };
  auto process = [&](u32x4 (&kreg)[2][4], u32x4 (&vreg)[8], int t, auto more, auto last) {
    bf16x8 kop[2][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int j = 0; j < 4; ++j) kop[mt][j] = as_bf16x8(kreg[mt][j]);
    f32x4 sc[NT][2];
    red.scores(kop, sc);
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(vstage + (4 * i + quad) * kVPitch + 16 * col) = vreg[i];
    if constexpr (decltype(more)::value) load(kreg, vreg, t + kUnitWaves);
    bf16x8 pb[1][NT];
    red.softmax(sc, u.end - t * kKeysPerTile, last, pb);
    __builtin_amdgcn_wave_barrier();
    const unsigned char* vrow = vstage + (quad * 4 + (col >> 2)) * kVPitch + 8 * (col & 3);
    red.pv(pb, [&](int mt, int nn) { return vrow + mt * 16 * kVPitch + 32 * nn; }, std::false_type{});
    __builtin_amdgcn_wave_barrier();
  };
  int t = u.t0 + wave;
  if (t < u.t1) {
    u32x4 kreg[2][4], vreg[8];
    load(kreg, vreg, t);
    for (; t + kUnitWaves < u.t1; t += kUnitWaves) process(kreg, vreg, t, std::true_type{}, std::false_type{});
    process(kreg, vreg, t, std::false_type{}, std::true_type{});
  }
  red.close();
  __syncthreads();  // every wave is done with its stage
  float* slots = reinterpret_cast<float*>(smem);
  publish_wave(red, slots, wave, lane);
  __syncthreads();

  // wave w merges the states for output dims [32w, 32w + 32)
  constexpr int SV = kSlotVals<8>;
  auto slot = [&](int w) { return slots + (size_t)w * (NT * SV * 64); };
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float wk[kUnitWaves], M = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < kUnitWaves; ++w) M = fmaxf(M, slot(w)[nt * SV * 64 + lane]);
#pragma unroll
    for (int w = 0; w < kUnitWaves; ++w) {
      wk[w] = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(slot(w)[nt * SV * 64 + lane] - M);
      l = fmaf(wk[w], slot(w)[(nt * SV + 1) * 64 + lane], l);
    }
    f32x4 o[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kUnitWaves; ++w)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[i][e] = fmaf(wk[w], slot(w)[(nt * SV + 2 + (2 * wave + i) * 4 + e) * 64 + lane], o[i][e]);
    }
    const int r = nt * 16 + col;
    if (r >= rows) continue;
    const RowPlace at = place_of(p, u, kvh, r);
    const float m = holds<true>(l) ? M * kLn2 : -INFINITY;
    if (u.state0 < 0) {
      const float inv = holds<true>(l) ? 1.0f / l : 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        *reinterpret_cast<uint2*>(p.out + at.out * D + 16 * (2 * wave + i) + 4 * quad) =
            make_uint2(pack_bf16x2(o[i][0] * inv, o[i][1] * inv), pack_bf16x2(o[i][2] * inv, o[i][3] * inv));
      if (p.lse && wave == 0 && quad == 0) p.lse[at.out] = holds<true>(l) ? m + logf(l) : -INFINITY;
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        *reinterpret_cast<f32x4*>(p.o_part + at.state * D + 16 * (2 * wave + i) + 4 * quad) = o[i];
      if (wave == 0 && quad == 0) {
        p.m_part[at.state] = m;
        p.l_part[at.state] = l;
      }
    }
  }
}

// More rows: each wave holds 16 NT of them, and all waves read the same tiles,
// which come straight into LDS, kStages - 1 ahead.  A wave loads a quarter of
// each tile; one barrier a tile, between the wait for a tile and the loads into
// the stage that the tile before it has left.  Only whole tiles (shared keys).
template <int NT>
__device__ __forceinline__ void shared_unit(const PrefixParams& p, const Unit& u, unsigned char* smem, int lane,
                                            int wave) {
  const int rows = u.rows_kvh & 255, kvh = u.rows_kvh >> 8;
  const int col = lane & 15, quad = lane >> 4;
  const uint32_t rs = (uint32_t)p.H_KV * (D * 2);
  TileReducer<NT, 8> red;
  red.scale_log2 = p.scale_log2;
  red.quad = quad;
  Pages pages;
  pages.start(p, u, lane);
  // block i of a tile: rows 4 i + [0, 4); position l % 16 of row r holds chunk (l % 16 - 2 r) mod 16 (tile.h)
  const int rr = lane >> 4, cp = lane & 15;
  const bool isv = wave >= 2;
  const int blk0 = (wave & 1) * 4;
  uint32_t off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    off[i] = (uint32_t)(4 * (blk0 + i) + rr) * rs + 16u * (uint32_t)((cp - 2 * rr) & 15);
  auto fetch = [&](int stage, int t) {
    int64_t elems;
    const bool in = pages.tile(p, t, kvh, lane, elems);
    const uint32_t bytes = (uint32_t)__builtin_amdgcn_readfirstlane(in ? 31u * rs + D * 2u : 0u);
    const __amdgpu_buffer_rsrc_t r = make_rsrc((isv ? p.v : p.k) + elems, bytes);
    unsigned char* at = smem + stage * kStageBytes + (isv ? kLdsTileBytes : 0) + blk0 * kBlockStride;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(at + i * kBlockStride), 16, off[i], 0, 0, 0);
  };
  uint32_t kro[2][4], vro[2][8];
  {
    const int kr = col & 3, vk = col >> 2, vm = col & 3;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        kro[mt][j] = lds_offset(smem) + (uint32_t)((4 * mt + (col >> 2)) * kBlockStride + kr * 256 +
                                                   16 * ((4 * j + quad + 2 * kr) & 15));
#pragma unroll
      for (int nn = 0; nn < 8; ++nn)
        vro[mt][nn] = lds_offset(smem) + (uint32_t)(kLdsTileBytes + (4 * mt + quad) * kBlockStride + vk * 256 +
                                                    16 * ((2 * nn + (vm >> 1) + 2 * vk) & 15) + 8 * (vm & 1));
    }
  }
  const int n = u.t1 - u.t0;
  for (int i = 0; i < kStages - 1 && i < n; ++i) fetch(i, u.t0 + i);
  load_rows(red, p, u, kvh, rows, wave * 16 * NT, col, quad);
  red.reset();
  // one tile: `ahead` tiles' loads stay in flight
  auto step = [&](auto stage, int i) {
    constexpr uint32_t so = decltype(stage)::value * kStageBytes;
    if (i + 2 < n)
      asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else if (i + 1 < n)
      asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (i + kStages - 1 < n) fetch((decltype(stage)::value + kStages - 1) % kStages, u.t0 + i + kStages - 1);
    bf16x8 kop[2][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        kop[mt][j] = as_bf16x8(
            *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>((uintptr_t)(kro[mt][j] + so)));
    f32x4 sc[NT][2];
    red.scores(kop, sc);
    bf16x8 pb[1][NT];
    red.softmax(sc, kKeysPerTile, std::false_type{}, pb);
    red.pv(pb, [&](int mt, int nn) { return vro[mt][nn] + so; }, std::true_type{});
  };
  static_assert(kStages == 4, "the loop below takes the stages in turn");
  int i = 0;
  for (; i + 4 <= n; i += 4) {
    step(std::integral_constant<int, 0>{}, i);
    step(std::integral_constant<int, 1>{}, i + 1);
    step(std::integral_constant<int, 2>{}, i + 2);
    step(std::integral_constant<int, 3>{}, i + 3);
  }
  if (i < n) step(std::integral_constant<int, 0>{}, i);
  if (i + 1 < n) step(std::integral_constant<int, 1>{}, i + 1);
  if (i + 2 < n) step(std::integral_constant<int, 2>{}, i + 2);
  red.close();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = wave * 16 * NT + nt * 16 + col;
    if (r >= rows) continue;
    const RowPlace at = place_of(p, u, kvh, r);
#pragma unroll
    for (int nn = 0; nn < 8; ++nn)
      *reinterpret_cast<f32x4*>(p.o_part + at.state * D + 16 * nn + 4 * quad) = red.o[nt][nn];
    if (quad == 0) {
      p.m_part[at.state] = holds<true>(red.l[nt]) ? red.m[nt] * kLn2 : -INFINITY;
      p.l_part[at.state] = red.l[nt];
    }
  }
}

__global__ void __launch_bounds__(64 * kUnitWaves, 2) unit_kernel(PrefixParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int total = __builtin_amdgcn_readfirstlane(p.head[0]);
  for (int w = blockIdx.x; w < total; w += gridDim.x) {
    // the unit, one integer a lane
    const int word = reinterpret_cast<const int32_t*>(p.units + w)[lane & 7];
    Unit u;
    u.table = __builtin_amdgcn_readlane(word, 0);
    u.end = __builtin_amdgcn_readlane(word, 1);
    u.t0 = __builtin_amdgcn_readlane(word, 2);
    u.t1 = __builtin_amdgcn_readlane(word, 3);
    u.seq0 = __builtin_amdgcn_readlane(word, 4);
    u.row0 = __builtin_amdgcn_readlane(word, 5);
    u.rows_kvh = __builtin_amdgcn_readlane(word, 6);
    u.state0 = __builtin_amdgcn_readlane(word, 7);
    const int rows = u.rows_kvh & 255;
    if (rows == 0) continue;
    __syncthreads();  // the unit before is done with the LDS
    // opaque, so that the addresses of all four kinds are not kept (and spilled) from unit to unit
    int ln = lane;
    asm volatile("" : "+v"(ln));
    if (rows <= 16)
      stream_unit<1>(p, u, smem, ln, wave);
    else if (rows <= 32)
      stream_unit<2>(p, u, smem, ln, wave);
    else if (rows <= 64)
      shared_unit<1>(p, u, smem, ln, wave);
    else
      shared_unit<2>(p, u, smem, ln, wave);
  }
}

// ---------------------------------------------------------------- merge

// A wave a row: states of the shared chunks, then of the row's own, in order.
// Lane i holds maximum and sum of chunk i of either kind, and output dims 2i and
// 2i + 1.
__global__ void __launch_bounds__(256) merge_kernel(PrefixParams p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + wave);
  if (row >= p.B * p.H_Q) return;
  const int b = div_by(row, p.div_hq), h = row - b * p.H_Q;
  const SeqStates s = p.seqs[b];
  if (s.own < 0) return;
  const int n = s.chunks + s.own;
  auto state = [&](int i) {
    return (int64_t)h + (i < s.chunks ? s.shared + (int64_t)i * s.stride : s.own0 + (int64_t)(i - s.chunks) * p.H_Q);
  };
  float m[2], l[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bool in = 64 * i + lane < n;
    m[i] = in ? p.m_part[state(64 * i + lane)] : -INFINITY;
    l[i] = in ? p.l_part[state(64 * i + lane)] : 0.f;
  }
  constexpr int kBatch = 16;
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  f32x2 a[kBatch];
  auto load = [&](int i0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (i0 + u < n) a[u] = *reinterpret_cast<const f32x2*>(p.o_part + state(i0 + u) * D + 2 * lane);
  };
  load(0);
  float M = -INFINITY, w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) M = fmaxf(M, holds<true>(l[i]) ? m[i] : -INFINITY);
  M = wave_max(M);
#pragma unroll
  for (int i = 0; i < 2; ++i) w[i] = holds<true>(l[i]) ? __builtin_amdgcn_exp2f((m[i] - M) * kLog2e) : 0.f;
  float L = 0.f, o0 = 0.f, o1 = 0.f;
  for (int i0 = 0; i0 < n; i0 += kBatch) {
    if (i0 > 0) load(i0);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (i0 + u >= n) break;
      const int i = i0 + u;
      const float wi = lane_value(i < 64 ? w[0] : w[1], i & 63), li = lane_value(i < 64 ? l[0] : l[1], i & 63);
      const bool live = holds<true>(li);
      L = fmaf(wi, li, L);
      o0 = fmaf(wi, live ? a[u].x : 0.f, o0);
      o1 = fmaf(wi, live ? a[u].y : 0.f, o1);
    }
  }
  const float inv = holds<true>(L) ? 1.0f / L : 0.f;
  *reinterpret_cast<uint32_t*>(p.out + (int64_t)row * D + 2 * lane) = pack_bf16x2(o0 * inv, o1 * inv);
  if (p.lse && lane == 0) p.lse[row] = holds<true>(L) ? M + logf(L) : -INFINITY;
}

// ---------------------------------------------------------------- host side

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? (int)DA_OK : da::fail(DA_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

// Sizes of a call's workspace: room for what the plan may choose, and at the
// least for one chunk of each prefix and of each sequence.
struct PrefixSizes {
  int64_t units, rows;
  size_t unit_at, seq_at, o_at, m_at, l_at, total;
};

PrefixSizes prefix_sizes(int B, int G, int H_Q, int H_KV, int cus) {
  const int64_t slots = 2 * cus, g = H_Q / H_KV;
  const int hpt = da::heads_per_tile(H_Q, H_KV, 1);
  const int64_t readers = g / hpt;
  PrefixSizes z{};
  // row tiles of all groups, their streams in whole bundles of 8
  const int64_t tiles = B * g / kSharedRows + G;
  z.units = 4 * slots + tiles * (H_KV + 7) + B * readers * (H_KV + (readers > 1 ? 7 : 0));
  z.rows = kSharedRows * slots + 2ll * B * H_Q;
  auto up = [](int64_t x) { return (size_t)((x + 255) / 256 * 256); };
  z.unit_at = 256;
  z.seq_at = z.unit_at + up(z.units * (int64_t)sizeof(Unit));
  z.o_at = z.seq_at + up(B * (int64_t)sizeof(SeqStates));
  z.m_at = z.o_at + up(z.rows * D * 4);
  z.l_at = z.m_at + up(z.rows * 4);
  z.total = z.l_at + up(z.rows * 4) + DA_ARRIVAL_BYTES;
  return z;
}

// Shapes the call takes; units and state rows are numbered with 32 bits.
int check_prefix_shape(int B, int G, int H_Q, int H_KV, int L_K_max, int d) {
  const int rc = da::check_shape(B, H_Q, H_KV, L_K_max, d);
  if (rc) return rc;
  if (B > DA_MAX_REQUESTS) return da::fail(DA_ERR_SHAPE, "B=%d exceeds %d", B, DA_MAX_REQUESTS);
  if (G < 0 || G > B) return da::fail(DA_ERR_SHAPE, "%d groups of %d sequences", G, B);
  if (H_KV > (1 << 16) || (int64_t)B * H_Q > (1 << 22))
    return da::fail(DA_ERR_SHAPE, "B=%d sequences of %d heads (%d KV heads) are too many for one call", B, H_Q, H_KV);
  return DA_OK;
}

}  // namespace

extern "C" {

size_t da_prefix_workspace_bytes(int B, int G, int H_Q, int H_KV, int num_cus) {
  if (check_prefix_shape(B, G, H_Q, H_KV, 0, D)) return 0;
  if (num_cus <= 0 && ensure_gfx950(&num_cus)) return 0;
  return prefix_sizes(B, G, H_Q, H_KV, num_cus).total;
}

int da_decode_attn_prefix(const void* q, const void* k_cache, const void* v_cache, const int32_t* block_table,
                          const int32_t* seq_lens, const int32_t* cu_groups, const int32_t* prefix_lens, void* out,
                          float* lse_out, int B, int G, int H_Q, int H_KV, int page_size, int max_pages, int num_pages,
                          int L_K_max, int d, float softmax_scale, int chunk_keys, void* workspace,
                          size_t workspace_bytes, void* stream) {
  da::clear_error();
  int rc = check_prefix_shape(B, G, H_Q, H_KV, L_K_max, d);
  if (!q || !out) return da::fail(DA_ERR_NULL, "q and out must be non-NULL");
  if (!block_table || !seq_lens) return da::fail(DA_ERR_NULL, "block_table and seq_lens must be non-NULL");
  if (G > 0 && (!cu_groups || !prefix_lens)) return da::fail(DA_ERR_NULL, "cu_groups and prefix_lens must be non-NULL");
  if ((!k_cache || !v_cache) && !(rc == DA_OK && L_K_max == 0))
    return da::fail(DA_ERR_NULL, "k_cache and v_cache must be non-NULL");
  if (rc) return rc;
  rc = da::check_page_table(B, page_size, max_pages, num_pages, L_K_max);
  if (rc) return rc;
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16))
    return da::fail(DA_ERR_ALIGN, "q, k_cache, v_cache and out must be 16-byte aligned");
  for (const void* x : {(const void*)block_table, (const void*)seq_lens, (const void*)cu_groups,
                        (const void*)prefix_lens, (const void*)lse_out})
    if (!aligned(x, 4)) return da::fail(DA_ERR_ALIGN, "tables, lengths, groups and lse_out must be 4-byte aligned");
  if (workspace && !aligned(workspace, 16)) return da::fail(DA_ERR_ALIGN, "workspace must be 16-byte aligned");
  int cus = 0;
  rc = ensure_gfx950(&cus);
  if (rc) return rc;
  const PrefixSizes z = prefix_sizes(B, G, H_Q, H_KV, cus);
  if (!workspace || workspace_bytes < z.total)
    return da::fail(DA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", z.total, workspace ? workspace_bytes : 0);
  PrefixParams p{};
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k_cache);
  p.v = static_cast<const uint16_t*>(v_cache);
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.cu = cu_groups;
  p.prefix_lens = prefix_lens;
  p.out = static_cast<uint16_t*>(out);
  p.lse = lse_out;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  p.head = reinterpret_cast<int32_t*>(ws);
  p.units = reinterpret_cast<Unit*>(ws + z.unit_at);
  p.seqs = reinterpret_cast<SeqStates*>(ws + z.seq_at);
  p.o_part = reinterpret_cast<float*>(ws + z.o_at);
  p.m_part = reinterpret_cast<float*>(ws + z.m_at);
  p.l_part = reinterpret_cast<float*>(ws + z.l_at);
  p.most_rows = z.rows;
  p.most_units = (int)z.units;
  p.B = B;
  p.G = G;
  p.H_Q = H_Q;
  p.H_KV = H_KV;
  p.g = H_Q / H_KV;
  p.hpt = da::heads_per_tile(H_Q, H_KV, 1);
  p.L_K = L_K_max;
  p.page_size = page_size;
  p.max_pages = max_pages;
  p.num_pages = num_pages;
  p.slots = 2 * cus;
  p.chunk_tiles = chunk_keys > 0 ? (int)(((int64_t)chunk_keys + kKeysPerTile - 1) / kKeysPerTile) : 0;
  p.div_page = make_div((uint32_t)page_size);
  p.div_g = make_div((uint32_t)p.g);
  p.div_heads = make_div((uint32_t)H_KV);
  p.div_hq = make_div((uint32_t)H_Q);
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)D)) * kLog2e;
  hipStream_t s = static_cast<hipStream_t>(stream);
  void* args[] = {&p};
  const int plan_smem = 4 * (4 * B + 5 * G + 1);
  rc = launched(hipLaunchKernel(reinterpret_cast<const void*>(&plan_kernel), dim3(1), dim3(kPlanThreads), args, plan_smem, s),
                "prefix plan");
  if (rc) return rc;
  rc = launched(hipLaunchKernel(reinterpret_cast<const void*>(&unit_kernel), dim3((uint32_t)p.slots),
                                dim3(64 * kUnitWaves), args, unit_smem(), s),
                "prefix attention");
  if (rc) return rc;
  return launched(hipLaunchKernel(reinterpret_cast<const void*>(&merge_kernel), dim3((uint32_t)((B * (int64_t)H_Q + 3) / 4)),
                                  dim3(256), args, 0, s),
                  "prefix merge");
}

}  // extern "C"
