// Decode attention of a batch whose sequences share prefixes.  Where the batch
// may hold enough keys for that to pay, three launches: its work cut into units on
// the device (plan_kernel), the chunk states of the units (unit_kernel), and their
// merge (merge_kernel).  Else the one launch of the windowed call, which reads
// shared keys for each sequence.  Entry points at the end.
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
  int32_t* head;      // workspace: units there are (in whole eights)
  uint32_t* tickets;  // of each XCD's lists, 128 bytes apart: the groups' units taken, the sequences'
  Unit* units;
  SeqStates* seqs;
  float* o_part;
  float* m_part;
  float* l_part;
  int64_t most_rows;  // state rows there is room for
  int most_units;
  int B, G, H_Q, H_KV, g, hpt, L_K, page_size, max_pages, num_pages;
  int slots;          // workgroups that run at once
  int own_tiles;      // head tiles of a KV head
  int chunk_tiles;    // 0: chosen on the device
  Div div_page, div_g, div_hq, div_readers, div_tiles;
  float scale_log2;
};

// ---------------------------------------------------------------- plan

constexpr int kFewGroups = 16;    // the chunks of so many are weighed against each other; of more, any will do
constexpr float kUnitTiles = 24;  // what a unit of a group costs besides its tiles, in tiles
constexpr int kWhole = 1 << 26;  // tiles: longer than any sequence

__device__ __forceinline__ int chunks_of(int tiles, int length) {
  const int n = (int)((uint32_t)(tiles + length - 1) / (uint32_t)length);
  return n < kMostGroupChunks ? n : kMostGroupChunks;
}

__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

// One workgroup.  A group's shared keys are its prefix length, or its shortest
// sequence's that has keys if that is less, in whole tiles; a group of one such
// sequence shares none.  They are cut into chunks for tiles of up to 128 of the
// group's query rows, and what each sequence has behind them into chunks for
// the heads of each KV head, by the rules beside the lengths below.  Units are
// dealt round robin to the XCDs; the row tiles of a chunk, which read the same
// keys, stand 8 apart, one behind the other in one XCD's list.
// Bound by latency (barriers, dependent LDS reads, a cold instruction cache).
template <int kPlanThreads>
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(PrefixParams p) {
  constexpr int kPlanWaves = kPlanThreads / 64;
  extern __shared__ int32_t lds[];
  __shared__ int4 sums[kPlanWaves];
  __shared__ int fit[kPlanWaves];
  __shared__ int backwards[kPlanWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* tiles = lds;            // [B] keys, then tiles of the sequence's own keys
  int32_t* group = tiles + p.B;    // [B] its group, or -1
  int32_t* unit_b = group + p.B;   // [B] its first chunk, counted over the batch
  int32_t* state_b = unit_b + p.B; // [B] its first state row / H_Q
  int32_t* cu = state_b + p.B;     // [G + 1]
  int32_t* shared = cu + p.G + 1;  // [G] shared keys, then tiles
  int32_t* reader = shared + p.G;  // [G] its first sequence that has keys
  int32_t* unit_g = reader + p.G;  // [G] sequences that have keys, then its first unit
  int32_t* state_g = unit_g + p.G; // [G]

  if (tid < 16) p.tickets[32 * tid] = 0;
  bool back = false;
  for (int i = tid; i < p.G; i += kPlanThreads) {
    const int c0 = max(0, min(p.cu[i], p.B)), c1 = max(0, min(p.cu[i + 1], p.B));
    back |= c0 > c1;
    cu[i] = c0;
    if (i == p.G - 1) cu[p.G] = c1;
    shared[i] = max(0, min(p.prefix_lens[i], p.L_K));
    reader[i] = p.B;
    unit_g[i] = 0;
  }
  for (int b = tid; b < p.B; b += kPlanThreads) tiles[b] = max(0, min(p.seq_lens[b], p.L_K));
  back = __any(back);
  if (lane == 0) backwards[wave] = back;
  __syncthreads();
  int G = p.G;
  for (int w = 0; w < kPlanWaves; ++w) G = backwards[w] ? 0 : G;  // groups that run backwards share nothing
  for (int b = tid; b < p.B; b += kPlanThreads) {
    const int L = tiles[b];
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
    // a sequence without keys belongs to no group
    if (L == 0) group[b] = -1;
    tiles[b] = L > 0 ? (L + kKeysPerTile - 1) / kKeysPerTile - first : 0;
  }
  __syncthreads();

  const int own_tiles = p.own_tiles;  // head tiles of a KV head
  auto row_tiles = [&](int i) { return ((cu[i + 1] - cu[i]) * p.g + kSharedRows - 1) / kSharedRows; };
  // units of `streams` streams of keys that `readers` units each read
  auto units_of = [&](int streams, int readers) { return readers == 1 ? streams : (streams + 7) / 8 * 8 * readers; };
  const int own_readers = p.H_KV * own_tiles;  // units that read a sequence's chunk, together whole rows of it
  // Lengths by the work there is; wave w tries them 2^w times as long, and the first that fit the workspace are taken.
  int length_g, length_b;
  int waves;  // of a workgroup that take a sequence's own chunks, each by itself; 0: a chunk is a workgroup's work
  {
    int work_g = 0, work_b = 0;
    for (int i = lane; i < G; i += 64) work_g += (int)min((int64_t)shared[i] * row_tiles(i), (int64_t)1 << 16);
    for (int b = lane; b < p.B; b += 64) work_b += min(tiles[b], 1 << 16);
    work_g = min(wave_total(work_g), (1 << 30) / p.H_KV) * p.H_KV;
    work_b = min(wave_total(work_b), (1 << 30) / (p.H_KV * own_tiles)) * (p.H_KV * own_tiles);
    // About a unit a CU of shared keys (128 tiles at most: more are dealt as they run out).  Shorter ones write more
    // states, whose merge costs as much: 32 sequences over 8192 keys in 256 units of 16 tiles 38.8 us, in 512 of 8 47.8;
    // 128 over 16384, with own parts, in units of 128 tiles 145 us, of 64 151.
    // Half as many of a sequence's own keys, a workgroup each.  Where there are many, a wave each: by four waves of a
    // workgroup, or by two where the shared keys are the larger work, whose tiles would wait behind them (128 sequences of
    // 100 to 1500 own keys, by two and by four: over 16384 shared ones 144 and 157 us, over 8192 134 and 117).  Chunks are
    // as long as two shares of the first waves (64 of 100 to 2000 keys over 8192: one share 87.5, two 84, four 110), or half
    // of one where there are two (the 144 us: 136).
    // Few long sequences are few chunks and so few waves: one of 800 000 keys, 8/1 heads, takes 454 us (the windowed call
    // 128), three of 20480, 64/16, 97 (90).
    waves = work_b < 24 * p.slots ? 0 : work_b > work_g ? 4 : 2;
    length_g = p.chunk_tiles > 0 ? p.chunk_tiles : min(max(work_g / (p.slots / 2), 4), 128);
    length_b = p.chunk_tiles > 0 ? p.chunk_tiles
               : waves > 0       ? min(max(waves == 2 ? work_b / (2 * p.slots) : work_b / p.slots, 8), 64)
                                 : min(max(work_b / (p.slots / 4), 4), 64);
    if (G <= kFewGroups && p.chunk_tiles == 0) {
      // A lane a length, from half of that to two and a half times: of the rounds in which the CUs take the units, and what
      // one costs, the least product (three groups of 64 sequences over 8192 keys: 288 units of 86 tiles, two rounds, 163 us;
      // 192 of 128 129).
      const int tried = max(length_g * (16 + lane) / 32, 4);
      const float of_length = __builtin_amdgcn_rcpf((float)tried);
      float units = 0.f, longest = 0.f;
      for (int i = 0; i < G; ++i) {
        const float T = (float)shared[i], n = fminf(ceilf(T * of_length - 1e-3f), (float)kMostGroupChunks);
        units = fmaf(n, (float)row_tiles(i), units);
        longest = fmaxf(longest, n > 0.f ? T * __builtin_amdgcn_rcpf(n) : 0.f);
      }
      const float cost = ceilf(units * (float)p.H_KV / (float)(p.slots / 2)) * (longest + kUnitTiles);
      const uint64_t least = __ballot(cost == -wave_max(-cost));
      length_g = __builtin_amdgcn_readlane(tried, least ? 63 - __builtin_clzll(least) : 16);
    }
    auto longer = [&](int length, int w) { return (int)min((int64_t)length << w, (int64_t)kWhole); };
    int w = 0;
    for (;; w += kPlanWaves) {
      const int lg = longer(length_g, w + wave), lb = longer(length_b, w + wave);
      int units = 0, rows = 0, chunks = 0;
      for (int i = lane; i < G; i += 64) {
        const int n = chunks_of(shared[i], lg);
        units += units_of(n * p.H_KV, row_tiles(i));
        rows += n * (cu[i + 1] - cu[i]);
      }
      for (int b = lane; b < p.B; b += 64) chunks += chunks_of(tiles[b], lb);
      rows += chunks;
      const int u = wave_total(min(units, 1 << 24)), r = wave_total(min(rows, 1 << 24));
      const int64_t own_units = (int64_t)((wave_total(chunks) + 7) / 8 * 8) * own_readers;
      const bool fits = u + 7 <= p.most_units && own_units <= p.most_units && (int64_t)r * p.H_Q <= p.most_rows;
      if (lane == 0) fit[wave] = fits;
      __syncthreads();
      int k = 0;
      while (k < kPlanWaves && !fit[k]) ++k;
      if (k < kPlanWaves || w + kPlanWaves >= 32) {  // whole prefixes and sequences always fit
        w += k;
        break;
      }
      __syncthreads();
    }
    length_g = longer(length_g, min(w, 31));
    length_b = longer(length_b, min(w, 31));
  }

  // first units and state rows: groups, then sequences, each thread some in a row
  const int per_g = (G + kPlanThreads - 1) / kPlanThreads, g0 = min(tid * per_g, G), g1 = min(g0 + per_g, G);
  const int per_b = (p.B + kPlanThreads - 1) / kPlanThreads, b0 = min(tid * per_b, p.B), b1 = min(b0 + per_b, p.B);
  // states of a sequence's own chunks; one that shares nothing and has one chunk writes its output
  auto state_chunks = [&](int b, int n) { return n == 1 && (group[b] < 0 || shared[group[b]] == 0) ? 0 : n; };
  int4 mine = make_int4(0, 0, 0, 0);
  for (int i = g0; i < g1; ++i) {
    const int n = chunks_of(shared[i], length_g);
    unit_g[i] = mine.x;
    state_g[i] = mine.y;
    mine.x += units_of(n * p.H_KV, row_tiles(i));
    mine.y += n * (cu[i + 1] - cu[i]);
  }
  for (int b = b0; b < b1; ++b) {
    const int n = chunks_of(tiles[b], length_b);
    unit_b[b] = mine.z;
    state_b[b] = mine.w;
    mine.z += n;
    mine.w += state_chunks(b, n);
  }
  int4 upto = make_int4(wave_scan(mine.x), wave_scan(mine.y), wave_scan(mine.z), wave_scan(mine.w));
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int4 all = make_int4(0, 0, 0, 0), before = make_int4(upto.x - mine.x, upto.y - mine.y, upto.z - mine.z, upto.w - mine.w);
  for (int w = 0; w < kPlanWaves; ++w) {
    const int4 x = sums[w];
    if (w < wave) before = make_int4(before.x + x.x, before.y + x.y, before.z + x.z, before.w + x.w);
    all = make_int4(all.x + x.x, all.y + x.y, all.z + x.z, all.w + x.w);
  }
  for (int i = g0; i < g1; ++i) {
    unit_g[i] += before.x;
    state_g[i] += before.y;
  }
  for (int b = b0; b < b1; ++b) {
    unit_b[b] += before.z;
    state_b[b] += all.y + before.w;
  }
  __syncthreads();
  for (int b = tid; b < p.B; b += kPlanThreads) {
    const int n = chunks_of(tiles[b], length_b), at = group[b];
    const int shared_chunks = at >= 0 ? chunks_of(shared[at], length_g) : 0;
    SeqStates s;
    s.shared = shared_chunks ? (state_g[at] + (b - cu[at])) * p.H_Q : 0;
    s.chunks = shared_chunks;
    s.stride = shared_chunks ? (cu[at + 1] - cu[at]) * p.H_Q : 0;
    s.own0 = state_b[b] * p.H_Q;
    s.own = n > 0 && state_chunks(b, n) == 0 ? -1 : n;
    p.seqs[b] = s;
  }
  // two lists, each in whole eights: the groups' units, then the sequences', whose chunks are dealt to the XCDs and
  // read there by all heads one behind the other
  const int padded = (all.x + 7) / 8 * 8, total = padded + (all.z + 7) / 8 * 8 * own_readers;
  if (tid == 0) {
    p.head[0] = padded;
    p.head[1] = total - padded;
    p.head[2] = waves;
  }
  for (int i = tid; i < padded; i += kPlanThreads) {
    Unit u{};
    if (i < all.x) {
      int lo = 0, hi = G;  // the last group that starts at or before it
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (unit_g[mid] <= i)
          lo = mid;
        else
          hi = mid;
      }
      const uint32_t T = (uint32_t)shared[lo], n = (uint32_t)chunks_of((int)T, length_g);
      const uint32_t readers = (uint32_t)row_tiles(lo);
      uint32_t stream = (uint32_t)(i - unit_g[lo]), reader_at = 0;
      if (readers > 1) {
        const uint32_t bundle = stream / (8 * readers), in = stream - bundle * 8 * readers;
        reader_at = in / 8;
        stream = bundle * 8 + in % 8;
      }
      const int kvh = (int)(stream / n);
      const uint32_t chunk = stream - (uint32_t)kvh * n;
      if (kvh < p.H_KV) {  // else it fills a bundle
        const int size = cu[lo + 1] - cu[lo];
        u.table = reader[lo];
        u.end = (int)T * kKeysPerTile;
        u.t0 = (int)(T * chunk / n);  // T < 2^26, at most 64 chunks
        u.t1 = (int)(T * (chunk + 1) / n);
        u.seq0 = cu[lo];
        u.row0 = (int)reader_at * kSharedRows;
        u.rows_kvh = min(size * p.g - u.row0, kSharedRows) | kvh << 8;
        u.state0 = (state_g[lo] + (int)chunk * size) * p.H_Q;
      }
    }
    p.units[i] = u;
  }
  // a sequence's chunk for one of its readers: chunk number c of the batch stands c mod 8 in bundle c / 8
  auto own_place = [&](int number, int own_reader) {
    return p.units + p.most_units + (int64_t)(number / 8) * 8 * own_readers + 8 * own_reader + number % 8;
  };
  for (int i = tid; i < p.B * own_readers; i += kPlanThreads) {
    const int b = div_by(i, p.div_readers), own_reader = i - b * own_readers;
    const uint32_t T = (uint32_t)tiles[b];
    const int n = chunks_of((int)T, length_b), first = group[b] < 0 ? 0 : shared[group[b]];
    const int kvh = div_by(own_reader, p.div_tiles);
    Unit u;
    u.table = b;
    u.end = max(0, min(p.seq_lens[b], p.L_K));
    u.seq0 = b;
    u.row0 = (own_reader - kvh * own_tiles) * p.hpt;
    u.rows_kvh = p.hpt | kvh << 8;
    for (int chunk = 0; chunk < n; ++chunk) {
      u.t0 = first + (int)(T * (uint32_t)chunk / (uint32_t)n);
      u.t1 = first + (int)(T * (uint32_t)(chunk + 1) / (uint32_t)n);
      u.state0 = n == 1 && first == 0 ? -1 : (state_b[b] + chunk) * p.H_Q;
      *own_place(unit_b[b] + chunk, own_reader) = u;
    }
  }
  const int fill = (8 - all.z % 8) % 8;  // of the last bundle
  for (int i = tid; i < fill * own_readers; i += kPlanThreads) {
    const int own_reader = i / fill;
    *own_place(all.z + i - own_reader * fill, own_reader) = Unit{};
  }
}

// ---------------------------------------------------------------- units

constexpr int kWaveStage = kKeysPerTile * (kVPitch + kKPitch);  // a wave's own tile of V and of K
constexpr int kStages = 4;
constexpr int kStageBytes = 2 * kLdsTileBytes;  // K and V of one tile
constexpr int unit_smem() {
  int most = kStages * kStageBytes;
  most = std::max(most, kUnitWaves * kWaveStage);
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

// One wave over the tiles t, t + STEP, ... of a unit of 16 NT rows or fewer: K
// and V by way of LDS (`vstage`, the wave's own), the next tile's loads in flight.
// ready(): called between the first loads and the first use of the LDS.
// Single waves (STEP 1) stream: 64 sequences of 500 to 4000 own keys, 64/8 heads,
// 140 -> 131 us.  Where several units read the same keys it costs instead: 128/1
// heads and 64 sequences of 1000 to 8000 97 -> 105, 37/1 258 -> 435.
template <int NT, typename Step, typename Ready>
__device__ __forceinline__ void stream_tiles(const PrefixParams& p, const Unit& u, TileReducer<NT, 8>& red,
                                             unsigned char* vstage, int t, Step, int lane, Ready ready) {
  constexpr int STEP = Step::value;
  constexpr int AUX = STEP == 1 ? 2 : 0;
  const int rows = u.rows_kvh & 255, kvh = u.rows_kvh >> 8;
  const int col = lane & 15, quad = lane >> 4;
  const uint32_t rs = (uint32_t)p.H_KV * (D * 2);
  Pages pages;
  pages.start(p, u, lane);
  red.scale_log2 = p.scale_log2;
  red.quad = quad;
  load_rows(red, p, u, kvh, rows, 0, col, quad);
  red.reset();
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
        kreg[mt][j] = __builtin_amdgcn_raw_buffer_load_b128(kt, (uint32_t)(16 * mt + 4 * j + quad) * rs + 16u * col, 0, AUX);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      vreg[i] = __builtin_amdgcn_raw_buffer_load_b128(vt, (uint32_t)(4 * i + quad) * rs + 16u * col, 0, AUX);
  };
  auto process = [&](u32x4 (&kreg)[2][4], u32x4 (&vreg)[8], int t, auto more, auto last) {
    unsigned char* kstage = vstage + kKeysPerTile * kVPitch;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<u32x4*>(kstage + (16 * mt + 4 * j + quad) * kKPitch + 16 * col) = kreg[mt][j];
    __builtin_amdgcn_wave_barrier();
    bf16x8 kop[2][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        kop[mt][j] = as_bf16x8(*reinterpret_cast<const u32x4*>(kstage + (16 * mt + col) * kKPitch + 16 * (4 * j + quad)));
    f32x4 sc[NT][2];
    red.scores(kop, sc);
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(vstage + (4 * i + quad) * kVPitch + 16 * col) = vreg[i];
    if constexpr (decltype(more)::value) load(kreg, vreg, t + STEP);
    bf16x8 pb[1][NT];
    red.softmax(sc, u.end - t * kKeysPerTile, last, pb);
    __builtin_amdgcn_wave_barrier();
    const unsigned char* vrow = vstage + (quad * 4 + (col >> 2)) * kVPitch + 8 * (col & 3);
    red.pv(pb, [&](int mt, int nn) { return vrow + mt * 16 * kVPitch + 32 * nn; }, std::false_type{});
    __builtin_amdgcn_wave_barrier();
  };
  u32x4 kreg[2][4], vreg[8];
  if (t < u.t1) load(kreg, vreg, t);
  ready();
  if (t < u.t1) {
    for (; t + STEP < u.t1; t += STEP) process(kreg, vreg, t, std::true_type{}, std::false_type{});
    process(kreg, vreg, t, std::false_type{}, std::true_type{});
  }
  red.close();
}

// 16 NT rows or fewer by a workgroup: the waves take one tile in four, and their
// states meet in LDS at the end (in wave order).
template <int NT, typename Next>
__device__ __forceinline__ void stream_unit(const PrefixParams& p, const Unit& u, unsigned char* smem, int lane,
                                            int wave, Next& next) {
  const int rows = u.rows_kvh & 255, kvh = u.rows_kvh >> 8;
  const int col = lane & 15, quad = lane >> 4;
  next.take();  // units of this kind are short: the ticket for the next one is here before they end
  TileReducer<NT, 8> red;
  stream_tiles(p, u, red, smem + wave * kWaveStage, u.t0 + wave, std::integral_constant<int, kUnitWaves>{},
               lane, [] { __syncthreads(); });  // the unit before is done with the LDS
  next.post();
  __syncthreads();  // every wave is done with its stage
  float* slots = reinterpret_cast<float*>(smem);
  publish_wave(red, slots, wave, lane);
  next.fetch();
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
      wk[w] = __builtin_amdgcn_exp2f(slot(w)[nt * SV * 64 + lane] - M);
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

// The same by one wave, tile after tile, without the others: what a batch of many
// sequences has behind its prefixes.
template <int NT, typename Ready>
__device__ __forceinline__ void wave_unit(const PrefixParams& p, const Unit& u, unsigned char* smem, int lane, int wave,
                                          Ready ready) {
  const int rows = u.rows_kvh & 255, kvh = u.rows_kvh >> 8;
  const int col = lane & 15, quad = lane >> 4;
  TileReducer<NT, 8> red;
  stream_tiles(p, u, red, smem + wave * kWaveStage, u.t0, std::integral_constant<int, 1>{}, lane, ready);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = nt * 16 + col;
    if (r >= rows) continue;
    const RowPlace at = place_of(p, u, kvh, r);
    const float l = red.l[nt], m = holds<true>(l) ? red.m[nt] * kLn2 : -INFINITY;
    if (u.state0 < 0) {
      const float inv = holds<true>(l) ? 1.0f / l : 0.f;
#pragma unroll
      for (int nn = 0; nn < 8; ++nn)
        *reinterpret_cast<uint2*>(p.out + at.out * D + 16 * nn + 4 * quad) =
            make_uint2(pack_bf16x2(red.o[nt][nn][0] * inv, red.o[nt][nn][1] * inv),
                       pack_bf16x2(red.o[nt][nn][2] * inv, red.o[nt][nn][3] * inv));
      if (p.lse && quad == 0) p.lse[at.out] = holds<true>(l) ? m + logf(l) : -INFINITY;
    } else {
#pragma unroll
      for (int nn = 0; nn < 8; ++nn)
        *reinterpret_cast<f32x4*>(p.o_part + at.state * D + 16 * nn + 4 * quad) = red.o[nt][nn];
      if (quad == 0) {
        p.m_part[at.state] = m;
        p.l_part[at.state] = l;
      }
    }
  }
}

// More rows: each wave holds 16 NT of them, and all waves read the same tiles,
// which come straight into LDS (rings of kStages tiles of K and of V; two waves
// load K, two V, half a tile each).  The scores of tile i + 1 are multiplied
// while the softmax of tile i is taken: K runs one tile ahead of V, so that a
// tile's products, exponentials and LDS reads do not wait for each other.  One
// barrier a tile, between the wait for a tile and the loads into the place that
// the tile before it has left.  Only whole tiles (shared keys).
template <int NT>
struct SharedRows {
  bf16x8 q[NT][4];
  float m[NT], l[NT];  // running maximum (log2 units) and this lane's part of the sum
  f32x4 o[NT][8];
};

// The largest of three, NaN where one is (v_maximum3_f32): fmaxf would have every product quieted first.  The compiler has
// to see that a product's result is read, and puts the wait there that the hardware does not have; it sees into no assembly.
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// max_rows (tile.h) with it.
__device__ __forceinline__ float top_of_rows(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __builtin_elementwise_maximum(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto c = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(c[0]), __uint_as_float(c[1]));
}

template <int NT, typename Next>
__device__ __forceinline__ void shared_unit(const PrefixParams& p, const Unit& u, unsigned char* smem, int lane,
                                            int wave, Next& next) {
  const int rows = u.rows_kvh & 255, kvh = u.rows_kvh >> 8;
  const int col = lane & 15, quad = lane >> 4;
  const uint32_t rs = (uint32_t)p.H_KV * (D * 2);
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
  // tiles in order; only where a page ends is the next one's place worked out
  const uint16_t* const pool = isv ? p.v : p.k;
  unsigned char* const ring = smem + (isv ? kStages * kLdsTileBytes : 0) + blk0 * kBlockStride;
  const uint16_t* at_tile = nullptr;
  uint32_t tile_bytes = 0;
  int next_tile = u.t0, in_page = 0;
  auto fetch = [&](int stage) {
    if (in_page == 0) {
      int64_t elems;
      const bool in = pages.tile(p, next_tile, kvh, lane, elems);
      at_tile = pool + elems;
      tile_bytes = in ? 31u * rs + D * 2u : 0u;
      const int key = next_tile * kKeysPerTile;
      in_page = (p.page_size - (key - div_by(key, p.div_page) * p.page_size)) / kKeysPerTile;
    }
    const __amdgpu_buffer_rsrc_t r = make_rsrc(at_tile, tile_bytes);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(ring + stage * kLdsTileBytes + i * kBlockStride), 16, off[i],
                                               0, 0, 0);
    at_tile += kKeysPerTile * (rs / 2);
    --in_page;
    ++next_tile;
  };
  // K and V of a tile as operands: where this lane's pieces of the tile's first half lie; those of the second, and of the
  // ring's other places, lie a constant further on
  uint32_t kro[4], vro[8];
  {
    const int kr = col & 3, vk = col >> 2, vm = col & 3;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      kro[j] = lds_offset(smem) +
               (uint32_t)((col >> 2) * kBlockStride + kr * 256 + 16 * ((4 * j + quad + 2 * kr) & 15));
#pragma unroll
    for (int nn = 0; nn < 8; ++nn)
      vro[nn] = lds_offset(smem) + (uint32_t)(kStages * kLdsTileBytes + quad * kBlockStride + vk * 256 +
                                              16 * ((2 * nn + (vm >> 1) + 2 * vk) & 15) + 8 * (vm & 1));
  }
  const int n = u.t1 - u.t0;
  // K waves run one tile further ahead
  const int deep = isv ? kStages - 1 : kStages;
  __syncthreads();  // the unit before is done with the LDS
  for (int i = 0; i < deep && i < n; ++i) fetch(i);
  SharedRows<NT> red;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    // rows past the unit's repeat its last one; nothing of theirs is stored
    const uint16_t* row = p.q + place_of(p, u, kvh, min(wave * 16 * NT + nt * 16 + col, rows - 1)).out * D + 8 * quad;
#pragma unroll
    for (int j = 0; j < 4; ++j) red.q[nt][j] = as_bf16x8(*reinterpret_cast<const u32x4*>(row + 32 * j));
    red.m[nt] = kNoScore;
    red.l[nt] = 0.f;
#pragma unroll
    for (int nn = 0; nn < 8; ++nn) red.o[nt][nn] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // of the ring's place `at`, a constant, `more` bytes behind it
  auto read_k = [&](bf16x8 (&kop)[2][4], auto at, uint32_t more) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        kop[mt][j] = as_bf16x8(*reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(
            (uintptr_t)(kro[j] + more + decltype(at)::value * kLdsTileBytes + mt * 4 * kBlockStride)));
  };
  // V of a tile, transposed (TileReducer::pv).  In assembly with its wait: for the
  // compiler's own form of the instruction it waits for every load into LDS.
  auto read_v = [&](s16x4 (&lo)[8], s16x4 (&hi)[8], auto at, uint32_t more) {
    constexpr int kFirst = decltype(at)::value * kLdsTileBytes, kSecond = kFirst + 4 * kBlockStride;
    static_assert(kSecond < 65536, "an offset has 16 bits");
    uint32_t from[8];
#pragma unroll
    for (int nn = 0; nn < 8; ++nn) from[nn] = vro[nn] + more;
#define DA_READ(lo, hi, i)                              \
  "ds_read_b64_tr_b16 %" #lo ", %" #i " offset:%24\n" \
  "ds_read_b64_tr_b16 %" #hi ", %" #i " offset:%25\n"
    asm volatile(DA_READ(0, 8, 16) DA_READ(1, 9, 17) DA_READ(2, 10, 18) DA_READ(3, 11, 19) DA_READ(4, 12, 20)
                     DA_READ(5, 13, 21) DA_READ(6, 14, 22) DA_READ(7, 15, 23) "s_waitcnt lgkmcnt(0)"
                 : "=&v"(lo[0]), "=&v"(lo[1]), "=&v"(lo[2]), "=&v"(lo[3]), "=&v"(lo[4]), "=&v"(lo[5]), "=&v"(lo[6]),
                   "=&v"(lo[7]), "=&v"(hi[0]), "=&v"(hi[1]), "=&v"(hi[2]), "=&v"(hi[3]), "=&v"(hi[4]), "=&v"(hi[5]),
                   "=&v"(hi[6]), "=&v"(hi[7])
                 : "v"(from[0]), "v"(from[1]), "v"(from[2]), "v"(from[3]), "v"(from[4]), "v"(from[5]), "v"(from[6]),
                   "v"(from[7]), "n"(kFirst), "n"(kSecond)
                 : "memory");
#undef DA_READ
  };
  auto scores = [&](const bf16x8 (&kop)[2][4], f32x4 (&sc)[NT][2]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) sc[nt][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
          sc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[mt][j], red.q[nt][j], sc[nt][mt], 0, 0, 0);
  };
  // Waits until all but two of this wave's tiles are there (`left` where that is less), then for the other waves.
  auto arrive = [&](int left) {
    if (left >= 2)
      asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else if (left == 1)
      asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  float tops[NT];  // of the scores in hand, over the rows' keys
  auto top_of = [&](const f32x4 (&sc)[NT][2]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const f32x4 a = sc[nt][0], c = sc[nt][1];
      const float last = __builtin_elementwise_maximum(c[2], c[3]);
      tops[nt] = p.scale_log2 * top_of_rows(max3(max3(a[0], a[1], a[2]), max3(a[3], c[0], c[1]), last));
    }
  };
  // Tile i from its scores `sc` and their maxima `tops`; leaves those of tile i + 1 there.  The tiles lie in the ring's
  // places at0 and at1, s0 and s1 bytes further on.  full: the loads go on behind tile i as far as the rings reach; more:
  // there is a tile i + 1.
  auto step = [&](f32x4 (&sc)[NT][2], int i, auto at0, auto at1, uint32_t s0, uint32_t s1, int place, auto more,
                  auto full) {
    // K(i + 1) and V(i) are needed, K up to i + 3 and V up to i + 2 on their way
    if constexpr (decltype(full)::value) {
      arrive(2);
      fetch((place + deep) % kStages);
    } else {
      arrive(decltype(more)::value ? (isv ? n - 1 - i : n - 2 - i) : 0);
      if (i + deep < n) fetch((place + deep) % kStages);
    }
    bf16x8 kop[2][4];
    if constexpr (decltype(more)::value) read_k(kop, at1, s1);
    // The maximum follows at once, so that a row's largest probability is exactly 1 (with a slack of 2^8 the products with
    // the old state's weight were rarer and 128 sequences over 16384 keys 5% faster, but the error against 64 bits 2.2e-3
    // and not 1.8e-3); 16 rows at a time, most tiles move none of them.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (__any(tops[nt] > red.m[nt])) {
        const float m = fmaxf(red.m[nt], tops[nt]);
        const float alpha = __builtin_amdgcn_exp2f(red.m[nt] - m);
        red.m[nt] = m;
        red.l[nt] *= alpha;
#pragma unroll
        for (int nn = 0; nn < 8; ++nn) red.o[nt][nn] *= alpha;
      }
    }
    f32x4 next[NT][2];
    if constexpr (decltype(more)::value) scores(kop, next);
    bf16x8 pb[NT];
    float xs[NT][8];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float(&x)[8] = xs[nt];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(sc[nt][e / 4][e % 4], p.scale_log2, -red.m[nt]));
      pb[nt] = as_bf16x8(u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                               pack_bf16x2(x[6], x[7])});
    }
    __builtin_amdgcn_sched_barrier(0);
    s16x4 vlo[8], vhi[8];
    read_v(vlo, vhi, at0, s0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float(&x)[8] = xs[nt];
      red.l[nt] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
#pragma unroll
    for (int nn = 0; nn < 8; ++nn) {
      const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vlo[nn], vhi[nn], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        red.o[nt][nn] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[nt], red.o[nt][nn], 0, 0, 0);
    }
    if constexpr (decltype(more)::value) {
      top_of(next);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) sc[nt][mt] = next[nt][mt];
    }
    // What the compiler would leave for the next step, which begins with a wait, is done behind this one's products, two
    // vector instructions each (128 sequences over 16384 shared keys alone 118 -> 111 us).
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) asm volatile("" : "+v"(red.l[nt]), "+v"(tops[nt]));
#pragma unroll
    for (int i = 0; i < 8 * NT; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr std::integral_constant<int, 0> place0{};
  f32x4 sc[NT][2];
  {
    arrive(n - 1);  // K(0)
    bf16x8 kop[2][4];
    read_k(kop, place0, 0u);
    scores(kop, sc);
    top_of(sc);
  }
  static_assert(kStages == 4, "the loop below takes the stages in turn");
  constexpr uint32_t T = kLdsTileBytes;
  constexpr std::integral_constant<int, 1> place1{};
  constexpr std::integral_constant<int, 2> place2{};
  constexpr std::integral_constant<int, 3> place3{};
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  int i = 0;
  for (; i + 3 + kStages < n; i += 4) {
    step(sc, i, place0, place1, 0, 0, 0, yes, yes);
    step(sc, i + 1, place1, place2, 0, 0, 1, yes, yes);
    step(sc, i + 2, place2, place3, 0, 0, 2, yes, yes);
    step(sc, i + 3, place3, place0, 0, 0, 3, yes, yes);
  }
  for (; i + 1 < n; ++i) step(sc, i, place0, place0, (uint32_t)(i & 3) * T, (uint32_t)((i + 1) & 3) * T, i & 3, yes, no);
  next.take();
  step(sc, i, place0, place0, (uint32_t)(i & 3) * T, 0, i & 3, no, no);
  next.post();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float l = sum_rows(red.l[nt]);
    const int r = wave * 16 * NT + nt * 16 + col;
    if (r >= rows) continue;
    const RowPlace at = place_of(p, u, kvh, r);
#pragma unroll
    for (int nn = 0; nn < 8; ++nn)
      *reinterpret_cast<f32x4*>(p.o_part + at.state * D + 16 * nn + 4 * quad) = red.o[nt][nn];
    if (quad == 0) {
      p.m_part[at.state] = holds<true>(l) ? red.m[nt] * kLn2 : -INFINITY;
      p.l_part[at.state] = l;
    }
  }
  __syncthreads();
  next.fetch();
}

__device__ __forceinline__ Unit unit_of(int word) {  // one integer a lane
  Unit u;
  u.table = __builtin_amdgcn_readlane(word, 0);
  u.end = __builtin_amdgcn_readlane(word, 1);
  u.t0 = __builtin_amdgcn_readlane(word, 2);
  u.t1 = __builtin_amdgcn_readlane(word, 3);
  u.seq0 = __builtin_amdgcn_readlane(word, 4);
  u.row0 = __builtin_amdgcn_readlane(word, 5);
  u.rows_kvh = __builtin_amdgcn_readlane(word, 6);
  u.state0 = __builtin_amdgcn_readlane(word, 7);
  return u;
}

// A workgroup's way through one of its XCD's lists: a ticket (thread 0), the
// unit's number for all (after post and a barrier), and the unit's words.
struct Next {
  const Unit* list;
  uint32_t* tickets;
  int* place;  // LDS, two: one is written while slow waves may still read the other
  int n, given;  // units of the list; of them given out without tickets
  int xcd, tid, lane;
  int turn, index, word;  // index < 0: none left
  uint32_t ticket;
  __device__ __forceinline__ void take() {
    if (given < n && tid == 0) ticket = __hip_atomic_fetch_add(tickets, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ __forceinline__ void post() {
    if (tid == 0) place[turn] = (uint32_t)given + ticket < (uint32_t)n ? given + (int)ticket : -1;
  }
  __device__ __forceinline__ void fetch() {
    index = __builtin_amdgcn_readfirstlane(place[turn]);
    turn ^= 1;
    load();
  }
  __device__ __forceinline__ void load() {
    if (index >= 0) word = reinterpret_cast<const int32_t*>(list + 8 * index + xcd)[lane & 7];
  }
  __device__ __forceinline__ void skip() {
    take();
    post();
    __syncthreads();
    fetch();
  }
};

// Each XCD has a list of the groups' units (bound by the matrix cores where they
// have many rows) and one of the sequences' own (bound by memory).  Up to half of
// its workgroups begin with the second, so that both kinds share the CUs, and
// each list is worked off by whoever comes to it: the first unit by the
// workgroup's number, the others by tickets.  A unit's result does not depend on
// who computes it.  Where there are many own units a wave takes one by itself.
__global__ void __launch_bounds__(64 * kUnitWaves, 2) unit_kernel(PrefixParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ int place[2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int xcd = blockIdx.x & 7, at = blockIdx.x >> 3, slots = gridDim.x >> 3;
  // the unit that the workgroup begins with, if it begins with one of a group's: loaded along with the lists' lengths
  const int begins = reinterpret_cast<const int32_t*>(p.units + 8 * at + xcd)[lane & 7];
  const int n_group = __builtin_amdgcn_readfirstlane(p.head[0]) / 8;
  const int n_own = __builtin_amdgcn_readfirstlane(p.head[1]) / 8;
  const int own_waves = __builtin_amdgcn_readfirstlane(p.head[2]);
  const bool by_wave = own_waves > 0;
  const int need = by_wave ? (n_own + own_waves - 1) >> (own_waves == 2 ? 1 : 2) : n_own;  // workgroups that the own units can use
  const int front = min(slots - min(slots / 2, need), n_group);
  // workgroups [0, front) begin with the groups' units, the others with the sequences'
  const int own_given = (slots - front) * (by_wave ? own_waves : 1);
  // one body for both lists: the kernel is long, and what a CU has not run yet it fetches in the middle of its work
#pragma nounroll
  for (int turn = 0; turn < 2; ++turn) {
    const bool of_group = (turn == 0) == (at < front);
    Next list{of_group ? p.units : p.units + p.most_units, p.tickets + 64 * xcd + (of_group ? 0 : 32), place,
              of_group ? n_group : n_own, of_group ? front : own_given, xcd, tid, lane, 0, -1, 0, 0};
    if (!of_group && by_wave) {
      auto take = [&]() {
        uint32_t t = 0;
        if (own_given < n_own && lane == 0)
          t = __hip_atomic_fetch_add(list.tickets, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return t;
      };
      auto number = [&](uint32_t t) {
        const uint32_t i = (uint32_t)own_given + (uint32_t)__builtin_amdgcn_readfirstlane((int)t);
        return own_given < n_own && i < (uint32_t)n_own ? (int)i : n_own;
      };
      auto words = [&](int i) {
        return i < n_own ? reinterpret_cast<const int32_t*>(list.list + 8 * i + xcd)[lane & 7] : 0;
      };
      int i = wave >= own_waves ? n_own : turn == 0 ? (at - front) * own_waves + wave : number(take());
      int word = words(i);
      while (i < n_own) {
        const Unit u = unit_of(word);
        const uint32_t t = take();
        // the next unit's words are on their way while this one's tiles are read
        auto ready = [&]() {
          i = number(t);
          word = words(i);
        };
        int ln = lane;
        asm volatile("" : "+v"(ln));
        if ((u.rows_kvh & 255) == 0)
          ready();
        else if ((u.rows_kvh & 255) <= 16)
          wave_unit<1>(p, u, smem, ln, wave, ready);
        else
          wave_unit<2>(p, u, smem, ln, wave, ready);
      }
      __syncthreads();
      continue;
    }
    if (turn == 0) {
      list.index = of_group ? at : at - front < n_own ? at - front : -1;
      list.word = begins;
      if (!of_group) list.load();
    } else if (list.given < list.n) {
      list.skip();
    }
    while (list.index >= 0) {
      const Unit u = unit_of(list.word);
      const int rows = u.rows_kvh & 255;
      // opaque, so that the addresses of all kinds are not kept (and spilled) from unit to unit
      int ln = lane;
      asm volatile("" : "+v"(ln));
      if (rows == 0)  // fills a bundle
        list.skip();
      else if (rows <= 16)
        stream_unit<1>(p, u, smem, ln, wave, list);
      else if (rows <= 32)
        stream_unit<2>(p, u, smem, ln, wave, list);
      else if (rows <= 64)
        shared_unit<1>(p, u, smem, ln, wave, list);
      else
        shared_unit<2>(p, u, smem, ln, wave, list);
    }
    __syncthreads();
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

// Bytes of K and V that the batch's sequences hold at most, shared keys counted for each, up to which they are all read:
// what is shared then comes out of L2 and the last-level cache at twice HBM's rate and more, and one launch does.  By
// those bytes, this call's sharing launches and the one launch (us; 64/8 heads): 5 MB 15 and 6.6, 75 MB 23 and 8.1, 276
// MB 30 and 18, 330 MB 30 and 25, 598 MB 34 and 43, 1140 MB 41 and 79.  Groups of more than 16 heads need the matrix
// cores twice as long for as many bytes: 32/1 heads 270 MB 42 and 27, 1080 MB 76 and 76.
// The bound decides, not the lengths: two sequences of 530 keys under one of 131072 17.6 us, by the one launch 8.9.
constexpr int64_t kUnsharedBytes = 384ll << 20;

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
  // of either list: row tiles of all groups, their streams in whole bundles of 8, or a chunk of each sequence
  const int64_t tiles = B * g / kSharedRows + G;
  z.units = 16 + 8 * slots + std::max<int64_t>(tiles * (H_KV + 7), (B + 7ll) * H_KV * readers);
  z.rows = kSharedRows * slots + 2ll * B * H_Q;
  auto up = [](int64_t x) { return (size_t)((x + 255) / 256 * 256); };
  z.unit_at = 256 + 16 * 128;
  z.seq_at = z.unit_at + up(2 * z.units * (int64_t)sizeof(Unit));
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
  const int64_t bytes = (int64_t)B * L_K_max * H_KV * D * 4;
  if (chunk_keys == 0 && workspace && workspace_bytes >= z.total && bytes <= kUnsharedBytes * (H_Q / H_KV > 16 ? 2 : 1)) {
    // a window that hides nothing, in as much workspace as this call asks for, taken at the end (where the counters are): a
    // larger one does not change which launches run, and with them the result's last bits
    const size_t spare = (workspace_bytes - z.total) / 256 * 256;
    const int rc1 = da_decode_attn_window(q, k_cache, v_cache, nullptr, block_table, seq_lens, page_size, max_pages,
                                          num_pages, out, lse_out, B, H_Q, H_KV, L_K_max, d, softmax_scale,
                                          std::max(L_K_max, 1), 0, 0, -1, static_cast<unsigned char*>(workspace) + spare,
                                          workspace_bytes - spare, stream);
    // more chunk states than that holds, or than one launch may write
    if (rc1 != DA_ERR_WORKSPACE && rc1 != DA_ERR_SHAPE) return rc1;
    da::clear_error();
  }
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
  p.tickets = reinterpret_cast<uint32_t*>(ws + 256);
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
  p.own_tiles = p.g / p.hpt;
  p.chunk_tiles = chunk_keys > 0 ? (int)(((int64_t)chunk_keys + kKeysPerTile - 1) / kKeysPerTile) : 0;
  p.div_page = make_div((uint32_t)page_size);
  p.div_g = make_div((uint32_t)p.g);
  p.div_hq = make_div((uint32_t)H_Q);
  p.div_readers = make_div((uint32_t)(H_KV * p.own_tiles));
  p.div_tiles = make_div((uint32_t)p.own_tiles);
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)D)) * kLog2e;
  hipStream_t s = static_cast<hipStream_t>(stream);
  void* args[] = {&p};
  const int plan_smem = 4 * (4 * B + 5 * G + 1);
  // few sequences: a wave a SIMD, whose instructions do not wait for three others' (B=2: 6.9 -> 5.9 us)
  const int plan_threads = (int64_t)B * H_KV <= 512 ? 256 : 1024;
  const void* plan = plan_threads == 256 ? reinterpret_cast<const void*>(&plan_kernel<256>)
                                         : reinterpret_cast<const void*>(&plan_kernel<1024>);
  rc = launched(hipLaunchKernel(plan, dim3(1), dim3(plan_threads), args, plan_smem, s), "prefix plan");
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
