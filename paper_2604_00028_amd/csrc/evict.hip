// A cache that is bounded by eviction: the attention weight each key received
// (weights_kernel), and the choice of the rows that stay (select_kernel) with
// their way into the places that come free (move_kernel).  Entry points at the
// end.
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

// ---------------------------------------------------------------- weights

constexpr int kWeightWaves = 4;
constexpr int kMostChunkTiles = 64;  // page ids of a chunk: one a lane

struct WeightParams {
  const uint16_t* q;
  const uint16_t* k;
  const int32_t* block_table;
  const int32_t* seq_lens;
  const float* lse;
  const float* in;
  float* out;
  int64_t stride;  // floats between the rows of two heads
  int B, H_Q, H_KV, g, L_K, page_size, max_pages, num_pages;
  int chunk_tiles, chunks;
  Div div_page, div_chunks, div_heads;
  float scale_log2, decay;
};

// out_j = decay in_j + sum_h exp(scale q_h k_j - lse_h) over the g query heads
// of a KV head.  A workgroup takes `chunk_tiles` tiles of 32 keys of one
// (sequence, KV head), its waves one tile in four; a wave's product has the
// heads as rows and the keys as columns (S = Q K^T, the operands of the
// attention kernels' S^T exchanged), so that a key's sum over 16 heads is three
// additions and two lane exchanges.  K is loaded row by row and takes its operand
// layout by way of LDS, the next tile's loads in flight while one is reduced.
// exp(x) = 2^(raw scale log2 e - lse log2 e), one fma and one exponential a
// score; in 32 bits throughout.  Up to 16 NT heads stay in registers; more (g >
// 64) are read anew for each tile.  AUX: the loads' cache policy (2: streaming).
//
// Bound by HBM: 32 sequences of 8192 keys of 8 heads (535 MB of K, 17 of
// weights) 95 us, 5.8 TB/s; K straight into the operand layout 112.
template <int NT, int AUX>
__global__ void __launch_bounds__(64 * kWeightWaves) weights_kernel(WeightParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  // the heads of a chunk side by side, and each sequence's chunks turned by one: chunks that only long sequences have
  // would else be the work of a few XCDs
  const int item = div_by((int)blockIdx.x, p.div_heads), kvh = (int)blockIdx.x - item * p.H_KV;
  const int b = div_by(item, p.div_chunks);
  const int turned = item - b * p.chunks + (b - div_by(b, p.div_chunks) * p.chunks);
  const int chunk = turned < p.chunks ? turned : turned - p.chunks;
  const int L = min(p.seq_lens[b], p.L_K);
  const int tiles = L > 0 ? (L + kKeysPerTile - 1) / kKeysPerTile : 0;
  const int first = chunk * p.chunk_tiles;
  const int end = min(first + p.chunk_tiles, tiles);
  int t = first + wave;
  if (t >= end) return;  // waves are independent
  const int pg0 = div_by(first * kKeysPerTile, p.div_page);
  const int pg1 = div_by(end * kKeysPerTile - 1, p.div_page);
  const int pages = pg0 + lane <= pg1 ? p.block_table[(int64_t)b * p.max_pages + pg0 + lane] : 0;

  const uint32_t rs = (uint32_t)p.H_KV * (D * 2);
  const int64_t row0 = (int64_t)b * p.H_Q + (int64_t)kvh * p.g;
  const __amdgpu_buffer_rsrc_t qr = make_rsrc(p.q + row0 * D, (uint32_t)p.g * (D * 2));
  const __amdgpu_buffer_rsrc_t lr = make_rsrc(p.lse + row0, (uint32_t)p.g * 4u);
  bf16x8 q[NT][4];
  float base[NT][4];  // -lse log2 e; -inf for rows past the heads, and for heads that saw nothing
  auto load_heads = [&](int h0) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        q[nt][j] = as_bf16x8(__builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       qr, (uint32_t)(h0 + nt * 16 + col) * (D * 2) + 64u * j + 16u * quad, 0, 0)));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int h = h0 + nt * 16 + quad * 4 + e;
        const float l = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(lr, (uint32_t)h * 4u, 0, 0));
        base[nt][e] = h < p.g && l != -INFINITY ? -l * kLog2e : -INFINITY;
      }
    }
  };
  load_heads(0);

  const float* in = p.in + ((int64_t)b * p.H_KV + kvh) * p.stride;
  float* out = p.out + ((int64_t)b * p.H_KV + kvh) * p.stride;
  const bool keep = p.decay != 0.f;
  __shared__ __attribute__((aligned(16))) unsigned char stages[kWeightWaves][kKeysPerTile * kKPitch];
  unsigned char* const stage = stages[wave];
  auto load = [&](u32x4 (&k)[2][4], float& old, int t) {
    const int key = t * kKeysPerTile, j = div_by(key, p.div_page);
    const int page = __builtin_amdgcn_readlane(pages, (j - pg0) & 63);
    const bool in_pool = page >= 0 && page < p.num_pages;  // a page outside the cache reads as zero keys
    const int rows = min(L - key, kKeysPerTile);
    const int64_t prow = (in_pool ? (int64_t)page : 0) * p.page_size + (key - j * p.page_size);
    const __amdgpu_buffer_rsrc_t kr =
        make_rsrc(p.k + (prow * p.H_KV + kvh) * D,
                  (uint32_t)__builtin_amdgcn_readfirstlane(in_pool ? (uint32_t)(rows - 1) * rs + D * 2u : 0u));
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        k[mt][i] = __builtin_amdgcn_raw_buffer_load_b128(kr, (uint32_t)(16 * mt + 4 * i + quad) * rs + 16u * col, 0, AUX);
    old = keep && lane < rows ? in[key + lane] : 0.f;
  };
  // rows of the tile to LDS, and back as operands: lane (col, quad) of (mt, i) holds dims [32 i + 8 quad, + 8) of key 16 mt + col
  auto put = [&](const u32x4 (&k)[2][4]) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u32x4*>(stage + (16 * mt + 4 * i + quad) * kKPitch + 16 * col) = k[mt][i];
    __builtin_amdgcn_wave_barrier();
  };
  auto reduce = [&](float old, int t) {
    u32x4 k[2][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        k[mt][i] = *reinterpret_cast<const u32x4*>(stage + (16 * mt + col) * kKPitch + 16 * (4 * i + quad));
    __builtin_amdgcn_wave_barrier();
    float sum[2] = {0.f, 0.f};
    for (int h0 = 0; h0 < p.g; h0 += 16 * NT) {
      if (NT == 4 && p.g > 64) load_heads(h0);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[nt][i], as_bf16x8(k[mt][i]), s, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e)  // an infinite key times a row of no head is NaN
            sum[mt] += base[nt][e] != -INFINITY ? __builtin_amdgcn_exp2f(fmaf(s[e], p.scale_log2, base[nt][e])) : 0.f;
        }
    }
    const float s0 = sum_rows(sum[0]), s1 = sum_rows(sum[1]);
    const int key = t * kKeysPerTile + lane;
    if (lane < kKeysPerTile && key < L) {
      const float w = lane < 16 ? s0 : s1;
      out[key] = keep ? fmaf(p.decay, old, w) : w;
    }
  };
  u32x4 k[2][4];
  float old;
  load(k, old, t);
  for (; t + kWeightWaves < end; t += kWeightWaves) {
    put(k);
    const float was = old;
    load(k, old, t + kWeightWaves);
    reduce(was, t);
  }
  put(k);
  reduce(old, t);
}

// ---------------------------------------------------------------- eviction

constexpr int kBins = 4096;       // of the second and third digit; of the first 256, in kCopies
constexpr int kCopies = 16;
constexpr int kListed = kBins / 2;  // moves whose rows are listed in LDS, in the histogram's place
constexpr int kMostKeys = 32768;    // keys that stay in LDS
constexpr int kMoveRows = 64;  // rows a workgroup of move_kernel takes at a time
constexpr int kFew = 5;        // evicted rows that are found one after the other
constexpr uint32_t kGates = 16;   // counters of workgroups that have ended
constexpr int kMovedAtOnce = 64;  // moves of a (sequence, KV head) that select_kernel makes itself

struct EvictParams {
  const int32_t* block_table;
  const int32_t* seq_lens;
  const int32_t* totals;
  const float* w_in;
  const int32_t* p_in;
  float* w_out;
  int32_t* p_out;
  int64_t stride;
  int32_t* moves;      // workspace: per (sequence, KV head) a count, then `most` target rows and `most` source rows
  int64_t move_ints;   // integers of one
  int most;
  int B, H_KV, L_K, budget, sinks, recent, page_size, max_pages, num_pages;
  Div div_page, div_heads;
  // moves, lengths and pages
  uint16_t* k;
  uint16_t* v;
  int32_t* lens_out;
  int32_t* free_pages;
  const int32_t* taken;
  int32_t* taken_out;   // nullable: pages are not given back
  int num_free;
  uint32_t* arrivals;   // no second launch: the workgroups that have ended
  int groups;           // workgroups a (sequence, KV head)
  Div div_groups;
};

// Weights in the order of unsigned numbers; NaN below all, both zeros alike.
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  return w != w ? 0u : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Sum over lanes 0 to 15's values before lane `n` (n <= 16, uniform).
__device__ __forceinline__ int row_sum_before(int x, int n) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  const int upto = __builtin_amdgcn_readlane(x, (n + 15) & 15);
  return n > 0 ? upto : 0;
}

// Sums of x and y over the threads before this one; *total: over all.  One
// barrier: `sums` is this call's own.
template <int WAVES>
__device__ __forceinline__ int2 scan_before(int x, int y, int2* sums, int2* total) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int sx = wave_scan(x), sy = wave_scan(y);
  if (lane == 63) sums[wave] = make_int2(sx, sy);
  __syncthreads();
  const int2 s = lane < WAVES ? sums[lane] : make_int2(0, 0);
  *total = make_int2(row_sum_before(s.x, 16), row_sum_before(s.y, 16));
  return make_int2(sx - x + row_sum_before(s.x, wave), sy - y + row_sum_before(s.y, wave));
}

// Keys of a sequence.  Where they are more than L_K, the rows past them may have no
// weights (whose stride need only hold L_K) and the sequence stays as it is: cut to
// L_K rows it would take later tokens' positions for its first ones, and lose the
// pages behind.  One that has had no more than L_K tokens holds no more keys.
__device__ __forceinline__ int counted(const EvictParams& p, int length, int total) {
  return length > p.L_K && total <= p.L_K ? p.L_K : max(0, length);
}

__device__ __forceinline__ int length_of(const EvictParams& p, int b) {
  return b < p.B ? counted(p, p.seq_lens[b], p.totals[b]) : 0;
}

// The lengths after the eviction, and the pages that come free: sequences in order,
// THREADS at a time, their pages past the budget by one scan, then a page a
// thread, its sequence by bisection.  One workgroup, after all others have read
// the lengths; length0: that of sequence `thread`, in_use: pages of the list.
template <int THREADS>
__device__ __forceinline__ void give_back(const EvictParams& p, int length0, int in_use) {
  constexpr int WAVES = THREADS / 64;
  const int tid = threadIdx.x;
  __shared__ int2 sums[2][WAVES];
  __shared__ int32_t starts[THREADS];
  const int first_page = (p.budget + p.page_size - 1) / p.page_size;
  auto length = [&](int b) { return b < THREADS ? length0 : length_of(p, b); };
  auto pages_gone = [&](int L) { return L > p.budget && L <= p.L_K ? div_by(L - 1, p.div_page) + 1 - first_page : 0; };
  const int taken = p.taken_out ? max(0, min(in_use, p.num_free)) : 0;
  int2 sum;
  int all = 0, done = 0;  // pages of all sequences, and of those before b0
  if (p.taken_out && p.B > THREADS) {
    for (int b = tid; b < p.B; b += THREADS) all += pages_gone(length(b));
    scan_before<WAVES>(all, 0, sums[0], &sum);
    all = sum.x;
  }
  for (int b0 = 0; b0 < p.B; b0 += THREADS) {
    const int L = length(b0 + tid);
    if (p.taken_out) {
      starts[tid] = scan_before<WAVES>(pages_gone(L), 0, sums[1], &sum).x;
      if (p.B <= THREADS) all = sum.x;
      const int at0 = taken - all + done;  // the place of the first page; the list has none for those below 0
      __syncthreads();
      for (int e = tid; e < sum.x; e += THREADS) {
        int lo = 0, hi = THREADS;  // the last sequence that starts at or before e
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (starts[mid] <= e)
            lo = mid;
          else
            hi = mid;
        }
        if (at0 + e >= 0)
          p.free_pages[at0 + e] = p.block_table[(int64_t)(b0 + lo) * p.max_pages + first_page + (e - starts[lo])];
      }
      done += sum.x;
      __syncthreads();
    }
    if (b0 + tid < p.B) p.lens_out[b0 + tid] = L > p.L_K ? L : min(L, p.budget);
  }
  if (p.taken_out && tid == 0) *p.taken_out = max(0, taken - all);
}

// The least of a row of 16 lanes, for each of them.
__device__ __forceinline__ uint64_t least_of_row(uint64_t x) {
  auto step = [&](auto turn) {
    constexpr int kTurn = 0x120 + decltype(turn)::value;  // row_ror
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, kTurn, 0xf, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), kTurn, 0xf, 0xf, false);
    const uint64_t y = (uint64_t)hi << 32 | lo;
    x = y < x ? y : x;
  };
  step(std::integral_constant<int, 8>{});
  step(std::integral_constant<int, 4>{});
  step(std::integral_constant<int, 2>{});
  step(std::integral_constant<int, 1>{});
  return x;
}

// The rows of one (sequence, KV head) that stay.  With more than `budget` rows,
// those of the `budget` largest keys do, where a key is the row's weight (all
// ones for a protected row), of equal ones the lowest rows.  The budget-th
// largest key comes from three histograms in LDS of 8, 12 and 12 bits: each
// fixes the bits of its digit and the number still to be found among the keys
// that share them.  Weights agree in their first bits, and additions to one
// address go one after the other, so the first histogram has a copy for each of
// 16 lanes.  A thread then ranks `each` consecutive rows: one scan over the
// threads numbers the equal keys, and another the evicted rows below the budget
// (holes) and the kept ones above it: the i-th of these moves into the i-th
// hole, in place and without an order among the moves.
//
// Up to kFew evicted rows, as where every step of a decode brings one, are found
// one after the other as the smallest key left, 1 us each where the histograms
// take 6, and the rows past the budget are loaded before it is known which stay.
//
// Bound by latency: one pass over weights and positions, coalesced, whose keys
// stay in LDS (KEEP; longer sequences read both anew for each step), two lookups
// a move.  32 sequences of 8 heads one key past 4096, in a graph: 9.6 us with all
// that follows (an empty kernel 2.5, the pass over the keys 2.6, the choice 1.3,
// the moves 0.8, the last workgroup's part the rest); eight past it 15.1 (about
// ten barriers).  With a thread's rows in registers, loaded and stored `each`
// apart, and one copy of the first histogram the choice by histograms took half as
// long again.
template <int THREADS, bool KEEP>
__device__ __forceinline__ void select_rows(const EvictParams& p) {
  constexpr int WAVES = THREADS / 64;
  static_assert(32 * kFew <= THREADS, "32 threads hold a row past the budget");
  static_assert(WAVES <= 16 && THREADS >= 256, "the waves' sums are scanned by 16 lanes; 256 threads have a first digit each");
  extern __shared__ uint32_t keys[];  // KEEP: [L_K]
  __shared__ __attribute__((aligned(16))) uint32_t hist[kBins];
  __shared__ int2 sums[5][WAVES];
  __shared__ uint32_t found[3][2];
  __shared__ int32_t pages[KEEP ? kMostKeys / kKeysPerTile : 1];
  __shared__ uint64_t lows[2][WAVES];
  __shared__ int gone[kFew];
  __shared__ int ties;  // not all keys equal to the last that stays do
  const int tid = threadIdx.x, lane = tid & 63;
  const int unit = blockIdx.x, b = div_by(unit, p.div_heads);
  const int total = p.totals[b], L = counted(p, p.seq_lens[b], total);
  const float* w_in = p.w_in + unit * p.stride;
  const int32_t* p_in = p.p_in + unit * p.stride;
  float* w_out = p.w_out + unit * p.stride;
  int32_t* p_out = p.p_out + unit * p.stride;
  int32_t* moves = p.moves + unit * p.move_ints;
  if (L <= p.budget || L > p.L_K) {
    const int rows = (int)min((int64_t)L, p.stride);
    if (tid == 0 && !p.arrivals) moves[0] = 0;
    if (w_in != w_out)
      for (int r = tid; r < rows; r += THREADS) w_out[r] = w_in[r];
    if (p_in != p_out)
      for (int r = tid; r < rows; r += THREADS) p_out[r] = p_in[r];
    return;
  }
  // the sequence's pages, for the way of rows at the end
  if constexpr (KEEP)
    for (int i = tid; i <= div_by(L - 1, p.div_page); i += THREADS) pages[i] = p.block_table[(int64_t)b * p.max_pages + i];
  const int evicted = L - p.budget;
  const bool few = evicted <= kFew, held = few && p.arrivals;
  auto pool_row_of = [&](int r, const int32_t* table) {
    const int j = div_by(r, p.div_page);
    const int page = table[j];
    return page >= 0 && page < p.num_pages ? page * p.page_size + (r - j * p.page_size) : -1;
  };
  // a sixteenth of a row of K or V: 16 lanes a row of K, 16 of V
  const int64_t pitch = (int64_t)p.H_KV * D;
  auto piece = [&](int i) { return (i & 16 ? p.v : p.k) + (int64_t)(unit - b * p.H_KV) * D + 8 * (i & 15); };
  // the rows past the budget, if they are few, are there when it is known which of them stay
  u32x4 held_row = {0u, 0u, 0u, 0u};  // a page outside the pool reads as zeros
  float held_w = 0.f;
  int held_at = 0;
  if (held) {
    if (tid < 32 * evicted) {
      const int from = pool_row_of(p.budget + tid / 32, p.block_table + (int64_t)b * p.max_pages);
      if (from >= 0) held_row = *reinterpret_cast<const u32x4*>(piece(tid) + from * pitch);
    }
    if (tid < evicted) {
      held_w = w_in[p.budget + tid];
      held_at = p_in[p.budget + tid];
    }
  }
  const int shift = (int)((uint32_t)total - (uint32_t)L);  // position of a row that no eviction has placed: row + shift
  auto placed = [&](int r, int at) { return at >= 0 ? at : (int)((uint32_t)r + (uint32_t)shift); };
  const int64_t newest = (int64_t)total - p.recent;
  auto key_of = [&](int at, float w) { return at < p.sinks || (int64_t)at >= newest ? 0xffffffffu : order_of(w); };
  auto key = [&](int r) {
    if constexpr (KEEP)
      return keys[r];
    else
      return key_of(placed(r, p_in[r]), w_in[r]);
  };
  if (!few) {
    for (int i = tid; i < kBins; i += THREADS) hist[i] = 0;
    __syncthreads();
  }
  // rows below the budget are written as if they stayed; what moves into the others follows
  for (int r8 = tid; r8 < L; r8 += 8 * THREADS) {
    float w[8];
    int at[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = min(r8 + i * THREADS, L - 1);
      w[i] = w_in[r];
      at[i] = p_in[r];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r8 + i * THREADS;
      if (r >= L) break;
      const int pos = placed(r, at[i]);
      const uint32_t k = key_of(pos, w[i]);
      if constexpr (KEEP) keys[r] = k;
      if (!few) atomicAdd(&hist[(k >> 24) * kCopies + (lane & (kCopies - 1))], 1u);
      if (r < p.budget) {
        if (w_in != w_out) w_out[r] = w[i];
        if (at[i] < 0 || p_in != p_out) p_out[r] = pos;
      }
    }
  }
  __syncthreads();

  // rows that move, listed within the sequence first
  int count, mover = -1;  // mover: this thread's row past the budget is the one that moves into the mover-th hole
  int32_t* to = reinterpret_cast<int32_t*>(hist);
  int32_t* from = to + kListed;
  if (few) {
    // One row after the other: the smallest key above the last one's, of equal ones the highest row.
    uint64_t last = 0;  // key and the row's complement; a row has one above 0
    for (int e = 0; e < evicted; ++e) {
      uint64_t least = ~(uint64_t)0;
      for (int r = tid; r < L; r += THREADS) {
        const uint64_t x = (uint64_t)key(r) << 32 | (uint32_t)~r;
        least = x > last && x < least ? x : least;
      }
      least = least_of_row(least);
      {
        const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)least, (uint32_t)least, false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(least >> 32), (uint32_t)(least >> 32), false, false);
        least = std::min((uint64_t)hi[0] << 32 | lo[0], (uint64_t)hi[1] << 32 | lo[1]);
      }
      {
        const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)least, (uint32_t)least, false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(least >> 32), (uint32_t)(least >> 32), false, false);
        least = std::min((uint64_t)hi[0] << 32 | lo[0], (uint64_t)hi[1] << 32 | lo[1]);
      }
      if (lane == 0) lows[e & 1][tid >> 6] = least;
      __syncthreads();
      last = least_of_row(lows[e & 1][lane & (WAVES - 1)]);
      if (tid == 0) gone[e] = (int)~(uint32_t)last;
    }
    __syncthreads();
    // lane e: of the evicted rows the e-th found, and row budget + e
    const int mine = lane < evicted ? gone[lane] : -1;
    int hole = 0;
    bool stays = lane < evicted;
    for (int e = 0; e < evicted; ++e) {
      hole += gone[e] < mine;
      stays = stays && gone[e] != p.budget + lane;
    }
    const uint64_t holes = __ballot(mine >= 0 && mine < p.budget), movers = __ballot(stays);
    if (tid < 64 && mine >= 0 && mine < p.budget) to[hole] = mine;
    if (tid < 64 && stays) {
      mover = __builtin_popcountll(movers & (((uint64_t)1 << lane) - 1));
      from[mover] = p.budget + lane;
    }
    count = __builtin_popcountll(holes);
  } else {
    uint32_t prefix = 0, mask = 0;
    uint32_t want = (uint32_t)p.budget;  // of the keys that share the prefix, the want-th largest is the last to stay
    int2 all;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int low = pass == 0 ? 24 : pass == 1 ? 12 : 0;
      if (pass > 0) {
#pragma unroll 4
        for (int r = tid; r < L; r += THREADS) {
          const uint32_t k = key(r);
          if ((k & mask) == prefix) atomicAdd(&hist[(k >> low) & (kBins - 1)], 1u);
        }
        __syncthreads();
      }
      // from the largest digit down: the first digit one a thread, the others kBins / THREADS
      constexpr int PER = kBins / THREADS;
      uint32_t c[PER], sum = 0;
      if (pass == 0) {
        if (tid < 256)
#pragma unroll
          for (int i = 0; i < kCopies; ++i) {
            const int at = (255 - tid) * kCopies + ((tid + i) & (kCopies - 1));
            sum += hist[at];
            hist[at] = 0;
          }
      } else {
        u32x4* const mine = reinterpret_cast<u32x4*>(hist + kBins - PER * (tid + 1));
#pragma unroll
        for (int i = 0; i < PER / 4; ++i) {
          const u32x4 x = mine[PER / 4 - 1 - i];
          mine[PER / 4 - 1 - i] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            c[4 * i + e] = x[3 - e];
            sum += x[3 - e];
          }
        }
      }
      uint32_t before = (uint32_t)scan_before<WAVES>((int)sum, 0, sums[pass], &all).x;
      if (before < want && want <= before + sum) {
        int digit = 255 - tid;
        if (pass > 0) {
          digit = kBins - 1 - PER * tid;
          sum = c[0];
#pragma unroll
          for (int i = 0; i < PER - 1; ++i)
            if (kBins - 1 - PER * tid - i == digit && want > before + c[i]) {
              before += c[i];
              sum = c[i + 1];
              --digit;
            }
        }
        found[pass][0] = (uint32_t)digit;
        found[pass][1] = want - before;
        if (pass == 2) ties = sum != want - before;
      }
      __syncthreads();
      prefix |= found[pass][0] << low;
      mask |= (pass == 0 ? 255u : kBins - 1u) << low;
      want = found[pass][1];
    }

    // the thread's rows: an odd number of them, so that the threads' keys lie in different banks
    const int each = ((L + THREADS - 1) / THREADS) | 1;
    const int r0 = (int)min((int64_t)tid * each, (int64_t)L), r1 = (int)min((int64_t)r0 + each, (int64_t)L);
    int rank0 = 0;
    if (ties) {
      int equal = 0;
#pragma unroll 4
      for (int r = r0; r < r1; ++r) equal += key(r) == prefix;
      rank0 = scan_before<WAVES>(equal, 0, sums[3], &all).x;
    } else {
      want = (uint32_t)L;  // a thread's rows are fewer
    }
    int rank = rank0, holes = 0, late = 0;
#pragma unroll 4
    for (int r = r0; r < r1; ++r) {
      const uint32_t k = key(r);
      const bool stays = k > prefix || (k == prefix && rank < (int)want);
      rank += k == prefix;
      holes += !stays && r < p.budget;
      late += stays && r >= p.budget;
    }
    const int2 first = scan_before<WAVES>(holes, late, sums[4], &all);
    count = min(all.x, p.most);
    if (count > kListed) {
      to = moves + 1;
      from = moves + 1 + p.most;
    }
    if (holes + late > 0) {
      rank = rank0;
      int hole = first.x, late_row = first.y;
      for (int r = r0; r < r1; ++r) {
        const uint32_t k = key(r);
        const bool stays = k > prefix || (k == prefix && rank < (int)want);
        rank += k == prefix;
        if (r < p.budget && !stays) {
          if (hole < count) to[hole] = r;
          ++hole;
        }
        if (r >= p.budget && stays) {
          if (late_row < count) from[late_row] = r;
          ++late_row;
        }
      }
    }
  }
  __syncthreads();
  if (tid == 0 && !p.arrivals) moves[0] = count;
  auto pool_row = [&](int r) {
    if constexpr (KEEP)
      return pool_row_of(r, pages);
    else
      return pool_row_of(r, p.block_table + (int64_t)b * p.max_pages);
  };
  if (held) {
    if (mover >= 0) {
      const int d = to[mover];
      w_out[d] = held_w;
      p_out[d] = placed(p.budget + tid, held_at);
    }
    for (int i = 0; i < count; ++i) {
      if (tid / 32 != from[i] - p.budget) continue;
      const int d = pool_row(to[i]);
      if (d >= 0) *reinterpret_cast<u32x4*>(piece(tid) + d * pitch) = held_row;
    }
    count = 0;  // done
  }
  for (int i = tid; i < count; i += THREADS) {
    const int d = to[i], s = from[i];
    w_out[d] = w_in[s];
    p_out[d] = placed(s, p_in[s]);
    if (!p.arrivals) {
      moves[1 + i] = pool_row(d);
      moves[1 + p.most + i] = pool_row(s);
    }
  }
  if (p.arrivals) {
    for (int i = tid; i < 32 * count; i += THREADS) {
      const int d = pool_row(to[i / 32]), s = pool_row(from[i / 32]);
      u32x4 x = {0u, 0u, 0u, 0u};
      if (s >= 0) x = *reinterpret_cast<const u32x4*>(piece(i) + s * pitch);
      if (d >= 0) *reinterpret_cast<u32x4*>(piece(i) + d * pitch) = x;
    }
  }
  __syncthreads();
  for (int r = p.budget + tid; r < L; r += THREADS) {
    w_out[r] = 0.f;
    p_out[r] = -1;
  }
}

// With `arrivals` the rows that move are few, and there is no second launch: each
// workgroup moves its own, and the last one to end (nobody waits) does the rest.
// 256 sequences and heads with 64 rows past the budget 16.7 us in a graph, with a
// second launch 17.2; with 128 19.8 and 19.7; with 256 25.7 and 25.2.
template <int THREADS, bool KEEP>
__global__ void __launch_bounds__(THREADS) select_kernel(EvictParams p) {
  int length0 = 0, in_use = 0;
  if (p.arrivals) {  // there when the last workgroup needs them
    length0 = length_of(p, threadIdx.x);
    if (p.taken_out) in_use = *p.taken;
  }
  select_rows<THREADS, KEEP>(p);
  if (!p.arrivals) return;
  __shared__ int last;
  __syncthreads();  // every thread is done with the lengths
  if (threadIdx.x == 0) {
    // the last at one of kGates counters goes on to the one of all: additions to one address go one after the other (256
    // workgroups at one 2.9 us)
    auto last_at = [](uint32_t* counter, uint32_t members) {
      const bool is = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == members - 1;
      if (is) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      return is;
    };
    const uint32_t gate = blockIdx.x % kGates;
    last = last_at(p.arrivals + (1 + gate) * da::kArrivalStride, (gridDim.x - gate + kGates - 1) / kGates) &&
           last_at(p.arrivals, min(gridDim.x, kGates));
  }
  __syncthreads();
  if (last) give_back<THREADS>(p, length0, in_use);
}

// The rows into their places, and (block 0) the lengths and the pages that come
// free.  A head's row of K or V is 16 lanes of 16 bytes; a wave moves four rows
// of both at a time.  Targets lie below the budget and sources above it, so no
// move meets another.
__global__ void __launch_bounds__(256) move_kernel(EvictParams p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (blockIdx.x > 0) {
    const int blk = (int)blockIdx.x - 1;
    const int unit = div_by(blk, p.div_groups), part = blk - unit * p.groups;
    const int h = unit - div_by(unit, p.div_heads) * p.H_KV;
    const int32_t* moves = p.moves + unit * p.move_ints;
    const int count = moves[0];
    const int32_t* to = moves + 1;
    const int32_t* from = moves + 1 + p.most;
    for (int i0 = part * kMoveRows; i0 < count; i0 += p.groups * kMoveRows) {
      u32x4 x[4][2];
      int d[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * 16 + wave * 4 + (lane >> 4);
        d[u] = i < count ? to[i] : -1;
        const int s = i < count ? from[i] : -1;
        x[u][0] = x[u][1] = u32x4{0u, 0u, 0u, 0u};  // a page outside the pool reads as zeros
        if (s >= 0) {
          const int64_t at = ((int64_t)s * p.H_KV + h) * D + 8 * (lane & 15);
          x[u][0] = *reinterpret_cast<const u32x4*>(p.k + at);
          x[u][1] = *reinterpret_cast<const u32x4*>(p.v + at);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (d[u] < 0) continue;
        const int64_t at = ((int64_t)d[u] * p.H_KV + h) * D + 8 * (lane & 15);
        *reinterpret_cast<u32x4*>(p.k + at) = x[u][0];
        *reinterpret_cast<u32x4*>(p.v + at) = x[u][1];
      }
    }
    return;
  }
  give_back<256>(p, length_of(p, threadIdx.x), p.taken_out ? *p.taken : 0);
}

// ---------------------------------------------------------------- host side

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? (int)DA_OK : da::fail(DA_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

constexpr int64_t kGridThreads = (int64_t)1 << 32;  // a launch has fewer

int most_moves(int L_K_max, int budget) { return std::max(0, std::min(budget, L_K_max - budget)); }

// Workspace bytes of an eviction, without the counters at its end.
int64_t move_bytes(int B, int H_KV, int L_K_max, int budget) {
  return 4ll * B * H_KV * (1 + 2ll * most_moves(L_K_max, budget));
}

// Threads that choose the rows of a (sequence, KV head).
int select_threads(int L_K_max) { return L_K_max <= 512 ? 256 : L_K_max <= 1024 ? 512 : 1024; }

}  // namespace

extern "C" {

int da_add_key_weights(const void* q, const void* k_cache, const int32_t* block_table, const int32_t* seq_lens,
                       const float* lse, const float* weights, float* weights_out, int64_t weight_stride, int B,
                       int H_Q, int H_KV, int page_size, int max_pages, int num_pages, int L_K_max, int d,
                       float softmax_scale, float decay, void* stream) {
  da::clear_error();
  int rc = da::check_shape(B, H_Q, H_KV, L_K_max, d);
  if (!q || !block_table || !seq_lens || !lse || !weights || !weights_out)
    return da::fail(DA_ERR_NULL, "q, block_table, seq_lens, lse, weights and weights_out must be non-NULL");
  if (!k_cache && !(rc == DA_OK && L_K_max == 0)) return da::fail(DA_ERR_NULL, "k_cache must be non-NULL");
  if (rc) return rc;
  rc = da::check_page_table(B, page_size, max_pages, num_pages, L_K_max);
  if (rc) return rc;
  if (H_Q / H_KV > (1 << 16)) return da::fail(DA_ERR_SHAPE, "%d query heads a KV head", H_Q / H_KV);
  if (weight_stride < L_K_max)
    return da::fail(DA_ERR_SHAPE, "weight_stride=%lld is less than L_K_max=%d", (long long)weight_stride, L_K_max);
  if (!(decay >= 0.f && decay <= 1.f)) return da::fail(DA_ERR_ARG, "decay must be in [0, 1]");
  if (!aligned(q, 16) || !aligned(k_cache, 16))
    return da::fail(DA_ERR_ALIGN, "q and k_cache must be 16-byte aligned");
  if (!aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(lse, 4) || !aligned(weights, 4) ||
      !aligned(weights_out, 4))
    return da::fail(DA_ERR_ALIGN, "block_table, seq_lens, lse and weights must be 4-byte aligned");
  const int64_t tiles = (L_K_max + kKeysPerTile - 1) / kKeysPerTile, units = (int64_t)B * H_KV;
  if (units * ((tiles + kMostChunkTiles - 1) / kMostChunkTiles) * (64 * kWeightWaves) >= kGridThreads)
    return da::fail(DA_ERR_SHAPE, "B=%d H_KV=%d L_K_max=%d: too many workgroups", B, H_KV, L_K_max);
  int cus = 0;
  rc = ensure_gfx950(&cus);
  if (rc || L_K_max == 0) return rc;
  WeightParams p{};
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k_cache);
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.lse = lse;
  p.in = weights;
  p.out = weights_out;
  p.stride = weight_stride;
  p.B = B;
  p.H_Q = H_Q;
  p.H_KV = H_KV;
  p.g = H_Q / H_KV;
  p.L_K = L_K_max;
  p.page_size = page_size;
  p.max_pages = max_pages;
  p.num_pages = num_pages;
  p.div_page = make_div((uint32_t)page_size);
  p.div_heads = make_div((uint32_t)H_KV);
  // sixteen workgroups a CU, of one tile a wave at least: they start as others end, so lengths even out.  Where they
  // become more than that and one a unit, chunks have their greatest length
  int64_t each = (tiles * units + 16 * cus - 1) / (16 * cus);
  each = std::min<int64_t>(std::max<int64_t>(4, (each + 3) / 4 * 4), kMostChunkTiles);
  p.chunk_tiles = (int)each;
  const int64_t chunks = (tiles + each - 1) / each;
  p.chunks = (int)chunks;
  p.div_chunks = make_div((uint32_t)chunks);
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)D)) * kLog2e;
  p.decay = decay;
  // keys that the caches cannot hold until the next call take the streaming hint (552 MB of keys and weights 108 ->
  // 94 us in a graph; 276 MB 44 -> 46, so not below)
  const int64_t keys = std::min((int64_t)num_pages * page_size, (int64_t)B * L_K_max);
  const bool stream_hint = (uint64_t)keys * H_KV * D * 2 > DA_RESIDENT_BYTES;
  auto pick = [&](auto hint) {
    constexpr int AUX = decltype(hint)::value;
    return p.g <= 16   ? reinterpret_cast<const void*>(&weights_kernel<1, AUX>)
           : p.g <= 32 ? reinterpret_cast<const void*>(&weights_kernel<2, AUX>)
                       : reinterpret_cast<const void*>(&weights_kernel<4, AUX>);
  };
  const void* fn = stream_hint ? pick(std::integral_constant<int, 2>{}) : pick(std::integral_constant<int, 0>{});
  void* args[] = {&p};
  return launched(hipLaunchKernel(fn, dim3((uint32_t)(units * chunks)), dim3(64 * kWeightWaves), args, 0,
                                  static_cast<hipStream_t>(stream)),
                  "key weight");
}

size_t da_evict_workspace_bytes(int B, int H_KV, int L_K_max, int budget) {
  // a workgroup a (sequence, KV head), and where those are many one more in move_kernel
  if (B <= 0 || B > DA_MAX_REQUESTS || H_KV <= 0 || L_K_max < 0 || budget < 1 ||
      ((int64_t)B * H_KV + 1) * select_threads(L_K_max) >= kGridThreads)
    return 0;
  const int64_t bytes = move_bytes(B, H_KV, L_K_max, budget);
  if (bytes >= ((int64_t)1 << 40)) return 0;
  return (size_t)((bytes + 255) / 256 * 256) + DA_ARRIVAL_BYTES;
}

int da_evict_kv(void* k_cache, void* v_cache, const int32_t* block_table, const int32_t* seq_lens,
                const int32_t* totals, const float* weights, const int32_t* positions, float* weights_out,
                int32_t* positions_out, int64_t weight_stride, int32_t* lens_out, int32_t* free_pages,
                const int32_t* taken, int32_t* taken_out, int num_free, int B, int H_KV, int page_size, int max_pages,
                int num_pages, int L_K_max, int d, int budget, int sinks, int recent, void* workspace,
                size_t workspace_bytes, void* stream) {
  da::clear_error();
  int rc = da::check_shape(B, H_KV, H_KV, L_K_max, d);
  if (!block_table || !seq_lens || !totals || !weights || !positions || !weights_out || !positions_out || !lens_out)
    return da::fail(DA_ERR_NULL, "tables, lengths, totals, weights and positions must be non-NULL");
  if ((!k_cache || !v_cache) && !(rc == DA_OK && L_K_max == 0))
    return da::fail(DA_ERR_NULL, "k_cache and v_cache must be non-NULL");
  if ((free_pages || taken_out) && (!taken || !taken_out || (!free_pages && num_free > 0)))
    return da::fail(DA_ERR_NULL, "free_pages, taken and taken_out go together");
  if (rc) return rc;
  rc = da::check_page_table(B, page_size, max_pages, num_pages, L_K_max);
  if (rc) return rc;
  if (B > DA_MAX_REQUESTS) return da::fail(DA_ERR_SHAPE, "B=%d exceeds %d", B, DA_MAX_REQUESTS);
  if ((int64_t)num_pages * page_size >= ((int64_t)1 << 31))
    return da::fail(DA_ERR_SHAPE, "num_pages=%d pages of %d rows: rows have 32 bits", num_pages, page_size);
  if (weight_stride < L_K_max)
    return da::fail(DA_ERR_SHAPE, "weight_stride=%lld is less than L_K_max=%d", (long long)weight_stride, L_K_max);
  if (num_free < 0) return da::fail(DA_ERR_SHAPE, "num_free=%d is negative", num_free);
  if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget)
    return da::fail(DA_ERR_ARG, "budget=%d must be positive and hold sinks=%d and recent=%d", budget, sinks, recent);
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16))
    return da::fail(DA_ERR_ALIGN, "k_cache and v_cache must be 16-byte aligned");
  for (const void* x : {(const void*)block_table, (const void*)seq_lens, (const void*)totals, (const void*)weights,
                        (const void*)positions, (const void*)weights_out, (const void*)positions_out,
                        (const void*)lens_out, (const void*)free_pages, (const void*)taken, (const void*)taken_out})
    if (!aligned(x, 4)) return da::fail(DA_ERR_ALIGN, "tables, lengths, weights and positions must be 4-byte aligned");
  if (workspace && !aligned(workspace, 16)) return da::fail(DA_ERR_ALIGN, "workspace must be 16-byte aligned");
  const size_t need = da_evict_workspace_bytes(B, H_KV, L_K_max, budget);
  if (need == 0) return da::fail(DA_ERR_SHAPE, "B=%d H_KV=%d L_K_max=%d: too many rows", B, H_KV, L_K_max);
  if (!workspace || workspace_bytes < need)
    return da::fail(DA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : 0);
  int cus = 0;
  rc = ensure_gfx950(&cus);
  if (rc) return rc;
  EvictParams p{};
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.totals = totals;
  p.w_in = weights;
  p.p_in = positions;
  p.w_out = weights_out;
  p.p_out = positions_out;
  p.stride = weight_stride;
  p.moves = static_cast<int32_t*>(workspace);
  p.most = most_moves(L_K_max, budget);
  p.move_ints = 1 + 2ll * p.most;
  p.B = B;
  p.H_KV = H_KV;
  p.L_K = L_K_max;
  p.budget = budget;
  p.sinks = sinks;
  p.recent = recent;
  p.page_size = page_size;
  p.max_pages = max_pages;
  p.num_pages = num_pages;
  p.div_page = make_div((uint32_t)page_size);
  p.div_heads = make_div((uint32_t)H_KV);
  p.k = static_cast<uint16_t*>(k_cache);
  p.v = static_cast<uint16_t*>(v_cache);
  p.lens_out = lens_out;
  p.free_pages = free_pages;
  p.taken = taken;
  p.taken_out = taken_out;
  p.num_free = num_free;
  const int64_t units = (int64_t)B * H_KV;
  // one launch where a sequence has few rows to move
  if (p.most <= kMovedAtOnce)
    p.arrivals = reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(workspace) + da::arrival_offset(workspace_bytes));
  void* args[] = {&p};
  const int threads = select_threads(L_K_max);
  const void* fn = threads == 256         ? reinterpret_cast<const void*>(&select_kernel<256, true>)
                   : threads == 512       ? reinterpret_cast<const void*>(&select_kernel<512, true>)
                   : L_K_max <= kMostKeys ? reinterpret_cast<const void*>(&select_kernel<1024, true>)
                                          : reinterpret_cast<const void*>(&select_kernel<1024, false>);
  const int smem = L_K_max <= kMostKeys ? 4 * L_K_max : 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  rc = launched(hipLaunchKernel(fn, dim3((uint32_t)units), dim3(threads), args, smem, s), "select");
  if (rc || p.arrivals) return rc;
  // eight workgroups a CU at most; a workgroup that finds nothing to move ends at once
  const int64_t parts = (p.most + kMoveRows - 1) / kMoveRows;
  p.groups = (int)std::max<int64_t>(1, std::min<int64_t>(parts, (8ll * cus + units - 1) / units));
  p.div_groups = make_div((uint32_t)p.groups);
  const int64_t grid = 1 + units * p.groups;
  return launched(hipLaunchKernel(reinterpret_cast<const void*>(&move_kernel), dim3((uint32_t)grid), dim3(256), args, 0, s),
                  "move");
}

}  // extern "C"
