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

struct Kv4Params {
  Params p;  // q, out, lse, chunk states, counters, block table, lengths, shape, window
  const unsigned char* cache;
  int chunk_tiles;   // tiles of 32 keys a chunk holds
  int blocks;        // tiles a page holds
  Div div_blocks;
  Div div_tiles;     // p.tiles
};

constexpr int kv4_smem_bytes(int NT) {
  return W * kKeysPerTile * kVPitch > W * merge_slot_bytes(NT) ? W * kKeysPerTile * kVPitch : W * merge_slot_bytes(NT);
}
static_assert(kv4_smem_bytes(1) >= (2 * (DA_MAX_SPLITS + 16) * 32 + 8 * 32) * 4, "the merge stages chunk maxima and sums");

template <int NT, bool NTL>
__global__ void __launch_bounds__(64 * W) kv4_kernel(Kv4Params a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int kv_aux = NTL ? 2 : 0;
  const Params& p = a.p;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;

  // ---- chunk and tile: all first chunks, then all second ones, ...
  const int chunk = div_by((int)blockIdx.x, a.div_tiles);
  const int tile = (int)blockIdx.x - chunk * p.tiles;
  const int b = div_by(tile, p.div_tps);
  const int head0 = (tile - b * p.tiles_per_seq) * p.hpt;
  const int kvh = div_by(head0, p.div_g);
  int L = p.seq_lens[b];
  L = L < 0 ? 0 : (L > p.L_K ? p.L_K : L);
  const Window wn = window_of(L, p.window > 0 ? p.window : L, p.window > 0 ? p.sinks : 0);
  const int vis = L - wn.skip;  // positions
  const int T = (vis + kKeysPerTile - 1) / kKeysPerTile;
  const int t0 = chunk * a.chunk_tiles;
  if (t0 >= T && chunk > 0) return;  // the whole workgroup
  const int chunks = max(1, (T + a.chunk_tiles - 1) / a.chunk_tiles);
  const int t1 = min(t0 + a.chunk_tiles, T);

  // ---- this wave's tiles: t0 + wave, + W, ...
  const int n = t1 > t0 + wave ? (t1 - t0 - wave + W - 1) / W : 0;
  // its page ids, 64 pages at a time, one per lane
  int pg_win = 0, pg_ids = 0;
  const int pg_last = n > 0 ? div_by(wn.key(kKeysPerTile * (t0 + wave + (n - 1) * W)) / kKeysPerTile, a.div_blocks) : -1;
  auto pages = [&](int first) {
    pg_win = first;
    pg_ids = first + lane <= pg_last ? p.block_table[(int64_t)b * p.max_pages + first + lane] : 0;
  };
  auto tile_key = [&](int i) { return wn.key(kKeysPerTile * (t0 + wave + i * W)); };  // first key of tile i
  if (n > 0) pages(div_by(tile_key(0) / kKeysPerTile, a.div_blocks));

  struct Tile {
    u32x4 k[2], v[2];
    uint32_t scales;
  };
  auto load = [&](Tile& t, int i) {
    const int kt = tile_key(i) / kKeysPerTile;
    const int j = div_by(kt, a.div_blocks);
    if (j - pg_win >= 64) pages(j);
    const int page = __builtin_amdgcn_readlane(pg_ids, (j - pg_win) & 63);
    const bool in = page >= 0 && page < p.num_pages;  // a page id outside the cache reads as zeros
    const int64_t at = (((int64_t)(in ? page : 0) * p.H_KV + kvh) * a.blocks + (kt - j * a.blocks)) * DA_KV4_TILE_BYTES;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(a.cache + at, in ? DA_KV4_TILE_BYTES : 0u);
    const uint32_t off = 64u * col + 16u * quad;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) t.k[mt] = __builtin_amdgcn_raw_buffer_load_b128(r, off + 1024u * mt, 0, kv_aux);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
      t.v[mt] = __builtin_amdgcn_raw_buffer_load_b128(r, off + 1024u * mt + (uint32_t)kKv4V, 0, kv_aux);
    t.scales =
        (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, (uint32_t)kKv4Scales + 16u * col + 4u * quad, 0, kv_aux);
  };

  TileReducer<NT, 8> red;
  red.scale_log2 = p.scale_log2;
  red.quad = quad;
  // Q in the order of the 4-bit rows: k-step j, lane group `quad` covers dims [32 quad + 8 j, +8)
  {
    const __amdgpu_buffer_rsrc_t qr = make_rsrc(p.q + ((int64_t)b * p.H_Q + head0) * D, (uint32_t)p.hpt * (D * 2));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        red.q[nt][j] = as_bf16x8(__builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       qr, (uint32_t)(nt * 16 + col) * (D * 2) + 64u * quad + 16u * j, 0, 0)));
  }
  red.reset();
  unsigned char* vstage = smem + wave * kKeysPerTile * kVPitch;

  auto reduce = [&](Tile& t, int i, bool more) {
    const int first = tile_key(i);
    const int nvalid = L - first;  // >= 1
    bf16x8 kop[2][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const float s = kv4_scale((t.scales >> (8 * mt)) & 0xffu);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 y;
        dequantise(t.k[mt][j], s, y);
        kop[mt][j] = as_bf16x8(y);
      }
    }
    f32x4 sc[NT][2];
    red.scores(kop, sc);
    const bool cut = nvalid < kKeysPerTile || wn.cuts(first);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      float s = kv4_scale((t.scales >> (16 + 8 * mt)) & 0xffu);
      // whatever an invisible row holds, its values come out finite: a zero probability cancels them
      const int row = 16 * mt + col;
      if (cut && (row >= nvalid || wn.hides(first, row))) s = 1.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 y;
        dequantise(t.v[mt][j], s, y);
        *reinterpret_cast<u32x4*>(vstage + row * kVPitch + 64 * quad + 16 * j) = y;
      }
    }
    if (more) load(t, i + 2);
    if (cut) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = mt * 16 + quad * 4 + e;
            sc[nt][mt][e] = row < nvalid && !wn.hides(first, row) ? sc[nt][mt][e] : -INFINITY;
          }
    }
    bf16x8 pb[1][NT];
    red.softmax(sc, kKeysPerTile, std::false_type{}, pb);
    __builtin_amdgcn_wave_barrier();
    const unsigned char* vrow = vstage + (quad * 4 + (col >> 2)) * kVPitch + 8 * (col & 3);
    red.pv(pb, [&](int mt, int nn) { return vrow + mt * 16 * kVPitch + 32 * nn; }, std::false_type{});
    __builtin_amdgcn_wave_barrier();
  };
  // two tiles in flight
  Tile even, odd;
  if (n > 0) load(even, 0);
  if (n > 1) load(odd, 1);
  for (int i = 0; i < n; i += 2) {
    reduce(even, i, i + 2 < n);
    if (i + 1 < n) reduce(odd, i + 1, i + 3 < n);
  }

  const int64_t rows = (int64_t)p.B * p.H_Q;
  const int64_t row0 = (int64_t)b * p.H_Q + head0;
  const bool direct = chunks == 1;
  red.close();
  __syncthreads();  // every wave is done with its stage
  publish_wave(red, reinterpret_cast<float*>(smem), wave, lane);
  __syncthreads();
  finish_chunk<NT, 8, W>(p, reinterpret_cast<const float*>(smem), direct, row0,
                         direct ? 0 : (int64_t)chunk * rows + row0, 0, wave, lane);
  if (direct) return;

  // The merge inside the launch: the hand-off of split_partial_kernel
  // (decode_attn.hip), with this sequence's chunk count.
  __shared__ int s_last;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) {
    uint32_t* counter = p.arrivals + (size_t)tile * da::kArrivalStride;
    const bool last =
        __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u == (uint32_t)chunks;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = last ? 1 : 0;
  }
  __syncthreads();
  if (!s_last) return;
  merge_tile<NT, W>(p, reinterpret_cast<float*>(smem), row0, rows, chunks, row0, tid);
}

// ---------------------------------------------------------------- host side

struct Kv4Plan {
  int heads_per_tile, tiles, chunk_tiles, chunks;
};

// num_splits <= 0: chosen.
Kv4Plan kv4_plan(int B, int H_Q, int H_KV, int keys, int num_splits, int cus) {
  Kv4Plan pl;
  pl.heads_per_tile = da::heads_per_tile(H_Q, H_KV, 1);
  pl.tiles = (int)((int64_t)B * H_Q / pl.heads_per_tile);
  const int T = std::max(1, (keys + kKeysPerTile - 1) / kKeysPerTile);
  // chunk states below 2 GiB, and a counter for every tile
  const int64_t most = std::min<int64_t>(DA_MAX_SPLITS, (((int64_t)1 << 31) - 1) / ((int64_t)B * H_Q * D * 4));
  int s = num_splits;
  if (s <= 0) {
    const int64_t want = (2ll * cus + pl.tiles - 1) / pl.tiles;  // two workgroups a CU
    s = (int)std::min<int64_t>(want, (T + 2 * W - 1) / (2 * W));  // two tiles a wave at least
  }
  if (pl.tiles > da::kMaxArrivalTiles) s = 1;
  s = (int)std::max<int64_t>(1, std::min<int64_t>(s, most));
  pl.chunk_tiles = (T + s - 1) / s;
  pl.chunks = (T + pl.chunk_tiles - 1) / pl.chunk_tiles;
  return pl;
}

int kv4_keys(int L_K_max, int window, int sinks) {
  return window > 0 ? da::window_keys(L_K_max, window, sinks) : L_K_max;
}

}  // namespace

extern "C" {

size_t da_kv4_workspace_bytes(int B, int H_Q, int H_KV, int L_K_max, int window, int sinks, int num_splits,
                              int num_cus) {
  if (da::check_shape(B, H_Q, H_KV, L_K_max, D) || window < 0 || sinks < 0 || num_splits > DA_MAX_SPLITS) return 0;
  if (num_cus <= 0 && ensure_gfx950(&num_cus)) return 0;
  const Kv4Plan pl = kv4_plan(B, H_Q, H_KV, kv4_keys(L_K_max, window, sinks), num_splits, num_cus);
  return pl.chunks > 1 ? da::workspace_layout(B, H_Q, D, pl.chunks).total : 0;
}

int da_decode_attn_kv4(const void* q, const void* cache, const int32_t* block_table, const int32_t* seq_lens, void* out,
                       float* lse_out, int B, int H_Q, int H_KV, int page_size, int max_pages, int num_pages,
                       int L_K_max, int d, float softmax_scale, int window, int sinks, int num_splits, void* workspace,
                       size_t workspace_bytes, void* stream) {
  da::clear_error();
  int rc = da::check_shape(B, H_Q, H_KV, L_K_max, d);
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
  int cus = 0;
  rc = ensure_gfx950(&cus);
  if (rc) return rc;
  const int keys = kv4_keys(L_K_max, window, sinks);
  const Kv4Plan pl = kv4_plan(B, H_Q, H_KV, keys, num_splits, cus);
  if ((int64_t)pl.tiles * pl.chunks >= (1 << 24))
    return da::fail(DA_ERR_SHAPE, "%d head tiles in %d chunks are too many workgroups", pl.tiles, pl.chunks);
  Kv4Params a{};
  da_plan dp{};
  dp.num_splits = pl.chunks;
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
  a.div_blocks = make_div((uint32_t)a.blocks);
  a.div_tiles = make_div((uint32_t)pl.tiles);
  if (pl.chunks > 1) {
    const da::WorkspaceLayout wl = da::workspace_layout(B, H_Q, D, pl.chunks);
    if (!workspace || workspace_bytes < wl.total)
      return da::fail(DA_ERR_WORKSPACE, "%d chunks need %zu workspace bytes, got %zu", pl.chunks, wl.total,
                      workspace ? workspace_bytes : (size_t)0);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    a.p.o_part = reinterpret_cast<float*>(ws + wl.o_off);
    a.p.m_part = reinterpret_cast<float*>(ws + wl.m_off);
    a.p.l_part = reinterpret_cast<float*>(ws + wl.l_off);
    a.p.arrivals = reinterpret_cast<uint32_t*>(ws + da::arrival_offset(workspace_bytes));
  }
  const bool ntl = (double)B * keys * H_KV * (DA_KV4_TILE_BYTES / kKeysPerTile) > (double)DA_RESIDENT_BYTES &&
                   pl.heads_per_tile == H_Q / H_KV;
  const void* fn;
  int smem;
  if (pl.heads_per_tile <= 16) {
    fn = ntl ? reinterpret_cast<const void*>(&kv4_kernel<1, true>) : reinterpret_cast<const void*>(&kv4_kernel<1, false>);
    smem = kv4_smem_bytes(1);
  } else {
    fn = ntl ? reinterpret_cast<const void*>(&kv4_kernel<2, true>) : reinterpret_cast<const void*>(&kv4_kernel<2, false>);
    smem = kv4_smem_bytes(2);
  }
  void* args[] = {&a};
  const hipError_t e =
      hipLaunchKernel(fn, dim3(pl.tiles * pl.chunks), dim3(64 * W), args, smem, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return da::fail(DA_ERR_HIP, "4-bit attention launch: %s", hipGetErrorString(e));
  return DA_OK;
}

}  // extern "C"
