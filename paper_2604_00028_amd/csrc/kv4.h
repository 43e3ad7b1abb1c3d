// The 4-bit K/V cache: its layout, and rows into and out of it.
//
// A tile is 32 keys of one KV head, DA_KV4_TILE_BYTES bytes: K codes 32 x 64
// bytes, V codes 32 x 64 bytes, then 256 scale bytes.  A row's byte i holds
// dims 2i (low half) and 2i + 1.  A value is code x 2^(scale byte - 127), one
// scale byte, 2 to 252 (255: NaN), for 32 dims: the FP4 (e2m1: 0, 0.5, 1, 1.5, 2,
// 3, 4, 6 and their negatives) and power-of-two scale formats that gfx950
// converts in one instruction, exactly into bf16.
//
// The order inside a tile is what the attention loads: lane (key % 16, block of
// 32 dims) of a wave reads 16 bytes of codes of each of two keys, 1 KiB
// contiguous a load, and one dword with its four scales (K and V of keys r and
// r + 16).
#pragma once

#include <stdint.h>

#include "decode_attn.h"
#include "tile.h"

namespace {

constexpr int kKv4V = 32 * 64;            // V codes
constexpr int kKv4Scales = 2 * 32 * 64;   // scale bytes

__device__ __forceinline__ int kv4_scale_at(int key, int block, int isv) {
  return kKv4Scales + 4 * (4 * (key & 15) + block) + (key >> 4) + 2 * isv;
}

__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes times the scale as bf16.
__device__ __forceinline__ void dequantise(uint32_t codes, float scale, u32x4& y) {
  y.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  y.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  y.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  y.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
}

// Eight bf16 values of a row, this lane's quarter of a block of 32 (the other
// three in the lanes of its quad): their codes, and the block's scale byte.
// The scale is the least power of two that leaves the largest magnitude at most
// 7 (a value between 6 and 7 becomes 6, which is no further off than a value
// between 4 and 6 can be), held to [2^-125, 2^125] so that neither a value nor
// half a unit leaves the normal range; codes are rounded to the nearest, ties to
// the even code.  A block with an infinity or NaN gets the scale byte 255 (NaN).
__device__ __forceinline__ uint32_t quantise(const u32x4& x, uint32_t* scale) {
  uint32_t top = 0;  // largest magnitude's bits; those of a NaN are above infinity's
#pragma unroll
  for (int e = 0; e < 4; ++e) top = max(top, max((x[e] & 0x7fffu) << 16, x[e] & 0x7fff0000u));
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, false));  // quad lanes 1, 0, 3, 2
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, false));  // quad lanes 2, 3, 0, 1
  // 1.75 x 2^2 = 7: a mantissa above 1.75 takes the next power
  int byte = (int)((top + 0x1fffffu) >> 23) - 2;
  byte = byte < 2 ? 2 : byte > 252 ? 252 : byte;
  const float s = kv4_scale((uint32_t)byte);
  uint32_t codes = 0;
#define DA_PAIR(i)                                                                                        \
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(x[i] << 16),                    \
                                                   __uint_as_float(x[i] & 0xffff0000u), s, i)
  DA_PAIR(0);
  DA_PAIR(1);
  DA_PAIR(2);
  DA_PAIR(3);
#undef DA_PAIR
  *scale = top >= 0x7f800000u ? 255u : (uint32_t)byte;
  return codes;
}

}  // namespace
