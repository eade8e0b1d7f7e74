// The paged 8-bit key-value cache: its layout, and the quantisation of one block.
//
// uint8 [pages][kv heads][kv8_tile_bytes(d)], per (page of 16 tokens, kv head):
//   K codes  [d/64][16 tokens][64 dims]: lane (token l % 16, g = l / 16) of a wave reads
//            the 16 dims 64 a + 16 g .. of its token, a whole 64-dim block in one
//            contiguous 1 KB access; the two halves of those 16 bytes are the lane's part of
//            two 16x16x32 matrix instructions.
//   V codes  [d/64][4 token quads][16][4][4]: lane (b = l % 16, g) reads tokens 4 g .. + 3 of
//            the dims 64 a + 16 c + b, c < 4.  Tokens 4 g .. + 3 are also those whose scores
//            that lane gets from K Q^T, so the probabilities go from one product to
//            the other without leaving the lane.
//   K scales, V scales  fp32 [16] each, one per token.
// One region of 32 d + 128 bytes: 33 cache lines at d = 128, read front to back.
#pragma once
#include "common.h"

namespace sevo {

__host__ __device__ constexpr uint32_t kv8_tile_bytes(int d) { return 32u * d + 128u; }
__host__ __device__ __forceinline__ uint32_t kv8_k_offset(int s, int e) {
  return (uint32_t)((e >> 6) * 1024 + s * 64 + (e & 63));
}
// (behind the 16 d bytes of K)
__host__ __device__ __forceinline__ uint32_t kv8_v_offset(int s, int e) {
  return (uint32_t)((e >> 6) * 1024 + (s >> 2) * 256 + (e & 15) * 16 + ((e >> 4) & 3) * 4 + (s & 3));
}

// The scale of a block whose largest magnitude has the bits a: max / 448, at least
// 2^-64.  A block that holds a NaN or an infinity (bits of at least 0x7F800000, above every
// finite magnitude) gets the scale NaN, and the codes 0 instead of NaN codes: a query
// that does not see the token then adds 0 * 0 for it.
__device__ __forceinline__ float kv8_scale(uint32_t a) {
  return a < 0x7F800000u ? fmaxf(__uint_as_float(a) * (1.f / 448.f), 0x1p-64f) : NAN;
}
// four values, times the reciprocals of their scales, to four codes (round to nearest even;
// |y| / s <= 448 (1 + 2^-22) rounds to at most 448)
__device__ __forceinline__ uint32_t kv8_pack(float y0, float y1, float y2, float y3) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y0, y1, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y2, y3, w, true);
  return (uint32_t)w;
}
// four values of one block
__device__ __forceinline__ uint32_t kv8_codes(float y0, float y1, float y2, float y3, float scale) {
  const float inv = 1.f / scale;
  const uint32_t w = kv8_pack(y0 * inv, y1 * inv, y2 * inv, y3 * inv);
  return scale == scale ? w : 0u;
}

}  // namespace sevo
