// The 8-bit key-value cache as it is written and read back: QK-norm + RoPE + append,
// pages of the bf16 pool to 8-bit pages, and 8-bit pages to the bf16 pool.
#include "kernels.h"
#include "kv8.h"

namespace sevo {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Calls whose data is larger than the last-level cache read their sources past the caches: kept
// there they would only put out what is about to be written.  Plain / past the caches, us:
// to 8 bits 407 MB 82.5 / 67.8, 288 MB 50.3 / 49.5, 199 MB 35.0 / 35.5; back 407 MB 84.6 / 81.4;
// append 290 MB 57.2 / 52.5, 212 MB 41.7 / 40.6.  With the stores below past the caches as well
// the 407 MB take 64 to 66 us and 70 to 72, 5.7 to 6.3 TB/s: bound by HBM.
constexpr size_t kOnceBytes = (size_t)256 << 20;
template <bool ONCE, typename V>
__device__ __forceinline__ V load(const V* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}

}  // namespace

// One workgroup per token and 4 NP * HPW of its heads.  D / 4 lanes hold a head, four
// dims each, so a wave reads HPW = 256 / D heads of the projection in one 1 KB access; the
// rotate-half partner of a dim is in the lane half a head away, the norm's sum and the
// block's largest magnitude are lane reductions.
template <int D, int NP, bool ONCE>
__global__ __launch_bounds__(256) void append8_kernel(RopeAppendArgs a, int n_rows,
                                                      uint8_t* __restrict__ pool) {
  constexpr int LPH = D / 4, HPW = 64 / LPH, HALF = D / 2;
  const int i = xcd_row(blockIdx.x, gridDim.x);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l = lane % LPH, e = 4 * l, m = e % HALF;
  const int H = a.hq + 2 * a.hkv;
  const int h0 = (blockIdx.y * 4 * NP + w) * HPW + lane / LPH;  // head of pass j: h0 + 4 HPW j
  const float* row = a.qkv + (size_t)i * H * D;
  f32x4 u[NP];
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    const int hh = h0 + 4 * HPW * j;
    u[j] = hh < H ? load<ONCE>(reinterpret_cast<const f32x4*>(row + (size_t)hh * D + e))
                  : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int p = a.positions[i];
  const bool pos_ok = p >= 0 && p < a.max_pos;
  f32x4 c{0.f, 0.f, 0.f, 0.f}, s = c;
  int page = -1;
  if (pos_ok) {
    c = *reinterpret_cast<const f32x4*>(a.rope_cos + (size_t)p * HALF + m);
    s = *reinterpret_cast<const f32x4*>(a.rope_sin + (size_t)p * HALF + m);
    const int pr = a.row_of_token ? a.row_of_token[i] : i;
    if ((p >> 4) < a.max_pages && pr >= 0 && pr < n_rows) {
      const int id = a.page_table[(size_t)pr * a.max_pages + (p >> 4)];
      if (id >= 0 && (int64_t)id < a.num_pages) page = id;
    }
  }
  if (e < HALF) s = -s;
  u32x2 gq{0u, 0u}, gk = gq;
  if (a.qk_norm) {
    gq = *reinterpret_cast<const u32x2*>(a.q_gain + e);
    gk = *reinterpret_cast<const u32x2*>(a.k_gain + e);
  }
  const int slot = p & 15;
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    const int hh = h0 + 4 * HPW * j;
    f32x4 v = u[j];
    if (a.qk_norm) {
      float ss = v.x * v.x + v.y * v.y + v.z * v.z + v.w * v.w;
      ss += lane_xor<1>(ss);
      ss += lane_xor<2>(ss);
      ss += lane_xor<4>(ss);
      ss += lane_xor<8>(ss);
      if constexpr (LPH == 32) ss = xor16_sum(ss);
      const float inv = 1.0f / sqrtf(ss / (float)D + a.eps);
      const u32x2 g = hh < a.hq ? gq : gk;
      const f32x4 n = {v.x * inv * bf16_lo(g.x), v.y * inv * bf16_hi(g.x), v.z * inv * bf16_lo(g.y),
                       v.w * inv * bf16_hi(g.y)};
      if (hh < a.hq + a.hkv) v = n;
    }
    f32x4 o;
#pragma unroll
    for (int x = 0; x < 4; ++x) o[x] = lane_xor<LPH / 2>(v[x]);
    if (hh < a.hq + a.hkv) {
#pragma unroll
      for (int x = 0; x < 4; ++x) v[x] = pos_ok ? v[x] * c[x] + o[x] * s[x] : 0.f;
    }
    uint32_t top = max(max(mag(v.x), mag(v.y)), max(mag(v.z), mag(v.w)));
    top = max(top, lane_xor<1>(top));
    top = max(top, lane_xor<2>(top));
    top = max(top, lane_xor<4>(top));
    top = max(top, lane_xor<8>(top));
    if constexpr (LPH == 32) top = max(top, lane_xor<16>(top));
    if (hh < a.hq) {
      *reinterpret_cast<u32x2*>(a.q_out + ((size_t)i * a.hq + hh) * D + e) =
          u32x2{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)};
    } else if (hh < H && page >= 0) {
      const float scale = kv8_scale(top);
      const uint32_t codes = kv8_codes(v.x, v.y, v.z, v.w, scale);
      const bool is_k = hh < a.hq + a.hkv;
      const int kh = is_k ? hh - a.hq : hh - a.hq - a.hkv;
      uint8_t* t = pool + ((size_t)page * a.hkv + kh) * kv8_tile_bytes(D);
      if (l == 0)
        reinterpret_cast<float*>(t + 32 * D)[(is_k ? 0 : kPage) + slot] = scale;
      if (is_k) {
        *reinterpret_cast<uint32_t*>(t + kv8_k_offset(slot, e)) = codes;
      } else {
        // dims 4 l .. + 3 are 16 bytes apart: one byte each
        uint8_t* d = t + 16 * D + kv8_v_offset(slot, e);
        d[0] = (uint8_t)codes;
        d[16] = (uint8_t)(codes >> 8);
        d[32] = (uint8_t)(codes >> 16);
        d[48] = (uint8_t)(codes >> 24);
      }
    }
  }
}

hipError_t launch_append8(const RopeAppendArgs& a, int n_rows, uint8_t* pool, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  const int per = a.d == 128 ? 8 : 16;  // heads of one pass of a workgroup
  const int passes = (a.hq + 2 * a.hkv + per - 1) / per;
  auto go = [&](auto kern, int np) {
    hipLaunchKernelGGL(kern, dim3(a.n, (passes + np - 1) / np), dim3(256), 0, st, a, n_rows, pool);
    return hipGetLastError();
  };
  if (a.n < 512)
    return a.d == 128 ? go(append8_kernel<128, 1, false>, 1) : go(append8_kernel<64, 1, false>, 1);
  const size_t bytes = (size_t)a.n * a.d * (6 * (size_t)a.hq + 10 * (size_t)a.hkv);
  if (bytes > kOnceBytes)
    return a.d == 128 ? go(append8_kernel<128, 6, true>, 6) : go(append8_kernel<64, 3, true>, 3);
  return a.d == 128 ? go(append8_kernel<128, 6, false>, 6) : go(append8_kernel<64, 3, false>, 3);
}

namespace {

// tile j of a call: its source and destination tiles, null where the id is outside the pool
struct TilePair {
  const char* src;
  char* dst;
};
__device__ __forceinline__ TilePair tile_pair(const KvPagesArgs& a, uint32_t tile, size_t src_bytes,
                                              size_t dst_bytes) {
  TilePair t{nullptr, nullptr};
  const uint32_t j = tile / (uint32_t)a.hkv, h = tile - j * (uint32_t)a.hkv;
  const int64_t s = a.src_pages ? a.src_pages[j] : (int64_t)j;
  const int64_t d = a.dst_pages ? a.dst_pages[j] : (int64_t)j;
  if (s >= 0 && s < a.src_num_pages)
    t.src = static_cast<const char*>(a.src) + ((size_t)s * a.hkv + h) * src_bytes;
  if (d >= 0 && d < a.dst_num_pages)
    t.dst = static_cast<char*>(a.dst) + ((size_t)d * a.hkv + h) * dst_bytes;
  return t;
}

template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const char* p, uint32_t off) {
  return p ? load<ONCE>(reinterpret_cast<const u32x4*>(p + off)) : u32x4{0u, 0u, 0u, 0u};
}

}  // namespace

// bf16 tiles (K [d/32][16][32], V [d][16]) to 8-bit tiles: a wave takes 128 / D tiles.  K: four
// lanes a token, eight dims of every 32-dim block each.  V: lane (b, token half, a) holds
// the dims 64 a + 16 c + b, c < 4, of eight tokens; a token's largest magnitude is over
// the lanes of its half.
template <int D, bool ONCE>
__global__ __launch_bounds__(256) void pack_kv8_kernel(KvPagesArgs a, uint32_t tiles) {
  constexpr int TPW = 128 / D, NI = D / 32;
  constexpr uint32_t kSrc = 64 * D, kDst = kv8_tile_bytes(D);
  const int lane = threadIdx.x & 63;
  const uint32_t wave = blockIdx.x * 4 + (threadIdx.x >> 6);
  const uint32_t waves = gridDim.x * 4;
  for (uint32_t t0 = wave * TPW; t0 < tiles; t0 += waves * TPW) {
    // K: tile by tile, the whole wave
    const int s = lane >> 2, q = lane & 3;
#pragma unroll
    for (int x = 0; x < TPW; ++x) {
      if (t0 + x >= tiles) break;
      const TilePair t = tile_pair(a, t0 + x, kSrc, kDst);
      if (!t.dst) continue;
      float y[NI][8];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const u32x4 v = load16<ONCE>(t.src, i * 1024 + lane * 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          y[i][2 * k] = bf16_lo(v[k]);
          y[i][2 * k + 1] = bf16_hi(v[k]);
          top = max(top, max(mag(y[i][2 * k]), mag(y[i][2 * k + 1])));
        }
      }
      top = max(top, lane_xor<1>(top));
      top = max(top, lane_xor<2>(top));
      const float scale = t.src ? kv8_scale(top) : 0.f;
      const float use = t.src ? scale : 1.f;
#pragma unroll
      for (int i = 0; i < NI; ++i)
        *reinterpret_cast<u32x2*>(t.dst + kv8_k_offset(s, 32 * i + 8 * q)) =
            u32x2{kv8_codes(y[i][0], y[i][1], y[i][2], y[i][3], use),
                  kv8_codes(y[i][4], y[i][5], y[i][6], y[i][7], use)};
      if (q == 0) reinterpret_cast<float*>(t.dst + 32 * D)[s] = scale;
    }
    // V: at d = 64 each half wave has a tile of its own
    const int h = lane & 1, b = (lane >> 1) & 15, up = lane >> 5;
    const uint32_t tile = D == 64 ? t0 + up : t0;
    TilePair t{nullptr, nullptr};
    if (tile < tiles) t = tile_pair(a, tile, kSrc, kDst);
    const int a64 = D == 64 ? 0 : up;
    float y[4][8];
    uint32_t top[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const u32x4 v = load16<ONCE>(t.src, 32 * D + (64 * a64 + 16 * c + b) * 32 + h * 16);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        y[c][2 * k] = bf16_lo(v[k]);
        y[c][2 * k + 1] = bf16_hi(v[k]);
        top[2 * k] = max(top[2 * k], mag(y[c][2 * k]));
        top[2 * k + 1] = max(top[2 * k + 1], mag(y[c][2 * k + 1]));
      }
    }
    float scale[8], inv[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t m = top[k];
      m = max(m, lane_xor<2>(m));
      m = max(m, lane_xor<4>(m));
      m = max(m, lane_xor<8>(m));
      m = max(m, lane_xor<16>(m));
      if constexpr (D == 128) m = max(m, lane_xor<32>(m));
      scale[k] = kv8_scale(m);
      inv[k] = 1.f / scale[k];
    }
    if (!t.dst) continue;
    bool nan = false;
#pragma unroll
    for (int k = 0; k < 8; ++k) nan |= scale[k] != scale[k];
    if (nan) {  // (rare: a token's codes are 0 where its block holds a NaN or an infinity)
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (scale[k] != scale[k]) y[c][k] = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (scale[k] != scale[k]) inv[k] = 0.f;
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      u32x4 w;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        w[c] = kv8_pack(y[c][4 * g] * inv[4 * g], y[c][4 * g + 1] * inv[4 * g + 1],
                        y[c][4 * g + 2] * inv[4 * g + 2], y[c][4 * g + 3] * inv[4 * g + 3]);
      // (past the caches: 2000 pages of 8 heads 42.4 -> 40.0 us, 4096 67.8 -> 66.3)
      __builtin_nontemporal_store(
          w, reinterpret_cast<u32x4*>(t.dst + 16 * D + a64 * 1024 + (2 * h + g) * 256 + b * 16));
    }
    if (b == 0 && (D == 64 || up == 0)) {
      float* vs = reinterpret_cast<float*>(t.dst + 32 * D) + kPage + 8 * h;
#pragma unroll
      for (int k = 0; k < 8; ++k) vs[k] = t.src ? scale[k] : 0.f;
    }
  }
}

// 8-bit tiles to bf16 tiles, the product of code and scale rounded once.  A wave a tile:
// K lane (token, 16 dims) as two 16-byte stores a 64-dim block, V lane (dims 16 c + b, four
// tokens) as 8-byte stores.
template <int D, bool ONCE>
__global__ __launch_bounds__(256) void unpack_kv8_kernel(KvPagesArgs a, uint32_t tiles) {
  constexpr int NA = D / 64;
  constexpr uint32_t kSrc = kv8_tile_bytes(D), kDst = 64 * D;
  const int lane = threadIdx.x & 63;
  const uint32_t wave = blockIdx.x * 4 + (threadIdx.x >> 6);
  const uint32_t waves = gridDim.x * 4;
  for (uint32_t tile = wave; tile < tiles; tile += waves) {
    const TilePair t = tile_pair(a, tile, kSrc, kDst);
    if (!t.dst) continue;
    const int s = lane >> 2, q = lane & 3, b = lane & 15, g = lane >> 4;
    u32x4 k[NA], v[NA];
#pragma unroll
    for (int x = 0; x < NA; ++x) {
      k[x] = load16<ONCE>(t.src, x * 1024 + lane * 16);
      v[x] = load16<ONCE>(t.src, 16 * D + x * 1024 + lane * 16);
    }
    const float ks = t.src ? reinterpret_cast<const float*>(t.src + 32 * D)[s] : 0.f;
    const u32x4 vsw = load16<ONCE>(t.src, 32 * D + 64 + g * 16);
    const f32x4 vs = __builtin_bit_cast(f32x4, vsw);
#pragma unroll
    for (int x = 0; x < NA; ++x) {
      uint32_t o[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)k[x][i], false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)k[x][i], true);
        o[2 * i] = pack_bf16x2(lo[0] * ks, lo[1] * ks);
        o[2 * i + 1] = pack_bf16x2(hi[0] * ks, hi[1] * ks);
      }
      // dims 64 x + 16 q .. + 15 of token s
      char* d = t.dst + (2 * x + (q >> 1)) * 1024 + s * 64 + (q & 1) * 32;
      // (past the caches: 4099 pages of 8 heads 81 -> 72 us, 2000 44 -> 38; V's 8-byte stores not: 79)
      __builtin_nontemporal_store(u32x4{o[0], o[1], o[2], o[3]}, reinterpret_cast<u32x4*>(d));
      __builtin_nontemporal_store(u32x4{o[4], o[5], o[6], o[7]}, reinterpret_cast<u32x4*>(d + 16));
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[x][c], false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[x][c], true);
        *reinterpret_cast<u32x2*>(t.dst + 32 * D + (64 * x + 16 * c + b) * 32 + g * 8) =
            u32x2{pack_bf16x2(lo[0] * vs.x, lo[1] * vs.y), pack_bf16x2(hi[0] * vs.z, hi[1] * vs.w)};
      }
    }
  }
}

hipError_t launch_pack_kv8(const KvPagesArgs& a, int to8, hipStream_t st) {
  const uint32_t tiles = (uint32_t)(a.count * a.hkv);
  if (tiles == 0) return hipSuccess;
  const uint32_t per = 4 * (to8 && a.d == 64 ? 2 : 1);  // tiles of one workgroup and pass
  const uint32_t need = (tiles + per - 1) / per;
  const dim3 grid(need < 65536 ? need : 65536);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a, tiles);
    return hipGetLastError();
  };
  if ((size_t)tiles * (96 * a.d + 128) > kOnceBytes) {
    if (to8) return a.d == 128 ? go(pack_kv8_kernel<128, true>) : go(pack_kv8_kernel<64, true>);
    return a.d == 128 ? go(unpack_kv8_kernel<128, true>) : go(unpack_kv8_kernel<64, true>);
  }
  if (to8) return a.d == 128 ? go(pack_kv8_kernel<128, false>) : go(pack_kv8_kernel<64, false>);
  return a.d == 128 ? go(unpack_kv8_kernel<128, false>) : go(unpack_kv8_kernel<64, false>);
}

}  // namespace sevo
