// Decode attention over the paged 8-bit cache: one or a few new tokens per candidate,
// split over the cache's length and joined.
//
//   z_u = scale ks_u (q . kc_u),  p = exp(z - max),  o = sum_u p_u vs_u vc_u / sum_u p_u
//
// with the codes kc, vc and the scales ks, vs of token u: the scales are one factor of a
// score and of a probability, so the codes themselves go into the matrix products, as
// bf16, which holds every e4m3 value exactly.  A query row (token t of the m new ones, head) sees
// the keys u < len - m + t + 1.
//
// Work: the pages of all candidates are cut into splits of about equal size, found on the
// device from the lengths alone (a candidate with few pages gets one split, whatever the page table's
// width), one 256-thread workgroup per (kv head, split).  Its waves take pairs of pages in
// turn, each with its own running maximum and sum, and meet in LDS at the end; a second
// kernel joins the splits of a candidate in order.  Per pair of pages and wave:
//   QK   S = K Q^T, 16x16x32 matrix instructions: rows = the page's tokens, columns = 16 query
//        rows.  Lane (column l % 16, g = l / 16) gets the scores of tokens 4 g .. + 3 of either page.
//   PV   O^T = V^T P^T: the 32-deep axis is the pair's tokens in the order in which the lanes hold
//        their scores, so p needs no exchange.  p vs is split into two bf16 parts, hi + lo
//        (to 2^-17 of itself): the probabilities keep their 32-bit accuracy.
// More than 16 query rows per kv head are further column tiles of the same page (NC), so
// the cache is read once for all new tokens.
#include "kernels.h"
#include "kv8.h"

namespace sevo {

namespace {

constexpr float kLazyLog2 = 8.f;  // the accumulators are rescaled when a maximum rises by more than 2^8

// the eight codes of two words to bf16, exactly
__device__ __forceinline__ bf16x8v codes_bf16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(
      bf16x8v,
      u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true))});
}

__device__ __forceinline__ int pages_of(const int32_t* lens, int i, int max_pages) {
  int len = lens[i];
  len = len < 0 ? 0 : (len > max_pages * kPage ? max_pages * kPage : len);
  return (len + kPage - 1) / kPage;
}

// The split plan, the same in every workgroup of both kernels: splits of at most `chunk`
// pages, chunk = max(kMinChunk, all pages / target); candidate i has max(1, ceil(pages_i /
// chunk)) of them.  Calls of a 256-thread workgroup.
struct Split {
  int cand, index, count, first;  // candidate, split of it, its number of splits, its first flat id
};
struct PlanLds {
  long long sum[4];
  int scan[4], cand, index, count, first;
};

__device__ __forceinline__ int wave_scan(int v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// flat >= 0: the split with that flat id (cand -1 behind the last); flat < 0: all of candidate ~flat
__device__ __forceinline__ Split find_split(const int32_t* lens, int n, int max_pages, int target,
                                            int flat, PlanLds& L) {
  const int t = threadIdx.x, w = t >> 6;
  long long own = 0;
  for (int i = t; i < n; i += 256) own += pages_of(lens, i, max_pages);
#pragma unroll
  for (int d = 32; d; d >>= 1) own += __shfl_xor(own, d);
  if ((t & 63) == 0) L.sum[w] = own;
  if (t == 0) L.cand = -1;
  __syncthreads();
  const long long all = L.sum[0] + L.sum[1] + L.sum[2] + L.sum[3];
  long long chunk = (all + target - 1) / target;
  if (chunk < kAttn8MinChunk) chunk = kAttn8MinChunk;
  int base = 0;
  for (int i0 = 0; i0 < n; i0 += 256) {
    const int i = i0 + t;
    int s = 0;
    if (i < n) {
      const int pg = pages_of(lens, i, max_pages);
      s = pg ? (int)((pg + chunk - 1) / chunk) : 1;
    }
    const int in = wave_scan(s);
    if ((t & 63) == 63) L.scan[w] = in;
    __syncthreads();
    int before = base;
    for (int x = 0; x < w; ++x) before += L.scan[x];
    const int first = before + in - s;
    if (flat >= 0 ? (s > 0 && flat >= first && flat < first + s) : i == ~flat) {
      L.cand = i;
      L.index = flat - first;
      L.count = s;
      L.first = first;
    }
    base += L.scan[0] + L.scan[1] + L.scan[2] + L.scan[3];
    __syncthreads();
  }
  // the same in every lane: scalars, so that what follows from them is scalar too
  return Split{__builtin_amdgcn_readfirstlane(L.cand), __builtin_amdgcn_readfirstlane(L.index),
               __builtin_amdgcn_readfirstlane(L.count), __builtin_amdgcn_readfirstlane(L.first)};
}

}  // namespace

template <int D, int NC>
__global__ __launch_bounds__(256, NC == 1 ? 2 : 1) void attn8_split_kernel(Attn8Args a) {
  constexpr int NA = D / 64;   // 64-dim blocks of a tile
  constexpr int NB = D / 16;   // 16-dim blocks of the output
  constexpr int kStride = D + 4;
  __shared__ PlanLds plan;
  __shared__ float w_m[4][16], w_l[4][16];
  __shared__ __align__(16) float w_acc[4][16][kStride];

  // workgroups in the order (split, kv head, NC column tiles): the heads of a page, adjacent in
  // the pool, are read together, each through the XCD that its workgroup number falls to
  const int per = a.hkv * a.col_tiles;
  const int flat = blockIdx.x / per, rest = blockIdx.x - flat * per;
  const int c = rest / a.col_tiles, cg = rest - c * a.col_tiles;
  const Split sp = find_split(a.seq_lens, a.n, a.max_pages, a.target, flat, plan);
  const int i = sp.cand;
  if (i < 0) return;
  int len = a.seq_lens[i];
  len = len < 0 ? 0 : (len > a.max_pages * kPage ? a.max_pages * kPage : len);
  const int npg = (len + kPage - 1) / kPage;
  int m = a.q_lens ? a.q_lens[i] : a.tokens;
  m = m < 0 ? 0 : (m > a.tokens ? a.tokens : m);
  // the candidate's pages in even shares, each an even number of pages
  const int share = ((npg + sp.count - 1) / sp.count + 1) & ~1;
  const int pbeg = sp.index * share;
  const int pend = min(npg, pbeg + share);

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int G = a.hq / a.hkv, cols = a.tokens * G;

  bf16x8v qf[NC][NA][2];
  int lim[NC];  // keys that the lane's column sees
#pragma unroll
  for (int t = 0; t < NC; ++t) {
    const int cc = (cg * NC + t) * 16 + col;
    const int tok = cc / G, head = cc - tok * G;
    const bool on = cc < cols && tok < m;
    lim[t] = on ? len - m + tok + 1 : 0;
    const bf16_t* qr = a.q + (((size_t)i * a.tokens + tok) * a.hq + (size_t)c * G + head) * D;
#pragma unroll
    for (int x = 0; x < NA; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 w{0u, 0u, 0u, 0u};
        if (on) w = *reinterpret_cast<const u32x4*>(qr + 64 * x + 16 * grp + 8 * h);
        qf[t][x][h] = __builtin_bit_cast(bf16x8v, w);
      }
  }
  // pages that every query row of the candidate sees in full need no mask (columns
  // without a row compute what is not stored)
  const int full = (len - m + 1) / kPage;
  float m_run[NC], l_run[NC];
  f32x4 acc[NC][NB];
#pragma unroll
  for (int t = 0; t < NC; ++t) {
    m_run[t] = -INFINITY;
    l_run[t] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int32_t* ptr = a.page_table + (size_t)i * a.max_pages;
  const int pairs = (pend - pbeg + 1) / 2;                 // pairs of the split
  const int mine = pairs > wave ? (pairs - wave + 3) / 4 : 0;  // the wave's: wave, wave + 4, ...
  // page ids of 64 of the wave's pairs, one pair per lane; -1: outside the pool
  int id0 = -1, id1 = -1;
  auto fetch_ids = [&](int k0) {
    const int pg = pbeg + 2 * (wave + 4 * (k0 + lane));
    id0 = id1 = -1;
    if (k0 + lane < mine) {
      const int x = ptr[pg];
      id0 = x >= 0 && x < a.num_pages ? x : -1;
      if (pg + 1 < pend) {
        const int y = ptr[pg + 1];
        id1 = y >= 0 && y < a.num_pages ? y : -1;
      }
    }
  };
  struct Page {
    u32x4 k[NA], v[NA], ks, vs;
  };
  constexpr uint32_t kTile = kv8_tile_bytes(D);
  const uint32_t koff = col * 64 + grp * 16, voff = lane * 16;
  auto load = [&](Page& r, int id) {
    const uint8_t* base = a.kv_pool + (id < 0 ? 0 : ((size_t)id * a.hkv + c) * kTile);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(base), 0, id < 0 ? 0 : (int)kTile, 0x00020000);
#pragma unroll
    for (int x = 0; x < NA; ++x)
      r.k[x] = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)koff, x * 1024, 2);
#pragma unroll
    for (int x = 0; x < NA; ++x)
      r.v[x] = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)voff, 16 * D + x * 1024, 2);
    r.ks = __builtin_amdgcn_raw_buffer_load_b128(rs, grp * 16, 32 * D, 2);
    r.vs = __builtin_amdgcn_raw_buffer_load_b128(rs, grp * 16, 32 * D + 64, 2);
  };

  // one pair of pages, the first at logical page pg; ok0, ok1: in the pool
  auto consume = [&](Page& A, Page& B, int pg, bool ok0, bool ok1) {
    const bool masked = pg + 2 > full || !ok0 || !ok1;
    const int u0 = pg * kPage + 4 * grp;  // the lane's tokens u0 .. + 3 and u0 + 16 .. + 3
    if (masked) {
      // what lies behind the last key may hold anything, also NaN codes
      const int n0 = len - u0, n1 = len - u0 - kPage;
      const uint32_t k0 = n0 >= 4 ? ~0u : (n0 <= 0 ? 0u : (1u << (8 * n0)) - 1u);
      const uint32_t k1 = n1 >= 4 ? ~0u : (n1 <= 0 ? 0u : (1u << (8 * n1)) - 1u);
#pragma unroll
      for (int x = 0; x < NA; ++x) {
        A.v[x] &= k0;
        B.v[x] &= k1;
      }
    }
    const f32x4 ks0 = __builtin_bit_cast(f32x4, A.ks) * a.scale_log2;
    const f32x4 ks1 = __builtin_bit_cast(f32x4, B.ks) * a.scale_log2;
    const f32x4 vs0 = __builtin_bit_cast(f32x4, A.vs), vs1 = __builtin_bit_cast(f32x4, B.vs);
    f32x4 s0[NC], s1[NC];
#pragma unroll
    for (int t = 0; t < NC; ++t) s0[t] = s1[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NA; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8v wa = codes_bf16(A.k[x][2 * h], A.k[x][2 * h + 1]);
        const bf16x8v wb = codes_bf16(B.k[x][2 * h], B.k[x][2 * h + 1]);
#pragma unroll
        for (int t = 0; t < NC; ++t) {
          s0[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa, qf[t][x][h], s0[t], 0, 0, 0);
          s1[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, qf[t][x][h], s1[t], 0, 0, 0);
        }
      }
    bf16x8v ph[NC], pl[NC];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
      float z[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        z[e] = s0[t][e] * ks0[e];
        z[4 + e] = s1[t][e] * ks1[e];
      }
      if (masked) {
        const int v0 = ok0 ? lim[t] - u0 : 0, v1 = ok1 ? lim[t] - u0 - kPage : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[e] = e < v0 ? z[e] : -INFINITY;
          z[4 + e] = e < v1 ? z[4 + e] : -INFINITY;
        }
      }
      float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])),
                        fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
      top = xor32_max(xor16_max(top));
      const bool raise = top > m_run[t] + kLazyLog2;
      if (__builtin_amdgcn_ballot_w64(raise)) {
        const float mn = raise ? top : m_run[t];
        const float alpha = raise ? __builtin_amdgcn_exp2f(m_run[t] - mn) : 1.f;  // 0 on the first page
        l_run[t] *= alpha;
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[t][b] *= alpha;
        m_run[t] = mn;
      }
      const float mz = m_run[t] == -INFINITY ? 0.f : m_run[t];
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float p[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float pr = __builtin_amdgcn_exp2f(z[e + y] - mz);
          l_run[t] += pr;
          const float vs = e < 4 ? vs0[(e + y) & 3] : vs1[(e + y) & 3];
          // a masked token's scale may be anything: it does not enter
          p[y] = masked && z[e + y] == -INFINITY ? 0.f : pr * vs;
        }
        const __bf16 h0 = (__bf16)p[0], h1 = (__bf16)p[1];
        hi[e / 2] = __builtin_bit_cast(uint32_t, bf16x2v{h0, h1});
        lo[e / 2] = pack_bf16x2(p[0] - (float)h0, p[1] - (float)h1);
      }
      ph[t] = __builtin_bit_cast(bf16x8v, u32x4{hi[0], hi[1], hi[2], hi[3]});
      pl[t] = __builtin_bit_cast(bf16x8v, u32x4{lo[0], lo[1], lo[2], lo[3]});
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const bf16x8v w = codes_bf16(A.v[b / 4][b % 4], B.v[b / 4][b % 4]);
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        acc[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, pl[t], acc[t][b], 0, 0, 0);
        acc[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, ph[t], acc[t][b], 0, 0, 0);
      }
    }
  };

  if (mine > 0) {
    fetch_ids(0);
    Page A0, B0, A1, B1;
    auto ida = [&](int k) { return __builtin_amdgcn_readlane(id0, k & 63); };
    auto idb = [&](int k) { return __builtin_amdgcn_readlane(id1, k & 63); };
    int a0 = ida(0), b0 = idb(0), a1 = -1, b1 = -1;
    load(A0, a0);
    load(B0, b0);
    for (int k = 0;;) {
      // the next pair's loads are in flight while this one is consumed (past the
      // wave's last pair the ids are -1: nothing is read)
      if (((k + 1) & 63) == 0) fetch_ids(k + 1);
      a1 = ida(k + 1);
      b1 = idb(k + 1);
      load(A1, a1);
      load(B1, b1);
      consume(A0, B0, pbeg + 2 * (wave + 4 * k), a0 >= 0, b0 >= 0);
      if (++k >= mine) break;
      if (((k + 1) & 63) == 0) fetch_ids(k + 1);
      a0 = ida(k + 1);
      b0 = idb(k + 1);
      load(A0, a0);
      load(B0, b0);
      consume(A1, B1, pbeg + 2 * (wave + 4 * k), a1 >= 0, b1 >= 0);
      if (++k >= mine) break;
    }
  }

  // the four waves of each column tile, in order; a candidate's only split is the result
#pragma unroll
  for (int t = 0; t < NC; ++t) {
    const float l = xor32_sum(xor16_sum(l_run[t]));
    if (t) __syncthreads();
    if (grp == 0) {
      w_m[wave][col] = m_run[t];
      w_l[wave][col] = l;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
      *reinterpret_cast<f32x4*>(&w_acc[wave][col][16 * b + 4 * grp]) = acc[t][b];
    __syncthreads();
    for (int idx = threadIdx.x; idx < 16 * D; idx += 256) {
      const int j = idx / D, e = idx - j * D;
      const int cc = (cg * NC + t) * 16 + j;
      const int tok = cc / G, head = c * G + cc - tok * G;
      if (cc >= cols) continue;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < 4; ++w) M = fmaxf(M, w_m[w][j]);
      const float mz = M == -INFINITY ? 0.f : M;
      float S = 0.f, O = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = exp2f(w_m[w][j] - mz);
        S += w_l[w][j] * f;
        O += w_acc[w][j][e] * f;
      }
      if (sp.count == 1) {
        if (tok < m || a.clear_rest)
          a.out[(((size_t)i * a.tokens + tok) * a.hq + head) * D + e] =
              f32_to_bf16(S == 0.f || tok >= m ? 0.f : O / S);
      } else {
        const size_t slot = ((size_t)flat * a.hkv + c) * cols + cc;
        a.part_acc[slot * D + e] = O;
        if (e == 0) {
          a.part_ml[slot * 2] = M;
          a.part_ml[slot * 2 + 1] = S;
        }
      }
    }
  }
}

// Joins the splits of one (candidate, kv head, query row), in split order within each wave and
// then over the waves, so the same call gives the same bits.
template <int D>
__global__ __launch_bounds__(256) void attn8_join_kernel(Attn8Args a) {
  constexpr int E = D / 64;
  __shared__ PlanLds plan;
  __shared__ float w_m[4], w_l[4], w_acc[4][D];
  const int rows = a.hq * a.tokens;
  const int i = blockIdx.x / rows;
  const Split sp = find_split(a.seq_lens, a.n, a.max_pages, a.target, ~i, plan);
  if (sp.count <= 1) return;
  const int G = a.hq / a.hkv, cols = a.tokens * G;
  const int c = (blockIdx.x - i * rows) / cols, cc = blockIdx.x - i * rows - c * cols;
  const int tok = cc / G, head = c * G + cc - tok * G;
  int m = a.q_lens ? a.q_lens[i] : a.tokens;
  m = m < 0 ? 0 : (m > a.tokens ? a.tokens : m);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  bf16_t* o = a.out + (((size_t)i * a.tokens + tok) * a.hq + head) * D;
  if (tok >= m) {
    if (a.clear_rest && threadIdx.x < D) o[threadIdx.x] = 0;
    return;
  }
  const size_t step = (size_t)a.hkv * cols;  // slots between a candidate's splits
  const size_t slot0 = ((size_t)sp.first * a.hkv + c) * cols + cc;
  float M = -INFINITY, S = 0.f, O[E];
#pragma unroll
  for (int e = 0; e < E; ++e) O[e] = 0.f;
  // a wave takes every fourth split, four of them in flight
  for (int s0 = w; s0 < sp.count; s0 += 16) {
    float ms[4], ls[4], ac[4][E];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int s = s0 + 4 * y;
      ms[y] = -INFINITY;
      ls[y] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) ac[y][e] = 0.f;
      if (s < sp.count) {
        const size_t slot = slot0 + s * step;
        ms[y] = a.part_ml[slot * 2];
        ls[y] = a.part_ml[slot * 2 + 1];
#pragma unroll
        for (int e = 0; e < E; ++e) ac[y][e] = a.part_acc[slot * D + lane + 64 * e];
      }
    }
    float top = M;
#pragma unroll
    for (int y = 0; y < 4; ++y) top = fmaxf(top, ms[y]);
    const float tz = top == -INFINITY ? 0.f : top;
    const float f0 = exp2f(M - tz);
    S *= f0;
#pragma unroll
    for (int e = 0; e < E; ++e) O[e] *= f0;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float f = exp2f(ms[y] - tz);
      S += ls[y] * f;
#pragma unroll
      for (int e = 0; e < E; ++e) O[e] += ac[y][e] * f;
    }
    M = top;
  }
  if (lane == 0) {
    w_m[w] = M;
    w_l[w] = S;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) w_acc[w][lane + 64 * e] = O[e];
  __syncthreads();
  if (threadIdx.x < D) {
    const int e = threadIdx.x;
    float T = fmaxf(fmaxf(w_m[0], w_m[1]), fmaxf(w_m[2], w_m[3]));
    T = T == -INFINITY ? 0.f : T;
    float L = 0.f, A = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float f = exp2f(w_m[x] - T);
      L += w_l[x] * f;
      A += w_acc[x][e] * f;
    }
    o[e] = f32_to_bf16(L == 0.f ? 0.f : A / L);
  }
}

template <int D>
static hipError_t launch_attn8_d(const Attn8Args& a, int nc, hipStream_t st) {
  const dim3 grid((unsigned)(a.hkv * a.col_tiles * a.max_splits));
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a); };
  if (nc == 1) go(attn8_split_kernel<D, 1>);
  else if (nc == 2) go(attn8_split_kernel<D, 2>);
  else go(attn8_split_kernel<D, 4>);
  hipError_t e = hipGetLastError();
  // pages that one split holds: every candidate has one, nothing to join
  if (e != hipSuccess || a.max_pages <= kAttn8MinChunk) return e;
  hipLaunchKernelGGL(attn8_join_kernel<D>, dim3((unsigned)(a.hq * a.tokens * a.n)), dim3(256),
                     0, st, a);
  return hipGetLastError();
}

Attn8Plan plan_attn8(int n, int hq, int hkv, int tokens, int max_pages) {
  Attn8Plan p;
  const int cols = tokens * (hq / hkv), tiles = (cols + 15) / 16;
  p.nc = tiles >= 3 ? 4 : tiles;
  p.col_tiles = (tiles + p.nc - 1) / p.nc;
  const int per = hkv * p.col_tiles;  // workgroups of a split
  p.target = (kAttn8Workgroups + per - 1) / per;
  // at most all pages / chunk + one more a candidate, and never more than the pages' own count
  const long long most = (long long)n * ((max_pages + kAttn8MinChunk - 1) / kAttn8MinChunk);
  const long long s = (long long)p.target + n;
  p.max_splits = s < most ? s : most;
  return p;
}

hipError_t launch_attn8(const Attn8Args& a, const Attn8Plan& p, hipStream_t st) {
  return a.d == 128 ? launch_attn8_d<128>(a, p.nc, st) : launch_attn8_d<64>(a, p.nc, st);
}

}  // namespace sevo
