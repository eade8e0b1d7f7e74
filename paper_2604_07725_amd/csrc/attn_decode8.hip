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
// width), one workgroup of four or eight waves per (kv head, split).  Its waves take pairs of pages in
// turn, each with its own running maximum and sum, and meet in LDS at the end; a second
// kernel joins the splits of a candidate in order.  Per pair of pages and wave:
//   QK   S = K Q^T, 16x16x32 matrix instructions: rows = the page's tokens, columns = 16 query
//        rows.  Lane (column l % 16, g = l / 16) gets the scores of tokens 4 g .. + 3 of either page.
//   PV   O^T = V^T P^T: the 32-deep axis is the pair's tokens in the order in which the lanes hold
//        their scores, so p needs no exchange.  p vs is split into two bf16 parts, hi + lo:
//        2^-17 of itself is lost (of one part 2^-8, as much as the output's own rounding loses).
// More than 16 query rows per kv head are further column tiles of the same page (NC), so
// the cache is read once for all new tokens.
//
// What bounds it: HBM for one token a candidate (16 flop a byte at 8 heads a kv head).  64
// candidates of 16k-32k keys, 8 x 128 heads, 3.32 GB: 512-528 us, 6.3-6.5 TB/s, what the read probe
// reaches; one candidate of 65537 keys, 138 MB: 30 us, of them 18 in the loop, the rest
// the two launches, the way to the first page (lengths, page ids, page: three memory latencies), workgroups
// without a split (the launch has 257 rows of them, the most of either plan below; 94 find one) and the join.  With 40 query rows (5 tokens of 8 heads; 16 candidates of 8k-16k keys, 209 MB, 48 us) the
// loop is bound by instructions: a wave issues one vector instruction in 8 clocks, and registers
// leave two waves a SIMD.
#include <algorithm>
#include <limits>

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

// the largest of three (the compiler's fmaxf first makes quiet every operand that it has lost track of,
// eight more instructions a column tile)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

__device__ __forceinline__ int keys_of(const int32_t* lens, int i, int max_pages) {
  const int len = lens[i];
  return len < 0 ? 0 : (len > max_pages * kPage ? max_pages * kPage : len);
}
__device__ __forceinline__ int pages_of(int keys) { return (keys + kPage - 1) / kPage; }

// The split plan, the same in every wave of both kernels: candidate i has max(1, ceil(pages_i /
// chunk)) splits.  The chunk is the least that gives all workgroups a place at once (then
// nothing waits for a second round that would be part empty: one candidate of 65537 keys 35 us
// against 42 for 3 rounds, with an earlier loop; 30 now); where that leaves chunks of more than kAttn8LongChunk pages, whose
// ends would be ragged, several rounds of shorter ones (64 candidates of 16k-32k: 8 workgroups per
// CU 515 us, 4 526, 2 575).
struct Split {
  int cand, index, count, first;  // candidate, split of it, its number of splits, its first flat id
  int len;                        // its keys
};

// sum over the wave, every lane gets it; inclusive scan (row shifts, then the rows' last lanes
// carried on): in registers, a shuffle through LDS costs 100 clocks a step
__device__ __forceinline__ int wave_sum_i(int v) {
  v += lane_xor<1>(v);
  v += lane_xor<2>(v);
  v += lane_xor<4>(v);
  v += lane_xor<8>(v);
  v += lane_xor<16>(v);
  return v + lane_xor<32>(v);
}
__device__ __forceinline__ int wave_scan_i(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast 15 into rows 1, 3
  return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast 31 into rows 2, 3
}

// flat >= 0: the split with that flat id (cand -1 behind the last); flat < 0: all of candidate ~flat.
// Each wave by itself, a candidate per lane: no barrier, and one read of the lengths where there
// are at most 64.
__device__ __forceinline__ Split find_split(const Attn8Args& a, int flat) {
  const int lane = threadIdx.x & 63;
  int keys = lane < a.n ? keys_of(a.seq_lens, lane, a.max_pages) : 0;
  int all = pages_of(keys);
  for (int i = lane + 64; i < a.n; i += 64) all += pages_of(keys_of(a.seq_lens, i, a.max_pages));
  all = __builtin_amdgcn_readfirstlane(wave_sum_i(all));  // (below 2^31: n max_pages is)
  int chunk = (all + a.one_round - 1) / a.one_round;
  if (chunk > kAttn8LongChunk) chunk = max(kAttn8LongChunk / 2, (all + a.rounds - 1) / a.rounds);
  chunk = max(chunk, a.min_chunk);
  int base = 0;
  Split r{-1, 0, 0, 0, 0};
  for (int i0 = 0; i0 < a.n; i0 += 64) {
    const int i = i0 + lane;
    if (i0) keys = i < a.n ? keys_of(a.seq_lens, i, a.max_pages) : 0;
    const int s = i < a.n ? max(1, (pages_of(keys) + chunk - 1) / chunk) : 0;
    const int in = wave_scan_i(s);
    const int first = base + in - s;
    const bool hit = flat >= 0 ? s > 0 && flat >= first && flat < first + s : i == ~flat;
    const uint64_t who = __builtin_amdgcn_ballot_w64(hit);
    if (who) {
      // scalars, so that what follows from them is scalar too
      const int l = __builtin_ctzll(who);
      r.cand = i0 + l;
      r.first = __builtin_amdgcn_readlane(first, l);
      r.count = __builtin_amdgcn_readlane(s, l);
      r.len = __builtin_amdgcn_readlane(keys, l);
      r.index = flat - r.first;
      break;
    }
    base += __builtin_amdgcn_readlane(in, 63);
  }
  return r;
}

// column cc (below 2^11) of a kv head's query rows: token cc / G, head cc % G of its group
__device__ __forceinline__ int token_of(const Attn8Args& a, int cc) {
  return (int)(((float)cc + 0.5f) * a.inv_group);
}
// running maxima start here: finite, so that what a column has not seen needs no case of its own, and at most
// any finite score
constexpr float kNoScore = -std::numeric_limits<float>::max();

// Waves per SIMD that the registers of NC column tiles leave room for.  At d = 128 two tiles fit three
// times with q in LDS and one tile's probabilities at a time (16 candidates of 8k-16k keys, 5 tokens of 32
// heads on 8: 94 -> 82 us; a second pair of pages in registers instead: 93); three tiles of d = 64
// as they are (32 candidates, 5 tokens of 32 heads on 4: 63 -> 58.5).
constexpr int waves8(int d, int nc) { return nc <= 2 || (nc == 3 && d == 64) ? 3 : 2; }

}  // namespace

template <int D, int NC, int PF, int W>
__global__ __launch_bounds__(64 * W, W == 4 ? waves8(D, NC) : 2) void attn8_split_kernel(Attn8Args a) {
  constexpr int NA = D / 64;   // 64-dim blocks of a tile
  constexpr int NB = D / 16;   // 16-dim blocks of the output
  constexpr int kStride = D + 4;
  __shared__ float w_m[W][16], w_l[W][16];
  __shared__ __align__(16) float w_acc[W][16][kStride];

  // workgroups in the order (split, kv head, NC column tiles): the heads of a page, adjacent in
  // the pool, are read together, each through the XCD that its workgroup number falls to
  const int flat = blockIdx.y;
  const int c = a.col_tiles == 1 ? blockIdx.x : blockIdx.x / a.col_tiles;
  const int cg = blockIdx.x - c * a.col_tiles;
  const Split sp = find_split(a, flat);
  const int i = sp.cand;
  if (i < 0) return;
  const int len = sp.len;
  const int npg = pages_of(len);
  // the candidate's pages in even shares, each an even number of pages
  const int share = ((npg + sp.count - 1) / sp.count + 1) & ~1;
  const int pbeg = sp.index * share;
  const int pend = min(npg, pbeg + share);

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int G = a.group, cols = a.tokens * G;

  const int32_t* ptr = a.page_table + (size_t)i * a.max_pages;
  const int pairs = (pend - pbeg + 1) / 2;                 // pairs of the split
  const int mine = pairs > wave ? (pairs - wave + W - 1) / W : 0;  // the wave's: wave, wave + W, ...
  // page ids of 64 of the wave's pairs, one pair per lane; -1: outside the pool
  int id0 = -1, id1 = -1;
  auto fetch_ids = [&](int k0) {
    const int pg = pbeg + 2 * (wave + W * (k0 + lane));
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
  fetch_ids(0);
  int m = a.q_lens ? a.q_lens[i] : a.tokens;
  m = m < 0 ? 0 : (m > a.tokens ? a.tokens : m);

  // The query rows' fragments, dims 64 x + 16 grp + 8 h .. + 7 of the lane's column: in registers,
  // or where those are short in LDS, once for the four waves.
  constexpr bool kQLds = NC >= 3 || (NC == 2 && D == 128);
  __shared__ __align__(16) u32x4 q_lds[kQLds ? NC * NA * 2 : 1][64];
  bf16x8v qf[kQLds ? 1 : NC][NA][2];
  int lim[NC];  // keys that the lane's column sees
#pragma unroll
  for (int t = 0; t < NC; ++t) {
    const int cc = (cg * NC + t) * 16 + col;
    const int tok = token_of(a, cc), head = cc - tok * G;
    const bool on = cc < cols && tok < m;
    lim[t] = on ? len - m + tok + 1 : 0;
    if (kQLds && (t & 3) != wave) continue;
    const bf16_t* qr = a.q + (((size_t)i * a.tokens + tok) * a.hq + (size_t)c * G + head) * D;
#pragma unroll
    for (int x = 0; x < NA; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 w{0u, 0u, 0u, 0u};
        if (on) w = *reinterpret_cast<const u32x4*>(qr + 64 * x + 16 * grp + 8 * h);
        if constexpr (kQLds) q_lds[(t * NA + x) * 2 + h][lane] = w;
        else qf[t][x][h] = __builtin_bit_cast(bf16x8v, w);
      }
  }
  if constexpr (kQLds) __syncthreads();
  auto q_frag = [&](int t, int x, int h, int at) {
    if constexpr (kQLds) return __builtin_bit_cast(bf16x8v, q_lds[(t * NA + x) * 2 + h][at]);
    else return qf[t][x][h];
  };
  // pages that every query row of the candidate sees in full need no mask (columns
  // without a row compute what is not stored)
  const int full = (len - m + 1) / kPage;
  float m_run[NC], l_run[NC];
  f32x4 acc[NC][NB];
#pragma unroll
  for (int t = 0; t < NC; ++t) {
    m_run[t] = kNoScore;
    l_run[t] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // PF pairs of pages in registers.  K of a later pair is read as soon as this pair's scores are
  // formed, the scales after its probabilities, V after its output, into the registers that just
  // became free: each load has PF iterations to arrive.
  constexpr uint32_t kTile = kv8_tile_bytes(D);
  const uint32_t koff = col * 64 + grp * 16, voff = lane * 16;
  struct Pair {
    u32x4 k[2][NA], v[2][NA], sk[2], sv[2];
    int id[2];
  };
  Pair set[PF];
  auto tile_of = [&](int id) {
    const uint8_t* base = a.kv_pool + (id < 0 ? 0 : ((size_t)id * a.hkv + c) * kTile);
    // no records, no read
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, id < 0 ? 0 : (int)kTile,
                                             0x00020000);
  };
  auto load_k = [&](Pair& r, int n) {  // the wave's n-th pair (past the last the ids are -1: nothing is read)
    if ((n & 63) == 0 && n) fetch_ids(n);
    r.id[0] = __builtin_amdgcn_readlane(id0, n & 63);
    r.id[1] = __builtin_amdgcn_readlane(id1, n & 63);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const __amdgpu_buffer_rsrc_t rs = tile_of(r.id[p]);
#pragma unroll
      for (int x = 0; x < NA; ++x)
        r.k[p][x] = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)koff, x * 1024, 2);
    }
  };
  auto load_s = [&](Pair& r) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const __amdgpu_buffer_rsrc_t rs = tile_of(r.id[p]);
      r.sk[p] = __builtin_amdgcn_raw_buffer_load_b128(rs, grp * 16, 32 * D, 2);
      r.sv[p] = __builtin_amdgcn_raw_buffer_load_b128(rs, grp * 16, 32 * D + 64, 2);
    }
  };
  auto load_v = [&](Pair& r) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const __amdgpu_buffer_rsrc_t rs = tile_of(r.id[p]);
#pragma unroll
      for (int x = 0; x < NA; ++x)
        r.v[p][x] = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)voff, 16 * D + x * 1024, 2);
    }
  };
  auto step = [&](Pair& r, int n) {
    const int pg = pbeg + 2 * (wave + W * n);  // the pair's first page
    const bool ok0 = r.id[0] >= 0, ok1 = r.id[1] >= 0;
    const bool masked = pg + 2 > full || !ok0 || !ok1;
    const int u0 = pg * kPage + 4 * grp;  // the lane's tokens u0 .. + 3 and u0 + 16 .. + 3
    int q_at = lane;  // opaque, or the reads of q would be moved out of the loop, into registers
    if constexpr (kQLds) asm volatile("" : "+v"(q_at));
    f32x4 s[NC][2];
#pragma unroll
    for (int t = 0; t < NC; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NA; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8v wa = codes_bf16(r.k[0][x][2 * h], r.k[0][x][2 * h + 1]);
        const bf16x8v wb = codes_bf16(r.k[1][x][2 * h], r.k[1][x][2 * h + 1]);
#pragma unroll
        for (int t = 0; t < NC; ++t) {
          const bf16x8v q = q_frag(t, x, h, q_at);
          s[t][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa, q, s[t][0], 0, 0, 0);
          s[t][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, q, s[t][1], 0, 0, 0);
        }
      }
    f32x4 ks[2], vs[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      ks[p] = __builtin_bit_cast(f32x4, r.sk[p]) * a.scale_log2;
      vs[p] = __builtin_bit_cast(f32x4, r.sv[p]);
    }
    if (masked) {
      // What lies behind the last key may hold anything, also NaN codes: no codes are kept of it.
      // A scale that is no number goes into the scores of those who see the token instead: as a
      // factor it would reach the others too (0 NaN).
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int left = len - u0 - kPage * p;
        const uint32_t keep = left >= 4 ? ~0u : (left <= 0 ? 0u : (1u << (8 * left)) - 1u);
#pragma unroll
        for (int x = 0; x < NA; ++x) r.v[p][x] &= keep;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float nan = vs[p][e] * 0.f;
          ks[p][e] += nan;
          vs[p][e] = nan == 0.f ? vs[p][e] : 0.f;
        }
      }
    }
    load_k(r, n + PF);
    // four column tiles go in two halves, two of d = 128 one by one, V's codes converted for each: the
    // probabilities of all take registers that are not there
    constexpr int H = NC == 4 ? 2 : (NC == 2 && D == 128 ? 1 : NC);
#pragma unroll
    for (int t0 = 0; t0 < NC; t0 += H) {
      bf16x8v ph[H], pl[H];
#pragma unroll
      for (int t = t0; t < t0 + H; ++t) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = s[t][e / 4][e & 3] * ks[e / 4][e & 3];
        if (masked) {
          const int v0 = ok0 ? lim[t] - u0 : 0, v1 = ok1 ? lim[t] - u0 - kPage : 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[e] = e < v0 ? z[e] : -INFINITY;
            z[4 + e] = e < v1 ? z[4 + e] : -INFINITY;
          }
        }
        float top = max3(max3(max3(z[0], z[1], z[2]), z[3], z[4]), max3(z[5], z[6], z[7]), z[7]);
        // (the column's largest is in one of its four lanes, and looked for only where one is too large)
        if (__builtin_amdgcn_ballot_w64(top > m_run[t] + kLazyLog2)) {
          top = xor32_max(xor16_max(top));
          const float mn = top > m_run[t] + kLazyLog2 ? top : m_run[t];
          const float alpha = __builtin_amdgcn_exp2f(m_run[t] - mn);  // 0 on the first page, 1 without a raise
          l_run[t] *= alpha;
#pragma unroll
          for (int b = 0; b < NB; ++b) acc[t][b] *= alpha;
          m_run[t] = mn;
        }
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          float p[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float pr = __builtin_amdgcn_exp2f(z[e + y] - m_run[t]);
            l_run[t] += pr;
            p[y] = pr * vs[e / 4][(e + y) & 3];
          }
          hi[e / 2] = pack_bf16x2(p[0], p[1]);
          asm("" : "+v"(hi[e / 2]));  // (else it is converted once more for what follows)
          // (p less its rounded value is exact)
          lo[e / 2] = pack_bf16x2(p[0] - bf16_lo(hi[e / 2]), p[1] - bf16_hi(hi[e / 2]));
        }
        ph[t - t0] = __builtin_bit_cast(bf16x8v, u32x4{hi[0], hi[1], hi[2], hi[3]});
        pl[t - t0] = __builtin_bit_cast(bf16x8v, u32x4{lo[0], lo[1], lo[2], lo[3]});
      }
      if (t0 + H == NC) load_s(r);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        uint32_t v0 = r.v[0][b / 4][b % 4], v1 = r.v[1][b / 4][b % 4];
        if constexpr (H < NC) asm("" : "+v"(v0), "+v"(v1));  // (not kept converted)
        const bf16x8v w = codes_bf16(v0, v1);
#pragma unroll
        for (int t = t0; t < t0 + H; ++t) {
          acc[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, pl[t - t0], acc[t][b], 0, 0, 0);
          acc[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, ph[t - t0], acc[t][b], 0, 0, 0);
        }
      }
    }
    load_v(r);
  };
  if (mine > 0) {
#pragma unroll
    for (int y = 0; y < PF; ++y) {
      load_k(set[y], y);
      load_s(set[y]);
      load_v(set[y]);
    }
    for (int n = 0;;) {
      step(set[0], n);
      if (++n >= mine) break;
      if constexpr (PF > 1) {
        step(set[PF - 1], n);
        if (++n >= mine) break;
      }
    }
  }

  // The waves of each column tile joined, in order: 16 threads a column, D / 16 dims each.
  // A candidate's only split is the result.
  constexpr int E = D / 16;
  const int j = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * E;
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
    const int cc = (cg * NC + t) * 16 + j;
    if (j < 16 && cc < cols) {
      float M = w_m[0][j];
#pragma unroll
      for (int w = 1; w < W; ++w) M = fmaxf(M, w_m[w][j]);
      float S = 0.f, O[E];
#pragma unroll
      for (int e = 0; e < E; ++e) O[e] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = __builtin_amdgcn_exp2f(w_m[w][j] - M);
        S += w_l[w][j] * f;
#pragma unroll
        for (int e = 0; e < E; ++e) O[e] += w_acc[w][j][e0 + e] * f;
      }
      if (sp.count == 1) {
        const int tok = token_of(a, cc), head = c * G + cc - tok * G;
        if (tok < m || a.clear_rest) {
          uint32_t o[E / 2];
          const float inv = S == 0.f ? 0.f : 1.f / S;
#pragma unroll
          for (int e = 0; e < E; e += 2)
            o[e / 2] = tok < m ? pack_bf16x2(O[e] * inv, O[e + 1] * inv) : 0u;
          uint32_t* dst = reinterpret_cast<uint32_t*>(
              a.out + (((size_t)i * a.tokens + tok) * a.hq + head) * D + e0);
#pragma unroll
          for (int e = 0; e < E / 2; ++e) dst[e] = o[e];
        }
      } else {
        const size_t slot = ((size_t)flat * a.hkv + c) * cols + cc;
        float* dst = a.part_acc + slot * D + e0;
#pragma unroll
        for (int e = 0; e < E; e += 4)
          *reinterpret_cast<f32x4*>(dst + e) = f32x4{O[e], O[e + 1], O[e + 2], O[e + 3]};
        if (e0 == 0) {
          a.part_ml[slot * 2] = M;
          a.part_ml[slot * 2 + 1] = S;
        }
      }
    }
  }
}

// Joins the splits of one query row, in a fixed order: the same call gives the same bits.  W waves a
// row (1: four rows a workgroup), each takes every W-th split, eight of them in flight: what it
// takes is a few memory latencies.
template <int D, int W>
__global__ __launch_bounds__(256) void attn8_join_kernel(Attn8Args a) {
  constexpr int E = D / 64;
  constexpr int U = 8;
  __shared__ float w_m[W], w_l[W], w_acc[W][D];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.group, cols = a.tokens * G;
  const int cc = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (cc >= cols) return;  // (behind the last row of the last workgroup, W = 1)
  const int c = blockIdx.y, i = blockIdx.z;
  const Split sp = find_split(a, ~i);
  if (sp.count <= 1) return;
  const int tok = token_of(a, cc), head = c * G + cc - tok * G;
  int m = a.q_lens ? a.q_lens[i] : a.tokens;
  m = m < 0 ? 0 : (m > a.tokens ? a.tokens : m);
  bf16_t* o = a.out + (((size_t)i * a.tokens + tok) * a.hq + head) * D;
  if (tok >= m) {
    if (a.clear_rest && (W == 1 || wave == 0))
#pragma unroll
      for (int e = 0; e < E; ++e) o[lane + 64 * e] = 0;
    return;
  }
  const size_t step = (size_t)a.hkv * cols;  // slots between a candidate's splits
  const size_t slot0 = ((size_t)sp.first * a.hkv + c) * cols + cc;
  float M = kNoScore, S = 0.f, O[E];
#pragma unroll
  for (int e = 0; e < E; ++e) O[e] = 0.f;
  for (int s0 = W == 1 ? 0 : wave; s0 < sp.count; s0 += 64 * W) {
    // a split per lane: its share of the sum; then the splits' rows, U of them in flight (past the
    // last one the last again, with the share 0)
    const int mine = min(64, (sp.count - s0 + W - 1) / W);
    float ml = kNoScore, ll = 0.f;
    if (lane < mine) {
      const float2 p = *reinterpret_cast<const float2*>(a.part_ml + (slot0 + (size_t)(s0 + W * lane) * step) * 2);
      ml = p.x;
      ll = p.y;
    }
    float ac[U][E];
    auto rows = [&](int y0) {
#pragma unroll
      for (int y = 0; y < U; ++y) {
        const float* r = a.part_acc + (slot0 + (size_t)(s0 + W * min(y0 + y, mine - 1)) * step) * D;
#pragma unroll
        for (int e = 0; e < E; ++e) ac[y][e] = r[lane + 64 * e];
      }
    };
    rows(0);
    const float top = fmaxf(M, wave_max(ml));
    const float f0 = __builtin_amdgcn_exp2f(M - top), f = lane < mine ? __builtin_amdgcn_exp2f(ml - top) : 0.f;
    S = S * f0 + wave_sum(ll * f);
#pragma unroll
    for (int e = 0; e < E; ++e) O[e] *= f0;
    for (int y0 = 0;;) {
#pragma unroll
      for (int y = 0; y < U; ++y) {
        const float fy = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), (y0 + y) & 63));
        const float g = y0 + y < mine ? fy : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) O[e] += ac[y][e] * g;
      }
      if ((y0 += U) >= mine) break;
      rows(y0);
    }
    M = top;
  }
  if constexpr (W > 1) {
    if (lane == 0) {
      w_m[wave] = M;
      w_l[wave] = S;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) w_acc[wave][lane + 64 * e] = O[e];
    __syncthreads();
    if (wave) return;
    M = w_m[0];
#pragma unroll
    for (int x = 1; x < W; ++x) M = fmaxf(M, w_m[x]);
    S = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) O[e] = 0.f;
#pragma unroll
    for (int x = 0; x < W; ++x) {
      const float f = __builtin_amdgcn_exp2f(w_m[x] - M);
      S += w_l[x] * f;
#pragma unroll
      for (int e = 0; e < E; ++e) O[e] += w_acc[x][lane + 64 * e] * f;
    }
  }
  const float inv = S == 0.f ? 0.f : 1.f / S;
#pragma unroll
  for (int e = 0; e < E; ++e) o[lane + 64 * e] = f32_to_bf16(O[e] * inv);
}

template <int D, int W>
static void launch_split8(const Attn8Args& a, int nc, hipStream_t st) {
  const dim3 grid((unsigned)(a.hkv * a.col_tiles), (unsigned)a.max_splits);
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(64 * W), 0, st, a); };
  if (nc == 1) go(attn8_split_kernel<D, 1, D == 64 ? 2 : 1, W>);
  else if (nc == 2) go(attn8_split_kernel<D, 2, 1, W>);
  else if (nc == 3) go(attn8_split_kernel<D, 3, 1, W>);
  else go(attn8_split_kernel<D, 4, 1, W>);
}

template <int D>
static hipError_t launch_attn8_d(const Attn8Args& a, const Attn8Plan& p, hipStream_t st) {
  if (p.waves == 8) launch_split8<D, 8>(a, p.nc, st);
  else launch_split8<D, 4>(a, p.nc, st);
  hipError_t e = hipGetLastError();
  // pages that one split holds: every candidate has one, nothing to join
  if (e != hipSuccess || a.max_pages <= a.min_chunk) return e;
  const unsigned cols = (unsigned)(a.tokens * a.group);
  auto join = [&](auto kern, unsigned groups) {
    hipLaunchKernelGGL(kern, dim3(groups, (unsigned)a.hkv, (unsigned)a.n), dim3(256), 0, st, a);
    return hipGetLastError();
  };
  // few candidates have many splits each, and few rows
  if (a.one_round > 12 * a.n) return join(attn8_join_kernel<D, 4>, cols);
  return join(attn8_join_kernel<D, 1>, (cols + 3) / 4);
}

Attn8Plan plan_attn8(int n, int hq, int hkv, int d, int tokens, int max_pages) {
  Attn8Plan p;
  const int cols = tokens * (hq / hkv), tiles = (cols + 15) / 16;
  p.col_tiles = (tiles + kAttn8MaxTiles - 1) / kAttn8MaxTiles;
  p.nc = (tiles + p.col_tiles - 1) / p.col_tiles;
  const int per = hkv * p.col_tiles;                          // workgroups of a split
  const int places = std::max(1, 256 * waves8(d, p.nc) / per);  // splits that are resident at once
  // all pages / chunk + n splits at most
  p.one_round = std::max(std::max(places - n, places / 2), 1);
  p.rounds = std::max(kAttn8Rounds * 256 / per, 1);
  // A join costs 5 us of the GPU and a launch: short candidates are one split, longer ones too where
  // they fill the CUs (splits / one, us among others: 4 candidates of 512-1024 keys, 8 heads, 13.8 /
  // 12.0, of 768-1536, in a graph, 9.5 / 11.5; 64 of 1280-2560 53 / 46, 64 of 256-4096 with 4 heads 33 / 39).
  const bool one = max_pages <= ((long long)n * per >= 256 ? kAttn8OneSplitMany : kAttn8OneSplit);
  p.min_chunk = one ? max_pages : kAttn8MinChunk;
  // A workgroup that has its CU to itself takes eight waves (four / eight, us in a graph, 32 heads on 8:
  // 4 candidates of 512-1024 keys 11.1 / 9.5, 16 12.3 / 10.5, of 4 tokens each 12.1 / 10.5;
  // sixteen waves 10.7, 12.0).
  p.waves = one && (long long)n * per <= 256 ? 8 : 4;
  const long long most = (long long)n * ((max_pages + p.min_chunk - 1) / p.min_chunk);
  const long long s = (long long)std::max(p.one_round, p.rounds) + n;
  p.max_splits = s < most ? s : most;
  return p;
}

hipError_t launch_attn8(const Attn8Args& a, const Attn8Plan& p, hipStream_t st) {
  return a.d == 128 ? launch_attn8_d<128>(a, p, st) : launch_attn8_d<64>(a, p, st);
}

}  // namespace sevo
