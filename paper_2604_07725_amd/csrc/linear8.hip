// Y = X W^T on 8-bit operands with a scale for each block of 128 (e4m3 codes;
// X: a scale per row and 128 columns, W: one per 128 rows and 128 columns):
//   Y[m][n] = sum over 128-column blocks b of
//             sx[b][m] sw[n / 128][b] (sum over k in b of X[m][k] W[n][k]).
// The inner sum of a block runs on the matrix cores, its scaled addition to the
// fp32 accumulator on the vector ALU (one FMA per element and block, the two
// scales multiplied once per row fragment).
//
// Two matrix instructions.  The 8-bit ones (16x16x128) have twice the rate of
// bf16 but add in fewer bits.  Measured: the products of eight neighbouring
// columns are cut toward zero at 2^-13 of the largest one's power of two (a subnormal
// operand counts with the exponent -6), then added as in fp32; this gives the bf16
// results bit for bit.  For normally distributed codes that is 1.4e-5 of a block's sum (norm),
// -1e-5 on average where all products have one sign, and up to 2e-4 of the sum of
// magnitudes where they differ by orders: below the 2^-8 of a result that is rounded
// to bf16, which is what these instructions are used for, unless blocks cancel.  A
// result kept in fp32 takes the bf16 instruction on the codes converted to bf16, which
// is exact (e4m3 has four significant bits): 1e-7.
//
// A operand = 16 weight rows, B operand = 16 activation rows, 128 columns: lane
// l holds row l % 16 and its 16-byte runs l / 16 and l / 16 + 4, so that a packed
// weight fragment is two contiguous 1 KB loads.  The order of k inside a block is
// the same on both sides and does not matter otherwise.  D: lane l holds activation
// row l % 16 and the four weight rows (output columns) 4 (l / 16) ..: one activation
// scale per lane, and stores of four consecutive columns.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace sevo {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// 16-row x 128-column operand fragment of one lane: its two 16-byte runs
union Frag8 {
  i32x8 v;
  u32x4 u[2];
};

__device__ __forceinline__ bf16x8v codes_to_bf16(uint32_t w0, uint32_t w1) {
  const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, false);
  const bf16x2v b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, true);
  const bf16x2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, false);
  const bf16x2v d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, true);
  return bf16x8v{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// the operand a product takes: the codes, or their bf16 values (32 columns a piece)
template <bool EXACT>
struct Operand;
template <>
struct Operand<false> {
  i32x8 v;
  Operand() = default;
  __device__ __forceinline__ explicit Operand(const Frag8& f) : v(f.v) {}
};
template <>
struct Operand<true> {
  bf16x8v v[4];
  Operand() = default;
  __device__ __forceinline__ explicit Operand(const Frag8& f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = codes_to_bf16(f.u[i >> 1][2 * (i & 1)], f.u[i >> 1][2 * (i & 1) + 1]);
  }
};

// the unscaled 16 x 16 product of one 128-column block
__device__ __forceinline__ f32x4 block_product(const Operand<false>& a, const Operand<false>& b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0,
                                                          0, 0, 0, 0);
}
__device__ __forceinline__ f32x4 block_product(const Operand<true>& a, const Operand<true>& b) {
  f32x4 d = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], d, 0, 0, 0);
  return d;
}

__device__ __forceinline__ void add_scaled(f32x4& acc, const f32x4& d, float s) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(d[e], s, acc[e]);
}

__device__ __forceinline__ void store4(void* out, size_t off, const f32x4& v, int bf16) {
  if (bf16)
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(out) + off) =
        uint2{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)};
  else
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + off) = v;
}

// Direct global -> LDS load of N bytes per lane at voff + soff (wave-uniform; the sum is
// checked against the records, so both have to fit in them); lane i's bytes land at lds + N i.
// ONCE: data that nothing else reads, past the caches.
template <int N, bool ONCE = false>
__device__ __forceinline__ void dma_s(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff,
                                      uint8_t* lds) {
  static_assert(N == 16 || N == 4, "bytes per lane");
  const auto dst = (__attribute__((address_space(3))) void*)lds;
  if constexpr (N == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, (int)voff, (int)soff, 0, ONCE ? 2 : 0);
  else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 4, (int)voff, (int)soff, 0, 0);
}

}  // namespace

// Few rows: a weight stream.  One workgroup per (RB 16-row weight blocks, K
// split, M tile of 16 MB rows); its four waves take the 128-column steps of the
// split in turn and sum their tiles through LDS.  The weights go to registers in
// fragments of contiguous 1 KB; the activations and their scales go through the
// wave's own LDS ring by direct loads of whole 128-byte rows (gathered per lane
// in fragment order they came at 16 bytes per clock and CU: 64 x 4096 x 4096 in M
// tiles of 64 13.6 -> 10.5 us, 32 x 4096 x 4096 8.7 -> 7.5).  Two steps are in flight under
// the products of a third (three or four: no faster, 16 x 6144 x 4096 7.6 / 7.6 / 8.2).
// Measured in graphs, weights cold: 8 x 51200 x 5120 52.7 us (5.0 TB/s), 16 x 6144 x 4096 7.6
// (3.3), of which 3.4 a launch; from 32 rows on the CU's path from L2 bounds it, on which
// the activations come too: 64 x 4096 x 12288 in four splits 14.0 (3.6), their sum 3.9.  M tiles of 64 rows read the
// weights half as often as those of 32: 64 x 10240 x 5120 to fp32 24.1 -> 20.4 (LDS tiles
// before), 128 x 6144 x 4096 to fp32 19.9 -> 15.5, 203 x 4096 x 4096 16.2 -> 14.3.
template <int MB, int RB, bool EXACT>
__global__ __launch_bounds__(256, 1) void linear8_kernel(Linear8Args a, int kb_chunk,
                                                         float* __restrict__ part) {
  constexpr int kStepBytes = MB * 2048 + 256;            // a step's rows and their scales
  constexpr int ND = 3;  // step buffers
  constexpr int kRing = 4 * ND * kStepBytes, kRed = 4 * RB * MB * 1024;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kRing > kRed ? kRing : kRed];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, q = lane >> 4;
  const int m0 = blockIdx.z * 16 * MB;
  const int KB = a.k >> 7, nrb = a.n_out >> 4;
  const int rb0 = blockIdx.x * RB;

  // row blocks past the matrix read block 0 and are never stored, and so do rows past m
  const uint8_t* wp[RB];
#pragma unroll
  for (int i = 0; i < RB; ++i) {
    const int rb = rb0 + i < nrb ? rb0 + i : 0;
    wp[i] = a.w + ((size_t)(rb >> 2) * KB * 4 + (rb & 3)) * 2048;
  }
  // place p of row r holds run p ^ (r / 2 % 8): see tile8_kernel
  const uint8_t* xb = a.x + (size_t)m0 * a.ldx;
  uint32_t x_voff[2 * MB];
#pragma unroll
  for (int f = 0; f < 2 * MB; ++f)
    x_voff[f] = (uint32_t)min(8 * f + (lane >> 3), a.m - 1 - m0) * (uint32_t)a.ldx +
                16 * ((lane & 7) ^ (4 * (f & 1) + (lane >> 4)));
  const uint32_t s_voff = 4u * min(lane, a.m - 1 - m0);
  const int x_off0 = r * 128 + (q ^ (r >> 1)) * 16, x_off1 = x_off0 ^ 64;
  // the RB (at most 8) row blocks lie in at most two 128-row scale blocks
  const float* ws0 = a.ws + (size_t)(rb0 >> 3) * KB;
  const float* ws1 = a.ws + (size_t)((min(rb0 + RB, nrb) - 1) >> 3) * KB;

  const int st0 = blockIdx.y * kb_chunk;
  const int nsteps = min(KB - st0, kb_chunk);
  const int cnt = nsteps > wave ? (nsteps - wave + 3) >> 2 : 0;  // steps of this wave

  struct Step {
    Frag8 w[RB];
    float sw0, sw1;
  };
  constexpr int kLoads = 2 * MB + 1 + 2 * RB;  // vector loads of a step
  uint8_t* ring = smem + wave * ND * kStepBytes;
  // j-th step of this wave into buffer `slot`; past the end the descriptors have no
  // records, and nothing is read
  auto load = [&](Step& f, int slot, int j) {
    const int st = st0 + wave + 4 * min(j, cnt - 1);
    const int records = j < cnt ? 0x7FFFFFFF : 0;
    auto rsrc = [&](const void* p) {
      return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, records, 0x00020000);
    };
    uint8_t* so = ring + slot * kStepBytes;
#pragma unroll
    for (int b = 0; b < 2 * MB; ++b) dma_s<16>(rsrc(xb), x_voff[b], st * 128u, so + 1024 * b);
    dma_s<4>(rsrc(a.xs + m0), s_voff, (uint32_t)st * (uint32_t)a.lds * 4u, so + 2048 * MB);
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)  // (read once: past the caches)
        f.w[i].u[h] = __builtin_amdgcn_raw_buffer_load_b128(rsrc(wp[i]), lane * 16 + 1024 * h, st * 8192, 2);
    f.sw0 = ws0[st];
    f.sw1 = ws1[st];
    __builtin_amdgcn_sched_barrier(0);
  };
  f32x4 acc[RB][MB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto mma = [&](const Step& f, int slot) {
    wait_vmcnt<(ND - 1) * kLoads>();  // the step's loads; the next steps' may still run
    __builtin_amdgcn_sched_barrier(0);
    const uint8_t* so = ring + slot * kStepBytes;
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      Frag8 xf;
      xf.u[0] = *reinterpret_cast<const u32x4*>(so + 2048 * b + x_off0);
      xf.u[1] = *reinterpret_cast<const u32x4*>(so + 2048 * b + x_off1);
      const float sx = *reinterpret_cast<const float*>(so + 2048 * MB + 64 * b + 4 * r);
      const Operand<EXACT> xo(xf);
      const float s0 = sx * f.sw0, s1 = sx * f.sw1;
#pragma unroll
      for (int i = 0; i < RB; ++i)
        add_scaled(acc[i][b], block_product(Operand<EXACT>(f.w[i]), xo),
                   (rb0 + i) >> 3 == rb0 >> 3 ? s0 : s1);
    }
    wait_lgkm0();  // the buffer is read before the next load into it is issued
    __builtin_amdgcn_sched_barrier(0);
  };
  if (cnt > 0) {
    Step f[ND];
#pragma unroll
    for (int b = 0; b < ND - 1; ++b) load(f[b], b, b);
    for (int j = 0; j < cnt; j += ND)
#pragma unroll
      for (int b = 0; b < ND; ++b) {
        constexpr int kBack = ND - 1;
        load(f[(b + kBack) % ND], (b + kBack) % ND, j + b + kBack);
        if (j + b < cnt) mma(f[b], b);
      }
  }
  wait_vmcnt<0>();  // the direct loads past the end have left the ring
  __syncthreads();
  f32x4(*red)[RB][MB][64] = reinterpret_cast<f32x4(*)[RB][MB][64]>(smem);
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int b = 0; b < MB; ++b) red[wave][i][b][lane] = acc[i][b];
  __syncthreads();
  for (int idx = threadIdx.x; idx < RB * MB * 64; idx += 256) {
    const int l = idx & 63, i = (idx >> 6) / MB, b = (idx >> 6) % MB;
    const f32x4 v = red[0][i][b][l] + red[1][i][b][l] + red[2][i][b][l] + red[3][i][b][l];
    const int m = m0 + 16 * b + (l & 15);
    const int n = (rb0 + i) * 16 + 4 * (l >> 4);
    if (m < a.m && rb0 + i < nrb) {
      if (part) *reinterpret_cast<f32x4*>(part + ((size_t)blockIdx.y * a.m + m) * a.n_out + n) = v;
      else store4(a.out, (size_t)m * a.ldo + n, v, a.out_bf16);
    }
  }
}

// The splits' partials [S][m][n_out], summed in split order, to the output type.
__global__ __launch_bounds__(256) void linear8_sum_kernel(const float* __restrict__ part, int S,
                                                          Linear8Args a) {
  const size_t mn = (size_t)a.m * a.n_out, total4 = mn / 4;
  for (size_t g = (size_t)blockIdx.x * blockDim.x + threadIdx.x; g < total4;
       g += (size_t)gridDim.x * blockDim.x) {
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < S; s0 += 4) {
      f32x4 p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (s0 + j < S) p[j] = *reinterpret_cast<const f32x4*>(part + (s0 + j) * mn + g * 4);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (s0 + j < S) v += p[j];
    }
    const size_t row = g * 4 / a.n_out;
    store4(a.out, row * a.ldo + (g * 4 - row * a.n_out), v, a.out_bf16);
  }
}

// Zeros the output rows of the entries without an expert, which stand behind the lists:
// every parts-th one, from the part-th on, by a whole workgroup.  listed: the entries
// with one, offsets[n_experts].
__device__ __forceinline__ void clear_unlisted(const Moe8Args& a, int listed, int part, int parts) {
  const int nk = a.n * a.top_k;
  for (int i = listed + part; i < nk; i += parts) {
    const int asg = a.assign[i], tok = asg / a.top_k;
    const size_t row = a.down ? (size_t)(asg - tok * a.top_k) * a.n + tok : (size_t)asg;
    for (int c = 8 * threadIdx.x; c < a.n_out; c += 8 * blockDim.x)
      *reinterpret_cast<u32x4*>(a.out + row * a.n_out + c) = u32x4{0, 0, 0, 0};
  }
}

// The product grouped by expert for few entries an expert: a stream of the chosen
// experts' weights.  A wave takes two 16-row weight blocks of one expert over the
// whole k, a workgroup 128 rows (one row of weight scales); the expert's entries come
// 16 at a time, gathered through its list, and each 16 read its weights again.
// 30B-A3B gate/up of 64 tokens, 8 of 128 experts each: 63 us, 6.3 TB/s.  Where tokens
// agree few experts have long lists: the same 8 for all 64 (four passes over 25 MB)
// 38 us, 16 between them 30, one expert in every token's 8 77.
__global__ __launch_bounds__(256) void moe8_kernel(Moe8Args a) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, q = lane >> 4;
  const int e = blockIdx.y;
  const int off = a.offsets[e], ne = a.offsets[e + 1] - off, listed = a.offsets[a.n_experts];
  if (a.clear) clear_unlisted(a, listed, blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y);
  const int KB = a.k >> 7, nrb = a.n_out >> 4;
  const int rb0 = blockIdx.x * 8 + 2 * wave;
  if (ne <= 0 || rb0 >= nrb) return;  // wave-uniform, no barrier follows
  const uint8_t* wp = a.w + (size_t)e * a.n_out * a.k +
                      ((size_t)(rb0 >> 2) * KB * 4 + (rb0 & 3)) * 2048 + lane * 16;
  const float* wsp = a.ws + ((size_t)e * ((a.n_out + 127) >> 7) + (rb0 >> 3)) * KB;
  struct Step {
    Frag8 w[2], x;
    float sx, sw;
  };
  for (int m0 = 0; m0 < ne; m0 += 16) {
    const int asg = a.assign[off + min(m0 + r, ne - 1)];
    const int tok = asg / a.top_k;
    const int row = a.down ? asg : tok;
    const uint8_t* xp = a.x + (size_t)row * a.ldx + 16 * q;
    const float* xsp = a.xs + row;
    f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
    auto load = [&](Step& f, int j) {
      const int st = min(j, KB - 1);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          f.w[i].u[h] = __builtin_nontemporal_load(
              reinterpret_cast<const u32x4*>(wp + (size_t)st * 8192 + 2048 * i + 1024 * h));
#pragma unroll
      for (int h = 0; h < 2; ++h)
        f.x.u[h] = *reinterpret_cast<const u32x4*>(xp + (size_t)st * 128 + 64 * h);
      f.sx = xsp[(size_t)st * a.lds];
      f.sw = wsp[st];
    };
    auto mma = [&](const Step& f) {
      const Operand<false> xo(f.x);
      const float s = f.sx * f.sw;
#pragma unroll
      for (int i = 0; i < 2; ++i) add_scaled(acc[i], block_product(Operand<false>(f.w[i]), xo), s);
    };
    Step f0, f1, f2;
    load(f0, 0);
    load(f1, 1);
    for (int j = 0; j < KB; j += 3) {
      load(f2, j + 2);
      __builtin_amdgcn_sched_barrier(0);
      mma(f0);
      __builtin_amdgcn_sched_barrier(0);
      load(f0, j + 3);
      __builtin_amdgcn_sched_barrier(0);
      if (j + 1 < KB) mma(f1);
      __builtin_amdgcn_sched_barrier(0);
      load(f1, j + 4);
      __builtin_amdgcn_sched_barrier(0);
      if (j + 2 < KB) mma(f2);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (m0 + r < ne) {
      const float wt = a.down ? a.weights[asg] : 1.f;
      const size_t out = a.down ? (size_t)(asg - tok * a.top_k) * a.n + tok : (size_t)asg;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        store4(a.out, out * a.n_out + (rb0 + h) * 16 + 4 * q, acc[h] * wt, 1);
    }
  }
}

// More rows: LDS tiles of BM x BN, NW waves in a grid of NW / (BN / 64) x BN / 64,
// each 16 XT rows x 64 columns.  A stage is one 128-column block: the X and W
// codes go straight from global memory to LDS (16 bytes a lane), as do the
// block's scales; NS stage buffers keep NS - 1 stages in flight.
//   * W pieces are the 1 KB halves of the packed fragments;
//   * an X piece is eight whole 128-byte rows, eight consecutive lanes each (a
//     lane per row in turn: 16 bytes per clock and CU instead of 57).  Place p of
//     row r holds run p ^ (r / 2 % 8), so that each quarter of a fragment read covers
//     all 64 banks.
// A workgroup takes tiles blockIdx.x, + gridDim.x, ...: the next tile's first
// stages load while this one's results are stored.
// Grouped (GR): the m-tiles are tiles of the experts' lists and a tile's rows are
// gathered per lane.
// Bounds: large products the matrix cores, at the clock that the power allows (8192 x
// 24576 x 4096 665 to 707 us by the card, 2.3 to 2.5 PFLOP/s; the library's product with one
// scale 658); some
// hundred rows the reads from LDS, 0.38 us a stage of 128 x 128 x 128 alone on a CU, and
// the way from L2, 0.5 to 0.6 with all CUs busy (512 x 8192 x 5120 29 us).
template <int BM, int BN, int NW, int NS, bool EXACT, bool GR>
__global__ __launch_bounds__(64 * NW) void tile8_kernel(Linear8Args a, int kb_chunk,
                                                    float* __restrict__ part, int tiles_m, Moe8Args g) {
  constexpr int WN = BN / 64, WM = NW / WN, XT = BM / WM / 16;
  static_assert(WN * WM == NW && XT * WM * 16 == BM && XT % 2 == 0, "wave grid");
  constexpr int XD = BM / 8 / NW, D = XD + BN / 8 / NW;  // X pieces and pieces of a wave and stage
  static_assert(XD * 8 * NW == BM && D * 8 * NW == BM + BN, "whole pieces");
  // Two meetings of the waves a stage where its activation tiles can be halved: see
  // the pipeline below.  U0 and U1 are the loads that each makes room for.
  constexpr bool TWO = NS == 2 && XT >= 4;
  constexpr int XH = TWO ? XD / 2 : XD;
  constexpr int U0 = TWO ? D - XD + XH : D + 1, U1 = D + 1 - U0;
  constexpr int kScales = (BM + BN) * 128;           // byte offset of a stage's scales
  constexpr int XS = (BM + 63) / 64;                 // waves that bring row scales, 64 each
  static_assert(XS < NW, "a wave for the weight scales");
  constexpr int STAGE = kScales + NW * 256;
  constexpr int kOutRow = 64 * 2 + 16;               // bytes of a staged bf16 output row of a wave
  constexpr int kTable = GR ? BM * 8 : 0;            // a tile's output rows and routing weights
  static_assert(NS * STAGE + kTable <= 160 * 1024 && NW * 16 * kOutRow <= STAGE, "LDS");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[NS * STAGE + kTable];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int r = lane & 15, q = lane >> 4;
  const int KB = a.k >> 7;
  const int tiles_n = (a.n_out + BN - 1) / BN;
  const int st0 = GR ? 0 : blockIdx.y * kb_chunk;
  const int nst = GR ? KB : min(KB - st0, kb_chunk);
  // grouped: each lane keeps the first tile, first entry and entries of experts lane + 64 j
  int e_tile[GR ? 4 : 1], e_first[GR ? 4 : 1], e_rows[GR ? 4 : 1];
  if constexpr (GR) {
    const int listed = g.offsets[g.n_experts];
    tiles_m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = lane + 64 * j;
      const bool in = e < g.n_experts;
      e_first[j] = in ? g.offsets[e] : 0;
      e_rows[j] = in ? g.offsets[e + 1] - e_first[j] : 0;
      const int tiles = (e_rows[j] + BM - 1) / BM;
      int incl = tiles;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(incl, o, kWave);
        if (lane >= o) incl += y;
      }
      e_tile[j] = in ? tiles_m + incl - tiles : 0x7FFFFFFF;
      tiles_m += __builtin_amdgcn_readlane(incl, 63);
    }
    if (g.clear) clear_unlisted(g, listed, blockIdx.x, gridDim.x);
  }
  const int total = tiles_m * tiles_n;

  // ---- the place of tile t: a contiguous range of tiles per XCD, in groups of 1024
  // rows.  All of it uniform over the workgroup.
  struct Place {
    int m0, n0, rows, ent0, expert;
  };
  auto find = [&](int t) {
    const int per = total >> 3;
    if (t < per * 8) t = (t & 7) * per + (t >> 3);
    constexpr int GM = 1024 / BM;
    const int first_m = t / (GM * tiles_n) * GM;
    const int gsize = min(GM, tiles_m - first_m);
    const int in_group = t - first_m * tiles_n;
    const int tm = first_m + in_group % gsize;
    Place p{tm * BM, in_group / gsize * BN, a.m, 0, 0};
    if constexpr (GR) {
      // the last expert whose first tile is at or before tm
      int n = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) n += __popcll(__ballot(e_tile[j] <= tm));
      p.expert = n - 1;
      auto of = [&](const int (&v)[4]) {
        const int j = p.expert >> 6;
        const int x = j == 0 ? v[0] : j == 1 ? v[1] : j == 2 ? v[2] : v[3];
        return __builtin_amdgcn_readlane(x, p.expert & 63);
      };
      p.m0 = (tm - of(e_tile)) * BM;
      p.ent0 = of(e_first);
      p.rows = of(e_rows);
    }
    return p;
  };
  // Piece (8 rows) of this wave's load i of X; the first XH are of rows that the waves
  // read before the middle of a stage.
  auto piece = [&](int i) {
    if constexpr (!TWO) return wave + NW * i;
    const int h = wave + NW * (i % XH);
    return h / XT * 2 * XT + h % XT + (i < XH ? 0 : XT);
  };
  // grouped: the entries of the rows that this lane loads (asg: of row threadIdx.x)
  int idx[XD], asg = 0;
  auto fetch = [&](const Place& p) {
    if constexpr (GR) {
#pragma unroll
      for (int i = 0; i < XD; ++i)
        idx[i] = g.assign[p.ent0 + min(p.m0 + 8 * piece(i) + (lane >> 3), p.rows - 1)];
      if (wave < XS) asg = g.assign[p.ent0 + min(p.m0 + 64 * wave + lane, p.rows - 1)];
    }
  };

  // ---- this wave's direct loads of a stage (D pieces and 64 scales): three
  // descriptors, offsets of the lane and of the piece and stage (scalar).  Every
  // offset of a row is in range (256 ldx and 256 k are below 2^31); past
  // the last stage the descriptors have no records, so that the loop issues without
  // a branch and nothing is read.
  const uint8_t* xb;   // what the X, W and scale offsets count from
  const uint8_t* wb;
  const float* sb;
  uint32_t x_voff[XD], w_soff[D - XD], s_voff, s_step;
  auto set_loads = [&](const Place& p) {
    const int base = GR ? 0 : p.m0;
    xb = a.x + (size_t)base * a.ldx;
    wb = a.w + (size_t)p.expert * a.n_out * a.k + (size_t)(p.n0 >> 6) * KB * 8192;
    auto x_row = [&](int entry, int i) {  // row i of the tile's matrix (scales past the end: the last)
      if constexpr (GR) return g.down ? entry : entry / g.top_k;
      else return min(p.m0 + i, p.rows - 1);
    };
#pragma unroll
    for (int i = 0; i < XD; ++i) {
      const int f = piece(i);
      const int run = (lane & 7) ^ (4 * (f & 1) + (lane >> 4));
      const int row = 8 * f + (lane >> 3);
      // Rows past the end: every dword of the lane is past the records, nothing is read and
      // zeros arrive (8192 tokens of 30B-A3B experts 262 + 189 us with the last row again in
      // their place, 255 + 186 so).
      x_voff[i] = p.m0 + row < p.rows ? (uint32_t)((size_t)(x_row(idx[i], row) - base) * a.ldx) + 16 * run
                                      : 0x80000000u;
    }
#pragma unroll
    for (int i = 0; i < D - XD; ++i) {
      const int c = wave + NW * i;  // 1 KB half c % 2 of fragment c / 2
      w_soff[i] = (uint32_t)(min(c >> 3, ((a.n_out - p.n0) >> 6) - 1) * KB * 8192 + (c & 7) * 1024);
    }
    if (wave < XS) {  // 64 of the rows' scales
      sb = a.xs + (size_t)st0 * a.lds;
      s_voff = 4u * x_row(asg, 64 * wave + lane);
      s_step = (uint32_t)a.lds * 4;
    } else {          // the weight blocks' scales (lane % 2: the tile's 128-column blocks)
      const int nblocks = (a.n_out + 127) >> 7;
      const int nb = min((p.n0 >> 7) + (lane & 1), nblocks - 1);
      sb = a.ws + (size_t)p.expert * nblocks * KB + st0;
      s_voff = 4u * nb * KB;
      s_step = 4;
    }
  };
  // loads [i0, i1) of stage st: the weights, the first XH of X, the scales, the rest of X
  auto issue = [&](int st, int i0, int i1) {
    uint8_t* so = smem + (st % NS) * STAGE;
    const int records = st < nst ? 0x7FFFFFFF : 0;
    auto rsrc = [&](const void* p) {
      return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, records, 0x00020000);
    };
    constexpr int DW = D - XD;
#pragma unroll
    for (int i = 0; i <= D; ++i) {
      if (i < i0 || i >= i1) continue;
      if (i < DW) {
        // (32-row tiles are for 32 entries an expert or fewer on average.  Where these are
        // spread evenly an expert has one tile and its weights are read once: 12 entries
        // an expert 81.5 + 51 -> 77.5 + 47 us.  An expert with a longer list has more tiles,
        // which read its weights past the caches too: with tiles that share them it costs 5%.)
        dma_s<16, GR && BM == 32>(rsrc(wb), lane * 16, (st0 + st) * 8192 + w_soff[i],
                                  so + BM * 128 + (wave + NW * i) * 1024);
      } else if (i == DW + XH) {
        dma_s<4>(rsrc(sb), s_voff, st * s_step, so + kScales + 256 * wave);
      } else {
        const int x = i - DW - (i > DW + XH);
        dma_s<16>(rsrc(xb), x_voff[x], (st0 + st) * 128, so + piece(x) * 1024);
      }
    }
  };

  // LDS byte offsets of this lane's runs, in a stage
  const int x_off0 = wm * XT * 2048 + r * 128 + (q ^ (r >> 1)) * 16;
  const int x_off1 = x_off0 ^ 64;
  const int w_off = BM * 128 + wn * 8192 + lane * 16;
  const int sx_off = kScales + (wm * XT * 16 + r) * 4;
  const int sw_off = kScales + 256 * (NW - 1) + (wn >> 1) * 4;
  Frag8 wf[4], xf[2];
  Operand<EXACT> wo[4], xo;
  auto read_w = [&](const uint8_t* so, int j) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      wf[j].u[h] = *reinterpret_cast<const u32x4*>(so + w_off + 2048 * j + 1024 * h);
  };
  auto read_x = [&](const uint8_t* so, int i) {
    xf[i & 1].u[0] = *reinterpret_cast<const u32x4*>(so + x_off0 + 2048 * i);
    xf[i & 1].u[1] = *reinterpret_cast<const u32x4*>(so + x_off1 + 2048 * i);
  };
  auto read_sx = [&](const uint8_t* so, int i) {
    return *reinterpret_cast<const float*>(so + sx_off + 64 * i);
  };
  auto read_sw = [&](const uint8_t* so) { return *reinterpret_cast<const float*>(so + sw_off); };

  // The loads are spread over steps (a product each) from the meeting on, one a step
  // where the steps suffice: issued together they fill the address queue, and the
  // waves wait for it instead of running products.
  constexpr int kSteps = TWO ? 2 * XT : 4 * XT;          // from a meeting to the next one
  constexpr int SP0 = U0 < kSteps ? U0 : kSteps;
  constexpr int kAfter = TWO ? D + 1 : 4 * (D + 1) / SP0;  // those issued when a stage begins
  static_assert(!TWO || U1 <= 4, "U1 within the four products after the meeting");
  constexpr int kFlight = (NS - (TWO ? 1 : 2)) * (D + 1);  // loads younger than those waited for

  int t = blockIdx.x;
  if (t >= total) return;  // uniform, before any barrier
  Place at = find(t), next = at;
  fetch(at);
  set_loads(at);
  for (int st = 0; st < NS - 1; ++st) issue(st, 0, D + 1);
  int stored = 0;  // 16-row blocks whose two stores each were issued behind those loads
  for (;;) {
    f32x4 acc[XT][4];
#pragma unroll
    for (int i = 0; i < XT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Pipeline.  The weight fragments and the first activation tile of a stage are
    // in registers when it begins.  Once its last activation tile is too, the
    // waves meet: what stage kt + 1 begins with has landed, and the buffer of stage kt
    // is free for the direct loads of stage kt + NS.  That tile's products run after the
    // meeting, each weight fragment replaced by the next stage's as soon as it is
    // done, so that neither the barrier nor the LDS latency leaves the matrix
    // cores without work.  A product is added to its accumulator two products
    // later; the last two of a stage in the next one.
    // TWO: the waves meet in the middle of the stage as well.  Its weights and the
    // first half of its activations are in registers by then: their places are free for
    // stage kt + NS half a stage earlier, and the second half is waited for here, half a
    // stage later.  So a load has NS - 1/2 stages to arrive in, not NS - 1.
    // The stores of the last tile stand between its loads and later ones: the waits for
    // the loads before them count them, or they would wait for the stores too.
    // Measured: 8192 x 25600 x 5120 906 -> 885 us, 8192 x 4096 x 12288 350 -> 335; with three
    // stages a load has time enough and the second meeting only costs (512 x 8192 x 5120
    // 29.3 -> 29.8).
    constexpr int kFirst = (NS - 2) * (D + 1) + (TWO ? U1 - 1 : 0);
    if (stored == XT) wait_vmcnt<kFirst + 2 * XT>();
    else if (stored > 0) wait_vmcnt<kFirst + 2>();
    else wait_vmcnt<kFirst>();
    lds_barrier();
    auto meet_mid = [&](int kt) {
      if (kt == 0 && stored == XT) wait_vmcnt<kFlight + 2 * XT>();
      else wait_vmcnt<kFlight>();
      wait_lgkm0();
      lds_barrier();
    };
    auto meet_end = [&]() {
      wait_vmcnt<kFlight - TWO>();
      wait_lgkm0();
      lds_barrier();
    };
    // grouped: what the end of the tile needs is loaded under its products
    t += gridDim.x;
    const bool more = t < total;
    const int asg_now = asg;
    float wt_now = 1.f;
    if constexpr (GR) {
      if (g.down && wave < XS) wt_now = g.weights[asg_now];
    }
    if (more) {
      next = find(t);
      fetch(next);
    }
    const int wrow = wm * XT * 16;             // this wave's first row in the tile
    const int left = at.rows - at.m0 - wrow;   // its rows with results
    // a wave without any only loads (its SIMD's other wave then has the matrix core)
    const int active = left > 0 ? nst : 0;
    if (!active) {
      issue(NS - 1, 0, D + 1);
      for (int kt = 0; kt < nst; ++kt) {
        if constexpr (TWO) {
          meet_mid(kt);
          issue(kt + NS, 0, U0);
        }
        meet_end();
        issue(kt + NS, TWO ? U0 : 0, D + 1);
      }
    } else {
      issue(NS - 1, 0, kAfter);
    }
    float sc[2], sw, sw_next;
#pragma unroll
    for (int j = 0; j < 4; ++j) read_w(smem, j);
    read_x(smem, 0);
    sw = read_sw(smem);
    sc[0] = read_sx(smem, 0) * sw;
    sc[1] = 0.f;
    f32x4 p[4];  // products on their way
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int kt = 0; kt < active; ++kt) {
      const uint8_t* so = smem + (kt % NS) * STAGE;
      const uint8_t* sn = smem + ((kt + 1) % NS) * STAGE;
#pragma unroll
      for (int i = 0; i < XT; ++i) {
        float s_read = 0.f;
        if (TWO && i == XT / 2 - 1) meet_mid(kt);
        if (i == XT - 1) meet_end();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (i < XT - 1) {
            if (j == 0) read_x(so, i + 1);
            if (j == 1) s_read = read_sx(so, i + 1);
          }
          if (j == 0) xo = Operand<EXACT>(xf[i & 1]);
          if (i == 0) wo[j] = Operand<EXACT>(wf[j]);
          p[j] = block_product(wo[j], xo);
          // two products back
          if (j >= 2) add_scaled(acc[i][j - 2], p[j - 2], sc[i & 1]);
          else add_scaled(acc[(i + XT - 1) % XT][j + 2], p[j + 2], sc[(i + 1) & 1]);
          if (i == XT - 1) {
            // (after the last stage these read a stale buffer that is never used)
            read_w(sn, j);
            if (j == 0) read_x(sn, 0);
            if (j == 1) sw_next = read_sw(sn);
            if (j == 1) s_read = read_sx(sn, 0);
          }
          if constexpr (TWO) {
            const int step = 4 * (i - (XT / 2 - 1)) + j;  // from the middle on
            if (step >= 0 && step < SP0) issue(kt + NS, step * U0 / SP0, (step + 1) * U0 / SP0);
            if (i == XT - 1 && j < U1) issue(kt + NS, U0 + j, U0 + j + 1);
          } else {
            const int step = (4 * i + j + 4) % (4 * XT);  // from the meeting on
            if (step < SP0)
              issue(i == XT - 1 ? kt + NS : kt + NS - 1, step * (D + 1) / SP0, (step + 1) * (D + 1) / SP0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (i == XT - 1) sw = sw_next;
        sc[(i + 1) & 1] = s_read * sw;
      }
    }
#pragma unroll
    for (int j = 2; j < 4; ++j) add_scaled(acc[XT - 1][j], p[j], sc[1]);

    // ---- the next tile's first stages, then this one's results
    wait_vmcnt<0>();   // (the stages that the loop issued past the last, in zeros)
    wait_lgkm0();
    lds_barrier();     // every wave is done with the stage buffers
    if (more) {
      set_loads(next);
      for (int st = 0; st < NS - 1; ++st) issue(st, 0, D + 1);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);  // the stores stay behind those loads
    int* t_row = reinterpret_cast<int*>(smem + NS * STAGE);  // grouped: output row, weight
    float* t_wt = reinterpret_cast<float*>(smem + NS * STAGE) + BM;
    if constexpr (GR) {
      if (threadIdx.x < BM) {
        const int tok = asg_now / g.top_k;
        t_row[threadIdx.x] = g.down ? (asg_now - tok * g.top_k) * g.n + tok : asg_now;
        t_wt[threadIdx.x] = wt_now;
      }
      wait_lgkm0();
      lds_barrier();
    }
    if (!EXACT && !part) {
      // bf16: sixteen rows at a time through the wave's share of the last stage
      // buffer (which those loads leave alone), to leave as whole 128-byte runs.
      // Lanes past the last row store it again, so that every block is two stores.
      uint8_t* ot = smem + (NS - 1) * STAGE + wave * 16 * kOutRow;
      const int col0 = at.n0 + wn * 64;
      stored = col0 < a.n_out ? max(0, min(XT, (left + 15) >> 4)) : 0;
      bf16_t* out = static_cast<bf16_t*>(a.out) + col0;
      if (!GR) out += (size_t)(at.m0 + wrow) * a.ldo;
      const auto orsrc = __builtin_amdgcn_make_buffer_rsrc(out, 0, 0x7FFFFFFF, 0x00020000);
      const uint32_t o_voff = (uint32_t)((lane >> 3) * (int)a.ldo + 8 * (lane & 7)) * 2;
      // LDS serves a wave's accesses in order: the fences only keep the compiler's
      auto block = [&](int i, bool whole) {
        const float wt = GR ? t_wt[wrow + 16 * i + r] : 1.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 v = GR ? acc[i][j] * wt : acc[i][j];
          *reinterpret_cast<uint2*>(ot + r * kOutRow + 32 * j + 8 * q) =
              uint2{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)};
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          int lr = 8 * h + (lane >> 3);
          if (!whole) lr = min(lr, left - 16 * i - 1);
          const u32x4 v = *reinterpret_cast<const u32x4*>(ot + lr * kOutRow + 16 * (lane & 7));
          if (whole && !GR) {
            __builtin_amdgcn_raw_buffer_store_b128(v, orsrc, o_voff, (16 * i + 8 * h) * (int)a.ldo * 2, 2);
          } else {
            const size_t row = GR ? (size_t)t_row[wrow + 16 * i + lr] : (size_t)(16 * i + lr);
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(out + row * a.ldo + 8 * (lane & 7)));
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      };
      if (left >= 16 * XT && stored == XT && (GR || a.ldo < 1 << 22)) {
#pragma unroll
        for (int i = 0; i < XT; ++i) block(i, true);
      } else {
#pragma unroll
        for (int i = 0; i < XT; ++i)
          if (i < stored) block(i, false);  // uniform over the wave
      }
    } else {
#pragma unroll
      for (int i = 0; i < XT; ++i) {
        if (16 * i + r >= left) continue;
        const size_t row = at.m0 + wrow + 16 * i + r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int col = at.n0 + wn * 64 + 16 * j + 4 * q;
          if (col >= a.n_out) continue;
          if (part)
            *reinterpret_cast<f32x4*>(part + ((size_t)blockIdx.y * a.m + row) * a.n_out + col) = acc[i][j];
          else
            store4(a.out, row * a.ldo + col, acc[i][j], a.out_bf16);
        }
      }
    }
    if (!more) break;
    at = next;
  }
}

// ------------------------------------------------------------------ plans and launches
namespace {

constexpr int kCUs = 256;

// What a plan takes (us), fitted to the timings within twice the best of their product,
// of 14916 of 24 row counts from 1 to 4096 and 16 matrices of 0.1 to 262 MB, weights cold,
// in graphs (7 to 12% rms; the plan with the least is 1.1% slower than the best of all
// on average, 23% at worst: 48 x 5120 x 25600 37.5 for 30.4).  LDS tiles: rounds of `cap`
// workgroups, a stage per 128-column block, dearer on a full chip, the operands' bytes,
// and with a K split the sum kernel and its partials.
struct TileCost {
  int bm, bn, cap;
  double fixed, round, stage, load, per_mb, split, split_mb;
};
constexpr TileCost kBf16Tiles[] = {
    {256, 256, kCUs, 3.53, 2.29, 1.11, 0.288, 0.0, 2.18, 0.378},
    {128, 256, kCUs, 2.83, 2.53, 0.675, 0.176, 0.031, 4.08, 0.311},
    {128, 128, kCUs, 3.89, 0.818, 0.377, 0.141, 0.031, 2.98, 0.376},
    {64, 256, kCUs, 4.0, 0.807, 0.443, 0.141, 0.074, 2.16, 0.392},
    {64, 128, 2 * kCUs, 3.89, 0.73, 0.342, 0.321, 0.05, 1.97, 0.463}};
constexpr TileCost kF32Tiles[] = {
    {},
    {128, 256, kCUs, 6.79, 1.81, 1.26, 0.339, 0.0, 1.03, 0.329},
    {128, 128, kCUs, 5.69, 0.651, 0.669, 0.224, 0.0, 1.45, 0.423},
    {64, 256, kCUs, 6.1, 0.0, 0.756, 0.304, 0.0, 0.928, 0.468},
    {64, 128, 2 * kCUs, 4.89, 0.273, 0.601, 0.504, 0.015, 1.53, 0.529}};
// The stream, in one round of a workgroup per CU (in more it starts and drains again):
// each wave takes every fourth step, whose time is that of its loads, 2 KB for each block
// of weight rows and of activation rows.
constexpr double kStreamFixed = 3.93, kStreamW = 0.156, kStreamX = 0.126, kStreamMB = 0.028,
                 kStreamSplit = 1.86, kStreamSplitMB = 1.04;
constexpr int kStreamRB[] = {1, 2, 3, 4, 6};

}  // namespace

Linear8Plan plan_linear8(int m, int n_out, int k, int out_bf16) {
  Linear8Plan best;
  double best_us = 1e30;
  const int KB = k >> 7;
  const double mbytes = 1e-6 * ((double)n_out + m) * k, out_mb = 4e-6 * m * n_out;
  for (int want : {1, 2, 3, 4, 6, 8}) {
    if (want > 1 && KB < 2 * want) break;
    const int chunk = (KB + want - 1) / want, s = (KB + chunk - 1) / chunk;
    for (int mb = 1; mb <= 4 && want <= 4; mb *= 2)
      for (int rb : kStreamRB) {
        if (mb > 1 && (rb > 4 || m <= 8 * mb)) continue;
        const int64_t wgs = (int64_t)((m + 16 * mb - 1) / (16 * mb)) * ((n_out / 16 + rb - 1) / rb) * s;
        if (wgs > kCUs) continue;
        const int steps = (chunk + 3) / 4;
        const double us = kStreamFixed + steps * (kStreamW * rb + kStreamX * mb) + kStreamMB * mbytes +
                          (s > 1 ? kStreamSplit + kStreamSplitMB * s * out_mb : 0.0);
        if (us < best_us) {
          best_us = us;
          best = Linear8Plan{s, chunk, rb, mb, 0};
        }
      }
    for (int i = 0; i < 5; ++i) {
      const TileCost& t = out_bf16 ? kBf16Tiles[i] : kF32Tiles[i];
      if (!t.bm) continue;
      const int64_t wgs = (int64_t)((m + t.bm - 1) / t.bm) * ((n_out + t.bn - 1) / t.bn) * s;
      // over many rounds the last one's idle CUs weigh less
      const double rounds = wgs <= 4 * t.cap ? (double)((wgs + t.cap - 1) / t.cap) : (double)wgs / t.cap + 0.5;
      const double full = std::min(1.0, (double)wgs / t.cap);
      const double us = t.fixed + rounds * (t.round + chunk * (t.stage + t.load * full)) +
                        t.per_mb * mbytes + (s > 1 ? t.split + t.split_mb * s * out_mb : 0.0);
      if (us < best_us) {
        best_us = us;
        best = Linear8Plan{s, chunk, 0, 0, i + 1};
      }
    }
  }
  return best;
}

size_t linear8_workspace_bytes(int m, int n_out, const Linear8Plan& p) {
  return p.splits > 1 ? (size_t)p.splits * m * n_out * sizeof(float) : 0;
}

namespace {

template <int MB, int RB>
hipError_t run_linear8(const Linear8Args& a, const Linear8Plan& p, float* part, hipStream_t st) {
  const dim3 grid((a.n_out / 16 + RB - 1) / RB, p.splits, (a.m + 16 * MB - 1) / (16 * MB));
  if (a.out_bf16)
    hipLaunchKernelGGL((linear8_kernel<MB, RB, false>), grid, dim3(256), 0, st, a, p.kb_chunk, part);
  else
    hipLaunchKernelGGL((linear8_kernel<MB, RB, true>), grid, dim3(256), 0, st, a, p.kb_chunk, part);
  return hipGetLastError();
}

// workgroups of LDS tiles that a CU holds at once
template <int BM, int BN, int NW, int NS>
constexpr int per_cu() {
  return NS * ((BM + BN) * 128 + NW * 256) <= 80 * 1024 ? 2 : 1;
}

template <int MB>
hipError_t run_stream(const Linear8Args& a, const Linear8Plan& p, float* part, hipStream_t st) {
  switch (p.rb) {
    case 1: return run_linear8<MB, 1>(a, p, part, st);
    case 2: return run_linear8<MB, 2>(a, p, part, st);
    case 3: return run_linear8<MB, 3>(a, p, part, st);
    case 4: return run_linear8<MB, 4>(a, p, part, st);
    case 6:
      if constexpr (MB == 1) return run_linear8<MB, 6>(a, p, part, st);
    default: return hipErrorInvalidValue;
  }
}

template <int BM, int BN, int NW, int NS>
hipError_t run_tile8(const Linear8Args& a, const Linear8Plan& p, float* part, hipStream_t st) {
  const int tiles_m = (a.m + BM - 1) / BM;
  const int tiles = tiles_m * ((a.n_out + BN - 1) / BN);
  const dim3 grid(std::min(tiles, std::max(1, kCUs * per_cu<BM, BN, NW, NS>() / p.splits)), p.splits);
  const Moe8Args none{};
  if (a.out_bf16) {
    hipLaunchKernelGGL((tile8_kernel<BM, BN, NW, NS, false, false>), grid, dim3(64 * NW), 0, st, a, p.kb_chunk,
                       part, tiles_m, none);
    return hipGetLastError();
  }
  if constexpr (BM * BN < 256 * 256) {  // the converted weights have no room beside 256 x 256 sums
    hipLaunchKernelGGL((tile8_kernel<BM, BN, NW, NS, true, false>), grid, dim3(64 * NW), 0, st, a, p.kb_chunk,
                       part, tiles_m, none);
    return hipGetLastError();
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_linear8(const Linear8Args& a, const Linear8Plan& p, float* workspace,
                          hipStream_t st) {
  if (a.m == 0) return hipSuccess;
  float* part = p.splits > 1 ? workspace : nullptr;
  hipError_t e;
  switch (p.tile) {
    case 1: e = run_tile8<256, 256, 8, 2>(a, p, part, st); break;
    case 2: e = run_tile8<128, 256, 8, 3>(a, p, part, st); break;
    case 3: e = run_tile8<128, 128, 8, 4>(a, p, part, st); break;
    case 4: e = run_tile8<64, 256, 8, 3>(a, p, part, st); break;
    case 5: e = run_tile8<64, 128, 4, 3>(a, p, part, st); break;
    default:
      e = p.mb == 1   ? run_stream<1>(a, p, part, st)
          : p.mb == 2 ? run_stream<2>(a, p, part, st)
                      : run_stream<4>(a, p, part, st);
  }
  if (e != hipSuccess || !part) return e;
  const size_t blocks = ((size_t)a.m * a.n_out / 4 + 255) / 256;
  hipLaunchKernelGGL(linear8_sum_kernel, dim3((unsigned)std::min<size_t>(blocks, 8192)), dim3(256), 0,
                     st, part, p.splits, a);
  return hipGetLastError();
}

// Rows of a tile by the entries an expert has on average, 0: the stream (30B-A3B
// gate/up + down, us, stream / tiles of 32 / 128 / 256 rows: 1 entry 40 + 22 / 40 + 28 / 48 + 31;
// 4 63 + 35 / 68 + 37 / 72 + 45 / 89 + 51; 5 71 + 38 / 70 + 39 / 74 + 45; 8 82 + 48 / 70 + 40 / 77 +
// 46 / 88 + 51; 24 - / 79 + 47 / 81 + 50 / 87 + 56; 32 - / 92 + 53 / 93 + 57 / 90 + 55; 40 - / 98 +
// 60 / 94 + 59; 64 - / 116 + 70 / 97 + 62 / 96 + 63; 128 - / - / 119 + 74 / 125 + 82; 200 - / - /
// 149 + 103 / 153 + 99; 256 - / - / 173 + 122 / 166 + 111; 512 - / - / 288 + 204 / 264 + 189).  64
// rows were never the best by more than 2%.  The lists' own lengths are on the device: the
// rule goes by their mean, and these times are of independent routings.  Where tokens agree
// the same rule gives, independent / 16 experts / the same 8 for every token: 64 tokens
// 65 + 35 / 30 + 16 / 38 + 20; 256 72 + 41 / 31 + 24 / 28 + 15; 512 93 + 53 / 54 + 34 / 43 + 27;
// 4096 166 + 108 / 120 + 76 / 101 + 67.
constexpr int kStreamEntries = 4;

namespace {

template <int BM, int BN, int NW, int NS>
hipError_t run_moe8(const Linear8Args& a, const Moe8Args& g, hipStream_t st) {
  // as many tiles as lists of any lengths can fill
  const int64_t entries = (int64_t)g.n * g.top_k;
  const int64_t tiles_m = std::min<int64_t>((entries + BM - 1) / BM + g.n_experts, entries);
  const int64_t tiles = tiles_m * ((g.n_out + BN - 1) / BN);
  const dim3 grid((unsigned)std::min<int64_t>(tiles, kCUs * per_cu<BM, BN, NW, NS>()));
  hipLaunchKernelGGL((tile8_kernel<BM, BN, NW, NS, false, true>), grid, dim3(64 * NW), 0, st, a, a.k >> 7,
                     nullptr, 0, g);
  return hipGetLastError();
}

}  // namespace

static int moe8_tile_rows(const Moe8Args& g) {
  const int64_t per = ((int64_t)g.n * g.top_k + g.n_experts - 1) / g.n_experts;
  return per <= kStreamEntries ? 0 : per <= 32 ? 32 : per <= 200 ? 128 : 256;
}

hipError_t launch_moe8(const Moe8Args& g, hipStream_t st) {
  if (g.n == 0) return hipSuccess;
  Linear8Args a{};
  a.n_out = g.n_out; a.k = g.k; a.x = g.x; a.ldx = g.ldx; a.xs = g.xs; a.lds = g.lds;
  a.w = g.w; a.ws = g.ws; a.out = g.out; a.ldo = g.n_out; a.out_bf16 = 1;
  switch (moe8_tile_rows(g)) {
    case 0:
      hipLaunchKernelGGL(moe8_kernel, dim3((g.n_out + 127) / 128, g.n_experts), dim3(256), 0, st, g);
      return hipGetLastError();
    case 32: return run_moe8<32, 256, 4, 2>(a, g, st);
    case 128: return run_moe8<128, 256, 8, 3>(a, g, st);
    default: return run_moe8<256, 256, 8, 2>(a, g, st);
  }
}

}  // namespace sevo
