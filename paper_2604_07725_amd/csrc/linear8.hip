// Y = X W^T on 8-bit operands with a scale for each block of 128 (e4m3 codes;
// X: a scale per row and 128 columns, W: one per 128 rows and 128 columns):
//   Y[m][n] = sum over 128-column blocks b of
//             sx[b][m] sw[n / 128][b] (sum over k in b of X[m][k] W[n][k]).
// The inner sum of a block runs on the matrix cores, its scaled addition to the
// fp32 accumulator on the vector ALU (one FMA per element and block, the two
// scales multiplied once per row fragment).
//
// Two matrix instructions.  The 8-bit ones (16x16x128) have twice the rate of
// bf16 but sum a block's products with a relative error of 1.4e-5 (measured, the
// same for 16x16x32 and 32x32x64, unbiased, independent of k), far below the
// 2^-9 of a result that is rounded to bf16, which is what they are used for.  A result kept in
// fp32 takes the bf16 instruction on the codes converted to bf16, which is
// exact (e4m3 has four significant bits): 1e-7.
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
  __device__ __forceinline__ explicit Operand(const Frag8& f) : v(f.v) {}
};
template <>
struct Operand<true> {
  bf16x8v v[4];
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

}  // namespace

// Few rows: a weight stream.  One workgroup per (RB 16-row weight blocks, K
// split, M tile of 16 MB rows); its four waves take the 128-column steps of the
// split in turn and sum their tiles through LDS.
template <int MB, int RB, bool EXACT>
__global__ __launch_bounds__(256, 1) void linear8_kernel(Linear8Args a, int kb_chunk,
                                                         float* __restrict__ part) {
  __shared__ f32x4 red[4][RB][MB][64];
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
    wp[i] = a.w + ((size_t)(rb >> 2) * KB * 4 + (rb & 3)) * 2048 + lane * 16;
  }
  const uint8_t* xp[MB];
  const float* xsp[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int row = min(m0 + 16 * b + r, a.m - 1);
    xp[b] = a.x + (size_t)row * a.ldx + 16 * q;
    xsp[b] = a.xs + row;
  }
  // the RB (at most 8) row blocks lie in at most two 128-row scale blocks
  const float* ws0 = a.ws + (size_t)(rb0 >> 3) * KB;
  const float* ws1 = a.ws + (size_t)((min(rb0 + RB, nrb) - 1) >> 3) * KB;

  const int st0 = blockIdx.y * kb_chunk;
  const int nsteps = min(KB - st0, kb_chunk);
  const int cnt = nsteps > wave ? (nsteps - wave + 3) >> 2 : 0;  // steps of this wave

  struct Step {
    Frag8 w[RB], x[MB];
    float sx[MB], sw0, sw1;
  };
  // j-th step of this wave; past the end it re-reads the last one
  auto load = [&](Step& f, int j) {
    const int st = st0 + wave + 4 * min(j, cnt - 1);
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        f.w[i].u[h] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(wp[i] + (size_t)st * 8192 + 1024 * h));
#pragma unroll
    for (int b = 0; b < MB; ++b) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        f.x[b].u[h] = *reinterpret_cast<const u32x4*>(xp[b] + (size_t)st * 128 + 64 * h);
      f.sx[b] = xsp[b][(size_t)st * a.lds];
    }
    f.sw0 = ws0[st];
    f.sw1 = ws1[st];
  };
  f32x4 acc[RB][MB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto mma = [&](const Step& f) {
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      const Operand<EXACT> xo(f.x[b]);
      const float s0 = f.sx[b] * f.sw0, s1 = f.sx[b] * f.sw1;
#pragma unroll
      for (int i = 0; i < RB; ++i)
        add_scaled(acc[i][b], block_product(Operand<EXACT>(f.w[i]), xo),
                   (rb0 + i) >> 3 == rb0 >> 3 ? s0 : s1);
    }
  };
  if (cnt > 0) {
    // three buffers: two steps of loads in flight under the products
    Step f0, f1, f2;
    load(f0, 0);
    load(f1, 1);
    for (int j = 0; j < cnt; j += 3) {
      load(f2, j + 2);
      __builtin_amdgcn_sched_barrier(0);
      mma(f0);
      __builtin_amdgcn_sched_barrier(0);
      load(f0, j + 3);
      __builtin_amdgcn_sched_barrier(0);
      if (j + 1 < cnt) mma(f1);
      __builtin_amdgcn_sched_barrier(0);
      load(f1, j + 4);
      __builtin_amdgcn_sched_barrier(0);
      if (j + 2 < cnt) mma(f2);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
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

// The same product grouped by expert.  A wave takes two 16-row weight blocks of
// one expert over the whole k, a workgroup 128 rows (one row of weight scales); the
// expert's entries come in tiles of 16 NB rows, gathered through its list.
template <int NB>
__global__ __launch_bounds__(256) void moe8_kernel(Moe8Args a) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, q = lane >> 4;
  const int e = blockIdx.y;
  const int off = a.offsets[e], ne = a.offsets[e + 1] - off;
  const int KB = a.k >> 7, nrb = a.n_out >> 4;
  const int rb0 = blockIdx.x * 8 + 2 * wave;
  if (ne <= 0 || rb0 >= nrb) return;  // wave-uniform, no barrier follows
  const uint8_t* wp = a.w + (size_t)e * a.n_out * a.k +
                      ((size_t)(rb0 >> 2) * KB * 4 + (rb0 & 3)) * 2048 + lane * 16;
  const float* wsp = a.ws + ((size_t)e * ((a.n_out + 127) >> 7) + (rb0 >> 3)) * KB;
  struct Step {
    Frag8 w[2], x[NB];
    float sx[NB], sw;
  };
  for (int m0 = 0; m0 < ne; m0 += 16 * NB) {
    const uint8_t* xp[NB];
    const float* xsp[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int asg = a.assign[off + min(m0 + 16 * b + r, ne - 1)];
      const int row = a.down ? asg : asg / a.top_k;
      xp[b] = a.x + (size_t)row * a.ldx + 16 * q;
      xsp[b] = a.xs + row;
    }
    f32x4 acc[2][NB];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto load = [&](Step& f, int j) {
      const int st = min(j, KB - 1);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          f.w[i].u[h] = __builtin_nontemporal_load(
              reinterpret_cast<const u32x4*>(wp + (size_t)st * 8192 + 2048 * i + 1024 * h));
#pragma unroll
      for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          f.x[b].u[h] = *reinterpret_cast<const u32x4*>(xp[b] + (size_t)st * 128 + 64 * h);
        f.sx[b] = xsp[b][(size_t)st * a.lds];
      }
      f.sw = wsp[st];
    };
    auto mma = [&](const Step& f) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const Operand<false> xo(f.x[b]);
        const float s = f.sx[b] * f.sw;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          add_scaled(acc[i][b], block_product(Operand<false>(f.w[i]), xo), s);
      }
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
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int i = m0 + 16 * b + r;
      if (i >= ne) continue;
      const int asg = a.assign[off + i];
      float wt = 1.f;
      size_t row = asg;
      if (a.down) {
        const int t = asg / a.top_k;
        row = (size_t)(asg - t * a.top_k) * a.n + t;
        wt = a.weights[asg];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
        store4(a.out, row * a.n_out + (rb0 + h) * 16 + 4 * q, acc[h][b] * wt, 1);
    }
  }
}

// ------------------------------------------------------------------ plans and launches
Linear8Plan plan_linear8(int m, int n_out, int k) {
  Linear8Plan p;
  p.mb = m > 32 ? 4 : m > 16 ? 2 : 1;
  const int KB = k >> 7, nrb = n_out >> 4;
  const int mt = (m + 16 * p.mb - 1) / (16 * p.mb);
  p.rb = 4;
  int s = 1;
  while (s < 8 && (long)((nrb + p.rb - 1) / p.rb) * mt * s < 256 && KB >= 8 * s) s *= 2;
  p.kb_chunk = (KB + s - 1) / s;
  p.splits = (KB + p.kb_chunk - 1) / p.kb_chunk;
  return p;
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

}  // namespace

hipError_t launch_linear8(const Linear8Args& a, const Linear8Plan& p, float* workspace,
                          hipStream_t st) {
  if (a.m == 0) return hipSuccess;
  float* part = p.splits > 1 ? workspace : nullptr;
  hipError_t e;
  if (p.mb == 4) e = run_linear8<4, 4>(a, p, part, st);
  else if (p.mb == 2) e = run_linear8<2, 4>(a, p, part, st);
  else e = run_linear8<1, 4>(a, p, part, st);
  if (e != hipSuccess || !part) return e;
  const size_t blocks = ((size_t)a.m * a.n_out / 4 + 255) / 256;
  hipLaunchKernelGGL(linear8_sum_kernel, dim3((unsigned)std::min<size_t>(blocks, 8192)), dim3(256), 0,
                     st, part, p.splits, a);
  return hipGetLastError();
}

int moe8_tile_rows(int64_t entries, int n_experts) { return entries < 96ll * n_experts ? 128 : 256; }

hipError_t launch_moe8(const Moe8Args& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  const long per = ((long)a.n * a.top_k + a.n_experts - 1) / a.n_experts;
  const dim3 grid((a.n_out + 127) / 128, a.n_experts);
  if (per <= 12) hipLaunchKernelGGL(moe8_kernel<1>, grid, dim3(256), 0, st, a);
  else if (per <= 24) hipLaunchKernelGGL(moe8_kernel<2>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(moe8_kernel<4>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace sevo
