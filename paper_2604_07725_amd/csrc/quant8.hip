// 8-bit activations: the residual add + RMSNorm and the bf16 / SwiGLU
// quantiser that feed the block-scaled products, and the packed 8-bit weight
// layout.  Codes are OCP e4m3 (largest value 448); a row's 128-column block b
// has one fp32 scale
//   s = max(amax / 448, 2^-64),   code = rne_e4m3(y / s),
// so y is held to half a step of 2^-4 of its block's range.  A block with a NaN
// or an infinity gets the scale NaN (its codes too), which every product that
// touches it shows.
#include "common.h"
#include "kernels.h"

namespace sevo {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kTop = 448.f;               // largest e4m3 value
constexpr float kLeastScale = 0x1p-64f;     // of a block of zeros

// max over the 16 lanes of a row of the wave, every lane gets it
__device__ __forceinline__ uint32_t row16_umax(uint32_t v) {
  v = max(v, lane_xor<1>(v));
  v = max(v, lane_xor<2>(v));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppRowHalfMirror, 0xF, 0xF, false));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDppRowMirror, 0xF, 0xF, false));
}

// The 128 values of a block, eight in each of 16 neighbouring lanes, to codes
// (returned, 8 bytes) and their scale.  Magnitudes are compared as integers:
// the order of finite values, with infinities and NaNs above them.
__device__ __forceinline__ u32x2 block_codes(const float (&y)[8], float* scale) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(y[i]) & 0x7FFFFFFFu);
  a = row16_umax(a);
  const float s = a < 0x7F800000u ? fmaxf(__uint_as_float(a) * (1.f / kTop), kLeastScale) : NAN;
  const float inv = 1.f / s;
  *scale = s;
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * inv, y[1] * inv, 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * inv, y[3] * inv, lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4] * inv, y[5] * inv, 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6] * inv, y[7] * inv, hi, true);
  return u32x2{(uint32_t)lo, (uint32_t)hi};
}

__device__ __forceinline__ void unpack8(const u32x4& w, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_lo(w[i]);
    v[2 * i + 1] = bf16_hi(w[i]);
  }
}

}  // namespace

// Workgroup per row; thread t owns columns 8 (t + T g) .. + 8, g < NG, in
// registers from the one read of x to the codes, so a block of 128 columns is 16
// lanes of one wave.  T and NG follow from the columns alone: a row's bits do not
// depend on the rows beside it.  Bound by HBM from about 1000 rows on: in graphs,
// 8192 x 2048 with eight bf16 partials 70 us (6.0 TB/s), 8192 x 4096 with one 54.9 (6.7
// TB/s); 4 x 4096 3.5 us, of which the launch is 3.4.  Half the threads with twice the
// columns each: 82, 55.0 and 4.0 (for 73, 55.2 and 3.5).  Codes are stored past the caches
// (8192 x 5120 with one partial 75.8 -> 67.7).
template <int T, int NG, typename P>
__global__ __launch_bounds__(T) void add_rmsnorm_fp8_kernel(AddNormFp8Args a, int past_cache) {
  __shared__ float red[T / 64];
  const int row = xcd_row(blockIdx.x, gridDim.x);
  float* xr = a.x + (size_t)row * a.cols;
  const P* pr = static_cast<const P*>(a.partials) + (size_t)row * a.cols;
  const size_t plane = (size_t)a.rows * a.cols;
  float v[NG][8];
  float ss = 0.f;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const int c = 8 * (threadIdx.x + T * g);
    if (c >= a.cols) continue;
    *reinterpret_cast<f32x4*>(&v[g][0]) = *reinterpret_cast<const f32x4*>(xr + c);
    *reinterpret_cast<f32x4*>(&v[g][4]) = *reinterpret_cast<const f32x4*>(xr + c + 4);
    if (a.n_partials > 0) {
      constexpr int kAtOnce = 4;  // partials loaded together, added in order
      auto add = [&](auto once) {
        auto get = [&](const P* src) {
          const u32x4* q = reinterpret_cast<const u32x4*>(src);
          if constexpr (decltype(once)::value) return __builtin_nontemporal_load(q);
          else return *q;
        };
        for (int s0 = 0; s0 < a.n_partials; s0 += kAtOnce) {
          float p[kAtOnce][8];
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j)
            if (s0 + j < a.n_partials) {
              const P* src = pr + (s0 + j) * plane + c;
              if constexpr (sizeof(P) == 2) {
                unpack8(get(src), p[j]);
              } else {
                *reinterpret_cast<u32x4*>(&p[j][0]) = get(src);
                *reinterpret_cast<u32x4*>(&p[j][4]) = get(src + 4);
              }
            }
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j)
            if (s0 + j < a.n_partials)
#pragma unroll
              for (int i = 0; i < 8; ++i) v[g][i] += p[j][i];
        }
      };
      if (past_cache) add(std::true_type{});
      else add(std::false_type{});
      *reinterpret_cast<f32x4*>(xr + c) = *reinterpret_cast<f32x4*>(&v[g][0]);
      *reinterpret_cast<f32x4*>(xr + c + 4) = *reinterpret_cast<f32x4*>(&v[g][4]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += v[g][i] * v[g][i];
  }
  ss = block_sum<T / 64>(ss, red);
  const float inv = 1.f / sqrtf(ss / (float)a.cols + a.eps);
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const int c = 8 * (threadIdx.x + T * g);
    if (c >= a.cols) continue;  // whole blocks: cols is a multiple of 128
    float gn[8], y[8];
    unpack8(*reinterpret_cast<const u32x4*>(a.gain + c), gn);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = v[g][i] * inv * gn[i];
    float s;
    const u32x2 q = block_codes(y, &s);
    __builtin_nontemporal_store(q, reinterpret_cast<u32x2*>(a.out + (size_t)row * a.cols + c));
    if ((threadIdx.x & 15) == 0) a.scales[(size_t)(c >> 7) * a.rows + row] = s;
    if (a.out_bf16) {
      u32x4 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = pack_bf16x2(y[2 * i], y[2 * i + 1]);
      *reinterpret_cast<u32x4*>(a.out_bf16 + (size_t)row * a.cols + c) = o;
    }
  }
}

int64_t add_rmsnorm_fp8_max_rows(int cols) {  // a workgroup each, of the most threads that cols takes
  return (((int64_t)1 << 32) - 1) / (cols <= 512 ? 64 : cols <= 2048 ? 256 : cols <= 4096 ? 512 : 1024);
}

hipError_t launch_add_rmsnorm_fp8(const AddNormFp8Args& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  // Partials are read past the caches once a call's data cannot stay in the last-level
  // one (256 MiB) anyway: there they would push out x, which the next norm reads (us,
  // plain / past the caches: 235 MB, 8192 x 4096 and one partial, 54.9 / 59.4; 302 MB, two,
  // 64.0 / 68.5; 352 MB, 8192 x 2048 and eight, 70.3 / 70.1 and with new partials each call
  // 80.6 / 68.8; 436 MB 95.3 / 88.5; 705 MB 158 / 133).
  const int past_cache =
      (size_t)a.rows * a.cols * (5 + (size_t)a.n_partials * (a.partials_bf16 ? 2 : 4)) > (size_t)320 << 20;
  auto go = [&](auto t_tag, auto ng_tag) {
    constexpr int T = decltype(t_tag)::value, NG = decltype(ng_tag)::value;
    if (a.partials_bf16)
      hipLaunchKernelGGL((add_rmsnorm_fp8_kernel<T, NG, bf16_t>), dim3(a.rows), dim3(T), 0, st, a, past_cache);
    else
      hipLaunchKernelGGL((add_rmsnorm_fp8_kernel<T, NG, float>), dim3(a.rows), dim3(T), 0, st, a, past_cache);
    return hipGetLastError();
  };
  using std::integral_constant;
  const int groups = (a.cols + 7) / 8;
  if (groups <= 64) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (groups <= 256) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (groups <= 512) return go(integral_constant<int, 512>{}, integral_constant<int, 1>{});
  if (groups <= 1024) return go(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  if (groups <= 2048) return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  return go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

// A wave takes four blocks (512 columns) of R consecutive rows, 16 lanes a
// block.  Lane j of a block's 16 keeps row j's scale, so that the scales of R
// rows leave as one run of a [k/128][m] row.  Bound by HBM: 8192 x 12288 SwiGLU in a
// graph 99 us, 5.1 TB/s.
template <int R, bool SWIGLU>
__global__ __launch_bounds__(256) void quantize_fp8_kernel(const bf16_t* __restrict__ x, int64_t ldx,
                                                           int m, int k, uint8_t* __restrict__ out,
                                                           float* __restrict__ scales) {
  const int lane = threadIdx.x & 63, j = lane & 15;
  const int quads = (k + 511) >> 9;
  const long unit = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int r0 = (int)(unit / quads) * R;
  const int c = (int)(unit % quads) * 512 + 8 * lane;
  if (r0 >= m || c >= k) return;  // whole 16-lane blocks leave; no barrier
  float keep = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = r0 + i;
    if (row >= m) break;
    const bf16_t* src = x + (size_t)row * ldx + c;
    float y[8];
    unpack8(*reinterpret_cast<const u32x4*>(src), y);
    if constexpr (SWIGLU) {
      float u[8];
      unpack8(*reinterpret_cast<const u32x4*>(src + k), u);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] / (1.f + __expf(-y[e])) * u[e];
    }
    float s;
    // past the caches (8192 x 4096 19.2 -> 18.3 us): the product that reads them comes later
    __builtin_nontemporal_store(block_codes(y, &s), reinterpret_cast<u32x2*>(out + (size_t)row * k + c));
    if (j == i) keep = s;
  }
  if (j < R && r0 + j < m) scales[(size_t)(c >> 7) * m + r0 + j] = keep;
}

int64_t quantize_fp8_max_rows(int k) {  // four rows of 512 columns a wave, four waves a workgroup
  return (((int64_t)1 << 26) - 4) / ((k + 511) / 512) * 4;
}

hipError_t launch_quantize_fp8(const bf16_t* x, int64_t ldx, int m, int k, int swiglu, uint8_t* out,
                               float* scales, hipStream_t st) {
  if (m == 0) return hipSuccess;
  const long quads = (k + 511) / 512;
  auto go = [&](auto kern, int rows) {
    const long units = (long)((m + rows - 1) / rows) * quads;
    hipLaunchKernelGGL(kern, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, st, x, ldx, m, k, out,
                       scales);
    return hipGetLastError();
  };
  // A row per wave while that leaves the chip short of waves, else four, whose loads
  // pass under each other and whose scales share a line (us in graphs, a row a wave / 2 /
  // 4 / 8 / 16: 64 x 12288 SwiGLU 3.5 / 3.8 / 5.0 / 7.0 / 11.4; 1024 x 4096 4.6 / 4.6 / 4.9 / 6.3 /
  // 9.5; 2048 x 4096, 16384 waves of a row, 6.6 / 6.4 / 6.4 / 7.1 / 10.2; 8192 x 12288 SwiGLU
  // 108.5 / 103.4 / 99.1 / 104.7 / 110.7).
  if ((long)m * quads < 16384)
    return swiglu ? go(quantize_fp8_kernel<1, true>, 1) : go(quantize_fp8_kernel<1, false>, 1);
  return swiglu ? go(quantize_fp8_kernel<4, true>, 4) : go(quantize_fp8_kernel<4, false>, 4);
}

// Row-major codes [n][k] -> the packed layout, one thread per 16-byte run of dst.
__global__ __launch_bounds__(256) void pack_weight_fp8_kernel(const uint8_t* __restrict__ src,
                                                              uint8_t* __restrict__ dst, size_t runs,
                                                              int k) {
  const int kb = k >> 7;
  for (size_t g = (size_t)blockIdx.x * blockDim.x + threadIdx.x; g < runs;
       g += (size_t)gridDim.x * blockDim.x) {
    const size_t blk = g >> 9;  // (superblock, 128-column step): 512 runs
    const int rem = (int)(g & 511);
    const size_t sb = blk / kb;
    const int st = (int)(blk - sb * kb);
    const size_t row = sb * 64 + (rem >> 7) * 16 + (rem & 15);
    const int col = st * 128 + ((rem & 127) >> 4) * 16;
    *reinterpret_cast<u32x4*>(dst + g * 16) =
        *reinterpret_cast<const u32x4*>(src + row * k + col);
  }
}

hipError_t launch_pack_weight_fp8(const uint8_t* src, uint8_t* dst, int64_t n, int k,
                                  hipStream_t st) {
  const size_t runs = (size_t)n * k / 16;
  if (runs == 0) return hipSuccess;
  const size_t blocks = (runs + 255) / 256;
  hipLaunchKernelGGL(pack_weight_fp8_kernel, dim3((unsigned)(blocks < 16384 ? blocks : 16384)),
                     dim3(256), 0, st, src, dst, runs, k);
  return hipGetLastError();
}

}  // namespace sevo
