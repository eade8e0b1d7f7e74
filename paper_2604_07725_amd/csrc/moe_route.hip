// Routing of tokens to experts from router logits: softmax or sigmoid scores, a
// balance bias that acts on the choice alone, groups of experts of which the
// best are kept, the top-k of what is left, and weights from the unbiased
// scores.  Scores are formed and compared in float64: a choice turns on the
// difference of two of them, and near-equal sigmoids of large logits are equal in
// fp32.  Ties go to the lower group and the lower expert index.
#include "common.h"
#include "kernels.h"

namespace sevo {

namespace {

constexpr int kMaxExperts = 256;
constexpr int kPerLane = kMaxExperts / 64;

__device__ __forceinline__ double lane_xor_f64(double v, int mask) {
  return __shfl_xor(v, mask, kWave);
}

// the wave's best (value, then lower index) of each lane's candidate; every lane gets it
__device__ __forceinline__ void wave_best(double& v, int& i) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const double ov = lane_xor_f64(v, o);
    const int oi = __shfl_xor(i, o, kWave);
    if (ov > v || (ov == v && oi < i)) {
      v = ov;
      i = oi;
    }
  }
}

}  // namespace

// One wave per token; lane l holds experts l, l + 64, ...
__global__ __launch_bounds__(64) void moe_route8_kernel(MoeRouteArgs a) {
  __shared__ double pick_s[kMaxExperts];
  const int t = blockIdx.x, lane = threadIdx.x;
  const float* lg = a.logits + (size_t)t * a.ld;
  double score[kPerLane], pick[kPerLane];
  double z[kPerLane], mx = -INFINITY;
#pragma unroll
  for (int j = 0; j < kPerLane; ++j) {
    const int e = lane + 64 * j;
    z[j] = e < a.n_experts ? (double)lg[e] : -INFINITY;
    mx = fmax(mx, z[j]);
  }
  if (a.sigmoid) {
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) score[j] = 1.0 / (1.0 + exp(-z[j]));
  } else {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mx = fmax(mx, lane_xor_f64(mx, o));
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
      score[j] = lane + 64 * j < a.n_experts ? exp(z[j] - mx) : 0.0;
      sum += score[j];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += lane_xor_f64(sum, o);
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) score[j] /= sum;
  }
  // a NaN is chosen after everything else
  uint32_t open = 0;  // bit j: expert lane + 64 j may be chosen
#pragma unroll
  for (int j = 0; j < kPerLane; ++j) {
    const int e = lane + 64 * j;
    pick[j] = -INFINITY;
    if (e < a.n_experts) {
      const double p = a.bias ? score[j] + (double)a.bias[e] : score[j];
      if (p == p) pick[j] = p;
      open |= 1u << j;
    }
  }
  if (a.top_groups < a.n_groups) {
    const int each = a.n_experts / a.n_groups;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
      if (lane + 64 * j < a.n_experts) pick_s[lane + 64 * j] = pick[j];
    __syncthreads();
    // lane g: the sum of group g's one or two best
    double g = -INFINITY;
    if (lane < a.n_groups) {
      double b0 = -INFINITY, b1 = -INFINITY;
      for (int i = 0; i < each; ++i) {
        const double v = pick_s[lane * each + i];
        if (v > b0) {
          b1 = b0;
          b0 = v;
        } else if (v > b1) {
          b1 = v;
        }
      }
      g = a.group_best == 2 ? b0 + b1 : b0;
      if (g != g) g = -INFINITY;  // +inf and -inf biases in one group
    }
    uint64_t kept = 0;
    for (int r = 0; r < a.top_groups; ++r) {
      double v = g;
      int i = lane < a.n_groups && !((kept >> lane) & 1) ? lane : kWave;
      if (i == kWave) v = -INFINITY;
      wave_best(v, i);
      kept |= 1ull << (i & 63);
    }
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
      if (!((kept >> (min(lane + 64 * j, a.n_experts - 1) / each)) & 1)) open &= ~(1u << j);
  }
  double sum = 0.0;
  double wt = 0.0;  // lane r: the score of choice r
  int ex = 0;
  for (int r = 0; r < a.top_k; ++r) {
    double v = -INFINITY;
    int i = 0x7FFFFFFF;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
      if (((open >> j) & 1) && (i == 0x7FFFFFFF || pick[j] > v)) {
        v = pick[j];
        i = lane + 64 * j;
      }
    wave_best(v, i);
    const int j = i >> 6;
    double sc = 0.0;
#pragma unroll
    for (int u = 0; u < kPerLane; ++u)
      if (u == j) sc = score[u];
    sc = __shfl(sc, i & 63, kWave);
    if (lane == (i & 63)) open &= ~(1u << j);
    if (lane == r) {
      wt = sc;
      ex = i;
    }
    sum += sc;
  }
  if (lane < a.top_k) {
    if (a.renormalise) wt /= sum + 1e-20;
    a.out_experts[(size_t)t * a.top_k + lane] = ex;
    a.out_weights[(size_t)t * a.top_k + lane] = (float)(wt * (double)a.scaling);
  }
}

hipError_t launch_moe_route8(const MoeRouteArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(moe_route8_kernel, dim3(a.n), dim3(64), 0, st, a);
  return hipGetLastError();
}

// Entry lists in one launch: workgroup e reads every entry twice, once to count
// those of lower experts (its list's first place) and its own, once to write its
// own in order: each thread holds eight consecutive entries of a chunk, and an
// entry's rank is the matches of the lanes and waves before it.  No sums pass
// between workgroups, and nothing depends on scheduling.
template <int T>
__global__ __launch_bounds__(T) void moe_lists_kernel(const int32_t* __restrict__ sel, int nk, int E,
                                                      int32_t* __restrict__ offsets,
                                                      int32_t* __restrict__ assign) {
  constexpr int W = T / 64, P = 8;  // entries a thread holds
  __shared__ int red[2][W];
  const int e = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto load = [&](int c0, int (&v)[P]) {
    const int i = c0 + P * tid;
    if (i + P <= nk) {
      *reinterpret_cast<u32x4*>(&v[0]) = *reinterpret_cast<const u32x4*>(sel + i);
      *reinterpret_cast<u32x4*>(&v[4]) = *reinterpret_cast<const u32x4*>(sel + i + 4);
    } else {
#pragma unroll
      for (int j = 0; j < P; ++j) v[j] = i + j < nk ? sel[i + j] : -1;
    }
  };
  int lower = 0, own = 0;
  for (int c0 = 0; c0 < nk; c0 += P * T) {
    int v[P];
    load(c0, v);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      lower += (uint32_t)v[j] < (uint32_t)e;  // (a negative id is in no list)
      own += v[j] == e;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lower += __shfl_xor(lower, o, kWave);
    own += __shfl_xor(own, o, kWave);
  }
  if (lane == 0) {
    red[0][wave] = lower;
    red[1][wave] = own;
  }
  __syncthreads();
  int first = 0, count = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    first += red[0][w];
    count += red[1][w];
  }
  if (tid == 0) {
    offsets[e] = first;
    if (e == E - 1) offsets[E] = first + count;
  }
  if (count == 0) return;  // uniform
  __syncthreads();
  int buf = 0;
  for (int c0 = 0; c0 < nk; c0 += P * T, buf ^= 1) {
    int v[P];
    load(c0, v);
    const uint64_t below = (1ull << lane) - 1;
    int rank = 0, total = 0;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint64_t b = __ballot(v[j] == e);
      rank += __popcll(b & below);
      total += __popcll(b);
    }
    if (lane == 0) red[buf][wave] = total;
    __syncthreads();  // (the other buffer's readers have passed the barrier before it is written)
    int at = first + rank;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (w < wave) at += red[buf][w];
      first += red[buf][w];
    }
#pragma unroll
    for (int j = 0; j < P; ++j)
      if (v[j] == e) assign[at++] = c0 + P * tid + j;
  }
}

// From this many entries on, reading all of them in every workgroup costs more
// than the three launches that count, scan and place.
constexpr int kOneLaunchEntries = 65536;

hipError_t launch_moe_lists(const int32_t* sel, int nk, int E, int32_t* offsets, int32_t* assign,
                            int32_t* scratch, hipStream_t st) {
  if (nk == 0) return hipSuccess;
  if (nk > kOneLaunchEntries)
    return launch_moe_plan(sel, nk, E, offsets, assign, st, nullptr, 256, scratch);
  if (nk <= 2048)
    hipLaunchKernelGGL(moe_lists_kernel<256>, dim3(E), dim3(256), 0, st, sel, nk, E, offsets, assign);
  else
    hipLaunchKernelGGL(moe_lists_kernel<1024>, dim3(E), dim3(1024), 0, st, sel, nk, E, offsets, assign);
  return hipGetLastError();
}

}  // namespace sevo
