// Routing of tokens to experts from router logits: softmax or sigmoid scores, a
// balance bias that acts on the choice alone, groups of experts of which the
// best are kept, the top-k of what is left, and weights from the unbiased
// scores.  Scores are defined and compared in float64: a choice turns on the
// difference of two of them, and near-equal sigmoids of large logits are equal in
// fp32.  Ties go to the lower group and the lower expert index.
//
// Sixteen lanes (a DPP row) per token.  32-bit keys choose the top_k + 2 best; their
// scores are then formed in float64, and these decide the choice and its order.
// The proof that no other expert belongs in it: the last one chosen is further
// above the best one not looked at than fp32 scores can be off; likewise the last
// group kept above the first left out.  A token without that proof, or with a
// NaN or an infinity in the way, runs again in float64 throughout.
//
// Nothing is bound by memory here (8192 x 256 logits are 8 MiB, 2 us): a wave is a
// chain of about a thousand instructions that run once, its reductions waiting for
// each other.  So four tokens share a wave, reductions stay in a DPP row and the
// float64 path is entered by few: one token in 4000 of the grouped case below, which
// is why its length still shows there (of 8192 tokens two, 3 us).  In a graph, times
// with the launch (3.4 us): 8192 tokens, 256 experts, sigmoid, bias, 4 of 8 groups, top
// 8: 15.5 us (float64 throughout: 24); 8192 x 128 softmax: 7.3 (19); 64 x 128: 6.0 (16).
#include "common.h"
#include "kernels.h"

namespace sevo {

namespace {

constexpr int kMaxExperts = 256;
constexpr int kPerLane = kMaxExperts / 64;

template <int J>
__device__ __forceinline__ double lane_xor_f64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = lane_xor<J>((uint32_t)u), hi = lane_xor<J>((uint32_t)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double row_sum_f64(double v) {
  v += lane_xor_f64<1>(v);
  v += lane_xor_f64<2>(v);
  v += lane_xor_f64<4>(v);
  return v + lane_xor_f64<8>(v);
}

// Order-preserving keys of doubles that are not NaN; kNanKey is below every one, and 0
// below that
constexpr uint64_t kNanKey = 1;
__device__ __forceinline__ uint64_t key_f64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return u ^ ((uint64_t)((int64_t)u >> 63) | 1ull << 63);
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = max(v, lane_xor<1>(v));
  v = max(v, lane_xor<2>(v));
  v = max(v, lane_xor<4>(v));
  v = max(v, lane_xor<8>(v));
  v = max(v, lane_xor<16>(v));
  return max(v, lane_xor<32>(v));
}
// the index that goes with the wave's largest key, of equal keys the lowest index.
// The high words nearly always decide.
__device__ __forceinline__ int wave_best(uint64_t key, int index) {
  const uint32_t hi = (uint32_t)(key >> 32);
  uint64_t who = __ballot(hi == wave_max_u32(hi));
  if (who & (who - 1)) {  // uniform
    const uint32_t lo = (who >> (threadIdx.x & 63)) & 1 ? (uint32_t)key : 0u;
    who &= __ballot(lo == wave_max_u32(lo));
    if (who & (who - 1))
      return (int)~wave_max_u32((who >> (threadIdx.x & 63)) & 1 ? ~(uint32_t)index : 0u);
  }
  return __builtin_amdgcn_readlane(index, __builtin_ctzll(who));
}

// One token in float64 throughout, by a wave; lane l holds experts l + 64 i.
// s: its own LDS, scores then choice values
__device__ __forceinline__ void route_f64(const MoeRouteArgs& a, int t, double (*s)[kMaxExperts]) {
  const int lane = threadIdx.x & 63;
  const float* lg = a.logits + (size_t)t * a.ld;
  float x[kPerLane], bias[kPerLane];
  float mx = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    const int e = min(lane + 64 * i, a.n_experts - 1);
    x[i] = lg[e];
    bias[i] = a.bias ? a.bias[e] : 0.f;
    mx = fmaxf(mx, x[i]);
    nan |= x[i] != x[i];
  }
  mx = wave_max(mx);
  if (!a.sigmoid && __ballot(nan)) mx = NAN;  // a softmax with a NaN is one throughout
  double p[kPerLane], sum = 0.0;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    p[i] = exp(a.sigmoid ? -(double)x[i] : (double)x[i] - (double)mx);
    if (lane + 64 * i < a.n_experts) sum += p[i];
  }
  sum = row_sum_f64(sum);
  sum += lane_xor_f64<16>(sum);
  sum += lane_xor_f64<32>(sum);
  uint64_t key[kPerLane];  // of the choice values; 0: not to be chosen
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    const int e = lane + 64 * i;
    p[i] = (a.sigmoid ? 1.0 : p[i]) / (a.sigmoid ? 1.0 + p[i] : sum);
    const double v = a.bias ? p[i] + (double)bias[i] : p[i];
    // a NaN is chosen after everything else, -inf too, and adds -inf to its group
    key[i] = e >= a.n_experts ? 0 : v == v ? key_f64(v) : kNanKey;
    s[0][e] = p[i];
    s[1][e] = v == v ? v : -INFINITY;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (a.top_groups < a.n_groups) {
    const int each = a.n_experts / a.n_groups;
    // lane g: the sum of group g's one or two best
    uint64_t g = 0;
    if (lane < a.n_groups) {
      double b0 = -INFINITY, b1 = -INFINITY;
#pragma unroll 8
      for (int i = 0; i < each; ++i) {
        const double v = s[1][lane * each + i];
        b1 = fmax(b1, fmin(b0, v));
        b0 = fmax(b0, v);
      }
      const double sum2 = a.group_best == 2 ? b0 + b1 : b0;
      g = sum2 == sum2 ? key_f64(sum2) : kNanKey;  // (+inf and -inf biases in one group)
    }
    uint64_t kept = 0;
#pragma unroll 1
    for (int r = 0; r < a.top_groups; ++r) {
      const int best = wave_best(g, lane);
      kept |= 1ull << best;
      if (lane == best) g = 0;
    }
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      if (!((kept >> (min(lane + 64 * i, a.n_experts - 1) / each)) & 1)) key[i] = 0;
  }
  double wt = 0.0;  // lane r: the score of choice r
  int ex = 0;
#pragma unroll 1
  for (int r = 0; r < a.top_k; ++r) {
    uint64_t k = key[0];
    int at = 0;
#pragma unroll
    for (int i = 1; i < kPerLane; ++i)
      if (key[i] > k) {
        k = key[i];
        at = i;
      }
    const int best = wave_best(k, lane + 64 * at);
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      if (lane + 64 * i == best) key[i] = 0;
    if (lane == r) ex = best;
  }
  if (lane < a.top_k) wt = s[0][ex];
  if (a.renormalise) wt /= row_sum_f64(wt) + 1e-20;  // (top_k is at most 16)
  if (lane < a.top_k) {
    a.out_experts[(size_t)t * a.top_k + lane] = ex;
    a.out_weights[(size_t)t * a.top_k + lane] = (float)(wt * (double)a.scaling);
  }
}

// The two largest of (a0 >= a1) and lane ^ J's pair, in both lanes
template <int J>
__device__ __forceinline__ void top2_xor(float& a0, float& a1) {
  const float o0 = lane_xor<J>(a0), o1 = lane_xor<J>(a1);
  a1 = fmaxf(fminf(a0, o0), fmaxf(a1, o1));
  a0 = fmaxf(a0, o0);
}

// over the 16 lanes of a row, every lane gets the result
template <typename T, typename F>
__device__ __forceinline__ T row_reduce(T v, F f) {
  v = f(v, lane_xor<1>(v));
  v = f(v, lane_xor<2>(v));
  v = f(v, lane_xor<4>(v));
  return f(v, lane_xor<8>(v));
}

// Order-preserving keys of floats, their low four bits the expert's place in its
// lane (the lower one larger): no two of a lane are equal.  0 is below every key.
__device__ __forceinline__ uint32_t key_of(float v, int j) {
  const uint32_t u = __float_as_uint(v);
  return ((u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) & ~15u) | (uint32_t)(15 - j);
}
__device__ __forceinline__ float value_of(uint32_t k) {
  k &= ~15u;
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// How far apart two fp32 values must be for their float64 ones to stand the same
// way.  exp(x) is off by 3 |x| 2^-24 relative (the difference, the factor log2 e and
// its product), the sum of a softmax, the reciprocal and the products by 5e-7.
// Without a bias that is relative: two scores at |x| under 25 by 1e-5 together, and
// under e^-25 by less than 1e-15.  With one, |x| e^-|x| < 0.4 bounds it absolutely:
// 6e-7 for each score, and the bias's sum rounds by 2^-24 of itself.  A group's sum of
// two is off by both of its members' errors and 2^-24 of itself: as its members can
// cancel (a large bias of either sign), by 1.2e-6 and 2^-23 of their magnitudes.
// A key adds 2^-19 of its value.
struct Apart {
  float off, key_off, base;
  __device__ __forceinline__ explicit Apart(bool bias)
      : off(bias ? 1.5e-6f : 5e-6f), key_off(bias ? 6e-6f : 1.3e-5f), base(bias ? 1.f : 1e-10f) {}
  // how far a group's value can be off, its members' magnitudes adding to mag
  __device__ __forceinline__ float group(float mag) const { return off * (base + mag); }
  __device__ __forceinline__ bool key(float a, float b) const { return a - b > key_off * (base + fabsf(a)); }
};

// rank of lane l's candidate (v, then lower e) among the 16 of its row: how many
// stand before it
template <int O>
__device__ __forceinline__ void rank_ror(double v, int e, int& rank) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  constexpr int kRor = 0x120 + O;  // row_ror: O
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, kRor, 0xF, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), kRor, 0xF, 0xF, false);
  const int oe = __builtin_amdgcn_update_dpp(0, e, kRor, 0xF, 0xF, false);
  const double o = __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  rank += o > v || (o == v && oe < e);
  if constexpr (O < 15) rank_ror<O + 1>(v, e, rank);
}

}  // namespace

// np experts per lane: lane l of a row holds experts np l .. + np - 1 (np at most P,
// 16 np at least n_experts).  fast 0: float64 throughout; else, where groups are
// left out, 16 np equals n_experts and n_groups divides 16.
template <int P>
__global__ __launch_bounds__(256) void moe_route8_kernel(MoeRouteArgs a, int np, int fast) {
  __shared__ double scratch[4][2][kMaxExperts];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, row = lane >> 4;
  const int t0 = (blockIdx.x * 4 + wave) * 4;  // the wave's first token
  if (t0 >= a.n) return;                       // (waves work alone: no barrier)
  const int tokens = min(4, a.n - t0);
  uint64_t bad_lanes = ~0ull;
  if (fast) {  // uniform
    const Apart apart(a.bias != nullptr);
    const int tr = min(row, tokens - 1);       // past the end: the last one again, not stored
    const int e0 = np * l16, eb = min(e0, a.n_experts - np);  // this lane's: eb + j, from e0 on
    auto rsrc = [](const void* p, int bytes) {
      return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
    };
    const float* lg = a.logits + (size_t)t0 * a.ld;
    const auto lr = rsrc(lg, ((tokens - 1) * (int)a.ld + a.n_experts) * 4);
    const int voff = (tr * (int)a.ld + eb) * 4;
    float c[P], b[P];
#pragma unroll
    for (int j = 0; j < P; ++j)
      c[j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(lr, voff + 4 * j, 0, 0));
    if (a.bias) {
      const auto br = rsrc(a.bias, a.n_experts * 4);
#pragma unroll
      for (int j = 0; j < P; ++j)
        b[j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(br, (eb + j) * 4, 0, 0));
    }
    float mx = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      c[j] = j < np && eb + j >= e0 ? c[j] : -INFINITY;
      bad |= c[j] != c[j];
      mx = fmaxf(mx, c[j]);
    }
    mx = row_reduce(mx, [](float x, float y) { return fmaxf(x, y); });
    bad |= !(fabsf(mx) < 1e30f);
    // without bias and groups the choice is by logit: scores rise with them
    const bool by_logit = a.bias == nullptr && a.top_groups == a.n_groups;
    float sum32 = 1.f;
    if (!a.sigmoid) {
      sum32 = 0.f;
#pragma unroll
      for (int j = 0; j < P; ++j) sum32 += __expf(c[j] - mx);
      sum32 = row_reduce(sum32, [](float x, float y) { return x + y; });
    }
    if (!by_logit) {
      const float scale = __builtin_amdgcn_rcpf(sum32);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const float x = __expf(a.sigmoid ? -c[j] : c[j] - mx);
        const float p = a.sigmoid ? __builtin_amdgcn_rcpf(1.f + x) : x * scale;
        c[j] = j < np && eb + j >= e0 ? (a.bias ? p + b[j] : p) : -INFINITY;
        bad |= c[j] != c[j];
      }
    }
    if (a.top_groups < a.n_groups) {
      const int seg = 16 / a.n_groups;  // lanes of a group: a power of two from 1 to 8
      float a0 = -INFINITY, a1 = -INFINITY;
#pragma unroll
      for (int j = 0; j < P; ++j) {
        a1 = fmaxf(a1, fminf(a0, c[j]));
        a0 = fmaxf(a0, c[j]);
      }
      if (seg > 1) top2_xor<1>(a0, a1);
      if (seg > 2) top2_xor<2>(a0, a1);
      if (seg > 4) top2_xor<4>(a0, a1);
      const float g = a.group_best == 2 ? a0 + a1 : a0;
      // a group's rank: how many are as large or larger
      int larger = 0;
      for (int o = seg; o < 16; o += seg)
        larger += __shfl(g, (lane & 48) | ((l16 + o) & 15), kWave) >= g;
      bad |= larger < a.top_groups && !(fabsf(g) < 1e30f);
      // the least that a group kept can be against the most that one left out can
      const float err = apart.group(fabsf(a0) + (a.group_best == 2 ? fabsf(a1) : 0.f));
      const float least = row_reduce(larger < a.top_groups ? g - err : INFINITY,
                                     [](float x, float y) { return fminf(x, y); });
      const float most = row_reduce(larger >= a.top_groups && g > -INFINITY ? g + err : -INFINITY,
                                    [](float x, float y) { return fmaxf(x, y); });
      bad |= !(least > most);
      // fewer kept than asked for: equal values stood at the border
      const uint64_t kept = __ballot(larger < a.top_groups && (l16 & (seg - 1)) == 0);
      bad |= __popc((uint32_t)(kept >> (lane & 48)) & 0xFFFFu) != a.top_groups;
#pragma unroll
      for (int j = 0; j < P; ++j) c[j] = larger >= a.top_groups ? -INFINITY : c[j];
    }
    uint32_t key[P];
#pragma unroll
    for (int j = 0; j < P; ++j) key[j] = j < np ? key_of(c[j], j) : 0u;
    // lane r of a row: candidate r, r < top_k + 2
    const int cand = min(a.top_k + 2, 16);
    int ex = -1;
    uint32_t ex_key = 0, best = 0;
    for (int r = 0; r <= cand; ++r) {
      uint32_t m = key[0];
#pragma unroll
      for (int j = 1; j < P; ++j) m = max(m, key[j]);
      best = row_reduce(m, [](uint32_t x, uint32_t y) { return max(x, y); });
      if (r == cand) break;  // the best one not looked at
      const uint32_t who = (uint32_t)(__ballot(m == best) >> (lane & 48)) & 0xFFFFu;
      bad |= (who & (who - 1)) != 0 && best != 0;  // two lanes with the same key
      if (l16 == r && best != 0) {
        const int owner = __ffs(who) - 1;
        ex = min(np * owner, a.n_experts - np) + 15 - (int)(best & 15u);
        ex_key = best;
      }
#pragma unroll
      for (int j = 0; j < P; ++j) key[j] = key[j] == best ? 0u : key[j];
    }
    // the candidates' float64 scores and choice values
    const float v32 = value_of(ex_key);
    const bool is = ex >= 0 && v32 > -INFINITY;
    double p = 0.0, v = -INFINITY;
    double x = 0.0;
    if (is) {
      x = (double)__uint_as_float(
          __builtin_amdgcn_raw_buffer_load_b32(lr, (tr * (int)a.ld + ex) * 4, 0, 0));
      p = exp(a.sigmoid ? -x : x - (double)mx);
      if (a.sigmoid) p = 1.0 / (1.0 + p);
    }
    double sum = 1.0;
    if (!a.sigmoid) {
      // The softmax's sum.  It scales all scores alike: in fp32 it will do for the
      // choice without a bias, and renormalised weights do not see it either (but
      // for the 1e-20).
      sum = (double)sum32;
      if (!a.renormalise || a.bias) {
        sum = 0.0;
#pragma unroll 1
        for (int j = 0; j < np; ++j)
          if (eb + j >= e0)
            sum += exp((double)__uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(lr, voff + 4 * j, 0, 0)) -
                       (double)mx);
        sum = row_sum_f64(sum);
      }
      p /= sum;
    }
    if (is) v = a.bias ? p + (double)a.bias[ex] : p;
    int rank = 0;
    rank_ror<1>(v, is ? ex : 0x7FFFFFFF, rank);
    // the last one chosen against the best one not looked at
    if (rank == a.top_k - 1) {
      const float rest = value_of(best);
      if (by_logit) {
        // further apart in the logits than their scores' float64 can confuse
        bad |= !is || (best != 0 && !((float)x - rest > 6e-6f * (1.f + fabsf((float)x)))) || (a.sigmoid && x > 16.0) ||
               x - (a.sigmoid ? 0.0 : (double)mx) < -600.0;
      } else {
        bad |= !is || (best != 0 && !apart.key((float)v, rest));
      }
      bad |= !(fabs(v) < 1e30);
    }
    double wt = rank < a.top_k ? p : 0.0;
    if (a.renormalise) {
      const double s = row_sum_f64(wt);
      bad |= !(s > 1e-10);
      wt /= s + 1e-20;
    }
    bad_lanes = __ballot(bad);
    if (is && rank < a.top_k && row < tokens && !(bad_lanes >> (lane & 48) & 0xFFFFu)) {
      const size_t o = (size_t)(t0 + row) * a.top_k + rank;
      a.out_experts[o] = ex;
      a.out_weights[o] = (float)(wt * (double)a.scaling);
    }
  }
#pragma unroll 1
  for (int i = 0; i < tokens; ++i)
    if (bad_lanes >> (16 * i) & 0xFFFFu) route_f64(a, t0 + i, scratch[wave]);
}

hipError_t launch_moe_route8(const MoeRouteArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  const int np = (a.n_experts + 15) / 16;
  // groups that are not whole runs of lanes, or rows too far apart for the
  // offsets of four: float64 throughout
  const int fast = (a.top_groups == a.n_groups ||
                    (a.n_experts == 16 * np && a.n_groups <= 16 && 16 % a.n_groups == 0)) &&
                   a.ld < 1 << 26;
  const dim3 grid((a.n + 15) / 16);
  if (np <= 4) hipLaunchKernelGGL(moe_route8_kernel<4>, grid, dim3(256), 0, st, a, np, fast);
  else if (np <= 8) hipLaunchKernelGGL(moe_route8_kernel<8>, grid, dim3(256), 0, st, a, np, fast);
  else hipLaunchKernelGGL(moe_route8_kernel<16>, grid, dim3(256), 0, st, a, np, fast);
  return hipGetLastError();
}

// Entry lists in one launch: workgroup e reads every entry once and counts those of
// lower experts (its list's first place) and its own; its own then go out in order.
// Workgroup E does the same for the entries without an expert, behind the lists.  A
// wave holds 512 C consecutive entries in registers, a lane eight of each 512, and an
// entry's rank is the matches of the waves, chunks and lanes before it: one barrier,
// no sums between workgroups, and nothing depends on scheduling.
template <int T, int C>
__global__ __launch_bounds__(T) void moe_lists_kernel(const int32_t* __restrict__ sel, int nk, int E,
                                                      int32_t* __restrict__ offsets,
                                                      int32_t* __restrict__ assign) {
  constexpr int W = T / 64, P = 8;  // entries of a lane and chunk
  __shared__ int red[2][W];
  const int e = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i0 = wave * 512 * C + P * lane;
  int v[C][P];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int i = i0 + 512 * c;
    if (i + P <= nk) {
      *reinterpret_cast<u32x4*>(&v[c][0]) = *reinterpret_cast<const u32x4*>(sel + i);
      *reinterpret_cast<u32x4*>(&v[c][4]) = *reinterpret_cast<const u32x4*>(sel + i + 4);
    } else {
#pragma unroll
      for (int j = 0; j < P; ++j) v[c][j] = i + j < nk ? sel[i + j] : -1;
    }
  }
  if (e == E) {  // uniform
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < P; ++j)
        if ((uint32_t)v[c][j] >= (uint32_t)E && i0 + 512 * c + j < nk) v[c][j] = E;
  }
  int lower = 0, own = 0;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int j = 0; j < P; ++j) {
      lower += (uint32_t)v[c][j] < (uint32_t)e;  // (a negative id is in no list)
      own += v[c][j] == e;
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
  int first = 0, at = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w < wave) at += red[1][w];
    first += red[0][w];
  }
  if (threadIdx.x == 0) offsets[e] = first;
  at += first;
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    int rank = at, total = 0;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint64_t b = __ballot(v[c][j] == e);
      rank += __popcll(b & below);
      total += __popcll(b);
    }
    if (total == 0) continue;  // uniform over the wave
#pragma unroll
    for (int j = 0; j < P; ++j)
      if (v[c][j] == e) assign[rank++] = i0 + 512 * c + j;
    at += total;
  }
}

// From this many entries on, reading all of them in every workgroup costs more
// than the launches that count, scan and place.
constexpr int kOneLaunchEntries = 65536;

hipError_t launch_moe_lists(const int32_t* sel, int nk, int E, int32_t* offsets, int32_t* assign,
                            int32_t* scratch, hipStream_t st) {
  if (nk == 0) return hipSuccess;
  if (nk > kOneLaunchEntries) {
    if (hipError_t e = launch_moe_plan(sel, nk, E, offsets, assign, st, nullptr, 256, scratch); e != hipSuccess)
      return e;
    return launch_moe_plan_rest(sel, nk, E, offsets, assign, scratch, st);
  }
  auto go = [&](auto kern, int threads) {
    hipLaunchKernelGGL(kern, dim3(E + 1), dim3(threads), 0, st, sel, nk, E, offsets, assign);
  };
  if (nk <= 2048) go(moe_lists_kernel<256, 1>, 256);
  else if (nk <= 8192) go(moe_lists_kernel<1024, 1>, 1024);
  else if (nk <= 32768) go(moe_lists_kernel<1024, 4>, 1024);
  else go(moe_lists_kernel<1024, 8>, 1024);
  return hipGetLastError();
}

}  // namespace sevo
