// Verification of drafted tokens (speculative sampling).  With p_t = softmax(target logits of
// position t / T) and q_t the distribution that draft x_t was drawn from:
//   x_t is accepted while u_t q_t(x_t) < p_t(x_t);
//   the token after the accepted ones: at a rejection from max(p_t - q_t, 0), normalised, else from
//   the row behind the last draft; drawn by the inverse distribution function in index order
//   with the candidate's last uniform number.
// What is emitted is distributed as the target's own samples.
//
// A choice is a comparison of sums over the whole vocabulary: one entry of 150 thousand differs
// from its neighbour by 1e-6 of the mass and less, so a sum in 32 bits would move
// choices.  Exponentials and sums are in 64 bits throughout (an entry x nats below its row's largest is off by
// (4 x + 6) 1e-16 of itself at most, that is 6e-16 of the largest: log2 e / T and its product are rounded).
// Three kernels (us: 64 candidates with 4 drafts and their distributions, 151936 entries, 350 MB):
//   1. per (row, 2048 entries): the largest logit and the sum of exponentials relative to it (57
//      to 64; 51 are the floor of its reads: the vector ALU, 14 operations an entry and 5 for the
//      chunk's sums, is busy most of the time);
//   2. (a draft distribution given) per (candidate, 2048 entries): the sum of max(p - q, 0) of the
//      row where the candidate's drafts end (20 to 24: 5 to find it, then the vector ALU, 2
//      exponentials an entry);
//   3. per candidate: the chunk that holds the drawn point, and in it the entry (7: a chain of
//      loads and scans).
// Kernel 2, or 3 where there is none, finds the number of accepted drafts from 1's sums, each workgroup
// for its candidate: a kernel of its own for it would cost a launch more.
#include "common.h"
#include "kernels.h"

namespace sevo {

namespace {

constexpr int kPer = kVerifyChunk / 256;  // entries of a thread

// 2^x in 64 bits: x = n + f, |f| <= 1/2, a degree-10 polynomial through the Chebyshev
// nodes of [-1/2, 1/2] (3e-16 relative), scaled by 2^n.  -inf and anything below -2000 give 0, NaN
// gives NaN.
__device__ __forceinline__ double exp2d(double x) {
  x = x < -2000.0 ? -2000.0 : x;
  const double n = __builtin_rint(x);
  const double f = x - n;
  double y = 7.072585949269223e-09;
  y = __builtin_fma(y, f, 1.0208690299958306e-07);
  y = __builtin_fma(y, f, 1.321544258792169e-06);
  y = __builtin_fma(y, f, 1.5252657260200837e-05);
  y = __builtin_fma(y, f, 0.0001540353044173605);
  y = __builtin_fma(y, f, 0.0013333558230164974);
  y = __builtin_fma(y, f, 0.009618129107606888);
  y = __builtin_fma(y, f, 0.05550410866444772);
  y = __builtin_fma(y, f, 0.24022650695910097);
  y = __builtin_fma(y, f, 0.69314718055995);
  y = __builtin_fma(y, f, 1.0);
  // (n of a NaN is not converted)
  return __builtin_amdgcn_ldexp(y, x == x ? (int)n : 0);
}

// the two words of a double through a lane permutation in registers
template <typename F>
__device__ __forceinline__ double by_words(double v, F&& f) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)f((uint32_t)b) | ((uint64_t)f((uint32_t)(b >> 32)) << 32));
}
template <int J>
__device__ __forceinline__ double lane_xor64(double v) {
  return by_words(v, [](uint32_t x) { return lane_xor<J>(x); });
}
__device__ __forceinline__ double row16_sum64(double v) {
  v += lane_xor64<1>(v);
  v += lane_xor64<2>(v);
  v += lane_xor64<4>(v);
  return v + lane_xor64<8>(v);
}
__device__ __forceinline__ double wave_sum64(double v) {
  v = row16_sum64(v);
  v += lane_xor64<16>(v);
  return v + lane_xor64<32>(v);
}
// lanes without a source get 0
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp64(double v) {
  return by_words(v, [](uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
  });
}
__device__ __forceinline__ double wave_scan64(double v) {  // inclusive
  v += dpp64<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
  v += dpp64<0x112, 0xF>(v);
  v += dpp64<0x114, 0xF>(v);
  v += dpp64<0x118, 0xF>(v);
  v += dpp64<0x142, 0xA>(v);  // row_bcast 15 into rows 1, 3
  return v + dpp64<0x143, 0xC>(v);  // row_bcast 31 into rows 2, 3
}
// the value of lane l, the same for all
__device__ __forceinline__ double lane64(double v, int l) {
  return by_words(v, [l](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); });
}

// entries v .. v + 3 of a row, -inf at and past vocab (nothing is read there)
__device__ __forceinline__ f32x4 row4(const float* row, int v, int vocab) {
  if (v + 4 <= vocab) return *reinterpret_cast<const f32x4*>(row + v);
  f32x4 r{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (v + k < vocab) r[k] = row[v + k];
  return r;
}

__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int i) {
  const int m = a.n_drafts ? a.n_drafts[i] : a.drafts;
  return m < 0 ? 0 : (m > a.drafts ? a.drafts : m);
}

// target rows first, [n][drafts + 1], then the draft rows, [n][drafts]
__device__ __forceinline__ size_t target_row(const VerifyArgs& a, int i, int t) {
  return (size_t)i * (a.drafts + 1) + t;
}
__device__ __forceinline__ size_t draft_row(const VerifyArgs& a, int i, int t) {
  return (size_t)a.n * (a.drafts + 1) + (size_t)i * a.drafts + t;
}
__device__ __forceinline__ const float* row_ptr(const VerifyArgs& a, size_t row) {
  const size_t targets = (size_t)a.n * (a.drafts + 1);
  return row < targets ? a.logits + row * a.ld : a.draft_logits + (row - targets) * a.ld_draft;
}

__device__ __forceinline__ double log2_scale(const VerifyArgs& a) {
  return 1.4426950408889634074 / (a.temp == 0.0 ? 1.0 : a.temp);
}


// The sums' exponential, factor * 2^(d c): factor * 2^(k / 256) from a table in LDS, times a degree-4
// polynomial on [-1/512, 1/512] (5e-18 relative), scaled by 2^n in the table entry's exponent.
// 256 entries make the index one instruction (a byte's shift): 64 candidates 97 -> 95 us.
// d at most 0; what is more than 2^reach below 1, also a -inf (and a NaN), is taken for 2^-reach
// (factor 2^-reach has to be a normal number).
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
struct Exp2Steps {  // 2^(j / 256), from exp's series
  double v[256];
  constexpr Exp2Steps() : v() {
    for (int j = 0; j < 256; ++j) {
      const double x = j * (0.69314718055994530942 / 256);
      double y = 1.0;
      for (int n = 20; n > 0; --n) y = 1.0 + y * x / n;
      v[j] = y;
    }
  }
};
__device__ const Exp2Steps kExp2Steps{};
struct ExpTable {
  u32x2 t[256];  // the exponent of entry j less j / 256: adding k / 256 to it gives n
};
__device__ __forceinline__ void make_table(ExpTable& T, double step, double factor) {
  u32x2 b = __builtin_bit_cast(u32x2, factor * step);
  b.y -= threadIdx.x << 12;
  T.t[threadIdx.x] = b;
}
struct ExpScale {
  double c256, least;
  __device__ __forceinline__ ExpScale(double c, double reach) : c256(256.0 * c), least(-reach / c) {}
};
__device__ __forceinline__ void exp_parts(const ExpTable& T, const ExpScale& E, double d, double& poly,
                                          double& entry) {
  const double magic = 6755399441055744.0;  // 1.5 2^52: the sum's low bits are d c256 rounded
  d = __builtin_fmax(d, E.least);
  const double t = __builtin_fma(d, E.c256, magic);
  const int k = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
  const double r = __builtin_fma(d, E.c256, magic - t);
  u32x2 b = T.t[(uint8_t)k];
  double y = 2.239395329901621e-12;
  y = __builtin_fma(y, r, 3.30830298371135e-09);
  y = __builtin_fma(y, r, 3.665565596910101e-06);
  y = __builtin_fma(y, r, 0.0027076061740622767);
  poly = __builtin_fma(y, r, 1.0);
  b.y += (uint32_t)k << 12;
  entry = __builtin_bit_cast(double, b);
}

// max(p - q, 0) of an entry, dz and dy its logits less their rows' largest, P and Q tables with the factors
// kShareUnit / the rows' sums.  Times 2^120 every share that float64 holds (2^-1074 and more of the mass, as a
// subnormal number) is a normal number, and what stands for less (2^-980 and below, kShareReach) is told from it:
// up to kNoShare, half the least share, nothing is left.  A -inf or a mask of the lowest number thus weighs
// nothing, in both kernels alike: the second sums what the third walks through, so a chunk
// with a sum has an entry with a weight.
constexpr double kShareUnit = 0x1p120, kShareReach = 1100.0, kNoShare = 0x1p-955;
__device__ __forceinline__ double share_left(const ExpTable& P, const ExpTable& Q, const ExpScale& E,
                                             double dz, double dy) {
  // no multiply-add into the difference: of equal rows nothing is left
#pragma clang fp contract(off)
  double pp, pe, qp, qe;
  exp_parts(P, E, dz, pp, pe);
  exp_parts(Q, E, dy, qp, qe);
  return pp * pe - qp * qe;
}

}  // namespace

// A wave per (row, 2048 entries), 32 a lane in registers from one read: no barrier but the
// table's, so that some waves' loads are in flight while others compute.
__global__ __launch_bounds__(256, 6) void verify_rows_kernel(VerifyArgs a) {
  __shared__ ExpTable T;
  constexpr int J = kVerifyChunk / 256;
  const int lane = threadIdx.x & 63;
  const unsigned job = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned row = job / a.chunks;
  const int chunk = job - row * a.chunks;
  const unsigned targets = a.n * (a.drafts + 1);
  // rows behind a candidate's last draft are not read, nor is anything past the last row
  bool on = row < targets + (a.draft_logits && a.temp != 0.0 ? a.n * a.drafts : 0);
  if (on) {
    const unsigned own = row < targets ? row : row - targets;
    const unsigned each = row < targets ? a.drafts + 1 : a.drafts;
    const int i = (int)(own / each);
    on = (int)(own - i * each) < drafts_of(a, i) + (row < targets ? 1 : 0);
  }
  const double step = kExp2Steps.v[threadIdx.x];
  f32x4 z[J];
  if (on) {
    const float* r = row_ptr(a, row);
    const int v0 = chunk * kVerifyChunk + lane * 4;
    if ((chunk + 1) * kVerifyChunk <= a.vocab) {
#pragma unroll
      for (int j = 0; j < J; ++j)
        z[j] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(r + v0 + 256 * j));
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) z[j] = row4(r, v0 + 256 * j, a.vocab);
    }
  }
  make_table(T, step, 1.0);
  __syncthreads();
  if (!on) return;
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < J; ++j) m = fmaxf(fmaxf(fmaxf(m, z[j].x), fmaxf(z[j].y, z[j].z)), z[j].w);
  m = wave_max(m);
  const ExpScale E(log2_scale(a), 900.0);
  const double md = m;
  double sum = 0.0;
  bool none = m == INFINITY;  // a NaN or a +inf: no distribution
#pragma unroll
  for (int j = 0; j < J; ++j) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      double y, e;
      exp_parts(T, E, (double)z[j][k] - md, y, e);
      sum = __builtin_fma(y, e, sum);
    }
    none |= __builtin_isunordered(z[j].x, z[j].y) | __builtin_isunordered(z[j].z, z[j].w);
    __builtin_amdgcn_sched_barrier(0);  // (four at a time: all at once take twice the registers)
  }
  if (m == -INFINITY) sum = 0.0;
  if (none) sum = NAN;
  sum = wave_sum64(sum);
  int arg = 0x7FFFFFFF;
  if (a.temp == 0.0) {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (z[j][k] == m) arg = min(arg, chunk * kVerifyChunk + lane * 4 + 256 * j + k);
    arg = wave_min(arg);
  }
  if (lane == 0) a.parts[(size_t)row * a.chunks + chunk] = VerifyPart{sum, m, arg};
}

namespace {

// a row's largest logit, its sum of exponentials, its first largest entry
using RowSum = VerifyPart;
struct Decision {
  int taken, count;
};
using VerifyLds = VerifyDecided;

// over the 16 lanes of a row of the wave, every lane gets it
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, lane_xor<1>(v));
  v = fmaxf(v, lane_xor<2>(v));
  v = fmaxf(v, lane_xor<4>(v));
  return fmaxf(v, lane_xor<8>(v));
}

// 16 lanes: the row's partials joined, every lane gets the result
constexpr int kPartsAhead = 5;  // partials of a lane in flight: 80 chunks, 163840 entries
__device__ __forceinline__ void load_parts(const VerifyArgs& a, size_t row, VerifyPart (&v)[kPartsAhead]) {
  const VerifyPart* p = a.parts + row * a.chunks;
#pragma unroll
  for (int u = 0; u < kPartsAhead; ++u) v[u] = p[min((int)(threadIdx.x & 15) + 16 * u, a.chunks - 1)];
}
__device__ __forceinline__ RowSum join_row(const VerifyArgs& a, size_t row,
                                           const VerifyPart (&v)[kPartsAhead]) {
  const int q = threadIdx.x & 15;
  const VerifyPart* p = a.parts + row * a.chunks;
  float m = -INFINITY;
#pragma unroll
  for (int u = 0; u < kPartsAhead; ++u) m = fmaxf(m, v[u].max);
  for (int k = q + 16 * kPartsAhead; k < a.chunks; k += 16) m = fmaxf(m, p[k].max);
  m = row16_max(m);
  const double mc = m == -INFINITY ? 0.0 : (double)m, c = log2_scale(a);
  double s = 0.0;
  int arg = 0x7FFFFFFF;
  auto add = [&](const VerifyPart& x) {
    s += x.sum * exp2d(((double)x.max - mc) * c);
    if (x.max == m) arg = min(arg, x.arg);
  };
#pragma unroll
  for (int u = 0; u < kPartsAhead; ++u)
    if (q + 16 * u < a.chunks) add(v[u]);
  for (int k = q + 16 * kPartsAhead; k < a.chunks; k += 16) add(p[k]);
  s = row16_sum64(s);
  arg = min(arg, lane_xor<1>(arg));
  arg = min(arg, lane_xor<2>(arg));
  arg = min(arg, lane_xor<4>(arg));
  arg = min(arg, lane_xor<8>(arg));
  return RowSum{s, m, arg};
}

// a sum that a distribution can have: not of a row with a NaN, a +inf or nothing above -inf
__device__ __forceinline__ bool fine(double s) { return s > 0.0 && s < INFINITY; }

// an entry's share of the row's largest one (c: log2_scale; no multiply-add, so that it is the same bits wherever
// it is computed)
__device__ __forceinline__ double share(float z, double largest, double c) {
#pragma clang fp contract(off)
  return exp2d(((double)z - largest) * c);
}
__device__ __forceinline__ double prob(const VerifyArgs& a, const RowSum& r, float z) {
  return share(z, r.max, log2_scale(a)) / r.sum;
}

// The sums of candidate i's rows into LDS, and how many drafts are accepted.  All threads: 16 lanes
// a row, so that a call with 4 drafts takes two memory latencies: the partials beside the count, the
// drafts and their uniform numbers; then the drafts' logits.
__device__ __forceinline__ Decision decide(const VerifyArgs& a, int i, VerifyLds& L) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const bool dist = a.draft_logits && a.temp != 0.0;
  const int rows = a.drafts + 1 + (dist ? a.drafts : 0);
  int x = -1;
  float u = 0.f;
  if (w == 0 && lane < a.drafts) {
    x = a.draft_tokens[(size_t)i * a.drafts + lane];
    u = a.uniforms[(size_t)i * (a.drafts + 1) + lane];
  }
  // (partials of rows behind the last draft are joined too, whatever they hold, and not looked at)
  const int count = drafts_of(a, i);
  auto row_of = [&](int r) {
    return r <= a.drafts ? target_row(a, i, r) : draft_row(a, i, r - a.drafts - 1);
  };
  int r = threadIdx.x >> 4;
  VerifyPart v[kPartsAhead];
  if (r < rows) load_parts(a, row_of(r), v);
  float zx = 0.f, yx = 0.f;
  // (rows behind the last draft may not be there)
  const bool known = lane < count && x >= 0 && x < a.vocab;
  if (known) {
    zx = row_ptr(a, target_row(a, i, lane))[x];
    if (dist) yx = row_ptr(a, draft_row(a, i, lane))[x];
  }
  for (; r < rows; r += 16) {
    if (r >= 16) load_parts(a, row_of(r), v);
    const RowSum s = join_row(a, row_of(r), v);
    if ((lane & 15) == 0) L.row[r <= a.drafts ? r : kVerifyMaxDrafts + r - a.drafts] = s;
  }
  __syncthreads();
  if (w == 0) {
    bool ok = true;
    if (lane < count) {
      const RowSum t = L.row[lane];
      ok = false;
      if (known && fine(t.sum))
        ok = a.temp == 0.0 ? x == t.arg
                           : (double)u * (dist ? prob(a, L.row[kVerifyMaxDrafts + 1 + lane], yx) : 1.0) <
                                 prob(a, t, zx);
    }
    const uint64_t bad = __builtin_amdgcn_ballot_w64(!ok);
    if (lane == 0) {
      L.taken = bad ? min(count, (int)__builtin_ctzll(bad)) : count;
      L.count = count;
    }
  }
  __syncthreads();
  return Decision{L.taken, count};
}

// The weights that the next token is drawn from, at entries v .. v + 3, where no draft distribution is
// taken off: p times the row's sum (the scale does not matter, and the sums of a flat row are exact), there
// with or without the rejected draft
struct Weights {
  const float* target;
  double mt, c;
  int without;  // -1: none
  int vocab;
  __device__ __forceinline__ void at(int v, double (&o)[4]) const {
    const f32x4 z = row4(target, v, vocab);
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = share(z[k], mt, c);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (v + k == without) o[k] = 0.0;
  }
};

__device__ __forceinline__ Weights weights(const VerifyArgs& a, int i, const Decision& d,
                                           const VerifyLds& L, bool residual) {
  Weights w;
  w.target = row_ptr(a, target_row(a, i, d.taken));
  w.mt = L.row[d.taken].max;
  w.c = log2_scale(a);
  w.without = residual ? a.draft_tokens[(size_t)i * a.drafts + d.taken] : -1;
  w.vocab = a.vocab;
  return w;
}

// and where it is: max(p - q, 0) of the row behind the accepted drafts
struct Residual {
  const float* target;
  const float* draft;
  double mt, md;
  ExpScale E;
  __device__ __forceinline__ Residual(const VerifyArgs& a, int i, const Decision& d, const VerifyLds& L)
      : target(row_ptr(a, target_row(a, i, d.taken))),
        draft(row_ptr(a, draft_row(a, i, d.taken))),
        mt(L.row[d.taken].max),
        md(L.row[kVerifyMaxDrafts + 1 + d.taken].max),
        E(log2_scale(a), kShareReach) {}
};

// sum of a chunk's weights over the workgroup, every thread gets it
__device__ __forceinline__ double chunk_sum(const Weights& W, int chunk, double* red) {
  double s = 0.0;
#pragma unroll
  for (int j = 0; j < kPer / 4; ++j) {
    double o[4];
    W.at(chunk * kVerifyChunk + threadIdx.x * 4 + 1024 * j, o);
    s += (o[0] + o[1]) + (o[2] + o[3]);
  }
  s = wave_sum64(s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

}  // namespace

// A workgroup per candidate and four chunks, a wave per chunk; the rows' 1 / sums are factors of the
// exponentials' tables.
__global__ __launch_bounds__(256, 4) void verify_rest_kernel(VerifyArgs a) {
  __shared__ VerifyLds L;
  __shared__ ExpTable P, Q;
  const int groups = (a.chunks + 3) / 4;
  const int i = blockIdx.x / groups;
  const int chunk = (blockIdx.x - i * groups) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const double step = kExp2Steps.v[threadIdx.x];
  const Decision d = decide(a, i, L);
  if (blockIdx.x == (unsigned)(i * groups)) {  // for the third kernel
    const uint32_t* from = reinterpret_cast<const uint32_t*>(&L);
    uint32_t* to = reinterpret_cast<uint32_t*>(a.decided + i);
    if (threadIdx.x < sizeof(VerifyLds) / 4) to[threadIdx.x] = from[threadIdx.x];
  }
  if (d.taken == d.count) return;
  const RowSum t = L.row[d.taken], q = L.row[kVerifyMaxDrafts + 1 + d.taken];
  if (!fine(t.sum) || !fine(q.sum)) {  // no difference of distributions
    if (chunk < a.chunks && (threadIdx.x & 63) == 0) a.rest_sum[(size_t)i * a.chunks + chunk] = 0.0;
    return;
  }
  const Residual R(a, i, d, L);
  const int v0 = chunk * kVerifyChunk + (threadIdx.x & 63) * 4;
  constexpr int J = kVerifyChunk / 256;
  f32x4 z[J], y[J];
  if ((chunk + 1) * kVerifyChunk <= a.vocab) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      z[j] = *reinterpret_cast<const f32x4*>(R.target + v0 + 256 * j);
      y[j] = *reinterpret_cast<const f32x4*>(R.draft + v0 + 256 * j);
    }
  } else {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      z[j] = row4(R.target, v0 + 256 * j, a.vocab);
      y[j] = row4(R.draft, v0 + 256 * j, a.vocab);
    }
  }
  make_table(P, step, kShareUnit / t.sum);
  make_table(Q, step, kShareUnit / q.sum);
  __syncthreads();
  if (chunk >= a.chunks) return;
  double s = 0.0;
#pragma unroll
  for (int j = 0; j < J; ++j) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      s += __builtin_fmax(share_left(P, Q, R.E, (double)z[j][k] - R.mt, (double)y[j][k] - R.md), kNoShare);
    __builtin_amdgcn_sched_barrier(0);
  }
  // (every entry added kNoShare at least; of entries that added no more exactly 0 is left)
  s = wave_sum64(s - 4 * J * kNoShare);
  if ((threadIdx.x & 63) == 0) a.rest_sum[(size_t)i * a.chunks + chunk] = s;
}

// DECIDED: the second kernel ran, and left what decide() finds
template <bool DECIDED>
__global__ __launch_bounds__(256) void verify_pick_kernel(VerifyArgs a) {
  __shared__ VerifyLds L;
  __shared__ double red[4], s_pre[4];
  __shared__ double s_total, s_target, s_before;
  __shared__ int s_chunk, s_tok;
  __shared__ ExpTable P, Q;
  const int i = blockIdx.x;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const double step = DECIDED ? kExp2Steps.v[threadIdx.x] : 0.0;
  const double point = a.uniforms[(size_t)i * (a.drafts + 1) + a.drafts];
  Decision d;
  if constexpr (DECIDED) {
    const uint32_t* from = reinterpret_cast<const uint32_t*>(a.decided + i);
    uint32_t* to = reinterpret_cast<uint32_t*>(&L);
    if (threadIdx.x < sizeof(VerifyLds) / 4) to[threadIdx.x] = from[threadIdx.x];
    __syncthreads();
    d = Decision{L.taken, L.count};
  } else {
    d = decide(a, i, L);
  }
  const RowSum row = L.row[d.taken];
  const bool valid = fine(row.sum);
  if (threadIdx.x == 0) s_tok = valid && a.temp == 0.0 ? row.arg : -1;
  if (valid && a.temp != 0.0) {  // the same in every thread
    bool residual = d.taken < d.count;
    Weights W = weights(a, i, d, L, residual && !DECIDED);
    if constexpr (DECIDED)
      if (residual) {  // (tables of a row that is no distribution are not used: the second kernel's sums are 0)
        make_table(P, step, kShareUnit / row.sum);
        make_table(Q, step, kShareUnit / L.row[kVerifyMaxDrafts + 1 + d.taken].sum);
      }
    const size_t prow = target_row(a, i, d.taken) * a.chunks;
    // the chunk without the rejected draft: summed again, a difference would lose the digits of what is left
    double left = 0.0;
    const int hole = W.without >= 0 && W.without < a.vocab ? W.without / kVerifyChunk : -1;
    if (hole >= 0) left = chunk_sum(W, hole, red);
    auto weight_of = [&](int k) -> double {
      if (DECIDED && residual) return a.rest_sum[(size_t)i * a.chunks + k];
      if (residual && k == hole) return left;
      const VerifyPart p = a.parts[prow + k];
      return p.sum * share(p.max, row.max, W.c);
    };
    for (int pass = 0;; ++pass) {
      // wave 0: total, then the first chunk whose running sum passes the drawn point
      if (w == 0) {
        const double first = lane < a.chunks ? weight_of(lane) : 0.0;
        double total = wave_sum64(first);
        for (int k0 = 64; k0 < a.chunks; k0 += 64)
          total += wave_sum64(k0 + lane < a.chunks ? weight_of(k0 + lane) : 0.0);
        const double target = point * total;
        int found = -1, last = -1;
        double before = 0.0, last_before = 0.0, run = 0.0;
        for (int k0 = 0; k0 < a.chunks && found < 0; k0 += 64) {
          const double x = k0 == 0 ? first : k0 + lane < a.chunks ? weight_of(k0 + lane) : 0.0;
          const double in = wave_scan64(x);
          const uint64_t over = __builtin_amdgcn_ballot_w64(x > 0.0 && run + in > target);
          const uint64_t some = __builtin_amdgcn_ballot_w64(x > 0.0);
          if (over) {
            const int l = __builtin_ctzll(over);
            found = k0 + l;
            before = run + lane64(in - x, l);
          }
          if (some) {
            const int l = 63 - __builtin_clzll(some);
            last = k0 + l;
            last_before = run + lane64(in - x, l);
          }
          run += lane64(in, 63);
        }
        // a point at the very end (a uniform number of 1, or rounding): the last entry
        if (found < 0) {
          found = last;
          before = last_before;
        }
        if (lane == 0) {
          s_total = total;
          s_target = target;
          s_chunk = found;
          s_before = before;
        }
      }
      __syncthreads();
      const bool good = s_total > 0.0 && s_total < INFINITY;
      if (good || !residual) break;
      // nothing left of the residual: the target's own distribution
      residual = false;
      W = weights(a, i, d, L, false);
      __syncthreads();
    }
    if (s_total > 0.0 && s_chunk >= 0) {
      // thread t: entries 16 t .. + 15 of the chunk, in index order
      const int v0 = s_chunk * kVerifyChunk + threadIdx.x * kPer;
      double o[kPer], own = 0.0;
#pragma unroll
      for (int j = 0; j < kPer / 4; ++j) {
        double q[4];
        if (DECIDED && residual) {
          const Residual R(a, i, d, L);
          const f32x4 z = row4(R.target, v0 + 4 * j, a.vocab), y = row4(R.draft, v0 + 4 * j, a.vocab);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const double r = share_left(P, Q, R.E, (double)z[k] - R.mt, (double)y[k] - R.md);
            q[k] = r > kNoShare ? r : 0.0;
          }
        } else {
          W.at(v0 + 4 * j, q);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          o[4 * j + k] = q[k];
          own += q[k];
        }
      }
      const double in = wave_scan64(own);
      if (lane == 63) s_pre[w] = in;
      __syncthreads();
      double run = s_before;
      for (int x = 0; x < w; ++x) run += s_pre[x];
      run += in - own;
      int tok = 0x7FFFFFFF, last = -1;
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        run += o[k];
        if (o[k] > 0.0) {
          last = v0 + k;
          if (run > s_target) tok = min(tok, v0 + k);
        }
      }
      // first entry past the point, or the chunk's last one with any weight
      tok = wave_min(tok);
      last = -wave_min(-last);
      __shared__ int w_tok[4], w_last[4];
      if (lane == 0) {
        w_tok[w] = tok;
        w_last[w] = last;
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        const int f = min(min(w_tok[0], w_tok[1]), min(w_tok[2], w_tok[3]));
        const int e = max(max(w_last[0], w_last[1]), max(w_last[2], w_last[3]));
        s_tok = f != 0x7FFFFFFF ? f : e;
      }
    }
  }
  __syncthreads();
  // outputs: the accepted drafts, the drawn token, then -1 and 0
  if (threadIdx.x <= a.drafts) {
    const int t = threadIdx.x;
    const size_t at = (size_t)i * (a.drafts + 1) + t;
    int tok = -1;
    float lp = 0.f;
    if (t <= d.taken) {
      tok = t < d.taken ? a.draft_tokens[(size_t)i * a.drafts + t] : s_tok;
      const RowSum r = L.row[t];
      lp = tok < 0 ? NAN
                   : (float)(((double)row_ptr(a, target_row(a, i, t))[tok] - (double)r.max) /
                                 (a.temp == 0.0 ? 1.0 : a.temp) -
                             log(r.sum));
    }
    a.out_tokens[at] = tok;
    a.out_logprobs[at] = lp;
    if (t == 0) a.out_accepted[i] = d.taken;
  }
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  const bool dist = a.draft_logits && a.temp != 0.0 && a.drafts > 0;
  const long long rows = (long long)a.n * (a.drafts + 1) + (dist ? (long long)a.n * a.drafts : 0);
  hipLaunchKernelGGL(verify_rows_kernel, dim3((unsigned)((rows * a.chunks + 3) / 4)), dim3(256), 0,
                     st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (dist) {
    hipLaunchKernelGGL(verify_rest_kernel, dim3((unsigned)(a.n * ((a.chunks + 3) / 4))), dim3(256),
                       0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_pick_kernel<true>, dim3((unsigned)a.n), dim3(256), 0, st, a);
  } else {
    hipLaunchKernelGGL(verify_pick_kernel<false>, dim3((unsigned)a.n), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace sevo
