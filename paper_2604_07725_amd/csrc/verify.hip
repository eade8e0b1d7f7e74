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
// choices.  Exponentials and sums are in 64 bits throughout (2^-50 relative each), which
// the rows' reads cover: bound by HBM, then by the vector ALU.  Three kernels:
//   1. per (row, 4096 entries): the largest logit and the sum of exponentials relative to it;
//   2. (a draft distribution given) per (candidate, 4096 entries): the sum of max(p - q, 0) of the
//      row where the candidate's drafts end;
//   3. per candidate: the chunk that holds the drawn point, and in it the entry.
// Kernels 2 and 3 find the number of accepted drafts from 1's sums, each workgroup for its
// candidate.
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

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ double wave_scan64(double v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
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

}  // namespace

__global__ __launch_bounds__(256) void verify_rows_kernel(VerifyArgs a) {
  __shared__ float s_max[4];
  __shared__ double s_sum[4];
  __shared__ int s_arg[4];
  const size_t row = blockIdx.x / a.chunks;
  const int chunk = blockIdx.x - (unsigned)(row * a.chunks);
  const size_t targets = (size_t)a.n * (a.drafts + 1);
  // rows behind a candidate's last draft are not read
  if (row < targets) {
    const int i = (int)(row / (a.drafts + 1));
    if ((int)(row - (size_t)i * (a.drafts + 1)) > drafts_of(a, i)) return;
  } else {
    const int i = (int)((row - targets) / a.drafts);
    if ((int)(row - targets - (size_t)i * a.drafts) >= drafts_of(a, i)) return;
  }
  const float* r = row_ptr(a, row);
  const int v0 = chunk * kVerifyChunk + threadIdx.x * 4;
  f32x4 z[kPer / 4];
#pragma unroll
  for (int j = 0; j < kPer / 4; ++j) z[j] = row4(r, v0 + 1024 * j, a.vocab);
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < kPer / 4; ++j) m = fmaxf(fmaxf(fmaxf(m, z[j].x), fmaxf(z[j].y, z[j].z)), z[j].w);
  m = wave_max(m);
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (lane == 0) s_max[w] = m;
  __syncthreads();
  m = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  const double c = log2_scale(a);
  const double mc = m == -INFINITY ? 0.0 : (double)m;
  double sum = 0.0;
  int arg = 0x7FFFFFFF;
#pragma unroll
  for (int j = 0; j < kPer / 4; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      sum += exp2d(((double)z[j][k] - mc) * c);
      if (z[j][k] == m) arg = min(arg, v0 + 1024 * j + k);
    }
  sum = wave_sum64(sum);
  arg = wave_min(arg);
  if (lane == 0) {
    s_sum[w] = sum;
    s_arg[w] = arg;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const size_t at = row * a.chunks + chunk;
    a.part_max[at] = m;
    a.part_sum[at] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
    a.part_arg[at] = min(min(s_arg[0], s_arg[1]), min(s_arg[2], s_arg[3]));
  }
}

namespace {

// a row's largest logit, its sum of exponentials, its first largest entry
struct RowSum {
  double sum;
  float max;
  int arg;
};
struct Decision {
  int taken, count;
};
struct VerifyLds {
  RowSum row[2 * kVerifyMaxDrafts + 1];  // targets 0 .. drafts, then the drafts' own
  int taken;
};

// one wave: the row's partials joined, every lane gets the result
__device__ __forceinline__ RowSum join_row(const VerifyArgs& a, size_t row) {
  const int lane = threadIdx.x & 63;
  const float* pm = a.part_max + row * a.chunks;
  const double* ps = a.part_sum + row * a.chunks;
  const int32_t* pa = a.part_arg + row * a.chunks;
  float m = -INFINITY;
  for (int k = lane; k < a.chunks; k += 64) m = fmaxf(m, pm[k]);
  m = wave_max(m);
  const double mc = m == -INFINITY ? 0.0 : (double)m, c = log2_scale(a);
  double s = 0.0;
  int arg = 0x7FFFFFFF;
  for (int k = lane; k < a.chunks; k += 64) {
    s += ps[k] * exp2d(((double)pm[k] - mc) * c);
    if (pm[k] == m) arg = min(arg, pa[k]);
  }
  return RowSum{wave_sum64(s), m, wave_min(arg)};
}

// a sum that a distribution can have: not of a row with a NaN, a +inf or nothing above -inf
__device__ __forceinline__ bool fine(double s) { return s > 0.0 && s < INFINITY; }

__device__ __forceinline__ double prob(const VerifyArgs& a, const RowSum& r, float z) {
  return exp2d(((double)z - (double)r.max) * log2_scale(a)) / r.sum;
}

// The sums of candidate i's rows into LDS, and how many drafts are accepted.  All threads.
__device__ __forceinline__ Decision decide(const VerifyArgs& a, int i, VerifyLds& L) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int count = drafts_of(a, i);
  const bool dist = a.draft_logits && a.temp != 0.0;
  const int rows = count + 1 + (dist ? count : 0);
  for (int r = w; r < rows; r += 4) {
    const RowSum s = join_row(a, r <= count ? target_row(a, i, r) : draft_row(a, i, r - count - 1));
    if (lane == 0) L.row[r <= count ? r : kVerifyMaxDrafts + r - count] = s;
  }
  __syncthreads();
  if (w == 0) {
    bool ok = true;
    if (lane < count) {
      const int x = a.draft_tokens[(size_t)i * a.drafts + lane];
      const RowSum r = L.row[lane];
      ok = false;
      if (x >= 0 && x < a.vocab && fine(r.sum)) {
        const double p = a.temp == 0.0 ? (x == r.arg ? 1.0 : 0.0)
                                       : prob(a, r, row_ptr(a, target_row(a, i, lane))[x]);
        double q = 1.0;
        if (dist) q = prob(a, L.row[kVerifyMaxDrafts + 1 + lane], row_ptr(a, draft_row(a, i, lane))[x]);
        ok = a.temp == 0.0 ? p == 1.0 : (double)a.uniforms[(size_t)i * (a.drafts + 1) + lane] * q < p;
      }
    }
    const uint64_t bad = __builtin_amdgcn_ballot_w64(!ok);
    if (lane == 0) L.taken = bad ? min(count, (int)__builtin_ctzll(bad)) : count;
  }
  __syncthreads();
  return Decision{L.taken, count};
}

// The weights that the next token is drawn from, at entries v .. v + 3: max(p - q, 0), or without a
// draft distribution p times the row's sum (the scale does not matter, and the sums of a flat
// row are exact), there with or without the rejected draft
struct Weights {
  const float* target;
  const float* draft;  // null: none
  double mt, inv_t, md, inv_d, c;
  int without;  // -1: none
  int vocab;
  __device__ __forceinline__ void at(int v, double (&o)[4]) const {
    // no multiply-add here: with a rounded product on either side, of equal rows nothing is left
#pragma clang fp contract(off)
    const f32x4 z = row4(target, v, vocab);
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = exp2d(((double)z[k] - mt) * c) * inv_t;
    if (draft) {
      const f32x4 y = row4(draft, v, vocab);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const double d = o[k] - exp2d(((double)y[k] - md) * c) * inv_d;
        o[k] = v + k < vocab && !(d < 0.0) ? d : 0.0;  // a NaN stays one
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (v + k == without) o[k] = 0.0;
  }
};

__device__ __forceinline__ Weights weights(const VerifyArgs& a, int i, const Decision& d,
                                           const VerifyLds& L, bool residual) {
  const RowSum t = L.row[d.taken];
  Weights w;
  w.target = row_ptr(a, target_row(a, i, d.taken));
  w.draft = nullptr;
  w.mt = t.max;
  w.inv_t = 1.0;
  w.md = 0.0;
  w.inv_d = 1.0;
  w.c = log2_scale(a);
  w.without = -1;
  w.vocab = a.vocab;
  if (residual && d.taken < d.count) {
    if (a.draft_logits) {
      const RowSum q = L.row[kVerifyMaxDrafts + 1 + d.taken];
      w.inv_t = 1.0 / t.sum;
      w.draft = row_ptr(a, draft_row(a, i, d.taken));
      w.md = q.max;
      w.inv_d = 1.0 / q.sum;
    } else {
      w.without = a.draft_tokens[(size_t)i * a.drafts + d.taken];
    }
  }
  return w;
}

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

__global__ __launch_bounds__(256) void verify_rest_kernel(VerifyArgs a) {
  __shared__ VerifyLds L;
  __shared__ double red[4];
  const int i = blockIdx.x / a.chunks, chunk = blockIdx.x - i * a.chunks;
  const Decision d = decide(a, i, L);
  if (d.taken == d.count) return;
  const Weights W = weights(a, i, d, L, true);
  const double s = chunk_sum(W, chunk, red);
  if (threadIdx.x == 0) a.rest_sum[(size_t)i * a.chunks + chunk] = s;
}

__global__ __launch_bounds__(256) void verify_pick_kernel(VerifyArgs a) {
  __shared__ VerifyLds L;
  __shared__ double red[4], s_pre[4];
  __shared__ double s_total, s_target, s_before;
  __shared__ int s_chunk, s_tok, s_last;
  const int i = blockIdx.x;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Decision d = decide(a, i, L);
  const RowSum row = L.row[d.taken];
  const bool valid = fine(row.sum);
  if (threadIdx.x == 0) {
    s_tok = valid && a.temp == 0.0 ? row.arg : -1;
    s_last = -1;
  }
  if (valid && a.temp != 0.0) {  // the same in every thread
    bool residual = d.taken < d.count;
    Weights W = weights(a, i, d, L, true);
    const size_t prow = target_row(a, i, d.taken) * a.chunks;
    // the chunk without the rejected draft: summed again, a difference would lose the digits of what is left
    double left = 0.0;
    const int hole = W.without >= 0 && W.without < a.vocab ? W.without / kVerifyChunk : -1;
    if (hole >= 0) left = chunk_sum(W, hole, red);
    auto weight_of = [&](int k) -> double {
      if (residual && a.draft_logits) return a.rest_sum[(size_t)i * a.chunks + k];
      if (residual && k == hole) return left;
      return a.part_sum[prow + k] * exp2d(((double)a.part_max[prow + k] - (double)row.max) * W.c);
    };
    for (int pass = 0;; ++pass) {
      // wave 0: total, then the first chunk whose running sum passes the drawn point
      if (w == 0) {
        double total = 0.0;
        for (int k0 = 0; k0 < a.chunks; k0 += 64)
          total += wave_sum64(k0 + lane < a.chunks ? weight_of(k0 + lane) : 0.0);
        const double target = (double)a.uniforms[(size_t)i * (a.drafts + 1) + a.drafts] * total;
        int found = -1, last = -1;
        double before = 0.0, last_before = 0.0, run = 0.0;
        for (int k0 = 0; k0 < a.chunks && found < 0; k0 += 64) {
          const double x = k0 + lane < a.chunks ? weight_of(k0 + lane) : 0.0;
          const double in = wave_scan64(x);
          const uint64_t over = __builtin_amdgcn_ballot_w64(x > 0.0 && run + in > target);
          const uint64_t some = __builtin_amdgcn_ballot_w64(x > 0.0);
          if (over) {
            const int l = __builtin_ctzll(over);
            found = k0 + l;
            before = run + __shfl(in - x, l);
          }
          if (some) {
            const int l = 63 - __builtin_clzll(some);
            last = k0 + l;
            last_before = run + __shfl(in - x, l);
          }
          run += __shfl(in, 63);
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
        W.at(v0 + 4 * j, q);
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
  hipLaunchKernelGGL(verify_rows_kernel, dim3((unsigned)(rows * a.chunks)), dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (dist) {
    hipLaunchKernelGGL(verify_rest_kernel, dim3((unsigned)((long long)a.n * a.chunks)), dim3(256), 0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(verify_pick_kernel, dim3((unsigned)a.n), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace sevo
