// Log probabilities of one given class per row, and the two losses of tuning that are functions of them.  With z a row's logits, a its
// class and l = z_a - log sum_j exp(z_j):
//   policy       row = -min(r A, clip(r) A) + k (exp(f - l) - (f - l) - 1), r = exp(l - o);   loss = sum of w row
//   preference   s = sum of w l over a sequence, m = beta ((s_c - f_c) - (s_r - f_r));   loss = mean of -(1 - e) log sig(m) - e log sig(-m)
//   both         dz_j = dloss/dl ([j = a] - softmax(z)_j)
// One read of the logits and one write of their gradient is what the memory has to do; the preference loss reads them twice, since what a row
// weighs is known only when all rows of its pair have been seen.
// Exponents, sums and what is stored are fp32; the numbers of a row (its logarithm, ratios, the sums of a sequence) are formed in fp64 where fp32 would
// lose what the difference of two large ones keeps.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "device_utils.h"
#include "kernels.h"
#include "logprob.h"
#include "row_device.h"

namespace tp {

namespace {

// exp(z - top) = 2^((z - base) c - shift) with shift = (top - base) c rounded once.  That rounding is a factor common to all of a row's
// exponentials, and to their sum, so it leaves the probabilities alone, and the log probability as long as it is formed from the
// same shift.  Where it could take an exponential out of range (logits of 1e7) the maximum is taken off first, at one more operation each.
struct Exponents {
  float base, shift;
  __device__ __forceinline__ explicit Exponents(float top) {
    base = fabsf(top * kLog2e) > 0x1p24f ? top : 0.f;
    shift = (top - base) * kLog2e;
  }
  __device__ __forceinline__ float power(float z) const { return fmaf(z - base, kLog2e, -shift); }
  __device__ __forceinline__ double log_probability(float z, float sum) const {
    return ((double)(z - base) * kLog2e - (double)shift) * 0.6931471805599453 - log((double)sum);
  }
};

// A row's term of the policy loss: its value and what it changes by with the log probability, both times the row's weight.
struct PolicyTerm {
  float loss, slope;
};
__device__ __forceinline__ PolicyTerm policy_term(const PolicyArgs& a, int row, float weight, double logp) {
  const float advantage = a.advantages[row];
  const double moved = logp - (double)a.old_logp[row];
  // which side of a border the ratio is on is decided before anything is rounded to fp32
  const bool above = advantage > 0.f && moved > a.log_high, below = advantage < 0.f && moved < a.log_low;
  const float gain = advantage == 0.f ? 0.f : expf((float)moved) * advantage;
  PolicyTerm t;
  t.loss = -(above ? (1.f + a.clip_high) * advantage : below ? (1.f - a.clip_low) * advantage : gain);
  t.slope = above || below ? 0.f : -gain;
  if (a.kl_weight > 0.f) {
    const float x = (float)((double)a.ref_logp[row] - logp), grown = expm1f(x);
    // exp(x) - 1 - x: its series where the difference would lose more than an ulp or two (x = 1/2: the ninth term is 3e-9 of it)
    float tail = fmaf(x, 1.f / 362880.f, 1.f / 40320.f);
    tail = fmaf(x, tail, 1.f / 5040.f);
    tail = fmaf(x, tail, 1.f / 720.f);
    tail = fmaf(x, tail, 1.f / 120.f);
    tail = fmaf(x, tail, 1.f / 24.f);
    tail = fmaf(x, tail, 1.f / 6.f);
    tail = fmaf(x, tail, 0.5f);
    t.loss = fmaf(a.kl_weight, fabsf(x) < 0.5f ? x * x * tail : grown - x, t.loss);
    t.slope = fmaf(-a.kl_weight, grown, t.slope);
  }
  t.loss *= weight;
  t.slope *= weight;
  return t;
}

// ---- any row, by a workgroup of its own ---------------------------------------------------------
constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ RowStats read_row(const T* lg, int classes, float* sm) {
  using TM = Team<kThreads>;
  float top = -INFINITY;
  for (int j = threadIdx.x; j < classes; j += kThreads) top = fmaxf(top, to_float(lg[j]));
  top = TM::over(top, sm, Max());
  const Exponents e(top);
  float sum = 0.f;
  for (int j = threadIdx.x; j < classes; j += kThreads) sum += __builtin_amdgcn_exp2f(e.power(to_float(lg[j])));
  return RowStats{top, TM::over(sum, sm, Add())};
}
// slope ([j = id] - softmax(z)_j), or zeros (slope 0: whatever the logits hold)
template <typename T>
__device__ __forceinline__ void write_row(const RowStats& r, const T* lg, T* dl, int classes, int id, float slope) {
  const Exponents e(r.top);
  const float scale = -slope / r.sum;
  for (int j = threadIdx.x; j < classes; j += kThreads) {
    float g = 0.f;
    if (slope != 0.f) {
      g = scale * __builtin_amdgcn_exp2f(e.power(to_float(lg[j])));
      if (j == id) g += slope;
    }
    dl[j] = from_float<T>(g);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void logprob_rows_kernel(LogprobArgs a) {
  __shared__ float sm[kThreads / 64];
  for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int id = a.ids[row];
    const bool counts = id >= 0 && (!a.weights || a.weights[row] != 0.f);
    const T* lg = (const T*)a.logits + (size_t)row * a.classes;
    RowStats r{0.f, 1.f};
    if (counts) r = read_row(lg, a.classes, sm);
    if (threadIdx.x == 0) {
      a.logp[row] = !counts ? 0.f : id < a.classes ? (float)Exponents(r.top).log_probability(to_float(lg[id]), r.sum) : __builtin_nanf("");
      if (a.stats) a.stats[row] = r;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void policy_rows_kernel(PolicyArgs a) {
  __shared__ float sm[kThreads / 64];
  for (long at = blockIdx.x; at < a.rows; at += gridDim.x) {
    const int row = (int)at, id = a.actions[row];
    const float weight = a.weights ? a.weights[row] : 1.f / (float)a.rows;
    const bool counts = id >= 0 && weight != 0.f, known = id < a.classes;
    const T* lg = (const T*)a.logits + (size_t)row * a.classes;
    RowStats r{0.f, 1.f};
    PolicyTerm t{0.f, 0.f};
    double logp = 0.0;
    if (counts && known) {
      r = read_row(lg, a.classes, sm);
      logp = Exponents(r.top).log_probability(to_float(lg[id]), r.sum);
      t = policy_term(a, row, weight, logp);
    } else if (counts) {
      logp = __builtin_nan("");
      t.loss = __builtin_nanf("");
    }
    if (threadIdx.x == 0) {
      a.row_loss[row] = t.loss;
      if (a.logp) a.logp[row] = (float)logp;
    }
    write_row(r, lg, (T*)a.dlogits + (size_t)row * a.classes, a.classes, id, t.slope);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void preference_rows_kernel(PreferenceArgs a) {
  const long rows = 2l * a.pairs * a.tokens;
  for (long row = blockIdx.x; row < rows; row += gridDim.x) {
    const int id = a.targets[row];
    const float weight = a.weights ? a.weights[row] : 1.f;
    const float slope = id >= 0 && weight != 0.f ? a.pull[row / a.tokens] * weight : 0.f;
    write_row(a.stats[row], (const T*)a.logits + (size_t)row * a.classes, (T*)a.dlogits + (size_t)row * a.classes, a.classes, id, slope);
  }
}

// ---- the sums -----------------------------------------------------------------------------------
// Of 1024 threads' values, in every thread of the first wave's first lane; sm: 16 doubles.
constexpr int kSumThreads = 1024;
__device__ __forceinline__ double block_sum(double s, double* sm) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += sm[w];
  __syncthreads();
  return s;
}
// out = sum of n values, over `by`
__global__ __launch_bounds__(kSumThreads) void loss_sum_kernel(const float* __restrict__ v, long n, double by, float* __restrict__ out) {
  __shared__ double sm[kSumThreads / 64];
  double s = 0.0;
  long i = threadIdx.x;
  for (; i + 7 * kSumThreads < n; i += 8 * kSumThreads) {  // eight loads on their way
    float x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = v[i + u * kSumThreads];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += (double)x[u];
  }
  for (; i < n; i += kSumThreads) s += (double)v[i];
  s = block_sum(s, sm);
  if (threadIdx.x == 0) *out = (float)(s / by);
}

// A workgroup a pair: the sums of its two sequences, its loss, and what a log probability of either weighs.
__global__ __launch_bounds__(kThreads) void preference_pairs_kernel(PreferenceArgs a) {
  __shared__ double sm[kThreads / 64];
  for (long pair = blockIdx.x; pair < a.pairs; pair += gridDim.x) {
    double ratio[2];
    for (int k = 0; k < 2; ++k) {
      const size_t row0 = (size_t)(2 * pair + k) * a.tokens;
      double s = 0.0;
      for (int t = threadIdx.x; t < a.tokens; t += kThreads) {
        const float weight = a.weights ? a.weights[row0 + t] : 1.f;
        if (a.targets[row0 + t] >= 0 && weight != 0.f) s += (double)weight * (double)a.logp[row0 + t];
      }
      ratio[k] = block_sum(s, sm) - (double)a.ref_logp[2 * pair + k];
    }
    if (threadIdx.x == 0) {
      const double m = a.beta * (ratio[0] - ratio[1]);
      // log sig(m) = min(m, 0) - log(1 + e^-|m|)
      const double e = exp(-fabs(m)), rest = log1p(e), big = 1.0 / (1.0 + e), small = e / (1.0 + e);
      const double right = m >= 0.0 ? big : small, wrong = m >= 0.0 ? small : big;  // sig(m), sig(-m)
      const double log_right = fmin(m, 0.0) - rest, log_wrong = fmin(-m, 0.0) - rest;
      double loss = 0.0;
      if (a.smoothing < 1.0) loss -= (1.0 - a.smoothing) * log_right;
      if (a.smoothing > 0.0) loss -= a.smoothing * log_wrong;
      const double pull = a.beta / a.pairs * (a.smoothing * right - (1.0 - a.smoothing) * wrong);
      a.pair_loss[pair] = m == m ? (float)loss : __builtin_nanf("");
      a.pull[2 * pair] = (float)pull;
      a.pull[2 * pair + 1] = (float)-pull;
    }
  }
}

unsigned row_blocks(long rows) { return (unsigned)std::min<long>(rows, 1 << 20); }

hipError_t sum_losses(hipStream_t s, const float* v, long n, double by, float* out) {
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(kSumThreads), 0, s, v, n, by, out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_logprobs(hipStream_t s, int elt, const LogprobArgs& a) {
  if (elt == ELT_BF16) hipLaunchKernelGGL(logprob_rows_kernel<uint16_t>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(logprob_rows_kernel<float>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_policy(hipStream_t s, int elt, const PolicyArgs& a) {
  if (elt == ELT_BF16) hipLaunchKernelGGL(policy_rows_kernel<uint16_t>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(policy_rows_kernel<float>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : sum_losses(s, a.row_loss, a.rows, 1.0, a.loss);
}

hipError_t launch_preference(hipStream_t s, int elt, const PreferenceArgs& a) {
  const long rows = 2l * a.pairs * a.tokens;
  hipError_t e = launch_logprobs(s, elt, LogprobArgs{(int)rows, a.classes, a.logits, a.targets, a.logp, a.stats, a.weights});
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(preference_pairs_kernel, dim3(row_blocks(a.pairs)), dim3(kThreads), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (elt == ELT_BF16) hipLaunchKernelGGL(preference_rows_kernel<uint16_t>, dim3(row_blocks(rows)), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(preference_rows_kernel<float>, dim3(row_blocks(rows)), dim3(kThreads), 0, s, a);
  e = hipGetLastError();
  return e != hipSuccess ? e : sum_losses(s, a.pair_loss, a.pairs, (double)a.pairs, a.loss);
}

}  // namespace tp
