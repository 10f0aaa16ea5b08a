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
#include <type_traits>

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

// A row's term of the policy loss: its value and what it changes by with the log probability, both times the row's weight.  In fp64: rows of both
// signs cancel, and a sum of rows rounded to fp32 was up to six times further off than one of fp32 exponentials.  It takes 3 us more than
// in fp32 (128000 rows of 50 classes in bf16 31 -> 34 us, 8192 of 32000 172 -> 175).
struct PolicyTerm {
  double loss;
  float slope;
};
__device__ __forceinline__ PolicyTerm policy_term(const PolicyArgs& a, int row, double weight, double logp) {
  const double advantage = (double)a.advantages[row];
  const double moved = logp - (double)a.old_logp[row];
  const bool above = advantage > 0.0 && moved > a.log_high, below = advantage < 0.0 && moved < a.log_low;
  const double gain = advantage == 0.0 ? 0.0 : exp(moved) * advantage;
  double loss = -(above ? (1.0 + a.clip_high) * advantage : below ? (1.0 - a.clip_low) * advantage : gain);
  double slope = above || below ? 0.0 : -gain;
  if (a.kl_weight > 0.0) {
    const double x = (double)a.ref_logp[row] - logp, grown = expm1(x);
    loss += a.kl_weight * (grown - x);
    slope -= a.kl_weight * grown;
  }
  return PolicyTerm{loss * weight, (float)(slope * weight)};
}

// row losses go as doubles
__device__ __forceinline__ void publish(double* p, double v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double published(const double* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// ---- any row, by a workgroup of its own ---------------------------------------------------------
constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ RowStats read_row(const T* lg, int classes, float* sm) {
  using TM = Team<kThreads>;
  float top = -INFINITY;
  for (int j = threadIdx.x; j < classes; j += kThreads) top = fmaxf(top, to_float(lg[j]));
  top = TM::over(top, sm, Max());
  const Exponents e(top);
  // Eight at a time in fp32, their sums in fp64: in one chain of classes / 256 the unlikely classes of a long row were lost beside a likely one
  // (200003 classes, 1 of them likely: log probability 2.4e-5 off, within 1.6e-6 now).  Eight loads are on
  // their way at a time, too: log probabilities of 1024 rows of 128256 classes in bf16 304 -> 186 us.
  auto grown = [&](int j) { return __builtin_amdgcn_exp2f(e.power(to_float(lg[j]))); };
  float sum = 0.f;
  int j = threadIdx.x;
  if (classes >= 8 * kThreads) {
    double all = 0.0;
    for (; j + 7 * kThreads < classes; j += 8 * kThreads) {
      float part = 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) part += grown(j + u * kThreads);
      all += (double)part;
    }
    for (; j < classes; j += kThreads) sum += grown(j);
    sum = (float)(all + (double)sum);
  } else {
    for (; j < classes; j += kThreads) sum += grown(j);
  }
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

__device__ __forceinline__ void store_row(const LogprobArgs& a, long row, const RowStats& r, double logp) {
  const float stored = (float)logp;
  a.logp[row] = stored;
  if (a.stats) {
    a.stats[row] = r;
    a.logp_rest[row] = float_to_bf16(fabsf(stored) < INFINITY ? (float)(logp - (double)stored) : 0.f);
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
      store_row(a, row, r, !counts ? 0.0 : id < a.classes ? Exponents(r.top).log_probability(to_float(lg[id]), r.sum) : __builtin_nan(""));
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void policy_rows_kernel(PolicyArgs a) {
  __shared__ float sm[kThreads / 64];
  for (long at = blockIdx.x; at < a.rows; at += gridDim.x) {
    const int row = (int)at, id = a.actions[row];
    const double weight = a.weights ? (double)a.weights[row] : 1.0 / a.rows;
    const bool counts = id >= 0 && weight != 0.0, known = id < a.classes;
    const T* lg = (const T*)a.logits + (size_t)row * a.classes;
    RowStats r{0.f, 1.f};
    PolicyTerm t{0.0, 0.f};
    double logp = 0.0;
    if (counts && known) {
      r = read_row(lg, a.classes, sm);
      logp = Exponents(r.top).log_probability(to_float(lg[id]), r.sum);
      t = policy_term(a, row, weight, logp);
    } else if (counts) {
      logp = __builtin_nan("");
      t.loss = __builtin_nan("");
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

// ---- rows that registers hold -------------------------------------------------------------------
// A row is read once and held, HELD units of 16 bytes for each of its NT threads, and its gradient written once; rows may start at any
// element (units lie at 16-byte addresses; the first and last, which other rows share, are read and written one by one).
template <typename T, int NT, int HELD>
struct Held {
  using TM = Team<NT>;
  static constexpr int V = kVec<T>;
  const T* unit0;
  int thread, classes, lead, whole_from, whole_to, units;
  float x[HELD][V];

  __device__ __forceinline__ Held(const T* lg, int classes_) : thread(TM::thread()), classes(classes_) {
    lead = (int)((uintptr_t)lg % 16 / sizeof(T));  // values of the first unit that are another row's
    whole_from = lead > 0;
    whole_to = (lead + classes) / V;               // units that are this row's alone
    units = (lead + classes + V - 1) / V;
    unit0 = lg - lead;
  }
  __device__ __forceinline__ void read() {
    uint4 raw[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int u = min(max(thread + NT * i, whole_from), whole_to - 1);
      raw[i] = *reinterpret_cast<const uint4*>(unit0 + (size_t)u * V);
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int u = thread + NT * i;
      unpack<T>(raw[i], x[i]);
      if (u < whole_from || u >= whole_to) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int j = u * V + e - lead;
          x[i][e] = u < units && j >= 0 && j < classes ? to_float(unit0[lead + j]) : -INFINITY;
        }
      }
    }
  }
  __device__ __forceinline__ float top(float* sm) const {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) m = fmaxf(m, x[i][e]);
    return TM::over(m, sm, Max());
  }
  // every value becomes its exponential; this thread's sum of them
  __device__ __forceinline__ float exponentials(const Exponents& ex) {
    if (ex.base != 0.f) {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) x[i][e] -= ex.base;
    }
    float sum[4] = {};  // short chains of additions
#pragma unroll
    for (int i = 0; i < HELD; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[i][e] = __builtin_amdgcn_exp2f(fmaf(x[i][e], kLog2e, -ex.shift));
        sum[e % 4] += x[i][e];
      }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  // The exponentials times `scale`, and `own` in the place of class id's (none: a negative one).  The thread that stores a unit replaces a value
  // of it, in program order.
  __device__ __forceinline__ void write(T* dl, float scale, int id, float own) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int u = thread + NT * i;
#pragma unroll
      for (int e = 0; e < V; ++e) x[i][e] *= scale;
      store(dl, u, x[i]);
    }
    if (id >= 0 && (lead + id) / V % NT == thread) dl[id] = from_float<T>(own);
  }
  __device__ __forceinline__ void write_zeros(T* dl) {
    const float none[V] = {};
    for (int u = thread; u < units; u += NT) store(dl, u, none);
  }
  __device__ __forceinline__ void store(T* dl, int u, const float (&v)[V]) const {
    if (u >= whole_from && u < whole_to) {
      *reinterpret_cast<uint4*>(dl - lead + (size_t)u * V) = pack<T>(v);
    } else if (u < units) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int j = u * V + e - lead;
        if (j >= 0 && j < classes) dl[j] = from_float<T>(v[e]);
      }
    }
  }
};
// Of 64 values a thread, two workgroups of 512 threads on a CU.
template <typename T, int HELD>
constexpr int kWavesASimd = HELD * kVec<T> == 64 ? 4 : 1;

template <typename T, int NT, int HELD>
__global__ __launch_bounds__(Team<NT>::kThreads, (kWavesASimd<T, HELD>)) void logprob_held_kernel(LogprobArgs a, int first_row) {
  using TM = Team<NT>;
  __shared__ float sm[TM::kThreads / 64];
  const long at = first_row + (long)blockIdx.x * TM::kRows + TM::which();
  if (at >= a.rows) return;
  const int row = (int)at;
  const int id = a.ids[row];
  const bool counts = id >= 0 && (!a.weights || a.weights[row] != 0.f);
  const T* lg = (const T*)a.logits + (size_t)row * a.classes;
  RowStats r{0.f, 1.f};
  float z = 0.f;
  if (counts) {
    if (id < a.classes) z = to_float(lg[id]);
    Held<T, NT, HELD> h(lg, a.classes);
    h.read();
    r.top = h.top(sm);
    r.sum = TM::over(h.exponentials(Exponents(r.top)), sm, Add());
  }
  if (TM::thread() == 0) {
    store_row(a, row, r, !counts ? 0.0 : id < a.classes ? Exponents(r.top).log_probability(z, r.sum) : __builtin_nan(""));
  }
}

// The sum of the losses, over `by`, by the workgroup that arrives last, where a counter is given.
__device__ __forceinline__ void finish_sum(uint32_t* counter, const double* row_loss, int rows, double by, float* loss) {
  __shared__ double sums[256];
  __shared__ int finishes;
  if (!counter) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's row losses have arrived
  __syncthreads();
  if (threadIdx.x == 0) finishes = last_to_arrive(counter, gridDim.x);
  __syncthreads();
  if (!finishes) return;
  if (threadIdx.x < 256) {
    double s = 0.0;
    for (int i = threadIdx.x; i < rows; i += 256) s += published(row_loss + i);
    sums[threadIdx.x] = s;
  }
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) sums[threadIdx.x] += sums[threadIdx.x + w];
    __syncthreads();
  }
  if (threadIdx.x == 0) *loss = (float)(sums[0] / by);
}

template <typename T, int NT, int HELD>
__global__ __launch_bounds__(Team<NT>::kThreads, (kWavesASimd<T, HELD>)) void policy_held_kernel(PolicyArgs a) {
  using TM = Team<NT>;
  __shared__ float sm[TM::kThreads / 64];
  const long at = a.first_row + (long)blockIdx.x * TM::kRows + TM::which();
  if (at < a.rows) {
    const int row = (int)at;
    const int id = a.actions[row];
    const double weight = a.weights ? (double)a.weights[row] : 1.0 / a.rows;
    const bool counts = id >= 0 && weight != 0.0, known = id < a.classes;
    const T* lg = (const T*)a.logits + (size_t)row * a.classes;
    T* dl = (T*)a.dlogits + (size_t)row * a.classes;
    Held<T, NT, HELD> h(lg, a.classes);
    PolicyTerm t{0.0, 0.f};
    double logp = 0.0;
    if (counts && known) {
      const float z = to_float(lg[id]);
      h.read();
      const Exponents ex(h.top(sm));
      const float sum = TM::over(h.exponentials(ex), sm, Add());
      logp = ex.log_probability(z, sum);
      t = policy_term(a, row, weight, logp);
      if (t.slope != 0.f) {
        const float scale = -t.slope / sum;
        h.write(dl, scale, id, t.slope + scale * __builtin_amdgcn_exp2f(ex.power(z)));
      }
    } else if (counts) {
      logp = __builtin_nan("");
      t.loss = __builtin_nan("");
    }
    if (t.slope == 0.f) h.write_zeros(dl);
    if (TM::thread() == 0) {
      publish(a.row_loss + row, t.loss);
      if (a.logp) a.logp[row] = (float)logp;
    }
  }
  finish_sum(a.counter, a.row_loss, a.rows, 1.0, a.loss);
}

template <typename T, int NT, int HELD>
__global__ __launch_bounds__(Team<NT>::kThreads, (kWavesASimd<T, HELD>)) void preference_held_kernel(PreferenceArgs a, int first_row) {
  using TM = Team<NT>;
  const int rows = 2 * a.pairs * a.tokens;
  const long at = first_row + (long)blockIdx.x * TM::kRows + TM::which();
  if (at >= rows) return;
  // From the last row to the first: what the pass before read last is what the last-level cache still has (8192 rows of 32000 classes in bf16
  // 150 -> 146 us).  Both passes over a few pairs at a time, 131 MB of them or 262, find more there and lose it to the ends of twice as many
  // launches: 250 us in all, 300 and 271 so.
  const int row = rows - 1 - (int)at;
  const int id = a.targets[row];
  const float weight = a.weights ? a.weights[row] : 1.f;
  const float slope = id >= 0 && weight != 0.f ? a.pull[row / a.tokens] * weight : 0.f;
  const T* lg = (const T*)a.logits + (size_t)row * a.classes;
  T* dl = (T*)a.dlogits + (size_t)row * a.classes;
  Held<T, NT, HELD> h(lg, a.classes);
  if (slope == 0.f) {
    h.write_zeros(dl);
    return;
  }
  const RowStats r = a.stats[row];
  const Exponents ex(r.top);
  const float scale = -slope / r.sum;
  const float z = id < a.classes ? to_float(lg[id]) : 0.f;
  h.read();
  h.exponentials(ex);
  h.write(dl, scale, id < a.classes ? id : -1, slope + scale * __builtin_amdgcn_exp2f(ex.power(z)));
}

// ---- the sums -----------------------------------------------------------------------------------
// Of a workgroup's values, in every thread; sm: a double for each wave.
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
// out = sum of n values, over `by`: workgroups of 8192 values and up, their sums added up by the one that arrives last, in their order.
// (128000 values by one workgroup 14 us, by 15 4.6.)
__global__ __launch_bounds__(kSumThreads) void loss_sum_kernel(const double* __restrict__ v, long n, double by, double* parts, uint32_t* counter,
                                                               float* __restrict__ out) {
  __shared__ double sm[kSumThreads / 64];
  __shared__ int finishes;
  const long step = (long)gridDim.x * kSumThreads;
  double s = 0.0;
  long i = (long)blockIdx.x * kSumThreads + threadIdx.x;
  for (; i + 7 * step < n; i += 8 * step) {  // eight loads on their way
    double x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = v[i + u * step];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += x[u];
  }
  for (; i < n; i += step) s += v[i];
  s = block_sum(s, sm);
  if (gridDim.x > 1) {
    if (threadIdx.x == 0) {
      publish(parts + blockIdx.x, s);
      finishes = last_to_arrive(counter, gridDim.x);
    }
    __syncthreads();
    if (!finishes) return;
    s = block_sum(threadIdx.x < gridDim.x ? published(parts + threadIdx.x) : 0.0, sm);
  }
  if (threadIdx.x == 0) *out = (float)(s / by);
}

// A workgroup a pair: the sums of its two sequences, whose rows lie one behind the other, its loss, and what a log probability of either weighs; the
// mean of the losses by the workgroup that arrives last, where a counter is given.  What rounding log
// probabilities to fp32 has left over is added: without it results of 1002 rows of 32003 classes were 4.5e-7 of their norm off, 6e-8 with it.  A thread has
// four rows on their way at a time (28736 rows of 592 classes, eight pairs: 7 us, row after row 9.5; log probabilities formed again in fp64 11.6).
__global__ __launch_bounds__(kSumThreads) void preference_pairs_kernel(PreferenceArgs a) {
  __shared__ double sm[kSumThreads / 64];
  for (long pair = blockIdx.x; pair < a.pairs; pair += gridDim.x) {
    const size_t row0 = (size_t)(2 * pair) * a.tokens;
    const long rows = 2l * a.tokens;
    const double ref[2] = {a.ref_logp[2 * pair], a.ref_logp[2 * pair + 1]};
    double s[2] = {0.0, 0.0};
    for (long i = threadIdx.x; i < rows; i += 4 * kSumThreads) {
      int id[4];
      float weight[4], logp[4], rest[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const size_t row = row0 + std::min(i + u * kSumThreads, rows - 1);
        id[u] = a.targets[row];
        weight[u] = a.weights ? a.weights[row] : 1.f;
        logp[u] = a.logp[row];
        rest[u] = to_float(a.logp_rest[row]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const long t = i + u * kSumThreads;
        const double term = t < rows && id[u] >= 0 && weight[u] != 0.f ? (double)weight[u] * ((double)logp[u] + (double)rest[u]) : 0.0;
        if (t < a.tokens) s[0] += term;
        else s[1] += term;
      }
    }
    double ratio[2];
    for (int k = 0; k < 2; ++k) ratio[k] = block_sum(s[k], sm) - ref[k];
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
      publish(a.pair_loss + pair, m == m ? loss : __builtin_nan(""));
      a.pull[2 * pair] = (float)pull;
      a.pull[2 * pair + 1] = (float)-pull;
    }
  }
  finish_sum(a.counter, a.pair_loss, a.pairs, (double)a.pairs, a.loss);
}

unsigned row_blocks(long rows) { return (unsigned)std::min<long>(rows, 1 << 20); }

hipError_t sum_losses(hipStream_t s, const double* v, long n, double by, double* parts, uint32_t* counter, float* out) {
  const long blocks = std::max<long>(1, std::min<long>(kSumParts, n / (8 * kSumThreads)));
  hipLaunchKernelGGL(loss_sum_kernel, dim3((unsigned)blocks), dim3(kSumThreads), 0, s, v, n, by, parts, counter, out);
  return hipGetLastError();
}

// Calls f with the threads of a row and the units each holds (two integral constants) and the workgroups, some of them at a time: a launch takes
// fewer than 2^32 threads, and drops what a grid has beyond.  False: rows that are not held, of too few units or too many.
template <typename T, class F>
bool held(int rows, int classes, const F& f) {
  constexpr int V = kVec<T>, W = 64 / V;  // units of 64 values
  const long units = classes / V + 2;     // with a first and a last one that are shared
  auto go = [&](auto nt, auto count) {
    constexpr int NT = decltype(nt)::value;
    const long blocks = ((long)rows + Team<NT>::kRows - 1) / Team<NT>::kRows, most = UINT32_MAX / Team<NT>::kThreads;
    for (long from = 0; from < blocks; from += most)
      f(nt, count, (unsigned)std::min(most, blocks - from), blocks, (int)(from * Team<NT>::kRows));
    return true;
  };
  auto n = [](auto v) { return v; };
#define TP_HELD(NT, COUNT) go(n(std::integral_constant<int, NT>()), n(std::integral_constant<int, COUNT>()))
  if (classes < 2 * V) return false;
  // Rows of up to 128 units have a quarter of a wave, so that what is done once a row, its logarithm in fp64 and its term, is done for four at a
  // time; rows that a wave can hold have one, and no barriers.  policy in bf16, with a wave for each 64 units up to 128 and a workgroup from there:
  // 128000 rows of 50 classes 89 -> 36 us, of 1001 145 -> 109, 64000 of 2000 141 -> 88, 51200 of 4001 167 -> 145; fp32, 51200 of 700 87 -> 49 (all
  // with terms in fp32).
  if (units <= 16) return TP_HELD(16, 1);
  if (units <= 16 * 2) return TP_HELD(16, 2);
  if (units <= 16 * 4) return TP_HELD(16, 4);
  if (units <= 16 * 8) return TP_HELD(16, 8);
  if (units <= 64 * 4) return TP_HELD(64, 4);
  if (units <= 64 * 8) return TP_HELD(64, 8);
  if constexpr (sizeof(T) == 4)
    if (units <= 256 * 4) return TP_HELD(256, 4);
  if (units <= 256 * W / 2) return TP_HELD(256, W / 2);
  if (units <= 256 * W) return TP_HELD(256, W);
  if (units <= 512 * W) return TP_HELD(512, W);
  if (units <= 1024 * W) return TP_HELD(1024, W);
#undef TP_HELD
  return false;
}
inline bool alike(const void* a, const void* b) { return ((uintptr_t)a - (uintptr_t)b) % 16 == 0; }

constexpr int kCounted = 128;  // workgroups up to which the last of them adds up the losses; more take a launch of their own

template <typename T>
hipError_t logprobs(hipStream_t s, const LogprobArgs& a) {
  const bool done = held<T>(a.rows, a.classes, [&](auto nt, auto count, unsigned blocks, long, int first_row) {
    constexpr int NT = decltype(nt)::value, HELD = decltype(count)::value;
    hipLaunchKernelGGL((logprob_held_kernel<T, NT, HELD>), dim3(blocks), dim3(Team<NT>::kThreads), 0, s, a, first_row);
  });
  if (!done) hipLaunchKernelGGL(logprob_rows_kernel<T>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t policy(hipStream_t s, PolicyArgs a) {
  bool counted = false;
  const bool done = alike(a.logits, a.dlogits) && held<T>(a.rows, a.classes, [&](auto nt, auto count, unsigned blocks, long all, int first_row) {
    constexpr int NT = decltype(nt)::value, HELD = decltype(count)::value;
    counted = all <= kCounted;
    PolicyArgs part = a;
    part.first_row = first_row;
    if (!counted) part.counter = nullptr;
    hipLaunchKernelGGL((policy_held_kernel<T, NT, HELD>), dim3(blocks), dim3(Team<NT>::kThreads), 0, s, part);
  });
  if (!done) hipLaunchKernelGGL(policy_rows_kernel<T>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || counted ? e : sum_losses(s, a.row_loss, a.rows, 1.0, a.parts, a.counter, a.loss);
}

template <typename T>
hipError_t preference(hipStream_t s, PreferenceArgs a) {
  const int rows = 2 * a.pairs * a.tokens;
  hipError_t e = logprobs<T>(s, LogprobArgs{rows, a.classes, a.logits, a.targets, a.logp, a.stats, a.logp_rest, a.weights});
  if (e != hipSuccess) return e;
  const bool counted = a.pairs <= kCounted;
  uint32_t* const counter = a.counter;
  if (!counted) a.counter = nullptr;
  hipLaunchKernelGGL(preference_pairs_kernel, dim3(row_blocks(a.pairs)), dim3(kSumThreads), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const bool done = alike(a.logits, a.dlogits) && held<T>(rows, a.classes, [&](auto nt, auto count, unsigned blocks, long, int first_row) {
    constexpr int NT = decltype(nt)::value, HELD = decltype(count)::value;
    hipLaunchKernelGGL((preference_held_kernel<T, NT, HELD>), dim3(blocks), dim3(Team<NT>::kThreads), 0, s, a, first_row);
  });
  if (!done) hipLaunchKernelGGL(preference_rows_kernel<T>, dim3(row_blocks(rows)), dim3(kThreads), 0, s, a);
  e = hipGetLastError();
  return e != hipSuccess || counted ? e : sum_losses(s, a.pair_loss, a.pairs, (double)a.pairs, a.parts, counter, a.loss);
}

}  // namespace

hipError_t launch_logprobs(hipStream_t s, int elt, const LogprobArgs& a) { return elt == ELT_BF16 ? logprobs<uint16_t>(s, a) : logprobs<float>(s, a); }
hipError_t launch_policy(hipStream_t s, int elt, const PolicyArgs& a) { return elt == ELT_BF16 ? policy<uint16_t>(s, a) : policy<float>(s, a); }
hipError_t launch_preference(hipStream_t s, int elt, const PreferenceArgs& a) {
  return elt == ELT_BF16 ? preference<uint16_t>(s, a) : preference<float>(s, a);
}

}  // namespace tp
