// Learning from a teacher's stored top logits, and from labels, at the last stage.  Per row, with z the student's logits, t the
// teacher's stored ones and w the weight of the label:
//   p = softmax(t / T) over the stored entries,  q = softmax(z / T),  s = softmax(z)
//   row loss = w (-log s_label) + (1 - w) T^2 sum_k p_k (log p_k - log q_id(k)),  loss = mean over the rows
//   dz_j = [w (s_j - [j = label]) + (1 - w) T (q_j - p_j)] / rows
// A row without stored entries (none, or all of them -inf) has no second term, and with w = 1 no row has.  Entries of the same class
// add up.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "device_utils.h"
#include "distill.h"
#include "kernels.h"
#include "row_device.h"

namespace tp {

namespace {

constexpr float kLn2 = 0.6931471805599453f;

// Exponents: exp(z / T) = 2^(power), power = z c - top c with c = log2(e) / T and the row's maximum `top`; exp(z) = 2^(T power).  top c is
// rounded once and its rounding, that of `max / T`, is large where all of a row's logits are: it cancels because every numerator, sum and
// logarithm of both exponentials is formed from this one power.  (With labels alone c = log2(e) and the power is that of exp(z) itself.)
// T = 3, logits around 1000 or 10000, the label's logarithm from z log2(e) - top log2(e) instead: cross entropy 4e-5 or 2e-4 off.
// Where top c is so large that its rounding alone could take an exponential out of range (T = 1e-6, logits of some thousands; T = 1e6, logits of 1e12) the maximum is
// taken off the logits themselves first, at one more operation for each of them.
struct Row {
  float base;          // what is taken off every logit first: 0 or top
  float scale, shift;  // c and top c, or 0 where top is taken off
  float to_hard;       // what turns the power into that of exp(z)
  float soft, hard;    // what the exponentials are multiplied with in the gradient
  __device__ __forceinline__ Row(const DistillArgs& a, float soft_scale, float top) {
    const bool only_hard = a.teacher_weight <= 0.f;
    scale = only_hard ? kLog2e : soft_scale;
    to_hard = only_hard ? 1.f : a.temperature;
    // From 2^24 on the rounding is 1 and more; it counts T times in exp(z).  (The second product may overflow to infinity, which is as good.)
    base = fabsf(top * scale) * fmaxf(1.f, to_hard) > 0x1p24f ? top : 0.f;
    shift = (top - base) * scale;
  }
  __device__ __forceinline__ float power_of_rest(float z) const { return fmaf(z, scale, -shift); }  // base is taken off z
  __device__ __forceinline__ float power(float z) const { return power_of_rest(z - base); }
  __device__ __forceinline__ float gradient(float z) const {
    const float p = power(z);
    float g = soft == 0.f ? 0.f : soft * __builtin_amdgcn_exp2f(p);
    if (hard != 0.f) g = fmaf(hard, __builtin_amdgcn_exp2f(p * to_hard), g);
    return g;
  }
};

// A thread's first entry and the row's label, fetched in two steps: the classes ahead of the row, their logits behind it, so that neither is
// waited for by itself.
struct First {
  int id = -1, label = -1;
  float teacher = 0.f, z = 0.f, z_label = 0.f;
  __device__ __forceinline__ First(const DistillArgs& a, int row, int thread) {
    if (thread < a.k) {
      id = a.ids[(size_t)row * a.k + thread];
      teacher = a.teacher[(size_t)row * a.k + thread];
    }
    if (a.label_weight > 0.f) label = a.labels[row];
  }
  template <typename T>
  __device__ __forceinline__ void logits(const DistillArgs& a, const T* lg) {
    if ((unsigned)id < (unsigned)a.classes) z = to_float(lg[id]);
    if ((unsigned)label < (unsigned)a.classes) z_label = to_float(lg[label]);
  }
};

// The stored entries and the label, behind the row's maximum and sums.  share[e] (LDS): what entry e takes off the gradient of its
// class, e = k for the label; id[e]: its class, -1 none.  Completes r and returns the row's loss in every thread.
template <int NT, typename T>
__device__ __forceinline__ float entries(const DistillArgs& a, float soft_scale, int row, const T* lg, const First& f, float sum_hard,
                                         float sum_soft, float* sm, float* share, int* id, Row* r) {
  using TM = Team<NT>;
  const int thread = TM::thread();
  const float inv_rows = 1.f / (float)a.rows;
  const float* t = a.teacher + (size_t)row * a.k;
  const int32_t* ids = a.ids + (size_t)row * a.k;
  float tm = -INFINITY;
  for (int e = thread; e < a.k; e += NT) {
    const int mine = e == thread ? f.id : ids[e];
    id[e] = mine < 0 ? -1 : mine;
    share[e] = mine < 0 ? -INFINITY : e == thread ? f.teacher : t[e];
    tm = fmaxf(tm, share[e] == share[e] ? share[e] : INFINITY);  // a NaN is an entry, too, and makes the sum NaN
  }
  tm = TM::over(tm, sm, Max());
  const bool has = tm != -INFINITY && a.teacher_weight > 0.f;
  float total = 0.f;
  for (int e = thread; e < a.k; e += NT) total += has ? __builtin_amdgcn_exp2f((share[e] - tm) * soft_scale) : 0.f;
  total = TM::over(total, sm, Add());
  const float log_total = __builtin_amdgcn_logf(total), log_soft = __builtin_amdgcn_logf(sum_soft);  // base 2
  const float weight = a.teacher_weight * a.temperature * inv_rows;
  float kl = 0.f;
  for (int e = thread; e < a.k; e += NT) {
    const float log_p = has ? (share[e] - tm) * soft_scale - log_total : -INFINITY;
    const float p = has ? __builtin_amdgcn_exp2f(log_p) : 0.f;
    share[e] = weight * p;
    if (id[e] >= a.classes) {
      kl = __builtin_nanf("");  // a class that does not exist: the loss says so
      id[e] = -1;
    } else if (id[e] >= 0 && p != 0.f) {
      const float z = e == thread ? f.z : to_float(lg[id[e]]);
      kl += p * (log_p - (r->power(z) - log_soft));
    }
  }
  kl = TM::over(kl, sm, Add()) * kLn2;
  float loss = a.teacher_weight > 0.f ? a.teacher_weight * a.temperature * a.temperature * kl : 0.f;
  if (a.label_weight > 0.f) {
    const bool known = (unsigned)f.label < (unsigned)a.classes;
    const float ce = known ? __builtin_amdgcn_logf(sum_hard) - r->power(f.z_label) * r->to_hard : __builtin_nanf("");
    loss += a.label_weight * kLn2 * ce;
    if (thread == 0) {
      id[a.k] = known ? f.label : -1;
      share[a.k] = a.label_weight * inv_rows;
    }
  } else if (thread == 0) {
    id[a.k] = -1;
  }
  r->hard = a.label_weight > 0.f ? a.label_weight * inv_rows / sum_hard : 0.f;
  r->soft = has ? weight / sum_soft : 0.f;
  return loss;
}

// The gradient of the entries' classes, behind the stores of the others: the first entry of a class takes off what all of it do.
template <int NT, typename T>
__device__ __forceinline__ void finish_entries(const DistillArgs& a, const T* lg, T* dl, const Row& r, const float* share, const int* id) {
  for (int e = Team<NT>::thread(); e <= a.k; e += NT) {
    const int mine = id[e];
    if (mine < 0) continue;
    float off = 0.f;
    bool first = true;
    for (int f = 0; f <= a.k; ++f)
      if (id[f] == mine) {
        first = first && f >= e;
        off += share[f];
      }
    if (first) dl[mine] = from_float<T>(r.gradient(to_float(lg[mine])) - off);
  }
}

// The mean of the row losses by the workgroup that arrives last, where a counter is given.
__device__ __forceinline__ void finish_mean(const DistillArgs& a) {
  __shared__ double sums[256];
  __shared__ int finishes;
  if (!a.counter) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's row losses have arrived
  __syncthreads();
  if (threadIdx.x == 0) finishes = last_to_arrive(a.counter, gridDim.x);
  __syncthreads();
  if (!finishes) return;
  if (threadIdx.x < 256) {
    double s = 0.0;
    for (int i = threadIdx.x; i < a.rows; i += 256) s += (double)published(a.row_loss + i);
    sums[threadIdx.x] = s;
  }
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) sums[threadIdx.x] += sums[threadIdx.x + w];
    __syncthreads();
  }
  if (threadIdx.x == 0) *a.loss = (float)(sums[0] / (double)a.rows);
}

// A value of which the compiler forgets what has been worked out from it before, and holds none of that.
__device__ __forceinline__ float afresh(float v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Which exponentials a row needs.  kOne: of one scale (the teacher or the labels alone, or a temperature of 1), held in the logits' place from the
// second step on; kTwo: both, whose power is held and whose exponentials are formed for the sums and again for the gradient.  8192 x 32000 in
// bf16: 217 us with one, 278 with two (holding both, which leaves a SIMD one wave, 407).
enum Exponentials : int { kOne = 0, kTwo = 1 };

// A row is read once and held in registers, HELD units of 16 bytes for each of its NT threads, and written once.
// Rows may start at any element: units lie at 16-byte addresses, and the first and last, which other rows share, are read and written one
// by one.  Reading and writing at the rate of a copy is the floor (218 us at 8192 x 32000); what comes near it is instructions, an exponential
// taking a wave 16 cycles and any other 4.
template <typename T, int NT, int HELD, int EXPS>
__global__ __launch_bounds__(Team<NT>::kThreads, HELD * kVec<T> == 64 ? 4 : 1) void distill_held_kernel(DistillArgs a) {
  using TM = Team<NT>;
  constexpr int V = kVec<T>;
  __shared__ float sm_all[TM::kThreads / 64];
  extern __shared__ float entry_lds[];  // for each row [k + 1] shares, [k + 1] classes
  const int thread = TM::thread(), row = a.first_row + blockIdx.x * TM::kRows + TM::which();
  float* sm = sm_all;
  float* share = entry_lds + TM::which() * 2 * (a.k + 1);
  int* id = reinterpret_cast<int*>(share + a.k + 1);
  const float soft_scale = kLog2e / a.temperature;
  if (row < a.rows) {
    const T* lg = (const T*)a.logits + (size_t)row * a.classes;
    T* dl = (T*)a.dlogits + (size_t)row * a.classes;
    const int lead = (int)((uintptr_t)lg % 16 / sizeof(T));  // values of the first unit that are another row's
    const int whole_from = lead > 0, whole_to = (lead + a.classes) / V;  // units that are this row's alone
    const int units = (lead + a.classes + V - 1) / V;
    const T* unit0 = lg - lead;
    First entry(a, row, thread);
    uint4 raw[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int u = min(max(thread + NT * i, whole_from), whole_to - 1);
      raw[i] = *reinterpret_cast<const uint4*>(unit0 + (size_t)u * V);
    }
    entry.logits(a, lg);
    float x[HELD][V];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int u = thread + NT * i;
      unpack<T>(raw[i], x[i]);
      if (u < whole_from || u >= whole_to) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int j = u * V + e - lead;
          x[i][e] = u < units && j >= 0 && j < a.classes ? to_float(lg[j]) : -INFINITY;
        }
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) top = fmaxf(top, x[i][e]);
    top = TM::over(top, sm, Max());
    Row r(a, soft_scale, top);
    if (r.base != 0.f) {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) x[i][e] -= r.base;
    }
    float soft = 0.f, hard = 0.f;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float power = r.power_of_rest(x[i][e]), one = __builtin_amdgcn_exp2f(power);
        soft += one;
        if constexpr (EXPS == kTwo) {
          hard += __builtin_amdgcn_exp2f(power * r.to_hard);
          x[i][e] = power;
        } else {
          x[i][e] = one;
        }
      }
    soft = TM::over(soft, sm, Add());
    hard = EXPS == kOne ? soft : TM::over(hard, sm, Add());
    const float loss = entries<NT>(a, soft_scale, row, lg, entry, hard, soft, sm, share, id, &r);
    if (thread == 0) publish(a.row_loss + row, loss);
    const float one = r.soft + r.hard;  // kOne: both are of the same exponential
    if (EXPS == kOne && one == 0.f) {   // a row without a term (a padded one, say) has no gradient, whatever its logits hold
#pragma unroll
      for (int i = 0; i < HELD; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) x[i][e] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int u = thread + NT * i;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if constexpr (EXPS == kOne) {
          x[i][e] *= one;
        } else {
          const float power = afresh(x[i][e]);
          x[i][e] = fmaf(r.hard, __builtin_amdgcn_exp2f(power * r.to_hard), r.soft * __builtin_amdgcn_exp2f(power));
        }
      }
      if (u >= whole_from && u < whole_to) {
        *reinterpret_cast<uint4*>(dl - lead + (size_t)u * V) = pack<T>(x[i]);
      } else if (u < units) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int j = u * V + e - lead;
          if (j >= 0 && j < a.classes) dl[j] = from_float<T>(x[i][e]);
        }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the row is stored before single values of it are replaced
    TM::sync();
    finish_entries<NT>(a, lg, dl, r, share, id);
  }
  finish_mean(a);
}

// Any row, read three times by a workgroup of its own.
constexpr int kThreads = 256;
template <typename T>
__global__ __launch_bounds__(kThreads) void distill_rows_kernel(DistillArgs a) {
  __shared__ float sm[kThreads / 64];
  extern __shared__ float entry_lds[];
  float* share = entry_lds;
  int* id = reinterpret_cast<int*>(share + a.k + 1);
  const float soft_scale = kLog2e / a.temperature;
  const bool labels = a.label_weight > 0.f;
  for (long at = blockIdx.x; at < a.rows; at += gridDim.x) {
    const int row = (int)at;
    const T* lg = (const T*)a.logits + (size_t)row * a.classes;
    T* dl = (T*)a.dlogits + (size_t)row * a.classes;
    First entry(a, row, threadIdx.x);
    entry.logits(a, lg);
    float top = -INFINITY;
    for (int j = threadIdx.x; j < a.classes; j += kThreads) top = fmaxf(top, to_float(lg[j]));
    top = Team<kThreads>::over(top, sm, Max());
    Row r(a, soft_scale, top);
    float hard = 0.f, soft = 0.f;
    for (int j = threadIdx.x; j < a.classes; j += kThreads) {
      const float power = r.power(to_float(lg[j]));
      soft += __builtin_amdgcn_exp2f(power);
      if (labels) hard += __builtin_amdgcn_exp2f(power * r.to_hard);
    }
    soft = Team<kThreads>::over(soft, sm, Add());
    if (labels) hard = Team<kThreads>::over(hard, sm, Add());
    const float loss = entries<kThreads>(a, soft_scale, row, lg, entry, hard, soft, sm, share, id, &r);
    if (threadIdx.x == 0) publish(a.row_loss + row, loss);
    for (int j = threadIdx.x; j < a.classes; j += kThreads) dl[j] = from_float<T>(r.gradient(to_float(lg[j])));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the row is stored before single values of it are replaced
    __syncthreads();
    finish_entries<kThreads>(a, lg, dl, r, share, id);
    __syncthreads();  // the entries' LDS is free
  }
  finish_mean(a);
}

constexpr int kCounted = 128;  // workgroups up to which the last of them forms the mean; more take a launch of its own
constexpr int kMeanThreads = 1024;
__global__ __launch_bounds__(kMeanThreads) void distill_mean_kernel(const float* __restrict__ row_loss, int rows, float* __restrict__ loss) {
  __shared__ double sums[kMeanThreads / 64];
  double s = 0.0;
  long i = threadIdx.x;
  for (; i + 7 * kMeanThreads < rows; i += 8 * kMeanThreads) {  // eight loads on their way
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = row_loss[i + u * kMeanThreads];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += (double)v[u];
  }
  for (; i < rows; i += kMeanThreads) s += (double)row_loss[i];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < kMeanThreads / 64; ++w) s += sums[w];
    *loss = (float)(s / (double)rows);
  }
}
hipError_t finish(hipStream_t s, const DistillArgs& a) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.counter) return e;
  hipLaunchKernelGGL(distill_mean_kernel, dim3(1), dim3(kMeanThreads), 0, s, a.row_loss, a.rows, a.loss);
  return hipGetLastError();
}

template <typename T, int NT, int HELD>
hipError_t launch_held(hipStream_t s, DistillArgs a) {
  using TM = Team<NT>;
  const long blocks = ((long)a.rows + TM::kRows - 1) / TM::kRows;
  if (blocks > kCounted) a.counter = nullptr;
  const size_t lds = (size_t)TM::kRows * 2 * (a.k + 1) * sizeof(float);
  const bool one = a.label_weight <= 0.f || a.teacher_weight <= 0.f || a.temperature == 1.f;
  auto kernel = one ? distill_held_kernel<T, NT, HELD, kOne> : distill_held_kernel<T, NT, HELD, kTwo>;
  // a launch takes fewer than 2^32 threads, and drops what a grid has beyond
  const long most = UINT32_MAX / TM::kThreads;
  for (long from = 0; from < blocks; from += most) {
    a.first_row = (int)(from * TM::kRows);
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(most, blocks - from)), dim3(TM::kThreads), lds, s, a);
  }
  return finish(s, a);
}

template <typename T>
hipError_t launch(hipStream_t s, DistillArgs a) {
  constexpr int V = kVec<T>;
  const long units = a.classes / V + 2;  // with a first and a last one that are shared
  // whole units to hold, and rows that start at the same place in a unit on both sides
  if (a.classes >= 2 * V && ((uintptr_t)a.logits - (uintptr_t)a.dlogits) % 16 == 0) {
    constexpr int W = 64 / V;  // units of 64 values
    if (units <= 64) return launch_held<T, 64, 1>(s, a);
    if (units <= 64 * 2) return launch_held<T, 64, 2>(s, a);
    if (units <= 256) return launch_held<T, 256, 1>(s, a);
    if (units <= 256 * W / 4) return launch_held<T, 256, W / 4>(s, a);
    if (units <= 256 * W / 2) return launch_held<T, 256, W / 2>(s, a);
    if (units <= 256 * W) return launch_held<T, 256, W>(s, a);
    if (units <= 512 * W) return launch_held<T, 512, W>(s, a);
    if (units <= 1024 * W) return launch_held<T, 1024, W>(s, a);
  }
  const int blocks = std::min(a.rows, 1 << 20);
  if (blocks > kCounted) a.counter = nullptr;
  hipLaunchKernelGGL(distill_rows_kernel<T>, dim3(blocks), dim3(kThreads), (size_t)2 * (a.k + 1) * sizeof(float), s, a);
  return finish(s, a);
}

}  // namespace

hipError_t launch_distill(hipStream_t s, int elt, const DistillArgs& a) { return elt == ELT_BF16 ? launch<uint16_t>(s, a) : launch<float>(s, a); }

}  // namespace tp
