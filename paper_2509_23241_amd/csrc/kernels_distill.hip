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

namespace tp {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

template <int NT, class Op>
__device__ __forceinline__ float over_block(float v, float* sm, const Op& op) {  // sm: NT / 64 floats, free on both sides
  v = over_lanes<32>(v, op);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sm[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) v = op(v, sm[i]);
    __syncthreads();
  }
  return v;
}

// What a row's sums come to, and the terms of its loss and gradient that belong to single classes
struct Row {
  float top;           // max z
  float hard, soft;    // what exp(z - top) and exp((z - top) / T) are multiplied with in the gradient
};

// The stored entries and the label, behind the row's maximum and sums.  share[e] (LDS): what entry e takes off the gradient of its
// class, e = k for the label; id[e]: its class, -1 none.  Returns the row's loss in every thread of the block.
template <int NT, typename T>
__device__ __forceinline__ float entries(const DistillArgs& a, int row, const T* lg, float top, float sum_hard, float sum_soft, float* sm,
                                         float* share, int* id, Row* r) {
  const float inv_t = 1.f / a.temperature, inv_rows = 1.f / (float)a.rows;
  const float* t = a.teacher + (size_t)row * a.k;
  const int32_t* ids = a.ids + (size_t)row * a.k;
  float tm = -INFINITY;
  for (int e = threadIdx.x; e < a.k; e += NT) {
    id[e] = ids[e] < 0 ? -1 : ids[e];
    share[e] = ids[e] < 0 ? -INFINITY : t[e];
    tm = fmaxf(tm, share[e] == share[e] ? share[e] : INFINITY);  // a NaN is an entry, too, and makes the sum NaN
  }
  tm = over_block<NT>(tm, sm, Max());
  const bool has = tm != -INFINITY && a.label_weight < 1.f;
  float total = 0.f;
  for (int e = threadIdx.x; e < a.k; e += NT) total += has ? expf((share[e] - tm) * inv_t) : 0.f;
  total = over_block<NT>(total, sm, Add());
  const float log_total = logf(total), log_soft = logf(sum_soft);
  const float c = (1.f - a.label_weight) * a.temperature * inv_rows;
  float kl = 0.f;
  for (int e = threadIdx.x; e < a.k; e += NT) {
    const float log_p = has ? (share[e] - tm) * inv_t - log_total : -INFINITY;
    const float p = has ? expf(log_p) : 0.f;
    share[e] = c * p;
    if (id[e] >= a.classes) {
      kl = __builtin_nanf("");  // a class that does not exist: the loss says so
      id[e] = -1;
    } else if (id[e] >= 0 && p != 0.f) {
      kl += p * (log_p - ((to_float(lg[id[e]]) - top) * inv_t - log_soft));
    }
  }
  kl = over_block<NT>(kl, sm, Add());
  float loss = a.label_weight < 1.f ? (1.f - a.label_weight) * a.temperature * a.temperature * kl : 0.f;
  if (a.label_weight > 0.f) {
    const int label = a.labels[row];
    const bool known = (unsigned)label < (unsigned)a.classes;
    loss += a.label_weight * (known ? logf(sum_hard) - (to_float(lg[label]) - top) : __builtin_nanf(""));
    if (threadIdx.x == 0) {
      id[a.k] = known ? label : -1;
      share[a.k] = a.label_weight * inv_rows;
    }
  } else if (threadIdx.x == 0) {
    id[a.k] = -1;
  }
  r->top = top;
  r->hard = a.label_weight > 0.f ? a.label_weight * inv_rows / sum_hard : 0.f;
  r->soft = has ? c / sum_soft : 0.f;
  return loss;
}

__device__ __forceinline__ float gradient(const Row& r, float z, float inv_t_log2, bool labels) {
  const float x = z - r.top;
  float g = r.soft * __builtin_amdgcn_exp2f(x * inv_t_log2);
  if (labels) g = fmaf(r.hard, __builtin_amdgcn_exp2f(x * kLog2e), g);
  return g;
}

// The gradient of the entries' classes, behind the stores of the others: the first entry of a class takes off what all of it do.
template <int NT, typename T>
__device__ __forceinline__ void finish_entries(const DistillArgs& a, const T* lg, T* dl, const Row& r, float inv_t_log2, const float* share,
                                               const int* id) {
  const bool labels = a.label_weight > 0.f;
  for (int e = threadIdx.x; e <= a.k; e += NT) {
    const int mine = id[e];
    if (mine < 0) continue;
    float off = 0.f;
    bool first = true;
    for (int f = 0; f <= a.k; ++f)
      if (id[f] == mine) {
        first = first && f >= e;
        off += share[f];
      }
    if (first) dl[mine] = from_float<T>(gradient(r, to_float(lg[mine]), inv_t_log2, labels) - off);
  }
}

// A workgroup per row, which is read three times.
template <typename T>
__global__ __launch_bounds__(kThreads) void distill_rows_kernel(DistillArgs a) {
  __shared__ float sm[kThreads / 64];
  extern __shared__ float entry_lds[];  // [k + 1] shares, [k + 1] classes
  float* share = entry_lds;
  int* id = reinterpret_cast<int*>(share + a.k + 1);
  const float inv_t_log2 = kLog2e / a.temperature;
  const bool labels = a.label_weight > 0.f;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* lg = (const T*)a.logits + (size_t)row * a.classes;
    T* dl = (T*)a.dlogits + (size_t)row * a.classes;
    float top = -INFINITY;
    for (int j = threadIdx.x; j < a.classes; j += kThreads) top = fmaxf(top, to_float(lg[j]));
    top = over_block<kThreads>(top, sm, Max());
    float hard = 0.f, soft = 0.f;
    for (int j = threadIdx.x; j < a.classes; j += kThreads) {
      const float x = to_float(lg[j]) - top;
      soft += __builtin_amdgcn_exp2f(x * inv_t_log2);
      if (labels) hard += __builtin_amdgcn_exp2f(x * kLog2e);
    }
    soft = over_block<kThreads>(soft, sm, Add());
    if (labels) hard = over_block<kThreads>(hard, sm, Add());
    Row r;
    const float loss = entries<kThreads>(a, row, lg, top, hard, soft, sm, share, id, &r);
    if (threadIdx.x == 0) publish(a.row_loss + row, loss);
    for (int j = threadIdx.x; j < a.classes; j += kThreads) dl[j] = from_float<T>(gradient(r, to_float(lg[j]), inv_t_log2, labels));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the row is stored before single values of it are replaced
    __syncthreads();
    finish_entries<kThreads>(a, lg, dl, r, inv_t_log2, share, id);
    __syncthreads();  // the entries' LDS is free
  }
}

}  // namespace

hipError_t launch_distill(hipStream_t s, int elt, const DistillArgs& a) {
  const size_t lds = (size_t)2 * (a.k + 1) * sizeof(float);
  const int blocks = std::min(a.rows, 1 << 20);
  if (elt == ELT_BF16) hipLaunchKernelGGL(distill_rows_kernel<uint16_t>, dim3(blocks), dim3(kThreads), lds, s, a);
  else hipLaunchKernelGGL(distill_rows_kernel<float>, dim3(blocks), dim3(kThreads), lds, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_mean(s, a.row_loss, a.rows, a.loss);
}

}  // namespace tp
