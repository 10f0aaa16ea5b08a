// What the kernels of windowed attention share.  Everything lives in an unnamed namespace: each translation unit has its own copy.
#pragma once
#include <hip/hip_runtime.h>

#include "local_attention.h"

namespace tp {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Shape {
  int S, heads, kv, dh, window, sinks;
  __host__ __device__ __forceinline__ size_t ld() const { return (size_t)(heads + 2 * kv) * dh; }
  __device__ __forceinline__ bool sees(int i, int j) const { return j <= i && (i - j < window || j < sinks); }
};
inline Shape shape_of(const LocalAttention& a) { return Shape{a.S, a.heads, a.kv, a.dh, a.window, a.sinks}; }

// Bucket of a distance >= 0: a first guess from the logarithm, then to the borders (one step at most, borders that coincide aside).
// first: the borders in LDS.
__device__ __forceinline__ int bucket_of(const DistanceBuckets& d, const int* first, int distance) {
  if (distance < d.half) return distance;
  int b = min(d.count - 1, d.half + (int)(__builtin_amdgcn_logf((float)distance / (float)d.half) * d.ratio));
  while (distance < first[b]) --b;
  while (b + 1 < d.count && distance >= first[b + 1]) ++b;
  return b;
}

}  // namespace

// On the matrix cores (kernels_local_mfma.hip): heads of up to 128 values in whole 16-byte units, tensors at 16-byte addresses.
bool local_mfma_supported(int elt, const LocalAttention& a);
hipError_t local_mfma_fwd(hipStream_t s, int elt, const LocalAttention& a, const void* x, const float* table, float* kept, void* out, void* out2,
                          float* lse);
// partials: local_mfma_table_rows() rows of [heads][buckets]; scratch: local_mfma_scratch_bytes()
hipError_t local_mfma_bwd(hipStream_t s, int elt, const LocalAttention& a, const void* x, const void* out, const void* dout, const float* lse,
                          const float* kept, void* dx, float* partials, void* scratch);
size_t local_mfma_scratch_bytes(int elt, const LocalAttention& a);
int local_mfma_table_rows(int elt, const LocalAttention& a);

}  // namespace tp
