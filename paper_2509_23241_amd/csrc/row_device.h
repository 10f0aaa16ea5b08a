// Device code shared by the losses on rows of logits: the threads of a row and its 16-byte units.  Everything lives in an unnamed
// namespace: each translation unit that includes this header gets its own copy.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_utils.h"

namespace tp {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// The threads of a row: a quarter or half of a wave, a wave, or a whole workgroup.
template <int NT>
struct Team {
  static_assert(NT >= 16, "lanes of a row of 16 meet by rotations of it");
  static constexpr int kRows = NT <= 64 ? 256 / NT : 1;  // rows of a workgroup
  static constexpr int kThreads = NT <= 64 ? 256 : NT;
  static __device__ __forceinline__ int thread() { return NT <= 64 ? threadIdx.x & (NT - 1) : threadIdx.x; }
  static __device__ __forceinline__ int which() { return NT <= 64 ? threadIdx.x / NT : 0; }
  // what the others have written to LDS and memory is there
  static __device__ __forceinline__ void sync() {
    if constexpr (NT <= 64) {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
      __syncthreads();
    }
  }
  // sm: NT / 64 floats, free on both sides
  template <class Op>
  static __device__ __forceinline__ float over(float v, float* sm, const Op& op) {
    v = over_lanes<(NT < 64 ? NT / 2 : 32)>(v, op);
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
};

template <typename T>
constexpr int kVec = 16 / sizeof(T);  // values of a 16-byte unit
template <typename T>
__device__ __forceinline__ void unpack(const uint4& u, float (&v)[kVec<T>]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      v[i] = __uint_as_float(w[i]);
    }
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float (&v)[kVec<T>]) {
  if constexpr (sizeof(T) == 2)
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  else
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}

}  // namespace

}  // namespace tp
