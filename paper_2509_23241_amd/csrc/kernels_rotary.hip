// Rotary positions: pair i of a head at position p is turned by the angle t = p * speed_i,
//   (u, v) -> a (u cos t - v sin t, u sin t + v cos t),  backward (the transposed turn) with -t.
// Memory carries it: a read and a write of the queries and keys, and of the values where the output lies elsewhere.  The sines and
// cosines are formed once for a workgroup's positions and used for all their heads.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "device_utils.h"
#include "kernels.h"
#include "rotary.h"

namespace tp {

namespace {

constexpr int kThreads = 256;

// a cos t and a sin t of `turns` whole turns per position.  The angle is reduced in fp64 to an eighth of a turn either way, where its
// rounding to fp32 is 2^-25 of a quarter turn at most: positions up to 2^31 keep 2^-24 and the function's own error.
__device__ __forceinline__ float2 turn_of(double turns, int position, float amplitude, bool back) {
  const double quarters = 4.0 * (turns * (double)position);
  const double whole = rint(quarters);
  float s, c;
  sincospif(0.5f * (float)(quarters - whole), &s, &c);
  const int q = (int)(whole - 4.0 * floor(whole * 0.25));  // 0 .. 3
  const float cs = q == 0 ? c : q == 1 ? -s : q == 2 ? -c : s;
  const float sn = q == 0 ? s : q == 1 ? c : q == 2 ? -s : -c;
  return make_float2(amplitude * cs, amplitude * (back ? -sn : sn));
}

// Any width and address, value by value, a workgroup a token.
template <typename T>
__global__ __launch_bounds__(kThreads) void rotary_any_kernel(Rotary r, RotarySpeeds speeds, bool back, const T* x, T* out) {
  __shared__ float2 turn[kMaxRotaryPairs];
  const int half = r.rotated / 2;
  const size_t row = (size_t)r.all * r.dh;
  for (long token = blockIdx.x; token < (long)r.seqs * r.S; token += gridDim.x) {
    if (threadIdx.x < half) turn[threadIdx.x] = turn_of(speeds.turns[threadIdx.x], r.first + (int)(token % r.S), r.amplitude, back);
    __syncthreads();
    const T* from = x + token * row;
    T* to = out + token * row;
    for (int i = threadIdx.x; i < r.turned * half; i += kThreads) {
      const int head = i / half, pair = i % half;
      const int u = head * r.dh + (r.halves ? pair : 2 * pair), v = u + (r.halves ? half : 1);
      const float a = to_float(from[u]), b = to_float(from[v]);
      const float2 t = turn[pair];
      to[u] = from_float<T>(a * t.x - b * t.y);
      to[v] = from_float<T>(a * t.y + b * t.x);
    }
    if (from != to) {
      const int rest = r.dh - r.rotated;
      for (int i = threadIdx.x; i < r.turned * rest; i += kThreads) {
        const int at = i / rest * r.dh + r.rotated + i % rest;
        to[at] = from[at];
      }
      for (size_t i = (size_t)r.turned * r.dh + threadIdx.x; i < row; i += kThreads) to[i] = from[i];
    }
    __syncthreads();
  }
}

}  // namespace

void rotary_speeds(int rotated, double base, double factor, double original, double low, double high, RotarySpeeds* out) {
  const double two_pi = 6.283185307179586476925286766559;
  for (int i = 0; i < kMaxRotaryPairs; ++i) {
    if (i >= rotated / 2) {
      out->turns[i] = 0.0;
      continue;
    }
    const double s = pow(base, -2.0 * i / rotated);
    double speed = s / factor;
    if (original > 0.0) {
      const double g = std::min(1.0, std::max(0.0, (original * s / two_pi - low) / (high - low)));
      speed = s * ((1.0 - g) / factor + g);
    }
    out->turns[i] = speed / two_pi;
  }
}

hipError_t launch_rotary(hipStream_t s, int elt, const Rotary& r, const RotarySpeeds& speeds, bool back, const void* x, void* out) {
  const unsigned blocks = (unsigned)std::min<long>((long)r.seqs * r.S, 1 << 20);
  if (elt == ELT_BF16)
    hipLaunchKernelGGL(rotary_any_kernel<uint16_t>, dim3(blocks), dim3(kThreads), 0, s, r, speeds, back, (const uint16_t*)x, (uint16_t*)out);
  else
    hipLaunchKernelGGL(rotary_any_kernel<float>, dim3(blocks), dim3(kThreads), 0, s, r, speeds, back, (const float*)x, (float*)out);
  return hipGetLastError();
}

}  // namespace tp
