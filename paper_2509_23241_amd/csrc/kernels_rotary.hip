// Rotary positions: pair i of a head at position p is turned by the angle t = p * speed_i,
//   (u, v) -> a (u cos t - v sin t, u sin t + v cos t),  backward (the transposed turn) with -t.
// Memory carries it: a read and a write of the queries and keys, and of the values where the output lies elsewhere.  The sines and
// cosines are formed once for a workgroup's positions and used for all their heads.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "device_utils.h"
#include "kernels.h"
#include "rotary.h"

namespace tp {

namespace {

constexpr int kThreads = 256;

// a cos t and a sin t of `turns` whole turns per position.  The angle is reduced in fp64 to an eighth of a turn either way, where its
// rounding to fp32 is 2^-25 of a quarter turn at most.  In fp64 it is off by 2^-51 of itself: less than 2^-24 up to positions of 2^27, 10^-6 at 2^31.
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

// ---- heads and their parts in whole units of 16 or 8 bytes -------------------------------------
// A workgroup takes some tokens: sines and cosines go into LDS, one or a few a thread, while the first units are on their way; every
// thread then turns several items at a time, all of them loaded before the first is used.  An item is two units of halves, whose values are
// pairs across them, or one unit of neighbours.  What is not turned is copied likewise where the output lies elsewhere.  Value by value
// (the kernel above) the same 8192 tokens take 127 us.
struct RotaryShape {
  int tokens;      // of a workgroup
  int units;       // of a token
  int head_units;  // of a head
  int items;       // of a head
  int rest;        // units of a turned head that are not turned
  uint32_t by_items, by_turned, by_copies, by_rest;  // multipliers that divide by .., heads that are turned, units of a token that are copied, ..
};
// n / d by the multiplier of divisor(d), exact for n * d < 2^32
inline uint32_t divisor(int d) { return d <= 1 ? 0u : (uint32_t)(((1ull << 32) + d - 1) / d); }
__device__ __forceinline__ int divided(int n, uint32_t mul) { return mul ? (int)__umulhi((uint32_t)n, mul) : n; }
constexpr int kTurns = 1024;  // pairs of a workgroup's tokens

// (an array of uint4 written under a condition stays in memory)
template <int BYTES>
struct UnitOf {
  typedef uint32_t kept __attribute__((ext_vector_type(BYTES / 4)));
  typedef std::conditional_t<BYTES == 16, uint4, uint2> type;
};
template <typename T, int BYTES>
__device__ __forceinline__ void values_of(const typename UnitOf<BYTES>::type& u, float (&v)[BYTES / sizeof(T)]) {
#pragma unroll
  for (int i = 0; i < BYTES / 4; ++i) {
    const uint32_t w = reinterpret_cast<const uint32_t*>(&u)[i];
    if constexpr (sizeof(T) == 2) {
      v[2 * i] = __uint_as_float(w << 16);
      v[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
    } else {
      v[i] = __uint_as_float(w);
    }
  }
}
template <typename T, int BYTES>
__device__ __forceinline__ typename UnitOf<BYTES>::type unit_of(const float (&v)[BYTES / sizeof(T)]) {
  uint32_t w[BYTES / 4];
#pragma unroll
  for (int i = 0; i < BYTES / 4; ++i) {
    if constexpr (sizeof(T) == 2) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    else w[i] = __float_as_uint(v[i]);
  }
  if constexpr (BYTES == 16) return make_uint4(w[0], w[1], w[2], w[3]);
  else return make_uint2(w[0], w[1]);
}

template <typename T, int BYTES, bool HALVES, bool COPY>
__global__ __launch_bounds__(kThreads) void rotary_units_kernel(Rotary r, RotaryShape sh, RotarySpeeds speeds, bool back, const T* x, T* out) {
  using unit_t = typename UnitOf<BYTES>::type;
  using kept_t = typename UnitOf<BYTES>::kept;
  constexpr int V = BYTES / sizeof(T), ITEMS = HALVES ? 4 : 8;
  __shared__ float2 turn[kTurns];
  const int half = r.rotated / 2;
  const long token0 = (long)blockIdx.x * sh.tokens;
  const int tokens = (int)min((long)sh.tokens, (long)r.seqs * r.S - token0);
  const unit_t* from = reinterpret_cast<const unit_t*>(x) + token0 * sh.units;
  unit_t* to = reinterpret_cast<unit_t*>(out) + token0 * sh.units;
  // what is copied: a batch of it is under way while the turns are made, the rest follows them
  const int values = sh.units - r.turned * sh.head_units, copies = COPY ? tokens * (values + r.turned * sh.rest) : 0;
  auto copied = [&](int i) {
    const int token = divided(i, sh.by_copies), u = i - token * (values + r.turned * sh.rest), head = divided(max(u - values, 0), sh.by_rest);
    return token * sh.units + (u < values ? r.turned * sh.head_units + u : (head + 1) * sh.head_units - sh.rest + u - values - head * sh.rest);
  };
  constexpr int BATCH = COPY ? 4 : 1;
  kept_t kept[BATCH];
  if constexpr (COPY) {
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = k * kThreads + (int)threadIdx.x;
      kept[k] = i < copies ? *reinterpret_cast<const kept_t*>(from + copied(i)) : kept_t(0);
    }
  }
  const int items = tokens * r.turned * sh.items, other = half / V;
  for (int i0 = 0; i0 < items; i0 += kThreads * ITEMS) {
    unit_t a[ITEMS], b[HALVES ? ITEMS : 1];
    int unit[ITEMS], at[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int i = i0 + k * kThreads + (int)threadIdx.x;
      const int head_of_all = divided(i, sh.by_items), item = i - head_of_all * sh.items;
      const int token = divided(head_of_all, sh.by_turned), head = head_of_all - token * r.turned;
      unit[k] = token * sh.units + head * sh.head_units + item;
      at[k] = token * half + item * (HALVES ? V : V / 2);
      if (i < items) {
        a[k] = from[unit[k]];
        if constexpr (HALVES) b[k] = from[unit[k] + other];
      }
    }
    if (i0 == 0) {
      for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
        const int token = i / half, pair = i - token * half;
        turn[i] = turn_of(speeds.turns[pair], r.first + (int)((token0 + token) % r.S), r.amplitude, back);
      }
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      if (i0 + k * kThreads + (int)threadIdx.x < items) {
        float u[V], p[V];
        values_of<T, BYTES>(a[k], u);
        if constexpr (HALVES) {
          float v[V], q[V];
          values_of<T, BYTES>(b[k], v);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float2 t = turn[at[k] + e];
            p[e] = u[e] * t.x - v[e] * t.y;
            q[e] = u[e] * t.y + v[e] * t.x;
          }
          to[unit[k] + other] = unit_of<T, BYTES>(q);
        } else {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const float2 t = turn[at[k] + e / 2];
            p[e] = u[e] * t.x - u[e + 1] * t.y;
            p[e + 1] = u[e] * t.y + u[e + 1] * t.x;
          }
        }
        to[unit[k]] = unit_of<T, BYTES>(p);
      }
    }
  }
  if constexpr (COPY) {
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = k * kThreads + (int)threadIdx.x;
      if (i < copies) *reinterpret_cast<kept_t*>(to + copied(i)) = kept[k];
    }
    for (int i = BATCH * kThreads + (int)threadIdx.x; i < copies; i += kThreads) {
      const int u = copied(i);
      to[u] = from[u];
    }
  }
}

// Rotary layers whose parts of heads are whole units at their addresses; false: others, and tokens of too many units for the divisions.
template <typename T, int BYTES>
bool launch_units(hipStream_t s, const Rotary& r, const RotarySpeeds& speeds, bool back, const T* x, T* out) {
  constexpr int V = BYTES / sizeof(T);
  const int half = r.rotated / 2;
  if (r.dh % V || (r.halves ? half : r.rotated) % V || (((uintptr_t)x | (uintptr_t)out) & (BYTES - 1))) return false;
  const long all = (long)r.seqs * r.S, units = (long)r.all * r.dh / V;
  // Four units a thread, as long as that leaves every CU two workgroups.  8192 tokens of 768 units, both ways with the values copied: 79 us with one token a
  // workgroup (403 MB, at 5.1 TB/s the rate of a copy), 95 with two, 112 with four; 3108 tokens of 200 units 15.4 with five, 22 with one.
  const long tokens = std::max<long>(1, std::min({all / 512, 1024 / units, (long)kTurns / half}));
  if ((tokens * units + 8 * kThreads) * units >= (1l << 32)) return false;
  RotaryShape sh;
  sh.tokens = (int)tokens;
  sh.units = (int)units;
  sh.head_units = r.dh / V;
  sh.items = (r.halves ? half : r.rotated) / V;
  sh.rest = (r.dh - r.rotated) / V;
  const int copies = sh.units - r.turned * sh.head_units + r.turned * sh.rest;
  sh.by_items = divisor(sh.items);
  sh.by_turned = divisor(r.turned);
  sh.by_copies = divisor(copies);
  sh.by_rest = divisor(sh.rest);
  auto go = [&](auto halves, auto copy) {
    // (a workgroup with a token or a thousand units has 4 KB and more: the 2^24 that a launch takes have more than there is)
    hipLaunchKernelGGL((rotary_units_kernel<T, BYTES, decltype(halves)::value, decltype(copy)::value>), dim3((unsigned)((all + tokens - 1) / tokens)),
                       dim3(kThreads), 0, s, r, sh, speeds, back, x, out);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  const bool copy = x != out;
  if (r.halves) copy ? go(Yes(), Yes()) : go(Yes(), No());
  else copy ? go(No(), Yes()) : go(No(), No());
  return true;
}

template <typename T>
hipError_t launch(hipStream_t s, const Rotary& r, const RotarySpeeds& speeds, bool back, const T* x, T* out) {
  if (!launch_units<T, 16>(s, r, speeds, back, x, out) && !launch_units<T, 8>(s, r, speeds, back, x, out)) {
    const unsigned blocks = (unsigned)std::min<long>((long)r.seqs * r.S, 1 << 20);
    hipLaunchKernelGGL(rotary_any_kernel<T>, dim3(blocks), dim3(kThreads), 0, s, r, speeds, back, x, out);
  }
  return hipGetLastError();
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
  if (elt == ELT_BF16) return launch<uint16_t>(s, r, speeds, back, (const uint16_t*)x, (uint16_t*)out);
  return launch<float>(s, r, speeds, back, (const float*)x, (float*)out);
}

}  // namespace tp
