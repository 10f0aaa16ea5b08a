// Windowed attention on the matrix cores, bf16 and fp32, for heads of up to 128 values in whole 16-byte units.
//
// A wave owns 32 rows -- queries in the forward pass and for dQ, keys for dK and dV -- with their fragments in registers, and walks over
// blocks of the other side, which its workgroup copies global -> LDS.  It forms the transposed score tile: MFMA rows = streamed rows,
// columns = own rows, so that a lane holds one own row (lane % 32) and 16 of a tile's 32 streamed rows, statistics of a query are scalars of
// its lane, and eight consecutive accumulator elements are the B fragment of the second product.
//   forward  S^T = K Q^T, online softmax, O^T += V^T P^T
//   dQ       S^T, dP^T = V dO^T, dS, dQ^T += K^T dS^T; leaves (lse, corrected delta) of its rows for the next launch
//   dK, dV   S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS, and the sums of dS by distance
// Own rows: a wave takes the item (block of 32 queries, query head) of its key head, heads fastest, so that the waves of a workgroup walk
// over nearly the same keys whether heads share them or not.
// Streamed tiles lie in LDS once, as panels of 128-byte rows whose 16-byte chunk c is in slot c ^ f(row), f = the bits 1, 2, 3 of the row
// number as 4, 2, 1: conflict free both for the 16-byte reads of the first products (row by row: the eight pairs of rows take all slots) and
// for the transposing reads of the second (four rows of 64 bytes: rows that are 256 bytes apart fall into different halves).
// Rows behind the last and columns behind the head's width are copied from zeros.
// Pairs that are not visible count as p = dS = 0, but a product with an infinity or NaN of their row is NaN: a wave whose result is not
// finite forms those rows again from the visible pairs alone.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "device_utils.h"
#include "kernels.h"
#include "local_attention_device.h"
#include "mfma_common.h"

namespace tp {

namespace {

constexpr float kSlack = 8.f;
constexpr float kLowest = -1e30f;  // running maximum of a row that has seen no key; scores below it are formed again, row by row
constexpr int kNear = 224;         // distances with a table entry and a sum of their own: 0 .. kNear - 1, and as far as a tile reaches beyond
constexpr int kPad = 96;           // a tile of 32 x 64 spans 95 distances
constexpr int kNearSize = kPad + kNear + kPad;

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Type;
template <>
struct Type<uint16_t> {
  static constexpr int kAhead = 4;  // fragments on their way from LDS
  using Frag = bf16x8;
  static __device__ __forceinline__ floatx16 mma(const Frag& a, const Frag& b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ bool skips(int, int) { return false; }  // one instruction: less than it takes to decide
  static __device__ __forceinline__ Frag zero() { return __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0)); }
  // P and dS enter the second products rounded to bf16, like every operand there: 2^-9 of each, on average less of their sum
  static __device__ __forceinline__ Frag pack(const float (&e)[8]) {
    return __builtin_bit_cast(bf16x8, make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])));
  }
  using Half = uint2;
  static __device__ __forceinline__ Half half(const float (&e)[4]) { return make_uint2(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3])); }
  static __device__ __forceinline__ Frag join(const Half& a, const Half& b) { return __builtin_bit_cast(bf16x8, make_uint4(a.x, a.y, b.x, b.y)); }
  // values d .. d + 7 of a row that holds `left` more of them (a multiple of 8, or none)
  static __device__ __forceinline__ Frag load(const uint16_t* p, int left) {
    return left > 0 ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(p)) : zero();
  }
  static __device__ __forceinline__ float dot(const Frag& a, const Frag& b, float s) {
#pragma unroll
    for (int t = 0; t < 8; ++t) s = fmaf((float)a[t], (float)b[t], s);
    return s;
  }
  static __device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8], int left) {
    if (left > 0)
      *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  }
};
template <>
struct Type<float> {
  static constexpr int kAhead = 2;
  using Frag = floatx8;
  static __device__ __forceinline__ floatx16 mma(const Frag& a, const Frag& b, floatx16 c) {
#pragma unroll
    for (int t = 0; t < 8; ++t) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[t], b[t], c, 0, 0, 0);
    return c;
  }
  // A product of columns from `col` on, which are all padding: not worth its eight instructions of 64 cycles.  Heads of 32 or 80 take 15 to
  // 20 % less time for it, those of 64 or 128 2 % more for asking.
  static __device__ __forceinline__ bool skips(int col, int dh) { return col >= dh; }
  static __device__ __forceinline__ Frag zero() { return Frag{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ Frag pack(const float (&e)[8]) {
    Frag f;
#pragma unroll
    for (int t = 0; t < 8; ++t) f[t] = e[t];
    return f;
  }
  using Half = floatx4;
  static __device__ __forceinline__ Half half(const float (&e)[4]) { return floatx4{e[0], e[1], e[2], e[3]}; }
  static __device__ __forceinline__ Frag join(const Half& a, const Half& b) { return floatx8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }
  static __device__ __forceinline__ Frag load(const float* p, int left) {  // left: a multiple of 4
    Frag f = zero();
    if (left > 0) {
      const float4 a = *reinterpret_cast<const float4*>(p);
      f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    }
    if (left > 4) {
      const float4 a = *reinterpret_cast<const float4*>(p + 4);
      f[4] = a.x; f[5] = a.y; f[6] = a.z; f[7] = a.w;
    }
    return f;
  }
  static __device__ __forceinline__ float dot(const Frag& a, const Frag& b, float s) {
#pragma unroll
    for (int t = 0; t < 8; ++t) s = fmaf(a[t], b[t], s);
    return s;
  }
  static __device__ __forceinline__ void store8(float* p, const float (&v)[8], int left) {
    if (left > 0) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    if (left > 4) *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
};

// ---- a streamed tile in LDS -------------------------------------------------------------------------------------------------
__device__ __forceinline__ int swizzle(int row) { return 4 * ((row >> 1) & 1) + 2 * ((row >> 2) & 1) + ((row >> 3) & 1); }

// A value whose functions are worked out where they are used, block by block, instead of once for all in registers that there are none of.
__device__ __forceinline__ int afresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// streamed rows of a block: a tile of them takes 16 KB or less
template <typename T, int DHP>
constexpr int kBlockRows = DHP * sizeof(T) <= 256 ? 64 : 32;

template <typename T, int DHP, int NW, int ROWS = kBlockRows<T, DHP>>
struct Tile {
  static constexpr int BR = ROWS, E = sizeof(T);
  static constexpr int kPanels = DHP * E / 128, kPanelBytes = BR * 128, kBytes = kPanels * kPanelBytes;
  static constexpr int kPerWave = kBytes / 1024 / NW;  // a wave instruction copies 8 rows of a panel
  // A lane's chunk of copy t lies 32 rows (whose swizzle is the same) or a panel beyond that of copy 0
  static constexpr int kAround = BR / 8 / NW;  // copies of a panel
  static_assert((BR / 8) % NW == 0, "a panel is copied by all waves alike");
  static __device__ __forceinline__ size_t beyond(int t, size_t ld) { return (t % kAround) * 8 * NW * ld * E + (t / kAround) * 128; }
  static __device__ __forceinline__ uint32_t offset(size_t ld, int wave, int lane) {
    const int r = 8 * wave + (lane >> 3);
    return (uint32_t)(r * ld * E + (((lane & 7) ^ swizzle(r)) * 16));
  }
  // base: the block's first row, ld its row stride.  whole: BR rows and DHP columns are there; else rows and `cols` of them
  static __device__ __forceinline__ void copy(uint32_t lds, const T* base, size_t ld, uint32_t off, bool whole, int rows, int cols, int wave, int lane) {
#pragma unroll
    for (int t = 0; t < kPerWave; ++t) {
      const uint32_t to = lds + (t / kAround) * kPanelBytes + (wave + NW * (t % kAround)) * 1024;
      const char* from = (const char*)base + beyond(t, ld);
      if (whole) {
        dma16(to, from, off);
      } else {
        const int r = 8 * (wave + NW * (t % kAround)) + (lane >> 3), byte = (t / kAround) * 128 + (((lane & 7) ^ swizzle(r)) * 16);
        dma_addr<16>(to, r < rows && byte < cols * E ? from + off : zero_chunk());
      }
    }
  }
  // Where in a tile this lane's fragments lie: constants away from one address for the first products and one for the second, with bits
  // 4 .. 6, the slot, as an exclusive or (tiles start at multiples of 128).  The two addresses stay in registers; left to the compiler, all their
  // variants do, and the kernels with 128-wide heads spill.
  static __device__ __forceinline__ uint32_t row_base(int lane) {
    const int r = lane & 31, half = lane >> 5;
    return r * 128 + (((E == 2 ? half : 2 * half) ^ swizzle(r)) * 16);
  }
  static __device__ __forceinline__ uint32_t col_base(int lane) {
    if constexpr (E == 2) {
      const int q = lane >> 4, s = lane & 15, k = 4 * (q >> 1) + (s >> 2);
      return k * 128 + (((2 * (q & 1) + ((s & 3) >> 1)) ^ swizzle(k)) * 16) + (s & 1) * 8;
    } else {
      const int k = 4 * (lane >> 5);
      return k * 128 + ((((lane & 31) >> 2) ^ swizzle(k)) * 16) + (lane & 3) * 4;
    }
  }
  template <class V>
  static __device__ __forceinline__ V read(uint32_t base, uint32_t flip, uint32_t beyond) {
    uint32_t at = base;
    if (flip) asm volatile("v_xor_b32 %0, %1, %2" : "=v"(at) : "i"(flip), "v"(base));
    typedef __attribute__((address_space(3))) const char* lds_ptr;
    return *reinterpret_cast<__attribute__((address_space(3))) const V*>((lds_ptr)(uintptr_t)at + beyond);
  }
  // A fragment of the first products: row 32 u + lane % 32, columns 16 kk + 8 (lane / 32) .. + 7; base: the first tile of the stage plus row_base
  static __device__ __forceinline__ typename Type<T>::Frag row_frag(uint32_t base, int u, int kk, int tile = 0) {
    if constexpr (E == 2) {
      return __builtin_bit_cast(bf16x8, read<uintx4>(base, 32 * (kk & 3), tile * kBytes + u * 4096 + (kk >> 2) * kPanelBytes));
    } else {
      const uint32_t beyond = tile * kBytes + u * 4096 + (kk >> 1) * kPanelBytes;
      const floatx4 a = read<floatx4>(base, 64 * (kk & 1), beyond), b = read<floatx4>(base, 64 * (kk & 1) + 16, beyond);
      return floatx8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
  }
  // A fragment of the second products: column 32 j + lane % 32 of rows 16 g + 8 (t / 4) + 4 (lane / 32) + t % 4, t = 0 .. 7, the order in
  // which the accumulators hold them; base: the first tile of the stage plus col_base
  static __device__ __forceinline__ typename Type<T>::Frag col_frag(uint32_t base, int j, int g, int tile = 0) {
    if constexpr (E == 2) {
      const uint32_t beyond = tile * kBytes + (j >> 1) * kPanelBytes + g * 2048;
      const shortx4 lo = read_turned(base, 64 * (j & 1), beyond), hi = read_turned(base, 64 * (j & 1) + 16, beyond + 1024);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      floatx8 f;
#pragma unroll
      for (int t = 0; t < 8; ++t)
        f[t] = read<float>(base, 64 * ((t >> 1) & 1) + 16 * (t >> 2), tile * kBytes + j * kPanelBytes + (16 * g + 8 * (t >> 2) + (t & 3)) * 128);
      return f;
    }
  }
  static __device__ __forceinline__ shortx4 read_turned(uint32_t base, uint32_t flip, uint32_t beyond) {
    uint32_t at = base;
    if (flip) asm volatile("v_xor_b32 %0, %1, %2" : "=v"(at) : "i"(flip), "v"(base));
    typedef __attribute__((address_space(3))) const char* lds_ptr;
    typedef __attribute__((address_space(3))) shortx4* turned_ptr;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((turned_ptr)((lds_ptr)(uintptr_t)at + beyond));
  }
};

// Products one behind the other whose A fragments come from LDS: load(i) is issued DEPTH products ahead.  Left to itself the compiler
// puts every read right in front of its product, and a wave waits out the LDS's latency 24 times a tile.
template <int N, int DEPTH, class Frag, class Load, class Use>
__device__ __forceinline__ void pipelined(Frag (&f)[DEPTH], const Load& load, const Use& use, bool preloaded = false) {
  if (!preloaded) {
#pragma unroll
    for (int i = 0; i < DEPTH && i < N; ++i) f[i] = load(i);
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    use(i, f[i % DEPTH]);
    if (i + DEPTH < N) f[i % DEPTH] = load(i + DEPTH);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// ---- the bias in LDS ----------------------------------------------------------------------------------------------------------
// The buckets of distances 0 .. kNear + kPad - 1, four to a word.  A lane fetches a word, its borders and its values at the same time; a search by
// distance, or a walk over the buckets' runs, waited for memory again and again: 8 to 9 of the 12 thousand cycles before the first tile.
struct NearBuckets {
  uint32_t of[(kNear + kPad) / 4];
};
inline NearBuckets near_buckets(const DistanceBuckets& d) {
  NearBuckets n{};
  if (d.count == 0) return n;
  for (int i = 0, b = 0; i < kNear + kPad; ++i) {
    while (b + 1 < d.count && i >= d.first[b + 1]) ++b;
    n.of[i / 4] |= (uint32_t)b << 8 * (i % 4);
  }
  return n;
}
// near[kPad + d], d = -kPad .. kNear + kPad - 1: the table by distance, in units of log2; beyond that by bucket.
struct BiasLds {
  float near[kNearSize];
  float value[kMaxBuckets];
  // by the WAVES waves that share it
  template <int WAVES>
  __device__ __forceinline__ void load(const DistanceBuckets& d, const NearBuckets& n, const float* row, int lane, int thread) {
    constexpr int kWords = (kNear + kPad) / 4, kEach = (kWords + 64 * WAVES - 1) / (64 * WAVES);
    uint32_t word[kEach];
#pragma unroll
    for (int c = 0; c < kEach; ++c) word[c] = n.of[min(thread + 64 * WAVES * c, kWords - 1)];
    // all values by every wave, which then reads its own
#pragma unroll
    for (int c = 0; c < kMaxBuckets / 64; ++c) value[lane + 64 * c] = row[min(lane + 64 * c, d.count - 1)] * kLog2e;
    for (int i = thread; i < kPad; i += 64 * WAVES) near[i] = 0.f;
#pragma unroll
    for (int c = 0; c < kEach; ++c) {
      const int at = min(thread + 64 * WAVES * c, kWords - 1);
      const uint32_t w = word[c];
      *reinterpret_cast<float4*>(near + kPad + 4 * at) = make_float4(value[w & 255], value[w >> 8 & 255], value[w >> 16 & 255], value[w >> 24]);
    }
  }
};
__device__ __forceinline__ void load_borders(const DistanceBuckets& d, int* first) {
  if ((int)threadIdx.x < d.count) first[threadIdx.x] = d.first[threadIdx.x];
}

// Buckets b0 .. b1 of a tile's distances dmin .. dmax, wave uniform; b0 = -1: near ones, by distance.
struct TileBuckets {
  int b0 = -1, b1 = -1;
  __device__ TileBuckets() {}
  __device__ __forceinline__ TileBuckets(const DistanceBuckets& d, const int* first, int dmin, int dmax) {
    const int last = d.first[d.count - 1];
    if (dmin < kNear && dmin < last) return;
    b0 = b1 = d.count - 1;
    if (dmin >= last) return;
    b0 = __builtin_amdgcn_readfirstlane(bucket_of(d, first, dmin));
    b1 = b0;
    while (b1 + 1 < d.count && __builtin_amdgcn_readfirstlane(first[b1 + 1]) <= dmax) ++b1;
  }
};
// What a lane's N (4 or 16) elements have added to their scaled scores.  Element r has distance base + SIGN * (8 (r / 4) + r % 4).
template <int SIGN, int N>
__device__ __forceinline__ void tile_bias(const BiasLds& bl, const TileBuckets& tb, const int* first, int base, float (&out)[N]) {
  if (tb.b0 < 0) {
    const float* at = bl.near + kPad + base;
#pragma unroll
    for (int r = 0; r < N; ++r) out[r] = at[SIGN * (8 * (r >> 2) + (r & 3))];
  } else {
    const float v = bl.value[tb.b0];
#pragma unroll
    for (int r = 0; r < N; ++r) out[r] = v;
    for (int b = tb.b0 + 1; b <= tb.b1; ++b) {
      const int from = first[b] - base;
      const float w = bl.value[b];
#pragma unroll
      for (int r = 0; r < N; ++r)
        if (SIGN * (8 * (r >> 2) + (r & 3)) >= from) out[r] = w;
    }
  }
}

// ---- turning a wave's transposed result through LDS for whole rows ----------------------------------------------------------------
constexpr int kTurnPitch = 64 + 4, kTurnBytes = 32 * kTurnPitch * 4;
// write(row, column, v[8]) for the 32 rows of acc^T
template <int TN, class Write>
__device__ __forceinline__ void turned_rows(const floatx16 (&acc)[TN], float factor, float* lds, int lane, const Write& write) {
#pragma unroll
  for (int c = 0; c < TN / 2; ++c) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const floatx16& a = acc[2 * c + j];
        *reinterpret_cast<float4*>(lds + (lane & 31) * kTurnPitch + 32 * j + 8 * g + 4 * (lane >> 5)) =
            make_float4(a[4 * g] * factor, a[4 * g + 1] * factor, a[4 * g + 2] * factor, a[4 * g + 3] * factor);
      }
    // one wave on both sides, whose LDS operations complete in order
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int r = 8 * p + (lane >> 3), col = 8 * (lane & 7);
      const float4 lo = *reinterpret_cast<const float4*>(lds + r * kTurnPitch + col), hi = *reinterpret_cast<const float4*>(lds + r * kTurnPitch + col + 4);
      const float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      write(r, 64 * c + col, v);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

// Sums of two waves over the same rows: one leaves its own in LDS, a lane's values 64 x 16 bytes apart, the other adds them to its own,
// each with a factor.
template <int TN>
__device__ __forceinline__ void hand_over(const floatx16 (&acc)[TN], floatx4* to) {
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) to[(j * 4 + r) * 64] = floatx4{acc[j][4 * r], acc[j][4 * r + 1], acc[j][4 * r + 2], acc[j][4 * r + 3]};
}
template <int TN>
__device__ __forceinline__ void take_over(floatx16 (&acc)[TN], const floatx4* from, float mine = 1.f, float its = 1.f) {
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const floatx4 v = from[(j * 4 + r) * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][4 * r + e] = fmaf(acc[j][4 * r + e], mine, v[e] * its);
    }
}

// ---- rows one by one ----------------------------------------------------------------------------------------------------------
template <int TN>
__device__ __forceinline__ bool finite(const floatx16 (&acc)[TN]) {
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) s = fmaf(acc[j][r], 0.f, s);  // 0, or NaN
  return s == 0.f;
}
// bit i: row i of the wave (lanes i and i + 32) is there and not finite
__device__ __forceinline__ uint32_t rows_to_redo(bool fine, bool there) {
  const uint64_t m = __builtin_amdgcn_ballot_w64(!fine && there);
  return (uint32_t)m | (uint32_t)(m >> 32);
}
template <typename T>
__device__ __forceinline__ float row_dot(const T* a, const T* b, int dh) {
  float s = 0.f;
  for (int d = 0; d < dh; ++d) s = fmaf(to_float(a[d]), to_float(b[d]), s);
  return s;
}
// acc[c] += w (of lane t) * row t's value in this lane's column, over the lanes in `which`
template <typename T>
__device__ __forceinline__ void add_rows(float (&acc)[2], float w, const T* rows, size_t ld, uint64_t which, int dh, int lane) {
  for (; which; which &= which - 1) {
    const int t = __builtin_ctzll(which);
    const float wt = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), t));
#pragma unroll
    for (int c = 0; c < 2; ++c)
      if (lane + 64 * c < dh) acc[c] = fmaf(wt, to_float(rows[(size_t)t * ld + lane + 64 * c]), acc[c]);
  }
}
// the tiles of 64 keys that query i sees something of: calls body(first key)
template <class Body>
__device__ __forceinline__ void visible_tiles(const Shape& a, int i, const Body& body) {
  const int lo = max(0, i - a.window + 1);
  for (int k0 = 0; k0 <= i; k0 += 64) {
    if (k0 >= a.sinks && k0 + 64 <= lo) k0 = lo / 64 * 64;
    body(k0);
  }
}

template <typename T, bool BIAS>
__device__ void redo_output_row(const Shape& a, const DistanceBuckets& db, const int* first, const BiasLds* bl, int i, const T* q, const T* k,
                                const T* v, T* out, T* out2, float* lse, float scale_log2, int lane) {
  const size_t ld = a.ld();
  float m = -INFINITY, l = 0.f, o[2] = {};
  visible_tiles(a, i, [&](int k0) {
    const int j = k0 + lane;
    const bool sees = j <= i && a.sees(i, j);
    float sc = -INFINITY;
    if (sees) {
      sc = row_dot(q + (size_t)i * ld, k + (size_t)j * ld, a.dh) * scale_log2;
      if (BIAS) sc += bl->value[bucket_of(db, first, i - j)];
    }
    const float mn = fmaxf(m, max_over_lanes(sc));
    // a NaN score is NaN in p, whatever the maximum; a row whose scores are all -inf is NaN through its sum of zero
    const float p = sc == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sc - mn);
    const float corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
    l = l * corr + sum_over_lanes(p);
    m = mn;
    o[0] *= corr;
    o[1] *= corr;
    add_rows(o, p, v + (size_t)k0 * ld, ld, __builtin_amdgcn_ballot_w64(sees), a.dh, lane);
  });
  const float inv = 1.f / l;
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (lane + 64 * c < a.dh) {
      out[lane + 64 * c] = from_float<T>(o[c] * inv);
      if (out2) out2[lane + 64 * c] = from_float<T>(o[c] * inv);
    }
  if (lane == 0) *lse = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <typename T, bool BIAS>
__device__ void redo_dq_row(const Shape& a, const DistanceBuckets& db, const int* first, const BiasLds* bl, int i, const T* q, const T* k,
                            const T* v, const T* dout_row, float l2, float delta, T* dq, float scale, int lane) {
  const size_t ld = a.ld();
  float acc[2] = {};
  visible_tiles(a, i, [&](int k0) {
    const int j = k0 + lane;
    const bool sees = j <= i && a.sees(i, j);
    float ds = 0.f;
    if (sees) {
      float e = row_dot(q + (size_t)i * ld, k + (size_t)j * ld, a.dh) * (scale * kLog2e) - l2;
      if (BIAS) e += bl->value[bucket_of(db, first, i - j)];
      ds = __builtin_amdgcn_exp2f(e) * (row_dot(dout_row, v + (size_t)j * ld, a.dh) - delta);
    }
    add_rows(acc, ds, k + (size_t)k0 * ld, ld, __builtin_amdgcn_ballot_w64(sees), a.dh, lane);
  });
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (lane + 64 * c < a.dh) dq[lane + 64 * c] = from_float<T>(acc[c] * scale);
}

// ---- forward --------------------------------------------------------------------------------------------------------------------
template <typename T>
struct FwdArgs {
  Shape a;
  DistanceBuckets db;
  NearBuckets near;
  const T* x;
  const float* table;
  float* kept;
  T *out, *out2;
  float* lse;
  float scale_log2;
};

// LDS behind the streamed tiles where there is a bias: the borders, then a table per wave
template <int NW>
constexpr size_t bias_lds(bool bias) { return bias ? kMaxBuckets * 4 + NW * sizeof(BiasLds) : 0; }

// Items of a workgroup: blocks of 32 queries x heads of key head kvh, and the blocks of keys they walk over
template <int BR, int NW>
struct QueryItems {
  int item, items, q_lo, q_hi, blk, g;  // this wave's item; the workgroup's queries
  int first_blk, sink_blks, count;      // streamed blocks: 0 .. sink_blks - 1, then from first_blk on
  __device__ __forceinline__ QueryItems(const Shape& a, int group, int nblk, int wg, int wave) {
    items = nblk * group;
    item = wg * NW + wave;
    blk = item / group;
    g = item - blk * group;
    q_lo = wg * NW / group * 32;
    q_hi = min(a.S - 1, min(wg * NW + NW - 1, items - 1) / group * 32 + 31);
    first_blk = max(0, q_lo - a.window + 1) / BR;
    sink_blks = min((a.sinks + BR - 1) / BR, first_blk);
    count = q_hi < q_lo ? 0 : sink_blks + q_hi / BR - first_blk + 1;
  }
  __device__ __forceinline__ int block(int t) const { return t < sink_blks ? t : first_blk + t - sink_blks; }
};

// Steps of 32 keys at three waves a SIMD: one wave's exponentials run beside another's products.  (Steps of 64 at two waves, a row rescaled at
// every new maximum: 55, 114 and, with a bias, 86 us of the following.)
// 8 x 1024 tokens, 16 heads of 128, window 256: 46 us; 1 x 16384, 8 heads on 2, window 1024: 104 us, 0.65 PFLOP/s; 8 x 1024, 16 heads, all
// keys: 55 us, with a bias 65.
// TEAMS: 1, a wave has 32 queries of a head to itself; 2, blocks have 64 keys and two waves take 32 each, for launches that leave SIMDs without
// a wave: their maxima, sums and outputs meet in LDS.
template <typename T, int DHP, int NW, int TEAMS, bool BIAS>
__global__ __launch_bounds__(64 * NW, TEAMS == 1 && (sizeof(T) == 2 || DHP == 64) ? 3 : 2) void local_fwd_kernel(FwdArgs<T> p) {
  using TY = Type<T>;
  using TL = Tile<T, DHP, NW, 32 * TEAMS>;
  constexpr int BR = TL::BR, kMine = BR / TEAMS, NT = kMine / 32, KK = DHP / 16, TN = DHP / 32;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Shape& a = p.a;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = a.heads / a.kv, b = blockIdx.x / a.kv, kvh = blockIdx.x - b * a.kv;
  const int S = a.S, dh = a.dh;
  const size_t ld = a.ld(), D = (size_t)a.heads * dh;
  const int team = wave / (NW / TEAMS);
  const QueryItems<BR, NW / TEAMS> it(a, group, (S + 31) / 32, gridDim.y - 1 - blockIdx.y, wave % (NW / TEAMS));
  const bool active = it.item < it.items;
  const int h = kvh * group + (active ? it.g : 0), qw = (active ? it.blk : 0) * 32;
  const T* base = p.x + (size_t)b * S * ld;
  const T* qbase = base + (size_t)h * dh;
  const T* kbase = base + D + (size_t)kvh * dh;
  const T* vbase = kbase + (size_t)a.kv * dh;
  const uint32_t lds0 = lds_addr_of(lds);
  constexpr size_t kStages = 2 * 2 * TL::kBytes, kTiles = kStages > NW * kTurnBytes ? kStages : NW * kTurnBytes;
  int* first = reinterpret_cast<int*>(lds + kTiles);
  BiasLds* bl = reinterpret_cast<BiasLds*>(lds + kTiles + kMaxBuckets * 4) + wave;
  const uint32_t off = TL::offset(ld, wave, lane), row_at = TL::row_base(lane), col_at = TL::col_base(lane);
  auto issue = [&](int t) {
    const int row = it.block(t) * BR;
    const uint32_t to = lds0 + (t & 1) * 2 * TL::kBytes;
    const bool whole = dh == DHP && row + BR <= S;
    TL::copy(to, kbase + (size_t)row * ld, ld, off, whole, S - row, dh, wave, lane);
    TL::copy(to + TL::kBytes, vbase + (size_t)row * ld, ld, off, whole, S - row, dh, wave, lane);
  };
  if (it.count > 0) issue(0);  // on its way while the wave's own rows are fetched
  const int query = min(qw + (lane & 31), S - 1);
  typename TY::Frag qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) qf[kk] = TY::load(qbase + (size_t)query * ld + 16 * kk + 8 * half, dh - 16 * kk - 8 * half);
  if constexpr (BIAS) {
    load_borders(p.db, first);
    const float* row = p.table + (size_t)h * p.db.count;
    bl->load<1>(p.db, p.near, row, lane, lane);
    if (b == 0 && active && it.blk == 0)
      for (int t = lane; t < p.db.count; t += 64) p.kept[(size_t)h * p.db.count + t] = row[t];
  }
  wait_vmcnt<0>();  // nothing but copies is in flight from here on
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(qf[kk]));

  floatx16 oacc[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[j][r] = 0.f;
  float mrun = kLowest, lsum = 0.f;
  const int q_last = min(qw + 31, S - 1);
  for (int t = 0; t < it.count; ++t) {
    wait_vmcnt<0>();
    lds_barrier();  // block t is there, and nobody reads the other stage any more
    if (t + 1 < it.count) issue(t + 1);
    const int skip = TEAMS == 1 ? 0 : team * kMine, kb = it.block(t) * BR + skip;
    // wave uniform: some pair of this wave and block is visible
    if (!active || kb > q_last || (kb >= a.sinks && kb + kMine - 1 <= qw - a.window)) continue;
    const uint32_t stage = lds0 + (t & 1) * 2 * TL::kBytes + skip * 128, lk = stage + row_at, lv = stage + col_at;
    floatx16 sacc[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[u][r] = 0.f;
    typename TY::Frag ahead[TY::kAhead];
    // the tiles in turn: no product waits for the one before it
    pipelined<NT * KK>(ahead, [&](int i) { return TL::row_frag(lk, i % NT, i / NT); },
                       [&](int i, const typename TY::Frag& f) { if (!TY::skips(16 * (i / NT), dh)) sacc[i % NT] = TY::mma(f, qf[i / NT], sacc[i % NT]); });
    auto v_frag = [&](int i) { return TL::col_frag(lv, i % TN, i / TN, 1); };
#pragma unroll
    for (int i = 0; i < TY::kAhead; ++i) ahead[i] = v_frag(i);
    __builtin_amdgcn_sched_barrier(0);
    const int dmin = qw - (kb + kMine - 1), dmax = qw + 31 - kb;
    const bool masked = !(dmin >= 0 && (dmax < a.window || kb + kMine <= a.sinks));
    // distance of element r of tile u: d0 - 32 u - 8 (r / 4) - r % 4
    const int d0 = query - kb - 4 * half, sink0 = a.sinks - kb - 4 * half;
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      if constexpr (BIAS) {
        float bias[16];
        tile_bias<-1>(*bl, TileBuckets(p.db, first, dmin + kMine - 32 * (u + 1), dmax - 32 * u), first, d0 - 32 * u, bias);
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[u][r] = fmaf(sacc[u][r], p.scale_log2, bias[r]);
      }
      if (masked) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int at = 32 * u + 8 * (r >> 2) + (r & 3);
          sacc[u][r] = (at <= d0) & ((at > d0 - a.window) | (at < sink0)) ? sacc[u][r] : -INFINITY;
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[u][r]);
    }
    const float factor = BIAS ? 1.f : p.scale_log2;  // what turns sacc into scores
    const float mnew = over_halves(mx, Max()) * factor;
    // A row's reference need not be its maximum: while no score lies above it by more than kSlack, the exponentials stay below 2^kSlack and
    // nothing is rescaled.  (Some row's maximum of 32 moves in nearly every block.)
    if (__builtin_amdgcn_ballot_w64(mnew > mrun + kSlack) != 0) {
      const float m = fmaxf(mrun, mnew), alpha = __builtin_amdgcn_exp2f(mrun - m);
      mrun = m;
      lsum *= alpha;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[j][r] *= alpha;
    }
    typename TY::Frag pf[2 * NT];
#pragma unroll
    for (int g = 0; g < 2 * NT; ++g) {
      float e[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        e[r] = __builtin_amdgcn_exp2f(fmaf(sacc[g >> 1][8 * (g & 1) + r], factor, -mrun));
        lsum += e[r];
      }
      pf[g] = TY::pack(e);
    }
    pipelined<2 * NT * TN>(ahead, v_frag, [&](int i, const typename TY::Frag& f) { if (!TY::skips(32 * (i % TN), dh)) oacc[i % TN] = TY::mma(f, pf[i / TN], oacc[i % TN]); }, true);
  }
  lds_barrier();  // the stages are free
  if constexpr (TEAMS == 2) {
    floatx4* theirs = reinterpret_cast<floatx4*>(lds) + (size_t)(wave % (NW / TEAMS)) * TN * 4 * 64 + lane;
    float2* stats = reinterpret_cast<float2*>(lds + (size_t)NW / TEAMS * TN * 4 * 64 * 16) + wave % (NW / TEAMS) * 64 + lane;
    if (team == 1) {
      hand_over(oacc, theirs);
      *stats = make_float2(mrun, lsum);
    }
    lds_barrier();
    if (team == 0) {
      const float2 other = *stats;
      const float m = fmaxf(mrun, other.x), mine = __builtin_amdgcn_exp2f(mrun - m), its = __builtin_amdgcn_exp2f(other.x - m);
      mrun = m;
      lsum = fmaf(lsum, mine, other.y * its);
      take_over(oacc, theirs, mine, its);
    }
    lds_barrier();
  }
  if (!active || team != 0) return;
  const float ltot = over_halves(lsum, Add());
  const float inv = 1.f / ltot;
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[j][r] *= inv;
  const bool there = qw + (lane & 31) < S;
  float* lse = p.lse + ((size_t)b * a.heads + h) * S;
  if (half == 0 && there) lse[query] = (mrun + __builtin_amdgcn_logf(ltot)) * kLn2;
  const size_t at = ((size_t)b * S + qw) * D + (size_t)h * dh;
  turned_rows(oacc, 1.f, reinterpret_cast<float*>(lds) + wave * (kTurnBytes / 4), lane, [&](int r, int col, const float (&v)[8]) {
    if (qw + r >= S) return;
    TY::store8(p.out + at + (size_t)r * D + col, v, dh - col);
    if (p.out2) TY::store8(p.out2 + at + (size_t)r * D + col, v, dh - col);
  });
  uint32_t redo = rows_to_redo(finite(oacc), there);
  if (redo) wait_vmcnt<0>();  // what they replace is stored
  for (; redo; redo &= redo - 1) {
    const int r = __builtin_ctz(redo);
    redo_output_row<T, BIAS>(a, p.db, first, bl, qw + r, qbase, kbase, vbase, p.out + at + (size_t)r * D,
                             p.out2 ? p.out2 + at + (size_t)r * D : nullptr, lse + qw + r, p.scale_log2, lane);
  }
}

// ---- backward -------------------------------------------------------------------------------------------------------------------
__host__ __device__ constexpr int stat_rows(int S) { return (S + 63) / 64 * 64; }

template <typename T>
struct BwdArgs {
  Shape a;
  DistanceBuckets db;
  NearBuckets near;
  int seqs_per_table;
  const T *x, *out, *dout;
  const float *lse, *kept;
  T* dx;
  float* stat;      // [seqs*heads][stat_rows(S)][2]: lse * log2(e) and the corrected delta, zeros behind the last token
  // parts of dK and dV: [parts][seqs*kv][S, or with one part sinks][2][dh], then of far pairs of the first keys [chunks][seqs*kv][sinks][2][dh]
  float* sums;
  float* partials;  // of the table: [seqs * gridDim.y][heads][buckets]
  int parts;        // of a walk over streamed blocks, in workgroups of their own
  int far_blocks, chunks;  // workgroups for far pairs of the first keys: blocks of keys x ranges of the walk; none: the others take these pairs
  float scale;
};

// Three products a tile at two waves a SIMD: 140 registers are q, dy and the sums.  8 x 1024 tokens, 16 heads of 128, window 256: 63 us;
// 1 x 16384, 8 heads, window 1024: 142 us, 0.71 PFLOP/s; 8 x 1024, 16 heads, all keys: 82 us, with a bias 97.
// TEAMS: 1, a wave has 32 queries of a head to itself; 2, two waves take one tile of every streamed block each, and their sums meet in LDS:
// for launches that leave SIMDs without a wave.
template <typename T, int DHP, int NW, int TEAMS, bool BIAS>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 || DHP == 64 ? 2 : 1) void local_dq_kernel(BwdArgs<T> p) {
  using TY = Type<T>;
  using TL = Tile<T, DHP, NW>;
  constexpr int BR = TL::BR, NT = BR / 32, KK = DHP / 16, TN = DHP / 32;
  static_assert(TEAMS == 1 || TEAMS == NT, "a team takes one tile of a block");
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Shape& a = p.a;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = a.heads / a.kv, b = blockIdx.x / a.kv, kvh = blockIdx.x - b * a.kv;
  const int S = a.S, dh = a.dh, SP = stat_rows(S);
  const size_t ld = a.ld(), D = (size_t)a.heads * dh;
  const int team = wave / (NW / TEAMS);
  const QueryItems<BR, NW / TEAMS> it(a, group, SP / 32, gridDim.y - 1 - blockIdx.y, wave % (NW / TEAMS));
  const bool active = it.item < it.items;
  const int h = kvh * group + (active ? it.g : 0), qw = (active ? it.blk : 0) * 32;
  const T* base = p.x + (size_t)b * S * ld;
  const T* qbase = base + (size_t)h * dh;
  const T* kbase = base + D + (size_t)kvh * dh;
  const T* vbase = kbase + (size_t)a.kv * dh;
  const uint32_t lds0 = lds_addr_of(lds);
  constexpr size_t kStages = 2 * 2 * TL::kBytes, kTiles = kStages > NW * kTurnBytes ? kStages : NW * kTurnBytes;
  int* first = reinterpret_cast<int*>(lds + kTiles);
  BiasLds* bl = reinterpret_cast<BiasLds*>(lds + kTiles + kMaxBuckets * 4) + wave;
  const uint32_t off = TL::offset(ld, wave, lane), row_at = TL::row_base(lane), col_at = TL::col_base(lane);
  auto issue = [&](int t) {
    const int row = it.block(t) * BR;
    const uint32_t to = lds0 + (t & 1) * 2 * TL::kBytes;
    const bool whole = dh == DHP && row + BR <= S;
    TL::copy(to, kbase + (size_t)row * ld, ld, off, whole, S - row, dh, wave, lane);
    TL::copy(to + TL::kBytes, vbase + (size_t)row * ld, ld, off, whole, S - row, dh, wave, lane);
  };
  if (it.count > 0) issue(0);  // on its way while the wave's own rows are fetched
  const bool there = active && qw + (lane & 31) < S;
  const int query = min(qw + (lane & 31), S - 1);
  const T* dorow = p.dout + ((size_t)b * S + query) * D + (size_t)h * dh;
  const T* orow = p.out + ((size_t)b * S + query) * D + (size_t)h * dh;
  typename TY::Frag qf[KK], df[KK];
  float delta = 0.f;
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    const int d = 16 * kk + 8 * half;
    df[kk] = TY::load(dorow + d, dh - d);
    delta = TY::dot(df[kk], TY::load(orow + d, dh - d), delta);
  }
  __builtin_amdgcn_sched_barrier(0);  // the output's registers are free again
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) qf[kk] = TY::load(qbase + (size_t)query * ld + 16 * kk + 8 * half, dh - 16 * kk - 8 * half);
  delta = over_halves(delta, Add());
  float l2 = p.lse[((size_t)b * a.heads + h) * S + query] * kLog2e;
  if constexpr (BIAS) {
    load_borders(p.db, first);
    bl->load<1>(p.db, p.near, p.kept + ((size_t)(b / p.seqs_per_table) * a.heads + h) * p.db.count, lane, lane);
  }
  wait_vmcnt<0>();
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(qf[kk]), "+v"(df[kk]));
  asm volatile("" : "+v"(l2), "+v"(delta));

  floatx16 acc[TN];
  float total = 0.f;
  const int q_last = min(qw + 31, S - 1);
  const float scale_log2 = p.scale * kLog2e;
  // Over the first `steps` blocks, the first of which is on its way; waves of queries below q_end.  With products, or the sums of dS alone.
  auto walk = [&](auto products, int steps, int q_end) __attribute__((always_inline)) {
    constexpr bool kProducts = decltype(products)::value;
    for (int t = 0; t < steps; ++t) {
      wait_vmcnt<0>();
      lds_barrier();
      if (t + 1 < steps) issue(t + 1);
      constexpr int kMine = BR / TEAMS;  // the wave's rows of the block
      const int skip = TEAMS == 1 ? 0 : team * 32, kb = it.block(t) * BR + skip;
      if (!active || qw >= q_end || kb > q_last || (kb >= a.sinks && kb + kMine - 1 <= qw - a.window)) continue;
      const uint32_t stage = lds0 + (t & 1) * 2 * TL::kBytes + skip * 128, lk = stage + row_at, lkc = stage + col_at;
      const int d0 = query - kb - 4 * half, sink0 = a.sinks - kb - 4 * half;
#pragma unroll
      for (int u = 0; u < NT / TEAMS; ++u) {
        // the tile's smallest and largest distance; wave uniform
        const int k0 = kb + 32 * u, dmin = qw - (k0 + 31), dmax = qw + 31 - k0;
        if (dmax < 0 || (dmin >= a.window && k0 >= a.sinks)) continue;
        const bool masked = !(dmin >= 0 && (dmax < a.window || k0 + 32 <= a.sinks));
        floatx16 sacc, pacc;
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[r] = pacc[r] = 0.f;
        typename TY::Frag ahead[TY::kAhead];
        pipelined<2 * KK>(ahead, [&](int i) { return TL::row_frag(lk, u, i >> 1, i & 1); },
                          [&](int i, const typename TY::Frag& f) {
                            if (TY::skips(16 * (i >> 1), dh)) return;
                            if (i & 1) pacc = TY::mma(f, df[i >> 1], pacc);
                            else sacc = TY::mma(f, qf[i >> 1], sacc);
                          });
        auto k_frag = [&](int i) { return TL::col_frag(lkc, i % TN, 2 * u + i / TN); };
        if constexpr (kProducts) {
#pragma unroll
          for (int i = 0; i < TY::kAhead; ++i) ahead[i] = k_frag(i);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (BIAS) {  // ahead of the mask: an entry of the table that only hidden pairs have may hold anything
          float bias[16];
          tile_bias<-1>(*bl, TileBuckets(p.db, first, dmin, dmax), first, d0 - 32 * u, bias);
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[r] = fmaf(sacc[r], scale_log2, bias[r]);
        }
        if (masked) {  // p = 0, and dS = 0 whatever dP holds
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int at = 32 * u + 8 * (r >> 2) + (r & 3);
            const bool sees = (at <= d0) & ((at > d0 - a.window) | (at < sink0));  // without branches
            sacc[r] = sees ? sacc[r] : -INFINITY;
            pacc[r] = sees ? pacc[r] : delta;
          }
        }
        typename TY::Frag dsf[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          float e[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int r = 8 * g + q;
            const float pr = __builtin_amdgcn_exp2f((BIAS ? sacc[r] : sacc[r] * scale_log2) - l2);
            const float ds = pr * (pacc[r] - delta);
            e[q] = ds;
            total += ds;
          }
          dsf[g] = TY::pack(e);
        }
        if constexpr (kProducts) pipelined<2 * TN>(ahead, k_frag, [&](int i, const typename TY::Frag& f) { if (!TY::skips(32 * (i % TN), dh)) acc[i % TN] = TY::mma(f, dsf[i / TN], acc[i % TN]); }, true);
      }
    }
  };
  // The delta of the stored y is off by what rounded y to bf16, 2^-9 of it: of a query with few keys that is as much as dS itself is rounded
  // by.  Queries that see at most 32 keys, the first 32 of a sequence among them, are walked over once before to correct it; the others' dS are
  // off by it, on average over their keys.  (2 and 8 keys: dq 0.0038 and 0.0027 of its norm off, so 0.0023 and 0.0024; the rounding of what is
  // stored alone is 0.0017.  From 40 keys on it makes no difference.)  A walk of its own, before there are sums: as a second pass of the other
  // it took the 128-wide heads' kernel 15 registers, and spilled.
  if constexpr (sizeof(T) == 2) {
    const bool all = a.window + a.sinks <= 32;
    if (all || it.q_lo == 0) {
      // of a sequence's first queries the first block of keys has all they see, and only the first team's tile of it
      walk(std::false_type(), all ? it.count : min(1, it.count), all ? S : 32);
      if (all) {
        lds_barrier();
        if constexpr (TEAMS == 2) {
          float* totals = reinterpret_cast<float*>(lds);
          totals[threadIdx.x] = total;
          lds_barrier();
          total += totals[threadIdx.x ^ (64 * NW / 2)];
          lds_barrier();
        }
        if (it.count > 0) issue(0);
      }
      delta += over_halves(total, Add());
      total = 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
  walk(std::true_type(), it.count, S);
  lds_barrier();
  if constexpr (TEAMS == 2) {  // the second team's sums to the first
    floatx4* mine = reinterpret_cast<floatx4*>(lds) + (size_t)(wave % (NW / TEAMS)) * TN * 4 * 64 + lane;
    float* totals = reinterpret_cast<float*>(lds + (size_t)NW / TEAMS * TN * 4 * 64 * 16) + wave % (NW / TEAMS) * 64 + lane;
    if (team == 1) {
      hand_over(acc, mine);
      *totals = total;
    }
    lds_barrier();
    if (team == 0) {
      take_over(acc, mine);
      total += *totals;
    }
    lds_barrier();
  }
  if (!active || team != 0) return;
  // what the rows of dS add up to is what delta was off by
  const float corrected = delta + over_halves(total, Add());
  if (half == 0)
    *reinterpret_cast<float2*>(p.stat + (((size_t)b * a.heads + h) * SP + qw + lane) * 2) = there ? make_float2(l2, corrected) : make_float2(0.f, 0.f);
  T* dq = p.dx + ((size_t)b * S + qw) * ld + (size_t)h * dh;
  turned_rows(acc, p.scale, reinterpret_cast<float*>(lds) + wave * (kTurnBytes / 4), lane, [&](int r, int col, const float (&v)[8]) {
    if (qw + r < S) TY::store8(dq + (size_t)r * ld + col, v, dh - col);
  });
  uint32_t redo = rows_to_redo(finite(acc), there);
  if (redo) wait_vmcnt<0>();
  for (; redo; redo &= redo - 1) {
    const int r = __builtin_ctz(redo), i = qw + r;
    auto of_row = [&](float v) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), r)); };
    redo_dq_row<T, BIAS>(a, p.db, first, bl, i, qbase, kbase, vbase, p.dout + ((size_t)b * S + i) * D + (size_t)h * dh, of_row(l2), of_row(delta),
                         dq + (size_t)r * ld, p.scale, lane);
  }
}

// Sums of dS by distance and, beyond the near ones, by bucket, per wave, in LDS: a wave's own additions stay in order.
struct TableSums {
  float near[kNearSize];
  float far[kMaxBuckets];
};

// What a lane has of the bucket that its wave's last far tiles lay in; distances ascend along a walk, so buckets change rarely.
struct FarSum {
  float sum = 0.f;
  int bucket = 0;  // wave uniform
  __device__ __forceinline__ void flush(TableSums& sums, int lane) {
    const float s = sum_over_lanes(sum);
    if (lane == 0) sums.far[bucket] += s;
    sum = 0.f;
  }
  __device__ __forceinline__ void start_tile(TableSums& sums, const TileBuckets& tb, int lane) {
    if (tb.b0 < 0 || tb.b0 == bucket) return;
    flush(sums, lane);
    bucket = tb.b0;
  }
};
// Sums along the diagonals of a tile of 32 queries (rows, in order) x 32 keys (lanes): with every row the sums move a lane up, so that a
// diagonal's stays with it, and take in the row's values; lanes 32 .. 63 add nothing and hold the diagonals that have left the tile.  After
// the last row lane l has the sum of (row - lane) = 31 - l.  (Adding every element to its distance in LDS instead: 16 float atomics a tile, which
// took 650 cycles each, 10 of the 13 thousand cycles of a tile.)
struct Diagonals {
  float sum = 0.f;
  __device__ __forceinline__ void row(float v) {
    sum = v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(sum), 0x138, 0xf, 0xf, true));  // wave_shr:1
  }
  // a lane's four rows below the others', of which lanes 0 .. 31 have the first and lanes 32 .. 63 the second four
  __device__ __forceinline__ void rows(const float (&ds)[4]) {
    float second[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const auto split = __builtin_amdgcn_permlane32_swap(__float_as_uint(ds[r]), 0u, false, false);
      second[r] = __uint_as_float(split[1]);
      row(__uint_as_float(split[0]));
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) row(second[r]);
  }
};
// ds: four elements with distances base .. base + 3
__device__ __forceinline__ void add_to_table(TableSums& sums, FarSum& far, Diagonals& diagonals, const TileBuckets& tb, const int* first, int count,
                                             int base, int lane, const float (&ds)[4]) {
  if (tb.b0 < 0) {
    diagonals.rows(ds);
  } else if (tb.b0 == tb.b1) {
    far.sum += (ds[0] + ds[1]) + (ds[2] + ds[3]);
  } else {
    for (int b = tb.b0; b <= tb.b1; ++b) {
      const int from = first[b] - base, to = b + 1 < count ? first[b + 1] - base : 4;
      float s = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) s += r >= from && r < to ? ds[r] : 0.f;
      s = sum_over_lanes(s);
      if (lane == 0) sums.far[b] += s;
    }
  }
}

template <int NW>
constexpr size_t dkv_bias_lds(bool bias) { return bias ? kMaxBuckets * 4 + sizeof(BiasLds) + NW * sizeof(TableSums) : 0; }

// TEAMS: 1, a wave owns 32 keys of 128; 2, two waves own the same 32 keys of 64 and take one tile of every streamed block each, which makes
// twice as many workgroups of half the length; their sums meet in LDS.
// Four products a tile; k, v and two sums take 192 of 256 registers.  8 x 1024 tokens, 16 heads of 128, window 256: 80 us; 1 x 16384, 8 heads
// on 2, window 1024: 219 us, 0.62 PFLOP/s; 8 x 1024, 16 heads, all keys: 105 us, with a bias 155 (sums by distance, and registers that spill).
template <typename T, int DHP, int NW, int TEAMS, bool BIAS>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 || DHP == 64 ? 2 : 1) void local_dkv_kernel(BwdArgs<T> p) {
  using TY = Type<T>;
  using TL = Tile<T, DHP, NW>;
  constexpr int BR = TL::BR, NT = BR / 32, KK = DHP / 16, TN = DHP / 32, kOwn = 32 * NW / TEAMS;
  static_assert(TEAMS == 1 || TEAMS == NT, "a team takes one tile of a block");
  constexpr int kStageBytes = 2 * TL::kBytes + 1024;  // Q, dO, statistics
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Shape& a = p.a;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = a.heads / a.kv, b = blockIdx.x / a.kv, kvh = blockIdx.x - b * a.kv;
  const int S = a.S, dh = a.dh, SP = stat_rows(S);
  const size_t ld = a.ld(), D = (size_t)a.heads * dh;
  // workgroups for the far pairs of first keys come first, then a workgroup for each block of keys, low ones (which more queries see) first
  const int fars = p.far_blocks * p.chunks;
  const bool far = (int)blockIdx.y < fars;
  const int chunk = far ? blockIdx.y / p.far_blocks : 0;
  const int part = far ? 0 : ((int)blockIdx.y - fars) % p.parts;
  const int k0 = (far ? (int)blockIdx.y - chunk * p.far_blocks : ((int)blockIdx.y - fars) / p.parts) * kOwn;
  const int team = wave / (NW / TEAMS);
  const int kw = k0 + wave % (NW / TEAMS) * 32, key = kw + (lane & 31);
  const bool active = kw < (far ? a.sinks : S);
  // Distances that count, from d_from up to an end: those in the window, of first keys without far workgroups all, and of far workgroups
  // those beyond the window.
  const bool to_last = far || p.far_blocks == 0;
  auto end_of = [&](int j) { return j >= a.sinks ? (far ? 0 : a.window) : to_last ? S : a.window; };
  const int d_from = far ? a.window : 0, d_to = end_of(kw);
  const int d_end = min(end_of(key), S - key);  // of this lane's key; copied rows behind the last token do not count
  // streamed blocks of queries
  const int blk0 = (k0 + d_from) / BR, blk1 = (int)min((long)S - 1, (long)k0 + kOwn - 2 + end_of(k0)) / BR + 1;
  // steps of the walk: the streamed blocks of each query head in turn; a part or a chunk takes a range of them
  const int nb = max(0, blk1 - blk0), pieces = far ? p.chunks : p.parts, piece = far ? chunk : part;
  const int t_begin = (int)((long)nb * group * piece / pieces), t_end = (int)((long)nb * group * (piece + 1) / pieces);
  const T* base = p.x + (size_t)b * S * ld;
  const T* kbase = base + D + (size_t)kvh * dh;
  const T* vbase = kbase + (size_t)a.kv * dh;
  const T* dobase = p.dout + (size_t)b * S * D;
  const uint32_t lds0 = lds_addr_of(lds);
  constexpr size_t kStages = 2 * kStageBytes, kTiles = kStages > NW * kTurnBytes ? kStages : NW * kTurnBytes;
  int* first = reinterpret_cast<int*>(lds + kTiles);
  BiasLds* bl = reinterpret_cast<BiasLds*>(lds + kTiles + kMaxBuckets * 4);
  TableSums* sums = reinterpret_cast<TableSums*>(bl + 1);
  auto table = [&](int h) { return p.kept + ((size_t)(b / p.seqs_per_table) * a.heads + h) * p.db.count; };
  auto start_head = [&](int g) {
    bl->load<NW>(p.db, p.near, table(kvh * group + g), lane, threadIdx.x);
    for (int i = threadIdx.x; i < (int)(NW * sizeof(TableSums) / 4); i += 64 * NW) reinterpret_cast<float*>(sums)[i] = 0.f;
  };
  auto issue = [&](int t) {
    const int g = t / nb, row = (blk0 + t - g * nb) * BR, h = kvh * group + g;
    const uint32_t to = lds0 + (t & 1) * kStageBytes;
    const int l = afresh(lane);
    const uint32_t offq = TL::offset(ld, wave, l), offd = TL::offset(D, wave, l);
    const bool whole = dh == DHP && row + BR <= S;
    TL::copy(to, base + (size_t)row * ld + (size_t)h * dh, ld, offq, whole, S - row, dh, wave, lane);
    TL::copy(to + TL::kBytes, dobase + (size_t)row * D + (size_t)h * dh, D, offd, whole, S - row, dh, wave, lane);
    // (lse, delta) of BR rows, over and over where they are fewer than the 64 lanes copy
    dma16(to + 2 * TL::kBytes, p.stat + (((size_t)b * a.heads + h) * SP + row) * 2, (uint32_t)(lane & (BR / 2 - 1)) * 16);
  };
  if (t_begin < t_end) issue(t_begin);  // on its way while the wave's own rows are fetched
  typename TY::Frag kf[KK], vf[KK];
  {
    const int j = min(key, S - 1);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int d = 16 * kk + 8 * half;
      kf[kk] = TY::load(kbase + (size_t)j * ld + d, dh - d);
      vf[kk] = TY::load(vbase + (size_t)j * ld + d, dh - d);
    }
  }
  if constexpr (BIAS) {
    load_borders(p.db, first);
    if (t_begin < t_end) start_head(t_begin / nb);
  }
  wait_vmcnt<0>();
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(kf[kk]), "+v"(vf[kk]));

  floatx16 ak[TN], av[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) ak[j][r] = av[j][r] = 0.f;
  const float scale_log2 = p.scale * kLog2e;
  FarSum far_sum;
  for (int g = 0; g < group; ++g) {
    const int n_begin = max(0, t_begin - g * nb), n_end = min(nb, t_end - g * nb);
    float* table_sums = BIAS ? p.partials + (((size_t)b * gridDim.y + blockIdx.y) * a.heads + kvh * group + g) * p.db.count : nullptr;
    if (n_begin >= n_end) {  // a head of other parts
      if (BIAS && (int)threadIdx.x < p.db.count) table_sums[threadIdx.x] = 0.f;
      continue;
    }
    if constexpr (BIAS) {
      if (g * nb > t_begin) start_head(g);
    }
    for (int n = n_begin; n < n_end; ++n) {
      const int t = g * nb + n;
      wait_vmcnt<0>();
      lds_barrier();
      if (t + 1 < t_end) issue(t + 1);
      constexpr int kMine = BR / TEAMS;  // the wave's rows of the block
      const int skip = TEAMS == 1 ? 0 : team * 32, qb = (blk0 + n) * BR + skip;
      // wave uniform: distances of the wave's pairs in this block
      const int dlo = qb - (kw + 31), dhi = qb + kMine - 1 - kw;
      if (!active || dhi < d_from || dlo >= d_to) continue;
      const uint32_t stage = (t & 1) * kStageBytes, lq = lds0 + stage + skip * 128 + TL::row_base(afresh(lane)), lqc = lds0 + stage + skip * 128 + TL::col_base(afresh(lane));
      const float* lstat = reinterpret_cast<const float*>(lds + stage + 2 * TL::kBytes) + 2 * skip;
      const int d0 = qb - key + 4 * half;
#pragma unroll
      for (int u = 0; u < NT / TEAMS; ++u) {
        const int tlo = dlo + 32 * u, thi = tlo + 62;  // the tile's smallest and largest distance
        if (thi < d_from || tlo >= d_to) continue;
        const bool masked = tlo < d_from || thi >= end_of(kw + 31) || qb + 32 * u + 32 > S;
        floatx16 sacc, pacc;
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[r] = pacc[r] = 0.f;
        typename TY::Frag ahead[BIAS ? 1 : 2];
        pipelined<2 * KK>(ahead, [&](int i) { return TL::row_frag(lq, u, i >> 1, i & 1); },
                          [&](int i, const typename TY::Frag& f) {
                            if (TY::skips(16 * (i >> 1), dh)) return;
                            if (i & 1) pacc = TY::mma(f, vf[i >> 1], pacc);
                            else sacc = TY::mma(f, kf[i >> 1], sacc);
                          });
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!BIAS) {
          if (masked) {  // p = 0; what else reaches dK and dV from a query that is not finite, those rows are formed again without
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int at = 32 * u + 8 * (r >> 2) + (r & 3);
              const bool counts = (at >= d_from - d0) & (at < d_end - d0);
              sacc[r] = counts ? sacc[r] : -INFINITY;
              pacc[r] = counts ? pacc[r] : 0.f;
            }
          }
        }
        TileBuckets tb;
        if constexpr (BIAS) tb = TileBuckets(p.db, first, tlo, thi);  // without a bias there are no borders to look at
        if constexpr (BIAS) far_sum.start_tile(sums[wave], tb, lane);
        Diagonals diagonals;
#pragma unroll
        for (int v = 0; v < 2; ++v) {  // elements 8 v .. 8 v + 7: streamed rows 32 u + 16 v ..
          typename TY::Half ph[2], dsh[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {  // four rows at a time, which keeps few of their values alive
            const int row = 32 * u + 16 * v + 8 * q;
            float bias[4];
            if constexpr (BIAS) tile_bias<1>(*bl, tb, first, d0 + row, bias);
            const float4* sp = reinterpret_cast<const float4*>(lstat + 2 * (row + 4 * half));
            const float4 s0 = sp[0], s1 = sp[1];
            const float l2v[4] = {s0.x, s0.z, s1.x, s1.z}, dlv[4] = {s0.y, s0.w, s1.y, s1.w};
            float pe[4], de[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const int r = 8 * v + 4 * q + w;
              pe[w] = __builtin_amdgcn_exp2f((BIAS ? fmaf(sacc[r], scale_log2, bias[w]) : sacc[r] * scale_log2) - l2v[w]);
              de[w] = pe[w] * (pacc[r] - dlv[w]);
            }
            if constexpr (BIAS) {
              // Here for the table's sums, which are not formed again: p = dS = 0 whatever the score, the bias, dP and the query's lse and delta
              // are.  (As a second selection behind the other: 32 x 200 tokens 27 -> 30 us.)  128-wide heads have no registers for what it takes of the
              // lane, and work it out here: 33 spilled ones -> 23, 8 x 1024 tokens, all keys, 158 -> 154 us.
              if (masked) {
                const int l = DHP == 128 ? afresh(lane) : lane, j = kw + (l & 31), at = qb - j + 4 * (l >> 5) + row, end = min(end_of(j), S - j);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                  const bool counts = (at + w >= d_from) & (at + w < end);
                  pe[w] = counts ? pe[w] : 0.f;
                  de[w] = counts ? de[w] : 0.f;
                }
              }
            }
            if constexpr (BIAS) add_to_table(sums[wave], far_sum, diagonals, tb, first, p.db.count, d0 + row, lane, de);
            ph[q] = TY::half(pe);
            dsh[q] = TY::half(de);
            if constexpr (BIAS) __builtin_amdgcn_sched_barrier(0);
          }
          const typename TY::Frag pf = TY::join(ph[0], ph[1]), dsf = TY::join(dsh[0], dsh[1]);
          pipelined<2 * TN>(ahead, [&](int i) { return TL::col_frag(lqc, i >> 1, 2 * u + v, i & 1); },
                            [&](int i, const typename TY::Frag& f) {
                              if (TY::skips(32 * (i >> 1), dh)) return;
                              if (i & 1) av[i >> 1] = TY::mma(f, pf, av[i >> 1]);
                              else ak[i >> 1] = TY::mma(f, dsf, ak[i >> 1]);
                            });
        }
        if constexpr (BIAS) {
          if (tb.b0 < 0) sums[wave].near[kPad + thi - lane] += diagonals.sum;
        }
      }
    }
    if constexpr (BIAS) {
      // this head's sums: over the waves and halves by distance, then by bucket
      far_sum.flush(sums[wave], lane);
      __syncthreads();
      float* by_distance = bl->near;
      for (int i = threadIdx.x; i < kNearSize; i += 64 * NW) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) s += sums[w].near[i];
        by_distance[i] = s;
      }
      __syncthreads();
      // a bucket by 16 lanes; one after the other by whole waves, 8 of 32 each, took 5 to 10 thousand cycles
      for (int bk = threadIdx.x / 16; bk < p.db.count; bk += 4 * NW) {
        const int to = bk + 1 < p.db.count ? min(first[bk + 1], kNear + kPad) : kNear + kPad;
        float s = (lane & 15) < NW ? sums[lane & 15].far[bk] : 0.f;
#pragma unroll 4
        for (int d = first[bk] + (lane & 15); d < to; d += 16) s += by_distance[kPad + d];
        s = sum_over_lanes<8>(s);
        if ((lane & 15) == 0) table_sums[bk] = s;
      }
      __syncthreads();
    }
  }
  lds_barrier();
  if constexpr (TEAMS == 2) {  // the second team's sums to the first
    floatx4* mine = reinterpret_cast<floatx4*>(lds) + (size_t)(wave % (NW / TEAMS)) * 2 * TN * 4 * 64 + lane;
    if (team == 1) {
      hand_over(ak, mine);
      hand_over(av, mine + TN * 4 * 64);
    }
    lds_barrier();
    if (team == 0) {
      take_over(ak, mine);
      take_over(av, mine + TN * 4 * 64);
    }
    lds_barrier();
  }
  if (!active || team != 0) return;
  // Where a row of dK and dV goes: to dx, or, if it is a sum of several workgroups', as fp32 to their parts: those of parts of the walk
  // hold all keys, those of far pairs the first ones.
  const int joined = far ? a.sinks : p.parts > 1 ? S : p.far_blocks > 0 ? a.sinks : 0;
  const size_t nz = gridDim.x, part_rows = p.parts > 1 ? S : a.sinks;
  float* to = p.sums + (far ? p.parts * nz * part_rows + (chunk * nz + blockIdx.x) * a.sinks : (part * nz + blockIdx.x) * part_rows) * 2 * dh;
  T* dk = p.dx + (size_t)b * S * ld + D + (size_t)kvh * dh;
  T* dv = dk + (size_t)a.kv * dh;
  const int there_end = far ? a.sinks : S;
  float* turn = reinterpret_cast<float*>(lds) + wave * (kTurnBytes / 4);
  auto store = [&](int which) {
    return [=](int r, int col, const float (&v)[8]) {
      const int j = kw + r;
      if (j >= there_end) return;
      if (j < joined) Type<float>::store8(to + ((size_t)j * 2 + which) * dh + col, v, dh - col);
      else TY::store8((which ? dv : dk) + (size_t)j * ld + col, v, dh - col);
    };
  };
  turned_rows(ak, p.scale, turn, lane, store(0));
  turned_rows(av, 1.f, turn, lane, store(1));
  uint32_t redo = rows_to_redo(finite(ak) && finite(av), key < there_end);
  if (redo) wait_vmcnt<0>();
  for (; redo; redo &= redo - 1) {
    const int j = kw + __builtin_ctz(redo);
    float rk[2] = {}, rv[2] = {};
    for (int g = 0; g < group; ++g) {
      const int h = kvh * group + g;
      // queries of this workgroup's steps that see the key
      const int n0 = max(0, t_begin - g * nb), n1 = min(nb, t_end - g * nb);
      const int from = max((blk0 + n0) * BR, j + d_from), to_i = (int)min((long)min(S, (blk0 + n1) * BR), (long)j + end_of(j));
      const T* q = base + (size_t)h * dh;
      const T* dO = dobase + (size_t)h * dh;
      for (int i0 = from; i0 < to_i; i0 += 64) {
        const int i = i0 + lane;
        float pr = 0.f, ds = 0.f;
        if (i < to_i) {
          const float2 st = *reinterpret_cast<const float2*>(p.stat + (((size_t)b * a.heads + h) * SP + i) * 2);
          float e = row_dot(q + (size_t)i * ld, kbase + (size_t)j * ld, dh) * scale_log2 - st.x;
          if (BIAS) e += table(h)[bucket_of(p.db, first, i - j)] * kLog2e;
          pr = __builtin_amdgcn_exp2f(e);
          ds = pr * (row_dot(dO + (size_t)i * D, vbase + (size_t)j * ld, dh) - st.y);
        }
        const uint64_t which = __builtin_amdgcn_ballot_w64(i < to_i);
        add_rows(rk, ds, q + (size_t)i0 * ld, ld, which, dh, lane);
        add_rows(rv, pr, dO + (size_t)i0 * D, D, which, dh, lane);
      }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int col = lane + 64 * c;
      if (col >= dh) continue;
      if (j < joined) {
        to[((size_t)j * 2) * dh + col] = rk[c] * p.scale;
        to[((size_t)j * 2 + 1) * dh + col] = rv[c];
      } else {
        dk[(size_t)j * ld + col] = from_float<T>(rk[c] * p.scale);
        dv[(size_t)j * ld + col] = from_float<T>(rv[c]);
      }
    }
  }
}

// dK and dV from the parts of several workgroups, always in the same order: `parts` of [nz][rows][2][dh], then `chunks` of [nz][sinks][2][dh]
template <typename T>
__global__ __launch_bounds__(256) void local_join_kernel(Shape a, int parts, int chunks, size_t nz, int rows, const float* __restrict__ sums,
                                                         T* __restrict__ dx) {
  const size_t quad = (size_t)blockIdx.x * 256 + threadIdx.x, row = 2 * a.dh / 4, count = nz * rows * row;  // of four values
  if (quad >= count) return;
  const size_t zj = quad / row, z = zj / rows;
  const int in = (int)(quad - zj * row) * 4, j = (int)(zj - z * rows);
  const int which = in >= a.dh, d = in - which * a.dh;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float* at) {
    const float4 v = *reinterpret_cast<const float4*>(at);
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  };
  for (int p = 0; p < parts; ++p) add(sums + ((size_t)p * count + quad) * 4);
  if (j < a.sinks)
    for (int c = 0; c < chunks; ++c) add(sums + (size_t)parts * count * 4 + (((size_t)c * nz + z) * a.sinks + j) * 2 * a.dh + in);
  const size_t b = z / a.kv, kvh = z - b * a.kv;
  T* to = dx + ((size_t)b * a.S + j) * a.ld() + (size_t)(a.heads + which * a.kv + kvh) * a.dh + d;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
  else *reinterpret_cast<float4*>(to) = s;
}

constexpr int kWaves = 4;

// How the dK, dV launch is cut up.  Measured, launch and join, us:
//   8 x 1024 tokens, 16 key heads of 128, window 256, 4 first keys: one team 81, two 88; with far workgroups 87 and 94
//   1 x 16384, 8 heads of 128 on 2, window 1024: one part 257, two 246, four 232, eight 290; two teams 253, 224, 231, 318
//   4 x 777, 6 heads of 80 on 2, window 300, a bias: one team, one part 172, four parts 67; two teams 97 and 52; far pairs in place 65
//   32 x 200, 8 heads of 64, window 64, a bias: far pairs in place 29, far workgroups 44
// and in fp32 the whole backward pass, planned with two workgroups a CU and with the one that heads above 64 leave room for:
//   8 x 300, 8 heads of 128, all keys: 190 and 157; 1 x 4096, 4 heads of 128 on one, window 512: 315 and 250; 4 x 512, 2 x 2048, 4 x 1024: the same
struct DkvPlan {
  int teams = 1, parts = 1;
  int far_blocks = 0, chunks = 0;  // workgroups for the far pairs of the first keys; none: those keys' own workgroups take them
  int rows = 0;                    // workgroups for a key head of a sequence
};
template <typename T, int DHP>
DkvPlan dkv_plan(const LocalAttention& a) {
  constexpr int BR = kBlockRows<T, DHP>;
  // workgroups the chip runs at a time: two on a CU, but one of fp32 heads above 64, whose waves take 384 registers
  constexpr double kSlots = sizeof(T) == 4 && DHP == 128 ? 256 : 512;
  // a step of a workgroup whose waves each take whole blocks; in fp32 its matrix instructions alone, at either width
  constexpr double kStep = sizeof(T) == 4 ? 7.0e-6 : 2.6e-6 * DHP / 128;
  const long nz = (long)a.seqs * a.kv, group = a.heads / a.kv;
  const bool causal = a.window >= a.S;
  DkvPlan best;
  double best_time = 0;
  for (int teams = 1; teams <= BR / 32; ++teams) {
    const int own = 128 / teams, blocks = (a.S + own - 1) / own;
    // Times in steps; starting and ending a workgroup cost three, and a step of two teams 0.6.
    auto steps = [&](long queries) { return (double)((std::min<long>(a.S, queries) + BR - 1) / BR * group); };
    const double step = teams == 1 ? 1.0 : 0.6, walk = steps((long)own + a.window), far_walk = steps(a.S - a.window);
    for (int parts = 1; parts <= 16 && (parts == 1 || walk >= 4 * parts); ++parts) {
      for (int apart = 0; apart <= (a.sinks > 0 && !causal); ++apart) {  // far pairs in workgroups of their own
        DkvPlan f;
        f.teams = teams;
        f.parts = parts;
        if (apart) {
          // chunks as long as a part; no more of them than give every CU four, since each leaves its sums in memory
          f.far_blocks = (a.sinks + own - 1) / own;
          const long most = std::max<long>(1, 1024 / (nz * f.far_blocks));
          f.chunks = (int)std::min<long>(most, (long)std::ceil(far_walk / std::max(4.0, walk / parts)));
        }
        f.rows = blocks * parts + f.far_blocks * f.chunks;
        const bool longer = a.sinks > 0 && !apart;  // the first keys' workgroups
        const double one = 3 + step * std::max(walk / parts, apart ? far_walk / f.chunks : 0.0);
        const double first = longer ? 3 + step * steps(a.S) / parts : one, firsts = longer ? (double)nz * parts * ((a.sinks + own - 1) / own) : 0;
        const double all = (double)nz * f.rows;
        // equal walks run in rounds; those of a causal triangle, the longest first, fill one another's gaps
        double time = causal ? std::max(one, all * (3 + step * walk / parts / 2) / kSlots)
                             : std::max(first, std::ceil((firsts * first / one + all - firsts) / kSlots) * one);
        // parts meet in memory: written and read at some 4 TB/s, and a launch
        if (parts > 1 || apart) time += 1 + (parts > 1 ? (double)parts * nz * a.S * 2 * a.dh * 8 / 4e12 / kStep : 0.0);
        if (best.rows == 0 || time < best_time) {
          best = f;
          best_time = time;
        }
      }
    }
  }
  return best;
}
inline DkvPlan dkv_plan(int elt, const LocalAttention& a) {
  if (elt == ELT_BF16) return a.dh <= 64 ? dkv_plan<uint16_t, 64>(a) : dkv_plan<uint16_t, 128>(a);
  return a.dh <= 64 ? dkv_plan<float, 64>(a) : dkv_plan<float, 128>(a);
}
inline size_t stat_floats(const LocalAttention& a) { return (size_t)a.seqs * a.heads * stat_rows(a.S) * 2; }
inline int join_rows(const LocalAttention& a, const DkvPlan& f) { return f.parts > 1 ? a.S : f.far_blocks ? a.sinks : 0; }
inline size_t sum_floats(const LocalAttention& a, const DkvPlan& f) {
  return (size_t)a.seqs * a.kv * 2 * a.dh * ((size_t)f.parts * join_rows(a, f) + (size_t)f.chunks * a.sinks);
}
inline unsigned query_groups(const LocalAttention& a, int rows, int items = kWaves) {
  return (unsigned)(((long)(rows + 31) / 32 * (a.heads / a.kv) + items - 1) / items);
}
// Forward and dQ: two waves for 32 queries where one each would not give every SIMD of the 256 CUs a wave, and there is more than one tile to
// share.  fp32, 4 x 512 tokens, 8 heads of 64 (512 waves): forward 32 -> 18 us, dQ 40 -> 24; bf16, 4 x 777, 6 heads of 80 on 2 (624): 25 -> 19 and
// 27 -> 21; 32 x 200, 8 heads (2048): 16.6 -> 17.8 and 15.5 -> 19.1; 16 tokens: 4.4 -> 5.0 and the same.
inline bool in_teams(const LocalAttention& a) {
  return a.S > 32 && (long)a.seqs * a.kv * ((stat_rows(a.S) / 32) * (a.heads / a.kv)) <= 1024;
}

template <class Kernel>
hipError_t allow_lds(Kernel kernel) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
}

template <typename T, int DHP, bool BIAS>
hipError_t run_fwd(hipStream_t s, const LocalAttention& a, const FwdArgs<T>& p) {
  auto launch = [&](auto kernel, auto teams) {
    constexpr int kTeams = decltype(teams)::value;
    constexpr size_t lds = std::max<size_t>(4 * Tile<T, DHP, kWaves, 32 * kTeams>::kBytes, kWaves * kTurnBytes) + bias_lds<kWaves>(BIAS);
    static_assert(lds <= 160 * 1024, "stages and tables do not fit the LDS of a CU");
    static hipError_t attr = allow_lds(kernel);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(kernel, dim3(a.seqs * a.kv, query_groups(a, a.S, kWaves / kTeams)), dim3(64 * kWaves), lds, s, p);
    return hipGetLastError();
  };
  if (in_teams(a)) return launch(local_fwd_kernel<T, DHP, kWaves, 2, BIAS>, std::integral_constant<int, 2>());
  return launch(local_fwd_kernel<T, DHP, kWaves, 1, BIAS>, std::integral_constant<int, 1>());
}

template <typename T, int DHP, bool BIAS>
hipError_t run_bwd(hipStream_t s, const LocalAttention& a, const BwdArgs<T>& p) {
  using TL = Tile<T, DHP, kWaves>;
  constexpr size_t lds_q = std::max<size_t>(4 * TL::kBytes, kWaves * kTurnBytes) + bias_lds<kWaves>(BIAS);
  constexpr size_t lds_kv = std::max<size_t>(2 * (2 * TL::kBytes + 1024), kWaves * kTurnBytes) + dkv_bias_lds<kWaves>(BIAS);
  static_assert(lds_kv <= 160 * 1024, "tiles and sums do not fit the LDS of a CU");
  constexpr int kTeams = TL::BR / 32;
  auto dq = local_dq_kernel<T, DHP, kWaves, 1, BIAS>;
  auto dq_teams = local_dq_kernel<T, DHP, kWaves, kTeams, BIAS>;
  auto dkv = local_dkv_kernel<T, DHP, kWaves, 1, BIAS>;
  auto dkv_teams = local_dkv_kernel<T, DHP, kWaves, kTeams, BIAS>;
  static hipError_t attr_q = allow_lds(dq), attr_q_teams = allow_lds(dq_teams), attr_kv = allow_lds(dkv), attr_teams = allow_lds(dkv_teams);
  if (attr_q != hipSuccess) return attr_q;
  if (attr_q_teams != hipSuccess) return attr_q_teams;
  if (attr_kv != hipSuccess) return attr_kv;
  if (attr_teams != hipSuccess) return attr_teams;
  const bool teams = kTeams > 1 && in_teams(a);
  hipLaunchKernelGGL(teams ? dq_teams : dq, dim3(a.seqs * a.kv, query_groups(a, stat_rows(a.S), teams ? kWaves / kTeams : kWaves)), dim3(64 * kWaves),
                     lds_q, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const DkvPlan f = dkv_plan<T, DHP>(a);
  hipLaunchKernelGGL(f.teams == 1 ? dkv : dkv_teams, dim3(a.seqs * a.kv, f.rows), dim3(64 * kWaves), lds_kv, s, p);
  e = hipGetLastError();
  const int rows = join_rows(a, f);
  if (e != hipSuccess || rows == 0) return e;
  const size_t nz = (size_t)a.seqs * a.kv, quads = nz * rows * 2 * a.dh / 4;
  hipLaunchKernelGGL(local_join_kernel<T>, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, p.a, f.parts, f.chunks, nz, rows, p.sums, p.dx);
  return hipGetLastError();
}

template <typename T>
hipError_t fwd(hipStream_t s, const LocalAttention& a, const T* x, const float* table, float* kept, T* out, T* out2, float* lse) {
  const DistanceBuckets db = make_distance_buckets(a.buckets, a.max_distance);
  const FwdArgs<T> p{shape_of(a), db, near_buckets(db), x, table, kept, out, out2, lse, kLog2e / sqrtf((float)a.dh)};
  if (a.dh <= 64) return a.buckets ? run_fwd<T, 64, true>(s, a, p) : run_fwd<T, 64, false>(s, a, p);
  return a.buckets ? run_fwd<T, 128, true>(s, a, p) : run_fwd<T, 128, false>(s, a, p);
}

template <typename T>
hipError_t bwd(hipStream_t s, const LocalAttention& a, const T* x, const T* out, const T* dout, const float* lse, const float* kept, T* dx,
               float* partials, float* scratch) {
  const DkvPlan f = a.dh <= 64 ? dkv_plan<T, 64>(a) : dkv_plan<T, 128>(a);
  const DistanceBuckets db = make_distance_buckets(a.buckets, a.max_distance);
  const BwdArgs<T> p{shape_of(a), db, near_buckets(db), a.seqs_per_table, x, out, dout, lse, kept, dx, scratch,
                     scratch + stat_floats(a), partials, f.parts, f.far_blocks, f.chunks, 1.0f / sqrtf((float)a.dh)};
  if (a.dh <= 64) return a.buckets ? run_bwd<T, 64, true>(s, a, p) : run_bwd<T, 64, false>(s, a, p);
  return a.buckets ? run_bwd<T, 128, true>(s, a, p) : run_bwd<T, 128, false>(s, a, p);
}

}  // namespace

bool local_mfma_supported(int elt, const LocalAttention& a) {
  const int es = elt == ELT_BF16 ? 2 : 4;
  const size_t ld = (size_t)(a.heads + 2 * a.kv) * a.dh;
  return a.dh <= 128 && a.dh * es % 16 == 0 && (long)a.seqs * a.kv <= (1 << 22) && 64 * ld * es < (1ull << 31) &&
         query_groups(a, stat_rows(a.S)) <= 65535 && dkv_plan(elt, a).rows <= 65535;
}

size_t local_mfma_scratch_bytes(int elt, const LocalAttention& a) {
  return (stat_floats(a) + sum_floats(a, dkv_plan(elt, a))) * sizeof(float);
}

int local_mfma_table_rows(int elt, const LocalAttention& a) {
  return a.seqs * dkv_plan(elt, a).rows;
}

hipError_t local_mfma_fwd(hipStream_t s, int elt, const LocalAttention& a, const void* x, const float* table, float* kept, void* out, void* out2,
                          float* lse) {
  if (elt == ELT_BF16) return fwd(s, a, (const uint16_t*)x, table, kept, (uint16_t*)out, (uint16_t*)out2, lse);
  return fwd(s, a, (const float*)x, table, kept, (float*)out, (float*)out2, lse);
}

hipError_t local_mfma_bwd(hipStream_t s, int elt, const LocalAttention& a, const void* x, const void* out, const void* dout, const float* lse,
                          const float* kept, void* dx, float* partials, void* scratch) {
  if (elt == ELT_BF16)
    return bwd(s, a, (const uint16_t*)x, (const uint16_t*)out, (const uint16_t*)dout, lse, kept, (uint16_t*)dx, partials, (float*)scratch);
  return bwd(s, a, (const float*)x, (const float*)out, (const float*)dout, lse, kept, (float*)dx, partials, (float*)scratch);
}

}  // namespace tp
