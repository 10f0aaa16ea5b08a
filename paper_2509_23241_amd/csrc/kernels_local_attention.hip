// Windowed attention with first keys that stay visible, shared key heads and a learned bias per distance bucket: forward and
// backward for any head width and address.
//   s_ij = q_i.k_j / sqrt(dh) + table[bucket(i - j)],  p = softmax over the visible j,  y_i = sum_j p_ij v_j
//   dP_ij = dy_i.v_j,  delta_i = sum_j p_ij dP_ij,  dS = p (dP - delta)
//   dq_i = sum_j dS_ij k_j / sqrt(dh),  dk_j = sum_i dS_ij q_i / sqrt(dh),  dv_j = sum_i p_ij dy_i,  dtable[b] = sum of dS over pairs of bucket b
// The rows of dS sum to zero only as far as delta is right, and dtable is a sum of millions of them: delta = dy.y with y as it is
// stored (rounded to bf16) puts it off by 1e-3.  The first launch of the backward pass (dQ) starts from that delta, adds up the rows of
// its dS, whose sum is what delta was off by, and leaves the corrected delta for the second launch, which forms dK, dV and dtable.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "device_utils.h"
#include "kernels.h"
#include "local_attention_device.h"

namespace tp {

namespace {

// A whole number, 32 bits a word, lowest first: up to 64 factors of at most 2^20.
struct Whole {
  uint32_t word[41] = {1};
  int words = 1;
  void times(uint32_t factor, int how_often) {
    for (; how_often > 0; --how_often) {
      uint64_t carry = 0;
      for (int i = 0; i < words; ++i) {
        carry += (uint64_t)word[i] * factor;
        word[i] = (uint32_t)carry;
        carry >>= 32;
      }
      if (carry) word[words++] = (uint32_t)carry;
    }
  }
  bool operator<(const Whole& b) const {
    if (words != b.words) return words < b.words;
    for (int i = words - 1; i >= 0; --i)
      if (word[i] != b.word[i]) return word[i] < b.word[i];
    return false;
  }
};

}  // namespace

DistanceBuckets make_distance_buckets(int buckets, int max_distance) {
  DistanceBuckets d{};
  d.count = buckets;
  if (buckets == 0) return d;
  d.half = buckets / 2;
  const int n = buckets - d.half;
  d.ratio = (float)(n / std::log2((double)max_distance / d.half));
  for (int b = 0; b <= d.half; ++b) d.first[b] = b;
  const double step = std::log((double)max_distance / d.half) / n;
  for (int t = 1; t < n; ++t) {
    // The border is off by less than 1e-8 here.  Where a whole number is nearer than that could decide (borders come as close as 1e-9), whole
    // numbers do: the smallest d with d^n >= half^(n - t) max_distance^t.
    const double border = d.half * std::exp(step * t);
    const int near = (int)std::lround(border);
    if (std::fabs(border - near) > 1e-6) {
      d.first[d.half + t] = (int)std::ceil(border);
    } else {
      Whole at, want;
      at.times((uint32_t)near, n);
      want.times((uint32_t)d.half, n - t);
      want.times((uint32_t)max_distance, t);
      d.first[d.half + t] = at < want ? near + 1 : near;
    }
  }
  return d;
}

namespace {

constexpr int kThreads = 256;

// ---- any head width and address -------------------------------------------------------------------------------------------
// A workgroup owns 16 rows (four per wave) and walks over the other side in tiles staged in LDS as fp32; lane = pair for the dot
// products, lane = column for the sums.
constexpr int kRows = 16, kMaxDh = 256, kRW = kRows / 4, kND = kMaxDh / 64;
inline int tile_rows(int dh) { return dh <= 192 ? 64 : 32; }  // two tiles and twice 16 rows fit the LDS

template <typename T>
__device__ __forceinline__ void stage_rows(float* dst, const T* base, size_t ld, int count, int dh) {
  for (int i = threadIdx.x; i < count * dh; i += kThreads) {
    const int r = i / dh, d = i - r * dh;
    dst[r * (dh + 1) + d] = to_float(base[(size_t)r * ld + d]);
  }
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

struct Bias {  // a head's table and the borders in LDS, in units of log2
  float value[kMaxBuckets];
  int first[kMaxBuckets];
  __device__ __forceinline__ void load(const DistanceBuckets& d, const float* row) {
    for (int b = threadIdx.x; b < d.count; b += blockDim.x) {
      value[b] = row[b] * kLog2e;
      first[b] = d.first[b];
    }
  }
};

template <typename T>
__global__ __launch_bounds__(kThreads) void local_fwd_any_kernel(Shape a, int tile, DistanceBuckets db, const T* __restrict__ x,
                                                                 const float* __restrict__ table, float* __restrict__ kept,
                                                                 T* __restrict__ out, T* __restrict__ out2, float* __restrict__ lse,
                                                                 float scale_log2) {
  extern __shared__ float sm[];
  __shared__ Bias bias;
  const int dh = a.dh, S = a.S, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int blocks = (S + kRows - 1) / kRows, h = blockIdx.y;
  const int b = blockIdx.x / blocks, q0 = (blockIdx.x - b * blocks) * kRows;
  const size_t ld = a.ld(), D = (size_t)a.heads * dh;
  const int g = h / (a.heads / a.kv);
  const T* base = x + (size_t)b * S * ld;
  const T* kbase = base + D + (size_t)g * dh;
  const T* vbase = kbase + (size_t)a.kv * dh;
  float* qs = sm;                        // [kRows][dh + 1]
  float* ks = qs + kRows * (dh + 1);     // [tile][dh + 1]
  float* vs = ks + tile * (dh + 1);
  if (db.count) {
    bias.load(db, table + (size_t)h * db.count);
    if (blockIdx.x == 0)
      for (int t = threadIdx.x; t < db.count; t += kThreads) kept[h * db.count + t] = table[h * db.count + t];
  }
  const int nq = min(kRows, S - q0);
  stage_rows(qs, base + (size_t)q0 * ld + (size_t)h * dh, ld, nq, dh);
  float m[kRW], l[kRW], o[kRW][kND];
#pragma unroll
  for (int r = 0; r < kRW; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < kND; ++c) o[r][c] = 0.f;
  }
  const int last = q0 + nq - 1, lo = max(0, q0 - a.window + 1);  // keys the rows' windows reach
  for (int k0 = 0; k0 <= last; k0 += tile) {
    if (k0 >= a.sinks && k0 + tile <= lo) {  // nothing before the window's first tile
      k0 = lo / tile * tile - tile;
      continue;
    }
    const int nk = min(tile, S - k0);
    __syncthreads();
    stage_rows(ks, kbase + (size_t)k0 * ld, ld, nk, dh);
    stage_rows(vs, vbase + (size_t)k0 * ld, ld, nk, dh);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRW; ++r) {
      const int qi = wave * kRW + r, i = q0 + qi, j = k0 + lane;
      if (qi >= nq || k0 > i) continue;  // wave uniform
      float sc = -INFINITY;
      if (lane < nk && a.sees(i, j)) {
        float acc = 0.f;
        for (int d = 0; d < dh; ++d) acc = fmaf(qs[qi * (dh + 1) + d], ks[lane * (dh + 1) + d], acc);
        sc = acc * scale_log2;
        if (db.count) sc += bias.value[bucket_of(db, bias.first, i - j)];
      }
      const uint64_t seen = __builtin_amdgcn_ballot_w64(lane < nk && a.sees(i, j));
      if (seen == 0) continue;
      const float mn = fmaxf(m[r], max_over_lanes(sc));
      const float p = sc == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sc - mn);
      const float corr = m[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[r] - mn);
      l[r] = l[r] * corr + sum_over_lanes(p);
      m[r] = mn;
#pragma unroll
      for (int c = 0; c < kND; ++c) {
        const int d = lane + 64 * c;
        float acc = o[r][c] * corr;
        if (64 * c < dh)
          for (uint64_t left = seen; left; left &= left - 1) {
            const int jj = __builtin_ctzll(left);
            const float pj = lane_value(p, jj);
            if (d < dh) acc = fmaf(pj, vs[jj * (dh + 1) + d], acc);
          }
        o[r][c] = acc;
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kRW; ++r) {
    const int qi = wave * kRW + r, i = q0 + qi;
    if (qi >= nq) continue;
    const float inv = 1.f / l[r];
#pragma unroll
    for (int c = 0; c < kND; ++c) {
      const int d = lane + 64 * c;
      if (d < dh) {
        const size_t at = ((size_t)b * S + i) * D + (size_t)h * dh + d;
        out[at] = from_float<T>(o[r][c] * inv);
        if (out2) out2[at] = from_float<T>(o[r][c] * inv);
      }
    }
    if (lane == 0) lse[((size_t)b * a.heads + h) * S + i] = (m[r] + __builtin_amdgcn_logf(l[r])) * kLn2;
  }
}

// dq; delta[(b*heads + h)*S + i], corrected by what the row's dS add up to
template <typename T>
__global__ __launch_bounds__(kThreads, 6) void local_dq_any_kernel(Shape a, int tile, DistanceBuckets db, int seqs_per_table,
                                                                const T* __restrict__ x, const T* __restrict__ out,
                                                                const T* __restrict__ dout, const float* __restrict__ lse,
                                                                const float* __restrict__ kept, T* __restrict__ dx,
                                                                float* __restrict__ delta, float scale) {
  extern __shared__ float sm[];
  __shared__ Bias bias;
  const int dh = a.dh, S = a.S, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int blocks = (S + kRows - 1) / kRows, h = blockIdx.y;
  const int b = blockIdx.x / blocks, q0 = (blockIdx.x - b * blocks) * kRows;
  const size_t ld = a.ld(), D = (size_t)a.heads * dh;
  const int g = h / (a.heads / a.kv);
  const T* base = x + (size_t)b * S * ld;
  const T* kbase = base + D + (size_t)g * dh;
  const T* vbase = kbase + (size_t)a.kv * dh;
  const T* obase = out + (size_t)b * S * D + (size_t)h * dh;
  const T* dobase = dout + (size_t)b * S * D + (size_t)h * dh;
  float* qs = sm;                        // [kRows][dh + 1]
  float* dos = qs + kRows * (dh + 1);
  float* ks = dos + kRows * (dh + 1);    // [tile][dh + 1]
  float* vs = ks + tile * (dh + 1);
  if (db.count) bias.load(db, kept + ((size_t)(b / seqs_per_table) * a.heads + h) * db.count);
  const int nq = min(kRows, S - q0);
  stage_rows(qs, base + (size_t)q0 * ld + (size_t)h * dh, ld, nq, dh);
  stage_rows(dos, dobase + (size_t)q0 * D, D, nq, dh);
  __syncthreads();
  float dl[kRW], l2[kRW], total[kRW], dq[kRW][kND];
#pragma unroll
  for (int r = 0; r < kRW; ++r) {
    const int qi = wave * kRW + r, i = q0 + qi;
    float s = 0.f;
    if (qi < nq)
      for (int d = lane; d < dh; d += 64) s = fmaf(dos[qi * (dh + 1) + d], to_float(obase[(size_t)i * D + d]), s);
    dl[r] = sum_over_lanes(s);
    l2[r] = qi < nq ? lse[((size_t)b * a.heads + h) * S + i] * kLog2e : 0.f;
    total[r] = 0.f;
#pragma unroll
    for (int c = 0; c < kND; ++c) dq[r][c] = 0.f;
  }
  const int last = q0 + nq - 1, lo = max(0, q0 - a.window + 1);
  auto walk = [&](auto products) {  // with products, or the sums of dS alone
    for (int k0 = 0; k0 <= last; k0 += tile) {
      if (k0 >= a.sinks && k0 + tile <= lo) {
        k0 = lo / tile * tile - tile;
        continue;
      }
      const int nk = min(tile, S - k0);
      __syncthreads();
      stage_rows(ks, kbase + (size_t)k0 * ld, ld, nk, dh);
      stage_rows(vs, vbase + (size_t)k0 * ld, ld, nk, dh);
      __syncthreads();
#pragma unroll
      for (int r = 0; r < kRW; ++r) {
        const int qi = wave * kRW + r, i = q0 + qi, j = k0 + lane;
        if (qi >= nq || k0 > i) continue;
        float ds = 0.f;
        const bool sees = lane < nk && a.sees(i, j);
        if (sees) {
          float sc = 0.f, dp = 0.f;
          for (int d = 0; d < dh; ++d) {
            sc = fmaf(qs[qi * (dh + 1) + d], ks[lane * (dh + 1) + d], sc);
            dp = fmaf(dos[qi * (dh + 1) + d], vs[lane * (dh + 1) + d], dp);
          }
          float e = sc * scale * kLog2e - l2[r];
          if (db.count) e += bias.value[bucket_of(db, bias.first, i - j)];
          ds = __builtin_amdgcn_exp2f(e) * (dp - dl[r]);
          total[r] += ds;
        }
        if constexpr (!decltype(products)::value) continue;
        const uint64_t seen = __builtin_amdgcn_ballot_w64(sees);
#pragma unroll
        for (int c = 0; c < kND; ++c) {
          const int d = lane + 64 * c;
          if (64 * c >= dh) continue;
          for (uint64_t left = seen; left; left &= left - 1) {
            const int jj = __builtin_ctzll(left);
            const float v = lane_value(ds, jj);
            if (d < dh) dq[r][c] = fmaf(v, ks[jj * (dh + 1) + d], dq[r][c]);
          }
        }
      }
    }
  };
  // Queries of at most 32 keys: what y was rounded to bf16 by is as much in dS as what rounds dS, and is taken out of delta ahead.
  if (sizeof(T) == 2 && (a.window + a.sinks <= 32 || q0 < 32)) {
    walk(std::false_type());
#pragma unroll
    for (int r = 0; r < kRW; ++r) {
      dl[r] += sum_over_lanes(total[r]);
      total[r] = 0.f;
    }
  }
  walk(std::true_type());
#pragma unroll
  for (int r = 0; r < kRW; ++r) {
    const int qi = wave * kRW + r, i = q0 + qi;
    if (qi >= nq) continue;
#pragma unroll
    for (int c = 0; c < kND; ++c) {
      const int d = lane + 64 * c;
      if (d < dh) dx[((size_t)b * S + i) * ld + (size_t)h * dh + d] = from_float<T>(dq[r][c] * scale);
    }
    const float off = sum_over_lanes(total[r]);
    if (lane == 0) delta[((size_t)b * a.heads + h) * S + i] = dl[r] + off;
  }
}

// dk, dv, and the partial sums of dtable, [workgroups of x][heads][buckets]: a workgroup takes row blocks blockIdx.x, + gridDim.x, ..
// of key head blockIdx.y.  The LDS holds the table's sums of all heads of the key head or, where those do not fit (BY_HEAD), of one, whose sums
// over a row block are added to the workgroup's own partial sums.  (Heads one by one where all would fit: 32 x 200 tokens, 8 heads of 20, 233 -> 265 us.)
template <typename T, bool BY_HEAD>
__global__ __launch_bounds__(kThreads) void local_dkv_any_kernel(Shape a, int tile, DistanceBuckets db, int seqs, int seqs_per_table,
                                                                 const T* __restrict__ x, const T* __restrict__ dout,
                                                                 const float* __restrict__ lse, const float* __restrict__ kept,
                                                                 const float* __restrict__ delta, T* __restrict__ dx,
                                                                 float* __restrict__ partials, float scale) {
  extern __shared__ float sm[];
  __shared__ Bias bias;
  const int dh = a.dh, S = a.S, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int blocks = (S + kRows - 1) / kRows, kvh = blockIdx.y, group = a.heads / a.kv;
  const size_t ld = a.ld(), D = (size_t)a.heads * dh;
  float* ks = sm;                        // [kRows][dh + 1]
  float* vs = ks + kRows * (dh + 1);
  float* qs = vs + kRows * (dh + 1);     // [tile][dh + 1]
  float* dos = qs + tile * (dh + 1);
  float* dl = dos + tile * (dh + 1);     // [tile]
  float* ls = dl + tile;                 // [tile]
  float* sums = ls + tile;               // [4 waves][group, or 1][buckets]
  float* table_sums = partials + ((size_t)blockIdx.x * a.heads + (size_t)kvh * group) * db.count;
  for (int t = threadIdx.x; t < 4 * (BY_HEAD ? 1 : group) * db.count; t += kThreads) sums[t] = 0.f;
  static_assert(kMaxBuckets <= kThreads, "a thread for each bucket of a head");
  if (BY_HEAD && (int)threadIdx.x < db.count)
    for (int n = 0; n < group; ++n) table_sums[(size_t)n * db.count + threadIdx.x] = 0.f;
  for (int at = blockIdx.x; at < seqs * blocks; at += gridDim.x) {
    const int b = at / blocks, j0 = (at - b * blocks) * kRows;
    const T* base = x + (size_t)b * S * ld;
    const T* kbase = base + D + (size_t)kvh * dh;
    const T* vbase = kbase + (size_t)a.kv * dh;
    const int nkeys = min(kRows, S - j0);
    __syncthreads();
    stage_rows(ks, kbase + (size_t)j0 * ld, ld, nkeys, dh);
    stage_rows(vs, vbase + (size_t)j0 * ld, ld, nkeys, dh);
    float dk[kRW][kND], dv[kRW][kND];
#pragma unroll
    for (int r = 0; r < kRW; ++r)
#pragma unroll
      for (int c = 0; c < kND; ++c) dk[r][c] = dv[r][c] = 0.f;
    for (int n = 0; n < group; ++n) {
      const int h = kvh * group + n;
      __syncthreads();
      if (db.count) bias.load(db, kept + ((size_t)(b / seqs_per_table) * a.heads + h) * db.count);
      // queries that see a key of the block: from its first on, all for first keys, else as far as the window reaches
      const int end = j0 < a.sinks ? S : (int)min((long)S, (long)j0 + nkeys - 1 + a.window);
      for (int i0 = j0 / tile * tile; i0 < end; i0 += tile) {
        const int ni = min(tile, S - i0);
        __syncthreads();
        stage_rows(qs, base + (size_t)i0 * ld + (size_t)h * dh, ld, ni, dh);
        stage_rows(dos, dout + ((size_t)b * S + i0) * D + (size_t)h * dh, D, ni, dh);
        for (int q = threadIdx.x; q < ni; q += kThreads) {
          const size_t row = ((size_t)b * a.heads + h) * S + i0 + q;
          dl[q] = delta[row];
          ls[q] = lse[row] * kLog2e;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRW; ++r) {
          const int kj = wave * kRW + r, j = j0 + kj, i = i0 + lane;
          if (kj >= nkeys || i0 + ni - 1 < j) continue;  // wave uniform
          float p = 0.f, ds = 0.f;
          int bucket = -1;
          const bool sees = lane < ni && a.sees(i, j);
          if (sees) {
            float sc = 0.f, dp = 0.f;
            for (int d = 0; d < dh; ++d) {
              sc = fmaf(qs[lane * (dh + 1) + d], ks[kj * (dh + 1) + d], sc);
              dp = fmaf(dos[lane * (dh + 1) + d], vs[kj * (dh + 1) + d], dp);
            }
            float e = sc * scale * kLog2e - ls[lane];
            if (db.count) {
              bucket = bucket_of(db, bias.first, i - j);
              e += bias.value[bucket];
            }
            p = __builtin_amdgcn_exp2f(e);
            ds = p * (dp - dl[lane]);
          }
          const uint64_t seen = __builtin_amdgcn_ballot_w64(sees);
          if (db.count) {
            // distances ascend with the lanes, so that each bucket's lanes are neighbours; they are added bucket by bucket
            for (uint64_t left = seen; left;) {
              const int which = __builtin_amdgcn_readlane(bucket, __builtin_ctzll(left));
              left &= ~__builtin_amdgcn_ballot_w64(bucket == which);
              const float s = sum_over_lanes(bucket == which ? ds : 0.f);
              if (lane == 0) sums[(BY_HEAD ? wave : wave * group + n) * db.count + which] += s;
            }
          }
#pragma unroll
          for (int c = 0; c < kND; ++c) {
            const int d = lane + 64 * c;
            if (64 * c >= dh) continue;
            for (uint64_t left = seen; left; left &= left - 1) {
              const int ii = __builtin_ctzll(left);
              const float pb = lane_value(p, ii), dsb = lane_value(ds, ii);
              if (d < dh) {
                dk[r][c] = fmaf(dsb, qs[ii * (dh + 1) + d], dk[r][c]);
                dv[r][c] = fmaf(pb, dos[ii * (dh + 1) + d], dv[r][c]);
              }
            }
          }
        }
      }
      if (BY_HEAD) {  // this head's sums to memory, and the LDS free for the next head's
        __syncthreads();
        if ((int)threadIdx.x < db.count) {
          float t = 0.f;
          for (int w = 0; w < 4; ++w) {
            t += sums[w * db.count + threadIdx.x];
            sums[w * db.count + threadIdx.x] = 0.f;
          }
          table_sums[(size_t)n * db.count + threadIdx.x] += t;
        }
      }
    }
#pragma unroll
    for (int r = 0; r < kRW; ++r) {
      const int kj = wave * kRW + r, j = j0 + kj;
      if (kj >= nkeys) continue;
#pragma unroll
      for (int c = 0; c < kND; ++c) {
        const int d = lane + 64 * c;
        if (d < dh) {
          T* row = dx + ((size_t)b * S + j) * ld + D + (size_t)kvh * dh + d;
          row[0] = from_float<T>(dk[r][c] * scale);
          row[(size_t)a.kv * dh] = from_float<T>(dv[r][c]);
        }
      }
    }
  }
  if (BY_HEAD) return;
  __syncthreads();
  for (int t = threadIdx.x; t < group * db.count; t += kThreads) {
    float s = 0.f;
    for (int w = 0; w < 4; ++w) s += sums[w * group * db.count + t];
    table_sums[t] = s;
  }
}

constexpr int kAnyTableRows = 512;  // partial sums of a table that the kernels above leave, at most
inline long any_blocks(const LocalAttention& a) { return a.seqs * (((long)a.S + kRows - 1) / kRows); }
inline int any_dkv_blocks(const LocalAttention& a) {
  return (int)(a.buckets ? std::min<long>(kAnyTableRows, any_blocks(a)) : any_blocks(a));
}
// LDS of the last kernel, which needs most
inline size_t any_lds(const LocalAttention& a, int table_heads) {
  const int tile = tile_rows(a.dh);
  return ((size_t)(2 * kRows + 2 * tile) * (a.dh + 1) + 2 * tile + (size_t)4 * table_heads * a.buckets) * sizeof(float);
}
inline bool tables_fit(const LocalAttention& a) { return any_lds(a, a.heads / a.kv) <= 156 * 1024; }

template <typename T>
hipError_t any_fwd(hipStream_t s, const LocalAttention& a, const T* x, const float* table, float* kept, T* out, T* out2, float* lse) {
  const int tile = tile_rows(a.dh);
  const size_t lds = (size_t)(kRows + 2 * tile) * (a.dh + 1) * sizeof(float);
  static hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(local_fwd_any_kernel<T>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, 158 * 1024);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(local_fwd_any_kernel<T>, dim3((unsigned)any_blocks(a), a.heads), dim3(kThreads), lds, s, shape_of(a), tile,
                     make_distance_buckets(a.buckets, a.max_distance), x, table, kept, out, out2, lse, kLog2e / sqrtf((float)a.dh));
  return hipGetLastError();
}

template <typename T>
hipError_t any_bwd(hipStream_t s, const LocalAttention& a, const T* x, const T* out, const T* dout, const float* lse, const float* kept,
                   T* dx, float* partials, float* delta) {
  const int tile = tile_rows(a.dh);
  const float scale = 1.0f / sqrtf((float)a.dh);
  const DistanceBuckets db = make_distance_buckets(a.buckets, a.max_distance);
  const size_t lds_q = (size_t)(2 * kRows + 2 * tile) * (a.dh + 1) * sizeof(float);
  static hipError_t attr_q = hipFuncSetAttribute(reinterpret_cast<const void*>(local_dq_any_kernel<T>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, 158 * 1024);
  auto dkv = tables_fit(a) ? local_dkv_any_kernel<T, false> : local_dkv_any_kernel<T, true>;
  static hipError_t attr_kv = hipFuncSetAttribute(reinterpret_cast<const void*>(local_dkv_any_kernel<T, false>),
                                                  hipFuncAttributeMaxDynamicSharedMemorySize, 158 * 1024);
  static hipError_t attr_by_head = hipFuncSetAttribute(reinterpret_cast<const void*>(local_dkv_any_kernel<T, true>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, 158 * 1024);
  if (attr_q != hipSuccess) return attr_q;
  if (attr_kv != hipSuccess) return attr_kv;
  if (attr_by_head != hipSuccess) return attr_by_head;
  hipLaunchKernelGGL(local_dq_any_kernel<T>, dim3((unsigned)any_blocks(a), a.heads), dim3(kThreads), lds_q, s, shape_of(a), tile, db,
                     a.seqs_per_table, x, out, dout, lse, kept, dx, delta, scale);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(dkv, dim3(any_dkv_blocks(a), a.kv), dim3(kThreads), any_lds(a, tables_fit(a) ? a.heads / a.kv : 1), s, shape_of(a), tile, db,
                     a.seqs, a.seqs_per_table, x, dout, lse, kept, delta, dx, partials, scale);
  return hipGetLastError();
}

}  // namespace

bool local_attention_supported(const LocalAttention& a) {
  return a.S >= 1 && a.dh >= 1 && a.dh <= kMaxDh && a.kv >= 1 && a.heads >= a.kv && a.heads % a.kv == 0 && a.heads <= 65535 &&
         any_blocks(a) <= (1 << 23);
}

size_t local_attention_scratch_bytes(int elt, const LocalAttention& a) {
  const size_t any = (size_t)a.seqs * a.heads * a.S * sizeof(float);
  return ((local_mfma_supported(elt, a) ? std::max(any, local_mfma_scratch_bytes(elt, a)) : any) + 255) / 256 * 256;
}

size_t local_attention_table_floats(int elt, const LocalAttention& a) {
  if (!a.buckets) return 0;
  const int rows = local_mfma_supported(elt, a) ? std::max(any_dkv_blocks(a), local_mfma_table_rows(elt, a)) : any_dkv_blocks(a);
  return (size_t)rows * a.heads * a.buckets;
}

static bool aligned(const void* a, const void* b, const void* c, const void* d) {
  return (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c | (uintptr_t)d) & 15) == 0;
}

hipError_t launch_local_attention_fwd(hipStream_t s, int elt, const LocalAttention& a, const void* x, const float* table, float* kept,
                                      void* out, void* out2, float* lse) {
  if (!local_attention_supported(a)) return hipErrorInvalidValue;
  if (local_mfma_supported(elt, a) && aligned(x, out, out2, nullptr)) return local_mfma_fwd(s, elt, a, x, table, kept, out, out2, lse);
  if (elt == ELT_BF16) return any_fwd(s, a, (const uint16_t*)x, table, kept, (uint16_t*)out, (uint16_t*)out2, lse);
  return any_fwd(s, a, (const float*)x, table, kept, (float*)out, (float*)out2, lse);
}

hipError_t launch_local_attention_bwd(hipStream_t s, int elt, const LocalAttention& a, const void* x, const void* out, const void* dout,
                                      const float* lse, const float* kept, void* dx, float* dtable, float* partials, void* scratch) {
  if (!local_attention_supported(a)) return hipErrorInvalidValue;
  hipError_t e;
  int rows;
  if (local_mfma_supported(elt, a) && aligned(x, out, dout, dx)) {
    e = local_mfma_bwd(s, elt, a, x, out, dout, lse, kept, dx, partials, scratch);
    rows = local_mfma_table_rows(elt, a);
  } else {
    float* delta = (float*)scratch;
    e = elt == ELT_BF16 ? any_bwd(s, a, (const uint16_t*)x, (const uint16_t*)out, (const uint16_t*)dout, lse, kept, (uint16_t*)dx, partials, delta)
                        : any_bwd(s, a, (const float*)x, (const float*)out, (const float*)dout, lse, kept, (float*)dx, partials, delta);
    rows = any_dkv_blocks(a);
  }
  if (e != hipSuccess || !a.buckets) return e;
  return launch_sum_partials(s, (size_t)a.heads * a.buckets, rows, partials, dtable);
}

}  // namespace tp
