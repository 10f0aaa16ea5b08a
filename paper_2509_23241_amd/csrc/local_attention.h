// Causal attention over a window of keys and a few first ones, with shared key heads and a learned bias per distance bucket.
// x: [seqs*S x (heads + 2 kv)*dh] (queries | keys | values; query head h reads key head h / (heads/kv)), out: [seqs*S x heads*dh].
// Query i of a sequence sees key j <= i where i - j < window or j < sinks; its scores are q.k / sqrt(dh) + table[h][bucket(i - j)].
// Activations in elt (0 fp32, 1 bf16), table, lse and all sums in fp32.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace tp {

constexpr int kMaxBuckets = 128;
constexpr int kMaxBucketDistance = 1 << 20;

// Bucket b starts at distance first[b]; the last has no end.  half = buckets / 2 distances have one each, the first of bucket
// half + t is the smallest whole d with d^n >= half^(n - t) * max_distance^t, n = buckets - half.
struct DistanceBuckets {
  int count;  // 0: no bias
  int half;
  float ratio;  // n / log2(max_distance / half)
  int first[kMaxBuckets];
};
DistanceBuckets make_distance_buckets(int buckets, int max_distance);

struct LocalAttention {
  int seqs, S, heads, kv, dh;
  int window;  // 1 .. S; S: all keys
  int sinks;   // 0 .. S
  int buckets, max_distance;  // 0, 0: no bias
  int seqs_per_table;         // backward: sequences that read the same kept table
};
bool local_attention_supported(const LocalAttention& a);

// table: [heads][buckets] or null.  kept (null without a table): a copy of the table is left there for the backward pass, which forms
// the probabilities again and must not read newer weights for that.  out2 (may be null): the output a second time.
hipError_t launch_local_attention_fwd(hipStream_t s, int elt, const LocalAttention& a, const void* x, const float* table, float* kept,
                                      void* out, void* out2, float* lse);
// dx from dout, the saved x, output and lse, and from the kept tables (seqs_per_table sequences each, one behind the other).
// dtable: [heads][buckets]; partials: local_attention_table_floats() floats for its sum; scratch: local_attention_scratch_bytes().
hipError_t launch_local_attention_bwd(hipStream_t s, int elt, const LocalAttention& a, const void* x, const void* out, const void* dout,
                                      const float* lse, const float* kept, void* dx, float* dtable, float* partials, void* scratch);
size_t local_attention_scratch_bytes(int elt, const LocalAttention& a);
size_t local_attention_table_floats(int elt, const LocalAttention& a);

}  // namespace tp
