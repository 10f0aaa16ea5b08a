// Log probabilities of given classes and the losses on them (see kernels_logprob.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tp {

// What is needed of a row once it has been read: its maximum and the sum of exp(z_j - top).
struct RowStats {
  float top, sum;
};

struct LogprobArgs {
  int rows, classes;
  const void* logits;   // [rows x classes] in elt
  const int32_t* ids;   // [rows], negative: no token
  float* logp;          // [rows]
  RowStats* stats;      // [rows], or null
  uint16_t* logp_rest;  // [rows] with stats: bf16, what rounding logp to fp32 has left over
  const float* weights; // [rows], or null: rows of weight 0 are left out, too
};
hipError_t launch_logprobs(hipStream_t s, int elt, const LogprobArgs& a);

// Partial sums of many losses
constexpr int kSumParts = 64;

struct PolicyArgs {
  int rows, classes;
  const void* logits;
  const int32_t* actions;
  const float *old_logp, *advantages;
  const float* weights;   // or null: 1 / rows
  const float* ref_logp;  // read where kl_weight > 0
  double log_low, log_high;  // log(1 - clip_low), log(1 + clip_high)
  double clip_low, clip_high, kl_weight;
  void* dlogits;
  float* logp;            // or null
  double* row_loss;       // scratch, [rows]
  double* parts;          // scratch, [kSumParts]
  uint32_t* counter;      // zero before the launch and after it
  float* loss;
  int first_row = 0;      // of this launch
};
hipError_t launch_policy(hipStream_t s, int elt, const PolicyArgs& a);

struct PreferenceArgs {
  int pairs, tokens, classes;  // rows = 2 pairs * tokens
  const void* logits;
  const int32_t* targets;
  const float* weights;   // or null: 1
  const float* ref_logp;  // [2 pairs]
  double beta, smoothing;
  void* dlogits;
  float* logp;            // [rows]
  RowStats* stats;        // scratch, [rows]
  uint16_t* logp_rest;    // scratch, [rows]
  float* pull;            // scratch, [2 pairs]: what a log probability of the sample weighs in the loss
  double* pair_loss;      // scratch, [pairs]
  double* parts;          // scratch, [kSumParts]
  uint32_t* counter;      // zero before the launch and after it
  float* loss;
};
hipError_t launch_preference(hipStream_t s, int elt, const PreferenceArgs& a);

}  // namespace tp
