// Rotary positions on packed queries | keys | values (see kernels_rotary.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tp {

constexpr int kMaxRotaryPairs = 128;  // heads of up to 256 values

struct Rotary {
  int seqs, S;       // samples and positions of each
  int turned, all;   // heads whose first `rotated` values are turned (queries and keys), and all of them (values behind)
  int dh, rotated;
  bool halves;       // pairs (i, i + rotated / 2), else (2i, 2i + 1)
  int first;         // position of a sample's first token
  float amplitude;
};
struct RotarySpeeds {
  double turns[kMaxRotaryPairs];  // of pair i per position, in whole turns
};
// The frequencies of a layer: base^(-2i / rotated), slowed down by `factor`, by parts where original > 0.  Host only.
void rotary_speeds(int rotated, double base, double factor, double original, double low, double high, RotarySpeeds* out);

// out = x with its pairs turned (back: by the negative angle); out may be x.  Any address of whole values.
hipError_t launch_rotary(hipStream_t s, int elt, const Rotary& r, const RotarySpeeds& speeds, bool back, const void* x, void* out);

}  // namespace tp
