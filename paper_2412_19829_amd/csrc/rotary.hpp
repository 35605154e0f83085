// Rotary positions: pairs of channels of a head turn by an angle that goes with the row's position,
//   (a, b) -> f (a cos - b sin, b cos + a sin),  angle = position x the pair's frequency,
// the channels behind the first `rot` of a head as they are.
#pragma once

#include "common.hpp"

namespace gformer {

struct RotaryArgs {
  const void *q, *k;             // [total, H, d], [total, Hkv, d]; k may be null
  void *q_out, *k_out;           // may be q and k themselves
  const float* freqs;            // [rot / 2]
  const int32_t *positions;      // [total], or null: row i of sequence s is at start[s] + i (start null: i)
  const int32_t *cu, *start;
  int n_seqs, total, H, Hkv, d, rot;
  int interleaved, inverse, zero_tail;
  float factor;
  int64_t qs[2], ks[2], qos[2], kos[2];   // (row, head) strides
};
bool rotary_fits(int total);
hipError_t launch_rotary(const RotaryArgs& a, bool bf16, hipStream_t s);

}  // namespace gformer
