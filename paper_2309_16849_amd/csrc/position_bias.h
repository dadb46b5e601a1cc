// position_bias.h -- buckets of a displacement for the learned position bias
// (device side; the same for the scores of kept neighbours and for the
// attention over cached frames).
#pragma once

#include "snls_internal.h"

#ifdef __HIPCC__

namespace snls {

// Edges are counted four at a time (the list is padded with +inf, which no
// displacement of a counting neighbour reaches).
SNLS_DEV int bias_bucket(float x, const Bias& b) {
  const float m = fabsf(x);
  int j = 0;
  for (int i = 0; i < b.nE; i += 4)
    j += (m >= b.edges[i]) + (m >= b.edges[i + 1]) + (m >= b.edges[i + 2]) + (m >= b.edges[i + 3]);
  return x < 0.f ? b.nE - j : b.nE + j;
}

SNLS_DEV int bias_step_bucket(int step, const Bias& b) { return min(max(step, -b.radius), b.radius) + b.radius; }

}  // namespace snls

#endif  // __HIPCC__
