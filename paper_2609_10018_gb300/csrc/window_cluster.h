// How many CTAs share a single token's keys (no CUDA here: tested on the host).
#pragma once

namespace elasto {

// A unit is a sequence, key head and part of its query heads; keys are those it may see. CTAs of a unit: until the SMs
// have two each (down to 128 keys a CTA), and where keys are many until there are enough CTAs to even out sequences of
// different lengths. most: the largest cluster that the device runs (a power of two).
inline int single_token_cluster(long long units, long long keys, int sms, int most) {
  int cluster = 1;
  while (2 * cluster <= most && ((units * cluster < 2 * sms && keys >= 256LL * cluster) ||
                                 (units * cluster < 8 * sms && keys >= 2048LL * cluster)))
    cluster *= 2;
  return cluster;
}

}  // namespace elasto
