// What the two kernels of attention behind shared prefixes agree on: how the keys of a prefix are cut, and where the
// results of the parts lie. (Host code too: the plan is tested without a GPU.)
#pragma once
#include <stdint.h>

namespace elasto {

constexpr int kPrefixTile = 128;  // rows of Q, and keys, of a tile

// A row is a query head at a query: rho = q row * hg + head of the tile. An item is one or two tiles of 128 rows of
// one prefix and key head (or part of its query heads); its key tiles are shared out over `split` CTAs. With one tile of
// rows (pair) the two groups of warps of a CTA take every other key tile and leave a part each.
struct PrefixPlan {
  int hg, nsub, qpt;  // query heads and queries of a tile, tiles across a head group
  int pair;           // 1: items of one tile of rows
  int split;          // CTAs of an item
  int64_t items;      // for each key head and part of its heads, at most (those that there are not end at once)
  int parts() const { return pair ? 2 * split : split; }
};

// rows: the queries that are to be expected; most: as many as there may be.
inline PrefixPlan prefix_plan(int64_t rows, int64_t most, int prefixes, int group, int heads_kv, int64_t max_prefix, int head_dim, int sms) {
  PrefixPlan p;
  p.nsub = (group + 31) / 32;
  p.hg = (group + p.nsub - 1) / p.nsub;
  p.qpt = kPrefixTile / p.hg;
  p.pair = rows <= static_cast<int64_t>(prefixes) * p.qpt;
  const int64_t step = p.pair ? p.qpt : 2LL * p.qpt;
  auto items = [&](int64_t n) {  // of n rows: each prefix's last item may be short, and each has a row at least
    const int64_t k = prefixes == 1 ? (n + step - 1) / step : n / step + prefixes;
    return k < n ? k : n;
  };
  p.items = items(most);
  const int64_t tiles = (max_prefix + kPrefixTile - 1) / kPrefixTile, ctas = items(rows) * heads_kv * p.nsub;
  // Microseconds: of a CTA's start and end, of a key tile, and of writing and reading a part of all rows.
  const double start = 4.0, tile = (p.pair ? 0.65 : 1.25) * (head_dim > 64 ? 1.0 : 0.7);
  const double part = static_cast<double>(rows) * group * heads_kv * (8.0 * head_dim + 16) * (p.pair ? 2 : 1) / 8e6;
  double best = 0.0;
  p.split = 1;
  for (int n = 1; n <= 64 && n <= tiles; ++n) {
    const double waves = static_cast<double>((ctas * n + sms - 1) / sms);
    const double cost = waves * (start + static_cast<double>((tiles + n - 1) / n) * tile) + n * part;
    if (n == 1 || cost < best) best = cost, p.split = n;
  }
  return p;
}

// Parts of the results: stat [part][key head x nsub][rho] (maximum and sum of each row) and
// sums [part][key head x nsub][channels / 4][rho] of four channels.
struct PrefixParts {
  float* sums;
  float* stat;
  int64_t rho;  // rows
  int hs, quads;  // key heads x nsub, head_dim / 4
#ifdef __CUDACC__
  __host__ __device__
#endif
  int64_t stat_at(int part, int h, int64_t row) const { return 2 * ((static_cast<int64_t>(part) * hs + h) * rho + row); }
#ifdef __CUDACC__
  __host__ __device__
#endif
  int64_t sums_at(int part, int h, int quad, int64_t row) const {
    return 4 * (((static_cast<int64_t>(part) * hs + h) * quads + quad) * rho + row);
  }
};

// The key tiles [first, last) of a CTA.
#ifdef __CUDACC__
__host__ __device__
#endif
inline int split_from(int tiles, int rank, int split) { return static_cast<int>(static_cast<int64_t>(tiles) * rank / split); }

}  // namespace elasto
