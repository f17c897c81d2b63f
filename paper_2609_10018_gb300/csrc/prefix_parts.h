// What the kernels of attention behind shared prefixes agree on: how the keys of a prefix and of the sequences are cut, and
// where the results of the parts lie. (No CUDA here but the attributes: the plan is tested on the host.)
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define ELASTO_HD __host__ __device__
#define ELASTO_D __device__ __forceinline__
#else
#define ELASTO_HD
#define ELASTO_D inline
#endif

namespace elasto {

constexpr int kPrefixTile = 128;                 // rows of Q, and keys, of a tile
constexpr int kPrefixSplit = 64, kOwnSplit = 64;  // CTAs that share keys at most
constexpr int kMaxParts = 2 * kPrefixSplit + kOwnSplit;

// A row is a query head at a query: rho = q row * hg + head of the tile. An item is one or two tiles of 128 rows of
// one prefix and key head (or part of its query heads); its key tiles are shared out over `split` CTAs. With one tile of
// rows (pair) the two groups of warps of a CTA take every other key tile and leave a part each.
struct PrefixPlan {
  int hg, nsub, qpt;  // query heads and queries of a tile, tiles across a head group
  int pair;           // 1: items of one tile of rows
  int split;          // CTAs of an item
  int64_t items;      // for each key head and part of its heads, at most (those that there are not end at once)
  int many;           // 1: blocks of 64 rows of a sequence's own attention, 0: of 16
  int blocks;         // of a sequence and key head
  int own_split;      // CTAs that share a block's own keys
  int own_parts;      // what they leave behind the prefix's parts: one each, none where they join, or where there are no own keys
  int fused;          // 1: the kernel of the own keys (of 16 rows) joins its rows itself, with the prefix's one part
  int prefix_parts() const { return pair ? 2 * split : split; }
  int parts() const { return prefix_parts() + own_parts; }
};

struct PrefixSizes {
  int64_t rows, most;  // queries that are to be expected, and as many as there may be
  int batch, max_queries, prefixes, group, heads_kv, head_dim;
  int64_t max_prefix, max_keys;
  int sms;
};

inline PrefixPlan prefix_plan(const PrefixSizes& z) {
  PrefixPlan p;
  p.nsub = (z.group + 31) / 32;
  p.hg = (z.group + p.nsub - 1) / p.nsub;
  p.qpt = kPrefixTile / p.hg;
  p.pair = z.rows <= static_cast<int64_t>(z.prefixes) * p.qpt;
  const int64_t step = p.pair ? p.qpt : 2LL * p.qpt;
  auto items = [&](int64_t n) {  // of n rows: each prefix's last item may be short, and each has a row at least
    const int64_t k = z.prefixes == 1 ? (n + step - 1) / step : n / step + z.prefixes;
    return k < n ? k : n;
  };
  p.items = items(z.most);
  // The sequences' own keys: blocks of 64 rows where a sequence has more than 512, in which fewer rows read the keys again.
  // Calls with blocks of 64 and of 16 rows, in us (32 / 8 heads of 128): 512 new tokens of two sequences with caches of 32768 1895 and
  // 2420, 256 of eight with 4096 549 and 543, 150 of four with 8192 311 and 357; where a block has few keys its start weighs
  // more: one prompt of 2048 behind 8192 331 and 323, eight of 512 behind 1024 195 and 163; below 512 rows 128 tokens of
  // eight with 4096 309 and 368, 64 of 32 with 1024 200 and 179, prompts of 128 behind 4096 251 and 243. In CTAs until the SMs have six each, with four
  // tiles of 64 keys at least; else of 16 rows, in CTAs of a warp until the SMs have twelve, with 256 keys at least: sequences
  // of different lengths even out.
  const int64_t rows = static_cast<int64_t>(z.max_queries) * z.group;
  p.many = z.max_queries > 1 && rows > 512;
  const int64_t of = p.many ? 64 : 16, enough = (p.many ? 6LL : 12LL) * z.sms;
  p.blocks = static_cast<int>((rows + of - 1) / of);
  const int64_t units = static_cast<int64_t>(p.blocks) * z.batch * z.heads_kv;
  p.own_split = 1;
  while (p.own_split < kOwnSplit && units * p.own_split < enough && z.max_keys >= 512LL * p.own_split) p.own_split *= 2;
  while (!p.many && p.own_split < 4 && units * p.own_split < z.sms && z.max_keys >= 64LL * p.own_split) p.own_split *= 2;
  // How many CTAs share a prefix's keys. Both kernels run at the same time, the prefixes' with an SM a CTA, the other
  // on what is left. In microseconds: of a prefix's CTA its start and end and its key tiles (which wait longer for their
  // keys, where it alone reads them, while the other kernel reads at the memory's rate: 64 sequences behind 8192 keys took
  // 48 us with five CTAs a key head, 45 with eight); of a part of all rows, written and read; of the own keys (about 0.6 of
  // the longest each) the memory's time, and an SM's for all their CTAs (three at a time, or as if nine of one warp: with
  // twelve, as there are, drafts of 32 sequences got an SM too few and took 38 us in place of 30).
  const int64_t tiles = (z.max_prefix + kPrefixTile - 1) / kPrefixTile, each = items(z.rows), ctas = each * z.heads_kv * p.nsub;
  const double start = 5.0, tile = (p.pair ? 0.7 : 1.4) * (z.head_dim > 64 ? 1.0 : 0.7);
  const double part = (static_cast<double>(z.rows) * z.group * z.heads_kv * (8.0 * z.head_dim + 16) / 8e6 + 0.15) * (p.pair ? 2 : 1);
  const double keys = 0.6 * static_cast<double>(z.max_keys);
  const double memory = keys * 4.0 * z.head_dim * z.heads_kv * z.batch / 6.5e6;
  const double sm = static_cast<double>(units) * p.own_split * (4.0 + 0.03 * keys / p.own_split) / (p.many ? 3 : 9);
  auto own_rate = [&](double sms) {  // of all own keys, a microsecond
    const double t = z.max_keys == 0 ? 0.0 : sms <= 0.0 ? 1e9 : sm / sms > memory ? sm / sms : memory;
    return t > 0.01 ? 1.0 / t : 100.0;
  };
  double best = 0.0;
  p.split = 1;
  for (int n = 1; n <= kPrefixSplit && n <= tiles; ++n) {
    const int64_t waves = (ctas * n + z.sms - 1) / z.sms;
    const double left = waves > 1 ? 0.0 : static_cast<double>(z.sms - ctas * n);
    const double slow = 1.0 + (memory > 10.0 && left > 0.0 ? 0.6 * (left < 60 ? left / 60 : 1.0) : 0.0) * z.prefixes / static_cast<double>(each);
    const double prefix = static_cast<double>(waves) * (start + static_cast<double>((tiles + n - 1) / n) * tile * slow);
    const double done = prefix * own_rate(left);  // of the own keys
    const double cost = prefix + (done < 1.0 ? (1.0 - done) / own_rate(z.sms) : 0.0) + n * part;
    if (n == 1 || cost < best) best = cost, p.split = n;
  }
  p.fused = z.max_keys > 0 && !p.many && p.own_split == 1 && p.prefix_parts() == 1 && ctas >= z.sms;
  p.own_parts = p.fused || z.max_keys == 0 ? 0 : p.own_split;
  return p;
}

// Parts of the results, those of the prefix and then those of the own keys: stat [part][key head x nsub][rho] (maximum and
// sum of each row; the sum's sign is turned where the weighted sums do not show what the row sees: in an own part values that
// some row sees were left out, or all scores of the part are -infinity) and
// sums [part][key head x nsub][rho / 32][channels / 4][rho % 32] of four channels (not written where the maximum is
// -infinity): what a warp writes or reads of 32 rows lies together, all channels of them in one piece of 16 KB at most.
struct PrefixParts {
  float* sums;
  float* stat;
  int64_t rho;    // rows, a multiple of 32
  int hs, quads;  // key heads x nsub, head_dim / 4
  ELASTO_HD int64_t stat_at(int part, int h, int64_t row) const { return 2 * ((static_cast<int64_t>(part) * hs + h) * rho + row); }
  ELASTO_HD int64_t sums_at(int part, int h, int64_t row) const {  // of the first four channels, 128 floats from four to the next
    return 4 * (((static_cast<int64_t>(part) * hs + h) * (rho >> 5) + (row >> 5)) * quads * 32 + (row & 31));
  }
};
constexpr int kQuadStep = 128;

// The first key tile of a CTA.
ELASTO_HD inline int split_from(int tiles, int rank, int split) {
  return static_cast<int>(static_cast<int64_t>(tiles) * rank / split);
}

// A warp's way over the tiles [t0, t1) of `keys` keys each that it shares with other warps, of which all rows see the first
// `least` keys. came(i): whether tile number i has come; each warp waits for itself, and one may give up where another has
// just seen the tile. meet(i, t, ok): a tile that some rows see in part, behind which all warps wait for one another; work(i, t).
// A warp that has given up does nothing more, but meets the others at every such tile all the same: without it
// they would wait for ever. Whether all tiles came.
template <typename CAME, typename MEET, typename WORK>
ELASTO_D bool walk_tiles(int t0, int t1, int keys, int least, CAME came, MEET meet, WORK work) {
  bool ok = true;
  for (int t = t0, i = 0; t < t1; ++t, ++i) {
    ok = ok && came(i);
    if (least - t * keys < keys) meet(i, t, ok);
    if (ok) work(i, t);
  }
  return ok;
}

}  // namespace elasto
