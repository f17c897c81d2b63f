// Attention in a sliding window, the first tokens staying visible (the definition
// is at elasto_op_window_attention), for chunks and whole sequences of queries.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale (q . k_j) - m)
//
// in one pass over the visible keys with the running maximum m and sum.
//
// A tile is 128 rows of Q: the `hg` query heads that share a key head, times
// 128 / hg consecutive queries, so grouped heads read K and V once and a tile
// spans few positions (fewer keys that only some of its rows see). A work item is
// two tiles of one sequence and key head; they share the K/V stream. Roles:
//   warp 0     TMA: Q of both tiles, then K and V tiles of 128 keys through a ring;
//   warp 1     tcgen05.mma: S = Q K^T into TMEM, O += P V with P read from TMEM;
//   warps 2-3  look through the V tiles that need it (below); at 64 channels warp 2 issues MMAs;
//   warps 4-11 two groups of four, one for each tile, a row a thread: scores from
//              TMEM to registers, mask, maximum, exp2, P back to TMEM (over S).
// While one group works on its scores the tensor cores run the other's products.
// O stays in TMEM; it is rescaled by its group only when a row's maximum has
// grown by more than 2^8 (else P simply is up to 2^8: exact in the sums, and the
// division at the end cancels it, as it does the power of two that keeps bf16 sums
// from overflowing). S(t) is issued after PV(t - 1), so its arrival
// also says that O is at rest.
//
// Key tiles have 128 keys, the last one and the one of the sinks 32 or 64 where
// that is enough; one that no row of a group sees is skipped for it. Tiles that all
// rows see wholly take no mask. In the others values that are not finite are set to
// zero before the product, since 0 * NaN would reach rows that do not see them. Rows
// that see such values get them at the end (put_bad_values): after such a tile, or
// where a result is not finite.
//
// Items differ in length (ragged sequences, causal rows, class tokens that see
// everything), so the grid has a block for each and the blocks that run take over
// those not yet started (cluster launch control), the longest first.
//
// Measured on a GB300 (captured calls): prompts of 8192, 7150 and 4140 tokens, 32 / 8 heads of 128, causal
// with a window of 1024: 249 us, 1.21 PFLOP/s of visible pairs. A pair of
// tiles costs ~2400 clocks a key tile where its products alone cost 2080 (the waits
// between S, softmax and PV that the other tile does not cover); the masked tiles at
// the window's two ends and an item's start and end are the rest. Four sequences
// of 4097 tokens, 12 heads of 64, 256 keys to either side and a class token: 77.5 us (when it was 76: 58
// without the class token: 7 more for its key tile in every item, the rest for its query, which sees all keys). A
// group's five tiles of the window are cut by it at both ends, and the softmax warps' chain (scores from TMEM, mask,
// maximum, exp2, P back) sets the pace, not the tensor cores (21 %).
// 16 queries against 8192 keys, 32 / 8 heads of 128: 19 us on clusters, 86 us without (Args::split).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int THREADS = 384;
// Registers of a thread: at launch, of the four producer and MMA warps, of the eight softmax warps.
constexpr int REGS = 168, REGS_FEW = 56, REGS_MANY = 224;
static_assert(128 * REGS_FEW + 256 * REGS_MANY <= THREADS * REGS, "register split");
constexpr int QT = 128, KT = 128;  // rows and keys of a tile
constexpr int HALF = 128 * 128;    // bytes of 128 rows of 64 16-bit values
constexpr int SMEM_LIMIT = 232448;
constexpr int TAIL = 768;             // barriers, items
constexpr int STAGING = 8 * 32 * 128;  // 32 rows of 64 channels of out for each softmax warp
constexpr int TMEM_COLS = 512, O_COL = 2 * KT;  // S (and P over it) of both groups, then O
constexpr int MAX_SPLIT = 8;
// Forms of the kernel: plain; with items for queries that see everything (make_item); an item's key tiles shared out
// over a cluster. (Apart, since what one needs in the loops cost the others: prompts 263 -> 287 us.)
enum Form { PLAIN, WIDE, SPLIT_KEYS };
constexpr float kLazy = 8.0f;  // log2 of how far a row's maximum may grow before O is rescaled

template <int DP>
struct Shape {
  static constexpr int halves = DP / 64, tile = halves * HALF;
  static constexpr int slots = DP == 128 ? 4 : 8;
  // MMA warps: at 64 channels one for each group, which then needs no step of the other (four images of 4097
  // tokens 84.9 -> 82.8 us); at 128, where the tensor cores have twice the work, two fell into step (prefill 272 -> 316 us).
  static constexpr int issuers = DP == 128 ? 1 : 2, lookers = 3 - issuers;
  static constexpr int smem = 1024 + (2 + slots) * tile + STAGING + TAIL;
};
static_assert(Shape<128>::smem <= SMEM_LIMIT && Shape<64>::smem <= SMEM_LIMIT, "shared memory");

struct Args {
  int batch, heads, heads_kv, group, head_dim;
  int causal, window, sinks;  // window and sinks cut to max_keys
  float scale_log2, down;  // P is 2^-down times the probability over the running maximum (sum_headroom)
  int max_queries, q_rows;
  const int* q_start;
  void* out;
  long long out_row, out_head;
  int max_keys, kv_rows;
  const int* kv_start;
  const int* kv_len;
  const uint16_t* v;
  long long v_batch, v_row, v_head;
  int hg, nsub, qpt;  // heads and queries of a tile, tiles across a head group
  int box_q;          // queries of 32 rows, 0 where hg does not divide 32
  int by_hg;          // row / hg = row * by_hg >> 16 (rows < 128, hg <= 32)
  int tiles;          // tiles (groups at work) of an item: 1 or 2
  int qtiles;         // items along the longest sequence's queries
  int wide;           // those in front of them for queries that see everything
  int items;
  int split;          // CTAs (a cluster) that share an item's key tiles, one tile of rows each
  Divisor per_q, by_nsub, by_heads_kv;  // items of a step along the queries; the axes of one
  int* status;
};

// Rows of q and keys of sequence b, cut to what the host allows.
__device__ __forceinline__ void sequence(const Args& a, int b, int& q0, int& nq, int& k0, int& nk) {
  q0 = b * a.max_queries, nq = a.max_queries;
  if (a.q_start) {
    q0 = min(max(a.q_start[b], 0), a.q_rows);
    nq = min(max(min(a.q_start[b + 1], a.q_rows) - q0, 0), a.max_queries);
  }
  k0 = 0, nk = a.max_keys;
  if (a.kv_start) {
    k0 = min(max(a.kv_start[b], 0), a.kv_rows);
    nk = min(max(min(a.kv_start[b + 1], a.kv_rows) - k0, 0), a.max_keys);
  } else if (a.kv_len) {
    nk = min(max(a.kv_len[b], 0), a.max_keys);
  }
}

// x[g] without an address, so that the arrays stay in registers.
template <typename T>
__device__ __forceinline__ T of(const T (&x)[2], int g) {
  return g ? x[1] : x[0];
}

// What every role derives alike for a work item. Key tile t holds the keys from base(t) on, width(t) of them; where
// `lead` is not 0 the first `lead` columns of tile 0 hold the first keys (the sinks) and only the rest follow base(0).
struct Item {
  int b, kvh, head0, nheads;    // first query head and how many of the tile's
  int q0, nq, k0, nk;
  int first[2], last[2];        // queries of each group's rows: [first, last] (empty: last < first)
  int tiles;                    // key tiles
  int sink_tiles, base0;        // those of the sinks alone, the first key of the others
  int sink_width, last_width;   // of the first of the sinks' and of the last tile (the others have KT keys)
  int lead;                     // columns of tile 0 for the sinks, in front of the band's first keys
  int with_sinks;               // tiles [0, with_sinks) hold sinks
  int from[2], to[2];           // and tiles [from, to] the keys that the group's rows see besides (none: to < from)
  int whole_from[2], whole_to[2];  // every row of the group sees every key of tiles [whole_from, whole_to]
  int pair;                     // 1: both groups have the same rows, group g the key tiles of parity g
  int begin, end;               // the CTA's tiles: [begin, end), all of them where a CTA has an item to itself

  __device__ __forceinline__ int base(int t) const { return t < sink_tiles ? t * KT : base0 + (t - sink_tiles) * KT; }
  __device__ __forceinline__ int width(int t) const {
    return t == tiles - 1 ? last_width : t < sink_tiles ? sink_width : KT;
  }
  __device__ __forceinline__ int key(int t, int col) const { return t == 0 && col < lead ? col : base(t) + col; }
  // The first and the last of the CTA's tiles that the group needs (none: last < first).
  __device__ __forceinline__ int first_tile(int g) const {
    const int f = of(from, g);
    return of(to, g) < f ? end : begin < with_sinks ? begin : max(f, begin);
  }
  __device__ __forceinline__ int last_tile(int g) const {
    const int f = of(from, g), band = min(of(to, g), end - 1), sinks = min(with_sinks, end) - 1;
    return of(to, g) < f ? -1 : band >= max(f, begin) ? max(band, sinks) : sinks >= begin ? sinks : -1;
  }
  // Some row of the group sees a key of the tile.
  template <int FORM>
  __device__ __forceinline__ bool needs(int g, int t) const {
    const int f = of(from, g), l = of(to, g);
    return l >= f && (FORM != WIDE || ((t ^ g) & pair) == 0) && (t < with_sinks || (t >= f && t <= l));
  }
  __device__ __forceinline__ bool whole(int g, int t) const { return t >= of(whole_from, g) && t <= of(whole_to, g); }
};

__device__ __forceinline__ int tile_width(int keys) { return keys <= 32 ? 32 : keys <= 64 ? 64 : KT; }

template <int FORM>
__device__ __forceinline__ Item make_item(const Args& a, int id, int rank) {
  Item it;
  int q = static_cast<int>(a.per_q.quotient(id)), r = id - q * static_cast<int>(a.per_q.d);
  if (a.causal) q = a.qtiles - 1 - q;  // the longest rows of keys first
  const int r1 = static_cast<int>(a.by_nsub.quotient(r)), sub = r - r1 * a.nsub;
  it.b = static_cast<int>(a.by_heads_kv.quotient(r1));
  it.kvh = r1 - it.b * a.heads_kv;
  it.head0 = it.kvh * a.group + sub * a.hg;
  it.nheads = min(a.hg, a.group - sub * a.hg);
  sequence(a, it.b, it.q0, it.nq, it.k0, it.nk);
  const int shift = it.nk - it.nq;
  // Queries that see everything, the first of a sequence, have items of their own: there all keys are visible (no
  // masks) and both groups share them; in a tile with other queries its 128 rows would take them all one after another.
  it.pair = 0;
  int wide = 0;
  if constexpr (FORM == WIDE) {
    wide = shift < 0 ? 0 : min(max(a.sinks - shift, 0), it.nq);
    q -= a.wide;
    if (q < 0) {
      const int first = (q + a.wide) * a.qpt, last = min(first + a.qpt, wide) - 1;
      it.base0 = it.sink_tiles = it.lead = it.with_sinks = it.sink_width = 0;
      it.tiles = last < first ? 0 : (it.nk + KT - 1) / KT;
      it.last_width = tile_width(it.nk - (it.tiles - 1) * KT);
      it.pair = it.tiles > 1;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        it.first[g] = first, it.last[g] = g <= it.pair ? last : first - 1;
        it.from[g] = g, it.to[g] = g <= it.pair ? it.tiles - 1 - (it.pair & (it.tiles - 1 - g)) : -1;
        it.whole_from[g] = 0, it.whole_to[g] = it.nk / KT - 1;
      }
      it.begin = 0, it.end = it.tiles;
      return it;
    }
  }
  int lo[2], hi[2], low = 0x7fffffff, high = -1, sinks = 0;  // the groups' bands of keys, and the item's
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    it.first[g] = wide + (q * a.tiles + g) * a.qpt;
    it.last[g] = g < a.tiles ? min(it.first[g] + a.qpt, it.nq) - 1 : it.first[g] - 1;
    const int pmax = shift + it.last[g], pmin = max(shift + it.first[g], 0);
    lo[g] = 0, hi[g] = -1;
    if (it.last[g] < it.first[g] || pmax < 0 || it.nk == 0) continue;
    if (a.causal) {
      lo[g] = max(0, pmin - a.window), hi[g] = pmax;
      sinks = max(sinks, min(a.sinks, pmax + 1));
    } else {
      sinks = min(a.sinks, it.nk);
      lo[g] = pmin < a.sinks ? 0 : max(0, pmin - a.window);
      hi[g] = pmin < a.sinks ? it.nk - 1 : max(min(it.nk - 1, pmax + a.window), sinks - 1);
    }
    low = min(low, lo[g]), high = max(high, hi[g]);
  }
  // The sinks: in the band's tiles where these begin close to them, else in the first columns of the band's first
  // tile where that saves a tile, else in tiles of their own.
  it.sink_tiles = it.lead = 0;
  if (sinks > 0) {
    const int cols = (sinks + 31) & ~31;
    if (low <= cols)
      low = 0;
    else if (cols < KT && (high - low) % KT + cols < KT)
      it.lead = cols, low -= cols;
    else
      it.sink_tiles = (sinks + KT - 1) / KT;
  }
  it.base0 = low;
  it.with_sinks = (sinks + KT - 1) / KT;
  it.sink_width = it.sink_tiles == 1 ? tile_width(sinks) : KT;
  it.tiles = high < 0 ? 0 : it.sink_tiles + (high - low) / KT + 1;
  it.last_width = tile_width(high + 1 - it.base(it.tiles - 1));
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    it.from[g] = 0, it.to[g] = -1, it.whole_from[g] = 0, it.whole_to[g] = -1;
    if (hi[g] < lo[g]) continue;
    it.from[g] = it.sink_tiles + (lo[g] - low) / KT;
    it.to[g] = it.sink_tiles + (hi[g] - low) / KT;
    const int pmin = shift + it.first[g], pmax = shift + it.last[g];
    if (pmin < 0) continue;
    // keys [pmax - window, until] (floor divisions: the differences may be negative)
    const int until = a.causal ? pmin : min(it.nk - 1, pmin + a.window);
    it.whole_from[g] = it.sink_tiles + max(it.lead > 0 ? 1 : 0, (pmax - a.window - low + KT - 1) >> 7);
    it.whole_to[g] = it.sink_tiles + ((until + 1 - low) >> 7) - 1;
  }
  it.begin = it.tiles * rank / a.split, it.end = it.tiles * (rank + 1) / a.split;
  return it;
}

// Bits [a, b] of a 32-bit word.
__device__ __forceinline__ uint32_t bits(int a, int b) {
  const uint32_t up = b < 0 ? 0u : b >= 31 ? 0xffffffffu : (2u << b) - 1u;
  return a <= 0 ? up : a > 31 ? 0u : up & (0xffffffffu << a);
}

// The columns of key tile t that the row at position p sees.
struct Seen {
  int a0, a1, b1;  // columns [a0, a1] and [0, b1]
  __device__ __forceinline__ uint32_t word(int w) const { return bits(a0 - 32 * w, a1 - 32 * w) | bits(0, b1 - 32 * w); }
};
__device__ __forceinline__ Seen seen_columns(const Args& a, const Item& it, int t, int p) {
  Seen s;
  const int base = it.base(t);
  int lo = max(p - a.window, 0), hi = a.causal ? p : min(p + a.window, it.nk - 1);
  int sinks = min(a.sinks, a.causal ? p + 1 : it.nk);
  if (!a.causal && p < a.sinks) lo = 0, hi = it.nk - 1;
  if (p < 0) hi = -1, sinks = 0;
  s.a0 = lo - base;
  s.a1 = t < it.sink_tiles || hi < 0 ? -1 : hi - base;
  s.b1 = sinks - 1 - (t == 0 && it.lead > 0 ? 0 : base);
  return s;
}

template <bool BF>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  return BF ? pack_bf16x2(lo, hi) : pack_f16x2(lo, hi);
}
template <bool BF>
__device__ __forceinline__ float2 unpack16(uint32_t w) {
  return BF ? make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u))
            : __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// Non-zero bits where one of the two values is infinite or NaN.
template <bool BF>
__device__ __forceinline__ uint32_t bad16(uint32_t w) {
  constexpr uint32_t e = BF ? 0x7f807f80u : 0x7c007c00u;
  const uint32_t x = (w & e) ^ e;  // a half of zeros: all exponent bits set
  return ((x & 0xffffu) == 0 ? 0xffffu : 0u) | ((x >> 16) == 0 ? 0xffff0000u : 0u);
}

// acc + 0 * w: NaN from the first infinite or NaN value on.
template <bool BF>
__device__ __forceinline__ void look16(uint32_t w, uint32_t& acc) {
  if constexpr (BF)
    asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(w), "r"(0u));
  else
    asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(w), "r"(0u));
}

// Sets the values of the first `rows` rows of a V tile that are not finite to zero (N
// threads, number r); the item's number goes to *flag if there were any.
template <bool BF, int DP, int N>
__device__ __forceinline__ void clear_bad_values(uint8_t* v, int rows, int r, int seq, volatile int* flag) {
  const int n = rows * 8;  // 16-byte pieces of 64 channels
  uint32_t acc = 0u;
#pragma unroll
  for (int h = 0; h < DP / 64; ++h)
    for (int i = r; i < n; i += 4 * N) {  // (rows is a multiple of 32)
      uint4 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = reinterpret_cast<const uint4*>(v + h * HALF)[i + N * k];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        look16<BF>(x[k].x, acc), look16<BF>(x[k].y, acc), look16<BF>(x[k].z, acc), look16<BF>(x[k].w, acc);
    }
  if (!__any_sync(0xffffffffu, bad16<BF>(acc) != 0)) return;
  *flag = seq;
  __threadfence_block();
  for (int h = 0; h < DP / 64; ++h)
    for (int i = r; i < n; i += N) {
      uint4* p = reinterpret_cast<uint4*>(v + h * HALF) + i;
      uint4 w = *p;
      w.x &= ~bad16<BF>(w.x), w.y &= ~bad16<BF>(w.y), w.z &= ~bad16<BF>(w.z), w.w &= ~bad16<BF>(w.w);
      *p = w;
    }
  fence_async_smem();
}

// A lane's four channels (2 lane, 2 lane + 1, and 64 more): which of them held values that are not finite, and their sums.
struct BadValues {
  uint32_t found[2];
  float2 sum[2];
};

// Adds what keys [from, to) hold. v: channel 2 lane of key 0.
template <bool BF>
__device__ __noinline__ BadValues look_through(BadValues x, const uint16_t* v, long long row, int from, int to, int channels) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (64 * i >= channels) continue;
#pragma unroll 8
    for (int j = from; j < to; ++j) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(v + j * row + 64 * i), bad = bad16<BF>(w);
      const float2 y = unpack16<BF>(w & bad);
      x.found[i] |= bad;
      x.sum[i].x += y.x, x.sum[i].y += y.y;
    }
  }
  return x;
}

// A channel in which a row sees an infinite or NaN value gets the sum of these, whatever their probabilities: the
// products leave them out where a tile is seen in part, and in other tiles make NaN of an infinity whose probability
// has rounded to 0. For rows row0 + i * step of the tile where bit i of `good` is set, by the warp. Rare, but without a
// second look at every key for every row: a row sees keys [0, s) and [lo, hi], and what all of them see is looked through
// once (8192 causal tokens, 8 heads of 128, an infinity at the start: 0.8 ms, 0.1 without; row by row 99).
template <bool BF>
__device__ __noinline__ void put_bad_values(const Args& a, const Item& it, int g, int row0, int step, uint32_t good, int lane) {
  __syncwarp();
  const int r = row0 + lane * step, q = r * a.by_hg >> 16, h = r - q * a.hg, qi = of(it.first, g) + q, p = it.nk - it.nq + qi;
  const bool on = (good >> lane & 1) && r < QT && q < a.qpt && qi <= of(it.last, g) && h < it.nheads && p >= 0;
  const uint32_t rows = __ballot_sync(0xffffffffu, on);
  if (rows == 0) return;
  const bool all = !a.causal && p < a.sinks;
  const int lo = all ? 0 : max(p - a.window, 0), hi = all ? it.nk - 1 : a.causal ? p : min(p + a.window, it.nk - 1);
  const int sinks = min(a.sinks, a.causal ? p + 1 : it.nk);
  const int lo_all = __reduce_max_sync(0xffffffffu, on ? lo : 0), hi_all = __reduce_min_sync(0xffffffffu, on ? hi : 0x7fffffff);
  const int sinks_all = __reduce_min_sync(0xffffffffu, on ? sinks : 0x7fffffff);
  const int channels = a.head_dim - 2 * lane;  // from this lane's first on
  const uint16_t* const v = a.v + (a.kv_start ? 0 : it.b * a.v_batch) + it.k0 * a.v_row + it.kvh * a.v_head + 2 * lane;
  BadValues shared = {{0u, 0u}, {{0.0f, 0.0f}, {0.0f, 0.0f}}};
  shared = look_through<BF>(shared, v, a.v_row, 0, sinks_all, channels);
  shared = look_through<BF>(shared, v, a.v_row, lo_all, hi_all + 1, channels);
  for (int i = 0; i < 32; ++i) {
    if (!(rows >> i & 1)) continue;
    const int l = __shfl_sync(0xffffffffu, lo, i), u = __shfl_sync(0xffffffffu, hi, i), n = __shfl_sync(0xffffffffu, sinks, i);
    BadValues x = look_through<BF>(shared, v, a.v_row, sinks_all, n, channels);
    x = look_through<BF>(x, v, a.v_row, l, min(lo_all, u + 1), channels);
    x = look_through<BF>(x, v, a.v_row, max(hi_all + 1, l), u + 1, channels);
    uint16_t* const out = static_cast<uint16_t*>(a.out) + static_cast<long long>(it.q0 + __shfl_sync(0xffffffffu, qi, i)) * a.out_row +
                          static_cast<long long>(it.head0 + __shfl_sync(0xffffffffu, h, i)) * a.out_head + 2 * lane;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (x.found[k]) {
        uint32_t* const o = reinterpret_cast<uint32_t*>(out + 64 * k);
        *o = (*o & ~x.found[k]) | (pack16<BF>(x.sum[k].x, x.sum[k].y) & x.found[k]);
      }
  }
  __syncwarp();
}

__device__ __forceinline__ float4 cluster_load4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ float2 cluster_load2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
  return v;
}

// The rows of a split item from the cluster's parts, in rank order, an equal share of the rows by each CTA (256 threads).
template <bool BF, int DP>
__device__ __forceinline__ void join(const Args& a, const Item& it, int rank, int thread, const float* part, const float2* stat,
                                     const int* bad_seq) {
  const int share = (QT + a.split - 1) / a.split, row0 = rank * share, row1 = min(row0 + share, QT);
  for (int e = thread; e < (row1 - row0) * (DP / 4); e += 256) {
    const int r = row0 + e / (DP / 4), piece = e % (DP / 4);
    const int q = r * a.by_hg >> 16, h = r - q * a.hg, qi = it.first[0] + q;
    if (q >= a.qpt || qi > it.last[0] || h >= it.nheads || 4 * piece >= a.head_dim) continue;
    const uint32_t ms = smem_addr(stat + r), os = smem_addr(part + r * DP + ((piece ^ (r & 7)) << 2));
    float2 st[MAX_SPLIT];
    float4 o[MAX_SPLIT];
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < MAX_SPLIT; ++k)
      if (k < a.split) st[k] = cluster_load2(cluster_map(ms, k)), o[k] = cluster_load4(cluster_map(os, k));
#pragma unroll
    for (int k = 0; k < MAX_SPLIT; ++k)
      if (k < a.split) top = fmaxf(top, st[k].x);
    float total = 0.0f, y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < MAX_SPLIT; ++k)
      if (k < a.split) {
        // (a part without a finite score has sums of zeros, or NaN that must stay)
        const float f = st[k].x == -INFINITY ? 1.0f : ex2_approx((st[k].x - top) * a.scale_log2);
        total += st[k].y * f;
        y[0] += o[k].x * f, y[1] += o[k].y * f, y[2] += o[k].z * f, y[3] += o[k].w * f;
      }
    const float inv = it.nk - it.nq + qi >= 0 ? 1.0f / total : 0.0f;
    uint32_t* const out = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + static_cast<long long>(it.q0 + qi) * a.out_row +
                                                      static_cast<long long>(it.head0 + h) * a.out_head + 4 * piece);
    *reinterpret_cast<uint2*>(out) = make_uint2(pack16<BF>(y[0] * inv, y[1] * inv), pack16<BF>(y[2] * inv, y[3] * inv));
  }
  bool bad = false;  // some CTA left values out, or has a sum that is not finite
  for (int k = 0; k < a.split; ++k) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(cluster_map(smem_addr(bad_seq), k)));
    bad |= v == 0;
  }
  if (!bad) return;
  named_bar_sync(1, 256);
  const Item copy = it;
  // a warp takes every eighth row, a lane each of them to see whether its sum is a number above 0
  const int lane = thread & 31, first = row0 + (thread >> 5), r = first + 8 * lane;
  float total = 0.0f;  // (whether it is 0 or NaN: the parts' weights do not matter)
  if (r < row1)
    for (int k = 0; k < a.split; ++k) total += cluster_load2(cluster_map(smem_addr(stat + r), k)).y;
  put_bad_values<BF>(a, copy, 0, first, 8, __ballot_sync(0xffffffffu, r < row1 && total > 0.0f), lane);
}

// A pair's second group hands its rows' maxima, sums and O to the first, 32 channels at a time through its staging
// (a row a thread, 16-byte pieces swizzled by the row); the first adds them to its own and returns the joint sum,
// and 0 beside it for a wait that gave up. n: pieces handed over so far. Out of line: they are rare, and the
// kernel's code has to fit the instruction caches.
template <int DP>
__device__ __noinline__ bool give(uint32_t o_tm, float2 stat, uint8_t* stage, uint64_t* given, uint64_t* taken, uint32_t n) {
  const int lane = threadIdx.x & 31;
  uint8_t* const row = stage + lane * 128;
  if (elect_one()) bulk_wait_read<0>();  // the staging's last store has read it
  __syncwarp();
  *reinterpret_cast<float2*>(row) = stat;
  mbar_arrive(given);
  for (int c = 0; c < DP; c += 32, ++n) {
    uint32_t o[32];
    tmem_ld_32x32b_x32(o_tm + c, o);
    tmem_ld_wait();
    if (!__all_sync(0xffffffffu, mbar_wait<true>(taken, n & 1))) return false;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      *reinterpret_cast<uint4*>(row + ((j ^ (lane & 7)) << 4)) = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
    mbar_arrive(given);
  }
  tc_fence_before();
  return __all_sync(0xffffffffu, mbar_wait<true>(taken, n & 1));
}
template <int DP>
__device__ __noinline__ float2 take_in(uint32_t o_tm, float2 own, float sc, const uint8_t* stage, uint64_t* given,
                                       uint64_t* taken, uint32_t n) {
  const int lane = threadIdx.x & 31;
  const uint8_t* const row = stage + lane * 128;
  if (!__all_sync(0xffffffffu, mbar_wait<true>(given, n & 1))) return make_float2(0.0f, 0.0f);
  const float2 other = *reinterpret_cast<const float2*>(row);
  mbar_arrive(taken);
  ++n;
  const float top = fmaxf(own.x, other.x);
  const float w0 = own.x == -INFINITY ? 0.0f : ex2_approx((own.x - top) * sc);
  const float w1 = other.x == -INFINITY ? 0.0f : ex2_approx((other.x - top) * sc);
  for (int c = 0; c < DP; c += 32, ++n) {
    uint32_t o[32];
    tmem_ld_32x32b_x32(o_tm + c, o);
    tmem_ld_wait();
    if (!__all_sync(0xffffffffu, mbar_wait<true>(given, n & 1))) return make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint4 x = *reinterpret_cast<const uint4*>(row + ((j ^ (lane & 7)) << 4));
      o[4 * j] = __float_as_uint(__uint_as_float(o[4 * j]) * w0 + __uint_as_float(x.x) * w1);
      o[4 * j + 1] = __float_as_uint(__uint_as_float(o[4 * j + 1]) * w0 + __uint_as_float(x.y) * w1);
      o[4 * j + 2] = __float_as_uint(__uint_as_float(o[4 * j + 2]) * w0 + __uint_as_float(x.z) * w1);
      o[4 * j + 3] = __float_as_uint(__uint_as_float(o[4 * j + 3]) * w0 + __uint_as_float(x.w) * w1);
    }
    mbar_arrive(taken);
    uint32_t lo[16], hi[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) lo[j] = o[j], hi[j] = o[16 + j];
    tmem_st_16(o_tm + c, lo);
    tmem_st_16(o_tm + c + 16, hi);
  }
  tmem_st_wait();
  return make_float2(own.y * w0 + other.y * w1, 1.0f);
}

template <bool BF, int DP, int FORM>
__global__ void __launch_bounds__(THREADS, 1)
    window_attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                            const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmK32,
                            const __grid_constant__ CUtensorMap tmV32, const __grid_constant__ CUtensorMap tmO,
                            const __grid_constant__ Args a) {
  using S = Shape<DP>;
  constexpr bool SPLIT = FORM == SPLIT_KEYS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* qbuf = smem;                 // [group] 128 rows, in halves of 64 channels
  uint8_t* ring = smem + 2 * S::tile;   // [slot] a K or V tile, in halves of 64 channels
  uint8_t* staging = ring + S::slots * S::tile;
  uint64_t* bars = reinterpret_cast<uint64_t*>(staging + STAGING);
  uint64_t* full = bars;                // [slot]
  uint64_t* empty = full + S::slots;    // [slot]
  uint64_t* q_full = empty + S::slots;  // [group]
  uint64_t* q_empty = q_full + 2;
  uint64_t* s_full = q_empty + 2;        // [group]
  uint64_t* p_full = s_full + 2;         // [group] four arrivals, of the warps
  uint64_t* o_full = p_full + 2;         // [group]
  uint64_t* drain = o_full + 2;          // [MMA warp]
  uint64_t* item_full = drain + 2;       // [2] item n is in items[n & 1]
  uint64_t* item_empty = item_full + 2;  // [2] read by the other warps
  uint64_t* answered = item_empty + 2;
  uint64_t* v_ready = answered + 1;      // [slot] the V tile there has been looked through
  uint64_t* given = v_ready + S::slots;  // 128 arrivals each: of a pair's second group, a piece of its result for
  uint64_t* taken = given + 1;           // the first is in its staging; of the first, that it has read it
  static_assert(3 * S::slots + 4 + 6 + 2 + 5 + 2 <= 48, "barriers");
  uint4* answer = reinterpret_cast<uint4*>(bars + 48);
  Item* items = reinterpret_cast<Item*>(answer + 1);  // [2]
  static_assert(48 * 8 + 16 + 2 * sizeof(Item) + 4 + 32 <= TAIL, "barriers and items");
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(items + 2);
  volatile int* bad_seq = reinterpret_cast<int*>(tmem_slot + 1);  // [8] item (by its number in this CTA) with bad values

  const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int rank = SPLIT ? static_cast<int>(blockIdx.x) % a.split : 0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::slots; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], i & 1 ? 3 : S::issuers);  // (V tiles, in the odd slots: the warps that look through them too)
      mbar_init(&v_ready[i], S::lookers);
    }
    for (int i = 0; i < 8; ++i) bad_seq[i] = -1;
    for (int g = 0; g < 2; ++g) {
      mbar_init(&q_full[g], 1);
      mbar_init(&q_empty[g], 1);
      mbar_init(&s_full[g], 1);
      mbar_init(&p_full[g], 4);
      mbar_init(&o_full[g], 1);
      mbar_init(&item_full[g], 1);
      mbar_init(&item_empty[g], 11);
    }
    mbar_init(&drain[0], 1);
    mbar_init(&drain[1], 1);
    mbar_init(answered, 1);
    mbar_init(given, 128);
    mbar_init(taken, 128);
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(static_cast<int>(*tmem_slot));
  pdl_wait();
  pdl_trigger();

  // Item n for a warp (all its lanes call): false after the last one, or when the wait gave up.
  auto take = [&](uint32_t n, Item& it) -> bool {
    if (!__all_sync(0xffffffffu, mbar_wait<true>(&item_full[n & 1], (n >> 1) & 1))) {
      if (lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
      return false;
    }
    it = items[n & 1];
    __syncwarp();
    if (lane == 0) mbar_arrive(&item_empty[n & 1]);
    return it.tiles >= 0;
  };
  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
  if (warp == 0) {
    // ------------------------------------------------------------ producer
    if (elect_one()) {
      tma_prefetch_desc(&tmQ);
      tma_prefetch_desc(&tmK);
      tma_prefetch_desc(&tmV);
      uint32_t seq = 0, nq[2] = {0, 0};  // K/V tiles and Q tiles issued
      bool ok = true;
      int id = SPLIT ? static_cast<int>(blockIdx.x) / a.split : static_cast<int>(blockIdx.x);
      for (uint32_t n = 0; ok; ++n) {
        ok = mbar_wait<true>(&item_empty[n & 1], ((n >> 1) & 1) ^ 1);
        if (!ok) break;
        Item it;
        it.tiles = -1;
        if (id >= 0) it = make_item<FORM>(a, id, rank);
        items[n & 1] = it;
        mbar_arrive(&item_full[n & 1]);
        if (id < 0) break;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (!ok || it.last_tile(g) < it.first_tile(g)) continue;
          ok = mbar_wait<true>(&q_empty[g], (nq[g] & 1) ^ 1);
          if (!ok) continue;
          mbar_expect_tx(&q_full[g], S::halves * a.hg * a.qpt * 128);
          for (int h = 0; h < S::halves; ++h)
            tma_load_3d(qbuf + g * S::tile + h * HALF, &tmQ, &q_full[g], 64 * h, it.head0, it.q0 + it.first[g]);
          ++nq[g];
        }
        const int batch = a.kv_start ? 0 : it.b;
        for (int t = SPLIT ? it.begin : 0; t < (SPLIT ? it.end : it.tiles) && ok; ++t) {
          const int width = it.width(t), row = it.k0 + it.base(t), lead = t == 0 ? it.lead : 0;
          for (int kv = 0; kv < 2 && ok; ++kv, ++seq) {
            const uint32_t slot = seq % S::slots;
            ok = mbar_wait<true>(&empty[slot], ((seq / S::slots) & 1) ^ 1);
            if (!ok) break;
            uint8_t* dst = ring + slot * S::tile;
            mbar_expect_tx(&full[slot], S::halves * width * 128);
            for (int h = 0; h < S::halves; ++h) {
              if (width == KT && lead == 0) {
                tma_load_4d(dst + h * HALF, kv ? &tmV : &tmK, &full[slot], 64 * h, it.kvh, row, batch);
              } else {
                for (int c = 0; c < width; c += 32)
                  tma_load_4d(dst + h * HALF + c * 128, kv ? &tmV32 : &tmK32, &full[slot], 64 * h, it.kvh, (c < lead ? it.k0 : row) + c, batch);
              }
            }
          }
        }
        if (!ok) break;
        if (SPLIT) {
          id = -1;
          continue;
        }
        // the next item, asked for once this one's loads are under way
        fence_async_smem();  // (the last answer has been read)
        mbar_expect_tx(answered, 16);
        request_block(answer, answered);
        ok = mbar_wait<true>(answered, n & 1);
        id = requested_block(answer);
      }
      if (!ok) record_status(a.status, ELASTO_ERR_TIMEOUT);
      // all copies have landed before the CTA exits
      for (uint32_t s = seq > S::slots ? seq - S::slots : 0; s < seq; ++s) mbar_wait<true>(&full[s % S::slots], (s / S::slots) & 1);
      for (int g = 0; g < 2; ++g)
        if (nq[g] > 0) mbar_wait<true>(&q_full[g], (nq[g] - 1) & 1);
    }
  } else if (warp <= S::issuers) {
    // ------------------------------------------------------------ MMA issuer
    // One warp for both groups alternates between them, a product and the scores that follow it each, so that the
    // one's run while the other group is at its scores. What the warp spends between MMAs paces the kernel too:
    // fields of the item in registers, and an MMA's operands, and the branches to it, known to be the same in all
    // lanes (tc_mma_warp).
    const int ksteps = (a.head_dim + 15) / 16;  // channels that the products take
    const uint32_t idesc_o = idesc_16_f32(QT, 16 * ksteps, !BF, false, true);
    constexpr uint32_t hi = sdesc_sw128_hi(1024);
    const uint32_t q_lo = sdesc_lo(smem_addr(qbuf), 16), kv_lo = sdesc_lo(smem_addr(ring), 0);
    constexpr uint32_t K_LBO = (16 >> 4) << 16, V_LBO = (HALF >> 4) << 16;  // leading byte offsets of K and V tiles
    uint32_t seq = 0, nq[2] = {0, 0}, np[2] = {0, 0};  // K/V tiles; of a group: items, P tiles
    bool ok = true, issued = false;
    Item it;
    for (uint32_t n = 0; ok && warp_uniform(take(n, it)); ++n) {
      const int tiles = warp_uniform(it.tiles), sink_tiles = warp_uniform(it.sink_tiles);
      const int sink_width = warp_uniform(it.sink_width), last_width = warp_uniform(it.last_width);
      const int begin = SPLIT ? warp_uniform(it.begin) : 0, end = SPLIT ? warp_uniform(it.end) : tiles;
      const int pair = FORM == WIDE ? warp_uniform(it.pair) : 0;
      int from[2], to[2], with_sinks[2], first[2], last[2];
      bool begun[2] = {false, false};
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        from[g] = warp_uniform(it.from[g]), to[g] = warp_uniform(it.to[g]);
        with_sinks[g] = warp_uniform(to[g] < from[g] ? 0 : it.with_sinks);
        first[g] = SPLIT ? warp_uniform(it.first_tile(g)) : with_sinks[g] > 0 ? 0 : from[g];
        last[g] = SPLIT ? warp_uniform(it.last_tile(g)) : max(to[g], with_sinks[g] - 1);
      }
      auto width = [&](int t) { return t == tiles - 1 ? last_width : t < sink_tiles ? sink_width : KT; };
      auto landed = [&](uint32_t s) {
        ok = ok && mbar_wait_warp<true>(&full[s % S::slots], (s / S::slots) & 1);
        tc_fence_after();
      };
      auto scores = [&](auto group, int t) {
        constexpr int g = decltype(group)::value;
        if (t >= end || !ok) return;
        const uint32_t slot = (seq + 2 * (t - begin)) % S::slots;
        if (S::issuers == 2 || g == 0) landed(seq + 2 * (t - begin));
        if (ok && ((t ^ g) & pair) == 0 && (t < with_sinks[g] || (t >= from[g] && t <= to[g]))) {
          if (t == first[g]) {
            ok = mbar_wait_warp<true>(&q_full[g], nq[g] & 1);
            if (!ok) return;
            ++nq[g];
            tc_fence_after();
          }
          const uint32_t k_lo = kv_lo + K_LBO + slot * (S::tile >> 4), idesc_s = idesc_16_f32(QT, width(t), !BF);
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            const uint32_t off = (k >> 2) * (HALF >> 4) + 2 * (k & 3);
            if (k < ksteps) tc_mma_warp_lo(tmem + g * KT, q_lo + g * (S::tile >> 4) + off, k_lo + off, hi, idesc_s, k != 0);
          }
          tc_commit_warp(&s_full[g]);
          if (t == last[g]) tc_commit_warp(&q_empty[g]);
          issued = true;
        }
        if (S::issuers == 2 || g == 1) tc_commit_warp(&empty[slot]);
      };
      auto product = [&](auto group, int t) {
        constexpr int g = decltype(group)::value;
        if (!ok) return;
        const uint32_t s = seq + 2 * (t - begin) + 1, slot = s % S::slots;
        if (S::issuers == 2 || g == 0) {
          landed(s);
          // (also where this group sees the tile wholly: what the other group sees in part is changed in place)
          ok = ok && mbar_wait_warp<true>(&v_ready[slot], (s / S::slots) & 1);
          tc_fence_after();
        }
        if (ok && ((t ^ g) & pair) == 0 && (t < with_sinks[g] || (t >= from[g] && t <= to[g]))) {
          ok = mbar_wait_warp<true>(&p_full[g], np[g] & 1);
          if (!ok) return;
          ++np[g];
          tc_fence_after();
          const uint32_t v_lo = kv_lo + V_LBO + slot * (S::tile >> 4);
          const int steps = width(t) / 16;
#pragma unroll
          for (int k = 0; k < KT / 16; ++k)
            if (k < steps)
              tc_mma_tmem_a_warp_lo(tmem + O_COL + g * DP, tmem + g * KT + 8 * k, v_lo + 128 * k, hi, idesc_o, begun[g] || k != 0);
          begun[g] = true;
          if (t == last[g]) tc_commit_warp(&o_full[g]);
        }
        if (S::issuers == 2 || g == 1) tc_commit_warp(&empty[slot]);
      };
      const std::integral_constant<int, 0> g0;
      const std::integral_constant<int, 1> g1;
      if constexpr (S::issuers == 2) {
        auto run = [&](auto g) {
          scores(g, begin);
          for (int t = begin; t < end && ok; ++t) {
            product(g, t);
            scores(g, t + 1);
          }
        };
        if (warp == 1)
          run(g0);
        else
          run(g1);
      } else {
        scores(g0, begin);
        scores(g1, begin);
        for (int t = begin; t < end && ok; ++t) {
          product(g0, t);
          scores(g0, t + 1);
          product(g1, t);
          scores(g1, t + 1);
        }
      }
      seq += 2 * (end - begin);
    }
    if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
    if (issued) {
      tc_commit_warp(&drain[warp - 1]);
      mbar_wait_warp<true>(&drain[warp - 1], 0);
    }
  } else if (warp < 4) {
    // ------------------------------------------------------------ a look through the V tiles with masks
    uint32_t seq = 0;
    bool ok = true;
    Item it;
    for (uint32_t n = 0; ok && take(n, it); ++n) {
      const int begin = SPLIT ? it.begin : 0, end = SPLIT ? it.end : it.tiles;
      for (int t = begin; t < end && ok; ++t) {
        // (every V tile is waited for and given back, so that no slot is ever two tiles ahead)
        const uint32_t vs = seq + 2 * (t - begin) + 1, slot = vs % S::slots;
        ok = mbar_wait_warp<true>(&full[slot], (vs / S::slots) & 1);
        if (!ok) break;
        const bool masked = (it.template needs<FORM>(0, t) && !it.whole(0, t)) || (it.template needs<FORM>(1, t) && !it.whole(1, t));
        if (masked) clear_bad_values<BF, DP, 32 * S::lookers>(ring + slot * S::tile, it.width(t), (warp - 4 + S::lookers) * 32 + lane, n, &bad_seq[n & 7]);
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&v_ready[slot]);
          mbar_arrive(&empty[slot]);
        }
      }
      seq += 2 * (end - begin);
    }
    if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
  } else {
    // ------------------------------------------------------------ softmax, a row a thread
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_MANY));
    const int g = (warp - 4) >> 2, r = (warp & 3) * 32 + lane;  // row of the tile = TMEM lane
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_tm = tmem + lanes + g * KT, o_tm = tmem + lanes + O_COL + g * DP;
    const float sc = a.scale_log2;
    uint8_t* const stage = staging + (warp - 4) * (STAGING / 8);
    // O's columns past those that the products write: zeros, so that the look for results that are not finite needs no
    // bound (with one prompts took 258 us in place of 251)
    for (int c = (a.head_dim + 15) & ~15; c < DP; c += 16) {
      uint32_t zero[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) zero[j] = 0u;
      tmem_st_16(o_tm + c, zero);
    }
    tmem_st_wait();
    uint32_t ns = 0, no = 0, nj = 0;  // score tiles and items of this group, pieces of results given or taken
    bool ok = true;
    Item it;
    for (uint32_t nth = 0; ok && take(nth, it); ++nth) {
      const int first = of(it.first, g), last = of(it.last, g);
      if (last < first) continue;
      const int own = r * a.by_hg >> 16;  // query of this row in the tile
      const int qi = first + own, head = r - own * a.hg;
      const bool mine = own < a.qpt && qi <= last && head < it.nheads;
      const int shift = it.nk - it.nq, p = shift + qi;
      const float lazy = mine ? kLazy : INFINITY;
      float m = -INFINITY, sum = 0.0f;
      bool any = false;
      // one key tile; MASKED: some row does not see some of its keys, or it has less than KT
      auto tile = [&](auto masked, int t) -> bool {
        constexpr int NC = KT / 32;
        constexpr bool MASKED = decltype(masked)::value;
        if (!__all_sync(0xffffffffu, mbar_wait<true>(&s_full[g], ns & 1))) return false;
        ++ns;
        tc_fence_after();
        uint32_t v[NC][32];
#pragma unroll
        for (int i = 0; i < NC; ++i) tmem_ld_32x32b_x32(s_tm + 32 * i, v[i]);
        tmem_ld_wait();
        uint32_t live = 15;  // words of 32 columns that some row of the warp sees
        if constexpr (MASKED) {
          const Seen s = seen_columns(a, it, t, p);
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            const uint32_t w = s.word(i);  // (no row sees a column past the tile's width)
            if (!__any_sync(0xffffffffu, w)) live &= ~(1u << i);
            if (__all_sync(0xffffffffu, w == 0xffffffffu) || !(live >> i & 1)) continue;
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (!(w >> j & 1)) v[i][j] = 0xff800000u;
          }
        }
        float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          if (MASKED && !(live >> i & 1)) continue;
#pragma unroll
          for (int j = 0; j < 32; j += 2)
            t4[(j >> 1) & 3] = max3(t4[(j >> 1) & 3], __uint_as_float(v[i][j]), __uint_as_float(v[i][j + 1]));
        }
        const float top = fmaxf(m, fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])));
        // (Rows without a query of this item have no vote: they hold a neighbour's values, or what an earlier kernel left in
        // shared memory, and a rescaling rounds every row's P anew. top - m is NaN while both are -inf: nothing seen yet,
        // nothing to rescale.)
        if (__any_sync(0xffffffffu, (top - m) * sc > lazy)) {
          const float keep = m == -INFINITY ? 0.0f : ex2_approx((m - top) * sc);
          if (any) {
            uint32_t o[32];
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
              tmem_ld_32x32b_x32(o_tm + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                const float2 x = mul2(make_float2(__uint_as_float(o[j]), __uint_as_float(o[j + 1])), make_float2(keep, keep));
                o[j] = __float_as_uint(x.x), o[j + 1] = __float_as_uint(x.y);
              }
              uint32_t lo[16], hi[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) lo[j] = o[j], hi[j] = o[16 + j];
              tmem_st_16(o_tm + c, lo);
              tmem_st_16(o_tm + c + 16, hi);
            }
            tmem_st_wait();
          }
          sum *= keep;
          m = top;
        }
        any = true;
        const float neg = m == -INFINITY ? 0.0f : fmaf(-m, sc, -a.down);
        const float2 sc2 = make_float2(sc, sc), neg2 = make_float2(neg, neg);
        float2 add[2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          uint32_t pk[16];
          if (MASKED && !(live >> i & 1)) {
#pragma unroll
            for (int j = 0; j < 16; ++j) pk[j] = 0u;
            tmem_st_16(s_tm + 16 * i, pk);
            continue;
          }
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float2 x = fma2(make_float2(__uint_as_float(v[i][j]), __uint_as_float(v[i][j + 1])), sc2, neg2);
            const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y));
            pk[j >> 1] = pack16<BF>(e.x, e.y);
            add[(j >> 1) & 1] = add2(add[(j >> 1) & 1], e);
          }
          tmem_st_16(s_tm + 16 * i, pk);
        }
        sum += (add[0].x + add[0].y) + (add[1].x + add[1].y);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[g]);
        return true;
      };
      for (int t = SPLIT ? it.begin : 0; t < (SPLIT ? it.end : it.tiles) && ok; ++t) {
        if (it.template needs<FORM>(g, t)) ok = it.whole(g, t) ? tile(std::false_type(), t) : tile(std::true_type(), t);
      }
      // ------------------------------------------------------------ result rows
      if (ok && any) {
        ok = __all_sync(0xffffffffu, mbar_wait<true>(&o_full[g], no & 1));
        ++no;
        tc_fence_after();
      }
      if constexpr (FORM == WIDE) {
        if (ok && it.pair) {
          const float2 stat = make_float2(m, sum);
          if (g) {
            ok = give<DP>(o_tm, stat, stage, given, taken, nj);
          } else {
            const float2 both = take_in<DP>(o_tm, stat, sc, stage + STAGING / 2, given, taken, nj);
            sum = both.x, ok = both.y != 0.0f;
          }
          nj += 1 + DP / 32;
          if (ok && g) continue;
        }
      }
      if (!ok) break;
      const bool sees = mine && p >= 0 && it.nk > 0;
      if constexpr (SPLIT) {
        // this CTA's maximum, sum and O of each row, for the cluster (the ring is done with: O is complete)
        float* const part = reinterpret_cast<float*>(ring) + r * DP;
        reinterpret_cast<float2*>(staging)[r] = make_float2(any ? m : -INFINITY, sum);
        float look = 0.0f;  // NaN after a value that is not finite
#pragma unroll 1
        for (int c = 0; c < DP; c += 32) {
          uint32_t o[32];
          if (any) {
            tmem_ld_32x32b_x32(o_tm + c, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = 0u;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)  // (16-byte pieces swizzled by the row: no bank conflicts)
            *reinterpret_cast<uint4*>(part + ((((c >> 2) + j) ^ (r & 7)) << 2)) = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
#pragma unroll
          for (int j = 0; j < 32; ++j) look = fmaf(__uint_as_float(o[j]), 0.0f, look);
        }
        if (sees && look != look && sum == sum) *bad_seq = static_cast<int>(nth);
        continue;
      }
      // the warp's 32 rows are whole queries of all the tile's heads
      const bool boxed = a.box_q > 0 && first + ((warp & 3) + 1) * a.box_q - 1 <= last && it.nheads == a.hg;
      const float inv = sees ? 1.0f / sum : 0.0f;  // (O of a row that sees nothing is 0)
      uint32_t look = 0u;  // NaN after a result that is not finite
      // (loops that are not unrolled: the kernel's code has to fit the instruction caches, where twice the code
      // made every part of it slower)
#pragma unroll 1
      for (int c0 = 0; c0 < DP; c0 += 64) {
#pragma unroll 1
        for (int c = 0; c < 64; c += 32) {
          uint32_t o[32];
          if (any) {
            tmem_ld_32x32b_x32(o_tm + c0 + c, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = 0u;
          }
          if (c == 0) {  // the staging's last store has read it
            if (elect_one()) bulk_wait_read<0>();
            __syncwarp();
          }
          // 16-byte pieces of a 128-byte row, so placed that writing a column and reading a row are without conflicts
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t pk[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 x = mul2(make_float2(__uint_as_float(o[8 * j + 2 * i]), __uint_as_float(o[8 * j + 2 * i + 1])), make_float2(inv, inv));
              pk[i] = pack16<BF>(x.x, x.y);
              look16<BF>(pk[i], look);
            }
            *reinterpret_cast<uint4*>(stage + lane * 128 + ((((c >> 3) + j) ^ (lane & 7)) << 4)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
          }
        }
        // Whole groups of rows leave by TMA. Else eight lanes write a row, 16 bytes each, so that whole sectors
        // leave together (a row a lane took ~100 clocks an instruction; this, with its addresses, 1300 a half).
        if (boxed) {
          fence_async_smem();
          __syncwarp();
          if (elect_one()) {
            tma_store_3d(&tmO, stage, c0, it.head0, it.q0 + first + (warp & 3) * a.box_q);
            bulk_commit();
          }
        } else {
          __syncwarp();
          uint16_t* const out = static_cast<uint16_t*>(a.out) + static_cast<long long>(it.q0 + first) * a.out_row +
                                static_cast<long long>(it.head0) * a.out_head + c0 + 8 * (lane & 7);
#pragma unroll 2
          for (int i = 0; i < 8; ++i) {
            const int k = 4 * i + (lane >> 3), row = (warp & 3) * 32 + k, q = row * a.by_hg >> 16, h = row - q * a.hg;
            if (c0 + 8 * (lane & 7) < a.head_dim && q < a.qpt && first + q <= last && h < it.nheads)
              *reinterpret_cast<uint4*>(out + q * a.out_row + h * a.out_head) =
                  *reinterpret_cast<const uint4*>(stage + k * 128 + (((lane & 7) ^ (k & 7)) << 4));
          }
        }
        __syncwarp();
      }
      // (a row whose sum is 0 or NaN has NaN in all channels)
      const uint32_t good = __ballot_sync(0xffffffffu, sees && sum > 0.0f);
      if (any && __any_sync(0xffffffffu, bad_seq[nth & 7] == static_cast<int>(nth) || ((good >> lane & 1) && bad16<BF>(look)))) {
        if (boxed) {
          if (elect_one()) bulk_wait_all();
          __syncwarp();
        }
        const Item copy = it;  // (in memory, which `it` itself is not)
        put_bad_values<BF>(a, copy, g, (warp & 3) * 32, 1, good, lane);
      }
      tc_fence_before();
    }
    if (elect_one()) bulk_wait_all();
    if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
    if constexpr (SPLIT) {
      __syncwarp();
      cluster_sync_all();
      join<BF, DP>(a, items[0], rank, threadIdx.x - 128, reinterpret_cast<const float*>(ring),
                   reinterpret_cast<const float2*>(staging), const_cast<const int*>(bad_seq));
    }
  }
  if constexpr (SPLIT) {
    __syncwarp();
    if (warp < 4) cluster_sync_all();
    cluster_sync_all();  // the peers have read this CTA's results
  }
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
  }
}

// [batch][rows][heads][channels] of 16-bit values in boxes of 64 channels x `box_heads` x `box_rows`.
bool map_of(CUtensorMap* tm, const void* p, bool bf, const elasto_window_attention_args& a, uint64_t heads, uint64_t rows,
            uint64_t batch, long long head_s, long long row_s, long long batch_s, uint32_t box_heads, uint32_t box_rows) {
  // (the stride of an axis of one element is never used; the encoder wants a multiple of 16 all the same)
  const uint64_t dims[4] = {static_cast<uint64_t>(a.head_dim), heads, rows, batch};
  const uint64_t strides[3] = {static_cast<uint64_t>(head_s) * 2, static_cast<uint64_t>(row_s) * 2,
                               static_cast<uint64_t>(batch_s) * 2};
  const uint32_t box[4] = {64, box_heads, box_rows, 1};
  return encode_tmap_16(tm, p, bf, batch_s >= 0 ? 4 : 3, dims, strides, box);
}

template <bool BF, int DP>
cudaError_t launch(const CUtensorMap (&tm)[6], const Args& a, cudaStream_t s) {
  if (a.split == 1)
    return launch_pdl(a.wide > 0 ? window_attention_kernel<BF, DP, WIDE> : window_attention_kernel<BF, DP, PLAIN>, dim3(a.items), dim3(THREADS), Shape<DP>::smem, s, tm[0], tm[1], tm[2],
                      tm[3], tm[4], tm[5], a);
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see launch_pdl
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.split;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(a.items * a.split);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = Shape<DP>::smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, window_attention_kernel<BF, DP, SPLIT_KEYS>, tm[0], tm[1], tm[2], tm[3], tm[4], tm[5], a);
}

// Clusters of n CTAs of the split kernels that the current device runs at once (one CTA takes an SM; asked for
// once a device and size).
cudaError_t max_clusters(int n, int* clusters) {
  static std::atomic<int> known[64][MAX_SPLIT + 1];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  *clusters = known[dev][n].load(std::memory_order_relaxed);
  if (*clusters > 0) return cudaSuccess;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = n;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3(n * (num_sms() / n));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = Shape<128>::smem;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaOccupancyMaxActiveClusters(clusters, window_attention_kernel<true, 128, SPLIT_KEYS>, &cfg);
  if (e != cudaSuccess) return e;
  if (*clusters <= 0) return cudaErrorInvalidConfiguration;
  known[dev][n].store(*clusters, std::memory_order_relaxed);
  return cudaSuccess;
}

cudaError_t init_attributes() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  // the register split adds up only if the kernels were built with the launch's count
  auto check = [&](auto* f) {
    cudaFuncAttributes at{};
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, f);
    if (e == cudaSuccess && at.numRegs != REGS) e = cudaErrorInvalidConfiguration;
  };
  auto all = [&](auto bf, auto dp) {
    auto one = [&](auto* f) {
      set(f, Shape<dp.value>::smem);
      check(f);
    };
    one(window_attention_kernel<bf.value, dp.value, PLAIN>);
    one(window_attention_kernel<bf.value, dp.value, WIDE>);
    one(window_attention_kernel<bf.value, dp.value, SPLIT_KEYS>);
  };
  const std::integral_constant<int, 64> d64;
  const std::integral_constant<int, 128> d128;
  all(std::true_type(), d64);
  all(std::false_type(), d64);
  all(std::true_type(), d128);
  all(std::false_type(), d128);
  return e;
}

}  // namespace

elasto_status window_attention_launch(const elasto_window_attention_args& u, int* status, cudaStream_t s) {
  static DeviceOnce once;
  ELASTO_CUDA_TRY(once(init_attributes));
  Args a{};
  a.batch = u.batch, a.heads = u.heads, a.heads_kv = u.heads_kv, a.group = u.heads / u.heads_kv, a.head_dim = u.head_dim;
  a.causal = u.causal != 0;
  a.window = u.window < 0 || u.window > u.max_keys ? u.max_keys : u.window;
  a.sinks = u.sinks > u.max_keys ? u.max_keys : u.sinks;
  a.scale_log2 = u.scale * 1.4426950408889634f;
  a.down = sum_headroom(u.dtype == ELASTO_BF16, u.max_keys);
  a.max_queries = static_cast<int>(std::min<long long>(u.max_queries, u.q_rows)), a.q_rows = static_cast<int>(u.q_rows), a.q_start = u.q_start;
  a.out = u.out, a.out_row = u.out_row, a.out_head = u.out_head;
  a.max_keys = u.max_keys, a.kv_rows = static_cast<int>(u.kv_rows), a.kv_start = u.kv_start, a.kv_len = u.kv_len;
  a.v = static_cast<const uint16_t*>(u.v), a.v_batch = u.v_batch, a.v_row = u.v_row, a.v_head = u.v_head;
  a.status = status;
  // heads of a tile: the whole group, or for more than 32 equal parts of it
  a.nsub = (a.group + 31) / 32;
  a.hg = (a.group + a.nsub - 1) / a.nsub;
  a.qpt = QT / a.hg;
  a.box_q = 32 % a.hg == 0 ? 32 / a.hg : 0;
  a.by_hg = (65536 + a.hg - 1) / a.hg;
  const long long per = static_cast<long long>(a.batch) * a.heads_kv * a.nsub;
  const long long rows = (a.max_queries + a.qpt - 1LL) / a.qpt;
  a.tiles = rows * per > num_sms() ? 2 : 1;  // one tile an item where the chip would be half empty
  long long qtiles = (rows + a.tiles - 1) / a.tiles;
  if (qtiles * per > 0x3fffffffLL) {
    set_error("elasto_op_window_attention: too many queries");
    return ELASTO_ERR_UNSUPPORTED;
  }
  a.qtiles = static_cast<int>(qtiles);
  // Few queries against many keys: the key tiles of an item shared out over a cluster, two at least for each CTA.
  long long keys = a.max_keys;  // of an item at most
  if (a.causal || a.sinks == 0) keys = std::min(keys, (a.causal ? 1LL : 2LL) * a.window + a.qpt + a.sinks);
  const long long key_tiles = (keys + KT - 1) / KT;
  // (As many as run at once: 16 clusters of 8 do not, and took 30 us where 16 of 7 take 18.)
  a.split = 1;
  if (a.tiles == 1)
    for (int n = static_cast<int>(std::min<long long>({MAX_SPLIT, num_sms() / (qtiles * per), key_tiles / 2})); n > 1 && a.split == 1; --n) {
      int clusters = 0;
      ELASTO_CUDA_TRY(max_clusters(n, &clusters));
      if (qtiles * per <= clusters) a.split = n;
    }
  // Items for queries that see everything, where the keys are more than three times those in an item's window: 4 x 4097
  // tokens with a window of 256 84.6 -> 77.9 us, 16000 tokens 216 -> 110; 4 x 2400 51.3 -> 50.9, but 8 x 1600 65.4 -> 67.7.
  // (Only while the items with them, and queries' numbers behind them, stay within an int.)
  const long long wide = (std::min(a.sinks, a.max_queries) + a.qpt - 1LL) / a.qpt;
  if (a.split == 1 && !a.causal && a.sinks > 0 && a.max_keys > 3 * (2LL * a.window + a.tiles * a.qpt) &&
      (qtiles + wide) * per <= 0x3fffffffLL && a.sinks + static_cast<long long>(a.max_queries) <= 1 << 30) {
    a.wide = static_cast<int>(wide);
    qtiles += wide;
  }
  a.items = static_cast<int>(qtiles * per);
  a.per_q = Divisor(static_cast<unsigned>(per)), a.by_nsub = Divisor(a.nsub), a.by_heads_kv = Divisor(a.heads_kv);
  const bool bf = u.dtype == ELASTO_BF16;
  const uint64_t kvb = u.kv_start ? 1 : u.batch;
  const long long kb = u.kv_start ? 0 : u.k_batch, vb = u.kv_start ? 0 : u.v_batch;
  CUtensorMap tm[6]{};
  if (!map_of(&tm[0], u.q, bf, u, u.heads, u.q_rows, 1, u.q_head, u.q_row, -1, a.hg, a.qpt) ||
      !map_of(&tm[1], u.k, bf, u, u.heads_kv, u.kv_rows, kvb, u.k_head, u.k_row, kb, 1, KT) ||
      !map_of(&tm[2], u.v, bf, u, u.heads_kv, u.kv_rows, kvb, u.v_head, u.v_row, vb, 1, KT) ||
      !map_of(&tm[3], u.k, bf, u, u.heads_kv, u.kv_rows, kvb, u.k_head, u.k_row, kb, 1, 32) ||
      !map_of(&tm[4], u.v, bf, u, u.heads_kv, u.kv_rows, kvb, u.v_head, u.v_row, vb, 1, 32) ||
      (a.box_q > 0 && !map_of(&tm[5], u.out, bf, u, u.heads, u.q_rows, 1, u.out_head, u.out_row, -1, a.hg, a.box_q))) {
    set_error("elasto_op_window_attention: cuTensorMapEncodeTiled failed (alignment, strides or size)");
    return ELASTO_ERR_UNSUPPORTED;
  }
  cudaError_t e;
  if (u.head_dim <= 64)
    e = bf ? launch<true, 64>(tm, a, s) : launch<false, 64>(tm, a, s);
  else
    e = bf ? launch<true, 128>(tm, a, s) : launch<false, 128>(tm, a, s);
  ELASTO_CUDA_TRY(e);
  return ELASTO_OK;
}

}  // namespace elasto
