// Attention behind shared prefixes (the definition is at elasto_op_prefix_attention): the prefixes' keys, each read
// once for all the sequences that share it.
//
//   m = max_j s_j,  l = sum_j exp(s_j - m),  o = sum_j exp(s_j - m) v_j,  s_j = scale q . k_j
//
// over a part of the prefix's keys, for every query head of every sequence; prefix_own.cu does the same with the
// sequences' own keys and joins the parts. All queries see all keys of their prefix, so there are no masks but at its
// end, and the queries of all its sequences are rows of the same tiles.
//
// Bound by the products. 8 prefixes of 2804 to 4097 keys, 3339 queries of 32 heads of 128 (456 CTAs with work, three waves): 150
// us, tensor pipe busy 63 % of the time; a pair of key tiles takes 1.4 us (1.32 at the rate of a library product). 256
// queries behind 16384 keys on 96 SMs, so that the own keys stream beside them: 63 us; 64 behind 8192 on 64 SMs: 21.
//
// Probabilities are rounded to the operand type, as tcgen05 takes P with V of the same type (P in two pieces would double half of
// the products). In bf16 that is an independent error of each term of rms 0.0017 of it, as large as that of rounding the result,
// and both together 0.0023 (relative 2-norm); in f16 an eighth of it. Maxima, sums (of the unrounded P), O and joins are fp32.
//
// A tile is 128 rows of Q: the hg query heads that share a key head, times 128 / hg consecutive queries. An item is two
// tiles that share the K/V stream or, where a prefix has no more rows than one, that tile for both groups of
// warps, each with every other key tile. Roles:
//   warp 0      TMA: Q, then K and V tiles of 128 keys through a ring;
//   warp 1      tcgen05.mma: S = Q K^T into TMEM, O += P V with P read from TMEM;
//   warp 2      zeroes the values behind the prefix's end (0 * NaN would reach the sums);
//   warps 4-11  two groups of four, a row a thread: scores from TMEM to registers, maximum, exp2, P back to
//               TMEM (over S). While one group works the tensor cores run the other's products.
// O stays in TMEM; it is rescaled by its group only when a row's maximum has grown by more than 2^8.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "prefix_own.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int THREADS = 384;
// Registers of a thread: at launch, of the four producer and MMA warps, of the eight softmax warps.
constexpr int REGS = 168, REGS_FEW = 88, REGS_MANY = 208;
static_assert(128 * REGS_FEW + 256 * REGS_MANY <= THREADS * REGS, "register split");
constexpr int QT = kPrefixTile, KT = kPrefixTile;
constexpr int HALF = 128 * 128;  // bytes of 128 rows of 64 16-bit values
constexpr int TAIL = 512;        // barriers, the item
constexpr int TMEM_COLS = 512, O_COL = 2 * KT;  // S (and P over it) of both groups, then O
constexpr float kLazy = 8.0f;                   // log2 of how far a row's maximum may grow before O is rescaled

template <int DP>
struct Shape {
  static constexpr int halves = DP / 64, tile = halves * HALF;
  static constexpr int slots = DP == 128 ? 5 : 8;  // (as many as fit: eight images 208 -> 202 us with the fifth)
  static constexpr int smem = 1024 + (2 + slots) * tile + TAIL;
};

struct Args {
  int batch, heads_kv, group, head_dim;
  float scale_log2, down;  // P is 2^-down times the probability over the running maximum (sum_headroom)
  int max_queries, q_rows;
  const int* q_start;
  int prefixes, max_prefix;
  const int* seq_start;
  const int* prefix_len;
  int hg, nsub, qpt;
  int by_hg;  // row / hg = row * by_hg >> 16 (rows < 128, hg <= 32)
  int pair, split;
  Divisor by_items, by_hs;
  PrefixParts parts;
  int* status;
};

struct Item {
  int prefix, from, to;  // query rows [from, to) of the item and what follows of its prefix
  int len;               // keys of the prefix
};

// The first query row of the sequences from seq_start[g] on.
__device__ __forceinline__ int first_row(const Args& a, int g) {
  int seq = g == 0 ? 0 : a.batch;
  if (a.seq_start) seq = min(max(a.seq_start[g], 0), a.batch);
  return a.q_start ? min(max(a.q_start[seq], 0), a.q_rows) : seq * a.max_queries;
}

// Item n over all prefixes (a warp; prefix -1: there is none).
__device__ __forceinline__ Item find_item(const Args& a, int n, int lane) {
  const int step = a.pair ? a.qpt : 2 * a.qpt;
  Item it = {-1, 0, 0, 0};
  for (int g0 = 0; g0 < a.prefixes; g0 += 32) {
    const int g = g0 + lane;
    int from = 0, to = 0;
    if (g < a.prefixes) from = first_row(a, g), to = max(first_row(a, g + 1), from);
    const int items = (to - from + step - 1) / step;
    int sum = items;  // of this lane's and the lanes' before
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    const uint32_t found = __ballot_sync(0xffffffffu, sum > n);
    if (found) {
      const int src = __ffs(found) - 1;
      it.prefix = g0 + src;
      it.from = __shfl_sync(0xffffffffu, from, src) + (n - __shfl_sync(0xffffffffu, sum - items, src)) * step;
      it.to = __shfl_sync(0xffffffffu, to, src);
      it.len = a.prefix_len ? min(max(a.prefix_len[it.prefix], 0), a.max_prefix) : a.max_prefix;
      return it;
    }
    n -= __shfl_sync(0xffffffffu, sum, 31);
  }
  return it;
}

template <bool BF>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  return BF ? pack_bf16x2(lo, hi) : pack_f16x2(lo, hi);
}

template <bool BF, int DP>
__global__ void __launch_bounds__(THREADS, 1)
    prefix_attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                            const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Args a) {
  using S = Shape<DP>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* qbuf = smem;                // [group] 128 rows, in halves of 64 channels
  uint8_t* ring = smem + 2 * S::tile;  // [slot] a K or V tile, in halves of 64 channels
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + S::slots * S::tile);  // [slot]
  uint64_t* empty = full + S::slots;                                        // [slot]
  uint64_t* q_full = empty + S::slots;
  uint64_t* s_full = q_full + 1;  // [group]
  uint64_t* p_full = s_full + 2;  // [group] four arrivals, of the warps
  uint64_t* o_full = p_full + 2;  // [group]
  uint64_t* drain = o_full + 2;
  uint64_t* last_full = drain + 1;     // the last V tile, where the prefix ends in it, has been copied,
  uint64_t* v_ready = last_full + 1;  // and zeroed behind the prefix's end
  static_assert(8 * (2 * S::slots + 10) + sizeof(Item) + 8 <= TAIL, "barriers and item");
  Item* found = reinterpret_cast<Item*>(v_ready + 1);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(found + 1);

  const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  // CTAs of one part of the keys of a key head are neighbours: they read the same K and V at the same time
  const int rest = static_cast<int>(a.by_items.quotient(blockIdx.x)), item = static_cast<int>(blockIdx.x - rest * a.by_items.d);
  const int rank = static_cast<int>(a.by_hs.quotient(rest)), h = rest - rank * static_cast<int>(a.by_hs.d);
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::slots; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    mbar_init(q_full, 1);
    for (int g = 0; g < 2; ++g) {
      mbar_init(&s_full[g], 1);
      mbar_init(&p_full[g], 4);
      mbar_init(&o_full[g], 1);
    }
    mbar_init(drain, 1);
    mbar_init(last_full, 1);
    mbar_init(v_ready, 1);
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, TMEM_COLS);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_trigger();
  if (warp == 0) {
    const Item it = find_item(a, item, lane);
    if (lane == 0) *found = it;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(static_cast<int>(*tmem_slot));

  const int kvh = h / a.nsub, head0 = kvh * a.group + (h - kvh * a.nsub) * a.hg, nheads = min(a.hg, (kvh + 1) * a.group - head0);
  const int prefix = warp_uniform(found->prefix), from = warp_uniform(found->from), to = warp_uniform(found->to);
  const int len = warp_uniform(found->len), tiles = (len + KT - 1) / KT;
  const int begin = prefix < 0 ? 0 : split_from(tiles, rank, a.split), end = prefix < 0 ? 0 : split_from(tiles, rank + 1, a.split);
  const int pair = a.pair;
  // group g's rows: from + g * qpt on (pair: the same rows, every other key tile)
  const bool second = pair || from + a.qpt < to;  // group 1 has rows
  const int left = len - (end - 1) * KT;  // keys of the last tile, where it is the prefix's
  const bool cut = end == tiles && left < KT;

  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
  if (begin >= end) {
    // nothing to do (the barriers below are common)
  } else if (warp == 0) {
    // ------------------------------------------------------------ producer
    if (elect_one()) {
      const int qtiles = pair || !second ? 1 : 2;
      mbar_expect_tx(q_full, qtiles * S::halves * a.hg * a.qpt * 128);
      for (int g = 0; g < qtiles; ++g)
        for (int c = 0; c < S::halves; ++c)
          tma_load_3d(qbuf + g * S::tile + c * HALF, &tmQ, q_full, 64 * c, head0, from + g * a.qpt);
      uint32_t seq = 0;
      bool ok = true;
      for (int t = begin; t < end && ok; ++t)
        for (int kv = 0; kv < 2 && ok; ++kv, ++seq) {
          const uint32_t slot = seq % S::slots;
          ok = mbar_wait<true>(&empty[slot], ((seq / S::slots) & 1) ^ 1);
          if (!ok) break;
          uint64_t* const bar = cut && kv && t == end - 1 ? last_full : &full[slot];
          mbar_expect_tx(bar, S::tile);
          for (int c = 0; c < S::halves; ++c)
            tma_load_4d(ring + slot * S::tile + c * HALF, kv ? &tmV : &tmK, bar, 64 * c, kvh, t * KT, prefix);
        }
      if (!ok) record_status(a.status, ELASTO_ERR_TIMEOUT);
      // all copies have landed before the CTA exits
      for (uint32_t s = seq > S::slots ? seq - S::slots : 0; s < seq; ++s) {
        if (cut && s == 2u * (end - begin) - 1)
          mbar_wait<true>(last_full, 0);
        else
          mbar_wait<true>(&full[s % S::slots], (s / S::slots) & 1);
      }
      mbar_wait<true>(q_full, 0);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    const int ksteps = (a.head_dim + 15) / 16;  // channels that the products take
    const uint32_t idesc_s = idesc_16_f32(QT, KT, !BF), idesc_o = idesc_16_f32(QT, 16 * ksteps, !BF, false, true);
    constexpr uint32_t hi = sdesc_sw128_hi(1024);
    const uint32_t q_lo = sdesc_lo(smem_addr(qbuf), 16), kv_lo = sdesc_lo(smem_addr(ring), 0);
    constexpr uint32_t K_LBO = (16 >> 4) << 16, V_LBO = (HALF >> 4) << 16;  // leading byte offsets of K and V tiles
    uint32_t np[2] = {0, 0};  // P tiles of a group
    bool ok = mbar_wait_warp<true>(q_full, 0);
    tc_fence_after();
    auto scores = [&](auto group, int t, bool first, bool last) {  // first and last of the groups that take the tile
      constexpr int g = decltype(group)::value;
      if (t >= end || !ok) return;
      const uint32_t s = 2 * (t - begin), slot = s % S::slots;
      if (first) {
        ok = mbar_wait_warp<true>(&full[slot], (s / S::slots) & 1);
        tc_fence_after();
      }
      if (!ok) return;
      const uint32_t k_lo = kv_lo + K_LBO + slot * (S::tile >> 4), q = q_lo + (pair ? 0 : g) * (S::tile >> 4);
#pragma unroll
      for (int k = 0; k < DP / 16; ++k) {
        const uint32_t off = (k >> 2) * (HALF >> 4) + 2 * (k & 3);
        if (k < ksteps) tc_mma_warp_lo(tmem + g * KT, q + off, k_lo + off, hi, idesc_s, k != 0);
      }
      tc_commit_warp(&s_full[g]);
      if (last) tc_commit_warp(&empty[slot]);
    };
    auto product = [&](auto group, int t, bool first, bool last) {
      constexpr int g = decltype(group)::value;
      if (t >= end || !ok) return;
      const uint32_t s = 2 * (t - begin) + 1, slot = s % S::slots;
      if (first) ok = cut && t == end - 1 ? mbar_wait_warp<true>(v_ready, 0) : mbar_wait_warp<true>(&full[slot], (s / S::slots) & 1);
      ok = ok && mbar_wait_warp<true>(&p_full[g], np[g] & 1);
      if (!ok) return;
      tc_fence_after();
      const uint32_t v_lo = kv_lo + V_LBO + slot * (S::tile >> 4);
      const int steps = cut && t == end - 1 ? (left + 15) / 16 : KT / 16;
#pragma unroll
      for (int k = 0; k < KT / 16; ++k)
        if (k < steps) tc_mma_tmem_a_warp_lo(tmem + O_COL + g * DP, tmem + g * KT + 8 * k, v_lo + 128 * k, hi, idesc_o, np[g] > 0 || k != 0);
      ++np[g];
      if (t + (pair ? 2 : 1) >= end) tc_commit_warp(&o_full[g]);
      if (last) tc_commit_warp(&empty[slot]);
    };
    const std::integral_constant<int, 0> g0;
    const std::integral_constant<int, 1> g1;
    // S(t + 1) of a group is issued after its product with P(t): its arrival also says that O is at rest
    if (pair) {
      scores(g0, begin, true, true);
      scores(g1, begin + 1, true, true);
      for (int t = begin; t < end && ok; t += 2) {
        product(g0, t, true, true);
        scores(g0, t + 2, true, true);
        product(g1, t + 1, true, true);
        scores(g1, t + 3, true, true);
      }
    } else if (second) {
      scores(g0, begin, true, false);
      scores(g1, begin, false, true);
      for (int t = begin; t < end && ok; ++t) {
        product(g0, t, true, false);
        scores(g0, t + 1, true, false);
        product(g1, t, false, true);
        scores(g1, t + 1, false, true);
      }
    } else {
      scores(g0, begin, true, true);
      for (int t = begin; t < end && ok; ++t) {
        product(g0, t, true, true);
        scores(g0, t + 1, true, true);
      }
    }
    if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
    tc_commit_warp(drain);
    mbar_wait_warp<true>(drain, 0);
  } else if (warp == 2) {
    // ------------------------------------------------------------ values behind the prefix's end
    if (cut) {
      const uint32_t slot = (2 * (end - 1 - begin) + 1) % S::slots;
      if (mbar_wait_warp<true>(last_full, 0)) {
        uint8_t* const v = ring + slot * S::tile;
        const int rows = ((left + 15) & ~15) - left;
        for (int i = lane; i < rows * 8 * S::halves; i += 32) {
          const int c = i / (rows * 8), e = i - c * rows * 8;
          *reinterpret_cast<uint4*>(v + c * HALF + (left + (e >> 3)) * 128 + (e & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(v_ready);
      } else if (lane == 0) {
        record_status(a.status, ELASTO_ERR_TIMEOUT);
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------ softmax, a row a thread
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_MANY));
    const int g = (warp - 4) >> 2, r = (warp & 3) * 32 + lane;  // row of the tile = TMEM lane
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_tm = tmem + lanes + g * KT, o_tm = tmem + lanes + O_COL + g * DP;
    const float sc = a.scale_log2;
    auto place = [&](int& query, int& head) {  // of this row; false: it has none
      const int q = r * a.by_hg >> 16;
      head = r - q * a.hg, query = from + (pair ? 0 : g) * a.qpt + q;
      return q < a.qpt && query < to && head < nheads;
    };
    float lazy = kLazy;
    {
      int query, head;
      if (!place(query, head)) lazy = INFINITY;  // (rows without a query have no vote on rescaling)
    }
    const uint32_t count = pair ? (end - begin + 1 - g) / 2 : g == 0 || second ? end - begin : 0;  // of this group's key tiles
    const bool last_cut = cut && count > 0 && (!pair || ((end - 1 - begin) & 1) == g);
    float m = -INFINITY, sum = 0.0f;
    uint32_t ns = 0;
    bool ok = true;
    auto tile = [&](auto masked) -> bool {
      constexpr int NC = KT / 32;
      constexpr bool MASKED = decltype(masked)::value;
      if (!__all_sync(0xffffffffu, mbar_wait<true>(&s_full[g], ns & 1))) return false;
      tc_fence_after();
      uint32_t v[NC][32];
#pragma unroll
      for (int i = 0; i < NC; ++i) tmem_ld_32x32b_x32(s_tm + 32 * i, v[i]);
      tmem_ld_wait();
      if constexpr (MASKED) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (32 * i + j >= left) v[i][j] = 0xff800000u;
      }
      float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int j = 0; j < 32; j += 2)
          t4[(j >> 1) & 3] = max3(t4[(j >> 1) & 3], __uint_as_float(v[i][j]), __uint_as_float(v[i][j + 1]));
      const float top = fmaxf(m, fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])));
      // (top - m is NaN while both are -inf: nothing seen yet, nothing to rescale)
      if (__any_sync(0xffffffffu, (top - m) * sc > lazy)) {
        const float keep = m == -INFINITY ? 0.0f : ex2_approx((m - top) * sc);
        if (ns > 0) {
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
            uint32_t lo[16], up[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) lo[j] = o[j], up[j] = o[16 + j];
            tmem_st_16(o_tm + c, lo);
            tmem_st_16(o_tm + c + 16, up);
          }
          tmem_st_wait();
        }
        sum *= keep;
        m = top;
      }
      ++ns;
      const float neg = m == -INFINITY ? 0.0f : fmaf(-m, sc, -a.down);
      const float2 sc2 = make_float2(sc, sc), neg2 = make_float2(neg, neg);
      float2 add[2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        uint32_t pk[16];
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
    for (uint32_t n = last_cut ? 1 : 0; n < count && ok; ++n) ok = tile(std::false_type());
    if (last_cut && ok) ok = tile(std::true_type());
    // ------------------------------------------------------------ the part's results
    if (ok && ns > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait<true>(&o_full[g], 0));
      tc_fence_after();
    }
    if (ok && ns > 0) {
      int query, head;
      const bool mine = place(query, head);
      const int part = pair ? 2 * rank + g : rank;
      const long long rho = static_cast<long long>(query) * a.hg + head;
      // (-0 where all scores of the part are -infinity: an infinite value among its keys shows in no weighted sum then)
      if (mine) *reinterpret_cast<float2*>(a.parts.stat + a.parts.stat_at(part, h, rho)) = make_float2(m, m == -INFINITY ? -sum : sum);
      float* const sums = a.parts.sums + a.parts.sums_at(part, h, rho);
#pragma unroll 1
      for (int c = 0; c < DP; c += 32) {
        uint32_t o[32];
        tmem_ld_32x32b_x32(o_tm + c, o);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (mine && c + 4 * j < a.head_dim)
            *reinterpret_cast<uint4*>(sums + (c / 4 + j) * kQuadStep) = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
      }
      tc_fence_before();
    }
    if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
  }
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
  }
}

cudaError_t init_attributes() {
  cudaError_t e = cudaSuccess;
  // the register split adds up only if the kernels were built with the launch's count
  auto set = [&](auto* f, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    cudaFuncAttributes at{};
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, f);
    if (e == cudaSuccess && at.numRegs != REGS) e = cudaErrorInvalidConfiguration;
  };
  set(prefix_attention_kernel<true, 64>, Shape<64>::smem);
  set(prefix_attention_kernel<false, 64>, Shape<64>::smem);
  set(prefix_attention_kernel<true, 128>, Shape<128>::smem);
  set(prefix_attention_kernel<false, 128>, Shape<128>::smem);
  return e;
}

// Rows of q that may belong to sequences (with q_start anywhere in q), and those to be expected.
int64_t queries(const elasto_prefix_attention_args& u) {
  const int64_t most = static_cast<int64_t>(u.batch) * u.max_queries;
  return u.q_start ? u.q_rows : std::min<int64_t>(most, u.q_rows);
}
PrefixPlan plan_of(const elasto_prefix_attention_args& u) {
  PrefixSizes z;
  z.most = queries(u), z.rows = std::min<int64_t>(z.most, static_cast<int64_t>(u.batch) * u.max_queries);
  z.batch = u.batch, z.max_queries = static_cast<int>(std::min<int64_t>(u.max_queries, u.q_rows)), z.prefixes = u.prefixes;
  z.group = u.heads / u.heads_kv, z.heads_kv = u.heads_kv, z.head_dim = u.head_dim;
  z.max_prefix = u.max_prefix, z.max_keys = u.max_keys, z.sms = num_sms() > 0 ? num_sms() : 152;
  return prefix_plan(z);
}
int64_t part_rows(const elasto_prefix_attention_args& u, const PrefixPlan& p) { return (queries(u) * p.hg + 31) & ~int64_t(31); }
// Floats of the parts' statistics and sums.
int64_t stat_floats(const elasto_prefix_attention_args& u, const PrefixPlan& p) {
  return 2 * p.parts() * static_cast<int64_t>(u.heads_kv) * p.nsub * part_rows(u, p);
}
int64_t sums_floats(const elasto_prefix_attention_args& u, const PrefixPlan& p) {
  return p.parts() * static_cast<int64_t>(u.heads_kv) * p.nsub * part_rows(u, p) * u.head_dim;
}

}  // namespace

elasto_status prefix_attention_workspace(const elasto_prefix_attention_args& u, size_t* bytes) {
  const PrefixPlan p = plan_of(u);
  // (past any memory, and where the 64-bit sizes below could wrap)
  if (static_cast<double>(p.parts()) * u.heads_kv * p.nsub * p.hg * static_cast<double>(queries(u)) * u.head_dim > 1e15) {
    set_error("elasto_op_prefix_attention: too many queries and heads for a workspace");
    return ELASTO_ERR_UNSUPPORTED;
  }
  *bytes = static_cast<size_t>(4 * (stat_floats(u, p) + sums_floats(u, p)));
  return ELASTO_OK;
}

elasto_status prefix_attention_launch(const elasto_prefix_attention_args& u, int* status, cudaStream_t s) {
  static DeviceOnce once;
  if (static_cast<int64_t>(std::min<int64_t>(u.max_queries, u.q_rows)) * (u.heads / u.heads_kv) > 0x3fffffff) {
    set_error("elasto_op_prefix_attention: too many queries");
    return ELASTO_ERR_UNSUPPORTED;
  }
  const PrefixPlan p = plan_of(u);
  size_t bytes = 0;
  if (const elasto_status st = prefix_attention_workspace(u, &bytes); st != ELASTO_OK) return st;
  if (u.workspace_bytes < bytes) {
    set_error("elasto_op_prefix_attention: the workspace is smaller than elasto_op_prefix_attention_workspace says");
    return ELASTO_ERR_INVALID_ARG;
  }
  ELASTO_CUDA_TRY(once(init_attributes));
  Args a{};
  a.batch = u.batch, a.heads_kv = u.heads_kv, a.group = u.heads / u.heads_kv, a.head_dim = u.head_dim;
  a.scale_log2 = u.scale * 1.4426950408889634f;
  a.down = sum_headroom(u.dtype == ELASTO_BF16, static_cast<int>(std::min<int64_t>(static_cast<int64_t>(u.max_prefix) + u.max_keys, 0x7fffffff)));
  a.max_queries = static_cast<int>(std::min<int64_t>(u.max_queries, u.q_rows)), a.q_rows = static_cast<int>(u.q_rows), a.q_start = u.q_start;
  a.prefixes = u.prefixes, a.max_prefix = u.max_prefix, a.seq_start = u.seq_start, a.prefix_len = u.prefix_len;
  a.hg = p.hg, a.nsub = p.nsub, a.qpt = p.qpt, a.by_hg = (65536 + p.hg - 1) / p.hg;
  a.pair = p.pair, a.split = p.split;
  const int hs = u.heads_kv * p.nsub;
  const int64_t ctas = p.items * hs * p.split;
  if (ctas > 0x7fffffffLL) {
    set_error("elasto_op_prefix_attention: too many queries");
    return ELASTO_ERR_UNSUPPORTED;
  }
  a.by_items = Divisor(static_cast<unsigned>(p.items)), a.by_hs = Divisor(hs);
  a.parts = {static_cast<float*>(u.workspace) + stat_floats(u, p), static_cast<float*>(u.workspace), part_rows(u, p), hs, u.head_dim / 4};
  a.status = status;
  const bool bf = u.dtype == ELASTO_BF16;
  auto keys = [&](CUtensorMap* tm, const void* data, long long head_s, long long row_s, long long batch_s) {
    const uint64_t dims[4] = {static_cast<uint64_t>(u.head_dim), static_cast<uint64_t>(u.heads_kv), static_cast<uint64_t>(u.prefix_rows),
                              static_cast<uint64_t>(u.prefixes)};
    const uint64_t strides[3] = {static_cast<uint64_t>(head_s) * 2, static_cast<uint64_t>(row_s) * 2, static_cast<uint64_t>(batch_s) * 2};
    const uint32_t box[4] = {64, 1, KT, 1};
    return encode_tmap_16(tm, data, bf, 4, dims, strides, box);
  };
  const uint64_t q_dims[3] = {static_cast<uint64_t>(u.head_dim), static_cast<uint64_t>(u.heads), static_cast<uint64_t>(u.q_rows)};
  const uint64_t q_strides[2] = {static_cast<uint64_t>(u.q_head) * 2, static_cast<uint64_t>(u.q_row) * 2};
  const uint32_t q_box[3] = {64, static_cast<uint32_t>(p.hg), static_cast<uint32_t>(p.qpt)};
  CUtensorMap tq, tk, tv;
  if (!encode_tmap_16(&tq, u.q, bf, 3, q_dims, q_strides, q_box) || !keys(&tk, u.prefix_k, u.prefix_k_head, u.prefix_k_row, u.prefix_k_batch) ||
      !keys(&tv, u.prefix_v, u.prefix_v_head, u.prefix_v_row, u.prefix_v_batch)) {
    set_error("elasto_op_prefix_attention: cuTensorMapEncodeTiled failed (alignment, strides or size)");
    return ELASTO_ERR_UNSUPPORTED;
  }
  // (the other kernels' checks come before the first is launched)
  PrefixOwn own;
  elasto_status st = prefix_own_plan(u, p, a.parts, a.down, status, &own);
  if (st != ELASTO_OK) return st;
  const dim3 grid(static_cast<unsigned>(ctas)), block(THREADS);
  cudaError_t e;
  if (u.head_dim <= 64)
    e = bf ? launch_pdl(prefix_attention_kernel<true, 64>, grid, block, Shape<64>::smem, s, tq, tk, tv, a)
           : launch_pdl(prefix_attention_kernel<false, 64>, grid, block, Shape<64>::smem, s, tq, tk, tv, a);
  else
    e = bf ? launch_pdl(prefix_attention_kernel<true, 128>, grid, block, Shape<128>::smem, s, tq, tk, tv, a)
           : launch_pdl(prefix_attention_kernel<false, 128>, grid, block, Shape<128>::smem, s, tq, tk, tv, a);
  ELASTO_CUDA_TRY(e);
  return prefix_own_launch(own, s);
}

}  // namespace elasto
