// Attention behind shared prefixes: the sequences' own keys, and the join of all parts.
//
// A block is 16 or 64 rows (query, head) of one sequence and key head; S = Q K^T and O += P V by m16n8k16 products (tcgen05
// would need 128 rows of one sequence: the prefix, where most of the work lies, has them), running maximum and sum of the
// softmax in one pass, P rounded to the operand type as in prefix_attention.cu. The own keys of a block are shared out over own_split CTAs, each of which leaves a part as
// prefix_attention.cu's CTAs do.
//   prefix_few_kernel    16 rows, single tokens and few: a CTA is one warp, which streams 16 keys at a time by TMA through
//     a ring of its own. Nothing is shared between warps, and while one of an SM's twelve CTAs starts or ends the others load.
//   prefix_many_kernel   64 rows, longer runs of tokens: four warps with 16 rows each, a fifth loads tiles of 64 keys.
// Neither waits for the prefixes' kernel: that one is bound by its products, these by reading the keys and values
// once, and both run at the same time. Only the last CTA waits before it ends, so that what waits for this kernel waits
// for both. The inputs are there all the same: no CTA of these kernels starts before every CTA of the prefixes' has waited for
// the work before the call, whose results then are in the L2. What is read without a wait of the kernel's own is therefore read
// from there, by TMA and by loads that pass over the L1 (where lines of a call before might be left).
//
// prefix_join_few_kernel, prefix_join_many_kernel: out = sum over parts of o exp(m - top) / sum of l exp(m - top), four
// channels a thread, in a fixed order. Where the prefixes' CTAs fill the chip by themselves and leave one part, prefix_few_kernel waits for them and joins its
// rows itself.
//
// prefix_few_kernel is bound by memory: 64 sequences' own keys to 1024 (8 key heads of 128) 33 us by itself, 5.1 TB/s; 256
// sequences' to 512, 57 us, 5.3 TB/s. The joins behind them: 5 to 9 us, reading parts that lie in the L2.
#include <algorithm>
#include <type_traits>

#include "prefix_own.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr float kLazy = 8.0f;  // log2 of how far a maximum may grow before O is rescaled
constexpr int JOIN_THREADS = 256;

// A CTA of one warp and its ring: 16 KB, twelve CTAs an SM. With 24 KB (eight) 64 and 256 single tokens, drafts and images took 0.99,
// 1.02, 1.10 and 1.04 of the time, with 32 KB (six) 1.00, 1.08, 1.19 and 1.11.
template <int DP>
struct Few {
  static constexpr int halves = DP / 64, half = 16 * 128, tile = halves * half, stage = 2 * tile;  // 16 keys of 64 channels
  static constexpr int stages = 16 * 1024 / stage;  // twelve CTAs an SM (see below)
  static constexpr int smem = 1024 + stages * stage + 64;
};

constexpr int KT = 64, WARPS = 4, THREADS = 32 * (WARPS + 1), ROWS = 64;
constexpr int HALF = KT * 128;                 // bytes of 64 keys of 64 channels
constexpr int QUAD = 4 * ROWS + 8;             // floats from four channels of all rows to the next four (no bank conflicts)
template <int DP>
struct Many {
  static constexpr int halves = DP / 64, tile = halves * HALF, stage = 2 * tile;
  static constexpr int stages = DP == 128 ? 2 : 4;  // three CTAs an SM
  static constexpr int smem = 1024 + stages * stage + 256;
  static_assert(stages * stage >= (DP / 4 * QUAD + 2 * ROWS) * 4, "the results take the ring's place");
};

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
template <bool BF>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (BF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool BF>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  return BF ? pack_bf16x2(lo, hi) : pack_f16x2(lo, hi);
}
// Bits of the halves of w that are infinite or NaN.
template <bool BF>
__device__ __forceinline__ uint32_t bad16(uint32_t w) {
  constexpr uint32_t e = BF ? 0x7f807f80u : 0x7c007c00u;
  const uint32_t x = (w & e) ^ e;
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

// The sum of the infinite and NaN values among n keys of a channel (v: its first key).
template <bool BF>
__device__ __noinline__ float bad_values(const uint16_t* v, long long row, int n) {
  float sum = 0.0f;
#pragma unroll 8
  for (int j = 0; j < n; ++j) {
    const uint16_t w = __ldcg(v + j * row);
    const float x = BF ? __uint_as_float(static_cast<uint32_t>(w) << 16) : __half2float(__ushort_as_half(w));
    if (!(fabsf(x) < INFINITY)) sum += x;
  }
  return sum;
}

// Values that the weighted sums may not show: some own ones have been set to 0 because other rows do not see them, or all scores
// of a part (of the own keys, of the prefix) are -infinity, whose weighted sums the joins pass over.
enum { LOOK_OWN = 1, LOOK_PREFIX = 2 };

// The result y of channel ch of a row that sees `seen` own keys and `len` of its prefix: the sum of the values that are not
// finite, if it sees such. (An infinite value whose probability has rounded to 0 gave NaN.)
template <bool BF>
__device__ __noinline__ float put_bad_value(const PrefixOwnArgs& a, float y, int b, int kvh, int k0, int seen, int prefix, int len, int ch, int look) {
  float s = 0.0f;
  if (seen > 0) s += bad_values<BF>(a.v + (a.kv_start ? 0 : b * a.v_batch) + k0 * a.v_row + kvh * a.v_head + ch, a.v_row, seen);
  if ((!(fabsf(y) < INFINITY) || (look & LOOK_PREFIX)) && len > 0) s += bad_values<BF>(a.pv + prefix * a.pv_batch + kvh * a.pv_head + ch, a.pv_row, len);
  return s != 0.0f ? s : y;  // (NaN too)
}
// The same of four channels.
template <bool BF>
__device__ __forceinline__ float4 put_bad_values(const PrefixOwnArgs& a, float4 y, int b, int kvh, int k0, int seen, int prefix, int len, int quad,
                                                 int look) {
  const float odd = fmaf(y.x, 0.0f, fmaf(y.y, 0.0f, fmaf(y.z, 0.0f, y.w * 0.0f)));
  auto one = [&](float x, int c) { return put_bad_value<BF>(a, x, b, kvh, k0, seen, prefix, len, 4 * quad + c, look); };
  if (odd != 0.0f || look) y = make_float4(one(y.x, 0), one(y.y, 1), one(y.z, 2), one(y.w, 3));
  return y;
}

// The keys of prefix g, and whether sequence b is behind it.
__device__ __forceinline__ int prefix_keys(const PrefixOwnArgs& a, int g) {
  return a.prefix_len ? min(max(__ldcg(a.prefix_len + g), 0), a.max_prefix) : a.max_prefix;
}
__device__ __forceinline__ bool behind(const PrefixOwnArgs& a, int b, int g) {
  return !a.seq_start || (__ldcg(a.seq_start + g) <= b && b < __ldcg(a.seq_start + g + 1));
}
// Rows of q and own keys of sequence b, cut to what the host allows.
__device__ __forceinline__ void sequence(const PrefixOwnArgs& a, int b, int& q0, int& nq, int& k0, int& nk) {
  q0 = b * a.max_queries, nq = a.max_queries, k0 = 0, nk = a.max_keys;
  if (a.q_start) {
    q0 = min(max(__ldcg(a.q_start + b), 0), a.q_rows);
    nq = min(max(min(__ldcg(a.q_start + b + 1), a.q_rows) - q0, 0), a.max_queries);
  }
  if (a.kv_start) {
    k0 = min(max(__ldcg(a.kv_start + b), 0), a.kv_rows);
    nk = min(max(min(__ldcg(a.kv_start + b + 1), a.kv_rows) - k0, 0), a.max_keys);
  } else if (a.kv_len) {
    nk = min(max(__ldcg(a.kv_len + b), 0), a.max_keys);
  }
}

// Whether part p of a prefix has key tiles.
__device__ __forceinline__ bool has_keys(const PrefixOwnArgs& a, int p, int len) {
  const int r = a.pair ? p >> 1 : p, key_tiles = (len + kPrefixTile - 1) / kPrefixTile;
  return split_from(key_tiles, r + 1, a.split) - split_from(key_tiles, r, a.split) > (a.pair ? p & 1 : 0);
}

// The running softmax of a warp's 16 rows (this lane's: r and r + 8, r = lane / 4) over N blocks of 16 keys, and the
// products. q: the rows; ks, vs: this lane's rows of the K and V tiles for ldmatrix; half: bytes from 64 channels to
// the next; left: keys that some row sees; vis: keys that the two rows see (MASKED: not all of them all).
template <bool BF, int DP>
struct Softmax {
  float o[DP / 8][4], m[2], sum[2];
  __device__ __forceinline__ Softmax() {
    m[0] = m[1] = -INFINITY, sum[0] = sum[1] = 0.0f;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
  }
  template <int N>
  __device__ __forceinline__ void step(const uint32_t (&q)[DP / 16][4], uint32_t ks, uint32_t vs, int half, int left, bool masked, const int (&vis)[2],
                                       float sc, float down, int lane) {
    const int c2 = 2 * (lane & 3), kswap = lane & 7, kpiece = (lane >> 3) & 1, vpiece = lane >> 4;
    float x[2 * N][4];
#pragma unroll
    for (int n = 0; n < 2 * N; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.0f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (16 * n >= left) continue;
#pragma unroll
      for (int k = 0; k < DP / 16; ++k) {
        uint32_t bk[4];
        ldmatrix4(ks + n * 2048 + (k >> 2) * half + (((2 * (k & 3) + kpiece) ^ kswap) << 4), bk);
        mma16816<BF>(x[2 * n], q[k], bk[0], bk[1]);
        mma16816<BF>(x[2 * n + 1], q[k], bk[2], bk[3]);
      }
    }
    if (masked) {
#pragma unroll
      for (int n = 0; n < 2 * N; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (8 * n + c2 + (j & 1) >= vis[j >> 1]) x[n][j] = -INFINITY;
    }
    float top[2], keep[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v = -INFINITY;
#pragma unroll
      for (int n = 0; n < 2 * N; ++n) v = max3(v, x[n][2 * h], x[n][2 * h + 1]);
      v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
      v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
      top[h] = fmaxf(m[h], v);
    }
    if (__any_sync(0xffffffffu, (top[0] - m[0]) * sc > kLazy || (top[1] - m[1]) * sc > kLazy)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        keep[h] = m[h] == -INFINITY ? 0.0f : ex2_approx((m[h] - top[h]) * sc);
        sum[h] *= keep[h];
        m[h] = top[h];
      }
#pragma unroll
      for (int j = 0; j < DP / 8; ++j) o[j][0] *= keep[0], o[j][1] *= keep[0], o[j][2] *= keep[1], o[j][3] *= keep[1];
    }
    uint32_t p[N][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float neg = m[h] == -INFINITY ? 0.0f : fmaf(-m[h], sc, -down);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        float e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = ex2_approx(fmaf(x[2 * n + (j >> 1)][2 * h + (j & 1)], sc, neg));
        sum[h] += (e[0] + e[1]) + (e[2] + e[3]);
        p[n][h] = pack16<BF>(e[0], e[1]);
        p[n][2 + h] = pack16<BF>(e[2], e[3]);
      }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (16 * n >= left) continue;
#pragma unroll
      for (int k = 0; k < DP / 16; ++k) {
        uint32_t bv[4];
        ldmatrix4_trans(vs + n * 2048 + (k >> 2) * half + (((2 * (k & 3) + vpiece) ^ kswap) << 4), bv);
        mma16816<BF>(o[2 * k], p[n], bv[0], bv[1]);
        mma16816<BF>(o[2 * k + 1], p[n], bv[2], bv[3]);
      }
    }
  }
  // the four lanes of a row: its sum
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
      sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
    }
  }
};

// The words of a row at p (`channels` of it) that a lane of the row's four has of the products' A operand, into q[..][h] and
// q[..][h + 2]. A lane loads whole 16-byte pieces from the L2, every fourth of the row's, and the four exchange
// words. (With loads of the single words eight images took 206 us in place of 199.)
template <int DP>
__device__ __forceinline__ void load_query(const uint16_t* p, int channels, int lane, int h, uint32_t (&q)[DP / 16][4]) {
  const int c = lane & 3;
  const bool odd = c & 1, up = c & 2;
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) {
    const int ch = 32 * m + 8 * c;
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (ch < channels) w = __ldcg(reinterpret_cast<const uint4*>(p + ch));
    // (the transpose of 4 x 4 words: pairs of lanes, then pairs of pairs)
    auto swap = [&](uint32_t& lo, uint32_t& hi, bool second, int with) {
      const uint32_t other = __shfl_xor_sync(0xffffffffu, second ? lo : hi, with);
      (second ? lo : hi) = other;
    };
    swap(w.x, w.y, odd, 1), swap(w.z, w.w, odd, 1);
    swap(w.x, w.z, up, 2), swap(w.y, w.w, up, 2);
    q[2 * m][h] = w.x, q[2 * m][h + 2] = w.y, q[2 * m + 1][h] = w.z, q[2 * m + 1][h + 2] = w.w;
  }
}

// Values of the V tile at v (64 channels of `half` bytes, `keys` keys, 128 bytes each) that no row sees, from key `left` on,
// become 0, and from key `from` on, where some rows do not see them, those that are not finite: 0 * NaN
// would reach these rows. (The rows that see them get them at the end.) Whether there were any; thread `t` of `threads`.
template <bool BF, int DP>
__device__ __forceinline__ bool clear_values(uint8_t* v, int half, int keys, int from, int left, int t, int threads) {
  auto piece = [&](int e) {
    const int row = from + e / (DP / 8), at = e % (DP / 8);
    return reinterpret_cast<uint4*>(v + (at >> 3) * half + row * 128 + ((at & 7) << 4));  // (the swizzle stays within a row)
  };
  const int seen = (min(left, keys) - from) * (DP / 8), all = (keys - from) * (DP / 8);
  uint32_t acc = 0u;
  for (int e = t; e < all; e += threads) {
    uint4* const p = piece(e);
    if (e < seen)
      look16<BF>(p->x, acc), look16<BF>(p->y, acc), look16<BF>(p->z, acc), look16<BF>(p->w, acc);
    else
      *p = make_uint4(0u, 0u, 0u, 0u);
  }
  const bool bad = bad16<BF>(acc) != 0u;
  if (bad)
    for (int e = t; e < seen; e += threads) {
      uint4* const p = piece(e);
      const uint4 w = *p;
      *p = make_uint4(w.x & ~bad16<BF>(w.x), w.y & ~bad16<BF>(w.y), w.z & ~bad16<BF>(w.z), w.w & ~bad16<BF>(w.w));
    }
  fence_async_smem();  // (before the next tile is copied there)
  return bad;
}

template <bool BF, int DP>
__global__ void __launch_bounds__(32)
    prefix_few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PrefixOwnArgs a) {
  using T = Few<DP>;
  constexpr int S = T::stages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S * T::stage);
  const int lane = threadIdx.x;
  const int unit = static_cast<int>(a.by_split.quotient(blockIdx.x)), rank = static_cast<int>(blockIdx.x) - unit * a.own_split;
  const int u1 = static_cast<int>(a.by_blocks.quotient(unit)), blk = unit - u1 * a.blocks;
  const int b = static_cast<int>(a.by_heads_kv.quotient(u1)), kvh = u1 - b * a.heads_kv;
  if (lane == 0) {
    for (int i = 0; i < S; ++i) mbar_init(&full[i], 1);
    fence_barrier_init();
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  __syncwarp();
  pdl_trigger();
  // (the inputs may be read at once, from the L2)
  int q0, nq, k0, nk;
  sequence(a, b, q0, nq, k0, nk);
  const int row0 = blk * 16, nrows = min(nq * a.group - row0, 16);
  if (nrows > 0) {
    auto query = [&](int row) { return static_cast<int>(a.by_group.quotient(row0 + row)); };
    auto visible = [&](int row) { return row < nrows ? min(max(nk - nq + query(row) + 1, 0), nk) : 0; };
    const int most = visible(nrows - 1), least = visible(0), subs = (most + 15) / 16;
    const int t0 = split_from(subs, rank, a.own_split), n = split_from(subs, rank + 1, a.own_split) - t0;
    auto request = [&](int i) {  // (one lane)
      uint8_t* const dst = smem + i % S * T::stage;
      mbar_expect_tx(&full[i % S], T::stage);
      for (int h = 0; h < T::halves; ++h) {
        tma_load_4d(dst + h * T::half, &tmK, &full[i % S], 64 * h, kvh, k0 + (t0 + i) * 16, a.kv_start ? 0 : b);
        tma_load_4d(dst + T::tile + h * T::half, &tmV, &full[i % S], 64 * h, kvh, k0 + (t0 + i) * 16, a.kv_start ? 0 : b);
      }
    };
    int asked = min(n, S);
    if (elect_one())
      for (int i = 0; i < asked; ++i) request(i);
    __syncwarp();
    int prefix = -1, len = 0;
    if (a.fused)
      for (int g0 = 0; g0 < a.prefixes && prefix < 0; g0 += 32) {
        const int g = g0 + lane, keys = g < a.prefixes ? prefix_keys(a, g) : 0;
        const uint32_t mine = __ballot_sync(0xffffffffu, g < a.prefixes && behind(a, b, g));
        if (mine) prefix = g0 + __ffs(mine) - 1, len = __shfl_sync(0xffffffffu, keys, __ffs(mine) - 1);
      }
    const int r = lane >> 2, c2 = 2 * (lane & 3);
    uint32_t q[DP / 16][4];  // the rows r and r + 8
    int vis[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = r + 8 * h, qi = query(row), head = row0 + row - qi * a.group;
      vis[h] = visible(row);
      const uint16_t* const p = a.q + static_cast<long long>(q0 + qi) * a.q_row + static_cast<long long>(kvh * a.group + head) * a.q_head;
      load_query<DP>(p, row < nrows ? a.head_dim : 0, lane, h, q);
    }
    const float sc = a.scale_log2;
    const int krow = (lane & 7) + (lane >> 4) * 8, vrow = lane & 15;  // this lane's in the ldmatrix loads of K and of V
    Softmax<BF, DP> x;
    bool ok = true, left_out = false;
    for (int i = 0; i < n; ++i) {
      const int s = i % S, key0 = (t0 + i) * 16;
      ok = mbar_wait_warp(&full[s], (i / S) & 1);
      if (!ok) break;
      uint8_t* const kb = smem + s * T::stage;
      const int whole = least - key0, left = most - key0;  // of these keys: those that all rows see, and that some row sees
      if (whole < 16) {
        left_out |= clear_values<BF, DP>(kb + T::tile, T::half, 16, max(whole, 0), left, lane, 32);
        __syncwarp();
      }
      const int seen[2] = {vis[0] - key0, vis[1] - key0};
      x.template step<1>(q, smem_addr(kb) + krow * 128, smem_addr(kb + T::tile) + vrow * 128, T::half, left, whole < 16, seen, sc, a.down, lane);
      __syncwarp();
      if (i + S < n) {
        if (elect_one()) request(i + S);
        __syncwarp();
        ++asked;
      }
    }
    if (!ok) {  // (the copies in flight land before the CTA exits)
      if (lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
      for (int i = max(0, asked - S); i < asked; ++i) mbar_wait_warp(&full[i % S], (i / S) & 1);
    }
    x.finish();
    left_out = __any_sync(0xffffffffu, left_out);
    if (a.fused) pdl_wait();  // (the prefix's part)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = r + 8 * h;
      if (row >= nrows) continue;
      const int qi = query(row), head = row0 + row - qi * a.group, sub = head / a.hg, hs = kvh * a.nsub + sub;
      const long long rho = static_cast<long long>(q0 + qi) * a.hg + (head - sub * a.hg);
      if (!a.fused) {
        const bool look = left_out || (x.m[h] == -INFINITY && n > 0 && vis[h] > 16 * t0);  // (it sees keys of this part)
        if ((lane & 3) == 0)
          *reinterpret_cast<float2*>(a.parts.stat + a.parts.stat_at(a.prefix_parts + rank, hs, rho)) = make_float2(x.m[h], look ? -x.sum[h] : x.sum[h]);
        if (x.m[h] == -INFINITY) continue;
        float* const sums = a.parts.sums + a.parts.sums_at(a.prefix_parts + rank, hs, rho) + (c2 & 3) + (c2 >> 2) * kQuadStep;
#pragma unroll
        for (int j = 0; j < DP / 8; ++j)
          if (8 * j < a.head_dim) *reinterpret_cast<float2*>(sums + 2 * j * kQuadStep) = make_float2(x.o[j][2 * h], x.o[j][2 * h + 1]);
        continue;
      }
      // the row's result: the lane's channels of the prefix's one part and of the own keys
      const float* const sums = a.parts.sums + a.parts.sums_at(0, hs, rho) + (c2 & 3) + (c2 >> 2) * kQuadStep;
      float2 st = make_float2(-INFINITY, 0.0f), p[DP / 8];
      if (len > 0) st = *reinterpret_cast<const float2*>(a.parts.stat + a.parts.stat_at(0, hs, rho));
#pragma unroll
      for (int j = 0; j < DP / 8; ++j) p[j] = len > 0 && 8 * j < a.head_dim ? *reinterpret_cast<const float2*>(sums + 2 * j * kQuadStep) : make_float2(0.0f, 0.0f);
      const float top = fmaxf(x.m[h], st.x);
      // (a part without a finite score has sums of zeros, or NaN that must stay)
      const float wo = x.m[h] == -INFINITY ? 1.0f : ex2_approx((x.m[h] - top) * sc), wp = st.x == -INFINITY ? 1.0f : ex2_approx((st.x - top) * sc);
      const float total = x.sum[h] * wo + fabsf(st.y) * wp;
      const int seen_own = visible(row);
      const float inv = len > 0 || seen_own > 0 ? 1.0f / total : 0.0f;
      uint16_t* const out = a.out + static_cast<long long>(q0 + qi) * a.out_row + static_cast<long long>(kvh * a.group + head) * a.out_head + c2;
#pragma unroll
      for (int j = 0; j < DP / 8; ++j) {
        if (8 * j >= a.head_dim) continue;
        float2 y = make_float2((x.o[j][2 * h] * wo + p[j].x * wp) * inv, (x.o[j][2 * h + 1] * wo + p[j].y * wp) * inv);
        if (total > 0.0f) {
          if (fmaf(y.x, 0.0f, y.y * 0.0f) != 0.0f || left_out)
            y = make_float2(put_bad_value<BF>(a, y.x, b, kvh, k0, seen_own, prefix, len, 8 * j + c2, 0),
                            put_bad_value<BF>(a, y.y, b, kvh, k0, seen_own, prefix, len, 8 * j + c2 + 1, 0));
        } else if (inv != 0.0f) {  // (a sum of 0 or NaN over visible keys)
          y.x = y.y = __int_as_float(0x7fc00000);
        }
        *reinterpret_cast<uint32_t*>(out + 8 * j) = pack16<BF>(y.x, y.y);
      }
    }
  }
  if (blockIdx.x == gridDim.x - 1) pdl_wait();
}

template <bool BF, int DP>
__global__ void __launch_bounds__(THREADS, 3)
    prefix_many_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PrefixOwnArgs a) {
  using T = Many<DP>;
  constexpr int S = T::stages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S * T::stage);
  uint64_t* empty = full + S;
  int* bad = reinterpret_cast<int*>(empty + S);  // values that some row sees have been left out
  const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int unit = static_cast<int>(a.by_split.quotient(blockIdx.x)), rank = static_cast<int>(blockIdx.x) - unit * a.own_split;
  const int u1 = static_cast<int>(a.by_blocks.quotient(unit)), blk = unit - u1 * a.blocks;
  const int b = static_cast<int>(a.by_heads_kv.quotient(u1)), kvh = u1 - b * a.heads_kv;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], WARPS);
    }
    *bad = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  __syncthreads();
  pdl_trigger();
  // (the inputs may be read at once, from the L2)
  int q0, nq, k0, nk;
  sequence(a, b, q0, nq, k0, nk);
  const int row0 = blk * ROWS, nrows = min(nq * a.group - row0, ROWS);
  if (nrows <= 0) {
    if (blockIdx.x == gridDim.x - 1) pdl_wait();
    return;
  }
  auto query = [&](int row) { return static_cast<int>(a.by_group.quotient(row0 + row)); };
  auto visible = [&](int row) { return row < nrows ? min(max(nk - nq + query(row) + 1, 0), nk) : 0; };
  const int most = visible(nrows - 1), least = visible(0);
  const int tiles = (most + KT - 1) / KT;
  const int t0 = split_from(tiles, rank, a.own_split), t1 = split_from(tiles, rank + 1, a.own_split);

  Softmax<BF, DP> x;
  const int r = lane >> 2, c2 = 2 * (lane & 3), base = 16 * warp;  // (of the warp's rows)
  if (warp == WARPS) {
    if (elect_one()) {
      bool ok = true;
      int i = 0;
      for (int t = t0; t < t1; ++t, ++i) {
        const int s = i % S;
        ok = mbar_wait(&empty[s], ((i / S) & 1) ^ 1);
        if (!ok) break;
        uint8_t* dst = smem + s * T::stage;
        mbar_expect_tx(&full[s], T::stage);
        for (int h = 0; h < T::halves; ++h) {
          tma_load_4d(dst + h * HALF, &tmK, &full[s], 64 * h, kvh, k0 + t * KT, a.kv_start ? 0 : b);
          tma_load_4d(dst + T::tile + h * HALF, &tmV, &full[s], 64 * h, kvh, k0 + t * KT, a.kv_start ? 0 : b);
        }
      }
      if (!ok) record_status(a.status, ELASTO_ERR_TIMEOUT);
      for (int k = max(0, i - S); k < i; ++k) mbar_wait(&full[k % S], (k / S) & 1);
    }
    __syncwarp();
  } else if (t0 < t1) {
    uint32_t q[DP / 16][4];  // the rows base + r and base + r + 8
    int vis[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = base + r + 8 * h, qi = query(row), head = row0 + row - qi * a.group;
      vis[h] = visible(row);
      const uint16_t* const p = a.q + static_cast<long long>(q0 + qi) * a.q_row + static_cast<long long>(kvh * a.group + head) * a.q_head;
      load_query<DP>(p, row < nrows ? a.head_dim : 0, lane, h, q);
    }
    const float sc = a.scale_log2;
    const int krow = (lane & 7) + (lane >> 4) * 8, vrow = lane & 15;
    const bool ok = walk_tiles(
        t0, t1, KT, least, [&](int i) { return mbar_wait_warp(&full[i % S], (i / S) & 1); },
        [&](int i, int t, bool come) {
          uint8_t* const v = smem + i % S * T::stage + T::tile;
          const int key0 = t * KT;
          if (come && clear_values<BF, DP>(v, HALF, KT, max(least - key0, 0), most - key0, threadIdx.x, 32 * WARPS)) *bad = 1;
          named_bar_sync(1, 32 * WARPS);
        },
        [&](int i, int t) {
          const int s = i % S, key0 = t * KT, whole = least - key0, left = most - key0;
          uint8_t* const kb = smem + s * T::stage;
#pragma unroll 1
          for (int n = 0; n < KT && n < left; n += 32) {  // (32 keys at a time: with 64 the registers do for two CTAs an SM)
            const int seen[2] = {vis[0] - key0 - n, vis[1] - key0 - n};
            x.template step<2>(q, smem_addr(kb) + (n + krow) * 128, smem_addr(kb + T::tile) + (n + vrow) * 128, HALF, left - n, whole < n + 32, seen, sc,
                               a.down, lane);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&empty[s]);
        });
    if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
  }
  __syncthreads();  // all tiles are consumed: the ring's memory takes the results, [channels / 4][row] of four channels
  float* const sums = reinterpret_cast<float*>(smem);
  float* const stat = sums + DP / 4 * QUAD;  // [row][maximum, sum]
  if (warp < WARPS) {
    x.finish();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = base + r + 8 * h;
      if ((lane & 3) == 0) *reinterpret_cast<float2*>(stat + 2 * row) = make_float2(x.m[h], x.sum[h]);
#pragma unroll
      for (int j = 0; j < DP / 8; ++j)
        *reinterpret_cast<float2*>(sums + (2 * j + (c2 >> 2)) * QUAD + 4 * row + (c2 & 3)) = make_float2(x.o[j][2 * h], x.o[j][2 * h + 1]);
    }
  }
  __syncthreads();
  const int quads = a.head_dim / 4;
  const bool left_out = *bad != 0;
  // a row a thread: what the addresses of a row take is reckoned once
  const int row = threadIdx.x & (ROWS - 1);
  if (row < nrows && threadIdx.x < 2 * ROWS) {
    const int qi = query(row), head = row0 + row - qi * a.group, sub = head / a.hg, hs = kvh * a.nsub + sub;
    const long long rho = static_cast<long long>(q0 + qi) * a.hg + (head - sub * a.hg);
    const float2 st = *reinterpret_cast<const float2*>(stat + 2 * row);
    float* const to = a.parts.sums + a.parts.sums_at(a.prefix_parts + rank, hs, rho);
    const bool look = left_out || (st.x == -INFINITY && t0 < t1 && visible(row) > KT * t0);  // (it sees keys of this part)
    if (threadIdx.x < ROWS) *reinterpret_cast<float2*>(a.parts.stat + a.parts.stat_at(a.prefix_parts + rank, hs, rho)) = make_float2(st.x, look ? -st.y : st.y);
    if (st.x != -INFINITY)
      for (int quad = threadIdx.x / ROWS; quad < quads; quad += 2)
        *reinterpret_cast<float4*>(to + quad * kQuadStep) = *reinterpret_cast<const float4*>(sums + quad * QUAD + 4 * row);
  }
  if (blockIdx.x == gridDim.x - 1) pdl_wait();
}

// Where a row (query, head) of a sequence is: its rows over all heads, those of a key head together as in the parts.
struct JoinRow {
  int query, head, kvh, h;
  long long rho;
};
__device__ __forceinline__ JoinRow join_row(const PrefixOwnArgs& a, int q0, int nq, int row) {
  JoinRow r;
  const int each = nq * a.group;
  r.kvh = row / each;
  const int own = row - r.kvh * each;
  r.query = static_cast<int>(a.by_group.quotient(own));
  const int in = own - r.query * a.group, sub = in / a.hg;
  r.head = r.kvh * a.group + in, r.h = r.kvh * a.nsub + sub;
  r.rho = static_cast<long long>(q0 + r.query) * a.hg + (in - sub * a.hg);
  return r;
}
// The prefix of sequence b (-1: none) and the number of its keys, by a CTA, a prefix a thread, so that all loads are on the
// way at once; and which parts have results, as bits.
struct Found {
  int prefix, len;
  uint32_t written[(kMaxParts + 31) / 32];
};
__device__ __forceinline__ void find_prefix(const PrefixOwnArgs& a, int b, int parts, Found& found) {
  if (threadIdx.x == 0) found.prefix = a.seq_start ? -1 : 0, found.len = a.seq_start ? 0 : a.max_prefix;
  __syncthreads();
  for (int g = threadIdx.x; g < a.prefixes; g += JOIN_THREADS) {
    const int n = prefix_keys(a, g);
    if (behind(a, b, g)) found.prefix = g, found.len = n;
  }
  __syncthreads();
  if (threadIdx.x < (parts + 31) / 32 * 32) {
    const int p = threadIdx.x;
    const uint32_t bits = __ballot_sync(0xffffffffu, p < a.prefix_parts ? has_keys(a, p, found.len) : p < parts);
    if ((p & 31) == 0) found.written[p >> 5] = bits;
  }
  __syncthreads();
}

// The join of few rows: 32 rows of a sequence and 32 channels a CTA, four channels of a row a thread, which asks for all
// its parts' statistics and sums (N at a time) at once.
template <bool BF, int N>
__global__ void __launch_bounds__(JOIN_THREADS)
    prefix_join_few_kernel(const __grid_constant__ PrefixOwnArgs a) {
  __shared__ Found found;
  const int b = static_cast<int>(a.by_join.quotient(blockIdx.x)), blk = static_cast<int>(blockIdx.x) - b * a.join_blocks;
  pdl_trigger();
  // (the inputs may be read before the wait, from the L2)
  int q0, nq, k0, nk;
  sequence(a, b, q0, nq, k0, nk);
  const int parts = a.prefix_parts + a.own_parts;
  find_prefix(a, b, parts, found);
  const int prefix = found.prefix, len = found.len;
  const int row = 32 * blk + (threadIdx.x >> 3), quads = a.head_dim / 4;
  if (blockIdx.x == gridDim.x - 1 && blockIdx.y == gridDim.y - 1) pdl_wait();  // (where all sequences are empty nothing else does)
  if (row >= nq * a.heads_kv * a.group) return;
  const JoinRow r = join_row(a, q0, nq, row);
  const float* const st0 = a.parts.stat + a.parts.stat_at(0, r.h, r.rho);
  const float* const y0 = a.parts.sums + a.parts.sums_at(0, r.h, r.rho);
  const long long st_step = a.parts.stat_at(1, 0, 0), y_step = a.parts.sums_at(1, 0, 0);
  const float sc = a.scale_log2;
  const int seen = min(max(nk - nq + r.query + 1, 0), nk);  // of the own keys
  uint16_t* const out = a.out + static_cast<long long>(q0 + r.query) * a.out_row + static_cast<long long>(r.head) * a.out_head;
  const int quad = 8 * blockIdx.y + (threadIdx.x & 7);
  if (quad >= quads) return;
  float top = -INFINITY, total = 0.0f;
  float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  int look = 0;
  pdl_wait();
  for (int p0 = 0; p0 < parts; p0 += N) {
    const uint32_t bits = found.written[p0 >> 5] >> (p0 & 31);
    float2 st[N];
    float4 o[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      st[k] = make_float2(-INFINITY, 0.0f), o[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (bits >> k & 1) {
        st[k] = *reinterpret_cast<const float2*>(st0 + (p0 + k) * st_step);
        o[k] = *reinterpret_cast<const float4*>(y0 + (p0 + k) * y_step + quad * kQuadStep);
      }
    }
    float up = top;
#pragma unroll
    for (int k = 0; k < N; ++k) up = fmaxf(up, st[k].x);
    const float f = top == -INFINITY ? 1.0f : ex2_approx((top - up) * sc);
    total *= f, y.x *= f, y.y *= f, y.z *= f, y.w *= f;
    top = up;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (__float_as_int(st[k].y) < 0) look |= p0 + k < a.prefix_parts ? LOOK_PREFIX : LOOK_OWN;
      // (a part without a finite score has a sum of 0, or NaN that must stay, and no weighted sums)
      const bool none = st[k].x == -INFINITY;
      const float w = none ? 1.0f : ex2_approx((st[k].x - top) * sc);
      total = fmaf(fabsf(st[k].y), w, total);
      y.x = none ? y.x : fmaf(o[k].x, w, y.x), y.y = none ? y.y : fmaf(o[k].y, w, y.y);
      y.z = none ? y.z : fmaf(o[k].z, w, y.z), y.w = none ? y.w : fmaf(o[k].w, w, y.w);
    }
  }
  const float inv = len > 0 || seen > 0 ? 1.0f / total : 0.0f;
  y = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
  if (total > 0.0f)
    y = put_bad_values<BF>(a, y, b, r.kvh, k0, seen, prefix, len, quad, look);
  else if (inv != 0.0f)  // (a sum of 0 or NaN over visible keys)
    y.x = y.y = y.z = y.w = __int_as_float(0x7fc00000);
  *reinterpret_cast<uint2*>(out + 4 * quad) = make_uint2(pack16<BF>(y.x, y.y), pack16<BF>(y.z, y.w));
}

// The join of many rows: a CTA has 64 of one sequence. First the weight of each part in each row, then
// the weighted sums, four channels of a row a thread: four neighbouring threads have a row, so that whole sectors of the
// parts and of out move.
template <bool BF>
__global__ void __launch_bounds__(JOIN_THREADS, 4)
    prefix_join_many_kernel(const __grid_constant__ PrefixOwnArgs a) {
  constexpr int GROUPS = JOIN_THREADS / ROWS;  // threads that share a row's parts
  extern __shared__ float weight[];            // [part][ROWS]: times 1 / the joint sum; -1: not to be read
  __shared__ float2 partial[GROUPS][ROWS];     // maximum and sum of a thread's parts
  __shared__ uint8_t looks[GROUPS][ROWS];      // and what they do not show
  __shared__ float base[ROWS];                 // 0, or NaN in rows without a sum above 0
  __shared__ int look[ROWS];                   // LOOK_OWN, LOOK_PREFIX
  __shared__ Found found;
  const int b = static_cast<int>(a.by_join.quotient(blockIdx.x)), blk = static_cast<int>(blockIdx.x) - b * a.join_blocks;
  pdl_trigger();
  int q0, nq, k0, nk;
  sequence(a, b, q0, nq, k0, nk);
  const int parts = a.prefix_parts + a.own_parts;
  find_prefix(a, b, parts, found);
  const int prefix = found.prefix, len = found.len;
  const int row0 = blk * ROWS, nrows = min(nq * a.heads_kv * a.group - row0, ROWS);
  if (nrows <= 0) {
    if (blockIdx.x == gridDim.x - 1) pdl_wait();
    return;
  }
  const float sc = a.scale_log2;
  auto factor = [&](float m, float top) { return m == -INFINITY ? 1.0f : ex2_approx((m - top) * sc); };
  {
    // (a part without a finite score has a sum of 0, or NaN that must stay)
    const int row = threadIdx.x & (ROWS - 1), g = threadIdx.x / ROWS;
    const JoinRow r = join_row(a, q0, nq, row0 + min(row, nrows - 1));
    const float* const st = a.parts.stat + a.parts.stat_at(0, r.h, r.rho);
    const long long step = a.parts.stat_at(1, 0, 0);
    float top = -INFINITY, total = 0.0f;
    int bits = 0;
    pdl_wait();
#pragma unroll 4
    for (int p = g; p < parts; p += GROUPS) {
      const float2 v = found.written[p >> 5] >> (p & 31) & 1 ? *reinterpret_cast<const float2*>(st + p * step) : make_float2(-INFINITY, 0.0f);
      if (__float_as_int(v.y) < 0) bits |= p < a.prefix_parts ? LOOK_PREFIX : LOOK_OWN;
      const float up = fmaxf(top, v.x);
      total = total * factor(top, up) + fabsf(v.y) * factor(v.x, up);
      top = up;
      weight[p * ROWS + row] = v.x;
    }
    partial[g][row] = make_float2(top, total), looks[g][row] = static_cast<uint8_t>(bits);
    __syncthreads();
    top = -INFINITY, total = 0.0f, bits = 0;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) top = fmaxf(top, partial[k][row].x);
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const float2 v = partial[k][row];
      bits |= looks[k][row];
      total += v.y * factor(v.x, top);
    }
    const float inv = 1.0f / total;
    for (int p = g; p < parts; p += GROUPS) {
      const float m = weight[p * ROWS + row];
      weight[p * ROWS + row] = m == -INFINITY ? -1.0f : ex2_approx((m - top) * sc) * inv;
    }
    if (g == 0) {
      const bool sees = len > 0 || min(nk - nq + r.query + 1, nk) > 0;
      base[row] = sees && !(total > 0.0f) ? __int_as_float(0x7fc00000) : 0.0f;
      look[row] = bits;
    }
    __syncthreads();
  }
  const int row = (threadIdx.x >> 2) & (ROWS - 1);
  if (row >= nrows) return;
  const JoinRow r = join_row(a, q0, nq, row0 + row);
  const int quads = a.head_dim / 4;
  const float* const sums = a.parts.sums + a.parts.sums_at(0, r.h, r.rho);
  const long long y_step = a.parts.sums_at(1, 0, 0);
  const float none = base[row];
  uint16_t* const out = a.out + static_cast<long long>(q0 + r.query) * a.out_row + static_cast<long long>(r.head) * a.out_head;
  // U times four channels at once, N parts on the way
  auto run = [&](auto un, auto pn) {
    constexpr int U = un.value, N = pn.value, STEP = JOIN_THREADS / ROWS;
    for (int quad0 = 4 * (threadIdx.x / (4 * ROWS)) + (threadIdx.x & 3); quad0 < quads; quad0 += U * STEP) {
      float4 y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) y[u] = make_float4(none, none, none, none);
      for (int p0 = 0; p0 < parts; p0 += N) {
        float w[N];
        float4 o[N][U];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          w[k] = p0 + k < parts ? weight[(p0 + k) * ROWS + row] : -1.0f;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            o[k][u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (w[k] != -1.0f && quad0 + u * STEP < quads)
              o[k][u] = *reinterpret_cast<const float4*>(sums + (p0 + k) * y_step + (quad0 + u * STEP) * kQuadStep);
          }
        }
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
          for (int u = 0; u < U; ++u)
            y[u].x = fmaf(o[k][u].x, w[k], y[u].x), y[u].y = fmaf(o[k][u].y, w[k], y[u].y), y[u].z = fmaf(o[k][u].z, w[k], y[u].z),
            y[u].w = fmaf(o[k][u].w, w[k], y[u].w);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int quad = quad0 + u * STEP;
        if (quad >= quads) continue;
        float4 z = y[u];
        if (none == 0.0f) z = put_bad_values<BF>(a, z, b, r.kvh, k0, min(max(nk - nq + r.query + 1, 0), nk), prefix, len, quad, look[row]);
        *reinterpret_cast<uint2*>(out + 4 * quad) = make_uint2(pack16<BF>(z.x, z.y), pack16<BF>(z.z, z.w));
      }
    }
  };
  if (parts <= 2)
    run(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
  else
    run(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
}

template <bool BF, int DP>
cudaError_t launch(const PrefixOwn& own, cudaStream_t s) {
  const PrefixOwnArgs& a = own.a;
  cudaError_t e = cudaSuccess;
  const dim3 grid(static_cast<unsigned>(own.units * a.own_split));
  if (own.many)
    e = launch_pdl(prefix_many_kernel<BF, DP>, grid, dim3(THREADS), Many<DP>::smem, s, own.k, own.v, a);
  else if (a.max_keys > 0)
    e = launch_pdl(prefix_few_kernel<BF, DP>, grid, dim3(32), Few<DP>::smem, s, own.k, own.v, a);
  if (e != cudaSuccess || a.fused) return e;
  const int parts = a.prefix_parts + a.own_parts;
  const unsigned blocks = static_cast<unsigned>(a.batch) * a.join_blocks;
  if (own.join_many) return launch_pdl(prefix_join_many_kernel<BF>, dim3(blocks), dim3(JOIN_THREADS), 4 * parts * ROWS, s, a);
  const dim3 grid2(blocks, (a.head_dim + 31) / 32);
  return launch_pdl(parts <= 4 ? prefix_join_few_kernel<BF, 4> : parts <= 8 ? prefix_join_few_kernel<BF, 8> : prefix_join_few_kernel<BF, 16>, grid2,
                    dim3(JOIN_THREADS), 0, s, a);
}

cudaError_t init_attributes() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  auto all = [&](auto bf) {
    constexpr bool B = bf.value;
    set(prefix_few_kernel<B, 64>, Few<64>::smem);
    set(prefix_few_kernel<B, 128>, Few<128>::smem);
    set(prefix_many_kernel<B, 64>, Many<64>::smem);
    set(prefix_many_kernel<B, 128>, Many<128>::smem);
    set(prefix_join_many_kernel<B>, 4 * ROWS * kMaxParts);
  };
  all(std::false_type());
  all(std::true_type());
  return e;
}

}  // namespace

elasto_status prefix_own_plan(const elasto_prefix_attention_args& u, const PrefixPlan& p, const PrefixParts& parts, float down, int* status,
                              PrefixOwn* own) {
  static DeviceOnce once;
  ELASTO_CUDA_TRY(once(init_attributes));
  PrefixOwnArgs a{};
  a.batch = u.batch, a.heads_kv = u.heads_kv, a.group = u.heads / u.heads_kv, a.head_dim = u.head_dim;
  a.scale_log2 = u.scale * 1.4426950408889634f, a.down = down;
  a.max_queries = static_cast<int>(std::min<int64_t>(u.max_queries, u.q_rows)), a.q_rows = static_cast<int>(u.q_rows);
  a.max_keys = u.max_keys, a.kv_rows = static_cast<int>(u.kv_rows);
  a.q_start = u.q_start, a.kv_start = u.max_keys > 0 ? u.kv_start : nullptr, a.kv_len = u.max_keys > 0 ? u.kv_len : nullptr;
  a.q = static_cast<const uint16_t*>(u.q), a.q_row = u.q_row, a.q_head = u.q_head;
  a.v = static_cast<const uint16_t*>(u.v), a.v_batch = u.v_batch, a.v_row = u.v_row, a.v_head = u.v_head;
  a.out = static_cast<uint16_t*>(u.out), a.out_row = u.out_row, a.out_head = u.out_head;
  a.prefixes = u.prefixes, a.max_prefix = u.max_prefix, a.seq_start = u.seq_start, a.prefix_len = u.prefix_len;
  a.pv = static_cast<const uint16_t*>(u.prefix_v), a.pv_batch = u.prefix_v_batch, a.pv_row = u.prefix_v_row, a.pv_head = u.prefix_v_head;
  a.hg = p.hg, a.nsub = p.nsub, a.pair = p.pair, a.split = p.split, a.parts = parts;
  a.prefix_parts = p.prefix_parts(), a.own_split = p.own_split, a.own_parts = p.own_parts;
  a.status = status;
  own->many = p.many != 0 && u.max_keys > 0;
  a.fused = p.fused;
  own->units = static_cast<int64_t>(p.blocks) * a.batch * a.heads_kv;
  if (own->units * a.own_split > 0x7fffffffLL) {
    set_error("elasto_op_prefix_attention: too many sequences or queries");
    return ELASTO_ERR_UNSUPPORTED;
  }
  a.blocks = p.blocks;
  // The join: 32 rows and channels a CTA, 64 rows and all channels from 40000 rows on (a small CTA's start then costs
  // more than its loads). The call with the first and with the second, in us (32 / 8 heads of 128): 131072 rows, 8 prompts of 512
  // behind 8192 keys, 520 and 466; 65536, one of 2048, 359 and 331; 81920, 64 of 40 behind 4096, 206 and 178; 32768, 64 drafts of 16
  // with 1024 own keys, 130 and 114; 16384, 512 single tokens, 179 and 175; 35840 rows of 4 key heads with 7 each 129 and 118 (so
  // the second gains from about 16000 rows on; how it does with fewer has not been measured).
  const int64_t all = static_cast<int64_t>(a.max_queries) * u.heads;
  own->join_many = all * a.batch > 40000;
  const int64_t join_rows = own->join_many ? ROWS : 32, join_blocks = (all + join_rows - 1) / join_rows;
  if (join_blocks * a.batch > 0x7fffffffLL || all > 0x3fffffff) {
    set_error("elasto_op_prefix_attention: too many sequences or queries");
    return ELASTO_ERR_UNSUPPORTED;
  }
  a.join_blocks = static_cast<int>(join_blocks);
  a.by_join = Divisor(a.join_blocks);
  a.by_split = Divisor(a.own_split), a.by_blocks = Divisor(a.blocks), a.by_heads_kv = Divisor(a.heads_kv), a.by_group = Divisor(a.group);
  own->a = a, own->bf = u.dtype == ELASTO_BF16;
  auto map_of = [&](CUtensorMap* tm, const void* data, long long head_s, long long row_s, long long batch_s) {
    const uint64_t dims[4] = {static_cast<uint64_t>(u.head_dim), static_cast<uint64_t>(u.heads_kv), static_cast<uint64_t>(u.kv_rows),
                              static_cast<uint64_t>(u.kv_start ? 1 : u.batch)};
    const uint64_t strides[3] = {static_cast<uint64_t>(head_s) * 2, static_cast<uint64_t>(row_s) * 2, u.kv_start ? 0 : static_cast<uint64_t>(batch_s) * 2};
    const uint32_t box[4] = {64, 1, own->many ? KT : 16u, 1};
    return encode_tmap_16(tm, data, own->bf, 4, dims, strides, box);
  };
  own->k = CUtensorMap{}, own->v = CUtensorMap{};
  if (u.max_keys > 0 && (!map_of(&own->k, u.k, u.k_head, u.k_row, u.k_batch) || !map_of(&own->v, u.v, u.v_head, u.v_row, u.v_batch))) {
    set_error("elasto_op_prefix_attention: cuTensorMapEncodeTiled failed (alignment, strides or size)");
    return ELASTO_ERR_UNSUPPORTED;
  }
  return ELASTO_OK;
}

elasto_status prefix_own_launch(const PrefixOwn& own, cudaStream_t s) {
  auto run = [&](auto bf) { return own.a.head_dim <= 64 ? launch<bf.value, 64>(own, s) : launch<bf.value, 128>(own, s); };
  ELASTO_CUDA_TRY(own.bf ? run(std::true_type()) : run(std::false_type()));
  return ELASTO_OK;
}

}  // namespace elasto
