// Attention behind shared prefixes: the sequences' own keys, and the join of all parts.
//
// prefix_own_kernel: a block is 16 or 64 rows (query, head) of one sequence and key head; its own keys, in tiles of 64, are
// shared out over own_split CTAs, each of which leaves a part as prefix_attention.cu's CTAs do. Warp 4 streams K and V
// tiles by TMA through a ring, and warps 0-3 form S = Q K^T and O += P V by m16n8k16 products, running maximum and sum
// of the softmax for themselves:
//   16 rows (single tokens and few): a warp takes 16 keys of each tile, all rows;
//   64 rows (longer runs of tokens): a warp takes 16 rows, all keys.
// (tcgen05 would need 128 rows of one sequence: the prefix, where most of the work lies, has them.) It does not wait for
// the prefixes' kernel: both run at the same time, that one bound by its products, this one by reading the keys and values
// once. Only its last CTA waits before it ends, so that what waits for this kernel waits for both.
//
// prefix_join_kernel: out = sum over parts of o exp(m - top) / sum of l exp(m - top), four channels a thread, in a fixed order.
#include <algorithm>
#include <type_traits>

#include "prefix_own.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int KT = 64, WARPS = 4, THREADS = 32 * (WARPS + 1);
constexpr int HALF = KT * 128;  // bytes of 64 keys of 64 channels
constexpr int JOIN_THREADS = 256;
static_assert(4 * 64 * (2 * kPrefixSplit + kOwnSplit) <= 40 * 1024, "the join's weights");
constexpr float kLazy = 8.0f;  // log2 of how far a maximum may grow before O is rescaled

template <int DP, bool MANY>
struct Shape {
  static constexpr int rows = MANY ? 64 : 16;
  static constexpr int halves = DP / 64, tile = halves * HALF, stage = 2 * tile;
  // CTAs an SM: three, of the blocks of 64 rows (whose registers do not allow for it) two
  static constexpr int ctas = MANY ? 2 : 3;
  static constexpr int stages = (DP == 128 ? 1 : 2) * (MANY ? 3 : 2);
  static constexpr int smem = 1024 + stages * stage + 256;
  static constexpr int part = MANY ? 0 : WARPS * 16 * DP;  // floats of the warps' O, of the block's
  static_assert(stages * stage >= (part + rows * DP + 2 * rows + (MANY ? 0 : WARPS * 32)) * 4, "the results take the ring's place");
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
    const uint16_t w = v[j * row];
    const float x = BF ? __uint_as_float(static_cast<uint32_t>(w) << 16) : __half2float(__ushort_as_half(w));
    if (!(fabsf(x) < INFINITY)) sum += x;
  }
  return sum;
}

// Rows of q and own keys of sequence b, cut to what the host allows.
__device__ __forceinline__ void sequence(const PrefixOwnArgs& a, int b, int& q0, int& nq, int& k0, int& nk) {
  q0 = b * a.max_queries, nq = a.max_queries, k0 = 0, nk = a.max_keys;
  if (a.q_start) {
    q0 = min(max(a.q_start[b], 0), a.q_rows);
    nq = min(max(min(a.q_start[b + 1], a.q_rows) - q0, 0), a.max_queries);
  }
  if (a.kv_start) {
    k0 = min(max(a.kv_start[b], 0), a.kv_rows);
    nk = min(max(min(a.kv_start[b + 1], a.kv_rows) - k0, 0), a.max_keys);
  } else if (a.kv_len) {
    nk = min(max(a.kv_len[b], 0), a.max_keys);
  }
}

template <bool BF, int DP, bool MANY>
__global__ void __launch_bounds__(THREADS, Shape<DP, MANY>::ctas)
    prefix_own_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ PrefixOwnArgs a) {
  using T = Shape<DP, MANY>;
  constexpr int S = T::stages, ROWS = T::rows, NS = MANY ? KT / 16 : 1;  // sub-tiles of 16 keys that a warp takes
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
  // The kernel before writes nothing but its parts, and waited for what came before it: the inputs may be read at once.
  int q0, nq, k0, nk;
  sequence(a, b, q0, nq, k0, nk);
  const int row0 = blk * ROWS, nrows = min(nq * a.group - row0, ROWS);
  if (nrows <= 0) {
    if (blockIdx.x == gridDim.x - 1) pdl_wait();
    return;
  }

  // visible own keys of a row of the block
  auto query = [&](int row) { return static_cast<int>(a.by_group.quotient(row0 + row)); };
  auto visible = [&](int row) { return row < nrows ? min(max(nk - nq + query(row) + 1, 0), nk) : 0; };
  const int most = visible(nrows - 1), least = visible(0);
  const int tiles = (most + KT - 1) / KT;
  const int t0 = split_from(tiles, rank, a.own_split), t1 = split_from(tiles, rank + 1, a.own_split);

  float o[DP / 8][4], m[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
  const int base = MANY ? 16 * warp : 0;  // of the warp's rows
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
    const int r = lane >> 2, c2 = 2 * (lane & 3);
    uint32_t q[DP / 16][4];  // the rows base + r and base + r + 8
    int vis[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = base + r + 8 * h, qi = query(row), head = row0 + row - qi * a.group;
      vis[h] = visible(row);
      const uint16_t* const p = a.q + static_cast<long long>(q0 + qi) * a.q_row + static_cast<long long>(kvh * a.group + head) * a.q_head;
#pragma unroll
      for (int k = 0; k < DP / 16; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int ch = 16 * k + c2 + 8 * j;
          q[k][h + 2 * j] = row < nrows && ch < a.head_dim ? *reinterpret_cast<const uint32_t*>(p + ch) : 0u;
        }
    }
    const float sc = a.scale_log2;
    // this lane's row and 16-byte piece in the ldmatrix loads of K and of V
    const int sub0 = MANY ? 0 : 16 * warp;
    const int krow = sub0 + (lane & 7) + (lane >> 4) * 8, kpiece = (lane >> 3) & 1;
    const int vrow = sub0 + (lane & 15), vpiece = lane >> 4;
    bool ok = true;
    int i = 0;
    for (int t = t0; t < t1 && ok; ++t, ++i) {
      const int s = i % S, key0 = t * KT + sub0;
      ok = mbar_wait_warp(&full[s], (i / S) & 1);
      if (!ok) break;
      uint8_t* const kb = smem + s * T::stage;
      const int left = most - key0;   // of the warp's keys, those that some row sees
      const int whole = least - key0;  // and those that all rows see
      // Values that no row sees become 0, and where some rows do not see them values that are not finite
      // do: 0 * NaN would reach those. (The rows that see these get them at the end.)
      if (whole < 16 * NS && left > 0) {
        const int from = max(whole, 0), thread = MANY ? static_cast<int>(threadIdx.x) : lane, threads = MANY ? 32 * WARPS : 32;
        auto piece = [&](int e) {
          const int row = sub0 + from + e / (DP / 8), at = e % (DP / 8);
          return reinterpret_cast<uint4*>(kb + T::tile + (at >> 3) * HALF + row * 128 + (((at & 7) ^ (row & 7)) << 4));
        };
        const int seen = (min(left, 16 * NS) - from) * (DP / 8), all = (16 * NS - from) * (DP / 8);
        uint32_t acc = 0u;
        for (int e = thread; e < all; e += threads) {
          uint4* const p = piece(e);
          if (e < seen)
            look16<BF>(p->x, acc), look16<BF>(p->y, acc), look16<BF>(p->z, acc), look16<BF>(p->w, acc);
          else
            *p = make_uint4(0u, 0u, 0u, 0u);
        }
        if (bad16<BF>(acc) != 0u) {
          *bad = 1;
          for (int e = thread; e < seen; e += threads) {
            uint4* const p = piece(e);
            const uint4 w = *p;
            *p = make_uint4(w.x & ~bad16<BF>(w.x), w.y & ~bad16<BF>(w.y), w.z & ~bad16<BF>(w.z), w.w & ~bad16<BF>(w.w));
          }
        }
        fence_async_smem();  // (before the next tile is copied there)
        if (MANY)
          named_bar_sync(1, 32 * WARPS);
        else
          __syncwarp();
      }
      if (left > 0) {
        float x[2 * NS][4];
#pragma unroll
        for (int n = 0; n < 2 * NS; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.0f;
        const uint32_t ks = smem_addr(kb) + krow * 128, vs = smem_addr(kb + T::tile) + vrow * 128;
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          if (16 * n >= left) continue;
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            uint32_t bk[4];
            ldmatrix4(ks + n * 2048 + (k >> 2) * HALF + (((2 * (k & 3) + kpiece) ^ (krow & 7)) << 4), bk);
            mma16816<BF>(x[2 * n], q[k], bk[0], bk[1]);
            mma16816<BF>(x[2 * n + 1], q[k], bk[2], bk[3]);
          }
        }
        if (whole < 16 * NS) {
#pragma unroll
          for (int n = 0; n < 2 * NS; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (key0 + 8 * n + c2 + (j & 1) >= vis[j >> 1]) x[n][j] = -INFINITY;
        }
        float top[2], keep[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v = -INFINITY;
#pragma unroll
          for (int n = 0; n < 2 * NS; ++n) v = max3(v, x[n][2 * h], x[n][2 * h + 1]);
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
        uint32_t p[NS][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float neg = m[h] == -INFINITY ? 0.0f : fmaf(-m[h], sc, -a.down);
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = ex2_approx(fmaf(x[2 * n + (j >> 1)][2 * h + (j & 1)], sc, neg));
            sum[h] += (e[0] + e[1]) + (e[2] + e[3]);
            p[n][h] = pack16<BF>(e[0], e[1]);
            p[n][2 + h] = pack16<BF>(e[2], e[3]);
          }
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          if (16 * n >= left) continue;
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            uint32_t bv[4];
            ldmatrix4_trans(vs + n * 2048 + (k >> 2) * HALF + (((2 * (k & 3) + vpiece) ^ (vrow & 7)) << 4), bv);
            mma16816<BF>(o[2 * k], p[n], bv[0], bv[1]);
            mma16816<BF>(o[2 * k + 1], p[n], bv[2], bv[3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[s]);
    }
    if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
  }
  __syncthreads();  // all tiles are consumed: the ring's memory takes the results, [channels / 4][row] of four channels
  float* const whole = reinterpret_cast<float*>(smem);  // of this CTA's block
  float* const cta = whole + ROWS * DP;                 // [row][maximum, sum]
  float* const part = cta + 2 * ROWS;                   // [warp] of 16 rows, and
  float* const stat = part + T::part;                   // [warp][row][maximum, sum]
  if (warp < WARPS) {
    const int r = lane >> 2, c2 = 2 * (lane & 3);
    float* const to = MANY ? whole : part + warp * 16 * DP;
    float* const st = MANY ? cta : stat + warp * 32;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
      sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
      const int row = base + r + 8 * h;
      if ((lane & 3) == 0) *reinterpret_cast<float2*>(st + 2 * row) = make_float2(m[h], sum[h]);
#pragma unroll
      for (int j = 0; j < DP / 8; ++j)
        *reinterpret_cast<float2*>(to + ((2 * j + (c2 >> 2)) * ROWS + row) * 4 + (c2 & 3)) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
    }
  }
  __syncthreads();
  const int quads = a.head_dim / 4;
  const float sc = a.scale_log2;
  const bool left_out = *bad != 0;
  // (a thread keeps its row: what the addresses of a row take is reckoned once)
  const int row = threadIdx.x & (ROWS - 1);
  if (row < nrows && threadIdx.x < THREADS / ROWS * ROWS) {
    const int qi = query(row), head = row0 + row - qi * a.group, sub = head / a.hg, h = kvh * a.nsub + sub;
    const long long rho = static_cast<long long>(q0 + qi) * a.hg + (head - sub * a.hg);
    float* const sums = a.parts.sums + a.parts.sums_at(a.prefix_parts + rank, h, rho);
    float f[WARPS];
    float top = -INFINITY, total = 0.0f;
    if constexpr (MANY) {
      const float2 st = *reinterpret_cast<const float2*>(cta + 2 * row);
      top = st.x, total = st.y;
    } else {
#pragma unroll
      for (int w = 0; w < WARPS; ++w) top = fmaxf(top, stat[32 * w + 2 * row]);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float2 st = *reinterpret_cast<const float2*>(stat + 32 * w + 2 * row);
        // (a part without a finite score has sums of zeros, or NaN that must stay)
        f[w] = st.x == -INFINITY ? 1.0f : ex2_approx((st.x - top) * sc);
        total = fmaf(st.y, f[w], total);
      }
    }
    if (threadIdx.x < ROWS)
      *reinterpret_cast<float2*>(a.parts.stat + a.parts.stat_at(a.prefix_parts + rank, h, rho)) = make_float2(top, left_out ? -total : total);
    if (top != -INFINITY)
      for (int quad = threadIdx.x / ROWS; quad < quads; quad += THREADS / ROWS) {
        float4 y;
        if constexpr (MANY) {
          y = *reinterpret_cast<const float4*>(whole + (quad * ROWS + row) * 4);
        } else {
          y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int w = 0; w < WARPS; ++w) {
            const float4 o4 = *reinterpret_cast<const float4*>(part + w * 16 * DP + (quad * ROWS + row) * 4);
            y.x = fmaf(o4.x, f[w], y.x), y.y = fmaf(o4.y, f[w], y.y), y.z = fmaf(o4.z, f[w], y.z), y.w = fmaf(o4.w, f[w], y.w);
          }
        }
        *reinterpret_cast<float4*>(sums + quad * kQuadStep) = y;
      }
  }
  if (blockIdx.x == gridDim.x - 1) pdl_wait();
}

// A CTA has ROWS rows (query, head) of one sequence, over all its heads. First the weight of each part in each row, then
// the weighted sums, four channels of a row a thread: four neighbouring threads have a row, so that whole sectors of the
// parts and of out move.
template <bool BF, int ROWS>
__global__ void __launch_bounds__(JOIN_THREADS)
    prefix_join_kernel(const __grid_constant__ PrefixOwnArgs a) {
  constexpr int GROUPS = JOIN_THREADS / ROWS;  // threads that share a row's parts
  extern __shared__ float weight[];            // [part][ROWS]: times 1 / the joint sum; -1: not to be read
  __shared__ float2 partial[GROUPS][ROWS];     // maximum and sum of a thread's parts (the sign: values left out)
  __shared__ float base[ROWS];                 // 0, or NaN in rows without a sum above 0
  __shared__ int look[ROWS];                   // 1: values that the row may see have been left out
  const int b = static_cast<int>(a.by_join.quotient(blockIdx.x)), blk = static_cast<int>(blockIdx.x) - b * a.join_blocks;
  pdl_trigger();
  // (the inputs may be read before the wait, as by prefix_own_kernel)
  int q0, nq, k0, nk;
  sequence(a, b, q0, nq, k0, nk);
  // its prefix: the last g with seq_start[g] <= b
  int prefix = 0, len = a.max_prefix;
  if (a.seq_start) {
    int lo = 0, hi = a.prefixes;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.seq_start[mid] <= b)
        lo = mid;
      else
        hi = mid;
    }
    prefix = a.seq_start[lo] <= b && b < a.seq_start[lo + 1] ? lo : -1;
    if (prefix < 0) len = 0;
  }
  if (prefix >= 0 && a.prefix_len) len = min(max(a.prefix_len[prefix], 0), a.max_prefix);
  const int heads = a.heads_kv * a.group, row0 = blk * ROWS, nrows = min(nq * heads - row0, ROWS);
  if (nrows <= 0) return;
  const int key_tiles = (len + kPrefixTile - 1) / kPrefixTile, parts = a.prefix_parts + (a.max_keys > 0 ? a.own_split : 0);
  auto written = [&](int p) {  // (a part without key tiles of its prefix is not)
    const int r = a.pair ? p >> 1 : p;
    return p >= a.prefix_parts || split_from(key_tiles, r + 1, a.split) - split_from(key_tiles, r, a.split) > (a.pair ? p & 1 : 0);
  };
  struct Row {
    int query, head, h;
    long long rho;
  };
  auto place = [&](int row) {
    Row r;
    r.query = static_cast<int>(a.by_heads.quotient(row0 + row)), r.head = row0 + row - r.query * heads;
    const int kvh = static_cast<int>(a.by_group.quotient(r.head)), in = r.head - kvh * a.group, sub = in / a.hg;
    r.h = kvh * a.nsub + sub;
    r.rho = static_cast<long long>(q0 + r.query) * a.hg + (in - sub * a.hg);
    return r;
  };
  const float sc = a.scale_log2;
  auto factor = [&](float m, float top) { return m == -INFINITY ? 1.0f : ex2_approx((m - top) * sc); };
  {
    // (a part without a finite score has a sum of 0, or NaN that must stay)
    const int row = threadIdx.x & (ROWS - 1), g = threadIdx.x / ROWS;
    const Row r = place(min(row, nrows - 1));
    const float* const st = a.parts.stat + a.parts.stat_at(0, r.h, r.rho);
    const long long step = a.parts.stat_at(1, 0, 0);
    float top = -INFINITY, total = 0.0f;
    bool left_out = false;
    pdl_wait();
#pragma unroll 4
    for (int p = g; p < parts; p += GROUPS) {
      const float2 v = written(p) ? *reinterpret_cast<const float2*>(st + p * step) : make_float2(-INFINITY, 0.0f);
      left_out |= __float_as_int(v.y) < 0;
      const float up = fmaxf(top, v.x);
      total = total * factor(top, up) + fabsf(v.y) * factor(v.x, up);
      top = up;
      weight[p * ROWS + row] = v.x;
    }
    partial[g][row] = make_float2(top, left_out ? -total : total);
    __syncthreads();
    top = -INFINITY, total = 0.0f, left_out = false;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) top = fmaxf(top, partial[k][row].x);
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const float2 v = partial[k][row];
      left_out |= __float_as_int(v.y) < 0;
      total += fabsf(v.y) * factor(v.x, top);
    }
    const float inv = 1.0f / total;
    for (int p = g; p < parts; p += GROUPS) {
      const float m = weight[p * ROWS + row];
      weight[p * ROWS + row] = m == -INFINITY ? -1.0f : ex2_approx((m - top) * sc) * inv;
    }
    if (g == 0) {
      const bool sees = len > 0 || min(nk - nq + r.query + 1, nk) > 0;
      base[row] = sees && !(total > 0.0f) ? __int_as_float(0x7fc00000) : 0.0f;
      look[row] = left_out;
    }
    __syncthreads();
  }
  const int row = (threadIdx.x >> 2) & (ROWS - 1);
  if (row >= nrows) return;
  const Row r = place(row);
  const int kvh = r.h / a.nsub, quads = a.head_dim / 4;
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
        float z[4] = {y[u].x, y[u].y, y[u].z, y[u].w};
        // (an infinite value whose probability has rounded to 0 gave NaN)
        const float odd = fmaf(z[0], 0.0f, fmaf(z[1], 0.0f, fmaf(z[2], 0.0f, z[3] * 0.0f)));
        if ((odd != 0.0f || look[row]) && none == 0.0f) {
          const int seen = min(max(nk - nq + r.query + 1, 0), nk);  // of the own keys
#pragma unroll 1
          for (int j = 0; j < 4; ++j) {
            const float was = j == 0 ? z[0] : j == 1 ? z[1] : j == 2 ? z[2] : z[3];
            float s = 0.0f;
            if (seen > 0) s += bad_values<BF>(a.v + (a.kv_start ? 0 : b * a.v_batch) + k0 * a.v_row + kvh * a.v_head + 4 * quad + j, a.v_row, seen);
            if (!(fabsf(was) < INFINITY) && len > 0)
              s += bad_values<BF>(a.pv + prefix * a.pv_batch + kvh * a.pv_head + 4 * quad + j, a.pv_row, len);
            if (s != 0.0f) z[0] = j == 0 ? s : z[0], z[1] = j == 1 ? s : z[1], z[2] = j == 2 ? s : z[2], z[3] = j == 3 ? s : z[3];  // (NaN too)
          }
        }
        *reinterpret_cast<uint2*>(out + 4 * quad) = make_uint2(pack16<BF>(z[0], z[1]), pack16<BF>(z[2], z[3]));
      }
    }
  };
  if (parts <= 2)
    run(std::integral_constant<int, ROWS == 64 ? 4 : 2>(), std::integral_constant<int, 2>());
  else
    run(std::integral_constant<int, 1>(), std::integral_constant<int, 16>());
}

template <bool BF, int DP, bool MANY>
cudaError_t launch(const PrefixOwn& own, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (own.keys)
    e = launch_pdl(prefix_own_kernel<BF, DP, MANY>, dim3(static_cast<unsigned>(own.units * own.a.own_split)), dim3(THREADS), Shape<DP, MANY>::smem, s,
                   own.k, own.v, own.a);
  if (e != cudaSuccess) return e;
  const int parts = own.a.prefix_parts + (own.keys ? own.a.own_split : 0), rows = own.join_rows;
  return launch_pdl(rows == 64 ? prefix_join_kernel<BF, 64> : prefix_join_kernel<BF, 16>, dim3(static_cast<unsigned>(own.a.batch) * own.a.join_blocks),
                    dim3(JOIN_THREADS), 4 * parts * rows, s, own.a);
}

cudaError_t init_attributes() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  auto both = [&](auto many) {
    constexpr bool M = many.value;
    set(prefix_own_kernel<true, 64, M>, Shape<64, M>::smem);
    set(prefix_own_kernel<false, 64, M>, Shape<64, M>::smem);
    set(prefix_own_kernel<true, 128, M>, Shape<128, M>::smem);
    set(prefix_own_kernel<false, 128, M>, Shape<128, M>::smem);
  };
  both(std::false_type());
  both(std::true_type());
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
  a.prefix_parts = p.prefix_parts(), a.own_split = p.own_split;
  a.status = status;
  own->many = p.many != 0, own->keys = u.max_keys > 0;
  own->units = static_cast<int64_t>(p.blocks) * a.batch * a.heads_kv;
  if (own->units * a.own_split > 0x7fffffffLL) {
    set_error("elasto_op_prefix_attention: too many sequences or queries");
    return ELASTO_ERR_UNSUPPORTED;
  }
  a.blocks = p.blocks;
  // the join: 64 rows a CTA where these fill the SMs, else 16
  const int64_t all = static_cast<int64_t>(a.max_queries) * u.heads;
  own->join_rows = (all + 63) / 64 * a.batch >= 2LL * num_sms() ? 64 : 16;
  const int64_t join_blocks = (all + own->join_rows - 1) / own->join_rows;
  if (join_blocks * a.batch > 0x7fffffffLL || all > 0x3fffffff) {
    set_error("elasto_op_prefix_attention: too many sequences or queries");
    return ELASTO_ERR_UNSUPPORTED;
  }
  a.join_blocks = static_cast<int>(join_blocks);
  a.by_join = Divisor(a.join_blocks), a.by_heads = Divisor(u.heads);
  a.by_split = Divisor(a.own_split), a.by_blocks = Divisor(a.blocks), a.by_heads_kv = Divisor(a.heads_kv), a.by_group = Divisor(a.group);
  own->a = a, own->bf = u.dtype == ELASTO_BF16;
  auto map_of = [&](CUtensorMap* tm, const void* data, long long head_s, long long row_s, long long batch_s) {
    const uint64_t dims[4] = {static_cast<uint64_t>(u.head_dim), static_cast<uint64_t>(u.heads_kv), static_cast<uint64_t>(u.kv_rows),
                              static_cast<uint64_t>(u.kv_start ? 1 : u.batch)};
    const uint64_t strides[3] = {static_cast<uint64_t>(head_s) * 2, static_cast<uint64_t>(row_s) * 2, u.kv_start ? 0 : static_cast<uint64_t>(batch_s) * 2};
    const uint32_t box[4] = {64, 1, KT, 1};
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
  auto run = [&](auto bf, auto many) {
    return own.a.head_dim <= 64 ? launch<bf.value, 64, many.value>(own, s) : launch<bf.value, 128, many.value>(own, s);
  };
  auto typed = [&](auto many) { return own.bf ? run(std::true_type(), many) : run(std::false_type(), many); };
  ELASTO_CUDA_TRY(own.many ? typed(std::true_type()) : typed(std::false_type()));
  return ELASTO_OK;
}

}  // namespace elasto
