// Attention behind shared prefixes: the sequences' own keys, joined with the parts that prefix_attention.cu left.
//
// A block is 16 or 64 rows (query, head) of one sequence and key head; a cluster of CTAs takes it, the own keys in tiles
// of 64 shared out over the CTAs. In a CTA warp 4 streams K and V tiles by TMA through a ring, and warps 0-3 form
// S = Q K^T and O += P V by m16n8k16 products, running maximum and sum of the softmax for themselves:
//   16 rows (single tokens and few): a warp takes 16 keys of each tile, all rows;
//   64 rows (longer runs of tokens): a warp takes 16 rows, all keys.
// (tcgen05 would need 128 rows of one sequence: the prefix, where most of the work lies, has them.) Then the warps' results
// are joined in shared memory, the CTAs' through distributed shared memory, and the prefix's parts, in a fixed order.
// This kernel starts while the prefixes' runs out (programmatic launch) and waits for it only before it reads the parts.
//
// Bound by reading the own keys and values once.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "prefix_own.h"
#include "ptx.cuh"
#include "window_cluster.h"

namespace elasto {

namespace {

constexpr int KT = 64, WARPS = 4, THREADS = 32 * (WARPS + 1);
constexpr int HALF = KT * 128;  // bytes of 64 keys of 64 channels
constexpr int MAX_CLUSTER = 8;
constexpr float kLazy = 8.0f;  // log2 of how far a maximum may grow before O is rescaled

template <int DP, bool MANY>
struct Shape {
  static constexpr int rows = MANY ? 64 : 16;
  static constexpr int halves = DP / 64, tile = halves * HALF, stage = 2 * tile;
  static constexpr int stages = DP == 128 ? 3 : 6;  // two CTAs an SM
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
__device__ __forceinline__ int cluster_load_int(uint32_t addr) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
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

// A softmax's running maximum, sum and four channels of its weighted sum.
struct Joined {
  float top, total;
  float4 y;
  // (a part without a finite score has sums of zeros, or NaN that must stay)
  __device__ __forceinline__ void add(float2 st, float4 o, float f) {
    const float w = st.x == -INFINITY ? 1.0f : f;
    total = fmaf(st.y, w, total);
    y.x = fmaf(o.x, w, y.x), y.y = fmaf(o.y, w, y.y), y.z = fmaf(o.z, w, y.z), y.w = fmaf(o.w, w, y.w);
  }
  __device__ __forceinline__ void rise(float to, float sc) {  // the maximum to at least `to`
    const float t = fmaxf(top, to), f = top == -INFINITY ? 1.0f : ex2_approx((top - t) * sc);
    total *= f, y.x *= f, y.y *= f, y.z *= f, y.w *= f;
    top = t;
  }
};

template <bool BF, int DP, bool MANY>
__global__ void __launch_bounds__(THREADS)
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
  const int rank = static_cast<int>(blockIdx.x) % a.cluster;
  const int unit = static_cast<int>(blockIdx.x) / a.cluster;
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
  // Nothing but the parts is written by the kernel before, and that one waited for what came before it: the inputs may be
  // read at once.

  // the sequence, cut to what the host allows
  int q0 = b * a.max_queries, nq = a.max_queries, k0 = 0, nk = a.max_keys;
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
  const int row0 = blk * ROWS, nrows = min(nq * a.group - row0, ROWS);
  if (nrows <= 0) return;  // (the whole cluster)
  // its prefix: the last g with seq_start[g] <= b
  int prefix = 0, len = a.max_prefix;
  if (a.seq_start) {
    int lo = 0, hi = a.prefixes;  // seq_start[lo] <= b < seq_start[hi], if there is one
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.seq_start[mid] <= b)
        lo = mid;
      else
        hi = mid;
    }
    prefix = a.seq_start[lo] <= b && b < a.seq_start[lo + 1] ? lo : -1;
  }
  if (prefix < 0)
    len = 0;
  else if (a.prefix_len)
    len = min(max(a.prefix_len[prefix], 0), a.max_prefix);

  // visible own keys of a row of the block
  auto query = [&](int row) { return static_cast<int>(a.by_group.quotient(row0 + row)); };
  auto visible = [&](int row) { return row < nrows ? min(max(nk - nq + query(row) + 1, 0), nk) : 0; };
  const int most = visible(nrows - 1), least = visible(0);
  const int tiles = (most + KT - 1) / KT;
  const int t0 = split_from(tiles, rank, a.cluster), t1 = split_from(tiles, rank + 1, a.cluster);

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
        bool any = false;
        for (int e = thread; e < (16 * NS - from) * (DP / 8); e += threads) {
          const int key = from + e / (DP / 8), row = sub0 + key, piece = e % (DP / 8);
          uint4* const p = reinterpret_cast<uint4*>(kb + T::tile + (piece >> 3) * HALF + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
          if (key >= left) {
            *p = make_uint4(0u, 0u, 0u, 0u);
          } else {
            const uint4 w = *p;
            const uint4 x = make_uint4(bad16<BF>(w.x), bad16<BF>(w.y), bad16<BF>(w.z), bad16<BF>(w.w));
            if ((x.x | x.y | x.z | x.w) != 0u) {
              *p = make_uint4(w.x & ~x.x, w.y & ~x.y, w.z & ~x.z, w.w & ~x.w);
              any = true;
            }
          }
        }
        if (any) *bad = 1;
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
  if constexpr (!MANY) {
    for (int e = threadIdx.x; e < quads * nrows; e += THREADS) {
      const int quad = e / nrows, row = e - quad * nrows;
      Joined x = {-INFINITY, 0.0f, make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
#pragma unroll
      for (int w = 0; w < WARPS; ++w) x.top = fmaxf(x.top, stat[32 * w + 2 * row]);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float2 st = *reinterpret_cast<const float2*>(stat + 32 * w + 2 * row);
        x.add(st, *reinterpret_cast<const float4*>(part + w * 16 * DP + (quad * ROWS + row) * 4), ex2_approx((st.x - x.top) * sc));
      }
      *reinterpret_cast<float4*>(whole + (quad * ROWS + row) * 4) = x.y;
      if (quad == 0) *reinterpret_cast<float2*>(cta + 2 * row) = make_float2(x.top, x.total);
    }
  }
  if (a.cluster > 1)
    cluster_sync_all();
  else
    __syncthreads();
  pdl_wait();  // the prefix's parts
  bool left_out = *bad != 0;
  for (int k = 0; k < a.cluster && a.cluster > 1; ++k) left_out |= cluster_load_int(cluster_map(smem_addr(bad), k)) != 0;
  const int key_tiles = (len + kPrefixTile - 1) / kPrefixTile, parts = a.pair ? 2 * a.split : a.split;
  // (a part without key tiles has not been written)
  auto written = [&](int part) {
    const int r = a.pair ? part >> 1 : part, n = split_from(key_tiles, r + 1, a.split) - split_from(key_tiles, r, a.split);
    return n > (a.pair ? part & 1 : 0);
  };
  for (int e = rank * THREADS + threadIdx.x; e < quads * nrows; e += a.cluster * THREADS) {
    const int quad = e / nrows, row = e - quad * nrows, qi = query(row), head = row0 + row - qi * a.group;
    const uint32_t ms = smem_addr(cta + 2 * row), ys = smem_addr(whole + (quad * ROWS + row) * 4);
    Joined x = {-INFINITY, 0.0f, make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
    if (a.cluster > 1) {
      float2 st[MAX_CLUSTER];
      float4 y[MAX_CLUSTER];
#pragma unroll
      for (int k = 0; k < MAX_CLUSTER; ++k)
        if (k < a.cluster) st[k] = cluster_load2(cluster_map(ms, k)), y[k] = cluster_load4(cluster_map(ys, k));
#pragma unroll
      for (int k = 0; k < MAX_CLUSTER; ++k)
        if (k < a.cluster) x.top = fmaxf(x.top, st[k].x);
#pragma unroll
      for (int k = 0; k < MAX_CLUSTER; ++k)
        if (k < a.cluster) x.add(st[k], y[k], ex2_approx((st[k].x - x.top) * sc));
    } else {
      const float2 st = *reinterpret_cast<const float2*>(cta + 2 * row);
      x = {st.x, st.y, *reinterpret_cast<const float4*>(whole + (quad * ROWS + row) * 4)};
    }
    if (key_tiles > 0) {
      const int sub = head / a.hg, h = kvh * a.nsub + sub;
      const long long rho = static_cast<long long>(q0 + qi) * a.hg + (head - sub * a.hg);
      constexpr int N = 8;  // parts on the way at once
      for (int p0 = 0; p0 < parts; p0 += N) {
        float2 st[N];
        float4 y[N];
        float top = x.top;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          st[k] = make_float2(-INFINITY, 0.0f), y[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (p0 + k < parts && written(p0 + k)) {
            st[k] = *reinterpret_cast<const float2*>(a.parts.stat + a.parts.stat_at(p0 + k, h, rho));
            y[k] = *reinterpret_cast<const float4*>(a.parts.sums + a.parts.sums_at(p0 + k, h, quad, rho));
          }
        }
#pragma unroll
        for (int k = 0; k < N; ++k) top = fmaxf(top, st[k].x);
        x.rise(top, sc);
#pragma unroll
        for (int k = 0; k < N; ++k) x.add(st[k], y[k], ex2_approx((st[k].x - x.top) * sc));
      }
    }
    const int seen = visible(row);
    float y[4] = {x.y.x, x.y.y, x.y.z, x.y.w};
    const float inv = 1.0f / x.total;
    uint32_t w[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // (an infinite value whose probability has rounded to 0 gave NaN; where the sum is 0 or NaN all channels are NaN)
      y[j] = seen > 0 || len > 0 ? y[j] * inv : 0.0f;
      const bool odd = !(fabsf(y[j]) < INFINITY);
      if ((odd || left_out) && x.total > 0.0f) {
        float s = 0.0f;
        if (seen > 0) s += bad_values<BF>(a.v + (a.kv_start ? 0 : b * a.v_batch) + k0 * a.v_row + kvh * a.v_head + 4 * quad + j, a.v_row, seen);
        if (odd && len > 0) s += bad_values<BF>(a.pv + prefix * a.pv_batch + kvh * a.pv_head + 4 * quad + j, a.pv_row, len);
        if (s != 0.0f) y[j] = s;  // (NaN too)
      }
    }
    w[0] = pack16<BF>(y[0], y[1]), w[1] = pack16<BF>(y[2], y[3]);
    *reinterpret_cast<uint2*>(a.out + static_cast<long long>(q0 + qi) * a.out_row + static_cast<long long>(kvh * a.group + head) * a.out_head + 4 * quad) =
        make_uint2(w[0], w[1]);
  }
  if (a.cluster > 1) cluster_sync_all();  // the peers have read this CTA's results
}

template <bool BF, int DP, bool MANY>
cudaError_t launch(const PrefixOwn& own, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see launch_pdl
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = own.a.cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(own.units * own.a.cluster));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = Shape<DP, MANY>::smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, prefix_own_kernel<BF, DP, MANY>, own.k, own.v, own.a);
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
  a.status = status;
  // 16 rows where a sequence has no more, or one query; else 64
  const int64_t rows = static_cast<int64_t>(a.max_queries) * a.group;
  own->many = a.max_queries > 1 && rows > 16;
  const int of = own->many ? 64 : 16;
  const int64_t blocks = (rows + of - 1) / of;
  own->units = blocks * a.batch * a.heads_kv;
  if (rows > 0x3fffffff || own->units > 0x7fffffffLL / MAX_CLUSTER) {
    set_error("elasto_op_prefix_attention: too many sequences or queries");
    return ELASTO_ERR_UNSUPPORTED;
  }
  a.blocks = static_cast<int>(blocks);
  a.cluster = u.max_keys > 0 ? single_token_cluster(own->units, u.max_keys, num_sms(), MAX_CLUSTER) : 1;
  a.by_blocks = Divisor(a.blocks), a.by_heads_kv = Divisor(a.heads_kv), a.by_group = Divisor(a.group);
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
