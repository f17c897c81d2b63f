// Attention in a sliding window for single tokens (elasto_op_window_attention with one
// query a sequence): bound by reading the visible keys and values once.
//
// A cluster of CTAs takes one sequence, key head and up to 16 of the query heads
// that share it; the visible keys (the sinks and the band of the window) are cut
// into tiles of 64 and shared out over the CTAs. In a CTA
//   warp 4      streams K and V tiles by TMA through a ring;
//   warps 0-3   take 16 keys of each tile: S = Q K^T and O += P V by m16n8k16
//               products with the heads as rows (tcgen05 would need 128 of them; the
//               arithmetic is hidden behind the loads either way), running maximum
//               and sum of the softmax for itself.
// At the end the warps' (maximum, sum, O) are joined in shared memory and the
// CTAs' through distributed shared memory, in a fixed order: one launch, no workspace.
// All heads stand at the same position, so a key is visible to all rows or none;
// values of hidden keys inside a tile are set to zero.
// 64 sequences of up to 8192 keys, 32 / 8 heads of 128, window 4095: 150 us, 6.3 TB/s (of 6.8 measured
// for a copy). One sequence: 5.6 us, the chain of launch, loads and the two joins.
#include <algorithm>
#include <atomic>

#include "common.h"
#include "ptx.cuh"
#include "window_cluster.h"

namespace elasto {

namespace {

constexpr int KT = 64, ROWS = 16, WARPS = 4, THREADS = 32 * (WARPS + 1);
constexpr int HALF = KT * 128;  // bytes of 64 keys of 64 channels
constexpr int MAX_CLUSTER = 16;
constexpr float kLazy = 8.0f;   // log2 of how far a maximum may grow before O is rescaled

template <int DP>
struct Shape {
  static constexpr int halves = DP / 64, tile = halves * HALF, stage = 2 * tile;
  static constexpr int stages = DP == 128 ? 3 : 6;  // two CTAs an SM
  static constexpr int smem = 1024 + stages * stage + 256;
  static_assert(stages * stage >= (WARPS + 1) * ROWS * DP * 4 + 1024, "the partial results take the ring's place");
};

struct Args {
  int batch, heads_kv, group, head_dim;
  int window, sinks;
  float scale_log2, down;  // P is 2^-down times the probability over the running maximum (sum_headroom)
  int q_rows, max_keys, kv_rows;
  const int* q_start;
  const int* kv_start;
  const int* kv_len;
  const uint16_t* q;
  long long q_row, q_head;
  const uint16_t* v;
  long long v_batch, v_row, v_head;
  uint16_t* out;
  long long out_row, out_head;
  int nsub, rows;  // parts of a head group, heads of a part
  int cluster;
  int* status;
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
__device__ __forceinline__ float cluster_load(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}

// The sum of the infinite and NaN values of a channel that the token sees, `y` where there are none. v: the channel
// of key 0; keys [0, sinks) and [lo, nk) are visible. (Rare, so by the thread key by key.)
template <bool BF>
__device__ __noinline__ float bad_values(const uint16_t* v, long long row, int sinks, int lo, int nk, float y) {
  float sum = 0.0f;
#pragma unroll 8
  for (int j = 0; j < sinks + nk - lo; ++j) {
    const uint16_t w = v[(j < sinks ? j : lo + j - sinks) * row];
    const float x = BF ? __uint_as_float(static_cast<uint32_t>(w) << 16) : __half2float(__ushort_as_half(w));
    if (!(fabsf(x) < INFINITY)) sum += x;
  }
  return sum == 0.0f ? y : sum;
}

template <bool BF, int DP>
__global__ void __launch_bounds__(THREADS)
    window_decode_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                         const __grid_constant__ Args a) {
  using T = Shape<DP>;
  constexpr int S = T::stages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S * T::stage);
  uint64_t* empty = full + S;
  const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int rank = static_cast<int>(blockIdx.x) % a.cluster;
  int unit = static_cast<int>(blockIdx.x) / a.cluster;
  const int sub = unit % a.nsub;
  unit /= a.nsub;
  const int kvh = unit % a.heads_kv, b = unit / a.heads_kv;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], WARPS);
    }
    fence_barrier_init();
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  // the sequence, cut to what the host allows
  int q0 = b, nq = 1, k0 = 0, nk = a.max_keys;
  if (a.q_start) {
    q0 = min(max(a.q_start[b], 0), a.q_rows);
    nq = min(a.q_start[b + 1], a.q_rows) > q0 ? 1 : 0;
  }
  if (a.kv_start) {
    k0 = min(max(a.kv_start[b], 0), a.kv_rows);
    nk = min(max(min(a.kv_start[b + 1], a.kv_rows) - k0, 0), a.max_keys);
  } else if (a.kv_len) {
    nk = min(max(a.kv_len[b], 0), a.max_keys);
  }
  if (nq == 0) return;  // (the whole cluster)
  // visible keys: [0, sinks) and [lo, nk); tiles of the one, then of the other
  int lo = max(nk - 1 - a.window, 0), sinks = min(a.sinks, lo);
  if (lo <= sinks) lo = 0, sinks = 0;
  const int sink_tiles = (sinks + KT - 1) / KT, tiles = nk == 0 ? 0 : sink_tiles + (nk - lo + KT - 1) / KT;
  const int t0 = static_cast<int>(static_cast<long long>(tiles) * rank / a.cluster);
  const int t1 = static_cast<int>(static_cast<long long>(tiles) * (rank + 1) / a.cluster);
  const int head0 = kvh * a.group + sub * a.rows, nheads = min(a.rows, a.group - sub * a.rows);

  float o[DP / 8][4], m[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
  if (warp == WARPS) {
    if (elect_one()) {
      bool ok = true;
      int i = 0;
      for (int t = t0; t < t1; ++t, ++i) {
        const int s = i % S, row = k0 + (t < sink_tiles ? t * KT : lo + (t - sink_tiles) * KT);
        ok = mbar_wait(&empty[s], ((i / S) & 1) ^ 1);
        if (!ok) break;
        uint8_t* dst = smem + s * T::stage;
        mbar_expect_tx(&full[s], T::stage);
        for (int h = 0; h < T::halves; ++h) {
          tma_load_4d(dst + h * HALF, &tmK, &full[s], 64 * h, kvh, row, a.kv_start ? 0 : b);
          tma_load_4d(dst + T::tile + h * HALF, &tmV, &full[s], 64 * h, kvh, row, a.kv_start ? 0 : b);
        }
      }
      if (!ok) record_status(a.status, ELASTO_ERR_TIMEOUT);
      for (int k = max(0, i - S); k < i; ++k) mbar_wait(&full[k % S], (k / S) & 1);
    }
    __syncwarp();
  } else {
    const int r = lane >> 2, c2 = 2 * (lane & 3);
    uint32_t q[DP / 16][4];  // the heads' rows r and r + 8
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = r + 8 * (j & 1), ch = 16 * k + c2 + 8 * (j >> 1);
        q[k][j] = row < nheads && ch < a.head_dim
                      ? *reinterpret_cast<const uint32_t*>(a.q + static_cast<long long>(q0) * a.q_row + (head0 + row) * a.q_head + ch)
                      : 0u;
      }
    const float sc = a.scale_log2;
    // this lane's row and 16-byte piece in the ldmatrix loads of K and of V
    const int krow = 16 * warp + (lane & 7) + (lane >> 4) * 8, kpiece = (lane >> 3) & 1;
    const int vrow = 16 * warp + (lane & 15), vpiece = lane >> 4;
    bool ok = true;
    int i = 0;
    for (int t = t0; t < t1 && ok; ++t, ++i) {
      const int s = i % S;
      const int first = (t < sink_tiles ? t * KT : lo + (t - sink_tiles) * KT) + 16 * warp;  // of this warp's keys
      const int left = (t < sink_tiles ? sinks : nk) - first;                                 // how many of them are visible
      ok = mbar_wait_warp(&full[s], (i / S) & 1);
      if (!ok) break;
      if (left > 0) {
        uint8_t* const kb = smem + s * T::stage;
        const uint32_t ks = smem_addr(kb) + krow * 128, vs = smem_addr(kb + T::tile) + vrow * 128;
        if (left < 16) {
          for (int e = lane; e < (16 - left) * DP / 8; e += 32) {
            const int row = 16 * warp + left + e / (DP / 8), piece = e % (DP / 8);
            *reinterpret_cast<uint4*>(kb + T::tile + (piece >> 3) * HALF + row * 128 + (piece & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_async_smem();  // (before the next tile is copied there)
          __syncwarp();
        }
        float x[2][4] = {};
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          uint32_t bk[4];
          ldmatrix4(ks + (k >> 2) * HALF + (((2 * (k & 3) + kpiece) ^ (krow & 7)) << 4), bk);
          mma16816<BF>(x[0], q[k], bk[0], bk[1]);
          mma16816<BF>(x[1], q[k], bk[2], bk[3]);
        }
        if (left < 16) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (8 * (j >> 2) + c2 + (j & 1) >= left) x[j >> 2][j & 3] = -INFINITY;
        }
        float top[2], keep[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v = fmaxf(fmaxf(x[0][2 * h], x[0][2 * h + 1]), fmaxf(x[1][2 * h], x[1][2 * h + 1]));
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
        uint32_t p[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float neg = m[h] == -INFINITY ? 0.0f : fmaf(-m[h], sc, -a.down);
          float e[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) e[j] = ex2_approx(fmaf(x[j >> 1][2 * h + (j & 1)], sc, neg));
          sum[h] += (e[0] + e[1]) + (e[2] + e[3]);
          p[h] = pack16<BF>(e[0], e[1]);
          p[2 + h] = pack16<BF>(e[2], e[3]);
        }
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
          uint32_t bv[4];
          ldmatrix4_trans(vs + (k >> 2) * HALF + (((2 * (k & 3) + vpiece) ^ (vrow & 7)) << 4), bv);
          mma16816<BF>(o[2 * k], p, bv[0], bv[1]);
          mma16816<BF>(o[2 * k + 1], p, bv[2], bv[3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[s]);
    }
    if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
  }
  __syncthreads();  // all tiles are consumed: the ring's memory takes the partial results
  float* const part = reinterpret_cast<float*>(smem);                 // [warp][head][channel]
  float* const whole = part + WARPS * ROWS * DP;                      // [head][channel] of this CTA
  float* const stat = whole + ROWS * DP;                              // [warp][head][maximum, sum]
  float* const cta = stat + WARPS * ROWS * 2;                         // [head][maximum, sum] of this CTA
  if (warp < WARPS) {
    const int r = lane >> 2, c2 = 2 * (lane & 3);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
      sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
      if ((lane & 3) == 0) {
        stat[(warp * ROWS + r + 8 * h) * 2] = m[h];
        stat[(warp * ROWS + r + 8 * h) * 2 + 1] = sum[h];
      }
#pragma unroll
      for (int j = 0; j < DP / 8; ++j)
        *reinterpret_cast<float2*>(part + (warp * ROWS + r + 8 * h) * DP + 8 * j + c2) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < nheads * DP; e += THREADS) {
    const int h = e / DP;
    float top = -INFINITY, total = 0.0f, y = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, stat[(w * ROWS + h) * 2]);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float mw = stat[(w * ROWS + h) * 2], f = mw == -INFINITY ? 0.0f : ex2_approx((mw - top) * a.scale_log2);
      // (a warp without a finite score has sums of zeros, or NaN that must stay)
      const float s = stat[(w * ROWS + h) * 2 + 1];
      total += mw == -INFINITY ? s : s * f;
      y += mw == -INFINITY ? part[w * ROWS * DP + e] : part[w * ROWS * DP + e] * f;
    }
    whole[e] = y;
    if (e % DP == 0) cta[2 * h] = top, cta[2 * h + 1] = total;
  }
  if (a.cluster > 1)
    cluster_sync_all();
  else
    __syncthreads();
  for (int e = rank * THREADS + threadIdx.x; e < nheads * DP; e += a.cluster * THREADS) {
    const int h = e / DP, ch = e % DP;
    const uint32_t ms = smem_addr(cta + 2 * h), ys = smem_addr(whole + e);
    float mk[MAX_CLUSTER], lk[MAX_CLUSTER], yk[MAX_CLUSTER], top = -INFINITY;
#pragma unroll
    for (int k = 0; k < MAX_CLUSTER; ++k)
      if (k < a.cluster) {
        mk[k] = cluster_load(cluster_map(ms, k));
        lk[k] = cluster_load(cluster_map(ms + 4, k));
        yk[k] = cluster_load(cluster_map(ys, k));
      }
#pragma unroll
    for (int k = 0; k < MAX_CLUSTER; ++k)
      if (k < a.cluster) top = fmaxf(top, mk[k]);
    float total = 0.0f, y = 0.0f;
#pragma unroll
    for (int k = 0; k < MAX_CLUSTER; ++k)
      if (k < a.cluster) {
        const float f = ex2_approx((mk[k] - top) * a.scale_log2);
        total += mk[k] == -INFINITY ? lk[k] : lk[k] * f;
        y += mk[k] == -INFINITY ? yk[k] : yk[k] * f;
      }
    if (ch < a.head_dim) {
      y = nk > 0 ? y / total : 0.0f;
      // (an infinite value whose probability has rounded to 0 gave NaN; where the sum is 0 or NaN all channels are NaN)
      if (!(fabsf(y) < INFINITY) && total > 0.0f)
        y = bad_values<BF>(a.v + (a.kv_start ? 0 : b * a.v_batch) + k0 * a.v_row + kvh * a.v_head + ch, a.v_row, sinks, lo, nk, y);
      a.out[static_cast<long long>(q0) * a.out_row + (head0 + h) * a.out_head + ch] =
          BF ? __bfloat16_as_ushort(__float2bfloat16_rn(y)) : __half_as_ushort(__float2half_rn(y));
    }
  }
  if (a.cluster > 1) cluster_sync_all();  // the peers have read this CTA's results
}

template <bool BF, int DP>
cudaError_t launch(const CUtensorMap& tk, const CUtensorMap& tv, const Args& a, unsigned units, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see launch_pdl
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(units * a.cluster);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = Shape<DP>::smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, window_decode_kernel<BF, DP>, tk, tv, a);
}

// 16 where the current device runs a cluster of that many of these CTAs, which not every one (or part of one) does, else
// 8, which all do. Asked for once a device.
int largest_cluster(bool narrow) {
  static std::atomic<int> known[64][2];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 8;
  int n = known[dev][narrow].load(std::memory_order_relaxed);
  if (n > 0) return n;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = MAX_CLUSTER;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3(MAX_CLUSTER);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = narrow ? Shape<64>::smem : Shape<128>::smem;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int clusters = 0;
  const cudaError_t e = narrow ? cudaOccupancyMaxActiveClusters(&clusters, window_decode_kernel<true, 64>, &cfg)
                               : cudaOccupancyMaxActiveClusters(&clusters, window_decode_kernel<true, 128>, &cfg);
  if (e != cudaSuccess) cudaGetLastError();  // (a size that the device does not know)
  n = e == cudaSuccess && clusters > 0 ? MAX_CLUSTER : 8;
  known[dev][narrow].store(n, std::memory_order_relaxed);
  return n;
}

cudaError_t init_attributes() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(f, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  };
  set(window_decode_kernel<true, 64>, Shape<64>::smem);
  set(window_decode_kernel<false, 64>, Shape<64>::smem);
  set(window_decode_kernel<true, 128>, Shape<128>::smem);
  set(window_decode_kernel<false, 128>, Shape<128>::smem);
  return e;
}

}  // namespace

elasto_status window_decode_launch(const elasto_window_attention_args& u, int* status, cudaStream_t s) {
  static DeviceOnce once;
  ELASTO_CUDA_TRY(once(init_attributes));
  Args a{};
  a.batch = u.batch, a.heads_kv = u.heads_kv, a.group = u.heads / u.heads_kv, a.head_dim = u.head_dim;
  a.window = u.window < 0 || u.window > u.max_keys ? u.max_keys : u.window;
  a.sinks = u.sinks > u.max_keys ? u.max_keys : u.sinks;
  a.scale_log2 = u.scale * 1.4426950408889634f;
  a.down = sum_headroom(u.dtype == ELASTO_BF16, u.max_keys);
  a.q_rows = static_cast<int>(u.q_rows), a.max_keys = u.max_keys, a.kv_rows = static_cast<int>(u.kv_rows);
  a.q_start = u.q_start, a.kv_start = u.kv_start, a.kv_len = u.kv_len;
  a.q = static_cast<const uint16_t*>(u.q), a.q_row = u.q_row, a.q_head = u.q_head;
  a.v = static_cast<const uint16_t*>(u.v), a.v_batch = u.v_batch, a.v_row = u.v_row, a.v_head = u.v_head;
  a.out = static_cast<uint16_t*>(u.out), a.out_row = u.out_row, a.out_head = u.out_head;
  a.nsub = (a.group + ROWS - 1) / ROWS;
  a.rows = (a.group + a.nsub - 1) / a.nsub;
  a.status = status;
  const long long units = static_cast<long long>(a.batch) * a.heads_kv * a.nsub;
  const long long keys = std::min<long long>(u.max_keys, static_cast<long long>(a.window) + 1 + a.sinks);
  a.cluster = single_token_cluster(units, keys, num_sms(), MAX_CLUSTER);
  if (a.cluster > 8) a.cluster = single_token_cluster(units, keys, num_sms(), largest_cluster(u.head_dim <= 64));
  if (units * a.cluster > 0x7fffffffLL) {
    set_error("elasto_op_window_attention: too many sequences");
    return ELASTO_ERR_UNSUPPORTED;
  }
  const bool bf = u.dtype == ELASTO_BF16;
  auto map_of = [&](CUtensorMap* tm, const void* p, long long head_s, long long row_s, long long batch_s) {
    const uint64_t dims[4] = {static_cast<uint64_t>(u.head_dim), static_cast<uint64_t>(u.heads_kv),
                              static_cast<uint64_t>(u.kv_rows), static_cast<uint64_t>(u.kv_start ? 1 : u.batch)};
    const uint64_t strides[3] = {static_cast<uint64_t>(head_s) * 2, static_cast<uint64_t>(row_s) * 2,
                                 u.kv_start ? 0 : static_cast<uint64_t>(batch_s) * 2};
    const uint32_t box[4] = {64, 1, KT, 1};
    return encode_tmap_16(tm, p, bf, 4, dims, strides, box);
  };
  CUtensorMap tk, tv;
  if (!map_of(&tk, u.k, u.k_head, u.k_row, u.k_batch) || !map_of(&tv, u.v, u.v_head, u.v_row, u.v_batch)) {
    set_error("elasto_op_window_attention: cuTensorMapEncodeTiled failed (alignment, strides or size)");
    return ELASTO_ERR_UNSUPPORTED;
  }
  const unsigned n = static_cast<unsigned>(units);
  cudaError_t e;
  if (u.head_dim <= 64)
    e = bf ? launch<true, 64>(tk, tv, a, n, s) : launch<false, 64>(tk, tv, a, n, s);
  else
    e = bf ? launch<true, 128>(tk, tv, a, n, s) : launch<false, 128>(tk, tv, a, n, s);
  ELASTO_CUDA_TRY(e);
  return ELASTO_OK;
}

}  // namespace elasto
