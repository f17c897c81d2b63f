// The e4m3 product of gemm_fp8.cu for few rows of A, where W's bytes and latency
// set the pace. Operands are exchanged: a CTA's accumulator is 128 columns of out
// (rows of W, the tensor core's M) by NT rows of A (its N), and the blocks of K
// are shared out over a cluster of CTAs, so that W is read by as many SMs as
// there are. Each CTA sums its blocks in registers as gemm_fp8.cu does; the
// cluster's sums are then added through distributed shared memory in rank order,
// each CTA finishing its share of the rows: one launch, no workspace, the same
// result every time.
// 8 x 4096 x 4096: 5.8 us (12.6 on 128 x 64 tiles without the split; W alone 2.5 us, the rest the chain launch,
// first loads, last sums); 8 x 8192 x 16384: 28.2 us, 4.8 TB/s.
#include <algorithm>

#include "act.cuh"
#include "common.h"
#include "fp8_common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int BM = 128, BK = 128, W_STAGE = BM * BK;
constexpr int SCALE_BLOCKS = 32;  // blocks whose scales are in shared memory at a time
constexpr int MAX_CLUSTER = 8;

template <int NT>
struct Shape {
  static constexpr int epi_warps = NT >= 64 ? 8 : 4, threads = 64 + 32 * epi_warps;
  static constexpr int stage = W_STAGE + NT * BK;
  static constexpr int ctas = NT == 128 ? 1 : 2;  // of an SM
  static constexpr int stages = std::min(6, 208 * 1024 / ctas / stage);
  static constexpr int ring = stages * stage;
  static_assert(ring >= NT * BM * 4, "the sums take the ring's place");
  static constexpr int smem = 1024 + ring + SCALE_BLOCKS * NT * 4 + 256;
  static constexpr int cols = NT / (epi_warps / 4);  // rows of A of an epilogue warp
  static constexpr int accs = NT == 128 ? 4 : std::min(8, 256 / NT);  // accumulators: the SM's CTAs share 512 columns
  static constexpr int tmem_cols = accs * NT;
};

__device__ __forceinline__ float4 cluster_load(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

template <int NT, int EPI>
__global__ void __launch_bounds__(Shape<NT>::threads)
    gemm_fp8_tokens_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                           const __grid_constant__ Fp8Gemm g, int nkb, int cluster) {
  using T = Shape<NT>;
  constexpr int S = T::stages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* sums = reinterpret_cast<float*>(smem);                // [row of A][row of W], once the ring is done with
  float* scales = reinterpret_cast<float*>(smem + T::ring);    // [block][row of A]
  uint64_t* full = reinterpret_cast<uint64_t*>(scales + SCALE_BLOCKS * NT);
  uint64_t* empty = full + S;
  uint64_t* tfull = empty + S;   // [accumulator]
  uint64_t* tempty = tfull + T::accs;
  uint64_t* drain = tempty + T::accs;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);

  const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int rank = static_cast<int>(blockIdx.x) % cluster;
  const unsigned tile = blockIdx.x / cluster;
  const unsigned nt = (g.N + BM - 1) / BM;
  const int n0 = static_cast<int>(tile % nt) * BM, m0 = static_cast<int>(tile / nt) * NT;
  const int kb0 = static_cast<int>(static_cast<long long>(rank) * nkb / cluster);
  const int kb1 = static_cast<int>((rank + 1LL) * nkb / cluster), blocks = kb1 - kb0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < T::accs; ++i) {
      mbar_init(&tfull[i], 1);
      mbar_init(&tempty[i], T::epi_warps);
    }
    mbar_init(drain, 1);
    fence_barrier_init();
  }
  if (warp == 0) {
    tmem_alloc(tmem_slot, T::tmem_cols);
    tmem_relinquish();
  }
  if (warp == 1 && elect_one()) {
    tma_prefetch_desc(&tmW);
    tma_prefetch_desc(&tmA);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(static_cast<int>(*tmem_slot));
  pdl_wait();
  pdl_trigger();

  constexpr int C = T::cols;
  const int q = warp & 3, h = warp >= 2 ? (warp - 2) >> 2 : 0;
  float2 acc[C / 2];
  if (warp == 0) {
    if (elect_one()) {
      bool ok = true;
      int i = 0;
      for (; i < blocks; ++i) {
        const int s = i % S;
        ok = mbar_wait(&empty[s], ((i / S) & 1) ^ 1);
        if (!ok) break;
        mbar_expect_tx(&full[s], T::stage);
        tma_load_2d(smem + s * T::stage, &tmW, &full[s], (kb0 + i) * BK, n0);
        tma_load_2d(smem + s * T::stage + W_STAGE, &tmA, &full[s], (kb0 + i) * BK, m0);
      }
      if (!ok) record_status(g.status, ELASTO_ERR_TIMEOUT);
      for (int k = max(0, i - S); k < i; ++k) mbar_wait(&full[k % S], (k / S) & 1);
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t idesc = idesc_e4m3_f32(BM, NT);
    bool ok = true;
    for (int i = 0; i < blocks; ++i) {
      const int s = i % S, p = i % T::accs;
      ok = mbar_wait_warp(&tempty[p], ((i / T::accs) & 1) ^ 1) && mbar_wait_warp(&full[s], (i / S) & 1);
      if (!ok) break;
      tc_fence_after();
      const uint32_t w_lo = sdesc_lo(smem_addr(smem + s * T::stage), 16), a_lo = sdesc_lo(smem_addr(smem + s * T::stage + W_STAGE), 16);
#pragma unroll
      for (int k = 0; k < BK / 32; ++k) tc_mma_f8_warp_lo(tmem + p * NT, w_lo + 2 * k, a_lo + 2 * k, sdesc_sw128_hi(1024), idesc, k != 0);
      tc_commit_warp(&empty[s]);
      tc_commit_warp(&tfull[p]);
    }
    if (!ok && lane == 0) record_status(g.status, ELASTO_ERR_TIMEOUT);
    if (blocks > 0) {
      tc_commit_warp(drain);
      mbar_wait_warp(drain, 0);
    }
  } else {
    const uint32_t tm = tmem + (static_cast<uint32_t>(q * 32) << 16) + h * C;
    const float* ws = g.w_scale + static_cast<size_t>(n0 / 128) * nkb;
    bool ok = true;
#pragma unroll
    for (int j = 0; j < C / 2; ++j) acc[j] = make_float2(0.0f, 0.0f);
    for (int i = 0; i < blocks; ++i) {
      if (i % SCALE_BLOCKS == 0) {  // products of the scales of the next blocks
        named_bar_sync(1, 32 * T::epi_warps);
        const int n = min(SCALE_BLOCKS, blocks - i) * NT;
        for (int e = threadIdx.x - 64; e < n; e += 32 * T::epi_warps) {
          const int b = kb0 + i + e / NT, m = min(m0 + e % NT, g.M - 1);
          scales[e] = __ldg(g.a_scale + static_cast<size_t>(b) * g.lds + m) * __ldg(ws + b);
        }
        named_bar_sync(1, 32 * T::epi_warps);
      }
      const int p = i % T::accs;
      ok = ok && __all_sync(0xffffffffu, mbar_wait(&tfull[p], (i / T::accs) & 1));
      if (!ok) continue;  // (the named barriers above count every warp)
      tc_fence_after();
      const float4* sc = reinterpret_cast<const float4*>(scales + (i % SCALE_BLOCKS) * NT + h * C);
      uint32_t v[C];
#pragma unroll
      for (int c = 0; c < C; c += 16) {
        uint32_t x[16];
        tmem_ld_16(tm + p * NT + c, x);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[c + j] = x[j];
      }
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&tempty[p]);
#pragma unroll
      for (int j = 0; j < C / 4; ++j) {
        const float4 s4 = sc[j];
        acc[2 * j] = fma2(make_float2(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1])), make_float2(s4.x, s4.y), acc[2 * j]);
        acc[2 * j + 1] = fma2(make_float2(__uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3])), make_float2(s4.z, s4.w),
                              acc[2 * j + 1]);
      }
    }
    if (!ok && lane == 0) record_status(g.status, ELASTO_ERR_TIMEOUT);
  }
  // every copy has landed and every product is done: the ring's memory takes the sums
  __syncthreads();
  if (warp >= 2) {
#pragma unroll
    for (int j = 0; j < C / 2; ++j) {
      sums[(h * C + 2 * j) * BM + q * 32 + lane] = acc[j].x;
      sums[(h * C + 2 * j + 1) * BM + q * 32 + lane] = acc[j].y;
    }
  }
  if (cluster > 1)
    cluster_sync_all();
  else
    __syncthreads();
  const int share = (NT + cluster - 1) / cluster;  // rows of A that each CTA finishes
  // a warp takes two rows of A at a time, a lane four columns of out; all loads of a pair are in flight at once
  constexpr int WARPS = T::threads / 32;
  const int n = n0 + 4 * lane, last = min(min((rank + 1) * share, NT), g.M - m0);
  float bias[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) bias[j] = g.bias && n + j < g.N ? __ldg(g.bias + n + j) : 0.0f;
  for (int c0 = rank * share + 2 * warp; c0 < last; c0 += 2 * WARPS) {
    float4 x[2][MAX_CLUSTER];
#pragma unroll
    for (int k = 0; k < MAX_CLUSTER; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (k < cluster) x[u][k] = cluster_load(cluster_map(smem_addr(sums + (c0 + u) * BM + 4 * lane), k));
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float y[4] = {x[u][0].x, x[u][0].y, x[u][0].z, x[u][0].w};
#pragma unroll
      for (int k = 1; k < MAX_CLUSTER; ++k)
        if (k < cluster) y[0] += x[u][k].x, y[1] += x[u][k].y, y[2] += x[u][k].z, y[3] += x[u][k].w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y[j] += bias[j];
        if constexpr (EPI == EPI_BIAS_GELU_BF16) y[j] = gelu(y[j]);
        if (c0 + u < last && n + j < g.N) fp8_store_one<EPI>(g.out, static_cast<long long>(m0 + c0 + u) * g.ldo + n + j, y[j]);
      }
    }
  }
  if (cluster > 1) cluster_sync_all();  // the peers have read this CTA's sums
  if (warp == 0) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, T::tmem_cols);
  }
}

template <int NT, int EPI>
cudaError_t launch(const Fp8Gemm& g, const CUtensorMap& tw, const CUtensorMap& ta, int nkb, int cluster, unsigned tiles,
                   cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see launch_pdl
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(tiles * cluster);
  cfg.blockDim = dim3(Shape<NT>::threads);
  cfg.dynamicSmemBytes = Shape<NT>::smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, gemm_fp8_tokens_kernel<NT, EPI>, tw, ta, g, nkb, cluster);
}

template <int NT>
cudaError_t launch_epi(const Fp8Gemm& g, const CUtensorMap& tw, const CUtensorMap& ta, int nkb, int cluster, unsigned tiles,
                       cudaStream_t s) {
  switch (g.epi) {
    case EPI_BIAS_BF16: return launch<NT, EPI_BIAS_BF16>(g, tw, ta, nkb, cluster, tiles, s);
    case EPI_BIAS_GELU_BF16: return launch<NT, EPI_BIAS_GELU_BF16>(g, tw, ta, nkb, cluster, tiles, s);
    case EPI_BIAS_RESID_F32: return launch<NT, EPI_BIAS_RESID_F32>(g, tw, ta, nkb, cluster, tiles, s);
    default: return launch<NT, EPI_BIAS_F32>(g, tw, ta, nkb, cluster, tiles, s);
  }
}

template <int NT>
void set_attributes(cudaError_t* e) {
  auto set = [&](auto* f) {
    if (*e == cudaSuccess) *e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<NT>::smem);
  };
  set(gemm_fp8_tokens_kernel<NT, EPI_BIAS_BF16>);
  set(gemm_fp8_tokens_kernel<NT, EPI_BIAS_GELU_BF16>);
  set(gemm_fp8_tokens_kernel<NT, EPI_BIAS_RESID_F32>);
  set(gemm_fp8_tokens_kernel<NT, EPI_BIAS_F32>);
}

}  // namespace

cudaError_t gemm_fp8_tokens_init_attributes() {
  cudaError_t e = cudaSuccess;
  set_attributes<16>(&e);
  set_attributes<32>(&e);
  set_attributes<64>(&e);
  set_attributes<128>(&e);
  return e;
}

namespace {

int rows_of_tile(int M) { return M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128; }
long long tiles_of(const Fp8Gemm& g, int nt) { return ((g.N + BM - 1LL) / BM) * ((g.M + nt - 1LL) / nt); }
// CTAs that share a tile's K: as many as the SMs hold at once, each with two blocks or more.
int cluster_of(long long tiles, int nt, int nkb) {
  int cluster = 1;
  while (cluster < MAX_CLUSTER && tiles * cluster * 2 <= (nt == 128 ? 1 : 2) * num_sms() && nkb >= 4 * cluster) cluster *= 2;
  return cluster;
}

}  // namespace

// Fitted to launches of 1 to 400 rows: 8 x 4096 x 4096 5.8 us (128-row tiles 13.6), 64 x 4096 x 1024 5.2
// (5.1), 128 x 2304 x 768 6.8 (4.5), 128 x 1000 x 8000 10.2 (20.0).
double gemm_fp8_tokens_cost(const Fp8Gemm& g, int nkb) {
  const int nt = rows_of_tile(g.M);
  const long long tiles = tiles_of(g, nt);
  const int cluster = cluster_of(tiles, nt, nkb), room = (nt == 128 ? 1 : 2) * num_sms();
  const long long waves = (tiles * cluster + room - 1) / room;
  return 2.6 + 0.03 * nt + (0.3 + 0.0016 * nt) * ((nkb + cluster - 1) / cluster) * waves;
}

elasto_fp8_tile gemm_fp8_tokens_tile(const Fp8Gemm& g, int nkb) {
  const int nt = rows_of_tile(g.M);
  return {nt, BM, 0, cluster_of(tiles_of(g, nt), nt, nkb)};
}

elasto_status gemm_fp8_tokens_launch(const Fp8Gemm& g, cudaStream_t s) {
  const int nt = rows_of_tile(g.M), nkb = static_cast<int>((g.K + BK - 1LL) / BK);
  const long long tiles = tiles_of(g, nt);
  const int cluster = cluster_of(tiles, nt, nkb);
  CUtensorMap tw, ta;
  if (tiles * cluster > 0x7fffffffLL || !encode_tmap_8(&tw, g.W, g.K, g.N, g.ldw, BM) ||
      !encode_tmap_8(&ta, g.A, g.K, g.M, g.lda, nt)) {
    set_error("elasto_op_gemm_fp8: cuTensorMapEncodeTiled failed (alignment or size)");
    return ELASTO_ERR_UNSUPPORTED;
  }
  const unsigned t = static_cast<unsigned>(tiles);
  cudaError_t e;
  if (nt == 16)
    e = launch_epi<16>(g, tw, ta, nkb, cluster, t, s);
  else if (nt == 32)
    e = launch_epi<32>(g, tw, ta, nkb, cluster, t, s);
  else if (nt == 64)
    e = launch_epi<64>(g, tw, ta, nkb, cluster, t, s);
  else
    e = launch_epi<128>(g, tw, ta, nkb, cluster, t, s);
  ELASTO_CUDA_TRY(e);
  return ELASTO_OK;
}

}  // namespace elasto
