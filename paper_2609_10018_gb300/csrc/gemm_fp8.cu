// Product of e4m3 rows with e4m3 weights, both with fp32 scales for blocks of 128:
//   out[m, n] = epi( sum_b as[b, m] ws[n / 128, b] sum_{k in block b} A[m, k] W[n, k] + bias[n] ).
//
// A 64 x 64 tile per CTA; each block of 128 columns is staged in shared memory as
// fp32 and summed in fp32, then scaled into the tile's sums.
#include "act.cuh"
#include "common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int T = 64, BK = 32, SCALE_BLOCK = 128;

__device__ __forceinline__ float e4m3_value(uint8_t v) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(v)));
  return __low2float(*reinterpret_cast<__half2*>(&h));
}

__global__ void __launch_bounds__(256) gemm_fp8_kernel(Fp8Gemm g) {
  __shared__ float sa[T][BK + 1], sw[T][BK + 1];
  pdl_wait();
  pdl_trigger();
  const int tiles_n = (g.N + T - 1) / T;
  const int m0 = static_cast<int>(blockIdx.x / tiles_n) * T, n0 = static_cast<int>(blockIdx.x % tiles_n) * T;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int nkb = (g.K + SCALE_BLOCK - 1) / SCALE_BLOCK;
  float acc[4][4] = {};
  for (int b = 0; b < nkb; ++b) {
    float part[4][4] = {};
    for (int k0 = b * SCALE_BLOCK; k0 < min(g.K, (b + 1) * SCALE_BLOCK); k0 += BK) {
      __syncthreads();
      for (int i = threadIdx.x; i < T * BK; i += 256) {
        const int r = i / BK, k = i % BK;
        sa[r][k] = m0 + r < g.M && k0 + k < g.K ? e4m3_value(g.A[static_cast<size_t>(m0 + r) * g.lda + k0 + k]) : 0.0f;
        sw[r][k] = n0 + r < g.N && k0 + k < g.K ? e4m3_value(g.W[static_cast<size_t>(n0 + r) * g.ldw + k0 + k]) : 0.0f;
      }
      __syncthreads();
#pragma unroll 8
      for (int k = 0; k < BK; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) part[i][j] = fmaf(sa[ty * 4 + i][k], sw[tx + 16 * j][k], part[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = m0 + ty * 4 + i;
      const float as = m < g.M ? g.a_scale[static_cast<size_t>(b) * g.lds + m] : 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int n = n0 + tx + 16 * j;
        if (m < g.M && n < g.N)
          acc[i][j] = fmaf(part[i][j], as * g.w_scale[static_cast<size_t>(n / SCALE_BLOCK) * nkb + b], acc[i][j]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty * 4 + i, n = n0 + tx + 16 * j;
      if (m >= g.M || n >= g.N) continue;
      const size_t at = static_cast<size_t>(m) * g.ldo + n;
      const float y = acc[i][j] + (g.bias ? g.bias[n] : 0.0f);
      if (g.epi == EPI_BIAS_BF16) static_cast<bf16*>(g.out)[at] = __float2bfloat16_rn(y);
      if (g.epi == EPI_BIAS_GELU_BF16) static_cast<bf16*>(g.out)[at] = __float2bfloat16_rn(gelu(y));
      if (g.epi == EPI_BIAS_F32) static_cast<float*>(g.out)[at] = y;
      if (g.epi == EPI_BIAS_RESID_F32) static_cast<float*>(g.out)[at] += y;
    }
}

}  // namespace

elasto_status gemm_fp8_launch(const Fp8Gemm& g, cudaStream_t s) {
  const long long tiles = ((g.M + T - 1LL) / T) * ((g.N + T - 1LL) / T);
  if (tiles > 0x7fffffffLL) {
    set_error("elasto_op_gemm_fp8: output too large");
    return ELASTO_ERR_UNSUPPORTED;
  }
  ELASTO_CUDA_TRY(launch_pdl(gemm_fp8_kernel, dim3(static_cast<unsigned>(tiles)), dim3(256), 0, s, g));
  return ELASTO_OK;
}

}  // namespace elasto
