// What the two e4m3 products share.
#pragma once
#include "common.h"

namespace elasto {

template <int EPI>
__device__ __forceinline__ void fp8_store_one(void* out, long long at, float x) {
  if constexpr (EPI == EPI_BIAS_F32)
    static_cast<float*>(out)[at] = x;
  else if constexpr (EPI == EPI_BIAS_RESID_F32)
    static_cast<float*>(out)[at] += x;
  else
    static_cast<bf16*>(out)[at] = __float2bfloat16_rn(x);
}

// For few rows of A (gemm_fp8_tokens.cu), and its estimated microseconds (nkb: blocks of 128 of K).
double gemm_fp8_tokens_cost(const Fp8Gemm& g, int nkb);
elasto_fp8_tile gemm_fp8_tokens_tile(const Fp8Gemm& g, int nkb);
elasto_status gemm_fp8_tokens_launch(const Fp8Gemm& g, cudaStream_t s);
cudaError_t gemm_fp8_tokens_init_attributes();

}  // namespace elasto
