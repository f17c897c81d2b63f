// Attention in a sliding window, the first tokens staying visible (the
// definition is at elasto_op_window_attention): a warp for each query and head,
// one visible key at a time with the running maximum and sum of the softmax.
#include "common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

template <bool BF>
__device__ __forceinline__ float value(const void* p, long long i) {
  const uint16_t b = static_cast<const uint16_t*>(p)[i];
  return BF ? __uint_as_float(static_cast<uint32_t>(b) << 16) : __half2float(__ushort_as_half(b));
}

template <bool BF>
__global__ void __launch_bounds__(256) window_attention_kernel(const __grid_constant__ elasto_window_attention_args a) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long unit = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int head = static_cast<int>(unit % a.heads), i = static_cast<int>(unit / a.heads % a.max_queries);
  const int b = static_cast<int>(unit / a.heads / a.max_queries);
  if (b >= a.batch) return;
  long long q0 = static_cast<long long>(b) * a.max_queries, nq = a.max_queries;
  if (a.q_start) {
    q0 = min(max(static_cast<long long>(a.q_start[b]), 0LL), a.q_rows);
    nq = min(min(static_cast<long long>(a.q_start[b + 1]), a.q_rows) - q0, nq);
  }
  long long k0 = 0, nk = a.max_keys;
  if (a.kv_start) {
    k0 = min(max(static_cast<long long>(a.kv_start[b]), 0LL), a.kv_rows);
    nk = min(min(static_cast<long long>(a.kv_start[b + 1]), a.kv_rows) - k0, nk);
  } else if (a.kv_len) {
    nk = min(static_cast<long long>(a.kv_len[b]), nk);
  }
  if (i >= nq) return;
  nk = max(nk, 0LL);
  const long long p = nk - nq + i, w = a.window < 0 ? a.max_keys : a.window;
  const int d = a.head_dim, kvh = head / (a.heads / a.heads_kv);
  float q[4], o[4] = {}, m = -INFINITY, sum = 0.0f;
  for (int t = 0; t < 4; ++t)
    q[t] = lane + 32 * t < d ? value<BF>(a.q, (q0 + i) * a.q_row + head * a.q_head + lane + 32 * t) * a.scale : 0.0f;
  for (long long j = 0; p >= 0 && j < nk; ++j) {
    const bool near = j >= p - w && j <= p + w;
    const bool seen = a.causal ? j <= p && (near || j < a.sinks) : near || j < a.sinks || p < a.sinks;
    if (!seen) continue;
    const long long kr = b * (a.kv_start ? 0LL : a.k_batch) + (k0 + j) * a.k_row + kvh * a.k_head;
    const long long vr = b * (a.kv_start ? 0LL : a.v_batch) + (k0 + j) * a.v_row + kvh * a.v_head;
    float x = 0.0f;
    for (int t = 0; t < 4; ++t)
      if (lane + 32 * t < d) x = fmaf(q[t], value<BF>(a.k, kr + lane + 32 * t), x);
    for (int s = 16; s > 0; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    const float top = fmaxf(m, x), keep = expf(m - top), e = expf(x - top);
    m = top;
    sum = fmaf(sum, keep, e);
    for (int t = 0; t < 4; ++t)
      if (lane + 32 * t < d) o[t] = fmaf(o[t], keep, e * value<BF>(a.v, vr + lane + 32 * t));
  }
  const bool any = p >= 0 && nk > 0;
  for (int t = 0; t < 4; ++t) {
    const float y = any ? o[t] / sum : 0.0f;
    const long long at = (q0 + i) * a.out_row + head * a.out_head + lane + 32 * t;
    if (lane + 32 * t < d) static_cast<uint16_t*>(a.out)[at] = BF ? __bfloat16_as_ushort(__float2bfloat16_rn(y)) : __half_as_ushort(__float2half_rn(y));
  }
}

}  // namespace

elasto_status window_attention_launch(const elasto_window_attention_args& a, int* status, cudaStream_t s) {
  const long long units = static_cast<long long>(a.batch) * a.max_queries * a.heads;
  if (units > 8LL * 0x7fffffffLL) {
    set_error("elasto_op_window_attention: too many queries");
    return ELASTO_ERR_UNSUPPORTED;
  }
  const dim3 grid(static_cast<unsigned>((units + 7) / 8));
  ELASTO_CUDA_TRY(a.dtype == ELASTO_BF16 ? launch_pdl(window_attention_kernel<true>, grid, dim3(256), 0, s, a)
                                         : launch_pdl(window_attention_kernel<false>, grid, dim3(256), 0, s, a));
  return ELASTO_OK;
}

}  // namespace elasto
