// Norms of queries and keys for each head, with the position rotation and the
// write to the K/V cache in the same pass:
//   y = x * rsqrt(mean(x^2) + eps) * gain,  pairs (a, b) -> (a c - b s, b c + a s).
//
// Bound by memory: q, k (and v) are read and written once, everything between in
// fp32 registers. A head lies in LANES = head_dim / 8 lanes, rounded up to a power
// of two, 16 bytes each; a warp holds 32 / LANES heads of one row at a time and
// walks over the row's heads. All of them turn by the same angles, so a lane's
// cosines, sines and gains are read once a row. The partner channel of the
// half-split form is rot_dim / 16 lanes away (rot_dim / 2 is a multiple of 8).
#include "common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

template <bool BF>
__device__ __forceinline__ void unpack8(const uint4& w, float (&v)[8]) {
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = BF ? make_float2(__uint_as_float(ws[j] << 16), __uint_as_float(ws[j] & 0xffff0000u))
                        : __half22float2(*reinterpret_cast<const __half2*>(&ws[j]));
    v[2 * j] = f.x;
    v[2 * j + 1] = f.y;
  }
}
template <bool BF>
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = BF ? pack_bf16x2(v[2 * j], v[2 * j + 1]) : pack_f16x2(v[2 * j], v[2 * j + 1]);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// chunks: warps that share a row, each taking every chunks-th group of heads.
template <bool BF, int LANES, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS)
    qk_norm_rope_kernel(const __grid_constant__ elasto_qk_norm_rope_args a, int chunks, int* status) {
  pdl_wait();
  pdl_trigger();
  constexpr int HPW = 32 / LANES;
  const int lane = threadIdx.x & 31, l = lane % LANES, sub = lane / LANES;
  const long long unit = static_cast<long long>(blockIdx.x) * WARPS + (threadIdx.x >> 5);
  const int row = static_cast<int>(unit / chunks), chunk = static_cast<int>(unit % chunks);
  if (row >= a.rows) return;
  const int e = 8 * l;  // first channel of this lane
  const bool on = e < a.head_dim, turns = e < a.rot_dim;
  const int half = a.rot_dim / 2;

  float c[8], s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) c[j] = 1.0f, s[j] = 0.0f;
  if (a.rot_dim > 0) {
    const int pos = a.positions[row];
    if (pos < 0 || pos >= a.n_positions) {
      if (lane == 0) record_status(status, ELASTO_ERR_INVALID_ARG);
      return;
    }
    if (turns) {
      const float* t = a.cos_sin + static_cast<size_t>(pos) * a.rot_dim;
      if constexpr (INTERLEAVED) {  // pairs e / 2 .. e / 2 + 3
        const float4 cc = *reinterpret_cast<const float4*>(t + e / 2);
        const float4 ss = *reinterpret_cast<const float4*>(t + half + e / 2);
        c[0] = cc.x, c[1] = cc.y, c[2] = cc.z, c[3] = cc.w;
        s[0] = ss.x, s[1] = ss.y, s[2] = ss.z, s[3] = ss.w;
      } else {
        const int p = e < half ? e : e - half;
        const float sign = e < half ? -1.0f : 1.0f;
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          const float4 cc = *reinterpret_cast<const float4*>(t + p + j);
          const float4 ss = *reinterpret_cast<const float4*>(t + half + p + j);
          c[j] = cc.x, c[j + 1] = cc.y, c[j + 2] = cc.z, c[j + 3] = cc.w;
          s[j] = sign * ss.x, s[j + 1] = sign * ss.y, s[j + 2] = sign * ss.z, s[j + 3] = sign * ss.w;
        }
      }
    }
  }
  int slot = row;
  if (a.slots && a.heads_k > 0) {
    slot = a.slots[row];
    if (slot >= a.n_slots) {
      if (lane == 0) record_status(status, ELASTO_ERR_INVALID_ARG);
      return;
    }
  }
  const float inv_d = 1.0f / static_cast<float>(a.head_dim);
  const int partner = lane - l + (e < half ? l + half / 8 : l - half / 8);

  // heads [0, n) of one of q and k
  auto heads = [&](const uint16_t* x, long long x_head, uint16_t* y, long long y_head, const float* gain, int n) {
    float g[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = 1.0f;
    if (gain && on) {
      const float4 g0 = *reinterpret_cast<const float4*>(gain + e), g1 = *reinterpret_cast<const float4*>(gain + e + 4);
      g[0] = g0.x, g[1] = g0.y, g[2] = g0.z, g[3] = g0.w, g[4] = g1.x, g[5] = g1.y, g[6] = g1.z, g[7] = g1.w;
    }
#pragma unroll 2
    for (int h0 = chunk * HPW; h0 < n; h0 += chunks * HPW) {
      const int h = h0 + sub;
      const bool mine = on && h < n;
      float v[8] = {};
      if (mine) unpack8<BF>(__ldcs(reinterpret_cast<const uint4*>(x + h * x_head + e)), v);
      float ss = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(v[j], v[j], ss);
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float r = rsqrtf(fmaf(ss, inv_d, a.eps));
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= r * g[j];
      if constexpr (INTERLEAVED) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x0 = v[2 * j], x1 = v[2 * j + 1];
          v[2 * j] = fmaf(x0, c[j], -x1 * s[j]);
          v[2 * j + 1] = fmaf(x1, c[j], x0 * s[j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float o = __shfl_sync(0xffffffffu, v[j], partner & 31);
          if (turns) v[j] = fmaf(v[j], c[j], o * s[j]);
        }
      }
      if (mine) *reinterpret_cast<uint4*>(y + h * y_head + e) = pack8<BF>(v);
    }
  };
  auto at = [](const void* p, long long r, long long row_stride) { return static_cast<const uint16_t*>(p) + r * row_stride; };
  auto to = [](void* p, long long r, long long row_stride) { return static_cast<uint16_t*>(p) + r * row_stride; };
  if (a.heads_q > 0) heads(at(a.q, row, a.q_row), a.q_head, to(a.q_out, row, a.q_out_row), a.q_out_head, a.q_gain, a.heads_q);
  if (a.heads_k > 0 && slot >= 0) {
    heads(at(a.k, row, a.k_row), a.k_head, to(a.k_out, slot, a.k_out_row), a.k_out_head, a.k_gain, a.heads_k);
    if (a.v) {
      const uint16_t* x = at(a.v, row, a.v_row);
      uint16_t* y = to(a.v_out, slot, a.v_out_row);
      for (int h = chunk * HPW + sub; h < a.heads_k; h += chunks * HPW)
        if (on) *reinterpret_cast<uint4*>(y + h * a.v_out_head + e) = __ldcs(reinterpret_cast<const uint4*>(x + h * a.v_head + e));
    }
  }
}

template <int LANES>
cudaError_t launch(const elasto_qk_norm_rope_args& a, int* status, cudaStream_t s) {
  // as many warps a row as leave each at least one group of heads, where the rows alone are few
  const int groups = (a.heads_q + a.heads_k + 32 / LANES - 1) / (32 / LANES);
  const long long wanted = 32LL * (num_sms() > 0 ? num_sms() : 152);
  int chunks = static_cast<int>(wanted / a.rows);
  chunks = chunks < 1 ? 1 : chunks > groups ? groups : chunks;
  const long long units = static_cast<long long>(a.rows) * chunks;
  const dim3 grid(static_cast<unsigned>((units + WARPS - 1) / WARPS)), block(THREADS);
  const bool bf = a.dtype == ELASTO_BF16;
  if (a.interleaved)
    return bf ? launch_pdl(qk_norm_rope_kernel<true, LANES, true>, grid, block, 0, s, a, chunks, status)
              : launch_pdl(qk_norm_rope_kernel<false, LANES, true>, grid, block, 0, s, a, chunks, status);
  return bf ? launch_pdl(qk_norm_rope_kernel<true, LANES, false>, grid, block, 0, s, a, chunks, status)
            : launch_pdl(qk_norm_rope_kernel<false, LANES, false>, grid, block, 0, s, a, chunks, status);
}

}  // namespace

cudaError_t qk_norm_rope_launch(const elasto_qk_norm_rope_args& a, int* status, cudaStream_t s) {
  const int lanes = a.head_dim / 8;
  if (lanes <= 1) return launch<1>(a, status, s);
  if (lanes <= 2) return launch<2>(a, status, s);
  if (lanes <= 4) return launch<4>(a, status, s);
  if (lanes <= 8) return launch<8>(a, status, s);
  if (lanes <= 16) return launch<16>(a, status, s);
  return launch<32>(a, status, s);
}

}  // namespace elasto
