// Rows to e4m3 with an fp32 scale for each block of 128 columns.
//
//   a = max(max |x|, 2^-100),  scale = a / 448,  q = rn_e4m3(x * (448 / a))
//
// in IEEE fp32 operations (two divisions a block, a multiplication a value), so
// the result is a function of the block alone. 448 is the largest e4m3; x * (448 /
// a) can pass it by an fp32 rounding only, which rounds back to 448. The floor
// 2^-100 keeps 448 / a finite for blocks of zeros and subnormals.
//
// Sixteen lanes hold a block: eight values each, read as 16 bytes (fp32: 32)
// and written as 8; the maximum goes round by four shuffles. Maxima are taken
// over the bits of |x| as integers, which orders numbers as numbers and puts
// infinities and then NaN above them: a NaN reaches the scale.
#include "common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int THREADS = 256, UNROLL = 4;
constexpr int PER_CTA = THREADS / 16 * UNROLL;  // blocks of 128 columns

// Two values to e4m3 (round to nearest even, saturating), the first in the low byte.
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int TYPE>
__device__ __forceinline__ float value_at(const void* x, size_t i) {
  if constexpr (TYPE == ELASTO_F32) return static_cast<const float*>(x)[i];
  if constexpr (TYPE == ELASTO_BF16) return __bfloat162float(static_cast<const bf16*>(x)[i]);
  return __half2float(static_cast<const __half*>(x)[i]);
}

template <int TYPE>
__device__ __forceinline__ float2 pair_at(uint32_t w) {
  if constexpr (TYPE == ELASTO_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// WIDE: rows of x start on 16 bytes and those of q on 8.
template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(THREADS)
    quantize_kernel(const void* __restrict__ x, long long ldx, uint8_t* __restrict__ q, long long ldq,
                    float* __restrict__ scale, long long lds, unsigned total, unsigned nb, int cols) {
  pdl_wait();
  pdl_trigger();
  const int l = threadIdx.x & 15;
  const unsigned first = blockIdx.x * PER_CTA + (threadIdx.x >> 4);
  float v[UNROLL][8];
  unsigned row[UNROLL], blk[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const unsigned i = first + u * (THREADS / 16);
    row[u] = i / nb;
    blk[u] = i - row[u] * nb;
    const int c = static_cast<int>(blk[u]) * 128 + l * 8;
    const size_t at = static_cast<size_t>(row[u]) * ldx + c;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[u][j] = 0.0f;
    if (i < total) {
      if (WIDE && c + 8 <= cols) {
        if constexpr (TYPE == ELASTO_F32) {
          const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(x) + at);
          const float4 a = __ldcs(p), b = __ldcs(p + 1);
          v[u][0] = a.x, v[u][1] = a.y, v[u][2] = a.z, v[u][3] = a.w;
          v[u][4] = b.x, v[u][5] = b.y, v[u][6] = b.z, v[u][7] = b.w;
        } else {
          const uint4 w = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + at));
          const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 f = pair_at<TYPE>(ws[j]);
            v[u][2 * j] = f.x;
            v[u][2 * j + 1] = f.y;
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < cols) v[u][j] = value_at<TYPE>(x, at + j);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const unsigned i = first + u * (THREADS / 16);
    uint32_t top = __float_as_uint(7.888609052210118e-31f);  // 2^-100
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[u][j]) & 0x7fffffffu);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (i >= total) continue;
    const float a = __uint_as_float(top), inv = __fdiv_rn(448.0f, a);
    const int c = static_cast<int>(blk[u]) * 128 + l * 8;
    if (l == 0) scale[static_cast<size_t>(blk[u]) * lds + row[u]] = __fdiv_rn(a, 448.0f);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = pack_e4m3x2(__fmul_rn(v[u][2 * j], inv), __fmul_rn(v[u][2 * j + 1], inv));
    uint8_t* const out = q + static_cast<size_t>(row[u]) * ldq + c;
    if (WIDE && c + 8 <= cols) {
      *reinterpret_cast<uint2*>(out) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < cols) out[j] = static_cast<uint8_t>(w[j >> 1] >> (8 * (j & 1)));
    }
  }
}

template <int TYPE>
cudaError_t launch(const void* x, long long ldx, uint8_t* q, long long ldq, float* scale, long long lds, int rows,
                   int cols, cudaStream_t s) {
  const unsigned nb = static_cast<unsigned>((cols + 127LL) / 128), total = static_cast<unsigned>(rows) * nb;
  const dim3 grid((total + PER_CTA - 1) / PER_CTA), block(THREADS);
  const long long size = TYPE == ELASTO_F32 ? 4 : 2;
  const bool wide = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx * size % 16 == 0 &&
                    reinterpret_cast<uintptr_t>(q) % 8 == 0 && ldq % 8 == 0;
  return wide ? launch_pdl(quantize_kernel<TYPE, true>, grid, block, 0, s, x, ldx, q, ldq, scale, lds, total, nb, cols)
              : launch_pdl(quantize_kernel<TYPE, false>, grid, block, 0, s, x, ldx, q, ldq, scale, lds, total, nb, cols);
}

}  // namespace

cudaError_t quantize_fp8_launch(const void* x, int x_type, long long ldx, uint8_t* q, long long ldq, float* scale,
                                long long lds, int rows, int cols, cudaStream_t s) {
  if (x_type == ELASTO_F32) return launch<ELASTO_F32>(x, ldx, q, ldq, scale, lds, rows, cols, s);
  if (x_type == ELASTO_BF16) return launch<ELASTO_BF16>(x, ldx, q, ldq, scale, lds, rows, cols, s);
  return launch<ELASTO_F16>(x, ldx, q, ldq, scale, lds, rows, cols, s);
}

}  // namespace elasto
