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
//
// Bound by the bytes read and written once, and close behind by issue slots (75 %:
// the multiplications, conversions and shuffles of eight values a lane). 50432 x 768
// bf16: 21.4 us, 5.5 TB/s (of 6.8 measured for a copy); 41238 x 6904 fp32: 213 us, as
// fast as a copy. Two blocks a half warp keep enough loads in flight at 2048 threads an
// SM (four blocks 24.1 us, 1536 threads 22.6, CTAs of 256 22.1). Rows that start on any
// value are read and written value by value: 50000 x 769 bf16 51.7 us, 10000 x 6901 87.1 (x 768 21.0, x 6904 36.7).
#include "common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int THREADS = 128, UNROLL = 2, MIN_CTAS = 16;
constexpr int PER_CTA = THREADS / 16 * UNROLL;  // blocks of 128 columns

// Two values to e4m3 (round to nearest even, saturating), the first in the low byte.
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Bits of one 16-bit value (in the low half) as fp32.
template <int TYPE>
__device__ __forceinline__ float value_of(uint32_t bits) {
  if constexpr (TYPE == ELASTO_BF16) return __uint_as_float(bits << 16);
  return __half2float(__ushort_as_half(static_cast<unsigned short>(bits)));
}
template <int TYPE>
__device__ __forceinline__ float2 pair_of16(uint32_t w) {
  if constexpr (TYPE == ELASTO_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// A lane's eight values as they lie in memory.
template <int TYPE>
struct Eight {
  static constexpr bool f32 = TYPE == ELASTO_F32;
  uint32_t w[f32 ? 8 : 4];

  __device__ __forceinline__ void load_wide(const void* x, size_t at) {
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(x) + at * (f32 ? 4 : 2));
    const uint4 a = __ldcs(p);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    if constexpr (f32) {
      const uint4 b = __ldcs(p + 1);
      w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
  }
  // the first n of them, the others 0
  __device__ __forceinline__ void load_some(const void* x, size_t at, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (f32) {
        w[j] = j < n ? static_cast<const uint32_t*>(x)[at + j] : 0u;
      } else {
        const uint32_t v = j < n ? static_cast<const uint16_t*>(x)[at + j] : 0u;
        w[j / 2] = j & 1 ? w[j / 2] | v << 16 : v;
      }
    }
  }
  // the largest |value|'s bits: of fp32, or of the 16-bit type
  __device__ __forceinline__ uint32_t top() const {
    if constexpr (f32) {
      uint32_t t = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) t = max(t, w[j] & 0x7fffffffu);
      return t;
    } else {
      const uint32_t t = max_u16x2(max_u16x2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), max_u16x2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
      return max(t & 0xffffu, t >> 16);
    }
  }
  __device__ __forceinline__ uint2 codes(float inv) const {
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float2 v;
      if constexpr (f32)
        v = make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
      else
        v = pair_of16<TYPE>(w[j]);
      v = mul2(v, make_float2(inv, inv));
      c[j] = pack_e4m3x2(v.x, v.y);
    }
    return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
  }
};

// WIDE: rows of x start on 16 bytes and those of q on 8.
template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(THREADS, MIN_CTAS)
    quantize_kernel(const void* __restrict__ x, long long ldx, uint8_t* __restrict__ q, long long ldq,
                    float* __restrict__ scale, long long lds, unsigned total, Divisor nb, int cols) {
  pdl_wait();
  pdl_trigger();
  const int l = threadIdx.x & 15;
  const unsigned first = blockIdx.x * PER_CTA + (threadIdx.x >> 4);
  Eight<TYPE> v[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const unsigned i = first + u * (THREADS / 16), row = nb.quotient(i);
    const int c = static_cast<int>(i - row * nb.d) * 128 + l * 8, left = i < total ? cols - c : 0;
    const size_t at = static_cast<size_t>(row) * ldx + c;
    if (WIDE && left >= 8)
      v[u].load_wide(x, at);
    else
      v[u].load_some(x, at, left);
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const unsigned i = first + u * (THREADS / 16), row = nb.quotient(i), blk = i - row * nb.d;
    uint32_t top = v[u].top();
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (i >= total) continue;
    if constexpr (TYPE != ELASTO_F32) top = __float_as_uint(value_of<TYPE>(top));
    const float a = __uint_as_float(max(top, 0x0d800000u));  // 2^-100 at least
    const uint2 c8 = v[u].codes(__fdiv_rn(448.0f, a));
    const int c = static_cast<int>(blk) * 128 + l * 8;
    if (l == 0) scale[static_cast<size_t>(blk) * lds + row] = __fdiv_rn(a, 448.0f);
    uint8_t* const out = q + static_cast<size_t>(row) * ldq + c;
    if (WIDE && c + 8 <= cols) {
      *reinterpret_cast<uint2*>(out) = c8;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < cols) out[j] = static_cast<uint8_t>((j < 4 ? c8.x : c8.y) >> (8 * (j & 3)));
    }
  }
}

template <int TYPE>
cudaError_t launch(const void* x, long long ldx, uint8_t* q, long long ldq, float* scale, long long lds, int rows,
                   int cols, cudaStream_t s) {
  const Divisor nb(static_cast<unsigned>((cols + 127LL) / 128));
  const unsigned total = static_cast<unsigned>(rows) * nb.d;
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
