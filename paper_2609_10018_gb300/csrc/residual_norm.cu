// The sum at a block's end and the norm before the next block, in one pass over the rows:
//   u = N_post(y),  s = x_factor x + y_scale gate u,  x_out = s,  z = N_pre(s) (1 + scale) + shift,
// z as rows of fp32, bf16 or f16 or, with a scale for each 128 columns, of e4m3.
#include <type_traits>

#include "common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int MAX_THREADS = 512, MAX_PIECES = 4, FEW_PIECES = 3, ROWS_THREADS = 128;
static_assert(8 * MAX_PIECES * MAX_THREADS >= 16384, "columns");

__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint32_t w, bool bf) {
  return bf ? make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u))
            : __half22float2(*reinterpret_cast<const __half2*>(&w));
}
__device__ __forceinline__ float unpack1(uint16_t w, bool bf) {
  return bf ? __uint_as_float(static_cast<uint32_t>(w) << 16) : __half2float(__ushort_as_half(w));
}
__device__ __forceinline__ uint32_t pack2(float a, float b, bool bf) { return bf ? pack_bf16x2(a, b) : pack_f16x2(a, b); }

// 32 bytes at once (aligned to them).
__device__ __forceinline__ void load32(const void* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store32(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

struct Args {
  elasto_residual_norm_args u;
  int log_threads;  // of a row: 8 to MAX_THREADS
  int* status;
};

// A lane's eight values of a piece as they lie in memory. VEC: eight neighbours; else each `step` columns from the last.
template <bool F32, bool VEC>
struct Raw {
  uint32_t w[F32 ? 8 : VEC ? 4 : 8];

  __device__ __forceinline__ void load(const void* row, int col, int step, int cols) {
    if constexpr (VEC) {
      if (col + 8 <= cols) {
        if constexpr (F32) {
          load32(static_cast<const float*>(row) + col, w);
        } else {
          const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(row) + col);
          w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
        }
        return;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = col + j < cols;
        if constexpr (F32) {
          w[j] = in ? static_cast<const uint32_t*>(row)[col + j] : 0u;
        } else {
          const uint32_t v = in ? static_cast<const uint16_t*>(row)[col + j] : 0u;
          w[j / 2] = j & 1 ? w[j / 2] | v << 16 : v;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = col + j * step < cols;
        if constexpr (F32)
          w[j] = in ? static_cast<const uint32_t*>(row)[col + j * step] : 0u;
        else
          w[j] = in ? static_cast<const uint16_t*>(row)[col + j * step] : 0u;
      }
    }
  }
  __device__ __forceinline__ void values(bool bf, float (&v)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (F32) {
        v[j] = __uint_as_float(w[j]);
      } else if constexpr (VEC) {
        const float2 p = unpack2(w[j / 2], bf);
        v[j] = j & 1 ? p.y : p.x;
      } else {
        v[j] = unpack1(static_cast<uint16_t>(w[j]), bf);
      }
    }
  }
};

// Eight values of a vector over the columns (fp32), or of a modulation's row.
template <bool VEC>
__device__ __forceinline__ void load_vector(const void* p, int type, int col, int step, int cols, float (&v)[8]) {
  if (type == ELASTO_F32) {
    if (VEC && col + 8 <= cols) {
      const float4 a = reinterpret_cast<const float4*>(static_cast<const float*>(p) + col)[0];
      const float4 b = reinterpret_cast<const float4*>(static_cast<const float*>(p) + col)[1];
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = col + j * step < cols ? static_cast<const float*>(p)[col + j * step] : 0.0f;
    }
  } else {
    Raw<false, VEC> r;
    r.load(p, col, step, cols);
    r.values(type == ELASTO_BF16, v);
  }
}

template <bool VEC>
__device__ __forceinline__ void store_row(void* row, int type, int col, int step, int cols, const float (&v)[8]) {
  if (type == ELASTO_F32) {
    if (VEC && col + 8 <= cols) {
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[j]);
      store32(static_cast<float*>(row) + col, w);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + j * step < cols) static_cast<float*>(row)[col + j * step] = v[j];
    }
    return;
  }
  const bool bf = type == ELASTO_BF16;
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = pack2(v[2 * j], v[2 * j + 1], bf);
  if (VEC && col + 8 <= cols) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(row) + col) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + j * step < cols) static_cast<uint16_t*>(row)[col + j * step] = static_cast<uint16_t>(w[j / 2] >> 16 * (j & 1));
  }
}

// T threads have a row, in pieces of eight values: a warp's (or, with fewer threads, the row's) lanes hold 8 W
// neighbouring columns together, W = min(T, 32), lane l the columns 8 l to 8 l + 7 of them (VEC) or l + W j.
template <bool X32, bool Y32, bool VEC, int PIECES>
__global__ void __launch_bounds__(MAX_THREADS)
    residual_norm_kernel(const __grid_constant__ Args args) {
  pdl_wait();
  pdl_trigger();
  const elasto_residual_norm_args& a = args.u;
  __shared__ float partial[4][MAX_THREADS / 32];
  const int T = 1 << args.log_threads, W = T < 32 ? T : 32;
  const int t = threadIdx.x & (T - 1), l = t & (W - 1), warp = t >> 5, lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * (blockDim.x >> args.log_threads) + (threadIdx.x >> args.log_threads);
  const bool on = row < a.rows;
  // (lanes of rows past the last go along with the last row, for the shuffles, and store nothing)
  const long long r = on ? row : a.rows - 1;
  const int step = VEC ? 1 : W, first = (t & ~31) * 8 + (VEC ? 8 * l : l);  // columns first + 8 T i (+ step j)
  int group = 0;
  if (a.group) group = a.group[r];

  Raw<X32, VEC> rx[PIECES];
  Raw<Y32, VEC> ry[PIECES];
  const uint8_t* const x = static_cast<const uint8_t*>(a.x) + r * a.x_row * (X32 ? 4 : 2);
  const uint8_t* const y = static_cast<const uint8_t*>(a.y) + r * a.y_row * (Y32 ? 4 : 2);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    rx[i].load(x, first + 8 * T * i, step, a.cols);
    if (a.y) ry[i].load(y, first + 8 * T * i, step, a.cols);
  }
  bool live = on;
  if (a.groups > 0 && static_cast<unsigned>(group) >= static_cast<unsigned>(a.groups)) {
    if (on && t == 0) record_status(args.status, ELASTO_ERR_INVALID_ARG);
    live = false, group = 0;
  }
  const long long mod_at = static_cast<long long>(group) * a.mod_row * (a.mod_type == ELASTO_F32 ? 4 : 2);
  auto modulation = [&](const void* p) { return static_cast<const uint8_t*>(p) + mod_at; };

  // The sum over the row's threads; `slot`: a place in shared memory for each of them.
  auto row_sum = [&](float v, int slot) {
    for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (T > 32) {
      if (lane == 0) partial[slot][warp] = v;
      __syncthreads();
      v = 0.0f;
      for (int w = 0; w < T / 32; ++w) v += partial[slot][w];
    }
    return v;
  };
  const float inv_n = 1.0f / static_cast<float>(a.cols);
  auto column = [&](int i, int j) { return first + 8 * T * i + step * j; };
  // v -> (v - mean) / sqrt(var + eps), or v / sqrt(mean v^2 + eps), times gain plus bias
  auto norm = [&](float (&v)[PIECES][8], int kind, const float* gain, const float* bias, int slot) {
    if (kind == ELASTO_NORM_NONE) return;
    float mean = 0.0f, sum = 0.0f;
    if (kind == ELASTO_NORM_LAYER) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += v[i][j];  // (columns past the last hold 0)
      mean = row_sum(sum, slot) * inv_n;
    }
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] -= mean;
        if (column(i, j) < a.cols) sum = fmaf(v[i][j], v[i][j], sum);
      }
    const float rs = rsqrtf(fmaf(row_sum(sum, slot + 1), inv_n, a.eps));
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float g[8];
      if (gain) load_vector<VEC>(gain, ELASTO_F32, column(i, 0), step, a.cols, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= gain ? rs * g[j] : rs;
      if (bias) {
        load_vector<VEC>(bias, ELASTO_F32, column(i, 0), step, a.cols, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += g[j];
      }
    }
  };

  float v[PIECES][8];
  if (a.y) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) ry[i].values(a.y_type == ELASTO_BF16, v[i]);
    norm(v, a.post_norm, a.post_gain, a.post_bias, 0);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float g[8], xs[8];
      if (a.y_scale) {
        load_vector<VEC>(a.y_scale, ELASTO_F32, column(i, 0), step, a.cols, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
      }
      if (a.gate) {
        load_vector<VEC>(modulation(a.gate), a.mod_type, column(i, 0), step, a.cols, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
      }
      rx[i].values(a.x_type == ELASTO_BF16, xs);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = fmaf(a.x_factor, xs[j], v[i][j]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      rx[i].values(a.x_type == ELASTO_BF16, v[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= a.x_factor;
    }
  }
  if (a.x_out && live) {
    uint8_t* const out = static_cast<uint8_t*>(a.x_out) + r * a.x_out_row * (X32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) store_row<VEC>(out, a.x_type, column(i, 0), step, a.cols, v[i]);
  }
  if (!a.z) return;
#pragma unroll
  for (int i = 0; i < PIECES; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (column(i, j) >= a.cols) v[i][j] = 0.0f;
  norm(v, a.pre_norm, a.pre_gain, a.pre_bias, 2);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    float g[8];
    if (a.scale) {
      load_vector<VEC>(modulation(a.scale), a.mod_type, column(i, 0), step, a.cols, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = fmaf(v[i][j], g[j], v[i][j]);
    }
    if (a.shift) {
      load_vector<VEC>(modulation(a.shift), a.mod_type, column(i, 0), step, a.cols, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] += g[j];
    }
  }
  if (a.z_type != ELASTO_E4M3) {
    if (!live) return;
    uint8_t* const out = static_cast<uint8_t*>(a.z) + r * a.z_row * (a.z_type == ELASTO_F32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) store_row<VEC>(out, a.z_type, column(i, 0), step, a.cols, v[i]);
    return;
  }
  // Blocks of 128 columns: 16 lanes' eight values (VEC, or rows of 16 threads), or 32 lanes' first and last four.
  uint8_t* const out = static_cast<uint8_t*>(a.z) + r * a.z_row;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    uint32_t top[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (column(i, j) < a.cols) top[j >> 2] = max(top[j >> 2], __float_as_uint(v[i][j]) & 0x7fffffffu);
    const bool two = !VEC && W == 32;
    if (!two) top[0] = max(top[0], top[1]);
    for (int o = two ? 16 : 8; o > 0; o >>= 1) {
      top[0] = max(top[0], __shfl_xor_sync(0xffffffffu, top[0], o));
      if (two) top[1] = max(top[1], __shfl_xor_sync(0xffffffffu, top[1], o));
    }
    if (!two) top[1] = top[0];
    if (!live) continue;
    const float a0 = __uint_as_float(max(top[0], 0x0d800000u)), a1 = __uint_as_float(max(top[1], 0x0d800000u));  // 2^-100 at least
    const float i0 = __fdiv_rn(448.0f, a0), i1 = two ? __fdiv_rn(448.0f, a1) : i0;
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float m = j < 2 ? i0 : i1;
      c[j] = pack_e4m3x2(v[i][2 * j] * m, v[i][2 * j + 1] * m);
    }
    const int col = column(i, 0);
    const int block = ((t & ~31) * 8 + 8 * T * i) / 128 + (VEC ? l >> 4 : 0);
    if ((VEC ? (l & 15) == 0 : l == 0) && block * 128 < a.cols) {
      a.z_scale[block * a.z_scale_row + r] = __fdiv_rn(a0, 448.0f);
      if (two && (block + 1) * 128 < a.cols) a.z_scale[(block + 1) * a.z_scale_row + r] = __fdiv_rn(a1, 448.0f);
    }
    if (VEC && col + 8 <= a.cols) {
      *reinterpret_cast<uint2*>(out + col) = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (column(i, j) < a.cols) out[column(i, j)] = static_cast<uint8_t>(c[j / 2] >> 8 * (j & 1));
    }
  }
}

template <bool X32, bool Y32, bool VEC>
cudaError_t launch(const Args& a, int pieces, cudaStream_t s) {
  const int block = a.log_threads <= 5 ? ROWS_THREADS : 1 << a.log_threads, rows = block >> a.log_threads;
  const dim3 grid((static_cast<unsigned>(a.u.rows) + rows - 1) / rows);
  switch (pieces) {
    case 1: return launch_pdl(residual_norm_kernel<X32, Y32, VEC, 1>, grid, dim3(block), 0, s, a);
    case 2: return launch_pdl(residual_norm_kernel<X32, Y32, VEC, 2>, grid, dim3(block), 0, s, a);
    case 3: return launch_pdl(residual_norm_kernel<X32, Y32, VEC, 3>, grid, dim3(block), 0, s, a);
    default: return launch_pdl(residual_norm_kernel<X32, Y32, VEC, 4>, grid, dim3(block), 0, s, a);
  }
}

}  // namespace

cudaError_t residual_norm_launch(const elasto_residual_norm_args& u, int* status, cudaStream_t s) {
  // rows of `row` values of a type that are read and written wide
  auto wide = [](const void* p, long long row, int type) {
    const int size = type == ELASTO_F32 ? 4 : type == ELASTO_E4M3 ? 1 : 2;
    return !p || (reinterpret_cast<uintptr_t>(p) % (8 * size) == 0 && row % 8 == 0);
  };
  auto vector = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  bool vec = wide(u.x, u.x_row, u.x_type) && wide(u.y, u.y_row, u.y_type) && wide(u.x_out, u.x_out_row, u.x_type) && wide(u.z, u.z_row, u.z_type);
  for (const void* p : {static_cast<const void*>(u.post_gain), static_cast<const void*>(u.post_bias), static_cast<const void*>(u.y_scale),
                        static_cast<const void*>(u.pre_gain), static_cast<const void*>(u.pre_bias)})
    vec = vec && vector(p);
  for (const void* p : {u.gate, u.shift, u.scale}) vec = vec && (!p || (vector(p) && u.mod_row % 8 == 0));
  Args a{u, u.z && u.z_type == ELASTO_E4M3 ? 4 : 3, status};  // (a block of 128 columns is 16 threads' at least)
  const int eights = (u.cols + 7) / 8;
  while (eights > FEW_PIECES << a.log_threads && (1 << a.log_threads) < MAX_THREADS) ++a.log_threads;
  const int pieces = (eights + (1 << a.log_threads) - 1) >> a.log_threads;
  const bool x32 = u.x_type == ELASTO_F32, y32 = u.y && u.y_type == ELASTO_F32;
  auto start = [&](auto x, auto y) {
    return vec ? launch<x.value, y.value, true>(a, pieces, s) : launch<x.value, y.value, false>(a, pieces, s);
  };
  const std::true_type yes;
  const std::false_type no;
  if (x32) return y32 ? start(yes, yes) : start(yes, no);
  return y32 ? start(no, yes) : start(no, no);
}

}  // namespace elasto
