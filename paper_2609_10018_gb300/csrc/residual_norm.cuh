// The sum at a block's end and the norm before the next block, in one pass over the rows:
//   u = N_post(y),  s = x_factor x + y_scale gate u,  x_out = s,  z = N_pre(s) (1 + scale) + shift,
// z as rows of fp32, bf16 or f16 or, with a scale for each 128 columns, of e4m3.
//
// Bound by memory: x and y are read and x_out and z written once. A row lies in the registers of 8 to 512 threads, eight
// values in each of up to four pieces. One CTA an SM stays and walks over the rows; a team of threads gets its next
// rows by bulk copies through a ring in shared memory, so that what is in flight depends neither on registers nor on how
// long a row's sums take. Gains and biases lie in shared memory, tables are read through the L1 cache. Sums in fp32; the
// variance is that about the mean, in a second pass over the registers.
//
// Rows that start on multiples of eight values (and have as many columns) are read and written eight values at a
// time. Of others the copies take the whole 16-byte pieces and plain loads the rest, and a lane has every 32nd
// column, so that a warp's accesses are neighbours.
//
// 50432 x 768, fp32 stream, 82 us, 5.7 TB/s (68.5 at a copy's rate; without norms 77); 32760 x 1536 bf16, gated and
// modulated, 71 us, 5.6 TB/s, issue slots at 57 %; 8191 x 5000 to e4m3 64 us, issue slots at 59 %. (With rows loaded by the
// threads that compute them, without a ring: 82.6, 124 and 151.)
#pragma once
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "ptx.cuh"

namespace elasto {

namespace residual {

constexpr int MAX_THREADS = 512, MAX_PIECES = 4, FEW_PIECES = 3;  // of a row
static_assert(8 * MAX_PIECES * MAX_THREADS >= 16384, "columns");
constexpr int CTA_THREADS = 768, MAX_TEAMS = CTA_THREADS / 32, MAX_STAGES = 4;
constexpr int SMEM_LIMIT = 224 * 1024;    // of a CTA, for its rings and vectors
constexpr int TABLES_LIMIT = 160 * 1024;  // the same where tables are read through the L1 cache

struct Args {
  elasto_residual_norm_args u;
  int log_threads, stages;
  unsigned units;                // at most 2^31
  int x_bytes, y_bytes;          // of a row (0: no y)
  int x_slot, y_slot;            // of a row's place in the ring
  long long x_step, y_step;      // bytes from a row to the next
  int in_smem;                   // the vectors are in shared memory (rows of fewer than 512 threads: always)
  int* status;
};

__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// The larger of two numbers; a NaN wins.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// 448 / a and a / 448 of a block whose largest magnitude is a (2^-100 at least).
__device__ __forceinline__ float2 block_scales(float top) {
  const float a = max_nan(top, 7.88860905e-31f);
  return make_float2(__fdiv_rn(448.0f, a), __fdiv_rn(a, 448.0f));
}
// Global to shared, counted on the mbarrier: 16-byte aligned, a multiple of 16 bytes.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_addr(dst)),
               "l"(src), "r"(bytes), "r"(smem_addr(bar))
               : "memory");
}

using Eight = float2[4];  // a lane's values of a piece

template <int TYPE>
struct Type {
  static constexpr int size = TYPE == ELASTO_F32 ? 4 : 2;
  static __device__ __forceinline__ float2 pair(uint32_t w) {
    return TYPE == ELASTO_BF16 ? make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u))
                               : __half22float2(*reinterpret_cast<const __half2*>(&w));
  }
  static __device__ __forceinline__ uint32_t bits(float2 v) { return TYPE == ELASTO_BF16 ? pack_bf16x2(v.x, v.y) : pack_f16x2(v.x, v.y); }
  static __device__ __forceinline__ void read8(const uint8_t* p, Eight& v) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    if constexpr (TYPE == ELASTO_F32) {
      const uint4 b = reinterpret_cast<const uint4*>(p)[1];
      v[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y)), v[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
      v[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y)), v[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
    } else {
      v[0] = pair(a.x), v[1] = pair(a.y), v[2] = pair(a.z), v[3] = pair(a.w);
    }
  }
  static __device__ __forceinline__ void write8(uint8_t* p, const Eight& v) {
    if constexpr (TYPE == ELASTO_F32)  // (32 bytes at once, aligned to them)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(__float_as_uint(v[0].x)),
                   "r"(__float_as_uint(v[0].y)), "r"(__float_as_uint(v[1].x)), "r"(__float_as_uint(v[1].y)), "r"(__float_as_uint(v[2].x)),
                   "r"(__float_as_uint(v[2].y)), "r"(__float_as_uint(v[3].x)), "r"(__float_as_uint(v[3].y))
                   : "memory");
    else
      *reinterpret_cast<uint4*>(p) = make_uint4(bits(v[0]), bits(v[1]), bits(v[2]), bits(v[3]));
  }
  static __device__ __forceinline__ float read1(const uint8_t* p) {
    if constexpr (TYPE == ELASTO_F32) return *reinterpret_cast<const float*>(p);
    return pair(*reinterpret_cast<const uint16_t*>(p)).x;
  }
  // two values, the one at p and the other at q (`both`: else the first alone)
  static __device__ __forceinline__ void write2(uint8_t* p, uint8_t* q, float2 v, bool first, bool second) {
    if constexpr (TYPE == ELASTO_F32) {
      if (first) *reinterpret_cast<float*>(p) = v.x;
      if (second) *reinterpret_cast<float*>(q) = v.y;
    } else {
      const uint32_t w = bits(v);
      if (first) *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w);
      if (second) *reinterpret_cast<uint16_t*>(q) = static_cast<uint16_t>(w >> 16);
    }
  }
};
// f(Type) of a type known at run time: a branch around whole loops, since one around a conversion is compiled into both
// conversions and a choice.
template <typename F>
__device__ __forceinline__ void by_type(int type, F f) {
  if (type == ELASTO_F32)
    f(Type<ELASTO_F32>());
  else if (type == ELASTO_BF16)
    f(Type<ELASTO_BF16>());
  else
    f(Type<ELASTO_F16>());
}

// What the copies leave of a row at `p`: `head` bytes in front of the first whole 16-byte piece, `tail` behind the last.
// The row lies as far behind a 16-byte boundary in shared memory as in global memory.
struct Edges {
  int at, head, tail, whole;
  __device__ __forceinline__ Edges(const uint8_t* p, int bytes) {
    at = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15);
    const int to16 = (16 - at) & 15;
    head = min(to16, bytes);
    tail = bytes > to16 ? (bytes - to16) & 15 : 0;
    whole = bytes - head - tail;
  }
};

// T = 2^LOG threads have a row; a team is max(T, 32) threads and takes a unit of 32 / T rows (T < 32) or one at a time.
// Thread t has of piece i the columns column(i, 0) to column(i, 7). Lanes past the row's last column compute along, on zeros.
// (T known to the compiler: as an argument, with loops of shuffles, 50432 x 768 took 91.7 us in place of 82, 32760 x 1536 94.5
// in place of 71.)
template <int LOG, int PIECES, bool VEC>
__global__ void __launch_bounds__(LOG == 9 ? 512 : CTA_THREADS, 1)
    residual_norm_kernel(const __grid_constant__ Args args) {
  constexpr int T = 1 << LOG, TEAM = T < 32 ? 32 : T, W = T < 32 ? T : 32;
  constexpr int rows_log = LOG < 5 ? 5 - LOG : 0;
  const elasto_residual_norm_args& a = args.u;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[MAX_TEAMS][MAX_STAGES];
  __shared__ __align__(16) float partial[5][MAX_TEAMS];
  __shared__ uint4 zeros[2];  // what lanes past the row's last column read
  const int teams = blockDim.x / TEAM, team = warp_uniform(threadIdx.x / TEAM), t = threadIdx.x & (T - 1), lane = threadIdx.x & 31;
  const int sub = rows_log > 0 ? lane >> LOG : 0;
  const bool leader = (threadIdx.x & (TEAM - 1)) == 0;
  const int row_bytes = args.x_slot + args.y_slot, stage_bytes = row_bytes << rows_log, S = args.stages;
  uint8_t* const ring = smem + team * S * stage_bytes;
  float* const vectors = reinterpret_cast<float*>(smem + teams * S * stage_bytes);
  if (leader)
    for (int s = 0; s < S; ++s) mbar_init(&full[team][s], 1);
  if (threadIdx.x < 2) zeros[threadIdx.x] = make_uint4(0u, 0u, 0u, 0u);
  fence_barrier_init();
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  const unsigned stride = gridDim.x * teams, units = args.units;
  const uint8_t* const x0 = static_cast<const uint8_t*>(a.x);
  const uint8_t* const y0 = static_cast<const uint8_t*>(a.y);
  auto request = [&](unsigned unit, int s) {  // (the leader)
    const long long row0 = static_cast<long long>(unit) << rows_log;
    const int rows = static_cast<int>(min(static_cast<long long>(1 << rows_log), a.rows - row0));
    int total = rows * (args.x_bytes + args.y_bytes);
    if constexpr (!VEC) {
      total = 0;
      for (int k = 0; k < rows; ++k)
        total += Edges(x0 + (row0 + k) * args.x_step, args.x_bytes).whole + Edges(y0 + (row0 + k) * args.y_step, args.y_bytes).whole;
    }
    mbar_expect_tx(&full[team][s], total);
    for (int k = 0; k < rows; ++k) {
      uint8_t* const dst = ring + s * stage_bytes + k * row_bytes;
      const uint8_t* const x = x0 + (row0 + k) * args.x_step;
      const uint8_t* const y = y0 + (row0 + k) * args.y_step;
      if constexpr (VEC) {
        bulk_load(dst, x, args.x_bytes, &full[team][s]);
        if (args.y_bytes) bulk_load(dst + args.x_slot, y, args.y_bytes, &full[team][s]);
      } else {
        const Edges ex(x, args.x_bytes), ey(y, args.y_bytes);
        if (ex.whole) bulk_load(dst + ex.at + ex.head, x + ex.head, ex.whole, &full[team][s]);
        if (ey.whole) bulk_load(dst + args.x_slot + ey.at + ey.head, y + ey.head, ey.whole, &full[team][s]);
      }
    }
  };
  const unsigned unit0 = blockIdx.x * teams + team;
  if (leader)
    for (int s = 0; s < S && unit0 + s * stride < units; ++s) request(unit0 + s * stride, s);

  // The vectors, padded with zeros to the columns that the threads have. Of eight columns a lane the first four of every
  // eight lie together for each 256 columns, then the others: a warp's reads are then without conflicts.
  constexpr int padded = (8 * T * PIECES + 255) & ~255;
  auto place = [](int c) { return VEC ? (c & ~255) | (c & 4) << 5 | (c & 248) >> 1 | (c & 3) : c; };
  int used = 0;
  auto keep = [&](const float* p) {  // where in `vectors` it lies, -1: none
    if (!p) return -1;
    const int at = used;
    if (LOG < 9 || args.in_smem)
      for (int c = threadIdx.x; c < padded; c += blockDim.x) vectors[at + place(c)] = c < a.cols ? p[c] : 0.0f;
    used += padded;
    return at;
  };
  const bool post = a.y && a.post_norm != ELASTO_NORM_NONE, pre = a.pre_norm != ELASTO_NORM_NONE;
  const int post_gain = keep(post ? a.post_gain : nullptr), post_bias = keep(post ? a.post_bias : nullptr);
  const int y_scale = keep(a.y ? a.y_scale : nullptr);
  const int pre_gain = keep(pre ? a.pre_gain : nullptr), pre_bias = keep(pre ? a.pre_bias : nullptr);
  __syncthreads();

  auto team_sync = [&] {
    if constexpr (T > 32)
      named_bar_sync(1 + team, TEAM);
    else
      __syncwarp();
  };
  auto row_sum = [&](float2 two, int slot) {
    float v = two.x + two.y;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (T > 32) {
      float* const p = &partial[slot][team * (T / 32)];  // (the barrier in the middle of a row lies between two uses)
      if (lane == 0) p[t >> 5] = v;
      named_bar_sync(1 + team, TEAM);
      v = 0.0f;
#pragma unroll
      for (int w = 0; w < T / 32; ++w) v += p[w];
    }
    return v;
  };
  const float inv_n = 1.0f / static_cast<float>(a.cols);
  auto column = [&](int i, int k) { return VEC ? 8 * (t + T * i) + k : (t & ~31) * 8 + (t & (W - 1)) + 8 * T * i + W * k; };
  // (pieces but the last are whole; of eight neighbouring columns all are the row's or none)
  auto inside = [&](int i, int k) { return i < PIECES - 1 || column(i, VEC ? 0 : k) < a.cols; };
  auto pieces = [&](auto f) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) f(i);
  };
  // a piece of a row at p, zeros past its end
  auto read = [&](auto type, const uint8_t* p, int i, Eight& v) {
    using Ty = decltype(type);
    if constexpr (VEC) {
      Ty::read8(p + column(i, 0) * Ty::size, v);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = make_float2(0.0f, 0.0f);
        if (inside(i, 2 * j)) v[j].x = Ty::read1(p + column(i, 2 * j) * Ty::size);
        if (inside(i, 2 * j + 1)) v[j].y = Ty::read1(p + column(i, 2 * j + 1) * Ty::size);
      }
    }
  };
  auto read_smem = [&](auto type, const uint8_t* p, int i, Eight& v) {
    if (VEC && !inside(i, 0)) p = reinterpret_cast<const uint8_t*>(zeros) - column(i, 0) * decltype(type)::size;
    read(type, p, i, v);
  };
  auto write = [&](auto type, uint8_t* p, int i, const Eight& v) {
    using Ty = decltype(type);
    if constexpr (VEC) {
      if (inside(i, 0)) Ty::write8(p + column(i, 0) * Ty::size, v);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        Ty::write2(p + column(i, 2 * j) * Ty::size, p + column(i, 2 * j + 1) * Ty::size, v[j], inside(i, 2 * j), inside(i, 2 * j + 1));
    }
  };
  auto read_vector = [&](int at, const float* p, int i, Eight& g) {
    if (LOG < 9 || args.in_smem) {
      if constexpr (VEC) {
        const float4 x = *reinterpret_cast<const float4*>(vectors + at + place(column(i, 0)));
        const float4 y = *reinterpret_cast<const float4*>(vectors + at + place(column(i, 0)) + 128);
        g[0] = make_float2(x.x, x.y), g[1] = make_float2(x.z, x.w), g[2] = make_float2(y.x, y.y), g[3] = make_float2(y.z, y.w);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) g[j] = make_float2(vectors[at + column(i, 2 * j)], vectors[at + column(i, 2 * j + 1)]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        g[j].x = inside(i, 2 * j) ? p[column(i, 2 * j)] : 0.0f;
        g[j].y = inside(i, 2 * j + 1) ? p[column(i, 2 * j + 1)] : 0.0f;
      }
    }
  };
  // v is centred (LAYER), and scaled where it is small; returns 1 / sqrt(mean v^2 + eps)
  auto root = [&](float2 (&v)[PIECES][4], int kind, int slot) {
    float2 sum = make_float2(0.0f, 0.0f);
    if (kind == ELASTO_NORM_LAYER) {
      pieces([&](int i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum = add2(sum, v[i][j]);
      });
      const float mean = -row_sum(sum, slot) * inv_n;
      sum = make_float2(0.0f, 0.0f);
      pieces([&](int i) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          v[i][j] = add2(v[i][j], make_float2(inside(i, 2 * j) ? mean : 0.0f, inside(i, 2 * j + 1) ? mean : 0.0f));
      });
    }
    // Where the mean square is near the smallest normal number the squares have lost bits, or all of themselves: v times 2^100
    // then, whose squares are exact enough and far from overflow (v < 2^-55 there). A second time around, since ordinary
    // rows pay for more code (8191 x 5000 to e4m3 62.9 us without, 64.2 so, 68.7 with the second sum written out behind the first).
    float m = 0.0f, eps = a.eps;
#pragma unroll 1
    for (int at = slot + 1;; at = 4) {
      pieces([&](int i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum = fma2(v[i][j], v[i][j], sum);
      });
      m = fmaf(row_sum(sum, at), inv_n, eps);
      const bool small = m < 0x1p-124f;
      if (at == 4 || !(T >= 32 ? small : __any_sync(0xffffffffu, small))) break;  // (the same in all threads of a row)
      const float up = small ? 0x1p100f : 1.0f;
      eps = eps * up * up;
      sum = make_float2(0.0f, 0.0f);
      pieces([&](int i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = mul2(v[i][j], make_float2(up, up));
      });
    }
    // (rsqrtf is off by up to two units in the last place; one step of Newton's method leaves half of one)
    const float rs = rsqrtf(m), e = fmaf(-m * rs, rs, 1.0f);
    return fabsf(e) < 1.0f ? fmaf(0.5f * rs, e, rs) : rs;
  };

  bool failed = false;
  int group = 0, s = 0, phase = 0;
  float edge[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // of the unit to come: a value in front of x's whole pieces, one behind, of y's
  auto fetch = [&](unsigned unit) {          // what comes of a unit without a copy
    const long long r = min((static_cast<long long>(unit) << rows_log) + sub, a.rows - 1LL);
    if (a.group) group = a.group[r];
    if constexpr (!VEC) {
      auto ends = [&](int type, const uint8_t* p, int bytes, float& head, float& tail) {
        const Edges e(p, bytes);
        const int size = type == ELASTO_F32 ? 4 : 2;
        if (t >= 8) return;
        // (bits as they lie in memory)
        if (size == 4) {
          if (4 * t < e.head) head = *reinterpret_cast<const float*>(p + 4 * t);
          if (4 * t < e.tail) tail = *reinterpret_cast<const float*>(p + bytes - e.tail + 4 * t);
        } else {
          if (2 * t < e.head) head = __uint_as_float(*reinterpret_cast<const uint16_t*>(p + 2 * t));
          if (2 * t < e.tail) tail = __uint_as_float(*reinterpret_cast<const uint16_t*>(p + bytes - e.tail + 2 * t));
        }
      };
      ends(a.x_type, x0 + r * args.x_step, args.x_bytes, edge[0], edge[1]);
      if (args.y_bytes) ends(a.y_type, y0 + r * args.y_step, args.y_bytes, edge[2], edge[3]);
    }
  };
  if (unit0 < units) fetch(unit0);
  for (unsigned unit = unit0; unit < units; unit += stride) {
    const long long row = (static_cast<long long>(unit) << rows_log) + sub;
    bool live = row < a.rows;  // (lanes of rows past the last go along with the last, for the shuffles, and store nothing)
    const long long r = min(row, a.rows - 1LL);
    const uint8_t* const x = x0 + r * args.x_step;
    const uint8_t* const y = y0 + r * args.y_step;
    uint8_t* const slot = ring + s * stage_bytes + (static_cast<int>(r - row) + sub) * row_bytes;
    uint8_t* const xs = slot + (VEC ? 0 : reinterpret_cast<uintptr_t>(x) & 15);
    uint8_t* const ys = slot + args.x_slot + (VEC ? 0 : reinterpret_cast<uintptr_t>(y) & 15);
    const int g0 = group;
    if (!failed && !mbar_wait_warp(&full[team][s], phase)) {  // (no row after it is stored; the barriers go on)
      failed = true;
      if (lane == 0) record_status(args.status, ELASTO_ERR_TIMEOUT);
      if (leader)  // (the copies in flight land before the CTA exits)
        for (int k = 0; k < S; ++k) mbar_wait(&full[team][(s + k) % S], s + k < S ? phase : phase ^ 1);
    }
    if constexpr (!VEC) {
      auto put = [&](int type, uint8_t* at, const uint8_t* p, int bytes, float head, float tail) {
        const Edges e(p, bytes);
        if (t >= 8 || !live) return;
        if (type == ELASTO_F32) {
          if (4 * t < e.head) *reinterpret_cast<float*>(at + 4 * t) = head;
          if (4 * t < e.tail) *reinterpret_cast<float*>(at + bytes - e.tail + 4 * t) = tail;
        } else {
          if (2 * t < e.head) *reinterpret_cast<uint16_t*>(at + 2 * t) = static_cast<uint16_t>(__float_as_uint(head));
          if (2 * t < e.tail) *reinterpret_cast<uint16_t*>(at + bytes - e.tail + 2 * t) = static_cast<uint16_t>(__float_as_uint(tail));
        }
      };
      put(a.x_type, xs, x, args.x_bytes, edge[0], edge[1]);
      if (args.y_bytes) put(a.y_type, ys, y, args.y_bytes, edge[2], edge[3]);
      fence_async_smem();  // (a later row's copy may write where these bytes lie)
      team_sync();
    }
    if (unit + stride < units) fetch(unit + stride);
    int g = g0;
    if (a.groups > 0 && static_cast<unsigned>(g) >= static_cast<unsigned>(a.groups)) {
      if (live && t == 0) record_status(args.status, ELASTO_ERR_INVALID_ARG);
      live = false, g = 0;
    }
    live = live && !failed;

    float2 v[PIECES][4];
    auto each = [&](auto f) {  // v = f(i, j, v)
      pieces([&](int i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = f(v[i][j]);
      });
    };
    // v = v f times the one vector plus the other (-1: none)
    auto normed = [&](float f, int gain, const float* gain_p, int bias, const float* bias_p) {
      if (gain >= 0 && bias >= 0) {
        pieces([&](int i) {
          Eight g, b;
          read_vector(gain, gain_p, i, g);
          read_vector(bias, bias_p, i, b);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[i][j] = fma2(mul2(v[i][j], make_float2(f, f)), g[j], b[j]);
        });
        return;
      }
      if (gain >= 0)
        pieces([&](int i) {
          Eight g;
          read_vector(gain, gain_p, i, g);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[i][j] = mul2(mul2(v[i][j], make_float2(f, f)), g[j]);
        });
      else
        each([&](float2 p) { return mul2(p, make_float2(f, f)); });
      if (bias >= 0)
        pieces([&](int i) {
          Eight b;
          read_vector(bias, bias_p, i, b);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[i][j] = add2(v[i][j], b[j]);
        });
    };
    auto with_table = [&](const void* p, auto op) {
      if (!p) return;
      by_type(a.mod_type, [&](auto type) {
        const uint8_t* const from = static_cast<const uint8_t*>(p) + g * a.mod_row * type.size;
        pieces([&](int i) {
          Eight f = {};
          if (!VEC || inside(i, 0)) read(type, from, i, f);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[i][j] = op(v[i][j], f[j]);
        });
      });
    };
    auto times = [](float2 p, float2 q) { return mul2(p, q); };
    auto plus = [](float2 p, float2 q) { return add2(p, q); };
    if (args.y_bytes) {
      by_type(a.y_type, [&](auto type) { pieces([&](int i) { read_smem(type, ys, i, v[i]); }); });
      if (post) normed(root(v, a.post_norm, 0), post_gain, a.post_gain, post_bias, a.post_bias);
      if (y_scale >= 0) normed(1.0f, y_scale, a.y_scale, -1, nullptr);
      with_table(a.gate, times);
    } else {
      each([](float2) { return make_float2(0.0f, 0.0f); });
    }
    by_type(a.x_type, [&](auto type) {
      pieces([&](int i) {
        Eight f;
        read_smem(type, xs, i, f);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = fma2(make_float2(a.x_factor, a.x_factor), f[j], v[i][j]);
      });
    });
    team_sync();  // the stage has been read
    if (leader && !failed && unit + S * stride < units) request(unit + S * stride, s);
    if (++s == S) s = 0, phase ^= 1;

    if (a.x_out && live)
      by_type(a.x_type, [&](auto type) {
        uint8_t* const out = static_cast<uint8_t*>(a.x_out) + r * a.x_out_row * type.size;
        pieces([&](int i) { write(type, out, i, v[i]); });
      });
    if (!a.z) continue;
    if (pre) normed(root(v, a.pre_norm, 2), pre_gain, a.pre_gain, pre_bias, a.pre_bias);
    with_table(a.scale, [](float2 p, float2 q) { return fma2(p, q, p); });
    with_table(a.shift, plus);
    if (a.z_type != ELASTO_E4M3) {
      if (live)
        by_type(a.z_type, [&](auto type) {
          uint8_t* const out = static_cast<uint8_t*>(a.z) + r * a.z_row * type.size;
          pieces([&](int i) { write(type, out, i, v[i]); });
        });
      continue;
    }
    if constexpr (LOG >= 4) {  // (e4m3 rows have 16 threads at least)
      // Blocks of 128 columns: 16 lanes' eight values of a piece, or (VEC not, 32 lanes) a warp's first and last four.
      // One lane of them divides, another for each block.
      constexpr bool TWO = !VEC && W == 32;
      const int l = TWO ? lane : lane & 15;
      float mine = 0.0f;
      pieces([&](int i) {
        float top[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float& p = top[TWO ? j >> 1 : 0];
          p = max_nan(p, max_nan(fabsf(v[i][j].x), fabsf(v[i][j].y)));  // (0 past the row's end)
        }
#pragma unroll
        for (int o = TWO ? 16 : 8; o > 0; o >>= 1) {
          top[0] = max_nan(top[0], __shfl_xor_sync(0xffffffffu, top[0], o));
          if (TWO) top[1] = max_nan(top[1], __shfl_xor_sync(0xffffffffu, top[1], o));
        }
        if (l == (TWO ? 2 * i : i)) mine = top[0];
        if (TWO && l == 2 * i + 1) mine = top[1];
      });
      const float2 d = block_scales(mine);
      uint8_t* const out = static_cast<uint8_t*>(a.z) + r * a.z_row;
      pieces([&](int i) {
        const float m0 = __shfl_sync(0xffffffffu, d.x, TWO ? 2 * i : (lane & 16) | i);
        const float m1 = TWO ? __shfl_sync(0xffffffffu, d.x, 2 * i + 1) : m0;
        const int block = (TWO ? (t & ~31) * 8 / 128 + (l & 1) : t >> 4) + T * i / 16;
        if ((TWO ? l >> 1 : l) == i && live && block * 128 < a.cols) a.z_scale[block * a.z_scale_row + r] = d.y;
        if (!live) return;
        uint32_t c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float m = TWO && j >= 2 ? m1 : m0;
          const float2 q = mul2(v[i][j], make_float2(m, m));
          c[j] = pack_e4m3x2(q.x, q.y);
        }
        if constexpr (VEC) {
          if (inside(i, 0)) *reinterpret_cast<uint2*>(out + column(i, 0)) = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (inside(i, 2 * j)) out[column(i, 2 * j)] = static_cast<uint8_t>(c[j]);
            if (inside(i, 2 * j + 1)) out[column(i, 2 * j + 1)] = static_cast<uint8_t>(c[j] >> 8);
          }
        }
      });
    }
  }
}

template <int LOG, int PIECES, bool VEC>
cudaError_t start(const Args& a, unsigned grid, int threads, int smem, cudaStream_t s) {
  static DeviceOnce once;
  const cudaError_t e =
      once([] { return cudaFuncSetAttribute(residual_norm_kernel<LOG, PIECES, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_LIMIT); });
  if (e != cudaSuccess) return e;
  return launch_pdl(residual_norm_kernel<LOG, PIECES, VEC>, dim3(grid), dim3(threads), smem, s, a);
}

template <bool VEC>
cudaError_t launch(const elasto_residual_norm_args& u, int* status, cudaStream_t s) {
  Args a{};
  a.u = u, a.status = status;
  auto size = [](int type) { return type == ELASTO_F32 ? 4 : 2; };
  const int eights = (u.cols + 7) / 8;
  a.log_threads = u.z && u.z_type == ELASTO_E4M3 ? 4 : 3;  // (a block of 128 columns is 16 threads' at least)
  while (eights > FEW_PIECES << a.log_threads && (1 << a.log_threads) < MAX_THREADS) ++a.log_threads;
  const int pieces = (eights + (1 << a.log_threads) - 1) >> a.log_threads;
  a.x_bytes = u.cols * size(u.x_type), a.y_bytes = u.y ? u.cols * size(u.y_type) : 0;
  a.x_slot = VEC ? a.x_bytes : (a.x_bytes + 30) & ~15;
  a.y_slot = VEC || !u.y ? a.y_bytes : (a.y_bytes + 30) & ~15;
  a.x_step = u.x_row * size(u.x_type), a.y_step = u.y ? u.y_row * size(u.y_type) : 0;
  const int rows = a.log_threads < 5 ? 32 >> a.log_threads : 1, team = 1 << std::max(a.log_threads, 5);
  a.units = (static_cast<unsigned>(u.rows) - 1) / rows + 1;
  int vectors = 0;
  for (const float* p : {u.y && u.post_norm ? u.post_gain : nullptr, u.y && u.post_norm ? u.post_bias : nullptr, u.y ? u.y_scale : nullptr,
                         u.pre_norm ? u.pre_gain : nullptr, u.pre_norm ? u.pre_bias : nullptr})
    if (p) vectors += 4 * (((8 * pieces << a.log_threads) + 255) & ~255);
  const int stage = rows * (a.x_slot + a.y_slot);
  a.in_smem = vectors + stage <= SMEM_LIMIT;  // (else, in rows of more than 8000 columns, they are read where they are)
  if (!a.in_smem) vectors = 0;
  // As many teams as have two stages each beside the vectors (one where not even one team has), and no more than
  // spread the rows over all SMs.
  const unsigned sms = num_sms() > 0 ? num_sms() : 152;
  const int room = (u.gate || u.shift || u.scale ? std::max(TABLES_LIMIT, vectors + stage) : SMEM_LIMIT) - vectors;
  int teams = std::max(1, std::min(CTA_THREADS / team, room / (2 * stage)));
  teams = static_cast<int>(std::min<unsigned>(teams, (a.units - 1) / sms + 1));
  const unsigned grid = std::min((a.units - 1) / teams + 1, sms);
  a.stages = std::min({room / (teams * stage), MAX_STAGES, static_cast<int>((a.units - 1) / (grid * teams)) + 1});
  const int smem = a.stages * teams * stage + vectors, threads = teams * team;
  auto with = [&](auto log) {
    constexpr int LOG = log.value;
    if constexpr (LOG < 5)
      if (pieces == 1) return start<LOG, 1, VEC>(a, grid, threads, smem, s);
    if constexpr (LOG == 9)
      if (pieces == 4) return start<LOG, 4, VEC>(a, grid, threads, smem, s);
    return pieces == 2 ? start<LOG, 2, VEC>(a, grid, threads, smem, s) : start<LOG, 3, VEC>(a, grid, threads, smem, s);
  };
  switch (a.log_threads) {
    case 3: return with(std::integral_constant<int, 3>());
    case 4: return with(std::integral_constant<int, 4>());
    case 5: return with(std::integral_constant<int, 5>());
    case 6: return with(std::integral_constant<int, 6>());
    case 7: return with(std::integral_constant<int, 7>());
    case 8: return with(std::integral_constant<int, 8>());
    default: return with(std::integral_constant<int, 9>());
  }
}

}  // namespace residual

// Rows value by value (residual_norm_any.cu).
cudaError_t residual_norm_any_launch(const elasto_residual_norm_args& u, int* status, cudaStream_t s);

}  // namespace elasto
