// Norms of queries and keys for each head, with the position rotation and the
// write to the K/V cache in the same pass:
//   y = x * rsqrt(mean(x^2) + eps) * gain,  pairs (a, b) -> (a c - b s, b c + a s).
//
// q, k (and v) are read and written once, everything between in fp32 registers. A
// head lies in LANES = head_dim / 8 lanes, rounded up to a power of two, 16 bytes
// each; a warp walks over the heads of one row, 32 / LANES at a time, or of several
// rows at once. q, and k with v, have CTAs of their own: a lane's cosines, sines and
// gains are then one set, read once a row and multiplied together before the heads
// are walked over. The partner channel of the half-split form is rot_dim / 16 lanes
// away (rot_dim / 2 is a multiple of 8).
//
// Bound by memory, with the loads a row needs before its heads (position, angles,
// gains) and issue slots (unpacking, the norm's and the partners' shuffles) close
// behind. 32776 rows of 12 + 12 heads of 64: 36.0 us, 5.6 TB/s of the 203 MB it reads
// and writes; the copy's 6.8 would take 29.9 us. (CTAs of 256 threads with three heads in flight a lane: 40.4; of
// 128 with six: 37.4.) With values, into a cache: 10000 rows of 32 + 8 heads of 128 46.6 us (36.9 by their
// bytes at a copy's rate), 32776 of 12 + 12 of 64 64.0 (45.7). Single tokens (64 rows): 2.7 to 3.0 us, the latency of one chain of loads.
// With positions on several axes: 32760 rows of 12 + 12 heads of 128, three axes, neighbours: 68.4 us, 5.9 TB/s; 32776 of 12 + 12
// of 64, f16, two axes, halves of each axis, no norm: 36.1 (29.7 at a copy's rate), issue slots at 65 %.
// The first with the half-split pairing 72.1; with axes in turn (a table row for each pair of a lane) 68.4 and half-split 71.8; with
// values, into a cache, 113 to 115.
#include <type_traits>

#include "common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int THREADS = 128, WARPS = THREADS / 32, MIN_CTAS = 7, BATCH = 4;

template <bool BF>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  return BF ? make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u))
            : __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// elasto_op_qk_norm_rope_axes: the same with a position for each axis.
struct AxesArgs : elasto_qk_norm_rope_args {
  int norm, axes;
  long long positions_row, positions_axis;
  uint64_t axis[4];           // of pair j: bits 2 (j % 32) of word j / 32
  short first[4], pairs[4];   // PAIRS_AXIS: an axis's first pair and their number
};

// Rows of a warp: 1 (its 32 / LANES groups of lanes take as many heads of it) or, SHARED, 2 to the rows_log
// (each row has its own groups). chunks: warps that share a row, each taking every chunks-th step of heads.
template <bool BF, int LANES, int PAIRS, bool SHARED, typename ARGS>
__global__ void __launch_bounds__(THREADS, MIN_CTAS)
    qk_norm_rope_kernel(const __grid_constant__ ARGS a, int rows_of_warp, int chunks, int* status) {
  pdl_wait();
  pdl_trigger();
  constexpr bool AXES = std::is_same<ARGS, AxesArgs>::value, INTERLEAVED = PAIRS == ELASTO_PAIRS_NEIGHBOURS;
  constexpr int HPW = 32 / LANES;
  const int rows_log = SHARED ? rows_of_warp : 0;
  const int lane = threadIdx.x & 31, l = lane % LANES, sub = lane / LANES;
  const bool both = a.heads_q > 0 && a.heads_k > 0;
  const bool keys = both ? blockIdx.x & 1 : a.heads_k > 0;  // this CTA's heads: k (and v), or q
  const unsigned unit = (both ? blockIdx.x >> 1 : blockIdx.x) * WARPS + (threadIdx.x >> 5);
  const unsigned first = (chunks == 1 ? unit : unit / chunks) << rows_log;  // of the warp's rows
  const int chunk = chunks == 1 ? 0 : static_cast<int>(unit - first * chunks);  // (chunks > 1 only with one row a warp)
  if (first >= static_cast<unsigned>(a.rows)) return;
  unsigned row = first;
  bool live = true;
  if constexpr (SHARED) {  // lanes of rows past the last go along, for the shuffles
    row = min(first + (sub & ((1u << rows_log) - 1)), static_cast<unsigned>(a.rows) - 1);
    live = row == first + (sub & ((1u << rows_log) - 1));
  }
  const int step = HPW >> rows_log, hsub = sub >> rows_log;  // heads of a row at a time, and this lane's
  const int e = 8 * l;  // first channel of this lane
  const bool on = e < a.head_dim, turns = e < a.rot_dim;
  const int half = a.rot_dim / 2;
  int pe = !turns || INTERLEAVED ? e : e < half ? e + half : e - half;  // the partner channels
  int pair = INTERLEAVED ? e / 2 : e < half ? e : e - half;             // the first of this lane's pairs
  bool front = e < half;                                                // it holds the first channels of them
  if constexpr (PAIRS == ELASTO_PAIRS_AXIS) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {  // (lengths are multiples of 8: a lane lies in one half of one axis)
      const int at = e - 2 * a.first[x], n = a.pairs[x];
      if (turns && at >= 0 && at < 2 * n) front = at < n, pe = front ? e + n : e - n, pair = a.first[x] + (front ? at : at - n);
    }
  }
  const int partner = lane - l + pe / 8;

  int slot = static_cast<int>(row), pos = 0;
  int axis_pos[4] = {0, 0, 0, 0};
  bool outside = false;
  if constexpr (AXES) {
    if (a.rot_dim > 0) {
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (x < a.axes) axis_pos[x] = a.positions[row * a.positions_row + x * a.positions_axis];
    }
  } else {
    if (a.rot_dim > 0) pos = a.positions[row];
  }
  if (a.slots && a.heads_k > 0) slot = a.slots[row];
  const int n = keys ? a.heads_k : a.heads_q;
  const long long x_head = keys ? a.k_head : a.q_head;
  const uint16_t* const x = static_cast<const uint16_t*>(keys ? a.k : a.q) + static_cast<long long>(row) * (keys ? a.k_row : a.q_row) + e;
  // (the first heads' values are requested before the angles are known)
  uint4 w[BATCH];
  auto request = [&](int h0) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int h = h0 + i * chunks * step + hsub;
      w[i] = make_uint4(0u, 0u, 0u, 0u);
      if (on && h < n) w[i] = *reinterpret_cast<const uint4*>(x + h * x_head);
    }
  };
  request(chunk * step);
  if constexpr (AXES) {
#pragma unroll
    for (int x = 0; x < 4; ++x) outside |= a.rot_dim > 0 && static_cast<unsigned>(axis_pos[x]) >= static_cast<unsigned>(a.n_positions);
  } else {
    outside = a.rot_dim > 0 && static_cast<unsigned>(pos) >= static_cast<unsigned>(a.n_positions);
  }
  if (outside || (a.slots && a.heads_k > 0 && slot >= a.n_slots)) {
    if (live && (SHARED ? l == 0 : lane == 0)) record_status(status, ELASTO_ERR_INVALID_ARG);
    if constexpr (!SHARED) return;
    live = false;
    pos = axis_pos[0] = axis_pos[1] = axis_pos[2] = axis_pos[3] = 0;
  }
  if (keys && slot < 0) {
    if constexpr (!SHARED) return;
    live = false;
  }
  const float inv_d = 1.0f / static_cast<float>(a.head_dim);

  // y = r (x own + partner's x * other), r = rsqrt(mean(x^2) + eps): the row's angles at this lane's
  // channels, with the gains
  float2 own[4], other[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) own[j] = make_float2(1.0f, 1.0f), other[j] = make_float2(0.0f, 0.0f);
  if (turns && AXES) {
    if constexpr (AXES) {
      constexpr int N = INTERLEAVED ? 4 : 8;  // pairs of a lane
      const uint32_t axis = static_cast<uint32_t>(a.axis[pair >> 5] >> 2 * (pair & 31)) & ((1u << 2 * N) - 1u);
      auto at = [&](uint32_t x) { return x == 0 ? axis_pos[0] : x == 1 ? axis_pos[1] : x == 2 ? axis_pos[2] : axis_pos[3]; };
      float c[N], s[N];
      if (axis == (axis & 3u) * (0x55555555u & ((1u << 2 * N) - 1u))) {  // one axis for all
        const float* const table = a.cos_sin + static_cast<size_t>(at(axis & 3u)) * a.rot_dim + pair;
#pragma unroll
        for (int j = 0; j < N; j += 4) {
          const float4 x = *reinterpret_cast<const float4*>(table + j), y = *reinterpret_cast<const float4*>(table + half + j);
          c[j] = x.x, c[j + 1] = x.y, c[j + 2] = x.z, c[j + 3] = x.w;
          s[j] = y.x, s[j + 1] = y.y, s[j + 2] = y.z, s[j + 3] = y.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float* const table = a.cos_sin + static_cast<size_t>(at(axis >> 2 * j & 3u)) * a.rot_dim + pair + j;
          c[j] = table[0], s[j] = table[half];
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (INTERLEAVED) {
          own[j] = make_float2(c[j], c[j]), other[j] = make_float2(-s[j], s[j]);
        } else {
          own[j] = make_float2(c[2 * j], c[2 * j + 1]);
          other[j] = front ? make_float2(-s[2 * j], -s[2 * j + 1]) : make_float2(s[2 * j], s[2 * j + 1]);
        }
      }
    }
  } else if (turns) {
    const float* table = a.cos_sin + static_cast<size_t>(pos) * a.rot_dim;
    if constexpr (INTERLEAVED) {  // pairs e / 2 .. e / 2 + 3
      const float4 c = *reinterpret_cast<const float4*>(table + e / 2);
      const float4 s = *reinterpret_cast<const float4*>(table + half + e / 2);
      own[0] = make_float2(c.x, c.x), own[1] = make_float2(c.y, c.y), own[2] = make_float2(c.z, c.z), own[3] = make_float2(c.w, c.w);
      other[0] = make_float2(-s.x, s.x), other[1] = make_float2(-s.y, s.y), other[2] = make_float2(-s.z, s.z);
      other[3] = make_float2(-s.w, s.w);
    } else {
      const int p = e < half ? e : e - half;
      const float sign = e < half ? -1.0f : 1.0f;
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const float4 c = *reinterpret_cast<const float4*>(table + p + 2 * j);
        const float4 s = *reinterpret_cast<const float4*>(table + half + p + 2 * j);
        own[j] = make_float2(c.x, c.y), own[j + 1] = make_float2(c.z, c.w);
        other[j] = make_float2(sign * s.x, sign * s.y), other[j + 1] = make_float2(sign * s.z, sign * s.w);
      }
    }
  }
  const float* const gain = keys ? a.k_gain : a.q_gain;
  if (gain && on) {
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      const float4 g = *reinterpret_cast<const float4*>(gain + e + 2 * j);   // of this lane's channels
      const float4 o = *reinterpret_cast<const float4*>(gain + pe + 2 * j);  // and of the partners'
      own[j] = mul2(own[j], make_float2(g.x, g.y)), own[j + 1] = mul2(own[j + 1], make_float2(g.z, g.w));
      other[j] = mul2(other[j], INTERLEAVED ? make_float2(o.y, o.x) : make_float2(o.x, o.y));
      other[j + 1] = mul2(other[j + 1], INTERLEAVED ? make_float2(o.w, o.z) : make_float2(o.z, o.w));
    }
  }
  const long long y_head = keys ? a.k_out_head : a.q_out_head;
  uint16_t* const y = static_cast<uint16_t*>(keys ? a.k_out : a.q_out) + (keys ? slot * a.k_out_row : static_cast<long long>(row) * a.q_out_row) + e;
  for (int h0 = chunk * step; h0 < n; h0 += BATCH * chunks * step) {
    if (h0 != chunk * step) request(h0);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int hb = h0 + i * chunks * step, h = hb + hsub;
      if (hb >= n) break;
      const uint32_t ws[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
      float2 v[4], ss = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = unpack2<BF>(ws[j]);
        ss = fma2(v[j], v[j], ss);
      }
      float sum = ss.x + ss.y;
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      float r = rsqrtf(fmaf(sum, inv_d, a.eps));
      if constexpr (AXES) r = a.norm ? r : 1.0f;
      uint32_t out[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 o = INTERLEAVED ? make_float2(v[j].y, v[j].x) : unpack2<BF>(__shfl_sync(0xffffffffu, ws[j], partner & 31));
        // (where nothing turns `other` is 0 and `o` the value itself or its neighbour: an infinite one, whose head
        // has r = 0, must not reach the neighbour as 0 * infinity)
        float2 z = mul2(v[j], own[j]);
        if ((!INTERLEAVED && !AXES) || turns) z = fma2(o, other[j], z);
        z = mul2(z, make_float2(r, r));
        out[j] = BF ? pack_bf16x2(z.x, z.y) : pack_f16x2(z.x, z.y);
      }
      if (on && live && h < n) *reinterpret_cast<uint4*>(y + h * y_head) = make_uint4(out[0], out[1], out[2], out[3]);
    }
  }
  if (keys && a.v) {
    const uint16_t* const xv = static_cast<const uint16_t*>(a.v) + static_cast<long long>(row) * a.v_row + e;
    uint16_t* const yv = static_cast<uint16_t*>(a.v_out) + slot * a.v_out_row + e;
#pragma unroll 4
    for (int h = chunk * step + hsub; h < n; h += chunks * step)
      if (on && live) *reinterpret_cast<uint4*>(yv + h * a.v_out_head) = __ldcs(reinterpret_cast<const uint4*>(xv + h * a.v_head));
  }
}

template <int LANES, typename ARGS>
cudaError_t launch(const ARGS& a, int pairing, int* status, cudaStream_t s) {
  // As many warps a row as leave each at least one step of heads, where the rows alone are few; as many rows a warp as
  // leave 32 warps for each SM and a lane eight heads, where they are many (what a lane sets up for a row then serves more
  // heads: 60000 rows of 1 + 1 heads of 64 42.1 -> 13.0 us, 32776 of 12 + 12 41.6 -> 35.7; with 16 heads a lane, 10000 rows
  // of 32 + 8 of 128, 46.5 -> 48.9).
  const int heads = a.heads_q > a.heads_k ? a.heads_q : a.heads_k, groups = (heads + 32 / LANES - 1) / (32 / LANES);
  const long long wanted = 32LL * (num_sms() > 0 ? num_sms() : 152);
  int chunks = static_cast<int>(wanted / a.rows), rows_log = 0;
  chunks = chunks < 1 ? 1 : chunks > groups ? groups : chunks;
  while ((LANES << rows_log) < 32 && (static_cast<long long>(a.rows) >> (rows_log + 1)) >= wanted &&
         (heads << rows_log) <= 8 * (32 / LANES))
    ++rows_log;
  const unsigned units = ((static_cast<unsigned>(a.rows) - 1) / (1u << rows_log) + 1) * chunks;  // (or at most 32 warps an SM)
  const dim3 grid((units + WARPS - 1) / WARPS * (a.heads_q > 0 && a.heads_k > 0 ? 2 : 1)), block(THREADS);
  auto start = [&](auto bf, auto pairs) {
    if constexpr (LANES < 32)
      if (rows_log > 0)
        return launch_pdl(qk_norm_rope_kernel<bf.value, LANES, pairs.value, true, ARGS>, grid, block, 0, s, a, rows_log, chunks, status);
    return launch_pdl(qk_norm_rope_kernel<bf.value, LANES, pairs.value, false, ARGS>, grid, block, 0, s, a, 0, chunks, status);
  };
  auto typed = [&](auto bf) {
    if (pairing == ELASTO_PAIRS_NEIGHBOURS) return start(bf, std::integral_constant<int, ELASTO_PAIRS_NEIGHBOURS>());
    if constexpr (std::is_same<ARGS, AxesArgs>::value)
      if (pairing == ELASTO_PAIRS_AXIS) return start(bf, std::integral_constant<int, ELASTO_PAIRS_AXIS>());
    return start(bf, std::integral_constant<int, ELASTO_PAIRS_HALF>());
  };
  return a.dtype == ELASTO_BF16 ? typed(std::true_type()) : typed(std::false_type());
}

template <typename ARGS>
cudaError_t launch_any(const ARGS& a, int pairing, int* status, cudaStream_t s) {
  const int lanes = a.head_dim / 8;
  if (lanes <= 1) return launch<1>(a, pairing, status, s);
  if (lanes <= 2) return launch<2>(a, pairing, status, s);
  if (lanes <= 4) return launch<4>(a, pairing, status, s);
  if (lanes <= 8) return launch<8>(a, pairing, status, s);
  if (lanes <= 16) return launch<16>(a, pairing, status, s);
  return launch<32>(a, pairing, status, s);
}

}  // namespace

cudaError_t qk_norm_rope_launch(const elasto_qk_norm_rope_args& a, int* status, cudaStream_t s) {
  return launch_any(a, a.interleaved ? ELASTO_PAIRS_NEIGHBOURS : ELASTO_PAIRS_HALF, status, s);
}

cudaError_t qk_norm_rope_axes_launch(const elasto_qk_norm_rope_axes_args& u, int* status, cudaStream_t s) {
  AxesArgs a{};
  a.dtype = u.dtype, a.rows = u.rows, a.heads_q = u.heads_q, a.heads_k = u.heads_k, a.head_dim = u.head_dim, a.rot_dim = u.rot_dim;
  a.eps = u.eps;
  a.q = u.q, a.q_row = u.q_row, a.q_head = u.q_head, a.k = u.k, a.k_row = u.k_row, a.k_head = u.k_head;
  a.v = u.v, a.v_row = u.v_row, a.v_head = u.v_head;
  a.q_out = u.q_out, a.q_out_row = u.q_out_row, a.q_out_head = u.q_out_head;
  a.k_out = u.k_out, a.k_out_row = u.k_out_row, a.k_out_head = u.k_out_head;
  a.v_out = u.v_out, a.v_out_row = u.v_out_row, a.v_out_head = u.v_out_head;
  a.q_gain = u.q_gain, a.k_gain = u.k_gain, a.cos_sin = u.cos_sin, a.positions = u.positions, a.n_positions = u.n_positions;
  a.slots = u.slots, a.n_slots = u.n_slots;
  a.norm = u.norm, a.axes = u.axes, a.positions_row = u.positions_row, a.positions_axis = u.positions_axis;
  for (int j = u.rot_dim / 2 - 1; j >= 0; --j) {
    const int x = u.axis_of[j];
    a.axis[j >> 5] |= static_cast<uint64_t>(x) << 2 * (j & 31);
    a.first[x] = static_cast<short>(j), ++a.pairs[x];
  }
  return launch_any(a, u.pairing, status, s);
}

}  // namespace elasto
