// Product of e4m3 rows with e4m3 weights, both with fp32 scales for blocks of 128:
//   out[m, n] = epi( sum_b as[b, m] ws[n / 128, b] sum_{k in block b} A[m, k] W[n, k] + bias[n] ).
//
// The scales are fp32 numbers, so the tensor core cannot apply them: the sum over
// a block of 128 columns is one accumulator in TMEM, and the running sum lives in
// registers, where block b is added as acc += part * (as ws). A k-block is one
// 128-byte row of A and W in the 128-byte swizzle: four K = 32 steps.
//   warp 0      TMA producer of a ring of A and W tiles;
//   warp 1      tcgen05.mma (kind::f8f6f4), block after block into two (256 columns) or
//               four accumulators in turn;
//   warps 4-11  read the finished accumulator while the other fills; two warps share
//               32 rows, each half of the tile's columns (a row a thread); after the
//               last block they add the bias and store.
//
// Large products run on CTA pairs (256 x 256 tiles: each SM loads half of W's tile),
// others on 128 x 128 and 128 x 64; tile_cost estimates which is quickest.
// 8192 x 8192 x 4096: 199 us captured in a graph, 2.8 PFLOP/s (e4m3's rate is about twice the 1.87 measured for bf16);
// called with new inputs each time 215. A block of K costs ~760 clocks where its MMAs take 512: MMA, commit, read-out and
// release follow one another, with only two accumulators in TMEM to overlap them.
// The column halves shorten that chain (207 -> 202 us). 50432 x 2304 x 768 to bf16: 104
// us, of which the last read-out and store of each tile are ~2 us in 6 blocks of K;
// its bytes alone would take 40.
#include <algorithm>

#include "act.cuh"
#include "common.h"
#include "fp8_common.h"
#include "ptx.cuh"

namespace elasto {

namespace {

constexpr int THREADS = 384, EPI_WARPS = 8;
constexpr int REGS = 168, REGS_FEW = 40, REGS_MANY = 232;  // at launch; of warps 0-3 and 4-11 after the split
static_assert(128 * REGS_FEW + 256 * REGS_MANY <= THREADS * REGS, "register split");
constexpr int BM = 128, BK = 128, A_STAGE = BM * BK;
constexpr int TMEM_COLS = 512;
constexpr int MAX_STAGES = 8;
constexpr int PIECE = 32 * 128;  // output staging of an epilogue warp: 32 rows of 128 bytes, two of them
constexpr int PIECES = 2 * EPI_WARPS * PIECE;
constexpr int TAIL = EPI_WARPS * 128 + 512;  // 32 values of the bias for each epilogue warp, barriers
constexpr int SMEM_LIMIT = 232448;

template <bool PAIR, int BN>
struct Tile {
  static constexpr int b_stage = (PAIR ? BN / 2 : BN) * BK, stage = A_STAGE + b_stage;
  static constexpr int room = (SMEM_LIMIT - 1024 - TAIL - PIECES) / stage;
  static constexpr int stages = room < MAX_STAGES ? room : MAX_STAGES;
  static constexpr int smem = 1024 + stages * stage + PIECES + TAIL;
  static constexpr int tm = PAIR ? 2 * BM : BM;
  static constexpr int cols = BN / 2;  // of an epilogue warp
  static constexpr int accs = BN == 256 ? 2 : 4;  // accumulators
  // Column halves of an accumulator, each with its own MMAs and barriers (256 columns: a half is read out while
  // the other's products run)
  static constexpr int halves = BN == 256 ? 2 : 1, half = BN / halves;
};

struct Args {
  int M, N, K, nkb;
  const float* a_scale;
  long long lds;
  const float* w_scale;
  const float* bias;
  void* out;
  long long ldo;
  int tma_cols;  // pieces of columns that end by this one leave by TMA (0: rows of out do not start on 16 bytes)
  int* status;
};

template <int EPI>
constexpr bool f32_out = EPI == EPI_BIAS_RESID_F32 || EPI == EPI_BIAS_F32;

// A warp's 32 rows x CW columns of out from shared memory (32-bit words: fp32 values or pairs of 16-bit ones;
// word w of row r at r * 32 + (w ^ r)), where rows start on any value. A row leaves in 4-byte words; one of
// 16-bit values that starts inside a word has a single value at either end and pairs across two words between.
template <int EPI, int CW>
__device__ __forceinline__ void store_rows(const Args& a, const uint32_t* t, int lane, int row0, int col0) {
  const int left = a.N - col0;
  if (row0 + 32 > a.M || left < CW) {  // the last rows or columns: value by value
#pragma unroll
    for (int c = lane; c < CW; c += 32) {
      const long long at = row0 * a.ldo + col0 + c;
#pragma unroll 8
      for (int i = 0; i < 32; ++i) {
        if (row0 + i >= a.M || c >= left) continue;
        if constexpr (f32_out<EPI>)
          fp8_store_one<EPI>(a.out, at + i * a.ldo, __uint_as_float(t[i * 32 + (c ^ i)]));
        else
          static_cast<uint16_t*>(a.out)[at + i * a.ldo] = static_cast<uint16_t>(t[i * 32 + ((c >> 1) ^ i)] >> (16 * (c & 1)));
      }
    }
    return;
  }
  if constexpr (f32_out<EPI>) {
    float* p = static_cast<float*>(a.out) + row0 * a.ldo + col0 + lane;
#pragma unroll 8
    for (int i = 0; i < 32; ++i, p += a.ldo) {
      const float y = __uint_as_float(t[i * 32 + (lane ^ i)]);
      *p = EPI == EPI_BIAS_RESID_F32 ? *p + y : y;
    }
  } else {
    constexpr int W = CW / 2, R = 32 / W;  // words of a row, rows at a time
    const int l = lane % W, sub = lane / W;
    // whether even and odd rows of this lane start inside a word
    const uint32_t first = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(a.out) >> 1) +
                           static_cast<uint32_t>(row0 + sub) * static_cast<uint32_t>(a.ldo) + col0;
    const bool in0 = first & 1, in1 = (first + R * static_cast<uint32_t>(a.ldo)) & 1;
    const uint32_t take0 = in0 ? 0x5432 : 0x3210, take1 = in1 ? 0x5432 : 0x3210;
    const bool on0 = !in0 || l < W - 1, on1 = !in1 || l < W - 1;
    uint16_t* p = static_cast<uint16_t*>(a.out) + (row0 + sub) * a.ldo + col0 + 2 * l;
    const long long step = R * a.ldo;
#pragma unroll 4
    for (int i = sub; i < 32; i += 2 * R, p += 2 * step) {
      const uint32_t w0 = __byte_perm(t[i * 32 + (l ^ i)], t[i * 32 + ((l + 1) ^ i)], take0);
      const uint32_t w1 = __byte_perm(t[(i + R) * 32 + (l ^ (i + R))], t[(i + R) * 32 + ((l + 1) ^ (i + R))], take1);
      if (on0) *reinterpret_cast<uint32_t*>(p + in0) = w0;
      if (on1) *reinterpret_cast<uint32_t*>(p + step + in1) = w1;
    }
    // the two ends of such rows, a row a lane
    const uint32_t own = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(a.out) >> 1) +
                         static_cast<uint32_t>(row0 + lane) * static_cast<uint32_t>(a.ldo) + col0;
    if (own & 1) {
      uint16_t* const r = static_cast<uint16_t*>(a.out) + (row0 + lane) * a.ldo + col0;
      r[0] = static_cast<uint16_t>(t[lane * 32 + lane]);
      r[CW - 1] = static_cast<uint16_t>(t[lane * 32 + ((W - 1) ^ lane)] >> 16);
    }
  }
}

// 32 finished columns of a warp's 32 rows, a row a lane: out[row0 + lane, col .. col + 32). part: which
// 64 bytes of a 128-byte staging row (16-bit types take two chunks). NARROW: one chunk of a 16-bit
// type is all the warp has; its rows are 64 bytes, not swizzled. tma: the piece leaves by TMA, else from `base`.
template <int EPI, bool NARROW>
__device__ __forceinline__ void store_chunk(const Args& a, const CUtensorMap* tmC, bool tma, uint8_t* base, uint8_t* piece, int part,
                                            int lane, int row0, int col, float2 (&x)[16]) {
  if constexpr (EPI == EPI_BIAS_GELU_BF16) {
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = gelu2(x[j]);
  }
  if (!tma) {
    uint32_t* const t = reinterpret_cast<uint32_t*>(base);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if constexpr (f32_out<EPI>) {
        t[lane * 32 + ((2 * j) ^ lane)] = __float_as_uint(x[j].x);
        t[lane * 32 + ((2 * j + 1) ^ lane)] = __float_as_uint(x[j].y);
      } else {
        t[lane * 32 + ((16 * part + j) ^ lane)] = pack_bf16x2(x[j].x, x[j].y);
      }
    }
    if (!f32_out<EPI> && !NARROW && part == 0) return;
    __syncwarp();
    store_rows<EPI, f32_out<EPI> || NARROW ? 32 : 64>(a, t, lane, row0, col - 32 * part);
    __syncwarp();
    return;
  }
  // 16-byte pieces of the staging row, swizzled as the box is
  uint8_t* const rowp = piece + lane * (NARROW ? 64 : 128);
  if constexpr (f32_out<EPI>) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      *reinterpret_cast<float4*>(rowp + ((j ^ (lane & 7)) << 4)) = make_float4(x[2 * j].x, x[2 * j].y, x[2 * j + 1].x, x[2 * j + 1].y);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint4*>(rowp + (NARROW ? j << 4 : ((4 * part + j) ^ (lane & 7)) << 4)) =
          make_uint4(pack_bf16x2(x[4 * j].x, x[4 * j].y), pack_bf16x2(x[4 * j + 1].x, x[4 * j + 1].y),
                     pack_bf16x2(x[4 * j + 2].x, x[4 * j + 2].y), pack_bf16x2(x[4 * j + 3].x, x[4 * j + 3].y));
    if (!NARROW) {
      if (part == 0) return;
      col -= 32;
    }
  }
  fence_async_smem();
  __syncwarp();
  if (elect_one()) {
    if (row0 < a.M) {
      if constexpr (EPI == EPI_BIAS_RESID_F32)
        tma_add_2d(tmC, piece, col, row0);
      else
        tma_store_2d(tmC, piece, col, row0);
    }
    bulk_commit();
  }
}

template <bool PAIR, int BN, int EPI>
__global__ void __launch_bounds__(THREADS, 1)
    gemm_fp8_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                    const __grid_constant__ CUtensorMap tmC, const __grid_constant__ Args a) {
  using T = Tile<PAIR, BN>;
  constexpr int S = T::stages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sA = smem;
  uint8_t* sB = smem + S * A_STAGE;
  uint8_t* pieces = smem + S * T::stage;
  float* sbias = reinterpret_cast<float*>(pieces + PIECES);
  uint64_t* full = reinterpret_cast<uint64_t*>(sbias + EPI_WARPS * 32);
  uint64_t* empty = full + MAX_STAGES;
  uint64_t* tfull = empty + MAX_STAGES;  // [accumulator]
  uint64_t* tempty = tfull + T::accs * T::halves;
  uint64_t* drain = tempty + T::accs * T::halves;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);

  const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int rank = PAIR ? warp_uniform(static_cast<int>(cluster_ctarank())) : 0;
  const int t_start = PAIR ? warp_uniform(static_cast<int>(cluster_id_x())) : static_cast<int>(blockIdx.x);
  const int t_stride = PAIR ? warp_uniform(static_cast<int>(cluster_count_x())) : static_cast<int>(gridDim.x);
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < T::accs * T::halves; ++i) {
      mbar_init(&tfull[i], 1);
      mbar_init(&tempty[i], (PAIR ? 2 : 1) * EPI_WARPS / T::halves);
    }
    mbar_init(drain, 1);
    fence_barrier_init();
  }
  if (warp == 0) {
    if constexpr (PAIR) {
      tmem_alloc_pair(tmem_slot, TMEM_COLS);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(tmem_slot, TMEM_COLS);
      tmem_relinquish();
    }
  }
  if (warp == 1 && elect_one()) {
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
  }
  tc_fence_before();
  if constexpr (PAIR)
    cluster_sync_all();
  else
    __syncthreads();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(static_cast<int>(*tmem_slot));
  pdl_wait();
  pdl_trigger();

  const int nt = (a.N + BN - 1) / BN, tiles = (a.M + T::tm - 1) / T::tm * nt, nkb = a.nkb;
  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
  if (warp == 0) {
    // ------------------------------------------------------------ producer
    if (elect_one()) {
      uint32_t seq = 0;
      bool ok = true;
      for (int t = t_start; t < tiles && ok; t += t_stride) {
        const int m0 = t / nt * T::tm + rank * BM, n0 = t % nt * BN + rank * (T::half / 2);
        for (int kb = 0; kb < nkb; ++kb, ++seq) {
          const uint32_t s = seq % S;
          ok = mbar_wait<true>(&empty[s], ((seq / S) & 1) ^ 1);
          if (!ok) break;
          if constexpr (PAIR) {
            const uint32_t lead = cluster_map(smem_addr(&full[s]), 0);
            if (rank == 0) mbar_expect_tx(&full[s], 2 * T::stage);
            tma_load_2d_pair(sA + s * A_STAGE, &tmA, lead, kb * BK, m0);
            for (int h = 0; h < T::halves; ++h)  // (each half's columns from both CTAs)
              tma_load_2d_pair(sB + s * T::b_stage + h * (T::b_stage / T::halves), &tmB, lead, kb * BK, n0 + h * T::half);
          } else {
            mbar_expect_tx(&full[s], T::stage);
            tma_load_2d(sA + s * A_STAGE, &tmA, &full[s], kb * BK, m0);
            tma_load_2d(sB + s * T::b_stage, &tmB, &full[s], kb * BK, n0);
          }
        }
      }
      if (!ok) record_status(a.status, ELASTO_ERR_TIMEOUT);
      // all copies have landed before the CTA exits (a pair's are counted on the even CTA's barriers)
      if (rank == 0)
        for (uint32_t q = seq > S ? seq - S : 0; q < seq; ++q) mbar_wait<true>(&full[q % S], (q / S) & 1);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    if (rank == 0) {
      const uint32_t idesc = idesc_e4m3_f32(T::tm, T::half);
      uint32_t seq = 0;
      bool ok = true;
      for (int t = t_start; t < tiles && ok; t += t_stride)
        for (int kb = 0; kb < nkb; ++kb, ++seq) {
          const uint32_t s = seq % S, acc = seq % T::accs;
          ok = mbar_wait_warp<true>(&full[s], (seq / S) & 1);
          if (!ok) break;
          const uint32_t a_lo = sdesc_lo(smem_addr(sA + s * A_STAGE), 16), b_lo = sdesc_lo(smem_addr(sB + s * T::b_stage), 16);
#pragma unroll
          for (int h = 0; h < T::halves; ++h) {
            const uint32_t i = acc * T::halves + h;
            ok = mbar_wait_warp<true>(&tempty[i], ((seq / T::accs) & 1) ^ 1);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < BK / 32; ++k) {
              const uint32_t b = b_lo + h * (T::b_stage / T::halves / 16) + 2 * k;
              if constexpr (PAIR)
                tc_mma_f8_pair_warp_lo(tmem + i * T::half, a_lo + 2 * k, b, sdesc_sw128_hi(1024), idesc, k != 0);
              else
                tc_mma_f8_warp_lo(tmem + i * T::half, a_lo + 2 * k, b, sdesc_sw128_hi(1024), idesc, k != 0);
            }
            if constexpr (PAIR)
              tc_commit_pair_multicast_warp(&tfull[i], 0x3);
            else
              tc_commit_warp(&tfull[i]);
          }
          if (!ok) break;
          if constexpr (PAIR)
            tc_commit_pair_multicast_warp(&empty[s], 0x3);
          else
            tc_commit_warp(&empty[s]);
        }
      if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
      if (seq > 0) {
        if constexpr (PAIR) {
          if (elect_one()) tc_commit_pair(drain);
        } else {
          tc_commit_warp(drain);
        }
        mbar_wait_warp<true>(drain, 0);
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------ sums and epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_MANY));
    constexpr int C = T::cols;
    const int q = warp & 3, h = (warp - 4) >> 2;
    const uint32_t tm = tmem + (static_cast<uint32_t>(q * 32) << 16) + h * C;
    uint8_t* const piece = pieces + (warp - 4) * 2 * PIECE;
    float* const sb = sbias + (warp - 4) * 32;
    uint32_t seq = 0;
    bool ok = true;
    // scales of the first two blocks and the bias of a tile, requested before the tile ahead of it is stored
    const float *as, *ws;
    float sa0, sw0, sa1, sw1, bias[C / 32];
    auto request = [&](int t) {
      if (t >= tiles) return;
      const int row = min(t / nt * T::tm + rank * BM + q * 32 + lane, a.M - 1), col = t % nt * BN + h * C;
      as = a.a_scale + row;
      ws = a.w_scale + static_cast<size_t>(min(col, a.N - 1) / 128) * nkb;
      const int k1 = nkb > 1 ? 1 : 0;
      sa0 = __ldg(as), sw0 = __ldg(ws), sa1 = __ldg(as + k1 * a.lds), sw1 = __ldg(ws + k1);
#pragma unroll
      for (int c = 0; c < C / 32; ++c)
        bias[c] = a.bias && col + 32 * c + lane < a.N ? __ldg(a.bias + col + 32 * c + lane) : 0.0f;
    };
    request(t_start);
    for (int t = t_start; t < tiles && ok; t += t_stride) {
      const int row0 = t / nt * T::tm + rank * BM + q * 32, col0 = t % nt * BN + h * C;
      float2 acc[C / 2];
#pragma unroll
      for (int j = 0; j < C / 2; ++j) acc[j] = make_float2(0.0f, 0.0f);
      float s0 = sa0 * sw0, s1 = sa1 * sw1;  // of this block and the next; the one after is on its way
      for (int kb = 0; kb < nkb; ++kb, ++seq) {
        const uint32_t p = seq % T::accs, pb = T::halves == 2 ? 2 * p + h : p;  // accumulator, and its barrier
        const float sa = kb + 2 < nkb ? __ldg(as + (kb + 2) * a.lds) : 0.0f, sw = kb + 2 < nkb ? __ldg(ws + kb + 2) : 0.0f;
        ok = __all_sync(0xffffffffu, mbar_wait<true>(&tfull[pb], (seq / T::accs) & 1));
        if (!ok) break;
        tc_fence_after();
        const float2 s2 = make_float2(s0, s0);
        auto add = [&](const uint32_t (&v)[32], int c) {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            acc[16 * c + j] = fma2(make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), s2, acc[16 * c + j]);
        };
        auto release = [&] {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if constexpr (PAIR)
              mbar_arrive_cluster(cluster_map(smem_addr(&tempty[pb]), 0));
            else
              mbar_arrive(&tempty[pb]);
          }
        };
        uint32_t v[2][32];
        tmem_ld_32x32b_x32(tm + p * BN, v[0]);
        if constexpr (C >= 64) tmem_ld_32x32b_x32(tm + p * BN + 32, v[1]);
        tmem_ld_wait();
        if constexpr (C < 128) release();
        add(v[0], 0);
        if constexpr (C == 128) tmem_ld_32x32b_x32(tm + p * BN + 64, v[0]);
        if constexpr (C >= 64) add(v[1], 1);
        if constexpr (C == 128) {
          tmem_ld_32x32b_x32(tm + p * BN + 96, v[1]);
          tmem_ld_wait();
          release();
          add(v[0], 2);
          add(v[1], 3);
        }
        s0 = s1;
        s1 = sa * sw;
      }
      if (!ok) break;
      float b[C / 32];
#pragma unroll
      for (int c = 0; c < C / 32; ++c) b[c] = bias[c];
      request(t + t_stride);
      constexpr bool narrow = C == 32 && !f32_out<EPI>;
      constexpr int per = f32_out<EPI> || narrow ? 1 : 2;  // chunks of a staging piece
#pragma unroll
      for (int c = 0; c < C / 32; ++c) {
        const int col = col0 + 32 * c, part = c % per;
        if (col - 32 * part >= a.N) continue;
        float2 x[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = acc[16 * c + j];
        if (a.bias) {  // broadcast from shared memory: shuffles took a quarter of the epilogue
          __syncwarp();
          sb[lane] = b[c];
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            const float4 b4 = reinterpret_cast<const float4*>(sb)[j / 2];
            x[j] = add2(x[j], make_float2(b4.x, b4.y));
            x[j + 1] = add2(x[j + 1], make_float2(b4.z, b4.w));
          }
        }
        const bool tma = col - 32 * part + 32 * per <= a.tma_cols;
        if (part == 0) {
          // The piece's last store has read it. The two pieces take turns within a tile only: the tile before may have
          // ended in this one (one piece a tile, or an odd number at the last columns).
          if (elect_one()) {
            if (c == 0 || !tma)
              bulk_wait_read<0>();
            else
              bulk_wait_read<1>();
          }
          __syncwarp();
        }
        store_chunk<EPI, narrow>(a, &tmC, tma, piece, piece + (c / per & 1) * PIECE, part, lane, row0, col, x);
      }
    }
    if (elect_one()) bulk_wait_all();
    if (!ok && lane == 0) record_status(a.status, ELASTO_ERR_TIMEOUT);
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_sync_all();
  if (warp == 0) {
    __syncwarp();
    tc_fence_after();
    if constexpr (PAIR)
      tmem_dealloc_pair(tmem, TMEM_COLS);
    else
      tmem_dealloc(tmem, TMEM_COLS);
  }
}

template <bool PAIR, int BN, int EPI>
cudaError_t launch(const Fp8Gemm& g, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc, const Args& a, cudaStream_t s) {
  using T = Tile<PAIR, BN>;
  const long long tiles = (g.M + T::tm - 1LL) / T::tm * ((g.N + BN - 1LL) / BN);
  if constexpr (PAIR) {
    int pairs = 0;
    const cudaError_t e = max_cta_pairs(reinterpret_cast<const void*>(gemm_fp8_kernel<PAIR, BN, EPI>), THREADS, T::smem, &pairs);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see launch_pdl
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(static_cast<unsigned>(2 * std::min<long long>(tiles, pairs)));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = T::smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, gemm_fp8_kernel<PAIR, BN, EPI>, ta, tb, tc, a);
  } else {
    return launch_pdl(gemm_fp8_kernel<PAIR, BN, EPI>, dim3(static_cast<unsigned>(std::min<long long>(tiles, num_sms()))),
                      dim3(THREADS), T::smem, s, ta, tb, tc, a);
  }
}

template <bool PAIR, int BN>
cudaError_t launch_epi(const Fp8Gemm& g, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tc, const Args& a, cudaStream_t s) {
  switch (g.epi) {
    case EPI_BIAS_BF16: return launch<PAIR, BN, EPI_BIAS_BF16>(g, ta, tb, tc, a, s);
    case EPI_BIAS_GELU_BF16: return launch<PAIR, BN, EPI_BIAS_GELU_BF16>(g, ta, tb, tc, a, s);
    case EPI_BIAS_RESID_F32: return launch<PAIR, BN, EPI_BIAS_RESID_F32>(g, ta, tb, tc, a, s);
    default: return launch<PAIR, BN, EPI_BIAS_F32>(g, ta, tb, tc, a, s);
  }
}

template <bool PAIR, int BN, int EPI>
void set_attributes(cudaError_t* e) {
  auto* f = gemm_fp8_kernel<PAIR, BN, EPI>;
  if (*e == cudaSuccess) *e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, Tile<PAIR, BN>::smem);
  cudaFuncAttributes at{};
  if (*e == cudaSuccess) *e = cudaFuncGetAttributes(&at, f);
  // the register split adds up only if the kernel was built with the launch's count
  if (*e == cudaSuccess && at.numRegs != REGS) *e = cudaErrorInvalidConfiguration;
}
template <bool PAIR, int BN>
void set_attributes_of(cudaError_t* e) {
  set_attributes<PAIR, BN, EPI_BIAS_BF16>(e);
  set_attributes<PAIR, BN, EPI_BIAS_GELU_BF16>(e);
  set_attributes<PAIR, BN, EPI_BIAS_RESID_F32>(e);
  set_attributes<PAIR, BN, EPI_BIAS_F32>(e);
}

// Estimated microseconds with 128 x 64, 128 x 128 or (CTA pairs) 256 x 256 tiles: waves of tiles, each
// its k-blocks and an epilogue. Fitted to launches of 1 to 50432 rows: 256 x 8192 x 8192 57 us in two
// waves of 64 columns, 23 in one of 128; 1000 x 1000 x 1160 6.2 us with 64 columns, 6.8 with 128.
double tile_cost(const Fp8Gemm& g, int nkb, int bn) {
  const int tm = bn == 256 ? 256 : 128, units = bn == 256 ? num_sms() / 2 : num_sms();
  const long long tiles = (g.M + tm - 1LL) / tm * ((g.N + bn - 1LL) / bn), waves = (tiles + units - 1) / units;
  const double block = bn == 256 ? 0.40 : bn == 128 ? 0.32 : 0.30, epilogue = bn == 256 ? 2.1 : bn == 128 ? 1.0 : 0.4;
  return 2.2 + waves * (nkb * block + epilogue);
}

int tile_columns(const Fp8Gemm& g, int nkb) {
  int bn = 64;
  for (int n : {128, 256})
    if (tile_cost(g, nkb, n) < tile_cost(g, nkb, bn)) bn = n;
  return bn;
}

cudaError_t init_attributes() {
  cudaError_t e = cudaSuccess;
  set_attributes_of<true, 256>(&e);
  set_attributes_of<false, 128>(&e);
  set_attributes_of<false, 64>(&e);
  return e == cudaSuccess ? gemm_fp8_tokens_init_attributes() : e;
}

}  // namespace

elasto_fp8_tile gemm_fp8_tile(const Fp8Gemm& g) {
  const int nkb = static_cast<int>((g.K + BK - 1LL) / BK), bn = tile_columns(g, nkb);
  if (gemm_fp8_tokens_cost(g, nkb) < tile_cost(g, nkb, bn)) return gemm_fp8_tokens_tile(g, nkb);
  return {bn == 256 ? 256 : 128, bn, bn == 256, 0};
}

elasto_status gemm_fp8_launch(const Fp8Gemm& g, cudaStream_t s) {
  if ((g.M + BM - 1LL) / BM * ((g.N + 63LL) / 64) > 0x7fffffffLL) {
    set_error("elasto_op_gemm_fp8: output too large");
    return ELASTO_ERR_UNSUPPORTED;
  }
  static DeviceOnce once;
  ELASTO_CUDA_TRY(once(init_attributes));
  const int nkb = static_cast<int>((g.K + BK - 1LL) / BK);
  const int bn = tile_columns(g, nkb);
  if (gemm_fp8_tokens_cost(g, nkb) < tile_cost(g, nkb, bn)) return gemm_fp8_tokens_launch(g, s);
  Args a{};
  a.M = g.M, a.N = g.N, a.K = g.K, a.nkb = nkb;
  a.a_scale = g.a_scale, a.lds = g.lds, a.w_scale = g.w_scale, a.bias = g.bias;
  a.out = g.out, a.ldo = g.ldo, a.status = g.status;
  const int size = g.epi == EPI_BIAS_RESID_F32 || g.epi == EPI_BIAS_F32 ? 4 : 2;
  const uintptr_t starts = reinterpret_cast<uintptr_t>(g.out) | static_cast<uintptr_t>(g.ldo * size);
  // (TMA stores whole 16-byte words of a row: where the last column is inside one, its piece leaves value by value)
  const bool tma = starts % 16 == 0;
  a.tma_cols = !tma ? 0 : static_cast<uintptr_t>(g.N) * size % 16 == 0 ? 0x7fffffff : g.N;
  CUtensorMap ta, tb, tc{};
  const uint64_t od[2] = {static_cast<uint64_t>(g.N), static_cast<uint64_t>(g.M)}, os[1] = {static_cast<uint64_t>(g.ldo) * size};
  const bool narrow = bn == 64 && size == 2;
  const uint32_t ob[2] = {narrow ? 32u : 128u / size, 32};
  if ((tma && !encode_tmap_plain(&tc, g.out, 2, od, os, ob, size == 4, !narrow)) ||
      !encode_tmap_8(&ta, g.A, g.K, g.M, g.lda, BM) || !encode_tmap_8(&tb, g.W, g.K, g.N, g.ldw, bn == 256 ? 64 : bn)) {
    set_error("elasto_op_gemm_fp8: cuTensorMapEncodeTiled failed (alignment or size)");
    return ELASTO_ERR_UNSUPPORTED;
  }
  if (bn == 256) {
    ELASTO_CUDA_TRY((launch_epi<true, 256>(g, ta, tb, tc, a, s)));
  } else if (bn == 128) {
    ELASTO_CUDA_TRY((launch_epi<false, 128>(g, ta, tb, tc, a, s)));
  } else {
    ELASTO_CUDA_TRY((launch_epi<false, 64>(g, ta, tb, tc, a, s)));
  }
  return ELASTO_OK;
}

}  // namespace elasto
