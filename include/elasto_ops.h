/*
 * elasto_ops.h -- stateless kernel-level entry points of libelasto. The first
 * part has the steps of the DN forward (Section 4.1, Eq. 2-7) that elasto_forward
 * composes, so that every kernel can be checked on its own against the fp64
 * definition of that step. The second part has operators for a caller's own attention
 * sublayers over long sequences with 8-bit weights; no model call runs them.
 *
 * All pointers are CUDA device memory of the current device, row-major,
 * caller-owned; in the first part 16-byte aligned, in the second as each call says. Calls are asynchronous on `stream` (void* =
 * cudaStream_t). `status_device` (nullable) is an int the kernels set to
 * ELASTO_ERR_TIMEOUT if one of their bounded device-side waits gives up (and to
 * what else a call says of it). Errors: ELASTO_ERR_INVALID_ARG for null pointers, non-positive or
 * unsupported sizes; ELASTO_ERR_CUDA for launch failures.
 */
#ifndef ELASTO_OPS_H
#define ELASTO_OPS_H

#include "elasto.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Epilogues fused into the tensor-core GEMM (acc = A W^T in fp32). */
typedef enum {
  ELASTO_EPI_BIAS_BF16 = 0,       /* out bf16 = acc + bias                  (QKV, Eq. 2) */
  ELASTO_EPI_BIAS_GELU_BF16 = 1,  /* out bf16 = GELU(acc + bias)            (FC1, Eq. 5): x Phi(x) in a fitted form,
                                     off by at most 2.52e-5 (more than rounding where the result is small) */
  ELASTO_EPI_BIAS_RESID_F32 = 2,  /* out fp32 += acc + bias                 (proj, FC2: residual) */
  ELASTO_EPI_BIAS_F32 = 3,        /* out fp32 = acc + bias */
  ELASTO_EPI_BIAS_RELU_BF16 = 4,  /* out bf16 = ReLU(acc + bias)            (conv + folded BN) */
  ELASTO_EPI_BIAS_RESID_RELU_BF16 = 5, /* out bf16 = ReLU(acc + bias + resid) (block output) */
  /* The same with A, W, resid and out in IEEE f16 (ResNet-50 path: f16 has
   * 3 more mantissa bits than bf16 at the same tensor-core rate) */
  ELASTO_EPI_BIAS_RELU_F16 = 6,       /* out f16 = ReLU(acc + bias)             (conv + folded BN) */
  ELASTO_EPI_BIAS_F16 = 7,            /* out f16 = acc + bias                   (shortcut projection) */
  ELASTO_EPI_BIAS_RESID_RELU_F16 = 8  /* out f16 = ReLU(acc + bias + resid)     (block output) */
} elasto_epilogue;

/* out[M,N] = epilogue(A[M,K] W[N,K]^T): A, W bf16 (f16 for the *_F16
 * epilogues), K contiguous; bias fp32 [N] or NULL (= 0); resid [M,N] of the
 * same 16-bit type only for the ..._RESID_RELU epilogues. Output
 * row stride is N. Requires K % 8 == 0, N % 2 == 0, M, N, K >= 1 (K may be 0:
 * then acc = 0). tcgen05 MMA (M = 128 tiles), TMA-fed, persistent grid. */
elasto_status elasto_op_gemm(void* stream, const void* A, const void* W, const float* bias, void* out,
                             const void* resid, int M, int N, int K, int epilogue, int* status_device);

/* y bf16 [rows, d] = LayerNorm(x fp32 [rows, d]) * gamma + beta, eps = 1e-6,
 * biased variance, statistics in fp32 (one warp per row). d % 64 == 0,
 * d <= 4096. */
elasto_status elasto_op_layernorm(void* stream, const float* x, const float* gamma, const float* beta,
                                  void* y, int rows, int d);

/* y fp32 [rows, cols] = softmax over each row of x fp32 [rows, cols]
 * (exp(x - max) / sum, one warp per row, warp-shuffle reductions). */
elasto_status elasto_op_softmax(void* stream, const float* x, float* y, int rows, int cols);

/* k x k convolution (Eq. 7's conv over the kept channels) as an implicit
 * GEMM: out f16 [B, Ho, Wo, N] = act(conv(x) + bias), Ho = (H + 2 pad - k) /
 * stride + 1 (likewise Wo), act = ReLU if relu != 0 else identity.
 *   x f16 [B, H, W, C] NHWC, C % 8 == 0;
 *   w f16 [N, k, k, Cp] with Cp = 16 if C <= 16, else C rounded up to 64;
 *     channels >= C zero (the packed layout the ResNet path uses: a k-block
 *     of the tensor-core GEMM is one 64-channel group of a tap, or for at most
 *     16 channels one tap);
 *   bias fp32 [N] or NULL. N % 2 == 0, stride 1 or 2.
 * No im2col buffer: x is read by 4-D TMA tiles (padding read as zeros). At
 * stride 1, N % 8 == 0 and where it is estimated faster, one tile per block of
 * output pixels and channel group holds the pixels of all taps (its halo); else
 * there is one per k-block, the stride by TMA traversal strides. */
elasto_status elasto_op_conv2d(void* stream, const void* x, int B, int H, int W, int C, const void* w, int N, int k,
                               int stride, int pad, const float* bias, int relu, void* out, int* status_device);

/* The tiles that elasto_op_gemm / elasto_op_conv2d cut a call of this size into
 * on the current device (16-byte aligned operands). Nothing is launched. */
typedef struct {
  int columns; /* output columns (channels) of a tile */
  int pair;    /* 1: a pair of CTAs shares a tile of 256 rows; 0: a CTA has 128 rows of its own */
  int halo;    /* 1: conv2d on halo tiles (always pairs); 0: a box of x per k-block */
  int ahead;   /* pieces of 32 rows x 128 bytes of a residual that an epilogue warp reads ahead;
                  0: no residual, or (RESID_F32) one that the stores add to */
} elasto_tile;
elasto_status elasto_op_gemm_tile(int M, int N, int K, int epilogue, elasto_tile* tile);
elasto_status elasto_op_conv2d_tile(int B, int H, int W, int C, int N, int k, int stride, int pad, elasto_tile* tile);

/* Multi-head attention over the kept heads (Eq. 3), all heads of width 64:
 * qkv bf16 [batch, n, 3, heads, 64] (q | k | v blocks, head-major, as the
 * QKV GEMM writes them) -> out bf16 [batch, n, heads * 64] (heads
 * concatenated in order, Eq. 2). Scale 1/8. 1 <= n <= 256. */
elasto_status elasto_op_attention(void* stream, const void* qkv, void* out, int batch, int n, int heads,
                                  int* status_device);

/* ------------------------------------------------------------------------
 * An attention sublayer over long token sequences with 8-bit weights: rows to
 * e4m3, products of e4m3 rows, norms and positions of queries and keys, and
 * attention in a sliding window. Forward only, like the rest of the library.
 * Strides are in elements. A call allocates nothing and keeps nothing; it may
 * be captured into a graph. */

/* Operand type of these calls besides ELASTO_F32 and ELASTO_BF16: IEEE f16. */
enum { ELASTO_F16 = 2 };

/* q e4m3 [rows, cols] and scale fp32 [ceil(cols / 128), rows]: each row of x
 * (x_type ELASTO_F32, _BF16 or _F16) in blocks of 128 columns, the last block
 * what is left. Of a block, in fp32 arithmetic:
 *   a = max(largest |x|, 2^-100),  scale[b, r] = a / 448,
 *   q = x * (448 / a) rounded to the nearest e4m3 (ties to even),
 * so x is about q * scale. A NaN in a block makes its scale and all its values
 * NaN; an infinity makes its scale infinite, its own value NaN and the others 0.
 * ldx, ldq >= cols: row strides; lds >= rows: stride of scale's rows. At most 2^31 - 128
 * columns and 2^31 - 1 blocks. Columns past cols are neither read nor written. q and scale
 * may not overlap x. x, q and scale need their types'
 * alignment; 16-byte rows of x and 8-byte rows of q are read and written wide. */
elasto_status elasto_op_quantize_fp8(void* stream, const void* x, int x_type, long long ldx, void* q, long long ldq,
                                     float* scale, long long lds, int rows, int cols);

/* out[M, N] = epilogue(acc), acc[m, n] = sum over blocks b of 128 columns of
 *   a_scale[b, m] * w_scale[n / 128, b] * (sum over the block of A[m, k] W[n, k])
 * in fp32. A e4m3 [M, K] (row stride lda) with a_scale fp32 [ceil(K / 128), M]
 * (row stride lds >= M), as elasto_op_quantize_fp8 makes them; W e4m3 [N, K] (row
 * stride ldw) with w_scale fp32 [ceil(N / 128), ceil(K / 128)], dense; bias fp32 [N] or
 * NULL. epilogue: ELASTO_EPI_BIAS_BF16, _BIAS_GELU_BF16 (the same fitted GELU), _BIAS_F32, or
 * _BIAS_RESID_F32 (out += acc + bias); out has row stride ldo >= N, columns past N are left alone,
 * and may not overlap the inputs.
 * M, N, K >= 1, M and N at most 2^31 - 256, of any remainder; A and W 16-byte aligned with lda and ldw multiples of
 * 16 (>= K); columns past K are not read. The result does not depend on lda, ldw,
 * ldo, and is the same in every call. */
elasto_status elasto_op_gemm_fp8(void* stream, const void* A, long long lda, const float* a_scale, long long lds,
                                 const void* W, long long ldw, const float* w_scale, const float* bias, void* out,
                                 long long ldo, int M, int N, int K, int epilogue, int* status_device);

/* The tiles that elasto_op_gemm_fp8 cuts a call of this size into on the current
 * device. Nothing is launched. */
typedef struct {
  int rows;    /* of A in a tile */
  int columns; /* of out */
  int pair;    /* 1: a pair of CTAs shares a tile */
  int split;   /* few rows of A: CTAs (a cluster) that share a tile's blocks of K; 0: the form for many rows */
} elasto_fp8_tile;
elasto_status elasto_op_gemm_fp8_tile(int M, int N, int K, elasto_fp8_tile* tile);

/* Queries and keys of `rows` tokens: each head of each row divided by the root
 * of its mean square (plus eps), multiplied by the gain of its channel, and its
 * first rot_dim channels rotated by the row's position; all in fp32, rounded
 * once. Keys, and values unchanged, optionally go to the rows of a cache.
 *   y = x * rsqrt(mean(x^2) + eps) * gain      (a head of zeros with eps 0: NaN)
 *   pair j of rot_dim / 2: channels (j, j + rot_dim / 2), or (2 j, 2 j + 1) if
 *   interleaved != 0, (a, b) -> (a c - b s, b c + a s), with c and s from row
 *   positions[r] of cos_sin: rot_dim / 2 cosines, then rot_dim / 2 sines.
 * Head h of row r of q is at q + r * q_row + h * q_head, and so on: the columns of
 * a QKV product's output are taken as they are. An output may be its own input
 * (the same strides, and for k and v no slots); else it must not overlap the inputs.
 * k and v of row r go to row slots[r] of k_out and v_out (slots NULL: row r). A
 * negative slot stores neither. Slots that are stored must differ from one another.
 * A row with a position outside [0, n_positions), or a slot >= n_slots, is left
 * out, and *status_device is set to ELASTO_ERR_INVALID_ARG.
 * Refused: head_dim not a multiple of 8 up to 256; rot_dim not a multiple of 16
 * up to head_dim (0: no rotation); strides that are no multiples of 8; data not
 * 16-byte aligned. */
typedef struct {
  int dtype; /* of q, k, v and the outputs: ELASTO_BF16 or ELASTO_F16 */
  int rows, heads_q, heads_k, head_dim, rot_dim, interleaved;
  float eps; /* >= 0 */
  const void* q; /* heads_q heads (0: no queries, q and q_out are not used) */
  long long q_row, q_head;
  const void* k; /* heads_k heads (0: no keys and values) */
  long long k_row, k_head;
  const void* v; /* heads_k heads, copied to v_out; or NULL */
  long long v_row, v_head;
  void* q_out;
  long long q_out_row, q_out_head;
  void* k_out;
  long long k_out_row, k_out_head;
  void* v_out;
  long long v_out_row, v_out_head;
  const float* q_gain; /* [head_dim], or NULL: ones */
  const float* k_gain;
  const float* cos_sin; /* [n_positions, rot_dim], 16-byte aligned (rot_dim 0: not used, nor are positions) */
  const int32_t* positions; /* [rows] */
  int n_positions;
  const int32_t* slots; /* [rows], or NULL */
  int n_slots;
} elasto_qk_norm_rope_args;
elasto_status elasto_op_qk_norm_rope(void* stream, const elasto_qk_norm_rope_args* args, int* status_device);

/* Attention of `batch` sequences in a sliding window, the first tokens staying
 * visible. A sequence with nq queries and nk keys has its queries at the last
 * positions: query i at p = nk - nq + i. It sees key j, 0 <= j < nk, if
 *   causal != 0:  j <= p and (j >= p - window or j < sinks);
 *   causal == 0:  |j - p| <= window or j < sinks or p < sinks (class tokens and
 *                 the like: seen by all, and seeing all);
 * window < 0: no limit. A query before the first key (p < 0) sees nothing.
 *   out = softmax over the visible keys of (scale q . k), times v;
 * a query that sees nothing gets zeros. Keys and values that no query sees, and
 * NaN or infinite ones at places hidden from a query, do not change its result. A
 * channel in which a query sees infinite or NaN values gets the sum of these, however
 * small their probabilities (NaN in any case where a score is NaN or +infinity, or all are -infinity).
 * heads is a multiple of heads_kv: head h reads key head h / (heads / heads_kv).
 * head_dim: a multiple of 8 up to 128. Scores, softmax statistics and sums in fp32, exp2 by
 * the hardware's approximation; the probabilities are rounded to the operand type for the
 * product with v, their sum is of the unrounded ones.
 * Queries: sequence b has the rows q_start[b] to q_start[b + 1] of q and out, at
 *   most max_queries; q_start NULL: max_queries rows each. q and out have q_rows rows
 *   (at most 2^30, as kv_rows).
 * Keys: packed, the rows kv_start[b] to kv_start[b + 1] of k and v, which have
 *   kv_rows rows; or (kv_start NULL) in a cache of kv_rows rows per sequence, k_batch
 *   and v_batch apart, the first kv_len[b] of them (kv_len NULL: max_keys). At most
 *   max_keys each; max_keys <= kv_rows.
 * Lengths on the device past these limits are cut to them; nothing is read or
 * written outside them. Rows of out that belong to no sequence are left as they were.
 * max_queries == 1 runs the single-token form; few queries against many keys, and single
 * tokens, share the keys out over several SMs and join their results in a fixed order.
 * *status_device is set to ELASTO_ERR_TIMEOUT if a device-side wait gives up.
 * Strides of q, k, v and out are multiples of 8, the data is 16-byte aligned.
 * out may not overlap the inputs. */
typedef struct {
  int dtype; /* of q, k, v and out: ELASTO_BF16 or ELASTO_F16 */
  int batch, heads, heads_kv, head_dim;
  int causal, window, sinks;
  float scale; /* > 0, at most 2.3e38 */
  int max_queries;
  long long q_rows;
  const int32_t* q_start; /* [batch + 1] or NULL */
  const void* q;
  long long q_row, q_head;
  void* out;
  long long out_row, out_head;
  int max_keys;
  long long kv_rows;
  const int32_t* kv_start; /* [batch + 1] or NULL */
  const int32_t* kv_len;   /* [batch] or NULL; only without kv_start */
  const void* k;
  long long k_batch, k_row, k_head;
  const void* v;
  long long v_batch, v_row, v_head;
} elasto_window_attention_args;
elasto_status elasto_op_window_attention(void* stream, const elasto_window_attention_args* args, int* status_device);

/* Self-test of the bounded device-side wait that every kernel above (and the
 * forward's kernels) uses instead of an unbounded spin: one thread waits on an
 * mbarrier of one arrival. armed != 0: the arrival is made first and the wait
 * returns at once (status untouched). armed == 0: nothing arrives, the wait
 * gives up after its limit (1 s), the kernel writes ELASTO_ERR_TIMEOUT to
 * *status_device (if it still holds 0) and returns; the context stays usable.
 * *elapsed_ns_device (uint64) receives the time waited. */
elasto_status elasto_op_bounded_wait(void* stream, int armed, int* status_device,
                                     unsigned long long* elapsed_ns_device);

/* Self-test of the grid-wide barrier of the one-image one-launch forward
 * (elasto_set_one_launch): a cooperative launch of one block per SM passes
 * two barriers (arrival counter and abort flag in sync_device, 2 uint32 of
 * device scratch, zeroed here on the stream). unreachable != 0: the second
 * barrier waits for arrivals that never come, gives up after its limit (1 s),
 * writes ELASTO_ERR_TIMEOUT to *status_device (if it still holds 0) and
 * raises the abort flag, so every block returns; the context stays usable.
 * *elapsed_ns_device (uint64): block 0's time in the two barriers. */
elasto_status elasto_op_grid_barrier(void* stream, int unreachable, unsigned* sync_device, int* status_device,
                                     unsigned long long* elapsed_ns_device);

#ifdef __cplusplus
}
#endif
#endif /* ELASTO_OPS_H */
