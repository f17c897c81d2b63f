// Stateless kernel-level entry points (elasto_ops.h): each DN forward step on
// its own, so every kernel can be checked against the fp64 definition of that
// step at arbitrary (odd, ragged) shapes.
#include "common.h"
#include "handle.h"
#include "elasto_internal.h"
#include "ptx.cuh"

using namespace elasto;

namespace {

bool aligned(const void* p, unsigned bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
bool strides8(long long a, long long b) { return a % 8 == 0 && b % 8 == 0 && a >= 0 && b >= 0; }
// a strided [rows, heads, head_dim] tensor of 16-bit values
bool tensor16(const void* p, long long row, long long head) { return p && aligned(p, 16) && strides8(row, head); }
elasto_status refuse(const char* what, elasto_status st = ELASTO_ERR_INVALID_ARG) {
  set_error(what);
  return st;
}

// What elasto_op_qk_norm_rope and its form for several axes refuse alike.
template <typename ROPE>
elasto_status check_qk_norm_rope(const ROPE& a, const char* call) {
  auto no = [&](const char* what, elasto_status st = ELASTO_ERR_INVALID_ARG) { return refuse((std::string(call) + what).c_str(), st); };
  if (a.dtype != ELASTO_BF16 && a.dtype != ELASTO_F16) return no(": dtype");
  if (a.rows <= 0 || a.heads_q < 0 || a.heads_k < 0 || a.heads_q + static_cast<long long>(a.heads_k) <= 0 ||
      a.heads_q + 2LL * a.heads_k > 65536)
    return no(": rows or heads");
  if (a.head_dim <= 0 || a.head_dim % 8 != 0 || a.head_dim > 256)
    return no(": head_dim must be a multiple of 8 up to 256", ELASTO_ERR_UNSUPPORTED);
  if (a.rot_dim < 0 || a.rot_dim % 16 != 0 || a.rot_dim > a.head_dim)
    return no(": rot_dim must be a multiple of 16 up to head_dim", ELASTO_ERR_UNSUPPORTED);
  if (!(a.eps >= 0.0f) || a.eps > 3.0e38f) return no(": eps");
  if (a.heads_q > 0 && (!tensor16(a.q, a.q_row, a.q_head) || !tensor16(a.q_out, a.q_out_row, a.q_out_head)))
    return no(": q or q_out (null, alignment or strides)");
  if (a.heads_k > 0 && (!tensor16(a.k, a.k_row, a.k_head) || !tensor16(a.k_out, a.k_out_row, a.k_out_head)))
    return no(": k or k_out (null, alignment or strides)");
  if (a.heads_k > 0 && (a.v || a.v_out) &&
      (!tensor16(a.v, a.v_row, a.v_head) || !tensor16(a.v_out, a.v_out_row, a.v_out_head)))
    return no(": v or v_out (null, alignment or strides)");
  if (a.heads_k > 0 && a.slots && (a.k == a.k_out || (a.v && a.v == a.v_out)))
    return no(": slots with an output that is its own input");
  if ((a.q == a.q_out && a.heads_q > 0 && (a.q_row != a.q_out_row || a.q_head != a.q_out_head)) ||
      (a.k == a.k_out && a.heads_k > 0 && (a.k_row != a.k_out_row || a.k_head != a.k_out_head)) ||
      (a.v && a.v == a.v_out && a.heads_k > 0 && (a.v_row != a.v_out_row || a.v_head != a.v_out_head)))
    return no(": an output that is its own input has other strides");
  if (!aligned(a.q_gain, 16) || !aligned(a.k_gain, 16)) return no(": gains misaligned");
  if (a.rot_dim > 0 && (!a.cos_sin || !aligned(a.cos_sin, 16) || !a.positions || !aligned(a.positions, 4) || a.n_positions <= 0))
    return no(": cos_sin, positions or n_positions");
  if (a.slots && (a.n_slots <= 0 || !aligned(a.slots, 4))) return no(": slots or n_slots");
  return ELASTO_OK;
}

// The sizes of a call with shared prefixes (what its workspace depends on).
elasto_status check_prefix_sizes(const elasto_prefix_attention_args& a, const char* call) {
  auto no = [&](const char* what, elasto_status st = ELASTO_ERR_INVALID_ARG) { return refuse((std::string(call) + what).c_str(), st); };
  if (a.dtype != ELASTO_BF16 && a.dtype != ELASTO_F16) return no(": dtype");
  if (a.batch <= 0 || a.heads <= 0 || a.heads_kv <= 0 || a.heads % a.heads_kv != 0 || a.max_queries <= 0 || a.max_prefix <= 0 || a.max_keys < 0)
    return no(": batch, heads, max_queries, max_prefix or max_keys");
  if (a.head_dim <= 0 || a.head_dim % 8 != 0 || a.head_dim > 128)
    return no(": head_dim must be a multiple of 8 up to 128", ELASTO_ERR_UNSUPPORTED);
  if (a.prefixes <= 0 || (a.prefixes > 1 && !a.seq_start)) return no(": prefixes, or several without seq_start");
  if (a.q_rows <= 0 || a.q_rows > 1 << 30 || a.prefix_rows <= 0 || a.prefix_rows > 1 << 30 || a.max_prefix > a.prefix_rows)
    return no(": q_rows or prefix_rows");
  if (a.max_keys > 0 && (a.kv_rows <= 0 || a.kv_rows > 1 << 30 || (!a.kv_start && a.max_keys > a.kv_rows))) return no(": kv_rows");
  return ELASTO_OK;
}

// The same call with no more keys of a sequence than rows there are: max_keys is a limit, and packed sequences may have fewer
// rows altogether.
elasto_prefix_attention_args with_keys_there_are(const elasto_prefix_attention_args& a) {
  elasto_prefix_attention_args u = a;
  if (u.max_keys > u.kv_rows && u.max_keys > 0) u.max_keys = static_cast<int>(u.kv_rows);
  return u;
}

// The bounded wait every kernel uses (mbar_wait: a time limit, then false),
// on an mbarrier of one arrival. armed != 0: that arrival is made first, so
// the wait returns at once; armed == 0: nothing ever arrives, the wait gives
// up after its limit and the kernel records ELASTO_ERR_TIMEOUT in *status
// and returns, leaving the context usable. *elapsed_ns: how long it waited.
__global__ void bounded_wait_kernel(int armed, int* status, unsigned long long* elapsed_ns) {
  __shared__ __align__(8) uint64_t bar;
  if (threadIdx.x != 0) return;
  mbar_init(&bar, 1);
  fence_barrier_init();
  if (armed) mbar_arrive(&bar);
  const uint64_t t0 = global_timer_ns();
  const bool ok = mbar_wait(&bar, 0);
  *elapsed_ns = global_timer_ns() - t0;
  if (!ok) record_status(status, ELASTO_ERR_TIMEOUT);
}

}  // namespace

extern "C" {

elasto_status elasto_op_bounded_wait(void* stream, int armed, int* status_device,
                                     unsigned long long* elapsed_ns_device) {
  clear_error();
  if (!status_device || !elapsed_ns_device) {
    set_error("elasto_op_bounded_wait: null argument");
    return ELASTO_ERR_INVALID_ARG;
  }
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  bounded_wait_kernel<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(armed, status_device, elapsed_ns_device);
  ELASTO_CUDA_TRY(cudaGetLastError());
  return ELASTO_OK;
}


elasto_status elasto_op_grid_barrier(void* stream, int unreachable, unsigned* sync_device, int* status_device,
                                     unsigned long long* elapsed_ns_device) {
  clear_error();
  if (!sync_device || !status_device || !elapsed_ns_device) {
    set_error("elasto_op_grid_barrier: null argument");
    return ELASTO_ERR_INVALID_ARG;
  }
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  ELASTO_CUDA_TRY(pk_barrier_selftest(static_cast<cudaStream_t>(stream), unreachable, sync_device, status_device,
                                      elapsed_ns_device));
  return ELASTO_OK;
}

elasto_status elasto_op_gemm(void* stream, const void* A, const void* W, const float* bias, void* out,
                             const void* resid, int M, int N, int K, int epilogue, int* status_device) {
  clear_error();
  if (!out || M <= 0 || N <= 0 || K < 0 || (K > 0 && (!A || !W)) || epilogue < 0 || epilogue > 8 ||
      ((epilogue == ELASTO_EPI_BIAS_RESID_RELU_BF16 || epilogue == ELASTO_EPI_BIAS_RESID_RELU_F16) && !resid)) {
    set_error("elasto_op_gemm: invalid arguments");
    return ELASTO_ERR_INVALID_ARG;
  }
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  GemmPlan p;
  st = gemm_plan(&p, static_cast<const bf16*>(A), M, static_cast<const bf16*>(W), N, K, bias, out, N, epilogue,
                 status_device);
  if (st != ELASTO_OK) return st;
  if (epilogue == ELASTO_EPI_BIAS_RESID_RELU_BF16 || epilogue == ELASTO_EPI_BIAS_RESID_RELU_F16) {
    st = gemm_set_residual_source(&p, resid, M);
    if (st != ELASTO_OK) return st;
  }
  ELASTO_CUDA_TRY(gemm_launch(p, M, static_cast<cudaStream_t>(stream)));
  return ELASTO_OK;
}

elasto_status elasto_op_conv2d(void* stream, const void* x, int B, int H, int W, int C, const void* w, int N, int k,
                               int stride, int pad, const float* bias, int relu, void* out, int* status_device) {
  clear_error();
  if (!x || !w || !out || B <= 0 || H <= 0 || W <= 0 || C <= 0 || N <= 0 || k <= 0 || stride <= 0 || pad < 0) {
    set_error("elasto_op_conv2d: invalid arguments");
    return ELASTO_ERR_INVALID_ARG;
  }
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  GemmPlan p;
  st = gemm_plan_conv(&p, x, B, H, W, C, k, stride, pad, w, N, bias, out, N, relu ? EPI_BIAS_RELU_F16 : EPI_BIAS_F16,
                      status_device);
  if (st != ELASTO_OK) return st;
  ELASTO_CUDA_TRY(gemm_launch(p, B, static_cast<cudaStream_t>(stream)));
  return ELASTO_OK;
}

elasto_status elasto_op_gemm_tile(int M, int N, int K, int epilogue, elasto_tile* tile) {
  clear_error();
  if (!tile || M <= 0 || N <= 0 || K < 0 || epilogue < 0 || epilogue > 8) {
    set_error("elasto_op_gemm_tile: invalid arguments");
    return ELASTO_ERR_INVALID_ARG;
  }
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  GemmPlan p;
  bf16* const any = reinterpret_cast<bf16*>(uintptr_t(1) << 20);  // (encoded, never read)
  st = gemm_plan(&p, any, M, any, N, K, nullptr, any, N, epilogue, nullptr);
  if (st != ELASTO_OK) return st;
  const bool ahead = p.epi == EPI_BIAS_RESID_F32 || p.epi == EPI_BIAS_RESID_RELU_BF16 || p.epi == EPI_BIAS_RESID_RELU_F16;
  *tile = {p.args.bn, p.args.pair, 0, ahead ? p.args.cbufs : 0};
  return ELASTO_OK;
}

elasto_status elasto_op_conv2d_tile(int B, int H, int W, int C, int N, int k, int stride, int pad, elasto_tile* tile) {
  clear_error();
  if (!tile || B <= 0 || H <= 0 || W <= 0 || C <= 0 || N <= 0 || k <= 0 || stride <= 0 || pad < 0) {
    set_error("elasto_op_conv2d_tile: invalid arguments");
    return ELASTO_ERR_INVALID_ARG;
  }
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  GemmPlan p;
  void* const any = reinterpret_cast<void*>(uintptr_t(1) << 20);  // (encoded, never read)
  st = gemm_plan_conv(&p, any, B, H, W, C, k, stride, pad, any, N, nullptr, any, N, EPI_BIAS_F16, nullptr);
  if (st != ELASTO_OK) return st;
  *tile = {p.use_halo ? p.halo.bn : p.args.bn, p.use_halo ? 1 : p.args.pair, p.use_halo ? 1 : 0, 0};
  return ELASTO_OK;
}

elasto_status elasto_op_layernorm(void* stream, const float* x, const float* gamma, const float* beta, void* y,
                                  int rows, int d) {
  clear_error();
  if (!x || !gamma || !beta || !y || rows <= 0 || d <= 0) {
    set_error("elasto_op_layernorm: invalid arguments");
    return ELASTO_ERR_INVALID_ARG;
  }
  if (d % 64 != 0 || d > 1024) {
    set_error("elasto_op_layernorm: d must be a multiple of 64 up to 1024");
    return ELASTO_ERR_UNSUPPORTED;
  }
  ELASTO_CUDA_TRY(
      layernorm_launch(x, gamma, beta, static_cast<bf16*>(y), rows, d, d, static_cast<cudaStream_t>(stream)));
  return ELASTO_OK;
}

elasto_status elasto_op_quantize_fp8(void* stream, const void* x, int x_type, long long ldx, void* q, long long ldq,
                                     float* scale, long long lds, int rows, int cols) {
  clear_error();
  if (!x || !q || !scale || rows <= 0 || cols <= 0 || ldx < cols || ldq < cols || lds < rows)
    return refuse("elasto_op_quantize_fp8: null pointer, size or stride");
  if (x_type != ELASTO_F32 && x_type != ELASTO_BF16 && x_type != ELASTO_F16)
    return refuse("elasto_op_quantize_fp8: x_type must be ELASTO_F32, ELASTO_BF16 or ELASTO_F16");
  if (!aligned(x, x_type == ELASTO_F32 ? 4 : 2) || !aligned(scale, 4))
    return refuse("elasto_op_quantize_fp8: x or scale misaligned for its type");
  if (static_cast<long long>(rows) * ((cols + 127LL) / 128) > 0x7fffffffLL)
    return refuse("elasto_op_quantize_fp8: more than 2^31 blocks", ELASTO_ERR_UNSUPPORTED);
  if (cols > 0x7fffffff - 127)  // (the last block's columns would pass an int)
    return refuse("elasto_op_quantize_fp8: more than 2^31 - 128 columns", ELASTO_ERR_UNSUPPORTED);
  if (q == x || scale == x || scale == q) return refuse("elasto_op_quantize_fp8: an output that is x or the other output");
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  ELASTO_CUDA_TRY(quantize_fp8_launch(x, x_type, ldx, static_cast<uint8_t*>(q), ldq, scale, lds, rows, cols,
                                      static_cast<cudaStream_t>(stream)));
  return ELASTO_OK;
}

elasto_status elasto_op_gemm_fp8(void* stream, const void* A, long long lda, const float* a_scale, long long lds,
                                 const void* W, long long ldw, const float* w_scale, const float* bias, void* out,
                                 long long ldo, int M, int N, int K, int epilogue, int* status_device) {
  clear_error();
  if (!A || !a_scale || !W || !w_scale || !out || M <= 0 || N <= 0 || K <= 0 || lda < K || ldw < K || lds < M || ldo < N)
    return refuse("elasto_op_gemm_fp8: null pointer, size or stride");
  if (M > 0x7fffffff - 255 || N > 0x7fffffff - 255)  // (a last tile's rows and columns would pass an int)
    return refuse("elasto_op_gemm_fp8: M or N above 2^31 - 256", ELASTO_ERR_UNSUPPORTED);
  if (!aligned(A, 16) || !aligned(W, 16) || lda % 16 != 0 || ldw % 16 != 0)
    return refuse("elasto_op_gemm_fp8: A and W need 16-byte aligned rows");
  if (epilogue != ELASTO_EPI_BIAS_BF16 && epilogue != ELASTO_EPI_BIAS_GELU_BF16 && epilogue != ELASTO_EPI_BIAS_RESID_F32 &&
      epilogue != ELASTO_EPI_BIAS_F32)
    return refuse("elasto_op_gemm_fp8: epilogue");
  const bool f32 = epilogue == ELASTO_EPI_BIAS_RESID_F32 || epilogue == ELASTO_EPI_BIAS_F32;
  if (!aligned(out, f32 ? 4 : 2) || !aligned(a_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4))
    return refuse("elasto_op_gemm_fp8: out, a scale or the bias misaligned for its type");
  if (out == A || out == W || out == a_scale || out == w_scale || out == bias)
    return refuse("elasto_op_gemm_fp8: out is one of the inputs");
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  return gemm_fp8_launch({static_cast<const uint8_t*>(A), lda, a_scale, lds, static_cast<const uint8_t*>(W), ldw, w_scale,
                          bias, out, ldo, M, N, K, epilogue, status_device},
                         static_cast<cudaStream_t>(stream));
}

elasto_status elasto_op_gemm_fp8_tile(int M, int N, int K, elasto_fp8_tile* tile) {
  clear_error();
  if (!tile || M <= 0 || N <= 0 || K <= 0) return refuse("elasto_op_gemm_fp8_tile: null pointer or size");
  if (M > 0x7fffffff - 255 || N > 0x7fffffff - 255)
    return refuse("elasto_op_gemm_fp8_tile: M or N above 2^31 - 256", ELASTO_ERR_UNSUPPORTED);
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  Fp8Gemm g{};
  g.M = M, g.N = N, g.K = K;
  *tile = gemm_fp8_tile(g);
  return ELASTO_OK;
}

elasto_status elasto_op_qk_norm_rope(void* stream, const elasto_qk_norm_rope_args* args, int* status_device) {
  clear_error();
  if (!args) return refuse("elasto_op_qk_norm_rope: null arguments");
  const elasto_qk_norm_rope_args& a = *args;
  elasto_status st = check_qk_norm_rope(a, "elasto_op_qk_norm_rope");
  if (st != ELASTO_OK) return st;
  st = check_device();
  if (st != ELASTO_OK) return st;
  ELASTO_CUDA_TRY(qk_norm_rope_launch(a, status_device, static_cast<cudaStream_t>(stream)));
  return ELASTO_OK;
}

elasto_status elasto_op_qk_norm_rope_axes(void* stream, const elasto_qk_norm_rope_axes_args* args, int* status_device) {
  clear_error();
  if (!args) return refuse("elasto_op_qk_norm_rope_axes: null arguments");
  const elasto_qk_norm_rope_axes_args& a = *args;
  elasto_status st = check_qk_norm_rope(a, "elasto_op_qk_norm_rope_axes");
  if (st != ELASTO_OK) return st;
  if (a.pairing != ELASTO_PAIRS_HALF && a.pairing != ELASTO_PAIRS_NEIGHBOURS && a.pairing != ELASTO_PAIRS_AXIS)
    return refuse("elasto_op_qk_norm_rope_axes: pairing");
  if (a.norm != 0 && a.norm != 1) return refuse("elasto_op_qk_norm_rope_axes: norm");
  if (a.rot_dim > 0) {
    if (a.axes < 1 || a.axes > 4 || !a.axis_of) return refuse("elasto_op_qk_norm_rope_axes: axes or axis_of");
    if (a.positions_row < 0 || a.positions_axis < 0) return refuse("elasto_op_qk_norm_rope_axes: strides of positions");
    unsigned seen = 0;  // axes with a run of pairs already
    for (int j = 0, run = 0; j < a.rot_dim / 2; ++j) {
      if (a.axis_of[j] >= a.axes) return refuse("elasto_op_qk_norm_rope_axes: an axis_of that is not below axes");
      if (a.pairing != ELASTO_PAIRS_AXIS) continue;
      if (j == 0 || a.axis_of[j] != a.axis_of[j - 1]) {
        if (run % 8 != 0 || (seen >> a.axis_of[j] & 1)) return refuse("elasto_op_qk_norm_rope_axes: runs of an axis's pairs");
        seen |= 1u << a.axis_of[j];
        run = 0;
      }
      ++run;
    }
  }
  st = check_device();
  if (st != ELASTO_OK) return st;
  ELASTO_CUDA_TRY(qk_norm_rope_axes_launch(a, status_device, static_cast<cudaStream_t>(stream)));
  return ELASTO_OK;
}

elasto_status elasto_op_residual_norm(void* stream, const elasto_residual_norm_args* args, int* status_device) {
  clear_error();
  if (!args) return refuse("elasto_op_residual_norm: null arguments");
  const elasto_residual_norm_args& a = *args;
  auto type = [](int t) { return t == ELASTO_F32 || t == ELASTO_BF16 || t == ELASTO_F16; };
  auto size = [](int t) { return t == ELASTO_F32 ? 4u : t == ELASTO_E4M3 ? 1u : 2u; };
  auto kind = [](int n) { return n == ELASTO_NORM_NONE || n == ELASTO_NORM_RMS || n == ELASTO_NORM_LAYER; };
  if (a.rows <= 0 || a.cols <= 0) return refuse("elasto_op_residual_norm: rows or cols");
  if (a.cols > 16384) return refuse("elasto_op_residual_norm: more than 16384 columns", ELASTO_ERR_UNSUPPORTED);
  if (!(a.eps >= 0.0f) || a.eps > 3.0e38f || !(a.x_factor >= -3.0e38f && a.x_factor <= 3.0e38f))
    return refuse("elasto_op_residual_norm: eps or x_factor");
  if (!type(a.x_type) || !a.x || !aligned(a.x, size(a.x_type)) || a.x_row < a.cols) return refuse("elasto_op_residual_norm: x (type, null, alignment or stride)");
  if (a.y && (!type(a.y_type) || !aligned(a.y, size(a.y_type)) || a.y_row < a.cols))
    return refuse("elasto_op_residual_norm: y (type, alignment or stride)");
  if (!a.x_out && !a.z) return refuse("elasto_op_residual_norm: no output");
  if (a.x_out && (!aligned(a.x_out, size(a.x_type)) || a.x_out_row < a.cols)) return refuse("elasto_op_residual_norm: x_out (alignment or stride)");
  if (a.z && ((!type(a.z_type) && a.z_type != ELASTO_E4M3) || !aligned(a.z, size(a.z_type)) || a.z_row < a.cols))
    return refuse("elasto_op_residual_norm: z (type, alignment or stride)");
  const bool fp8 = a.z && a.z_type == ELASTO_E4M3;
  if (fp8 && (!a.z_scale || !aligned(a.z_scale, 4) || a.z_scale_row < a.rows))
    return refuse("elasto_op_residual_norm: z_scale (null, alignment or stride)");
  if (!kind(a.post_norm) || !kind(a.pre_norm)) return refuse("elasto_op_residual_norm: post_norm or pre_norm");
  for (const float* p : {a.post_gain, a.post_bias, a.y_scale, a.pre_gain, a.pre_bias})
    if (!aligned(p, 4)) return refuse("elasto_op_residual_norm: a gain, a bias or y_scale misaligned");
  if (a.groups < 0 || !aligned(a.group, 4)) return refuse("elasto_op_residual_norm: groups or group");
  if (a.groups == 0 && (a.group || a.gate || a.shift || a.scale)) return refuse("elasto_op_residual_norm: group or tables with groups 0");
  if (a.gate || a.shift || a.scale) {
    if (!type(a.mod_type) || a.mod_row < a.cols) return refuse("elasto_op_residual_norm: mod_type or mod_row");
    for (const void* p : {a.gate, a.shift, a.scale})
      if (!aligned(p, size(a.mod_type))) return refuse("elasto_op_residual_norm: gate, shift or scale misaligned");
  }
  if (a.x_out == a.x && a.x_out_row != a.x_row) return refuse("elasto_op_residual_norm: x_out is x with another row stride");
  const void* const inputs[] = {a.x, a.y, a.post_gain, a.post_bias, a.y_scale, a.pre_gain, a.pre_bias, a.group, a.gate, a.shift, a.scale};
  for (const void* p : inputs)
    if (p && ((p == a.x_out && p != a.x) || p == a.z || (fp8 && p == a.z_scale)))
      return refuse("elasto_op_residual_norm: an output that is an input");
  if ((a.z && a.z == a.x_out) || (fp8 && (a.z_scale == a.z || a.z_scale == a.x_out)) || (a.y && a.y == a.x_out))
    return refuse("elasto_op_residual_norm: two outputs, or y and x_out, are one");
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  ELASTO_CUDA_TRY(residual_norm_launch(a, status_device, static_cast<cudaStream_t>(stream)));
  return ELASTO_OK;
}

elasto_status elasto_op_window_attention(void* stream, const elasto_window_attention_args* args, int* status_device) {
  clear_error();
  if (!args) return refuse("elasto_op_window_attention: null arguments");
  const elasto_window_attention_args& a = *args;
  if (a.dtype != ELASTO_BF16 && a.dtype != ELASTO_F16) return refuse("elasto_op_window_attention: dtype");
  if (a.batch <= 0 || a.heads <= 0 || a.heads_kv <= 0 || a.heads % a.heads_kv != 0 || a.max_queries <= 0 || a.max_keys <= 0)
    return refuse("elasto_op_window_attention: batch, heads, max_queries or max_keys");
  if (a.head_dim <= 0 || a.head_dim % 8 != 0 || a.head_dim > 128)
    return refuse("elasto_op_window_attention: head_dim must be a multiple of 8 up to 128", ELASTO_ERR_UNSUPPORTED);
  if (a.sinks < 0 || !(a.scale > 0.0f) || a.scale > 2.3e38f) return refuse("elasto_op_window_attention: sinks or scale");
  if (!tensor16(a.q, a.q_row, a.q_head) || !tensor16(a.out, a.out_row, a.out_head))
    return refuse("elasto_op_window_attention: q or out (null, alignment or strides)");
  if (!tensor16(a.k, a.k_row, a.k_head) || !tensor16(a.v, a.v_row, a.v_head) || !strides8(a.k_batch, a.v_batch))
    return refuse("elasto_op_window_attention: k or v (null, alignment or strides)");
  if (a.q_rows <= 0 || a.kv_rows <= 0 || a.q_rows > 1 << 30 || a.kv_rows > 1 << 30 || a.max_keys > a.kv_rows)
    return refuse("elasto_op_window_attention: q_rows or kv_rows");
  if (!a.q_start && static_cast<long long>(a.batch) * a.max_queries > a.q_rows)
    return refuse("elasto_op_window_attention: q_rows is less than batch * max_queries");
  if (a.kv_start && a.kv_len) return refuse("elasto_op_window_attention: kv_start and kv_len exclude one another");
  if (!aligned(a.q_start, 4) || !aligned(a.kv_start, 4) || !aligned(a.kv_len, 4))
    return refuse("elasto_op_window_attention: starts or lengths misaligned");
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  if (a.max_queries == 1) return window_decode_launch(a, status_device, static_cast<cudaStream_t>(stream));
  return window_attention_launch(a, status_device, static_cast<cudaStream_t>(stream));
}

elasto_status elasto_op_prefix_attention_workspace(const elasto_prefix_attention_args* args, size_t* bytes) {
  clear_error();
  if (!args || !bytes) return refuse("elasto_op_prefix_attention_workspace: null arguments");
  elasto_status st = check_prefix_sizes(*args, "elasto_op_prefix_attention_workspace");
  if (st != ELASTO_OK) return st;
  st = check_device();
  if (st != ELASTO_OK) return st;
  return prefix_attention_workspace(with_keys_there_are(*args), bytes);
}

elasto_status elasto_op_prefix_attention(void* stream, const elasto_prefix_attention_args* args, int* status_device) {
  clear_error();
  if (!args) return refuse("elasto_op_prefix_attention: null arguments");
  const elasto_prefix_attention_args& a = *args;
  elasto_status st = check_prefix_sizes(a, "elasto_op_prefix_attention");
  if (st != ELASTO_OK) return st;
  if (!(a.scale > 0.0f) || a.scale > 2.3e38f) return refuse("elasto_op_prefix_attention: scale");
  if (!tensor16(a.q, a.q_row, a.q_head) || !tensor16(a.out, a.out_row, a.out_head))
    return refuse("elasto_op_prefix_attention: q or out (null, alignment or strides)");
  if (!tensor16(a.prefix_k, a.prefix_k_row, a.prefix_k_head) || !tensor16(a.prefix_v, a.prefix_v_row, a.prefix_v_head) ||
      !strides8(a.prefix_k_batch, a.prefix_v_batch))
    return refuse("elasto_op_prefix_attention: prefix_k or prefix_v (null, alignment or strides)");
  if (!a.q_start && static_cast<long long>(a.batch) * a.max_queries > a.q_rows)
    return refuse("elasto_op_prefix_attention: q_rows is less than batch * max_queries");
  if (a.max_keys > 0) {
    if (!tensor16(a.k, a.k_row, a.k_head) || !tensor16(a.v, a.v_row, a.v_head) || !strides8(a.k_batch, a.v_batch))
      return refuse("elasto_op_prefix_attention: k or v (null, alignment or strides)");
    if (a.kv_start && a.kv_len) return refuse("elasto_op_prefix_attention: kv_start and kv_len exclude one another");
    if (a.out == a.k || a.out == a.v || a.workspace == a.k || a.workspace == a.v)
      return refuse("elasto_op_prefix_attention: out or the workspace is an input");
  }
  if (!aligned(a.q_start, 4) || !aligned(a.seq_start, 4) || !aligned(a.prefix_len, 4) || !aligned(a.kv_start, 4) || !aligned(a.kv_len, 4))
    return refuse("elasto_op_prefix_attention: starts or lengths misaligned");
  if (a.out == a.q || a.out == a.prefix_k || a.out == a.prefix_v || a.workspace == a.out || a.workspace == a.q || a.workspace == a.prefix_k ||
      a.workspace == a.prefix_v)
    return refuse("elasto_op_prefix_attention: out or the workspace is an input, or both are one");
  if (!a.workspace || !aligned(a.workspace, 16)) return refuse("elasto_op_prefix_attention: workspace (null or alignment)");
  st = check_device();
  if (st != ELASTO_OK) return st;
  return prefix_attention_launch(with_keys_there_are(a), status_device, static_cast<cudaStream_t>(stream));
}

elasto_status elasto_op_softmax(void* stream, const float* x, float* y, int rows, int cols) {
  clear_error();
  if (!x || !y || rows <= 0 || cols <= 0) {
    set_error("elasto_op_softmax: invalid arguments");
    return ELASTO_ERR_INVALID_ARG;
  }
  ELASTO_CUDA_TRY(softmax_launch(x, y, rows, cols, static_cast<cudaStream_t>(stream)));
  return ELASTO_OK;
}

elasto_status elasto_op_attention(void* stream, const void* qkv, void* out, int batch, int n, int heads,
                                  int* status_device) {
  clear_error();
  if (!qkv || !out || batch <= 0 || n <= 0 || heads <= 0) {
    set_error("elasto_op_attention: invalid arguments");
    return ELASTO_ERR_INVALID_ARG;
  }
  elasto_status st = check_device();
  if (st != ELASTO_OK) return st;
  AttnPlan p;
  st = attn_plan(&p, static_cast<const bf16*>(qkv), static_cast<bf16*>(out), batch, n, heads, status_device);
  if (st != ELASTO_OK) return st;
  ELASTO_CUDA_TRY(attn_launch(p, batch, static_cast<cudaStream_t>(stream)));
  return ELASTO_OK;
}

}  // extern "C"
