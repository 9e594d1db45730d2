// C ABI of the operators on token sequences: argument validation and dispatch.  The contract of every entry point is in
// include/im2win.h.
#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int64_t kMost = (int64_t)1 << 31;
constexpr int64_t kMostRows = kMost - 4096;          // tokens, sequences: the kernels count in 32 bits, up to some chunks beyond the last one

bool known_dtype(im2win_dtype dtype) { return dtype == IM2WIN_F32 || dtype == IM2WIN_F16 || dtype == IM2WIN_BF16; }

// What the sequence operators have in common: rows, sequences, pools.
im2win_status take_sequences(const im2win_sequences* given, int32_t tokens, int32_t sequences, int32_t slots, bool pools,
                             Sequences* s) {
  *s = {nullptr, nullptr, nullptr, tokens, sequences, slots};
  if (given) {
    s->cu = given->cu_seqlens;
    s->slots = given->slots;
    s->resume = given->resume;
  }
  if (tokens < 0 || sequences < 1 || slots < 0) return IM2WIN_ERR_INVALID_ARG;
  if (!s->cu && tokens % sequences != 0) return IM2WIN_ERR_INVALID_ARG;
  if ((pools || s->slots) && slots < 1) return IM2WIN_ERR_INVALID_ARG;
  if (tokens > kMostRows || sequences > kMostRows) return IM2WIN_ERR_UNSUPPORTED;
  if (pools && !s->slots && slots < sequences) return IM2WIN_ERR_INVALID_ARG;
  if (!aligned_to(s->cu, 4) || !aligned_to(s->slots, 4)) return IM2WIN_ERR_MISALIGNED;
  return IM2WIN_OK;
}

im2win_status from_launch(cudaError_t e) {
  if (e == cudaErrorInvalidConfiguration) return IM2WIN_ERR_UNSUPPORTED;      // (more blocks than a grid holds)
  return e == cudaSuccess ? IM2WIN_OK : IM2WIN_ERR_CUDA;
}

im2win_status check_attention(const im2win_attention_shape* s, im2win_dtype dtype) {
  if (!s) return IM2WIN_ERR_NULL_POINTER;
  if (!known_dtype(dtype) || s->tokens < 0 || s->sequences < 1 || s->slots < 0 || s->max_len < 0 || s->heads < 1 ||
      s->qk_heads < 1 || s->heads % s->qk_heads != 0 || s->dk < 1 || s->dv < 1)
    return IM2WIN_ERR_INVALID_ARG;
  if (s->tokens > kMostRows || s->sequences > kMostRows || s->dk > 256 || (int64_t)s->heads * s->dv >= kMost ||
      (int64_t)s->heads * s->dk >= kMost)
    return IM2WIN_ERR_UNSUPPORTED;
  return IM2WIN_OK;
}

im2win_status check_int4(const im2win_int4_shape* s, im2win_dtype dtype) {
  if (!s) return IM2WIN_ERR_NULL_POINTER;
  if (!known_dtype(dtype) || s->M < 1 || s->N < 1 || s->K < 1 || s->x_stride < s->K || s->y_stride < s->N || s->group < 1)
    return IM2WIN_ERR_INVALID_ARG;
  if (s->M > 16 || (s->group != 32 && s->group != 64 && s->group % 128 != 0) || s->K > kMost - 4096 || s->N > kMost - 4096)
    return IM2WIN_ERR_UNSUPPORTED;
  return IM2WIN_OK;
}

im2win_status check_delta(const im2win_delta_shape* s, im2win_dtype dtype) {
  if (!s) return IM2WIN_ERR_NULL_POINTER;
  if (!known_dtype(dtype) || s->tokens < 0 || s->sequences < 1 || s->slots < 0 || s->max_len < 0 || s->heads < 1 ||
      s->qk_heads < 1 || s->heads % s->qk_heads != 0 || s->dk < 1 || s->dv < 1 || (s->normalize != 0 && s->normalize != 1))
    return IM2WIN_ERR_INVALID_ARG;
  if (s->tokens > kMostRows || s->sequences > kMostRows || s->dk > 256 || (int64_t)s->heads * s->dv >= kMost ||
      (int64_t)s->heads * s->dk >= kMost)
    return IM2WIN_ERR_UNSUPPORTED;
  return IM2WIN_OK;
}

im2win_status check_int8(const im2win_int8_shape* s, im2win_dtype dtype) {
  if (!s) return IM2WIN_ERR_NULL_POINTER;
  if (!known_dtype(dtype) || s->M < 0 || s->N < 1 || s->K < 1 || s->x_stride < s->K || s->y_stride < s->N) return IM2WIN_ERR_INVALID_ARG;
  if (s->K > 131071 || s->M > kMostRows || s->N > kMostRows) return IM2WIN_ERR_UNSUPPORTED;
  return IM2WIN_OK;
}

}  // namespace
}  // namespace im2win

using namespace im2win;

extern "C" {

im2win_status im2win_causal_conv1d(const void* x, const void* weight, const float* bias, void* y, const void* state_in,
                                   void* state_out, const im2win_sequences* seqs, const im2win_conv1d_shape* shape,
                                   im2win_dtype dtype, void* cuda_stream) {
  if (!shape || !weight) return IM2WIN_ERR_NULL_POINTER;
  if (!known_dtype(dtype) || shape->channels < 1 || shape->taps < 1 || shape->taps > 8 || (shape->silu != 0 && shape->silu != 1) ||
      shape->x_stride < shape->channels || shape->y_stride < shape->channels)
    return IM2WIN_ERR_INVALID_ARG;
  Sequences s;
  const im2win_status st = take_sequences(seqs, shape->tokens, shape->sequences, shape->slots, state_in || state_out, &s);
  if (st != IM2WIN_OK) return st;
  if (shape->tokens > 0 && (!x || !y)) return IM2WIN_ERR_NULL_POINTER;
  if (shape->channels >= kMost - 4096) return IM2WIN_ERR_UNSUPPORTED;
  const size_t es = element_bytes(dtype);
  for (const void* at : {x, weight, (const void*)y, state_in, (const void*)state_out})
    if (!aligned_to(at, es)) return IM2WIN_ERR_MISALIGNED;
  if (!aligned_to(bias, 4)) return IM2WIN_ERR_MISALIGNED;
  return from_launch(launch_causal_conv1d(x, weight, bias, y, state_in, state_out, s, *shape, dtype,
                                          static_cast<cudaStream_t>(cuda_stream)));
}

im2win_status im2win_linear_attention_workspace_size(const im2win_attention_shape* shape, im2win_dtype dtype, size_t* bytes) {
  const im2win_status st = check_attention(shape, dtype);
  if (st != IM2WIN_OK) return st;
  size_t packed = 0, equal = 0;                      // with cu_seqlens and without
  bool segmented;
  attention_by_chunks(*shape, dtype, true, &packed, &segmented);
  if (shape->tokens % shape->sequences == 0) attention_by_chunks(*shape, dtype, false, &equal, &segmented);
  if (bytes) *bytes = packed > equal ? packed : equal;
  return IM2WIN_OK;
}

const char* im2win_linear_attention_kernel_name(const im2win_attention_shape* shape, im2win_dtype dtype) {
  if (check_attention(shape, dtype) != IM2WIN_OK) return "none";
  size_t bytes;
  bool segmented;
  if (!attention_by_chunks(*shape, dtype, true, &bytes, &segmented)) return "tokens";
  return segmented ? "chunks+segments" : "chunks";
}

im2win_status im2win_linear_attention(const void* q, const void* k, const void* v, const float* log_decay, void* o,
                                      const float* state_in, float* state_out, const im2win_sequences* seqs, void* workspace,
                                      size_t workspace_bytes, const im2win_attention_shape* shape, im2win_dtype dtype,
                                      void* cuda_stream) {
  if (!shape || !workspace) return IM2WIN_ERR_NULL_POINTER;
  im2win_status st = check_attention(shape, dtype);
  if (st != IM2WIN_OK) return st;
  const int64_t qk_row = (int64_t)shape->qk_heads * shape->dk, v_row = (int64_t)shape->heads * shape->dv;
  if (shape->q_stride < qk_row || shape->k_stride < qk_row || shape->v_stride < v_row || shape->o_stride < v_row ||
      (shape->decay_stride != 0 && shape->decay_stride < shape->heads))
    return IM2WIN_ERR_INVALID_ARG;
  AttentionArgs a = {q, k, v, log_decay, o, state_in, state_out, workspace, {}, *shape, dtype};
  st = take_sequences(seqs, shape->tokens, shape->sequences, shape->slots, state_in || state_out, &a.seqs);
  if (st != IM2WIN_OK) return st;
  if (shape->tokens > 0 && (!q || !k || !v || !log_decay || !o)) return IM2WIN_ERR_NULL_POINTER;
  const size_t es = element_bytes(dtype);
  for (const void* at : {q, k, v, (const void*)o})
    if (!aligned_to(at, es)) return IM2WIN_ERR_MISALIGNED;
  if (!aligned_to(log_decay, 4) || !aligned_to(state_in, 16) || !aligned_to(state_out, 16) || !aligned_to(workspace, 16))
    return IM2WIN_ERR_MISALIGNED;
  size_t need = 0;
  bool segmented;
  const bool chunks = attention_by_chunks(*shape, dtype, a.seqs.cu != nullptr, &need, &segmented);
  if (workspace_bytes < need) return IM2WIN_ERR_WORKSPACE_TOO_SMALL;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return from_launch(chunks ? launch_attention_chunks(a, stream) : launch_attention_tokens(a, stream));
}

const char* im2win_matvec_int4_kernel_name(const im2win_int4_shape* shape, im2win_dtype dtype) {
  if (check_int4(shape, dtype) != IM2WIN_OK) return "none";
  return matvec_by_ring(*shape, dtype) ? "ring" : "registers";
}

im2win_status im2win_matvec_int4(const void* x, const uint8_t* weight, const void* scales, const uint8_t* zeros,
                                 const float* bias, void* y, const im2win_int4_shape* shape, im2win_dtype dtype,
                                 void* cuda_stream) {
  if (!x || !weight || !scales || !y) return IM2WIN_ERR_NULL_POINTER;
  const im2win_status st = check_int4(shape, dtype);
  if (st != IM2WIN_OK) return st;
  const size_t es = element_bytes(dtype);
  for (const void* at : {x, scales, (const void*)y})
    if (!aligned_to(at, es)) return IM2WIN_ERR_MISALIGNED;
  if (!aligned_to(bias, 4)) return IM2WIN_ERR_MISALIGNED;
  return from_launch(launch_matvec_int4(x, weight, scales, zeros, bias, y, *shape, dtype, static_cast<cudaStream_t>(cuda_stream)));
}

const char* im2win_gated_delta_rule_kernel_name(const im2win_delta_shape* shape, im2win_dtype dtype) {
  if (check_delta(shape, dtype) != IM2WIN_OK) return "none";
  return delta_by_chunks(*shape, true) ? "chunks" : "tokens";
}

im2win_status im2win_gated_delta_rule(const void* q, const void* k, const void* v, const float* log_decay, const float* beta,
                                      void* o, const float* state_in, float* state_out, const im2win_sequences* seqs,
                                      const im2win_delta_shape* shape, im2win_dtype dtype, void* cuda_stream) {
  im2win_status st = check_delta(shape, dtype);
  if (st != IM2WIN_OK) return st;
  const int64_t qk_row = (int64_t)shape->qk_heads * shape->dk, v_row = (int64_t)shape->heads * shape->dv;
  if (shape->q_stride < qk_row || shape->k_stride < qk_row || shape->v_stride < v_row || shape->o_stride < v_row ||
      (shape->decay_stride != 0 && shape->decay_stride < shape->heads) || (shape->beta_stride != 0 && shape->beta_stride < shape->heads))
    return IM2WIN_ERR_INVALID_ARG;
  DeltaArgs a = {q, k, v, log_decay, beta, o, state_in, state_out, {}, *shape, dtype};
  st = take_sequences(seqs, shape->tokens, shape->sequences, shape->slots, state_in || state_out, &a.seqs);
  if (st != IM2WIN_OK) return st;
  if (shape->tokens > 0 && (!q || !k || !v || !log_decay || !beta || !o)) return IM2WIN_ERR_NULL_POINTER;
  const size_t es = element_bytes(dtype);
  for (const void* at : {q, k, v, (const void*)o})
    if (!aligned_to(at, es)) return IM2WIN_ERR_MISALIGNED;
  if (!aligned_to(log_decay, 4) || !aligned_to(beta, 4) || !aligned_to(state_in, 16) || !aligned_to(state_out, 16))
    return IM2WIN_ERR_MISALIGNED;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return from_launch(delta_by_chunks(*shape, a.seqs.cu != nullptr) ? launch_delta_chunks(a, stream) : launch_delta_tokens(a, stream));
}

im2win_status im2win_rms_norm(const void* x, const void* residual, const void* weight, void* residual_out, void* y, float* scales,
                              const im2win_norm_shape* shape, im2win_dtype dtype, void* cuda_stream) {
  if (!shape) return IM2WIN_ERR_NULL_POINTER;
  if (!known_dtype(dtype) || shape->rows < 0 || shape->channels < 1 || !(shape->eps >= 0.0f) || shape->x_stride < shape->channels ||
      shape->y_stride < shape->channels || (residual && shape->residual_stride < shape->channels) ||
      (residual_out && (!residual || shape->residual_out_stride < shape->channels)))
    return IM2WIN_ERR_INVALID_ARG;
  if (shape->rows > kMostRows || shape->channels > kMostRows) return IM2WIN_ERR_UNSUPPORTED;
  const size_t es = element_bytes(dtype);
  for (const void* at : {x, residual, weight, (const void*)residual_out})
    if (!aligned_to(at, es)) return IM2WIN_ERR_MISALIGNED;
  if (!aligned_to(scales, 4) || (!scales && !aligned_to(y, es))) return IM2WIN_ERR_MISALIGNED;
  if (shape->rows == 0) return IM2WIN_OK;
  if (!x || !y) return IM2WIN_ERR_NULL_POINTER;
  return from_launch(launch_rms_norm(x, residual, weight, residual_out, y, scales, *shape, dtype, static_cast<cudaStream_t>(cuda_stream)));
}

const char* im2win_matmul_int8_kernel_name(const im2win_int8_shape* shape, im2win_dtype dtype) {
  if (check_int8(shape, dtype) != IM2WIN_OK) return "none";
  return matmul_int8_by_tiles(*shape) ? "tiles" : "registers";
}

im2win_status im2win_matmul_int8(const int8_t* x, const float* x_scales, const int8_t* weight, const float* scales, const float* bias,
                                 void* y, const im2win_int8_shape* shape, im2win_dtype dtype, void* cuda_stream) {
  const im2win_status st = check_int8(shape, dtype);
  if (st != IM2WIN_OK) return st;
  if (!weight || !scales || (shape->M > 0 && (!x || !x_scales || !y))) return IM2WIN_ERR_NULL_POINTER;
  if (!aligned_to(y, element_bytes(dtype))) return IM2WIN_ERR_MISALIGNED;
  for (const float* at : {x_scales, scales, bias})
    if (!aligned_to(at, 4)) return IM2WIN_ERR_MISALIGNED;
  if (shape->M == 0) return IM2WIN_OK;
  const Int8Args a = {x, x_scales, weight, scales, bias, y, *shape, dtype};
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const bool tiles = matmul_int8_by_tiles(*shape) && aligned_to(x, 16) && aligned_to(weight, 16);
  return from_launch(tiles ? launch_matmul_int8_tiles(a, stream) : launch_matmul_int8_registers(a, stream));
}

}  // extern "C"
