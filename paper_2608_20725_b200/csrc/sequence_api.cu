// C ABI of the operators on token sequences: argument validation and dispatch.  The contract of every entry point is in
// include/im2win.h.
#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int64_t kMost = (int64_t)1 << 31;

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
  if (pools && !s->slots && slots < sequences) return IM2WIN_ERR_INVALID_ARG;
  if (!aligned_to(s->cu, 4) || !aligned_to(s->slots, 4)) return IM2WIN_ERR_MISALIGNED;
  return IM2WIN_OK;
}

im2win_status from_launch(cudaError_t e) {
  if (e == cudaErrorInvalidConfiguration) return IM2WIN_ERR_UNSUPPORTED;      // (more blocks than a grid holds)
  return e == cudaSuccess ? IM2WIN_OK : IM2WIN_ERR_CUDA;
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

}  // extern "C"
