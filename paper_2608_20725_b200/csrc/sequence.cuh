// What the kernels on token sequences share: element types, where a sequence's rows and state lie, and the pieces of sequences
// that blocks take.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/im2win.h"

namespace im2win {

// im2win_sequences with what bounds its values.  Nothing on the host has seen the device arrays, so every value read from them is
// clamped to the tensors before it is used.
struct Sequences {
  const int32_t* cu;
  const int32_t* slots;
  const uint8_t* resume;
  int32_t tokens, sequences, pool;       // rows, sequences, states in a pool
};

struct SequenceRows {
  int32_t begin, end;
};

__device__ __forceinline__ SequenceRows rows_of(const Sequences& s, int b) {
  SequenceRows r;
  if (s.cu) {
    r.begin = min(max(__ldg(s.cu + b), 0), s.tokens);
    r.end = min(max(__ldg(s.cu + b + 1), r.begin), s.tokens);
  } else {
    const int32_t len = s.tokens / s.sequences;
    r.begin = b * len;
    r.end = r.begin + len;
  }
  return r;
}

// Pool element of sequence b, or -1: padding.
__device__ __forceinline__ int slot_of(const Sequences& s, int b) {
  if (!s.slots) return b;
  const int32_t slot = __ldg(s.slots + b);
  return slot < 0 || slot >= s.pool ? -1 : slot;
}

__device__ __forceinline__ bool resumes(const Sequences& s, int b) { return !s.resume || __ldg(s.resume + b) != 0; }

// Pieces of at most L rows.  Sequence b has the numbers cu[b] / L + b and up, as many as it has pieces and at least one (an empty
// sequence has a state to copy); since floor(x + y) >= floor(x) + floor(y) these never reach the next sequence's, so that no sums
// over the lengths are needed, and there are at most tokens / L + sequences of them.  Numbers in between have no rows.
inline int64_t number_of_pieces(int64_t tokens, int64_t sequences, int64_t L, bool has_cu) {
  if (has_cu) return tokens / L + sequences;
  const int64_t len = tokens / sequences, per = (len + L - 1) / L;
  return sequences * (per > 0 ? per : 1);
}

struct Piece {
  int32_t sequence;
  int64_t first;                         // its first row, at or behind rows.end: nothing to do (but for the first piece of a sequence)
  SequenceRows rows;                     // of the whole sequence
};

// Every thread of the block gets the same answer; all of them call it.  One look at the array and a count: a search would read it
// log2(sequences) times in turn, half a microsecond each.
__device__ __forceinline__ Piece find_piece(const Sequences& s, int64_t id, int32_t L) {
  Piece p;
  if (!s.cu) {
    const int32_t len = s.tokens / s.sequences;
    const int32_t per = len > L ? (int32_t)(((int64_t)len + L - 1) / L) : 1;
    p.sequence = (int32_t)((uint32_t)id / (uint32_t)per);
    p.rows = rows_of(s, p.sequence);
    p.first = p.rows.begin + ((uint32_t)id % (uint32_t)per) * (int64_t)L;
    return p;
  }
  int below = 0;
  for (int32_t b0 = 0; b0 < s.sequences; b0 += (int32_t)blockDim.x) {
    const int32_t b = b0 + (int32_t)threadIdx.x;
    const bool at_or_below = b < s.sequences && (int64_t)(min(max(__ldg(s.cu + b), 0), s.tokens) / L) + b <= id;
    below += __syncthreads_count(at_or_below);
  }
  p.sequence = max(min(below, s.sequences) - 1, 0);
  p.rows = rows_of(s, p.sequence);
  const int64_t index = id - ((int64_t)(p.rows.begin / L) + p.sequence);
  p.first = index < 0 ? (int64_t)s.tokens + L : p.rows.begin + index * L;      // (negative: a cu_seqlens that falls)
  return p;
}

// Elements as floats and back, rounded once to nearest even.
template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// The larger one; a NaN is larger than anything.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// N elements that are loaded and stored at once.
template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// Two floats whose sums and products go through the paired fp32 instructions.
struct Pair {
  uint64_t v;
};
__device__ __forceinline__ Pair pair(float a, float b) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(a), "f"(b));
  return p;
}
__device__ __forceinline__ void split(Pair p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v)); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

inline bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline size_t element_bytes(im2win_dtype dtype) { return dtype == IM2WIN_F32 ? 4 : 2; }

cudaError_t launch_causal_conv1d(const void* x, const void* weight, const float* bias, void* y, const void* state_in,
                                 void* state_out, const Sequences& seqs, const im2win_conv1d_shape& shape, im2win_dtype dtype,
                                 cudaStream_t stream);


struct AttentionArgs {
  const void* q;
  const void* k;
  const void* v;
  const float* decay;
  void* o;
  const float* state_in;
  float* state_out;
  void* workspace;
  Sequences seqs;
  im2win_attention_shape shape;
  im2win_dtype dtype;
};
cudaError_t launch_attention_tokens(const AttentionArgs& a, cudaStream_t stream);
// Whether the sizes go by chunks, and the workspace that takes.
bool attention_by_chunks(const im2win_attention_shape& s, im2win_dtype dtype, bool has_cu, size_t* workspace_bytes, bool* segmented);
cudaError_t launch_attention_chunks(const AttentionArgs& a, cudaStream_t stream);
// Whether rows that start on 16-byte boundaries come through the ring of bulk copies.
bool matvec_by_ring(const im2win_int4_shape& s, im2win_dtype dtype);
cudaError_t launch_matvec_int4(const void* x, const uint8_t* weight, const void* scales, const uint8_t* zeros, const float* bias,
                               void* y, const im2win_int4_shape& shape, im2win_dtype dtype, cudaStream_t stream);

struct DeltaArgs {
  const void* q;
  const void* k;
  const void* v;
  const float* decay;
  const float* beta;
  void* o;
  const float* state_in;
  float* state_out;
  Sequences seqs;
  im2win_delta_shape shape;
  im2win_dtype dtype;
};
constexpr float kNormalizeEps = 1e-6f;     // added to the sum of squares of a row of q or k
cudaError_t launch_delta_tokens(const DeltaArgs& a, cudaStream_t stream);
bool delta_by_chunks(const im2win_delta_shape& s, bool has_cu);
cudaError_t launch_delta_chunks(const DeltaArgs& a, cudaStream_t stream);

cudaError_t launch_rms_norm(const void* x, const void* residual, const void* weight, void* residual_out, void* y, float* scales,
                            const im2win_norm_shape& shape, im2win_dtype dtype, cudaStream_t stream);

struct Int8Args {
  const int8_t* x;
  const float* x_scales;
  const int8_t* weight;
  const float* scales;
  const float* bias;
  void* y;
  im2win_int8_shape shape;
  im2win_dtype dtype;
};
// Whether rows that start on 16-byte boundaries come by TMA.
bool matmul_int8_by_tiles(const im2win_int8_shape& s);
cudaError_t launch_matmul_int8_tiles(const Int8Args& a, cudaStream_t stream);
cudaError_t launch_matmul_int8_registers(const Int8Args& a, cudaStream_t stream);

}  // namespace im2win
