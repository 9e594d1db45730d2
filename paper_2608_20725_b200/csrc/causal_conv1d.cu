// Causal depthwise convolution along the tokens of packed sequences (im2win_causal_conv1d).
//
//   z[t][c] = bias[c] + sum_i w[c][i] x[t - (K-1) + i][c],   K = taps <= 8, rows before a sequence's first from its state.
//
// Every row is read once and written once and meets 2K operations an element, so the memory bounds it.  A thread owns VEC
// neighbouring channels (16 bytes) and walks down the rows of a piece of a sequence with the window's K-1 last rows in registers:
// each element is loaded once, plus K-1 rows at the start of a piece.  Rows are loaded in batches of kBatch, so that as many loads
// are under way.  The thread that has a sequence's first piece reads its old state and writes the new one, which is the old
// state's rows and the last rows of x: no other thread touches either, so that both may lie in the same buffer.
#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int kThreads = 128;
constexpr int kBatch = 8;                // rows whose loads are in flight together

struct Conv1dParams {
  const void* x;
  const void* weight;
  const float* bias;
  void* y;
  const void* state_in;
  void* state_out;
  Sequences seqs;
  int64_t x_stride, y_stride;
  int32_t channels, blocks, L;           // blocks: of kThreads * VEC channels; L: rows of a piece
};

// z / (1 + exp(-z)).  fp32: as it stands.  16-bit results: exp2 and the reciprocal of the special function units, whose errors of
// 2^-22 (and 2^-24 |z| from the product) are far below the result's 2^-9 or 2^-12; the exact forms take 20 more instructions, which
// the memory does not hide.
template <typename T>
__device__ __forceinline__ float silu_of(float z) {
  if constexpr (sizeof(T) == 4) return z / (1.0f + expf(-z));
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return z * r;
}

template <typename T, int VEC, int TAPS, bool SILU>
__global__ void __launch_bounds__(kThreads) conv1d_kernel(const Conv1dParams p) {
  using V = Vec<T, VEC>;
  const uint32_t id = blockIdx.x / (uint32_t)p.blocks;
  const Piece piece = find_piece(p.seqs, id, p.L);
  const int c = ((int)(blockIdx.x % (uint32_t)p.blocks) * kThreads + (int)threadIdx.x) * VEC;
  const int slot = slot_of(p.seqs, piece.sequence);
  const bool leads = piece.first == piece.rows.begin;                  // the first piece of its sequence
  if (c >= p.channels || slot < 0 || (!leads && piece.first >= piece.rows.end)) return;
  const int first = (int)piece.first, end = (int)min(piece.first + p.L, (int64_t)piece.rows.end);
  const T* x = static_cast<const T*>(p.x) + c;
  const int64_t state_at = ((int64_t)slot * (TAPS - 1)) * p.channels + c;
  const T* state = p.state_in && resumes(p.seqs, piece.sequence) ? static_cast<const T*>(p.state_in) + state_at : nullptr;

  // row t of the sequence's x, or of its state where t lies before its first row
  auto row = [&](int t) -> V {
    if (t >= piece.rows.begin) return *reinterpret_cast<const V*>(x + t * p.x_stride);
    if (state) return *reinterpret_cast<const V*>(state + (int64_t)(t - piece.rows.begin + TAPS - 1) * p.channels);
    V zero;
#pragma unroll
    for (int j = 0; j < VEC; ++j) zero.v[j] = from_float<T>(0.0f);
    return zero;
  };

  V weights[TAPS];                       // this thread's VEC * TAPS elements as they lie: element j * TAPS + i is w[j][i]
  V raw[TAPS > 1 ? TAPS - 1 : 1];
#pragma unroll
  for (int i = 0; i < TAPS; ++i)
    weights[i] = *reinterpret_cast<const V*>(static_cast<const T*>(p.weight) + (int64_t)c * TAPS + i * VEC);
#pragma unroll
  for (int i = 0; i < TAPS - 1; ++i) raw[i] = row(first - (TAPS - 1) + i);
  float w[TAPS][VEC], b[VEC], win[TAPS][VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
#pragma unroll
    for (int i = 0; i < TAPS; ++i) w[i][j] = to_float(weights[(j * TAPS + i) / VEC].v[(j * TAPS + i) % VEC]);
    b[j] = p.bias ? __ldg(p.bias + c + j) : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < TAPS - 1; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) win[i][j] = to_float(raw[i].v[j]);

  if (TAPS > 1 && p.state_out && leads) {
    T* out = static_cast<T*>(p.state_out) + state_at;
#pragma unroll
    for (int i = 0; i < TAPS - 1; ++i) raw[i] = row(piece.rows.end - (TAPS - 1) + i);
#pragma unroll
    for (int i = 0; i < TAPS - 1; ++i) *reinterpret_cast<V*>(out + (int64_t)i * p.channels) = raw[i];
  }

  T* y = static_cast<T*>(p.y) + c;
  for (int t0 = first; t0 < end; t0 += kBatch) {
    V in[kBatch];
#pragma unroll
    for (int r = 0; r < kBatch; ++r)
      if (t0 + r < end) in[r] = *reinterpret_cast<const V*>(x + (int64_t)(t0 + r) * p.x_stride);
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      if (t0 + r >= end) break;
      V out;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        win[TAPS - 1][j] = to_float(in[r].v[j]);
        float z = b[j];
#pragma unroll
        for (int i = 0; i < TAPS; ++i) z = fmaf(w[i][j], win[i][j], z);
        if (SILU) z = silu_of<T>(z);
        out.v[j] = from_float<T>(z);
#pragma unroll
        for (int i = 0; i < TAPS - 1; ++i) win[i][j] = win[i + 1][j];
      }
      *reinterpret_cast<V*>(y + (int64_t)(t0 + r) * p.y_stride) = out;
    }
  }
}

template <typename T, int VEC, int TAPS>
cudaError_t launch(const Conv1dParams& p, int64_t grid, bool silu, cudaStream_t stream) {
  if (silu)
    conv1d_kernel<T, VEC, TAPS, true><<<(unsigned)grid, kThreads, 0, stream>>>(p);
  else
    conv1d_kernel<T, VEC, TAPS, false><<<(unsigned)grid, kThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

template <typename T, int VEC>
cudaError_t launch_taps(Conv1dParams& p, const im2win_conv1d_shape& s, cudaStream_t stream) {
  p.blocks = (s.channels + kThreads * VEC - 1) / (kThreads * VEC);
  p.L = 32;
  const int64_t grid = number_of_pieces(s.tokens, s.sequences, p.L, p.seqs.cu != nullptr) * p.blocks;
  if (grid >= ((int64_t)1 << 31)) return cudaErrorInvalidConfiguration;
  const bool silu = s.silu != 0;
  switch (s.taps) {
    case 1: return launch<T, VEC, 1>(p, grid, silu, stream);
    case 2: return launch<T, VEC, 2>(p, grid, silu, stream);
    case 3: return launch<T, VEC, 3>(p, grid, silu, stream);
    case 4: return launch<T, VEC, 4>(p, grid, silu, stream);
    case 5: return launch<T, VEC, 5>(p, grid, silu, stream);
    case 6: return launch<T, VEC, 6>(p, grid, silu, stream);
    case 7: return launch<T, VEC, 7>(p, grid, silu, stream);
    default: return launch<T, VEC, 8>(p, grid, silu, stream);
  }
}

template <typename T>
cudaError_t launch_type(Conv1dParams& p, const im2win_conv1d_shape& s, cudaStream_t stream) {
  constexpr int kVec = 16 / (int)sizeof(T);
  const bool vectors = s.channels % kVec == 0 && s.x_stride % kVec == 0 && s.y_stride % kVec == 0 && aligned_to(p.x, 16) &&
                       aligned_to(p.y, 16) && aligned_to(p.weight, 16) && aligned_to(p.state_in, 16) && aligned_to(p.state_out, 16);
  return vectors ? launch_taps<T, kVec>(p, s, stream) : launch_taps<T, 1>(p, s, stream);
}

}  // namespace

cudaError_t launch_causal_conv1d(const void* x, const void* weight, const float* bias, void* y, const void* state_in,
                                 void* state_out, const Sequences& seqs, const im2win_conv1d_shape& s, im2win_dtype dtype,
                                 cudaStream_t stream) {
  Conv1dParams p = {x, weight, bias, y, state_in, state_out, seqs, s.x_stride, s.y_stride, s.channels, 0, 0};
  switch (dtype) {
    case IM2WIN_F32: return launch_type<float>(p, s, stream);
    case IM2WIN_F16: return launch_type<__half>(p, s, stream);
    default: return launch_type<__nv_bfloat16>(p, s, stream);
  }
}

}  // namespace im2win
