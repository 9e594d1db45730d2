// Causal depthwise convolution along the tokens of packed sequences (im2win_causal_conv1d).
//
//   z[t][c] = bias[c] + sum_i w[c][i] x[t - (K-1) + i][c],   K = taps <= 8, rows before a sequence's first from its state.
//
// Every row is read once and written once and meets 2K operations an element, so the memory bounds it.  A thread owns VEC
// neighbouring channels (16 bytes) and walks down the rows of a piece of a sequence with the window's K-1 last rows in registers:
// each element is loaded once, plus K-1 rows at the start of a piece.  The next kBatch rows are loaded while kBatch are worked on.  The thread that has a sequence's first piece reads its old state and writes the new one, which is the old
// state's rows and the last rows of x: no other thread touches either, so that both may lie in the same buffer.
//
// 16384 tokens of 4096 channels, bf16, 4 taps, activation: 60 us, 4.5 TB/s (41 us at the measured 6.53 TB/s; 54 without the
// activation).  An element then takes 8 instructions and two of the special function units, which makes 28 and 31 us of the SMs'
// time: what is over the memory's time is what of the three does not overlap.
#include <type_traits>

#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int kThreads = 128;
constexpr int kBatch = 4;                // rows that are loaded while the kBatch before them are worked on

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
// 2^-22 (and 2^-24 |z| from the product) are far below the result's 2^-9 or 2^-12.
template <typename T>
__device__ __forceinline__ Pair silu_of(Pair z) {
  float a, b;
  if constexpr (sizeof(T) == 4) {
    split(z, a, b);
    return pair(a / (1.0f + expf(-a)), b / (1.0f + expf(-b)));
  } else {
    constexpr float kScale = -1.4426950408889634f;
    split(mul2(z, pair(kScale, kScale)), a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    split(add2(pair(a, b), pair(1.0f, 1.0f)), a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return mul2(z, pair(a, b));
  }
}

// Two neighbouring elements as floats and back.
template <typename T> __device__ __forceinline__ Pair load2(const T* at) { return pair(to_float(at[0]), to_float(at[1])); }
template <> __device__ __forceinline__ Pair load2<__nv_bfloat16>(const __nv_bfloat16* at) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(at);
  return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <typename T> __device__ __forceinline__ void store2(T* at, Pair p) {
  float a, b;
  split(p, a, b);
  if constexpr (sizeof(T) == 4) {
    at[0] = a;
    at[1] = b;
  } else if constexpr (sizeof(T) == 2) {
    uint32_t w;
    if constexpr (std::is_same<T, __half>::value)
      asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    else
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    *reinterpret_cast<uint32_t*>(at) = w;
  }
}

template <typename T, int VEC, int TAPS, bool SILU>
__global__ void __launch_bounds__(kThreads, TAPS <= 4 ? 4 : 2) conv1d_kernel(const Conv1dParams p) {
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
  constexpr int kPairs = (VEC + 1) / 2;          // (a single channel: a pair whose second is not used)
  Pair w[TAPS][kPairs], b[kPairs], win[TAPS][kPairs];
  auto elements = [&](const V& v, int j) {
    if constexpr (VEC > 1) return load2<T>(v.v + 2 * j);
    return pair(to_float(v.v[0]), 0.0f);
  };
#pragma unroll
  for (int j = 0; j < kPairs; ++j) {
#pragma unroll
    for (int i = 0; i < TAPS; ++i) {
      auto weight = [&](int c) { return c < VEC ? to_float(weights[(c * TAPS + i) / VEC].v[(c * TAPS + i) % VEC]) : 0.0f; };
      w[i][j] = pair(weight(2 * j), weight(2 * j + 1));
    }
    b[j] = pair(p.bias ? __ldg(p.bias + c + 2 * j) : 0.0f, p.bias && VEC > 1 ? __ldg(p.bias + c + 2 * j + 1) : 0.0f);
  }
#pragma unroll
  for (int i = 0; i < TAPS - 1; ++i)
#pragma unroll
    for (int j = 0; j < kPairs; ++j) win[i][j] = elements(raw[i], j);

  if (TAPS > 1 && p.state_out && leads) {
    T* out = static_cast<T*>(p.state_out) + state_at;
#pragma unroll
    for (int i = 0; i < TAPS - 1; ++i) raw[i] = row(piece.rows.end - (TAPS - 1) + i);
#pragma unroll
    for (int i = 0; i < TAPS - 1; ++i) *reinterpret_cast<V*>(out + (int64_t)i * p.channels) = raw[i];
  }

  const T* x_next = x + (int64_t)first * p.x_stride;
  T* y_next = static_cast<T*>(p.y) + c + (int64_t)first * p.y_stride;
  auto work = [&](const V& in) {                 // a row: its sums, the window one further
    V out;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      win[TAPS - 1][j] = elements(in, j);
      Pair z = b[j];
#pragma unroll
      for (int i = 0; i < TAPS; ++i) z = fma2(w[i][j], win[i][j], z);
      if (SILU) z = silu_of<T>(z);
      if constexpr (VEC > 1) {
        store2<T>(out.v + 2 * j, z);
      } else {
        float first_of, second_of;
        split(z, first_of, second_of);
        out.v[0] = from_float<T>(first_of);
      }
#pragma unroll
      for (int i = 0; i < TAPS - 1; ++i) win[i][j] = win[i + 1][j];
    }
    *reinterpret_cast<V*>(y_next) = out;
    y_next += p.y_stride;
  };
  int left = end - first;
  if (left >= kBatch) {
    V next[kBatch];
#pragma unroll
    for (int r = 0; r < kBatch; ++r, x_next += p.x_stride) next[r] = *reinterpret_cast<const V*>(x_next);
    for (; left >= 2 * kBatch; left -= kBatch) {
      V in[kBatch];
#pragma unroll
      for (int r = 0; r < kBatch; ++r) in[r] = next[r];
#pragma unroll
      for (int r = 0; r < kBatch; ++r, x_next += p.x_stride) next[r] = *reinterpret_cast<const V*>(x_next);
#pragma unroll
      for (int r = 0; r < kBatch; ++r) work(in[r]);
    }
#pragma unroll
    for (int r = 0; r < kBatch; ++r) work(next[r]);
    left -= kBatch;
  }
#pragma unroll 1
  for (; left > 0; --left, x_next += p.x_stride) work(*reinterpret_cast<const V*>(x_next));
}

// One row of each sequence: a thread takes SEQS sequences, all of whose rows it loads at once, with one set of weights.  (256 sequences
// of 8192 channels, bf16, 4 taps: 6.2 us, by the kernel above, a row at a time, 15.5.)
template <typename T, int VEC, int TAPS, bool SILU, int SEQS>
__global__ void __launch_bounds__(kThreads) conv1d_step_kernel(const Conv1dParams p) {
  using V = Vec<T, VEC>;
  constexpr int kPairs = (VEC + 1) / 2;
  const int b0 = (int)(blockIdx.x / (uint32_t)p.blocks) * SEQS;
  const int c = ((int)(blockIdx.x % (uint32_t)p.blocks) * kThreads + (int)threadIdx.x) * VEC;
  if (c >= p.channels) return;
  const int n = min(SEQS, p.seqs.sequences - b0);
  V rows[SEQS][TAPS], weights[TAPS];
  int64_t state_at[SEQS];
#pragma unroll
  for (int i = 0; i < SEQS; ++i) {
    const int slot = i < n ? slot_of(p.seqs, b0 + i) : -1;
    state_at[i] = slot < 0 ? -1 : (int64_t)slot * (TAPS - 1) * p.channels + c;
  }
#pragma unroll
  for (int i = 0; i < TAPS; ++i)
    weights[i] = *reinterpret_cast<const V*>(static_cast<const T*>(p.weight) + (int64_t)c * TAPS + i * VEC);
#pragma unroll
  for (int i = 0; i < SEQS; ++i) {
    if (state_at[i] < 0) continue;
    const bool from_state = p.state_in && resumes(p.seqs, b0 + i);
#pragma unroll
    for (int r = 0; r < TAPS - 1; ++r) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) rows[i][r].v[j] = from_float<T>(0.0f);
      if (from_state) rows[i][r] = *reinterpret_cast<const V*>(static_cast<const T*>(p.state_in) + state_at[i] + (int64_t)r * p.channels);
    }
    rows[i][TAPS - 1] = *reinterpret_cast<const V*>(static_cast<const T*>(p.x) + c + (b0 + i) * p.x_stride);
  }
  float bias[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) bias[j] = p.bias ? __ldg(p.bias + c + j) : 0.0f;
  auto elements = [&](const V& v, int j) {
    if constexpr (VEC > 1) return load2<T>(v.v + 2 * j);
    return pair(to_float(v.v[0]), 0.0f);
  };
  Pair w[TAPS][kPairs];
#pragma unroll
  for (int j = 0; j < kPairs; ++j)
#pragma unroll
    for (int i = 0; i < TAPS; ++i) {
      auto weight = [&](int e) { return e < VEC ? to_float(weights[(e * TAPS + i) / VEC].v[(e * TAPS + i) % VEC]) : 0.0f; };
      w[i][j] = pair(weight(2 * j), weight(2 * j + 1));
    }
#pragma unroll
  for (int i = 0; i < SEQS; ++i) {
    if (state_at[i] < 0) continue;
    V out;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      Pair z = pair(bias[2 * j], VEC > 1 ? bias[(2 * j + 1) % VEC] : 0.0f);
#pragma unroll
      for (int r = 0; r < TAPS; ++r) z = fma2(w[r][j], elements(rows[i][r], j), z);
      if (SILU) z = silu_of<T>(z);
      if constexpr (VEC > 1) {
        store2<T>(out.v + 2 * j, z);
      } else {
        float first_of, second_of;
        split(z, first_of, second_of);
        out.v[0] = from_float<T>(first_of);
      }
    }
    *reinterpret_cast<V*>(static_cast<T*>(p.y) + c + (b0 + i) * p.y_stride) = out;
    if (TAPS > 1 && p.state_out) {
#pragma unroll
      for (int r = 0; r < TAPS - 1; ++r)
        *reinterpret_cast<V*>(static_cast<T*>(p.state_out) + state_at[i] + (int64_t)r * p.channels) = rows[i][r + 1];
    }
  }
}

template <typename T, int VEC, int TAPS, int SEQS>
cudaError_t launch_step(const Conv1dParams& p, bool silu, cudaStream_t stream) {
  const int64_t grid = ((int64_t)p.seqs.sequences + SEQS - 1) / SEQS * p.blocks;
  if (grid >= ((int64_t)1 << 31)) return cudaErrorInvalidConfiguration;
  if (silu)
    conv1d_step_kernel<T, VEC, TAPS, true, SEQS><<<(unsigned)grid, kThreads, 0, stream>>>(p);
  else
    conv1d_step_kernel<T, VEC, TAPS, false, SEQS><<<(unsigned)grid, kThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

template <typename T, int VEC, int TAPS>
cudaError_t launch(const Conv1dParams& p, int64_t grid, bool silu, cudaStream_t stream) {
  if (!p.seqs.cu && p.seqs.tokens == p.seqs.sequences) {       // a row each; several to a thread where there is a block an SM even so
    constexpr int kSeqs = TAPS <= 4 ? 4 : 2;
    if ((int64_t)p.seqs.sequences * p.blocks >= 148 * kSeqs) return launch_step<T, VEC, TAPS, kSeqs>(p, silu, stream);
    return launch_step<T, VEC, TAPS, 1>(p, silu, stream);
  }
  if (silu)
    conv1d_kernel<T, VEC, TAPS, true><<<(unsigned)grid, kThreads, 0, stream>>>(p);
  else
    conv1d_kernel<T, VEC, TAPS, false><<<(unsigned)grid, kThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

template <typename T, int VEC>
cudaError_t launch_taps(Conv1dParams& p, const im2win_conv1d_shape& s, cudaStream_t stream) {
  p.blocks = (s.channels + kThreads * VEC - 1) / (kThreads * VEC);
  // Rows of a piece: 64, fewer where that leaves under seven blocks an SM (16384 tokens of 4096 channels, bf16, with the activation:
  // 80, 71, 73, 84 us with 16, 32, 64, 128 at three blocks an SM, 63 and 61 with 32 and 64 at four).
  int64_t grid = 0;
  for (p.L = 64;; p.L /= 2) {
    grid = number_of_pieces(s.tokens, s.sequences, p.L, p.seqs.cu != nullptr) * p.blocks;
    if (grid >= 1000 || p.L == 16) break;
  }
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
