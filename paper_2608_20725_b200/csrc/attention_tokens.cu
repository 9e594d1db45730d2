// Linear attention with a decay for each head, token by token (im2win_linear_attention):
//
//   S <- exp(g) S + k^T v,   o = scale q S,   S [dk][dv] fp32.
//
// A block owns a head of a sequence and a tile of dv; S stays in its registers from the first token to the last: warp w has rows
// w*R.. of S, a lane VEC neighbouring columns of each.  For one token the state, read and written, is all the traffic there is,
// and every thread has its R loads under way at once.  o is the sum over the warps' rows, through shared memory, in their order.
//
// One token of each of 128 sequences, 32 heads of 128 x 128: 93 us, 5.7 TB/s of states (81 at the measured 6.53).  Prompts run here in
// fp32 and with dk above 128: 0.4 us a token (412 tokens of heads of 48 x 80), 0.7 (128 x 128), 1.9 (256 x 128), the latency of a token's
// loads, sums and barrier.  A sequence is one block's, however long and however much of the GPU is idle: 16384 tokens of 128 x 128 in fp32 take
// 10.8 ms with 8 heads as with 32, and 30.6 ms with 32 heads of 256 x 128 in bf16, where the formula by chunks in plain matrix products
// takes 2.5, 8.2 and 14.3.
//
// exp(g) as a float is off by up to 2^-25 of itself, the same way at every token of a head whose decay is constant: after n tokens n
// times as much.  Decays near 1, which remember many tokens, are therefore applied as S + S (exp(g) - 1), whose error is that of the
// sum, and over more than one token what each sum rounds off is kept and added to the next (against 64 bits, 412 tokens, decays of
// 0.7 to 0.999: 3e-6 without, 1e-7 with).
#include <float.h>

#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int kWarps = 8;

struct TokensParams {
  const void* q;
  const void* k;
  const void* v;
  const float* decay;
  void* o;
  const float* state_in;
  float* state_out;
  uint32_t* status;                      // status block of the workspace: cleared, nothing here waits
  Sequences seqs;
  int64_t q_stride, k_stride, v_stride, o_stride, decay_stride;
  int32_t heads, share, dk, dv, tiles;   // share: heads of v to one of q and k; tiles: of dv
  float scale;
};

// R: rows of S of a warp (dk <= kWarps * R); VEC: columns of a lane, dv a multiple of it; BATCH: tokens loaded while the BATCH
// before them are worked on
template <typename T, int R, int VEC, int BATCH>
__global__ void __launch_bounds__(kWarps * 32) tokens_kernel(const TokensParams p) {
  using VF = Vec<float, VEC>;
  __shared__ __align__(16) float partial[BATCH > 1 ? 2 : 1][BATCH][kWarps][32 * VEC];
  __shared__ __align__(16) float qk[kWarps][BATCH][2][R];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x == 0 && threadIdx.x < 64) p.status[threadIdx.x] = 0;
  const int tile = (int)(blockIdx.x % (uint32_t)p.tiles);
  const uint32_t rest = blockIdx.x / (uint32_t)p.tiles;
  const int head = (int)(rest % (uint32_t)p.heads), b = (int)(rest / (uint32_t)p.heads);
  const int slot = slot_of(p.seqs, b);
  if (slot < 0) return;
  const SequenceRows rows = rows_of(p.seqs, b);
  const int col = (tile * 32 + lane) * VEC;
  const bool live = col < p.dv;
  const int row0 = warp * R;
  const int64_t state_at = ((int64_t)slot * p.heads + head) * p.dk * p.dv + (int64_t)row0 * p.dv + col;

  float S[R][VEC], rest_of[BATCH > 1 ? R : 1][VEC];        // rest_of: what the sums so far have rounded off
  const bool from_state = p.state_in != nullptr && live && resumes(p.seqs, b);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    VF f;
#pragma unroll
    for (int j = 0; j < VEC; ++j) f.v[j] = 0.0f;
    if (from_state && row0 + r < p.dk) f = *reinterpret_cast<const VF*>(p.state_in + state_at + (int64_t)r * p.dv);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      S[r][j] = f.v[j];
      if (BATCH > 1) rest_of[r][j] = 0.0f;
    }
  }
  const bool has_row = lane < R && row0 + lane < p.dk;
  const int64_t qk_at = (int64_t)(head / p.share) * p.dk + row0 + lane;
  const T* q = static_cast<const T*>(p.q) + qk_at;
  const T* k = static_cast<const T*>(p.k) + qk_at;
  const T* v = static_cast<const T*>(p.v) + (int64_t)head * p.dv + col;
  T* o = static_cast<T*>(p.o) + (int64_t)head * p.dv + tile * 32 * VEC;

  float qn[BATCH], kn[BATCH], gn[BATCH], vn[BATCH][VEC];
  auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int64_t t = t0 + i;
      const bool there = t < rows.end;
      qn[i] = there && has_row ? to_float(q[t * p.q_stride]) : 0.0f;
      kn[i] = there && has_row ? to_float(k[t * p.k_stride]) : 0.0f;
      gn[i] = there ? p.decay[t * p.decay_stride + head] : 0.0f;
#pragma unroll
      for (int j = 0; j < VEC; ++j) vn[i][j] = there && live ? to_float(v[t * p.v_stride + j]) : 0.0f;
    }
  };
  load(rows.begin);
  int buffer = 0;
  for (int t0 = rows.begin; t0 < rows.end; t0 += BATCH) {
    const int n = min(BATCH, rows.end - t0);
    float g[BATCH], vv[BATCH][VEC];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      if (lane < R) {
        qk[warp][i][0][lane] = qn[i];
        qk[warp][i][1][lane] = kn[i];
      }
      g[i] = gn[i];
#pragma unroll
      for (int j = 0; j < VEC; ++j) vv[i][j] = vn[i][j];
    }
    __syncwarp();
    if (BATCH > 1) load(t0 + BATCH);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      if (i >= n) break;
      float sum[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[j] = 0.0f;
      if (g[i] > -0.5f) {
        const float less = expm1f(g[i]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (row0 + r >= p.dk) break;           // (a row that is not there must not meet an infinity of v)
          const float qq = qk[warp][i][0][r], kk = qk[warp][i][1][r];
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const float s = S[r][j];
            const float part = fabsf(s) <= FLT_MAX ? s : 0.0f;       // (an infinity stays one: it is not added to its own negative)
            if (BATCH > 1) {
              const float d = fmaf(part, less, fmaf(kk, vv[i][j], rest_of[r][j]));
              const float t = s + d;
              const float off = d - (t - s);
              rest_of[r][j] = fabsf(t) <= FLT_MAX ? off : 0.0f;
              S[r][j] = t;
            } else {
              S[r][j] = s + fmaf(part, less, kk * vv[i][j]);
            }
            sum[j] = fmaf(qq, S[r][j], sum[j]);
          }
        }
      } else {
        const float decay = expf(g[i]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (row0 + r >= p.dk) break;
          const float qq = qk[warp][i][0][r], kk = qk[warp][i][1][r];
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            S[r][j] = fmaf(decay, S[r][j], kk * vv[i][j]);
            if (BATCH > 1) rest_of[r][j] = 0.0f;
            sum[j] = fmaf(qq, S[r][j], sum[j]);
          }
        }
      }
      VF out;
#pragma unroll
      for (int j = 0; j < VEC; ++j) out.v[j] = sum[j];
      *reinterpret_cast<VF*>(&partial[buffer][i][warp][lane * VEC]) = out;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n * 32 * VEC; i += kWarps * 32) {
      const int t = i / (32 * VEC), c = i % (32 * VEC);
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum += partial[buffer][t][w][c];
      if (tile * 32 * VEC + c < p.dv) o[(int64_t)(t0 + t) * p.o_stride + c] = from_float<T>(sum * p.scale);
    }
    if (BATCH > 1) buffer ^= 1;                  // (the next batch's barrier comes before anyone writes this one again)
  }
  if (!p.state_out || !live) return;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (row0 + r >= p.dk) break;
    VF out;
#pragma unroll
    for (int j = 0; j < VEC; ++j) out.v[j] = S[r][j];
    *reinterpret_cast<VF*>(p.state_out + state_at + (int64_t)r * p.dv) = out;
  }
}

template <typename T, int R, int VEC>
cudaError_t launch(TokensParams& p, int32_t sequences, bool step, cudaStream_t stream) {
  p.tiles = (p.dv + 32 * VEC - 1) / (32 * VEC);
  const int64_t grid = (int64_t)sequences * p.heads * p.tiles;
  if (grid >= ((int64_t)1 << 31)) return cudaErrorInvalidConfiguration;
  if (step)
    tokens_kernel<T, R, VEC, 1><<<(unsigned)grid, kWarps * 32, 0, stream>>>(p);
  else
    tokens_kernel<T, R, VEC, 4><<<(unsigned)grid, kWarps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

// The columns of a lane: as many as dv fills and its alignment allows, fewer while there would be under two blocks an SM (a block's
// time goes by its columns), and no more registers than a thread has.
template <typename T, int R>
cudaError_t launch_rows(TokensParams& p, int32_t sequences, bool step, cudaStream_t stream) {
  const int64_t columns = (int64_t)sequences * p.heads * p.dv;
  if (R <= 16 && p.dv % 4 == 0 && p.dv > 64 && columns >= 296 * 128) return launch<T, R, R <= 16 ? 4 : 2>(p, sequences, step, stream);
  if (p.dv % 2 == 0 && p.dv > 32 && columns >= 296 * 64) return launch<T, R, 2>(p, sequences, step, stream);
  return launch<T, R, 1>(p, sequences, step, stream);
}

template <typename T>
cudaError_t launch_type(TokensParams& p, int32_t sequences, bool step, cudaStream_t stream) {
  if (p.dk <= 64) return launch_rows<T, 8>(p, sequences, step, stream);
  if (p.dk <= 128) return launch_rows<T, 16>(p, sequences, step, stream);
  return launch_rows<T, 32>(p, sequences, step, stream);
}

}  // namespace

cudaError_t launch_attention_tokens(const AttentionArgs& a, cudaStream_t stream) {
  const im2win_attention_shape& s = a.shape;
  TokensParams p = {a.q, a.k, a.v, a.decay, a.o, a.state_in, a.state_out, static_cast<uint32_t*>(a.workspace), a.seqs, s.q_stride, s.k_stride, s.v_stride, s.o_stride,
                    s.decay_stride, s.heads, s.heads / s.qk_heads, s.dk, s.dv, 0, s.scale};
  const bool step = !a.seqs.cu && s.tokens <= s.sequences;
  switch (a.dtype) {
    case IM2WIN_F32: return launch_type<float>(p, s.sequences, step, stream);
    case IM2WIN_F16: return launch_type<__half>(p, s.sequences, step, stream);
    default: return launch_type<__nv_bfloat16>(p, s.sequences, step, stream);
  }
}

}  // namespace im2win
