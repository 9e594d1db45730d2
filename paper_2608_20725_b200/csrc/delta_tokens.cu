// The gated delta rule, token by token (im2win_gated_delta_rule):
//
//   u = beta (v - a k S),   S <- a S + k^T u,   o = scale q S,   a = exp(g),   S [dk][dv] fp32.
//
// A block owns a head of a sequence and a tile of dv; S stays in its registers from the first token to the last: warp w has rows
// w*R.. of S, a lane VEC neighbouring columns of each.  For one token the state, read and written, is all the traffic there is, and
// every thread has its R loads under way at once.
//
// o needs the new S, u the old one: both sums over dk are made of the old one, o = scale (a (q S_old) + (q k) u), so that a token has
// one exchange between the warps (k S, q S of every column, and the sums q k, q q, k k; the last two where rows are divided by
// their norms) and one barrier.
//
// exp(g) as a float is off by up to 2^-25 of itself, the same way at every token of a head whose decay is constant; decays near 1,
// which remember many tokens, are applied as S + S (exp(g) - 1), whose error is that of the sum.
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
  const float* beta;
  void* o;
  const float* state_in;
  float* state_out;
  Sequences seqs;
  int64_t q_stride, k_stride, v_stride, o_stride, decay_stride, beta_stride;
  int32_t heads, share, dk, dv, tiles;   // share: heads of v to one of q and k; tiles: of dv
  int32_t normalize;
  float scale;
};

// R: rows of S of a warp (dk <= kWarps * R); VEC: columns of a lane, dv a multiple of it; BATCH: tokens loaded while the BATCH before
// them are worked on.  Single tokens: registers for two blocks of 64 numbers a thread on an SM, four of fewer.  (One token of each of 128 sequences, 32 heads
// of 128 x 128, states in one order: 64 numbers a thread, one, two, three blocks 143, 104, 120 us; 32 numbers, as the registers fell, two blocks, 110, three 102,
// four 100, and 93 in any order of a pool: 5.7 TB/s; 80 at the measured 6.56.)
template <typename T, int R, int VEC, int BATCH>
__global__ void __launch_bounds__(kWarps * 32, BATCH > 1 ? 1 : R * VEC >= 64 ? 2 : 4) delta_tokens_kernel(const TokensParams p) {
  using VF = Vec<float, VEC>;
  __shared__ __align__(16) float sums[BATCH > 1 ? 2 : 1][2][kWarps][32 * VEC];       // of k S and q S
  __shared__ float products[BATCH > 1 ? 2 : 1][3][kWarps];                           // of q k, q q, k k
  __shared__ __align__(16) float qk[kWarps][BATCH][2][R];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
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

  float S[R][VEC];
  const bool from_state = p.state_in != nullptr && live && resumes(p.seqs, b);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    VF f;
#pragma unroll
    for (int j = 0; j < VEC; ++j) f.v[j] = 0.0f;
    if (from_state && row0 + r < p.dk) f = *reinterpret_cast<const VF*>(p.state_in + state_at + (int64_t)r * p.dv);
#pragma unroll
    for (int j = 0; j < VEC; ++j) S[r][j] = f.v[j];
  }
  const bool has_row = lane < R && row0 + lane < p.dk;
  const int64_t qk_at = (int64_t)(head / p.share) * p.dk + row0 + lane;
  const T* q = static_cast<const T*>(p.q) + qk_at;
  const T* k = static_cast<const T*>(p.k) + qk_at;
  const T* v = static_cast<const T*>(p.v) + (int64_t)head * p.dv + col;
  T* o = static_cast<T*>(p.o) + (int64_t)head * p.dv + col;

  float qn[BATCH], kn[BATCH], gn[BATCH], bn[BATCH], vn[BATCH][VEC];
  auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int64_t t = t0 + i;
      const bool there = t < rows.end;
      qn[i] = there && has_row ? to_float(q[t * p.q_stride]) : 0.0f;
      kn[i] = there && has_row ? to_float(k[t * p.k_stride]) : 0.0f;
      gn[i] = there ? p.decay[t * p.decay_stride + head] : 0.0f;
      bn[i] = there ? p.beta[t * p.beta_stride + head] : 0.0f;
#pragma unroll
      for (int j = 0; j < VEC; ++j) vn[i][j] = there && live ? to_float(v[t * p.v_stride + j]) : 0.0f;
    }
  };
  load(rows.begin);
  int buffer = 0;
  for (int t0 = rows.begin; t0 < rows.end; t0 += BATCH) {
    const int n = min(BATCH, rows.end - t0);
    float g[BATCH], beta[BATCH], vv[BATCH][VEC], dots[BATCH][3];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      if (lane < R) {
        qk[warp][i][0][lane] = qn[i];
        qk[warp][i][1][lane] = kn[i];
      }
      g[i] = gn[i];
      beta[i] = bn[i];
      dots[i][0] = qn[i] * kn[i];
      dots[i][1] = qn[i] * qn[i];
      dots[i][2] = kn[i] * kn[i];
#pragma unroll
      for (int j = 0; j < VEC; ++j) vv[i][j] = vn[i][j];
    }
    __syncwarp();
    if (BATCH > 1) load(t0 + BATCH);
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
#pragma unroll
      for (int m = 0; m < 3; ++m)
#pragma unroll
        for (int s = R <= 8 ? 4 : R <= 16 ? 8 : 16; s > 0; s /= 2) dots[i][m] += __shfl_xor_sync(0xffffffffu, dots[i][m], s);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      if (i >= n) break;
      float ks[VEC], qs[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) ks[j] = qs[j] = 0.0f;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (row0 + r >= p.dk) break;             // (a row that is not there must not meet an infinity)
        const float qq = qk[warp][i][0][r], kk = qk[warp][i][1][r];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          ks[j] = fmaf(kk, S[r][j], ks[j]);
          qs[j] = fmaf(qq, S[r][j], qs[j]);
        }
      }
      VF out;
#pragma unroll
      for (int j = 0; j < VEC; ++j) out.v[j] = ks[j];
      *reinterpret_cast<VF*>(&sums[buffer][0][warp][lane * VEC]) = out;
#pragma unroll
      for (int j = 0; j < VEC; ++j) out.v[j] = qs[j];
      *reinterpret_cast<VF*>(&sums[buffer][1][warp][lane * VEC]) = out;
      if (lane < 3) products[buffer][lane][warp] = lane == 0 ? dots[i][0] : lane == 1 ? dots[i][1] : dots[i][2];
      __syncthreads();
      float all[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < VEC; ++j) ks[j] = qs[j] = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const VF a = *reinterpret_cast<const VF*>(&sums[buffer][0][w][lane * VEC]);
        const VF c = *reinterpret_cast<const VF*>(&sums[buffer][1][w][lane * VEC]);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          ks[j] += a.v[j];
          qs[j] += c.v[j];
        }
#pragma unroll
        for (int m = 0; m < 3; ++m) all[m] += products[buffer][m][w];
      }
      if (BATCH > 1) buffer ^= 1;                // (the next token's barrier comes before anyone writes this one again)
      float rq = 1.0f, rk = 1.0f;
      if (p.normalize) {
        rq = rsqrtf(all[1] + kNormalizeEps);
        rk = rsqrtf(all[2] + kNormalizeEps);
      }
      const bool near_one = g[i] > -0.5f;
      const float a = expf(g[i]), less = expm1f(g[i]);
      float u[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) u[j] = beta[i] * fmaf(-a * rk, ks[j], vv[i][j]);
      if (warp == i && live) {
        const float qk_all = all[0] * rq * rk;
#pragma unroll
        for (int j = 0; j < VEC; ++j) o[(int64_t)(t0 + i) * p.o_stride + j] = from_float<T>(p.scale * fmaf(qk_all, u[j], a * rq * qs[j]));
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) u[j] *= rk;
      if (near_one) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float kk = qk[warp][i][1][r];
#pragma unroll
          for (int j = 0; j < VEC; ++j) S[r][j] += fmaf(S[r][j], less, kk * u[j]);
        }
      } else {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float kk = qk[warp][i][1][r];
#pragma unroll
          for (int j = 0; j < VEC; ++j) S[r][j] = fmaf(S[r][j], a, kk * u[j]);
        }
      }
    }
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
    delta_tokens_kernel<T, R, VEC, 1><<<(unsigned)grid, kWarps * 32, 0, stream>>>(p);
  else
    delta_tokens_kernel<T, R, VEC, 4><<<(unsigned)grid, kWarps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

// The columns of a lane: as many as dv fills and its alignment allows, fewer while there would be under two blocks an SM (a block's
// time goes by its columns), and no more registers than a thread has.
template <typename T, int R>
cudaError_t launch_rows(TokensParams& p, int32_t sequences, bool step, cudaStream_t stream) {
  const int64_t columns = (int64_t)sequences * p.heads * p.dv;
  if constexpr (R <= 16) {
    if ((R <= 8 || !step) && p.dv % 4 == 0 && p.dv > 64 && columns >= 296 * 128) return launch<T, R, 4>(p, sequences, step, stream);
  }
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

cudaError_t launch_delta_tokens(const DeltaArgs& a, cudaStream_t stream) {
  const im2win_delta_shape& s = a.shape;
  TokensParams p = {a.q, a.k, a.v, a.decay, a.beta, a.o, a.state_in, a.state_out, a.seqs, s.q_stride, s.k_stride, s.v_stride, s.o_stride,
                    s.decay_stride, s.beta_stride, s.heads, s.heads / s.qk_heads, s.dk, s.dv, 0, s.normalize, s.scale};
  const bool step = !a.seqs.cu && s.tokens <= s.sequences;
  switch (a.dtype) {
    case IM2WIN_F32: return launch_type<float>(p, s.sequences, step, stream);
    case IM2WIN_F16: return launch_type<__half>(p, s.sequences, step, stream);
    default: return launch_type<__nv_bfloat16>(p, s.sequences, step, stream);
  }
}

}  // namespace im2win
