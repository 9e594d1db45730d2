// The gated delta rule by chunks of 64 tokens (im2win_gated_delta_rule).
//
// With G_i the sum of log_decay up to and including token i of a chunk, S the state before it, n its tokens and k, q as normalised,
//
//   A_ij = beta_i exp(G_i - G_j) k_i . k_j  (j < i),   T = (1 + A)^-1,   R_i = beta_i (v_i - exp(G_i) k_i S),   U = T R,
//   o_i  = scale ( exp(G_i) q_i S  +  sum_{j <= i} exp(G_i - G_j) (q_i . k_j) u_j ),
//   S   <- exp(G_n) S + sum_j exp(G_n - G_j) k_j^T u_j.
//
// A sequence's chunks follow one another: a block has a head of a sequence and a tile of the columns of dv, which need nothing of one
// another.  Its time is that chain's, so it is kept within a warp: a warp has 16 columns, and S^T, R^T, U^T and o^T [16][..] are
// accumulators of the warps' own matrix instructions (m16n8k16), whose layout is that of the next product's left operand.  Nothing
// between the three dependent products leaves the warp's registers.  (On tcgen05 each of them goes through tensor memory and a barrier,
// and the split below, which is made of S, R and U in every chunk, costs the same issue slots.)  Four more warps make
// A, T and the weights of the next chunk meanwhile; the two sides meet at a barrier a chunk.
//
// The state is fp32 and stays so: operands are split into two fp16 pieces, 22 bits.  Every row of an operand is brought to below 2^15 by
// a power of two first, so that what a piece leaves off is below 2^-39 of its row's largest element, whatever the type's range.  k and q
// of 16 bits are one piece, of fp32 two; S, R and U are two pieces (S k, U k: two products a term; T R: three); T is inverted in fp32: 16 x 16
// blocks by substitution, then two levels of -T_22 A_21 T_11.  For o of 16 bits S, P and U are rounded to fp16 once, which is finer than
// o's own rounding; of fp32 they are two pieces too.
//
// Infinities and NaNs: a token whose k, beta or decay is not finite, and those behind it, get a beta of 0, a weight of NaN for o and a
// decay of NaN for S.  A column whose R or U is not finite from some token on is cleaned from there on, before it meets the zeros of T and P, and its
// o and S are made NaN.
#include <float.h>

#include <algorithm>

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "sequence.cuh"

namespace im2win {
namespace {

using ptx::smem_u32;

constexpr int kChunk = 64;
constexpr int kHelpers = 4;              // warps that prepare chunks
constexpr int kAPitch = 68;              // floats

struct ChunkParams {
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
  int32_t heads, share, dk, dv, tiles;
  int32_t normalize, qk_vectors, v_vectors, o_vectors;         // rows in whole 16-byte vectors
  float scale;
};

// What the helpers say of the tokens of a chunk.
struct alignas(16) Weights {
  float of_x[kChunk];                    // beta exp(G_i) of k S, without the scale of k
  float of_v[kChunk];                    // beta
  float of_t[kChunk];                    // undoes T's scale of a row
  float to_end[kChunk];                  // exp(G_n - G_j), without the scale of k
  float of_q[kChunk];                    // scale exp(G_i) of q S, without the scale of q
  float of_p[kChunk];                    // undoes P's scale of a row
  float total, total_rest;               // exp(G_n) in two parts
  float pad[2];
};

struct Scratch {
  float A[kChunk][kAPitch];              // A, then T
  float k_row[kChunk], q_row[kChunk];    // what k and q in pieces are multiplied by
  float whole[kChunk], part[kChunk];     // G_i in powers of two: its floor and the rest
  float beta[kChunk];
  uint32_t bad_k[kChunk / 32], bad_q[kChunk / 32];             // rows that are not finite
};

template <typename T, int DK>
struct Layout {
  static constexpr int kPieces = sizeof(T) == 4 ? 2 : 1;
  static constexpr uint32_t kRows = kChunk * DK * 2;           // a piece of k or q
  static constexpr uint32_t kSquare = kChunk * kChunk * 2;     // a piece of T or P
  static constexpr uint32_t kQAt = kPieces * kRows, kTAt = 2 * kPieces * kRows, kPAt = kTAt + 2 * kSquare;
  static constexpr uint32_t kWeightsAt = kPAt + kPieces * kSquare;
  static constexpr uint32_t kStage = kWeightsAt + sizeof(Weights);
  static constexpr uint32_t kScratchAt = 2 * kStage;
  static constexpr uint32_t kVAt = (kScratchAt + sizeof(Scratch) + 127) / 128 * 128;
  static constexpr uint32_t kV = sizeof(T) == 2 ? kChunk * 32 : 0;         // a warp's columns of v, and of o on its way out
  static constexpr uint32_t bytes(int warps) { return kVAt + 2 * kV * warps; }
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// A power of two that brings numbers of at most `top` to below 2^15, and its reciprocal.
__device__ __forceinline__ float scale_for(float top) {
  const int e = (int)(__float_as_uint(top) >> 23 & 255u);
  return __uint_as_float((uint32_t)min(max(268 - e, 1), 253) << 23);
}
__device__ __forceinline__ float unscale_for(float scale) { return __uint_as_float((254u << 23) - __float_as_uint(scale)); }

__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ float2 unpack_half(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
// Two scaled numbers as pieces.
__device__ __forceinline__ void split(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pack_half(a, b);
  const float2 h = unpack_half(hi);
  lo = pack_half(a - h.x, b - h.y);
}

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void stmatrix_trans(uint32_t addr, const uint32_t (&r)[4]) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3])
               : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void sync_helpers() { asm volatile("bar.sync 1, %0;" ::"n"(kHelpers * 32) : "memory"); }

// Byte of a 16-byte unit of row r of rows of N elements of 16 bits (units swizzled by the row, so that the matrix loads have no conflicts).
template <int N>
__device__ __forceinline__ uint32_t unit_at(int r, int unit) {
  return (uint32_t)(r * N * 2 + ((unit ^ (r & 7)) << 4));
}

// ------------------------------------------------------------------------------------------------ the helpers

// Eight elements of a row as floats; 0 beyond `columns` and where the row is not there.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int at, int columns, bool there, bool vectors, float (&x)[8]) {
  if (vectors) {
    if constexpr (sizeof(T) == 2) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (there && at < columns) w = __ldg(reinterpret_cast<const uint4*>(row + at));
      const Vec<T, 8> e = *reinterpret_cast<const Vec<T, 8>*>(&w);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = to_float(e.v[j]);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (there && at + 4 * h < columns) w = __ldg(reinterpret_cast<const float4*>(row + at + 4 * h));
        x[4 * h] = w.x, x[4 * h + 1] = w.y, x[4 * h + 2] = w.z, x[4 * h + 3] = w.w;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = there && at + j < columns ? to_float(row[at + j]) : 0.0f;
  }
}

// Rows of q or k of a chunk to shared memory, scaled, in pieces: two threads a row.  Leaves what a row is multiplied by (the norm's and the
// scale's reciprocals) and says which rows are not finite (they come out as 0).
template <typename T, int DK>
__device__ __forceinline__ void prepare_rows(const ChunkParams& p, const T* from, int64_t stride, int first, int end, uint32_t to, float* factor,
                                             uint32_t* bad) {
  using L = Layout<T, DK>;
  const int t = threadIdx.x & (kHelpers * 32 - 1), r = t >> 1, half = t & 1, lane = threadIdx.x & 31;
  const bool there = first + r < end;
  const T* row = from + (there ? (int64_t)(first + r) * stride : 0);
  constexpr int kUnits = DK / 16;                              // of a thread: every second one of its row
  float x[kUnits][8];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) load8<T>(row, (2 * i + half) * 8, p.dk, there, p.qk_vectors, x[i]);
  float top = 0.0f, squares = 0.0f;
#pragma unroll
  for (int i = 0; i < kUnits; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      top = max_nan(top, fabsf(x[i][j]));
      squares = fmaf(x[i][j], x[i][j], squares);
    }
  top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
  squares += __shfl_xor_sync(0xffffffffu, squares, 1);
  const bool odd = !(top <= FLT_MAX);
  const float scale = scale_for(top);
  const uint32_t odd_rows = __ballot_sync(0xffffffffu, odd);   // (two bits a row)
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) split(odd ? 0.0f : x[i][2 * j] * scale, odd ? 0.0f : x[i][2 * j + 1] * scale, hi[j], lo[j]);
    const uint32_t at = to + unit_at<DK>(r, 2 * i + half);
    ptx::st_shared16(at, hi[0], hi[1], hi[2], hi[3]);
    if (L::kPieces == 2) ptx::st_shared16(at + L::kRows, lo[0], lo[1], lo[2], lo[3]);
  }
  if (half == 0) factor[r] = odd ? 0.0f : (p.normalize ? rsqrtf(squares + kNormalizeEps) : 1.0f) * unscale_for(scale);
  if (lane == 0) {
    uint32_t rows = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) rows |= (odd_rows >> (2 * i) & 1u) << i;
    reinterpret_cast<uint16_t*>(bad)[(t >> 5)] = (uint16_t)rows;
  }
}

// One warp: lane l has tokens 2l and 2l+1.  Sums of log_decay are of whole numbers of 2^-44 powers of two: exact.
__device__ __forceinline__ void prepare_weights(const ChunkParams& p, const float (&g)[2], const float (&b)[2], int tokens, Scratch& s, Weights& w) {
  constexpr float kNaN = __builtin_nanf("");
  const int lane = threadIdx.x & 31;
  auto powers = [](float x) -> int64_t {                       // (beyond 2^+-1000 nothing changes in fp32)
    return __double2ll_rn((double)fminf(fmaxf(x, -700.0f), 700.0f) * (1.4426950408889634074 * 17592186044416.0));
  };
  int64_t a[2];
  uint32_t odd[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    a[i] = powers(g[i]);
    const bool row = (s.bad_k[lane >> 4] >> ((2 * lane + i) & 31) & 1u) != 0;
    odd[i] = __ballot_sync(0xffffffffu, row || !(g[i] < __int_as_float(0x7f800000)) || !(fabsf(b[i]) <= FLT_MAX));
  }
  // the first token from which nothing is finite any more
  const int first0 = odd[0] ? 2 * (__ffs(odd[0]) - 1) : kChunk, first1 = odd[1] ? 2 * (__ffs(odd[1]) - 1) + 1 : kChunk;
  const int broken = min(first0, first1);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (2 * lane + i >= broken) a[i] = 0;                      // (so that nothing that is finite meets what is not)
  int64_t sum = a[0] + a[1];
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int64_t other = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += other;
  }
  const int64_t all = __shfl_sync(0xffffffffu, sum, 31);
  auto fraction = [](int64_t x) { return (float)((uint32_t)(x >> 20) & 0xffffffu) * 5.9604644775390625e-8f; };
  auto power = [&](int64_t x) {
    return exp2f(fraction(x)) * __uint_as_float((uint32_t)(min(max((int)(x >> 44), -127), 127) + 127) << 23);
  };
  const int64_t G[2] = {sum - a[1], sum};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = 2 * lane + i;
    const bool gone = t >= broken;
    const float beta = gone ? 0.0f : b[i], from_start = power(G[i]);
    const bool bad_q = (s.bad_q[lane >> 4] >> (t & 31) & 1u) != 0;
    s.whole[t] = (float)(int)(G[i] >> 44);
    s.part[t] = fraction(G[i]);
    s.beta[t] = beta;
    w.of_x[t] = beta * from_start * s.k_row[t];
    w.of_v[t] = beta;
    w.to_end[t] = power(all - G[i]) * s.k_row[t];
    w.of_q[t] = gone || bad_q ? kNaN : p.scale * from_start * s.q_row[t];
  }
  if (lane == 0) {
    const double exact = exp2((double)all * (1.0 / 17592186044416.0));
    const float total = (float)exact;
    w.total = broken < tokens ? kNaN : total;
    w.total_rest = (float)(exact - (double)total);
  }
}

// T in the place of A.
__device__ __forceinline__ void invert(Scratch& s) {
  const int t = threadIdx.x & (kHelpers * 32 - 1), warp = t >> 5, lane = t & 31;
  {
    const int b0 = warp * 16, j = lane & 15;                   // (both halves of the warp do the same)
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = i == j ? 1.0f : 0.0f;
#pragma unroll
    for (int k = 0; k < 15; ++k)
#pragma unroll
      for (int i = k + 1; i < 16; ++i) x[i] = fmaf(-s.A[b0 + i][b0 + k], x[k], x[i]);
    __syncwarp();
    if (lane < 16) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s.A[b0 + i][b0 + j] = x[i];
    }
  }
  sync_helpers();
  {
    const int c0 = (t >> 6) * 32, r0 = c0 + 16, r = r0 + ((t & 63) >> 2), c = c0 + (t & 3) * 4;
    float4 m = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto add = [&](float a, const float4& b) {
      m.x = fmaf(a, b.x, m.x), m.y = fmaf(a, b.y, m.y), m.z = fmaf(a, b.z, m.z), m.w = fmaf(a, b.w, m.w);
    };
#pragma unroll
    for (int k = 0; k < 16; ++k) add(s.A[r][c0 + k], *reinterpret_cast<const float4*>(&s.A[c0 + k][c]));
    sync_helpers();
    *reinterpret_cast<float4*>(&s.A[r][c]) = m;
    sync_helpers();
    m = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < 16; ++k) add(-s.A[r][r0 + k], *reinterpret_cast<const float4*>(&s.A[r0 + k][c]));
    sync_helpers();
    *reinterpret_cast<float4*>(&s.A[r][c]) = m;
  }
  sync_helpers();
  {
    const int r = 32 + (t >> 3) * 2, c = (t & 7) * 4;
    float4 m[2];
    auto product = [&](int rows_at, int from) {                // rows r, r + 1 of A[..][rows_at ..] times rows `from`.. of columns c
      m[0] = m[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < 32; k += 4) {
        const float4 a0 = *reinterpret_cast<const float4*>(&s.A[r][rows_at + k]), a1 = *reinterpret_cast<const float4*>(&s.A[r + 1][rows_at + k]);
        const float f0[4] = {a0.x, a0.y, a0.z, a0.w}, f1[4] = {a1.x, a1.y, a1.z, a1.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 b = *reinterpret_cast<const float4*>(&s.A[from + k + i][c]);
          m[0].x = fmaf(f0[i], b.x, m[0].x), m[0].y = fmaf(f0[i], b.y, m[0].y), m[0].z = fmaf(f0[i], b.z, m[0].z), m[0].w = fmaf(f0[i], b.w, m[0].w);
          m[1].x = fmaf(f1[i], b.x, m[1].x), m[1].y = fmaf(f1[i], b.y, m[1].y), m[1].z = fmaf(f1[i], b.z, m[1].z), m[1].w = fmaf(f1[i], b.w, m[1].w);
        }
      }
    };
    product(0, 0);
    sync_helpers();
    *reinterpret_cast<float4*>(&s.A[r][c]) = m[0];
    *reinterpret_cast<float4*>(&s.A[r + 1][c]) = m[1];
    sync_helpers();
    product(32, 32);
    sync_helpers();
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<float4*>(&s.A[r + i][c]) = make_float4(-m[i].x, -m[i].y, -m[i].z, -m[i].w);
  }
  sync_helpers();
}

// Chunk of rows [first, end) into `stage`.
template <typename T, int DK>
__device__ __forceinline__ void prepare(const ChunkParams& p, int head, int first, int end, uint32_t smem, uint8_t* generic, uint32_t stage,
                                        Scratch& s) {
  using L = Layout<T, DK>;
  const int warp = (threadIdx.x >> 5) & (kHelpers - 1), lane = threadIdx.x & 31;
  Weights& w = *reinterpret_cast<Weights*>(generic + stage + L::kWeightsAt);
  float g[2] = {0.0f, 0.0f}, b[2] = {0.0f, 0.0f};
  if (warp == 0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t t = first + 2 * lane + i;
      if (t < end) {
        g[i] = p.decay[t * p.decay_stride + head];
        b[i] = p.beta[t * p.beta_stride + head];
      }
    }
  }
  const int64_t at = (int64_t)(head / p.share) * p.dk;
  const uint32_t kt = smem + stage, qt = kt + L::kQAt;
  prepare_rows<T, DK>(p, static_cast<const T*>(p.k) + at, p.k_stride, first, end, kt, s.k_row, s.bad_k);
  prepare_rows<T, DK>(p, static_cast<const T*>(p.q) + at, p.q_stride, first, end, qt, s.q_row, s.bad_q);
  sync_helpers();
  if (warp == 0) prepare_weights(p, g, b, end - first, s, w);
  sync_helpers();

  // 16 rows of k k^T and 16 of q k^T a warp, up to the diagonal
  const int mi = lane >> 3, r8 = lane & 7, group = lane >> 2, pair = (lane & 3) * 2;
  auto square = [&](uint32_t rows, int m, float (&acc)[8][4]) {
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
#pragma unroll 2
    for (int ks = 0; ks < DK / 16; ++ks) {
      uint32_t a[L::kPieces][4];
#pragma unroll
      for (int i = 0; i < L::kPieces; ++i) ldmatrix(rows + i * L::kRows + unit_at<DK>(m * 16 + (mi & 1) * 8 + r8, 2 * ks + (mi >> 1)), a[i]);
#pragma unroll
      for (int np = 0; np < 4; ++np) {
        if (np > m) break;
        uint32_t k0[4];
        ldmatrix(kt + unit_at<DK>(np * 16 + (mi >> 1) * 8 + r8, 2 * ks + (mi & 1)), k0);
        if (L::kPieces == 2) {
          uint32_t k1[4];
          ldmatrix(kt + L::kRows + unit_at<DK>(np * 16 + (mi >> 1) * 8 + r8, 2 * ks + (mi & 1)), k1);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            mma(acc[2 * np + h], a[0], k1[2 * h], k1[2 * h + 1]);
            mma(acc[2 * np + h], a[L::kPieces - 1], k0[2 * h], k0[2 * h + 1]);
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) mma(acc[2 * np + h], a[0], k0[2 * h], k0[2 * h + 1]);
      }
    }
  };
  auto weigh = [&](int m, float (&acc)[8][4], float f0, float f1, bool with_diagonal) {
    const int i0 = m * 16 + group;
    const float w0 = s.whole[i0], w1 = s.whole[i0 + 8], p0 = s.part[i0], p1 = s.part[i0 + 8];
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      if (n > 2 * m + 1) break;
      const int j = n * 8 + pair;
      const float2 wj = *reinterpret_cast<const float2*>(&s.whole[j]), pj = *reinterpret_cast<const float2*>(&s.part[j]);
      const float2 kj = *reinterpret_cast<const float2*>(&s.k_row[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = i0 + (e >> 1) * 8, jj = j + (e & 1);
        const float power = ((e >> 1 ? w1 : w0) - (e & 1 ? wj.y : wj.x)) + ((e >> 1 ? p1 : p0) - (e & 1 ? pj.y : pj.x));
        const float x = acc[n][e] * (e >> 1 ? f1 : f0) * (e & 1 ? kj.y : kj.x) * exp2f(power);
        acc[n][e] = jj < i || (with_diagonal && jj == i) ? x : 0.0f;
      }
    }
  };
  {
    float acc[8][4];
    const int m = warp, i0 = m * 16 + group;
    square(kt, m, acc);
    weigh(m, acc, s.beta[i0] * s.k_row[i0], s.beta[i0 + 8] * s.k_row[i0 + 8], false);
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      if (n > 2 * m + 1) break;
      *reinterpret_cast<float2*>(&s.A[i0][n * 8 + pair]) = make_float2(acc[n][0], acc[n][1]);
      *reinterpret_cast<float2*>(&s.A[i0 + 8][n * 8 + pair]) = make_float2(acc[n][2], acc[n][3]);
    }
  }
  {
    float acc[8][4];
    const int m = kHelpers - 1 - warp, i0 = m * 16 + group;
    square(qt, m, acc);
    weigh(m, acc, p.scale * s.q_row[i0], p.scale * s.q_row[i0 + 8], true);
    float top[2] = {0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      if (n > 2 * m + 1) break;
#pragma unroll
      for (int e = 0; e < 4; ++e) top[e >> 1] = fmaxf(top[e >> 1], fabsf(acc[n][e]));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
      top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2));
      const float scale = scale_for(top[h]);
      const int i = i0 + 8 * h;
      if ((lane & 3) == 0) w.of_p[i] = unscale_for(scale);
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        if (n > 2 * m + 1) break;
        uint32_t hi, lo;
        split(acc[n][2 * h] * scale, acc[n][2 * h + 1] * scale, hi, lo);
        uint8_t* to = generic + stage + L::kPAt + unit_at<kChunk>(i, n) + pair * 2;
        *reinterpret_cast<uint32_t*>(to) = hi;
        if (L::kPieces == 2) *reinterpret_cast<uint32_t*>(to + L::kSquare) = lo;
      }
    }
  }
  sync_helpers();
  invert(s);
  {
    const int t = threadIdx.x & (kHelpers * 32 - 1), r = t >> 1, half = t & 1;
    const int blocks = (r >> 4) + 1;                           // of 16 columns, up to the diagonal's
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i >= blocks) break;
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        const float4 x = *reinterpret_cast<const float4*>(&s.A[r][i * 16 + half * 8 + j]);
        top = fmaxf(fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y))), fmaxf(fabsf(x.z), fabsf(x.w)));
      }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const float scale = scale_for(top);
    if (half == 0) w.of_t[r] = unscale_for(scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i >= blocks) break;
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 x = *reinterpret_cast<const float2*>(&s.A[r][i * 16 + half * 8 + 2 * j]);
        split(x.x * scale, x.y * scale, hi[j], lo[j]);
      }
      const uint32_t to = kt + L::kTAt + unit_at<kChunk>(r, 2 * i + half);
      ptx::st_shared16(to, hi[0], hi[1], hi[2], hi[3]);
      ptx::st_shared16(to + L::kSquare, lo[0], lo[1], lo[2], lo[3]);
    }
  }
}

// ------------------------------------------------------------------------------------------------ the columns of a warp

// Rows g and g + 8 of accumulators over tokens: from the first token on whose number is not finite all become 0; `from` says which.
__device__ __noinline__ void clean_copy(float (&x)[8][4], int (&from)[2]) {
  const int pair = (threadIdx.x & 3) * 2;
  int first[2] = {from[0], from[1]};
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (!(fabsf(x[n][e]) <= FLT_MAX)) first[e >> 1] = min(first[e >> 1], n * 8 + pair + (e & 1));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    first[h] = min(first[h], __shfl_xor_sync(0xffffffffu, first[h], 1));
    first[h] = min(first[h], __shfl_xor_sync(0xffffffffu, first[h], 2));
    from[h] = first[h];
  }
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n * 8 + pair + (e & 1) >= from[e >> 1]) x[n][e] = 0.0f;
}
// (The copy keeps x itself in registers where this is not called.)
__device__ __forceinline__ void clean(float (&x)[8][4], int (&from)[2]) {
  float copy[8][4];
  int first[2] = {from[0], from[1]};
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) copy[n][e] = x[n][e];
  clean_copy(copy, first);
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[n][e] = copy[n][e];
  from[0] = first[0];
  from[1] = first[1];
}

// The largest magnitude of rows g and g + 8, in all four lanes that share them; a NaN where there is one.
template <int N>
__device__ __forceinline__ void largest(const float (&x)[N][4], float (&top)[2]) {
  top[0] = top[1] = 0.0f;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) top[e >> 1] = max_nan(top[e >> 1], fabsf(x[n][e]));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    top[h] = max_nan(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
    top[h] = max_nan(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2));
  }
}

// Left operand of step ks of a product along the columns of x (its tiles 2 ks and 2 ks + 1), scaled, in pieces.
template <int N>
__device__ __forceinline__ void operand(const float (&x)[N][4], int ks, const float (&scale)[2], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f = scale[i & 1];
    split(x[2 * ks + (i >> 1)][2 * (i & 1)] * f, x[2 * ks + (i >> 1)][2 * (i & 1) + 1] * f, hi[i], lo[i]);
  }
}

template <typename T, int DK>
struct Columns {
  using L = Layout<T, DK>;
  static constexpr bool kFull = L::kPieces == 2;               // fp32: o too from two pieces

  const ChunkParams& p;
  uint32_t smem, v_at;
  uint8_t* generic;
  int head, col0, lane, mi, r8, group, pair;
  float S[DK / 8][4];

  __device__ __forceinline__ Columns(const ChunkParams& p_, uint32_t smem_, uint8_t* generic_, int head_, int col0_, int warp)
      : p(p_), smem(smem_), v_at(smem_ + L::kVAt + 2 * L::kV * warp), generic(generic_), head(head_), col0(col0_) {
    lane = threadIdx.x & 31;
    mi = lane >> 3, r8 = lane & 7, group = lane >> 2, pair = (lane & 3) * 2;
  }
  __device__ __forceinline__ void states(const float* from) {
#pragma unroll
    for (int n = 0; n < DK / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = n * 8 + pair + (e & 1), c = col0 + group + 8 * (e >> 1);
        S[n][e] = from && d < p.dk && c < p.dv ? from[(int64_t)d * p.dv + c] : 0.0f;
      }
  }
  __device__ __forceinline__ void store_states(float* to) const {
#pragma unroll
    for (int n = 0; n < DK / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = n * 8 + pair + (e & 1), c = col0 + group + 8 * (e >> 1);
        if (d < p.dk && c < p.dv) to[(int64_t)d * p.dv + c] = S[n][e];
      }
  }
  // (16 bits) 64 rows of 16 columns, 32 bytes each, the halves of every second four rows swapped
  static __device__ __forceinline__ uint32_t v_unit(int t, int half) { return (uint32_t)(t * 32 + ((half ^ (t >> 2 & 1)) << 4)); }
  __device__ __forceinline__ void load_v(int buffer, int first, int end) const {
    if constexpr (sizeof(T) == 2) {
      const T* v = static_cast<const T*>(p.v) + (int64_t)head * p.dv + col0;
      const uint32_t to = v_at + buffer * L::kV;
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + (lane >> 1), half = lane & 1;
        const bool row = first + t < end;
        const T* from = v + (row ? (int64_t)(first + t) * p.v_stride + half * 8 : 0);
        if (p.v_vectors) {
          const bool there = row && col0 + half * 8 < p.dv;
          copy16(to + v_unit(t, half), there ? from : v, there);
        } else {
          const uint16_t* e = reinterpret_cast<const uint16_t*>(from);
          uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (row && col0 + half * 8 + j < p.dv) w[j / 2] |= (uint32_t)e[j] << (16 * (j & 1));
          ptx::st_shared16(to + v_unit(t, half), w[0], w[1], w[2], w[3]);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }

  __device__ __forceinline__ void chunk(int c, int first, int end) {
    const uint32_t kt = smem + (c & 1) * L::kStage, qt = kt + L::kQAt, tt = kt + L::kTAt, pt = kt + L::kPAt;
    const Weights& w = *reinterpret_cast<const Weights*>(generic + (c & 1) * L::kStage + L::kWeightsAt);
    load_v((c + 1) & 1, first + kChunk, end);
    float v32[kFull ? 8 : 1][4];
    if constexpr (kFull) {
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = first + n * 8 + pair + (e & 1), at = col0 + group + 8 * (e >> 1);
          v32[n][e] = t < end && at < p.dv ? static_cast<const float*>(p.v)[(int64_t)t * p.v_stride + (int64_t)head * p.dv + at] : 0.0f;
        }
    }

    // k S and q S
    float X[8][4], O[8][4], top[2], scale[2], per_s[2];
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) X[n][e] = O[n][e] = 0.0f;
    largest(S, top);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      scale[h] = scale_for(top[h]);
      per_s[h] = unscale_for(scale[h]);
    }
#pragma unroll
    for (int ks = 0; ks < DK / 16; ++ks) {
      uint32_t hi[4], lo[4];
      operand(S, ks, scale, hi, lo);
#pragma unroll
      for (int np = 0; np < 4; ++np) {
        const uint32_t at = unit_at<DK>(np * 16 + (mi >> 1) * 8 + r8, 2 * ks + (mi & 1));
        uint32_t b[4], a[4];
        ldmatrix(kt + at, b);
        ldmatrix(qt + at, a);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          mma(X[2 * np + h], lo, b[2 * h], b[2 * h + 1]);
          if (kFull) mma(O[2 * np + h], lo, a[2 * h], a[2 * h + 1]);
          mma(X[2 * np + h], hi, b[2 * h], b[2 * h + 1]);
          mma(O[2 * np + h], hi, a[2 * h], a[2 * h + 1]);
        }
        if (kFull) {
          ldmatrix(kt + L::kRows + at, b);
          ldmatrix(qt + L::kRows + at, a);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            mma(X[2 * np + h], hi, b[2 * h], b[2 * h + 1]);
            mma(O[2 * np + h], hi, a[2 * h], a[2 * h + 1]);
          }
        }
      }
    }

    // R, in the place of k S
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncwarp();
#pragma unroll
    for (int np = 0; np < 4; ++np) {
      uint32_t vv[4] = {0, 0, 0, 0};
      if constexpr (!kFull) ptx::ldmatrix_x4_trans(v_at + (c & 1) * L::kV + v_unit(np * 16 + (mi >> 1) * 8 + r8, mi & 1), vv);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = 2 * np + h;
        const float2 fx = *reinterpret_cast<const float2*>(&w.of_x[n * 8 + pair]), fv = *reinterpret_cast<const float2*>(&w.of_v[n * 8 + pair]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float value;
          if constexpr (kFull) {
            value = v32[n][e];
          } else {
            const Vec<T, 2> two = *reinterpret_cast<const Vec<T, 2>*>(&vv[2 * h + (e >> 1)]);
            value = to_float(two.v[e & 1]);
          }
          X[n][e] = fmaf(e & 1 ? fv.y : fv.x, value, -(e & 1 ? fx.y : fx.x) * per_s[e >> 1] * X[n][e]);
        }
      }
    }
    int from[2] = {kChunk, kChunk};
    largest(X, top);
    bool odd = __any_sync(0xffffffffu, !(max_nan(top[0], top[1]) <= FLT_MAX));
    if (odd) {
      clean(X, from);
      largest(X, top);
    }
    float per_r[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      scale[h] = scale_for(top[h]);
      per_r[h] = unscale_for(scale[h]);
    }

    // U (times R's scale)
    float U[8][4];
    {
      uint32_t hi[4][4], lo[4][4];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) operand(X, kk, scale, hi[kk], lo[kk]);
#pragma unroll
      for (int np = 0; np < 4; ++np) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) U[2 * np + h][e] = 0.0f;
#pragma unroll
        for (int kk = 0; kk <= np; ++kk) {
          const uint32_t at = tt + unit_at<kChunk>(np * 16 + (mi >> 1) * 8 + r8, 2 * kk + (mi & 1));
          uint32_t b[4], bl[4];
          ldmatrix(at, b);
          ldmatrix(at + L::kSquare, bl);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            mma(U[2 * np + h], lo[kk], b[2 * h], b[2 * h + 1]);
            mma(U[2 * np + h], hi[kk], bl[2 * h], bl[2 * h + 1]);
            mma(U[2 * np + h], hi[kk], b[2 * h], b[2 * h + 1]);
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 f = *reinterpret_cast<const float2*>(&w.of_t[(2 * np + h) * 8 + pair]);
#pragma unroll
          for (int e = 0; e < 4; ++e) U[2 * np + h][e] *= e & 1 ? f.y : f.x;
        }
      }
    }
    largest(U, top);
    if (__any_sync(0xffffffffu, !(max_nan(top[0], top[1]) <= FLT_MAX))) {
      odd = true;
      clean(U, from);
      largest(U, top);
    }

    // o
    {
      uint32_t hi[4][4], lo[4][4];
      float per_o[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        scale[h] = scale_for(top[h]);
        per_o[h] = unscale_for(scale[h]) * per_r[h];
      }
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) operand(U, kk, scale, hi[kk], lo[kk]);
#pragma unroll
      for (int np = 0; np < 4; ++np) {
        float I[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) I[h][e] = 0.0f;
#pragma unroll
        for (int kk = 0; kk <= np; ++kk) {
          const uint32_t at = pt + unit_at<kChunk>(np * 16 + (mi >> 1) * 8 + r8, 2 * kk + (mi & 1));
          uint32_t b[4];
          ldmatrix(at, b);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (kFull) mma(I[h], lo[kk], b[2 * h], b[2 * h + 1]);
            mma(I[h], hi[kk], b[2 * h], b[2 * h + 1]);
          }
          if (kFull) {
            ldmatrix(at + L::kSquare, b);
#pragma unroll
            for (int h = 0; h < 2; ++h) mma(I[h], hi[kk], b[2 * h], b[2 * h + 1]);
          }
        }
        uint32_t out[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int n = 2 * np + h, t = n * 8 + pair;
          const float2 fq = *reinterpret_cast<const float2*>(&w.of_q[t]), fp = *reinterpret_cast<const float2*>(&w.of_p[t]);
          float y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y[e] = fmaf((e & 1 ? fq.y : fq.x) * per_s[e >> 1], O[n][e], (e & 1 ? fp.y : fp.x) * per_o[e >> 1] * I[h][e]);
            if (odd && t + (e & 1) >= from[e >> 1]) y[e] = __builtin_nanf("");
          }
          if constexpr (kFull) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int row = first + t + (e & 1), at = col0 + group + 8 * (e >> 1);
              if (row < end && at < p.dv) static_cast<float*>(p.o)[(int64_t)row * p.o_stride + (int64_t)head * p.dv + at] = y[e];
            }
          } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              Vec<T, 2> two;
              two.v[0] = from_float<T>(y[2 * i]);
              two.v[1] = from_float<T>(y[2 * i + 1]);
              out[2 * h + i] = *reinterpret_cast<const uint32_t*>(&two);
            }
          }
        }
        if constexpr (!kFull) stmatrix_trans(v_at + (c & 1) * L::kV + v_unit(np * 16 + (mi >> 1) * 8 + r8, mi & 1), out);
      }
    }

    // S
    {
      uint32_t hi[4][4], lo[4][4];
      float per_u[2];
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        const float2 f = *reinterpret_cast<const float2*>(&w.to_end[n * 8 + pair]);
#pragma unroll
        for (int e = 0; e < 4; ++e) U[n][e] *= e & 1 ? f.y : f.x;
      }
      largest(U, top);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        scale[h] = scale_for(top[h]);
        per_u[h] = unscale_for(scale[h]) * per_r[h];
      }
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) operand(U, kk, scale, hi[kk], lo[kk]);
      const float total = w.total, rest = w.total_rest;
#pragma unroll
      for (int np = 0; np < DK / 16; ++np) {
        float added[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) added[h][e] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const uint32_t at = kt + unit_at<DK>(kk * 16 + (mi & 1) * 8 + r8, 2 * np + (mi >> 1));
          uint32_t b[4];
          ptx::ldmatrix_x4_trans(at, b);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            mma(added[h], lo[kk], b[2 * h], b[2 * h + 1]);
            mma(added[h], hi[kk], b[2 * h], b[2 * h + 1]);
          }
          if (kFull) {
            ptx::ldmatrix_x4_trans(at + L::kRows, b);
#pragma unroll
            for (int h = 0; h < 2; ++h) mma(added[h], hi[kk], b[2 * h], b[2 * h + 1]);
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float& s = S[2 * np + h][e];
            s = fmaf(s, total, fmaf(s, rest, added[h][e] * per_u[e >> 1]));
            if (odd && from[e >> 1] < kChunk) s = __builtin_nanf("");
          }
      }
    }

    if constexpr (!kFull) {
      __syncwarp();
      T* o = static_cast<T*>(p.o) + (int64_t)head * p.dv + col0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + (lane >> 1), half = lane & 1;
        if (first + t < end) {
          const uint4 y = *reinterpret_cast<const uint4*>(generic + (v_at - smem) + (c & 1) * L::kV + v_unit(t, half));
          T* to = o + (int64_t)(first + t) * p.o_stride + half * 8;
          if (p.o_vectors) {
            if (col0 + half * 8 < p.dv) *reinterpret_cast<uint4*>(to) = y;
          } else {
            const Vec<T, 8> e = *reinterpret_cast<const Vec<T, 8>*>(&y);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (col0 + half * 8 + j < p.dv) to[j] = e.v[j];
          }
        }
      }
      __syncwarp();
    }
  }
};

// W warps of 16 columns each, then the helpers.
template <typename T, int DK, int W>
__global__ void __launch_bounds__((W + kHelpers) * 32, 1) delta_chunks_kernel(const ChunkParams p) {
  using L = Layout<T, DK>;
  extern __shared__ __align__(128) uint8_t dynamic_smem[];
  const uint32_t smem = smem_u32(dynamic_smem);
  Scratch& scratch = *reinterpret_cast<Scratch*>(dynamic_smem + L::kScratchAt);
  const int warp = ptx::warp_index();
  const uint32_t tile = blockIdx.x % (uint32_t)p.tiles, rest = blockIdx.x / (uint32_t)p.tiles;
  const int head = (int)(rest % (uint32_t)p.heads), b = (int)(rest / (uint32_t)p.heads);
  const int slot = slot_of(p.seqs, b);
  if (slot < 0) return;
  const SequenceRows rows = rows_of(p.seqs, b);
  const int chunks = (rows.end - rows.begin + kChunk - 1) / kChunk;
  const int64_t state_at = ((int64_t)slot * p.heads + head) * p.dk * p.dv;
  if (warp >= W) {
    if constexpr (W == 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    // (above the diagonal blocks nothing is written, and the products of T's halves meet it)
    for (int i = threadIdx.x - W * 32; i < kChunk * kAPitch; i += kHelpers * 32) (&scratch.A[0][0])[i] = 0.0f;
    for (int c = 0; c < chunks; ++c) {
      const int first = rows.begin + c * kChunk;
      prepare<T, DK>(p, head, first, min(first + kChunk, rows.end), smem, dynamic_smem, (c & 1) * L::kStage, scratch);
      __syncthreads();
    }
  } else {
    if constexpr (W == 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int col0 = ((int)tile * W + warp) * 16;
    Columns<T, DK> mine(p, smem, dynamic_smem, head, col0, warp);
    const bool live = col0 < p.dv;
    mine.states(live && p.state_in && resumes(p.seqs, b) ? p.state_in + state_at : nullptr);
    if (live) mine.load_v(0, rows.begin, rows.end);
    for (int c = 0; c < chunks; ++c) {
      __syncthreads();
      if (live) mine.chunk(c, rows.begin + c * kChunk, rows.end);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (live && p.state_out) mine.store_states(p.state_out + state_at);
  }
}

template <typename T, int DK, int W>
cudaError_t launch(ChunkParams& p, int32_t sequences, cudaStream_t stream) {
  constexpr uint32_t kBytes = Layout<T, DK>::bytes(W);
  static_assert(kBytes <= 227 * 1024, "");
  static bool attr_done[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!attr_done[dev]) {
    cudaError_t e = cudaFuncSetAttribute(delta_chunks_kernel<T, DK, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes);
    if (e != cudaSuccess) return e;
    // A build whose blocks start with fewer registers than the warpgroups ask for later would wait for them without end: not launched.
    cudaFuncAttributes built;
    e = cudaFuncGetAttributes(&built, delta_chunks_kernel<T, DK, W>);
    if (e != cudaSuccess) return e;
    if (W == 8 && built.numRegs * (W + kHelpers) * 32 < W * 32 * 208 + kHelpers * 32 * 88) return cudaErrorNotSupported;
    attr_done[dev] = true;
  }
  p.tiles = (p.dv + 16 * W - 1) / (16 * W);
  const int64_t grid = (int64_t)sequences * p.heads * p.tiles;
  if (grid >= ((int64_t)1 << 31)) return cudaErrorInvalidConfiguration;
  delta_chunks_kernel<T, DK, W><<<(unsigned)grid, (W + kHelpers) * 32, kBytes, stream>>>(p);
  return cudaGetLastError();
}

template <typename T, int DK>
cudaError_t launch_width(ChunkParams& p, int32_t sequences, cudaStream_t stream) {
  const int64_t columns = (int64_t)sequences * p.heads * ((p.dv + 15) / 16);
  if constexpr (sizeof(T) == 2) {
    if (p.dv > 64 && columns >= 148 * 8) return launch<T, DK, 8>(p, sequences, stream);
  }
  if (p.dv > 32 && columns >= 148 * 4) return launch<T, DK, 4>(p, sequences, stream);
  return launch<T, DK, 2>(p, sequences, stream);
}

template <typename T>
cudaError_t launch_type(ChunkParams& p, int32_t sequences, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  auto on = [&](const void* at, int64_t stride) { return aligned_to(at, 16) && stride % V == 0; };
  p.qk_vectors = p.dk % V == 0 && on(p.q, p.q_stride) && on(p.k, p.k_stride);
  p.v_vectors = p.dv % V == 0 && on(p.v, p.v_stride);
  p.o_vectors = p.dv % V == 0 && on(p.o, p.o_stride);
  return p.dk <= 64 ? launch_width<T, 64>(p, sequences, stream) : launch_width<T, 128>(p, sequences, stream);
}

}  // namespace

bool delta_by_chunks(const im2win_delta_shape& s, bool has_cu) {
  const int64_t longest = has_cu ? (s.max_len > 0 ? std::min(s.max_len, s.tokens) : s.tokens) : s.tokens / s.sequences;
  return s.dk <= 128 && longest > 16;
}

cudaError_t launch_delta_chunks(const DeltaArgs& a, cudaStream_t stream) {
  const im2win_delta_shape& s = a.shape;
  ChunkParams p = {a.q, a.k, a.v, a.decay, a.beta, a.o, a.state_in, a.state_out, a.seqs, s.q_stride, s.k_stride, s.v_stride, s.o_stride,
                   s.decay_stride, s.beta_stride, s.heads, s.heads / s.qk_heads, s.dk, s.dv, 0, s.normalize, 0, 0, 0, s.scale};
  switch (a.dtype) {
    case IM2WIN_F32: return launch_type<float>(p, s.sequences, stream);
    case IM2WIN_F16: return launch_type<__half>(p, s.sequences, stream);
    default: return launch_type<__nv_bfloat16>(p, s.sequences, stream);
  }
}

}  // namespace im2win
