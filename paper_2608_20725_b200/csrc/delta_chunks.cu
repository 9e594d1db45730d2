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
// and the split below, which is made of S, R and U in every chunk, costs the same issue slots.)  Four more warps, a team, make k, q, T, P
// and the weights of a chunk ahead; of 16-bit rows there are two teams, each with every second chunk.
//
// The state is fp32 and stays so.  The products with k and q, and the one that adds to S, are of two fp16 pieces, 22 bits: every row of an operand is
// brought to below 2^15 by a power of two first, so that what a piece leaves off is below 2^-39 of its row's largest element, whatever the type's range.
// That suits rows along dk, which are summed up anyway, and what all tokens of a chunk add to S.  R, U, T and P are another matter: tokens meet only
// those before them, which may be smaller by any factor, so that a scale for all of them would take their bits.  T R and P U are products of TF32
// pieces (11 and 11 bits), which have fp32's exponents; P U for o of bf16 of bf16 pieces (8 and 8, off by at most 2^-16: o's own rounding is 2^-9; S, P and
// U in one piece of 11 bits each put o off by 2% more, and 1e-3 of its norm away from what sums in fp32 give).  k and q of 16 bits are
// one piece, of fp32 two; S, R and U are two pieces (S k, U k: two products a term; T R and P U: three); T is inverted in blocks of 16 x 16, those on the
// diagonal by substitution in fp32, the others by TF32 products too.  Against 64 bits the states of 600 tokens are off by 2.3e-7 of their norm (of fp32
// rows by 3.3e-7, and o by 5.7e-7; token by token both are 2e-7).
//
// What bounds it (128 x 128, bf16): a chunk of 64 tokens takes a block of 32 columns 6.1 to 6.5 us by the box; its chains and o alone 4.4, a team alone,
// with every second chunk, 9.8.  Both are some 4000 instructions a warp, one after the other at about five cycles each (what the products, 8 cycles of an
// SM's quarter each, take is 2 us of the chain's).  The instruction cache is part of it: the code of a chunk, some 80 KB of which each warp runs its own part,
// misses it 500 times a chunk, which is why the code of helpers and of the warps that make o exists once and in loops.  One prompt of 16384 tokens, 32 heads
// of 128 x 128, bf16: 1560 to 1660 us (62 at 6.56 TB/s), fp16 1535 to 1630; token by token 22200.  13 prompts of 9001 tokens, 24 heads of 64 x 128, fp16:
// 364 (22), token by token 4090.
//
// Infinities and NaNs: a token whose k, beta or decay is not finite, and those behind it, get a beta of 0, a weight of NaN for o and a
// decay of NaN for S.  A column whose R or U is not finite from some token on is cleaned from there on, before it meets the zeros of T and P, and its
// o and S are made NaN.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "sequence.cuh"

namespace im2win {
namespace {

using ptx::smem_u32;

constexpr int kChunk = 64;

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
  float to_end[kChunk];                  // exp(G_n - G_j), without the scale of k
  float of_q[kChunk];                    // scale exp(G_i) of q S, without the scale of q
  float total, total_rest;               // exp(G_n) in two parts
  float pad[2];
};

constexpr int kBlock = 256;              // floats of a 16 x 16 block
struct Scratch {
  float A[6 * kBlock];                   // its blocks left of the diagonal, by rows of blocks
  float k_row[kChunk], q_row[kChunk];    // what k and q in pieces are multiplied by
  int whole[kChunk];                     // G_i in powers of two: its floor; the rest is in the factors of A's and P's rows and columns
  float of_a[kChunk], of_p[kChunk], of_column[kChunk];
  uint32_t bad_k[kChunk / 32], bad_q[kChunk / 32];             // rows that are not finite
  int broken;                            // the first token from which nothing is finite any more
  int64_t all;                           // G_n
};

// TEAMS of four helper warps, each with a chunk of its own.
template <typename T, int DK, int TEAMS>
struct Layout {
  static constexpr int kPieces = sizeof(T) == 4 ? 2 : 1;
  static constexpr int kSlots = TEAMS + 1;                     // chunks that are ready or being made
  static constexpr uint32_t kRows = kChunk * DK * 2;           // a piece of k or q
  static constexpr uint32_t kTriangle = 10 * kBlock * 4;       // T or P: their 16 x 16 blocks up to the diagonal, by rows of blocks
  static constexpr uint32_t kQAt = kPieces * kRows, kTAt = 2 * kPieces * kRows, kPAt = kTAt + kTriangle;
  // P U of bf16 rows: of two bf16 pieces each
  static constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  static constexpr uint32_t kWeightsAt = kPAt + kTriangle;
  static constexpr uint32_t kStage = (kWeightsAt + sizeof(Weights) + 127) / 128 * 128;
  static constexpr uint32_t kScratchAt = kSlots * kStage, kScratch = (sizeof(Scratch) + 127) / 128 * 128;
  static constexpr uint32_t kColumnsAt = kScratchAt + TEAMS * kScratch;
  // of a warp with columns: two chunks of v (16 bits), where o leaves through too; then, where another warp makes o, what it needs: S as operands, U,
  // three pairs a lane
  static constexpr uint32_t kV = sizeof(T) == 2 ? kChunk * 32 : 0;
  static constexpr uint32_t kSAt = 2 * kV, kUAt = kSAt + DK / 16 * 1024, kPairsAt = kUAt + 8 * 512;
  template <bool SPLIT> static constexpr uint32_t kColumns = SPLIT ? kPairsAt + 3 * 256 : 2 * kV;
};

// A power of two that brings numbers of at most `top` to below 2^15, and its reciprocal.
__device__ __forceinline__ float scale_for(float top) {
  const int e = (int)(__float_as_uint(top) >> 23 & 255u);
  return __uint_as_float((uint32_t)min(max(268 - e, 1), 253) << 23);
}
__device__ __forceinline__ float unscale_for(float scale) { return __uint_as_float((254u << 23) - __float_as_uint(scale)); }
// The same for an operand in TF32 pieces, which have fp32's exponents: only where the smaller piece would fall below fp32's range, or rounding pass it.
__device__ __forceinline__ float scale_for_tf32(float top) { return top < 0x1p-40f ? scale_for(top) : top > 0x1p120f ? 0x1p-8f : 1.0f; }

// 2^x of x in -1..1.
__device__ __forceinline__ float exp2_fraction(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
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
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Left: lane l has rows l / 4 and that + 8 of columns l % 4 (0, 1) and that + 4 (2, 3); right: rows l % 4 and that + 4 of column l / 4.
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pack_bf16(a, b);
  lo = pack_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
}
// x rounded to 22 bits, away from 0 in the middle (a NaN stays one: as a whole number it may not).
__device__ __forceinline__ float rounded_22(float x) { return fmaf(x, 0.0f, __uint_as_float((__float_as_uint(x) + 2u) & ~3u)); }
// Left operand from a tile of accumulators (rows g and g + 8, columns along its tokens) in pieces: rounded to 11 bits, and the rest, of which
// the instruction takes 11.  (By whole numbers: the conversion instruction takes its time, one prompt of 16384 tokens 1706 instead of 1634 us.)  Of its eight
// columns the even ones are taken for the first four, and so are the rows of right_tf32.
__device__ __forceinline__ void left_tf32(const float (&x)[4], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int to = (e & 1) * 2 + (e >> 1);
    hi[to] = (__float_as_uint(x[e]) + 0x1000u) & 0xffffe000u;
    lo[to] = __float_as_uint(x[e] - __uint_as_float(hi[to]));
  }
}
// A tile of R or U, rows scaled.
__device__ __forceinline__ void scaled(const float (&x)[4], const float (&scale)[2], float (&y)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = x[e] * scale[e >> 1];
}
// Right operand, of two numbers that are rounded to 22 bits: the first 11 of them, and the others.
__device__ __forceinline__ void right_tf32(const float* two, uint32_t (&hi)[2], uint32_t (&lo)[2]) {
  const float2 b = *reinterpret_cast<const float2*>(two);
  hi[0] = __float_as_uint(b.x) & 0xffffe000u;
  hi[1] = __float_as_uint(b.y) & 0xffffe000u;
  lo[0] = __float_as_uint(b.x - __uint_as_float(hi[0]));
  lo[1] = __float_as_uint(b.y - __uint_as_float(hi[1]));
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

// Byte of a 16-byte unit of row r of rows of N elements of 16 bits (units swizzled by the row, so that the matrix loads have no conflicts).
template <int N>
__device__ __forceinline__ uint32_t unit_at(int r, int unit) {
  return (uint32_t)(r * N * 2 + ((unit ^ (r & 7)) << 4));
}

// Block (i, k) of a triangle of 16 x 16 blocks with its diagonal, and without it; in a block, float (r, c), the halves of every second two rows
// swapped: eight rows of four pairs, as the matrix instructions take them, have no conflicts.
__host__ __device__ constexpr int block_at(int i, int k) { return (i * (i + 1) / 2 + k) * kBlock; }
__host__ __device__ constexpr int left_block_at(int i, int k) { return (i * (i - 1) / 2 + k) * kBlock; }
__host__ __device__ constexpr int float_at(int r, int c) { return r * 16 + (c ^ ((r & 2) << 2)); }
// The same of 16 bits: byte of half a row (16 bytes) r of block (i, k), the halves of every second four rows swapped, and of a piece.
__host__ __device__ constexpr int half_row_at(int i, int k, int r, int half) {
  return (i * (i + 1) / 2 + k) * 512 + r * 32 + ((half ^ (r >> 2 & 1)) << 4);
}
constexpr int kPieceOfP = 10 * 512;

// ------------------------------------------------------------------------------------------------ the helpers

// Eight elements of a row; 0 beyond `columns` and where the row is not there.
__device__ __forceinline__ void load8(const float* row, int at, int columns, bool there, float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (there && at + 4 * h < columns) w = __ldg(reinterpret_cast<const float4*>(row + at + 4 * h));
    x[4 * h] = w.x, x[4 * h + 1] = w.y, x[4 * h + 2] = w.z, x[4 * h + 3] = w.w;
  }
}

// Two elements of 16 bits: whether they are fp16 as they come, the larger magnitudes (a NaN is larger than anything), and both as floats.
template <typename T> struct Half;
template <> struct Half<__half> {
  static constexpr bool kExact = true;
  static __device__ __forceinline__ uint32_t largest(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("{\n\t.reg .b32 m;\n\tabs.f16x2 m, %2;\n\tmax.NaN.f16x2 %0, %1, m;\n\t}" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return unpack_half(w); }
};
template <> struct Half<__nv_bfloat16> {
  static constexpr bool kExact = false;
  static __device__ __forceinline__ uint32_t largest(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("{\n\t.reg .b32 m;\n\tabs.bf16x2 m, %2;\n\tmax.NaN.bf16x2 %0, %1, m;\n\t}" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
};

// A team of four warps that makes chunks.
template <typename T, int DK, int TEAMS>
struct Helpers {
  using L = Layout<T, DK, TEAMS>;

  const ChunkParams& p;
  uint32_t smem;
  uint8_t* generic;
  Scratch& s;
  int head, team, t, warp, lane;
  float g[2], b[2];                                            // (the first warp) of the next chunk

  __device__ __forceinline__ Helpers(const ChunkParams& p_, uint32_t smem_, uint8_t* generic_, int head_, int team_, int t_)
      : p(p_), smem(smem_), generic(generic_), s(*reinterpret_cast<Scratch*>(generic_ + L::kScratchAt + team_ * L::kScratch)), head(head_), team(team_),
        t(t_), warp(t_ >> 5), lane(t_ & 31) {}

  __device__ __forceinline__ void sync() const { asm volatile("bar.sync %0, 128;" ::"r"(14 + team) : "memory"); }

  // The team's next chunk: its decays and betas to registers, its rows to the L2 cache.
  __device__ __forceinline__ void fetch(int first, int end) {
    if (warp == 0) {
      g[0] = g[1] = b[0] = b[1] = 0.0f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t at = (int64_t)first + 2 * lane + i;
        if (at < end) {
          g[i] = p.decay[at * p.decay_stride + head];
          b[i] = p.beta[at * p.beta_stride + head];
        }
      }
    }
    const int64_t row = (int64_t)first + (t >> 1);
    const int64_t at = (int64_t)(head / p.share) * p.dk;
    constexpr int kLine = 128 / sizeof(T);
    if (row < end)
      for (int e = (t & 1) * kLine; e < p.dk; e += 2 * kLine) {
        asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const T*>(p.k) + at + row * p.k_stride + e));
        asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const T*>(p.q) + at + row * p.q_stride + e));
      }
  }

  // Rows of q or k of a chunk to shared memory, in pieces, scaled where they are not fp16 already.  Leaves what a row is multiplied by (the
  // norm's and the scale's reciprocals) and says which rows are not finite (they come out as 0).
  // Four threads have a row: rows base up to base + 31.
  __device__ __forceinline__ void rows(int base, const T* from, int64_t stride, int first, int end, uint32_t to, float* factor, uint32_t* bad) const {
    constexpr int kShare = 4, kUnits = DK / 8 / kShare;        // 16-byte units (of 16-bit elements) of a thread: every fourth one
    const int r = base + t / kShare, part = t % kShare;
    const bool there = first + r < end;
    const T* row = from + (there ? (int64_t)(first + r) * stride : 0);
    float top = 0.0f, squares[2] = {0.0f, 0.0f}, scale = 1.0f;
    if constexpr (sizeof(T) == 2) {
      uint4 x[kUnits];
      uint32_t most = 0;
      if (p.qk_vectors) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
          const int at = (i * kShare + part) * 8;
          x[i] = make_uint4(0, 0, 0, 0);
          if (there && at < p.dk) x[i] = __ldg(reinterpret_cast<const uint4*>(row + at));
        }
      } else {
        const uint16_t* e = reinterpret_cast<const uint16_t*>(row);
#pragma unroll 1
        for (int i = 0; i < kUnits; ++i) {
          const int at = (i * kShare + part) * 8;
          uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (there && at + j < p.dk) w[j / 2] |= (uint32_t)e[at + j] << (16 * (j & 1));
          ptx::st_shared16(to + unit_at<DK>(r, i * kShare + part), w[0], w[1], w[2], w[3]);
        }
#pragma unroll
        for (int i = 0; i < kUnits; ++i) x[i] = *reinterpret_cast<const uint4*>(generic + (to - smem) + unit_at<DK>(r, i * kShare + part));
      }
#pragma unroll
      for (int i = 0; i < kUnits; ++i)
#pragma unroll
        for (uint32_t w : {x[i].x, x[i].y, x[i].z, x[i].w}) {
          if (!Half<T>::kExact) most = Half<T>::largest(most, w);
          const float2 f = Half<T>::unpack(w);
          squares[0] = fmaf(f.x, f.x, squares[0]);
          squares[1] = fmaf(f.y, f.y, squares[1]);
        }
      if (Half<T>::kExact) {
        top = squares[0] + squares[1];                         // (of fp16 it is finite where the elements are)
      } else {
        const float2 f = Half<T>::unpack(most);
        top = max_nan(f.x, f.y);
      }
#pragma unroll
      for (int d = 1; d < kShare; d *= 2) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, d));
      const bool odd = !(top <= FLT_MAX);
      if (!Half<T>::kExact) scale = scale_for(top);
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (!Half<T>::kExact) {
            const float2 g = Half<T>::unpack(w[j]);
            w[j] = pack_half(g.x * scale, g.y * scale);
          }
          if (odd) w[j] = 0;
        }
        ptx::st_shared16(to + unit_at<DK>(r, i * kShare + part), w[0], w[1], w[2], w[3]);
      }
    } else {
      float x[kUnits][8];
      if (p.qk_vectors) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) load8(row, (i * kShare + part) * 8, p.dk, there, x[i]);
      } else {
#pragma unroll
        for (int i = 0; i < kUnits; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int at = (i * kShare + part) * 8 + j;
            x[i][j] = there && at < p.dk ? row[at] : 0.0f;
          }
      }
#pragma unroll
      for (int i = 0; i < kUnits; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          top = max_nan(top, fabsf(x[i][j]));
          squares[j & 1] = fmaf(x[i][j], x[i][j], squares[j & 1]);
        }
#pragma unroll
      for (int d = 1; d < kShare; d *= 2) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, d));
      const bool odd = !(top <= FLT_MAX);
      scale = scale_for(top);
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          split(x[i][2 * j] * scale, x[i][2 * j + 1] * scale, hi[j], lo[j]);
          if (odd) hi[j] = lo[j] = 0;
        }
        const uint32_t at = to + unit_at<DK>(r, i * kShare + part);
        ptx::st_shared16(at, hi[0], hi[1], hi[2], hi[3]);
        ptx::st_shared16(at + L::kRows, lo[0], lo[1], lo[2], lo[3]);
      }
    }
    squares[0] += squares[1];
#pragma unroll
    for (int d = 1; d < kShare; d *= 2) squares[0] += __shfl_xor_sync(0xffffffffu, squares[0], d);
    const bool odd = !(top <= FLT_MAX);
    const uint32_t odd_rows = __ballot_sync(0xffffffffu, odd); // (four bits a row)
    if (part == 0) factor[r] = odd ? 0.0f : (p.normalize ? rsqrtf(squares[0] + kNormalizeEps) : 1.0f) * unscale_for(scale);
    if (lane == 0) {
      uint32_t bits = 0;
      if (odd_rows) {
#pragma unroll 1
        for (int i = 0; i < 32 / kShare; ++i) bits |= (odd_rows >> (kShare * i) & 1u) << i;
      }
      reinterpret_cast<uint8_t*>(bad)[r >> 3] = (uint8_t)bits;
    }
  }

  // What the weigher keeps of its tokens, 2l and 2l+1, from k's weights to q's.
  struct Sums {
    int broken;                          // the first token from which nothing is finite any more
    float from_start[2], part[2];        // exp(G_i), and its part of a power of two
  };
  // One warp: lane l has tokens 2l and 2l+1.  Sums of log_decay are of whole numbers of 2^-44 powers of two: exact.
  __device__ __forceinline__ void weights_of_k(Weights& w, Sums& kept) const {
    auto powers = [](float x) -> int64_t {                     // (beyond 2^+-1000 nothing changes in fp32)
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
    const int first0 = odd[0] ? 2 * (__ffs(odd[0]) - 1) : kChunk, first1 = odd[1] ? 2 * (__ffs(odd[1]) - 1) + 1 : kChunk;
    const int broken = min(first0, first1);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (2 * lane + i >= broken) a[i] = 0;                    // (so that nothing that is finite meets what is not)
    int64_t sum = a[0] + a[1];
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int64_t other = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += other;
    }
    const int64_t all = __shfl_sync(0xffffffffu, sum, 31);
    kept.broken = broken;
    auto fraction = [](int64_t x) { return (float)((uint32_t)(x >> 20) & 0xffffffu) * 5.9604644775390625e-8f; };
    auto power = [&](int64_t x) { return exp2_fraction(fraction(x)) * power_of_two((int)(x >> 44)); };
    const int64_t G[2] = {sum - a[1], sum};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = 2 * lane + i;
      const float beta = at >= broken ? 0.0f : b[i], k_row = s.k_row[at];
      kept.part[i] = exp2_fraction(fraction(G[i]));
      kept.from_start[i] = kept.part[i] * power_of_two((int)(G[i] >> 44));
      s.whole[at] = (int)(G[i] >> 44);
      s.of_a[at] = beta * k_row * kept.part[i];
      s.of_column[at] = k_row * exp2_fraction(-fraction(G[i]));
      w.of_x[at] = beta * kept.from_start[i] * k_row;
      w.of_v[at] = beta;
      w.to_end[at] = power(all - G[i]) * k_row;
    }
    if (lane == 0) {
      s.broken = broken;
      s.all = all;
    }
  }
  __device__ __forceinline__ void weights_of_q(Weights& w, const Sums& kept) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = 2 * lane + i;
      const float q_row = s.q_row[at];
      const bool bad_q = (s.bad_q[lane >> 4] >> (at & 31) & 1u) != 0;
      s.of_p[at] = q_row * kept.part[i];
      w.of_q[at] = at >= kept.broken || bad_q ? __builtin_nanf("") : p.scale * kept.from_start[i] * q_row;
    }
  }
  // (by a warp that has little else to do: 64-bit powers take their time)
  __device__ __forceinline__ void total(Weights& w, int tokens) const {
    if (lane == 0) {
      const double exact = exp2((double)s.all * (1.0 / 17592186044416.0));
      const float rounded = (float)exact;
      w.total = s.broken < tokens ? __builtin_nanf("") : rounded;
      w.total_rest = (float)(exact - (double)rounded);
    }
  }

  // 16 rows (m) of products with k: the blocks left of the diagonal's, and that one.  (One piece of code for all warps and both k and q, loops rolled:
  // the code that a block's warps run for a chunk, each its own part, has to fit the instruction cache.  With a variant for each m, 140 KB in all,
  // a chunk of 32 columns of 128 x 128 took 14.4 us.)
  struct Square {
    float left[6][4], diagonal[2][4];
  };
  __device__ __forceinline__ void square(uint32_t rows_at, uint32_t kt, int m, Square& acc) const {
    const int mi = lane >> 3, r8 = lane & 7;
#pragma unroll
    for (int n = 0; n < 6; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc.left[n][i] = 0.0f;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc.diagonal[n][i] = 0.0f;
    const uint32_t a_at = rows_at + (m * 16 + (mi & 1) * 8 + r8) * DK * 2, b_at = kt + ((mi >> 1) * 8 + r8) * DK * 2, d_at = b_at + m * 16 * DK * 2;
#pragma unroll 2
    for (int ks = 0; ks < DK / 16; ++ks) {
      const uint32_t ua = (2 * ks + (mi >> 1)) ^ r8, ub = (2 * ks + (mi & 1)) ^ r8;            // (as unit_at)
      uint32_t a[L::kPieces][4], b[4][L::kPieces][4];
#pragma unroll
      for (int i = 0; i < L::kPieces; ++i) {
        ldmatrix(a_at + ua * 16 + i * L::kRows, a[i]);
        ldmatrix(d_at + ub * 16 + i * L::kRows, b[3][i]);
      }
#pragma unroll
      for (int np = 0; np < 3; ++np)
        if (np < m) {
#pragma unroll
          for (int i = 0; i < L::kPieces; ++i) ldmatrix(b_at + ub * 16 + np * 16 * DK * 2 + i * L::kRows, b[np][i]);
        }
#pragma unroll
      for (int np = 3; np >= 0; --np)                          // (the last one: the diagonal's)
        if (np < m || np == 3) {
#pragma unroll
          for (int u = L::kPieces == 2 ? 0 : 2; u < 3; ++u)    // (the small products first)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t(&f)[4] = b[np][u == 0 ? L::kPieces - 1 : 0];
              mma(np == 3 ? acc.diagonal[h] : acc.left[(np == 3 ? 0 : 2 * np) + h], a[u == 1 ? L::kPieces - 1 : 0], f[2 * h], f[2 * h + 1]);
            }
        }
    }
  }
  static __device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(min(max(e, -127), 127) + 127) << 23); }
  // times exp(G_i - G_j) and the factors of row and column; 0 above the diagonal, and on it for A.  Left of the diagonal's block
  // exp(G_i - G_j) is taken apart at the block's first token: what has i is the row's, what has j the column's.
  __device__ __forceinline__ void weigh(int m, Square& acc, const float* of_row, int diagonal) const {
    const int i0 = m * 16 + (lane >> 2), pair = (lane & 3) * 2;
    const int w[2] = {s.whole[i0], s.whole[i0 + 8]}, middle = s.whole[m * 16];
    const float f[2] = {of_row[i0], of_row[i0 + 8]}, near[2] = {f[0] * power_of_two(w[0] - middle), f[1] * power_of_two(w[1] - middle)};
#pragma unroll
    for (int n = 0; n < 6; ++n) {
      if (n >= 2 * m) break;
      const int2 wj = *reinterpret_cast<const int2*>(&s.whole[n * 8 + pair]);
      const float2 kj = *reinterpret_cast<const float2*>(&s.of_column[n * 8 + pair]);
      const float far[2] = {kj.x * power_of_two(middle - wj.x), kj.y * power_of_two(middle - wj.y)};
#pragma unroll
      for (int e = 0; e < 4; ++e) acc.left[n][e] *= near[e >> 1] * far[e & 1];
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int j = m * 16 + n * 8 + pair;
      const int2 wj = *reinterpret_cast<const int2*>(&s.whole[j]);
      const float2 kj = *reinterpret_cast<const float2*>(&s.of_column[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = acc.diagonal[n][e] * (f[e >> 1] * (e & 1 ? kj.y : kj.x)) * power_of_two(w[e >> 1] - (e & 1 ? wj.y : wj.x));
        acc.diagonal[n][e] = j + (e & 1) < i0 + (e >> 1) * 8 + diagonal ? x : 0.0f;
      }
    }
  }
  // Row m of the blocks of A (the diagonal's block as it is, into T's place) or of P, rounded to what their products take.
  template <bool OF_P>
  __device__ __forceinline__ void store(int m, const Square& acc, float* left, float* diagonal) const {
    const int at = float_at(lane >> 2, (lane & 3) * 2);
    auto put = [&](const float(&x)[4], float* to, bool exact) {
      *reinterpret_cast<float2*>(to) = exact ? make_float2(x[0], x[1]) : make_float2(rounded_22(x[0]), rounded_22(x[1]));
      *reinterpret_cast<float2*>(to + 8 * 16) = exact ? make_float2(x[2], x[3]) : make_float2(rounded_22(x[2]), rounded_22(x[3]));
    };
#pragma unroll
    for (int n = 0; n < 2; ++n) put(acc.diagonal[n], diagonal + (at ^ (n * 8)), !OF_P);
#pragma unroll
    for (int n = 0; n < 6; ++n) {
      if (n >= 2 * m) break;
      put(acc.left[n], left + (n >> 1) * kBlock + (at ^ ((n & 1) * 8)), false);
    }
  }
  // The same of P in bf16 pieces.
  __device__ __forceinline__ void store_bf16(int m, const Square& acc, uint8_t* to) const {
    auto put = [&](const float(&x)[4], int n) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t hi, lo;
        split_bf16(x[2 * h], x[2 * h + 1], hi, lo);
        uint8_t* at = to + half_row_at(m, n >> 1, (lane >> 2) + 8 * h, n & 1) + (lane & 3) * 4;
        *reinterpret_cast<uint32_t*>(at) = hi;
        *reinterpret_cast<uint32_t*>(at + kPieceOfP) = lo;
      }
    };
#pragma unroll
    for (int n = 0; n < 2; ++n) put(acc.diagonal[n], 2 * m + n);
#pragma unroll
    for (int n = 0; n < 6; ++n) {
      if (n >= 2 * m) break;
      put(acc.left[n], n);
    }
  }
  // The inverse of 1 and a diagonal block of A, in its place: by substitution, a column a lane.
  __device__ __forceinline__ void invert_block(float* d) const {
    const int j = lane & 15;                                   // (both halves of the warp do the same)
    float x[16];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float sum[2] = {i == j ? 1.0f : 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < i; k += 4) {
        const float4 a = *reinterpret_cast<const float4*>(d + float_at(i, k));
        sum[0] = fmaf(-a.x, x[k], sum[0]);
        if (k + 1 < i) sum[1] = fmaf(-a.y, x[k + 1], sum[1]);
        if (k + 2 < i) sum[0] = fmaf(-a.z, x[k + 2], sum[0]);
        if (k + 3 < i) sum[1] = fmaf(-a.w, x[k + 3], sum[1]);
      }
      x[i] = sum[0] + sum[1];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) d[float_at(i, j)] = rounded_22(x[i]);
  }

  // 16 columns J of T below the diagonal block: T_iJ = -T_ii sum_k A_ik T_kJ, i downward.  They are worked on transposed, so that what one product
  // gives is the next one's left operand.  By TF32 instructions, whose exponents need no scales: operands in two pieces, three products a term.
  __device__ __forceinline__ void columns_of_t(int J, float* T_blocks) const {
    const int g = lane >> 2, pair = (lane & 3) * 2, right = float_at(g, pair), turned = pair * 16 + (g ^ ((pair & 2) << 2));
    float x[2][4];
#pragma unroll 1
    for (int i = J + 1; i < 4; ++i) {
      float d[2][4], small[2][2][4];
#pragma unroll 1
      for (int k = J; k <= i; ++k) {                           // (the last step: T_ii times the sum of the others)
        if (k < i) {
          const float* at = T_blocks + block_at(k, J);         // rows of x are columns of T
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[n][e] = at[(turned ^ ((e >> 1) * 8)) + (n * 8 + (e & 1)) * 16];
        } else {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[n][e] = -(d[n][e] + (small[0][n][e] + small[1][n][e]));
        }
        if (k == J || k == i) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[n][e] = small[0][n][e] = small[1][n][e] = 0.0f;
        }
        const float* from = k < i ? s.A + left_block_at(i, k) : T_blocks + block_at(i, i);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          uint32_t ah[4], al[4], bh[2][2], bl[2][2];
          left_tf32(x[ks], ah, al);
#pragma unroll
          for (int n = 0; n < 2; ++n) right_tf32(from + n * 8 * 16 + (right ^ (ks * 8)), bh[n], bl[n]);
#pragma unroll
          for (int n = 0; n < 2; ++n) mma_tf32(d[n], ah, bh[n][0], bh[n][1]);
#pragma unroll
          for (int n = 0; n < 2; ++n) mma_tf32(small[0][n], al, bh[n][0], bh[n][1]);
#pragma unroll
          for (int n = 0; n < 2; ++n) mma_tf32(small[1][n], ah, bl[n][0], bl[n][1]);
        }
      }
      float* to = T_blocks + block_at(i, J);
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[(turned ^ ((e >> 1) * 8)) + (n * 8 + (e & 1)) * 16] = rounded_22(d[n][e] + (small[0][n][e] + small[1][n][e]));
      __syncwarp();
    }
  }

  // Chunk of rows first up to first + 64 (or end) into `stage`; the team's next one, two chunks on where there are two teams, is fetched.
  __device__ __forceinline__ void prepare(int first, int end, uint32_t stage) {
    Weights& w = *reinterpret_cast<Weights*>(generic + stage + L::kWeightsAt);
    const int64_t at = (int64_t)(head / p.share) * p.dk;
    const uint32_t kt = smem + stage, qt = kt + L::kQAt;
    const T* k = static_cast<const T*>(p.k) + at;
    const T* q = static_cast<const T*>(p.q) + at;
    // (each piece of code once, loops rolled: see square)
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
      const bool of_q = i > 1;
      rows((i & 1) * 32, of_q ? q : k, of_q ? p.q_stride : p.k_stride, first, end, of_q ? qt : kt, of_q ? s.q_row : s.k_row, of_q ? s.bad_q : s.bad_k);
    }
    sync();
    if (warp == 0) {
      Sums kept;
      weights_of_k(w, kept);
      weights_of_q(w, kept);
    }
    fetch(first + TEAMS * kChunk, end);
    // (A warp has row tile `warp` of A and of P, and column tile `warp` of T: what is long of the ones is short of the other.)
#pragma unroll 1
    for (int of_q = 0; of_q < 2; ++of_q) {
      Square acc;
      square(of_q ? qt : kt, kt, warp, acc);
      if (!of_q) sync();                                       // (the weights)
      weigh(warp, acc, of_q ? s.of_p : s.of_a, of_q);
      if (of_q) {
        float* P = reinterpret_cast<float*>(generic + stage + L::kPAt);
        if constexpr (L::kBf16) store_bf16(warp, acc, generic + stage + L::kPAt);
        else store<true>(warp, acc, P + block_at(warp, 0), P + block_at(warp, warp));
      } else {
        float* T_blocks = reinterpret_cast<float*>(generic + stage + L::kTAt);
        store<false>(warp, acc, s.A + left_block_at(warp, 0), T_blocks + block_at(warp, warp));
        invert_block(T_blocks + block_at(warp, warp));
        sync();
        columns_of_t(warp, T_blocks);
      }
    }
    if (warp == 3) total(w, min(end - first, kChunk));
  }
};

// ------------------------------------------------------------------------------------------------ the columns of a warp

// Rows g and g + 8 of accumulators over tokens: from the first token on whose number is not finite all become 0; `from` says which.
__device__ __forceinline__ void clean(float (&x)[8][4], int (&from)[2]) {
  const int pair = (threadIdx.x & 3) * 2;
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (!(fabsf(x[n][e]) <= FLT_MAX)) from[e >> 1] = min(from[e >> 1], n * 8 + pair + (e & 1));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    from[h] = min(from[h], __shfl_xor_sync(0xffffffffu, from[h], 1));
    from[h] = min(from[h], __shfl_xor_sync(0xffffffffu, from[h], 2));
  }
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n * 8 + pair + (e & 1) >= from[e >> 1]) x[n][e] = 0.0f;
}

// The largest magnitude of rows g and g + 8, in all four lanes that share them; a NaN where there is one.
template <int N>
__device__ __forceinline__ void largest(const float (&x)[N][4], float (&top)[2]) {
  float m[4][2];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float two = max_nan(fabsf(x[n][2 * h]), fabsf(x[n][2 * h + 1]));
      m[n & 3][h] = n < 4 ? two : max_nan(m[n & 3][h], two);
    }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    top[h] = max_nan(max_nan(m[0][h], m[1][h]), max_nan(m[2][h], m[3][h]));
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

// 16 columns of a head.  SPLIT: one warp has the chain from S to S, another one makes o from S and U in fp16, which the first leaves in shared memory; it says
// so at two barriers of the pair.  Otherwise one warp does both.
template <typename T, int DK, bool SPLIT, int TEAMS>
struct Columns {
  using L = Layout<T, DK, TEAMS>;
  static constexpr bool kFull = L::kPieces == 2;               // fp32 rows
  static_assert(!(kFull && SPLIT), "");

  const ChunkParams& p;
  uint32_t smem, at0;
  uint8_t* generic;
  int head, col0, index, lane, mi, r8, group, pair;

  __device__ __forceinline__ Columns(const ChunkParams& p_, uint32_t smem_, uint8_t* generic_, int head_, int col0_, int index_)
      : p(p_), smem(smem_), at0(L::kColumnsAt + L::template kColumns<SPLIT> * index_), generic(generic_), head(head_), col0(col0_), index(index_) {
    lane = threadIdx.x & 31;
    mi = lane >> 3, r8 = lane & 7, group = lane >> 2, pair = (lane & 3) * 2;
  }
  __device__ __forceinline__ void states(const float* from, float (&S)[DK / 8][4]) const {
#pragma unroll
    for (int n = 0; n < DK / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = n * 8 + pair + (e & 1), c = col0 + group + 8 * (e >> 1);
        S[n][e] = from && d < p.dk && c < p.dv ? from[(int64_t)d * p.dv + c] : 0.0f;
      }
  }
  __device__ __forceinline__ void store_states(float* to, const float (&S)[DK / 8][4]) const {
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
      const uint32_t to = smem + at0 + buffer * L::kV;
      if (p.v_vectors) {
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
          const int t = i * 16 + (lane >> 1), half = lane & 1;
          const bool there = first + t < end && col0 + half * 8 < p.dv;
          copy16(to + v_unit(t, half), there ? v + (int64_t)(first + t) * p.v_stride + half * 8 : v, there);
        }
      } else {
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
          const int t = i * 16 + (lane >> 1), half = lane & 1;
          const bool row = first + t < end;
          const uint16_t* e = reinterpret_cast<const uint16_t*>(v + (row ? (int64_t)(first + t) * p.v_stride + half * 8 : 0));
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

  // What the warp that makes o waits for: S of a chunk (which == 0), its U (1).
  __device__ __forceinline__ void announce(int which) const { asm volatile("bar.arrive %0, 64;" ::"r"(2 + 2 * index + which) : "memory"); }
  __device__ __forceinline__ void await(int which) const { asm volatile("bar.sync %0, 64;" ::"r"(2 + 2 * index + which) : "memory"); }
  template <typename V>
  __device__ __forceinline__ V& lane_pair(int which) const { return reinterpret_cast<V*>(generic + at0 + L::kPairsAt + which * 256)[lane]; }

  // O += S q of 32 tokens (half), one step of dk: the products of the small pieces, of the large ones, or both.  (What an instruction adds to an
  // accumulator is cut off, not rounded: small products that come first lose less.)
  template <bool SMALL, bool LARGE>
  __device__ __forceinline__ void multiply_q(uint32_t qt, int half, int ks, const uint32_t (&hi)[4], const uint32_t (&lo)[4], float (&O)[4][4]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t at = qt + unit_at<DK>((2 * half + i) * 16 + (mi >> 1) * 8 + r8, 2 * ks + (mi & 1));
      uint32_t a[4];
      ldmatrix(at, a);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (SMALL) mma(O[2 * i + h], lo, a[2 * h], a[2 * h + 1]);
        if (LARGE) mma(O[2 * i + h], hi, a[2 * h], a[2 * h + 1]);
      }
      if (kFull && SMALL) {
        ldmatrix(at + L::kRows, a);
#pragma unroll
        for (int h = 0; h < 2; ++h) mma(O[2 * i + h], hi, a[2 * h], a[2 * h + 1]);
      }
    }
  }

  // o of 32 tokens (half): q S, which O holds, and P U; tile(n, x) gives U's tokens 8 n up to 8 n + 7.  16 bits: to shared memory.
  template <typename Tile>
  __device__ __forceinline__ void finish_o(uint32_t P_at, const Weights& w, int half, const float (&O)[4][4], const float (&per_s)[2],
                                           const float (&per_o)[2], const Tile& tile, bool odd, const int (&from)[2], uint32_t out_at, int first,
                                           int end) const {
    constexpr int kSmall = kFull ? 4 : 1;                      // fp32 rows: sums of the small products of their own (o off by 5.7e-7 instead of 7.4e-7)
    float I[4][4], small[kSmall][4];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) I[n][e] = small[n < kSmall ? n : 0][e] = 0.0f;
    auto block = [&](int kk) {                                 // of 16 tokens of U
      if constexpr (L::kBf16) {
        uint32_t hi[4], lo[4], b[2][4], bl[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float x[4];
          tile(2 * kk + i, x);
          split_bf16(x[0], x[1], hi[2 * i], lo[2 * i]);
          split_bf16(x[2], x[3], hi[2 * i + 1], lo[2 * i + 1]);
          if (kk > 2 * half + i) continue;
          const uint32_t at = smem + P_at + half_row_at(2 * half + i, kk, (mi >> 1) * 8 + r8, mi & 1);
          ldmatrix(at, b[i]);
          ldmatrix(at + kPieceOfP, bl[i]);
        }
#pragma unroll
        for (int m = 0; m < 3; ++m)                            // (the small products first)
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            if (kk > 2 * half + (t >> 1)) continue;
            const uint32_t(&f)[4] = m == 1 ? bl[t >> 1] : b[t >> 1];
            mma_bf16(I[t], m == 0 ? lo : hi, f[2 * (t & 1)], f[2 * (t & 1) + 1]);
          }
      } else {
        const float* P = reinterpret_cast<const float*>(generic + P_at);
#pragma unroll
        for (int n = 2 * kk; n < 2 * kk + 2; ++n) {
          float x[4];
          uint32_t hi[4], lo[4], bh[4][2], bl[4][2];
          tile(n, x);
          left_tf32(x, hi, lo);
#pragma unroll
          for (int t = 0; t < 4; ++t)                          // (P is 0 where its tokens come before U's)
            if (n <= 4 * half + t)
              right_tf32(P + block_at(2 * half + (t >> 1), kk) + (t & 1) * 8 * 16 + float_at(group, (n & 1) * 8 + pair), bh[t], bl[t]);
#pragma unroll
          for (int m = 0; m < 3; ++m)
#pragma unroll
            for (int t = 0; t < 4; ++t)
              if (n <= 4 * half + t) {
                const uint32_t(&f)[2] = m == 1 ? bl[t] : bh[t];
                mma_tf32(kFull && m < 2 ? small[t < kSmall ? t : 0] : I[t], m == 0 ? lo : hi, f[0], f[1]);
              }
        }
      }
    };
    if constexpr (SPLIT) {                                     // (less code for the instruction cache: the long prompt 1616 to 1559 us)
#pragma unroll 1
      for (int kk = 0; kk < 2 * half + 2; ++kk) block(kk);
    } else {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        if (kk < 2 * half + 2) block(kk);
    }
    if constexpr (kFull) {
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) I[n][e] += small[n][e];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t out[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = (4 * half + 2 * i + h) * 8 + pair;
        const float2 fq = *reinterpret_cast<const float2*>(&w.of_q[t]);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          y[e] = fmaf((e & 1 ? fq.y : fq.x) * per_s[e >> 1], O[2 * i + h][e], p.scale * per_o[e >> 1] * I[2 * i + h][e]);
        if (odd) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t + (e & 1) >= from[e >> 1]) y[e] = __builtin_nanf("");
        }
        if constexpr (kFull) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = first + t + (e & 1), at = col0 + group + 8 * (e >> 1);
            if (row < end && at < p.dv) static_cast<float*>(p.o)[(int64_t)row * p.o_stride + (int64_t)head * p.dv + at] = y[e];
          }
        } else {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            Vec<T, 2> two;
            two.v[0] = from_float<T>(y[2 * j]);
            two.v[1] = from_float<T>(y[2 * j + 1]);
            out[2 * h + j] = *reinterpret_cast<const uint32_t*>(&two);
          }
        }
      }
      if constexpr (!kFull) stmatrix_trans(smem + out_at + v_unit((2 * half + i) * 16 + (mi >> 1) * 8 + r8, mi & 1), out);
    }
  }
  // (16 bits) o of the chunk from shared memory to where it belongs
  __device__ __forceinline__ void store_o(uint32_t out_at, int first, int end) const {
    if constexpr (!kFull) {
      __syncwarp();
      T* o = static_cast<T*>(p.o) + (int64_t)head * p.dv + col0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = i * 16 + (lane >> 1), half = lane & 1;
        if (first + t < end) {
          const uint4 y = *reinterpret_cast<const uint4*>(generic + out_at + v_unit(t, half));
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

  // o of chunk c, by the warp beside the chain's.
  __device__ __forceinline__ void chunk_o(int c, uint32_t stage, int first, int end) const {
    const Weights& w = *reinterpret_cast<const Weights*>(generic + stage + L::kWeightsAt);
    float O[2][4][4];
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) O[n >> 2][n & 3][e] = 0.0f;
    auto handed_s = [&](int i, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
      const uint4* from = reinterpret_cast<const uint4*>(generic + at0 + L::kSAt) + i * 32 + lane;
      const uint4 x = from[0];
      hi[0] = x.x, hi[1] = x.y, hi[2] = x.z, hi[3] = x.w;
      const uint4 y = from[DK / 16 * 32];
      lo[0] = y.x, lo[1] = y.y, lo[2] = y.z, lo[3] = y.w;
    };
    await(0);
#pragma unroll 1
    for (int ks = 0; ks < DK / 16; ++ks) {
      uint32_t hi[4], lo[4];
      handed_s(ks, hi, lo);
#pragma unroll
      for (int half = 0; half < 2; ++half) multiply_q<true, true>(smem + stage + L::kQAt, half, ks, hi, lo, O[half]);
    }
    await(1);
    const float2 ps = lane_pair<float2>(0), po = lane_pair<float2>(1);
    const int2 f = lane_pair<int2>(2);
    const float per_s[2] = {ps.x, ps.y}, per_o[2] = {po.x, po.y};
    const int from[2] = {f.x, f.y};
    const bool odd = __any_sync(0xffffffffu, min(f.x, f.y) < kChunk);
#pragma unroll
    for (int half = 0; half < 2; ++half)
      finish_o(stage + L::kPAt, w, half, O[half], per_s, per_o,
               [&](int n, float(&x)[4]) {
                 const float4 y = reinterpret_cast<const float4*>(generic + at0 + L::kUAt)[n * 32 + lane];
                 x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
               },
               odd, from, at0 + (c & 1) * L::kV, first, end);
    store_o(at0 + (c & 1) * L::kV, first, end);        // (v of the chunk has been read: seen with U)
  }

  // S of chunk c, and its o too where no other warp makes it.
  __device__ __forceinline__ void chunk(int c, uint32_t stage, int first, int end, float (&S)[DK / 8][4]) const {
    const uint32_t kt = smem + stage, qt = kt + L::kQAt;
    const float* T_blocks = reinterpret_cast<const float*>(generic + stage + L::kTAt);
    const Weights& w = *reinterpret_cast<const Weights*>(generic + stage + L::kWeightsAt);
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

    // k S
    constexpr bool kBeside = !SPLIT && !kFull;                 // q S beside k S (of fp32 rows there are not the registers)
    float X[8][4], O[kBeside ? 2 : 1][4][4], top[2], scale[2], scale_s[2], per_s[2];
    auto clear = [](float (&x)[4][4]) {
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = 0.0f;
    };
    if constexpr (kBeside) clear(O[0]), clear(O[1]);
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) X[n][e] = 0.0f;
    largest(S, top);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      scale_s[h] = scale_for(top[h]);
      per_s[h] = unscale_for(scale_s[h]);
    }
#pragma unroll
    for (int ks = 0; ks < DK / 16; ++ks) {
      uint32_t hi[4], lo[4];
      operand(S, ks, scale_s, hi, lo);
      if constexpr (SPLIT) {
        const uint32_t to = smem + at0 + L::kSAt + (ks * 32 + lane) * 16;
        ptx::st_shared16(to, hi[0], hi[1], hi[2], hi[3]);
        ptx::st_shared16(to + DK / 16 * 512, lo[0], lo[1], lo[2], lo[3]);
      }
      if constexpr (kBeside) {
#pragma unroll
        for (int half = 0; half < 2; ++half) multiply_q<true, true>(qt, half, ks, hi, lo, O[half]);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {                   // (four accumulators, so that a product does not wait for the one before)
        uint32_t b[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) ldmatrix(kt + unit_at<DK>((2 * half + i) * 16 + (mi >> 1) * 8 + r8, 2 * ks + (mi & 1)), b[i]);
#pragma unroll
        for (int n = 0; n < 4; ++n) mma(X[4 * half + n], lo, b[n >> 1][2 * (n & 1)], b[n >> 1][2 * (n & 1) + 1]);
#pragma unroll
        for (int n = 0; n < 4; ++n) mma(X[4 * half + n], hi, b[n >> 1][2 * (n & 1)], b[n >> 1][2 * (n & 1) + 1]);
        if (kFull) {
#pragma unroll
          for (int i = 0; i < 2; ++i) ldmatrix(kt + L::kRows + unit_at<DK>((2 * half + i) * 16 + (mi >> 1) * 8 + r8, 2 * ks + (mi & 1)), b[i]);
#pragma unroll
          for (int n = 0; n < 4; ++n) mma(X[4 * half + n], hi, b[n >> 1][2 * (n & 1)], b[n >> 1][2 * (n & 1) + 1]);
        }
      }
    }
    if constexpr (SPLIT) {
      lane_pair<float2>(0) = make_float2(per_s[0], per_s[1]);
      announce(0);
    }

    // R, in the place of k S
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncwarp();
#pragma unroll
    for (int np = 0; np < 4; ++np) {
      uint32_t vv[4] = {0, 0, 0, 0};
      if constexpr (!kFull) ptx::ldmatrix_x4_trans(smem + at0 + (c & 1) * L::kV + v_unit(np * 16 + (mi >> 1) * 8 + r8, mi & 1), vv);
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
      scale[h] = scale_for_tf32(top[h]);
      per_r[h] = unscale_for(scale[h]);
    }

    // U (times R's scale): eight tokens of R at a time with four tiles of T's rows
    float U[8][4];
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) U[n][e] = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      float x[4];
      uint32_t hi[4], lo[4];
      scaled(X[n], scale, x);
      left_tf32(x, hi, lo);
#pragma unroll
      for (int t0 = n / 4 * 4; t0 < 8; t0 += 4) {
        uint32_t bh[4][2], bl[4][2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (n <= t0 + t)
            right_tf32(T_blocks + block_at((t0 + t) >> 1, n >> 1) + (t & 1) * 8 * 16 + float_at(group, (n & 1) * 8 + pair), bh[t], bl[t]);
#pragma unroll
        for (int m = 0; m < 3; ++m)                            // (the small products first)
#pragma unroll
          for (int t = 0; t < 4; ++t)
            if (n <= t0 + t) {
              const uint32_t(&f)[2] = m == 1 ? bl[t] : bh[t];
              mma_tf32(U[t0 + t], m == 0 ? lo : hi, f[0], f[1]);
            }
      }
    }
    largest(U, top);
    if (__any_sync(0xffffffffu, !(max_nan(top[0], top[1]) <= FLT_MAX))) {
      odd = true;
      clean(U, from);
      largest(U, top);
    }

    // o, or what the other warp makes it from
    {
      float per_o[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        scale[h] = scale_for_tf32(top[h]);
        per_o[h] = unscale_for(scale[h]) * per_r[h];
      }
      if constexpr (SPLIT) {
#pragma unroll
        for (int n = 0; n < 8; ++n)
          reinterpret_cast<float4*>(generic + at0 + L::kUAt)[n * 32 + lane] =
              make_float4(U[n][0] * scale[0], U[n][1] * scale[0], U[n][2] * scale[1], U[n][3] * scale[1]);
        lane_pair<float2>(1) = make_float2(per_o[0], per_o[1]);
        lane_pair<int2>(2) = make_int2(from[0], from[1]);
        announce(1);
      } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float(&q_s)[4][4] = O[kBeside ? half : 0];
          if constexpr (!kBeside) {                            // (S is taken apart again, 32 tokens at a time)
            clear(q_s);
#pragma unroll
            for (int ks = 0; ks < DK / 16; ++ks) {
              uint32_t hi[4], lo[4];
              operand(S, ks, scale_s, hi, lo);
              multiply_q<true, false>(qt, half, ks, hi, lo, q_s);
            }
#pragma unroll
            for (int ks = 0; ks < DK / 16; ++ks) {
              uint32_t hi[4], lo[4];
              operand(S, ks, scale_s, hi, lo);
              multiply_q<false, true>(qt, half, ks, hi, lo, q_s);
            }
          }
          finish_o(stage + L::kPAt, w, half, q_s, per_s, per_o, [&](int n, float(&x)[4]) { scaled(U[n], scale, x); }, odd, from, at0 + (c & 1) * L::kV,
                   first, end);
        }
        store_o(at0 + (c & 1) * L::kV, first, end);
      }
    }

    // S
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
    uint32_t hi[4][4], lo[4][4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) operand(U, kk, scale, hi[kk], lo[kk]);
    const float total = w.total, rest = w.total_rest;
#pragma unroll
    for (int np = 0; np < DK / 16; np += 2) {
      float added[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) added[n][e] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        uint32_t b[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) ptx::ldmatrix_x4_trans(kt + unit_at<DK>(kk * 16 + (mi & 1) * 8 + r8, 2 * (np + i) + (mi >> 1)), b[i]);
#pragma unroll
        for (int n = 0; n < 4; ++n) mma(added[n], lo[kk], b[n >> 1][2 * (n & 1)], b[n >> 1][2 * (n & 1) + 1]);
#pragma unroll
        for (int n = 0; n < 4; ++n) mma(added[n], hi[kk], b[n >> 1][2 * (n & 1)], b[n >> 1][2 * (n & 1) + 1]);
        if (kFull) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            ptx::ldmatrix_x4_trans(kt + L::kRows + unit_at<DK>(kk * 16 + (mi & 1) * 8 + r8, 2 * (np + i) + (mi >> 1)), b[i]);
#pragma unroll
          for (int n = 0; n < 4; ++n) mma(added[n], hi[kk], b[n >> 1][2 * (n & 1)], b[n >> 1][2 * (n & 1) + 1]);
        }
      }
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float& s = S[2 * np + n][e];
          s = fmaf(s, total, fmaf(s, rest, added[n][e] * per_u[e >> 1]));
        }
    }
    if (odd) {
#pragma unroll
      for (int n = 0; n < DK / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (from[e >> 1] < kChunk) S[n][e] = __builtin_nanf("");
    }
  }
};

// How a block's warps share the work: W with the chains of 16 columns each, with SPLIT as many that make o, then TEAMS of four helpers.  Registers: of
// the warpgroups with columns and of the helpers' (0: as launched); they ask for no more than the block is launched with.
template <int W_, bool SPLIT_, int TEAMS_, int CHAIN, int HELP>
struct Shape {
  static constexpr int W = W_, TEAMS = TEAMS_, kWarps = SPLIT_ ? 2 * W_ : W_, kThreads = (kWarps + 4 * TEAMS_) * 32;
  static constexpr bool SPLIT = SPLIT_;
  static constexpr int kChain = CHAIN, kHelp = HELP, kAsked = kWarps * 32 * CHAIN + 4 * TEAMS_ * 32 * HELP;
  static_assert(CHAIN == 0 || (kWarps % 4 == 0 && kAsked <= 65536 / kThreads / 8 * 8 * kThreads), "");
};

// Chunk c is ready, and chunk c - 1 done with: a barrier for even and one for odd chunks, at which a team does not wait for the other one's chunks.
template <int THREADS>
__device__ __forceinline__ void chunk_barrier(int c, bool wait) {
  if (wait) asm volatile("bar.sync %0, %1;" ::"r"((c & 1) * 13), "n"(THREADS) : "memory");
  else asm volatile("bar.arrive %0, %1;" ::"r"((c & 1) * 13), "n"(THREADS) : "memory");
}

template <typename T, int DK, typename F>
__global__ void __launch_bounds__(F::kThreads, 1) delta_chunks_kernel(const ChunkParams p) {
  using L = Layout<T, DK, F::TEAMS>;
  constexpr int W = F::W;
  extern __shared__ __align__(128) uint8_t dynamic_smem[];
  const uint32_t smem = smem_u32(dynamic_smem);
  const int warp = ptx::warp_index();
  const uint32_t tile = blockIdx.x % (uint32_t)p.tiles, rest = blockIdx.x / (uint32_t)p.tiles;
  const int head = (int)(rest % (uint32_t)p.heads), b = (int)(rest / (uint32_t)p.heads);
  const int slot = slot_of(p.seqs, b);
  if (slot < 0) return;
  const SequenceRows rows = rows_of(p.seqs, b);
  const int chunks = (rows.end - rows.begin + kChunk - 1) / kChunk;
  const int64_t state_at = ((int64_t)slot * p.heads + head) * p.dk * p.dv;
  uint32_t stage = 0;
  auto next = [&]() { stage = stage == (L::kSlots - 1) * L::kStage ? 0 : stage + L::kStage; };
  if (warp >= F::kWarps) {
    if constexpr (F::kChain > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F::kHelp));
    const int t = (int)threadIdx.x - F::kWarps * 32, team = (warp - F::kWarps) >> 2;
    Helpers<T, DK, F::TEAMS> helpers(p, smem, dynamic_smem, head, team, t & 127);
    helpers.fetch(rows.begin + team * kChunk, rows.end);
    // (Chunk c goes where chunk c - slots was.  Of one team that is the chunk before the last: done with at the barrier behind it.  Of two, the team
    // begins chunk c behind the barrier of chunk c - 2, where c - 3 is done with.)
    for (int c = 0; c < chunks; ++c, next()) {
      const bool mine = F::TEAMS == 1 || (c & 1) == team;
      if (mine) helpers.prepare(rows.begin + c * kChunk, rows.end, stage);
      chunk_barrier<F::kThreads>(c, mine);
    }
  } else {
    if constexpr (F::kChain > 0) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(F::kChain));
    const int index = F::SPLIT && warp >= W ? warp - W : warp, col0 = ((int)tile * W + index) * 16;
    const Columns<T, DK, F::SPLIT, F::TEAMS> mine(p, smem, dynamic_smem, head, col0, index);
    const bool live = col0 < p.dv;
    if (!F::SPLIT || warp < W) {
      float S[DK / 8][4];
      mine.states(live && p.state_in && resumes(p.seqs, b) ? p.state_in + state_at : nullptr, S);
      if (live) mine.load_v(0, rows.begin, rows.end);
      for (int c = 0; c < chunks; ++c, next()) {
        chunk_barrier<F::kThreads>(c, true);
        if (live) mine.chunk(c, stage, rows.begin + c * kChunk, rows.end, S);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (live && p.state_out) mine.store_states(p.state_out + state_at, S);
    } else if constexpr (F::SPLIT) {
      for (int c = 0; c < chunks; ++c, next()) {
        chunk_barrier<F::kThreads>(c, true);
        if (live) mine.chunk_o(c, stage, rows.begin + c * kChunk, rows.end);
      }
    }
  }
}

template <typename T, int DK, typename F>
cudaError_t launch(ChunkParams& p, int32_t sequences, cudaStream_t stream) {
  using L = Layout<T, DK, F::TEAMS>;
  constexpr uint32_t kBytes = L::kColumnsAt + F::W * L::template kColumns<F::SPLIT>;
  static_assert(kBytes <= 227 * 1024, "");
  static bool attr_done[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!attr_done[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(delta_chunks_kernel<T, DK, F>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes);
    if (e != cudaSuccess) return e;
    // A build whose blocks start with fewer registers than the warpgroups ask for later would wait for them without end: not launched.
    cudaFuncAttributes built;
    const cudaError_t asked = cudaFuncGetAttributes(&built, delta_chunks_kernel<T, DK, F>);
    if (asked != cudaSuccess) return asked;
    if (F::kChain > 0 && built.numRegs * F::kThreads < F::kAsked) return cudaErrorNotSupported;
    attr_done[dev] = true;
  }
  p.tiles = (p.dv + 16 * F::W - 1) / (16 * F::W);
  const int64_t grid = (int64_t)sequences * p.heads * p.tiles;
  if (grid >= ((int64_t)1 << 31)) return cudaErrorInvalidConfiguration;
  delta_chunks_kernel<T, DK, F><<<(unsigned)grid, F::kThreads, kBytes, stream>>>(p);
  return cudaGetLastError();
}

// The columns of a block: 32 while that gives no more blocks than there are SMs, 64 beyond.  (A chunk of 64 tokens, 128 x 128 in bf16, takes a block of
// 32 columns 6.1 to 6.5 us; of 64 columns, with all SMs at work, 9.7: four prompts of 8192 tokens in all 620.)  fp32: its pieces leave shared memory
// for one team, and registers for o beside the chain.
template <typename T, int DK>
cudaError_t launch_width(ChunkParams& p, int32_t sequences, cudaStream_t stream) {
  const bool wide = p.dv > 32 && (int64_t)sequences * p.heads * ((p.dv + 31) / 32) > 148;
  if constexpr (sizeof(T) == 4) {
    if (wide) return launch<T, DK, Shape<4, false, 1, 0, 0>>(p, sequences, stream);
    return launch<T, DK, Shape<2, false, 1, 0, 0>>(p, sequences, stream);
  } else {
    if (!wide) return launch<T, DK, Shape<2, true, 2, 224, 136>>(p, sequences, stream);
    return launch<T, DK, Shape<4, false, 2, 232, 136>>(p, sequences, stream);
  }
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
