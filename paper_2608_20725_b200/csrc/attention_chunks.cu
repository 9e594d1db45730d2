// Linear attention with a decay for each head, by chunks of 64 tokens on the tensor cores (im2win_linear_attention).
//
// With G_i the sum of log_decay up to and including token i of a chunk, S the state before it and n its tokens:
//
//   o_i  = scale ( exp(G_i) q_i S  +  sum_{j <= i} exp(G_i - G_j) (q_i . k_j) v_j )        "inter" and "intra"
//   S   <- exp(G_n) S + sum_j exp(G_n - G_j) k_j^T v_j                                      "added"
//
// A block has one head, a tile of 128 columns of dv and a run of chunks of one sequence.  S stays in its registers, transposed: a
// thread has a column of dv and a quarter of dk.  All products with S or v are made transposed, so that their 128 rows are dv:
//
//   inter^T [dv][64 tokens] = S^T (16 bits, tensor memory) x q        added^T [dv][dk] = v^T x (weighted k)
//   intra^T [dv][64 tokens] = v^T x P,  P_ij = exp(G_i - G_j) (q_i . k_j)
//
// v^T and the weighted k are read as they lie, rows of tokens, as operands whose 64 elements of a row are innermost along M or N
// (transposed by the descriptor); the 64 x 64 products q . k are one more (64 rows: by the warps
// they would take issue slots, which are short) and come to registers to be weighted and masked.
//
// What is rounded to 16 bits: P and the copy of S that meets q, once each, as the result o is; their errors and o's own rounding are of
// one size and independent.  The weighted k are not: the state is carried from call to call in fp32 and has to stay fp32, so they go
// through the tensor cores as three pieces whose sum is the fp32 product (of bf16: cut off; of fp16: each 2^12 times what it stands for
// beside the one before, which the sums of the products undo as they go; off by 2^-62 of a chunk's largest).  fp16 has no room for large or
// small numbers: the weighted k, each column of S and each row of P are brought to 2^13 by a power of two for each chunk, of their largest.
// log_decay is summed in 64 bits, differences are split into whole and fractional powers of two, so that no cancellation is left
// behind a strong decay.  A product of a masked 0, or of a piece that is 0 or has the other sign, with an infinity of v is a NaN: a
// chunk whose k or v hold any has its intra part made again from the terms j <= i alone, and what it adds to the state from fp32 products.
//
// What bounds it: a chunk of 64 tokens (128 x 128, bf16) takes 2.5 us of an SM; its 64 KB take 1.5 us of an SM's part of the memory's
// bandwidth and its products 0.7 us of the tensor cores.  The rest is the workers' instructions (pieces of k, S, P, o: half of the issue slots)
// and what they wait for each other: pieces and S of the next chunk cannot start before this one's products are done.  One sequence of 16384
// tokens, 32 heads of 128 x 128: 298 us (83 at 6.53 TB/s for rows read and written once), of which the segments' own sums are 100;
// 13 sequences of 9001 tokens, 24 heads of 64 x 128, fp16: 120 (22).  fp16 pays for its range: scales for k, for the rows of P and for the
// columns of S, and a third piece of k (16384 tokens, 32 heads of 128 x 128: 385 us, 357 with two pieces).
//
// Long sequences are cut into segments of several chunks where there are too few heads and sequences for the GPU: one launch sums up
// what each segment adds to a zero state, a second one runs over the segments of a sequence and leaves each one's starting state, and
// the main one then has all segments at once.
#include <float.h>
#include <stdlib.h>

#include <algorithm>

#define IM2WIN_INLINE_SLOW_WAIT          // (register counts set by warpgroup leave no room for calls)
#include "common.cuh"
#include "ptx_sm100.cuh"
#include "sequence.cuh"

namespace im2win {
namespace {

using namespace ptx;

constexpr int kChunk = 64;               // tokens
constexpr int kThreads = 512;           // that have a part of S; two more warps
constexpr int kAllThreads = kThreads + 128;
// Registers: 640 threads are launched with 96 each; four warpgroups of workers take what the fifth gives back (512 x 104 + 128 x 64).
// What the workers spill goes to the L2 cache, since shared memory leaves none of the first level: with dk 128 some 40 bytes a thread
// even so, in bf16 and fp16.
constexpr int kWorkerRegisters = 104, kHelperRegisters = 64;
constexpr int kQuarters = kThreads / 128; // parts of dk, and of a chunk's tokens, of the threads that have a column of dv
constexpr int kStages = 3;
constexpr int kIssueWarp = 16;          // one thread of it starts loads and products
constexpr int kDecayWarp = 17;          // sends o out, sums up log_decay, two chunks ahead
constexpr int kTile = 128;               // columns of dv of a block: rows of the products
constexpr uint32_t kPanel = 64 * 128;    // 64 rows of 64 16-bit elements, 128-byte swizzle

struct ChunkParams {
  const void* q;
  const void* k;
  const void* v;
  const float* decay;
  void* o;
  const float* state_in;
  float* state_out;
  float* added;                          // [segments][heads][dk][dv]: what each adds, then (segmented) its starting state
  float2* totals;                        // [segments][heads]: decay of a whole segment, in two parts
  uint32_t* status;
  Sequences seqs;
  int64_t q_stride, k_stride, v_stride, o_stride, decay_stride;
  int32_t heads, share, dk, dv, tiles, L;
  int32_t segmented, by_map, o_by_map;   // by_map: rows of q, k and v start on 16-byte boundaries; o_by_map: those of o too
  int32_t drop;                          // testing aid: head 0 does not say that the products of this chunk are done (-1: all do)
  float scale;
};

// q, k, v as [tokens][heads][dk or dv] in boxes of 64 tokens of 64 elements of a head, o in boxes of 64 tokens of 128.
struct alignas(64) ChunkMaps {
  CUtensorMap q, k, v, o;
};

template <typename T> struct Kind;
template <> struct Kind<__nv_bfloat16> {
  static constexpr int kPieces = 3;
  static constexpr int kPieceBits = 0;
  static constexpr bool kScaled = false;
  static constexpr uint32_t kFormats = (1u << 7) | (1u << 10);
  // The larger magnitudes, two at once; a NaN is larger than anything.
  static __device__ __forceinline__ uint32_t largest(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("{\n\t.reg .b32 m;\n\tabs.bf16x2 m, %2;\n\tmax.NaN.bf16x2 %0, %1, m;\n\t}" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ bool odd(uint32_t top) { return ((top & 0x7fff7fffu) + 0x00800080u) & 0x80008000u; }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
  }
  static __device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
  static __device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
  // Two numbers as pieces: the upper half, the upper half of the rest, the rest of that (exact: 24 bits).
  static __device__ __forceinline__ void split(float a, float b, uint32_t (&piece)[3]) {
    const float a1 = a - __uint_as_float(__float_as_uint(a) & 0xffff0000u), b1 = b - __uint_as_float(__float_as_uint(b) & 0xffff0000u);
    piece[0] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    piece[1] = __byte_perm(__float_as_uint(a1), __float_as_uint(b1), 0x7632);
    const float a2 = a1 - __uint_as_float(__float_as_uint(a1) & 0xffff0000u), b2 = b1 - __uint_as_float(__float_as_uint(b1) & 0xffff0000u);
    piece[2] = __byte_perm(__float_as_uint(a2), __float_as_uint(b2), 0x7632);
  }
};
template <> struct Kind<__half> {
  static constexpr int kPieces = 3;
  static constexpr int kPieceBits = 12;                        // a piece is that many bits above what it stands for, beside the one before
  static constexpr bool kScaled = true;
  static constexpr uint32_t kFormats = 0;
  static __device__ __forceinline__ uint32_t largest(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("{\n\t.reg .b32 m;\n\tabs.f16x2 m, %2;\n\tmax.NaN.f16x2 %0, %1, m;\n\t}" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ bool odd(uint32_t top) { return ((top & 0x7fff7fffu) + 0x04000400u) & 0x80008000u; }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
  }
  static __device__ __forceinline__ float low(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w & 0xffffu))); }
  static __device__ __forceinline__ float high(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
  // Two numbers below 2^14 as pieces: rounded, 2^12 times the rest rounded (at most half of the 8 that are a last place there, times
  // 2^12: 2^14 again), and that once more: exact down to 2^-25, off by at most 2^-49 below.
  static __device__ __forceinline__ void split(float a, float b, uint32_t (&piece)[3]) {
    constexpr float kUp = (float)(1 << kPieceBits);
    piece[0] = pack(a, b);
    const float a1 = (a - low(piece[0])) * kUp, b1 = (b - high(piece[0])) * kUp;
    piece[1] = pack(a1, b1);
    piece[2] = pack((a1 - low(piece[1])) * kUp, (b1 - high(piece[1])) * kUp);
  }
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t ld_shared_u16(uint32_t addr) {
  unsigned short v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared4(uint32_t addr, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// MMA with A in tensor memory (its elements two a column along K) and B by descriptor.
__device__ __forceinline__ void umma_f16_ta(uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The same from descriptors, added to D times 2^-DOWN.
template <int DOWN>
__device__ __forceinline__ void umma_f16_onto_scaled(uint32_t tmem_d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc) {
  static_assert(DOWN >= 0 && DOWN <= 15, "");
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %2};\n\t"
      "mov.b64 db, {%3, %4};\n\t"
      "setp.eq.b32 p, 0, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p, %6;\n\t}"
      ::"r"(tmem_d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "n"(DOWN)
      : "memory");
}
// Descriptor halves of an operand whose rows of 64 elements (128 bytes, 128-byte swizzle) run along M or N: panels of 64 of them
// kPanel bytes apart (leading offset), groups of eight rows, along K, 1024 bytes apart (stride offset).
__device__ __forceinline__ uint32_t desc_lo_mn(uint32_t saddr) { return ((saddr & 0x3ffffu) >> 4) | ((kPanel >> 4) << 16); }
constexpr uint32_t kDescHi = kSmemDescHiSw128;
constexpr uint32_t kAlongM = 1u << 15, kAlongN = 1u << 16;     // of the instruction descriptor: A, B lie that way

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// The decays of one chunk, all relative to its start.
struct alignas(16) Decays {
  float whole[kChunk], part[kChunk];     // G_i in powers of two: its floor and the rest
  float from_start[kChunk];              // exp(G_i) scale E, E of the state before the chunk
  float to_end[kChunk];                  // exp(G_n - G_i) / E, E of the state behind it
  float total, behind;                   // exp(G_n), rounded; E behind the chunk
};

// A power of two that brings numbers of at most `bits` (of a float) to below 2^14.
__device__ __forceinline__ float scale_for(uint32_t bits) {
  const int e = (int)(bits >> 23);
  if (e == 0) return 1.0f;
  return __uint_as_float((uint32_t)min(max(127 + 13 - (e - 127), 1), 253) << 23);
}
__device__ __forceinline__ float unscale_for(float scale) { return __uint_as_float((254u << 23) - __float_as_uint(scale)); }     // its reciprocal
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
__device__ __forceinline__ void raise_max(uint32_t* at, uint32_t bits) {
  const uint32_t m = __reduce_max_sync(0xffffffffu, bits);
  if ((threadIdx.x & 31) == 0) atomicMax(at, m);
}

// S <- exp(G_n) S + added, for the decay of a segment, in two parts.
__device__ __forceinline__ float carry(float s, float2 total, float added) { return fmaf(s, total.x, fmaf(s, total.y, added)); }

// exp2(power) as the float below it and the rest, so that an infinity times either has its sign (and no rest where nothing is left).
__device__ __forceinline__ float2 two_parts(double power) {
  const double all = exp2(power);
  const float hi = __double2float_rz(all);
  const float lo = (float)(all - (double)hi);
  return make_float2(hi, hi > 0.0f && lo < FLT_MIN ? FLT_MIN : lo);
}

// One warp: lane l has tokens 2l and 2l+1.  Returns G_n (powers of two).  Sums are of whole numbers of 2^-44: exact, and without
// the 64-bit floating-point units, which took 1300 cycles for sums and powers.
// The states in registers are S / E: a chunk multiplies them by exp(G_n) rounded to a float, and what that is off, the same at every
// chunk of a constant decay, goes into E, a double, instead: S is off by less than a rounding of its sums after any number of chunks.
__device__ __forceinline__ double chunk_decays(float g0, float g1, float scale, double& E, Decays& d) {
  constexpr float kNaN = __builtin_nanf("");
  const int lane = threadIdx.x & 31;
  auto powers = [](float g) -> int64_t {                       // (beyond 2^+-1000 nothing changes in fp32)
    return __double2ll_rn((double)fminf(fmaxf(g, -700.0f), 700.0f) * (1.4426950408889634074 * 17592186044416.0));
  };
  const int64_t a = powers(g0), b = powers(g1);
  const uint32_t nan0 = __ballot_sync(0xffffffffu, g0 != g0), nan1 = __ballot_sync(0xffffffffu, g1 != g1);
  int64_t sum = a + b;
#pragma unroll
  for (int s = 1; s < 32; s *= 2) {
    const int64_t other = __shfl_up_sync(0xffffffffu, sum, s);
    if (lane >= s) sum += other;
  }
  const int64_t all = __shfl_sync(0xffffffffu, sum, 31);
  auto fraction = [](int64_t x) { return (float)((uint32_t)(x >> 20) & 0xffffffu) * 5.9604644775390625e-8f; };
  auto power_of_two = [](int64_t x) { return __uint_as_float((uint32_t)(min(max((int)(x >> 44), -127), 128) + 127) << 23); };
  const int64_t G[2] = {sum - b, sum};
  const double end = nan0 | nan1 ? (double)kNaN : (double)all * (1.0 / 17592186044416.0);
  const double exact = exp2(end);
  const float total = (float)exact;
  const float before = (float)E * scale;
  if (total > 1e-30f && total < 1e30f) E += E * (double)__fdividef((float)(exact - (double)total), total);
  const float per = 1.0f / (float)E;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t rest = all - G[i];
    float whole = (float)(int)(G[i] >> 44), from = exp2f(fraction(G[i])) * power_of_two(G[i]) * before;
    float to_end = exp2f(fraction(rest)) * power_of_two(rest) * per;
    if (nan0 | nan1) {                                         // behind a NaN every sum is one
      const uint32_t behind0 = (2u << lane) - 1u, behind1 = i ? (2u << lane) - 1u : (1u << lane) - 1u;
      if ((nan0 & behind0) | (nan1 & behind1)) whole = from = kNaN;
      to_end = kNaN;
    }
    d.whole[2 * lane + i] = whole;
    d.part[2 * lane + i] = fraction(G[i]);
    d.from_start[2 * lane + i] = from;
    d.to_end[2 * lane + i] = to_end;
  }
  if (lane == 0) {
    d.total = total;
    d.behind = (float)E;
  }
  return end;
}

// Shared memory: three stages of k, v and q, the pieces of the weighted k (two sets where o is not made), P, o on its way out.
template <typename T, int DK, bool OUT>
struct Layout {
  static constexpr uint32_t kQK = DK / 64 * kPanel;            // q or k of a chunk
  static constexpr uint32_t kV = 2 * kPanel;
  static constexpr uint32_t kStage = (OUT ? 2 : 1) * kQK + kV;
  static constexpr uint32_t kPieces = Kind<T>::kPieces * kQK;
  static constexpr uint32_t kPiecesAt = kStages * kStage;
  static constexpr uint32_t kPAt = kPiecesAt + (OUT ? 1 : 2) * kPieces;
  static constexpr uint32_t kOAt = kPAt + kPanel;
  static constexpr uint32_t kBytes = (OUT ? kOAt + kChunk * kTile * 2 : kPAt) + 1024;
  // columns of tensor memory: added (two where o is not made), two of inter, two of intra, q . k, the copy of S
  static constexpr uint32_t kAdded = 0, kInter = DK, kIntra = DK + 128, kDots = DK + 256, kS = DK + 320;
  static constexpr uint32_t kColumns = OUT ? 512 : 2 * DK;
};

// N columns of tensor memory, 32 bits each, of this warp's lanes.
template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[N]) {
  static_assert(N == 16 || N == 32, "");
  if constexpr (N == 32) {
    tmem_ld32_issue(taddr, r);
  } else {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
  }
}
// 16 lanes and 16 columns: r[4n + 2h + i] is row lane / 4 + 8h, column 8n + 2 (lane % 4) + i.
__device__ __forceinline__ void tmem_ld_16x16(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
// The wait for a load into r[] (naming the registers keeps every use of them behind it).
template <int N>
__device__ __forceinline__ void tmem_ld_done(uint32_t (&r)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y),
               "r"(z)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

// A wait that has mostly come about (a look costs a fifth of the time of a try that may suspend).
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* status) {
  if (mbar_test_wait(bar, parity)) return true;
  return mbar_wait(bar, parity, abort_flag, status);
}

// Barriers of the workers and the two helping warps.
__device__ __forceinline__ void sync_all() { asm volatile("bar.sync 1, %0;" ::"n"(kThreads + 64) : "memory"); }
__device__ __forceinline__ bool sync_or(bool any) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "bar.red.or.pred p, 1, %2, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)any), "n"(kThreads + 64)
      : "memory");
  return r != 0;
}

// The order of work for chunk c, between its barrier and the next chunk's:
//   issue warp    the loads of chunk c+2; q . k of chunk c+1; inter, added and intra of chunk c
//   decay warp    the store of o of chunk c-2, the decays of chunk c+2
//   all others    P of chunk c+1; o of chunk c-1 to shared memory; S with what chunk c added
// and before the barrier: weighted k in pieces, the copy of S, P of chunk c to where the products read them.
template <typename T, int DK, bool OUT>
__global__ void __launch_bounds__(kAllThreads, 1) chunk_kernel(const __grid_constant__ ChunkMaps maps, const ChunkParams p) {
  using K = Kind<T>;
  using L = Layout<T, DK, OUT>;
  constexpr int kMine = DK / kQuarters;                        // columns of S of a thread
  constexpr int kTokens = kChunk / kQuarters;                  // rows of o of a thread
  extern __shared__ uint8_t dynamic_smem[];
  __shared__ Decays decays[4];
  __shared__ __align__(8) uint64_t bars[kStages + 5];          // stages loaded; added done (two), intra, q . k done, o stored; all products done
  __shared__ uint32_t tmem_base_at, abort_flag, odd_values[4], largest[4];       // largest: of the weighted k
  __shared__ uint32_t column_largest[K::kScaled && OUT ? 4 : 1][kTile];          // fp16: of each column of S
  // and the exponents of the largest of each row of P, a byte for each quarter of its columns, and what undoes the row's scale
  __shared__ __align__(16) uint32_t row_exponents[K::kScaled ? 2 : 1][kChunk];
  __shared__ __align__(16) float row_unscale[K::kScaled ? 2 : 1][kChunk];
  const uint32_t smem = (smem_u32(dynamic_smem) + 1023u) & ~1023u;
  const int warp = warp_index(), lane = threadIdx.x & 31, tid = threadIdx.x;
  const uint32_t tile = blockIdx.x % (uint32_t)p.tiles, rest = blockIdx.x / (uint32_t)p.tiles;
  const int head = (int)(rest % (uint32_t)p.heads);
  const uint32_t id = rest / (uint32_t)p.heads;
  const Piece piece = find_piece(p.seqs, id, p.L);
  const int slot = slot_of(p.seqs, piece.sequence);
  const bool leads = piece.first == piece.rows.begin;
  if (slot < 0 || (!leads && piece.first >= piece.rows.end)) return;
  const int first = (int)piece.first, end = (int)min(piece.first + p.L, (int64_t)piece.rows.end);
  const bool last = end == piece.rows.end;
  if (!OUT && last) return;                                    // (nothing starts behind it)

  const int chunks = (end - first + kChunk - 1) / kChunk, whole = p.by_map ? (end - first) / kChunk : 0;

  const uint32_t loaded = smem_u32(bars), done = smem_u32(bars + kStages), intra_done = smem_u32(bars + kStages + 1),
                 dots_done = smem_u32(bars + kStages + 2), stored = smem_u32(bars + kStages + 3), drained = smem_u32(bars + kStages + 4);
  if (warp == 0) tmem_alloc(smem_u32(&tmem_base_at), L::kColumns);
  if (tid == 0) {
    for (int i = 0; i < kStages + 5; ++i) mbar_init(smem_u32(bars + i), 1);
    abort_flag = 0;
    for (int i = 0; i < 4; ++i) largest[i] = odd_values[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async_smem();
  }
  if (K::kScaled && OUT && tid < 4 * kTile) column_largest[tid / kTile][tid % kTile] = 0;
  if (K::kScaled && tid < 2 * kChunk) row_exponents[tid / kChunk][tid % kChunk] = 0;     // (as the quarters above the diagonal stay)
  if (OUT && tid < kPanel / 16) st_shared16(smem + L::kPAt + tid * 16, 0, 0, 0, 0);      // (above the diagonal it stays 0)
  auto wait = [&](uint32_t bar, uint32_t phase) { return wait_for(bar, phase & 1, &abort_flag, p.status); };

  // A whole chunk: one thread, by TMA (elements beyond a head's read as 0).
  auto load_whole = [&](int c) {
    const uint32_t base = smem + (c % kStages) * L::kStage, bar = loaded + (c % kStages) * 8;
    const int t0 = first + c * kChunk;
    mbar_arrive_expect_tx(bar, L::kStage);
#pragma unroll
    for (int i = 0; i < DK / 64; ++i) {
      tma_load_3d(base + i * kPanel, &maps.k, i * 64, head / p.share, t0, bar);
      if (OUT) tma_load_3d(base + L::kQK + L::kV + i * kPanel, &maps.q, i * 64, head / p.share, t0, bar);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) tma_load_3d(base + L::kQK + i * kPanel, &maps.v, (int)tile * kTile + i * 64, head, t0, bar);
  };
  // The last chunk of a sequence: the workers; the rows of the next sequence, and those behind the last, as 0.  Rows that do not start
  // on 16-byte boundaries: every chunk, an element at a time.
  auto load_rows = [&](uint32_t to, const T* from, int64_t stride, int columns, int t0, int units) {
    const int shift = units == 16 ? 4 : 3;
#pragma unroll 1
    for (int u = tid; u < kChunk * units; u += kThreads) {
      const int r = u >> shift, cc = u & (units - 1);
      const uint32_t at = to + (cc / 8) * kPanel + r * 128 + (((cc % 8) ^ (r & 7)) << 4);
      const bool row_there = t0 + r < end;
      if (p.by_map) {
        const bool there = row_there && cc * 8 < columns;
        copy16(at, from + (there ? (t0 + r) * stride + cc * 8 : 0), there);
      } else {
        const unsigned short* row = reinterpret_cast<const unsigned short*>(from) + (row_there ? (t0 + r) * stride : 0);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t lo = row_there && cc * 8 + 2 * i < columns ? row[cc * 8 + 2 * i] : 0;
          const uint32_t hi = row_there && cc * 8 + 2 * i + 1 < columns ? row[cc * 8 + 2 * i + 1] : 0;
          w[i] = lo | hi << 16;
        }
        st_shared16(at, w[0], w[1], w[2], w[3]);
      }
    }
  };
  auto load_part = [&](int c) {
    const uint32_t base = smem + (c % kStages) * L::kStage;
    const int t0 = first + c * kChunk;
    const int64_t qk_at = (int64_t)(head / p.share) * p.dk;
    load_rows(base, static_cast<const T*>(p.k) + qk_at, p.k_stride, p.dk, t0, DK / 8);
    if (OUT) load_rows(base + L::kQK + L::kV, static_cast<const T*>(p.q) + qk_at, p.q_stride, p.dk, t0, DK / 8);
    load_rows(base + L::kQK, static_cast<const T*>(p.v) + (int64_t)head * p.dv + tile * kTile, p.v_stride, p.dv - (int)tile * kTile, t0, 16);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto load_decay = [&](int c, float& g0, float& g1) {
    const int t = first + c * kChunk + 2 * lane;
    g0 = t < end ? p.decay[(int64_t)t * p.decay_stride + head] : 0.0f;
    g1 = t + 1 < end ? p.decay[(int64_t)(t + 1) * p.decay_stride + head] : 0.0f;
  };

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_at, lanes = (uint32_t)(warp & 3) << 21;      // this warp's 32 lanes
  // q . k of chunk c: one thread
  auto issue_dots = [&](int c) {
    const uint32_t kt = smem + (c % kStages) * L::kStage, qt = kt + L::kQK + L::kV;
#pragma unroll
    for (int ks = 0; ks < DK / 16; ++ks)
      umma_f16_lohi(tmem + L::kDots, smem_desc_lo(qt + (ks / 4) * kPanel + (ks % 4) * 32), smem_desc_lo(kt + (ks / 4) * kPanel + (ks % 4) * 32),
                    K::kFormats | instr_desc_f16(64, 64), ks > 0);
    umma_commit(dots_done);
  };
  bool failed = false;
  if (warp >= kThreads / 32) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kHelperRegisters));
    bool odd_1 = false, odd_2 = false;
    if (warp == kIssueWarp) {
      // (Waits by the whole warp, issue by one elected lane: operands of the tensor cores and of TMA are uniform registers, which they stay
      // in where the compiler sees no other branch.)
      if (elect_one()) {
        if (0 < whole) load_whole(0);
        if (1 < whole) load_whole(1);
      }
      __syncwarp();
      if (OUT && 0 < whole) {
        failed = !wait(loaded, 0);
        if (elect_one()) issue_dots(0);
        __syncwarp();
      }
      sync_all();
      int c = 0;
      for (; c < chunks; ++c) {
        const uint32_t kt = smem + (c % kStages) * L::kStage, vt = kt + L::kQK, qt = vt + L::kV;
        const uint32_t pieces = smem + L::kPiecesAt + (OUT ? 0 : (c & 1) * L::kPieces);
        if (c >= whole) {
          sync_all();
          tc_fence_after();
          if (OUT && elect_one()) issue_dots(c);
          __syncwarp();
        }
        if (K::kScaled) sync_all();
        failed = sync_or(failed);
        if (failed) break;
        tc_fence_after();
        const bool odd_0 = *(volatile uint32_t*)&odd_values[c & 3] != 0;
        if (OUT && c + 1 < whole) {
          failed = !wait(loaded + ((c + 1) % kStages) * 8, (c + 1) / kStages);
          if (elect_one()) issue_dots(c + 1);
          __syncwarp();
        }
        if (elect_one()) {
          if (OUT) {
#pragma unroll
            for (int ks = 0; ks < DK / 16; ++ks)
              umma_f16_ta(tmem + L::kInter + (c & 1) * 64, tmem + L::kS + ks * 8, smem_desc_lo(qt + (ks / 4) * kPanel + (ks % 4) * 32), kDescHi,
                          K::kFormats | instr_desc_f16(128, 64), ks > 0);
          }
#pragma unroll
          for (int n = K::kPieces - 1; n >= 0; --n)            // the smallest pieces first
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
              const uint32_t to = tmem + L::kAdded + (OUT ? 0 : (c & 1) * DK), a = desc_lo_mn(vt + ks * 2048),
                             b = desc_lo_mn(pieces + n * L::kQK + ks * 2048);
              constexpr uint32_t kDesc = K::kFormats | kAlongM | kAlongN | instr_desc_f16(128, DK);
              if (K::kPieceBits > 0 && ks == 0 && n < K::kPieces - 1)
                umma_f16_onto_scaled<K::kPieceBits>(to, a, kDescHi, b, kDescHi, kDesc);
              else
                umma_f16_ab(to, a, kDescHi, b, kDescHi, kDesc, n < K::kPieces - 1 || ks > 0);
            }
          if (c != p.drop || head != 0) umma_commit(done + (OUT ? 0 : (c & 1) * 8));
          if (OUT) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              umma_f16_ab(tmem + L::kIntra + (c & 1) * 64, desc_lo_mn(vt + ks * 2048), kDescHi, smem_desc_lo(smem + L::kPAt + ks * 32), kDescHi,
                          K::kFormats | kAlongM | instr_desc_f16(128, 64), ks > 0);
            umma_commit(intra_done);
            if (c + 2 < whole) load_whole(c + 2);              // (the products of the chunk before are done: seen before the barrier)
          }
        }
        __syncwarp();
        if (!OUT && c > 0) failed = !wait(done + ((c - 1) & 1) * 8, (c - 1) >> 1) || failed;
        if (OUT ? odd_0 : odd_1) sync_all();                   // (the workers have read P, k and v)
        if (!OUT && c + 2 < whole && elect_one()) load_whole(c + 2);
        __syncwarp();
        odd_1 = odd_0;
      }
      // Its loads and products under way end before the block does and gives its tensor memory back.
      if (failed)
        for (int i = c; i < c + 2 && i < whole; ++i) wait(loaded + (i % kStages) * 8, i / kStages);
      if (elect_one()) umma_commit(drained);
      __syncwarp();
      wait(drained, 0);
    } else if (warp == kDecayWarp) {
      double all_decay = 0.0, E = 1.0;
      float g0 = 0.0f, g1 = 0.0f;
      if (chunks > 0) {
        load_decay(0, g0, g1);
        all_decay = chunk_decays(g0, g1, p.scale, E, decays[0]);
        load_decay(1, g0, g1);
      }
      sync_all();
      if (chunks > 1) all_decay += chunk_decays(g0, g1, p.scale, E, decays[1]);
      for (int c = 0; c < chunks; ++c) {
        if (c + 2 < chunks) load_decay(c + 2, g0, g1);
        if (c >= whole) sync_all();
        if (K::kScaled) sync_all();
        if (sync_or(false)) {
          all_decay = (double)__builtin_nanf("");
          break;
        }
        const bool odd_0 = *(volatile uint32_t*)&odd_values[c & 3] != 0;
        if (OUT && elect_one()) {
          if (p.o_by_map && c > 1 && !odd_2) {
            tma_store_3d(&maps.o, smem + L::kOAt, (int)tile * kTile, head, first + (c - 2) * kChunk);
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          }
          mbar_arrive(stored);
        }
        __syncwarp();
        // (in the places of the chunk two before, a barrier behind its last use and one before its first)
        if (c + 2 < chunks) all_decay += chunk_decays(g0, g1, p.scale, E, decays[(c + 2) & 3]);
        __syncwarp();
        if (lane == 0) {
          odd_values[(c + 2) & 3] = 0;
          if (K::kScaled) largest[(c + 2) & 3] = 0;
        }
        if (K::kScaled && OUT) {
#pragma unroll
          for (int i = 0; i < kTile; i += 32) column_largest[(c + 2) & 3][i + lane] = 0;
        }
        if (OUT ? odd_0 : odd_1) sync_all();
        odd_2 = odd_1;
        odd_1 = odd_0;
      }
      if (OUT) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
      __syncwarp();
      asm volatile("bar.arrive 2, %0;" ::"n"(kThreads + 32) : "memory");
      if (!OUT && tile == 0) {
        const float2 total = two_parts(all_decay);
        if (lane == 0) p.totals[(int64_t)id * p.heads + head] = total;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kWorkerRegisters));
    const int quarter = warp >> 2, row = (warp & 3) * 32 + lane;           // row: of the transposed products, a column of dv
    const int col = (int)tile * kTile + row;
    const bool live = col < p.dv;
    const int64_t state_size = (int64_t)p.dk * p.dv;
    if (whole == 0 && chunks > 0) load_part(0);
    // the starting state
    float S[kMine];
    {
      const float* from = nullptr;
      if (OUT && live) {
        if (p.segmented && !(leads && last))                   // (of a sequence that is cut)
          from = p.added + ((int64_t)id * p.heads + head) * state_size;
        else if (p.state_in && resumes(p.seqs, piece.sequence))
          from = p.state_in + ((int64_t)slot * p.heads + head) * state_size;
      }
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        const int d = quarter * kMine + j;
        S[j] = from && d < p.dk ? from[(int64_t)d * p.dv + col] : 0.0f;
      }
    }
    // element e of row t of panels at `at`
    auto element = [&](uint32_t at, int t, int e) {
      return K::low(ld_shared_u16(at + (e >> 6) * kPanel + t * 128 + ((((uint32_t)(e & 63) >> 3) ^ (t & 7)) << 4) + (e & 7) * 2));
    };
    // P of chunk c, whose q . k are done (its 16 x 16 blocks that reach below the diagonal, one to a warp: rows 16 rb, columns 16 quarter)
    const int rb = warp & 3;
    const bool makes_p = OUT && quarter <= rb;
    float P[2][4];
    auto make_p = [&](int c) {
      const Decays& d = decays[c & 3];
      uint32_t dots[8];
      tmem_ld_16x16(tmem + lanes + L::kDots + quarter * 16, dots);
      const int ti = rb * 16 + (lane >> 2), tj = quarter * 16 + 2 * (lane & 3);
      const float wi[2] = {d.whole[ti], d.whole[ti + 8]}, pi[2] = {d.part[ti], d.part[ti + 8]};
      tmem_ld_done(dots);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float2 wj = *reinterpret_cast<const float2*>(&d.whole[tj + 8 * n]), pj = *reinterpret_cast<const float2*>(&d.part[tj + 8 * n]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float power = (wi[i >> 1] - (i & 1 ? wj.y : wj.x)) + (pi[i >> 1] - (i & 1 ? pj.y : pj.x));
          const float w = __uint_as_float(dots[4 * n + i]) * (exp2_fast(power) * p.scale);
          P[n][i] = tj + 8 * n + (i & 1) <= ti + 8 * (i >> 1) ? w : 0.0f;
        }
      }
      if (K::kScaled) {
        // (a row for itself: its q, and the decays behind it, may be far from another's)
        float top[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
          top[h] = fmaxf(fmaxf(fabsf(P[0][2 * h]), fabsf(P[0][2 * h + 1])), fmaxf(fabsf(P[1][2 * h]), fabsf(P[1][2 * h + 1])));
        if (fmaxf(top[0], top[1]) > FLT_MAX) {                 // (of the finite ones)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            top[h] = __uint_as_float(max(max(finite_bits(P[0][2 * h]), finite_bits(P[0][2 * h + 1])),
                                         max(finite_bits(P[1][2 * h]), finite_bits(P[1][2 * h + 1]))));
        }
        uint32_t both = __float_as_uint(top[0]) >> 23 | (__float_as_uint(top[1]) >> 23) << 16;
        both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 1));
        both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 2));
        if ((lane & 3) == 0) {
          uint8_t* to = reinterpret_cast<uint8_t*>(&row_exponents[c & 1][ti]) + quarter;
          to[0] = (uint8_t)both;
          to[32] = (uint8_t)(both >> 16);
        }
      }
    };
    // o of chunk c, whose products are done, two rows a register
    auto make_o = [&](int c, float scale_s, bool odd, uint32_t (&y)[kTokens / 2]) {
      const Decays& d = decays[c & 3];
      const float is = unscale_for(scale_s);
      uint32_t inter[kTokens], intra[kTokens];
      tmem_ld(tmem + lanes + L::kInter + (c & 1) * 64 + quarter * kTokens, inter);
      tmem_ld(tmem + lanes + L::kIntra + (c & 1) * 64 + quarter * kTokens, intra);
      tmem_ld_done(inter);
      tmem_ld_done(intra);
      if (odd) {                                                 // from the terms j <= i alone
        const uint32_t vt = smem + (c % kStages) * L::kStage + L::kQK;
#pragma unroll 1
        for (int i = 0; i < kTokens; ++i) {
          const int ti = quarter * kTokens + i;
          float sum = 0.0f;
#pragma unroll 1
          for (int j = 0; j <= ti; ++j) sum = fmaf(element(smem + L::kPAt, ti, j), element(vt, j, row), sum);
#pragma unroll
          for (int u = 0; u < kTokens; ++u)
            if (u == i) intra[u] = __float_as_uint(sum);
        }
      }
#pragma unroll
      for (int i = 0; i < kTokens; i += 4) {
        const float4 from = *reinterpret_cast<const float4*>(&d.from_start[quarter * kTokens + i]);
        float4 unscale = make_float4(1.0f, 1.0f, 1.0f, 1.0f);
        if constexpr (K::kScaled) unscale = *reinterpret_cast<const float4*>(&row_unscale[c & 1][quarter * kTokens + i]);
        const float f[4] = {from.x, from.y, from.z, from.w}, ip[4] = {unscale.x, unscale.y, unscale.z, unscale.w};
#pragma unroll
        for (int u = 0; u < 4; u += 2)
          y[(i + u) / 2] = K::pack(fmaf(f[u] * is, __uint_as_float(inter[i + u]), __uint_as_float(intra[i + u]) * ip[u]),
                                   fmaf(f[u + 1] * is, __uint_as_float(inter[i + u + 1]), __uint_as_float(intra[i + u + 1]) * ip[u + 1]));
      }
    };
    auto store_o = [&](int c, const uint32_t (&y)[kTokens / 2]) {
      const int t0 = first + c * kChunk + quarter * kTokens;
      unsigned short* at = static_cast<unsigned short*>(p.o) + (int64_t)head * p.dv + col + (int64_t)t0 * p.o_stride;
      const int n = live ? end - t0 : 0;
#pragma unroll
      for (int i = 0; i < kTokens; ++i)
        if (i < n) at[(int64_t)i * p.o_stride] = (unsigned short)(y[i / 2] >> (16 * (i & 1)));
    };
    auto stage_o = [&](const uint32_t (&y)[kTokens / 2]) {
      const uint32_t to = smem + L::kOAt + quarter * kTokens * (kTile * 2) + row * 2;
#pragma unroll
      for (int i = 0; i < kTokens; ++i)
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + i * kTile * 2), "h"((unsigned short)(y[i / 2] >> (16 * (i & 1)))) : "memory");
    };
    // what chunk c added, once its products are done
    auto add = [&](int c, float scale_k, bool odd) {
      const Decays& d = decays[c & 3];
      uint32_t added[kMine];
      tmem_ld(tmem + lanes + L::kAdded + (OUT ? 0 : (c & 1) * DK) + quarter * kMine, added);
      const float total = d.total;
      tmem_ld_done(added);
      if (odd) {                                                 // from the products in fp32
        const uint32_t base = smem + (c % kStages) * L::kStage;
        const int n = min(kChunk, end - (first + c * kChunk));
#pragma unroll 1
        for (int i = 0; i < kMine; ++i) {
          float sum = 0.0f;
#pragma unroll 1
          for (int t = 0; t < n; ++t) sum = fmaf(element(base, t, quarter * kMine + i) * d.to_end[t], element(base + L::kQK, t, row), sum);
#pragma unroll
          for (int u = 0; u < kMine; ++u)
            if (u == i) added[u] = __float_as_uint(sum * scale_k);
        }
      }
      const float ik = unscale_for(scale_k);
#pragma unroll
      for (int j = 0; j < kMine; ++j) S[j] = fmaf(S[j], total, __uint_as_float(added[j]) * ik);
    };

    // infinities and NaNs among v of chunk c
    auto look_at_v = [&](int c) {
      const uint32_t vt = smem + (c % kStages) * L::kStage + L::kQK;
      uint32_t top = 0;
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint4 vv = ld_shared16(vt + (tid + m * kThreads) * 16);
        top = K::largest(K::largest(K::largest(K::largest(top, vv.x), vv.y), vv.z), vv.w);
      }
      if (K::odd(top)) odd_values[c & 3] = 1;
    };
    float prev_k = 1.0f, prev_s = 1.0f;                        // the chunk before's scales,
    bool odd_1 = false;                                        // whether its k and v hold infinities or NaNs
    sync_all();                                                // (the first decays)
    if (OUT && 0 < whole) {
      failed = !wait(dots_done, 0);
      tc_fence_after();
      if (makes_p) make_p(0);
      failed = !wait(loaded, 0) || failed;
      look_at_v(0);
    }
    for (int c = 0; c < chunks; ++c) {
      const uint32_t kt = smem + (c % kStages) * L::kStage, vt = kt + L::kQK;
      const uint32_t pieces = smem + L::kPiecesAt + (OUT ? 0 : (c & 1) * L::kPieces);
      if (c >= whole) {                                        // the last one, in part
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        fence_proxy_async_smem();
        sync_all();
        if (OUT) {
          failed = !wait(dots_done, c) || failed;
          tc_fence_after();
          if (makes_p) make_p(c);
        }
      } else if (!OUT) {                                       // (otherwise waited for with the chunk before)
        failed = !wait(loaded + (c % kStages) * 8, c / kStages) || failed;
      }

      constexpr int kUnits = DK / 8, kVectors = kChunk * kUnits / kThreads;
      uint4 kk[kVectors];
      if (c >= whole || !OUT) look_at_v(c);
#pragma unroll
      for (int m = 0; m < kVectors; ++m) {
        const int u = tid + m * kThreads, r = u / kUnits, cc = u % kUnits;
        kk[m] = ld_shared16(kt + (cc / 8) * kPanel + r * 128 + (((cc % 8) ^ (r & 7)) << 4));
      }
      uint32_t tops[kVectors], top = 0;
#pragma unroll
      for (int m = 0; m < kVectors; ++m) {
        tops[m] = K::largest(K::largest(K::largest(K::largest(0, kk[m].x), kk[m].y), kk[m].z), kk[m].w);
        top = K::largest(top, tops[m]);
      }
      const bool odd_k = K::odd(top);
      if (odd_k) odd_values[c & 3] = 1;
      float scale_k = 1.0f, scale_s = 1.0f;
      if (K::kScaled) {
        // The largest of the weighted k: the weights of tokens far from the chunk's end are far from 1, below it or, where decays grow, above.
        uint32_t km = 0;
#pragma unroll
        for (int m = 0; m < kVectors; ++m) {
          uint32_t t = tops[m];
          if (odd_k) {                                         // (of the finite ones)
            t = 0;
#pragma unroll
            for (uint32_t w : {kk[m].x, kk[m].y, kk[m].z, kk[m].w}) {
              if ((w & 0x7c00u) != 0x7c00u) t = __vmaxu2(t, w & 0x7fffu);
              if ((w & 0x7c000000u) != 0x7c000000u) t = __vmaxu2(t, w & 0x7fff0000u);
            }
          }
          km = max(km, finite_bits(fmaxf(K::low(t), K::high(t)) * decays[c & 3].to_end[(tid + m * kThreads) / kUnits]));
        }
        raise_max(&largest[c & 3], km);
        if (OUT) {
          float sm = 0.0f;
#pragma unroll
          for (int j = 0; j < kMine; ++j) sm = fmaxf(sm, fabsf(S[j]));
          if (sm > FLT_MAX) {                                  // (an infinity: the largest of the others; NaNs do not count)
            sm = 0.0f;
#pragma unroll
            for (int j = 0; j < kMine; ++j) sm = fmaxf(sm, fabsf(S[j]) <= FLT_MAX ? fabsf(S[j]) : 0.0f);
          }
          atomicMax(&column_largest[c & 3][row], __float_as_uint(sm));
        }
        sync_all();
        scale_k = scale_for(largest[c & 3]);
        if (OUT) scale_s = scale_for(column_largest[c & 3][row]);
      }
      if (OUT) {
        uint32_t r[kMine / 2];
#pragma unroll
        for (int i = 0; i < kMine / 2; ++i) r[i] = K::pack(S[2 * i] * scale_s, S[2 * i + 1] * scale_s);
        tmem_st(tmem + lanes + L::kS + quarter * (kMine / 2), r);
      }
      {
        const Decays& d = decays[c & 3];
#pragma unroll
        for (int m = 0; m < kVectors; ++m) {
          const int u = tid + m * kThreads, r = u / kUnits, cc = u % kUnits;
          const float w = d.to_end[r] * scale_k;
          const uint32_t words[4] = {kk[m].x, kk[m].y, kk[m].z, kk[m].w};
          uint32_t out[K::kPieces][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t piece_of[K::kPieces];
            K::split(K::low(words[i]) * w, K::high(words[i]) * w, piece_of);
#pragma unroll
            for (int n = 0; n < K::kPieces; ++n) out[n][i] = piece_of[n];
          }
          const uint32_t at = (cc / 8) * kPanel + r * 128 + (((cc % 8) ^ (r & 7)) << 4);
#pragma unroll
          for (int n = 0; n < K::kPieces; ++n) st_shared16(pieces + n * L::kQK + at, out[n][0], out[n][1], out[n][2], out[n][3]);
        }
      }
      if (OUT) {
        if (c > 0) failed = !wait(intra_done, c - 1) || failed;      // (it read P)
        if (makes_p) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int ti = rb * 16 + (lane >> 2) + 8 * i;
            float scale_p = 1.0f;
            if constexpr (K::kScaled) {
              const uint32_t e = row_exponents[c & 1][ti];
              scale_p = scale_for(max(max(e & 255u, e >> 8 & 255u), max(e >> 16 & 255u, e >> 24)) << 23);
              if (quarter == 0 && (lane & 3) == 0) row_unscale[c & 1][ti] = unscale_for(scale_p);
            }
#pragma unroll
            for (int n = 0; n < 2; ++n)
              st_shared4(smem + L::kPAt + ti * 128 + (((quarter * 2 + n) ^ (ti & 7)) << 4) + (lane & 3) * 4,
                         K::pack(P[n][2 * i] * scale_p, P[n][2 * i + 1] * scale_p));
          }
        }
        tmem_st_wait();
      }
      fence_proxy_async_smem();
      tc_fence_before();
      failed = sync_or(failed);
      if (failed) break;
      tc_fence_after();
      const bool odd_0 = *(volatile uint32_t*)&odd_values[c & 3] != 0;     // (set before the barrier: every thread sees the same)
      if (c + 1 >= whole && c + 1 < chunks) load_part(c + 1);
      if (OUT) {
        if (c > 0 && !odd_1) {                                 // (an odd chunk's has been stored)
          uint32_t y[kTokens / 2];
          make_o(c - 1, prev_s, false, y);
          if (p.o_by_map && c + 1 < chunks) {
            failed = !wait(stored, c) || failed;
            stage_o(y);
          } else {
            store_o(c - 1, y);
          }
        }
        if (c + 1 < whole) {
          failed = !wait(dots_done, c + 1) || failed;
          tc_fence_after();
          if (makes_p) make_p(c + 1);
          failed = !wait(loaded + ((c + 1) % kStages) * 8, (c + 1) / kStages) || failed;
          look_at_v(c + 1);
        }
        failed = !wait(done, c) || failed;
        tc_fence_after();
        add(c, scale_k, odd_0);
        if (odd_0) {
          failed = !wait(intra_done, c) || failed;
          tc_fence_after();
          uint32_t y[kTokens / 2];
          make_o(c, scale_s, true, y);
          store_o(c, y);
          sync_all();                                          // (P and v have been read)
        }
        prev_s = scale_s;
      } else {
        if (c > 0) {
          failed = !wait(done + ((c - 1) & 1) * 8, (c - 1) >> 1) || failed;
          tc_fence_after();
          add(c - 1, prev_k, odd_1);
        }
        if (odd_1) sync_all();                                 // (k and v of the chunk before have been read)
        prev_k = scale_k;
      }
      odd_1 = odd_0;
    }
    if (!failed && chunks > 0) {
      const int z = chunks - 1;
      if (OUT) {
        if (!odd_1) {
          wait(intra_done, z);
          tc_fence_after();
          uint32_t y[kTokens / 2];
          make_o(z, prev_s, false, y);
          store_o(z, y);
        }
      } else {
        wait(done + (z & 1) * 8, z >> 1);
        tc_fence_after();
        add(z, prev_k, odd_1);
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    float* to = nullptr;
    if (!OUT)
      to = p.added + ((int64_t)id * p.heads + head) * state_size;
    else if (p.state_out && last)
      to = p.state_out + ((int64_t)slot * p.heads + head) * state_size;
    // Should a wait have given up, what there is of o and S is not to be taken for results.  (The rows of o under way have arrived.)
    asm volatile("bar.sync 2, %0;" ::"n"(kThreads + 32) : "memory");
    const bool gave_up = *(volatile uint32_t*)&abort_flag != 0;
    if (OUT && gave_up && live) {
      unsigned short* at = static_cast<unsigned short*>(p.o) + (int64_t)head * p.dv + col;
      for (int t = first + quarter; t < end; t += kQuarters) at[(int64_t)t * p.o_stride] = 0x7fff;         // (a NaN of either type)
    }
    if (to && live) {
      const float E = gave_up ? __builtin_nanf("") : chunks > 0 ? decays[(chunks - 1) & 3].behind : 1.0f;
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        const int e = quarter * kMine + j;
        if (e < p.dk) to[(int64_t)e * p.dv + col] = S[j] * E;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_dealloc(tmem, L::kColumns);
}

// The starting state of every segment of a sequence that is cut, in the place of what it adds: a thread has W numbers of a head's
// state and runs over the segments.
template <int W>
__global__ void __launch_bounds__(256) segment_states_kernel(const ChunkParams p, const float* pool, int32_t blocks) {
  const uint32_t rest = blockIdx.x / (uint32_t)blocks;
  const int head = (int)(rest % (uint32_t)p.heads), b = (int)(rest / (uint32_t)p.heads);
  const SequenceRows rows = rows_of(p.seqs, b);
  const int32_t len = rows.end - rows.begin;
  const int slot = slot_of(p.seqs, b);
  using V = Vec<float, W>;
  const int64_t size = (int64_t)p.dk * p.dv, e = ((int64_t)(blockIdx.x % (uint32_t)blocks) * 256 + threadIdx.x) * W;
  if (len <= p.L || slot < 0 || e >= size) return;
  const int32_t n = (len + p.L - 1) / p.L;
  // (as find_piece numbers them)
  const int64_t id0 = p.seqs.cu ? (int64_t)(rows.begin / p.L) + b : (int64_t)b * n;
  V s = {};
  if (pool && resumes(p.seqs, b)) s = *reinterpret_cast<const V*>(pool + ((int64_t)slot * p.heads + head) * size + e);
  constexpr int kAhead = 4;
  for (int i0 = 0; i0 < n; i0 += kAhead) {
    V added[kAhead];
    float2 total[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i0 + i + 1 >= n) break;                              // (the last one's sum is not made)
      const int64_t at = (id0 + i0 + i) * p.heads + head;
      added[i] = *reinterpret_cast<const V*>(p.added + at * size + e);
      total[i] = p.totals[at];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i0 + i >= n) break;
      *reinterpret_cast<V*>(p.added + ((id0 + i0 + i) * p.heads + head) * size + e) = s;
      if (i0 + i + 1 >= n) break;
#pragma unroll
      for (int u = 0; u < W; ++u) s.v[u] = carry(s.v[u], total[i], added[i].v[u]);
    }
  }
}

struct ChunkPlan {
  bool eligible;
  int32_t tiles, L;
  int64_t segments;                      // 0: every sequence is one
  size_t totals_off, added_off, bytes;
};

// Segments by an estimate, in chunks' times (2.6 us): a launch takes as long as its rounds of the longest pieces, or as all of its
// work spread over 148 SMs if that is longer, four for the start and end of a block; where sequences are cut, what the segments but the
// last add comes before, at 0.65 of the time, and two more launches.  (One sequence of 16384 tokens, 32 heads of 128 x 128, bf16: 256
// chunks in one piece 628 us, in 2, 4, 5, 8, 9, 12, 18 segments 547, 301, 377, 321, 298, 343, 338: the estimate takes 9.  Of 8192 tokens 1,
// 2, 4, 5, 9: 322, 294, 173, 215, 186: it takes 4.  13 sequences of up to 2488, 24 heads of 64 x 128, fp16: 1, 2, 3 segments 121, 182, 158:
// it takes 1.)
ChunkPlan plan_chunks(const im2win_attention_shape& s, im2win_dtype dtype, bool has_cu) {
  ChunkPlan c = {};
  const int64_t longest = has_cu ? (s.max_len > 0 ? (s.max_len < s.tokens ? s.max_len : s.tokens) : s.tokens) : s.tokens / s.sequences;
  // Not the shortest prompts: up to 16 tokens the recurrence, which waits for nothing but its loads, is as fast.  (Rows that start anywhere
  // come an element at a time: 13 prompts of 9001 tokens, 24 heads of 61 x 123, 253 us, where 64 x 128 takes 120 and its recurrence 2600.)
  c.eligible = dtype != IM2WIN_F32 && s.dk <= 128 && longest > 16;
  if (!c.eligible) return c;
  c.tiles = (s.dv + kTile - 1) / kTile;
  const int64_t blocks = (int64_t)s.heads * c.tiles;
  const int64_t chunks = (longest + kChunk - 1) / kChunk;
  // sequences of the longest one's length that there can be
  int64_t like = s.tokens / longest;
  if (like < 1) like = 1;
  double best = 0;
  int64_t best_n = 1;
  constexpr double kEnds = 4.0, kAdds = 0.65, kLaunches = 7.0;
  const double work = (double)((s.tokens / kChunk + s.sequences) * blocks);
  for (int64_t n = 1; n <= chunks && n <= 64; ++n) {
    const int64_t per = (chunks + n - 1) / n;
    auto launch_time = [&](int64_t longest_pieces, double all_chunks, double pieces) {
      return std::max((double)((longest_pieces + 147) / 148) * ((double)per + kEnds), (all_chunks + pieces * kEnds) / 148.0);
    };
    const double pieces = (double)(number_of_pieces(s.tokens, s.sequences, n == 1 ? (int64_t)1 << 40 : per * kChunk, has_cu) * blocks);
    double cost = launch_time(like * blocks * n, work, pieces);
    if (n > 1) cost += kAdds * launch_time(like * blocks * (n - 1), (double)(like * blocks * (n - 1) * per), (double)(like * blocks * (n - 1))) + kLaunches;
    if (n == 1 || cost < best) { best = cost; best_n = n; }
  }
  if (const char* v = debug_getenv("IM2WIN_SEGMENTS")) best_n = std::min<int64_t>(std::max(atoi(v), 1), chunks);    // testing aid
  c.totals_off = c.added_off = c.bytes = kStatusBytes;
  c.L = INT32_MAX;
  if (best_n > 1) {
    c.L = (int32_t)((chunks + best_n - 1) / best_n * kChunk);
    c.segments = number_of_pieces(s.tokens, s.sequences, c.L, has_cu);
    c.added_off = c.totals_off + (size_t)((c.segments * s.heads * (int64_t)sizeof(float2) + 255) / 256 * 256);
    c.bytes = c.added_off + (size_t)(c.segments * s.heads * (int64_t)s.dk * s.dv * 4);
  }
  return c;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
EncodeTiledFn get_encode_fn() {
  static EncodeTiledFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<EncodeTiledFn>(f);
  }();
  return fn;
}

bool encode(EncodeTiledFn fn, CUtensorMap* map, im2win_dtype dtype, const void* at, int64_t tokens, int64_t heads, int64_t size, int64_t stride,
            uint32_t box_elements, CUtensorMapSwizzle swizzle) {
  const cuuint64_t dims[3] = {(cuuint64_t)size, (cuuint64_t)heads, (cuuint64_t)tokens};
  const cuuint64_t strides[2] = {(cuuint64_t)size * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[3] = {box_elements, 1, kChunk}, one[3] = {1, 1, 1};
  return fn(map, dtype == IM2WIN_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(at), dims, strides,
            box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DK, bool OUT>
cudaError_t launch(const ChunkMaps& maps, const ChunkParams& p, int64_t pieces, cudaStream_t stream) {
  constexpr uint32_t kBytes = Layout<T, DK, OUT>::kBytes;
  static bool attr_done[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!attr_done[dev]) {
    cudaError_t e = cudaFuncSetAttribute(chunk_kernel<T, DK, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes);
    if (e != cudaSuccess) return e;
    // A build whose blocks start with fewer registers than the warpgroups ask for later would wait for them without end: not launched.
    cudaFuncAttributes built;
    e = cudaFuncGetAttributes(&built, chunk_kernel<T, DK, OUT>);
    if (e != cudaSuccess) return e;
    if (built.numRegs * kAllThreads < kThreads * kWorkerRegisters + (kAllThreads - kThreads) * kHelperRegisters) return cudaErrorNotSupported;
    attr_done[dev] = true;
  }
  const int64_t grid = pieces * p.heads * p.tiles;             // (launch_all has seen that it fits)
  chunk_kernel<T, DK, OUT><<<(unsigned)grid, kAllThreads, kBytes, stream>>>(maps, p);
  return cudaGetLastError();
}

template <typename T, int DK>
cudaError_t launch_all(const ChunkMaps& maps, ChunkParams& p, const ChunkPlan& plan, const AttentionArgs& a, cudaStream_t stream) {
  const int64_t pieces = plan.segments ? plan.segments : number_of_pieces(a.shape.tokens, a.shape.sequences, p.L, a.seqs.cu != nullptr);
  const int32_t width = p.dk * p.dv % 4 == 0 ? 4 : 1;
  const int32_t blocks = (int32_t)(((int64_t)p.dk * p.dv + 256 * width - 1) / (256 * width));
  const int64_t grid = (int64_t)blocks * p.heads * a.shape.sequences, most = (int64_t)1 << 31;
  if (pieces * p.heads * p.tiles >= most || (plan.segments && grid >= most)) return cudaErrorInvalidConfiguration;
  if (cudaMemsetAsync(p.status, 0, kStatusBytes, stream) != cudaSuccess) return cudaErrorUnknown;
  // Testing aids: a chunk that head 0 drops (ChunkParams) of the launch that makes o, or of the one that sums up; waits then give up
  // after 4096 polls (word 1 of the status block).
  const char* drop = debug_getenv("IM2WIN_ATTENTION_DROP");
  const char* drop_sums = debug_getenv("IM2WIN_ATTENTION_DROP_SUMS");
  if ((drop || drop_sums) && cudaMemsetAsync(reinterpret_cast<uint8_t*>(p.status) + 5, 0x10, 1, stream) != cudaSuccess) return cudaErrorUnknown;
  if (plan.segments) {
    p.drop = drop_sums ? atoi(drop_sums) : -1;
    cudaError_t e = launch<T, DK, false>(maps, p, pieces, stream);
    if (e != cudaSuccess) return e;
    if (width == 4)
      segment_states_kernel<4><<<(unsigned)grid, 256, 0, stream>>>(p, a.state_in, blocks);
    else
      segment_states_kernel<1><<<(unsigned)grid, 256, 0, stream>>>(p, a.state_in, blocks);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    p.segmented = 1;
  }
  p.drop = drop ? atoi(drop) : -1;
  return launch<T, DK, true>(maps, p, pieces, stream);
}

}  // namespace

bool attention_by_chunks(const im2win_attention_shape& s, im2win_dtype dtype, bool has_cu, size_t* workspace_bytes, bool* segmented) {
  const ChunkPlan plan = plan_chunks(s, dtype, has_cu);
  *workspace_bytes = plan.eligible ? plan.bytes : kStatusBytes;
  *segmented = plan.eligible && plan.segments > 0;
  return plan.eligible;
}

cudaError_t launch_attention_chunks(const AttentionArgs& a, cudaStream_t stream) {
  const im2win_attention_shape& s = a.shape;
  const ChunkPlan plan = plan_chunks(s, a.dtype, a.seqs.cu != nullptr);
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  ChunkParams p = {a.q, a.k, a.v, a.decay, a.o, a.state_in, a.state_out, reinterpret_cast<float*>(ws + plan.added_off),
                   reinterpret_cast<float2*>(ws + plan.totals_off), reinterpret_cast<uint32_t*>(ws), a.seqs, s.q_stride, s.k_stride,
                   s.v_stride, s.o_stride, s.decay_stride, s.heads, s.heads / s.qk_heads, s.dk, s.dv, plan.tiles, plan.L, 0, 0, 0, -1, s.scale};
  const EncodeTiledFn fn = get_encode_fn();
  if (!fn) return cudaErrorNotSupported;
  p.by_map = s.dk % 8 == 0 && s.dv % 8 == 0 && s.q_stride % 8 == 0 && s.k_stride % 8 == 0 && s.v_stride % 8 == 0 && aligned_to(a.q, 16) &&
             aligned_to(a.k, 16) && aligned_to(a.v, 16);
  p.o_by_map = p.by_map && s.o_stride % 8 == 0 && aligned_to(a.o, 16);
  ChunkMaps maps = {};
  const CUtensorMapSwizzle rows = CU_TENSOR_MAP_SWIZZLE_128B;
  if (p.by_map && (!encode(fn, &maps.q, a.dtype, a.q, s.tokens, s.qk_heads, s.dk, s.q_stride, 64, rows) ||
      !encode(fn, &maps.k, a.dtype, a.k, s.tokens, s.qk_heads, s.dk, s.k_stride, 64, rows) ||
      !encode(fn, &maps.v, a.dtype, a.v, s.tokens, s.heads, s.dv, s.v_stride, 64, rows) ||
      (p.o_by_map && !encode(fn, &maps.o, a.dtype, a.o, s.tokens, s.heads, s.dv, s.o_stride, kTile, CU_TENSOR_MAP_SWIZZLE_NONE))))
    return cudaErrorInvalidValue;
  if (a.dtype == IM2WIN_F16)
    return s.dk <= 64 ? launch_all<__half, 64>(maps, p, plan, a, stream) : launch_all<__half, 128>(maps, p, plan, a, stream);
  return s.dk <= 64 ? launch_all<__nv_bfloat16, 64>(maps, p, plan, a, stream) : launch_all<__nv_bfloat16, 128>(maps, p, plan, a, stream);
}

}  // namespace im2win
