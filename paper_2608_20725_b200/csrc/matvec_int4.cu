// A few rows times a matrix of 4-bit weights with group scales (im2win_matvec_int4):
//
//   y[m][n] = bias[n] + sum_groups s[n][j] * sum_{k in group j} (w[n][k] - z[n][j]) x[m][k].
//
// The matrix is read once, half a byte a weight, which should bound it for up to 16 rows.  The products run on mma.sync (16 rows of the
// matrix x 8 columns of x x 16 terms): w - z lies in -15..15, which both 16-bit types hold exactly, and so are the products; a group's
// sum comes out of the accumulators in fp32 and meets its scale there.  Making the 16-bit numbers takes 11 instructions for eight weights.
// What bounds it now: the instructions around the products (making the numbers, scales, sums), which take half of the issue slots, and
// what they wait for.  28672 x 8192, whose 117 MB the ring below alone brings in 26 us (18 at the measured bandwidth), 8 rows of bf16, calls
// from a graph: 73 us with groups of 64 and zero points, 68 without these, 56 with groups of 128, 92 with 32; groups of 128 with 1, 2, 4, 16
// rows 54, 55, 55, 85; 8 rows of fp32 127.  Between events around a single call, which counts some 6 us more, groups of 64 with zero points
// took 82, and 64 with scales that were not loaded: they are single loads of 2 to 16 bytes, rows apart.  The products themselves are hidden: a
// quarter of an SM makes one in 9 cycles, and without them the times are the same.  Paired fp32 multiply-adds in their place were slower from
// one row on (80, 127, 224 us for 1, 2, 4 rows).  Registers are at their limit of 128: groups of 64 with up to 8 columns of x spill 44 bytes in
// bf16 and 12 in fp16, the forms of 16 and 24 columns up to 40 and 96.
//
// The order of the terms of a product is free as long as both operands agree.  Lane (g = lane/4, t = lane%4) holds rows g and g+8 of
// a tile of the matrix and the t-th of four equal parts of a group's elements, so that it loads neighbouring bytes; of a word's eight
// nibbles n0..n7 a mask gives (n0, n4), (n1, n5), (n2, n6), (n3, n7), and x is brought into that order instead.
// fp32 rows of x are three rows of bf16 pieces each, cut off so that their sum is exact; a column of the product for each.
//
// A block stays on an SM and takes its part of the rows, in tiles of 32; its 16 warps share a tile's elements along K, 128 each of 2048
// at a time, keep x for theirs in registers from one tile to the next, and add their sums up at the end of a tile, in their order.  The matrix
// comes through a ring of kSlots such chunks in shared memory, row by row (bulk copies; loads to registers two blocks ahead took 100 us in
// the place of 84).  Rows of more than a pass of K (4096 elements for 8 columns of x, 2048 for more columns or for groups of 32:
// what registers hold; 8192 spilled, 90 us in the place of 82) go in passes, whose sums are kept for kMostGroups tiles at a time.  Rows that do not start on 16-byte boundaries, and a K that is no
// multiple of 128, go through registers (matvec_any_kernel), and so do scales or zero points that cannot be loaded a block at once.
#include <stdlib.h>

#include <type_traits>

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int kWarps = 16;
constexpr int kMostX = 128 * 1024;                     // shared memory for x of matvec_any_kernel; longer rows go in passes over K,
constexpr int kMostGroups = 8;                         // whose sums are kept for so many tiles or groups of rows at a time

struct Int4Params {
  const void* x;
  const uint8_t* weight;
  const void* scales;
  const uint8_t* zeros;
  const float* bias;
  void* y;
  int64_t x_stride, y_stride;
  int32_t M, N, K, group, groups, row_bytes, blocks;   // blocks: of 128 elements along K
  int32_t pass, wk;                                    // blocks of a pass, warps that share a group of rows along K
  int32_t vec_w, vec_x, ring;                          // whether rows of the matrix and of x can be loaded whole; matvec_kernel or the other
  uint32_t polls;                                      // looks, of a microsecond at most, before a wait gives up
  int32_t drop;                                        // testing aid: a warp of block 0 does not say that it is done with this tile (-1: all do)
};

template <typename T> struct Mma;
template <> struct Mma<__half> {
  static constexpr uint32_t kMagic = 0x64006400u;      // 1024: the nibble is its lowest bits
  static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b) {
    const __half2 r = __hsub2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <> struct Mma<__nv_bfloat16> {
  static constexpr uint32_t kMagic = 0x43004300u;      // 128
  static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

// Piece `which` (0 to 2) of an fp32 number as bf16 bits: the upper half of what the pieces before it leave, so that the three add up
// to it exactly.  Infinities and NaNs are their own first piece.
__device__ __forceinline__ uint32_t bf16_piece(float x, int which) {
  const uint32_t bits = __float_as_uint(x);
  if ((bits & 0x7f800000u) == 0x7f800000u) return which ? 0u : (bits & 0x007fffffu) ? 0x7fc0u : bits >> 16;
  if (which == 0) return bits >> 16;
  const float r1 = x - __uint_as_float(bits & 0xffff0000u);
  const uint32_t bits1 = __float_as_uint(r1);
  if (which == 1) return bits1 >> 16;
  return __float_as_uint(r1 - __uint_as_float(bits1 & 0xffff0000u)) >> 16;
}

// W words (8 elements each) of a row of the matrix; bytes beyond the row's end read as 0 (x is 0 there).
template <int W>
__device__ __forceinline__ void load_weights(const uint8_t* row, int at, int row_bytes, bool vec, uint32_t* w) {
  if (vec && at + 4 * W <= row_bytes) {
    const Vec<uint32_t, W> v = *reinterpret_cast<const Vec<uint32_t, W>*>(row + at);
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = v.v[i];
    return;
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    w[i] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + 4 * i + j < row_bytes) w[i] |= (uint32_t)row[at + 4 * i + j] << (8 * j);
  }
}

// Eight elements of a column of x from element `at`, as the four pairs (0, 4), (1, 5), (2, 6), (3, 7).
template <typename T>
__device__ __forceinline__ void load_x(const T* row, int at, int K, bool vec, int piece, uint32_t* out) {
  if constexpr (sizeof(T) == 2) {
    uint32_t r[4];
    if (vec && at + 8 <= K) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(row + at));
      r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = at + 2 * i < K ? reinterpret_cast<const uint16_t*>(row)[at + 2 * i] : 0;
        const uint32_t hi = at + 2 * i + 1 < K ? reinterpret_cast<const uint16_t*>(row)[at + 2 * i + 1] : 0;
        r[i] = lo | hi << 16;
      }
    }
    out[0] = __byte_perm(r[0], r[2], 0x5410);
    out[1] = __byte_perm(r[0], r[2], 0x7632);
    out[2] = __byte_perm(r[1], r[3], 0x5410);
    out[3] = __byte_perm(r[1], r[3], 0x7632);
  } else {
    float f[8];
    if (vec && at + 8 <= K) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(row + at)), b = __ldg(reinterpret_cast<const float4*>(row + at + 4));
      f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = at + i < K ? row[at + i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = bf16_piece(f[i], piece) | bf16_piece(f[i + 4], piece) << 16;
  }
}

// PARTS: groups in 128 elements (1: groups of 128 and multiples, 2: of 64, 4: of 32).  NT: tiles of 8 columns of x.
// Everything may be ragged and unaligned.
template <typename T, int PARTS, int NT>
__global__ void __launch_bounds__(kWarps * 32, 1) matvec_any_kernel(const Int4Params p) {
  using M16 = typename std::conditional<sizeof(T) == 4, __nv_bfloat16, T>::type;   // what the products are made of
  using MM = Mma<M16>;
  constexpr int TILES = 1;                       // of 16 rows in a warp
  constexpr int kWords = 4 / PARTS;              // of a lane, row and group
  constexpr int kPieces = sizeof(T) == 4 ? 3 : 1;
  constexpr int kRows = 2 * TILES;               // of the matrix in a lane
  constexpr int kGroupRows = 16 * TILES;
  extern __shared__ uint4 xs[];                  // [block][word][column][t]: a lane's eight elements of a word, as pairs
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int columns = p.M * kPieces;
  // behind x: the warps' sums of a group of rows, and what passes over K have added up so far
  float (*sums)[kGroupRows][NT * 8 + 1] = reinterpret_cast<float (*)[kGroupRows][NT * 8 + 1]>(xs + p.pass * 16 * columns);
  float (*kept)[kGroupRows][NT * 8] = reinterpret_cast<float (*)[kGroupRows][NT * 8]>(sums + kWarps);
  const int wk = p.wk, part_k = warp % wk, sub = warp / wk, subs = kWarps / wk;    // subs groups of rows side by side
  const int all_groups = (p.N + kGroupRows * subs - 1) / (kGroupRows * subs);

  struct Stage {
    uint32_t w[kRows][4];
    Vec<T, PARTS> scale[kRows];
    Vec<uint8_t, PARTS> zero[kRows];
  };
  const int first_group = blockIdx.x, my_groups = (all_groups - first_group + (int)gridDim.x - 1) / (int)gridDim.x;
  for (int batch = 0; batch < my_groups; batch += kMostGroups) {
    const int n_groups = min(kMostGroups, my_groups - batch);
    for (int b0 = 0; b0 < p.blocks; b0 += p.pass) {
      const int nb = min(p.pass, p.blocks - b0);
      // x of this pass
      if (b0 > 0 || batch == 0 || p.pass < p.blocks) {
        __syncthreads();
        for (int c = 0; c < columns; ++c) {
          const T* row = static_cast<const T*>(p.x) + (int64_t)(c / kPieces) * p.x_stride;
          for (int u = threadIdx.x; u < nb * 16; u += kWarps * 32) {
            // word `word` of block b and lane t: the part's elements, the lane's among them, the word's among those
            const int ut = u & 3, word = (u >> 2) & 3, b = u >> 4, part = word / kWords, w = word % kWords;
            const int e = (b0 + b) * 128 + part * (128 / PARTS) + ut * (kWords * 8) + 8 * w;
            uint32_t pairs[4];
            load_x<T>(row, e, p.K, p.vec_x, c % kPieces, pairs);
            xs[((u >> 2) * columns + c) * 4 + ut] = make_uint4(pairs[0], pairs[1], pairs[2], pairs[3]);
          }
        }
        __syncthreads();
      }
      const int turns = (nb + wk - 1) / wk;
      auto first_row = [&](int group) { return ((first_group + (batch + group) * (int)gridDim.x) * subs + sub) * kGroupRows; };
      int next_group = 0, next_turn = 0;         // what is fetched next
      int64_t row_at = 0;                        // this lane's first row of that group
      auto fetch = [&](Stage& s) {
        if (next_turn == 0) row_at = first_row(next_group) + g;
        const int block = b0 + part_k + next_turn * wk;
        const bool there = next_group < n_groups && block < b0 + nb;
        if (++next_turn == turns) {
          next_turn = 0;
          ++next_group;
        }
        if (!there) return;
        const int j0 = PARTS > 1 ? block * PARTS : p.group == 128 ? block : (int)((int64_t)block * 128 / p.group);
        const uint8_t* weight = p.weight + row_at * p.row_bytes + block * 64 + t * (kWords * 4);
        const T* scales = static_cast<const T*>(p.scales) + row_at * p.groups + j0;
        const uint8_t* zeros = p.zeros ? p.zeros + row_at * p.groups + j0 : nullptr;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          if (row_at + r * 8 >= p.N) break;      // (rows beyond the last: whatever was there is worked on and dropped)
          const uint8_t* w = weight + (int64_t)(r * 8) * p.row_bytes;
          const int64_t at = (int64_t)(r * 8) * p.groups;
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
              const int off = block * 64 + part * (64 / PARTS) + t * (kWords * 4);
              load_weights<kWords>(w + part * (64 / PARTS) - off, off, p.row_bytes, p.vec_w, &s.w[r][part * kWords]);
              const bool group_there = j0 + part < p.groups;
              s.scale[r].v[part] = group_there ? scales[at + part] : from_float<T>(0.0f);
              if (zeros) s.zero[r].v[part] = group_there ? zeros[at + part] : 0;
            }
        }
      };
      float total[TILES][NT][4];
      auto work = [&](int group, int turn, const Stage& s) {
        const int b = part_k + turn * wk;
        if (turn == 0) {
#pragma unroll
          for (int tile = 0; tile < TILES; ++tile)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) total[tile][i][r] = 0.0f;
        }
        if (b < nb) {
#pragma unroll
          for (int part = 0; part < PARTS; ++part) {
            uint4 bx[NT][kWords];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
              for (int w = 0; w < kWords; ++w)
                bx[i][w] = i * 8 + g < columns ? xs[((b * 4 + part * kWords + w) * columns + i * 8 + g) * 4 + t] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int tile = 0; tile < TILES; ++tile) {
              uint32_t zero[2];
#pragma unroll
              for (int i = 0; i < 2; ++i)
                zero[i] = MM::kMagic + (p.zeros ? (uint32_t)(s.zero[2 * tile + i].v[part] & 15) * 0x10001u : 0x80008u);
              float acc[NT][4] = {};
#pragma unroll
              for (int w = 0; w < kWords; ++w) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  uint32_t a[4];
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    const uint32_t word = s.w[2 * tile + (i & 1)][part * kWords + w];
                    a[i] = MM::sub(((word >> (8 * h + 4 * (i >> 1))) & 0x000f000fu) | MM::kMagic, zero[i & 1]);
                  }
#pragma unroll
                  for (int i = 0; i < NT; ++i) MM::mma(acc[i], a, h ? bx[i][w].z : bx[i][w].x, h ? bx[i][w].w : bx[i][w].y);
                }
              }
              const float sa = to_float(s.scale[2 * tile].v[part]), sb = to_float(s.scale[2 * tile + 1].v[part]);
#pragma unroll
              for (int i = 0; i < NT; ++i) {
                total[tile][i][0] = fmaf(sa, acc[i][0], total[tile][i][0]);
                total[tile][i][1] = fmaf(sa, acc[i][1], total[tile][i][1]);
                total[tile][i][2] = fmaf(sb, acc[i][2], total[tile][i][2]);
                total[tile][i][3] = fmaf(sb, acc[i][3], total[tile][i][3]);
              }
            }
          }
        }
        if (turn != turns - 1) return;
        // the group's sums of all warps
#pragma unroll
        for (int tile = 0; tile < TILES; ++tile)
#pragma unroll
          for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[warp][tile * 16 + g + 8 * (r >> 1)][i * 8 + 2 * t + (r & 1)] = total[tile][i][r];
        __syncthreads();
        const int n_first = first_row(group) - sub * kGroupRows, rows_log = 31 - __clz(kGroupRows * subs);
        const bool more = b0 + nb < p.blocks;
        for (int at = threadIdx.x; at < kGroupRows * subs * p.M; at += kWarps * 32) {
          const int n = at & (kGroupRows * subs - 1), m = at >> rows_log, r = n % kGroupRows;
          if (n_first + n >= p.N) continue;
          float y = 0.0f;
          for (int w = 0; w < wk; ++w)
#pragma unroll
            for (int i = kPieces - 1; i >= 0; --i) y += sums[n / kGroupRows * wk + w][r][m * kPieces + i];
          if (b0 > 0) y += kept[group][r][m];     // (passes only where a group has all the warps)
          if (more) {
            kept[group][r][m] = y;
          } else {
            if (p.bias) y += p.bias[n_first + n];
            static_cast<T*>(p.y)[(int64_t)m * p.y_stride + n_first + n] = from_float<T>(y);
          }
        }
        __syncthreads();
      };
      Stage even = {}, odd = {};
      fetch(even);
      fetch(odd);
      int group = 0, turn = 0;
      auto step = [&]() {
        if (++turn == turns) {
          turn = 0;
          ++group;
        }
        return group < n_groups;
      };
      for (;;) {
        work(group, turn, even);
        fetch(even);
        if (!step()) break;
        work(group, turn, odd);
        fetch(odd);
        if (!step()) break;
      }
    }
  }
}

template <typename T, int PARTS, int NT>
cudaError_t launch_any(Int4Params& p, cudaStream_t stream) {
  constexpr int kSums = 4 * 16 * (kWarps * (NT * 8 + 1) + kMostGroups * NT * 8);
  static_assert(kMostX + kSums <= 227 * 1024, "more shared memory than a block can have");
  const int block_bytes = 4 * 4 * 16 * p.M * (sizeof(T) == 4 ? 3 : 1);
  p.pass = kMostX / block_bytes;                 // (20 to 512)
  if (p.pass >= p.blocks)
    p.pass = p.blocks;
  else if (p.pass > kWarps)
    p.pass -= p.pass % kWarps;
  p.wk = 1;
  while (p.wk < kWarps && (p.wk < p.pass || p.pass < p.blocks)) p.wk *= 2;
  static bool attr_done[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  auto kernel = matvec_any_kernel<T, PARTS, NT>;
  if (!attr_done[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostX + kSums);
    if (e != cudaSuccess) return e;
    attr_done[dev] = true;
  }
  const int64_t group = 16 * (kWarps / p.wk), groups = (p.N + group - 1) / group;
  kernel<<<(unsigned)(groups < 148 ? groups : 148), kWarps * 32, p.pass * block_bytes + kSums, stream>>>(p);
  return cudaGetLastError();
}

constexpr int kSlots = 4;
constexpr int kTileRows = 32;                    // rows of a tile: two products high, so that what a warp does but products counts half
constexpr int kChunkBlocks = kWarps;             // blocks of 128 elements of a chunk: one for each warp

// A row of a chunk takes 1024 bytes and 64 / PARTS: the words that a warp reads at once then lie in different banks.
template <int PARTS>
constexpr int kRowPitch = kChunkBlocks * 64 + 64 / PARTS;

// One look at a barrier, of a microsecond at most.
__device__ __forceinline__ bool try_wait_1us(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 1000;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

template <typename T, int PARTS, int NT, int TURNS>
__global__ void __launch_bounds__(kWarps * 32, 1) matvec_kernel(const Int4Params p) {
  using M16 = typename std::conditional<sizeof(T) == 4, __nv_bfloat16, T>::type;   // what the products are made of
  using MM = Mma<M16>;
  constexpr int kWords = 4 / PARTS;              // of a lane, row and group
  constexpr int kPieces = sizeof(T) == 4 ? 3 : 1;
  constexpr int kRows = kTileRows / 8;           // of a lane
  constexpr uint32_t kSlot = kTileRows * kRowPitch<PARTS>;
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ __align__(8) uint64_t bars[2 * kSlots];           // full, empty
  __shared__ uint32_t gave_up;
  float (*sums)[kTileRows][NT * 8 + 1] = reinterpret_cast<float (*)[kTileRows][NT * 8 + 1]>(ring + kSlots * kSlot);
  float (*kept)[kTileRows][NT * 8] = reinterpret_cast<float (*)[kTileRows][NT * 8]>(sums + kWarps);
  const int lane = threadIdx.x & 31, warp = ptx::warp_index(), g = lane >> 2, t = lane & 3;
  const int columns = p.M * kPieces;
  const uint32_t ring_at = ptx::smem_u32(ring), full = ptx::smem_u32(bars), empty = ptx::smem_u32(bars + kSlots);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      ptx::mbar_init(full + i * 8, kWarps);      // a warp copies two rows each
      ptx::mbar_init(empty + i * 8, kWarps);
    }
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    ptx::fence_proxy_async_smem();
  }
  __syncthreads();
  // the block's rows: 16 at a time, of which every block has as many as the others or one more
  const int units = (p.N + 15) / 16, unit = (int)((int64_t)units * blockIdx.x / gridDim.x);
  const int first = unit * 16, last = min((int)((int64_t)units * (blockIdx.x + 1) / gridDim.x) * 16, p.N);
  const int mine = (last - first + kTileRows - 1) / kTileRows;
  bool failed = false;
  // Waits are for copies and warps of this block, which end by themselves.  Should one not within some four seconds, it gives up, the
  // others with it, and y is NaN from that tile on.
  auto wait = [&](uint32_t bar, uint32_t parity) {             // (the whole warp, of one mind)
    uint32_t left = failed ? 0 : p.polls;
    bool there = false;
    while (left-- > 0) {
      there = __all_sync(0xffffffffu, try_wait_1us(bar, parity));
      if (there || ((left & 255u) == 0u && *(volatile uint32_t*)&gave_up)) break;
    }
    if (there) return;
    failed = true;
    gave_up = 1;
  };
  uint32_t fill_slot = 0, fill_parity = 1, use_slot = 0, use_parity = 0;       // (the first wait for an empty slot passes)
  const uint32_t words_at = g * kRowPitch<PARTS> + warp * 64 + t * (kWords * 4);
  for (int batch = 0; batch < mine; batch += kMostGroups) {
    const int n_tiles = min(kMostGroups, mine - batch);
    for (int b0 = 0; b0 < p.blocks; b0 += TURNS * kChunkBlocks) {
      const int nb = min(TURNS * kChunkBlocks, p.blocks - b0), turns = (nb + kChunkBlocks - 1) / kChunkBlocks;
      auto first_row = [&](int tile) { return first + (batch + tile) * kTileRows; };
      uint4 bx[TURNS][NT][4];
#pragma unroll
      for (int turn = 0; turn < TURNS; ++turn)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int word = 0; word < 4; ++word) {
            const int c = i * 8 + g, b = turn * kChunkBlocks + warp;
            uint32_t pairs[4] = {0, 0, 0, 0};
            if (c < columns && b < nb)
              load_x<T>(static_cast<const T*>(p.x) + (int64_t)(c / kPieces) * p.x_stride,
                        (b0 + b) * 128 + word / kWords * (128 / PARTS) + t * (kWords * 8) + 8 * (word % kWords), p.K, true, c % kPieces, pairs);
            bx[turn][i][word] = make_uint4(pairs[0], pairs[1], pairs[2], pairs[3]);
          }
      // this warp's two rows of the next chunk to be filled
      int fill_tile = 0, fill_turn = 0;
      const uint8_t* from = nullptr;
      int64_t second = 0;                        // from the first of the two rows to the other
      auto fill = [&]() {
        if (fill_tile >= n_tiles || failed) return;
        if (fill_turn == 0) {
          const int row = min(first_row(fill_tile) + 2 * warp, p.N - 1);
          from = p.weight + (int64_t)row * p.row_bytes + (int64_t)b0 * 64;
          second = row + 1 < p.N ? p.row_bytes : 0;
        }
        wait(empty + fill_slot * 8, fill_parity);
        if (failed) return;
        if (ptx::elect_one()) {
          const uint32_t bytes = (uint32_t)min(kChunkBlocks, nb - fill_turn * kChunkBlocks) * 64;
          const uint32_t to = ring_at + fill_slot * kSlot + 2 * warp * kRowPitch<PARTS>, bar = full + fill_slot * 8;
          ptx::mbar_arrive_expect_tx(bar, 2 * bytes);
          ptx::bulk_load(to, from, bytes, bar);
          ptx::bulk_load(to + kRowPitch<PARTS>, from + second, bytes, bar);
        }
        __syncwarp();
        from += kChunkBlocks * 64;
        if (++fill_slot == kSlots) {
          fill_slot = 0;
          fill_parity ^= 1;
        }
        if (++fill_turn == turns) {
          fill_turn = 0;
          ++fill_tile;
        }
      };
      Vec<T, PARTS> scale[TURNS][kRows];         // fetched a tile ahead
      Vec<uint8_t, PARTS> zero[TURNS][kRows];
      const T* scales = nullptr;                 // of this lane's first row of the tile that is fetched
      const uint8_t* zeros = nullptr;
      uint32_t row_off[kRows];
      auto fetch_scales = [&](int tile, int turn) {
        const int b = b0 + turn * kChunkBlocks + warp;
        if (tile >= n_tiles || turn * kChunkBlocks + warp >= nb) return;
        const uint32_t j0 = PARTS > 1 ? b * PARTS : p.group == 128 ? b : (uint32_t)((int64_t)b * 128 / p.group);
        if (turn == 0) {
          const int row = min(first_row(tile) + g, p.N - 1);
          const int64_t at = (int64_t)row * p.groups;
          scales = static_cast<const T*>(p.scales) + at;
          if (p.zeros) zeros = p.zeros + at;
#pragma unroll
          for (int r = 0; r < kRows; ++r) row_off[r] = (uint32_t)min(8 * r, p.N - 1 - row) * (uint32_t)p.groups;
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          scale[turn][r] = *reinterpret_cast<const Vec<T, PARTS>*>(scales + (row_off[r] + j0));
          if (p.zeros) zero[turn][r] = *reinterpret_cast<const Vec<uint8_t, PARTS>*>(zeros + (row_off[r] + j0));
        }
      };
#pragma unroll
      for (int turn = 0; turn < TURNS; ++turn) fetch_scales(0, turn);
      // A slot is filled again a chunk after the one it held is done with, so that no warp waits for the slowest at every chunk; short
      // runs need no slot twice and start with all they have.
      const int ahead = n_tiles * turns < kSlots ? kSlots - 1 : kSlots - 2;
      for (int i = 0; i < ahead; ++i) fill();
      float total[kRows / 2][NT][4];
      for (int tile = 0; tile < n_tiles; ++tile) {
#pragma unroll
        for (int h = 0; h < kRows / 2; ++h)
#pragma unroll
          for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) total[h][i][r] = 0.0f;
#pragma unroll
        for (int turn = 0; turn < TURNS; ++turn) {
          if (turn >= turns) break;
          fill();
          wait(full + use_slot * 8, use_parity);
          if (turn * kChunkBlocks + warp < nb) {
            uint32_t words[kRows][4];
            const uint8_t* at = ring + use_slot * kSlot + words_at;
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
              for (int part = 0; part < PARTS; ++part) {
                const Vec<uint32_t, kWords> v = *reinterpret_cast<const Vec<uint32_t, kWords>*>(at + 8 * r * kRowPitch<PARTS> + part * (64 / PARTS));
#pragma unroll
                for (int w = 0; w < kWords; ++w) words[r][part * kWords + w] = v.v[w];
              }
            float s[kRows][PARTS];
            uint32_t z[kRows][PARTS];
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
              for (int part = 0; part < PARTS; ++part) {
                s[r][part] = to_float(scale[turn][r].v[part]);
                z[r][part] = MM::kMagic + (p.zeros ? (uint32_t)(zero[turn][r].v[part] & 15) * 0x10001u : 0x80008u);
              }
            fetch_scales(tile + 1, turn);
            auto products = [&](auto high) {     // of 16 or 32 rows
              constexpr int H = decltype(high)::value;
#pragma unroll
              for (int part = 0; part < PARTS; ++part) {
                float acc[H][NT][4] = {};  // (products of different rows in turn: one that adds to the last waits 40 cycles for it)
#pragma unroll
                for (int w = 0; w < kWords; ++w)
#pragma unroll
                  for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                      uint32_t a[4];
#pragma unroll
                      for (int i = 0; i < 4; ++i)
                        a[i] = MM::sub(((words[2 * h + (i & 1)][part * kWords + w] >> (8 * half + 4 * (i >> 1))) & 0x000f000fu) | MM::kMagic,
                                       z[2 * h + (i & 1)][part]);
#pragma unroll
                      for (int i = 0; i < NT; ++i) {
                        const uint4 x = bx[turn][i][part * kWords + w];
                        MM::mma(acc[h][i], a, half ? x.z : x.x, half ? x.w : x.y);
                      }
                    }
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                  for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) total[h][i][r] = fmaf(s[2 * h + (r >> 1)][part], acc[h][i][r], total[h][i][r]);
              }
            };
            if (last - first_row(tile) > 16)
              products(std::integral_constant<int, 2>());
            else
              products(std::integral_constant<int, 1>());
          }
          __syncwarp();
          if (failed) continue;
          if (lane == 0 && !(tile == p.drop && warp == 3 && blockIdx.x == 0)) ptx::mbar_arrive(empty + use_slot * 8);
          if (++use_slot == kSlots) {
            use_slot = 0;
            use_parity ^= 1;
          }
        }
#pragma unroll
        for (int h = 0; h < kRows / 2; ++h)
#pragma unroll
          for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[warp][h * 16 + g + 8 * (r >> 1)][i * 8 + 2 * t + (r & 1)] = failed ? __int_as_float(0x7fffffff) : total[h][i][r];
        __syncthreads();
        const int n0 = first_row(tile);
        const bool more = b0 + nb < p.blocks;
        for (int at = threadIdx.x; at < kTileRows * p.M; at += kWarps * 32) {
          const int n = at % kTileRows, m = at / kTileRows;
          if (n0 + n >= last) continue;
          float y = 0.0f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w)
#pragma unroll
            for (int i = kPieces - 1; i >= 0; --i) y += sums[w][n][m * kPieces + i];
          if (b0 > 0) y += kept[tile][n][m];     // (this thread's own)
          if (more) {
            kept[tile][n][m] = y;
          } else {
            if (p.bias) y += p.bias[n0 + n];
            static_cast<T*>(p.y)[(int64_t)m * p.y_stride + n0 + n] = from_float<T>(y);
          }
        }
        __syncthreads();
      }
    }
  }
  if (failed) {                                  // copies under way end before the block does
    failed = false;
    while (!failed && (use_slot != fill_slot || use_parity == fill_parity)) {
      wait(full + use_slot * 8, use_parity);
      if (++use_slot == kSlots) {
        use_slot = 0;
        use_parity ^= 1;
      }
    }
  }
}

template <typename T, int PARTS, int NT, int TURNS>
cudaError_t launch_ring(const Int4Params& p, cudaStream_t stream) {
  constexpr int kBytes = kSlots * kTileRows * kRowPitch<PARTS> + 4 * kTileRows * (kWarps * (NT * 8 + 1) + kMostGroups * NT * 8);
  static_assert(kBytes + 1024 <= 227 * 1024, "more shared memory than a block can have");
  static bool attr_done[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  auto kernel = matvec_kernel<T, PARTS, NT, TURNS>;
  if (!attr_done[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    attr_done[dev] = true;
  }
  const int64_t units = ((int64_t)p.N + 15) / 16;
  kernel<<<(unsigned)(units < 148 ? units : 148), kWarps * 32, kBytes, stream>>>(p);
  return cudaGetLastError();
}

// Chunks of a pass by what registers hold: 32 of them x, or 16 to 48 with smaller groups or more columns and their sums.
template <typename T, int PARTS, int NT>
cudaError_t launch(Int4Params& p, cudaStream_t stream) {
  if (!p.ring) return launch_any<T, PARTS, NT>(p, stream);
  return launch_ring<T, PARTS, NT, NT == 1 && PARTS < 4 ? 2 : 1>(p, stream);
}

template <typename T, int PARTS>
cudaError_t launch_columns(Int4Params& p, cudaStream_t stream) {
  const int columns = p.M * (sizeof(T) == 4 ? 3 : 1);
  if (columns <= 8) return launch<T, PARTS, 1>(p, stream);
  if constexpr (sizeof(T) == 4) {
    if (columns <= 24) return launch<T, PARTS, 3>(p, stream);
    // more than eight rows of fp32: eight at a time, which reads the matrix twice
    Int4Params rest = p;
    p.M = 8;
    rest.M -= 8;
    rest.x = static_cast<const T*>(p.x) + 8 * p.x_stride;
    rest.y = static_cast<T*>(p.y) + 8 * p.y_stride;
    const cudaError_t e = launch<T, PARTS, 3>(p, stream);
    return e != cudaSuccess ? e : launch_columns<T, PARTS>(rest, stream);
  }
  if constexpr (sizeof(T) == 2) return launch<T, PARTS, 2>(p, stream);
}

template <typename T>
cudaError_t launch_type(Int4Params& p, cudaStream_t stream) {
  p.vec_w = p.row_bytes % 16 == 0 && aligned_to(p.weight, 16);
  p.vec_x = (p.x_stride * (int64_t)sizeof(T)) % 16 == 0 && aligned_to(p.x, 16);
  // (a row then has whole blocks of 128 elements, and a block's scales and zero points are loaded at once)
  const size_t parts = p.group == 32 ? 4 : p.group == 64 ? 2 : 1;
  p.ring = p.K % 128 == 0 && p.vec_w && p.vec_x && aligned_to(p.scales, parts * sizeof(T)) && aligned_to(p.zeros, parts);
  if (p.group == 32) return launch_columns<T, 4>(p, stream);
  if (p.group == 64) return launch_columns<T, 2>(p, stream);
  return launch_columns<T, 1>(p, stream);
}

}  // namespace

bool matvec_by_ring(const im2win_int4_shape& s, im2win_dtype dtype) {
  return s.K % 128 == 0 && s.x_stride * (int64_t)element_bytes(dtype) % 16 == 0;
}

cudaError_t launch_matvec_int4(const void* x, const uint8_t* weight, const void* scales, const uint8_t* zeros, const float* bias,
                               void* y, const im2win_int4_shape& s, im2win_dtype dtype, cudaStream_t stream) {
  Int4Params p = {x, weight, scales, zeros, bias, y, s.x_stride, s.y_stride, s.M, s.N, s.K, s.group,
                  (int32_t)(((int64_t)s.K + s.group - 1) / s.group), (int32_t)(((int64_t)s.K + 1) / 2),
                  (int32_t)(((int64_t)s.K + 127) / 128), 0, 0, 0, 0, 0, 1u << 22, -1};
  if (const char* v = debug_getenv("IM2WIN_MATVEC_DROP")) {    // testing aid
    p.drop = atoi(v);
    p.polls = 4096;
  }
  switch (dtype) {
    case IM2WIN_F32: return launch_type<float>(p, stream);
    case IM2WIN_F16: return launch_type<__half>(p, stream);
    default: return launch_type<__nv_bfloat16>(p, stream);
  }
}

}  // namespace im2win
