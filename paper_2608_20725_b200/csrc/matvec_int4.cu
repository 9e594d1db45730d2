// A few rows times a matrix of 4-bit weights with group scales (im2win_matvec_int4):
//
//   y[m][n] = bias[n] + sum_groups s[n][j] * sum_{k in group j} (w[n][k] - z[n][j]) x[m][k].
//
// The matrix is read once, half a byte a weight, which bounds it for up to 16 rows.  At the memory's rate a lane of an SM has
// under three instructions for each weight; one multiply-add a weight and row would take most of them already, so the products run
// on mma.sync (16 rows of the matrix x 8 columns of x x 16 terms): what is left is 10 to 12 instructions for eight weights to make
// them 16-bit numbers.  w - z lies in -15..15, which both 16-bit types hold exactly, and so are the products; a group's sum comes out
// of the accumulators in fp32 and meets its scale there.  (tcgen05 wants its 128 rows of weights in shared or tensor memory: for
// 8 columns that would be more work than the products.)
//
// The order of the terms of a product is free as long as both operands agree.  Lane (g = lane/4, t = lane%4) holds rows g and g+8 of
// a tile of the matrix and the t-th of four equal parts of a group's elements, so that it loads neighbouring bytes; of a word's eight
// nibbles n0..n7 a mask gives (n0, n4), (n1, n5), (n2, n6), (n3, n7), and x is brought into that order instead.
// fp32 rows of x are three rows of bf16 pieces each, cut off so that their sum is exact; a column of the product for each.
//
// A block stays on an SM and takes groups of rows in turn.  It brings x into shared memory once, as the products want it (for a batch
// of 8, twice the bytes that 16 rows of the matrix have: fetched for each such tile it would be most of the traffic); its 16 warps
// share a group's elements along K, each loading its next two blocks of 128 elements while it works on one, and add their sums up in
// their order.  Measured, without zero points / with, at 6.53 TB/s: see launch_columns.
#include <type_traits>

#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int kWarps = 16;
constexpr int kMostX = 128 * 1024;                     // shared memory for x; longer rows go in passes over K,
constexpr int kMostGroups = 8;                         // whose sums are kept for so many groups of rows at a time

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
  int32_t vec_w, vec_x, vec_s;                         // whether rows of the matrix, of x, and a block's scales can be loaded whole
};

template <typename T> struct Mma;
template <> struct Mma<__half> {
  static constexpr uint32_t kMagic = 0x64006400u;      // 1024: the nibble is its lowest bits
  static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b) {
    const __half2 r = __hsub2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
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
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
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

// PARTS: groups in 128 elements (1: groups of 128 and multiples, 2: of 64, 4: of 32).  NT: tiles of 8 columns of x.  TILES: of 16 rows.
// WHOLE: K is a multiple of 128 and everything can be loaded as vectors.
template <typename T, int PARTS, int NT, int TILES, bool WHOLE>
__global__ void __launch_bounds__(kWarps * 32, 1) matvec_kernel(const Int4Params p) {
  using M16 = typename std::conditional<sizeof(T) == 4, __nv_bfloat16, T>::type;   // what the products are made of
  using MM = Mma<M16>;
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
          if (WHOLE) {
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
              const Vec<uint32_t, kWords> v = *reinterpret_cast<const Vec<uint32_t, kWords>*>(w + part * (64 / PARTS));
#pragma unroll
              for (int i = 0; i < kWords; ++i) s.w[r][part * kWords + i] = v.v[i];
            }
            s.scale[r] = *reinterpret_cast<const Vec<T, PARTS>*>(scales + at);
            if (zeros) s.zero[r] = *reinterpret_cast<const Vec<uint8_t, PARTS>*>(zeros + at);
          } else {
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
              const int off = block * 64 + part * (64 / PARTS) + t * (kWords * 4);
              load_weights<kWords>(w + part * (64 / PARTS) - off, off, p.row_bytes, p.vec_w, &s.w[r][part * kWords]);
              const bool group_there = j0 + part < p.groups;
              s.scale[r].v[part] = group_there ? scales[at + part] : from_float<T>(0.0f);
              if (zeros) s.zero[r].v[part] = group_there ? zeros[at + part] : 0;
            }
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

template <typename T, int PARTS, int NT, int TILES, bool WHOLE>
cudaError_t launch_one(Int4Params& p, cudaStream_t stream) {
  constexpr int kSums = 4 * 16 * TILES * (kWarps * (NT * 8 + 1) + kMostGroups * NT * 8);
  static_assert(kMostX + kSums <= 227 * 1024, "more shared memory than a block can have");
  const int block_bytes = 4 * 4 * 16 * p.M * (sizeof(T) == 4 ? 3 : 1);
  p.pass = kMostX / block_bytes;                 // (10 to 512)
  if (p.pass >= p.blocks)
    p.pass = p.blocks;
  else if (p.pass > kWarps)
    p.pass -= p.pass % kWarps;
  p.wk = 1;
  while (p.wk < kWarps && (p.wk < p.pass || p.pass < p.blocks)) p.wk *= 2;
  static bool attr_done[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  auto kernel = matvec_kernel<T, PARTS, NT, TILES, WHOLE>;
  if (!attr_done[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostX + kSums);
    if (e != cudaSuccess) return e;
    attr_done[dev] = true;
  }
  const int64_t group = 16 * TILES * (kWarps / p.wk), groups = (p.N + group - 1) / group;
  kernel<<<(unsigned)(groups < 148 ? groups : 148), kWarps * 32, p.pass * block_bytes + kSums, stream>>>(p);
  return cudaGetLastError();
}

template <typename T, int PARTS, int NT>
cudaError_t launch(Int4Params& p, cudaStream_t stream) {
  const bool whole = p.K % 128 == 0 && p.vec_w && p.vec_x && p.vec_s;
  return whole ? launch_one<T, PARTS, NT, NT <= 2 ? 2 : 1, true>(p, stream) : launch_one<T, PARTS, NT, 1, false>(p, stream);
}

template <typename T, int PARTS>
cudaError_t launch_columns(Int4Params& p, cudaStream_t stream) {
  const int columns = p.M * (sizeof(T) == 4 ? 3 : 1);
  if (columns <= 8) return launch<T, PARTS, 1>(p, stream);
  if constexpr (sizeof(T) == 4) return columns <= 24 ? launch<T, PARTS, 3>(p, stream) : launch<T, PARTS, 6>(p, stream);
  if constexpr (sizeof(T) == 2) return launch<T, PARTS, 2>(p, stream);
}

template <typename T>
cudaError_t launch_type(Int4Params& p, cudaStream_t stream) {
  p.vec_w = p.row_bytes % 16 == 0 && aligned_to(p.weight, 16);
  p.vec_x = (p.x_stride * (int64_t)sizeof(T)) % 16 == 0 && aligned_to(p.x, 16);
  p.vec_s = (p.group >= 128 || p.groups % 4 == 0) && aligned_to(p.scales, 16) && aligned_to(p.zeros, 4);
  if (p.group == 32) return launch_columns<T, 4>(p, stream);
  if (p.group == 64) return launch_columns<T, 2>(p, stream);
  return launch_columns<T, 1>(p, stream);
}

}  // namespace

cudaError_t launch_matvec_int4(const void* x, const uint8_t* weight, const void* scales, const uint8_t* zeros, const float* bias,
                               void* y, const im2win_int4_shape& s, im2win_dtype dtype, cudaStream_t stream) {
  Int4Params p = {x, weight, scales, zeros, bias, y, s.x_stride, s.y_stride, s.M, s.N, s.K, s.group,
                  (int32_t)(((int64_t)s.K + s.group - 1) / s.group), (int32_t)(((int64_t)s.K + 1) / 2),
                  (int32_t)(((int64_t)s.K + 127) / 128), 0, 0, 0, 0, 0};
  switch (dtype) {
    case IM2WIN_F32: return launch_type<float>(p, stream);
    case IM2WIN_F16: return launch_type<__half>(p, stream);
    default: return launch_type<__nv_bfloat16>(p, stream);
  }
}

}  // namespace im2win
