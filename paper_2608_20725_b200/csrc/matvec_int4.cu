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
// The eight warps of a block take turns at the blocks of 128 elements along K and add their sums up at the end, in their order.
// A warp works on TILES tiles of rows, so that x, as many bytes as 8 rows of fp16 have for 16 of the matrix, is fetched (from the
// caches) once for all of them, and loads the next block's weights, scales and zeros before it works on this one's.
#include <type_traits>

#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int kWarps = 8;

struct Int4Params {
  const void* x;
  const uint8_t* weight;
  const void* scales;
  const uint8_t* zeros;
  const float* bias;
  void* y;
  int64_t x_stride, y_stride;
  int32_t M, N, K, group, groups, row_bytes, blocks;   // blocks: of 128 elements along K
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

// PARTS: groups in 128 elements (1: groups of 128 and multiples, 2: of 64, 4: of 32).  NT: tiles of 8 columns of x.
template <typename T, int PARTS, int NT, int TILES, bool ZEROS>
__global__ void __launch_bounds__(kWarps * 32) matvec_kernel(const Int4Params p) {
  using M16 = typename std::conditional<sizeof(T) == 4, __nv_bfloat16, T>::type;   // what the products are made of
  using MM = Mma<M16>;
  constexpr int kWords = 4 / PARTS;              // of a lane, row and group
  constexpr int kPieces = sizeof(T) == 4 ? 3 : 1;
  constexpr int kRows = 2 * TILES;               // of the matrix in a lane
  __shared__ float sums[kWarps][16 * TILES][NT * 8 + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * 16 * TILES;
  auto row_of = [&](int r) { return min(n0 + r * 8 + g, p.N - 1); };               // (rows beyond the last are computed and dropped)
  const T* x[NT];
  int piece[NT];
  bool column[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int c = i * 8 + g;
    column[i] = c < p.M * kPieces;
    piece[i] = kPieces == 3 ? c % 3 : 0;
    x[i] = static_cast<const T*>(p.x) + (int64_t)(column[i] ? c / kPieces : 0) * p.x_stride;
  }

  struct Stage {
    uint32_t w[kRows][4];
    Vec<T, PARTS> scale[kRows];
    Vec<uint8_t, PARTS> zero[ZEROS ? kRows : 1];
  };
  auto fetch = [&](int block, Stage& s) {
    const int j0 = PARTS > 1 ? block * PARTS : (int)((int64_t)block * 128 / p.group);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int row = row_of(r);
      const uint8_t* from = p.weight + (int64_t)row * p.row_bytes;
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
        load_weights<kWords>(from, block * 64 + part * (64 / PARTS) + t * (kWords * 4), p.row_bytes, p.vec_w, &s.w[r][part * kWords]);
      const int64_t at = (int64_t)row * p.groups + j0;
      const T* scale = static_cast<const T*>(p.scales) + at;
      if (PARTS == 1 || p.vec_s) {
        s.scale[r] = *reinterpret_cast<const Vec<T, PARTS>*>(scale);
        if (ZEROS) s.zero[r] = *reinterpret_cast<const Vec<uint8_t, PARTS>*>(p.zeros + at);
      } else {
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          const bool there = j0 + part < p.groups;
          s.scale[r].v[part] = there ? scale[part] : from_float<T>(0.0f);
          if (ZEROS) s.zero[r].v[part] = there ? p.zeros[at + part] : 0;
        }
      }
    }
  };

  float total[TILES][NT][4] = {};
  Stage next;
  if (warp < p.blocks) fetch(warp, next);
  for (int block = warp; block < p.blocks; block += kWarps) {
    const Stage s = next;
    if (block + kWarps < p.blocks) fetch(block + kWarps, next);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      uint32_t bx[NT][kWords][4];
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
#pragma unroll
          for (int h = 0; h < 4; ++h) bx[i][w][h] = 0;
          if (column[i])
            load_x<T>(x[i], block * 128 + part * (128 / PARTS) + t * (kWords * 8) + 8 * w, p.K, p.vec_x, piece[i], bx[i][w]);
        }
#pragma unroll
      for (int tile = 0; tile < TILES; ++tile) {
        uint32_t zero[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
          zero[i] = MM::kMagic + (ZEROS ? (uint32_t)(s.zero[2 * tile + i].v[part] & 15) * 0x10001u : 0x80008u);
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
            for (int i = 0; i < NT; ++i) MM::mma(acc[i], a, bx[i][w][2 * h], bx[i][w][2 * h + 1]);
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
#pragma unroll
  for (int tile = 0; tile < TILES; ++tile)
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) sums[warp][tile * 16 + g + 8 * (r >> 1)][i * 8 + 2 * t + (r & 1)] = total[tile][i][r];
  __syncthreads();
  for (int at = threadIdx.x; at < 16 * TILES * p.M; at += kWarps * 32) {
    const int n = at % (16 * TILES), m = at / (16 * TILES);
    if (n0 + n >= p.N) continue;
    float y = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w)
#pragma unroll
      for (int i = kPieces - 1; i >= 0; --i) y += sums[w][n][m * kPieces + i];
    if (p.bias) y += p.bias[n0 + n];
    static_cast<T*>(p.y)[(int64_t)m * p.y_stride + n0 + n] = from_float<T>(y);
  }
}

template <typename T, int PARTS, int NT, int TILES>
cudaError_t launch(const Int4Params& p, cudaStream_t stream) {
  const unsigned grid = (unsigned)((p.N + 16 * TILES - 1) / (16 * TILES));
  if (p.zeros)
    matvec_kernel<T, PARTS, NT, TILES, true><<<grid, kWarps * 32, 0, stream>>>(p);
  else
    matvec_kernel<T, PARTS, NT, TILES, false><<<grid, kWarps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

// Tiles of a warp: more where that leaves two blocks an SM and more.
template <typename T, int PARTS, int NT>
cudaError_t launch_tiles(const Int4Params& p, cudaStream_t stream) {
  if constexpr (NT <= 2)
    if (p.N >= 296 * 32) return launch<T, PARTS, NT, 2>(p, stream);
  return launch<T, PARTS, NT, 1>(p, stream);
}

template <typename T, int PARTS>
cudaError_t launch_columns(const Int4Params& p, cudaStream_t stream) {
  const int columns = p.M * (sizeof(T) == 4 ? 3 : 1);
  if (columns <= 8) return launch_tiles<T, PARTS, 1>(p, stream);
  if (columns <= 16) return launch_tiles<T, PARTS, 2>(p, stream);
  if constexpr (sizeof(T) == 4) {
    if (columns <= 24) return launch_tiles<T, PARTS, 3>(p, stream);
    return launch_tiles<T, PARTS, 6>(p, stream);
  }
  return cudaErrorInvalidValue;
}

template <typename T>
cudaError_t launch_type(Int4Params& p, cudaStream_t stream) {
  p.vec_w = p.row_bytes % 16 == 0 && aligned_to(p.weight, 16);
  p.vec_x = (p.x_stride * (int64_t)sizeof(T)) % 16 == 0 && aligned_to(p.x, 16);
  p.vec_s = p.groups % 4 == 0 && aligned_to(p.scales, 16) && aligned_to(p.zeros, 4);
  if (p.group == 32) return launch_columns<T, 4>(p, stream);
  if (p.group == 64) return launch_columns<T, 2>(p, stream);
  return launch_columns<T, 1>(p, stream);
}

}  // namespace

cudaError_t launch_matvec_int4(const void* x, const uint8_t* weight, const void* scales, const uint8_t* zeros, const float* bias,
                               void* y, const im2win_int4_shape& s, im2win_dtype dtype, cudaStream_t stream) {
  Int4Params p = {x, weight, scales, zeros, bias, y, s.x_stride, s.y_stride, s.M, s.N, s.K, s.group,
                  (int32_t)(((int64_t)s.K + s.group - 1) / s.group), (int32_t)(((int64_t)s.K + 1) / 2),
                  (int32_t)(((int64_t)s.K + 127) / 128), 0, 0, 0};
  switch (dtype) {
    case IM2WIN_F32: return launch_type<float>(p, stream);
    case IM2WIN_F16: return launch_type<__half>(p, stream);
    default: return launch_type<__nv_bfloat16>(p, stream);
  }
}

}  // namespace im2win
