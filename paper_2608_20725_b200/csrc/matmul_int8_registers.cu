// Rows times a matrix in 8-bit integers, for rows that start anywhere (im2win_matmul_int8):
//
//   y[m][n] = bias[n] + x_scales[m] scales[n] sum_k x[m][k] w[n][k],   sums in 32-bit integers.
//
// A block makes 128 x 128 of y, eight warps 64 x 32 each with the warps' own matrix instruction (16 x 8 x 32), or 64 x 64 where there are few.  Rows of 64 bytes go through registers
// to shared memory, where they lie on 80 bytes (no conflicts), one step ahead of the products.  A row that starts off a word is put together
// from the words it lies on.  (16384 x 8192 x 4096, 2174 us; tiles by TMA take 337.)
//
// Up to 8 rows of x would leave most of a tile without work: a warp then has two rows of the matrix, a lane every 32nd 16 bytes of them, which meet
// all rows of x, staged in shared memory, by products of four bytes (dp4a); the lanes' sums are added at the end.  (5 rows x 4001 x 8001: 31 us; of
// 16 rows, 48, it is slower than the tiles.)
#include <algorithm>

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int kStep = 64, kPitch = kStep + 16, kThreads = 256;

struct Bytes {
  const int8_t* at;
  int64_t stride, size;                  // size: bytes from the first one to the last one, with the gaps between rows
  int32_t rows, K;
};

// 16 bytes of row r from k on, 0 beyond its end.
__device__ __forceinline__ uint4 load16(const Bytes& t, int64_t r, int k) {
  uint32_t w[4] = {0, 0, 0, 0};
  if (r < t.rows && k < t.K) {
    const int64_t from = r * t.stride + k;
    const int8_t* at = t.at + from;
    const uintptr_t address = reinterpret_cast<uintptr_t>(at);
    const int n = min(16, t.K - k);
    if (n == 16 && (address & 15) == 0) return __ldg(reinterpret_cast<const uint4*>(at));
    const int off = (int)(address & 3);
    if (n == 16 && from >= off && from - off + 20 <= t.size) {           // (five whole words, all within the tensor)
      const uint32_t* word = reinterpret_cast<const uint32_t*>(at - off);
      uint32_t v[5];
#pragma unroll
      for (int i = 0; i < 5; ++i) v[i] = __ldg(word + i);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(v[i], v[i + 1], off * 8);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < n) w[i / 4] |= (uint32_t)(uint8_t)__ldg(at + i) << (8 * (i % 4));
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

// Tiles of TILE x TILE (128: eight warps, 64: four).  The CTAs of a cluster share a tile's K; each then finishes a share of its rows from all their sums.
template <typename T, int TILE>
__global__ void __launch_bounds__(TILE * 2) matmul_int8_kernel(const Int8Args p, const Bytes x, const Bytes weight, const int32_t share) {
  constexpr int kThreads = TILE * 2, kI = TILE / 32, kUnits = TILE * 4 / kThreads;
  __shared__ __align__(16) uint8_t tiles[2][2][TILE * kPitch];
  static_assert(TILE == 128 || sizeof(tiles) >= TILE * TILE * 4, "");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t m0 = (int64_t)blockIdx.y * TILE, n0 = (int64_t)(blockIdx.x / share) * TILE;
  const int rank = share > 1 ? (int)ptx::cluster_ctarank() : 0;
  const int steps = (p.shape.K + kStep - 1) / kStep, per = (steps + share - 1) / share;
  const int k_end = min(p.shape.K, (rank + 1) * per * kStep);
  const int wm = (warp & 1) * (TILE / 2), wn = (warp >> 1) * 32;
  int32_t acc[kI][4][4] = {};
  uint4 next[2][kUnits];
  auto load = [&](int k) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int u = tid + i * kThreads;
      next[0][i] = load16(x, m0 + u / 4, k + (u % 4) * 16);
      next[1][i] = load16(weight, n0 + u / 4, k + (u % 4) * 16);
    }
  };
  int buffer = 0;
  if (rank * per * kStep < k_end) load(rank * per * kStep);
  for (int k = rank * per * kStep; k < k_end; k += kStep) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int u = tid + i * kThreads;
        *reinterpret_cast<uint4*>(&tiles[buffer][t][(u / 4) * kPitch + (u % 4) * 16]) = next[t][i];
      }
    __syncthreads();
    if (k + kStep < k_end) load(k + kStep);
    const uint32_t a_at = (uint32_t)__cvta_generic_to_shared(&tiles[buffer][0][(wm + (lane & 15)) * kPitch + (lane >> 4) * 16]);
    const uint32_t b_at = (uint32_t)__cvta_generic_to_shared(&tiles[buffer][1][(wn + (lane & 7) + (lane >> 4) * 8) * kPitch + (lane >> 3 & 1) * 16]);
#pragma unroll
    for (int s = 0; s < kStep / 32; ++s) {
      uint32_t a[kI][4], b[2][4];
#pragma unroll
      for (int i = 0; i < kI; ++i) ldmatrix_x4(a_at + i * 16 * kPitch + s * 32, a[i]);
#pragma unroll
      for (int j = 0; j < 2; ++j) ldmatrix_x4(b_at + j * 16 * kPitch + s * 32, b[j]);
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                       : "+r"(acc[i][j][0]), "+r"(acc[i][j][1]), "+r"(acc[i][j][2]), "+r"(acc[i][j][3])
                       : "r"(a[i][0]), "r"(a[i][1]), "r"(a[i][2]), "r"(a[i][3]), "r"(b[j / 2][j % 2 * 2]), "r"(b[j / 2][j % 2 * 2 + 1]));
    }
    buffer ^= 1;                         // (the next barrier comes before anyone writes this one again)
  }
  T* y = static_cast<T*>(p.y);
  auto finish = [&](int64_t m, int64_t n, int32_t sum, float x_scale) {
    const float v = __fmul_rn((float)sum * x_scale, p.scales[n]);         // (rounded before the bias is added, as by tiles)
    y[m * p.shape.y_stride + n] = from_float<T>(p.bias ? v + p.bias[n] : v);
  };
  if constexpr (TILE == 64) {
    if (share > 1) {
      int32_t* sums = reinterpret_cast<int32_t*>(&tiles[0][0][0]);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sums[(wm + i * 16 + (e >> 1) * 8 + (lane >> 2)) * TILE + wn + j * 8 + (lane & 3) * 2 + (e & 1)] = acc[i][j][e];
      ptx::cluster_sync_all();
      for (int u = rank * kThreads + tid; u < TILE * TILE; u += share * kThreads) {
        int32_t sum = 0;
        for (int r = 0; r < share; ++r) {
          int32_t part;
          asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(part) : "r"(ptx::mapa_shared((uint32_t)__cvta_generic_to_shared(sums + u), r)) : "memory");
          sum += part;
        }
        const int64_t m = m0 + u / TILE, n = n0 + u % TILE;
        if (m < p.shape.M && n < p.shape.N) finish(m, n, sum, p.x_scales[m]);
      }
      ptx::cluster_sync_all();           // (no CTA leaves while another may still read its sums)
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < kI; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t m = m0 + wm + i * 16 + h * 8 + (lane >> 2);
      if (m >= p.shape.M) continue;
      const float xs = p.x_scales[m];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int64_t n = n0 + wn + j * 8 + (lane & 3) * 2 + e;
          if (n < p.shape.N) finish(m, n, acc[i][j][2 * h + e], xs);
        }
    }
}

// Tiles of 128 where there are two for each SM; otherwise of 64, and clusters of up to eight CTAs share a tile's K until there are some eight for each SM: a step of
// 64 takes some 2 us, most of it its loads' latency, which other CTAs on the SM fill.  (64 x 4001 x 8001 in tiles of 128 and one CTA each 289 us, so 45.)
template <typename T>
cudaError_t launch_tiles(const Int8Args& a, const Bytes& x, const Bytes& weight, cudaStream_t stream) {
  auto tiles = [&](int64_t size, int64_t tile) { return (size + tile - 1) / tile; };
  const im2win_int8_shape& s = a.shape;
  if (tiles(s.M, 128) * tiles(s.N, 128) >= 296) {
    matmul_int8_kernel<T, 128><<<dim3((unsigned)tiles(s.N, 128), (unsigned)tiles(s.M, 128)), 256, 0, stream>>>(a, x, weight, 1);
    return cudaGetLastError();
  }
  const int64_t all = tiles(s.M, 64) * tiles(s.N, 64), steps = tiles(s.K, kStep);
  int share = 1;
  while (share < 8 && all * share * 2 <= 1184 && steps >= share * 2 * 4) share *= 2;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)share; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(tiles(s.N, 64) * share), (unsigned)tiles(s.M, 64));
  cfg.blockDim = dim3(128, 1, 1);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, matmul_int8_kernel<T, 64>, a, x, weight, (int32_t)share);
}

constexpr int kFewStep = 2048;           // bytes of K of x that are staged
constexpr int kFewRows = 2;              // of the matrix, of a warp

template <typename T, int MOST>
__global__ void __launch_bounds__(kThreads) matmul_int8_few_kernel(const Int8Args p, const Bytes x, const Bytes weight) {
  __shared__ __align__(16) uint4 staged[MOST][kFewStep / 16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, M = p.shape.M;
  const int64_t n0 = ((int64_t)blockIdx.x * (kThreads / 32) + warp) * kFewRows;
  int32_t acc[kFewRows][MOST] = {};
  for (int k0 = 0; k0 < p.shape.K; k0 += kFewStep) {
    const int units = (min(kFewStep, p.shape.K - k0) + 15) / 16;
    __syncthreads();
    for (int i = threadIdx.x; i < M * units; i += kThreads) staged[i / units][i % units] = load16(x, i / units, k0 + i % units * 16);
    __syncthreads();
    for (int u = lane; u < units; u += 32) {
      uint4 w[kFewRows];
#pragma unroll
      for (int n = 0; n < kFewRows; ++n) w[n] = load16(weight, n0 + n, k0 + u * 16);
#pragma unroll
      for (int m = 0; m < MOST; ++m) {
        if (m >= M) break;
        const uint4 v = staged[m][u];
#pragma unroll
        for (int n = 0; n < kFewRows; ++n) {
          acc[n][m] = __dp4a((int)v.x, (int)w[n].x, acc[n][m]);
          acc[n][m] = __dp4a((int)v.y, (int)w[n].y, acc[n][m]);
          acc[n][m] = __dp4a((int)v.z, (int)w[n].z, acc[n][m]);
          acc[n][m] = __dp4a((int)v.w, (int)w[n].w, acc[n][m]);
        }
      }
    }
  }
  T* y = static_cast<T*>(p.y);
#pragma unroll
  for (int n = 0; n < kFewRows; ++n)
#pragma unroll
    for (int m = 0; m < MOST; ++m) {
      if (m >= M) break;
      const int32_t sum = __reduce_add_sync(0xffffffffu, acc[n][m]);
      if (lane == m && n0 + n < p.shape.N) {
        const float v = __fmul_rn((float)sum * p.x_scales[m], p.scales[n0 + n]);
        y[m * p.shape.y_stride + n0 + n] = from_float<T>(p.bias ? v + p.bias[n0 + n] : v);
      }
    }
}

template <typename T>
cudaError_t launch_few(const Int8Args& a, const Bytes& x, const Bytes& weight, cudaStream_t stream) {
  constexpr int kOfBlock = kThreads / 32 * kFewRows;
  const unsigned grid = (unsigned)(((int64_t)a.shape.N + kOfBlock - 1) / kOfBlock);
  if (a.shape.M <= 4) matmul_int8_few_kernel<T, 4><<<grid, kThreads, 0, stream>>>(a, x, weight);
  else matmul_int8_few_kernel<T, 8><<<grid, kThreads, 0, stream>>>(a, x, weight);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_matmul_int8_registers(const Int8Args& a, cudaStream_t stream) {
  constexpr int32_t kMostRows = 65535 * 64;                    // of a grid
  if (a.shape.M > kMostRows) {
    for (int64_t m = 0; m < a.shape.M; m += kMostRows) {
      Int8Args part = a;
      part.x += m * a.shape.x_stride;
      part.x_scales += m;
      part.y = static_cast<uint8_t*>(a.y) + m * a.shape.y_stride * (int64_t)element_bytes(a.dtype);
      part.shape.M = (int32_t)std::min<int64_t>(a.shape.M - m, kMostRows);
      const cudaError_t e = launch_matmul_int8_registers(part, stream);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  const im2win_int8_shape& s = a.shape;
  const Bytes x = {a.x, s.x_stride, (int64_t)(s.M - 1) * s.x_stride + s.K, s.M, s.K};
  const Bytes weight = {a.weight, s.K, (int64_t)s.N * s.K, s.N, s.K};
  if (s.M <= 8) {
    switch (a.dtype) {
      case IM2WIN_F32: return launch_few<float>(a, x, weight, stream);
      case IM2WIN_F16: return launch_few<__half>(a, x, weight, stream);
      default: return launch_few<__nv_bfloat16>(a, x, weight, stream);
    }
  }
  switch (a.dtype) {
    case IM2WIN_F32: return launch_tiles<float>(a, x, weight, stream);
    case IM2WIN_F16: return launch_tiles<__half>(a, x, weight, stream);
    default: return launch_tiles<__nv_bfloat16>(a, x, weight, stream);
  }
}

}  // namespace im2win
