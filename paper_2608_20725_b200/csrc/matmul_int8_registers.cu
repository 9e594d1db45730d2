// Rows times a matrix in 8-bit integers, for rows that start anywhere (im2win_matmul_int8):
//
//   y[m][n] = bias[n] + x_scales[m] scales[n] sum_k x[m][k] w[n][k],   sums in 32-bit integers.
//
// A block makes 128 x 128 of y, eight warps 64 x 32 each with the warps' own matrix instruction (16 x 8 x 32).  Rows of 64 bytes go through registers
// to shared memory, where they lie on 80 bytes (no conflicts), one step ahead of the products.  A row that starts off a word is put together
// from the words it lies on.
#include "sequence.cuh"

namespace im2win {
namespace {

constexpr int kTile = 128, kStep = 64, kPitch = kStep + 16, kThreads = 256;

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

template <typename T>
__global__ void __launch_bounds__(kThreads) matmul_int8_kernel(const Int8Args p, const Bytes x, const Bytes weight) {
  __shared__ __align__(16) uint8_t tiles[2][2][kTile * kPitch];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
  const int wm = (warp & 1) * 64, wn = (warp >> 1) * 32;
  int32_t acc[4][4][4] = {};
  uint4 next[2][2];
  auto load = [&](int k) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int u = tid + i * kThreads;
      next[0][i] = load16(x, m0 + u / 4, k + (u % 4) * 16);
      next[1][i] = load16(weight, n0 + u / 4, k + (u % 4) * 16);
    }
  };
  load(0);
  int buffer = 0;
  for (int k = 0; k < p.shape.K; k += kStep) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int u = tid + i * kThreads;
        *reinterpret_cast<uint4*>(&tiles[buffer][t][(u / 4) * kPitch + (u % 4) * 16]) = next[t][i];
      }
    __syncthreads();
    if (k + kStep < p.shape.K) load(k + kStep);
    const uint32_t a_at = (uint32_t)__cvta_generic_to_shared(&tiles[buffer][0][(wm + (lane & 15)) * kPitch + (lane >> 4) * 16]);
    const uint32_t b_at = (uint32_t)__cvta_generic_to_shared(&tiles[buffer][1][(wn + (lane & 7) + (lane >> 4) * 8) * kPitch + (lane >> 3 & 1) * 16]);
#pragma unroll
    for (int s = 0; s < kStep / 32; ++s) {
      uint32_t a[4][4], b[2][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) ldmatrix_x4(a_at + i * 16 * kPitch + s * 32, a[i]);
#pragma unroll
      for (int j = 0; j < 2; ++j) ldmatrix_x4(b_at + j * 16 * kPitch + s * 32, b[j]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                       : "+r"(acc[i][j][0]), "+r"(acc[i][j][1]), "+r"(acc[i][j][2]), "+r"(acc[i][j][3])
                       : "r"(a[i][0]), "r"(a[i][1]), "r"(a[i][2]), "r"(a[i][3]), "r"(b[j / 2][j % 2 * 2]), "r"(b[j / 2][j % 2 * 2 + 1]));
    }
    buffer ^= 1;                         // (the next barrier comes before anyone writes this one again)
  }
  T* y = static_cast<T*>(p.y);
#pragma unroll
  for (int i = 0; i < 4; ++i)
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
          if (n >= p.shape.N) continue;
          const float v = (float)acc[i][j][2 * h + e] * xs * p.scales[n];
          y[m * p.shape.y_stride + n] = from_float<T>(p.bias ? v + p.bias[n] : v);
        }
    }
}

}  // namespace

cudaError_t launch_matmul_int8_registers(const Int8Args& a, cudaStream_t stream) {
  const im2win_int8_shape& s = a.shape;
  const Bytes x = {a.x, s.x_stride, (int64_t)(s.M - 1) * s.x_stride + s.K, s.M, s.K};
  const Bytes weight = {a.weight, s.K, (int64_t)s.N * s.K, s.N, s.K};
  const dim3 grid((unsigned)(((int64_t)s.N + kTile - 1) / kTile), (unsigned)(((int64_t)s.M + kTile - 1) / kTile));
  if (grid.y > 65535) return cudaErrorInvalidConfiguration;
  switch (a.dtype) {
    case IM2WIN_F32: matmul_int8_kernel<float><<<grid, kThreads, 0, stream>>>(a, x, weight); break;
    case IM2WIN_F16: matmul_int8_kernel<__half><<<grid, kThreads, 0, stream>>>(a, x, weight); break;
    default: matmul_int8_kernel<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(a, x, weight); break;
  }
  return cudaGetLastError();
}

}  // namespace im2win
