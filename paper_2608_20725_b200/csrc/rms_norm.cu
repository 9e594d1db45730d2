// Root-mean-square norm of rows behind the addition of a residual, into their type or into 8 bits (im2win_rms_norm):
//
//   h = x + residual (rounded),   y = h w / sqrt(mean(h^2) + eps),   or   y = nearest(127 h w / top), scale = top / (127 sqrt(..)),
//
// with top the largest |h w| of the row.  A row is read once: its threads keep h in registers from the sum of squares to y.  Rows that
// no block's registers hold (above 32768 elements of 16 bits, 16384 of 32 or where rows do not lie on vectors) are read again.
//
// In 8 bits the root drops out of which number is nearest: h w of 16-bit elements is exact in fp32, of fp32 ones in 64 bits, and its
// quotient by the row's largest is looked at in fp32 first; where that comes within 1e-4 of halfway between two numbers, n and n + 1 (of its 127 it is
// off by up to 127 * 3 * 2^-24 = 2.3e-5), the sign of 254 h w - (2 n + 1) top decides, exactly.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "sequence.cuh"

namespace im2win {
namespace {

constexpr float kSmall = 0x1p-100f;      // of eps, and of the mean of squares

struct NormParams {
  const void* x;
  const void* residual;
  const void* weight;
  void* residual_out;
  void* y;
  float* scales;
  int64_t x_stride, residual_stride, residual_out_stride, y_stride;
  int32_t rows, channels;
  float eps;
};

// 127 z / top, which lies within n .. n + 1 (but for what tells halves from one another), rounded to the nearest whole number, ties to the even one: by the
// sign of 254 |z| - (2 n + 1) top.  z and top are products of two elements, exact in 64 bits; what they are multiplied by here brings fp32 ones to 56 bits.
template <typename T>
__device__ __forceinline__ int nearest_of(double z, double top, float n) {
  const double size = fabs(z), odd = 2.0f * n + 1.0f, a = __dmul_rn(254.0, size), b = __dmul_rn(odd, top);
  double d = a - b;
  if constexpr (sizeof(T) == 4) d += fma(254.0, size, -a) - fma(odd, top, -b);           // (a and b all but agree: both differences are exact)
  const float r = d > 0.0 ? n + 1.0f : d < 0.0 ? n : 2.0f * rintf(0.5f * (n + 0.5f));
  return z < 0.0 ? -(int)r : (int)r;
}
template <typename T>
__device__ __forceinline__ int nearest(float product, float per_top, float h, float w, double top) {
  const float t = product * per_top;
  const float r = rintf(t);
  if (fabsf(t - r) < 0.4999f) return (int)r;
  return nearest_of<T>((double)h * (double)w, top, floorf(fabsf(t)));
}
template <typename T>
__device__ __forceinline__ int nearest_in_64(double z, double top) {
  const double t = z * 127.0 / top, r = rint(t);
  return fabs(t - r) < 0.4999 ? (int)r : nearest_of<T>(z, top, (float)floor(fabs(t)));
}

// WARP: a row is a warp's (a block has four), otherwise all of the block's.  V: elements of a vector; N vectors a thread, or (N == 0) any
// number, read twice.  BYTES: y in 8 bits, a kernel of its own for its registers.  (16384 rows of 4096 bf16 with a residual, 84 us at 6.4 TB/s, took 127 with
// both in one kernel and the residual's loads behind a question each.)  SMALL: eps is so small that rows may be too, which is looked at; asking costs
// 131072 rows of 128 a tenth of their time, which is instructions.
template <typename T, int V, int N, bool WARP, bool BYTES, bool SMALL>
__global__ void __launch_bounds__(WARP ? 128 : 1024) rms_norm_kernel(const NormParams p) {
  using VT = Vec<T, V>;
  using VB = Vec<int8_t, V>;
  __shared__ float shared_sum[32], shared_top[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = WARP ? (int64_t)blockIdx.x * 4 + warp : (int64_t)blockIdx.x;
  if (row >= p.rows) return;                                   // (a whole warp, or nobody)
  const int tid = WARP ? lane : (int)threadIdx.x, threads = WARP ? 32 : (int)blockDim.x;
  const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
  const T* residual = p.residual ? static_cast<const T*>(p.residual) + row * p.residual_stride : nullptr;
  T* out = p.residual_out ? static_cast<T*>(p.residual_out) + row * p.residual_out_stride : nullptr;
  const T* weight = static_cast<const T*>(p.weight);
  const int vectors = p.channels / V;                          // (V divides the channels)

  auto at = [&](const T* from, int i) { return *reinterpret_cast<const VT*>(from + (int64_t)i * V); };
  auto add = [&](VT& h, const VT& r) {
#pragma unroll
    for (int j = 0; j < V; ++j) h.v[j] = from_float<T>(to_float(h.v[j]) + to_float(r.v[j]));
  };
  auto load = [&](int i) {
    VT h = at(x, i);
    if (residual) add(h, at(residual, i));
    return h;
  };
  auto weights = [&](int i) {
    VT w;
    if (weight) {
      w = *reinterpret_cast<const VT*>(weight + (int64_t)i * V);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) w.v[j] = from_float<T>(1.0f);
    }
    return w;
  };
  float sum = 0.0f, top = 0.0f;
  auto look = [&](const VT& h, int i) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum = fmaf(to_float(h.v[j]), to_float(h.v[j]), sum);
    if (BYTES) {
      const VT w = weights(i);
#pragma unroll
      for (int j = 0; j < V; ++j) top = max_nan(top, fabsf(to_float(h.v[j]) * to_float(w.v[j])));
    }
  };
  VT kept[N > 0 ? N : 1], first;
  if constexpr (N == 1 && WARP && !BYTES) {                      // (short rows: their weights before the sums)
    if (tid < vectors) first = weights(tid);
  }
  if constexpr (N > 0) {
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (tid + n * threads < vectors) kept[n] = at(x, tid + n * threads);
    if (residual) {
      VT more[N];                                              // (all loads under way before the first sum)
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (tid + n * threads < vectors) more[n] = at(residual, tid + n * threads);
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (tid + n * threads < vectors) {
          add(kept[n], more[n]);
          if (out) *reinterpret_cast<VT*>(out + (int64_t)(tid + n * threads) * V) = kept[n];
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (tid + n * threads < vectors) look(kept[n], tid + n * threads);
  } else {
    for (int i = tid; i < vectors; i += threads) {
      const VT h = load(i);
      if (out) *reinterpret_cast<VT*>(out + (int64_t)i * V) = h;
      look(h, i);
    }
  }
#pragma unroll
  for (int s = 16; s > 0; s /= 2) {
    sum += __shfl_xor_sync(0xffffffffu, sum, s);
    top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, s));
  }
  if constexpr (!WARP) {
    if (lane == 0) {
      shared_sum[warp] = sum;
      shared_top[warp] = top;
    }
    __syncthreads();
    const bool there = lane < threads / 32;
    sum = there ? shared_sum[lane] : 0.0f;
    top = there ? shared_top[lane] : 0.0f;
#pragma unroll
    for (int s = 16; s > 0; s /= 2) {
      sum += __shfl_xor_sync(0xffffffffu, sum, s);
      top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, s));
    }
  }
  auto each = [&](auto&& work) {                                 // work(h, its number) of all of the thread's vectors
    if constexpr (N > 0) {
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (tid + n * threads < vectors) work(kept[n], tid + n * threads);
    } else {
      for (int i = tid; i < vectors; i += threads) work(out ? *reinterpret_cast<const VT*>(out + (int64_t)i * V) : load(i), i);
    }
  };
  // Squares that fp32 may not hold, in a mean that eps does not lift: those of h times 2^96 are summed instead, and the rate is that of h times 2^96.  (Down
  // to 2^-100 what is lost of a square is below 2^-49 of the mean.)  Rows of zeros without eps have a rate of 0.
  constexpr float kUp = 0x1p96f;
  const float mean = sum / (float)p.channels + p.eps;
  const bool small = SMALL && mean < kSmall;                     // (the same for all threads of the row)
  auto raised_rate = [&]() {
    float sum = 0.0f;
    each([&](const VT& h, int) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float a = to_float(h.v[j]) * kUp;
        sum = fmaf(a, a, sum);
      }
    });
#pragma unroll
    for (int s = 16; s > 0; s /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    if constexpr (!WARP) {
      __syncthreads();
      if (lane == 0) shared_sum[warp] = sum;
      __syncthreads();
      sum = lane < threads / 32 ? shared_sum[lane] : 0.0f;
#pragma unroll
      for (int s = 16; s > 0; s /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    }
    const float raised = sum / (float)p.channels + p.eps * kUp * kUp;
    return raised > 0.0f ? rsqrtf(raised) : 0.0f;
  };

  if constexpr (!BYTES) {
    T* y = static_cast<T*>(p.y) + row * p.y_stride;
    float up = 1.0f, rate;
    if (small) up = kUp, rate = raised_rate();
    else rate = rsqrtf(mean);
    each([&](const VT& h, int i) {
      const VT w = N == 1 && WARP ? first : weights(i);
      VT r;
#pragma unroll
      for (int j = 0; j < V; ++j) r.v[j] = from_float<T>((SMALL ? to_float(h.v[j]) * up : to_float(h.v[j])) * rate * to_float(w.v[j]));
      *reinterpret_cast<VT*>(y + (int64_t)i * V) = r;
    });
    return;
  } else {
    const bool fine = top <= FLT_MAX;                            // (not of a NaN)
    // fp32: the largest product in 64 bits, and all below 2^-90: products that fp32 does not hold exactly
    const bool in_64 = sizeof(T) == 4 || top < 8e-28f;
    double exact_top = top;
    if (fine && in_64) {                                         // (the same for all threads of the row)
      double most = 0.0;
      each([&](const VT& h, int i) {
        const VT w = weights(i);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float a = to_float(h.v[j]), b = to_float(w.v[j]);
          if (fabsf(a * b) == top) most = fmax(most, fabs((double)a * (double)b));
        }
      });
#pragma unroll
      for (int s = 16; s > 0; s /= 2) most = fmax(most, __shfl_xor_sync(0xffffffffu, most, s));
      if constexpr (!WARP) {
        __shared__ double shared_most[32];
        if (lane == 0) shared_most[warp] = most;
        __syncthreads();
        most = lane < threads / 32 ? shared_most[lane] : 0.0;
#pragma unroll
        for (int s = 16; s > 0; s /= 2) most = fmax(most, __shfl_xor_sync(0xffffffffu, most, s));
      }
      exact_top = most;
    }
    const float raised = small ? raised_rate() : 0.0f;
    if (tid == 0) p.scales[row] = !fine ? __int_as_float(0x7fffffff) : small ? (float)(exact_top * (double)kUp) * raised / 127.0f : top * rsqrtf(mean) / 127.0f;
    int8_t* y = static_cast<int8_t*>(p.y) + row * p.y_stride;
    const bool zero = !fine || exact_top == 0.0;
    const float per_top = zero ? 0.0f : 127.0f / top;
    auto finish = [&](const VT& h, int i, auto tiny) {
      const VT w = weights(i);
      VB r;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float a = to_float(h.v[j]), b = to_float(w.v[j]);
        if constexpr (tiny.value) r.v[j] = zero ? 0 : (int8_t)nearest_in_64<T>((double)a * (double)b, exact_top);
        else r.v[j] = (int8_t)nearest<T>(a * b, per_top, a, b, exact_top);
      }
      *reinterpret_cast<VB*>(y + (int64_t)i * V) = r;
    };
    if (zero || top < 8e-28f) each([&](const VT& h, int i) { finish(h, i, std::true_type{}); });         // (products lose bits, and 127 / top is out of range)
    else each([&](const VT& h, int i) { finish(h, i, std::false_type{}); });
  }
}

// Rows of up to 1024 elements (128 where they do not lie on vectors) are a warp's; others a block's of as many threads as make four
// vectors each or fewer, and one each where there are few rows and a row's time is its latency.
template <typename T, int V, bool BYTES, bool SMALL>
cudaError_t launch(const NormParams& p, cudaStream_t stream) {
  constexpr int kMost = V > 1 ? 4 : 16;
  const int64_t vectors = p.channels / V;
  if (vectors <= 128) {
    const unsigned grid = (unsigned)(((int64_t)p.rows + 3) / 4);
    if (vectors <= 32)
      rms_norm_kernel<T, V, 1, true, BYTES, SMALL><<<grid, 128, 0, stream>>>(p);
    else
      rms_norm_kernel<T, V, 4, true, BYTES, SMALL><<<grid, 128, 0, stream>>>(p);
    return cudaGetLastError();
  }
  const bool few = p.rows <= 592;
  auto threads_for = [&](int each) { return (int)((vectors + each * 32 - 1) / (each * 32) * 32); };
  if (few && vectors <= 1024)
    rms_norm_kernel<T, V, 1, false, BYTES, SMALL><<<p.rows, threads_for(1), 0, stream>>>(p);
  else if (vectors <= 512)
    rms_norm_kernel<T, V, 2, false, BYTES, SMALL><<<p.rows, threads_for(2), 0, stream>>>(p);
  else if (vectors <= 1024 * 4)
    rms_norm_kernel<T, V, 4, false, BYTES, SMALL><<<p.rows, std::min(threads_for(4), 1024), 0, stream>>>(p);
  else if (V == 1 && vectors <= 1024 * kMost)
    rms_norm_kernel<T, V, kMost, false, BYTES, SMALL><<<p.rows, threads_for(kMost), 0, stream>>>(p);
  else
    rms_norm_kernel<T, V, 0, false, BYTES, SMALL><<<p.rows, 1024, 0, stream>>>(p);
  return cudaGetLastError();
}

template <typename T, int V>
cudaError_t launch_kind(const NormParams& p, cudaStream_t stream) {
  if (p.eps < kSmall) return p.scales ? launch<T, V, true, true>(p, stream) : launch<T, V, false, true>(p, stream);
  return p.scales ? launch<T, V, true, false>(p, stream) : launch<T, V, false, false>(p, stream);
}

template <typename T>
cudaError_t launch_type(const NormParams& p, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  auto rows_on = [&](const void* at, int64_t stride, int64_t size) { return !at || (aligned_to(at, V * size) && stride % V == 0); };
  if (p.channels % V == 0 && rows_on(p.x, p.x_stride, sizeof(T)) && rows_on(p.residual, p.residual_stride, sizeof(T)) &&
      rows_on(p.residual_out, p.residual_out_stride, sizeof(T)) && rows_on(p.weight, 0, sizeof(T)) &&
      rows_on(p.y, p.y_stride, p.scales ? 1 : sizeof(T)))
    return launch_kind<T, V>(p, stream);
  return launch_kind<T, 1>(p, stream);
}

}  // namespace

cudaError_t launch_rms_norm(const void* x, const void* residual, const void* weight, void* residual_out, void* y, float* scales,
                            const im2win_norm_shape& s, im2win_dtype dtype, cudaStream_t stream) {
  const NormParams p = {x, residual, weight, residual_out, y, scales, s.x_stride, s.residual_stride, s.residual_out_stride, s.y_stride,
                        s.rows, s.channels, s.eps};
  switch (dtype) {
    case IM2WIN_F32: return launch_type<float>(p, stream);
    case IM2WIN_F16: return launch_type<__half>(p, stream);
    default: return launch_type<__nv_bfloat16>(p, stream);
  }
}

}  // namespace im2win
