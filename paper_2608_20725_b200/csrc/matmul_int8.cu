// Rows times a matrix in 8-bit integers on the tensor cores (im2win_matmul_int8):
//
//   y[m][n] = bias[n] + x_scales[m] scales[n] sum_k x[m][k] w[n][k],   sums in 32-bit integers (tcgen05.mma kind::i8).
//
// Tiles of 128 rows x BN columns, or, by a pair of CTAs (cta_group::2), of 256 x BN, each CTA with 128 rows of x and half of the matrix's rows.  One warp
// starts the copies (TMA, blocks of 128 bytes along K with the 128-byte swizzle, a ring of stages), one issues the products, eight turn finished
// sums into y while the next tile's run: two accumulators in tensor memory.  CTAs stay on their SM and take tile after tile.
#include <algorithm>

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "sequence.cuh"

namespace im2win {
namespace {

using namespace ptx;

constexpr int kRows = 128;               // of x, of a CTA's tile
constexpr int kBlock = 128;              // elements (bytes) along K of a copy
constexpr int kMaxStages = 12;
constexpr int kFinishers = 8;            // warps that make y
constexpr int kFirstFinisher = 4;
constexpr int kThreads = (kFirstFinisher + kFinishers) * 32;
constexpr int kGroup = 8;                // row tiles that are worked on together, so that what is read of x and the matrix stays in the L2 cache

struct MatmulParams {
  const float* x_scales;
  const float* scales;
  const float* bias;
  void* y;
  int64_t y_stride;
  int32_t M, N, blocks;                  // blocks: of K, of as many bytes as a stage has
  int32_t tiles_m, tiles_n;              // tiles_m: of the CTA or the pair
  int32_t x_rows, parts, stages;         // rows of x of a copy; 128-byte parts of a stage; stages
  int32_t vectors;                       // whether rows of y start on 16-byte boundaries
  uint32_t polls;                        // looks, of a microsecond at most, before a wait gives up
  int32_t drop;                          // testing aid: the first CTA (pair) does not say that the sums of this tile of its are done (-1: it does)
};

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

template <bool PAIR>
__device__ __forceinline__ void umma_i8(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  if constexpr (PAIR) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %5};\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kSmemDescHiSw128)
        : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %5};\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kSmemDescHiSw128)
        : "memory");
  }
}
// Signed 8-bit A and B, both along K, 32-bit integer sums, M x N tile.
__host__ __device__ constexpr uint32_t instr_desc_i8(int M, int N) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

template <typename T, int BN, bool PAIR>
struct Tile {
  static constexpr uint32_t kRingBytes = (sizeof(T) == 4 ? 184 : 200) * 1024;          // (beside what turns y)
  static constexpr int kMatrixRows = PAIR ? BN / 2 : BN;       // that a CTA stages
  static constexpr uint32_t kB = kMatrixRows * kBlock;
  static constexpr uint32_t kColumns = 2 * BN;                 // of tensor memory
};

// Tile number w as (tile of rows, tile of columns): row tiles by groups, within a group the columns outermost.
__device__ __forceinline__ void place(const MatmulParams& p, int64_t w, int& tm, int& tn) {
  const int64_t per = (int64_t)kGroup * p.tiles_n;
  const int group = (int)(w / per), first = group * kGroup, rows = min(kGroup, p.tiles_m - first);
  const int rest = (int)(w - group * per);
  tn = rest / rows;
  tm = first + rest % rows;
}

template <typename T, int BN, bool PAIR>
__device__ __forceinline__ void matmul_body(const CUtensorMap& x_map, const CUtensorMap& matrix_map, const MatmulParams& p) {
  using L = Tile<T, BN, PAIR>;
  extern __shared__ uint8_t dynamic_smem[];
  __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 4];   // stages full, empty; sums done, taken (two)
  __shared__ uint32_t tmem_base_at, gave_up;
  __shared__ __align__(16) float factors[kFinishers][2][32];   // scales and bias of a warp's columns
  __shared__ T turned[kFinishers][32][sizeof(T) == 4 ? 33 : 34];           // 32 x 32 of y on their way to rows that start anywhere
  const uint32_t ring = (smem_u32(dynamic_smem) + 1023u) & ~1023u;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const int64_t first = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  const uint32_t full = smem_u32(bars), empty = smem_u32(bars + kMaxStages), done = smem_u32(bars + 2 * kMaxStages),
                 taken = smem_u32(bars + 2 * kMaxStages + 2);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kMaxStages; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(done + 8 * i, 1);
      mbar_init(taken + 8 * i, (PAIR ? 2 : 1) * kFinishers);
    }
    gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) tmem_alloc_pair(smem_u32(&tmem_base_at), L::kColumns);
    else tmem_alloc(smem_u32(&tmem_base_at), L::kColumns);
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();                                // the peer's barriers exist before anything arrives on them
  tc_fence_after();
  const uint32_t tmem = tmem_base_at;
  // Waits are for copies, products and warps of the CTA or pair, which end by themselves.  Should one not within some four seconds, it gives up,
  // the others with it, and y is NaN from that tile on.
  bool failed = false;
  auto wait = [&](uint32_t bar, uint32_t parity) {             // (the whole warp, of one mind)
    uint32_t left = failed ? 0 : p.polls;
    bool there = false;
    while (left-- > 0) {
      there = __all_sync(0xffffffffu, try_wait_1us(bar, parity));
      if (there || ((left & 255u) == 0u && *(volatile uint32_t*)&gave_up)) break;
    }
    if (there) return true;
    failed = true;
    gave_up = 1;
    return false;
  };

  const uint32_t x_bytes = (uint32_t)p.x_rows * kBlock, part_bytes = x_bytes + L::kB, stage_bytes = p.parts * part_bytes;

  if (warp == 0) {
    const bool elected = elect_one();
    const uint32_t to_full = PAIR ? mapa_shared(full, 0) : full;             // the leader's
    int stage = 0;
    uint32_t phase = 1;                                        // (the first wait for an empty stage passes)
    for (int64_t w = first; w < tiles && !failed; w += step) {
      int tm, tn;
      place(p, w, tm, tn);
      const int m0 = (PAIR ? 2 * tm + (int)rank : tm) * kRows, n0 = tn * BN + (int)rank * L::kMatrixRows;
      for (int b = 0; b < p.blocks; ++b) {
        if (!wait(empty + 8 * stage, phase)) break;
        if (elected) {
          const uint32_t bar = to_full + 8 * stage;
          uint32_t to = ring + stage * stage_bytes;
          // (What lies beyond a matrix reads as 0 and counts; in a pair the leader announces the bytes of both.  Of few rows no more than those, eight at a
          // time, are copied; what the products find in the others' place makes sums that are not looked at.)
          if (rank == 0) mbar_arrive_expect_tx(full + 8 * stage, (PAIR ? 2u : 1u) * stage_bytes);
          for (int i = 0; i < p.parts; ++i, to += part_bytes) {
            const int k = (b * p.parts + i) * kBlock;
            if (PAIR) {
              tma_load_2d_pair(to, &x_map, k, m0, bar);
              tma_load_2d_pair(to + x_bytes, &matrix_map, k, n0, bar);
            } else {
              tma_load_2d(to, &x_map, k, m0, bar);
              tma_load_2d(to + x_bytes, &matrix_map, k, n0, bar);
            }
          }
        }
        __syncwarp();
        if (++stage == p.stages) stage = 0, phase ^= 1;
      }
    }
  } else if (warp == 1 && rank == 0) {
    constexpr uint32_t kDesc = instr_desc_i8(PAIR ? 2 * kRows : kRows, BN);
    const bool elected = elect_one();
    int stage = 0;
    uint32_t phase = 0, it = 0;
    for (int64_t w = first; w < tiles && !failed; w += step, ++it) {
      const uint32_t buffer = it & 1;
      if (!wait(taken + 8 * buffer, (it >> 1 & 1) ^ 1)) break;
      tc_fence_after();
      const uint32_t to = tmem + buffer * BN;
      for (int b = 0; b < p.blocks; ++b) {
        if (!wait(full + 8 * stage, phase)) break;
        if (elected) {
          uint32_t a = smem_desc_lo(ring + stage * stage_bytes);
          for (int i = 0; i < p.parts; ++i, a += part_bytes >> 4) {
            const uint32_t m = a + (x_bytes >> 4);
#pragma unroll
            for (int j = 0; j < kBlock / 32; ++j) umma_i8<PAIR>(to, a + 2 * j, m + 2 * j, kDesc, b > 0 || i > 0 || j > 0);
          }
          if (PAIR) umma_commit_pair(empty + 8 * stage);
          else umma_commit(empty + 8 * stage);
        }
        __syncwarp();
        if (++stage == p.stages) stage = 0, phase ^= 1;
      }
      if (!failed && elected && !(first == 0 && (int)it == p.drop)) {
        if (PAIR) umma_commit_pair(done + 8 * buffer);
        else umma_commit(done + 8 * buffer);
      }
      __syncwarp();
    }
  } else if (warp >= kFirstFinisher) {
    const int index = warp - kFirstFinisher;
    constexpr int kParts = BN >= 64 ? 2 : 1;                   // of the columns; otherwise the upper four warps have nothing to do
    const int row = (warp & 3) * 32 + lane, part = index >> 2;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;
    const uint32_t to_taken = PAIR ? mapa_shared(taken, 0) : taken;
    uint32_t it = 0;
    for (int64_t w = first; w < tiles; w += step, ++it) {
      int tm, tn;
      place(p, w, tm, tn);
      const uint32_t buffer = it & 1;
      const int m = (PAIR ? 2 * tm + (int)rank : tm) * kRows + row;
      const float x_scale = m < p.M ? p.x_scales[m] : 0.0f;
      wait(done + 8 * buffer, it >> 1 & 1);
      tc_fence_after();
      if (part < kParts) {
#pragma unroll 1
        for (int c = part * (BN / kParts); c < (part + 1) * (BN / kParts); c += 32) {
          const int n0 = tn * BN + c;
          if (n0 >= p.N) break;
          uint32_t sum[32];
          if (!failed) tmem_ld32_issue(tmem + lanes + buffer * BN + c, sum);
          __syncwarp();
          const bool there = n0 + lane < p.N;
          factors[index][0][lane] = there ? __ldg(p.scales + n0 + lane) : 0.0f;
          factors[index][1][lane] = there && p.bias ? __ldg(p.bias + n0 + lane) : 0.0f;
          __syncwarp();
          if (!failed) tmem_ld_wait_for(sum);
          if (m < p.M) {
            float v[32];
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              const float4 f = *reinterpret_cast<const float4*>(&factors[index][0][j]), a = *reinterpret_cast<const float4*>(&factors[index][1][j]);
              const float fs[4] = {f.x, f.y, f.z, f.w}, as[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                v[j + e] = __fmul_rn((float)(int32_t)sum[j + e] * x_scale, fs[e]);
                if (p.bias) v[j + e] += as[e];
                if (failed) v[j + e] = __builtin_nanf("");
              }
            }
            T* to = static_cast<T*>(p.y) + (int64_t)m * p.y_stride + n0;
            if (p.vectors && n0 + 32 <= p.N) {
              constexpr int V = 16 / sizeof(T);
#pragma unroll
              for (int j = 0; j < 32; j += V) {
                Vec<T, V> out;
#pragma unroll
                for (int e = 0; e < V; ++e) out.v[e] = from_float<T>(v[j + e]);
                *reinterpret_cast<Vec<T, V>*>(to + j) = out;
              }
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j) turned[index][lane][j] = from_float<T>(v[j]);
            }
          }
          if (!(p.vectors && n0 + 32 <= p.N)) {                // a row at a time
            __syncwarp();
            const int rows = min(32, p.M - (m - lane));
            T* to = static_cast<T*>(p.y) + (int64_t)(m - lane) * p.y_stride + n0 + lane;
            if (there)
              for (int r = 0; r < rows; ++r) to[(int64_t)r * p.y_stride] = turned[index][r][lane];
          }
          __syncwarp();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) mbar_arrive_cluster(to_taken + 8 * buffer);
        else mbar_arrive(taken + 8 * buffer);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*(volatile uint32_t*)&gave_up) {
    for (int i = 0; i < 64; ++i) __nanosleep(1000);            // copies and products under way end before the CTA does
    __syncthreads();
  }
  if (PAIR) cluster_sync_all();                                // no CTA leaves while its peer may still signal or read it
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem, L::kColumns);
    else tmem_dealloc(tmem, L::kColumns);
  }
}

template <typename T, int BN>
__global__ void __launch_bounds__(kThreads, 1)
matmul_int8_tiles_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap matrix_map, const MatmulParams p) {
  matmul_body<T, BN, false>(x_map, matrix_map, p);
}
template <typename T, int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
matmul_int8_pairs_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap matrix_map, const MatmulParams p) {
  matmul_body<T, BN, true>(x_map, matrix_map, p);
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

bool encode(EncodeTiledFn fn, CUtensorMap* map, const int8_t* at, int64_t rows, int64_t K, int64_t stride, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
  const cuuint32_t box[2] = {(cuuint32_t)kBlock, (cuuint32_t)box_rows}, one[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(at), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int BN, bool PAIR>
cudaError_t launch(const Int8Args& a, cudaStream_t stream) {
  using L = Tile<T, BN, PAIR>;
  constexpr uint32_t kBytes = L::kRingBytes + 1024;
  const im2win_int8_shape& s = a.shape;
  static bool attr_done[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  void (*kernel)(CUtensorMap, CUtensorMap, MatmulParams);
  if constexpr (PAIR) kernel = matmul_int8_pairs_kernel<T, BN>;
  else kernel = matmul_int8_tiles_kernel<T, BN>;
  if (!attr_done[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes);
    if (e != cudaSuccess) return e;
    attr_done[dev] = true;
  }
  const EncodeTiledFn fn = get_encode_fn();
  if (!fn) return cudaErrorNotSupported;
  CUtensorMap x_map, matrix_map;
  const int x_rows = s.M >= kRows ? kRows : (s.M + 7) / 8 * 8;
  if (!encode(fn, &x_map, a.x, s.M, s.K, s.x_stride, x_rows) || !encode(fn, &matrix_map, a.weight, s.N, s.K, s.K, L::kMatrixRows))
    return cudaErrorInvalidValue;
  const int rows = PAIR ? 2 * kRows : kRows;
  MatmulParams p = {a.x_scales, a.scales, a.bias, a.y, s.y_stride, s.M, s.N, 0, (int32_t)(((int64_t)s.M + rows - 1) / rows),
                    (int32_t)(((int64_t)s.N + BN - 1) / BN), x_rows, 1, 0, 0, 4000000u, -1};
  // A stage takes some 0.2 us whatever it holds (8 rows x 4096 x 4096: 10.4 us with 32 stages' worth, 7.8 with 8), so that small ones are put together, and the ring is to
  // hold four of them.  (Of few rows of x the products read on behind them: the last stage ends 16 KB before the ring does.)
  const uint32_t part = x_rows * kBlock + L::kB, most = L::kRingBytes - (kRows - x_rows) * kBlock;
  while (p.parts < 4 && 2 * p.parts * part <= most / 4 && p.parts * kBlock < s.K) p.parts *= 2;
  p.stages = std::min<int>(kMaxStages, most / (p.parts * part));
  p.blocks = (s.K + p.parts * kBlock - 1) / (p.parts * kBlock);
  p.vectors = aligned_to(a.y, 16) && s.y_stride * sizeof(T) % 16 == 0;
  if (const char* v = debug_getenv("IM2WIN_MATMUL_DROP")) {    // testing aid
    p.drop = atoi(v);
    p.polls = 4096;
  }
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  const unsigned grid = PAIR ? 2 * (unsigned)std::min<int64_t>(tiles, 74) : (unsigned)std::min<int64_t>(tiles, 148);
  kernel<<<grid, kThreads, kBytes, stream>>>(x_map, matrix_map, p);
  return cudaGetLastError();
}

// Tiles: pairs of CTAs where there are more rows than a CTA's; the columns of a tile by an estimate, the rounds of tiles times a tile's time, which goes
// by its columns and what it costs besides.
struct Choice {
  bool pair;
  int bn;
};
Choice choose(const im2win_int8_shape& s) {
  Choice best = {s.M > kRows, 0};
  int64_t least = 0;
  for (int bn : {256, 128, 64, 32}) {
    if (best.pair && bn < 64) break;
    const int64_t tiles = ((int64_t)s.M + (best.pair ? 255 : 127)) / (best.pair ? 256 : 128) * (((int64_t)s.N + bn - 1) / bn);
    const int64_t slots = best.pair ? 74 : 148, cost = (tiles + slots - 1) / slots * (bn + 32);
    if (!best.bn || cost < least) best.bn = bn, least = cost;
  }
  return best;
}

template <typename T>
cudaError_t launch_type(const Int8Args& a, cudaStream_t stream) {
  const Choice c = choose(a.shape);
  if (c.pair) {
    if (c.bn == 256) return launch<T, 256, true>(a, stream);
    if (c.bn == 128) return launch<T, 128, true>(a, stream);
    return launch<T, 64, true>(a, stream);
  }
  if (c.bn == 256) return launch<T, 256, false>(a, stream);
  if (c.bn == 128) return launch<T, 128, false>(a, stream);
  if (c.bn == 64) return launch<T, 64, false>(a, stream);
  return launch<T, 32, false>(a, stream);
}

}  // namespace

bool matmul_int8_by_tiles(const im2win_int8_shape& s) { return s.K % 16 == 0 && s.x_stride % 16 == 0; }

cudaError_t launch_matmul_int8_tiles(const Int8Args& a, cudaStream_t stream) {
  switch (a.dtype) {
    case IM2WIN_F32: return launch_type<float>(a, stream);
    case IM2WIN_F16: return launch_type<__half>(a, stream);
    default: return launch_type<__nv_bfloat16>(a, stream);
  }
}

}  // namespace im2win
