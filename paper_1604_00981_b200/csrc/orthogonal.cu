// The orthogonalised update (declared in include/sgdb.h): Newton-Schulz products of a matrix,
// alone and as the rule of a whole server iteration.
//
//   X <- U / (|U|_F + eps), then `steps` times, over the shorter side:
//     A = X X^T,  B = a I + b A + c A^2,  X <- B X        (tall: A = X^T X, X <- X B)
//
// Each product is one launch of product_kernel: tcgen05 matrix instructions on fp16 operands with fp32
// accumulators in tensor memory.  X, A and B are kept as fp16 times kScale: the largest singular
// value of X is at most about 1.2, so every element is far below fp16's largest number, and elements
// down to 2^-22 keep all 11 bits of their significand, three more than bf16 has.  The rounding of
// X, A and B adds a relative error of about 1.3e-3 to the result after five steps (bf16 operands: 1e-2).
// A and B are symmetric: only tiles that touch the upper triangle are computed, and stored twice.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>

#include "sgdb_host.cuh"
#include "sgdb_rows.cuh"
#include "sgdb_tensor.cuh"

namespace sgdb {
namespace {

constexpr float kScale = 256.0f;
constexpr int kTileM = 128;
constexpr int kTileK = 64;              // 128 bytes of fp16: one swizzled row of shared memory
constexpr int kBoxBytes = 64 * 64 * 2;  // every copy is a box of 64 x 64 elements
constexpr int kNormBlocks = 64;         // partial sums of squares per matrix
constexpr unsigned long long kPatienceNs = kWaitLimitNs;

enum : int { OUT_GRAM = 0, OUT_POLY = 1, OUT_APPLY = 2, OUT_FINAL = 3, OUT_THETA = 4 };

struct ProductParams {
  int M, N, K, batch;
  int a_mn, b_mn;  // 1: the operand's rows run along K in memory (k is the slow index)
  int tiles_m, tiles_n, tiles;  // per matrix; `tiles` counts those that are computed
  __half* out;                  // GRAM, POLY, APPLY: fp16 times kScale
  const __half* addend;         // POLY: A
  long long ld, stride;         // of out (and addend), elements
  float ca, cb, cc;             // POLY: a, b, c
  void* final_out;              // FINAL: dt_out; THETA: fp32 parameters
  int dt_out;
  long long ld_final, stride_final;
  float keep, rate;  // THETA: theta <- keep theta - rate O
  int32_t* info;     // optional: [1] != SGDB_OK: do nothing; receives SGDB_ERR_TIMEOUT
};

template <int TN>
struct Shape {
  static constexpr int kBoxesA = kTileM / 64, kBoxesB = TN / 64;
  static constexpr int kStageBytes = (kBoxesA + kBoxesB) * kBoxBytes;
  static constexpr int kStages = TN == 256 ? 4 : 6;
  static constexpr int kStaging = 4 * 32 * 33 * 4;  // one 32 x 33 fp32 block per epilogue warp
  static constexpr int kSmem = kStages * kStageBytes + kStaging + 1024;
  static constexpr int kTmemColumns = 2 * TN;
};

// Row and column tile of the i-th computed tile of a matrix.
template <int TN, bool SYM>
__device__ __forceinline__ void tile_at(const ProductParams& p, int i, int* tm, int* tn) {
  if (!SYM) {
    *tm = i / p.tiles_n;
    *tn = i % p.tiles_n;
    return;
  }
  int row = 0, first = 0;
  while (true) {
    first = row * kTileM / TN;  // the first column tile that reaches the diagonal
    const int n = p.tiles_n - first;
    if (i < n) break;
    i -= n;
    ++row;
  }
  *tm = row;
  *tn = first + i;
}

// One product.  Warp 0 issues the copies of 64-wide slices of both operands into a ring, warp 1 the matrix
// instructions, warps 2..5 read the finished tile from tensor memory while the next one is computed.
template <int TN, int OUT>
__global__ void __launch_bounds__(192, 1)
    product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const ProductParams p) {
  using S = Shape<TN>;
  constexpr bool kSym = OUT == OUT_GRAM || OUT == OUT_POLY;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  float* staging = reinterpret_cast<float*>(smem + S::kStages * S::kStageBytes);
  __shared__ __align__(8) uint64_t s_full[S::kStages], s_empty[S::kStages], s_done[2], s_free[2], s_end;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(smem_addr(&s_full[i]), 1);
      mbar_init(smem_addr(&s_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&s_done[i]), 1);
      mbar_init(smem_addr(&s_free[i]), 4);
    }
    mbar_init(smem_addr(&s_end), 1);
    s_abort = 0;
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc(smem_addr(&s_tmem), S::kTmemColumns);
  tcgen05_before_sync();
  __syncthreads();
  tcgen05_after_sync();
  const uint32_t tmem = s_tmem;
  pdl_launch_dependents();
  pdl_wait();
  const bool idle = p.info != nullptr && p.info[1] != SGDB_OK;
  const int total = idle ? 0 : p.tiles * p.batch;
  const int k_blocks = (p.K + kTileK - 1) / kTileK;

  if (warp == 0 && lane == 0) {
    fence_proxy_async();
    uint32_t it = 0;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < total; tile += gridDim.x) {
      int tm, tn;
      const int z = tile / p.tiles;
      tile_at<TN, kSym>(p, tile % p.tiles, &tm, &tn);
      for (int kb = 0; kb < k_blocks; ++kb, ++it) {
        const uint32_t stage = it % S::kStages, round = it / S::kStages;
        if (!mbar_wait_for(smem_addr(&s_empty[stage]), (round & 1) ^ 1, &s_abort, kPatienceNs)) {
          ok = false;
          break;
        }
        const uint32_t bar = smem_addr(&s_full[stage]);
        mbar_arrive_expect_tx(bar, S::kStageBytes);
        uint32_t dst = smem_addr(smem + stage * S::kStageBytes);
#pragma unroll
        for (int b = 0; b < S::kBoxesA + S::kBoxesB; ++b, dst += kBoxBytes) {
          const bool is_a = b < S::kBoxesA;
          const int mn = is_a ? tm * kTileM + b * 64 : tn * TN + (b - S::kBoxesA) * 64;
          const bool slow_k = is_a ? p.a_mn : p.b_mn;
          tma_load_3d(dst, is_a ? &map_a : &map_b, slow_k ? mn : kb * kTileK, slow_k ? kb * kTileK : mn, z, bar);
        }
      }
    }
    // nothing may be in flight when the block ends: the last slots are consumed or, after a wait that ran out, at least filled
    for (uint32_t i = it > S::kStages ? it - S::kStages : 0; i < it; ++i) {
      int ignore = 0;
      uint64_t* bar = ok ? &s_empty[i % S::kStages] : &s_full[i % S::kStages];
      (void)mbar_wait_for(smem_addr(bar), (i / S::kStages) & 1, &ignore, kPatienceNs);
    }
  } else if (warp == 1 && lane == 0) {
    const uint32_t idesc = mma_descriptor_f16(kTileM, TN, p.a_mn, p.b_mn);
    const uint64_t desc_a = smem_descriptor(p.a_mn), desc_b = smem_descriptor(p.b_mn);
    const uint32_t step_a = p.a_mn ? 2048 : 32, step_b = p.b_mn ? 2048 : 32;  // bytes from one K of 16 to the next
    uint32_t it = 0, count = 0;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < total; tile += gridDim.x, ++count) {
      const uint32_t buf = count & 1;
      if (!mbar_wait_for(smem_addr(&s_free[buf]), ((count >> 1) & 1) ^ 1, &s_abort, kPatienceNs)) {
        ok = false;
        break;
      }
      tcgen05_after_sync();
      for (int kb = 0; kb < k_blocks; ++kb, ++it) {
        const uint32_t stage = it % S::kStages;
        if (!mbar_wait_for(smem_addr(&s_full[stage]), (it / S::kStages) & 1, &s_abort, kPatienceNs)) {
          ok = false;
          break;
        }
        tcgen05_after_sync();
        const uint32_t at = smem_addr(smem + stage * S::kStageBytes);
#pragma unroll
        for (int k = 0; k < kTileK / 16; ++k)
          mma_f16(tmem + buf * TN, desc_a + ((at + k * step_a) >> 4), desc_b + ((at + S::kBoxesA * kBoxBytes + k * step_b) >> 4),
                  idesc, (kb | k) != 0);
        mma_commit(smem_addr(&s_empty[stage]));
      }
      if (ok) mma_commit(smem_addr(&s_done[buf]));
    }
    if (!ok) {  // the instructions issued so far end before tensor memory is given back
      int ignore = 0;
      mma_commit(smem_addr(&s_end));
      (void)mbar_wait_for(smem_addr(&s_end), 0, &ignore, kPatienceNs);
    }
  } else if (warp >= 2) {
    const int quarter = warp & 3;  // the lanes of tensor memory that this warp may read
    float(*block)[33] = reinterpret_cast<float(*)[33]>(staging + quarter * 32 * 33);
    uint32_t count = 0;
    for (int tile = blockIdx.x; tile < total; tile += gridDim.x, ++count) {
      const uint32_t buf = count & 1;
      int tm, tn;
      const long long z = tile / p.tiles;
      tile_at<TN, kSym>(p, tile % p.tiles, &tm, &tn);
      if (!mbar_wait_for(smem_addr(&s_done[buf]), (count >> 1) & 1, &s_abort, kPatienceNs)) break;
      tcgen05_after_sync();
      const int row0 = tm * kTileM + quarter * 32;
      for (int c0 = 0; c0 < TN; c0 += 32) {
        const int col0 = tn * TN + c0;
        if (col0 >= p.N || row0 >= p.M || (kSym && col0 + 31 < row0)) continue;
        float acc[32];
        tmem_load32(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + buf * TN + c0, acc);
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 32; ++c) block[lane][c] = acc[c];
        __syncwarp();
        const int col = col0 + lane;
        for (int r = 0; r < 32; ++r) {
          const int row = row0 + r;
          if (row >= p.M) break;
          if (col >= p.N || (kSym && col < row)) continue;
          float v = block[r][lane];
          if (OUT == OUT_FINAL) {
            store_any(p.final_out, p.dt_out, z * p.stride_final + row * p.ld_final + col, v * (1.0f / (kScale * kScale)));
          } else if (OUT == OUT_THETA) {
            float* theta = static_cast<float*>(p.final_out) + z * p.stride_final + row * p.ld_final + col;
            *theta = fmaf(-p.rate, v * (1.0f / (kScale * kScale)), p.keep * *theta);
          } else {
            v *= 1.0f / kScale;
            const long long at = z * p.stride + row * p.ld + col;
            if (OUT == OUT_POLY) {
              v = fmaf(p.cc, v, p.cb * __half2float(p.addend[at]));
              if (row == col) v += p.ca * kScale;
              if (kSym) block[r][lane] = v;
            } else if (kSym) {
              block[r][lane] = v;
            }
            p.out[at] = __float2half_rn(v);
          }
        }
        if (kSym) {  // the mirror image: lanes along the rows
          __syncwarp();
          const int row = row0 + lane;
          for (int c = 0; c < 32 && col0 + c < p.N; ++c)
            if (row < col0 + c && row < p.M)
              p.out[z * p.stride + (col0 + c) * p.ld + row] = __float2half_rn(block[lane][c]);
        }
      }
      tcgen05_before_sync();
      if (lane == 0) mbar_arrive(smem_addr(&s_free[buf]));
    }
  }
  __syncwarp();
  tcgen05_before_sync();
  __syncthreads();
  tcgen05_after_sync();
  if (threadIdx.x == 0 && s_abort != 0 && p.info != nullptr) p.info[1] = SGDB_ERR_TIMEOUT;
  if (warp == 1) tmem_dealloc(tmem, S::kTmemColumns);
}

// ---------------------------------------------------------------- before the products

struct NormParams {
  const void* u;  // dt_in
  int dt_in;
  int rows, cols;
  long long ld, stride;
  float *velocity, *combined;  // step: fp32 momentum in/out, and where u = g + mu m goes; u holds the mean g
  float mu;
  int nesterov;
  double* partials;  // [batch][kNormBlocks]
  __half* x;
  long long ldx, stride_x;
  float eps;
  const int32_t* info;
};

// Partial sums of squares of each matrix, in 64 bits: the square of an fp32 number may be out of fp32's range.
__global__ void __launch_bounds__(256) square_sum_kernel(const NormParams p) {
  pdl_launch_dependents();
  pdl_wait();
  if (p.info != nullptr && p.info[1] != SGDB_OK) return;
  __shared__ double s[8];
  double sum = 0.0;
  const long long z = blockIdx.y, n = static_cast<long long>(p.rows) * p.cols;
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < n; i += kNormBlocks * 256) {
    float v;
    if (p.velocity != nullptr) {
      const long long at = z * n + i;
      const float g = static_cast<const float*>(p.u)[at];
      const float m = fmaf(p.mu, p.velocity[at], g);
      v = p.nesterov ? fmaf(p.mu, m, g) : m;
      p.velocity[at] = m;
      p.combined[at] = v;
    } else {
      v = load_any(p.u, p.dt_in, z * p.stride + i / p.cols * p.ld + i % p.cols);
    }
    sum += static_cast<double>(v) * v;
  }
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int w = 0; w < 8; ++w) sum += s[w];
    p.partials[z * kNormBlocks + blockIdx.x] = sum;
  }
}

// X = kScale U / (|U| + eps) in fp16.
__global__ void __launch_bounds__(256) normalise_kernel(const NormParams p) {
  pdl_launch_dependents();
  pdl_wait();
  if (p.info != nullptr && p.info[1] != SGDB_OK) return;
  const long long z = blockIdx.y, n = static_cast<long long>(p.rows) * p.cols;
  double sum = 0.0;
  for (int b = 0; b < kNormBlocks; ++b) sum += p.partials[z * kNormBlocks + b];
  const double factor = static_cast<double>(kScale) / (sqrt(sum) + static_cast<double>(p.eps));
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<long long>(gridDim.x) * 256) {
    const long long row = i / p.cols, col = i % p.cols;
    const float v = p.velocity != nullptr ? p.combined[z * n + i] : load_any(p.u, p.dt_in, z * p.stride + row * p.ld + col);
    p.x[z * p.stride_x + row * p.ldx + col] = __float2half_rn(static_cast<float>(v * factor));
  }
}

// ---------------------------------------------------------------- host side

long long round_up(long long n, long long to) { return (n + to - 1) / to * to; }

struct Plan {
  int batch, rows, cols, side;  // side: the shorter one
  long long ldx, stride_x, lds, stride_s;
  size_t x0, x1, a, b, partials, mean, total;  // byte offsets in the workspace
};

bool make_plan(int32_t batch, int64_t rows, int64_t cols, bool step, Plan* q) {
  if (batch < 0 || batch > SGDB_MAX_MATRICES || rows < 1 || cols < 1 || rows > SGDB_MAX_SIDE || cols > SGDB_MAX_SIDE) return false;
  if (((rows + 63) / 64) * ((cols + 63) / 64) * batch > 0x3fffffff) return false;  // tiles are counted in 32 bits
  q->batch = batch;
  q->rows = static_cast<int>(rows);
  q->cols = static_cast<int>(cols);
  q->side = q->rows < q->cols ? q->rows : q->cols;
  q->ldx = round_up(cols, 8);
  q->stride_x = q->ldx * rows;
  q->lds = round_up(q->side, 8);
  q->stride_s = q->lds * q->side;
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at = static_cast<size_t>(round_up(static_cast<long long>(at + bytes), 256));
    return here;
  };
  const size_t n = static_cast<size_t>(batch);
  q->x0 = take(n * q->stride_x * 2);
  q->x1 = take(n * q->stride_x * 2);
  q->a = take(n * q->stride_s * 2);
  q->b = take(n * q->stride_s * 2);
  q->partials = take(n * kNormBlocks * sizeof(double));
  q->mean = at;
  if (step) take(n * static_cast<size_t>(rows) * static_cast<size_t>(cols) * sizeof(float));
  q->total = at + 256;  // room to start on a multiple of 256 bytes
  return true;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

// Boxes of 64 x 64 of `batch` fp16 matrices [rows x cols], 128-byte swizzle, zeros outside.
sgdb_status_t make_map(CUtensorMap* map, void* base, int rows, int cols, long long ld, long long stride, int batch) {
  const EncodeTiled encode = encode_tiled();
  if (encode == nullptr) return SGDB_ERR_CUDA;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(batch)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(stride) * 2};
  const cuuint32_t box[3] = {64, 64, 1}, unit[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, base, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SGDB_OK : SGDB_ERR_CUDA;
}

template <typename... Args, typename... Given>
sgdb_status_t launch_dependent(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, cudaStream_t s, Given... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<Args>(args)...);
  return launch_status();
}

template <int TN, int OUT>
sgdb_status_t launch_product_t(const CUtensorMap& a, const CUtensorMap& b, ProductParams p, const DeviceInfo* dev, cudaStream_t s) {
  constexpr bool kSym = OUT == OUT_GRAM || OUT == OUT_POLY;
  p.tiles_m = (p.M + kTileM - 1) / kTileM;
  p.tiles_n = (p.N + TN - 1) / TN;
  p.tiles = 0;
  for (int i = 0; i < p.tiles_m; ++i) p.tiles += p.tiles_n - (kSym ? i * kTileM / TN : 0);
  const long long total = static_cast<long long>(p.tiles) * p.batch;
  auto kernel = product_kernel<TN, OUT>;
  static std::atomic<bool> allowed[kMaxDevices];
  if (!allowed[dev->index].load(std::memory_order_relaxed)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<TN>::kSmem) != cudaSuccess)
      return launch_status();
    allowed[dev->index].store(true, std::memory_order_relaxed);
  }
  const unsigned grid = static_cast<unsigned>(total < dev->sms ? total : dev->sms);
  return launch_dependent(kernel, dim3(grid), 192, Shape<TN>::kSmem, s, a, b, p);
}

template <int OUT>
sgdb_status_t launch_product(const CUtensorMap& a, const CUtensorMap& b, const ProductParams& p, const DeviceInfo* dev, cudaStream_t s) {
  return launch_product_t<128, OUT>(a, b, p, dev, s);
}

bool rule_ok(const sgdb_newton_schulz_t* ns) {
  return ns != nullptr && ns->steps >= 1 && ns->steps <= SGDB_MAX_STEPS && std::isfinite(ns->a) && std::isfinite(ns->b) &&
         std::isfinite(ns->c) && ns->eps >= 0.0f && !std::isinf(ns->eps);
}

// X is in place (q.x0): the products, and what is done with the last one.
sgdb_status_t run_products(const Plan& q, const sgdb_newton_schulz_t& ns, char* ws, int last, ProductParams final_params,
                           int32_t* info, const DeviceInfo* dev, cudaStream_t s) {
  __half* x[2] = {reinterpret_cast<__half*>(ws + q.x0), reinterpret_cast<__half*>(ws + q.x1)};
  __half *a = reinterpret_cast<__half*>(ws + q.a), *b = reinterpret_cast<__half*>(ws + q.b);
  CUtensorMap map_x[2], map_a, map_b;
  sgdb_status_t st = SGDB_OK;
  for (int i = 0; i < 2 && st == SGDB_OK; ++i) st = make_map(&map_x[i], x[i], q.rows, q.cols, q.ldx, q.stride_x, q.batch);
  if (st == SGDB_OK) st = make_map(&map_a, a, q.side, q.side, q.lds, q.stride_s, q.batch);
  if (st == SGDB_OK) st = make_map(&map_b, b, q.side, q.side, q.lds, q.stride_s, q.batch);
  if (st != SGDB_OK) return st;
  const bool tall = q.rows > q.cols;
  for (int i = 0; i < ns.steps; ++i) {
    const CUtensorMap& mx = map_x[i & 1];
    ProductParams p{};
    p.batch = q.batch;
    p.info = info;
    p.ld = q.lds;
    p.stride = q.stride_s;
    p.M = p.N = q.side;
    // A = X X^T; tall: A = X^T X, whose operands run along K
    p.K = tall ? q.rows : q.cols;
    p.a_mn = p.b_mn = tall;
    p.out = a;
    st = launch_product<OUT_GRAM>(mx, mx, p, dev, s);
    if (st != SGDB_OK) return st;
    p.K = q.side;
    p.a_mn = p.b_mn = 0;
    p.out = b;
    p.addend = a;
    p.ca = ns.a, p.cb = ns.b, p.cc = ns.c;
    st = launch_product<OUT_POLY>(map_a, map_a, p, dev, s);
    if (st != SGDB_OK) return st;
    const bool end = i + 1 == ns.steps;
    ProductParams r = end ? final_params : ProductParams{};
    r.batch = q.batch;
    r.info = info;
    r.M = q.rows;
    r.N = q.cols;
    r.K = q.side;
    r.a_mn = 0;
    r.b_mn = tall ? 0 : 1;  // wide: B X, X's rows are K
    r.out = x[(i + 1) & 1];
    r.ld = q.ldx;
    r.stride = q.stride_x;
    const CUtensorMap &first = tall ? mx : map_b, &second = tall ? map_b : mx;
    st = !end ? launch_product<OUT_APPLY>(first, second, r, dev, s)
              : last == OUT_THETA ? launch_product<OUT_THETA>(first, second, r, dev, s)
                                  : launch_product<OUT_FINAL>(first, second, r, dev, s);
    if (st != SGDB_OK) return st;
  }
  return SGDB_OK;
}

sgdb_status_t run_normalise(const NormParams& p, int batch, const DeviceInfo* dev, cudaStream_t s) {
  sgdb_status_t st = launch_dependent(square_sum_kernel, dim3(kNormBlocks, batch), 256, 0, s, p);
  if (st != SGDB_OK) return st;
  const long long n = static_cast<long long>(p.rows) * p.cols;
  const long long want = (n + 1023) / 1024, cap = (8ll * dev->sms + batch - 1) / batch;
  return launch_dependent(normalise_kernel, dim3(static_cast<unsigned>(want < cap ? want : cap), batch), 256, 0, s, p);
}

char* align_workspace(void* p) { return reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(p) + 255) & ~static_cast<uintptr_t>(255)); }

}  // namespace
}  // namespace sgdb

using namespace sgdb;

extern "C" {

size_t sgdb_orthogonalize_workspace_bytes(int32_t batch, int64_t rows, int64_t cols) {
  Plan q;
  return make_plan(batch, rows, cols, false, &q) ? q.total : 0;
}

size_t sgdb_step_orthogonal_workspace_bytes(int32_t batch, int64_t rows, int64_t cols) {
  Plan q;
  return make_plan(batch, rows, cols, true, &q) ? q.total : 0;
}

sgdb_status_t sgdb_orthogonalize(const void* d_u, sgdb_dtype_t dt, int32_t batch, int64_t rows, int64_t cols, int64_t ldu,
                                 int64_t stride_u, const sgdb_newton_schulz_t* ns, void* d_out, sgdb_dtype_t dt_out, int64_t ldout,
                                 int64_t stride_out, void* d_workspace, size_t workspace_bytes, int32_t* d_info, void* stream) {
  Plan q;
  if (!dtype_ok(dt) || !dtype_ok(dt_out) || !make_plan(batch, rows, cols, false, &q) || !rule_ok(ns)) return SGDB_ERR_INVALID_ARG;
  if (ldu < cols || ldout < cols) return SGDB_ERR_INVALID_ARG;
  if (batch > 1 && (stride_u < (rows - 1) * ldu + cols || stride_out < (rows - 1) * ldout + cols)) return SGDB_ERR_INVALID_ARG;
  if (batch == 0) return SGDB_OK;
  if (!array_ok(d_u, dt) || !array_ok(d_out, dt_out) || d_workspace == nullptr || workspace_bytes < q.total)
    return SGDB_ERR_INVALID_ARG;
  if (d_info != nullptr && !array_ok(d_info, SGDB_F32)) return SGDB_ERR_INVALID_ARG;
  const DeviceInfo* dev = nullptr;
  sgdb_status_t st = device_info(&dev);
  if (st != SGDB_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  char* ws = align_workspace(d_workspace);
  NormParams n{};
  n.u = d_u;
  n.dt_in = dt;
  n.rows = q.rows;
  n.cols = q.cols;
  n.ld = ldu;
  n.stride = stride_u;
  n.partials = reinterpret_cast<double*>(ws + q.partials);
  n.x = reinterpret_cast<__half*>(ws + q.x0);
  n.ldx = q.ldx;
  n.stride_x = q.stride_x;
  n.eps = ns->eps;
  n.info = d_info;
  st = run_normalise(n, batch, dev, s);
  if (st != SGDB_OK) return st;
  ProductParams f{};
  f.final_out = d_out;
  f.dt_out = dt_out;
  f.ld_final = ldout;
  f.stride_final = stride_out;
  return run_products(q, *ns, ws, OUT_FINAL, f, d_info, dev, s);
}

sgdb_status_t sgdb_step_orthogonal(const void* d_grad, sgdb_dtype_t dt, int32_t batch, int64_t rows, int64_t cols, int64_t ld,
                                   const float* d_arrival, const int32_t* d_tags, int32_t t, int32_t N, int32_t b, float* d_theta,
                                   float* d_momentum, const sgdb_orthogonal_opt_t* opt, uint8_t* d_mask, int32_t* d_order,
                                   int32_t* d_info, void* d_workspace, size_t workspace_bytes, void* stream) {
  Plan q;
  if (opt == nullptr || !dtype_ok(dt) || !make_plan(batch, rows, cols, true, &q) || !rule_ok(&opt->newton_schulz))
    return SGDB_ERR_INVALID_ARG;
  if (!std::isfinite(opt->lr) || !std::isfinite(opt->momentum) || !std::isfinite(opt->weight_decay) || !std::isfinite(opt->scale))
    return SGDB_ERR_INVALID_ARG;
  const int64_t P = static_cast<int64_t>(batch) * rows * cols;
  if (d_grad == nullptr || !is_aligned16(d_grad) || ld < P || !array_ok(d_theta, SGDB_F32) || !array_ok(d_momentum, SGDB_F32))
    return SGDB_ERR_INVALID_ARG;
  if (batch > 0 && (d_workspace == nullptr || workspace_bytes < q.total)) return SGDB_ERR_INVALID_ARG;
  sgdb_status_t st = sgdb_select(d_arrival, d_tags, t, N, b, d_mask, d_order, d_info, stream);
  if (st != SGDB_OK || batch == 0) return st;
  const DeviceInfo* dev = nullptr;
  st = device_info(&dev);
  if (st != SGDB_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  char* ws = align_workspace(d_workspace);
  float* mean = reinterpret_cast<float*>(ws + q.mean);
  st = sgdb_aggregate(d_grad, dt, P, ld, N, d_order, d_info, mean, stream);
  if (st != SGDB_OK) return st;
  NormParams n{};
  n.u = mean;
  n.dt_in = SGDB_F32;
  n.rows = q.rows;
  n.cols = q.cols;
  n.velocity = d_momentum;
  n.combined = mean;  // element by element, after it has been read
  n.mu = opt->momentum;
  n.nesterov = opt->nesterov != 0;
  n.partials = reinterpret_cast<double*>(ws + q.partials);
  n.x = reinterpret_cast<__half*>(ws + q.x0);
  n.ldx = q.ldx;
  n.stride_x = q.stride_x;
  n.eps = opt->newton_schulz.eps;
  n.info = d_info;
  st = run_normalise(n, batch, dev, s);
  if (st != SGDB_OK) return st;
  ProductParams f{};
  f.final_out = d_theta;
  f.ld_final = cols;
  f.stride_final = rows * cols;
  f.keep = static_cast<float>(1.0 - static_cast<double>(opt->lr) * static_cast<double>(opt->weight_decay));
  f.rate = opt->lr * opt->scale;
  return run_products(q, opt->newton_schulz, ws, OUT_THETA, f, d_info, dev, s);
}

}  // extern "C"
