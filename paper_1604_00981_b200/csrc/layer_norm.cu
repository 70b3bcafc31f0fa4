// Layer norm of a worker's activations, forward and backward (declared in include/sgdb.h).
//
//   mu = mean(x), r = 1/sqrt(mean((x - mu)^2) + eps), n = (x - mu) r, y = n gamma + beta
//   h = dy gamma, dx = r (h - mean(h) - n mean(h n)), dgamma = sum over rows of dy n, dbeta = sum of dy
//
// Both passes are bound by HBM: every element is read once into registers, where the sums
// of its row are taken, and written once.  The variance is taken around the mean that the
// registers give (two sums over the same registers), so large offsets lose nothing.
#include <cuda_runtime.h>

#include <cmath>

#include "sgdb_host.cuh"
#include "sgdb_rows.cuh"

namespace sgdb {
namespace {

constexpr int kMaxThreads = 512;  // threads of a block that works on one row
constexpr int kWarpRows = 8;      // rows that a block of the narrow form works on at a time, one per warp
constexpr int kMaxPartials = 592; // rows of partial sums of dgamma and dbeta, at most

struct LayerNormParams {
  const void *x, *gamma, *beta;
  void* y;
  float *mean, *rstd;
  long long ldx, ldy, T;
  int D, dt_w;
  float eps;
};

struct LayerNormBackParams {
  const void *dy, *x, *gamma;
  const float *mean, *rstd;
  void* dx;
  float* partials;  // [blocks][2 D]: sums of dy n, then sums of dy
  long long lddy, ldx, lddx, T;
  int D, dt_w;
};

// Sum over the threads that share a row; every one of them gets it.  `slots` are two arrays of
// shared memory used in turn, so that one barrier per sum is enough.
template <bool WARP>
__device__ __forceinline__ float row_sum(float v, float* slots) {
  v = warp_sum(v);
  if (WARP) return v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) slots[warp] = v;
  __syncthreads();
  return warp_sum(lane < warps ? slots[lane] : 0.0f);
}
template <bool WARP>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2* slots) {
  a = warp_sum(a);
  b = warp_sum(b);
  if (WARP) return make_float2(a, b);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) slots[warp] = make_float2(a, b);
  __syncthreads();
  const float2 s = lane < warps ? slots[lane] : make_float2(0.0f, 0.0f);
  return make_float2(warp_sum(s.x), warp_sum(s.y));
}

// Forward.  A row belongs to a block (or, WARP, to a warp): thread i holds the chunks i, i + threads, ... of it,
// C of them, with gamma and beta for the same columns, which serve every row of the persistent block.
// The next row's chunks are on their way while this row's sums are taken.
template <typename T, int V, int C, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kWarpRows : kMaxThreads) layer_norm_kernel(const LayerNormParams p) {
  using Ch = Chunk<T, V>;
  __shared__ float s_sum[2][32];
  const int threads = WARP ? 32 : blockDim.x;
  const int i = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int rows = WARP ? kWarpRows : 1;
  const long long step = static_cast<long long>(gridDim.x) * rows;
  long long row = static_cast<long long>(blockIdx.x) * rows + (WARP ? threadIdx.x >> 5 : 0);
  const float inv_d = 1.0f / static_cast<float>(p.D);
  const T* x = static_cast<const T*>(p.x);
  T* y = static_cast<T*>(p.y);

  float gamma[C][V], beta[C][V];
  typename Ch::Raw next[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (i + c * threads) * V;
    next[c] = (row < p.T && col < p.D) ? Ch::load(x + row * p.ldx + col) : Ch::zero();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      gamma[c][e] = (col < p.D && p.gamma != nullptr) ? load_any(p.gamma, p.dt_w, col + e) : 1.0f;
      beta[c][e] = (col < p.D && p.beta != nullptr) ? load_any(p.beta, p.dt_w, col + e) : 0.0f;
    }
  }
  for (; row < p.T; row += step) {
    float v[C][V];
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      Ch::unpack(next[c], v[c]);
#pragma unroll
      for (int e = 0; e < V; ++e) sum += v[c][e];  // columns past D hold zeros
    }
    const long long following = row + step;
    if (following < p.T) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (i + c * threads) * V;
        if (col < p.D) next[c] = Ch::load(x + following * p.ldx + col);
      }
    }
    const float mean = row_sum<WARP>(sum, s_sum[0]) * inv_d;
    float square = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const bool in = (i + c * threads) * V < p.D;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[c][e] -= mean;
        if (in) square += v[c][e] * v[c][e];
      }
    }
    const float rstd = __frsqrt_rn(row_sum<WARP>(square, s_sum[1]) * inv_d + p.eps);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (i + c * threads) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) v[c][e] = fmaf(v[c][e] * rstd, gamma[c][e], beta[c][e]);
      if (col < p.D) Ch::store(y + row * p.ldy + col, v[c]);
    }
    if (i == 0) {
      if (p.mean != nullptr) p.mean[row] = mean;
      if (p.rstd != nullptr) p.rstd[row] = rstd;
    }
  }
}

// Forward for rows that no block's registers hold: one block per row, the row is read three times (from L2
// after the first).
template <typename T>
__global__ void __launch_bounds__(kMaxThreads) layer_norm_wide_kernel(const LayerNormParams p) {
  __shared__ float s_sum[2][32];
  const float inv_d = 1.0f / static_cast<float>(p.D);
  for (long long row = blockIdx.x; row < p.T; row += gridDim.x) {
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    T* y = static_cast<T*>(p.y) + row * p.ldy;
    float sum = 0.0f;
    for (int col = threadIdx.x; col < p.D; col += blockDim.x) sum += widen<T>(x[col]);
    const float mean = row_sum<false>(sum, s_sum[0]) * inv_d;
    float square = 0.0f;
    for (int col = threadIdx.x; col < p.D; col += blockDim.x) {
      const float d = widen<T>(x[col]) - mean;
      square += d * d;
    }
    const float rstd = __frsqrt_rn(row_sum<false>(square, s_sum[1]) * inv_d + p.eps);
    for (int col = threadIdx.x; col < p.D; col += blockDim.x) {
      const float g = p.gamma != nullptr ? load_any(p.gamma, p.dt_w, col) : 1.0f;
      const float b = p.beta != nullptr ? load_any(p.beta, p.dt_w, col) : 0.0f;
      y[col] = narrow<T>(fmaf((widen<T>(x[col]) - mean) * rstd, g, b));
    }
    if (threadIdx.x == 0) {
      if (p.mean != nullptr) p.mean[row] = mean;
      if (p.rstd != nullptr) p.rstd[row] = rstd;
    }
  }
}

// Backward: as the forward pass, with the thread's columns of dgamma and dbeta summed in registers over the
// rows of the block.  Each block writes its sums once; sum_partials_kernel adds the blocks' sums in
// their order, so the result does not change from run to run.
template <typename T, int V, int C, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kWarpRows : kMaxThreads) layer_norm_back_kernel(const LayerNormBackParams p) {
  using Ch = Chunk<T, V>;
  __shared__ float2 s_sum[2][32];
  __shared__ float s_cols[WARP ? 2 * 32 * C * V : 1];
  const int threads = WARP ? 32 : blockDim.x;
  const int i = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int rows = WARP ? kWarpRows : 1;
  const long long step = static_cast<long long>(gridDim.x) * rows;
  long long row = static_cast<long long>(blockIdx.x) * rows + (WARP ? threadIdx.x >> 5 : 0);
  const float inv_d = 1.0f / static_cast<float>(p.D);
  const T* x = static_cast<const T*>(p.x);
  const T* dy = static_cast<const T*>(p.dy);
  T* dx = static_cast<T*>(p.dx);

  float gamma[C][V], dgamma[C][V], dbeta[C][V];
  typename Ch::Raw next_x[C], next_dy[C];
  float next_mean = 0.0f, next_rstd = 0.0f;
  if (row < p.T) {
    next_mean = p.mean[row];
    next_rstd = p.rstd[row];
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (i + c * threads) * V;
    const bool in = row < p.T && col < p.D;
    next_x[c] = in ? Ch::load(x + row * p.ldx + col) : Ch::zero();
    next_dy[c] = in ? Ch::load(dy + row * p.lddy + col) : Ch::zero();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      gamma[c][e] = (col < p.D && p.gamma != nullptr) ? load_any(p.gamma, p.dt_w, col + e) : 1.0f;
      dgamma[c][e] = dbeta[c][e] = 0.0f;
    }
  }
  int turn = 0;
  for (; row < p.T; row += step) {
    float n[C][V], h[C][V];
    const float mean = next_mean, rstd = next_rstd;
    float sum_h = 0.0f, sum_hn = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      Ch::unpack(next_x[c], n[c]);
      Ch::unpack(next_dy[c], h[c]);  // columns past D hold zeros here, so they add nothing below
#pragma unroll
      for (int e = 0; e < V; ++e) {
        n[c][e] = (n[c][e] - mean) * rstd;
        dgamma[c][e] = fmaf(h[c][e], n[c][e], dgamma[c][e]);
        dbeta[c][e] += h[c][e];
        h[c][e] *= gamma[c][e];
        sum_h += h[c][e];
        sum_hn = fmaf(h[c][e], n[c][e], sum_hn);
      }
    }
    const long long following = row + step;
    if (following < p.T) {
      next_mean = p.mean[following];
      next_rstd = p.rstd[following];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (i + c * threads) * V;
        if (col < p.D) {
          next_x[c] = Ch::load(x + following * p.ldx + col);
          next_dy[c] = Ch::load(dy + following * p.lddy + col);
        }
      }
    }
    const float2 sums = row_sum2<WARP>(sum_h, sum_hn, s_sum[turn]);
    turn ^= 1;
    const float mean_h = sums.x * inv_d, mean_hn = sums.y * inv_d;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (i + c * threads) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) h[c][e] = rstd * (h[c][e] - mean_h - n[c][e] * mean_hn);
      if (col < p.D) Ch::store(dx + row * p.lddx + col, h[c]);
    }
  }

  if (p.partials == nullptr) return;
  float* out = p.partials + static_cast<long long>(blockIdx.x) * 2 * p.D;
  if (WARP) {  // the warps' sums in their order
    for (int w = 0; w < kWarpRows; ++w) {
      if (threadIdx.x >> 5 == w) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const int at = (c * V + e) * 32 + i;
            s_cols[at] = (w == 0 ? 0.0f : s_cols[at]) + dgamma[c][e];
            s_cols[32 * C * V + at] = (w == 0 ? 0.0f : s_cols[32 * C * V + at]) + dbeta[c][e];
          }
      }
      __syncthreads();
    }
    if (threadIdx.x >= 32) return;
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (i + c * threads) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (col < p.D) {
        out[col + e] = WARP ? s_cols[(c * V + e) * 32 + i] : dgamma[c][e];
        out[p.D + col + e] = WARP ? s_cols[32 * C * V + (c * V + e) * 32 + i] : dbeta[c][e];
      }
    }
  }
}

// Backward for rows that no block's registers hold: dx with one block per row ...
template <typename T>
__global__ void __launch_bounds__(kMaxThreads) layer_norm_back_wide_kernel(const LayerNormBackParams p) {
  __shared__ float2 s_sum[2][32];
  const float inv_d = 1.0f / static_cast<float>(p.D);
  int turn = 0;
  for (long long row = blockIdx.x; row < p.T; row += gridDim.x) {
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const T* dy = static_cast<const T*>(p.dy) + row * p.lddy;
    T* dx = static_cast<T*>(p.dx) + row * p.lddx;
    const float mean = p.mean[row], rstd = p.rstd[row];
    float sum_h = 0.0f, sum_hn = 0.0f;
    for (int col = threadIdx.x; col < p.D; col += blockDim.x) {
      const float h = widen<T>(dy[col]) * (p.gamma != nullptr ? load_any(p.gamma, p.dt_w, col) : 1.0f);
      sum_h += h;
      sum_hn = fmaf(h, (widen<T>(x[col]) - mean) * rstd, sum_hn);
    }
    const float2 sums = row_sum2<false>(sum_h, sum_hn, s_sum[turn]);
    turn ^= 1;
    for (int col = threadIdx.x; col < p.D; col += blockDim.x) {
      const float h = widen<T>(dy[col]) * (p.gamma != nullptr ? load_any(p.gamma, p.dt_w, col) : 1.0f);
      dx[col] = narrow<T>(rstd * (h - sums.x * inv_d - (widen<T>(x[col]) - mean) * rstd * (sums.y * inv_d)));
    }
  }
}

// ... and the sums of dgamma and dbeta with one thread per column and one block row per slice of the rows.
template <typename T>
__global__ void __launch_bounds__(256) layer_norm_back_columns_kernel(const LayerNormBackParams p) {
  const long long col = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  if (col >= p.D) return;
  const long long first = p.T * blockIdx.y / gridDim.y, last = p.T * (blockIdx.y + 1) / gridDim.y;
  float dgamma = 0.0f, dbeta = 0.0f;
  for (long long row = first; row < last; ++row) {
    const float g = widen<T>(static_cast<const T*>(p.dy)[row * p.lddy + col]);
    const float n = (widen<T>(static_cast<const T*>(p.x)[row * p.ldx + col]) - p.mean[row]) * p.rstd[row];
    dgamma = fmaf(g, n, dgamma);
    dbeta += g;
  }
  float* out = p.partials + static_cast<long long>(blockIdx.y) * 2 * p.D;
  out[col] = dgamma;
  out[p.D + col] = dbeta;
}

// Adds the partial sums of dgamma and dbeta: 32 columns per block, 16 warps that each take every sixteenth
// partial sum, then the warps' sums in their order.
constexpr int kSumWarps = 16;
__global__ void __launch_bounds__(32 * kSumWarps) sum_partials_kernel(const float* partials, int count, int D, void* dgamma,
                                                                     void* dbeta, int dt) {
  __shared__ float s[kSumWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long col = static_cast<long long>(blockIdx.x) * 32 + lane;  // of 2 D
  float sum = 0.0f;
  if (col < 2ll * D) {
#pragma unroll 8
    for (int b = warp; b < count; b += kSumWarps) sum += partials[static_cast<long long>(b) * 2 * D + col];
  }
  s[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && col < 2ll * D) {
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kSumWarps; ++w) sum += s[w][lane];
    if (col < D) {
      if (dgamma != nullptr) store_any(dgamma, dt, col, sum);
    } else if (dbeta != nullptr) {
      store_any(dbeta, dt, col - D, sum);
    }
  }
}

// Blocks of `kernel` that are resident at once, asked once per kernel, block size and device.
template <typename Kernel>
sgdb_status_t resident_blocks(Kernel kernel, int threads, const DeviceInfo* dev, std::atomic<int>* known, int* out) {
  std::atomic<int>& k = known[dev->index * (kMaxThreads / 32 + 1) + threads / 32];
  int per_sm = k.load(std::memory_order_relaxed);
  if (per_sm == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, 0) != cudaSuccess) return launch_status();
    if (per_sm < 1) per_sm = 1;
    k.store(per_sm, std::memory_order_relaxed);
  }
  *out = per_sm * dev->sms;
  return SGDB_OK;
}
using Known = std::atomic<int>[kMaxDevices * (kMaxThreads / 32 + 1)];

int round32(int n) { return (n + 31) & ~31; }

template <typename T, int V, int C, bool WARP>
sgdb_status_t run_forward(const LayerNormParams& p, const DeviceInfo* dev, cudaStream_t s) {
  static Known known;
  const int chunks = (p.D + V - 1) / V;
  const int threads = WARP ? 32 * kWarpRows : round32((chunks + C - 1) / C);
  int grid = 0;
  auto kernel = layer_norm_kernel<T, V, C, WARP>;
  const sgdb_status_t st = resident_blocks(kernel, threads, dev, known, &grid);
  if (st != SGDB_OK) return st;
  const long long want = WARP ? (p.T + kWarpRows - 1) / kWarpRows : p.T;
  if (want < grid) grid = static_cast<int>(want);
  kernel<<<grid, threads, 0, s>>>(p);
  return launch_status();
}

template <typename T>
sgdb_status_t forward(const LayerNormParams& p, bool vec, const DeviceInfo* dev, cudaStream_t s) {
  constexpr int V = kChunk16<T>;
  if (vec) {
    const int n = p.D / V;
    if (n <= 32) return run_forward<T, V, 1, true>(p, dev, s);
    if (n <= 64) return run_forward<T, V, 2, true>(p, dev, s);
    if (n <= 128) return run_forward<T, V, 4, true>(p, dev, s);
    if (n <= 4 * kMaxThreads) return run_forward<T, V, 4, false>(p, dev, s);
  } else {
    if (p.D <= 128) return run_forward<T, 1, 4, true>(p, dev, s);
    if (p.D <= 4 * kMaxThreads) return run_forward<T, 1, 4, false>(p, dev, s);
    if (p.D <= 16 * kMaxThreads) return run_forward<T, 1, 16, false>(p, dev, s);
  }
  const long long cap = 4ll * dev->sms;
  layer_norm_wide_kernel<T><<<static_cast<unsigned>(p.T < cap ? p.T : cap), kMaxThreads, 0, s>>>(p);
  return launch_status();
}

template <typename T, int V, int C, bool WARP>
sgdb_status_t run_backward(const LayerNormBackParams& p, const DeviceInfo* dev, cudaStream_t s, int* partials) {
  static Known known;
  const int chunks = (p.D + V - 1) / V;
  const int threads = WARP ? 32 * kWarpRows : round32((chunks + C - 1) / C);
  int grid = 0;
  auto kernel = layer_norm_back_kernel<T, V, C, WARP>;
  const sgdb_status_t st = resident_blocks(kernel, threads, dev, known, &grid);
  if (st != SGDB_OK) return st;
  const long long want = WARP ? (p.T + kWarpRows - 1) / kWarpRows : p.T;
  if (want < grid) grid = static_cast<int>(want);
  if (grid > kMaxPartials) grid = kMaxPartials;
  *partials = grid;
  kernel<<<grid, threads, 0, s>>>(p);
  return launch_status();
}

template <typename T>
sgdb_status_t backward(const LayerNormBackParams& p, bool vec, const DeviceInfo* dev, cudaStream_t s, int* partials) {
  constexpr int V = kChunk16<T>;
  constexpr int kMost = sizeof(T) == 2 ? 2 : 4;  // chunks per thread: 16 columns
  if (vec) {
    const int n = p.D / V;
    if (n <= 32) return run_backward<T, V, 1, true>(p, dev, s, partials);
    if (n <= 64) return run_backward<T, V, 2, true>(p, dev, s, partials);
    if (n <= kMaxThreads) return run_backward<T, V, 1, false>(p, dev, s, partials);
    if (n <= kMost * kMaxThreads) return run_backward<T, V, kMost, false>(p, dev, s, partials);
  } else {
    if (p.D <= 128) return run_backward<T, 1, 4, true>(p, dev, s, partials);
    if (p.D <= 4 * kMaxThreads) return run_backward<T, 1, 4, false>(p, dev, s, partials);
    if (p.D <= 16 * kMaxThreads) return run_backward<T, 1, 16, false>(p, dev, s, partials);
  }
  const long long cap = 4ll * dev->sms;
  layer_norm_back_wide_kernel<T><<<static_cast<unsigned>(p.T < cap ? p.T : cap), kMaxThreads, 0, s>>>(p);
  sgdb_status_t st = launch_status();
  if (st != SGDB_OK || p.partials == nullptr) return st;
  *partials = static_cast<int>(p.T < 64 ? p.T : 64);
  layer_norm_back_columns_kernel<T><<<dim3((p.D + 255) / 256, *partials), 256, 0, s>>>(p);
  return launch_status();
}

bool sizes_ok(int64_t tokens, int64_t width) { return tokens >= 0 && width >= 1 && width <= SGDB_MAX_WIDTH; }

}  // namespace
}  // namespace sgdb

using namespace sgdb;

extern "C" {

sgdb_status_t sgdb_layer_norm(const void* d_x, sgdb_dtype_t dt, int64_t tokens, int64_t width, int64_t ldx, const void* d_gamma,
                              const void* d_beta, sgdb_dtype_t dt_w, float eps, void* d_y, int64_t ldy, float* d_mean,
                              float* d_rstd, void* stream) {
  if (!dtype_ok(dt) || !dtype_ok(dt_w) || !sizes_ok(tokens, width) || ldx < width || ldy < width) return SGDB_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || std::isinf(eps)) return SGDB_ERR_INVALID_ARG;
  if (tokens == 0) return SGDB_OK;
  if (!array_ok(d_x, dt) || !array_ok(d_y, dt)) return SGDB_ERR_INVALID_ARG;
  if ((d_gamma != nullptr && !array_ok(d_gamma, dt_w)) || (d_beta != nullptr && !array_ok(d_beta, dt_w))) return SGDB_ERR_INVALID_ARG;
  if ((d_mean != nullptr && !array_ok(d_mean, SGDB_F32)) || (d_rstd != nullptr && !array_ok(d_rstd, SGDB_F32)))
    return SGDB_ERR_INVALID_ARG;
  const DeviceInfo* dev = nullptr;
  const sgdb_status_t st = device_info(&dev);
  if (st != SGDB_OK) return st;
  const LayerNormParams p{d_x, d_gamma, d_beta, d_y, d_mean, d_rstd, ldx, ldy, tokens, static_cast<int>(width), dt_w, eps};
  const bool vec = rows_aligned16(d_x, ldx, dt) && rows_aligned16(d_y, ldy, dt) &&
                   (width * static_cast<int64_t>(dtype_size(dt))) % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return dt == SGDB_BF16 ? forward<BF16>(p, vec, dev, s) : forward<float>(p, vec, dev, s);
}

size_t sgdb_layer_norm_backward_workspace_bytes(int64_t tokens, int64_t width) {
  if (!sizes_ok(tokens, width)) return 0;
  const int64_t rows = tokens < kMaxPartials ? tokens : kMaxPartials;
  return static_cast<size_t>(rows) * 2 * static_cast<size_t>(width) * sizeof(float);
}

sgdb_status_t sgdb_layer_norm_backward(const void* d_dy, int64_t lddy, const void* d_x, int64_t ldx, sgdb_dtype_t dt,
                                       int64_t tokens, int64_t width, const void* d_gamma, sgdb_dtype_t dt_w,
                                       const float* d_mean, const float* d_rstd, void* d_dx, int64_t lddx, void* d_dgamma,
                                       void* d_dbeta, sgdb_dtype_t dt_g, void* d_workspace, size_t workspace_bytes,
                                       void* stream) {
  if (!dtype_ok(dt) || !dtype_ok(dt_w) || !dtype_ok(dt_g) || !sizes_ok(tokens, width)) return SGDB_ERR_INVALID_ARG;
  if (lddy < width || ldx < width || lddx < width) return SGDB_ERR_INVALID_ARG;
  if (tokens > 0 && (!array_ok(d_dy, dt) || !array_ok(d_x, dt) || !array_ok(d_dx, dt) || !array_ok(d_mean, SGDB_F32) ||
                     !array_ok(d_rstd, SGDB_F32)))
    return SGDB_ERR_INVALID_ARG;
  if (d_gamma != nullptr && !array_ok(d_gamma, dt_w)) return SGDB_ERR_INVALID_ARG;
  if ((d_dgamma != nullptr && !array_ok(d_dgamma, dt_g)) || (d_dbeta != nullptr && !array_ok(d_dbeta, dt_g)))
    return SGDB_ERR_INVALID_ARG;
  const bool sums = d_dgamma != nullptr || d_dbeta != nullptr;
  if (sums && tokens > 0 &&
      (!array_ok(d_workspace, SGDB_F32) || workspace_bytes < sgdb_layer_norm_backward_workspace_bytes(tokens, width)))
    return SGDB_ERR_INVALID_ARG;
  const DeviceInfo* dev = nullptr;
  sgdb_status_t st = device_info(&dev);
  if (st != SGDB_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int partials = 0;
  if (tokens > 0) {
    const LayerNormBackParams p{d_dy, d_x, d_gamma, d_mean, d_rstd, d_dx, sums ? static_cast<float*>(d_workspace) : nullptr,
                                lddy, ldx, lddx, tokens, static_cast<int>(width), dt_w};
    const bool vec = rows_aligned16(d_dy, lddy, dt) && rows_aligned16(d_x, ldx, dt) && rows_aligned16(d_dx, lddx, dt) &&
                     (width * static_cast<int64_t>(dtype_size(dt))) % 16 == 0;
    st = dt == SGDB_BF16 ? backward<BF16>(p, vec, dev, s, &partials) : backward<float>(p, vec, dev, s, &partials);
    if (st != SGDB_OK) return st;
  }
  if (!sums) return SGDB_OK;
  // no tokens: the sums are zero
  const unsigned blocks = static_cast<unsigned>((2 * width + 31) / 32);
  sum_partials_kernel<<<blocks, 32 * kSumWarps, 0, s>>>(static_cast<const float*>(d_workspace), partials, static_cast<int>(width),
                                                        d_dgamma, d_dbeta, dt_g);
  return launch_status();
}

}  // extern "C"
