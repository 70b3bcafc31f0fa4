// Layer norm of a worker's activations, forward and backward (declared in include/sgdb.h).
//
//   mu = mean(x), r = 1/sqrt(mean((x - mu)^2) + eps), n = (x - mu) r, y = n gamma + beta
//   h = dy gamma, dx = r (h - mean(h) - n mean(h n)), dgamma = sum over rows of dy n, dbeta = sum of dy
//
// Both passes are bound by HBM: every element is read once into registers, where the sums
// of its row are taken, and written once.  The variance is taken around the mean that the
// registers give (two sums over the same registers), so large offsets lose nothing.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <cmath>

#include "sgdb_host.cuh"
#include "sgdb_rows.cuh"

namespace sgdb {
namespace {

namespace cg = cooperative_groups;

constexpr int kMaxThreads = 512;  // threads of a block that works on one row
constexpr int kWarpRows = 8;      // rows that a block of the narrow form works on at a time, one per warp
constexpr int kDepth = 3;         // rows on their way, and one more
constexpr int kCluster = 2;       // blocks that add their sums of dgamma and dbeta before they write them
constexpr int kMaxPartials = 592; // rows of partial sums of dgamma and dbeta, at most

struct LayerNormParams {
  const void *x, *gamma, *beta;
  void* y;
  float *mean, *rstd;
  long long ldx, ldy, T;
  int D, dt_w;
  float eps;
  bool chunked;  // y's rows lie against 16-byte boundaries as x's do
};

struct LayerNormBackParams {
  const void *dy, *x, *gamma;
  const float *mean, *rstd;
  void* dx;
  float* partials;  // [blocks or clusters][2 D]: sums of dy n, then sums of dy
  long long lddy, ldx, lddx, T;
  int D, dt_w;
  bool chunked;  // dx's rows lie against 16-byte boundaries as x's do
};

// Sum over the threads that share a row; every one of them gets it.  `slots`: shared memory, two arrays used in turn, so
// that one barrier per sum is enough.
template <bool WARP>
__device__ __forceinline__ float row_sum(float v, float* slots) {
  v = warp_sum(v);
  if (WARP) return v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) slots[warp] = v;
  __syncthreads();
  // at most 16 warps: half a warp's lanes hold them all
  v = (lane & 15) < warps ? slots[lane & 15] : 0.0f;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Two such sums at once: after the first exchange even lanes carry a, odd lanes b.
template <bool WARP>
__device__ __forceinline__ float2 row_sum2(float a, float b, float* slots) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const bool odd = lane & 1;
  float v = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
#pragma unroll
  for (int o = 2; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (!WARP) {
    if (lane < 2) slots[2 * warp + lane] = v;
    __syncthreads();
    v = lane < 2 * warps ? slots[lane] : 0.0f;
#pragma unroll
    for (int o = 2; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  }
  const float other = __shfl_xor_sync(0xffffffffu, v, 1);
  return odd ? make_float2(other, v) : make_float2(v, other);
}

// A thread's share of a row: C chunks of 16 bytes, `threads` chunks apart, as pairs for the paired fp32 instructions.
//
// Chunks lie on 16-byte boundaries of memory, rows need not: a row begins `shift` elements into its first chunk.  Rows that a
// multiple of 8 rows (bf16; fp32: 4) lies between have the same shift, and so have all rows of one block when the number of
// blocks is such a multiple: a thread's columns are then the same in all its rows, whatever the width.  Elements of a row's
// first and last chunk that are not the row's are read, never used and never written.
//
// The rows on their way are a ring of DEPTH rows in shared memory, of which each thread copies and reads its own chunks
// only, so that no barrier is needed.  STREAMS rows (x, or x and dy) come together.
// FIT: every thread has C chunks, all whole (FULL); some threads have fewer (PARTS); or some chunks are not the row's as a
// whole (EDGES).
enum : int { FIT_FULL = 0, FIT_PARTS = 1, FIT_EDGES = 2 };
template <typename T, int C, int STREAMS, int DEPTH, int FIT>
struct Share {
  static constexpr int V = kChunk16<T>;
  using Ch = Chunk<T, V>;
  static constexpr int kPairs = C * V / 2;
  static constexpr bool EDGES = FIT == FIT_EDGES;
  int col[C];            // first column of each chunk, from -shift on
  bool in[C], whole[C];  // whether the row has some of it, and all of it
  uint32_t base, apart;  // shared memory: this thread's first chunk, distance of its chunks
  int slot, D;

  static size_t bytes(int block) { return static_cast<size_t>(DEPTH) * STREAMS * C * block * 16; }  // shared memory of a block

  __device__ __forceinline__ Share(uint8_t* smem, int i, int threads, int D_, int shift) : slot(0), D(D_) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      col[c] = (i + c * threads) * V - shift;
      in[c] = FIT == FIT_FULL || col[c] < D;
      whole[c] = EDGES ? col[c] >= 0 && col[c] + V <= D : in[c];
    }
    base = smem_addr(smem) + threadIdx.x * 16;
    apart = blockDim.x * 16;
  }
  __device__ __forceinline__ uint32_t at(int s, int stream) const { return base + (s * STREAMS + stream) * C * apart; }
  // Starts the copies of a row into slot s.
  __device__ __forceinline__ void fetch(int s, int stream, const T* row) const {
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (in[c]) copy16_async(at(s, stream) + c * apart, row + col[c]);
  }
  // The oldest row's values; columns that the row does not have are zero.
  __device__ __forceinline__ void take(int stream, Pair (&v)[kPairs]) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      uint4 raw = in[c] ? lds128(at(slot, stream) + c * apart) : Ch::zero();
      if (EDGES && in[c] && !whole[c]) {
        const uint4 m = mask(c);
        raw = make_uint4(raw.x & m.x, raw.y & m.y, raw.z & m.z, raw.w & m.w);
      }
      float u[V];
      Ch::unpack(raw, u);
      put(v, c, u);
    }
  }
  // Ones in the bits of chunk c's elements that are the row's.
  __device__ __forceinline__ uint4 mask(int c) const {
    const int first = col[c] < 0 ? -col[c] * static_cast<int>(sizeof(T)) : 0;  // bytes
    const int last = col[c] + V > D ? (D - col[c]) * static_cast<int>(sizeof(T)) : 16;
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int a = first - 4 * q, b = last - 4 * q;  // the word's bytes a .. b - 1; of them there are 0, 2 (bf16) or 4
      const uint32_t from = a <= 0 ? 0xffffffffu : a >= 4 ? 0u : 0xffff0000u;
      const uint32_t to = b >= 4 ? 0xffffffffu : b <= 0 ? 0u : 0x0000ffffu;
      w[q] = from & to;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void advance() { slot = slot == DEPTH - 1 ? 0 : slot + 1; }
  // chunked: the output's rows lie against the boundaries as the input's do
  __device__ __forceinline__ void store(T* row, const Pair (&v)[kPairs], bool chunked) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!in[c]) continue;
      float u[V];
      get(v, c, u);
      const uint4 raw = Ch::pack(u);
      if (!EDGES || (whole[c] && chunked)) {
        Ch::store_raw(row + col[c], raw);
      } else if (chunked) {
        store_part(row + col[c], raw, col[c] < 0 ? -col[c] : 0, col[c] + V > D ? D - col[c] : V);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (col[c] + e >= 0 && col[c] + e < D) row[col[c] + e] = narrow<T>(u[e]);
      }
    }
  }
  static __device__ __forceinline__ void put(Pair* v, int c, const float (&u)[V]) {
#pragma unroll
    for (int e = 0; e < V; e += 2) v[(c * V + e) / 2] = pair(u[e], u[e + 1]);
  }
  static __device__ __forceinline__ void get(const Pair* v, int c, float (&u)[V]) {
#pragma unroll
    for (int e = 0; e < V; e += 2) {
      const float2 d = split(v[(c * V + e) / 2]);
      u[e] = d.x;
      u[e + 1] = d.y;
    }
  }
  // Zeros in columns that the row does not have.
  __device__ __forceinline__ void clear_outside(Pair (&v)[kPairs]) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (whole[c]) continue;
      if (!EDGES || !in[c]) {
#pragma unroll
        for (int k = 0; k < V / 2; ++k) v[c * V / 2 + k] = 0;
        continue;
      }
      const uint4 m = mask(c);
      const uint32_t w[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
      for (int k = 0; k < V / 2; ++k) {
        const uint32_t lo = sizeof(T) == 2 ? __byte_perm(w[k], 0, 0x1010) : w[2 * k & 3];
        const uint32_t hi = sizeof(T) == 2 ? __byte_perm(w[k], 0, 0x3232) : w[(2 * k + 1) & 3];
        v[c * V / 2 + k] &= (static_cast<Pair>(hi) << 32) | lo;
      }
    }
  }
  // Parameters of the share's columns.
  __device__ __forceinline__ void parameters(const void* p, int dt, float otherwise, Pair (&v)[kPairs]) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float u[V];
#pragma unroll
      for (int e = 0; e < V; ++e)
        u[e] = (EDGES ? col[c] + e >= 0 && col[c] + e < D : in[c]) && p != nullptr ? load_any(p, dt, col[c] + e) : otherwise;
      put(v, c, u);
    }
  }
};

// Forward.  A row belongs to a block (or, WARP, to a warp): thread i holds the chunks i, i + threads, ... of it,
// C of them, with gamma and beta for the same columns, which serve every row of the persistent block.
template <typename T, int C, bool WARP, int FIT>
__global__ void __launch_bounds__(WARP ? 32 * kWarpRows : kMaxThreads) layer_norm_kernel(const LayerNormParams p) {
  using Sh = Share<T, C, 1, kDepth, FIT>;
  constexpr int kPairs = Sh::kPairs;
  constexpr bool EDGES = FIT == FIT_EDGES;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float s_sum[2][16];
  const int threads = WARP ? 32 : blockDim.x;
  const int i = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int rows = WARP ? kWarpRows : 1;
  const long long step = static_cast<long long>(gridDim.x) * rows;
  long long row = static_cast<long long>(blockIdx.x) * rows + (WARP ? threadIdx.x >> 5 : 0);
  const float inv_d = 1.0f / static_cast<float>(p.D);
  const T* x = static_cast<const T*>(p.x);
  T* y = static_cast<T*>(p.y);
  Sh share(smem, i, threads, p.D, EDGES ? shift_of(x + row * p.ldx) : 0);
  pdl_wait();
#pragma unroll
  for (int k = 0; k < kDepth - 1; ++k) {
    if (row + k * step < p.T) share.fetch(k, 0, x + (row + k * step) * p.ldx);
    copy_commit();
  }
  Pair gamma[kPairs], beta[kPairs];
  share.parameters(p.gamma, p.dt_w, 1.0f, gamma);
  share.parameters(p.beta, p.dt_w, 0.0f, beta);
  for (; row < p.T; row += step) {
    Pair v[kPairs];
    copy_wait<kDepth - 2>();
    share.take(0, v);
    const long long coming = row + (kDepth - 1) * step;
    if (coming < p.T) share.fetch(share.slot == 0 ? kDepth - 1 : share.slot - 1, 0, x + coming * p.ldx);
    copy_commit();
    share.advance();
    Pair sum = v[0];
#pragma unroll
    for (int k = 1; k < kPairs; ++k) sum = add2(sum, v[k]);  // columns that the row does not have hold zeros
    const float mean = row_sum<WARP>(total(sum), s_sum[0]) * inv_d;
    const Pair minus_mean = pair(-mean);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) v[k] = add2(v[k], minus_mean);
    share.clear_outside(v);
    Pair square = 0;
#pragma unroll
    for (int k = 0; k < kPairs; ++k) square = fma2(v[k], v[k], square);
    const float rstd = __frsqrt_rn(row_sum<WARP>(total(square), s_sum[1]) * inv_d + p.eps);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) v[k] = fma2(mul2(v[k], pair(rstd)), gamma[k], beta[k]);
    share.store(y + row * p.ldy, v, p.chunked);
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
  __shared__ float s_sum[2][16];
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

// The blocks of a cluster add their `sums` [2][D]: each takes a share of the columns of all.  Out of line, so that the
// loop over the rows keeps its registers to itself.
__device__ __noinline__ void add_over_cluster(float* sums, int D, float* partials) {
  cg::cluster_group cluster = cg::this_cluster();
  const int blocks = static_cast<int>(cluster.num_blocks());
  cluster.sync();
  float* out = partials + static_cast<long long>(blockIdx.x / blocks) * 2 * D;
  for (int col = cluster.block_rank() * blockDim.x + threadIdx.x; col < 2 * D; col += blocks * blockDim.x) {
    float sum = 0.0f;
#pragma unroll 8
    for (int r = 0; r < blocks; ++r) sum += cluster.map_shared_rank(sums, r)[col];
    out[col] = sum;
  }
  cluster.sync();  // no block leaves while another may still read its sums
}

// Backward: as the forward pass, with the thread's columns of dgamma and dbeta summed in registers over the
// rows of the block.  The blocks of a cluster add their sums through distributed shared memory and each writes its share of
// the columns; sum_partials_kernel adds the clusters' (WARP: the blocks') sums.  All in a fixed order: the result does
// not change from run to run.  8192x4096 bf16:
// 45.0 us with clusters of 2, 46.1 without, 49.8 with 4 and 56 with 8, whose blocks do not fill the GPU.
template <typename T, int C, bool WARP, int THREADS, int BLOCKS, int FIT>
__global__ void __launch_bounds__(THREADS, BLOCKS) layer_norm_back_kernel(const LayerNormBackParams p) {
  using Sh = Share<T, C, 2, kDepth, FIT>;
  constexpr int kPairs = Sh::kPairs, V = Sh::V;
  constexpr bool EDGES = FIT == FIT_EDGES;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float s_sum[2][32];
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
  Sh share(smem, i, threads, p.D, EDGES ? shift_of(x + row * p.ldx) : 0);
  const auto fetch = [&](int slot, long long r) {
    if (r < p.T) {
      share.fetch(slot, 0, x + r * p.ldx);
      share.fetch(slot, 1, dy + r * p.lddy);
    }
    copy_commit();
  };
  pdl_wait();
#pragma unroll
  for (int k = 0; k < kDepth - 1; ++k) fetch(k, row + k * step);

  Pair gamma[kPairs], dgamma[kPairs], dbeta[kPairs];
  float next_mean = 0.0f, next_rstd = 0.0f;
  if (row < p.T) {
    next_mean = p.mean[row];
    next_rstd = p.rstd[row];
  }
  share.parameters(p.gamma, p.dt_w, 1.0f, gamma);
#pragma unroll
  for (int k = 0; k < kPairs; ++k) dgamma[k] = dbeta[k] = 0;
  int turn = 0;
  for (; row < p.T; row += step) {
    const float mean = next_mean, rstd = next_rstd;
    copy_wait<kDepth - 2>();
    fetch(share.slot == 0 ? kDepth - 1 : share.slot - 1, row + (kDepth - 1) * step);
    if (row + step < p.T) {
      next_mean = p.mean[row + step];
      next_rstd = p.rstd[row + step];
    }
    const Pair minus_mean = pair(-mean), r2 = pair(rstd);
    Pair n[kPairs], h[kPairs], sum_h = 0, sum_hn = 0;
    share.take(0, n);
    share.take(1, h);  // zero in columns that the row does not have, so that these add nothing below
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      const Pair d = add2(n[k], minus_mean);
      n[k] = mul2(d, r2);
      dgamma[k] = fma2(h[k], n[k], dgamma[k]);
      dbeta[k] = add2(dbeta[k], h[k]);
      h[k] = mul2(h[k], gamma[k]);
      sum_h = add2(sum_h, h[k]);
      // Where a chunk may have columns that the row does not have: of h (x - mean), with the factor rstd behind the sum.  n is
      // -mean rstd there, which may be infinite, and 0 times that is not 0.
      sum_hn = fma2(h[k], FIT == FIT_FULL ? n[k] : d, sum_hn);
    }
    float2 sums = row_sum2<WARP>(total(sum_h), total(sum_hn), s_sum[turn]);
    if (FIT != FIT_FULL) sums.y *= rstd;
    turn ^= 1;
    const Pair minus_mean_h = pair(-sums.x * inv_d), minus_mean_hn = pair(-sums.y * inv_d);
#pragma unroll
    for (int k = 0; k < kPairs; ++k) h[k] = mul2(r2, fma2(n[k], minus_mean_hn, add2(h[k], minus_mean_h)));
    share.store(dx + row * p.lddx, h, p.chunked);
    share.advance();
  }

  if (p.partials == nullptr) return;
  float g[C][V], b[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    Sh::get(dgamma, c, g[c]);
    Sh::get(dbeta, c, b[c]);
  }
  if constexpr (WARP) {  // the warps' sums in their order, by column: shifts differ from warp to warp
    for (int w = 0; w < kWarpRows; ++w) {
      if (threadIdx.x >> 5 == w) {
#pragma unroll
        for (int k = 0; k < C * V; ++k) {
          const int col = share.col[k / V] + k % V;
          if (EDGES ? col >= 0 && col < p.D : share.in[k / V]) {
            s_cols[col] = (w == 0 ? 0.0f : s_cols[col]) + g[k / V][k % V];
            s_cols[32 * C * V + col] = (w == 0 ? 0.0f : s_cols[32 * C * V + col]) + b[k / V][k % V];
          }
        }
      }
      __syncthreads();
    }
    float* out = p.partials + static_cast<long long>(blockIdx.x) * 2 * p.D;
    for (int col = threadIdx.x; col < p.D; col += blockDim.x) {
      out[col] = s_cols[col];
      out[p.D + col] = s_cols[32 * C * V + col];
    }
  } else {
    // the ring is empty: its place takes this block's sums, [2][D]
    float* sums = reinterpret_cast<float*>(smem);
    copy_wait<0>();
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int col = share.col[c] + e;
        if (EDGES ? col >= 0 && col < p.D : share.in[c]) {
          sums[col] = g[c][e];
          sums[p.D + col] = b[c][e];
        }
      }
    }
    add_over_cluster(sums, p.D, p.partials);
  }
}

// Backward for rows that no block's registers hold: dx with one block per row ...
template <typename T>
__global__ void __launch_bounds__(kMaxThreads) layer_norm_back_wide_kernel(const LayerNormBackParams p) {
  __shared__ float s_sum[2][32];
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
  pdl_wait();
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

// Blocks of `kernel` that are resident at once, asked once per kernel, block size and device.  `most`: shared memory of the
// kernel's largest block, which it is allowed then.
template <typename Kernel>
sgdb_status_t resident_blocks(Kernel kernel, int threads, size_t smem, size_t most, const DeviceInfo* dev, std::atomic<int>* known, int* out) {
  std::atomic<int>& k = known[dev->index * (kMaxThreads / 32 + 1) + threads / 32];
  int per_sm = k.load(std::memory_order_relaxed);
  if (per_sm == 0) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most)) != cudaSuccess)
      return launch_status();
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem) != cudaSuccess) return launch_status();
    if (per_sm < 1) per_sm = 1;
    k.store(per_sm, std::memory_order_relaxed);
  }
  *out = per_sm * dev->sms;
  return SGDB_OK;
}
using Known = std::atomic<int>[kMaxDevices * (kMaxThreads / 32 + 1)];

int round32(int n) { return (n + 31) & ~31; }

// Blocks of a persistent kernel: as many as are resident and have work, in multiples of 8 where rows are shifted against
// the chunks.
int whole_grid(long long want, int resident, bool shifted) {
  if (want < resident) resident = static_cast<int>(want);
  return shifted && resident > 8 ? resident & ~7 : shifted ? 8 : resident;
}

template <typename T, int C, bool WARP, int FIT>
sgdb_status_t run_forward(const LayerNormParams& p, int chunks, bool shifted, const DeviceInfo* dev, cudaStream_t s) {
  static Known known;
  const int threads = WARP ? 32 * kWarpRows : round32((chunks + C - 1) / C);
  int resident = 0;
  auto kernel = layer_norm_kernel<T, C, WARP, FIT>;
  const size_t smem = Share<T, C, 1, kDepth, FIT>::bytes(threads), most = Share<T, C, 1, kDepth, FIT>::bytes(WARP ? threads : kMaxThreads);
  const sgdb_status_t st = resident_blocks(kernel, threads, smem, most, dev, known, &resident);
  if (st != SGDB_OK) return st;
  const int grid = whole_grid(WARP ? (p.T + kWarpRows - 1) / kWarpRows : p.T, resident, shifted && !WARP);
  return launch_dependent(kernel, dim3(grid), threads, smem, s, p);
}

// How rows lie against 16-byte boundaries.
struct Boundaries {
  int chunks;    // 16-byte chunks that a row touches at most; 0: x and dy differ
  bool shifted;  // rows begin at different distances from the boundaries
  bool edges;    // some chunks are not a row's as a whole, or the output's rows lie otherwise
};

// The narrowest fit for rows of b.chunks chunks in C chunks per thread.
template <int C, bool WARP>
int fit_of(const Boundaries& b) {
  if (b.edges) return FIT_EDGES;
  return b.chunks == C * (WARP ? 32 : round32((b.chunks + C - 1) / C)) ? FIT_FULL : FIT_PARTS;
}

template <typename T, int C, bool WARP>
sgdb_status_t forward_fit(const LayerNormParams& p, const Boundaries& b, const DeviceInfo* dev, cudaStream_t s) {
  switch (fit_of<C, WARP>(b)) {
    case FIT_FULL: return run_forward<T, C, WARP, FIT_FULL>(p, b.chunks, b.shifted, dev, s);
    case FIT_PARTS: return run_forward<T, C, WARP, FIT_PARTS>(p, b.chunks, b.shifted, dev, s);
    default: return run_forward<T, C, WARP, FIT_EDGES>(p, b.chunks, b.shifted, dev, s);
  }
}

template <typename T>
sgdb_status_t forward(const LayerNormParams& p, const Boundaries& b, const DeviceInfo* dev, cudaStream_t s) {
  if (b.chunks <= 32) return forward_fit<T, 1, true>(p, b, dev, s);
  if (b.chunks <= 64) return forward_fit<T, 2, true>(p, b, dev, s);
  if (b.chunks <= 128) return forward_fit<T, 4, true>(p, b, dev, s);
  if (b.chunks <= 4 * kMaxThreads) return forward_fit<T, 4, false>(p, b, dev, s);
  const long long cap = 4ll * dev->sms;
  layer_norm_wide_kernel<T><<<static_cast<unsigned>(p.T < cap ? p.T : cap), kMaxThreads, 0, s>>>(p);
  return launch_status();
}

template <typename T, int C, bool WARP, int THREADS, int BLOCKS, int FIT>
sgdb_status_t run_backward(const LayerNormBackParams& p, int chunks, bool shifted, const DeviceInfo* dev, cudaStream_t s, int* partials) {
  static Known known;
  const int threads = WARP ? THREADS : round32((chunks + C - 1) / C);
  auto kernel = layer_norm_back_kernel<T, C, WARP, THREADS, BLOCKS, FIT>;
  const size_t smem = Share<T, C, 2, kDepth, FIT>::bytes(threads);
  const long long want = WARP ? (p.T + kWarpRows - 1) / kWarpRows : p.T;
  const int cluster = !WARP && (want >= 8 || shifted) ? kCluster : 1;  // blocks then come in multiples of 8
  cudaLaunchConfig_t cfg{};
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  // blocks that are resident at once, in whole clusters
  std::atomic<int>& known_here = known[dev->index * (kMaxThreads / 32 + 1) + threads / 32];
  int resident = known_here.load(std::memory_order_relaxed);
  if (resident == 0) {
    // the kernel's largest block
    const size_t most = Share<T, C, 2, kDepth, FIT>::bytes(THREADS);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most)) != cudaSuccess)
      return launch_status();
    attr[0].val.clusterDim.x = WARP ? 1 : kCluster;
    cfg.gridDim = dim3(16 * dev->sms / kCluster * kCluster);
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&resident, kernel, &cfg) != cudaSuccess) return launch_status();
    if (resident < 1) return SGDB_ERR_UNSUPPORTED;
    resident *= WARP ? 1 : kCluster;
    if (resident > kMaxPartials) resident = kMaxPartials;
    known_here.store(resident, std::memory_order_relaxed);
    attr[0].val.clusterDim.x = cluster;
  }
  cfg.gridDim = dim3(whole_grid(want, resident, cluster > 1 || shifted));
  cfg.numAttrs = 2;
  *partials = static_cast<int>(cfg.gridDim.x) / cluster;
  (void)cudaLaunchKernelEx(&cfg, kernel, p);
  return launch_status();
}

template <typename T, int C, bool WARP, int THREADS, int BLOCKS>
sgdb_status_t backward_fit(const LayerNormBackParams& p, const Boundaries& b, const DeviceInfo* dev, cudaStream_t s, int* partials) {
  switch (fit_of<C, WARP>(b)) {
    case FIT_FULL: return run_backward<T, C, WARP, THREADS, BLOCKS, FIT_FULL>(p, b.chunks, b.shifted, dev, s, partials);
    case FIT_PARTS: return run_backward<T, C, WARP, THREADS, BLOCKS, FIT_PARTS>(p, b.chunks, b.shifted, dev, s, partials);
    default: return run_backward<T, C, WARP, THREADS, BLOCKS, FIT_EDGES>(p, b.chunks, b.shifted, dev, s, partials);
  }
}

template <typename T>
sgdb_status_t backward(const LayerNormBackParams& p, const Boundaries& b, const DeviceInfo* dev, cudaStream_t s, int* partials) {
  constexpr int kWarpThreads = 32 * kWarpRows;
  if (b.chunks > 0) {
    if (b.chunks <= 32) return backward_fit<T, 1, true, kWarpThreads, 1>(p, b, dev, s, partials);
    if (b.chunks <= 64) return backward_fit<T, 2, true, kWarpThreads, 1>(p, b, dev, s, partials);
    // 65 to 128 chunks: a warp per row (16384x512 fp32 21.5 us, 30.5 with two chunks per thread of a block), but a block
    // - for edges in bf16, whose masks take the registers of that (this kernel alone, us, with a block / a warp / two chunks per
    //   thread of a block: 300x700 7.3 / 17.3 / 8.4, 2000x700 10.3 / 18.3 / 11.6, 16384x700 31.5 / 35.0 / 37.0; 523, 901 and 1001
    //   columns alike);
    // - for few rows of bf16 or with edges, where a row's latency counts (300x1024 bf16 6.8 / 12.4, 2400 rows 10.9 / 15.0, 4800
    //   rows 14.2 / 17.2, 16384 rows 30.7 / 29.8; 300x501 fp32 5.6 / 11.1, 4800 rows 13.0 / 16.2, 16384 rows 30.1 / 29.6); fp32
    //   without edges has half the elements in a chunk (300x512 5.3 / 5.4, 4800 rows 11.9 / 10.7)
    if (b.chunks <= 128) {
      constexpr long long kFewRows = 8192;
      const bool block = sizeof(T) == 2 ? b.edges || p.T <= kFewRows : b.edges && p.T <= kFewRows;
      return block ? backward_fit<T, 1, false, 128, 6>(p, b, dev, s, partials) : backward_fit<T, 4, true, kWarpThreads, 1>(p, b, dev, s, partials);
    }
    if (b.chunks <= 512) return backward_fit<T, 2, false, 256, 2>(p, b, dev, s, partials);
    if (b.chunks <= 1024) return backward_fit<T, 2, false, 512, 1>(p, b, dev, s, partials);
    if (sizeof(T) == 4 && b.chunks <= 2048) return backward_fit<T, sizeof(T) == 4 ? 4 : 2, false, 512, 1>(p, b, dev, s, partials);
  }
  const long long cap = 4ll * dev->sms;
  layer_norm_back_wide_kernel<T><<<static_cast<unsigned>(p.T < cap ? p.T : cap), kMaxThreads, 0, s>>>(p);
  sgdb_status_t st = launch_status();
  if (st != SGDB_OK || p.partials == nullptr) return st;
  // slices of at least 32 rows from 64 slices on, up to what the workspace has room for: few terms per sum, few sums to write
  const long long slices = p.T < 64 ? p.T : p.T < 32ll * 64 ? 64 : p.T < 32ll * kMaxPartials ? p.T / 32 : kMaxPartials;
  *partials = static_cast<int>(slices);
  layer_norm_back_columns_kernel<T><<<dim3((p.D + 255) / 256, *partials), 256, 0, s>>>(p);
  return launch_status();
}

// Whether every row of one array begins as far from a 16-byte boundary as the same row of another.
bool same_boundaries(const void* a, int64_t lda, const void* b, int64_t ldb, int dt, int64_t rows) {
  const int64_t size = static_cast<int64_t>(dtype_size(dt));
  const uintptr_t differ = reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b);
  return (differ & 15) == 0 && (rows <= 1 || ((lda - ldb) * size) % 16 == 0);
}

Boundaries boundaries_of(const void* a, int64_t ld, int dt, int64_t rows, int64_t width) {
  const int64_t size = static_cast<int64_t>(dtype_size(dt)), per = 16 / size;
  Boundaries b;
  b.shifted = rows > 1 && (ld * size) % 16 != 0;
  const int64_t most = b.shifted ? per - 1 : static_cast<int64_t>(reinterpret_cast<uintptr_t>(a) & 15) / size;
  b.chunks = static_cast<int>((width + most + per - 1) / per);
  b.edges = most != 0 || width % per != 0;
  return b;
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
  const LayerNormParams p{d_x, d_gamma, d_beta, d_y, d_mean, d_rstd, ldx, ldy, tokens, static_cast<int>(width), dt_w, eps,
                          same_boundaries(d_x, ldx, d_y, ldy, dt, tokens)};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Boundaries b = boundaries_of(d_x, ldx, dt, tokens, width);
  b.edges = b.edges || !p.chunked;
  return dt == SGDB_BF16 ? forward<BF16>(p, b, dev, s) : forward<float>(p, b, dev, s);
}

size_t sgdb_layer_norm_backward_workspace_bytes(int64_t tokens, int64_t width) {
  if (!sizes_ok(tokens, width)) return 0;
  // blocks come in multiples of 8 when rows are shifted against 16-byte boundaries
  const int64_t rows = tokens < 8 ? 8 : tokens < kMaxPartials ? tokens : kMaxPartials;
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
                                lddy, ldx, lddx, tokens, static_cast<int>(width), dt_w,
                                same_boundaries(d_x, ldx, d_dx, lddx, dt, tokens)};
    Boundaries b = boundaries_of(d_x, ldx, dt, tokens, width);
    b.edges = b.edges || !p.chunked;
    if (!same_boundaries(d_x, ldx, d_dy, lddy, dt, tokens)) b.chunks = 0;
    st = dt == SGDB_BF16 ? backward<BF16>(p, b, dev, s, &partials) : backward<float>(p, b, dev, s, &partials);
    if (st != SGDB_OK) return st;
  }
  if (!sums) return SGDB_OK;
  // no tokens: the sums are zero
  const unsigned blocks = static_cast<unsigned>((2 * width + 31) / 32);
  return launch_dependent(sum_partials_kernel, dim3(blocks), 32 * kSumWarps, 0, s, static_cast<const float*>(d_workspace), partials,
                          static_cast<int>(width), d_dgamma, d_dbeta, static_cast<int>(dt_g));
}

}  // extern "C"
