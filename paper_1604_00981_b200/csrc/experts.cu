// Tokens to their experts and back (declared in include/sgdb.h): the stable sort of the (token, choice)
// pairs by expert, the copy of the tokens into the experts' rows, the weighted sum back, and the gradients.
//
//   slot(t, j)   row of pair (t, j) among the experts' rows, which are sorted by (expert, t, j); -1: dropped
//   dispatch     xs[slot(t, j)] = x[t]
//   combine      out[t] = sum over j of w[t, j] ys[slot(t, j)]
//   backward     dys[slot(t, j)] = w[t, j] dout[t],  dw[t, j] = <ys[slot(t, j)], dout[t]>
//
// The sort is bound by latency, everything else by HBM: each row is read once and written once.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "sgdb_host.cuh"
#include "sgdb_rows.cuh"

namespace sgdb {
namespace {

namespace cg = cooperative_groups;

constexpr int kRouteThreads = 1024;
constexpr int kRouteWarps = kRouteThreads / 32;
constexpr int kRouteBlocks = 8;  // blocks of the cluster that sorts many pairs together

// The sort is one launch of one block, or of one cluster of 8 blocks that exchange their counts through
// distributed shared memory.  Each warp owns a contiguous run of pairs and counts its experts; the counts of
// the runs before it (warps, then blocks) and of the experts before give the first row of each (run, expert);
// a second walk through the run hands the rows out in order.  No atomics decide an order: the result is stable.
__global__ void __launch_bounds__(kRouteThreads) route_kernel(const int32_t* __restrict__ ids, int pairs, int E,
                                                             int32_t* __restrict__ offsets, int32_t* __restrict__ slot,
                                                             int32_t* __restrict__ source) {
  extern __shared__ int smem[];
  int* hist = smem;                       // [kRouteWarps][E]
  int* block_count = hist + kRouteWarps * E;  // [E]
  __shared__ int s_scan[32];
  cg::cluster_group cluster = cg::this_cluster();
  const int blocks = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned below = (1u << lane) - 1u;

  const int per_block = (pairs + blocks - 1) / blocks;
  const int per_warp = ((per_block + kRouteWarps - 1) / kRouteWarps + 31) & ~31;
  const long long first = static_cast<long long>(rank) * kRouteWarps * per_warp + static_cast<long long>(warp) * per_warp;
  const int begin = static_cast<int>(first < pairs ? first : pairs);
  const int end = static_cast<int>(first + per_warp < pairs ? first + per_warp : pairs);

  int* mine = hist + warp * E;
  for (int e = lane; e < E; e += 32) mine[e] = 0;
  __syncwarp();
  for (int base = begin; base < end; base += 32) {
    const int at = base + lane;
    int id = at < end ? ids[at] : -1;
    if (id < 0 || id >= E) id = -1;
    const unsigned same = __match_any_sync(0xffffffffu, id);
    if (id >= 0 && (same & below) == 0) mine[id] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  // per expert: the warps' counts become the counts of the warps before
  for (int e = tid; e < E; e += kRouteThreads) {
    int sum = 0;
    for (int w = 0; w < kRouteWarps; ++w) {
      const int n = hist[w * E + e];
      hist[w * E + e] = sum;
      sum += n;
    }
    block_count[e] = sum;
  }
  cluster.sync();
  // E <= kRouteThreads: thread e owns expert e
  int before = 0, total = 0;
  if (tid < E) {
    for (int r = 0; r < blocks; ++r) {
      const int n = cluster.map_shared_rank(block_count, r)[tid];
      if (r < rank) before += n;
      total += n;
    }
  }
  // exclusive scan of the experts' totals over the block
  int scan = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int n = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += n;
  }
  if (lane == 31) s_scan[warp] = scan;
  __syncthreads();
  if (warp == 0) {
    int v = s_scan[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int n = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += n;
    }
    s_scan[lane] = v;
  }
  __syncthreads();
  const int exclusive = scan - total + (warp > 0 ? s_scan[warp - 1] : 0);
  const int used = s_scan[31];
  if (tid < E) {
    if (rank == 0) {
      offsets[tid] = exclusive;
      if (tid == 0) offsets[E] = used;
    }
    for (int w = 0; w < kRouteWarps; ++w) hist[w * E + tid] += exclusive + before;
  }
  __syncthreads();
  for (int base = begin; base < end; base += 32) {
    const int at = base + lane;
    int id = at < end ? ids[at] : -1;
    if (id < 0 || id >= E) id = -1;
    const unsigned same = __match_any_sync(0xffffffffu, id);
    int to = -1;
    if (id >= 0) to = mine[id] + __popc(same & below);
    __syncwarp();
    if (id >= 0 && (same & below) == 0) mine[id] += __popc(same);
    __syncwarp();
    if (at < end) {
      slot[at] = to;
      if (to >= 0) source[to] = at;
    }
  }
  for (int r = used + rank * kRouteThreads + tid; r < pairs; r += blocks * kRouteThreads) source[r] = -1;
  cluster.sync();  // no block leaves while another may still read its counts
}

struct ExpertParams {
  const void *in, *ys;
  void* out;
  const int32_t *slot, *offsets;
  const float* weights;
  float* dweights;
  long long ld_in, ld_ys, ld_out;
  long long tokens;
  int D, k, E;
};

// Rows from the last used one on, which belong to no pair, are zero.
template <typename T, int V>
__device__ __forceinline__ void zero_tail(T* out, long long ld, const int32_t* offsets, int E, long long pairs, int D,
                                          long long warp, long long warps, int lane) {
  using Ch = Chunk<T, V>;
  long long used = offsets[E];
  if (used < 0) used = 0;
  for (long long r = used + warp; r < pairs; r += warps)
    for (int col = lane * V; col < D; col += 32 * V) Ch::store_raw(out + r * ld + col, Ch::zero());
}

// dispatch: a warp takes a piece of a token's row, reads it once and writes it k times.
constexpr int kCopyThreads = 256;
constexpr int kUnroll = 4;
template <typename T, int V>
__global__ void __launch_bounds__(kCopyThreads) dispatch_kernel(const ExpertParams p) {
  using Ch = Chunk<T, V>;
  const int lane = threadIdx.x & 31;
  const long long warp = (static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x) >> 5;
  const long long warps = (static_cast<long long>(gridDim.x) * kCopyThreads) >> 5;
  constexpr int kPiece = 32 * V * kUnroll;
  const int pieces = (p.D + kPiece - 1) / kPiece;
  const long long pairs = p.tokens * p.k;
  const T* x = static_cast<const T*>(p.in);
  T* xs = static_cast<T*>(p.out);
  for (long long w = warp; w < p.tokens * pieces; w += warps) {
    const long long t = w / pieces;
    const int col0 = static_cast<int>(w % pieces) * kPiece + lane * V;
    const int to = lane < p.k ? p.slot[t * p.k + lane] : -1;
    typename Ch::Raw v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (col0 + u * 32 * V < p.D) v[u] = Ch::load(x + t * p.ld_in + col0 + u * 32 * V);
    for (int j = 0; j < p.k; ++j) {
      const int row = __shfl_sync(0xffffffffu, to, j);
      if (row < 0 || row >= pairs) continue;
      T* out = xs + row * p.ld_out;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (col0 + u * 32 * V < p.D) Ch::store_raw(out + col0 + u * 32 * V, v[u]);
    }
  }
  zero_tail<T, V>(xs, p.ld_out, p.offsets, p.E, pairs, p.D, warp, warps, lane);
}

// combine: a warp takes a piece of a token's row and adds the k rows in the order of the choices, in fp32.
template <typename T, int V>
__global__ void __launch_bounds__(kCopyThreads) combine_kernel(const ExpertParams p) {
  using Ch = Chunk<T, V>;
  const int lane = threadIdx.x & 31;
  const long long warp = (static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x) >> 5;
  const long long warps = (static_cast<long long>(gridDim.x) * kCopyThreads) >> 5;
  constexpr int kPiece = 32 * V * kUnroll;
  const int pieces = (p.D + kPiece - 1) / kPiece;
  const long long pairs = p.tokens * p.k;
  const T* ys = static_cast<const T*>(p.in);
  T* out = static_cast<T*>(p.out);
  for (long long w = warp; w < p.tokens * pieces; w += warps) {
    const long long t = w / pieces;
    const int col0 = static_cast<int>(w % pieces) * kPiece + lane * V;
    int from = -1;
    float weight = 1.0f;
    if (lane < p.k) {
      from = p.slot[t * p.k + lane];
      if (p.weights != nullptr) weight = p.weights[t * p.k + lane];
    }
    float sum[kUnroll][V];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) sum[u][e] = 0.0f;
    for (int j = 0; j < p.k; ++j) {
      const int row = __shfl_sync(0xffffffffu, from, j);
      const float wj = __shfl_sync(0xffffffffu, weight, j);
      if (row < 0 || row >= pairs) continue;
      const T* y = ys + row * p.ld_in;
      typename Ch::Raw raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (col0 + u * 32 * V < p.D) raw[u] = Ch::load(y + col0 + u * 32 * V);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (col0 + u * 32 * V < p.D) {
          float v[V];
          Ch::unpack(raw[u], v);
#pragma unroll
          for (int e = 0; e < V; ++e) sum[u][e] = fmaf(wj, v[e], sum[u][e]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (col0 + u * 32 * V < p.D) Ch::store(out + t * p.ld_out + col0 + u * 32 * V, sum[u]);
  }
}

// combine's gradients: a warp takes a pair; the token's row of dout comes from L2 for all but its first pair.
template <typename T, int V>
__global__ void __launch_bounds__(kCopyThreads) combine_back_kernel(const ExpertParams p) {
  using Ch = Chunk<T, V>;
  const int lane = threadIdx.x & 31;
  const long long warp = (static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x) >> 5;
  const long long warps = (static_cast<long long>(gridDim.x) * kCopyThreads) >> 5;
  const long long pairs = p.tokens * p.k;
  const T* dout = static_cast<const T*>(p.in);
  const T* ys = static_cast<const T*>(p.ys);
  T* dys = static_cast<T*>(p.out);
  for (long long pair = warp; pair < pairs; pair += warps) {
    const int row = p.slot[pair];
    float dot = 0.0f;
    if (row >= 0 && row < pairs) {
      const T* g = dout + (pair / p.k) * p.ld_in;
      const float w = p.weights != nullptr ? p.weights[pair] : 1.0f;
      for (int col = lane * V; col < p.D; col += 32 * V * kUnroll) {
        typename Ch::Raw rg[kUnroll], ry[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (col + u * 32 * V < p.D) {
            rg[u] = Ch::load(g + col + u * 32 * V);
            ry[u] = Ch::load(ys + row * p.ld_ys + col + u * 32 * V);
          }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (col + u * 32 * V < p.D) {
            float a[V], b[V];
            Ch::unpack(rg[u], a);
            Ch::unpack(ry[u], b);
#pragma unroll
            for (int e = 0; e < V; ++e) {
              dot = fmaf(a[e], b[e], dot);
              a[e] *= w;
            }
            Ch::store(dys + row * p.ld_out + col + u * 32 * V, a);
          }
      }
    }
    dot = warp_sum(dot);
    if (lane == 0 && p.dweights != nullptr) p.dweights[pair] = dot;
  }
  zero_tail<T, V>(dys, p.ld_out, p.offsets, p.E, pairs, p.D, warp, warps, lane);
}

bool sizes_ok(int64_t tokens, int32_t k, int64_t width) {
  return tokens >= 0 && k >= 1 && k <= SGDB_MAX_CHOICES && width >= 1 && width <= SGDB_MAX_WIDTH && tokens <= SGDB_MAX_PAIRS / k;
}

// Blocks for `warps` units of work, at most eight per SM at a time: the kernels stride over the rest.
unsigned grid_for(long long warps, const DeviceInfo* dev) {
  const long long want = (warps + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  const long long cap = 8ll * dev->sms;
  return static_cast<unsigned>(want < 1 ? 1 : want < cap ? want : cap);
}

long long pieces_of(int D, int V) { return (D + 32 * V * kUnroll - 1) / (32 * V * kUnroll); }

}  // namespace
}  // namespace sgdb

using namespace sgdb;

extern "C" {

sgdb_status_t sgdb_route(const int32_t* d_expert, int64_t tokens, int32_t k, int32_t E, int32_t* d_offsets, int32_t* d_slot,
                         int32_t* d_source, void* stream) {
  if (!sizes_ok(tokens, k, 1) || E < 1 || E > SGDB_MAX_EXPERTS) return SGDB_ERR_INVALID_ARG;
  if (!array_ok(d_offsets, SGDB_F32)) return SGDB_ERR_INVALID_ARG;
  if (tokens > 0 && (!array_ok(d_expert, SGDB_F32) || !array_ok(d_slot, SGDB_F32) || !array_ok(d_source, SGDB_F32)))
    return SGDB_ERR_INVALID_ARG;
  const DeviceInfo* dev = nullptr;
  const sgdb_status_t st = device_info(&dev);
  if (st != SGDB_OK) return st;
  const int pairs = static_cast<int>(tokens * k);
  const size_t smem = static_cast<size_t>(kRouteWarps + 1) * static_cast<size_t>(E) * sizeof(int);
  static std::atomic<int> smem_allowed[kMaxDevices];
  if (static_cast<int>(smem) > smem_allowed[dev->index].load(std::memory_order_relaxed)) {
    if (cudaFuncSetAttribute(route_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess)
      return launch_status();
    smem_allowed[dev->index].store(static_cast<int>(smem), std::memory_order_relaxed);
  }
  const int blocks = pairs > 4 * kRouteThreads ? kRouteBlocks : 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kRouteThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = blocks;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  (void)cudaLaunchKernelEx(&cfg, route_kernel, d_expert, pairs, static_cast<int>(E), d_offsets, d_slot, d_source);
  return launch_status();
}

sgdb_status_t sgdb_dispatch(const void* d_x, sgdb_dtype_t dt, int64_t tokens, int64_t width, int64_t ldx, const int32_t* d_slot,
                            int32_t k, const int32_t* d_offsets, int32_t E, void* d_xs, int64_t ldxs, void* stream) {
  if (!dtype_ok(dt) || !sizes_ok(tokens, k, width) || E < 1 || E > SGDB_MAX_EXPERTS || ldx < width || ldxs < width)
    return SGDB_ERR_INVALID_ARG;
  if (tokens == 0) return SGDB_OK;
  if (!array_ok(d_x, dt) || !array_ok(d_xs, dt) || !array_ok(d_slot, SGDB_F32) || !array_ok(d_offsets, SGDB_F32))
    return SGDB_ERR_INVALID_ARG;
  const DeviceInfo* dev = nullptr;
  const sgdb_status_t st = device_info(&dev);
  if (st != SGDB_OK) return st;
  ExpertParams p{};
  p.in = d_x, p.out = d_xs, p.slot = d_slot, p.offsets = d_offsets;
  p.ld_in = ldx, p.ld_out = ldxs, p.tokens = tokens, p.D = static_cast<int>(width), p.k = k, p.E = E;
  const bool vec = rows_aligned16(d_x, ldx, dt) && rows_aligned16(d_xs, ldxs, dt) &&
                   (width * static_cast<int64_t>(dtype_size(dt))) % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const auto launch = [&](auto kernel, int V) { kernel<<<grid_for(tokens * pieces_of(p.D, V), dev), kCopyThreads, 0, s>>>(p); };
  if (dt == SGDB_BF16)
    vec ? launch(dispatch_kernel<BF16, 8>, 8) : launch(dispatch_kernel<BF16, 1>, 1);
  else
    vec ? launch(dispatch_kernel<float, 4>, 4) : launch(dispatch_kernel<float, 1>, 1);
  return launch_status();
}

sgdb_status_t sgdb_combine(const void* d_ys, sgdb_dtype_t dt, int64_t tokens, int64_t width, int64_t ldys, const int32_t* d_slot,
                           int32_t k, const float* d_weights, void* d_out, int64_t ldout, void* stream) {
  if (!dtype_ok(dt) || !sizes_ok(tokens, k, width) || ldys < width || ldout < width) return SGDB_ERR_INVALID_ARG;
  if (tokens == 0) return SGDB_OK;
  if (!array_ok(d_ys, dt) || !array_ok(d_out, dt) || !array_ok(d_slot, SGDB_F32)) return SGDB_ERR_INVALID_ARG;
  if (d_weights != nullptr && !array_ok(d_weights, SGDB_F32)) return SGDB_ERR_INVALID_ARG;
  const DeviceInfo* dev = nullptr;
  const sgdb_status_t st = device_info(&dev);
  if (st != SGDB_OK) return st;
  ExpertParams p{};
  p.in = d_ys, p.out = d_out, p.slot = d_slot, p.weights = d_weights;
  p.ld_in = ldys, p.ld_out = ldout, p.tokens = tokens, p.D = static_cast<int>(width), p.k = k;
  const bool vec = rows_aligned16(d_ys, ldys, dt) && rows_aligned16(d_out, ldout, dt) &&
                   (width * static_cast<int64_t>(dtype_size(dt))) % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const auto launch = [&](auto kernel, int V) { kernel<<<grid_for(tokens * pieces_of(p.D, V), dev), kCopyThreads, 0, s>>>(p); };
  if (dt == SGDB_BF16)
    vec ? launch(combine_kernel<BF16, 8>, 8) : launch(combine_kernel<BF16, 1>, 1);
  else
    vec ? launch(combine_kernel<float, 4>, 4) : launch(combine_kernel<float, 1>, 1);
  return launch_status();
}

sgdb_status_t sgdb_combine_backward(const void* d_dout, int64_t lddout, const void* d_ys, int64_t ldys, sgdb_dtype_t dt,
                                    int64_t tokens, int64_t width, const int32_t* d_slot, int32_t k, const float* d_weights,
                                    const int32_t* d_offsets, int32_t E, void* d_dys, int64_t lddys, float* d_dweights,
                                    void* stream) {
  if (!dtype_ok(dt) || !sizes_ok(tokens, k, width) || E < 1 || E > SGDB_MAX_EXPERTS) return SGDB_ERR_INVALID_ARG;
  if (lddout < width || ldys < width || lddys < width) return SGDB_ERR_INVALID_ARG;
  if (tokens == 0) return SGDB_OK;
  if (!array_ok(d_dout, dt) || !array_ok(d_ys, dt) || !array_ok(d_dys, dt) || !array_ok(d_slot, SGDB_F32) ||
      !array_ok(d_offsets, SGDB_F32))
    return SGDB_ERR_INVALID_ARG;
  if ((d_weights != nullptr && !array_ok(d_weights, SGDB_F32)) || (d_dweights != nullptr && !array_ok(d_dweights, SGDB_F32)))
    return SGDB_ERR_INVALID_ARG;
  const DeviceInfo* dev = nullptr;
  const sgdb_status_t st = device_info(&dev);
  if (st != SGDB_OK) return st;
  ExpertParams p{};
  p.in = d_dout, p.ys = d_ys, p.out = d_dys, p.slot = d_slot, p.offsets = d_offsets, p.weights = d_weights;
  p.dweights = d_dweights;
  p.ld_in = lddout, p.ld_ys = ldys, p.ld_out = lddys, p.tokens = tokens, p.D = static_cast<int>(width), p.k = k, p.E = E;
  const bool vec = rows_aligned16(d_dout, lddout, dt) && rows_aligned16(d_ys, ldys, dt) && rows_aligned16(d_dys, lddys, dt) &&
                   (width * static_cast<int64_t>(dtype_size(dt))) % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const auto launch = [&](auto kernel) { kernel<<<grid_for(tokens * k, dev), kCopyThreads, 0, s>>>(p); };
  if (dt == SGDB_BF16)
    vec ? launch(combine_back_kernel<BF16, 8>) : launch(combine_back_kernel<BF16, 1>);
  else
    vec ? launch(combine_back_kernel<float, 4>) : launch(combine_back_kernel<float, 1>);
  return launch_status();
}

}  // extern "C"
