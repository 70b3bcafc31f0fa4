// The balance loss of a layer of experts with the experts' counts, and its gradient (declared in include/sgdb.h).
//
//   p_t = softmax of token t's logits,  c_e = pairs of expert e among the n tokens that count
//   loss = sum over e of E c_e / (n n k) P_e  with  P_e = sum over the tokens of p_te
//   slope_e = E (c_e - mean of c) / (n n k),  gradient  dx_te = g p_te (slope_e - sum over j of p_tj slope_j)
//
// A row's probabilities add up to one, so what the slopes have in common has no part in the gradient; without it the difference
// loses no digits when the experts' counts are nearly alike, as they are when the loss has done its work.
//
// One pass over the logits each way; the backward pass takes the softmax anew from the row that it has to read anyway, which
// is more exact than a stored logarithm and needs no memory per token.  Sums over the tokens go through a partial sum per
// block, which a second kernel adds in the blocks' order.
#include <cuda_runtime.h>

#include <type_traits>

#include "sgdb_host.cuh"
#include "sgdb_rows.cuh"

namespace sgdb {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxBlocks = 128;       // of the forward pass: partial sums per expert
constexpr int kFinalThreads = 1024;

struct BalanceParams {
  const void* logits;
  long long ld, tokens;
  int E, k;
  const int32_t* expert;
  const uint8_t* mask;  // or null: all tokens count
  float* sums;          // [blocks][E]
  int32_t* counts;      // [blocks][E + 1]: pairs of each expert, and tokens that count
  const float *grad, *slope;
  void* dlogits;
  long long ld_out;
};

// A token belongs to a group of L lanes, each of which has CHUNKS times V columns: V columns at (c * L + lane) * V.
template <typename T, int L, int CHUNKS>
struct Row {
  static constexpr int V = kChunk16<T>;
  float x[CHUNKS * V];
  template <bool VEC>
  __device__ __forceinline__ void load(const T* row, int lane, int E) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int col = (c * L + lane) * V;
      float v[V];
      if (VEC && col + V <= E) {
        GradTraits<T>::unpack(*reinterpret_cast<const uint4*>(row + col), v);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = col + e < E ? widen<T>(row[col + e]) : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) x[c * V + e] = v[e];
    }
  }
  static __device__ __forceinline__ float over_group(float v, bool largest) {
#pragma unroll
    for (int o = 1; o < L; o *= 2) {
      const float w = __shfl_xor_sync(0xffffffffu, v, o);
      v = largest ? fmaxf(v, w) : v + w;
    }
    return v;
  }
  // x becomes the softmax; a row without any probability (all -inf) becomes zeros, one with NaN or +inf NaN
  __device__ __forceinline__ void softmax() {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < CHUNKS * V; ++i) top = fmaxf(top, x[i]);
    top = over_group(top, true);
    if (top == -INFINITY) top = 0.0f;  // exp(-inf - 0) is zero; NaN, which fmaxf passes over, stays in the sum
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < CHUNKS * V; ++i) {
      x[i] = expf(x[i] - top);
      sum += x[i];
    }
    sum = over_group(sum, false);
    const float r = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int i = 0; i < CHUNKS * V; ++i) x[i] *= r;
  }
};

template <typename T, int L, int CHUNKS, bool VEC>
__global__ void __launch_bounds__(kThreads) balance_kernel(const BalanceParams p) {
  using R = Row<T, L, CHUNKS>;
  constexpr int V = R::V, kTokens = 32 / L;  // tokens of a warp at a time
  extern __shared__ float s_dynamic[];
  float* s_sums = s_dynamic;  // [warps][columns of a warp's lanes], then the block's counts
  constexpr int kColumns = L * CHUNKS * V;
  int32_t* s_counts = reinterpret_cast<int32_t*>(s_dynamic + kWarps * kColumns);  // [E + 1]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_group = lane % L;
  for (int e = threadIdx.x; e <= p.E; e += kThreads) s_counts[e] = 0;
  __syncthreads();
  pdl_wait();
  const T* logits = static_cast<const T*>(p.logits);
  float sum[CHUNKS * V];
#pragma unroll
  for (int i = 0; i < CHUNKS * V; ++i) sum[i] = 0.0f;
  int counted = 0;
  // a warp's share is contiguous rows of several groups; whole warps stay together for the sums over groups
  const long long step = static_cast<long long>(gridDim.x) * kWarps * kTokens;
  for (long long t0 = (static_cast<long long>(blockIdx.x) * kWarps + warp) * kTokens; t0 < p.tokens; t0 += step) {
    const long long t = t0 + lane / L;
    const bool counts = t < p.tokens && (p.mask == nullptr || p.mask[t] != 0);
    R row;
    if (counts) {
      row.template load<VEC>(logits + t * p.ld, in_group, p.E);
    } else {
#pragma unroll
      for (int i = 0; i < CHUNKS * V; ++i) row.x[i] = -INFINITY;
    }
    row.softmax();
#pragma unroll
    for (int i = 0; i < CHUNKS * V; ++i) sum[i] += row.x[i];
    if (counts) {
      if (in_group == 0) ++counted;
      for (int j = in_group; j < p.k; j += L) {
        const int e = p.expert[t * p.k + j];
        if (e >= 0 && e < p.E) atomicAdd(&s_counts[e], 1);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < CHUNKS * V; ++i) {
#pragma unroll
    for (int o = L; o < 32; o *= 2) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
  }
  if (lane < L) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int e = 0; e < V; ++e) s_sums[warp * kColumns + (c * L + lane) * V + e] = sum[c * V + e];
  }
  counted = __reduce_add_sync(0xffffffffu, counted);
  if (lane == 0 && counted > 0) atomicAdd(&s_counts[p.E], counted);
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += kThreads) {
    float total = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) total += s_sums[w * kColumns + e];
    p.sums[static_cast<long long>(blockIdx.x) * p.E + e] = total;
  }
  for (int e = threadIdx.x; e <= p.E; e += kThreads) p.counts[static_cast<long long>(blockIdx.x) * (p.E + 1) + e] = s_counts[e];
}

// The blocks' sums, in their order: a thread for each expert (several where there are few, each with a run of the blocks).
__global__ void __launch_bounds__(kFinalThreads) balance_final_kernel(const float* __restrict__ sums, const int32_t* __restrict__ counts, int blocks,
                                                                      int E, int k, float* __restrict__ loss, int32_t* __restrict__ total_counts,
                                                                      float* __restrict__ slope) {
  __shared__ float s_sum[kFinalThreads];
  __shared__ int32_t s_count[kFinalThreads];
  __shared__ double s_loss[kFinalThreads / 32];
  __shared__ int32_t s_tokens;
  __shared__ unsigned long long s_pairs;
  pdl_wait();
  int columns = 32;
  while (columns < E) columns *= 2;
  const int runs = kFinalThreads / columns, e = threadIdx.x % columns, run = threadIdx.x / columns;
  const int per_run = (blocks + runs - 1) / runs;
  float sum = 0.0f;
  int32_t count = 0;
  if (e < E) {
#pragma unroll 8
    for (int b = run * per_run; b < min(blocks, (run + 1) * per_run); ++b) {
      sum += sums[static_cast<long long>(b) * E + e];
      count += counts[static_cast<long long>(b) * (E + 1) + e];
    }
  }
  s_sum[threadIdx.x] = sum;
  s_count[threadIdx.x] = count;
  if (threadIdx.x == 0) s_pairs = 0;
  __syncthreads();
  const int here = __reduce_add_sync(0xffffffffu, count);
  if ((threadIdx.x & 31) == 0) atomicAdd(&s_pairs, static_cast<unsigned long long>(here));
  if (threadIdx.x < 32) {
    int n = 0;
    for (int b = threadIdx.x; b < blocks; b += 32) n += counts[static_cast<long long>(b) * (E + 1) + E];
    n = __reduce_add_sync(0xffffffffu, n);
    if (threadIdx.x == 0) s_tokens = n;
  }
  __syncthreads();
  double part = 0.0;
  if (run == 0 && e < E) {
    for (int r = 1; r < runs; ++r) {
      sum += s_sum[r * columns + e];
      count += s_count[r * columns + e];
    }
    const double n = s_tokens, factor = s_tokens > 0 ? E / (n * n * k) : 0.0;
    total_counts[e] = count;
    slope[e] = static_cast<float>(factor * (count - static_cast<double>(s_pairs) / E));
    part = factor * count * sum;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
  if ((threadIdx.x & 31) == 0) s_loss[threadIdx.x >> 5] = part;
  __syncthreads();
  if (threadIdx.x == 0) {
    part = 0.0;
    for (int w = 0; w < kFinalThreads / 32; ++w) part += s_loss[w];
    *loss = static_cast<float>(part);
  }
}

template <typename T, int L, int CHUNKS, bool VEC>
__global__ void __launch_bounds__(kThreads) balance_back_kernel(const BalanceParams p) {
  using R = Row<T, L, CHUNKS>;
  constexpr int V = R::V, kTokens = 32 / L;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_group = lane % L;
  pdl_wait();
  const float g = *p.grad;
  float slope[CHUNKS * V];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int col = (c * L + in_group) * V + e;
      slope[c * V + e] = col < p.E ? p.slope[col] : 0.0f;
    }
  const long long step = static_cast<long long>(gridDim.x) * kWarps * kTokens;
  for (long long t0 = (static_cast<long long>(blockIdx.x) * kWarps + warp) * kTokens; t0 < p.tokens; t0 += step) {
    const long long t = t0 + lane / L;
    const bool counts = t < p.tokens && (p.mask == nullptr || p.mask[t] != 0);
    R row;
    if (counts) {
      row.template load<VEC>(static_cast<const T*>(p.logits) + t * p.ld, in_group, p.E);
    } else {
#pragma unroll
      for (int i = 0; i < CHUNKS * V; ++i) row.x[i] = -INFINITY;
    }
    row.softmax();
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < CHUNKS * V; ++i) dot = fmaf(row.x[i], slope[i], dot);
    dot = R::over_group(dot, false);
    if (t >= p.tokens) continue;  // behind the last vote of the loop's body
    T* out = static_cast<T*>(p.dlogits) + t * p.ld_out;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int col = (c * L + in_group) * V;
      float v[V];
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = counts ? g * row.x[c * V + e] * (slope[c * V + e] - dot) : 0.0f;
      if (VEC && col + V <= p.E) {
        *reinterpret_cast<uint4*>(out + col) = Chunk<T, V>::pack(v);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (col + e < p.E) out[col + e] = narrow<T>(v[e]);
      }
    }
  }
}

// Calls f with the element type, the lanes of a token, the chunks of a lane and whether chunks may be read whole.
template <typename F>
sgdb_status_t with_row(int dt, int E, bool vec, F&& f) {
  using std::bool_constant;
  using std::integral_constant;
  const auto vectored = [&](auto one, auto lanes, auto chunks) {
    return vec ? f(one, lanes, chunks, bool_constant<true>{}) : f(one, lanes, chunks, bool_constant<false>{});
  };
  const auto shaped = [&](auto one) {
    constexpr int V = kChunk16<decltype(one)>;
    const int chunks = (E + V - 1) / V;
    const integral_constant<int, 1> c1;
    if (chunks <= 2) return vectored(one, integral_constant<int, 2>{}, c1);
    if (chunks <= 8) return vectored(one, integral_constant<int, 8>{}, c1);
    if (chunks <= 32) return vectored(one, integral_constant<int, 32>{}, c1);
    if (chunks <= 64) return vectored(one, integral_constant<int, 32>{}, integral_constant<int, 2>{});
    if constexpr (V == 4) {
      if (chunks > 128) return vectored(one, integral_constant<int, 32>{}, integral_constant<int, 8>{});
    }
    return vectored(one, integral_constant<int, 32>{}, integral_constant<int, 4>{});
  };
  return dt == SGDB_BF16 ? shaped(BF16{}) : shaped(float{});
}

bool sizes_ok(int64_t tokens, int32_t k, int32_t E) {
  return tokens >= 0 && k >= 1 && k <= SGDB_MAX_CHOICES && E >= 1 && E <= SGDB_MAX_EXPERTS && tokens <= SGDB_MAX_PAIRS / k;
}

int blocks_for(int64_t tokens, int per_block, int most) {
  const int64_t want = (tokens + per_block - 1) / per_block;
  return static_cast<int>(want < 1 ? 1 : want < most ? want : most);
}

}  // namespace
}  // namespace sgdb

using namespace sgdb;

extern "C" {

size_t sgdb_balance_loss_workspace_bytes(int64_t tokens, int32_t E) {
  if (!sizes_ok(tokens, 1, E)) return 0;
  return static_cast<size_t>(kMaxBlocks) * (2 * E + 1) * 4;
}

sgdb_status_t sgdb_balance_loss(const void* d_logits, sgdb_dtype_t dt, int64_t tokens, int32_t E, int64_t ld, const int32_t* d_expert, int32_t k,
                                const uint8_t* d_mask, float* d_loss, int32_t* d_counts, float* d_slope, void* d_workspace, size_t workspace_bytes,
                                void* stream) {
  if (!dtype_ok(dt) || !sizes_ok(tokens, k, E) || ld < E) return SGDB_ERR_INVALID_ARG;
  if (!array_ok(d_loss, SGDB_F32) || !array_ok(d_counts, SGDB_F32) || !array_ok(d_slope, SGDB_F32)) return SGDB_ERR_INVALID_ARG;
  if (!array_ok(d_workspace, SGDB_F32) || workspace_bytes < sgdb_balance_loss_workspace_bytes(tokens, E)) return SGDB_ERR_INVALID_ARG;
  if (tokens > 0 && (!array_ok(d_logits, dt) || !array_ok(d_expert, SGDB_F32))) return SGDB_ERR_INVALID_ARG;
  BalanceParams p{};
  p.logits = d_logits, p.ld = ld, p.tokens = tokens, p.E = E, p.k = k, p.expert = d_expert, p.mask = d_mask;
  p.sums = static_cast<float*>(d_workspace);
  p.counts = reinterpret_cast<int32_t*>(p.sums + static_cast<size_t>(kMaxBlocks) * E);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int blocks = 1;
  const sgdb_status_t st = with_row(dt, E, rows_aligned16(d_logits, ld, dt), [&](auto one, auto lanes, auto chunks, auto vec) {
    using T = decltype(one);
    blocks = blocks_for(tokens, kWarps * 32 / lanes(), kMaxBlocks);
    const size_t smem = (static_cast<size_t>(kWarps) * lanes() * chunks() * kChunk16<T> + E + 1) * 4;
    return launch_dependent(balance_kernel<T, lanes(), chunks(), vec()>, dim3(blocks), kThreads, smem, s, p);
  });
  if (st != SGDB_OK) return st;
  return launch_dependent(balance_final_kernel, dim3(1), kFinalThreads, 0, s, static_cast<const float*>(p.sums), static_cast<const int32_t*>(p.counts), blocks,
                          static_cast<int>(E), static_cast<int>(k), d_loss, d_counts, d_slope);
}

sgdb_status_t sgdb_balance_loss_backward(const float* d_grad, const void* d_logits, sgdb_dtype_t dt, int64_t tokens, int32_t E, int64_t ld,
                                         const uint8_t* d_mask, const float* d_slope, void* d_dlogits, int64_t ldd, void* stream) {
  if (!dtype_ok(dt) || !sizes_ok(tokens, 1, E) || ld < E || ldd < E) return SGDB_ERR_INVALID_ARG;
  if (tokens == 0) return SGDB_OK;
  if (!array_ok(d_grad, SGDB_F32) || !array_ok(d_logits, dt) || !array_ok(d_slope, SGDB_F32) || !array_ok(d_dlogits, dt)) return SGDB_ERR_INVALID_ARG;
  const DeviceInfo* dev = nullptr;
  const sgdb_status_t st = device_info(&dev);
  if (st != SGDB_OK) return st;
  BalanceParams p{};
  p.logits = d_logits, p.ld = ld, p.tokens = tokens, p.E = E, p.mask = d_mask, p.grad = d_grad, p.slope = d_slope, p.dlogits = d_dlogits, p.ld_out = ldd;
  const bool vec = rows_aligned16(d_logits, ld, dt) && rows_aligned16(d_dlogits, ldd, dt);
  return with_row(dt, E, vec, [&](auto one, auto lanes, auto chunks, auto is_vec) {
    const int blocks = blocks_for(tokens, kWarps * 32 / lanes(), 8 * dev->sms);
    return launch_dependent(balance_back_kernel<decltype(one), lanes(), chunks(), is_vec()>, dim3(blocks), kThreads, 0, static_cast<cudaStream_t>(stream), p);
  });
}

}  // extern "C"
