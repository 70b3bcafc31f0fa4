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

#include <type_traits>

#include "sgdb_host.cuh"
#include "sgdb_rows.cuh"

namespace sgdb {
namespace {

namespace cg = cooperative_groups;

constexpr int kRouteThreads = 512;
constexpr int kRouteWarps = kRouteThreads / 32;
constexpr int kRouteHeld = 4;    // groups of 128 pairs whose loads are in flight together
constexpr int kRouteList = 512;  // pairs of its expert that a warp can note down
constexpr int kRouteCluster = 8; // blocks that share an expert, at most

// The sort: a block, or a cluster of blocks where there are few experts, for each expert.  It looks through all pairs (which
// come from L2 for all but the first), counts those of lower experts, whose rows come before its own, and hands out its
// rows in the pairs' order: a warp owns a contiguous run of pairs, votes tell the lanes their places, and the
// warp notes its pairs down until the counts before it are known.  E times the work of a counting sort, spread over all SMs.
// 65,536 pairs to 64 experts: 8.3 us (1024 threads: 11.5); with the counting
// sort in one cluster of 8 blocks 14.5 us.
__global__ void __launch_bounds__(kRouteThreads) route_kernel(const int32_t* __restrict__ ids, int pairs, int E, bool wide,
                                                             int32_t* __restrict__ offsets, int32_t* __restrict__ slot,
                                                             int32_t* __restrict__ source) {
  __shared__ int s_equal[kRouteWarps], s_less[kRouteWarps];
  __shared__ __align__(8) int s_block[2];
  __shared__ int s_list[kRouteWarps][kRouteList];
  pdl_launch_dependents();
  pdl_wait();
  cg::cluster_group cluster = cg::this_cluster();
  const int blocks = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
  const int e = blockIdx.x / blocks, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const unsigned below = (1u << lane) - 1u;
  const int runs = blocks * kRouteWarps;
  const int per_warp = ((pairs + runs - 1) / runs + 127) & ~127;
  const long long first = static_cast<long long>(rank * kRouteWarps + warp) * per_warp;
  const int begin = static_cast<int>(first < pairs ? first : pairs);
  const int end = static_cast<int>(first + per_warp < pairs ? first + per_warp : pairs);

  // four consecutive pairs of this lane; -1 where there is none (which no expert is)
  const auto load = [&](int at) {
    if (wide && at + 4 <= end) return *reinterpret_cast<const int4*>(ids + at);
    return make_int4(at < end ? ids[at] : -1, at + 1 < end ? ids[at + 1] : -1, at + 2 < end ? ids[at + 2] : -1,
                     at + 3 < end ? ids[at + 3] : -1);
  };
  // the warp's pairs of expert e in order, from number `next` on: found(pair, number)
  const auto walk = [&](int next, auto&& every, auto&& found) {
    for (int base = begin; base < end; base += 128 * kRouteHeld) {
      int4 v[kRouteHeld];
#pragma unroll
      for (int h = 0; h < kRouteHeld; ++h) v[h] = load(base + h * 128 + lane * 4);
#pragma unroll
      for (int h = 0; h < kRouteHeld; ++h) {
        const int at = base + h * 128 + lane * 4, id[4] = {v[h].x, v[h].y, v[h].z, v[h].w};
        int to = next;
        bool mine = false;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          every(at + c, id[c]);
          const unsigned votes = __ballot_sync(0xffffffffu, id[c] == e);
          to += __popc(votes & below);
          next += __popc(votes);
          mine |= id[c] == e;
        }
        if (mine) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (id[c] == e) found(at + c, to++);
        }
      }
    }
    return next;
  };

  int less = 0;
  const int equal = walk(
      0,
      [&](int at, int id) {
        less += static_cast<unsigned>(id) < static_cast<unsigned>(e);  // negative ids are large
        if (e == 0 && at < end && (id < 0 || id >= E)) slot[at] = -1;  // the first expert's blocks write down who is dropped
      },
      [&](int pair, int number) {
        if (number < kRouteList) s_list[warp][number] = pair;
      });
  less = __reduce_add_sync(0xffffffffu, less);
  if (lane == 0) {
    s_equal[warp] = equal;
    s_less[warp] = less;
  }
  __syncthreads();
  const int before_here = __reduce_add_sync(0xffffffffu, lane < warp ? s_equal[lane] : 0);
  int lower = __reduce_add_sync(0xffffffffu, lane < kRouteWarps ? s_less[lane] : 0),
      mine = __reduce_add_sync(0xffffffffu, lane < kRouteWarps ? s_equal[lane] : 0), before = before_here;
  if (blocks > 1) {
    if (threadIdx.x == 0) {
      s_block[0] = lower;
      s_block[1] = mine;
    }
    cluster.sync();
    const int2 theirs = lane < blocks ? *reinterpret_cast<const int2*>(cluster.map_shared_rank(s_block, lane)) : make_int2(0, 0);
    lower = __reduce_add_sync(0xffffffffu, theirs.x);
    mine = __reduce_add_sync(0xffffffffu, theirs.y);
    before += __reduce_add_sync(0xffffffffu, lane < rank ? theirs.y : 0);
    cluster.sync();  // no block leaves while another may still read its counts
  }
  const int row0 = lower + before;
  if (equal <= kRouteList) {
    __syncwarp();
    for (int i = lane; i < equal; i += 32) {
      const int pair = s_list[warp][i];
      slot[pair] = row0 + i;
      source[row0 + i] = pair;
    }
  } else {
    walk(row0, [](int, int) {},
         [&](int pair, int row) {
           slot[pair] = row;
           source[row] = pair;
         });
  }
  if (rank == 0 && threadIdx.x == 0) offsets[e] = lower;
  if (e == E - 1) {  // the last one, what is not in use
    const int used = lower + mine;
    if (rank == 0 && threadIdx.x == 0) offsets[E] = used;
    for (int r = used + rank * kRouteThreads + threadIdx.x; r < pairs; r += blocks * kRouteThreads) source[r] = -1;
  }
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
  int pieces;  // of a row: 32 * U chunks each
};

// Rows are written in chunks of 16 bytes on 16-byte boundaries.  A row that is ALIGNED begins and ends on them; any other
// begins `shift` elements into its first chunk, and the elements of its first and last chunk are written one by one.

// 16 bytes from any element on: the one or two chunks on 16-byte boundaries that hold them are loaded first, so that many
// can be under way, and put together when they are used.
template <typename T, bool ALIGNED>
struct Window {
  uint4 lo, hi;
  uint32_t off;
  // Of the elements from p on, `first` to `last` - 1 exist; only chunks that hold some of these are loaded.
  __device__ __forceinline__ void load(const T* p, int first, int last) {
    if (ALIGNED) {
      lo = __ldcs(reinterpret_cast<const uint4*>(p));
      return;
    }
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    off = at & 15;
    const uint4* chunk = reinterpret_cast<const uint4*>(at - off);
    lo = hi = make_uint4(0, 0, 0, 0);
    if (first * static_cast<int>(sizeof(T)) + static_cast<int>(off) < 16) lo = chunk[0];
    if (last * static_cast<int>(sizeof(T)) + static_cast<int>(off) > 16) hi = chunk[1];
  }
  __device__ __forceinline__ uint4 get() const {
    if (ALIGNED) return lo;
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    const bool by8 = off & 8, by4 = off & 4, by2 = off & 2;
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = by8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = by4 ? w[i + 1] : w[i];
    if (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], by2 ? 16 : 0);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

template <typename T, bool ALIGNED>
__device__ __forceinline__ void store_chunk(T* p, int first, int last, const uint4& v) {
  constexpr int V = kChunk16<T>;
  if (ALIGNED || (first == 0 && last == V)) {
    __stcs(reinterpret_cast<uint4*>(p), v);
    return;
  }
  union {
    uint4 all;
    T one[V];
  } u;
  u.all = v;
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e >= first && e < last) p[e] = u.one[e];
}

// A lane's chunk of a row that is written: number `index` of the row's chunks.
template <typename T, bool ALIGNED>
struct Place {
  int col, first, last;  // column of its first element (negative before the row), elements that exist
  __device__ __forceinline__ Place(const T* row, int index, int D) {
    constexpr int V = kChunk16<T>;
    col = index * V - (ALIGNED ? 0 : shift_of(row));
    first = !ALIGNED && col < 0 ? -col : 0;
    last = !ALIGNED && col + V > D ? D - col : V;
  }
  __device__ __forceinline__ bool exists(int D) const { return col < D; }
};

constexpr int kCopyThreads = 256;

// Rows from the last used one on, which belong to no pair, are zero.
template <typename T, bool ALIGNED>
__device__ __forceinline__ void zero_tail(T* out, long long ld, const int32_t* offsets, int E, long long pairs, int D,
                                          long long warp, long long warps, int lane) {
  long long used = offsets[E];
  if (used < 0) used = 0;
  for (long long r = used + warp; r < pairs; r += warps) {
    T* row = out + r * ld;
    for (int i = lane;; i += 32) {
      const Place<T, ALIGNED> at(row, i, D);
      if (!at.exists(D)) break;
      store_chunk<T, ALIGNED>(row + at.col, at.first, at.last, make_uint4(0, 0, 0, 0));
    }
  }
}

// dispatch: a warp takes a piece of a token's row, reads it (from cache after the first time, when rows are not aligned
// and each copy needs its own chunks) and writes it k times.
template <typename T, bool ALIGNED, int U>
__global__ void __launch_bounds__(kCopyThreads) dispatch_kernel(const ExpertParams p) {
  const int lane = threadIdx.x & 31;
  const long long warp = (static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x) >> 5;
  const long long warps = (static_cast<long long>(gridDim.x) * kCopyThreads) >> 5;
  const long long pairs = p.tokens * p.k;
  const T* x = static_cast<const T*>(p.in);
  T* xs = static_cast<T*>(p.out);
  // While the sort before this kernel runs, the tokens come into L2, whose contents are never stale (8192x2048 bf16, 8 of 64
  // experts: sort and dispatch 60 -> 56 us).
  for (long long w = warp; w < p.tokens * p.pieces && w < 4 * warps; w += warps) {
    const T* at = x + (w / p.pieces) * p.ld_in + (w % p.pieces) * 32 * U * kChunk16<T>;
    const long long left = p.D - (w % p.pieces) * 32 * U * kChunk16<T>;
    if (lane * (128 / static_cast<int>(sizeof(T))) < left && lane * 128 < 32 * U * 16)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(at + lane * (128 / static_cast<int>(sizeof(T)))));
  }
  pdl_wait();
  for (long long w = warp; w < p.tokens * p.pieces; w += warps) {
    const long long t = w / p.pieces;
    const int chunk0 = static_cast<int>(w % p.pieces) * 32 * U + lane;
    const int to = lane < p.k ? p.slot[t * p.k + lane] : -1;
    const T* in = x + t * p.ld_in;
    Window<T, ALIGNED> v[U];
    if (ALIGNED) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const Place<T, ALIGNED> at(in, chunk0 + 32 * u, p.D);
        if (at.exists(p.D)) v[u].load(in + at.col, at.first, at.last);
      }
    }
    for (int j = 0; j < p.k; ++j) {
      const int row = __shfl_sync(0xffffffffu, to, j);
      if (row < 0 || row >= pairs) continue;
      T* out = xs + row * p.ld_out;
      if (!ALIGNED) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const Place<T, ALIGNED> at(out, chunk0 + 32 * u, p.D);
          if (at.exists(p.D)) v[u].load(in + at.col, at.first, at.last);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const Place<T, ALIGNED> at(out, chunk0 + 32 * u, p.D);
        if (at.exists(p.D)) store_chunk<T, ALIGNED>(out + at.col, at.first, at.last, v[u].get());
      }
    }
  }
  zero_tail<T, ALIGNED>(xs, p.ld_out, p.offsets, p.E, pairs, p.D, warp, warps, lane);
}

// combine: a warp takes a piece of a token's row and adds the k rows in the order of the choices, in fp32.
template <typename T, bool ALIGNED, int U>
__global__ void __launch_bounds__(kCopyThreads, ALIGNED ? 1 : 4) combine_kernel(const ExpertParams p) {
  constexpr int V = kChunk16<T>;
  const int lane = threadIdx.x & 31;
  const long long warp = (static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x) >> 5;
  const long long warps = (static_cast<long long>(gridDim.x) * kCopyThreads) >> 5;
  const long long pairs = p.tokens * p.k;
  const T* ys = static_cast<const T*>(p.in);
  pdl_wait();
  for (long long w = warp; w < p.tokens * p.pieces; w += warps) {
    const long long t = w / p.pieces;
    const int chunk0 = static_cast<int>(w % p.pieces) * 32 * U + lane;
    T* out = static_cast<T*>(p.out) + t * p.ld_out;
    int from = -1;
    float weight = 1.0f;
    if (lane < p.k) {
      from = p.slot[t * p.k + lane];
      if (p.weights != nullptr) weight = p.weights[t * p.k + lane];
    }
    float sum[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) sum[u][e] = 0.0f;
    for (int j = 0; j < p.k; ++j) {
      const int row = __shfl_sync(0xffffffffu, from, j);
      const float wj = __shfl_sync(0xffffffffu, weight, j);
      if (row < 0 || row >= pairs) continue;
      const T* y = ys + row * p.ld_in;
      Window<T, ALIGNED> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const Place<T, ALIGNED> at(out, chunk0 + 32 * u, p.D);
        if (at.exists(p.D)) raw[u].load(y + at.col, at.first, at.last);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (Place<T, ALIGNED>(out, chunk0 + 32 * u, p.D).exists(p.D)) {
          float v[V];
          GradTraits<T>::unpack(raw[u].get(), v);
#pragma unroll
          for (int e = 0; e < V; ++e) sum[u][e] = fmaf(wj, v[e], sum[u][e]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const Place<T, ALIGNED> at(out, chunk0 + 32 * u, p.D);
      if (at.exists(p.D)) store_chunk<T, ALIGNED>(out + at.col, at.first, at.last, Chunk<T, V>::pack(sum[u]));
    }
  }
}

// combine's gradients: a warp (BLOCK: a block, where there are few pairs) takes a pair; the token's row of dout comes from
// L2 for all but its first pair.
template <typename T, bool ALIGNED, bool BLOCK, int U>
__global__ void __launch_bounds__(kCopyThreads, ALIGNED ? 1 : 4) combine_back_kernel(const ExpertParams p) {
  constexpr int V = kChunk16<T>;
  __shared__ float s_dot[kCopyThreads / 32];
  const int lane = threadIdx.x & 31;
  const long long warp = (static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x) >> 5;
  const long long warps = (static_cast<long long>(gridDim.x) * kCopyThreads) >> 5;
  const long long pairs = p.tokens * p.k;
  const int i0 = BLOCK ? threadIdx.x : lane;
  constexpr int kLanes = BLOCK ? kCopyThreads : 32;
  T* dys = static_cast<T*>(p.out);
  pdl_wait();
  for (long long pair = BLOCK ? blockIdx.x : warp; pair < pairs; pair += BLOCK ? gridDim.x : warps) {
    const int row = p.slot[pair];
    float dot = 0.0f;
    if (row >= 0 && row < pairs) {
      const T* g = static_cast<const T*>(p.in) + (pair / p.k) * p.ld_in;
      const T* y = static_cast<const T*>(p.ys) + row * p.ld_ys;
      T* out = dys + row * p.ld_out;
      const float w = p.weights != nullptr ? p.weights[pair] : 1.0f;
      for (int i = i0; Place<T, ALIGNED>(out, i, p.D).exists(p.D); i += kLanes * U) {
        Window<T, ALIGNED> rg[U], ry[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const Place<T, ALIGNED> at(out, i + u * kLanes, p.D);
          if (at.exists(p.D)) {
            rg[u].load(g + at.col, at.first, at.last);
            ry[u].load(y + at.col, at.first, at.last);
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const Place<T, ALIGNED> at(out, i + u * kLanes, p.D);
          if (at.exists(p.D)) {
            float a[V], b[V];
            GradTraits<T>::unpack(rg[u].get(), a);
            GradTraits<T>::unpack(ry[u].get(), b);
#pragma unroll
            for (int e = 0; e < V; ++e) {
              if (ALIGNED || (e >= at.first && e < at.last)) dot = fmaf(a[e], b[e], dot);
              a[e] *= w;
            }
            store_chunk<T, ALIGNED>(out + at.col, at.first, at.last, Chunk<T, V>::pack(a));
          }
        }
      }
    }
    if (p.dweights == nullptr) continue;
    dot = warp_sum(dot);
    if (!BLOCK) {
      if (lane == 0) p.dweights[pair] = dot;
    } else {
      if (lane == 0) s_dot[threadIdx.x >> 5] = dot;
      __syncthreads();
      if (threadIdx.x == 0) {
        dot = 0.0f;
#pragma unroll
        for (int i = 0; i < kCopyThreads / 32; ++i) dot += s_dot[i];
        p.dweights[pair] = dot;
      }
      __syncthreads();
    }
  }
  zero_tail<T, ALIGNED>(dys, p.ld_out, p.offsets, p.E, pairs, p.D, warp, warps, lane);
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

// Chunks of a row: there may be one more when it is not aligned.
int chunks_of(int64_t width, int dt, bool aligned) {
  const int64_t per = 16 / static_cast<int64_t>(dtype_size(dt));
  return static_cast<int>((width + per - 1 + (aligned ? 0 : per - 1)) / per);
}

// Calls f with the element type, whether rows are aligned, and the chunks that a lane holds at a time: four (two where
// each needs two loads), for the loads in flight, or one where a row has no more than a warp's lanes, for the warps on an SM (131,072 rows of 130
// bf16 elements: the gradients take 46 us with one, 78 us with four).
template <typename F>
sgdb_status_t with_shape(int dt, bool aligned, bool narrow, F&& f) {
  using std::bool_constant;
  using std::integral_constant;
  const auto typed = [&](auto one) {
    if (aligned)
      return narrow ? f(one, bool_constant<true>{}, integral_constant<int, 1>{}) : f(one, bool_constant<true>{}, integral_constant<int, 4>{});
    return narrow ? f(one, bool_constant<false>{}, integral_constant<int, 1>{}) : f(one, bool_constant<false>{}, integral_constant<int, 2>{});
  };
  return dt == SGDB_BF16 ? typed(BF16{}) : typed(float{});
}

template <typename Kernel>
sgdb_status_t launch_rows(Kernel kernel, long long warps, const ExpertParams& p, const DeviceInfo* dev, void* stream) {
  return launch_dependent(kernel, dim3(grid_for(warps, dev)), kCopyThreads, 0, static_cast<cudaStream_t>(stream), p);
}

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
  // two blocks fit on an SM; none should have less than a few thousand pairs
  int blocks = 1;
  while (blocks < kRouteCluster && 2 * blocks * E <= 2 * dev->sms && pairs > 4096 * blocks) blocks *= 2;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(E * blocks);
  cfg.blockDim = dim3(kRouteThreads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = blocks;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, route_kernel, d_expert, pairs, static_cast<int>(E), is_aligned16(d_expert), d_offsets, d_slot, d_source);
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
  const bool aligned = rows_aligned16(d_x, ldx, dt) && rows_aligned16(d_xs, ldxs, dt) &&
                       (width * static_cast<int64_t>(dtype_size(dt))) % 16 == 0;
  const int chunks = chunks_of(width, dt, aligned);
  return with_shape(dt, aligned, chunks <= 32, [&](auto one, auto is_aligned, auto unroll) {
    p.pieces = (chunks + 32 * unroll() - 1) / (32 * unroll());
    return launch_rows(dispatch_kernel<decltype(one), is_aligned(), unroll()>, tokens * p.pieces, p, dev, stream);
  });
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
  const bool aligned = rows_aligned16(d_ys, ldys, dt) && rows_aligned16(d_out, ldout, dt) &&
                       (width * static_cast<int64_t>(dtype_size(dt))) % 16 == 0;
  const int chunks = chunks_of(width, dt, aligned);
  return with_shape(dt, aligned, chunks <= 32, [&](auto one, auto is_aligned, auto unroll) {
    p.pieces = (chunks + 32 * unroll() - 1) / (32 * unroll());
    return launch_rows(combine_kernel<decltype(one), is_aligned(), unroll()>, tokens * p.pieces, p, dev, stream);
  });
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
  const bool aligned = rows_aligned16(d_dout, lddout, dt) && rows_aligned16(d_ys, ldys, dt) && rows_aligned16(d_dys, lddys, dt) &&
                       (width * static_cast<int64_t>(dtype_size(dt))) % 16 == 0;
  const bool few = tokens * k < 4ll * dev->sms;  // not one warp for each scheduler: a block takes a pair
  return with_shape(dt, aligned, chunks_of(width, dt, aligned) <= 32, [&](auto one, auto is_aligned, auto unroll) {
    using T = decltype(one);
    return few ? launch_rows(combine_back_kernel<T, is_aligned(), true, unroll()>, tokens * k * (kCopyThreads / 32), p, dev, stream)
               : launch_rows(combine_back_kernel<T, is_aligned(), false, unroll()>, tokens * k, p, dev, stream);
  });
}

}  // extern "C"
