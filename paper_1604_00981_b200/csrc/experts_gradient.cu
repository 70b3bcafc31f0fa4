// The gradient of the experts' matrices (declared in include/sgdb.h; the 8-bit format: sgdb_f8.cuh):
//
//   dw[e][n][k] = sum over expert e's rows s of dy[s][n] x[s][k],   x[s][k] = q 2^(byte of (s, k / 128))
//
// x is the checkpoint that the forward pass kept, its products' operand in 8 bits.  Its values times their scales are exact
// in bf16, so the products of bf16 matrix instructions, summed in fp32 in tensor memory, are those of x and dy as they are.
// A dy in fp32 is cut into three bf16 numbers of 8 bits each whose sum it is, at three times the products: rounded to one, the
// result would have an error of 1.6e-3 instead of 3e-7.
//
// K of the instruction are the tokens, 64 to a slot of the ring; its M are k and its N are n, 256 each for a pair of blocks, so
// that a lane of tensor memory is a k and a warp's stores run along a row of dw.  Both operands lie in shared memory as in
// global memory, with the tokens as the slow index.  Eight warps load them through registers, which is where x is
// widened and where tokens behind the expert's last become zeros: a copy engine could do neither, and what lies there may
// be NaN.
//
// Few tiles and many tokens: the tokens are cut into `splits` ranges whose sums go to the workspace; a second kernel
// adds them in order.
#include <cuda.h>
#include <cuda_runtime.h>

#include "sgdb_f8.cuh"
#include "sgdb_host.cuh"
#include "sgdb_tensor.cuh"

namespace sgdb {
namespace {

constexpr int kTile = 256;       // k, and n, of a pair's tile
constexpr int kTokens = 64;      // of a slot of the ring
constexpr int kLoaders = 256;    // threads
constexpr int kThreads = kLoaders + 4 * 32 + 32;
constexpr int kGroupBytes = kTokens * 128;  // 64 columns of bf16
constexpr int kOperandBytes = 2 * kGroupBytes;

// Of dy in type T: numbers in bf16 for each of its elements, and slots of the ring, which is 192 KB.
template <typename T>
struct Shape {
  static constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
  static constexpr int kStageBytes = (1 + kParts) * kOperandBytes;
  static constexpr int kStages = 196608 / kStageBytes;
  static constexpr int kSmem = kStages * kStageBytes + 1024;
};

// The first 8 bits of a number's significand, and what is left: exact both.
__device__ __forceinline__ float leading_bits(float v, float* rest) {
  const float lead = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  *rest = (__float_as_uint(v) & 0x7fffffffu) == 0x7f800000u ? 0.0f : v - lead;
  return lead;
}
constexpr int kTmemColumns = 512;
constexpr int kPairs = 74;       // what the rule for the splits counts on
constexpr int kSplitTokens = 512;

struct GradientParams {
  const void* dy;
  long long lddy;
  const uint8_t *x, *x_scale;
  long long ldx, ldxs;
  const int32_t* offsets;  // or null: one expert has all rows
  void* dw;
  long long lddw, stride;
  int rows, N, K, E, tiles_n, tiles_k, splits, dt_out;
  bool vec_dy, vec_x;
  float* partial;  // [unit][n][k] where splits > 1
  int32_t* info;
  unsigned long long wait_limit_ns;
};

// What a pair works on at a time: a tile of dw of expert e and a range of its tokens.
struct Unit {
  int e, n0, k0, n_mma, begin, end;
  __device__ __forceinline__ Unit(const GradientParams& p, long long index) {
    const int split = static_cast<int>(index % p.splits);
    long long tile = index / p.splits;
    const int tk = static_cast<int>(tile % p.tiles_k);
    tile /= p.tiles_k;
    const int tn = static_cast<int>(tile % p.tiles_n);
    e = static_cast<int>(tile / p.tiles_n);
    n0 = tn * kTile, k0 = tk * kTile;
    n_mma = min(kTile, (p.N - n0 + 15) & ~15);
    int a = 0, b = p.rows;
    if (p.offsets != nullptr) {
      a = min(max(p.offsets[e], 0), p.rows);
      b = max(a, min(max(p.offsets[e + 1], 0), p.rows));
    }
    const int share = ((b - a + p.splits - 1) / p.splits + kTokens - 1) / kTokens * kTokens;
    begin = min(static_cast<long long>(b), a + static_cast<long long>(split) * share);
    end = min(static_cast<long long>(b), static_cast<long long>(begin) + share);
  }
  __device__ __forceinline__ int slots() const { return (end - begin + kTokens - 1) / kTokens; }
};

// A loader thread's share of a slot: 16 bytes of bf16 (32 of fp32) of four tokens of dy, 16 bytes of two tokens of x.
template <typename T>
struct Held {
  uint4 dy[4 * sizeof(T) / 2], x[2];
  uint32_t scale[2];
};

template <typename T, int FORMAT>
struct Loader {
  const GradientParams& p;
  long long index, units, step;
  int slot, slots, rank, thread;
  Unit u;
  __device__ __forceinline__ Loader(const GradientParams& p_, long long first, long long step_, long long units_, int rank_)
      : p(p_), index(first), units(units_), step(step_), slot(0), slots(0), rank(rank_), thread(threadIdx.x), u(p_, first) {
    slots = u.slots();
    settle();
  }
  __device__ __forceinline__ void settle() {
    while (slot >= slots) {
      index += step;
      if (index >= units) return;
      u = Unit(p, index);
      slot = 0;
      slots = u.slots();
    }
  }
  // Four consecutive elements of 4 bytes, or eight of 2, of which those before `n` exist.
  __device__ __forceinline__ uint4 load16(const T* at, int n) const {
    constexpr int V = kChunk16<T>;
    if (n <= 0) return make_uint4(0, 0, 0, 0);
    if (p.vec_dy && n >= V) return *reinterpret_cast<const uint4*>(at);
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = e < n ? widen<T>(at[e]) : 0.0f;
    return Chunk<T, V>::pack(v);
  }
  // Begins the loads of the next slot; false behind the last.
  __device__ __forceinline__ bool load(Held<T>& h) {
    if (index >= units) return false;
    const int first = u.begin + slot * kTokens;
    {
      constexpr int kParts = sizeof(T) / 2;  // loads of 16 bytes for eight elements
      const int half = u.n_mma >> 1, chunk = thread & 15, n = u.n0 + rank * half + chunk * 8;
      const int there = chunk * 8 < half ? p.N - n : 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int token = first + (thread >> 4) + 16 * i;
        const T* at = static_cast<const T*>(p.dy) + token * p.lddy + n;
#pragma unroll
        for (int q = 0; q < kParts; ++q) h.dy[kParts * i + q] = load16(at + q * kChunk16<T>, token < u.end ? there - q * kChunk16<T> : 0);
      }
    }
    const int k = u.k0 + rank * 128 + (thread & 7) * 16;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int token = first + (thread >> 3) + 32 * i;
      h.x[i] = make_uint4(0, 0, 0, 0);
      h.scale[i] = 127;
      if (token < u.end && k < p.K) {
        const uint8_t* at = p.x + token * p.ldx + k;
        h.scale[i] = p.x_scale[token * p.ldxs + (k >> 7)];
        if (p.vec_x && k + 16 <= p.K) {
          h.x[i] = *reinterpret_cast<const uint4*>(at);
        } else {
          uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (k + e < p.K) w[e >> 2] |= static_cast<uint32_t>(at[e]) << (8 * (e & 3));
          h.x[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
    ++slot;
    settle();
    return true;
  }
  // To shared memory, as bf16: 128 bytes of 64 columns for each token, in the layout of the 128-byte swizzle.
  __device__ __forceinline__ void store(const Held<T>& h, uint32_t at) const {
    const auto place = [&](int token, int chunk) { return (chunk >> 3) * kGroupBytes + token * 128 + (((chunk & 7) ^ (token & 7)) << 4); };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int token = (thread >> 3) + 32 * i, chunk = (thread & 7) * 2;
      const float scale = scale_value(h.scale[i]);
      const uint32_t raw[4] = {h.x[i].x, h.x[i].y, h.x[i].z, h.x[i].w};
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 two = widen_f8x2(static_cast<uint16_t>(raw[j >> 1] >> (16 * (j & 1))), FORMAT);
        w[j] = pack_bf16(two.x * scale, two.y * scale);
      }
      // lanes of the second 64 columns store their chunks in the other order: no two of eight to the same banks
      const bool swap = (thread & 4) != 0;
      const uint32_t a = at + place(token, chunk), b = at + place(token, chunk + 1);
      st_shared_v4(swap ? b : a, swap ? w[4] : w[0], swap ? w[5] : w[1], swap ? w[6] : w[2], swap ? w[7] : w[3]);
      st_shared_v4(swap ? a : b, swap ? w[0] : w[4], swap ? w[1] : w[5], swap ? w[2] : w[6], swap ? w[3] : w[7]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t to = at + kOperandBytes + place((thread >> 4) + 16 * i, thread & 15);
      if constexpr (sizeof(T) == 2) {
        st_shared_v4(to, h.dy[i].x, h.dy[i].y, h.dy[i].z, h.dy[i].w);
      } else {
        float v[8];
        const uint4 lo = h.dy[2 * i], hi = h.dy[2 * i + 1];
        v[0] = __uint_as_float(lo.x), v[1] = __uint_as_float(lo.y), v[2] = __uint_as_float(lo.z), v[3] = __uint_as_float(lo.w);
        v[4] = __uint_as_float(hi.x), v[5] = __uint_as_float(hi.y), v[6] = __uint_as_float(hi.z), v[7] = __uint_as_float(hi.w);
#pragma unroll
        for (int part = 0; part < 3; ++part) {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float a = leading_bits(v[2 * j], &v[2 * j]), b = leading_bits(v[2 * j + 1], &v[2 * j + 1]);
            w[j] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
          }
          st_shared_v4(to + part * kOperandBytes, w[0], w[1], w[2], w[3]);
        }
      }
    }
  }
};

template <typename T, int FORMAT>
__global__ void __launch_bounds__(kThreads, 1) experts_gradient_kernel(const __grid_constant__ GradientParams p) {
  constexpr int kStages = Shape<T>::kStages, kStageBytes = Shape<T>::kStageBytes;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t ring = (smem_addr(smem_raw) + 1023) & ~1023u;  // the same offset in both blocks of a pair
  __shared__ __align__(8) uint64_t s_full[kStages], s_empty[kStages], s_done[2], s_free[2], s_end;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort, s_partner_abort;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_addr(&s_full[i]), 2 * kLoaders / 32);
      mbar_init(smem_addr(&s_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&s_done[i]), 1);
      mbar_init(smem_addr(&s_free[i]), 8);
    }
    mbar_init(smem_addr(&s_end), 1);
    s_abort = s_partner_abort = 0;
    fence_barrier_init();
  }
  if (warp == 12) tmem_alloc<true>(smem_addr(&s_tmem), kTmemColumns);
  tcgen05_before_sync();
  __syncthreads();
  cluster_sync();  // the partner's barriers are ready before anything arrives at them
  tcgen05_after_sync();
  pdl_wait();
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
  const long long units = static_cast<long long>(p.E) * p.tiles_n * p.tiles_k * p.splits;
  const long long first = blockIdx.x >> 1, step = gridDim.x >> 1;

  if (warp < kLoaders / 32) {
    Loader<T, FORMAT> loader(p, first, step, units, rank);
    uint32_t it = 0;
    const auto put = [&](const Held<T>& h) {
      const uint32_t slot = it % kStages;
      if (!wait_phase(smem_addr(&s_empty[slot]), ((it / kStages) & 1) ^ 1, &s_abort, p.wait_limit_ns)) return false;
      loader.store(h, ring + slot * kStageBytes);
      fence_proxy_async_shared();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(cluster_address(smem_addr(&s_full[slot]), 0));
      ++it;
      return true;
    };
    Held<T> h0, h1;  // two slots' loads are under way while a third is stored
    bool v0 = loader.load(h0), v1 = loader.load(h1), ok = true;
    while (v0) {
      ok = put(h0);
      if (!ok) break;
      v0 = loader.load(h0);
      if (!v1) break;
      ok = put(h1);
      if (!ok) break;
      v1 = loader.load(h1);
    }
    // the last slots are consumed: the arrivals that say so have come to both blocks before these end
    for (uint32_t i = it > kStages ? it - kStages : 0; ok && i < it; ++i)
      ok = wait_phase(smem_addr(&s_empty[i % kStages]), (i / kStages) & 1, &s_abort, p.wait_limit_ns);
  } else if (warp == 12) {
    if (rank == 0) {
      const bool leader = elect_one();
      uint32_t it = 0, count = 0;
      bool ok = true;
      for (long long index = first; ok && index < units; index += step) {
        const Unit u(p, index);
        const int slots = u.slots();
        if (slots == 0) continue;
        const uint32_t buf = count & 1, idesc = mma_descriptor_bf16_slow_k(kTile, u.n_mma);
        if (!wait_phase(smem_addr(&s_free[buf]), ((count >> 1) & 1) ^ 1, &s_abort, p.wait_limit_ns)) {
          ok = false;
          break;
        }
        tcgen05_after_sync();
        for (int s = 0; s < slots; ++s, ++it) {
          const uint32_t slot = it % kStages;
          if (!wait_phase(smem_addr(&s_full[slot]), (it / kStages) & 1, &s_abort, p.wait_limit_ns)) {
            ok = false;
            break;
          }
          tcgen05_after_sync();
          if (leader) {
            // 8 tokens every 1024 bytes, 64 columns every kGroupBytes
            const uint64_t a = (static_cast<uint64_t>(kGroupBytes >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61) |
                               ((ring + slot * kStageBytes) >> 4);
#pragma unroll
            for (int part = 0; part < Shape<T>::kParts; ++part)
#pragma unroll
              for (int k = 0; k < kTokens / 16; ++k)
                mma_f16<true>(tmem + buf * kTile, a + 128 * k, a + ((1 + part) * kOperandBytes >> 4) + 128 * k, idesc, (s | part | k) != 0);
            mma_commit<true>(smem_addr(&s_empty[slot]));
          }
          __syncwarp();
        }
        if (ok && leader) mma_commit<true>(smem_addr(&s_done[buf]));
        ++count;
      }
      // the instructions issued so far end before shared and tensor memory are given back, whoever gave up
      int ignore = 0;
      if (leader) mma_commit<true>(smem_addr(&s_end), 1);
      (void)wait_phase(smem_addr(&s_end), 0, &ignore, kWaitLimitNs);
    }
  } else {
    const int quarter = warp & 3;  // the lanes of tensor memory that this warp may read
    uint32_t count = 0;
    for (long long index = first; index < units; index += step) {
      const Unit u(p, index);
      const bool empty = u.slots() == 0;
      const uint32_t buf = count & 1;
      if (!empty) {
        if (!wait_phase(smem_addr(&s_done[buf]), (count >> 1) & 1, &s_abort, p.wait_limit_ns)) break;
        tcgen05_after_sync();
      }
      const uint32_t acc = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + buf * kTile;
      const int in_tile = rank * 128 + quarter * 32 + lane, k = u.k0 + in_tile;
      if (k - lane < p.K) {
        for (int c = 0; c < u.n_mma; c += 16) {
          float v[16];
          if (empty) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0.0f;
          } else {
            tmem_load16(acc + c, v);
            tmem_load_wait(v);
          }
          if (p.splits > 1) {
            float* to = p.partial + (index * kTile + c) * kTile + in_tile;
#pragma unroll
            for (int i = 0; i < 16; ++i) to[i * kTile] = v[i];
          } else if (k < p.K) {
            const long long at = u.e * p.stride + static_cast<long long>(u.n0 + c) * p.lddw + k;
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (u.n0 + c + i < p.N) store_any(p.dw, p.dt_out, at + i * p.lddw, v[i]);
          }
        }
      }
      if (!empty) {
        tcgen05_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(cluster_address(smem_addr(&s_free[buf]), 0));
        ++count;
      }
    }
  }
  __syncwarp();
  tcgen05_before_sync();
  __syncthreads();
  // no block leaves, or gives tensor memory back, while its partner may still reach it; here each tells whether it gave up
  if (threadIdx.x == 0 && s_abort != 0) st_shared_cluster(cluster_address(smem_addr(&s_partner_abort), cluster_rank() ^ 1), 1);
  __syncwarp();
  cluster_sync();
  tcgen05_after_sync();
  if (threadIdx.x == 0 && (s_abort != 0 || s_partner_abort != 0) && p.info != nullptr) p.info[1] = SGDB_ERR_TIMEOUT;
  if (warp == 12) tmem_dealloc<true>(tmem, kTmemColumns);
}

// The ranges' sums, in their order.
__global__ void __launch_bounds__(256) gradient_sum_kernel(const __grid_constant__ GradientParams p) {
  pdl_wait();
  const long long rows = static_cast<long long>(p.E) * p.N;
  for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
    const int e = static_cast<int>(r / p.N), n = static_cast<int>(r % p.N);
    for (int k = threadIdx.x; k < p.K; k += blockDim.x) {
      const long long tile = (static_cast<long long>(e) * p.tiles_n + n / kTile) * p.tiles_k + k / kTile;
      const float* from = p.partial + (tile * p.splits * kTile + n % kTile) * kTile + k % kTile;
      float sum = 0.0f;
      for (int s = 0; s < p.splits; ++s) sum += from[static_cast<long long>(s) * kTile * kTile];
      store_any(p.dw, p.dt_out, e * p.stride + n * p.lddw + k, sum);
    }
  }
}

// One range where the tiles keep the pairs busy; otherwise as many as there are pairs for them, of kSplitTokens at least if
// the experts are alike.
int splits_of(int64_t rows, int64_t N, int64_t K, int32_t E) {
  const int64_t tiles = ((N + kTile - 1) / kTile) * ((K + kTile - 1) / kTile) * E;
  const int64_t room = kPairs / tiles, useful = rows / E / kSplitTokens;
  const int64_t n = room < useful ? room : useful;
  return n < 1 ? 1 : static_cast<int>(n);
}

bool sizes_ok(int64_t rows, int64_t N, int64_t K, int32_t E) {
  return rows >= 0 && rows <= SGDB_MAX_PAIRS && N >= 1 && N <= SGDB_MAX_WIDTH && K >= 1 && K <= SGDB_MAX_WIDTH && E >= 1 && E <= SGDB_MAX_EXPERTS;
}

template <typename T, int FORMAT>
sgdb_status_t launch_gradient(const GradientParams& p, const DeviceInfo* dev, cudaStream_t s) {
  auto kernel = experts_gradient_kernel<T, FORMAT>;
  constexpr int kSmem = Shape<T>::kSmem;
  cudaLaunchConfig_t cfg{};
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  static std::atomic<int> resident[kMaxDevices];  // pairs that run at once: more would be a second round
  int most = resident[dev->index].load(std::memory_order_relaxed);
  if (most == 0) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return launch_status();
    cfg.gridDim = dim3(dev->sms / 2 * 2);
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&most, kernel, &cfg) != cudaSuccess) return launch_status();
    if (most < 1) return SGDB_ERR_UNSUPPORTED;
    resident[dev->index].store(most, std::memory_order_relaxed);
  }
  const long long want = static_cast<long long>(p.E) * p.tiles_n * p.tiles_k * p.splits;
  cfg.gridDim = dim3(static_cast<unsigned>(want < most ? want : most) * 2);
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, kernel, p);
  return launch_status();
}

}  // namespace
}  // namespace sgdb

using namespace sgdb;

extern "C" {

size_t sgdb_experts_gradient_workspace_bytes(int64_t rows, int64_t width, int64_t depth, int32_t E) {
  if (!sizes_ok(rows, width, depth, E)) return 0;
  const int splits = splits_of(rows, width, depth, E);
  const size_t tiles = static_cast<size_t>((width + kTile - 1) / kTile) * ((depth + kTile - 1) / kTile) * E;
  return splits > 1 ? tiles * splits * kTile * kTile * 4 : 4;
}

sgdb_status_t sgdb_experts_gradient(const void* d_dy, sgdb_dtype_t dt, int64_t rows, int64_t width, int64_t lddy, const void* d_x, sgdb_f8_t format,
                                    int64_t depth, int64_t ldx, const uint8_t* d_x_scale, int64_t ldxs, const int32_t* d_offsets, int32_t E, void* d_dw,
                                    sgdb_dtype_t dt_dw, int64_t lddw, int64_t stride_dw, void* d_workspace, size_t workspace_bytes, int32_t* d_info,
                                    void* stream) {
  if (!dtype_ok(dt) || !dtype_ok(dt_dw) || (format != SGDB_E4M3 && format != SGDB_E5M2) || !sizes_ok(rows, width, depth, E)) return SGDB_ERR_INVALID_ARG;
  if (lddy < width || ldx < depth || ldxs < blocks_of(depth) || lddw < depth || (E > 1 && stride_dw < (width - 1) * lddw + depth))
    return SGDB_ERR_INVALID_ARG;
  if (d_offsets == nullptr && E != 1) return SGDB_ERR_INVALID_ARG;
  if (!array_ok(d_dw, dt_dw) || (rows > 0 && (!array_ok(d_dy, dt) || d_x == nullptr || d_x_scale == nullptr))) return SGDB_ERR_INVALID_ARG;
  if ((d_offsets != nullptr && !array_ok(d_offsets, SGDB_F32)) || (d_info != nullptr && !array_ok(d_info, SGDB_F32))) return SGDB_ERR_INVALID_ARG;
  GradientParams p{};
  p.splits = splits_of(rows, width, depth, E);
  if (p.splits > 1 && (!array_ok(d_workspace, SGDB_F32) || workspace_bytes < sgdb_experts_gradient_workspace_bytes(rows, width, depth, E)))
    return SGDB_ERR_INVALID_ARG;
  const DeviceInfo* dev = nullptr;
  sgdb_status_t st = device_info(&dev);
  if (st != SGDB_OK) return st;
  p.dy = d_dy, p.lddy = lddy, p.x = static_cast<const uint8_t*>(d_x), p.ldx = ldx, p.x_scale = d_x_scale, p.ldxs = ldxs, p.offsets = d_offsets;
  p.dw = d_dw, p.dt_out = dt_dw, p.lddw = lddw, p.stride = E > 1 ? stride_dw : 0;
  p.rows = static_cast<int>(rows), p.N = static_cast<int>(width), p.K = static_cast<int>(depth), p.E = E;
  p.tiles_n = (p.N + kTile - 1) / kTile, p.tiles_k = (p.K + kTile - 1) / kTile;
  p.vec_dy = rows_aligned16(d_dy, lddy, dt), p.vec_x = is_aligned16(d_x) && ldx % 16 == 0;
  p.partial = static_cast<float*>(d_workspace), p.info = d_info, p.wait_limit_ns = wait_limit_ns();
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (dt == SGDB_BF16)
    st = format == SGDB_E4M3 ? launch_gradient<BF16, SGDB_E4M3>(p, dev, s) : launch_gradient<BF16, SGDB_E5M2>(p, dev, s);
  else
    st = format == SGDB_E4M3 ? launch_gradient<float, SGDB_E4M3>(p, dev, s) : launch_gradient<float, SGDB_E5M2>(p, dev, s);
  if (st != SGDB_OK || p.splits == 1) return st;
  const long long lines = static_cast<long long>(E) * width, cap = 8ll * dev->sms;
  return launch_dependent(gradient_sum_kernel, dim3(static_cast<unsigned>(lines < cap ? lines : cap)), 256, 0, s, p);
}

}  // extern "C"
