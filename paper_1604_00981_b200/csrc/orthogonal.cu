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
// A and B are symmetric: only tiles that touch the upper triangle are computed and stored.  A product that needs a block
// below it loads the block above, whose rows run along K, and tells the matrix instruction so: each instruction says for
// each operand which of its two indices is the fast one.
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
constexpr int kTileK = 64;              // 128 bytes of fp16: one swizzled row of shared memory
constexpr int kBoxBytes = 64 * 64 * 2;  // every copy to shared memory is a box of 64 x 64 elements
constexpr int kStoreBytes = 32 * 64 * 2;  // every copy from it a box of 32 x 64
constexpr int kNormBlocks = 296;        // partial sums of squares per matrix, at most
constexpr unsigned long long kPatienceNs = kWaitLimitNs;

// What becomes of a finished tile: fp16 for the next product (GRAM, POLY, APPLY), the result through a tensor copy (BF16),
// the result element by element (FINAL), the parameters' update (THETA).
enum : int { OUT_GRAM = 0, OUT_POLY = 1, OUT_APPLY = 2, OUT_BF16 = 3, OUT_FINAL = 4, OUT_THETA = 5 };

struct ProductParams {
  int M, N, K, batch;
  // For each operand: 1 if its rows run along K in memory (k is the slow index); for a symmetric operand the
  // granularity g to which its upper triangle is in memory: (r, c) is there when c >= r / g * g
  int a_slow, b_slow, a_sym, b_sym;
  int tiles_n, tiles;           // tiles per row of tiles; tiles that are computed per matrix
  const __half* addend;         // POLY: A
  long long ld, stride;         // of the addend, elements
  float ca, cb, cc;             // POLY: a, b, c
  void* final_out;              // FINAL: dt_out; THETA: fp32 parameters
  int dt_out;
  long long ld_final, stride_final;
  float keep, rate;  // THETA: theta <- keep theta - rate O
  int32_t* info;     // optional: [1] != SGDB_OK: do nothing; receives SGDB_ERR_TIMEOUT
};

template <bool PAIR, int TN>
struct Shape {
  static constexpr int kTileM = PAIR ? 256 : 128;              // rows of a tile
  static constexpr int kBoxesA = 2;                            // per block: 128 rows
  static constexpr int kBoxesB = TN / 64 / (PAIR ? 2 : 1);     // per block
  static constexpr int kStageBytes = (kBoxesA + kBoxesB) * kBoxBytes;
  static constexpr int kWarps = TN >= 128 ? 8 : 4;             // that empty the accumulators
  static constexpr int kThreads = 64 + 32 * kWarps;
  static constexpr int kStages = 6;
  static constexpr int kSmem = kStages * kStageBytes + kWarps * kStoreBytes + 1024;
  static constexpr int kTmemColumns = 2 * TN;                  // two accumulators
  static constexpr int kColumns = TN / (kWarps / 4);           // per warp
};

// Row and column tile of the i-th computed tile of a matrix.
template <int TM, int TN, bool SYM>
__device__ __forceinline__ void tile_at(const ProductParams& p, int i, int* tm, int* tn) {
  if (!SYM) {
    *tm = i / p.tiles_n;
    *tn = i % p.tiles_n;
    return;
  }
  int row = 0, first = 0;
  while (true) {
    first = row * TM / TN;  // the first column tile that reaches the diagonal
    const int n = p.tiles_n - first;
    if (i < n) break;
    i -= n;
    ++row;
  }
  *tm = row;
  *tn = first + i;
}

// The rows [row0, row0 + rows) of an operand are loaded with K as the slow index in the slices of K before the one that
// is returned.  For a symmetric operand: where the rows' part above the diagonal is not all there, its mirror image is.
__device__ __forceinline__ int slow_slices(int slow, int sym, int row0, int rows) {
  return sym != 0 ? (row0 + rows - 1) / sym * sym / kTileK : slow != 0 ? 0x7fffffff : 0;
}

__device__ __forceinline__ void st_shared_v4(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// 16-bit outputs: 32 rows x 64 columns of the accumulator, lane = row.  Scaled, rounded, put into shared memory in the
// layout of the 128-byte swizzle and copied out from there.
template <int OUT>
__device__ __forceinline__ void emit_16bit(const ProductParams& p, const CUtensorMap* map, uint32_t acc, uint32_t stage,
                                           const uint4 (&addend)[8], int z, int row0, int col0, int lane) {
  float v[2][32];
  tmem_load32(acc, v[0]);
  tmem_load32(acc + 32, v[1]);
  tmem_load_wait(v[0]);
  tmem_load_wait(v[1]);
  uint32_t word[32];
  const int diagonal = row0 + lane - col0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    constexpr float kFactor = OUT == OUT_BF16 ? 1.0f / (kScale * kScale) : 1.0f / kScale;
    float lo = v[i >> 4][(2 * i) & 31] * kFactor, hi = v[i >> 4][(2 * i + 1) & 31] * kFactor;
    if (OUT == OUT_POLY) {
      const uint32_t w = (i & 3) == 0 ? addend[i >> 2].x : (i & 3) == 1 ? addend[i >> 2].y : (i & 3) == 2 ? addend[i >> 2].z : addend[i >> 2].w;
      const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&w));
      lo = fmaf(p.cc, lo, fmaf(p.cb, a.x, diagonal == 2 * i ? p.ca * kScale : 0.0f));
      hi = fmaf(p.cc, hi, fmaf(p.cb, a.y, diagonal == 2 * i + 1 ? p.ca * kScale : 0.0f));
    }
    if (OUT == OUT_BF16) {
      word[i] = pack_bf16(lo, hi);
    } else {
      const __half2 h = __floats2half2_rn(lo, hi);
      word[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  bulk_wait_read();  // this lane's earlier copy has read the staging block (only lane 0 has one)
  __syncwarp();
#pragma unroll
  for (int q = 0; q < 8; ++q)
    st_shared_v4(stage + lane * 128 + ((q ^ (lane & 7)) << 4), word[4 * q], word[4 * q + 1], word[4 * q + 2], word[4 * q + 3]);
  fence_proxy_async_shared();
  __syncwarp();
  if (lane == 0) {
    tma_store_3d(map, col0, row0, z, stage);
    bulk_commit();
  }
}

// The old parameters of 32 rows x 32 columns, lane = column.
__device__ __forceinline__ void load_theta(const ProductParams& p, long long z, int row0, int col0, int lane, float (&old)[32]) {
  const float* theta = static_cast<const float*>(p.final_out) + z * p.stride_final + row0 * p.ld_final + col0 + lane;
#pragma unroll
  for (int r = 0; r < 32; ++r) old[r] = row0 + r < p.M && col0 + lane < p.N ? theta[r * p.ld_final] : 0.0f;
}

// The last product, any type and alignment: 32 rows x 32 columns through shared memory, so that a warp writes along a row.
template <int OUT>
__device__ __forceinline__ void emit_final(const ProductParams& p, uint32_t acc, float* block, const float (&old)[32], long long z, int row0,
                                           int col0, int lane) {
  float v[32];
  tmem_load32(acc, v);
  tmem_load_wait(v);
  __syncwarp();
#pragma unroll
  for (int c = 0; c < 32; ++c) block[lane * 32 + (c ^ lane)] = v[c] * (1.0f / (kScale * kScale));
  __syncwarp();
  const int col = col0 + lane;
  if (col >= p.N) return;
  const long long at = z * p.stride_final + row0 * p.ld_final + col;
#pragma unroll
  for (int r = 0; r < 32; ++r) {
    if (row0 + r >= p.M) continue;
    const float o = block[r * 32 + (lane ^ r)];
    if (OUT == OUT_THETA)
      static_cast<float*>(p.final_out)[at + r * p.ld_final] = fmaf(-p.rate, o, p.keep * old[r]);
    else
      store_any(p.final_out, p.dt_out, at + r * p.ld_final, o);
  }
}

// The bounded wait of the other kernels, with some probes before it reads the clock, which takes longer than most waits.
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
#pragma unroll 1
  for (int i = 0; i < 128; ++i)
    if (mbar_try_wait(bar, parity)) return true;
  return mbar_wait_for(bar, parity, abort_flag, kPatienceNs);
}

// One product.  Warp 0 issues the copies of 64-wide slices of both operands into a ring, warp 1 the matrix instructions,
// the other warps read the finished tile from one accumulator while the next tile is summed in the other.
// PAIR: two blocks on neighbouring SMs share a tile of 256 rows; each holds 128 rows of A and of the accumulator and half
// of the columns of B, so that shared memory is read half as often per product; the first block's warp 1 issues for both.
template <bool PAIR, int TN, int OUT>
__global__ void __launch_bounds__(Shape<PAIR, TN>::kThreads, 1)
    product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ CUtensorMap map_out, const ProductParams p) {
  using S = Shape<PAIR, TN>;
  constexpr bool kSym = OUT == OUT_GRAM || OUT == OUT_POLY;
  extern __shared__ uint8_t smem_raw[];
  // the same offset in both blocks of a pair: dynamic shared memory starts at the same address in every block
  const uint32_t ring = (smem_addr(smem_raw) + 1023) & ~1023u;
  const uint32_t staging = ring + S::kStages * S::kStageBytes;
  __shared__ __align__(8) uint64_t s_full[S::kStages], s_empty[S::kStages], s_done[2], s_free[2], s_end;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // warp: known to be uniform
  const uint32_t rank = PAIR ? cluster_rank() : 0;

  if (threadIdx.x == 0) {
    prefetch_map(&map_a);
    prefetch_map(&map_b);
    if (OUT <= OUT_BF16) prefetch_map(&map_out);
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(smem_addr(&s_full[i]), 1);
      mbar_init(smem_addr(&s_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&s_done[i]), 1);
      mbar_init(smem_addr(&s_free[i]), S::kWarps * (PAIR ? 2 : 1));
    }
    mbar_init(smem_addr(&s_end), 1);
    s_abort = 0;
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc<PAIR>(smem_addr(&s_tmem), S::kTmemColumns);
  tcgen05_before_sync();
  __syncthreads();
  if (PAIR) cluster_sync();  // the partner's barriers are ready before anything arrives at them
  tcgen05_after_sync();
  const uint32_t tmem = s_tmem;
  pdl_launch_dependents();
  pdl_wait();
  const bool idle = p.info != nullptr && p.info[1] != SGDB_OK;
  const int total = idle ? 0 : p.tiles * p.batch;
  const int k_blocks = (p.K + kTileK - 1) / kTileK;
  const int first_tile = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;

  // Warps 0 and 1 run their loops as whole warps, so that addresses and descriptors stay in uniform registers, and one
  // elected lane issues.
  if (warp == 0) {
    const bool leader = elect_one();
    fence_proxy_async();
    uint32_t it = 0;
    bool ok = true;
    for (int tile = first_tile; ok && tile < total; tile += step) {
      int tm, tn;
      const int z = tile / p.tiles;
      tile_at<S::kTileM, TN, kSym>(p, tile % p.tiles, &tm, &tn);
      const int row0 = tm * S::kTileM + rank * 128, col0 = tn * TN + rank * S::kBoxesB * 64;
      const int slow_a = slow_slices(p.a_slow, p.a_sym, tm * S::kTileM, S::kTileM), slow_b = slow_slices(p.b_slow, p.b_sym, tn * TN, TN);
      for (int kb = 0; kb < k_blocks; ++kb, ++it) {
        const uint32_t slot = it % S::kStages, round = it / S::kStages;
        if (!wait_phase(smem_addr(&s_empty[slot]), (round & 1) ^ 1, &s_abort)) {
          ok = false;
          break;
        }
        uint32_t bar = smem_addr(&s_full[slot]);
        if (rank == 0 && leader) mbar_arrive_expect_tx(bar, S::kStageBytes * (PAIR ? 2 : 1));
        if (PAIR) bar = cluster_address(bar, 0);
        uint32_t dst = ring + slot * S::kStageBytes;
#pragma unroll
        for (int b = 0; b < S::kBoxesA + S::kBoxesB; ++b, dst += kBoxBytes) {
          const bool is_a = b < S::kBoxesA;
          const int mn = is_a ? row0 + b * 64 : col0 + (b - S::kBoxesA) * 64;
          const bool slow_k = kb < (is_a ? slow_a : slow_b);
          const int x = slow_k ? mn : kb * kTileK, y = slow_k ? kb * kTileK : mn;
          if (leader) {
            if (PAIR)
              tma_load_3d_pair(dst, is_a ? &map_a : &map_b, x, y, z, bar);
            else
              tma_load_3d(dst, is_a ? &map_a : &map_b, x, y, z, bar);
          }
        }
      }
    }
    // nothing may be in flight when the block ends: the last slots are consumed; after a wait that ran out they are at
    // least filled (the pair's second block cannot see that and gives its copies a millisecond)
    for (uint32_t i = it > S::kStages ? it - S::kStages : 0; i < it && (ok || rank == 0); ++i) {
      int ignore = 0;
      uint64_t* bar = ok ? &s_empty[i % S::kStages] : &s_full[i % S::kStages];
      (void)wait_phase(smem_addr(bar), (i / S::kStages) & 1, &ignore);
    }
    if (!ok && rank != 0)
      for (const unsigned long long end = global_timer_ns() + 1000000ull; global_timer_ns() < end;) {
      }
  } else if (warp == 1 && rank == 0) {
    const bool leader = elect_one();
    uint32_t it = 0, count = 0;
    bool ok = true;
    for (int tile = first_tile; ok && tile < total; tile += step, ++count) {
      const uint32_t buf = count & 1;
      if (!wait_phase(smem_addr(&s_free[buf]), ((count >> 1) & 1) ^ 1, &s_abort)) {
        ok = false;
        break;
      }
      tcgen05_after_sync();
      int tm, tn;
      tile_at<S::kTileM, TN, kSym>(p, tile % p.tiles, &tm, &tn);
      const int slow_a = slow_slices(p.a_slow, p.a_sym, tm * S::kTileM, S::kTileM), slow_b = slow_slices(p.b_slow, p.b_sym, tn * TN, TN);
      for (int kb = 0; kb < k_blocks; ++kb, ++it) {
        const uint32_t slot = it % S::kStages;
        const bool is_slow_a = kb < slow_a, is_slow_b = kb < slow_b;
        const uint32_t idesc = mma_descriptor_f16(S::kTileM, TN, is_slow_a, is_slow_b);
        // start address, then 16-byte units from one K of 16 to the next
        const uint64_t desc_a = smem_descriptor(is_slow_a) + ((ring + slot * S::kStageBytes) >> 4);
        const uint64_t desc_b = smem_descriptor(is_slow_b) + ((ring + slot * S::kStageBytes + S::kBoxesA * kBoxBytes) >> 4);
        const uint32_t step_a = is_slow_a ? 2048 >> 4 : 32 >> 4, step_b = is_slow_b ? 2048 >> 4 : 32 >> 4;
        if (!wait_phase(smem_addr(&s_full[slot]), (it / S::kStages) & 1, &s_abort)) {
          ok = false;
          break;
        }
        tcgen05_after_sync();
        if (leader) {
#pragma unroll
          for (int k = 0; k < kTileK / 16; ++k)
            mma_f16<PAIR>(tmem + buf * TN, desc_a + k * step_a, desc_b + k * step_b, idesc, (kb | k) != 0);
          mma_commit<PAIR>(smem_addr(&s_empty[slot]));
        }
        __syncwarp();
      }
      if (ok && leader) mma_commit<PAIR>(smem_addr(&s_done[buf]));
    }
    if (!ok) {  // the instructions issued so far end before tensor memory is given back
      int ignore = 0;
      if (leader) mma_commit<PAIR>(smem_addr(&s_end));
      (void)wait_phase(smem_addr(&s_end), 0, &ignore);
    }
  } else if (warp >= 2) {
    const int quarter = warp & 3;  // the lanes of tensor memory that this warp may read
    const int columns0 = (warp - 2) / 4 * S::kColumns;
    const uint32_t stage = staging + (warp - 2) * kStoreBytes;
    uint32_t count = 0;
    for (int tile = first_tile; tile < total; tile += step, ++count) {
      const uint32_t buf = count & 1;
      int tm, tn;
      const long long z = tile / p.tiles;
      tile_at<S::kTileM, TN, kSym>(p, tile % p.tiles, &tm, &tn);
      const int row0 = tm * S::kTileM + rank * 128 + quarter * 32;
      constexpr int kChunk = OUT <= OUT_BF16 ? 64 : 32;
      [[maybe_unused]] uint4 addend[8];
      [[maybe_unused]] float old[32];
      // what the tile is combined with is on its way while the tile is computed
      const auto load_addend = [&](int c0) {  // 64 columns of this lane's row of A; rows are padded to multiples of 64
        const int col0 = tn * TN + c0, row = row0 + lane;
        const bool in = row < p.M && col0 < p.N;
        const uint4* from = reinterpret_cast<const uint4*>(p.addend + z * p.stride + row * p.ld + col0);
#pragma unroll
        for (int q = 0; q < 8; ++q) addend[q] = in ? from[q] : make_uint4(0, 0, 0, 0);
      };
      if (OUT == OUT_POLY) load_addend(columns0);
      if (OUT == OUT_THETA) load_theta(p, z, row0, tn * TN + columns0, lane, old);
      if (!wait_phase(smem_addr(&s_done[buf]), (count >> 1) & 1, &s_abort)) break;
      tcgen05_after_sync();
      const uint32_t acc = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + buf * TN;
      for (int c = 0; c < S::kColumns; c += kChunk) {
        const int col0 = tn * TN + columns0 + c;
        if (col0 >= p.N || row0 >= p.M) break;
        if constexpr (OUT <= OUT_BF16) {
          emit_16bit<OUT>(p, &map_out, acc + columns0 + c, stage, addend, static_cast<int>(z), row0, col0, lane);
          if (OUT == OUT_POLY && c + kChunk < S::kColumns) load_addend(columns0 + c + kChunk);
        } else {
          emit_final<OUT>(p, acc + columns0 + c, reinterpret_cast<float*>(smem_raw + (stage - smem_addr(smem_raw))), old, z, row0, col0, lane);
          if (OUT == OUT_THETA && c + kChunk < S::kColumns) load_theta(p, z, row0, col0 + kChunk, lane, old);
        }
      }
      tcgen05_before_sync();
      __syncwarp();
      if (lane == 0) {
        const uint32_t bar = smem_addr(&s_free[buf]);
        if (PAIR)
          mbar_arrive_cluster(cluster_address(bar, 0));
        else
          mbar_arrive(bar);
      }
    }
    if (OUT <= OUT_BF16) bulk_wait_all();  // the copies are complete before the block ends
  }
  __syncwarp();
  tcgen05_before_sync();
  __syncthreads();
  if (PAIR) cluster_sync();  // no block leaves, or gives tensor memory back, while its partner may still reach it
  tcgen05_after_sync();
  if (threadIdx.x == 0 && s_abort != 0 && p.info != nullptr) p.info[1] = SGDB_ERR_TIMEOUT;
  if (warp == 1) tmem_dealloc<PAIR>(tmem, S::kTmemColumns);
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
  double* partials;  // [batch][kNormBlocks], the first n_partials in use
  int n_partials;
  __half* x;
  long long ldx, stride_x;
  float eps;
  const int32_t* info;
};

// U is walked through in pieces of a row: a warp takes 32 chunks of 8 elements (VEC: 16-byte accesses) or of one element,
// kPieces times.
constexpr int kPieces = 4;
constexpr int kNormThreads = 256;

template <typename T, bool VEC>
struct PieceTraits {
  static constexpr int kV = VEC ? 8 : 1;
  static constexpr int kWidth = 32 * kV * kPieces;
};

template <typename T, bool VEC>
__device__ __forceinline__ void load_piece(const T* p, float (&v)[VEC ? 8 : 1]) {
  if constexpr (!VEC) {
    v[0] = widen<T>(*p);
  } else if constexpr (sizeof(T) == 2) {
    GradTraits<BF16>::unpack(*reinterpret_cast<const uint4*>(p), v);
  } else {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
}

template <bool VEC>
__device__ __forceinline__ void store_piece(float* p, const float (&v)[VEC ? 8 : 1]) {
  if constexpr (!VEC) {
    *p = v[0];
  } else {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// Partial sums of squares of each matrix, in 64 bits: the square of an fp32 number may be out of fp32's range.  MOMENTUM
// (U is the mean gradient): m <- mu m + g and u = g + mu m or m on the way.
template <typename T, bool VEC, bool MOMENTUM>
__global__ void __launch_bounds__(kNormThreads) square_sum_kernel(const NormParams p) {
  using P = PieceTraits<T, VEC>;
  pdl_launch_dependents();
  pdl_wait();
  if (p.info != nullptr && p.info[1] != SGDB_OK) return;
  __shared__ double s[kNormThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per_row = (p.cols + P::kWidth - 1) / P::kWidth, warps = gridDim.x * (kNormThreads / 32);
  const long long z = blockIdx.y, units = static_cast<long long>(p.rows) * per_row;
  double sum = 0.0;
  for (long long unit = blockIdx.x * (kNormThreads / 32) + warp; unit < units; unit += warps) {
    const int row = static_cast<int>(unit / per_row), col0 = static_cast<int>(unit % per_row) * P::kWidth + lane * P::kV;
    const long long at = z * p.stride + row * p.ld;
    float v[kPieces][P::kV], m[kPieces][P::kV];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int col = col0 + i * 32 * P::kV;
      if (col < p.cols) {
        load_piece<T, VEC>(static_cast<const T*>(p.u) + at + col, v[i]);
        if (MOMENTUM) load_piece<float, VEC>(p.velocity + at + col, m[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int col = col0 + i * 32 * P::kV;
      if (col < p.cols) {
#pragma unroll
        for (int e = 0; e < P::kV; ++e) {
          if (MOMENTUM) {
            m[i][e] = fmaf(p.mu, m[i][e], v[i][e]);
            v[i][e] = p.nesterov ? fmaf(p.mu, m[i][e], v[i][e]) : m[i][e];
          }
          sum = fma(static_cast<double>(v[i][e]), static_cast<double>(v[i][e]), sum);
        }
        if (MOMENTUM) {
          store_piece<VEC>(p.velocity + at + col, m[i]);
          store_piece<VEC>(p.combined + at + col, v[i]);
        }
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int w = 0; w < kNormThreads / 32; ++w) sum += s[w];
    p.partials[z * kNormBlocks + blockIdx.x] = sum;
  }
}

// X = kScale U / (|U| + eps) in fp16.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kNormThreads) normalise_kernel(const NormParams p) {
  using P = PieceTraits<T, VEC>;
  pdl_launch_dependents();
  pdl_wait();
  if (p.info != nullptr && p.info[1] != SGDB_OK) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per_row = (p.cols + P::kWidth - 1) / P::kWidth, warps = gridDim.x * (kNormThreads / 32);
  const long long z = blockIdx.y, units = static_cast<long long>(p.rows) * per_row;
  double sum = 0.0;
  for (int b = lane; b < p.n_partials; b += 32) sum += p.partials[z * kNormBlocks + b];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const double factor = static_cast<double>(kScale) / (sqrt(sum) + static_cast<double>(p.eps));
  // within fp32's range one product in 32 bits; outside it, where U or 1/|U| would not be a normal number, in 64
  const bool plain = factor > 1e-36 && factor < 1e36;
  const float factor32 = static_cast<float>(factor);
  for (long long unit = blockIdx.x * (kNormThreads / 32) + warp; unit < units; unit += warps) {
    const int row = static_cast<int>(unit / per_row), col0 = static_cast<int>(unit % per_row) * P::kWidth + lane * P::kV;
    const T* u = static_cast<const T*>(p.u) + z * p.stride + row * p.ld;
    __half* x = p.x + z * p.stride_x + row * p.ldx;
    float v[kPieces][P::kV];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int col = col0 + i * 32 * P::kV;
      if (col < p.cols) load_piece<T, VEC>(u + col, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int col = col0 + i * 32 * P::kV;
      if (col < p.cols) {
#pragma unroll
        for (int e = 0; e < P::kV; ++e) v[i][e] = plain ? v[i][e] * factor32 : static_cast<float>(v[i][e] * factor);
        if constexpr (VEC) {
          uint32_t w[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const __half2 h = __floats2half2_rn(v[i][2 * q], v[i][2 * q + 1]);
            w[q] = *reinterpret_cast<const uint32_t*>(&h);
          }
          *reinterpret_cast<uint4*>(x + col) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
          x[col] = __float2half_rn(v[i][0]);
        }
      }
    }
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
  q->ldx = round_up(cols, 64);
  q->stride_x = q->ldx * rows;
  q->lds = round_up(q->side, 64);
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

// Boxes of 64 columns and box_rows rows of `batch` 16-bit matrices [rows x cols], 128-byte swizzle, zeros outside.
sgdb_status_t make_map(CUtensorMap* map, void* base, int rows, int cols, long long ld, long long stride, int batch, int box_rows,
                       CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_FLOAT16) {
  const EncodeTiled encode = encode_tiled();
  if (encode == nullptr) return SGDB_ERR_CUDA;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(batch)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(stride) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_rows), 1}, unit[3] = {1, 1, 1};
  const CUresult r = encode(map, type, 3, base, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SGDB_OK : SGDB_ERR_CUDA;
}

struct Maps {  // of one fp16 operand: as it is read and as it is written
  CUtensorMap load, store;
};

sgdb_status_t make_maps(Maps* m, void* base, int rows, int cols, long long ld, long long stride, int batch) {
  const sgdb_status_t st = make_map(&m->load, base, rows, cols, ld, stride, batch, 64);
  return st != SGDB_OK ? st : make_map(&m->store, base, rows, cols, ld, stride, batch, 32);
}

// Programmatic dependent launch: the kernel's start overlaps its predecessor's end; it waits itself before it reads.
template <typename... Args, typename... Given>
sgdb_status_t launch_dependent(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s, Given... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<Args>(args)...);
  return launch_status();
}

// Tiles that are computed of a product of M x N, and those in a row of tiles.
template <bool PAIR, int TN>
long long count_tiles(int M, int N, bool sym, int* tiles_n) {
  constexpr int TM = Shape<PAIR, TN>::kTileM;
  const int tiles_m = (M + TM - 1) / TM;
  *tiles_n = (N + TN - 1) / TN;
  long long n = 0;
  for (int i = 0; i < tiles_m; ++i) n += *tiles_n - (sym ? i * TM / TN : 0);
  return n;
}

template <bool PAIR, int TN, int OUT>
sgdb_status_t launch_product_t(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& out, ProductParams p, const DeviceInfo* dev,
                               cudaStream_t s) {
  using S = Shape<PAIR, TN>;
  p.tiles = static_cast<int>(count_tiles<PAIR, TN>(p.M, p.N, OUT == OUT_GRAM || OUT == OUT_POLY, &p.tiles_n));
  const long long total = static_cast<long long>(p.tiles) * p.batch;
  auto kernel = product_kernel<PAIR, TN, OUT>;
  static std::atomic<bool> allowed[kMaxDevices];
  if (!allowed[dev->index].load(std::memory_order_relaxed)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem) != cudaSuccess) return launch_status();
    allowed[dev->index].store(true, std::memory_order_relaxed);
  }
  constexpr int kCluster = PAIR ? 2 : 1;
  const long long most = dev->sms / kCluster;
  return launch_dependent(kernel, dim3(static_cast<unsigned>(total < most ? total : most) * kCluster), S::kThreads, S::kSmem, kCluster, s, a, b,
                          out, p);
}

enum : int { TILE_PAIR_256, TILE_PAIR_128, TILE_64 };

int tile_rows(int tile) { return tile == TILE_PAIR_256 || tile == TILE_PAIR_128 ? 256 : 128; }

// Large tiles where there are two and more for each pair of SMs, small ones where there is not even one of 128 x 128 per SM
// (256 x 256, 256 x 128, 128 x 64 for one matrix: 4096 1.05, 1.15, 2.37 ms; 2048 273, 241, 416 us; 1000 167, 122, 106 us).
int pick_tile(int M, int N, int batch, bool sym, const DeviceInfo* dev) {
  int unused;
  if (count_tiles<true, 256>(M, N, sym, &unused) * batch >= dev->sms) return TILE_PAIR_256;
  return count_tiles<false, 128>(M, N, sym, &unused) * batch >= dev->sms ? TILE_PAIR_128 : TILE_64;
}

template <int OUT>
sgdb_status_t launch_product(int tile, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& out, const ProductParams& p,
                             const DeviceInfo* dev, cudaStream_t s) {
  switch (tile) {
    case TILE_PAIR_256: return launch_product_t<true, 256, OUT>(a, b, out, p, dev, s);
    case TILE_PAIR_128: return launch_product_t<true, 128, OUT>(a, b, out, p, dev, s);
    default: return launch_product_t<false, 64, OUT>(a, b, out, p, dev, s);
  }
}

bool rule_ok(const sgdb_newton_schulz_t* ns) {
  return ns != nullptr && ns->steps >= 1 && ns->steps <= SGDB_MAX_STEPS && std::isfinite(ns->a) && std::isfinite(ns->b) &&
         std::isfinite(ns->c) && ns->eps >= 0.0f && !std::isinf(ns->eps);
}

// X is in place (q.x0): the products, and what is done with the last one.  `result`: the map of the output when `last` is
// OUT_BF16.
sgdb_status_t run_products(const Plan& q, const sgdb_newton_schulz_t& ns, char* ws, int last, const ProductParams& final_params,
                           const CUtensorMap* result, int32_t* info, const DeviceInfo* dev, cudaStream_t s) {
  __half* x[2] = {reinterpret_cast<__half*>(ws + q.x0), reinterpret_cast<__half*>(ws + q.x1)};
  __half *a = reinterpret_cast<__half*>(ws + q.a), *b = reinterpret_cast<__half*>(ws + q.b);
  Maps map_x[2], map_a, map_b;
  sgdb_status_t st = SGDB_OK;
  for (int i = 0; i < 2 && st == SGDB_OK; ++i) st = make_maps(&map_x[i], x[i], q.rows, q.cols, q.ldx, q.stride_x, q.batch);
  if (st == SGDB_OK) st = make_maps(&map_a, a, q.side, q.side, q.lds, q.stride_s, q.batch);
  if (st == SGDB_OK) st = make_maps(&map_b, b, q.side, q.side, q.lds, q.stride_s, q.batch);
  if (st != SGDB_OK) return st;
  const bool tall = q.rows > q.cols;
  const int length = tall ? q.rows : q.cols;
  const int tile_gram = pick_tile(q.side, q.side, q.batch, true, dev), tile_poly = pick_tile(q.side, q.side, q.batch, true, dev),
            tile_apply = pick_tile(q.rows, q.cols, q.batch, false, dev);
  for (int i = 0; i < ns.steps; ++i) {
    const CUtensorMap& mx = map_x[i & 1].load;
    ProductParams p{};
    p.batch = q.batch;
    p.info = info;
    p.M = p.N = q.side;
    // A = X X^T; tall: A = X^T X, whose operands run along K
    p.K = length;
    p.a_slow = p.b_slow = tall;
    st = launch_product<OUT_GRAM>(tile_gram, mx, mx, map_a.store, p, dev, s);
    if (st != SGDB_OK) return st;
    p.K = q.side;
    p.a_sym = p.b_sym = tile_rows(tile_gram);
    p.addend = a;
    p.ld = q.lds;
    p.stride = q.stride_s;
    p.ca = ns.a, p.cb = ns.b, p.cc = ns.c;
    st = launch_product<OUT_POLY>(tile_poly, map_a.load, map_a.load, map_b.store, p, dev, s);
    if (st != SGDB_OK) return st;
    const bool end = i + 1 == ns.steps;
    ProductParams r = end ? final_params : ProductParams{};
    r.batch = q.batch;
    r.info = info;
    r.M = q.rows;
    r.N = q.cols;
    r.K = q.side;
    // wide: B X, X's rows run along K; tall: X B
    r.a_sym = tall ? 0 : tile_rows(tile_poly);
    r.b_sym = tall ? tile_rows(tile_poly) : 0;
    r.b_slow = 1;
    const CUtensorMap &first = tall ? mx : map_b.load, &second = tall ? map_b.load : mx, &next = map_x[(i + 1) & 1].store;
    const int out = end ? last : OUT_APPLY;
    st = out == OUT_APPLY   ? launch_product<OUT_APPLY>(tile_apply, first, second, next, r, dev, s)
         : out == OUT_BF16  ? launch_product<OUT_BF16>(tile_apply, first, second, *result, r, dev, s)
         : out == OUT_THETA ? launch_product<OUT_THETA>(tile_apply, first, second, next, r, dev, s)
                            : launch_product<OUT_FINAL>(tile_apply, first, second, next, r, dev, s);
    if (st != SGDB_OK) return st;
  }
  return SGDB_OK;
}

template <typename T, bool VEC>
sgdb_status_t run_normalise_t(NormParams p, int batch, const DeviceInfo* dev, cudaStream_t s) {
  constexpr int kWidth = PieceTraits<T, VEC>::kWidth;
  const long long units = static_cast<long long>(p.rows) * ((p.cols + kWidth - 1) / kWidth);
  const long long want = (units + kNormThreads / 32 - 1) / (kNormThreads / 32);
  const auto blocks = [&](long long per_sm, long long most) {
    long long cap = (per_sm * dev->sms + batch - 1) / batch;
    if (cap > most) cap = most;
    return static_cast<unsigned>(want < cap ? want : cap);
  };
  p.n_partials = static_cast<int>(blocks(4, kNormBlocks));
  const dim3 sums(p.n_partials, batch);
  sgdb_status_t st;
  if constexpr (sizeof(T) == 4)
    st = p.velocity != nullptr ? launch_dependent(square_sum_kernel<T, VEC, true>, sums, kNormThreads, 0, 1, s, p)
                               : launch_dependent(square_sum_kernel<T, VEC, false>, sums, kNormThreads, 0, 1, s, p);
  else
    st = launch_dependent(square_sum_kernel<T, VEC, false>, sums, kNormThreads, 0, 1, s, p);
  if (st != SGDB_OK) return st;
  if (p.velocity != nullptr) p.u = p.combined;
  return launch_dependent(normalise_kernel<T, VEC>, dim3(blocks(8, 1 << 20), batch), kNormThreads, 0, 1, s, p);
}

sgdb_status_t run_normalise(const NormParams& p, int batch, const DeviceInfo* dev, cudaStream_t s) {
  const bool vec = rows_aligned16(p.u, p.ld, p.dt_in) && (batch == 1 || rows_aligned16(p.u, p.stride, p.dt_in)) && p.cols % 8 == 0 &&
                   is_aligned16(p.velocity);
  if (p.dt_in == SGDB_BF16)
    return vec ? run_normalise_t<BF16, true>(p, batch, dev, s) : run_normalise_t<BF16, false>(p, batch, dev, s);
  return vec ? run_normalise_t<float, true>(p, batch, dev, s) : run_normalise_t<float, false>(p, batch, dev, s);
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
  if (dt_out == SGDB_BF16 && rows_aligned16(d_out, ldout, dt_out) && (batch == 1 || stride_out % 8 == 0)) {
    CUtensorMap result;
    st = make_map(&result, d_out, q.rows, q.cols, ldout, batch == 1 ? q.rows * ldout : stride_out, batch, 32, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16);
    return st != SGDB_OK ? st : run_products(q, *ns, ws, OUT_BF16, f, &result, d_info, dev, s);
  }
  return run_products(q, *ns, ws, OUT_FINAL, f, nullptr, d_info, dev, s);
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
  n.ld = cols;
  n.stride = rows * cols;
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
  return run_products(q, opt->newton_schulz, ws, OUT_THETA, f, nullptr, d_info, dev, s);
}

}  // extern "C"
