// The orthogonalised update (declared in include/sgdb.h): Newton-Schulz products of a matrix,
// alone and as the rule of a whole server iteration.
//
//   X <- U / (|U|_F + eps), then `steps` times, over the shorter side:
//     A = X X^T,  B = a I + b A + c A^2,  X <- B X        (tall: A = X^T X, X <- X B)
//
// All products of a call are one cooperative launch of newton_schulz_kernel, whose blocks work through the tiles of all
// products in order; a tile starts when the tiles of its matrix in the product before are done, which counters in global
// memory tell.  The products are tcgen05 matrix instructions on fp16 operands with fp32
// accumulators in tensor memory.  X, A and B are kept as fp16 times kScale: with the
// usual coefficients the largest singular value of X is at most about 1.2, far below fp16's largest number (rules that could
// leave its range are refused, see rule_in_range), and elements
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
constexpr int kTileK = 128;               // depth of a slot of the ring
constexpr int kStoreBytes = 32 * 64 * 2;  // every copy from shared memory is a box of 32 x 64 elements
constexpr int kNormBlocks = 296;        // partial sums of squares per matrix, at most

// What becomes of a finished tile: fp16 for the next product (GRAM, POLY, APPLY); of the last one, the result through a
// tensor copy (BF16) or element by element (FINAL), or the parameters' update (THETA).
enum : int { OUT_GRAM = 0, OUT_POLY = 1, OUT_APPLY = 2, OUT_BF16 = 3, OUT_FINAL = 4, OUT_THETA = 5 };

// Tensor maps.  A row of a box is 64 elements, 128 bytes, swizzled.  An operand is read in boxes of 128 rows, or of 64
// where a block's share of it has no more, and written in boxes of 32.
enum : int { MAP_X0 = 0, MAP_X1 = 1, MAP_A = 2, MAP_B = 3, MAP_RESULT = 4, kMaps = 5 };
struct Maps {
  CUtensorMap load[4], load64[4], store[kMaps];
};

struct ChainParams {
  int rows, cols, side, length;  // of each matrix; its shorter and its longer side
  int batch, phases;             // phases: three products a step
  int tiles_sym, tiles_apply;    // tiles that are computed per matrix: of A and B, of X
  int tiles_n_sym, tiles_n_apply;  // tiles in a row of tiles
  int tn_sym, tn_apply;          // columns of a tile
  int* done;                     // [batch][phases]: arrivals of finished pieces of tiles
  const __half* a;               // A, for B = a I + b A + c A^2
  long long lda, stride_a;       // elements
  float ca, cb, cc;
  void* final_out;               // FINAL: dt_out; THETA: fp32 parameters
  int dt_out;
  long long ld_final, stride_final;
  float keep, rate;  // THETA: theta <- keep theta - rate O
  const int* go;     // 0: the selection refused, nothing is to be done.  Not info, which a block that gives up writes
                     // while others may still be starting: all blocks have to decide alike
  int32_t* info;     // optional: [1] receives SGDB_ERR_TIMEOUT
  unsigned long long wait_limit_ns;  // patience of each wait (see mbar_wait_for)
};

// The product of a phase: A = X X^T (tall: X^T X), B = a I + b A + c A^2, X <- B X (tall: X B).
struct Product {
  int kind, M, N, K, tiles, tiles_n, tn;
  int map_a, map_b, map_out;
  // for each operand: its rows run along K in memory (k is the slow index); or it is symmetric, of which (r, c) is
  // in memory where c >= r / g * g, with g the rows of a tile
  bool a_slow, b_slow, a_sym, b_sym;
};
__device__ __forceinline__ Product product_of(const ChainParams& p, int phase) {
  Product q;
  const int step = phase / 3;
  const bool tall = p.rows > p.cols;
  q.kind = phase % 3;
  const bool sym = q.kind != OUT_APPLY;
  q.M = sym ? p.side : p.rows;
  q.N = sym ? p.side : p.cols;
  q.K = q.kind == OUT_GRAM ? p.length : p.side;
  q.tiles = sym ? p.tiles_sym : p.tiles_apply;
  q.tiles_n = sym ? p.tiles_n_sym : p.tiles_n_apply;
  q.tn = sym ? p.tn_sym : p.tn_apply;
  const int x = MAP_X0 + (step & 1);
  q.map_a = q.kind == OUT_GRAM ? x : q.kind == OUT_POLY ? MAP_A : tall ? x : MAP_B;
  q.map_b = q.kind == OUT_GRAM ? x : q.kind == OUT_POLY ? MAP_A : tall ? MAP_B : x;
  q.map_out = q.kind == OUT_GRAM ? MAP_A : q.kind == OUT_POLY ? MAP_B : MAP_X0 + ((step + 1) & 1);
  q.a_slow = q.kind == OUT_GRAM && tall;
  q.b_slow = q.kind == OUT_GRAM ? tall : q.kind == OUT_APPLY && !tall;
  q.a_sym = q.kind == OUT_POLY || (q.kind == OUT_APPLY && !tall);
  q.b_sym = q.kind == OUT_POLY || (q.kind == OUT_APPLY && tall);
  return q;
}

// PAIR: tiles of 256 rows and 256 or 128 columns, from product to product; otherwise of 128 rows and 64 columns.
template <bool PAIR>
struct Shape {
  static constexpr int kTileM = PAIR ? 256 : 128;              // rows of a tile
  static constexpr int kTileN = PAIR ? 256 : 64;               // columns, at most
  static constexpr int kRowsB = PAIR ? 128 : 64;               // of B, per block, at most; of A 128
  static constexpr int kBytesA = 128 * kTileK * 2, kBytesB = kRowsB * kTileK * 2;
  static constexpr int kStageBytes = kBytesA + kBytesB;
  static constexpr int kWarps = PAIR ? 8 : 4;                  // that empty the accumulators
  static constexpr int kThreads = 64 + 32 * kWarps;
  static constexpr int kStages = 196608 / kStageBytes;         // 192 KB
  static constexpr int kSmem = kStages * kStageBytes + kWarps * kStoreBytes + 1024;
  static constexpr int kTmemColumns = 2 * kTileN;              // two accumulators
  static constexpr int kArrivals = PAIR ? 2 : 1;               // per tile
};

// A block's (pair's) walk through the tiles of all phases: every `step`-th of them.
struct Walk {
  int phase, index, step;  // index: within the phase, over all matrices
  Product q;
  __device__ __forceinline__ Walk(const ChainParams& p, int first, int step_) : phase(0), index(first), step(step_), q(product_of(p, 0)) {
    settle(p);
  }
  __device__ __forceinline__ void settle(const ChainParams& p) {
    while (phase < p.phases && index >= q.tiles * p.batch) {
      index -= q.tiles * p.batch;
      q = product_of(p, ++phase);
    }
  }
  __device__ __forceinline__ bool at_end(const ChainParams& p) const { return phase >= p.phases; }
  __device__ __forceinline__ void next(const ChainParams& p) {
    index += step;
    settle(p);
  }
  // Matrix, row of tiles and column of tiles.
  template <int TM>
  __device__ __forceinline__ void place(int* z, int* tm, int* tn) const {
    *z = index / q.tiles;
    int i = index - *z * q.tiles;
    if (q.kind == OUT_APPLY) {
      *tm = i / q.tiles_n;
      *tn = i - *tm * q.tiles_n;
      return;
    }
    int row = 0;
    while (true) {
      const int n = q.tiles_n - row * TM / q.tn;  // from the first column tile that reaches the diagonal on
      if (i < n) break;
      i -= n;
      ++row;
    }
    *tm = row;
    *tn = row * TM / q.tn + i;
  }
};

// The rows [row0, row0 + rows) of an operand are loaded with K as the slow index in the slices of K before the one that
// is returned.  For a symmetric operand: where the rows' part above the diagonal is not all there, its mirror image is.
template <int TM>
__device__ __forceinline__ int slow_slices(bool slow, bool sym, int row0, int rows) {
  return sym ? (row0 + rows - 1) / TM * TM / kTileK : slow ? 0x7fffffff : 0;
}

// Waits until the tiles of matrix z in the phase before are done; for a whole warp, with the same answer in all lanes.
__device__ __forceinline__ bool wait_done(const ChainParams& p, int phase, int z, int arrivals, volatile int* abort_flag) {
  if (phase == 0) return true;
  const int want = product_of(p, phase - 1).tiles * arrivals;
  const int* at = p.done + static_cast<long long>(z) * p.phases + phase - 1;
  unsigned long long deadline = 0;
  for (uint32_t spin = 0;; ++spin) {
    int have;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(have) : "l"(at) : "memory");
    if (__all_sync(0xffffffffu, have >= want)) return true;
    if (p.wait_limit_ns == 0) break;  // no patience at all: one probe decides
    if ((spin & 63u) == 63u) {
      const unsigned long long now = global_timer_ns();
      if (deadline == 0) deadline = now + p.wait_limit_ns;
      if (__any_sync(0xffffffffu, *abort_flag != 0 || now > deadline)) break;
    }
  }
  *abort_flag = 1;
  return false;
}

__device__ __forceinline__ void st_shared_v4(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// 16-bit outputs: 32 rows x 64 columns of the accumulator, lane = row.  Scaled, rounded, put into shared memory in the
// layout of the 128-byte swizzle and copied out from there.
template <int OUT>
__device__ __forceinline__ void emit_16bit(const ChainParams& p, const CUtensorMap* map, uint32_t acc, uint32_t stage,
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
__device__ __forceinline__ void load_theta(const ChainParams& p, long long z, int row0, int col0, int lane, float (&old)[32]) {
  const float* theta = static_cast<const float*>(p.final_out) + z * p.stride_final + row0 * p.ld_final + col0 + lane;
#pragma unroll
  for (int r = 0; r < 32; ++r) old[r] = row0 + r < p.rows && col0 + lane < p.cols ? theta[r * p.ld_final] : 0.0f;
}

// The last product, any type and alignment: 32 rows x 32 columns through shared memory, so that a warp writes along a row.
template <int OUT>
__device__ __forceinline__ void emit_final(const ChainParams& p, uint32_t acc, float* block, const float (&old)[32], long long z, int row0,
                                           int col0, int lane) {
  float v[32];
  tmem_load32(acc, v);
  tmem_load_wait(v);
  __syncwarp();
#pragma unroll
  for (int c = 0; c < 32; ++c) block[lane * 32 + (c ^ lane)] = v[c] * (1.0f / (kScale * kScale));
  __syncwarp();
  const int col = col0 + lane;
  if (col >= p.cols) return;
  const long long at = z * p.stride_final + row0 * p.ld_final + col;
#pragma unroll
  for (int r = 0; r < 32; ++r) {
    if (row0 + r >= p.rows) continue;
    const float o = block[r * 32 + (lane ^ r)];
    if (OUT == OUT_THETA)
      static_cast<float*>(p.final_out)[at + r * p.ld_final] = fmaf(-p.rate, o, p.keep * old[r]);
    else
      store_any(p.final_out, p.dt_out, at + r * p.ld_final, o);
  }
}

// The bounded wait of the other kernels for a whole warp, with the same answer in all lanes, and with some probes before it
// reads the clock.
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns) {
  if (limit_ns != 0) {
#pragma unroll 1
    for (int i = 0; i < 128; ++i)
      if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  }
  return __all_sync(0xffffffffu, mbar_wait_for(bar, parity, abort_flag, limit_ns));
}

// A slot's share of an operand: ROWS rows (along M or N) from `row` on, kTileK columns from `k` on, as boxes that a
// descriptor of smem_descriptor describes.
template <bool PAIR, int ROWS>
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* map, const CUtensorMap* map64, bool slow_k, int row, int k, int z,
                                             uint32_t bar) {
  const auto box = [&](uint32_t to, const CUtensorMap* m, int x, int y) {
    if (PAIR)
      tma_load_3d_pair(to, m, x, y, z, bar);
    else
      tma_load_3d(to, m, x, y, z, bar);
  };
  if (slow_k) {
#pragma unroll
    for (int i = 0; i < ROWS; i += 64) box(dst + i * kTileK * 2, map, row + i, k);
  } else {
#pragma unroll
    for (int i = 0; i < kTileK; i += 64) box(dst + ROWS * i * 2, ROWS == 64 ? map64 : map, k + i, row);
  }
}

// After a wait that ran out: ends when all copies into this block's (pair's) ring have landed.  The copies of both blocks of
// a pair are counted by the first one's barriers, but the blocks may have stopped at different slots.  A slot that both have
// filled completes by itself; for one that only one of them has, the other's part is entered here by one thread of the first
// block.  The lead is at most the ring: a slot is filled again only when the matrix instructions have read both shares.
// `issued`: slots filled by each block.
template <bool PAIR>
__device__ __noinline__ void end_copies(const ChainParams& p, const uint64_t* full, uint32_t issued0, uint32_t issued1) {
  using S = Shape<PAIR>;
  const uint32_t low = issued0 < issued1 ? issued0 : issued1, high = issued0 < issued1 ? issued1 : issued0;
  const uint32_t from = high > S::kStages ? high - S::kStages : 0;
  uint32_t at = 0;  // number of a tile's first slot
  for (Walk w(p, PAIR ? blockIdx.x >> 1 : blockIdx.x, PAIR ? gridDim.x >> 1 : gridDim.x); at < high && !w.at_end(p); w.next(p)) {
    const uint32_t next = at + (w.q.K + kTileK - 1) / kTileK;
    const uint32_t share = S::kBytesA + (PAIR ? w.q.tn >> 1 : 64) * kTileK * 2;  // bytes of one block
    for (uint32_t i = at > from ? at : from; i < next && i < high; ++i) {
      const uint32_t bar = smem_addr(&full[i % S::kStages]);
      if (i >= low) {
        if (issued0 > i)
          mbar_complete_tx(bar, share);  // the first block expects both shares
        else
          mbar_arrive_expect_tx(bar, share);  // nobody expects the second block's
      }
      int ignore = 0;
      (void)mbar_wait_for(bar, (i / S::kStages) & 1, &ignore, kWaitLimitNs);
    }
    at = next;
  }
}

// All products.  Warp 0 issues the copies of 128-wide slices of both operands into a ring, warp 1 the matrix instructions,
// the other warps read the finished tile from one accumulator while the next tile is summed in the other.
// PAIR: two blocks on neighbouring SMs share a tile of 256 rows; each holds 128 rows of A and of the accumulator and half
// of the columns of B, so that shared memory is read half as often per product; the first block's warp 1 issues for both.
template <bool PAIR, int LAST>
__global__ void __launch_bounds__(Shape<PAIR>::kThreads, 1)
    newton_schulz_kernel(const __grid_constant__ Maps maps, const __grid_constant__ ChainParams p) {
  using S = Shape<PAIR>;
  constexpr int TM = S::kTileM;
  extern __shared__ uint8_t smem_raw[];
  // the same offset in both blocks of a pair: dynamic shared memory starts at the same address in every block
  const uint32_t ring = (smem_addr(smem_raw) + 1023) & ~1023u;
  const uint32_t staging = ring + S::kStages * S::kStageBytes;
  __shared__ __align__(8) uint64_t s_full[S::kStages], s_empty[S::kStages], s_done[2], s_free[2], s_end;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort, s_partner_abort;
  __shared__ int s_left[2];          // one of the warps that empty the accumulators gave up, at an even or an odd tile
  __shared__ uint32_t s_issued[2];   // slots filled by this block or by the pair's two
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // warp: known to be uniform
  const uint32_t rank = PAIR ? cluster_rank() : 0;

  const int go = __ldcg(p.go);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 4; ++i) {
      prefetch_map(&maps.load[i]);
      prefetch_map(&maps.load64[i]);
    }
    for (int i = 0; i < kMaps - (LAST == OUT_BF16 ? 0 : 1); ++i) prefetch_map(&maps.store[i]);
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(smem_addr(&s_full[i]), 1);
      mbar_init(smem_addr(&s_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&s_done[i]), 1);
      mbar_init(smem_addr(&s_free[i]), S::kWarps * (PAIR ? 2 : 1));
    }
    mbar_init(smem_addr(&s_end), 1);
    s_abort = s_partner_abort = s_left[0] = s_left[1] = 0;
    s_issued[0] = s_issued[1] = 0;
    fence_barrier_init();
  }
  if (go == 0) return;  // the same for every block
  if (warp == 1) tmem_alloc<PAIR>(smem_addr(&s_tmem), S::kTmemColumns);
  tcgen05_before_sync();
  __syncthreads();
  if (PAIR) cluster_sync();  // the partner's barriers are ready before anything arrives at them
  tcgen05_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
  const int first = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;

  // Warps 0 and 1 run their loops as whole warps, so that addresses and descriptors stay in uniform registers, and one
  // elected lane issues.
  if (warp == 0) {
    const bool leader = elect_one();
    uint32_t it = 0;
    bool ok = true;
    for (Walk w(p, first, step); ok && !w.at_end(p); w.next(p)) {
      int tm, tn, z;
      w.place<TM>(&z, &tm, &tn);
      if (!wait_done(p, w.phase, z, S::kArrivals, &s_abort)) {
        ok = false;
        break;
      }
      fence_proxy_async();  // what the counter tells of was written by other blocks' copies; now come this one's
      const int rows_b = PAIR ? w.q.tn >> 1 : 64;  // of B, per block
      const int row0 = tm * TM + rank * 128, col0 = tn * w.q.tn + rank * rows_b;
      const int slow_a = slow_slices<TM>(w.q.a_slow, w.q.a_sym, tm * TM, TM), slow_b = slow_slices<TM>(w.q.b_slow, w.q.b_sym, tn * w.q.tn, w.q.tn);
      const CUtensorMap *map_a = &maps.load[w.q.map_a], *map_b = &maps.load[w.q.map_b], *map_b64 = &maps.load64[w.q.map_b];
      const int k_blocks = (w.q.K + kTileK - 1) / kTileK;
      for (int kb = 0; kb < k_blocks; ++kb, ++it) {
        const uint32_t slot = it % S::kStages, round = it / S::kStages;
        if (!wait_phase(smem_addr(&s_empty[slot]), (round & 1) ^ 1, &s_abort, p.wait_limit_ns)) {
          ok = false;
          break;
        }
        if (leader) {
          uint32_t bar = smem_addr(&s_full[slot]);
          if (rank == 0) mbar_arrive_expect_tx(bar, (S::kBytesA + rows_b * kTileK * 2) * (PAIR ? 2 : 1));
          if (PAIR) bar = cluster_address(bar, 0);
          const uint32_t dst = ring + slot * S::kStageBytes;
          load_operand<PAIR, 128>(dst, map_a, nullptr, kb < slow_a, row0, kb * kTileK, z, bar);
          if (rows_b == 128)
            load_operand<PAIR, 128>(dst + S::kBytesA, map_b, nullptr, kb < slow_b, col0, kb * kTileK, z, bar);
          else
            load_operand<PAIR, 64>(dst + S::kBytesA, map_b, map_b64, kb < slow_b, col0, kb * kTileK, z, bar);
        }
        __syncwarp();
      }
    }
    if (leader) s_issued[rank] = it;
    // the last slots are consumed: the arrivals that say so have come to both blocks of a pair before these end
    for (uint32_t i = it > S::kStages ? it - S::kStages : 0; ok && i < it; ++i)
      ok = wait_phase(smem_addr(&s_empty[i % S::kStages]), (i / S::kStages) & 1, &s_abort, p.wait_limit_ns);
  } else if (warp == 1 && rank == 0) {
    const bool leader = elect_one();
    uint32_t it = 0, count = 0;
    bool ok = true;
    for (Walk w(p, first, step); ok && !w.at_end(p); w.next(p), ++count) {
      const uint32_t buf = count & 1;
      int tm, tn, z;
      w.place<TM>(&z, &tm, &tn);
      const int slow_a = slow_slices<TM>(w.q.a_slow, w.q.a_sym, tm * TM, TM), slow_b = slow_slices<TM>(w.q.b_slow, w.q.b_sym, tn * w.q.tn, w.q.tn);
      const int k_blocks = (w.q.K + kTileK - 1) / kTileK;
      if (!wait_phase(smem_addr(&s_free[buf]), ((count >> 1) & 1) ^ 1, &s_abort, p.wait_limit_ns)) {
        ok = false;
        break;
      }
      tcgen05_after_sync();
      for (int kb = 0; kb < k_blocks; ++kb, ++it) {
        const uint32_t slot = it % S::kStages;
        const bool is_slow_a = kb < slow_a, is_slow_b = kb < slow_b;
        const uint32_t idesc = mma_descriptor_f16(TM, w.q.tn, is_slow_a, is_slow_b);
        const uint32_t at = (ring + slot * S::kStageBytes) >> 4;
        const uint64_t desc_a = smem_descriptor(is_slow_a) + at, desc_b = smem_descriptor(is_slow_b) + (at + (S::kBytesA >> 4));
        // 16-byte units from one K of 16 to the next, and from one 64 to the next
        const uint32_t step_a = is_slow_a ? 128 : 2, step_b = is_slow_b ? 128 : 2;
        const uint32_t half_a = is_slow_a ? 512 : 128 * 128 >> 4, half_b = is_slow_b ? 512 : (PAIR ? w.q.tn >> 1 : 64) * 128 >> 4;
        if (!wait_phase(smem_addr(&s_full[slot]), (it / S::kStages) & 1, &s_abort, p.wait_limit_ns)) {
          ok = false;
          break;
        }
        tcgen05_after_sync();
        if (leader) {
#pragma unroll
          for (int k = 0; k < kTileK / 16; ++k)
            mma_f16<PAIR>(tmem + buf * S::kTileN, desc_a + ((k & 3) * step_a + (k >> 2) * half_a), desc_b + ((k & 3) * step_b + (k >> 2) * half_b),
                          idesc, (kb | k) != 0);
          mma_commit<PAIR>(smem_addr(&s_empty[slot]));
        }
        __syncwarp();
      }
      if (ok && leader) mma_commit<PAIR>(smem_addr(&s_done[buf]));
    }
    // the instructions issued so far end before shared and tensor memory are given back, whoever gave up
    int ignore = 0;
    if (leader) mma_commit<PAIR>(smem_addr(&s_end), 1);
    (void)wait_phase(smem_addr(&s_end), 0, &ignore, kWaitLimitNs);
  } else if (warp >= 2) {
    const int quarter = warp & 3;  // the lanes of tensor memory that this warp may read
    const uint32_t stage = staging + (warp - 2) * kStoreBytes;
    float* block = reinterpret_cast<float*>(smem_raw + (stage - smem_addr(smem_raw)));
    // The warps meet at every tile but those of the last product, and go on or leave together: one that gives up says so
    // before the meeting, the others read it behind it.  The two flags are used in turn, so that a warp that is ahead, at the
    // next tile, does not write the one that is being read.
    const auto meet = [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * S::kWarps) : "memory"); };
    const auto leave = [&](uint32_t buf) {
      if (lane == 0) *static_cast<volatile int*>(&s_left[buf]) = 1;
      __syncwarp();
      meet();
    };
    uint32_t count = 0;
    for (Walk w(p, first, step); !w.at_end(p); w.next(p), ++count) {
      const uint32_t buf = count & 1;
      int tm, tn, z;
      w.place<TM>(&z, &tm, &tn);
      const int columns = PAIR ? w.q.tn >> 1 : 64, columns0 = PAIR ? (warp - 2) / 4 * columns : 0;  // this warp's share of the tile
      const int row0 = tm * TM + rank * 128 + quarter * 32, col_first = tn * w.q.tn + columns0;
      const bool last = w.phase == p.phases - 1;
      const int out = last ? LAST : w.q.kind;
      // B's tile needs A's, which is in memory when the operands of this product are; it is on its way while the tile is
      // computed.  64 columns of this lane's row; rows are padded to multiples of 64
      uint4 addend[8] = {};
      const auto load_addend = [&](int c) {
        const uint4* from = reinterpret_cast<const uint4*>(p.a + z * p.stride_a + (row0 + lane) * p.lda + col_first + c);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (row0 + lane < p.side && col_first + c < p.side) addend[i] = __ldcg(from + i);
      };
      if (out == OUT_POLY) {
        if (!wait_done(p, w.phase, z, S::kArrivals, &s_abort)) {
          leave(buf);  // B is never the last product
          break;
        }
        load_addend(0);
      }
      if (!wait_phase(smem_addr(&s_done[buf]), (count >> 1) & 1, &s_abort, p.wait_limit_ns)) {
        if (!last) leave(buf);
        break;
      }
      tcgen05_after_sync();
      const uint32_t acc = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + buf * S::kTileN + columns0;
      if (row0 < w.q.M && col_first < w.q.N) {
        if (!last || LAST == OUT_BF16) {
          const CUtensorMap* map = &maps.store[LAST == OUT_BF16 && last ? MAP_RESULT : w.q.map_out];
          for (int c = 0; c < columns && col_first + c < w.q.N; c += 64) {
            const int col0 = col_first + c;
            if (out == OUT_POLY) {
              emit_16bit<OUT_POLY>(p, map, acc + c, stage, addend, z, row0, col0, lane);
              if (c + 64 < columns) load_addend(c + 64);
            } else if (LAST == OUT_BF16 && last) {
              emit_16bit<OUT_BF16>(p, map, acc + c, stage, addend, z, row0, col0, lane);
            } else {
              emit_16bit<OUT_APPLY>(p, map, acc + c, stage, addend, z, row0, col0, lane);
            }
          }
        } else if constexpr (LAST != OUT_BF16) {
          for (int c = 0; c < columns && col_first + c < w.q.N; c += 32) {
            float old[32];
            if (LAST == OUT_THETA) load_theta(p, z, row0, col_first + c, lane, old);
            emit_final<LAST>(p, acc + c, block, old, z, row0, col_first + c, lane);
          }
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
        bulk_wait_all();  // the copies are complete
      }
      if (!last) {  // one arrival for the block's part of the tile
        meet();
        if (threadIdx.x == 64) {
          asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(p.done + static_cast<long long>(z) * p.phases + w.phase) : "memory");
        }
        // read behind the arrival, which is what others wait for; one for a tile that is not whole only lets them compute what
        // the time-out declares lost
        if (*static_cast<volatile int*>(&s_left[buf]) != 0) break;
      }
    }
  }
  __syncwarp();
  tcgen05_before_sync();
  __syncthreads();
  // no block leaves, or gives tensor memory back, while its partner may still reach it; here each tells whether it gave up
  if (PAIR) {
    if (threadIdx.x == 0 && s_abort != 0) st_shared_cluster(cluster_address(smem_addr(&s_partner_abort), cluster_rank() ^ 1), 1);
    __syncwarp();
    cluster_sync();
  }
  tcgen05_after_sync();
  // Otherwise every slot has been read by the matrix instructions, which are done.  (Ranks and sizes are read anew here: kept
  // from the beginning they cost the loops above registers, and up to 12 % of the whole chain.)
  if (s_abort != 0 || (PAIR && s_partner_abort != 0)) {
    if (PAIR) {
      if (threadIdx.x == 0 && cluster_rank() != 0) st_shared_cluster(cluster_address(smem_addr(&s_issued[1]), 0), s_issued[1]);
      __syncwarp();
      cluster_sync();
    }
    if (threadIdx.x == 0 && (!PAIR || cluster_rank() == 0)) end_copies<PAIR>(p, s_full, s_issued[0], PAIR ? s_issued[1] : s_issued[0]);
    __syncthreads();
    if (PAIR) cluster_sync();
    if (threadIdx.x == 0 && p.info != nullptr) p.info[1] = SGDB_ERR_TIMEOUT;
  }
  if (warp == 1) tmem_dealloc<PAIR>(tmem, S::kTmemColumns);
}

// ---------------------------------------------------------------- before the products

struct NormParams {
  const void* u;  // dt_in
  int dt_in;
  int rows, cols;
  long long ld, stride;
  double* partials;  // [batch][kNormBlocks], the first n_partials in use
  int n_partials;
  __half* x;
  long long ldx, stride_x;
  float eps;
  int *done, n_done;  // the products' counters, set to zero here
  const int32_t* info;
  int* go;  // set here: whether the products are to run
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

// Partial sums of squares of each matrix, in 64 bits: the square of an fp32 number may be out of fp32's range.
template <typename T, bool VEC>
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
    float v[kPieces][P::kV];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int col = col0 + i * 32 * P::kV;
      if (col < p.cols) load_piece<T, VEC>(static_cast<const T*>(p.u) + at + col, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      if (col0 + i * 32 * P::kV < p.cols) {
#pragma unroll
        for (int e = 0; e < P::kV; ++e) sum = fma(static_cast<double>(v[i][e]), static_cast<double>(v[i][e]), sum);
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
  const bool refused = p.info != nullptr && p.info[1] != SGDB_OK;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.go = !refused;
  if (refused) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per_row = (p.cols + P::kWidth - 1) / P::kWidth, warps = gridDim.x * (kNormThreads / 32);
  const long long z = blockIdx.y, units = static_cast<long long>(p.rows) * per_row;
  double sum = 0.0;
  for (int b = lane; b < p.n_partials; b += 32) sum += p.partials[z * kNormBlocks + b];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int i = threadIdx.x; i < p.n_done; i += kNormThreads) p.done[i] = 0;
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
  size_t x0, x1, a, b, partials, done, go, u, total;  // byte offsets in the workspace
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
  q->done = take(n * 3 * SGDB_MAX_STEPS * sizeof(int));
  q->go = take(sizeof(int));
  q->u = at;
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

// Tiles that are computed of a product of M x N, and those in a row of tiles.
long long count_tiles(int tm, int tn, int M, int N, bool sym, int* tiles_n) {
  const int tiles_m = (M + tm - 1) / tm;
  *tiles_n = (N + tn - 1) / tn;
  long long n = 0;
  for (int i = 0; i < tiles_m; ++i) n += *tiles_n - (sym ? i * tm / tn : 0);
  return n;
}

template <bool PAIR, int LAST>
sgdb_status_t launch_chain(const Maps& maps, ChainParams p, const DeviceInfo* dev, cudaStream_t s) {
  using S = Shape<PAIR>;
  constexpr int kCluster = PAIR ? 2 : 1;
  const long long sym = count_tiles(S::kTileM, p.tn_sym, p.side, p.side, true, &p.tiles_n_sym);
  const long long apply = count_tiles(S::kTileM, p.tn_apply, p.rows, p.cols, false, &p.tiles_n_apply);
  p.tiles_sym = static_cast<int>(sym);
  p.tiles_apply = static_cast<int>(apply);
  auto kernel = newton_schulz_kernel<PAIR, LAST>;
  cudaLaunchConfig_t cfg{};
  cfg.blockDim = dim3(S::kThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kCluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeCooperative;
  attr[1].val.cooperative = 1;
  cfg.attrs = attr;
  // blocks (pairs) that are resident at once: the blocks wait for one another, so there may be no more
  static std::atomic<int> resident[kMaxDevices];
  int most = resident[dev->index].load(std::memory_order_relaxed);
  if (most == 0) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem) != cudaSuccess) return launch_status();
    cfg.gridDim = dim3(dev->sms / kCluster * kCluster);
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&most, kernel, &cfg) != cudaSuccess) return launch_status();
    if (most < 1) return SGDB_ERR_UNSUPPORTED;
    resident[dev->index].store(most, std::memory_order_relaxed);
  }
  const long long want = (sym > apply ? sym : apply) * p.batch;
  cfg.gridDim = dim3(static_cast<unsigned>(want < most ? want : most) * kCluster);
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, kernel, maps, p);
  return launch_status();
}

// What a product takes in each tile shape, in microseconds, fitted to measurements of 23 shapes and batches from 64 to 4096:
// its latency (from one tile's end to the counter to the next tile's operands), and per round of tiles a cost and one
// for each 128 of K.  With one shape for all products the fit is within 25 % everywhere and picks the fastest of the
// three for all of the 23, for example (256 x 256 / 256 x 128 / 128 x 64): one of 256 x 256 108 / 80 / 62 us, 1024 x 1024
// 162 / 112 / 95, 2048 x 2048 244 / 204 / 294, 4096 x 4096 1028 / 1248 / 2286, 16 of 512 x 1408 189 / 178 / 217, 8 of
// 1024 x 2048 297 / 338 / 511.  Pairs then choose their columns for the symmetric products and for X apart.
struct TileCost {
  int rows, columns, blocks;
  double latency, round, depth;
};
constexpr TileCost kPair256{256, 256, 2, 3.7, 0.5, 0.79}, kPair128{256, 128, 2, 2.7, 1.0, 0.45}, kSingle64{128, 64, 1, 2.4, 0.3, 0.42};

// The two symmetric products, or X's, of one step.
double product_cost(const TileCost& c, const Plan& q, bool sym, const DeviceInfo* dev) {
  int unused;
  const long long tiles = count_tiles(c.rows, c.columns, sym ? q.side : q.rows, sym ? q.side : q.cols, sym, &unused);
  double rounds = static_cast<double>(tiles) * q.batch / (dev->sms / c.blocks);
  // one matrix's products follow one another; of several, the tiles of one fill the gaps of the others
  rounds = q.batch == 1 ? std::ceil(rounds) : std::fmax(1.0, rounds);
  const auto at = [&](int depth) { return c.latency + rounds * (c.round + (depth + kTileK - 1) / kTileK * c.depth); };
  return sym ? at(q.rows + q.cols - q.side) + at(q.side) : at(q.side);
}

template <int LAST>
sgdb_status_t launch_chain(const Maps& maps, ChainParams p, const Plan& q, const DeviceInfo* dev, cudaStream_t s) {
  double pair = 0.0;
  for (const bool sym : {true, false}) {
    const double wide = product_cost(kPair256, q, sym, dev), narrow = product_cost(kPair128, q, sym, dev);
    (sym ? p.tn_sym : p.tn_apply) = wide < narrow ? 256 : 128;
    pair += std::fmin(wide, narrow);
  }
  if (pair <= product_cost(kSingle64, q, true, dev) + product_cost(kSingle64, q, false, dev)) return launch_chain<true, LAST>(maps, p, dev, s);
  p.tn_sym = p.tn_apply = 64;
  return launch_chain<false, LAST>(maps, p, dev, s);
}

bool rule_ok(const sgdb_newton_schulz_t* ns) {
  return ns != nullptr && ns->steps >= 1 && ns->steps <= SGDB_MAX_STEPS && std::isfinite(ns->a) && std::isfinite(ns->b) &&
         std::isfinite(ns->c) && ns->eps >= 0.0f && !std::isinf(ns->eps);
}

// Whether X, A and B, times kScale, stay within fp16 for every U.  The singular values of X begin in [0, 1] and go through
// s p(s^2) with p(t) = a + b t + c t^2; no element of a matrix is larger than its largest singular value.  2 % per step
// are left for the roundings.  The last X is not kept in fp16.
bool rule_in_range(const sgdb_newton_schulz_t& ns) {
  constexpr double kMost = 65504.0 / kScale, kRoom = 1.02;
  const double a = ns.a, b = ns.b, c = ns.c;
  const auto p = [&](double t) { return a + t * (b + t * c); };
  double most = kRoom;  // singular value of X
  for (int step = 0; step < ns.steps; ++step) {
    const double t1 = most * most;
    double of_b = std::fmax(std::fabs(p(0.0)), std::fabs(p(t1)));
    if (c != 0.0 && -b / (2.0 * c) > 0.0 && -b / (2.0 * c) < t1) of_b = std::fmax(of_b, std::fabs(p(-b / (2.0 * c))));
    if (!(most <= kMost && t1 <= kMost && of_b * kRoom <= kMost)) return false;
    // the extremes of s p(s^2): the end, and where a + 3 b t + 5 c t^2 = 0
    double next = most * std::fabs(p(t1));
    const double root = std::sqrt(9.0 * b * b - 20.0 * a * c);  // not a number: none
    for (const double t : {c != 0.0 ? (-3.0 * b + root) / (10.0 * c) : -a / (3.0 * b), c != 0.0 ? (-3.0 * b - root) / (10.0 * c) : -1.0})
      if (t > 0.0 && t < t1) next = std::fmax(next, std::sqrt(t) * std::fabs(p(t)));
    most = next * kRoom;
  }
  return true;
}

// X is in place (q.x0): the products, and what is done with the last one, which f's final_ members and `last` tell.
// `result`: the output's map when `last` is OUT_BF16.
sgdb_status_t run_products(const Plan& q, const sgdb_newton_schulz_t& ns, char* ws, int last, const ChainParams& f,
                           const CUtensorMap* result, int32_t* info, const DeviceInfo* dev, cudaStream_t s) {
  Maps maps;
  __half* const base[4] = {reinterpret_cast<__half*>(ws + q.x0), reinterpret_cast<__half*>(ws + q.x1), reinterpret_cast<__half*>(ws + q.a),
                           reinterpret_cast<__half*>(ws + q.b)};
  sgdb_status_t st = SGDB_OK;
  for (int i = 0; i < 4 && st == SGDB_OK; ++i) {
    const bool x = i == MAP_X0 || i == MAP_X1;
    const int rows = x ? q.rows : q.side, cols = x ? q.cols : q.side;
    const long long ld = x ? q.ldx : q.lds, stride = x ? q.stride_x : q.stride_s;
    st = make_map(&maps.load[i], base[i], rows, cols, ld, stride, q.batch, 128);
    if (st == SGDB_OK) st = make_map(&maps.load64[i], base[i], rows, cols, ld, stride, q.batch, 64);
    if (st == SGDB_OK) st = make_map(&maps.store[i], base[i], rows, cols, ld, stride, q.batch, 32);
  }
  if (st != SGDB_OK) return st;
  maps.store[MAP_RESULT] = result != nullptr ? *result : maps.store[MAP_X0];
  ChainParams p = f;
  p.rows = q.rows;
  p.cols = q.cols;
  p.side = q.side;
  p.length = q.rows > q.cols ? q.rows : q.cols;
  p.batch = q.batch;
  p.phases = 3 * ns.steps;
  p.done = reinterpret_cast<int*>(ws + q.done);
  p.a = base[MAP_A];
  p.lda = q.lds;
  p.stride_a = q.stride_s;
  p.ca = ns.a, p.cb = ns.b, p.cc = ns.c;
  p.go = reinterpret_cast<const int*>(ws + q.go);
  p.info = info;
  p.wait_limit_ns = wait_limit_ns();
  return last == OUT_BF16    ? launch_chain<OUT_BF16>(maps, p, q, dev, s)
         : last == OUT_THETA ? launch_chain<OUT_THETA>(maps, p, q, dev, s)
                             : launch_chain<OUT_FINAL>(maps, p, q, dev, s);
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
  const sgdb_status_t st = launch_dependent(square_sum_kernel<T, VEC>, sums, kNormThreads, 0, s, p);
  if (st != SGDB_OK) return st;
  return launch_dependent(normalise_kernel<T, VEC>, dim3(blocks(8, 1 << 20), batch), kNormThreads, 0, s, p);
}

sgdb_status_t run_normalise(const NormParams& p, int batch, const DeviceInfo* dev, cudaStream_t s) {
  const bool vec = rows_aligned16(p.u, p.ld, p.dt_in) && (batch == 1 || rows_aligned16(p.u, p.stride, p.dt_in)) && p.cols % 8 == 0;
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
  if (!rule_in_range(*ns)) return SGDB_ERR_UNSUPPORTED;
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
  n.n_done = batch * 3 * ns->steps;
  n.info = d_info;
  n.done = reinterpret_cast<int*>(ws + q.done);
  n.go = reinterpret_cast<int*>(ws + q.go);
  st = run_normalise(n, batch, dev, s);
  if (st != SGDB_OK) return st;
  ChainParams f{};
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
  if (!array_ok(d_theta, SGDB_F32) || !array_ok(d_momentum, SGDB_F32)) return SGDB_ERR_INVALID_ARG;
  if (batch > 0 && (d_workspace == nullptr || workspace_bytes < q.total)) return SGDB_ERR_INVALID_ARG;
  if (!rule_in_range(opt->newton_schulz)) return SGDB_ERR_UNSUPPORTED;
  const DeviceInfo* dev = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  char* ws = align_workspace(d_workspace);
  float* u = batch > 0 ? reinterpret_cast<float*>(ws + q.u) : nullptr;
  sgdb_status_t st = select_and_velocity(d_grad, dt, static_cast<int64_t>(batch) * rows * cols, ld, d_arrival, d_tags, t, N, b, d_momentum, u,
                                         opt->momentum, opt->nesterov != 0, d_mask, d_order, d_info, s);
  if (st != SGDB_OK || batch == 0) return st;
  st = device_info(&dev);
  if (st != SGDB_OK) return st;
  NormParams n{};
  n.u = u;
  n.dt_in = SGDB_F32;
  n.rows = q.rows;
  n.cols = q.cols;
  n.ld = cols;
  n.stride = rows * cols;
  n.partials = reinterpret_cast<double*>(ws + q.partials);
  n.x = reinterpret_cast<__half*>(ws + q.x0);
  n.ldx = q.ldx;
  n.stride_x = q.stride_x;
  n.eps = opt->newton_schulz.eps;
  n.n_done = batch * 3 * opt->newton_schulz.steps;
  n.info = d_info;
  n.done = reinterpret_cast<int*>(ws + q.done);
  n.go = reinterpret_cast<int*>(ws + q.go);
  st = run_normalise(n, batch, dev, s);
  if (st != SGDB_OK) return st;
  ChainParams f{};
  f.final_out = d_theta;
  f.ld_final = cols;
  f.stride_final = rows * cols;
  f.keep = static_cast<float>(1.0 - static_cast<double>(opt->lr) * static_cast<double>(opt->weight_decay));
  f.rate = opt->lr * opt->scale;
  return run_products(q, opt->newton_schulz, ws, OUT_THETA, f, nullptr, d_info, dev, s);
}

}  // extern "C"
