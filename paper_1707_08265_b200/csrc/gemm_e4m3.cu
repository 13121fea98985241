// ScaledInnerProduct  Y[m,n] = sum_b sx[m,b] sw[n/128,b] sum_{k in block b} Xq[m,k] Wq[n,k]: e4m3 operands with a scale for
// each block of 128 along K, fp32 accumulation, fp32 or bf16 output.  Hand-written for sm_100a.
//
// The scales change every 128 elements of K, so the tensor unit may accumulate over one block only (four
// tcgen05.mma.kind::f8f6f4 of K = 32).  TMEM accumulators take turns: while the tensor unit works on the next block, the
// epilogue warps read this block's sums with tcgen05.ld and add them, times their scale, to fp32 registers (packed FMAs).
// One block is one TMA stage (128-byte rows, 128-byte swizzle).
// The scale is the fp32 product of the operands' two.  Multiplying by one and then by the other where that product leaves the
// normal range was tried: 8192 x 8192 x 4096 287 us for 256 with a condition in the loop over the columns, 315 to 340 with a loop
// of its own for those blocks (the sums hold all registers); the range is documented instead.
//
//   gemm_e4m3_kernel      many rows: two CTAs of a cluster work on one tile of 256 rows of X x 256 rows of W
//                         (tcgen05.mma.cta_group::2), so that a CTA copies 32 KB a block instead of the 48 KB of a 128 x 256 tile
//                         of its own.  A thread holds one row of Y and 128 columns, its scale is one number a block; persistent
//                         pairs in an L2-friendly tile order.  Measured, 8192 x 8192 x 4096: 250 us by itself (2.2 PFLOP/s), 308 us
//                         in a loop under the power limit (1.8).  A block of a tile takes 0.52 us: its products alone 0.28, with
//                         the copies 0.37 (13 TB/s out of L2), with the hand-over of the accumulators but no work on them 0.41.
//                         TMEM holds two blocks' sums, so the products of a block wait for the work on the one before the last.
//                         Slower: accumulators of half a tile (A is read twice), 16 epilogue warps of 64 columns (spills), a
//                         release before the last sums (no gain).
//   gemm_e4m3_few_kernel  few rows: the operands change places (128 rows of W x 16..128 rows of X), so that the tile's height is
//                         filled by weights and hardly any product is wasted; the K blocks of a tile are split over the
//                         CTAs of a cluster, whose partial sums meet in shared memory in a fixed order.  5 x 8192 x 4096: 11.4 us, one call
//                         after another (34 MB of weights: 5.1 us at the measured bandwidth; the rest is the first bytes' latency
//                         and the join); 256 x 8192 x 16384: a block 0.5 us, copies out of L2
// Every wait is bounded; when one runs out the kernel records DRAGON_ERR_TIMEOUT, lets its copies and products in flight
// land, frees its TMEM and returns.
#include <algorithm>
#include <cstdlib>

#include "device_util.h"
#include "plan.h"
#include "tcgen05_util.h"

namespace dragon {
namespace {

constexpr int kBlockK = 128;        // one scale block = one 128-byte swizzle row of e4m3 = one stage
constexpr int kUmmaK = 32;
constexpr int kBufs = 4;            // accumulators in TMEM that take turns

// instruction descriptor of kind::f8f6f4: D = f32, A = B = e4m3 (both codes 0), K-major, M x N
constexpr uint32_t idesc_e4m3(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// two neighbouring columns' sums as one 64-bit register: acc += v * s
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pack(float lo, float hi) { Pair p; asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi)); return p; }
__device__ __forceinline__ float2 unpack(Pair p) { float2 v; asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p)); return v; }
__device__ __forceinline__ void fma_pair(Pair& acc, uint32_t v0, uint32_t v1, Pair s) {
  Pair v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(v0), "r"(v1));
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(v), "l"(s));
}

// the same by a pair: 256 rows of A and N columns over both CTAs' shared memory and TMEM
__device__ __forceinline__ void umma_e4m3_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

struct Gemm8Args {
  const float *sx, *sw;
  void* y;
  int ydt, M, N, K, kb;        // kb: blocks along K
  int tiles_m, tiles_n;
  int split;                   // few rows: CTAs of a cluster that share a tile's blocks
  int* status;
  int* status_clear;
  long long wait_budget;
  int drop_first_load;         // failure-detection test: the first stage's signal never comes
};

// barriers and flags of a CTA, behind its stages
struct Sync {
  uint32_t full, empty, part_full, part_empty, drain;
  uint32_t* tmem_slot;
  volatile int* abort_flag;
};
__device__ __forceinline__ Sync sync_area(unsigned char* p, int stages) {
  uint64_t* bars = reinterpret_cast<uint64_t*>(p);
  Sync s;
  s.full = smem_u32(bars);
  s.empty = s.full + 8 * stages;
  s.part_full = s.empty + 8 * stages;
  s.part_empty = s.part_full + 8 * kBufs;
  s.drain = s.part_empty + 8 * kBufs;
  s.tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * stages + 2 * kBufs + 1);
  s.abort_flag = reinterpret_cast<volatile int*>(s.tmem_slot + 1);
  return s;
}
__device__ __forceinline__ void sync_init(const Sync& s, int stages, int epilogue_warps) {
  for (int i = 0; i < stages; ++i) { mbar_init(s.full + 8 * i, 1); mbar_init(s.empty + 8 * i, 1); }
  for (int b = 0; b < kBufs; ++b) { mbar_init(s.part_full + 8 * b, 1); mbar_init(s.part_empty + 8 * b, epilogue_warps); }
  mbar_init(s.drain, 1);
  s.abort_flag[0] = 0;
  s.abort_flag[1] = 0;         // nobody sets this one: for waits that must not be cut short
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ bool wait_or_abort(const Sync& s, const Gemm8Args& g, uint32_t bar, uint32_t parity) {
  if (mbar_wait(bar, parity, s.abort_flag, g.wait_budget)) return true;
  *s.abort_flag = 1;
  atomicExch(g.status, DRAGON_ERR_TIMEOUT);
  return false;
}
// the copies that nobody consumed must land before the shared memory goes away (full budget, whatever the pipeline's is)
__device__ __forceinline__ void drain_copies(const Sync& s, int first, int issued, int stages) {
  for (int i = max(first, issued > stages ? issued - stages : 0); i < issued; ++i) mbar_wait(s.full + 8 * (i % stages), (i / stages) & 1, s.abort_flag + 1);
}

// ... and the products in flight (the thread that issued them) before their operands and the TMEM do
__device__ __forceinline__ void drain_products(const Sync& s) {
  umma_commit(s.drain);
  mbar_wait(s.drain, 0, s.abort_flag + 1);
}

// The MMA issuer's work on one block: wait for an accumulator and the stage, four products, hand both on
__device__ __forceinline__ bool issue_block(const Sync& s, const Gemm8Args& g, int it, int stages, uint32_t a_addr, uint32_t b_addr, uint32_t tmem, int columns, uint32_t idesc) {
  const int buf = it % kBufs, st = it % stages;
  if (!wait_or_abort(s, g, s.part_empty + 8 * buf, ((it / kBufs) & 1) ^ 1)) return false;
  if (!wait_or_abort(s, g, s.full + 8 * st, (it / stages) & 1)) return false;
  fence_after();
  const uint64_t a = make_smem_desc(a_addr), b = make_smem_desc(b_addr);
#pragma unroll
  for (int k = 0; k < kBlockK / kUmmaK; ++k) umma_e4m3(tmem + buf * columns, a + 2 * k, b + 2 * k, idesc, k > 0 ? 1u : 0u);   // 32 bytes along the swizzle row
  umma_commit(s.empty + 8 * st);
  umma_commit(s.part_full + 8 * buf);
  return true;
}

// ---- many rows ------------------------------------------------------------------------------------------------

constexpr int kTileM = 256, kTileN = 256, kStages = 6;          // of a pair; a CTA holds 128 rows of X and 128 of W
constexpr int kEpiWarps = 8, kEpiThreads = 32 * kEpiWarps;      // two warps a quarter of the lanes, 128 columns of it each: all the registers there are
constexpr int kFetchWarps = 2;
constexpr int kThreads = 64 + kEpiThreads + 32 * kFetchWarps;   // TMA, MMA, epilogue, scales
constexpr int kTileBufs = 2;                                    // accumulators that take turns: all of TMEM
constexpr int kEpiCols = kTileN * 4 / kEpiWarps;                // columns of a warp
constexpr uint32_t kHalfBytes = 128 * kBlockK, kStageBytes = 2 * kHalfBytes;
constexpr int kScaleBlocks = 16;                                // blocks whose scales are fetched together
// scales of kScaleBlocks blocks: of this CTA's 128 rows of X, and of the tile's two 128-row blocks of W; two sets
struct TileScales { float x[kScaleBlocks][128]; float w[2][kScaleBlocks]; };
constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + 256 + 2 * sizeof(TileScales);

__device__ __forceinline__ void copy_async4(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
// the fetching threads copy the scales of blocks b0.. of the tile at (row0, n-block nb0); what is outside repeats the last
__device__ __forceinline__ void fetch_scales(const Gemm8Args& g, TileScales& to, int tid, int row0, int nb0, int b0) {
  for (int r = tid; r < 128; r += 32 * kFetchWarps) {
    const float* sx = g.sx + (size_t)min(row0 + r, g.M - 1) * g.kb;
#pragma unroll
    for (int b = 0; b < kScaleBlocks; ++b) copy_async4(&to.x[b][r], sx + min(b0 + b, g.kb - 1));
  }
  for (int i = tid; i < 2 * kScaleBlocks; i += 32 * kFetchWarps) {
    const int h = i / kScaleBlocks, b = i % kScaleBlocks;
    copy_async4(&to.w[h][b], g.sw + (size_t)min(nb0 + h, (g.N - 1) / 128) * g.kb + min(b0 + b, g.kb - 1));
  }
}

// A warp holds 32 rows, a row to a lane; written like that, every 16 bytes would be half a sector of its own (a tile of bf16
// took 5 us; with the exchanges below 2).  Eight neighbouring lanes exchange pieces of 16 bytes: piece u of lane p becomes
// piece p of lane u.
__device__ __forceinline__ void exchange(uint32_t& lo, uint32_t& hi, int lane, int b) {
  const uint32_t got = __shfl_xor_sync(0xffffffffu, lane & b ? lo : hi, b);
  if (lane & b) lo = got; else hi = got;
}
__device__ __forceinline__ void exchange_pieces(uint32_t (&v)[32], int lane) {
#pragma unroll
  for (int b = 1; b < 8; b <<= 1)
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (!(u & b))
#pragma unroll
        for (int i = 0; i < 4; ++i) exchange(v[4 * u + i], v[4 * (u | b) + i], lane, b);
}
// 32 rows' lines of 128 bytes (of 16-byte pieces whose first column is below `cols`), each written as a whole by 8 lanes
template <bool kF32>
__device__ __forceinline__ void store_lines(char* y, size_t row_bytes, int rows_left, int col0, int cols, uint32_t (&v)[32], int lane) {
  exchange_pieces(v, lane);
  if (col0 + (lane & 7) * (kF32 ? 4 : 8) >= cols) return;
  char* at = y + (lane & 24) * row_bytes + (lane & 7) * 16;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if ((lane & 24) + i < rows_left) *reinterpret_cast<uint4*>(kF32 ? at : at + i * row_bytes) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    if (kF32) at += row_bytes;           // (one address in registers, where four parts of a row would spill them)
  }
}
// ... and where rows do not start at 16-byte boundaries: word u of lane p becomes word p of lane u, and the warp writes one
// row after another
template <bool kF32>
__device__ __forceinline__ void store_words(char* y, size_t row_bytes, int rows_left, int col0, int cols, uint32_t (&v)[32], int lane) {
#pragma unroll
  for (int b = 1; b < 32; b <<= 1)
#pragma unroll
    for (int u = 0; u < 32; ++u)
      if (!(u & b)) exchange(v[u], v[u | b], lane, b);
  const int left = cols - col0 - (kF32 ? lane : 2 * lane);
  char* at = y + 4 * lane;
#pragma unroll
  for (int r = 0; r < 32; ++r, at += row_bytes) {
    if (r >= rows_left) break;
    if (kF32) {
      if (left > 0) *reinterpret_cast<uint32_t*>(at) = v[r];
    } else if (cols % 2 == 0) {
      if (left > 0) *reinterpret_cast<uint32_t*>(at) = v[r];
    } else {
      if (left > 0) *reinterpret_cast<unsigned short*>(at) = (unsigned short)v[r];
      if (left > 1) *reinterpret_cast<unsigned short*>(at + 2) = (unsigned short)(v[r] >> 16);
    }
  }
}

// One kernel for each way to write a tile: with all of them in one the registers spill (285 us instead of 260).
template <bool kF32, bool kLines>
__global__ void __launch_bounds__(kThreads, 1)
gemm_e4m3_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_w, const Gemm8Args g) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), tiles = (raw + 1023u) & ~1023u;
  const Sync s = sync_area(smem_raw + (tiles - raw) + (size_t)kStages * kStageBytes, kStages);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_tiles = g.tiles_m * g.tiles_n, n_units = (int)(gridDim.x >> 1), unit = (int)(blockIdx.x >> 1);
  const uint32_t rank = cluster_ctarank();
  if (threadIdx.x == 0) {
    sync_init(s, kStages, 2 * kEpiWarps);                       // (both CTAs' epilogue warps; only the first CTA's part_empty is used)
    if (g.status_clear && blockIdx.x == 0) *g.status_clear = 0;
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s.tmem_slot)), "r"((uint32_t)(2 * kTileN)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *s.tmem_slot;
  cluster_sync_all();                                           // nobody signals a barrier of the other CTA before it is initialised
  const uint32_t full_first = map_to_cta(s.full, 0);            // the pair counts its copies on the first CTA's barriers
  if (warp == 0) {
    if (lane == 0) {
      bool ok = true;
      int issued = 0;
      for (int t = unit; t < n_tiles && ok; t += n_units) {
        int tm, tn;
        tile_coords(t, g.tiles_m, g.tiles_n, &tm, &tn);
        for (int b = 0; b < g.kb; ++b, ++issued) {
          const int st = issued % kStages;
          if (!wait_or_abort(s, g, s.empty + 8 * st, ((issued / kStages) & 1) ^ 1)) { ok = false; break; }
          if (g.drop_first_load && issued == 0) continue;
          const uint32_t dst = tiles + (uint32_t)st * kStageBytes;
          if (rank == 0) mbar_expect_tx(s.full + 8 * st, 2 * kStageBytes);
          tma_load_2d_pair(dst, &tmap_x, b * kBlockK, tm * kTileM + (int)rank * 128, full_first + 8 * st);
          tma_load_2d_pair(dst + kHalfBytes, &tmap_w, b * kBlockK, tn * kTileN + (int)rank * 128, full_first + 8 * st);
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      int it = 0;
      bool ok = true;
      for (int t = unit; t < n_tiles && ok; t += n_units)
        for (int b = 0; b < g.kb && ok; ++b, ++it) {
          const int st = it % kStages;
          const int buf = it % kTileBufs;
          ok = wait_or_abort(s, g, s.part_empty + 8 * buf, ((it / kTileBufs) & 1) ^ 1) && wait_or_abort(s, g, s.full + 8 * st, (it / kStages) & 1);
          if (!ok) break;
          fence_after();
          const uint32_t at = tiles + (uint32_t)st * kStageBytes;
          const uint64_t da = make_smem_desc(at), db = make_smem_desc(at + kHalfBytes);
#pragma unroll
          for (int k = 0; k < kBlockK / kUmmaK; ++k) umma_e4m3_pair(tmem + buf * kTileN, da + 2 * k, db + 2 * k, idesc_e4m3(kTileM, kTileN), k > 0 ? 1u : 0u);
          umma_commit_pair(s.empty + 8 * st);
          umma_commit_pair(s.part_full + 8 * buf);
        }
    }
  } else if (warp >= 2 + kEpiWarps) {
    // scales, kScaleBlocks blocks at a time: a set is filled while the epilogue works with the other one, and handed over
    // at a barrier that says both "it is filled" and "the other one is free"
    TileScales* scales = reinterpret_cast<TileScales*>(smem_raw + (tiles - raw) + (size_t)kStages * kStageBytes + 256);
    int set = 0;
    for (int t = unit; t < n_tiles; t += n_units) {
      int tm, tn;
      tile_coords(t, g.tiles_m, g.tiles_n, &tm, &tn);
      for (int b0 = 0; b0 < g.kb; b0 += kScaleBlocks, set ^= 1) {
        fetch_scales(g, scales[set], (int)threadIdx.x - 64 - kEpiThreads, tm * kTileM + (int)rank * 128, tn * 2, b0);
        asm volatile("cp.async.wait_all;" ::: "memory");
        asm volatile("bar.sync 1, %0;" ::"n"(kEpiThreads + 32 * kFetchWarps) : "memory");
      }
    }
  } else {
    // warp w reads TMEM lanes 32 (w % 4) .. + 31 (rows of this CTA's half of the tile) and kEpiCols columns (inside one
    // 128-row block of W)
    const int q = warp & 3, first_col = ((warp - 2) >> 2) * kEpiCols;
    const uint32_t part_empty_first = map_to_cta(s.part_empty, 0);
    const TileScales* scales = reinterpret_cast<const TileScales*>(smem_raw + (tiles - raw) + (size_t)kStages * kStageBytes + 256);
    const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)first_col;
    int it = 0, set = 0;
    bool ok = true;
    for (int t = unit; t < n_tiles; t += n_units) {
      Pair acc[kEpiCols / 2];
#pragma unroll
      for (int j = 0; j < kEpiCols / 2; ++j) acc[j] = 0;
      for (int b0 = 0; b0 < g.kb; b0 += kScaleBlocks, set ^= 1) {
        asm volatile("bar.sync 1, %0;" ::"n"(kEpiThreads + 32 * kFetchWarps) : "memory");
        const float* xs = &scales[set].x[0][q * 32 + lane];
        const float* ws = scales[set].w[first_col / 128];
        const int n = min(kScaleBlocks, g.kb - b0);
#pragma unroll 1
        for (int i = 0; i < n && ok; ++i, ++it) {
          const float s1 = xs[i * 128] * ws[i];
          const Pair sc = pack(s1, s1);
          const int buf = it % kTileBufs;
          ok = __all_sync(0xffffffffu, mbar_wait(s.part_full + 8 * buf, (it / kTileBufs) & 1, s.abort_flag, g.wait_budget));
          if (!ok) { if (lane == 0) { *s.abort_flag = 1; atomicExch(g.status, DRAGON_ERR_TIMEOUT); } break; }
          fence_after();
#pragma unroll
          for (int c = 0; c < kEpiCols; c += 16) {
            uint32_t v[16];
            tmem_ld16(from + (uint32_t)(buf * kTileN + c), v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 8; ++j) fma_pair(acc[c / 2 + j], v[2 * j], v[2 * j + 1], sc);
          }
          fence_before();
          __syncwarp();
          if (lane == 0) {
            if (rank == 0) mbar_arrive(s.part_empty + 8 * buf);
            else mbar_arrive_remote_relaxed(part_empty_first + 8 * buf);
          }
        }
      }
      int tm, tn;
      tile_coords(t, g.tiles_m, g.tiles_n, &tm, &tn);
      if (!ok) continue;
      const int row0 = tm * kTileM + (int)rank * 128 + q * 32;
      constexpr int kCols = kF32 ? 32 : 64, kBytes = kF32 ? 4 : 2;         // 128 bytes of a row at a time
      const size_t row_bytes = (size_t)g.N * kBytes;
      const int col0 = tn * kTileN + first_col;
      char* y = static_cast<char*>(g.y) + (size_t)row0 * row_bytes + (size_t)col0 * kBytes;
#pragma unroll
      for (int h = 0; h < kEpiCols / kCols; ++h) {
        if (!kLines) asm volatile("" ::: "memory");     // (one part after another, or registers spill)
        uint32_t v[32];
#pragma unroll
        for (int j = 0; j < kCols / 2; ++j) {
          const float2 p = unpack(acc[kCols / 2 * h + j]);
          if (kF32) { v[2 * j] = __float_as_uint(p.x); v[2 * j + 1] = __float_as_uint(p.y); }
          else v[j] = bf16_pair(p.x, p.y);
        }
        if (kLines) store_lines<kF32>(y + 128 * h, row_bytes, g.M - row0, col0 + kCols * h, g.N, v, lane);
        else store_words<kF32>(y + 128 * h, row_bytes, g.M - row0, col0 + kCols * h, g.N, v, lane);
      }
    }
  }
  fence_before();
  __syncthreads();
  if (*s.abort_flag) {
    if (threadIdx.x == 0) {   // the copies are counted on the first CTA's barriers: give them time instead (they take microseconds)
      const long long t0 = clock64();
      while (clock64() - t0 < 20000000LL) { }
    }
    if (threadIdx.x == 32 && rank == 0) {
      umma_commit_pair(s.drain);
      mbar_wait(s.drain, 0, s.abort_flag + 1);
    }
    __syncthreads();
  }
  cluster_sync_all();          // neither CTA leaves while the other may still signal its barriers or read its tiles
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)(2 * kTileN)) : "memory");
}

// ---- few rows -------------------------------------------------------------------------------------------------

// NT rows of X a tile; from 64 on more epilogue warps share its columns, 32 each
constexpr int few_warps(int nt) { return nt == 128 ? 16 : nt == 64 ? 8 : 4; }
constexpr int few_threads(int nt) { return 64 + 32 * few_warps(nt); }             // TMA, MMA, epilogue
constexpr int few_ctas(int nt) { return nt == 128 ? 1 : 2; }                      // per SM
constexpr int few_stages(int nt) { return nt <= 32 ? 5 : nt == 64 ? 4 : 6; }
constexpr uint32_t few_stage_bytes(int nt) { return (128 + nt) * kBlockK; }
constexpr size_t few_smem(int nt) { return 1024 + (size_t)few_stages(nt) * few_stage_bytes(nt) + 256 + kScaleBlocks * nt * sizeof(float); }

template <int NT>
__global__ void __launch_bounds__(few_threads(NT), few_ctas(NT))
gemm_e4m3_few_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_w, const Gemm8Args g) {
  constexpr int kSt = few_stages(NT), kWarps = few_warps(NT), kCols = NT * 4 / kWarps;      // columns (rows of X) of a warp
  constexpr uint32_t kSB = few_stage_bytes(NT), kColumns = kBufs * NT;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), tiles = (raw + 1023u) & ~1023u;
  unsigned char* base = smem_raw + (tiles - raw);
  const Sync s = sync_area(base + (size_t)kSt * kSB, kSt);
  float* scales = reinterpret_cast<float*>(base + (size_t)kSt * kSB + 256);      // [kScaleBlocks][NT]: scale of X times scale of W
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n0 = blockIdx.x * 128, m0 = blockIdx.y * NT, part = blockIdx.z;
  const int b0 = (int)((long long)g.kb * part / g.split), b1 = (int)((long long)g.kb * (part + 1) / g.split);
  int issued = 0, first_issued = 0;
  auto copy_block = [&](int b) {
    const uint32_t bar = s.full + 8 * (issued % kSt), dst = tiles + (uint32_t)(issued % kSt) * kSB;
    mbar_expect_tx(bar, kSB);
    tma_load_2d(dst, &tmap_w, b * kBlockK, n0, bar);
    tma_load_2d(dst + 128 * kBlockK, &tmap_x, b * kBlockK, m0, bar);
  };
  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_w) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_x) : "memory");
    sync_init(s, kSt, kWarps);
    // the first copies go out at once: the stages are free, and nobody else touches their barriers before the one below
    for (; issued < kSt && b0 + issued < b1; ++issued) {
      if (g.drop_first_load && issued == 0) { first_issued = 1; continue; }
      copy_block(b0 + issued);
    }
    if (g.status_clear && blockIdx.x == 0 && blockIdx.y == 0 && part == 0) *g.status_clear = 0;
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s.tmem_slot)), "r"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *s.tmem_slot;
  Pair acc[kCols / 2];         // epilogue: row n0 + its TMEM lane of W, kCols rows of X from c0 on
#pragma unroll
  for (int j = 0; j < kCols / 2; ++j) acc[j] = 0;
  const int q = warp & 3, e = q * 32 + lane;      // epilogue warps 2..: quadrants 2, 3, 0, 1
  const int c0 = ((warp - 2) >> 2) * kCols, tid = (warp - 2) * 32 + lane;
  if (warp == 0) {
    if (lane == 0) {
      for (; b0 + issued < b1; ++issued) {
        if (!wait_or_abort(s, g, s.empty + 8 * (issued % kSt), ((issued / kSt) & 1) ^ 1)) break;
        copy_block(b0 + issued);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      bool ok = true;
      for (int it = 0; it < b1 - b0 && ok; ++it) {
        const uint32_t a = tiles + (uint32_t)(it % kSt) * kSB;
        ok = issue_block(s, g, it, kSt, a, a + 128 * kBlockK, tmem, NT, idesc_e4m3(128, NT));
      }
    }
  } else {
    // kScaleBlocks blocks' scales at a time: the next ones are in registers before they are needed
    constexpr int kThreadsE = 32 * kWarps, kPer = kScaleBlocks * NT / kThreadsE;
    const float* sw = g.sw + (size_t)blockIdx.x * g.kb;
    float next_x[kPer], next_w[kPer];
    auto fetch = [&](int b) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int k = i * kThreadsE + tid, row = m0 + k % NT, at = min(b + k / NT, b1 - 1);
        next_x[i] = row < g.M ? __ldg(g.sx + (size_t)row * g.kb + at) : 0.f;
        next_w[i] = __ldg(sw + at);
      }
    };
    fetch(b0);
    bool ok = true;
    for (int it = 0; it < b1 - b0; ++it) {
      const int buf = it % kBufs;
      if (it % kScaleBlocks == 0) {
        if (it) asm volatile("bar.sync 1, %0;" ::"n"(kThreadsE) : "memory");      // everyone is done with the last ones
#pragma unroll
        for (int i = 0; i < kPer; ++i) scales[i * kThreadsE + tid] = next_x[i] * next_w[i];
        if (it + kScaleBlocks < b1 - b0) fetch(b0 + it + kScaleBlocks);
        asm volatile("bar.sync 1, %0;" ::"n"(kThreadsE) : "memory");
      }
      ok = __all_sync(0xffffffffu, ok && mbar_wait(s.part_full + 8 * buf, (it / kBufs) & 1, s.abort_flag, g.wait_budget));
      if (!ok) {                                           // (the barriers above count every warp)
        if (lane == 0) { *s.abort_flag = 1; atomicExch(g.status, DRAGON_ERR_TIMEOUT); }
        continue;
      }
      fence_after();
      const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * NT + c0);
      const float4* sc = reinterpret_cast<const float4*>(scales + it % kScaleBlocks * NT + c0);
      constexpr int kChunk = kCols < 32 ? kCols : 32;
#pragma unroll
      for (int c = 0; c < kCols / kChunk; ++c) {
        uint32_t v[kChunk];
        if (kChunk == 16) tmem_ld16(from, v);
        else tmem_ld32(from + 32 * c, v);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < kChunk / 4; ++j) {
          const float4 f = sc[kChunk / 4 * c + j];
          fma_pair(acc[kChunk / 2 * c + 2 * j], v[4 * j], v[4 * j + 1], pack(f.x, f.y));
          fma_pair(acc[kChunk / 2 * c + 2 * j + 1], v[4 * j + 2], v[4 * j + 3], pack(f.z, f.w));
        }
      }
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(s.part_empty + 8 * buf);
    }
    if (g.split == 1) {
      if (ok && n0 + e < g.N)
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
          const float v = j & 1 ? unpack(acc[j / 2]).y : unpack(acc[j / 2]).x;
          if (m0 + c0 + j < g.M) store_any<1>(g.y, g.ydt, (size_t)(m0 + c0 + j) * g.N + n0 + e, &v);
        }
    }
  }
  fence_before();
  __syncthreads();
  if (*s.abort_flag) {
    if (threadIdx.x == 0) drain_copies(s, first_issued, issued, kSt);
    if (threadIdx.x == 32) drain_products(s);
    __syncthreads();
  }
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kColumns) : "memory");
  if (g.split == 1) return;
  // the cluster's partial sums: each CTA lays its own down (the stages are free now), then sums a share of the rows of X
  float* sums = reinterpret_cast<float*>(base);
  if (warp >= 2) {
#pragma unroll
    for (int j = 0; j < kCols; ++j) sums[(c0 + j) * 128 + e] = j & 1 ? unpack(acc[j / 2]).y : unpack(acc[j / 2]).x;
  }
  cluster_sync_all();
  if (warp >= 2) {
    const uint32_t mine = smem_u32(sums);
    const int step = g.split * (kWarps / 4);      // rows of X go round the CTAs and their groups of four warps
    // eight rows at a time: their loads from the other CTAs' shared memory are in flight together
    for (int j0 = part + g.split * ((warp - 2) >> 2); j0 < NT && m0 + j0 < g.M; j0 += 8 * step) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
      for (int p = 0; p < g.split; ++p) {
        const uint32_t from = map_to_cta(mine, (uint32_t)p) + (uint32_t)e * 4;
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = min(j0 + i * step, NT - 1);
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w[i]) : "r"(from + (uint32_t)j * 512) : "memory");
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += w[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = j0 + i * step;
        if (j < NT && m0 + j < g.M && n0 + e < g.N) store_any<1>(g.y, g.ydt, (size_t)(m0 + j) * g.N + n0 + e, &v[i]);
      }
    }
  }
  cluster_sync_all();          // nobody leaves while its sums are read
}

// ---- host side ------------------------------------------------------------------------------------------------

// row-major e4m3 [rows, K] with boxes of box_rows x 128 bytes; outside the tensor a copy reads zeros
bool make_tmap8(CUtensorMap* map, const void* ptr, int64_t rows, int64_t k, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)k};
  cuuint32_t box[2] = {(cuuint32_t)kBlockK, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// once per device and kernel: the shared-memory attribute
cudaError_t allow_smem(const void* kern, size_t bytes, int variant) {
  static std::mutex mu;
  static bool done[64][8] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (done[dev][variant]) return cudaSuccess;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) done[dev][variant] = true;
  return e;
}

struct FewConfig {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  FewConfig(int nt, dim3 grid, cudaStream_t st) {
    cfg.gridDim = grid;
    cfg.blockDim = dim3(few_threads(nt));
    cfg.dynamicSmemBytes = few_smem(nt);
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = grid.z;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
};
// How many CTAs in clusters of `split` the GPU holds at once: fewer than its SMs suggest, as a cluster stays inside one group
// of SMs (16 clusters of 8 CTAs of an SM each do not fit: 2025 x 64 x 2912 took 30 us in two waves, in clusters of 4 16 us)
template <int NT> int few_capacity(int split, int sm_count) {
  static std::mutex mu;
  static int known[64][4] = {};
  const int at = split == 1 ? 0 : split == 2 ? 1 : split == 4 ? 2 : 3;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  std::lock_guard<std::mutex> lock(mu);
  if (!known[dev][at]) {
    FewConfig c(NT, dim3(1, 1, split), nullptr);
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, gemm_e4m3_few_kernel<NT>, &c.cfg) != cudaSuccess || clusters < 1) {
      (void)cudaGetLastError();
      clusters = few_ctas(NT) * sm_count / split;
    }
    known[dev][at] = clusters * split;
  }
  return known[dev][at];
}

template <int NT>
cudaError_t launch_few(const CUtensorMap& tx, const CUtensorMap& tw, Gemm8Args g, int variant, int sm_count, cudaStream_t st) {
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(gemm_e4m3_few_kernel<NT>), few_smem(NT), variant);
  if (e != cudaSuccess) return e;
  const int64_t ctas = (int64_t)((g.N + 127) / 128) * ((g.M + NT - 1) / NT);
  // eight parts pay for their join only where a tile is small: 1 x 512 x 4096 10.8 us for 12.2 with four, 128 x 128 x 2912 16.8 for 14.4
  const int most = NT == 128 ? 4 : 8;
  // where an SM holds one CTA all clusters must find room, a second wave costs more than longer parts; where it holds two, the
  // clusters that do not fit start beside others (5 x 8192 x 4096: 64 clusters of 4 11.3 us, of 2 12.3)
  auto room = [&](int split) { return few_ctas(NT) == 1 ? few_capacity<NT>(split, sm_count) : few_ctas(NT) * sm_count; };
  while (g.split < most && g.kb >= 4 * g.split && ctas * g.split * 2 <= room(2 * g.split)) g.split *= 2;
  FewConfig c(NT, dim3((g.N + 127) / 128, (g.M + NT - 1) / NT, g.split), st);
  return cudaLaunchKernelEx(&c.cfg, gemm_e4m3_few_kernel<NT>, tx, tw, g);
}
template <bool kF32, bool kLines>
cudaError_t launch_pairs(const CUtensorMap& tx, const CUtensorMap& tw, const Gemm8Args& g, int pairs, int variant, cudaStream_t st) {
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(gemm_e4m3_kernel<kF32, kLines>), kSmem, variant);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * std::min(g.tiles_m * g.tiles_n, pairs));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, gemm_e4m3_kernel<kF32, kLines>, tx, tw, g);
}

}  // namespace

int launch_gemm_e4m3(const StepRun& r) {
  const Shape &sx = r.mems[r.s.rd[g8::XQ]].shape, &sw = r.mems[r.s.rd[g8::WQ]].shape;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  Gemm8Args g{reinterpret_cast<const float*>(r.rd(g8::SX)), reinterpret_cast<const float*>(r.rd(g8::SW)), r.wr(g8::Y), r.wr_type(g8::Y),
              (int)sx.d[0], (int)sw.d[0], (int)sx.d[1], (int)((sx.d[1] + 127) / 128), 0, 0, 1, r.status, r.status_clear, kWaitBudgetCycles, 0};
  // failure-detection test only, as for InnerProduct: a short budget and a first wait for a signal that nothing sends
  if (const char* e = std::getenv("DRAGON_GEMM_WAIT_BUDGET")) { const long long b = std::atoll(e); if (b > 0) g.wait_budget = std::min(b, kWaitBudgetCycles); }
  if (const char* e = std::getenv("DRAGON_GEMM_DROP_FIRST_LOAD")) g.drop_first_load = e[0] == '1';
  const int64_t tiles_m = (g.M + kTileM - 1) / kTileM, tiles_n = (g.N + kTileN - 1) / kTileN;
  if (tiles_m * tiles_n > 0x3fffffffLL) { set_error("ScaledInnerProduct: too many tiles"); return DRAGON_ERR_UNSUPPORTED; }
  g.tiles_m = (int)tiles_m;
  g.tiles_n = (int)tiles_n;
  // The small tiles where rows are few or the GPU holds all of them at once, their blocks split while CTAs find room; otherwise
  // the large ones.  Small and large: 777 x 2056 x 2064 18.7 us and 20.8, 256 x 2048 x 8192 21 and 39, 256 x 8192 x 4096 28 and
  // 27, 512 x 8192 x 4096 49 and 28, 2048 x 2048 x 2048 31 and 20.
  const int pairs = r.sm_count / 2;
  const bool few = g.M <= 128 || ((g.M + 127) / 128) * (int64_t)((g.N + 127) / 128) <= r.sm_count;
  const int nt = g.M <= 16 ? 16 : g.M <= 32 ? 32 : g.M <= 64 ? 64 : 128;
  CUtensorMap tx, tw;
  if (!make_tmap8(&tx, r.rd(g8::XQ), g.M, g.K, few ? nt : 128) || !make_tmap8(&tw, r.rd(g8::WQ), g.N, g.K, 128)) {
    set_error("ScaledInnerProduct: cannot encode the TMA descriptors (no CUDA driver?)");
    return DRAGON_ERR_CUDA;
  }
  cudaError_t e;
  if (few) {
    e = nt == 16 ? launch_few<16>(tx, tw, g, 1, r.sm_count, st) : nt == 32 ? launch_few<32>(tx, tw, g, 2, r.sm_count, st)
        : nt == 64 ? launch_few<64>(tx, tw, g, 3, r.sm_count, st) : launch_few<128>(tx, tw, g, 4, r.sm_count, st);
  } else {
    const bool lines = g.N % (g.ydt == DRAGON_F32 ? 4 : 8) == 0;
    if (g.ydt == DRAGON_F32) e = lines ? launch_pairs<true, true>(tx, tw, g, pairs, 0, st) : launch_pairs<true, false>(tx, tw, g, pairs, 5, st);
    else e = lines ? launch_pairs<false, true>(tx, tw, g, pairs, 6, st) : launch_pairs<false, false>(tx, tw, g, pairs, 7, st);
  }
  if (e != cudaSuccess) { set_error("ScaledInnerProduct: launch failed: %s", cudaGetErrorString(e)); return DRAGON_ERR_CUDA; }
  return DRAGON_OK;
}

}  // namespace dragon
