// What the tensor-core kernels of attention share: tiles of 128 rows of a head in shared memory, products of them, TMEM access.
//
// A tile is one or two chunks of 64 elements of the head: 128 rows of 128 bytes in the 128-byte swizzle, as a TMA copy of a
// (64, 1, 128) box leaves them.  The map's innermost extent is the head's width, so a narrower head reads zeros.
#pragma once
#include <algorithm>
#include <cstdlib>
#include <mutex>

#include "attention_util.h"
#include "device_util.h"
#include "plan.h"
#include "tcgen05_util.h"

namespace dragon {
namespace {

constexpr uint32_t kChunkBytes = 128 * 128;

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// All loads out of TMEM that this thread has asked for are there.  The registers of one of them go through the statement: nothing is
// computed from them in front of it (the loads fill them some time after their own statement), nor are they used for anything else
// before.  With several loads, one statement for each; only the first has something to wait for.
__device__ __forceinline__ void tmem_load32(uint32_t taddr, uint32_t* v) {
  __syncwarp();
  tmem_ld32(taddr, v);
}
__device__ __forceinline__ void tmem_loaded32(uint32_t* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31]) :: "memory");
}
__device__ __forceinline__ void tmem_loaded16(uint32_t* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]) :: "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A wait of a whole warp.  It is left by a vote, by all lanes together: the tcgen05 statements that follow are for a whole warp at
// once (.sync.aligned), which the compiler does not know of them; lanes that left a wait one by one could reach them apart
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long budget) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  const long long t0 = clock64();
  for (;;) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if (__any_sync(0xffffffffu, *abort_flag != 0 || clock64() - t0 > budget)) return false;
  }
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// One lane of a warp that is whole, the same one every time: it issues products and copies.  The loops around them, waits included,
// are run by the whole warp: these instructions take their operands from registers that a warp has once, and in a loop that one lane
// ran alone (if (lane == 0) around all of it) three products of eight were seen with another product's descriptor
__device__ __forceinline__ bool elected() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes)::"memory");
  return yes != 0;
}
// An arrival of lanes that a condition picks, without a branch: a branch on the lane in a loop lets the compiler make two loops of it,
// one for the lanes that take it and one for the others, and the warp then runs apart in front of statements that want it whole
__device__ __forceinline__ void mbar_arrive_if(uint32_t bar, bool yes) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"((uint32_t)yes) : "memory");
}
// (with a warp barrier in front)
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* v) {
  __syncwarp();
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
  __syncwarp();
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
        "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* v) {
  __syncwarp();
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
        "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
        "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
        "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(taddr) : "memory");
}
// 2^x, results below 2^-126 as 0
__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// the largest of three, NaN if one of them is
__device__ __forceinline__ float most_of(float a, float b, float c) { float d; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }

// rows of a tile along M or N, the head's elements along K: 16 of them are 32 bytes on
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) { return make_smem_desc(addr); }
// the head's elements along N, rows of the tile along K: 16 rows are 2048 bytes on, the next 64 elements a chunk
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(kChunkBytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// D = f32, A = B = bf16, A K-major
constexpr uint32_t idesc_bf16(int m, int n, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void umma_ss(uint32_t d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// A out of TMEM: 16 bf16 of every row in 8 columns
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}

// X Y^T over the head's elements, `steps` times 16 of them.  The descriptors of a step differ from the tile's by constants: what the
// one issuing thread computes between two products is as little as can be (an address computed for each took longer than the product)
template <int kChunks> __device__ __forceinline__ void product_over_head(uint32_t d, uint32_t x, uint32_t y, int steps, uint32_t idesc) {
  const uint64_t dx = desc_k(x), dy = desc_k(y);
#pragma unroll
  for (int k = 0; k < 4 * kChunks; ++k) {
    const uint64_t off = (k >> 2) * (kChunkBytes >> 4) + (k & 3) * 2;
    if (k < steps) umma_ss(d, dx + off, dy + off, idesc, k > 0);
  }
}
// P Y over the 128 rows of the tile Y, P out of TMEM: 16 rows' columns after one another, the second 64 rows' `half` columns on
template <int kHalf, int kFirst = 0, int kLast = 8> __device__ __forceinline__ void product_over_rows(uint32_t d, uint32_t p, uint32_t y, uint32_t idesc, bool accumulate) {
  const uint64_t dy = desc_mn(y);
#pragma unroll
  for (int k = kFirst; k < kLast; ++k) umma_ts(d, p + kHalf * (k >> 2) + 8 * (k & 3), dy + 128 * k, idesc, accumulate || k > 0);
}

// ---- units of work ---------------------------------------------------------------------------

struct Unit {
  int seq, a, b;        // the sequence (-1: none) and its rows
  int row0;             // first row of tile 0, from a
  int first_pos;        // position of row a (paged: behind the tokens that were there)
  int keys;             // keys there are
  int spare, spares;    // seq < 0: which of how many units that have the rows of none (spare as large as the rows: not one of them)
};

// Up to so many packed sequences are walked over, more are searched: 64 of up to 100 rows with gradients take 37.2 us walked over and 43.0
// searched (units without rows stand among the others then), 128 of up to 300 rows 221 and 215, 600 of up to 300 rows 1243 and 939
constexpr int kWalked = 64;
// Which block of rows this unit has: blocks of a sequence from its end (those that see most keys go first)
// (blocks: those that the grid has room for, each_blocks: of a sequence, where all are equally long, 0: starts; block_rows: a power of two)
__device__ __forceinline__ void find_unit(const Sequences& q, int blocks, int each_blocks, int unit, int block_rows, Unit* u, int lane) {
  u->seq = -1;
  if (each_blocks) {
    const int s = unit % q.count;
    q.rows_of(s, &u->a, &u->b);
    u->seq = s;
    u->row0 = (each_blocks - 1 - unit / q.count) * block_rows;
    return;
  }
  if (q.count <= kWalked) {      // blocks counted from the first sequence on, 32 sequences at a time: units without rows are all behind the others
    int before = 0;
    for (int s0 = 0; s0 < q.count; s0 += 32) {
      int x = 0, y = 0;
      if (s0 + lane < q.count) q.rows_of(s0 + lane, &x, &y);
      const int n = (y - x + block_rows - 1) / block_rows;
      int sum = n;
#pragma unroll
      for (int k = 1; k < 32; k <<= 1) { const int t = __shfl_up_sync(0xffffffffu, sum, k); if (lane >= k) sum += t; }
      const int local = unit - before;
      const unsigned hit = __ballot_sync(0xffffffffu, local >= sum - n && local < sum);
      if (hit) {
        const int w = __ffs(hit) - 1;
        u->seq = s0 + w;
        u->a = __shfl_sync(0xffffffffu, x, w);
        u->b = __shfl_sync(0xffffffffu, y, w);
        u->row0 = (__shfl_sync(0xffffffffu, sum, w) - 1 - local) * block_rows;
        return;
      }
      before += __shfl_sync(0xffffffffu, sum, 31);
    }
    u->spare = unit - before;
    u->spares = blocks - before;
    return;
  }
  // Sequence s has the units from starts[s] / block_rows + s on: the numbers ascend, leave every sequence room for its blocks and come from
  // starts alone, so that a unit finds its sequence in a search of 32 probes a turn (a walk over all of them in every CTA took 46.3 ms
  // for 16384 rows in as many sequences with gradients, the search takes 3.3).  A unit behind its sequence's last block has nothing
  // to do; those in front of the first sequence and behind the last have the rows of none.
  const int shift = 31 - __clz(block_rows);
  auto start = [&](int s) { return min(max(__ldg(q.starts + s), 0), q.rows); };
  int s = -1, step = 1;      // s: the last sequence whose units begin here or before
  while (32 * step < q.count) step *= 32;
  for (int from = 0; step; step >>= 5) {
    const int probe = from + lane * step;
    const unsigned behind = ~__ballot_sync(0xffffffffu, probe < q.count && (start(probe) >> shift) + probe <= unit);
    const int n = behind ? __ffs(behind) - 1 : 32;
    if (n == 0) break;
    s = from += (n - 1) * step;
  }
  if (s >= 0) {
    q.rows_of(s, &u->a, &u->b);
    const int block = unit - (u->a >> shift) - s, n = (u->b - u->a + block_rows - 1) >> shift;
    if (block < n) {
      u->seq = s;
      u->row0 = (n - 1 - block) * block_rows;
      return;
    }
  }
  const int first = start(0), behind = (max(start(q.count), first) >> shift) + q.count;      // units behind the last sequence's
  const bool nothing = s >= 0 && unit < behind;
  u->spare = nothing ? q.rows : s < 0 ? unit : (first >> shift) + unit - behind;
  u->spares = (first >> shift) + blocks - behind;
}

// row i of those that belong to no sequence, -1 behind them
__device__ __forceinline__ int row_of_none(const Sequences& q, int i) {
  const int first = q.starts ? min(max(__ldg(q.starts), 0), q.rows) : 0;
  const int last = q.starts ? min(max(__ldg(q.starts + q.count), first), q.rows) : q.rows;
  return i < first ? i : i < first + q.rows - last ? last + i - first : -1;
}

// ---- host ----------------------------------------------------------------------------------

// bf16 [rows, heads * width] as (element of a head, head, row), boxes of 64 elements x box_heads heads x box_rows rows
bool head_map(CUtensorMap* map, const void* ptr, int64_t rows, int heads, int width, int box_rows, int box_heads = 1) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)heads, (cuuint64_t)rows};
  cuuint64_t strides[2] = {(cuuint64_t)width * 2, (cuuint64_t)width * heads * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// whether a tile of queries holds all heads of a group
bool packs(int group) { return (group & (group - 1)) == 0 && group <= 128; }

// blocks of rows that a grid needs room for, and those of a sequence where all are equally long
void count_blocks(const Sequences& q, int block_rows, int* blocks, int* each_blocks) {
  *each_blocks = q.starts ? 0 : (q.each + block_rows - 1) / block_rows;
  *blocks = q.starts ? (q.rows + block_rows - 1) / block_rows + q.count + (q.count > kWalked) : *each_blocks * q.count;      // (one at least for rows of none)
}

// a kernel's dynamic shared memory, once per device (set: one flag a device)
int allow_smem(const void* kernel, size_t bytes, bool* set, const char* who) {
  static std::mutex mu;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { set_error("%s: no current device", who); return DRAGON_ERR_CUDA; }
  std::lock_guard<std::mutex> lock(mu);
  if (set[dev]) return DRAGON_OK;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != cudaSuccess) { set_error("%s: %s", who, cudaGetErrorString(e)); return DRAGON_ERR_CUDA; }
  set[dev] = true;
  return DRAGON_OK;
}

// failure-detection tests only: <name>_WAIT_BUDGET=<clock cycles> shortens the waits, <name>_DROP_FIRST_LOAD=1 leaves out the first copy
void wait_settings(const char* name, long long* budget, int* drop) {
  *budget = kWaitBudgetCycles;
  *drop = 0;
  if (const char* e = std::getenv((std::string(name) + "_WAIT_BUDGET").c_str())) { const long long b = std::atoll(e); if (b > 0) *budget = std::min(b, kWaitBudgetCycles); }
  if (const char* e = std::getenv((std::string(name) + "_DROP_FIRST_LOAD").c_str())) *drop = e[0] == '1';
}

}  // namespace
}  // namespace dragon
