// Attention's forward pass on the tensor cores: y = softmax(scale q k^T) v over packed sequences or over a paged cache.
// Hand-written for sm_100a.
//
// A CTA works on one or two tiles of 128 query rows that see the same keys: where the heads of a group are a power of two, all of them
// for 128 / group neighbouring rows of the sequence in each tile; otherwise the same 128 rows of two heads of a group, or rows
// of one head.  Keys and values pass once, 128 at a time:
//   S_t = Q_t K^T              tcgen05.mma, both operands in shared memory (TMA, 128-byte swizzle), S_t in TMEM
//   P_t = exp2(scale' S_t - m) one thread a row: the running maximum m and sum stay in its registers; P_t goes back over S_t as
//                              bf16 (its sum is taken in fp32 before the rounding)
//   O_t += P_t V               tcgen05.mma with P_t as the A operand out of TMEM, V as it lies in memory (MN-major)
// While the softmax threads of one tile work, the tensor unit works for the other (of the CTA, or of the SM's other CTA).
// Bound: exponentials and products alike.  A round (two tiles against 128 keys, heads of 128) has 2048 cycles of each and takes 3200; a
// CTA's start and end another 14000.  16384 causal rows, 8 heads on 2 of 128: 420 us, 1.31 PFLOP/s on a cool GPU (with gradients, one after
// another under the power limit, all launches take some 15 % more).  m only moves when a row's maximum has grown
// by more than 2^8 (P_t and the sum then stay below 2^8 times their scale, far inside bf16 and fp32): O_t in TMEM is rescaled
// that seldom that the softmax threads do it themselves.  S_t of the next keys is issued behind O_t's product, so a completed
// S_t says that O_t may be touched.  Where there are few units of work (few rows or heads, long contexts) the keys of one are split over
// several CTAs.
// Warps: four softmax warps a tile (a warp its TMEM lanes), then TMA, MMA.  Every wait is bounded.
#include <algorithm>
#include <cstdlib>

#include "attention_rows.h"
#include "attention_tiles.h"

namespace dragon {
namespace {

constexpr int fwd_threads(int tiles) { return 128 * tiles + 64; }
constexpr int fwd_stages(int tiles, int chunks) { return tiles * (chunks == 1 ? 2 : 1); }      // of K and of V each
constexpr size_t fwd_smem(int tiles, int chunks) { return 1024 + (size_t)(tiles + 2 * fwd_stages(tiles, chunks)) * chunks * kChunkBytes + 512; }
constexpr float kRescale = 8.f;

struct FwdArgs {
  RowArgs r;
  int pack_shift;       // log2 of the heads in a tile
  int by_heads;         // (one head a tile) the two tiles are two heads' of the same rows, not two blocks of rows
  int columns;          // units side by side: key heads (several heads a tile), pairs of heads, or heads
  int blocks;           // blocks of rows that the grid has room for
  int each_blocks;      // of a sequence, where all are equally long (0: starts)
  int few;              // paged: sequences of at most so many rows are not this kernel's
  long long budget;
  int drop_first_load;
};

template <bool kPaged, int kTiles, int kChunks>
__global__ void __launch_bounds__(fwd_threads(kTiles), 3 - kTiles)
attention_fwd(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ FwdArgs a) {
  constexpr int kSt = fwd_stages(kTiles, kChunks), kTmaWarp = 4 * kTiles, kMmaWarp = kTmaWarp + 1;
  constexpr uint32_t kTile = kChunks * kChunkBytes;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t q_at = base, k_at = base + kTiles * kTile, v_at = k_at + kSt * kTile;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem_raw + (base - raw) + (kTiles + 2 * kSt) * kTile);
  const uint32_t q_full = smem_u32(bars), k_full = q_full + 16, k_empty = k_full + 8 * kSt, v_full = k_empty + 8 * kSt, v_empty = v_full + 8 * kSt;
  const uint32_t s_full = v_empty + 8 * kSt, p_full = s_full + 16, o_full = p_full + 32, v_clean = o_full + 16, drain = v_clean + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 12 + 4 * kSt);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  __shared__ Unit unit;
  if (kPaged) after_the_launch_before();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pack = 1 << a.pack_shift, tile_rows = 128 >> a.pack_shift, block_rows = a.by_heads ? 128 : kTiles * tile_rows;      // rows: of the sequence
  const int column = blockIdx.x % a.columns, group = a.r.heads / a.r.kv_heads, heads_here = a.by_heads ? 2 : pack;
  const int head0 = column * heads_here, kvh = head0 / group;

  // three warps side by side: barriers, the unit of work, TMEM
  if (warp == 1 && elected()) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_v) : "memory");
    for (int t = 0; t < kTiles; ++t) { mbar_init(q_full + 8 * t, 1); mbar_init(s_full + 8 * t, 1); mbar_init(p_full + 16 * t, 4); mbar_init(p_full + 16 * t + 8, 4); mbar_init(o_full + 8 * t, 1); }
    for (int s = 0; s < kSt; ++s) { mbar_init(k_full + 8 * s, 1); mbar_init(k_empty + 8 * s, 1); mbar_init(v_full + 8 * s, 1); mbar_init(v_empty + 8 * s, 1); }
    mbar_init(v_clean, 32);
    mbar_init(drain, 1);
    abort_flag[0] = abort_flag[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (blockIdx.x == 0 && blockIdx.y == 0 && a.r.status_clear) *a.r.status_clear = 0;
  }
  if (blockIdx.x == 0 && blockIdx.y == 0 && !a.r.seq.in_order()) report(a.r.status, DRAGON_ERR_INVALID_ARG);
  if (warp == 0) {
    Unit u;
    find_unit(a.r.seq, a.blocks, a.each_blocks, blockIdx.x / a.columns, block_rows, &u, lane);
    if (u.seq >= 0) {
      u.keys = u.b - u.a;
      u.first_pos = 0;
      if (kPaged) {
        bool fits;
        u.keys = a.r.pages.tokens(u.seq, &fits);
        if (!fits) report(a.r.status, DRAGON_ERR_INVALID_ARG);
        u.first_pos = u.keys - (u.b - u.a);
      }
    }
    if (lane == 0) unit = u;
  }
  if (warp == kMmaWarp) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(256u * kTiles) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const Unit u = unit;
  const uint32_t tmem = *tmem_slot;
  auto give_tmem_back = [&]() {
    __syncwarp();
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256u * kTiles) : "memory");
  };
  next_launch_may_come();
  if (u.seq < 0) {      // rows of no sequence: zeros, shared out among the units that are left over
    if (kPaged && a.r.splits > 1) { give_tmem_back(); return; }      // (where the parts are put together)
    const int wide = heads_here * a.r.width;
    for (int i = u.spare, row; (row = row_of_none(a.r.seq, i)) >= 0; i += u.spares) {
      const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (a.r.out) for (int c = 8 * threadIdx.x; c < wide; c += 8 * fwd_threads(kTiles)) store_any<8>(a.r.out, a.r.ot, ((size_t)row * a.r.heads + head0) * a.r.width + c, zero);
      if (a.r.lse && threadIdx.x < heads_here) a.r.lse[(size_t)(head0 + threadIdx.x) * a.r.seq.rows + row] = kInf;
    }
    give_tmem_back();
    return;
  }
  const int n_rows = u.b - u.a;
  if (kPaged && has_few_rows(n_rows, group, a.few)) { give_tmem_back(); return; }
  // the tiles of keys that any row of the unit sees
  const int last_row = min(u.row0 + block_rows, n_rows) - 1;      // (row0 < n_rows)
  const int key_end = a.r.causal ? max(0, min(u.keys, u.first_pos + last_row + 1)) : u.keys;
  const int key_begin = a.r.window ? max(0, u.first_pos + u.row0 - a.r.window + 1) : 0;
  int j0 = key_begin / 128, n_tiles = key_end > key_begin ? (key_end + 127) / 128 - j0 : 0;
  if (a.r.splits > 1) {
    const int each = (n_tiles + a.r.splits - 1) / a.r.splits, skip = min(n_tiles, (int)blockIdx.y * each);
    j0 += skip;
    n_tiles = min(each, n_tiles - skip);
  }
  const bool ragged = u.keys - (j0 + n_tiles - 1) * 128 < 128;      // the last tile has rows behind the sequence's last key

  auto wait_warp = [&](uint32_t bar, uint32_t parity) {
    if (mbar_wait_warp(bar, parity, abort_flag, a.budget)) return true;
    *abort_flag = 1;
    report(a.r.status, DRAGON_ERR_TIMEOUT);
    return false;
  };
  int issued_k = 0, issued_v = 0;
  if (warp == kTmaWarp) {
    if (n_tiles > 0 && elected()) {
      for (int t = 0; t < kTiles; ++t) {
        mbar_expect_tx(q_full + 8 * t, kTile);
        for (int c = 0; c < kChunks; ++c)
          tma_load_3d(q_at + t * kTile + c * kChunkBytes, &tm_q, 64 * c, a.by_heads ? head0 + t : head0, u.a + u.row0 + (a.by_heads ? 0 : tile_rows * t), q_full + 8 * t);
      }
    }
    __syncwarp();
    bool ok = true;
    for (int j = 0; j < n_tiles && ok; ++j) {
      const int s = j % kSt, turn = j / kSt;
      for (int which = 0; which < 2; ++which) {
        const CUtensorMap* tm = which ? &tm_v : &tm_k;
        const uint32_t full = (which ? v_full : k_full) + 8 * s, dst = (which ? v_at : k_at) + s * kTile;
        ok = wait_warp((which ? v_empty : k_empty) + 8 * s, (turn & 1) ^ 1);
        if (!ok) break;
        if (which) issued_v = j + 1; else issued_k = j + 1;
        if (a.drop_first_load && j == 0 && !which) continue;      // failure-detection test: this stage's signal never comes
        if (!kPaged) {
          if (elected()) {
            mbar_expect_tx(full, kTile);
            for (int c = 0; c < kChunks; ++c) tma_load_3d(dst + c * kChunkBytes, tm, 64 * c, kvh, u.a + (j0 + j) * 128, full);
          }
          __syncwarp();
        } else {
          const int page = 1 << a.r.pages.shift, box = min(page, 128), at = (j0 + j) * 128 + lane * box;
          const bool mine = lane < 128 / box, there = mine && at < u.keys;
          const int number = there ? a.r.pages.page_of(u.seq, at) : -1, none = a.r.pages.pool << a.r.pages.shift;      // behind the cache: zeros
          const int row = a.r.pages.in_pool(number) ? (number << a.r.pages.shift) + (at & (page - 1)) : none;
          if (__any_sync(0xffffffffu, there && row == none)) report(a.r.status, DRAGON_ERR_INVALID_ARG);
          for (int p = 0; p < 128 / box; ++p) {      // (each lane has looked up a page; one lane issues all copies)
            const int from = __shfl_sync(0xffffffffu, row, p);
            if (elected()) {
              if (p == 0) mbar_expect_tx(full, kTile);
              for (int c = 0; c < kChunks; ++c) tma_load_3d(dst + c * kChunkBytes + p * box * 128, tm, 64 * c, kvh, from, full);
            }
            __syncwarp();
          }
        }
      }
    }
    if (ok && ragged && n_tiles > 0) {
      // what stands behind the sequence's last key (other sequences, a page's unused rows) is not to meet a probability of 0
      const int j = n_tiles - 1, keep = u.keys - (j0 + j) * 128;
      if (wait_warp(v_full + 8 * (j % kSt), (j / kSt) & 1)) {
        unsigned char* tile = smem_raw + (v_at - raw) + (j % kSt) * kTile;
        for (int c = 0; c < kChunks; ++c)
          for (int i = lane; i < (128 - keep) * 8; i += 32) *reinterpret_cast<uint4*>(tile + c * kChunkBytes + keep * 128 + 16 * i) = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(v_clean);
      }
    }
  } else if (warp == kMmaWarp) {
    if (n_tiles > 0) {
      const int k_steps = (a.r.width + 15) / 16, n_out = 16 * k_steps;
      const uint32_t idesc_s = idesc_bf16(128, 128, false), idesc_o = idesc_bf16(128, n_out, true);
      auto commit = [&](uint32_t bar) { if (elected()) umma_commit(bar); __syncwarp(); };
      auto product_s = [&](int t, int j) {
        fence_after();
        if (elected()) {
          product_over_head<kChunks>(tmem + 128 * t, q_at + t * kTile, k_at + (j % kSt) * kTile, k_steps, idesc_s);
          umma_commit(s_full + 8 * t);
        }
        __syncwarp();
      };
      bool ok = wait_warp(k_full, 0);
      for (int t = 0; t < kTiles && ok; ++t) {
        ok = wait_warp(q_full + 8 * t, 0);
        if (ok) product_s(t, 0);
      }
      if (ok) commit(k_empty);
      for (int j = 0; j < n_tiles && ok; ++j) {
        const int s = j % kSt;
        ok = wait_warp(v_full + 8 * s, (j / kSt) & 1);
        if (ok && ragged && j == n_tiles - 1) ok = wait_warp(v_clean, 0);
        for (int t = 0; t < kTiles && ok; ++t) {
          if (!(ok = wait_warp(p_full + 16 * t, j & 1))) break;
          fence_after();
          if (elected()) product_over_rows<32, 0, 4>(tmem + 128 * (kTiles + t), tmem + 128 * t, v_at + s * kTile, idesc_o, j > 0);
          __syncwarp();
          if (!(ok = wait_warp(p_full + 16 * t + 8, j & 1))) break;
          fence_after();
          if (elected()) {
            product_over_rows<32, 4, 8>(tmem + 128 * (kTiles + t), tmem + 128 * t, v_at + s * kTile, idesc_o, true);
            if (t == kTiles - 1) umma_commit(v_empty + 8 * s);
          }
          __syncwarp();
          if (j + 1 < n_tiles) {
            if (t == 0 && !(ok = wait_warp(k_full + 8 * ((j + 1) % kSt), ((j + 1) / kSt) & 1))) break;
            product_s(t, j + 1);
          } else {
            commit(o_full + 8 * t);
          }
        }
        if (ok && j + 1 < n_tiles) commit(k_empty + 8 * ((j + 1) % kSt));
      }
    }
  } else {
    const int t = warp >> 2, e = (warp & 3) * 32 + lane;
    const int head = a.by_heads ? head0 + t : head0 + (e & (pack - 1));
    const int i = u.row0 + (a.by_heads ? 0 : tile_rows * t) + (e >> a.pack_shift);      // this thread's row of the sequence
    const int pos = u.first_pos + i;
    const bool mine = i < n_rows;
    // the keys that the row sees
    const int hi = !mine ? 0 : a.r.causal ? min(pos + 1, u.keys) : u.keys, lo = a.r.window ? max(0, pos - a.r.window + 1) : 0;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_at = tmem + lanes + 128 * t, o_at = tmem + lanes + 128 * (kTiles + t);
    float top = -kInf, sum = 0.f;
    bool ok = true;
    for (int j = 0; j < n_tiles; ++j) {
      ok = wait_warp(s_full + 8 * t, j & 1);
      if (!ok) break;
      fence_after();
      uint32_t s[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_load32(s_at + 32 * c, s + 32 * c);
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_loaded32(s + 32 * c);
      const int k0 = (j0 + j) * 128;
      if (!__all_sync(0xffffffffu, lo <= k0 && k0 + 128 <= hi)) {
#pragma unroll
        for (int c = 0; c < 128; ++c) if (k0 + c < lo || k0 + c >= hi) s[c] = 0xff800000u;
      }
      float m[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) m[c] = __uint_as_float(s[c]);
#pragma unroll
      for (int c = 4; c < 124; c += 2) m[(c >> 1) & 3] = most_of(m[(c >> 1) & 3], __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
      m[0] = most_of(m[0], __uint_as_float(s[124]), __uint_as_float(s[125]));
      m[1] = most_of(m[1], __uint_as_float(s[126]), __uint_as_float(s[127]));
      const float most = most_of(most_of(m[0], m[1], m[2]), m[3], m[3]);      // (a NaN among the scores makes everything of the row NaN)
      if (j == 0) {
        top = most;
      } else {
        const bool grown = !((most - top) * a.r.scale <= kRescale) && most != -kInf;      // (from -inf on: infinite; NaN)
        if (__any_sync(0xffffffffu, grown)) {
          const float f = grown ? exp2_fast((top - most) * a.r.scale) : 1.f;
          if (grown) top = most;
          sum *= f;
#pragma unroll 1
          for (int c = 0; c < a.r.width; c += 16) {
            uint32_t o[16];
            tmem_ld16(o_at + c, o);
            tmem_loaded16(o);
#pragma unroll
            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
            tmem_st16(o_at + c, o);
          }
        }
      }
      const float shift = top == -kInf ? 0.f : top * a.r.scale;
      const Pair factor = pair_of(a.r.scale, a.r.scale), less = pair_of(-shift, -shift);
      Pair part[2] = {0, 0};
#pragma unroll
      for (int c = 0; c < 2; ++c) {      // the products of the first 64 keys start while the others are worked on
        uint32_t p[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          const float2 x = both(fma_pair(pair_of(s[64 * c + 2 * k], s[64 * c + 2 * k + 1]), factor, less));
          const float x0 = exp2_fast(x.x), x1 = exp2_fast(x.y);
          part[k & 1] = add_pair(part[k & 1], pair_of(x0, x1));
          p[k] = bf16_pair(x0, x1);
        }
        tmem_st32(s_at + 32 * c, p);
        tmem_st_wait();
        fence_before();
        __syncwarp();
        mbar_arrive_if(p_full + 16 * t + 8 * c, lane == 0);
      }
      const float2 more = both(add_pair(part[0], part[1]));
      sum += more.x + more.y;
    }
    if (ok && n_tiles > 0) {
      ok = wait_warp(o_full + 8 * t, 0);
      fence_after();
    }
    if (ok) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (a NaN stays one)
      const int row = u.a + i;
      const size_t at = ((size_t)row * a.r.heads + head) * a.r.width;
      bool fine = fabsf(sum) < kInf;
#pragma unroll 1
      for (int c = 0; c < a.r.width; c += 16) {
        uint32_t o[16];
        float v[16];
        if (n_tiles > 0) { tmem_ld16(o_at + c, o); tmem_loaded16(o); }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          v[k] = n_tiles > 0 ? __uint_as_float(o[k]) * inv : 0.f;
          fine &= fabsf(v[k]) < kInf;
        }
        if (a.r.splits > 1) {
          float* to = a.r.part + ((size_t)blockIdx.y * a.r.seq.rows * a.r.heads * a.r.width + at + c);
          if (mine && n_tiles > 0) {
            store_any<8>(to, DRAGON_F32, 0, v);
            if (c + 8 < a.r.width) store_any<8>(to, DRAGON_F32, 8, v + 8);
          }
        } else if (mine && a.r.out) {
          store_any<8>(a.r.out, a.r.ot, at + c, v);
          if (c + 8 < a.r.width) store_any<8>(a.r.out, a.r.ot, at + c + 8, v + 8);
        }
        if (!kPaged && a.r.splits == 1 && mine && a.r.rest) {
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = behind_bf16(v[k]);
          store_any<8>(a.r.rest, DRAGON_BF16, at + c, v);
          if (c + 8 < a.r.width) store_any<8>(a.r.rest, DRAGON_BF16, at + c + 8, v + 8);
        }
      }
      if (a.r.splits > 1) {      // (where the parts are put together a row that is not finite is computed again)
        if (mine) a.r.part_lse[((size_t)blockIdx.y * a.r.seq.rows + row) * a.r.heads + head] = sum == 0.f ? -kInf : top * a.r.scale + log2f(sum);
        fine = true;
      }
      if (!kPaged && a.r.splits == 1 && mine && a.r.lse) a.r.lse[(size_t)head * a.r.seq.rows + row] = sum == 0.f ? kInf : top * a.r.scale + log2f(sum);
      __syncwarp();
      for (unsigned again = __ballot_sync(0xffffffffu, mine && !fine); again; again &= again - 1)
        attend_row<kPaged>(a.r, __shfl_sync(0xffffffffu, head, __ffs(again) - 1), __shfl_sync(0xffffffffu, row, __ffs(again) - 1), lane);
    }
  }
  fence_before();
  __syncthreads();
  if (*abort_flag) {      // an unwind: copies and products that have been asked for end before their memory goes away
    if (warp == kMmaWarp) {
      if (elected()) umma_commit(drain);
      __syncwarp();
      mbar_wait_warp(drain, 0, abort_flag + 1, kWaitBudgetCycles);
    }
    if (threadIdx.x == 32 * kTmaWarp) {
      for (int t = 0; t < kTiles && n_tiles > 0; ++t) mbar_wait(q_full + 8 * t, 0, abort_flag + 1);
      for (int k = std::max(a.drop_first_load ? 1 : 0, issued_k - kSt); k < issued_k; ++k) mbar_wait(k_full + 8 * (k % kSt), (k / kSt) & 1, abort_flag + 1);
      for (int k = std::max(0, issued_v - kSt); k < issued_v; ++k) mbar_wait(v_full + 8 * (k % kSt), (k / kSt) & 1, abort_flag + 1);
    }
    __syncthreads();
  }
  give_tmem_back();
}

template <bool kPaged, int kTiles, int kChunks> int launch_fwd(const FwdArgs& a, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t st, const char* who) {
  static bool set[64] = {};
  const auto kernel = attention_fwd<kPaged, kTiles, kChunks>;
  constexpr size_t bytes = fwd_smem(kTiles, kChunks);
  const int rc = allow_smem(reinterpret_cast<const void*>(kernel), bytes, set, who);
  if (rc != DRAGON_OK) return rc;
  const long long grid = (long long)a.blocks * a.columns;
  if (grid > 0x7fffffffLL) { set_error("%s: too many blocks of rows", who); return DRAGON_ERR_UNSUPPORTED; }
  const dim3 ctas((unsigned)grid, a.r.splits), threads(fwd_threads(kTiles));
  if (kPaged) return launch_behind(kernel, ctas, threads, bytes, st, who, q, k, v, a);
  kernel<<<ctas, threads, bytes, st>>>(q, k, v, a);
  return launched(who);
}

}  // namespace

// units of work that the kernel has at least room for, without splits
int64_t attention_units(int64_t rows, int64_t sequences, int heads, int kv_heads) {
  const int group = heads / kv_heads;
  const int64_t block = packs(group) ? 256 / group : group % 2 == 0 ? 128 : 256;
  return std::max<int64_t>(sequences, (rows + block - 1) / block) * (packs(group) ? kv_heads : group % 2 == 0 ? heads / 2 : heads);
}

// Tiles of a CTA: one, with two CTAs on an SM, or two that share the copies of keys and values.  Two CTAs overlap start and end of one
// with the other's work, and their units are half as long; heads of 64 and less: always (1 x 16384 rows, 8 heads of 64: 415 us with two
// tiles, 392 with one).  With wider heads there is room for one stage of keys and values only: two tiles (16384 rows, 8 heads on 2 of
// 128: 420 us, 445 with one), but where a unit meets few keys (1 x 12001, window 1024, heads of 96: 57 us with two tiles, 51 with one), where
// a causal call has units for less than two rounds of the GPU (7807 rows, 8 heads: 161 and 144), or the second tile had no rows (15 new rows
// of 14 sequences of 4200, 9 heads on 3: 102 and 68).
static int tiles_of(const RowArgs& r, bool paged, int sm_count) {
  if (r.width <= 64) return 1;
  const int group = r.heads / r.kv_heads, count = std::max(1, r.seq.count);
  const int64_t each = (r.seq.rows + count - 1) / count, room = paged ? std::min<int64_t>((int64_t)r.pages.most << r.pages.shift, 0x7fffffff) : each;
  const bool falling = r.causal && !r.window && !paged;
  const int64_t pairs = ((r.window ? std::min<int64_t>(room, (int64_t)r.window + 128) : room) + 127) / 128;
  if (each * (packs(group) ? group : 1) <= 128 || pairs <= (falling ? 32 : 16)) return 1;
  return falling && attention_units(r.seq.rows, count, r.heads, r.kv_heads) < 2 * (int64_t)sm_count ? 1 : 2;
}

// rows: what the row functions need as well; key_rows: rows of k and v in memory; few: rows x group of a sequence up to which another kernel has it
int launch_attention_forward(const RowArgs& rows, bool paged, int64_t key_rows, int few, int sm_count, cudaStream_t st, const char* who) {
  FwdArgs a = {};
  a.r = rows;
  const int group = rows.heads / rows.kv_heads;
  const bool packed = packs(group);
  while (packed && (1 << a.pack_shift) < group) ++a.pack_shift;
  const bool wide = rows.width > 64;
  const int tiles = tiles_of(rows, paged, sm_count);
  a.by_heads = tiles == 2 && !packed && group % 2 == 0;
  a.columns = packed ? rows.kv_heads : a.by_heads ? rows.heads / 2 : rows.heads;
  const int block = a.by_heads ? 128 : 128 * tiles >> a.pack_shift;
  count_blocks(rows.seq, block, &a.blocks, &a.each_blocks);
  a.few = few;
  wait_settings("DRAGON_ATTENTION", &a.budget, &a.drop_first_load);
  CUtensorMap q, k, v;
  const int box = paged ? std::min(1 << rows.pages.shift, 128) : 128;
  if (!head_map(&q, rows.q, rows.seq.rows, rows.heads, rows.width, 128 >> a.pack_shift, 1 << a.pack_shift) || !head_map(&k, rows.k, key_rows, rows.kv_heads, rows.width, box) ||
      !head_map(&v, rows.v, key_rows, rows.kv_heads, rows.width, box)) {
    set_error("%s: cannot encode the TMA descriptors (no CUDA driver?)", who);
    return DRAGON_ERR_CUDA;
  }
  const auto launch = [&](auto t, auto c) {
    return paged ? launch_fwd<true, t, c>(a, q, k, v, st, who) : launch_fwd<false, t, c>(a, q, k, v, st, who);
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  return !wide ? launch(one, one) : tiles == 1 ? launch(one, two) : launch(two, two);
}

}  // namespace dragon
