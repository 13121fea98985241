// Attention's gradient on the tensor cores, with the probabilities computed again from q, k and every row's log2 sum.
// Hand-written for sm_100a.
//
//   p = exp2(scale' q k^T - lse), dp = dy v^T, ds = p (dp - delta), delta = sum(dy y) of a row
//   dv = p^T dy, dk = scale ds^T q (over the query heads that share the key head), dq = scale ds k
//
// Two kinds of CTA, so that every sum has one owner and its order is fixed (no atomics); q k^T and dy v^T are computed by both (7
// products of a tile where one pass needs 5):
//   keys:  a CTA has 128 keys of a key head and meets every tile of queries that sees them, of every head of the group.  It
//          computes S^T = K Q^T and dP^T = V dY^T, so that P^T and dS^T lie in TMEM as the A operands of dV += P^T dY and
//          dK += dS^T Q (dY and Q as they lie in memory, MN-major).
//   rows:  a CTA has 128 rows of a head and meets their keys: S = Q K^T, dP = dY V^T, dQ += dS K.
// Where the heads of a group are a power of two a tile of queries has all of them, for 128 / group neighbouring rows of the sequence:
// short sequences fill it (14 sequences of 28 rows, 8 heads a group: 54 us forwards and backwards with tiles of one head, 31 so).
// One tile pair is 128 x 128; two warps share a row (64 columns each).  The products are issued in an order in which the tensor
// unit has work while the threads compute: keys: dV(i), S(i+1), dK(i), dP(i+1); rows: S(i+1), dP(i+1), dQ(i) (dP has two buffers).
// Warps: 0..7 mathematics, 8 TMA, 9 MMA.  Every wait is bounded.
// Bound: keys, a round has 2048 cycles of products and took 3245, about 3200 by the launch's time since the products of half of P^T start
// early; rows, 1536 and 2288; what is left over is one product waiting for the threads' results of another.  16384 causal rows, 8 heads on
// 2 of 128: 1395 us on a cool GPU, 0.99 PFLOP/s of the formula's five products (1.38 of the seven), some 15 % more under its power limit.
// Both kinds are one launch, keys first: theirs are the longest (all heads of a group), and the rows' fill the SMs that run out of them.
#include <algorithm>

#include "attention_rows.h"
#include "attention_tiles.h"

namespace dragon {
namespace {

constexpr int kBwdThreads = 320;
// Stages of the first operand (q, or k), which is held until the end of a round, and of the second (dy, or v).  rows: with two
// stages of k its next tile came too late (a round 2970 cycles)
constexpr int bwd_stages1(bool keys, int chunks) { return chunks == 1 ? 4 : keys ? 2 : 3; }
constexpr int bwd_stages2(int chunks) { return chunks == 1 ? 4 : 2; }
constexpr size_t bwd_smem(bool keys, int chunks) {
  return 1024 + (size_t)(2 + bwd_stages1(keys, chunks) + bwd_stages2(chunks)) * chunks * kChunkBytes + (keys ? bwd_stages1(keys, chunks) * 1024 : 0) + 512;
}

struct BwdArgs {
  RowArgs r;
  int pack_shift;           // log2 of the heads in a tile of queries
  int blocks[2], each_blocks[2];      // of rows, of keys
  int key_ctas;             // the first CTAs have keys, the others rows
  long long budget;
  int drop_first_load;
};

template <bool kKeys, int kChunks>
__device__ __forceinline__ void bwd_cta(const CUtensorMap& tm_q, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CUtensorMap& tm_dy, const BwdArgs& a, int cta) {
  constexpr int kSt1 = bwd_stages1(kKeys, kChunks), kSt2 = bwd_stages2(kChunks);
  constexpr uint32_t kTile = kChunks * kChunkBytes;
  // columns of TMEM
  constexpr uint32_t kS = 0, kDp = 128, kAcc1 = kKeys ? 256 : 384, kAcc2 = 384;      // (rows: the second buffer of dP at 256)
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t x1 = base, x2 = x1 + kTile, y1 = x2 + kTile, y2 = y1 + kSt1 * kTile;      // the CTA's own tiles, and the stages of those it meets
  float* stats = reinterpret_cast<float*>(smem_raw + (base - raw) + (2 + kSt1 + kSt2) * kTile);      // keys: [stage][-lse, -delta][128]
  uint64_t* bars = reinterpret_cast<uint64_t*>(stats + (kKeys ? kSt1 * 256 : 0));
  const uint32_t x_full = smem_u32(bars), y1_full = x_full + 8, y1_empty = y1_full + 8 * kSt1, y2_full = y1_empty + 8 * kSt1, y2_empty = y2_full + 8 * kSt2;
  const uint32_t st_full = y2_empty + 8 * kSt2, st_empty = st_full + 8 * kSt1;
  const uint32_t s_full = st_empty + 8 * kSt1, dp_full = s_full + 8, p_full = dp_full + 16, ds_full = p_full + 16, acc_full = ds_full + 16, drain = acc_full + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 1 + 4 * kSt1 + 2 * kSt2 + 9);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  __shared__ Unit unit;
  __shared__ unsigned again[2][8];      // rows of a warp whose dk or dq, and whose dv, is not finite
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = a.r.heads / a.r.kv_heads;
  const int shift = a.pack_shift, pack = 1 << shift, tile_rows = 128 >> shift;      // rows of the sequence in a tile of queries
  const int own_rows = kKeys ? 128 : tile_rows, own_heads = kKeys ? 1 : pack, n_heads = kKeys ? a.r.kv_heads : a.r.heads;
  const int splits = kKeys ? a.r.key_splits : a.r.splits;
  int part = 0;
  if (splits > 1) { part = cta % splits; cta /= splits; }      // (divisions that most calls do without)
  const int columns = n_heads / own_heads, head0 = cta % columns * own_heads;      // the first of the CTA's heads

  // three warps side by side: barriers, the unit of work, TMEM
  if (warp == 1 && elected()) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_v) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_dy) : "memory");
    mbar_init(x_full, 1);
    for (int s = 0; s < kSt1; ++s) { mbar_init(y1_full + 8 * s, 1); mbar_init(y1_empty + 8 * s, 1); mbar_init(st_full + 8 * s, 32); mbar_init(st_empty + 8 * s, 8); }
    for (int s = 0; s < kSt2; ++s) { mbar_init(y2_full + 8 * s, 1); mbar_init(y2_empty + 8 * s, 1); }
    mbar_init(s_full, 1); mbar_init(dp_full, 1); mbar_init(dp_full + 8, 1); mbar_init(p_full, 8); mbar_init(p_full + 8, 8); mbar_init(ds_full, 8); mbar_init(ds_full + 8, 8); mbar_init(acc_full, 1); mbar_init(drain, 1);
    abort_flag[0] = abort_flag[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    Unit u;
    find_unit(a.r.seq, a.blocks[kKeys], a.each_blocks[kKeys], cta / columns, own_rows, &u, lane);
    if (u.seq >= 0 && kKeys && a.r.causal) u.row0 = (u.b - u.a - 1) / 128 * 128 - u.row0;      // the first keys are seen by most rows
    if (lane == 0) unit = u;
  }
  if (warp == 9) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const Unit u = unit;
  const uint32_t tmem = *tmem_slot;
  auto give_tmem_back = [&]() {
    __syncwarp();
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  };
  next_launch_may_come();
  after_the_launch_before();
  if (u.seq < 0) {      // rows of no sequence: zeros, shared out among the units that are left over
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int i = u.spare, row; (row = row_of_none(a.r.seq, i)) >= 0; i += u.spares)
      for (int c = 8 * threadIdx.x; c < own_heads * a.r.width; c += 8 * kBwdThreads) {
        const size_t at = ((size_t)row * n_heads + head0) * a.r.width + c;
        if (kKeys && a.r.dk) store_any<8>(a.r.dk, a.r.dkt, at, zero);
        if (kKeys && a.r.dv) store_any<8>(a.r.dv, a.r.dvt, at, zero);
        if (!kKeys) store_any<8>(a.r.out, a.r.ot, at, zero);
      }
    give_tmem_back();
    return;
  }
  const int n_rows = u.b - u.a, last = min(u.row0 + own_rows, n_rows) - 1;      // own rows: row0 .. last
  // the tiles it meets: keys: rows that see any of the own keys; rows: keys that any of the own rows sees
  int first = 0, end = n_rows;
  if (kKeys) {
    if (a.r.causal) first = u.row0;
    if (a.r.window) end = (int)min((long long)n_rows, (long long)last + a.r.window);
  } else {
    if (a.r.causal) end = last + 1;
    if (a.r.window) first = max(0, u.row0 - a.r.window + 1);
  }
  const int met_rows = kKeys ? tile_rows : 128, t0 = first / met_rows, tiles = (end + met_rows - 1) / met_rows - t0, all = tiles * (kKeys ? group >> shift : 1);
  int skip = 0, n = all, h_skip = 0, tile_skip = 0;      // this CTA's part of them
  if (splits > 1) {
    const int each = (all + splits - 1) / splits;
    skip = min(all, part * each);
    n = min(each, all - skip);
    h_skip = skip / tiles;
    tile_skip = skip - h_skip * tiles;
  }
  float* const to = splits > 1 ? (kKeys ? a.r.part_k : a.r.part) + (size_t)part * a.r.seq.rows * n_heads * a.r.width : nullptr;
  float* const to_v = splits > 1 && kKeys ? a.r.part_v + (size_t)part * a.r.seq.rows * n_heads * a.r.width : nullptr;
  if (n == 0) {      // (more parts than tiles)
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int wide = own_heads * a.r.width;
    for (int i = 8 * threadIdx.x; i < (last - u.row0 + 1) * wide; i += 8 * kBwdThreads) {
      const size_t at = ((size_t)(u.a + u.row0 + i / wide) * n_heads + head0) * a.r.width + i % wide;
      store_any<8>(to, DRAGON_F32, at, zero);
      if (kKeys) store_any<8>(to_v, DRAGON_F32, at, zero);
    }
    give_tmem_back();
    return;
  }

  auto wait_warp = [&](uint32_t bar, uint32_t parity) {
    if (mbar_wait_warp(bar, parity, abort_flag, a.budget)) return true;
    *abort_flag = 1;
    report(a.r.status, DRAGON_ERR_TIMEOUT);
    return false;
  };
  int issued1 = 0, issued2 = 0;
  if (warp == 8) {
    if (elected()) {
      mbar_expect_tx(x_full, 2 * kTile);
      for (int c = 0; c < kChunks; ++c) {
        tma_load_3d(x1 + c * kChunkBytes, kKeys ? &tm_k : &tm_q, 64 * c, head0, u.a + u.row0, x_full);
        tma_load_3d(x2 + c * kChunkBytes, kKeys ? &tm_v : &tm_dy, 64 * c, head0, u.a + u.row0, x_full);
      }
    }
    __syncwarp();
    bool ok = true;
    int h = kKeys ? head0 * group + h_skip : head0 / group, tile = tile_skip;
    for (int i = 0; i < n && ok; ++i, ++tile) {
      if (tile == tiles) { tile = 0; ++h; }
      const int s = i % kSt1, turn = i / kSt1, row = u.a + (t0 + tile) * met_rows;
      ok = wait_warp(y1_empty + 8 * s, (turn & 1) ^ 1);
      if (!ok) break;
      issued1 = i + 1;
      const bool leave_out = a.drop_first_load && i == 0;      // (failure-detection test: the first stage's signal never comes)
      if (elected() && !leave_out) {
        mbar_expect_tx(y1_full + 8 * s, kTile);
        for (int c = 0; c < kChunks; ++c) tma_load_3d(y1 + s * kTile + c * kChunkBytes, kKeys ? &tm_q : &tm_k, 64 * c, h, row, y1_full + 8 * s);
      }
      __syncwarp();
      if (kKeys) {      // -lse and -delta of the tile's rows; a row behind the sequence's last has probabilities 0
        ok = wait_warp(st_empty + 8 * s, (turn & 1) ^ 1);
        if (!ok) break;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = (t0 + tile) * tile_rows + ((32 * k + lane) >> shift);
          const size_t at = (size_t)(h + (lane & (pack - 1) & 31) + (32 * k & (pack - 1))) * a.r.seq.rows + u.a + r;
          stats[s * 256 + 32 * k + lane] = r < n_rows ? -__ldg(a.r.lse + at) : -kInf;
          stats[s * 256 + 128 + 32 * k + lane] = r < n_rows ? -__ldg(a.r.delta + at) : 0.f;
        }
        mbar_arrive(st_full + 8 * s);
      }
      const int s2 = i % kSt2;
      ok = wait_warp(y2_empty + 8 * s2, ((i / kSt2) & 1) ^ 1);
      if (!ok) break;
      issued2 = i + 1;
      if (elected()) {
        mbar_expect_tx(y2_full + 8 * s2, kTile);
        for (int c = 0; c < kChunks; ++c) tma_load_3d(y2 + s2 * kTile + c * kChunkBytes, kKeys ? &tm_dy : &tm_v, 64 * c, h, row, y2_full + 8 * s2);
      }
      __syncwarp();
    }
  } else if (warp == 9) {
    const int k_steps = (a.r.width + 15) / 16;
    const uint32_t idesc_s = idesc_bf16(128, 128, false), idesc_acc = idesc_bf16(128, 16 * k_steps, true);
    auto commit = [&](uint32_t bar) { if (elected()) umma_commit(bar); __syncwarp(); };
    auto dp_at = [&](int i) { return kDp + (kKeys ? 0 : 128 * (i & 1)); };
    auto issue_s = [&](int i) {
      if (!wait_warp(y1_full + 8 * (i % kSt1), (i / kSt1) & 1)) return false;
      fence_after();
      if (elected()) {
        product_over_head<kChunks>(tmem + kS, x1, y1 + (i % kSt1) * kTile, k_steps, idesc_s);
        umma_commit(s_full);
      }
      __syncwarp();
      return true;
    };
    auto issue_dp = [&](int i) {
      if (!wait_warp(y2_full + 8 * (i % kSt2), (i / kSt2) & 1)) return false;
      fence_after();
      if (elected()) {
        product_over_head<kChunks>(tmem + dp_at(i), x2, y2 + (i % kSt2) * kTile, k_steps, idesc_s);
        umma_commit(dp_full + (kKeys ? 0 : 8 * (i & 1)));
        if (!kKeys) umma_commit(y2_empty + 8 * (i % kSt2));
      }
      __syncwarp();
      return true;
    };
    auto accumulate = [&](uint32_t d, uint32_t p, uint32_t y, bool more, uint32_t empty) {
      fence_after();
      if (elected()) {
        product_over_rows<64>(tmem + d, tmem + p, y, idesc_acc, more);
        umma_commit(empty);
      }
      __syncwarp();
    };
    bool ok = wait_warp(x_full, 0) && issue_s(0) && issue_dp(0);
    for (int i = 0; i < n && ok; ++i) {
      const int s = i % kSt1, s2 = i % kSt2;
      if (kKeys) {
        // rows 0..31 and 64..95 of the tile, then the others
        if (!(ok = wait_warp(p_full, i & 1))) break;
        fence_after();
        if (elected()) {
          product_over_rows<64, 0, 2>(tmem + kAcc2, tmem + kS, y2 + s2 * kTile, idesc_acc, i > 0);
          product_over_rows<64, 4, 6>(tmem + kAcc2, tmem + kS, y2 + s2 * kTile, idesc_acc, true);
        }
        __syncwarp();
        if (!(ok = wait_warp(p_full + 8, i & 1))) break;
        fence_after();
        if (elected()) {
          product_over_rows<64, 2, 4>(tmem + kAcc2, tmem + kS, y2 + s2 * kTile, idesc_acc, true);
          product_over_rows<64, 6, 8>(tmem + kAcc2, tmem + kS, y2 + s2 * kTile, idesc_acc, true);
          umma_commit(y2_empty + 8 * s2);
        }
        __syncwarp();
        if (i + 1 < n && !(ok = issue_s(i + 1))) break;
        if (!(ok = wait_warp(ds_full, i & 1))) break;
        accumulate(kAcc1, kDp, y1 + s * kTile, i > 0, y1_empty + 8 * s);
        if (i + 1 < n && !(ok = issue_dp(i + 1))) break;
      } else {
        if (i + 1 < n) {
          if (!(ok = wait_warp(p_full, i & 1))) break;      // S has been read
          fence_after();
          if (!(ok = issue_s(i + 1) && issue_dp(i + 1))) break;
        }
        if (!(ok = wait_warp(ds_full + 8 * (i & 1), (i >> 1) & 1))) break;
        accumulate(kAcc1, dp_at(i), y1 + s * kTile, i > 0, y1_empty + 8 * s);
      }
    }
    if (ok) commit(acc_full);
  } else {
    const int e = (warp & 3) * 32 + lane, half = warp >> 2;
    const int row = u.row0 + (kKeys ? e : e >> shift), head = head0 + (kKeys ? 0 : e & (pack - 1));      // own row of the sequence (a key, or a query)
    const bool mine = row < n_rows;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    float lse = kInf, delta = 0.f;
    if (!kKeys && mine) {
      lse = a.r.lse[(size_t)head * a.r.seq.rows + u.a + row];
      delta = a.r.delta[(size_t)head * a.r.seq.rows + u.a + row];
    }
    const Pair factor = pair_of(a.r.scale, a.r.scale);
    bool ok = true;
    for (int i = 0, tile = tile_skip; i < n; ++i, ++tile) {
      if (tile == tiles) tile = 0;
      const int r0 = (t0 + tile) * met_rows, c0 = r0 + 64 * half;      // the tile's first row; (rows) this thread's first column
      // columns [lo, hi) are seen
      int lo, hi;
      if (kKeys) {
        lo = a.r.causal ? (min(max(row - r0, 0), tile_rows) << shift) - 64 * half : 0;
        hi = a.r.window ? ((int)min((long long)tile_rows, max(0LL, (long long)row + a.r.window - r0)) << shift) - 64 * half : 64;
      } else {
        hi = (a.r.causal ? min(row + 1, n_rows) : n_rows) - c0;
        lo = a.r.window ? row - a.r.window + 1 - c0 : 0;
      }
      const float4* st = reinterpret_cast<const float4*>(stats + (i % kSt1) * 256 + 64 * half);
      ok = wait_warp(s_full, i & 1);
      if (ok && kKeys) ok = wait_warp(st_full + 8 * (i % kSt1), (i / kSt1) & 1);
      if (!ok) break;
      fence_after();
      // 32 columns at a time: the next ones are on their way out of TMEM, and results into it, while these are worked on
      const bool all_seen = __all_sync(0xffffffffu, lo <= 0 && hi >= 64);
      const uint32_t s_at = tmem + lanes + kS + 64 * half;
      uint32_t v[64];
      float p[64];
      tmem_load32(s_at, v);
      if (kKeys) tmem_loaded32(v);
      tmem_load32(s_at + 32, v + 32);
      if (!kKeys) {      // (the next S may be written as soon as this one has been read)
        tmem_loaded32(v);
        tmem_loaded32(v + 32);
        fence_before();
        __syncwarp();
        mbar_arrive_if(p_full, lane == 0);
      }
#pragma unroll
      for (int h = 0; h < 64; h += 32) {
        if (kKeys && h) tmem_loaded32(v + 32);
#pragma unroll
        for (int c = h; c < h + 32; c += 4) {
          float4 l = make_float4(-lse, -lse, -lse, -lse);
          if (kKeys) l = st[c / 4];
          const float2 x = both(fma_pair(pair_of(v[c], v[c + 1]), factor, pair_of(l.x, l.y))), y = both(fma_pair(pair_of(v[c + 2], v[c + 3]), factor, pair_of(l.z, l.w)));
          p[c] = exp2_fast(x.x); p[c + 1] = exp2_fast(x.y); p[c + 2] = exp2_fast(y.x); p[c + 3] = exp2_fast(y.y);
        }
        if (!all_seen) {
#pragma unroll
          for (int c = h; c < h + 32; ++c) if (c < lo || c >= hi) p[c] = 0.f;
        }
        if (kKeys) {
          uint32_t w[16];
#pragma unroll
          for (int c = 0; c < 16; ++c) w[c] = bf16_pair(p[h + 2 * c], p[h + 2 * c + 1]);
          tmem_st16(s_at + h / 2, w);
          tmem_st_wait();
          fence_before();
          __syncwarp();
          mbar_arrive_if(p_full + h / 4, lane == 0);      // (the products of the first half start while the second is worked on)
        }
      }
      const uint32_t dp = tmem + lanes + kDp + (kKeys ? 0 : 128 * (i & 1)) + 64 * half;
      ok = wait_warp(dp_full + (kKeys ? 0 : 8 * (i & 1)), (kKeys ? i : i >> 1) & 1);
      if (!ok) break;
      fence_after();
      tmem_load32(dp, v);
      tmem_loaded32(v);
      tmem_load32(dp + 32, v + 32);
#pragma unroll
      for (int h = 0; h < 64; h += 32) {
        if (h) tmem_loaded32(v + 32);
        uint32_t w[16];
#pragma unroll
        for (int c = h; c < h + 32; c += 4) {
          float4 d = make_float4(-delta, -delta, -delta, -delta);
          if (kKeys) d = st[32 + c / 4];
          const float2 x = both(mul_pair(pair_of(p[c], p[c + 1]), add_pair(pair_of(v[c], v[c + 1]), pair_of(d.x, d.y))));
          const float2 y = both(mul_pair(pair_of(p[c + 2], p[c + 3]), add_pair(pair_of(v[c + 2], v[c + 3]), pair_of(d.z, d.w))));
          w[(c - h) / 2] = bf16_pair(x.x, x.y);
          w[(c - h) / 2 + 1] = bf16_pair(y.x, y.y);
        }
        tmem_st16(dp + h / 2, w);
      }
      tmem_st_wait();
      fence_before();
      __syncwarp();
      // (rows: S and dP of the next round are there by now, so a warp can be here again before another one has come here for this round:
      // two barriers, in turn)
      mbar_arrive_if(ds_full + (kKeys ? 0 : 8 * (i & 1)), lane == 0);
      if (kKeys) mbar_arrive_if(st_empty + 8 * (i % kSt1), lane == 0);
    }
    if (ok) {
      ok = wait_warp(acc_full, 0);
      fence_after();
    }
    bool fine[2] = {true, true};
    if (ok) {      // a warp writes half of the head's elements
      const size_t at = ((size_t)(u.a + row) * n_heads + head) * a.r.width;
      auto write = [&](uint32_t acc, void* out, int type, float factor, bool* fine) {
#pragma unroll 1
        for (int c = 32 * kChunks * half; c < min(a.r.width, 32 * kChunks * (half + 1)); c += 16) {
          uint32_t o[16];
          float f[16];
          tmem_ld16(tmem + lanes + acc + c, o);
          tmem_loaded16(o);
#pragma unroll
          for (int k = 0; k < 16; ++k) { f[k] = __uint_as_float(o[k]) * factor; *fine &= fabsf(f[k]) < kInf; }
          if (mine && out) {
            store_any<8>(out, type, at + c, f);
            if (c + 8 < a.r.width) store_any<8>(out, type, at + c + 8, f + 8);
          }
        }
      };
      const bool parts = splits > 1;
      if (kKeys) {
        write(kAcc1, parts ? to : a.r.dk, parts ? DRAGON_F32 : a.r.dkt, a.r.raw_scale, fine);
        write(kAcc2, parts ? to_v : a.r.dv, parts ? DRAGON_F32 : a.r.dvt, 1.f, fine + 1);
      } else {
        write(kAcc1, parts ? to : a.r.out, parts ? DRAGON_F32 : a.r.ot, a.r.raw_scale, fine);
      }
      fine[0] |= parts || (kKeys && !a.r.dk);      // (where the parts are added up a row that is not finite is computed again)
      fine[1] |= parts || !kKeys || !a.r.dv;
    }
    // rows that are not finite: again, after both halves have been written (every warp comes here, after an unwind too)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const unsigned bad = __ballot_sync(0xffffffffu, mine && !fine[k]);
      if (lane == 0) again[k][warp] = bad;
    }
    __syncwarp();
    asm volatile("bar.sync 1, 256;" ::: "memory");
    {      // the two warps of 32 rows take turns
      const unsigned bad1 = again[0][warp & 3] | again[0][(warp & 3) + 4], bad2 = again[1][warp & 3] | again[1][(warp & 3) + 4];
      int turn = 0;
      for (unsigned b = bad1 | bad2; b; b &= b - 1) {
        if ((turn++ & 1) != half) continue;
        const int r = (warp & 3) * 32 + __ffs(b) - 1, first_row = u.a + u.row0;
        const unsigned bit = b & (0u - b);
        if (kKeys) dkv_of_row(a.r, head0, first_row + r, lane, bad1 & bit, bad2 & bit);
        else dq_of_row(a.r, head0 + (r & (pack - 1)), first_row + (r >> shift), lane);
      }
    }
  }
  fence_before();
  __syncthreads();
  if (*abort_flag) {      // an unwind: copies and products that have been asked for end before their memory goes away
    if (warp == 9) {
      if (elected()) umma_commit(drain);
      __syncwarp();
      mbar_wait_warp(drain, 0, abort_flag + 1, kWaitBudgetCycles);
    }
    if (threadIdx.x == 256) {
      mbar_wait(x_full, 0, abort_flag + 1);
      for (int k = std::max(a.drop_first_load ? 1 : 0, issued1 - kSt1); k < issued1; ++k) mbar_wait(y1_full + 8 * (k % kSt1), (k / kSt1) & 1, abort_flag + 1);
      for (int k = std::max(0, issued2 - kSt2); k < issued2; ++k) mbar_wait(y2_full + 8 * (k % kSt2), (k / kSt2) & 1, abort_flag + 1);
    }
    __syncthreads();
  }
  give_tmem_back();
}

template <int kChunks>
__global__ void __launch_bounds__(kBwdThreads, 1)
attention_bwd(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
              const __grid_constant__ CUtensorMap tm_dy, const __grid_constant__ BwdArgs a) {
  if ((int)blockIdx.x < a.key_ctas) bwd_cta<true, kChunks>(tm_q, tm_k, tm_v, tm_dy, a, blockIdx.x);
  else bwd_cta<false, kChunks>(tm_q, tm_k, tm_v, tm_dy, a, blockIdx.x - a.key_ctas);
}

// delta = sum(dy y) of every row and head, y with what its rounding left out: in a row that sees few keys dp - delta is small, and
// with the rounded y alone dq and dk of short sequences were off by 0.0030 of their norm, not 0.0024.  A head in the next power of two of lanes, 8 elements a lane
__global__ void __launch_bounds__(256) attention_delta(const __grid_constant__ RowArgs a, int lanes) {
  next_launch_may_come();
  after_the_launch_before();
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.status_clear) *a.status_clear = 0;
  const int lane = threadIdx.x & 31, l = lane & (lanes - 1);
  const long long i = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * (32 / lanes) + lane / lanes, n = (long long)a.seq.rows * a.heads;      // row by row, head by head
  float sum = 0.f;
  if (i < n && 8 * l < a.width) {
    float y[8], d[8];
    load_any<8>(a.y, a.yt, (size_t)i * a.width + 8 * l, y);
    load_any<8>(a.dy, DRAGON_BF16, (size_t)i * a.width + 8 * l, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += y[e] * d[e];
    if (a.rest) {
      load_any<8>(a.rest, DRAGON_BF16, (size_t)i * a.width + 8 * l, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += y[e] * d[e];
    }
  }
  for (int s = lanes >> 1; s; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
  if (i < n && l == 0) a.delta[(size_t)(i % a.heads) * a.seq.rows + i / a.heads] = sum;
}

template <int kChunks> int launch_bwd(const BwdArgs& a, long long ctas, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const CUtensorMap& dy, cudaStream_t st) {
  static const char* who = "Attention's gradient";
  static bool set[64] = {};
  constexpr size_t bytes = std::max(bwd_smem(true, kChunks), bwd_smem(false, kChunks));
  const int rc = allow_smem(reinterpret_cast<const void*>(attention_bwd<kChunks>), bytes, set, who);
  if (rc != DRAGON_OK) return rc;
  if (ctas > 0x7fffffffLL) { set_error("%s: too many blocks of rows", who); return DRAGON_ERR_UNSUPPORTED; }
  return launch_behind(attention_bwd<kChunks>, dim3((unsigned)ctas), dim3(kBwdThreads), bytes, st, who, q, k, v, dy, a);
}

}  // namespace

// CTAs of both kinds that there are at least, without splits, and the rows of a sequence in a tile of queries
void attention_bwd_units(int64_t rows, int64_t sequences, int heads, int kv_heads, int64_t* row_units, int64_t* key_units, int* tile_rows) {
  const int group = heads / kv_heads, pack = packs(group) ? group : 1;
  *tile_rows = 128 / pack;
  *row_units = std::max<int64_t>(sequences, (rows + *tile_rows - 1) / *tile_rows) * (heads / pack);
  *key_units = std::max<int64_t>(sequences, (rows + 127) / 128) * kv_heads;
}

int launch_attention_backward(const RowArgs& rows, cudaStream_t st) {
  BwdArgs a = {};
  a.r = rows;
  const int group = rows.heads / rows.kv_heads;
  while (packs(group) && 1 << a.pack_shift < group) ++a.pack_shift;
  const int tile_rows = 128 >> a.pack_shift, pack = 1 << a.pack_shift;
  count_blocks(rows.seq, tile_rows, &a.blocks[0], &a.each_blocks[0]);
  count_blocks(rows.seq, 128, &a.blocks[1], &a.each_blocks[1]);
  wait_settings("DRAGON_ATTENTION", &a.budget, &a.drop_first_load);
  CUtensorMap q, k, v, dy;
  if (!head_map(&q, rows.q, rows.seq.rows, rows.heads, rows.width, tile_rows, pack) || !head_map(&k, rows.k, rows.seq.rows, rows.kv_heads, rows.width, 128) ||
      !head_map(&v, rows.v, rows.seq.rows, rows.kv_heads, rows.width, 128) || !head_map(&dy, rows.dy, rows.seq.rows, rows.heads, rows.width, tile_rows, pack)) {
    set_error("Attention's gradient: cannot encode the TMA descriptors (no CUDA driver?)");
    return DRAGON_ERR_CUDA;
  }
  int lanes = 1;
  while (lanes * 8 < rows.width) lanes *= 2;
  const long long warps = ((long long)rows.seq.rows * rows.heads * lanes + 31) / 32;
  int rc = launch_behind(attention_delta, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, st, "Attention's gradient", rows, lanes);
  const long long key_ctas = rows.dk || rows.dv ? (long long)a.blocks[1] * rows.kv_heads * rows.key_splits : 0;
  const long long ctas = key_ctas + (rows.out ? (long long)a.blocks[0] * (rows.heads / pack) * rows.splits : 0);
  a.key_ctas = (int)std::min(key_ctas, 0x7fffffffLL);
  if (rc == DRAGON_OK && ctas) rc = rows.width > 64 ? launch_bwd<2>(a, ctas, q, k, v, dy, st) : launch_bwd<1>(a, ctas, q, k, v, dy, st);
  return rc;
}

}  // namespace dragon
