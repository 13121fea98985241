// CacheWrite: the rows of new tokens to their places in a cache of pages.  Bound: HBM and, for a decoding step's few rows, the
// launch.  A warp copies one row of one cache, 16 bytes a lane; keys and values of the same table are one launch.
//
// PagedAttention for few rows (a decoding step): every key and value is read once and used by few rows (the query heads that
// share its head, times the new tokens), so HBM is the bound, and what counts is that enough copies are in flight and that all
// SMs have some.  The keys of a sequence and key head are split over CTAs; in a CTA each of four warps walks its own groups of 16
// keys through its own ring of stages (cp.async; no barrier between warps), with mma.sync products of 16 rows and an online
// softmax in registers (a tile of tcgen05 would have 128 rows, of which 8 were real).  A group of 16 keys lies in one page.
// One sequence of 95225 tokens, 32 heads on 8 of 128: 67 us, 5.8 TB/s (this kernel alone; the whole step 75 to 79).
// What the warps and the CTAs have is put together by their maxima, in a fixed order.  Sequences with more rows go to the
// tensor-core kernel for tiles (attention_tcgen05.cu), whose keys are split likewise.
#include <cuda_runtime.h>

#include <algorithm>

#include "attention_rows.h"
#include "attention_tiles.h"

namespace dragon {
int launch_attention_forward(const RowArgs& rows, bool paged, int64_t key_rows, int few, int sm_count, cudaStream_t st, const char* who);
int64_t attention_units(int64_t rows, int64_t sequences, int heads, int kv_heads);
namespace {

constexpr int kWriteWarps = 8;
constexpr int kPartsMost = 128;       // parts of a sequence's keys

struct WriteArgs {
  const uint4* rows[kCachesPerLaunch];
  uint4* cache[kCachesPerLaunch];
  int vectors[kCachesPerLaunch];      // 16-byte vectors of a row
  int pool[kCachesPerLaunch];         // pages of the cache
  Sequences seq;
  Pages pages;
  int* status;
  int* status_clear;
};

__global__ void __launch_bounds__(32 * kWriteWarps) cache_write(const __grid_constant__ WriteArgs a) {
  next_launch_may_come();
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    if (threadIdx.x == 0 && a.status_clear) *a.status_clear = 0;
    if (!a.seq.in_order()) report(a.status, DRAGON_ERR_INVALID_ARG);
  }
  const int lane = threadIdx.x & 31, row = blockIdx.x * kWriteWarps + (threadIdx.x >> 5), c = blockIdx.y;
  if (row >= a.seq.rows) return;
  const int s = a.seq.of_row(row);
  if (s < 0) return;
  int r0, r1;
  a.seq.rows_of(s, &r0, &r1);
  // (a position behind the table's room is no place: the row is reported, not written)
  const int p = max(__ldg(a.pages.lengths + s), 0) - (r1 - r0) + (row - r0);
  if (p < 0) return;
  const int page = (p >> a.pages.shift) < a.pages.most ? a.pages.page_of(s, p) : -1;
  if (page < 0 || page >= a.pool[c]) {
    if (lane == 0) report(a.status, DRAGON_ERR_INVALID_ARG);
    return;
  }
  const int n = a.vectors[c];
  const uint4* from = a.rows[c] + (size_t)row * n;
  uint4* to = a.cache[c] + (((size_t)page << a.pages.shift) + (p & ((1 << a.pages.shift) - 1))) * n;
  int i = lane;
  for (; i + 96 < n; i += 128) {
    const uint4 v0 = __ldg(from + i), v1 = __ldg(from + i + 32), v2 = __ldg(from + i + 64), v3 = __ldg(from + i + 96);
    to[i] = v0; to[i + 32] = v1; to[i + 64] = v2; to[i + 96] = v3;
  }
  for (; i < n; i += 32) to[i] = __ldg(from + i);
}

// ---- few rows ------------------------------------------------------------------------------------

constexpr int kFewWarps = 4, kFewStages = 2, kFewMost = 32;      // kFewMost: rows (times heads of a group) of a sequence
constexpr int few_pitch(int steps) { return steps * 32 + 16; }      // bytes of a key in a stage: an odd number of 16, for ldmatrix
constexpr int few_smem(int steps, int m) { return std::max(kFewWarps * kFewStages * 2 * 16 * few_pitch(steps), kFewWarps * 16 * m * (16 * steps + 4) * 4) + 16; }

// CTAs of it that an SM holds, by shared memory and registers.  Two stages and a CTA more were faster than three stages (64 sequences of
// 2000 to 4000 tokens 160 -> 148 us)
constexpr int few_resident(int steps, int m) {
  return std::min(227 * 1024 / (few_smem(steps, m) + 2048), m == 1 ? 5 : steps <= 2 ? 4 : steps <= 4 ? 3 : 2);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool real) {      // zeros where it is not real
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_of(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// where a part of few rows stands among those of its split; r: new row of the sequence x group + head of the group
__device__ __forceinline__ size_t few_item(const RowArgs& a, int s, int kvh, int r, int row, int head) {
  return a.slots ? ((size_t)s * a.kv_heads + kvh) * a.slots + r : (size_t)row * a.heads + head;
}

// kSteps: 16 elements of the head each; kM: 16 rows each
template <int kSteps, int kM> __global__ void __launch_bounds__(32 * kFewWarps, few_resident(kSteps, kM)) paged_few(const __grid_constant__ RowArgs a, int few, int columns) {
  constexpr int kPitch = few_pitch(kSteps), kRows = 16 * kM, kStage = 2 * 16 * kPitch, kOut = 16 * kSteps + 4;
  extern __shared__ __align__(16) unsigned char smem_few[];
  __shared__ float warp_top[kFewWarps][kRows], warp_sum_of[kFewWarps][kRows];
  __shared__ int row_bad[kRows];
  next_launch_may_come();
  after_the_launch_before();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x % a.splits, column = blockIdx.x / a.splits % columns, s = blockIdx.x / a.splits / columns;
  const int kvh = column % a.kv_heads, tile = column / a.kv_heads, group = a.heads / a.kv_heads;
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  if (blockIdx.x == 0 && !a.seq.in_order()) report(a.status, DRAGON_ERR_INVALID_ARG);
  int r0, r1;
  a.seq.rows_of(s, &r0, &r1);
  if (!has_few_rows(r1 - r0, group, few)) return;
  const int rows = (r1 - r0) * group, first = tile * kRows;      // row r: new token r / group, head r % group of the group
  if (first >= rows) return;
  bool fits;
  const int tokens = a.pages.tokens(s, &fits), base = tokens - (r1 - r0);
  if (!fits && threadIdx.x == 0) report(a.status, DRAGON_ERR_INVALID_ARG);
  // keys that any row of the tile sees, in groups of 16; this CTA's part of them
  const int low = base + first / group, high = base + (min(first + kRows, rows) - 1) / group;      // positions of the first and last row
  const int g_end = max(0, min(high + 1, tokens) + 15) / 16, g_begin = a.window ? max(0, low - a.window + 1) / 16 : 0;
  const int each = (max(0, g_end - g_begin) + a.splits - 1) / a.splits, my0 = g_begin + split * each, my1 = min(g_end, my0 + each);
  // q: A fragments of this thread
  uint32_t q[kM][kSteps][4];
  int pos[kM][2];      // positions of its rows
#pragma unroll
  for (int m = 0; m < kM; ++m)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int r = first + 16 * m + 8 * b + g;
      const bool real = r < rows;
      pos[m][b] = real ? base + r / group : -1;
      const unsigned short* from = a.q + ((size_t)(r0 + (real ? r / group : 0)) * a.heads + kvh * group + (real ? r % group : 0)) * a.width;
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int at = 16 * k + 8 * c + 2 * t;
          q[m][k][b + 2 * c] = real && at < a.width ? __ldg(reinterpret_cast<const unsigned*>(from + at)) : 0u;
        }
    }
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem_few) + warp * kFewStages * kStage;
  // the elements behind the head's width are never copied: zeros once (q's are zeros too, but 0 times what was there may be NaN)
  if (16 * kSteps > a.width) {
    const int gap = 16 * kSteps - a.width;      // a multiple of 8
    for (int i = lane; i < kFewStages * 32 * (gap / 8); i += 32) {
      const int line = i / (gap / 8), c = a.width / 8 + i % (gap / 8);
      *reinterpret_cast<uint4*>(smem_few + warp * kFewStages * kStage + line * kPitch + 16 * c) = make_uint4(0, 0, 0, 0);
    }
  }
  const int vectors = a.width / 8;
  auto number_of = [&](int grp) { return grp < my1 ? a.pages.page_of(s, 16 * grp) : 0; };
  auto issue = [&](int grp, int slot, int number) {
    if (grp < my1) {
      const bool good = a.pages.in_pool(number);
      if (!good && lane == 0) report(a.status, DRAGON_ERR_INVALID_ARG);
      const int k0 = 16 * grp, in_page = k0 & ((1 << a.pages.shift) - 1);
      const size_t line = good ? ((size_t)number << a.pages.shift) + in_page : 0;
      const size_t pitch = (size_t)a.kv_heads * a.width, from = line * pitch + (size_t)kvh * a.width;
      const uint32_t dst = ring + slot * kStage;
      for (int i = lane; i < 16 * vectors; i += 32) {
        const int key = i / vectors, c = i - key * vectors;
        const bool real = good && k0 + key < tokens;
        const size_t off = from + (real ? (size_t)key * pitch : 0) + 8 * c;
        copy16(dst + key * kPitch + 16 * c, a.k + off, real);
        copy16(dst + (16 + key) * kPitch + 16 * c, a.v + off, real);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float o[kM][2 * kSteps][4], top[kM][2], sum[kM][2];
#pragma unroll
  for (int m = 0; m < kM; ++m) {
    top[m][0] = top[m][1] = -kInf;
    sum[m][0] = sum[m][1] = 0.f;
#pragma unroll
    for (int n = 0; n < 2 * kSteps; ++n) o[m][n][0] = o[m][n][1] = o[m][n][2] = o[m][n][3] = 0.f;
  }
  int grp = my0 + warp, number = number_of(grp);
#pragma unroll
  for (int st = 0; st < kFewStages - 1; ++st) {
    const int now = number;
    number = number_of(grp + kFewWarps * (st + 1));
    issue(grp + kFewWarps * st, st, now);
  }
  __syncwarp();
  int slot = 0;
  for (; grp < my1; grp += kFewWarps) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 2) : "memory");
    __syncwarp();
    {
      const int now = number, ahead = grp + kFewWarps * (kFewStages - 1);
      number = number_of(ahead + kFewWarps);
      issue(ahead, slot == 0 ? kFewStages - 1 : slot - 1, now);
    }
    const uint32_t keys = ring + slot * kStage, values = keys + 16 * kPitch;
    slot = slot == kFewStages - 1 ? 0 : slot + 1;
    float x[kM][2][4];
#pragma unroll
    for (int m = 0; m < kM; ++m)
#pragma unroll
      for (int n = 0; n < 2; ++n) x[m][n][0] = x[m][n][1] = x[m][n][2] = x[m][n][3] = 0.f;
    const uint32_t k_lane = keys + ((lane >> 4) * 8 + (lane & 7)) * kPitch + ((lane >> 3) & 1) * 16;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      uint32_t b[4];
      ldsm4(k_lane + 32 * k, b);
#pragma unroll
      for (int m = 0; m < kM; ++m) { mma16(x[m][0], q[m][k], b[0], b[1]); mma16(x[m][1], q[m][k], b[2], b[3]); }
    }
    const int k0 = 16 * grp;
    uint32_t p[kM][4];
#pragma unroll
    for (int m = 0; m < kM; ++m) {
      if (!__all_sync(0xffffffffu, k0 + 15 <= min(pos[m][0], pos[m][1]) && (!a.window || k0 > max(pos[m][0], pos[m][1]) - a.window))) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int key = k0 + 8 * n + 2 * t + (c & 1), at = pos[m][c >> 1];
            if (key > at || (a.window && key <= at - a.window)) x[m][n][c] = -kInf;
          }
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float most = fmaxf(fmaxf(x[m][0][2 * b], x[m][0][2 * b + 1]), fmaxf(x[m][1][2 * b], x[m][1][2 * b + 1]));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const bool grown = most > top[m][b];
        if (__any_sync(0xffffffffu, grown)) {
          const float f = grown ? exp2_of((top[m][b] - most) * a.scale) : 1.f;
          if (grown) top[m][b] = most;
          sum[m][b] *= f;
#pragma unroll
          for (int n = 0; n < 2 * kSteps; ++n) { o[m][n][2 * b] *= f; o[m][n][2 * b + 1] *= f; }
        }
        const float shift = top[m][b] == -kInf ? 0.f : top[m][b] * a.scale;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float e = exp2_of(fmaf(x[m][n][2 * b + c], a.scale, -shift));
            x[m][n][2 * b + c] = e;
            sum[m][b] += e;
          }
      }
      p[m][0] = bf16_pair(x[m][0][0], x[m][0][1]);
      p[m][1] = bf16_pair(x[m][0][2], x[m][0][3]);
      p[m][2] = bf16_pair(x[m][1][0], x[m][1][1]);
      p[m][3] = bf16_pair(x[m][1][2], x[m][1][3]);
    }
    const uint32_t v_lane = values + (((lane >> 3) & 1) * 8 + (lane & 7)) * kPitch + (lane >> 4) * 16;
#pragma unroll
    for (int n = 0; n < kSteps; ++n) {
      uint32_t b[4];
      ldsm4_t(v_lane + 32 * n, b);
#pragma unroll
      for (int m = 0; m < kM; ++m) { mma16(o[m][2 * n], p[m], b[0], b[1]); mma16(o[m][2 * n + 1], p[m], b[2], b[3]); }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();      // the rings are free
  float* outs = reinterpret_cast<float*>(smem_few);      // [warp][row][kOut]
#pragma unroll
  for (int m = 0; m < kM; ++m)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      float l = sum[m][b];
      l += __shfl_xor_sync(0xffffffffu, l, 1);
      l += __shfl_xor_sync(0xffffffffu, l, 2);
      const int r = 16 * m + 8 * b + g;
      if (t == 0) { warp_top[warp][r] = top[m][b]; warp_sum_of[warp][r] = l; }
#pragma unroll
      for (int n = 0; n < 2 * kSteps; ++n)
        *reinterpret_cast<float2*>(outs + (warp * kRows + r) * kOut + 8 * n + 2 * t) = make_float2(o[m][n][2 * b], o[m][n][2 * b + 1]);
    }
  if (threadIdx.x < kRows) row_bad[threadIdx.x] = 0;
  __syncthreads();
  const bool parts = a.splits > 1;
  for (int i = threadIdx.x; i < kRows * vectors; i += 32 * kFewWarps) {
    const int r = i / vectors, c = 8 * (i - r * vectors);
    if (first + r >= rows) continue;
    float most = -kInf;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) most = fmaxf(most, warp_top[w][r]);
    const float shift = most == -kInf ? 0.f : most;
    float l = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float f = exp2_of((warp_top[w][r] - shift) * a.scale);
      l += f * warp_sum_of[w][r];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += f * outs[(w * kRows + r) * kOut + c + e];
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;      // (a NaN stays one)
    bool fine = fabsf(l) < kInf;
#pragma unroll
    for (int e = 0; e < 8; ++e) { v[e] *= inv; fine &= fabsf(v[e]) < kInf; }
    const int row = r0 + (first + r) / group, head = kvh * group + (first + r) % group;
    const size_t at = ((size_t)row * a.heads + head) * a.width + c;
    if (parts) {
      const size_t item = split * (size_t)a.part_items + few_item(a, s, kvh, first + r, row, head);
      if (my1 > my0) store_any<8>(a.part, DRAGON_F32, item * a.width + c, v);
      if (c == 0) a.part_lse[item] = l == 0.f ? -kInf : most * a.scale + log2f(l);
    } else {
      store_any<8>(a.out, a.ot, at, v);
      if (!fine) row_bad[r] = 1;
    }
  }
  if (parts) return;      // (where the parts are put together a row that is not finite is computed again)
  __syncthreads();
  for (int r = warp; r < kRows && first + r < rows; r += kFewWarps)
    if (row_bad[r]) attend_row<true>(a, kvh * group + (first + r) % group, r0 + (first + r) / group, lane);
}

// The parts of every row put together; rows of no sequence get zeros.  A row and head for `ways` warps (1 or 8), which share its
// parts, 4 elements a lane.  by_sequence: only rows of sequences of few rows (the others have no parts).
__global__ void __launch_bounds__(256) paged_join(const __grid_constant__ RowArgs a, const float* tile_part, const float* tile_lse, int few, int few_splits, int tile_splits,
                                                  int ways, int by_sequence) {
  __shared__ float sums[8][132];
  after_the_launch_before();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, way = warp & (ways - 1), group = a.heads / a.kv_heads;
  const long long item = ((long long)blockIdx.x * 8 + warp) / ways;
  int row, head, s, splits = 0;
  const float *part = a.part, *lse = a.part_lse;
  size_t from = 0, stride = a.part_items;      // its first part, and from one to the next
  if (by_sequence) {
    const int slots = a.kv_heads * few, slot = (int)(item % slots), r = slot % few;
    s = (int)(item / slots);
    if (s >= a.seq.count) return;
    int r0, r1;
    a.seq.rows_of(s, &r0, &r1);
    if (!has_few_rows(r1 - r0, group, few) || r >= (r1 - r0) * group) return;
    row = r0 + r / group;
    head = slot / few * group + r % group;
    splits = few_splits;
    from = few_item(a, s, slot / few, r, row, head);
  } else {
    if (item >= (long long)a.seq.rows * a.heads) return;
    row = (int)(item / a.heads);
    head = (int)(item % a.heads);
    s = a.seq.of_row(row);
    if (s >= 0) {
      int r0, r1;
      a.seq.rows_of(s, &r0, &r1);
      const bool is_few = has_few_rows(r1 - r0, group, few);
      splits = is_few ? few_splits : tile_splits;
      if (splits == 1) return;      // written already
      if (is_few) {
        from = few_item(a, s, head / group, (row - r0) * group + head % group, row, head);
      } else {
        from = (size_t)row * a.heads + head;
        stride = (size_t)a.seq.rows * a.heads;
        part = tile_part;
        lse = tile_lse;
      }
    }
  }
  float most = -kInf;
  for (int p = lane; p < splits; p += 32) most = fmaxf(most, lse[p * stride + from]);
#pragma unroll
  for (int k = 16; k; k >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, k));
  const float shift = most == -kInf ? 0.f : most;
  float total = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
  // loads without a condition, so that they are on their way together; what a part without keys left (it wrote nothing) is not taken
  const bool in = 4 * lane < a.width;
  lse += from;
  part += from * a.width + (in ? 4 * lane : 0);
  const size_t step = stride * a.width;
  for (int p0 = way; p0 < splits; p0 += 4 * ways) {
    float l[4];
    float4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int p = min(p0 + k * ways, splits - 1);
      l[k] = lse[p * stride];
      x[k] = *reinterpret_cast<const float4*>(part + p * step);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (p0 + k * ways >= splits || l[k] == -kInf) continue;
      const float w = exp2f(l[k] - shift);
      total += w;
      v[0] += w * x[k].x; v[1] += w * x[k].y; v[2] += w * x[k].z; v[3] += w * x[k].w;
    }
  }
  if (ways > 1) {      // (the CTA has one row and head: it came here as a whole)
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[warp][4 * lane + e] = v[e];
    if (lane == 0) sums[warp][128] = total;
    __syncthreads();
    if (warp) return;
    for (int w = 1; w < 8; ++w) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += sums[w][4 * lane + e];
      total += sums[w][128];
    }
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  bool fine = fabsf(total) < kInf;
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[e] *= inv; fine &= fabsf(v[e]) < kInf; }
  if (in) {
    const size_t at = ((size_t)row * a.heads + head) * a.width + 4 * lane;
    if (a.ot == DRAGON_F32) *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2*>(reinterpret_cast<unsigned short*>(a.out) + at) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
  }
  if (!__all_sync(0xffffffffu, fine)) {
    __syncwarp();
    attend_row<true>(a, head, row, lane);
  }
}

// How a PagedAttention is run: its kernels, and into how many parts each splits a sequence's keys.  Lengths are on the device, so
// the rule goes by the room that the table has for a sequence.
struct PagedPlan {
  bool few, tiles, join;
  int most_few;                       // rows x group of a sequence that the kernel for few rows takes
  int few_rows;                       // of one CTA
  int few_splits, tile_splits;
  int slots;                          // numbering of the few rows' parts (RowArgs), and how many of a split
  int64_t few_items;
  // the workspace in floats: log sums and results of the few rows' parts, then of the tiles'
  int64_t few_lse, few_part, tile_lse, tile_part, floats;
};

// Parts: as many as bring the CTAs to `waves` times what the GPU holds at once, of at least `least` keys each
int parts_of(int64_t units, int64_t room, int64_t ctas, int64_t least) {
  return (int)std::max<int64_t>(1, std::min({(ctas + units - 1) / units, (room + least - 1) / least, (int64_t)kPartsMost}));
}

PagedPlan plan_paged(int64_t rows, int64_t sequences, bool starts, int64_t room, int heads, int kv_heads, int width, int sm_count) {
  PagedPlan p = {};
  const int group = heads / kv_heads;
  const int64_t each = rows / sequences * group;      // without starts: rows x group of every sequence
  // with starts any sequence may have few rows or many; one of more than kFewMost goes to the kernel of tiles.  16 rows a CTA suffice
  // for the single new rows that are usual
  p.most_few = starts && group <= 16 ? 16 : kFewMost;
  p.few = starts ? group <= kFewMost : each <= kFewMost;
  p.tiles = starts ? rows * group > p.most_few || !p.few : !p.few;
  if (!p.few) p.most_few = 0;
  p.few_rows = p.most_few > 16 && (starts || each > 16) ? 32 : 16;
  // few rows: as many parts as the GPU holds at once (one sequence of 95225 tokens, the whole step: 88 us with 512 CTAs, 79 with the 440 that are there
  // together); with more sequences than that, whose lengths differ, parts of which some eight CTAs an SM come
  const int64_t units = sequences * kv_heads, slots = few_resident((width + 31) / 32 * 2, p.few_rows / 16) * (int64_t)sm_count;
  p.few_splits = p.few ? parts_of(units, room, units <= slots ? slots / units * units : 8 * (int64_t)sm_count, 256) : 1;
  p.tile_splits = p.tiles ? parts_of(attention_units(rows, sequences, heads, kv_heads), room, sm_count, 512) : 1;
  p.join = starts ? p.few_splits > 1 || p.tile_splits > 1 || !p.tiles : p.few_splits > 1 || p.tile_splits > 1;
  // (numbered by rows with 64 sequences of single new rows, by slots with a chunk of 16384 rows, 64 heads on 8: 8.5 MB where all rows would take 29.8 GB)
  const int64_t most = std::min<int64_t>(p.most_few, starts ? rows * group : each), by_slots = sequences * kv_heads * most;
  p.slots = by_slots < rows * heads ? (int)most : 0;
  p.few_items = p.slots ? by_slots : rows * heads;
  auto take = [&](int64_t floats) { const int64_t at = p.floats; p.floats += (floats + 63) & ~(int64_t)63; return at; };
  const int64_t few = p.few_splits > 1 ? p.few_splits * p.few_items : 0, tile = p.tile_splits > 1 ? p.tile_splits * rows * heads : 0;
  p.few_lse = take(few); p.few_part = take(few * width);
  p.tile_lse = take(tile); p.tile_part = take(tile * width);
  return p;
}
PagedPlan plan_of(const Step& s, const std::vector<MemRef>& mems, int sm_count) {
  const Shape &q = mems[s.rd[pa::Q]].shape, &pages = mems[s.rd[pa::PAGES]].shape;
  return plan_paged(q.d[0], pages.d[0], s.rd[pa::STARTS] >= 0, std::min<int64_t>(pages.d[1] * (int64_t)s.num[pn::PAGE], 0x7fffffff), (int)s.num[pn::HEADS],
                    (int)s.num[pn::KV_HEADS], (int)(q.d[1] / (int64_t)s.num[pn::HEADS]), sm_count);
}

template <int kSteps> int launch_few(const RowArgs& a, const PagedPlan& p, int most_rows, cudaStream_t st) {
  static bool set[2][64] = {};
  const bool wide = p.few_rows > 16;
  const void* kernel = wide ? reinterpret_cast<const void*>(paged_few<kSteps, 2>) : reinterpret_cast<const void*>(paged_few<kSteps, 1>);
  const int bytes = few_smem(kSteps, wide ? 2 : 1);
  const int rc = allow_smem(kernel, bytes, set[wide], "PagedAttention");
  if (rc != DRAGON_OK) return rc;
  const int columns = a.kv_heads * ((most_rows + p.few_rows - 1) / p.few_rows);
  const long long grid = (long long)p.few_splits * columns * a.seq.count;
  if (grid > 0x7fffffffLL) { set_error("PagedAttention: too many sequences and heads"); return DRAGON_ERR_UNSUPPORTED; }
  const dim3 ctas((unsigned)grid), threads(32 * kFewWarps);
  return wide ? launch_behind(paged_few<kSteps, 2>, ctas, threads, bytes, st, "PagedAttention", a, p.most_few, columns)
              : launch_behind(paged_few<kSteps, 1>, ctas, threads, bytes, st, "PagedAttention", a, p.most_few, columns);
}

}  // namespace

cudaError_t launch_cache_write(const StepRun& r) {
  const Step& s = r.s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  WriteArgs a = {};
  const Shape &tb = r.mems[s.rd[cw::PAGES]].shape;
  const int caches = (int)s.wr.size();
  int live = 0;
  a.pages.pages = reinterpret_cast<const int*>(r.rd(cw::PAGES));
  a.pages.lengths = reinterpret_cast<const int*>(r.rd(cw::LENGTHS));
  a.pages.most = (int)tb.d[1];
  while ((1 << a.pages.shift) < (int)s.num[0]) ++a.pages.shift;
  for (int c = 0; c < caches; ++c) {
    const int in = cw::CACHE + 2 * c;
    if (s.wr[c] < 0) continue;
    const MemRef &m = r.mems[s.rd[in]], &rows = r.mems[s.rd[in + 1]];
    if (r.rd(in) != r.wr(c)) {      // not in place
      const cudaError_t e = cudaMemcpyAsync(r.wr(c), r.rd(in), m.bytes(), cudaMemcpyDeviceToDevice, st);
      if (e != cudaSuccess) return e;
    }
    a.rows[live] = reinterpret_cast<const uint4*>(r.rd(in + 1));
    a.cache[live] = reinterpret_cast<uint4*>(r.wr(c));
    a.vectors[live] = (int)(m.shape.d[1] * dtype_bytes(m.dtype) / 16);
    a.pool[live] = (int)(m.shape.d[0] >> a.pages.shift);
    a.seq.rows = (int)rows.shape.d[0];
    ++live;
  }
  a.seq.starts = reinterpret_cast<const int*>(r.rd(cw::STARTS));
  a.seq.count = (int)tb.d[0];
  a.seq.each = std::max(1, a.seq.rows / a.seq.count);
  a.status = r.status;
  a.status_clear = r.status_clear;
  cache_write<<<dim3((a.seq.rows + kWriteWarps - 1) / kWriteWarps, live), 32 * kWriteWarps, 0, st>>>(a);
  return cudaGetLastError();
}

int paged_launches(const Step& s, const std::vector<MemRef>& mems, int sm_count) {
  const PagedPlan p = plan_of(s, mems, sm_count);
  return p.few + p.tiles + p.join;
}
size_t paged_scratch_bytes(const Step& s, const std::vector<MemRef>& mems, int sm_count) {
  return plan_of(s, mems, sm_count).floats * sizeof(float);
}

int launch_paged_attention(const StepRun& r) {
  const std::vector<double>& n = r.s.num;
  const Shape &sh = r.mems[r.s.rd[pa::Q]].shape, &tb = r.mems[r.s.rd[pa::PAGES]].shape;
  const PagedPlan p = plan_of(r.s, r.mems, r.sm_count);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  RowArgs a = {};
  a.q = reinterpret_cast<const unsigned short*>(r.rd(pa::Q));
  a.k = reinterpret_cast<const unsigned short*>(r.rd(pa::K));
  a.v = reinterpret_cast<const unsigned short*>(r.rd(pa::V));
  a.out = r.wr(pa::Y); a.ot = r.wr_type(pa::Y);
  a.heads = (int)n[pn::HEADS]; a.kv_heads = (int)n[pn::KV_HEADS]; a.width = (int)(sh.d[1] / a.heads);
  a.causal = 1; a.window = (int)n[pn::WINDOW];
  a.scale = (float)(n[pn::SCALE] * 1.4426950408889634);
  a.seq.rows = (int)sh.d[0]; a.seq.count = (int)tb.d[0];
  a.seq.starts = reinterpret_cast<const int*>(r.rd(pa::STARTS));
  a.seq.each = a.seq.rows / a.seq.count;
  a.pages.pages = reinterpret_cast<const int*>(r.rd(pa::PAGES));
  a.pages.lengths = reinterpret_cast<const int*>(r.rd(pa::LENGTHS));
  a.pages.most = (int)tb.d[1];
  while ((1 << a.pages.shift) < (int)n[pn::PAGE]) ++a.pages.shift;
  a.pages.pool = (int)(r.mems[r.s.rd[pa::K]].shape.d[0] >> a.pages.shift);
  a.status = r.status;
  a.status_clear = r.status_clear;
  float* const ws = reinterpret_cast<float*>(r.ws + r.s.scratch_off);
  int rc = DRAGON_OK;
  if (p.few) {
    a.splits = p.few_splits;
    a.part_lse = ws + p.few_lse;
    a.part = ws + p.few_part;
    a.part_items = p.few_items;
    a.slots = p.slots;
    const int most_rows = std::min<int64_t>(p.most_few, a.seq.starts ? (int64_t)a.seq.rows * (a.heads / a.kv_heads) : (int64_t)a.seq.each * (a.heads / a.kv_heads));
    const int steps = (a.width + 15) / 16;
    rc = steps <= 2 ? launch_few<2>(a, p, most_rows, st) : steps <= 4 ? launch_few<4>(a, p, most_rows, st) : steps <= 6 ? launch_few<6>(a, p, most_rows, st)
                                                                                                          : launch_few<8>(a, p, most_rows, st);
  }
  if (rc == DRAGON_OK && p.tiles) {
    RowArgs t = a;
    t.splits = p.tile_splits;
    t.part_lse = ws + p.tile_lse;
    t.part = ws + p.tile_part;
    rc = launch_attention_forward(t, true, r.mems[r.s.rd[pa::K]].shape.d[0], p.most_few, r.sm_count, st, "PagedAttention");
  }
  if (rc == DRAGON_OK && p.join) {
    const bool by_sequence = a.seq.starts && p.tiles && p.tile_splits == 1;
    const int ways = std::max(p.few_splits, p.tile_splits) > 8 ? 8 : 1;
    const long long items = by_sequence ? (long long)a.seq.count * a.kv_heads * p.most_few : (long long)a.seq.rows * a.heads;
    rc = launch_behind(paged_join, dim3((unsigned)((items * ways + 7) / 8)), dim3(256), 0, st, "PagedAttention", a, (const float*)(ws + p.tile_part), (const float*)(ws + p.tile_lse), p.most_few, p.few_splits, p.tile_splits, ways, (int)by_sequence);
  }
  return rc;
}

}  // namespace dragon
