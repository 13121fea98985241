// Attention one row at a time: a warp computes a row of a head from the keys it sees and nothing else.  The tensor-core kernels
// multiply whole tiles, so that a masked key's infinities and NaN reach a row as 0 x inf; a row whose result is not finite is
// computed again here, which gives what the formula gives.  Where all is finite among what its tiles held and it does not see, a few
// hundred rows beside those that it sees, the tiles' result, which is in place already, is the formula's and stays.  (Where everything is
// NaN, as in a training run that has come apart, a row ends at the first key.)
#pragma once
#include <cuda_runtime.h>

#include "attention_util.h"
#include "device_util.h"
#include "plan.h"

namespace dragon {

constexpr float kInf = __builtin_huge_valf();

struct RowArgs {
  const unsigned short *q, *k, *v, *dy;
  const void* y;            // backwards: the forward result
  void* out;                // y, or dq
  void *dk, *dv;
  unsigned short* rest;     // what y's rounding to bf16 left out (nullptr: not wanted)
  float* lse;
  float* delta;
  int yt, ot, dkt, dvt;
  int heads, kv_heads, width, causal, window;
  float scale;              // of q k, times log2 e
  float raw_scale;
  Sequences seq;
  Pages pages;
  // what a CTA meets split over `splits` CTAs.  Forwards: every part's result and the log2 of its sum (-inf: no keys), [split][row][head];
  // backwards: every part's dq, and with key_splits dk and dv, which are added up
  int splits, key_splits;
  float *part, *part_lse, *part_k, *part_v;
  // PagedAttention's few rows: results of a split, and where slots is not 0 so many of every sequence and key head (new row x group +
  // head of the group) instead of [row][head]: with starts there may be many rows, of which only those of short sequences have parts
  long long part_items;
  int slots;
  int* status;
  int* status_clear;
};

namespace {

__device__ __forceinline__ float at(const unsigned short* p, size_t i) { return bf16_low(__ldg(p + i)); }
__device__ __forceinline__ void put(void* p, int t, size_t i, float v) { store_any<1>(p, t, i, &v); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int s = 16; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
  return v;
}

// what rounding to bf16 leaves out of v
__device__ __forceinline__ float behind_bf16(float v) { return v - __bfloat162float(__float2bfloat16_rn(v)); }

// first and last + 1 of the keys that the row at position i of its sequence (of n rows) sees
__device__ __forceinline__ void seen_by(const RowArgs& a, int i, int n, int* first, int* last) {
  *first = a.window ? max(0, i - a.window + 1) : 0;
  *last = a.causal ? i + 1 : n;
}

// x . y over the head, both in memory and 16-byte aligned (width: a multiple of 8).  kAtOnce, here and below: how far loops are unrolled, that
// their loads are on their way together
template <int kAtOnce> __device__ __forceinline__ float dot_of(const unsigned short* x, const unsigned short* y, int width) {
  float d[2] = {0.f, 0.f};
#pragma unroll kAtOnce
  for (int c = 0; c < width; c += 8) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(x + c)), w = __ldg(reinterpret_cast<const uint4*>(y + c));
    d[0] += bf16_low(u.x) * bf16_low(w.x) + bf16_low(u.y) * bf16_low(w.y) + bf16_low(u.z) * bf16_low(w.z) + bf16_low(u.w) * bf16_low(w.w);
    d[1] += bf16_high(u.x) * bf16_high(w.x) + bf16_high(u.y) * bf16_high(w.y) + bf16_high(u.z) * bf16_high(w.z) + bf16_high(u.w) * bf16_high(w.w);
  }
  return d[0] + d[1];
}
// A lane's elements of a head: 4 lane .. 4 lane + 3 (none where that is behind the width).  out += factor * a row in memory
__device__ __forceinline__ void add_row(float* out, float factor, const unsigned short* row, int width, int lane) {
  if (4 * lane >= width) return;
  const uint2 u = __ldg(reinterpret_cast<const uint2*>(row + 4 * lane));
  out[0] += factor * bf16_low(u.x);
  out[1] += factor * bf16_high(u.x);
  out[2] += factor * bf16_low(u.y);
  out[3] += factor * bf16_high(u.y);
}
__device__ __forceinline__ void put_row(void* p, int t, size_t base, const float* v, int width, int lane) {
  if (4 * lane >= width) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) put(p, t, base + 4 * lane + e, v[e]);
}
// whether this lane's elements of a row are all NaN: no more that is added changes them
__device__ __forceinline__ bool all_nan(const float* v, int width, int lane) {
  return 4 * lane >= width || (v[0] != v[0] && v[1] != v[1] && v[2] != v[2] && v[3] != v[3]);
}
__device__ __forceinline__ bool nan_in_memory(const void* p, int t, size_t base, int width, int lane) {      // a row; a warp
  bool all = true;
  for (int c = lane; c < width; c += 32) {
    const float v = t == DRAGON_F32 ? reinterpret_cast<const float*>(p)[base + c] : bf16_low(reinterpret_cast<const unsigned short*>(p)[base + c]);
    all &= v != v;
  }
  return __all_sync(0xffffffffu, all);
}

// f(0) .. f(n - 1)
template <int kAtOnce, typename F> __device__ __forceinline__ void for_each_of(int n, F f) {
  if (n == 32) {
#pragma unroll kAtOnce
    for (int k = 0; k < 32; ++k) f(k);
  } else {
#pragma unroll 1
    for (int k = 0; k < n; ++k) f(k);
  }
}

// whether a head's elements in memory (16-byte aligned) are all below a limit in magnitude, given as the upper bits of it
constexpr uint32_t kFinite = 0x7f80, kTame = (127 + 56) << 7;      // infinity; 2^56: 0 times one below it is 0, and so is 0 times a product of two heads
template <int kAtOnce> __device__ __forceinline__ bool below(const unsigned short* x, int width, uint32_t limit) {
  bool fine = true;
#pragma unroll kAtOnce
  for (int c = 0; c < width; c += 8) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(x + c));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) fine &= (w[i] & 0x7fffu) < limit && (w[i] >> 16 & 0x7fffu) < limit;
  }
  return fine;
}
// Rows that a tile may have held beside those that a row sees: of 256 neighbouring rows and of the 128 keys of a tile, forwards; of 128 and 128
// backwards
constexpr int kBesideForward = 384, kBesideBackward = 256;
// Whether the tiles' result of a row that sees the rows [first, last) is the formula's although it is not finite: of those beside them, from `from`
// on and before `to`, none is so large that 0 times it may not be 0, and it is NaN throughout or one of those that the row sees is not
// finite (otherwise a sum of finite values has left fp32's range, where the row by itself may stay within it).  fine(i, limit): row i; a warp
template <typename F> __device__ __forceinline__ bool result_stands(int first, int last, int from, int to, int beside, bool nan, int lane, F fine) {
  bool ok = true;
  for (int i = max(from, first - beside) + lane; i < first; i += 32) ok &= fine(i, kTame);
  for (int i = last + lane; i < min((long long)to, (long long)last + beside); i += 32) ok &= fine(i, kTame);
  if (!__all_sync(0xffffffffu, ok)) return false;
  if (nan) return true;
  for (int i = first; i < last; i += 32)
    if (__any_sync(0xffffffffu, i + lane < last && !fine(min(i + lane, last - 1), kFinite))) return true;
  return false;
}

// Each of the three meets 32 rows at a time: a lane's score is that of one of them, and then the lanes share out the head's elements.
// (16384 rows, 8 heads on 2 of 128 with gradients, 1.8 ms where all is finite: an infinity in the first value 1374 ms when a row met its keys one
// by one and wherever its result was not finite, 4.4 now; in the last gradient 1144 and 155; in a whole column of values 91.)

// y and lse of a row, where its tiles' result (in place by now) may be something else
template <bool kPaged> __device__ __noinline__ void attend_row(const RowArgs& a, int h, int row, int lane) {
  // (unrolled here, these loops made a decoding step's kernel, which hardly ever comes here, 1 us longer: 8.4 us -> 9.8 for 3 sequences of 200)
  constexpr int kAtOnce = kPaged ? 1 : 8;
  const int kvh = h / (a.heads / a.kv_heads);
  const int s = a.seq.of_row(row);
  const size_t base = (size_t)row * a.heads * a.width + (size_t)h * a.width;
  float acc[4] = {0.f, 0.f, 0.f, 0.f}, top = -kInf, sum = 0.f;
  int first = 0, last = 0, r0 = 0, there = 0;      // there: keys of the sequence
  if (s >= 0) {
    int r1;
    a.seq.rows_of(s, &r0, &r1);
    if (kPaged) {
      bool fits;
      const int tokens = a.pages.tokens(s, &fits);
      if (!fits) report(a.status, DRAGON_ERR_INVALID_ARG);
      there = tokens;
      const int p = tokens - (r1 - r0) + (row - r0);
      if (p >= 0) { last = p + 1; first = a.window ? max(0, p - a.window + 1) : 0; }
    } else {
      there = r1 - r0;
      seen_by(a, row - r0, r1 - r0, &first, &last);
    }
  }
  const size_t pitch = (size_t)a.kv_heads * a.width, column = (size_t)kvh * a.width;
  if (result_stands(first, last, 0, there, kBesideForward, a.out && nan_in_memory(a.out, a.ot, base, a.width, lane), lane, [&](int j, uint32_t limit) {
        int kr = r0 + j;
        if (kPaged) {
          const int page = a.pages.page_of(s, j);
          if (!a.pages.in_pool(page)) return true;
          kr = (page << a.pages.shift) + (j & ((1 << a.pages.shift) - 1));
        }
        return below<kAtOnce>(a.v + kr * pitch + column, a.width, limit);
      })) return;
  for (int j0 = first; j0 < last; j0 += 32) {
    const int j = j0 + min(lane, last - j0 - 1), n = min(32, last - j0);
    int kr = r0 + j;      // -1: a page of none, whose keys and values are zeros
    if (kPaged) {
      const int page = a.pages.page_of(s, j);
      kr = a.pages.in_pool(page) ? (page << a.pages.shift) + (j & ((1 << a.pages.shift) - 1)) : -1;
      if (kr < 0) report(a.status, DRAGON_ERR_INVALID_ARG);
    }
    const float d = kr < 0 ? 0.f : dot_of<kAtOnce>(a.q + base, a.k + kr * pitch + column, a.width) * a.scale;
    float now = fmaxf(top, d);
#pragma unroll
    for (int k = 16; k; k >>= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, k));
    const float shift = now == -kInf ? 0.f : now, f = exp2f(top - shift), p = lane < n ? exp2f(d - shift) : 0.f;
    sum = sum * f + warp_sum(p);
    top = now;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= f;
    for_each_of<kAtOnce>(n, [&](int k) {
      const float pk = __shfl_sync(0xffffffffu, p, k);
      const int from = __shfl_sync(0xffffffffu, kr, k);
      if (!kPaged || from >= 0) add_row(acc, pk, a.v + from * pitch + column, a.width, lane);
    });
    if (sum != sum) break;      // NaN from here on whatever follows
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (a NaN stays one)
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] *= inv;
  if (a.out) put_row(a.out, a.ot, base, acc, a.width, lane);
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = behind_bf16(acc[e]);
  if (a.rest) put_row(a.rest, DRAGON_BF16, base, acc, a.width, lane);
  if (a.lse && lane == 0) a.lse[(size_t)h * a.seq.rows + row] = sum == 0.f ? kInf : top + log2f(sum);
}

// dq of a row, likewise.  A delta or dy of its own that is not finite makes the zeros of keys that it does not see NaN
__device__ __noinline__ void dq_of_row(const RowArgs& a, int h, int row, int lane) {
  const int kvh = h / (a.heads / a.kv_heads);
  const int s = a.seq.of_row(row);
  const size_t base = (size_t)row * a.heads * a.width + (size_t)h * a.width, pitch = (size_t)a.kv_heads * a.width, column = (size_t)kvh * a.width;
  float dq[4] = {0.f, 0.f, 0.f, 0.f};
  const size_t st = (size_t)h * a.seq.rows + row;
  const float delta = a.delta[st], lse = a.lse[st];
  int first = 0, last = 0, r0 = 0, r1 = 0;
  if (s >= 0) { a.seq.rows_of(s, &r0, &r1); seen_by(a, row - r0, r1 - r0, &first, &last); }
  // (behind the sequence's last key other rows may stand in the tile)
  if (fabsf(delta) < 0x1p126f && below<8>(a.dy + base, a.width, kTame) && result_stands(first, last, 0, a.seq.rows - r0, kBesideBackward, nan_in_memory(a.out, a.ot, base, a.width, lane), lane, [&](int j, uint32_t limit) {
        return below<8>(a.k + (size_t)(r0 + j) * pitch + column, a.width, limit) && below<8>(a.v + (size_t)(r0 + j) * pitch + column, a.width, limit);
      })) return;
  for (int j0 = first; j0 < last; j0 += 32) {
    const int n = min(32, last - j0);
    const size_t kb = (size_t)(r0 + j0 + min(lane, n - 1)) * pitch + column;
    const float p = exp2f(dot_of<8>(a.q + base, a.k + kb, a.width) * a.scale - lse), ds = p * (dot_of<8>(a.dy + base, a.v + kb, a.width) - delta) * a.raw_scale;
    for_each_of<8>(n, [&](int k) { add_row(dq, __shfl_sync(0xffffffffu, ds, k), a.k + (size_t)(r0 + j0 + k) * pitch + column, a.width, lane); });
    if (__all_sync(0xffffffffu, all_nan(dq, a.width, lane))) break;
  }
  if (a.out) put_row(a.out, a.ot, base, dq, a.width, lane);
}

// dk and dv of a key row (those that are wanted), over the heads that share it, likewise.  A row of its own that is not finite makes the zeros of rows that do not
// see it NaN
__device__ __noinline__ void dkv_of_row(const RowArgs& a, int kvh, int row, int lane, bool want_k, bool want_v) {
  const int group = a.heads / a.kv_heads;
  const int s = a.seq.of_row(row);
  const size_t kb = (size_t)row * a.kv_heads * a.width + (size_t)kvh * a.width;
  float dk[4] = {0.f, 0.f, 0.f, 0.f}, dv[4] = {0.f, 0.f, 0.f, 0.f};
  int r0 = 0, r1 = 0;
  if (s >= 0) a.seq.rows_of(s, &r0, &r1);
  const int j = row - r0, n = r1 - r0, i0 = a.causal ? j : 0, i1 = a.window ? min(n, j + a.window) : n;
  const bool nan = (!want_k || nan_in_memory(a.dk, a.dkt, kb, a.width, lane)) && (!want_v || nan_in_memory(a.dv, a.dvt, kb, a.width, lane));
  if (below<8>(a.k + kb, a.width, kTame) && below<8>(a.v + kb, a.width, kTame) && result_stands(i0, max(i0, i1), 0, a.seq.rows - r0, kBesideBackward, nan, lane, [&](int i, uint32_t limit) {
        bool fine = true;
        for (int h = kvh * group; fine && h < (kvh + 1) * group; ++h) {
          const size_t at = ((size_t)(r0 + i) * a.heads + h) * a.width;
          fine = fabsf(a.delta[(size_t)h * a.seq.rows + r0 + i]) < (limit == kTame ? 0x1p126f : kInf) && below<8>(a.q + at, a.width, limit) && below<8>(a.dy + at, a.width, limit);
        }
        return fine;
      })) return;
  bool open = s >= 0;      // until everything is NaN
  for (int h = kvh * group; open && h < (kvh + 1) * group; ++h)
    for (int i = i0; open && i < i1; i += 32) {
      const int here = min(32, i1 - i);
      const size_t first = ((size_t)(r0 + i) * a.heads + h) * a.width, pitch = (size_t)a.heads * a.width, mine = first + min(lane, here - 1) * pitch;
      const size_t st = (size_t)h * a.seq.rows + r0 + i + min(lane, here - 1);
      const float p = exp2f(dot_of<8>(a.q + mine, a.k + kb, a.width) * a.scale - a.lse[st]), ds = p * (dot_of<8>(a.dy + mine, a.v + kb, a.width) - a.delta[st]) * a.raw_scale;
      for_each_of<8>(here, [&](int k) {
        if (want_k) add_row(dk, __shfl_sync(0xffffffffu, ds, k), a.q + first + k * pitch, a.width, lane);
        if (want_v) add_row(dv, __shfl_sync(0xffffffffu, p, k), a.dy + first + k * pitch, a.width, lane);
      });
      open = !__all_sync(0xffffffffu, (!want_k || all_nan(dk, a.width, lane)) && (!want_v || all_nan(dv, a.width, lane)));
    }
  if (want_k) put_row(a.dk, a.dkt, kb, dk, a.width, lane);
  if (want_v) put_row(a.dv, a.dvt, kb, dv, a.width, lane);
}

// Launches of one operator behind one another: a kernel's CTAs may be there, and prepare what needs no results, before the launch in
// front has ended (a launch of 2 to 3 us is hidden that way).  Each launch lets the next one come as soon as all of its CTAs run,
// and each thread waits for the end of the launch before (which has waited for the one before it) ahead of its first access to memory
// that a kernel writes.
__device__ __forceinline__ void next_launch_may_come() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void after_the_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

int launched(const char* who) {
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) return DRAGON_OK;
  set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
  return DRAGON_ERR_CUDA;
}

template <typename... P, typename... A> int launch_behind(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const char* who, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  if (e == cudaSuccess) return launched(who);
  cudaGetLastError();
  set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
  return DRAGON_ERR_CUDA;
}

}  // namespace
}  // namespace dragon
