// Attention one row at a time: a warp computes a row of a head from the keys it sees and nothing else.  The tensor-core kernels
// multiply whole tiles, so that a masked key's infinities and NaN reach a row as 0 x inf; a row whose result is not finite is
// computed again here, which gives what the formula gives.  (Where everything is NaN, as in a training run that has come apart, it
// ends at the first key.)
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

// y and lse of a row
template <bool kPaged> __device__ __noinline__ void attend_row(const RowArgs& a, int h, int row, int lane) {
  const int kvh = h / (a.heads / a.kv_heads);
  const int s = a.seq.of_row(row);
  const size_t base = (size_t)row * a.heads * a.width + (size_t)h * a.width;
  float q[4], acc[4] = {0.f, 0.f, 0.f, 0.f}, top = -kInf, sum = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) q[e] = lane + 32 * e < a.width ? at(a.q, base + lane + 32 * e) : 0.f;
  int first = 0, last = 0, r0 = 0;
  if (s >= 0) {
    int r1;
    a.seq.rows_of(s, &r0, &r1);
    if (kPaged) {
      bool fits;
      const int tokens = a.pages.tokens(s, &fits);
      if (!fits) report(a.status, DRAGON_ERR_INVALID_ARG);
      const int p = tokens - (r1 - r0) + (row - r0);
      if (p >= 0) { last = p + 1; first = a.window ? max(0, p - a.window + 1) : 0; }
    } else {
      seen_by(a, row - r0, r1 - r0, &first, &last);
    }
  }
  for (int j = first; j < last; ++j) {
    size_t kr;
    bool ok = true;
    if (kPaged) {
      const int page = a.pages.page_of(s, j);
      ok = a.pages.in_pool(page);
      if (!ok) report(a.status, DRAGON_ERR_INVALID_ARG);
      kr = ((size_t)page << a.pages.shift) + (j & ((1 << a.pages.shift) - 1));
    } else {
      kr = (size_t)(r0 + j);
    }
    const size_t kb = kr * a.kv_heads * a.width + (size_t)kvh * a.width;
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) if (ok && lane + 32 * e < a.width) d += q[e] * at(a.k, kb + lane + 32 * e);
    d = warp_sum(d) * a.scale;
    const float now = fmaxf(top, d), shift = now == -kInf ? 0.f : now, f = exp2f(top - shift), p = exp2f(d - shift);
    sum = sum * f + p;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = acc[e] * f + (ok && lane + 32 * e < a.width ? p * at(a.v, kb + lane + 32 * e) : 0.f);
    top = now;
    if (sum != sum) break;      // NaN from here on whatever follows
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (a NaN stays one)
#pragma unroll
  for (int e = 0; e < 4; ++e) if (a.out && lane + 32 * e < a.width) put(a.out, a.ot, base + lane + 32 * e, acc[e] * inv);
#pragma unroll
  for (int e = 0; e < 4; ++e) if (a.rest && lane + 32 * e < a.width) put(a.rest, DRAGON_BF16, base + lane + 32 * e, behind_bf16(acc[e] * inv));
  if (a.lse && lane == 0) a.lse[(size_t)h * a.seq.rows + row] = sum == 0.f ? kInf : top + log2f(sum);
}

// dq of a row
__device__ __noinline__ void dq_of_row(const RowArgs& a, int h, int row, int lane) {
  const int kvh = h / (a.heads / a.kv_heads);
  const int s = a.seq.of_row(row);
  const size_t base = (size_t)row * a.heads * a.width + (size_t)h * a.width;
  float q[4], d[4], dq[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool in = lane + 32 * e < a.width;
    q[e] = in ? at(a.q, base + lane + 32 * e) : 0.f;
    d[e] = in ? at(a.dy, base + lane + 32 * e) : 0.f;
  }
  const size_t st = (size_t)h * a.seq.rows + row;
  const float delta = a.delta[st];
  int first = 0, last = 0, r0 = 0, r1 = 0;
  if (s >= 0) { a.seq.rows_of(s, &r0, &r1); seen_by(a, row - r0, r1 - r0, &first, &last); }
  const float lse = a.lse[st];
  for (int j = first; j < last; ++j) {
    const size_t kb = (size_t)(r0 + j) * a.kv_heads * a.width + (size_t)kvh * a.width;
    float x = 0.f, dp = 0.f, k[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool in = lane + 32 * e < a.width;
      k[e] = in ? at(a.k, kb + lane + 32 * e) : 0.f;
      x += q[e] * k[e];
      if (in) dp += d[e] * at(a.v, kb + lane + 32 * e);
    }
    const float p = exp2f(warp_sum(x) * a.scale - lse), ds = p * (warp_sum(dp) - delta) * a.raw_scale;
#pragma unroll
    for (int e = 0; e < 4; ++e) dq[e] += ds * k[e];
    if (ds != ds) break;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (a.out && lane + 32 * e < a.width) put(a.out, a.ot, base + lane + 32 * e, dq[e]);
}

// dk and dv of a key row, over the heads that share it
__device__ __noinline__ void dkv_of_row(const RowArgs& a, int kvh, int row, int lane) {
  const int group = a.heads / a.kv_heads;
  const int s = a.seq.of_row(row);
  const size_t kb = (size_t)row * a.kv_heads * a.width + (size_t)kvh * a.width;
  float k[4], v[4], dk[4] = {0.f, 0.f, 0.f, 0.f}, dv[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool in = lane + 32 * e < a.width;
    k[e] = in ? at(a.k, kb + lane + 32 * e) : 0.f;
    v[e] = in ? at(a.v, kb + lane + 32 * e) : 0.f;
  }
  int r0 = 0, r1 = 0;
  if (s >= 0) a.seq.rows_of(s, &r0, &r1);
  const int j = row - r0, n = r1 - r0, i0 = a.causal ? j : 0, i1 = a.window ? min(n, j + a.window) : n;
  bool open = s >= 0;      // until everything is NaN
  for (int h = kvh * group; open && h < (kvh + 1) * group; ++h)
    for (int i = i0; open && i < i1; ++i) {
      const size_t base = (size_t)(r0 + i) * a.heads * a.width + (size_t)h * a.width, st = (size_t)h * a.seq.rows + r0 + i;
      float x = 0.f, dp = 0.f, q[4], d[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = lane + 32 * e < a.width;
        q[e] = in ? at(a.q, base + lane + 32 * e) : 0.f;
        d[e] = in ? at(a.dy, base + lane + 32 * e) : 0.f;
        x += q[e] * k[e];
        dp += d[e] * v[e];
      }
      const float p = exp2f(warp_sum(x) * a.scale - a.lse[st]), ds = p * (warp_sum(dp) - a.delta[st]) * a.raw_scale;
#pragma unroll
      for (int e = 0; e < 4; ++e) { dk[e] += ds * q[e]; dv[e] += p * d[e]; }
      open = p == p;
    }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (lane + 32 * e < a.width) {
      if (a.dk) put(a.dk, a.dkt, kb + lane + 32 * e, dk[e]);
      if (a.dv) put(a.dv, a.dvt, kb + lane + 32 * e, dv[e]);
    }
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
