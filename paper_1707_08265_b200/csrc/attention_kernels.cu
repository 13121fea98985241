// Attention over packed sequences, forward and backward, and over a paged cache: one warp for each row of a head.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "attention_util.h"
#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

constexpr float kInf = __builtin_huge_valf();

struct RowArgs {
  const unsigned short *q, *k, *v, *dy;
  const void* y;            // backwards: the forward result
  void* out;                // y, or dq
  void *dk, *dv;
  float* lse;
  float* delta;
  int yt, ot, dkt, dvt;
  int heads, kv_heads, width, causal, window;
  float scale;              // of q k, times log2 e
  float raw_scale;
  Sequences seq;
  Pages pages;
  int* status;
  int* status_clear;
};

__device__ __forceinline__ float at(const unsigned short* p, size_t i) { return bf16_low(__ldg(p + i)); }
__device__ __forceinline__ void put(void* p, int t, size_t i, float v) { store_any<1>(p, t, i, &v); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int s = 16; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
  return v;
}

// first and last + 1 of the keys that the row at position i of its sequence (of n rows) sees
__device__ __forceinline__ void seen_by(const RowArgs& a, int i, int n, int* first, int* last) {
  *first = a.window ? max(0, i - a.window + 1) : 0;
  *last = a.causal ? i + 1 : n;
}

template <bool kPaged> __global__ void __launch_bounds__(128) row_attention(const RowArgs a) {
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    if (threadIdx.x == 0 && a.status_clear) *a.status_clear = 0;
    if (!a.seq.in_order()) report(a.status, DRAGON_ERR_INVALID_ARG);
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y, kvh = h / (a.heads / a.kv_heads);
  const int row = blockIdx.x * 4 + warp;
  if (row >= a.seq.rows) return;
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
    const float now = fmaxf(top, d), f = exp2f(top - now), p = exp2f(d - now);
    sum = sum * f + p;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = acc[e] * f + (ok && lane + 32 * e < a.width ? p * at(a.v, kb + lane + 32 * e) : 0.f);
    top = now;
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) if (a.out && lane + 32 * e < a.width) put(a.out, a.ot, base + lane + 32 * e, acc[e] * inv);
  if (a.lse && lane == 0) a.lse[(size_t)h * a.seq.rows + row] = sum > 0.f ? top + log2f(sum) : kInf;
}

// dq of a row, and delta = sum(dy y)
__global__ void __launch_bounds__(128) row_attention_dq(const RowArgs a) {
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0 && a.status_clear) *a.status_clear = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y, kvh = h / (a.heads / a.kv_heads);
  const int row = blockIdx.x * 4 + warp;
  if (row >= a.seq.rows) return;
  const int s = a.seq.of_row(row);
  const size_t base = (size_t)row * a.heads * a.width + (size_t)h * a.width;
  float q[4], d[4], dq[4] = {0.f, 0.f, 0.f, 0.f}, delta = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool in = lane + 32 * e < a.width;
    q[e] = in ? at(a.q, base + lane + 32 * e) : 0.f;
    d[e] = in ? at(a.dy, base + lane + 32 * e) : 0.f;
    float y = 0.f;
    if (in) load_any<1>(a.y, a.yt, base + lane + 32 * e, &y);
    delta += y * d[e];
  }
  delta = warp_sum(delta);
  const size_t st = (size_t)h * a.seq.rows + row;
  if (lane == 0) a.delta[st] = delta;
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
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (a.out && lane + 32 * e < a.width) put(a.out, a.ot, base + lane + 32 * e, dq[e]);
}

// dk and dv of a key row, over the heads that share it
__global__ void __launch_bounds__(128) row_attention_dkv(const RowArgs a) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, kvh = blockIdx.y, group = a.heads / a.kv_heads;
  const int row = blockIdx.x * 4 + warp;
  if (row >= a.seq.rows) return;
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
  for (int h = kvh * group; s >= 0 && h < (kvh + 1) * group; ++h)
    for (int i = i0; i < i1; ++i) {
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
    }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (lane + 32 * e < a.width) {
      if (a.dk) put(a.dk, a.dkt, kb + lane + 32 * e, dk[e]);
      if (a.dv) put(a.dv, a.dvt, kb + lane + 32 * e, dv[e]);
    }
}

int launched(const char* who) {
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) return DRAGON_OK;
  set_error("%s: launch failed: %s", who, cudaGetErrorString(e));
  return DRAGON_ERR_CUDA;
}

RowArgs row_args(const StepRun& r) {
  const std::vector<double>& n = r.s.num;
  const Shape& sh = r.mems[r.s.rd[at::Q]].shape;
  RowArgs a = {};
  a.q = reinterpret_cast<const unsigned short*>(r.rd(at::Q));
  a.k = reinterpret_cast<const unsigned short*>(r.rd(at::K));
  a.v = reinterpret_cast<const unsigned short*>(r.rd(at::V));
  a.heads = (int)n[an::HEADS]; a.kv_heads = (int)n[an::KV_HEADS]; a.width = (int)(sh.d[1] / a.heads);
  a.causal = n[an::CAUSAL] != 0.0; a.window = (int)n[an::WINDOW];
  a.raw_scale = (float)n[an::SCALE]; a.scale = (float)(n[an::SCALE] * 1.4426950408889634);
  a.seq.rows = (int)sh.d[0];
  a.seq.starts = reinterpret_cast<const int*>(r.rd(at::STARTS));
  a.seq.count = a.seq.starts ? (int)r.mems[r.s.rd[at::STARTS]].shape.d[0] - 1 : (int)n[an::SEQUENCES];
  a.seq.each = a.seq.rows / a.seq.count;
  a.status = r.status;
  a.status_clear = r.status_clear;
  return a;
}

}  // namespace

size_t attention_bwd_scratch_bytes(int64_t rows, int64_t heads) { return (size_t)(rows * heads) * sizeof(float); }
int attention_bwd_launches(const Step&) { return 2; }
int paged_launches(const Step&, const std::vector<MemRef>&) { return 1; }
size_t paged_scratch_bytes(int64_t, int64_t, int64_t, int64_t, int64_t, int) { return 0; }

int launch_attention(const StepRun& r) {
  RowArgs a = row_args(r);
  a.out = r.wr(at::Y); a.ot = r.wr_type(at::Y);
  a.lse = reinterpret_cast<float*>(r.wr(at::LSE));
  row_attention<false><<<dim3((a.seq.rows + 3) / 4, a.heads), 128, 0, reinterpret_cast<cudaStream_t>(r.stream)>>>(a);
  return launched("Attention");
}

int launch_attention_bwd(const StepRun& r) {
  RowArgs a = row_args(r);
  a.y = r.rd(at::Y_IN); a.yt = r.rd_type(at::Y_IN);
  a.lse = reinterpret_cast<float*>(r.rd(at::LSE_IN));
  a.dy = reinterpret_cast<const unsigned short*>(r.rd(at::DY));
  a.out = r.wr(at::DQ); a.ot = r.wr_type(at::DQ);
  a.dk = r.wr(at::DK); a.dkt = r.wr_type(at::DK);
  a.dv = r.wr(at::DV); a.dvt = r.wr_type(at::DV);
  a.delta = reinterpret_cast<float*>(r.ws + r.s.scratch_off);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  row_attention_dq<<<dim3((a.seq.rows + 3) / 4, a.heads), 128, 0, st>>>(a);
  row_attention_dkv<<<dim3((a.seq.rows + 3) / 4, a.kv_heads), 128, 0, st>>>(a);
  return launched("Attention's gradient");
}

int launch_paged_attention(const StepRun& r) {
  const std::vector<double>& n = r.s.num;
  const Shape &sh = r.mems[r.s.rd[pa::Q]].shape, &tb = r.mems[r.s.rd[pa::PAGES]].shape;
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
  a.pages.shift = 0;
  while ((1 << a.pages.shift) < (int)n[pn::PAGE]) ++a.pages.shift;
  a.pages.pool = (int)(r.mems[r.s.rd[pa::K]].shape.d[0] >> a.pages.shift);
  a.status = r.status;
  a.status_clear = r.status_clear;
  row_attention<true><<<dim3((a.seq.rows + 3) / 4, a.heads), 128, 0, reinterpret_cast<cudaStream_t>(r.stream)>>>(a);
  return launched("PagedAttention");
}

}  // namespace dragon
