// Attention's steps of the plan: their operands for the kernels.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "attention_rows.h"

namespace dragon {
int launch_attention_forward(const RowArgs& rows, bool paged, int64_t key_rows, int few, int sm_count, cudaStream_t st, const char* who);
int launch_attention_backward(const RowArgs& rows, cudaStream_t st);
int64_t attention_units(int64_t rows, int64_t sequences, int heads, int kv_heads);
void attention_bwd_units(int64_t rows, int64_t sequences, int heads, int kv_heads, int64_t* row_units, int64_t* key_units, int* tile_rows);
namespace {

// Into how many parts a CTA's work is split: what takes the least time by a model in cycles, of a CTA's fixed costs, of a pair of tiles,
// and of what putting the parts together costs.  A sequence's length is on the device where there are starts: the average stands
// for it (whatever the lengths, the result is the same).  A causal block of rows sees half of what the last one sees, on average.  The
// cycles are those of two tiles a CTA and heads of 128 and stand for the other forms too (one tile a CTA, narrower heads), whose rounds
// and fixed costs are smaller alike.
// One sequence of 12909 rows and one head forwards: 239 us in one part, 77 in more; 12 heads of 7 sequences of 148 rows with
// gradients: 37 us in one part, 51 in the two that would fill the GPU.
struct AttentionPlan { int fwd, rows, keys; };
constexpr int kMostParts = 16;
constexpr double kFwdPair = 3200, kKeysPair = 3245, kRowsPair = 2288, kFwdFixed = 14000, kBwdFixed = 9000, kJoinFixed = 14000, kBytesACycle = 3400;
AttentionPlan plan_of(const Step& s, const std::vector<MemRef>& mems, int sm_count) {
  const Shape& sh = mems[s.rd[at::Q]].shape;
  const std::vector<double>& n = s.num;
  const bool starts = s.rd[at::STARTS] >= 0;
  const int64_t rows = sh.d[0], count = starts ? mems[s.rd[at::STARTS]].shape.d[0] - 1 : (int64_t)n[an::SEQUENCES];
  const int heads = (int)n[an::HEADS], kv = (int)n[an::KV_HEADS];
  const int64_t window = (int64_t)n[an::WINDOW], each = std::max<int64_t>(1, rows / std::max<int64_t>(1, count));
  const double falling = n[an::CAUSAL] != 0.0 && !window ? 0.5 : 1.0, row_bytes = (double)rows * sh.d[1] * 2 * sizeof(float);      // of a part, written and read
  AttentionPlan p = {1, 1, 1};
  double best = 0;
  auto better = [&](double t) { const bool is = best == 0 || t < best; if (is) best = t; return is; };
  if (s.kind == ST_ATTN) {
    const int64_t units = attention_units(rows, count, heads, kv), pairs = ((window ? std::min(each, window + 256) : each) + 127) / 128;
    for (int64_t k = 1; k <= std::min<int64_t>(pairs, kMostParts); ++k) {
      const double share = units * (pairs * kFwdPair * falling + k * kFwdFixed) / sm_count, longest = kFwdFixed + (pairs + k - 1) / k * kFwdPair;
      if (better(std::max(share, longest) + (k > 1 ? kJoinFixed + k * row_bytes / kBytesACycle : 0))) p.fwd = (int)k;
    }
    return p;
  }
  int64_t row_units, key_units;
  int tile_rows;
  attention_bwd_units(rows, count, heads, kv, &row_units, &key_units, &tile_rows);
  const int64_t met = window ? std::min(each, window + 128) : each, by_key = (met + tile_rows - 1) / tile_rows * (heads / kv) * tile_rows / 128, by_row = (met + 127) / 128;
  for (int64_t k = 1; k <= std::min<int64_t>(by_key, kMostParts); ++k)
    for (int64_t r = 1; r <= std::min<int64_t>(by_row, kMostParts); ++r) {
      const double share = (key_units * (by_key * kKeysPair * falling + k * kBwdFixed) + row_units * (by_row * kRowsPair * falling + r * kBwdFixed)) / sm_count;
      const double longest = kBwdFixed + std::max((by_key + k - 1) / k * kKeysPair, (by_row + r - 1) / r * kRowsPair);
      const double parts = ((r > 1 ? (double)r : 0) + (k > 1 ? 2.0 * k * kv / heads : 0)) * row_bytes / kBytesACycle;
      if (better(std::max(share, longest) + (k > 1 || r > 1 ? kJoinFixed : 0) + parts)) { p.keys = (int)k; p.rows = (int)r; }
    }
  return p;
}
size_t delta_floats(int64_t rows, int64_t heads) { return (size_t)((rows * heads + 63) & ~(int64_t)63); }

// The parts of every row and head put together: a warp each, 4 elements a lane, in the order of the parts
__global__ void __launch_bounds__(256) attention_join(const __grid_constant__ RowArgs a) {
  after_the_launch_before();
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), items = (long long)a.seq.rows * a.heads;
  if (item >= items) return;
  const int row = (int)(item / a.heads), head = (int)(item % a.heads);
  if (a.seq.of_row(row) < 0) return;      // written already
  float most = -kInf;
  for (int p = 0; p < a.splits; ++p) most = fmaxf(most, a.part_lse[p * items + item]);
  const float shift = most == -kInf ? 0.f : most;
  float total = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
  const bool in = 4 * lane < a.width;
#pragma unroll 4
  for (int p = 0; p < a.splits; ++p) {
    const float l = a.part_lse[p * items + item], w = exp2f(l - shift);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);      // (no keys: nothing was written)
    if (in && l != -kInf) x = *reinterpret_cast<const float4*>(a.part + (p * items + item) * a.width + 4 * lane);
    total += w;
    v[0] += w * x.x; v[1] += w * x.y; v[2] += w * x.z; v[3] += w * x.w;
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  bool fine = fabsf(total) < kInf;
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[e] *= inv; fine &= fabsf(v[e]) < kInf; }
  if (a.lse && lane == 0) a.lse[(size_t)head * a.seq.rows + row] = total == 0.f ? kInf : shift + log2f(total);
  const size_t at = item * a.width + 4 * lane;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (a.out && in) put(a.out, a.ot, at + e, v[e]);
    if (a.rest && in) put(a.rest, DRAGON_BF16, at + e, behind_bf16(v[e]));
  }
  if (!__all_sync(0xffffffffu, fine)) {
    __syncwarp();
    attend_row<false>(a, head, row, lane);
  }
}

// The parts of the gradients added up: the first dq_items are rows of dq, the others rows of dk and dv
__global__ void __launch_bounds__(256) attention_bwd_join(const __grid_constant__ RowArgs a, long long dq_items, long long items) {
  after_the_launch_before();
  const int lane = threadIdx.x & 31;
  long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (item >= items) return;
  const bool keys = item >= dq_items;
  if (keys) item -= dq_items;
  const int heads = keys ? a.kv_heads : a.heads, row = (int)(item / heads), head = (int)(item % heads);
  if (a.seq.of_row(row) < 0) return;      // written already
  const size_t at = item * a.width + 4 * lane, stride = (size_t)a.seq.rows * heads * a.width;
  const bool in = 4 * lane < a.width;
  auto sum = [&](const float* part, int parts, float* v) {
    v[0] = v[1] = v[2] = v[3] = 0.f;
#pragma unroll 4
    for (int p = 0; p < parts && in; ++p) {
      const float4 x = *reinterpret_cast<const float4*>(part + p * stride + at);
      v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
    }
    return fabsf(v[0]) < kInf && fabsf(v[1]) < kInf && fabsf(v[2]) < kInf && fabsf(v[3]) < kInf;
  };
  float v[4], w[4];
  const bool fine = __all_sync(0xffffffffu, !keys ? sum(a.part, a.splits, v) : !a.dk || sum(a.part_k, a.key_splits, v));
  const bool fine_v = __all_sync(0xffffffffu, !keys || !a.dv || sum(a.part_v, a.key_splits, w));
#pragma unroll
  for (int e = 0; e < 4 && in; ++e) {
    if (!keys) put(a.out, a.ot, at + e, v[e]);
    if (keys && a.dk) put(a.dk, a.dkt, at + e, v[e]);
    if (keys && a.dv) put(a.dv, a.dvt, at + e, w[e]);
  }
  __syncwarp();
  if (keys && !(fine && fine_v)) dkv_of_row(a, head, row, lane, !fine, !fine_v);
  else if (!fine) dq_of_row(a, head, row, lane);
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
  a.splits = 1;
  a.status = r.status;
  a.status_clear = r.status_clear;
  return a;
}

}  // namespace

size_t attention_scratch_bytes(const Step& s, const std::vector<MemRef>& mems, int sm_count) {
  const Shape& sh = mems[s.rd[at::Q]].shape;
  const AttentionPlan p = plan_of(s, mems, sm_count);
  const size_t rows = (size_t)sh.d[0], heads = (size_t)s.num[an::HEADS], kv = (size_t)s.num[an::KV_HEADS], width = (size_t)sh.d[1] / heads;
  if (s.kind == ST_ATTN) return p.fwd > 1 ? p.fwd * rows * heads * (width + 1) * sizeof(float) : 0;
  return (delta_floats(rows, heads) + (p.rows > 1 ? p.rows * rows * heads * width : 0) + (p.keys > 1 ? 2 * p.keys * rows * kv * width : 0)) * sizeof(float);
}
int attention_launches(const Step& s, const std::vector<MemRef>& mems, int sm_count) {
  const AttentionPlan p = plan_of(s, mems, sm_count);
  if (s.kind == ST_ATTN) return 1 + (p.fwd > 1);
  const bool rows = s.wr[at::DQ] >= 0, keys = s.wr[at::DK] >= 0 || s.wr[at::DV] >= 0;
  return 2 + ((p.rows > 1 && rows) || (p.keys > 1 && keys));
}

int launch_attention(const StepRun& r) {
  RowArgs a = row_args(r);
  a.out = r.wr(at::Y); a.ot = r.wr_type(at::Y);
  a.lse = reinterpret_cast<float*>(r.wr(at::LSE));
  a.splits = plan_of(r.s, r.mems, r.sm_count).fwd;
  a.part = reinterpret_cast<float*>(r.ws + r.s.scratch_off);
  a.part_lse = a.part + (size_t)a.splits * a.seq.rows * a.heads * a.width;
  if (r.s.wr.size() > at::REST) a.rest = reinterpret_cast<unsigned short*>(r.wr(at::REST));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const int rc = launch_attention_forward(a, false, a.seq.rows, 0, r.sm_count, st, "Attention");
  if (rc != DRAGON_OK || a.splits == 1) return rc;
  const long long items = (long long)a.seq.rows * a.heads;
  return launch_behind(attention_join, dim3((unsigned)((items + 7) / 8)), dim3(256), 0, st, "Attention", a);
}

int launch_attention_bwd(const StepRun& r) {
  RowArgs a = row_args(r);
  a.y = r.rd(at::Y_IN); a.yt = r.rd_type(at::Y_IN);
  a.lse = reinterpret_cast<float*>(r.rd(at::LSE_IN));
  a.rest = reinterpret_cast<unsigned short*>(r.rd(at::REST_IN));
  a.dy = reinterpret_cast<const unsigned short*>(r.rd(at::DY));
  a.out = r.wr(at::DQ); a.ot = r.wr_type(at::DQ);
  a.dk = r.wr(at::DK); a.dkt = r.wr_type(at::DK);
  a.dv = r.wr(at::DV); a.dvt = r.wr_type(at::DV);
  a.delta = reinterpret_cast<float*>(r.ws + r.s.scratch_off);
  const AttentionPlan p = plan_of(r.s, r.mems, r.sm_count);
  a.splits = p.rows;
  a.key_splits = p.keys;
  a.part = a.delta + delta_floats(a.seq.rows, a.heads);
  a.part_k = a.part + (p.rows > 1 ? (size_t)p.rows * a.seq.rows * a.heads * a.width : 0);
  a.part_v = a.part_k + (p.keys > 1 ? (size_t)p.keys * a.seq.rows * a.kv_heads * a.width : 0);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const int rc = launch_attention_backward(a, st);
  const bool rows = p.rows > 1 && a.out, keys = p.keys > 1 && (a.dk || a.dv);
  if (rc != DRAGON_OK || (!rows && !keys)) return rc;
  const long long items = (long long)a.seq.rows * ((rows ? a.heads : 0) + (keys ? a.kv_heads : 0));
  return launch_behind(attention_bwd_join, dim3((unsigned)((items + 7) / 8)), dim3(256), 0, st, "Attention's gradient", a, rows ? (long long)a.seq.rows * a.heads : 0LL, items);
}

}  // namespace dragon
