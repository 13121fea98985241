// Attention's steps of the plan: their operands for the kernels.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "attention_rows.h"

namespace dragon {
int launch_attention_forward(const RowArgs& rows, bool paged, int64_t key_rows, int few, cudaStream_t st, const char* who);
int launch_attention_backward(const RowArgs& rows, cudaStream_t st);
namespace {

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

int launch_attention(const StepRun& r) {
  RowArgs a = row_args(r);
  a.out = r.wr(at::Y); a.ot = r.wr_type(at::Y);
  a.lse = reinterpret_cast<float*>(r.wr(at::LSE));
  if (r.s.wr.size() > at::REST) a.rest = reinterpret_cast<unsigned short*>(r.wr(at::REST));
  return launch_attention_forward(a, false, a.seq.rows, 0, reinterpret_cast<cudaStream_t>(r.stream), "Attention");
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
  return launch_attention_backward(a, reinterpret_cast<cudaStream_t>(r.stream));
}

}  // namespace dragon
