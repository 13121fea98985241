// CacheWrite: the rows of new tokens to their places in a cache of pages.
//
// Bound: HBM and, for a decoding step's few rows, the launch.  A warp copies one row of one cache, 16 bytes a lane; keys and
// values of the same table are one launch.
#include <cuda_runtime.h>

#include <algorithm>

#include "attention_util.h"
#include "plan.h"

namespace dragon {
namespace {

constexpr int kWriteWarps = 8;

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

}  // namespace dragon
