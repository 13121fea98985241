// Root-mean-square norm of rows with the residual's addition in front and 8-bit output behind, its gradient, and
// block scales / e4m3 values of a tensor in memory.
//   forward   h = x + r,  y = h * rstd * g,  rstd = 1 / sqrt(mean(h^2) + eps);  s = max(amax(y) / 448, 2^-126) per 1 x 128
//             block, q = e4m3(y / s)
//   gradient  dh = skip + rstd * (t - h * rstd^2 * mean(t h)),  t = dy g;   dg = sum over rows of dy h rstd
// Bound: bytes.  A row stays in the registers of its threads between the reduction and the output, so everything is read
// and written once; the statistics are fp32 sums.  Row lengths that do not fit take a second pass over the row.
#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

constexpr int kMaxRowThreads = 512;

struct RowShape {
  int threads, rows;   // threads per row (a power of two, at least 32), rows per CTA
  int vec, per;        // elements per access (8 or 1), accesses per thread
  bool in_registers;
};

// Threads per row and accesses per thread: 8 elements (16 bytes of bf16) per access where rows are 16-byte aligned
// (a length that is a multiple of 8), single elements otherwise; rows beyond 16384 (single elements: 8192) do not fit.
RowShape row_shape(int64_t cols) {
  RowShape s;
  s.vec = cols % 8 == 0 ? 8 : 1;
  const int64_t n = cols / s.vec;
  s.per = s.vec == 1 ? 16 : n <= 512 ? 1 : n <= 1024 ? 2 : 4;
  s.in_registers = n <= (int64_t)s.per * kMaxRowThreads;
  s.threads = 32;
  while (s.threads < kMaxRowThreads && (int64_t)s.threads * s.per < n) s.threads *= 2;
  s.rows = s.threads < 128 ? 128 / s.threads : 1;
  return s;
}

struct NormArgs {
  const void *x, *r, *gain;
  void *h, *y, *q;
  float* s;
  int xdt, rdt, gdt, sum_dt, ydt;   // sum_dt: h's declared type
  int rows, cols, threads;
  float eps;
  int* status_clear;
};

// sums over the `threads` threads of a row (threads / 32 warps); every thread of the CTA takes part
__device__ __forceinline__ float2 row_sum2(float2 v, int threads, float2* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if (threads == 32) return v;
  const int warp = threadIdx.x >> 5, per_row = threads >> 5, first = warp / per_row * per_row;
  if ((threadIdx.x & 31) == 0) sh[warp] = v;
  __syncthreads();
  float2 t = sh[first];
  for (int i = 1; i < per_row; ++i) { t.x += sh[first + i].x; t.y += sh[first + i].y; }
  __syncthreads();
  return t;
}

template <int XDT, int RDT, int V, int PER>
__global__ void __launch_bounds__(kMaxRowThreads) norm_kernel(const NormArgs a) {
  __shared__ float2 sh[kMaxRowThreads / 32];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int t = threadIdx.x & (a.threads - 1);
  const int rows_per_cta = blockDim.x / a.threads;
  const long long row = (long long)blockIdx.x * rows_per_cta + threadIdx.x / a.threads;
  const bool in = row < a.rows;
  const size_t base = (size_t)(in ? row : 0) * a.cols;
  Raw<XDT, V> rx[PER];
  Raw<RDT, V> rr[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = (t + k * a.threads) * V;
    if (in && j < a.cols) { rx[k].load(a.x, base + j); rr[k].load(a.r, base + j); }
  }
  float h[PER][V], g[PER][V];
  float2 sum = make_float2(0.f, 0.f);
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = (t + k * a.threads) * V;
    if (j < a.cols) load_any<V>(a.gain, a.gdt, j, g[k]);
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = (t + k * a.threads) * V;
    if (in && j < a.cols) {
      float r[V];
      rx[k].get(h[k]);
      rr[k].get(r);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if (RDT >= 0) h[k][e] += r[e];
        if (a.sum_dt == DRAGON_BF16) h[k][e] = bf16_rounded(h[k][e]);
        sum.x += h[k][e] * h[k][e];
      }
      if (a.h) store_any<V>(a.h, a.sum_dt, base + j, h[k]);
    }
  }
  sum = row_sum2(sum, a.threads, sh);
  const float rstd = rsqrtf(sum.x / (float)a.cols + a.eps);
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = (t + k * a.threads) * V;
    const bool mine = in && j < a.cols;
    float y[V];
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      y[e] = mine ? h[k][e] * rstd * g[k][e] : 0.f;
      if (a.ydt == DRAGON_BF16) y[e] = bf16_rounded(y[e]);
      m = max(m, magnitude(y[e]));
    }
    if (mine && a.y) store_any<V>(a.y, a.ydt, base + j, y);
    if (V == 8 && (a.s || a.q)) {       // 16 neighbouring threads hold a block of 128
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      const float s = scale_of(m);
      if (mine && a.s && (threadIdx.x & 15) == 0) a.s[(size_t)row * ((a.cols + 127) / 128) + j / 128] = s;
      if (mine && a.q) {
        const float inv = __frcp_rn(s);
        uint2 w;
        w.x = e4m3_pair(y[0] * inv, y[1 % V] * inv) | (e4m3_pair(y[2 % V] * inv, y[3 % V] * inv) << 16);
        w.y = e4m3_pair(y[4 % V] * inv, y[5 % V] * inv) | (e4m3_pair(y[6 % V] * inv, y[7 % V] * inv) << 16);
        *reinterpret_cast<uint2*>(reinterpret_cast<unsigned char*>(a.q) + base + j) = w;
      }
    }
  }
}

// Any row length, one CTA per row: a pass for the sum of squares, one for the output (a warp per block of 128 columns,
// four elements a lane).  Also the form for 8-bit output of rows whose length is no multiple of 8.
__global__ void __launch_bounds__(kMaxRowThreads) norm_loop_kernel(const NormArgs a) {
  __shared__ float2 sh[kMaxRowThreads / 32];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const size_t row = blockIdx.x, base = row * a.cols;
  auto sum_at = [&](int j) {
    float h, r = 0.f;
    load_any<1>(a.x, a.xdt, base + j, &h);
    if (a.r) { load_any<1>(a.r, a.rdt, base + j, &r); h += r; }
    return a.sum_dt == DRAGON_BF16 ? bf16_rounded(h) : h;
  };
  float2 sum = make_float2(0.f, 0.f);
  for (int j = threadIdx.x; j < a.cols; j += kMaxRowThreads) {
    const float h = sum_at(j);
    if (a.h) store_any<1>(a.h, a.sum_dt, base + j, &h);
    sum.x += h * h;
  }
  sum = row_sum2(sum, kMaxRowThreads, sh);
  const float rstd = rsqrtf(sum.x / (float)a.cols + a.eps);
  const int lane = threadIdx.x & 31, n_blocks = (a.cols + 127) / 128;
  for (int b = threadIdx.x >> 5; b < n_blocks; b += kMaxRowThreads / 32) {
    float y[4];
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = b * 128 + e * 32 + lane;
      y[e] = 0.f;
      if (j < a.cols) {
        float g;
        load_any<1>(a.gain, a.gdt, j, &g);
        y[e] = sum_at(j) * rstd * g;
        if (a.ydt == DRAGON_BF16) y[e] = bf16_rounded(y[e]);
        if (a.y) store_any<1>(a.y, a.ydt, base + j, &y[e]);
      }
      m = max(m, magnitude(y[e]));
    }
    if (!a.s && !a.q) continue;
    m = __reduce_max_sync(0xffffffffu, m);
    const float s = scale_of(m), inv = __frcp_rn(s);
    if (a.s && lane == 0) a.s[row * n_blocks + b] = s;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = b * 128 + e * 32 + lane;
      if (a.q && j < a.cols) reinterpret_cast<unsigned char*>(a.q)[base + j] = e4m3_of(y[e] * inv);
    }
  }
}

struct NormBwdArgs {
  const void *h, *dy, *gain, *skip;
  void* dh;
  float* part;      // partial sums over rows of dy h rstd: one row of cols floats per row slot of the grid
  int hdt, dydt, gdt, sdt, dhdt;
  int rows, cols, threads;
  float eps;
  int* status_clear;
};

// Persistent: a row slot (the threads of one row) walks the rows with the grid's stride, so that every thread keeps the
// running sums of dg for its own columns and writes them once.
template <int HDT, int DYDT, int SDT, int V, int PER>
__global__ void __launch_bounds__(kMaxRowThreads) norm_bwd_kernel(const NormBwdArgs a) {
  __shared__ float2 sh[kMaxRowThreads / 32];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int t = threadIdx.x & (a.threads - 1);
  const int rows_per_cta = blockDim.x / a.threads;
  const long long slot = (long long)blockIdx.x * rows_per_cta + threadIdx.x / a.threads, step = (long long)gridDim.x * rows_per_cta;
  const long long passes = (a.rows + step - 1) / step;     // the same number for every thread of the CTA (barriers)
  float g[PER][V], dg[PER][V];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = (t + k * a.threads) * V;
    if (j < a.cols) load_any<V>(a.gain, a.gdt, j, g[k]);
#pragma unroll
    for (int e = 0; e < V; ++e) dg[k][e] = 0.f;
  }
  const float inv_cols = 1.f / (float)a.cols;
  for (long long pass = 0; pass < passes; ++pass) {
    const long long row = slot + pass * step;
    const bool in = row < a.rows;
    const size_t base = (size_t)(in ? row : 0) * a.cols;
    Raw<HDT, V> rh[PER];
    Raw<DYDT, V> ry[PER];
    Raw<SDT, V> rs[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (in && j < a.cols) { rh[k].load(a.h, base + j); ry[k].load(a.dy, base + j); rs[k].load(a.skip, base + j); }
    }
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (in && j < a.cols) {
        float h[V], dy[V];
        rh[k].get(h);
        ry[k].get(dy);
#pragma unroll
        for (int e = 0; e < V; ++e) { sum.x += h[e] * h[e]; sum.y += dy[e] * g[k][e] * h[e]; }
      }
    }
    sum = row_sum2(sum, a.threads, sh);
    const float rstd = rsqrtf(sum.x * inv_cols + a.eps);
    const float c = rstd * rstd * (sum.y * inv_cols);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (in && j < a.cols) {
        float h[V], dy[V], s[V], o[V];
        rh[k].get(h);
        ry[k].get(dy);
        rs[k].get(s);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          o[e] = s[e] + rstd * (dy[e] * g[k][e] - h[e] * c);
          dg[k][e] += dy[e] * (h[e] * rstd);
        }
        if (a.dh) store_any<V>(a.dh, a.dhdt, base + j, o);
      }
    }
  }
  if (a.part) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (j < a.cols) store_any<V>(a.part, DRAGON_F32, (size_t)slot * a.cols + j, dg[k]);
    }
  }
}

// any row length: two passes over the row; the running sums of dg stay in memory (each column belongs to one thread)
__global__ void __launch_bounds__(kMaxRowThreads) norm_bwd_loop_kernel(const NormBwdArgs a) {
  __shared__ float2 sh[kMaxRowThreads / 32];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  bool first = true;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, first = false) {
    const size_t base = (size_t)row * a.cols;
    float2 sum = make_float2(0.f, 0.f);
    for (int j = threadIdx.x; j < a.cols; j += kMaxRowThreads) {
      float h, dy, g;
      load_any<1>(a.h, a.hdt, base + j, &h);
      load_any<1>(a.dy, a.dydt, base + j, &dy);
      load_any<1>(a.gain, a.gdt, j, &g);
      sum.x += h * h;
      sum.y += dy * g * h;
    }
    sum = row_sum2(sum, kMaxRowThreads, sh);
    const float rstd = rsqrtf(sum.x / (float)a.cols + a.eps);
    const float c = rstd * rstd * (sum.y / (float)a.cols);
    for (int j = threadIdx.x; j < a.cols; j += kMaxRowThreads) {
      float h, dy, g, s = 0.f;
      load_any<1>(a.h, a.hdt, base + j, &h);
      load_any<1>(a.dy, a.dydt, base + j, &dy);
      load_any<1>(a.gain, a.gdt, j, &g);
      if (a.skip) load_any<1>(a.skip, a.sdt, base + j, &s);
      const float o = s + rstd * (dy * g - h * c);
      if (a.dh) store_any<1>(a.dh, a.dhdt, base + j, &o);
      if (a.part) {
        float* p = a.part + (size_t)blockIdx.x * a.cols + j;
        *p = (first ? 0.f : *p) + dy * (h * rstd);
      }
    }
  }
}

int norm_bwd_grid(int64_t rows, const RowShape& s, int sm_count) {
  const int64_t ctas = (rows + s.rows - 1) / s.rows;
  return (int)std::min<int64_t>(ctas, (int64_t)sm_count * (s.threads * s.rows > 256 ? 2 : 4));
}

template <int XDT, int RDT>
cudaError_t launch_norm_typed(const NormArgs& a, const RowShape& s, int grid, cudaStream_t st) {
  const int block = s.threads * s.rows;
  if (s.vec == 1) norm_kernel<XDT, RDT, 1, 16><<<grid, block, 0, st>>>(a);
  else if (s.per == 1) norm_kernel<XDT, RDT, 8, 1><<<grid, block, 0, st>>>(a);
  else if (s.per == 2) norm_kernel<XDT, RDT, 8, 2><<<grid, block, 0, st>>>(a);
  else norm_kernel<XDT, RDT, 8, 4><<<grid, block, 0, st>>>(a);
  return cudaGetLastError();
}
template <int HDT, int DYDT, int SDT>
cudaError_t launch_norm_bwd_typed(const NormBwdArgs& a, const RowShape& s, int grid, cudaStream_t st) {
  const int block = s.threads * s.rows;
  if (s.vec == 1) norm_bwd_kernel<HDT, DYDT, SDT, 1, 16><<<grid, block, 0, st>>>(a);
  else if (s.per == 1) norm_bwd_kernel<HDT, DYDT, SDT, 8, 1><<<grid, block, 0, st>>>(a);
  else if (s.per == 2) norm_bwd_kernel<HDT, DYDT, SDT, 8, 2><<<grid, block, 0, st>>>(a);
  else norm_bwd_kernel<HDT, DYDT, SDT, 8, 4><<<grid, block, 0, st>>>(a);
  return cudaGetLastError();
}

struct QuantArgs {
  const void* x;
  const float* s_in;
  float* s;
  unsigned char* q;
  int xdt, block_rows;
  int rows, cols, col_blocks;
  long long n_blocks;
  int* status_clear;
};

// 1 x 128 blocks, or given scales of either kind: a warp per block of a row, four elements a lane
__global__ void __launch_bounds__(256) quant_row_kernel(const QuantArgs a) {
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int lane = threadIdx.x & 31;
  for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < a.n_blocks; i += (long long)gridDim.x * 8) {
    const long long row = i / a.col_blocks;
    const int b = (int)(i - row * a.col_blocks);
    const size_t base = (size_t)row * a.cols;
    float v[4];
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = b * 128 + e * 32 + lane;
      v[e] = 0.f;
      if (j < a.cols) load_any<1>(a.x, a.xdt, base + j, &v[e]);
      m = max(m, magnitude(v[e]));
    }
    float s;
    if (a.s_in) s = __ldg(a.s_in + (size_t)(row / a.block_rows) * a.col_blocks + b);
    else s = scale_of(__reduce_max_sync(0xffffffffu, m));
    if (a.s && lane == 0) a.s[i] = s;
    const float inv = __frcp_rn(s);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = b * 128 + e * 32 + lane;
      if (a.q && j < a.cols) a.q[base + j] = e4m3_of(v[e] * inv);
    }
  }
}

// 128 x 128 blocks: a CTA per block, which stays in registers between the maximum and the rounding (16 rows a warp)
__global__ void __launch_bounds__(256) quant_tile_kernel(const QuantArgs a) {
  __shared__ unsigned sh[8];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long tile_row = blockIdx.x / a.col_blocks;
  const int b = (int)(blockIdx.x - tile_row * a.col_blocks);
  float v[16][4];
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const long long row = tile_row * 128 + i * 8 + warp;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = b * 128 + e * 32 + lane;
      v[i][e] = 0.f;
      if (row < a.rows && j < a.cols) load_any<1>(a.x, a.xdt, (size_t)row * a.cols + j, &v[i][e]);
      m = max(m, magnitude(v[i][e]));
    }
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if (lane == 0) sh[warp] = m;
  __syncthreads();
  for (int i = 0; i < 8; ++i) m = max(m, sh[i]);
  const float s = scale_of(m), inv = __frcp_rn(s);
  if (a.s && threadIdx.x == 0) a.s[blockIdx.x] = s;
  if (!a.q) return;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const long long row = tile_row * 128 + i * 8 + warp;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = b * 128 + e * 32 + lane;
      if (row < a.rows && j < a.cols) a.q[(size_t)row * a.cols + j] = e4m3_of(v[i][e] * inv);
    }
  }
}

}  // namespace

int norm_bwd_partials(int64_t rows, int64_t cols, int sm_count) {
  const RowShape s = row_shape(cols);
  if (!s.in_registers) return (int)std::min<int64_t>(rows, (int64_t)sm_count * 2);
  return norm_bwd_grid(rows, s, sm_count) * s.rows;
}

cudaError_t launch_norm(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const Shape& sh = r.mems[r.s.rd[nm::X]].shape;
  NormArgs a{r.rd(nm::X), r.rd(nm::R), r.rd(nm::GAIN), r.wr(nm::H), r.wr(nm::Y), r.wr(nm::Q), reinterpret_cast<float*>(r.wr(nm::S)),
             r.rd_type(nm::X), r.rd_type(nm::R), r.rd_type(nm::GAIN), r.s.sum_dtype, r.s.round_dtype, (int)sh.rows(), (int)sh.cols(), 0,
             (float)r.s.attr, r.status_clear};
  const RowShape s = row_shape(a.cols);
  if (!s.in_registers || (s.vec == 1 && (a.s || a.q))) {
    norm_loop_kernel<<<a.rows, kMaxRowThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  a.threads = s.threads;
  const int grid = (int)(((int64_t)a.rows + s.rows - 1) / s.rows);
  const int rdt = a.r ? a.rdt : -1;
  if (a.xdt == DRAGON_F32)
    return rdt < 0 ? launch_norm_typed<DRAGON_F32, -1>(a, s, grid, st) : rdt == DRAGON_F32 ? launch_norm_typed<DRAGON_F32, DRAGON_F32>(a, s, grid, st)
                                                                         : launch_norm_typed<DRAGON_F32, DRAGON_BF16>(a, s, grid, st);
  return rdt < 0 ? launch_norm_typed<DRAGON_BF16, -1>(a, s, grid, st) : rdt == DRAGON_F32 ? launch_norm_typed<DRAGON_BF16, DRAGON_F32>(a, s, grid, st)
                                                                        : launch_norm_typed<DRAGON_BF16, DRAGON_BF16>(a, s, grid, st);
}

cudaError_t launch_colsum_finish(const float* part, int n_part, int cols, void* out, int dtype, cudaStream_t st);

cudaError_t launch_norm_bwd(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const Shape& sh = r.mems[r.s.rd[nb::H]].shape;
  void* dg = r.wr(nb::DGAIN);
  NormBwdArgs a{r.rd(nb::H), r.rd(nb::DY), r.rd(nb::GAIN), r.rd(nb::SKIP), r.wr(nb::DH), dg ? reinterpret_cast<float*>(r.ws + r.s.colpart_off) : nullptr,
                r.rd_type(nb::H), r.rd_type(nb::DY), r.rd_type(nb::GAIN), r.rd_type(nb::SKIP), r.wr_type(nb::DH), (int)sh.rows(), (int)sh.cols(), 0,
                (float)r.s.attr, r.status_clear};
  const RowShape s = row_shape(a.cols);
  cudaError_t e;
  if (!s.in_registers) {
    norm_bwd_loop_kernel<<<(int)std::min<int64_t>(a.rows, (int64_t)r.sm_count * 2), kMaxRowThreads, 0, st>>>(a);
    e = cudaGetLastError();
  } else {
    a.threads = s.threads;
    const int grid = norm_bwd_grid(a.rows, s, r.sm_count);
    const int sdt = a.skip ? a.sdt : -1;
#define DRAGON_NB(H, D) (sdt < 0 ? launch_norm_bwd_typed<H, D, -1>(a, s, grid, st) : sdt == DRAGON_F32 ? launch_norm_bwd_typed<H, D, DRAGON_F32>(a, s, grid, st) \
                                                                                     : launch_norm_bwd_typed<H, D, DRAGON_BF16>(a, s, grid, st))
    if (a.hdt == DRAGON_F32) e = a.dydt == DRAGON_F32 ? DRAGON_NB(DRAGON_F32, DRAGON_F32) : DRAGON_NB(DRAGON_F32, DRAGON_BF16);
    else e = a.dydt == DRAGON_F32 ? DRAGON_NB(DRAGON_BF16, DRAGON_F32) : DRAGON_NB(DRAGON_BF16, DRAGON_BF16);
#undef DRAGON_NB
  }
  if (e != cudaSuccess || !dg) return e;
  return launch_colsum_finish(a.part, r.s.n_colpart, a.cols, dg, r.wr_type(nb::DGAIN), st);
}

cudaError_t launch_quant(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const Shape& sh = r.mems[r.s.rd[qt::X]].shape;
  QuantArgs a{r.rd(qt::X), reinterpret_cast<const float*>(r.rd(qt::SIN)), reinterpret_cast<float*>(r.wr(qt::S)), reinterpret_cast<unsigned char*>(r.wr(qt::Q)),
              r.rd_type(qt::X), (int)r.s.attr, (int)sh.d[0], (int)sh.d[1], (int)((sh.d[1] + 127) / 128), 0, r.status_clear};
  if (a.block_rows == 128 && !a.s_in) {
    const int64_t tiles = (sh.d[0] + 127) / 128 * a.col_blocks;
    if (tiles > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    quant_tile_kernel<<<(unsigned)tiles, 256, 0, st>>>(a);
  } else {
    a.n_blocks = (long long)sh.d[0] * a.col_blocks;
    quant_row_kernel<<<(unsigned)std::min<long long>((a.n_blocks + 7) / 8, (long long)r.sm_count * 8), 256, 0, st>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace dragon
