// Root-mean-square norm of rows with the residual's addition in front and 8-bit output behind, its gradient, and
// block scales / e4m3 values of a tensor in memory.
//   forward   h = x + r,  y = h * rstd * g,  rstd = 1 / sqrt(mean(h^2) + eps);  s = max(amax(y) / 448, 2^-126) per 1 x 128
//             block, q = e4m3(y / s)
//   gradient  dh = skip + rstd * (t - h * rstd^2 * mean(t h)),  t = dy g;   dg = sum over rows of dy h rstd
// Bound: bytes.  A row stays in the registers of its threads between the reduction and the output, so everything is read
// and written once; the statistics are fp32 sums.  Row lengths that do not fit take a second pass over the row.
// Measured, bf16, the kernel by itself: norm with residual and sum 8192 x 4096 48 us (5.6 TB/s), 16384 x 4096 87 us (6.2), in fp32
// 8192 x 8192 210 us (5.1); with scales and e4m3 values for y 4099 x 5000 35 us (4.1), 16384 x 4096 88 us (5.3; a division for each
// lane and access instead 93); rows of 5001 80 us (single elements), of 5002 57 (pairs), of 5000 36; gradient with the residual
// branch's 8192 x 4096 64 us (5.2).  To 8 bits, rows that are not 16-byte aligned or do not fit take two passes by single elements:
// 4099 x 5001 108 us (4.9 times its bytes at the copy rate), 5490 x 532 23 (7.2; in fp32 4.0).  Issue slots used and DRAM's share,
// by ncu: 4099 x 5000 to 8 bits 0.63 and 0.42, 4099 x 5001 0.69 and 0.18, 5490 x 532 to 8 bits 0.68 and 0.07.
#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

constexpr int kMaxRowThreads = 512;

struct RowShape {
  int threads, rows;   // threads per row (whole warps), rows per CTA
  int vec, per;        // elements per access (8 or 1), accesses per thread
  bool in_registers;
};

// Threads per row and accesses per thread: 8 elements (16 bytes of bf16) per access where rows are 16-byte aligned (a length
// that is a multiple of 8), pairs for other even lengths, single elements for odd ones; rows beyond 16384 (8192) do not fit.
// With many rows a thread takes up to four accesses of 8, so that a row is few warps and an SM holds many rows in flight;
// with fewer rows than two per SM there is nothing else to run, and a row is spread over as many threads as it can use.
RowShape row_shape(int64_t rows, int64_t cols) {
  RowShape s;
  s.vec = cols % 8 == 0 ? 8 : cols % 2 == 0 ? 2 : 1;
  const int64_t n = cols / s.vec;
  if (s.vec == 8) s.per = n <= 256 || (rows <= 256 && n <= kMaxRowThreads) ? 1 : n <= 512 || (rows <= 256 && n <= 2 * kMaxRowThreads) ? 2 : 4;
  else s.per = n <= 2 * 256 ? 2 : n <= 8 * 256 || s.vec == 2 ? 8 : 16;
  s.in_registers = n <= (int64_t)s.per * kMaxRowThreads;
  s.threads = (int)std::min<int64_t>(kMaxRowThreads, ((n + s.per - 1) / s.per + 31) / 32 * 32);
  s.rows = s.threads <= 64 ? 128 / s.threads : 1;
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

// sums over the `threads` threads of a row (threads / 32 warps); every thread of the CTA takes part.  Scratch is written
// once per call in alternating halves, so that one barrier is enough.
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
  return t;
}

// DT: the type of x, r and h (-1: they differ); RDT: that of r, or -2 without a residual
template <int DT, int RDT, int V, int PER>
__global__ void __launch_bounds__(kMaxRowThreads, DT == DRAGON_BF16 && V == 8 && PER <= 2 ? 3 : 2) norm_kernel(const NormArgs a) {
  __shared__ float2 sh[kMaxRowThreads / 32];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int slot = threadIdx.x / a.threads, t = threadIdx.x - slot * a.threads;
  const long long row = (long long)blockIdx.x * (blockDim.x / a.threads) + slot;
  const bool in = row < a.rows;
  const size_t base = (size_t)(in ? row : 0) * a.cols;
  Raw<DT, V> h[PER];
  {
    Raw<RDT, V> r[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (in && j < a.cols) { h[k].load(a.x, a.xdt, base + j); r[k].load(a.r, a.rdt, base + j); }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (RDT != -2 && in && j < a.cols) {
        float u[V], w[V];
        h[k].get(u);
        r[k].get(w);
#pragma unroll
        for (int e = 0; e < V; ++e) u[e] += w[e];
        h[k].set(u);
      }
    }
  }
  float2 sum = make_float2(0.f, 0.f);
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = (t + k * a.threads) * V;
    if (in && j < a.cols) {
      float u[V];
      h[k].get(u);
      if (DT == -1 && a.sum_dt == DRAGON_BF16) {
#pragma unroll
        for (int e = 0; e < V; ++e) u[e] = bf16_rounded(u[e]);
        h[k].set(u);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) sum.x += u[e] * u[e];
      if (a.h) h[k].store(a.h, a.sum_dt, base + j);
    }
  }
  sum = row_sum2(sum, a.threads, sh);
  const float rstd = rsqrtf(sum.x / (float)a.cols + a.eps);
  float y[PER][V];
  unsigned m = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = (t + k * a.threads) * V;
    unsigned mk = 0;
    if (in && j < a.cols) {
      float g[V];
      load_any<V>(a.gain, a.gdt, j, g);
      h[k].get(y[k]);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        y[k][e] = y[k][e] * rstd * g[e];
        if (a.ydt == DRAGON_BF16) y[k][e] = bf16_rounded(y[k][e]);
        mk = max(mk, magnitude(y[k][e]));
      }
      if (a.y) store_any<V>(a.y, a.ydt, base + j, y[k]);
    }
    if (V == 8 && (a.s || a.q)) {       // 16 neighbouring threads hold a block of 128; lane l % PER of them keeps block k's maximum
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) mk = max(mk, __shfl_xor_sync(0xffffffffu, mk, o));
      if (t % PER == k) m = mk;
    }
  }
  if (V == 8 && (a.s || a.q)) {         // the scales, two correctly rounded divisions each, of PER blocks at once
    const float s = scale_of(m), inv = __frcp_rn(s);
    const int l = t & 15, first = (t - l + l * a.threads) * V;
    if (a.s && in && l < PER && first < a.cols) a.s[(size_t)row * ((a.cols + 127) / 128) + first / 128] = s;
    if (a.q)
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const float inv_k = __shfl_sync(0xffffffffu, inv, (threadIdx.x & 16) + k);
        const int j = (t + k * a.threads) * V;
        if (in && j < a.cols) store_e4m3<V>(reinterpret_cast<unsigned char*>(a.q) + base + j, y[k], inv_k);
      }
  }
}

// Any row length, one CTA of T threads per row: a pass for the sum of squares, one for the output (a warp per block of 128 columns,
// four elements a lane).  Also the form for 8-bit output of rows whose length is no multiple of 8.
template <int T>
__global__ void __launch_bounds__(T) norm_loop_kernel(const NormArgs a) {
  __shared__ float2 sh[T / 32];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const size_t row = blockIdx.x, base = row * a.cols;
  auto sum_at = [&](int j) {
    float h, r = 0.f;
    load_any<1>(a.x, a.xdt, base + j, &h);
    if (a.r) { load_any<1>(a.r, a.rdt, base + j, &r); h += r; }
    return a.sum_dt == DRAGON_BF16 ? bf16_rounded(h) : h;
  };
  float2 sum = make_float2(0.f, 0.f);
  for (int j = threadIdx.x; j < a.cols; j += T) {
    const float h = sum_at(j);
    if (a.h) store_any<1>(a.h, a.sum_dt, base + j, &h);
    sum.x += h * h;
  }
  sum = row_sum2(sum, T, sh);
  const float rstd = rsqrtf(sum.x / (float)a.cols + a.eps);
  const int lane = threadIdx.x & 31, n_blocks = (a.cols + 127) / 128;
  for (int b = threadIdx.x >> 5; b < n_blocks; b += T / 32) {
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
// running sums of dg for its own columns; a CTA's slots (short rows: up to 16) add theirs in their order and write one partial
// row, so that two CTAs an SM leave no more than 296 for the sum that follows (14500 x 60: 61 us with a row for every slot, 17 so).  DT: the type of h and dy (-1: they differ), SDT: that of
// the residual branch's gradient (-2: none).
template <int DT, int SDT, int V, int PER> constexpr int norm_bwd_ctas() { return V * PER <= 8 ? 2 : 1; }      // of 512 threads, by registers
template <int DT, int SDT, int V, int PER>
__global__ void __launch_bounds__(kMaxRowThreads, norm_bwd_ctas<DT, SDT, V, PER>()) norm_bwd_kernel(const NormBwdArgs a) {
  constexpr bool kAhead = DT == DRAGON_BF16 && SDT != -1 && V == 8 && PER == 2;      // the next row's loads go out before this row's sums
  __shared__ float2 sh[2][kMaxRowThreads / 32];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int slot_in = threadIdx.x / a.threads, t = threadIdx.x - slot_in * a.threads;
  const int rows_per_cta = blockDim.x / a.threads;
  const long long slot = (long long)blockIdx.x * rows_per_cta + slot_in, step = (long long)gridDim.x * rows_per_cta;
  const int passes = (int)((a.rows + step - 1) / step);     // the same number for every thread of the CTA (barriers)
  float g[PER][V], dg[PER][V];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = (t + k * a.threads) * V;
    if (j < a.cols) load_any<V>(a.gain, a.gdt, j, g[k]);
#pragma unroll
    for (int e = 0; e < V; ++e) dg[k][e] = 0.f;
  }
  const float inv_cols = 1.f / (float)a.cols;
  Raw<DT, V> rh[PER], ry[PER];
  Raw<SDT, V> rs[PER];
  auto load = [&](long long row) {
    if (row >= a.rows) return;
    const size_t base = (size_t)row * a.cols;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (j < a.cols) { rh[k].load(a.h, a.hdt, base + j); ry[k].load(a.dy, a.dydt, base + j); rs[k].load(a.skip, a.sdt, base + j); }
    }
  };
  if (kAhead) load(slot);
  for (int pass = 0; pass < passes; ++pass) {
    const long long row = slot + pass * step;
    const bool in = row < a.rows;
    const size_t base = (size_t)(in ? row : 0) * a.cols;
    if (!kAhead) load(row);
    Raw<DT, V> ch[PER], cy[PER];
    Raw<SDT, V> cs[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) { ch[k] = rh[k]; cy[k] = ry[k]; cs[k] = rs[k]; }
    if (kAhead) load(row + step);
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (in && j < a.cols) {
        float h[V], dy[V];
        ch[k].get(h);
        cy[k].get(dy);
#pragma unroll
        for (int e = 0; e < V; ++e) { sum.x += h[e] * h[e]; sum.y += dy[e] * g[k][e] * h[e]; }
      }
    }
    sum = row_sum2(sum, a.threads, sh[pass & 1]);
    const float rstd = rsqrtf(sum.x * inv_cols + a.eps);
    const float c = rstd * rstd * (sum.y * inv_cols);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (in && j < a.cols) {
        float h[V], dy[V], s[V], o[V];
        ch[k].get(h);
        cy[k].get(dy);
        cs[k].get(s);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          o[e] = s[e] + rstd * (dy[e] * g[k][e] - h[e] * c);
          dg[k][e] += dy[e] * (h[e] * rstd);
        }
        if (a.dh) store_any<V>(a.dh, a.dhdt, base + j, o);
      }
    }
  }
  if (a.part && rows_per_cta == 1) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = (t + k * a.threads) * V;
      if (j < a.cols) store_any<V>(a.part, DRAGON_F32, (size_t)blockIdx.x * a.cols + j, dg[k]);
    }
  } else if (a.part) {
    extern __shared__ float total[];               // cols
    for (int s = 0; s < rows_per_cta; ++s) {
      if (slot_in == s)
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          const int j = (t + k * a.threads) * V;
          if (j < a.cols)
#pragma unroll
            for (int e = 0; e < V; ++e) total[j + e] = s ? total[j + e] + dg[k][e] : dg[k][e];
        }
      __syncthreads();
    }
    for (int j = threadIdx.x; j < a.cols; j += blockDim.x) a.part[(size_t)blockIdx.x * a.cols + j] = total[j];
  }
}

// any row length: two passes over the row; the running sums of dg stay in memory (each column belongs to one thread)
__global__ void __launch_bounds__(kMaxRowThreads) norm_bwd_loop_kernel(const NormBwdArgs a) {
  __shared__ float2 sh[2][kMaxRowThreads / 32];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  bool first = true;
  int half = 0;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, first = false) {
    const size_t base = (size_t)row * a.cols;
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int j = threadIdx.x; j < a.cols; j += kMaxRowThreads) {
      float h, dy, g;
      load_any<1>(a.h, a.hdt, base + j, &h);
      load_any<1>(a.dy, a.dydt, base + j, &dy);
      load_any<1>(a.gain, a.gdt, j, &g);
      sum.x += h * h;
      sum.y += dy * g * h;
    }
    sum = row_sum2(sum, kMaxRowThreads, sh[half]);
    half ^= 1;
    const float rstd = rsqrtf(sum.x / (float)a.cols + a.eps);
    const float c = rstd * rstd * (sum.y / (float)a.cols);
#pragma unroll 4
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

// the gradient's CTAs take as many rows as fit 512 threads where rows are short; enough CTAs to fill the SMs at the kernel's
// occupancy
RowShape norm_bwd_shape(int64_t rows, int64_t cols) {
  RowShape s = row_shape(rows, cols);
  s.rows = s.threads <= 128 ? kMaxRowThreads / s.threads : 1;
  return s;
}
int norm_bwd_grid(int64_t rows, const RowShape& s, int sm_count) {
  const int64_t ctas = (rows + s.rows - 1) / s.rows;
  const int per_sm = std::max(1, (s.vec * s.per <= 8 ? 1024 : 512) / (s.threads * s.rows));
  return (int)std::min<int64_t>(ctas, (int64_t)sm_count * per_sm);
}

template <int DT, int RDT>
cudaError_t launch_norm_typed(const NormArgs& a, const RowShape& s, int grid, cudaStream_t st) {
  const int block = s.threads * s.rows;
  if (s.vec == 2) {
    if (s.per == 2) norm_kernel<DT, RDT, 2, 2><<<grid, block, 0, st>>>(a);
    else norm_kernel<DT, RDT, 2, 8><<<grid, block, 0, st>>>(a);
  } else if (s.vec == 1) {
    if (s.per == 2) norm_kernel<DT, RDT, 1, 2><<<grid, block, 0, st>>>(a);
    else if (s.per == 8) norm_kernel<DT, RDT, 1, 8><<<grid, block, 0, st>>>(a);
    else norm_kernel<DT, RDT, 1, 16><<<grid, block, 0, st>>>(a);
  } else if (s.per == 1) norm_kernel<DT, RDT, 8, 1><<<grid, block, 0, st>>>(a);
  else if (s.per == 2) norm_kernel<DT, RDT, 8, 2><<<grid, block, 0, st>>>(a);
  else norm_kernel<DT, RDT, 8, 4><<<grid, block, 0, st>>>(a);
  return cudaGetLastError();
}
template <int DT, int SDT>
cudaError_t launch_norm_bwd_typed(const NormBwdArgs& a, const RowShape& s, int grid, cudaStream_t st) {
  const int block = s.threads * s.rows;
  const size_t smem = s.rows > 1 ? (size_t)a.cols * sizeof(float) : 0;      // (at most 16 KB)
  if (s.vec == 2) {
    if (s.per == 2) norm_bwd_kernel<DT, SDT, 2, 2><<<grid, block, smem, st>>>(a);
    else norm_bwd_kernel<DT, SDT, 2, 8><<<grid, block, smem, st>>>(a);
  } else if (s.vec == 1) {
    if (s.per == 2) norm_bwd_kernel<DT, SDT, 1, 2><<<grid, block, smem, st>>>(a);
    else if (s.per == 8) norm_bwd_kernel<DT, SDT, 1, 8><<<grid, block, smem, st>>>(a);
    else norm_bwd_kernel<DT, SDT, 1, 16><<<grid, block, smem, st>>>(a);
  } else if (s.per == 1) norm_bwd_kernel<DT, SDT, 8, 1><<<grid, block, smem, st>>>(a);
  else if (s.per == 2) norm_bwd_kernel<DT, SDT, 8, 2><<<grid, block, smem, st>>>(a);
  else norm_bwd_kernel<DT, SDT, 8, 4><<<grid, block, smem, st>>>(a);
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

// 1 x 128 blocks, or given scales of either kind, in rows of any length: a warp per block of a row, four elements a lane, four
// blocks in flight (their scales as below).  8192 x 8191 bf16: 112 us (46 for 8192 columns), element by element 186; bound by
// instructions (vectors joined across lanes, edges written by themselves: 0.76 of the issue slots used, DRAM 0.19, by ncu).
constexpr int kTogether = 4;
template <int DT>
__global__ void __launch_bounds__(256) quant_row_kernel(const QuantArgs a) {
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int lane = threadIdx.x & 31;
  const long long total = (long long)a.rows * a.cols;
  for (long long first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * kTogether; first < a.n_blocks; first += (long long)gridDim.x * 8 * kTogether) {
    typename Quad<DT>::Vec own[kTogether], behind = {};
    Quad<DT> raw[kTogether];
    size_t at[kTogether];
    int n[kTogether];
    float s = 1.f;
    long long row = first >> 31 ? first / a.col_blocks : (long long)((unsigned)first / (unsigned)a.col_blocks);
    int b = (int)(first - row * a.col_blocks);
#pragma unroll
    for (int k = 0; k < kTogether; ++k, ++b) {
      if (b == a.col_blocks) { b = 0; ++row; }
      n[k] = 0;
      at[k] = 0;
      own[k] = {};
      if (first + k >= a.n_blocks) continue;
      at[k] = (size_t)row * a.cols + (size_t)b * 128;
      n[k] = min(128, a.cols - b * 128);
      own[k] = vector_from<DT>(a.x, at[k], total - (long long)at[k], lane);
      if (lane == k) behind = vector_from<DT>(a.x, at[k], total - (long long)at[k], 32);
      if (a.s_in && lane % kTogether == k) s = __ldg(a.s_in + (size_t)(a.block_rows == 1 ? row : row >> 7) * a.col_blocks + b);
    }
#pragma unroll
    for (int k = 0; k < kTogether; ++k) raw[k] = quads_of<DT>(own[k], behind, k, at[k], lane);
    if (!a.s_in) {
      unsigned m = 0;
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        const unsigned mk = __reduce_max_sync(0xffffffffu, n[k] ? largest_magnitude(raw[k], n[k] - 4 * lane) : 0);
        if (lane % kTogether == k) m = mk;
      }
      s = scale_of(m);
    }
    if (a.s && lane < kTogether && first + lane < a.n_blocks) a.s[first + lane] = s;
    if (!a.q) continue;
    const float inv = __frcp_rn(s);
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      const float inv_k = __shfl_sync(0xffffffffu, inv, k);
      if (n[k]) store_byte_quads(a.q, at[k], n[k], e4m3_of(raw[k], inv_k), lane);
    }
  }
}

// The same for rows of a multiple of 8 elements: 16 lanes a block, 8 elements a lane, kTogether blocks of a half warp in
// flight, whose scales (two correctly rounded divisions each) are computed by as many lanes at once.  kWhole: the length is a
// multiple of 128, so block i is elements 128 i .. 128 i + 127 of the tensor.  16384 x 4096 bf16: 47 us (4.3 TB/s), with persistent
// CTAs and a division per lane 61; instructions as much as bytes (0.63 of the issue slots used, DRAM 0.51, by ncu).
constexpr int kQuantBlocks = 16 * kTogether;      // blocks of a CTA
template <int DT, bool kWhole>
__global__ void __launch_bounds__(256, 4) quant_row_vec_kernel(const QuantArgs a) {
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int l = threadIdx.x & 15;
  for (long long i0 = (long long)blockIdx.x * kQuantBlocks; i0 < a.n_blocks; i0 += (long long)gridDim.x * kQuantBlocks) {
    const long long first = i0 + (threadIdx.x >> 4);
    Raw<DT, 8> raw[kTogether];
    size_t at[kTogether];
    float given[kTogether];
    bool in[kTogether];
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      const long long i = first + k * 16;
      in[k] = i < a.n_blocks;
      at[k] = (size_t)i * 128 + l * 8;
      long long row = 0;
      int b = 0;
      if (!kWhole || a.s_in) {
        row = i >> 31 ? i / a.col_blocks : (long long)((unsigned)i / (unsigned)a.col_blocks);
        b = (int)(i - row * a.col_blocks);
      }
      if (!kWhole) {
        in[k] = in[k] && b * 128 + l * 8 < a.cols;
        at[k] = (size_t)row * a.cols + b * 128 + l * 8;
      }
      given[k] = 1.f;              // (a lane behind the row's end too takes its part of the scales)
      if (in[k]) raw[k].load(a.x, a.xdt, at[k]);
      if (a.s_in && i < a.n_blocks) given[k] = __ldg(a.s_in + (size_t)(a.block_rows == 1 ? row : row >> 7) * a.col_blocks + b);
    }
    // lane l holds the scale of the half warp's block l % kTogether
    unsigned m = 0;
    float s = 1.f;
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      if (a.s_in) { if (l % kTogether == k) s = given[k]; continue; }
      unsigned mk = in[k] ? largest_magnitude(raw[k]) : 0;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) mk = max(mk, __shfl_xor_sync(0xffffffffu, mk, o));
      if (l % kTogether == k) m = mk;
    }
    if (!a.s_in) s = scale_of(m);
    if (a.s && l < kTogether && first + l * 16 < a.n_blocks) a.s[first + l * 16] = s;
    if (!a.q) continue;
    const float inv = __frcp_rn(s);
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      const float inv_k = __shfl_sync(0xffffffffu, inv, (threadIdx.x & 16) + k);
      float v[8];
      raw[k].get(v);
      if (in[k]) store_e4m3<8>(a.q + at[k], v, inv_k);
    }
  }
}

// 128 x 128 blocks (8192 x 8192 bf16: 38 us, 5.3 TB/s): a CTA per block, which stays in registers between the maximum and the
// rounding.  kVec: 16 lanes a row, 8 elements a lane, 16 rows at a time; otherwise (rows that are not 16-byte aligned) a warp a
// row, four elements a lane: 8192 x 8191 85 us (0.70 of the issue slots, DRAM 0.24), element by element 407.
__device__ __forceinline__ float tile_scale(unsigned m, unsigned* sh) {
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, sh[i]);
  return scale_of(m);
}
template <int DT, bool kVec>
__global__ void __launch_bounds__(256) quant_tile_kernel(const QuantArgs a) {
  constexpr int kLanes = kVec ? 16 : 32, kPer = 128 * kLanes / 256;     // rows per thread
  __shared__ unsigned sh[8];
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int lane = threadIdx.x % kLanes, line = threadIdx.x / kLanes;
  const long long tile_row = blockIdx.x / a.col_blocks;
  const int b = (int)(blockIdx.x - tile_row * a.col_blocks);
  const int rows = (int)min(128LL, a.rows - tile_row * 128), cols = min(128, a.cols - b * 128);      // of this block
  const size_t first = (size_t)tile_row * 128 * a.cols + (size_t)b * 128;
  unsigned m = 0;
  if constexpr (kVec) {
    Raw<DT, 8> raw[kPer];
    const bool in = lane * 8 < cols;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (in && i * 16 + line < rows) raw[i].load(a.x, a.xdt, first + (size_t)(i * 16 + line) * a.cols + lane * 8);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (in && i * 16 + line < rows) m = max(m, largest_magnitude(raw[i]));
    const float s = tile_scale(m, sh), inv = __frcp_rn(s);
    if (a.s && threadIdx.x == 0) a.s[blockIdx.x] = s;
    if (!a.q) return;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (in && i * 16 + line < rows) {
        float v[8];
        raw[i].get(v);
        store_e4m3<8>(a.q + first + (size_t)(i * 16 + line) * a.cols + lane * 8, v, inv);
      }
  } else {
    Quad<DT> raw[kPer];
    typename Quad<DT>::Vec behind = {};
    const long long total = (long long)a.rows * a.cols;
    auto place = [&](int i) { return first + (size_t)(i * 8 + line) * a.cols; };
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i * 8 + line < rows) raw[i].u = vector_from<DT>(a.x, place(i), total - (long long)place(i), lane);
    if (lane < kPer && lane * 8 + line < rows) behind = vector_from<DT>(a.x, place(lane), total - (long long)place(lane), 32);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i * 8 + line < rows) {
        raw[i] = quads_of<DT>(raw[i].u, behind, i, place(i), lane);
        m = max(m, largest_magnitude(raw[i], cols - 4 * lane));
      }
    const float s = tile_scale(m, sh), inv = __frcp_rn(s);
    if (a.s && threadIdx.x == 0) a.s[blockIdx.x] = s;
    if (!a.q) return;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i * 8 + line < rows) store_byte_quads(a.q, place(i), cols, e4m3_of(raw[i], inv), lane);
  }
}

}  // namespace

int norm_bwd_partials(int64_t rows, int64_t cols, int sm_count) {
  const RowShape s = norm_bwd_shape(rows, cols);
  if (!s.in_registers) return (int)std::min<int64_t>(rows, (int64_t)sm_count * 2);
  return norm_bwd_grid(rows, s, sm_count);
}

cudaError_t launch_norm(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const Shape& sh = r.mems[r.s.rd[nm::X]].shape;
  NormArgs a{r.rd(nm::X), r.rd(nm::R), r.rd(nm::GAIN), r.wr(nm::H), r.wr(nm::Y), r.wr(nm::Q), reinterpret_cast<float*>(r.wr(nm::S)),
             r.rd_type(nm::X), r.rd_type(nm::R), r.rd_type(nm::GAIN), r.s.sum_dtype, r.s.round_dtype, (int)sh.rows(), (int)sh.cols(), 0,
             (float)r.s.attr, r.status_clear};
  const RowShape s = row_shape(a.rows, a.cols);
  if (!s.in_registers || (s.vec != 8 && (a.s || a.q))) {
    if (a.cols <= 1024) norm_loop_kernel<128><<<a.rows, 128, 0, st>>>(a);      // 5490 x 532 bf16 to 8 bits 23 us, with 512 threads 31
    else norm_loop_kernel<kMaxRowThreads><<<a.rows, kMaxRowThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  a.threads = s.threads;
  const int grid = (int)(((int64_t)a.rows + s.rows - 1) / s.rows);
  const bool same = a.xdt == a.sum_dt && (!a.r || a.rdt == a.xdt);
  if (!same) return a.r ? launch_norm_typed<-1, -1>(a, s, grid, st) : launch_norm_typed<-1, -2>(a, s, grid, st);
  if (a.xdt == DRAGON_F32) return a.r ? launch_norm_typed<DRAGON_F32, DRAGON_F32>(a, s, grid, st) : launch_norm_typed<DRAGON_F32, -2>(a, s, grid, st);
  return a.r ? launch_norm_typed<DRAGON_BF16, DRAGON_BF16>(a, s, grid, st) : launch_norm_typed<DRAGON_BF16, -2>(a, s, grid, st);
}

cudaError_t launch_colsum_finish(const float* part, int n_part, int cols, void* out, int dtype, cudaStream_t st);

cudaError_t launch_norm_bwd(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const Shape& sh = r.mems[r.s.rd[nb::H]].shape;
  void* dg = r.wr(nb::DGAIN);
  NormBwdArgs a{r.rd(nb::H), r.rd(nb::DY), r.rd(nb::GAIN), r.rd(nb::SKIP), r.wr(nb::DH), dg ? reinterpret_cast<float*>(r.ws + r.s.colpart_off) : nullptr,
                r.rd_type(nb::H), r.rd_type(nb::DY), r.rd_type(nb::GAIN), r.rd_type(nb::SKIP), r.wr_type(nb::DH), (int)sh.rows(), (int)sh.cols(), 0,
                (float)r.s.attr, r.status_clear};
  const RowShape s = norm_bwd_shape(a.rows, a.cols);
  cudaError_t e;
  if (!s.in_registers) {
    norm_bwd_loop_kernel<<<(int)std::min<int64_t>(a.rows, (int64_t)r.sm_count * 2), kMaxRowThreads, 0, st>>>(a);
    e = cudaGetLastError();
  } else {
    a.threads = s.threads;
    const int grid = norm_bwd_grid(a.rows, s, r.sm_count);
    const bool same = a.hdt == a.dydt && (!a.skip || a.sdt == a.hdt);
    if (!same) e = a.skip ? launch_norm_bwd_typed<-1, -1>(a, s, grid, st) : launch_norm_bwd_typed<-1, -2>(a, s, grid, st);
    else if (a.hdt == DRAGON_F32) e = a.skip ? launch_norm_bwd_typed<DRAGON_F32, DRAGON_F32>(a, s, grid, st) : launch_norm_bwd_typed<DRAGON_F32, -2>(a, s, grid, st);
    else e = a.skip ? launch_norm_bwd_typed<DRAGON_BF16, DRAGON_BF16>(a, s, grid, st) : launch_norm_bwd_typed<DRAGON_BF16, -2>(a, s, grid, st);
  }
  if (e != cudaSuccess || !dg) return e;
  return launch_colsum_finish(a.part, r.s.n_colpart, a.cols, dg, r.wr_type(nb::DGAIN), st);
}

cudaError_t launch_quant(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const Shape& sh = r.mems[r.s.rd[qt::X]].shape;
  QuantArgs a{r.rd(qt::X), reinterpret_cast<const float*>(r.rd(qt::SIN)), reinterpret_cast<float*>(r.wr(qt::S)), reinterpret_cast<unsigned char*>(r.wr(qt::Q)),
              r.rd_type(qt::X), (int)r.s.attr, (int)sh.d[0], (int)sh.d[1], (int)((sh.d[1] + 127) / 128), 0, r.status_clear};
  const bool vec = a.cols % 8 == 0, f32 = a.xdt == DRAGON_F32;
  if (a.block_rows == 128 && !a.s_in) {
    const int64_t tiles = (sh.d[0] + 127) / 128 * a.col_blocks;
    if (tiles > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    if (vec) f32 ? quant_tile_kernel<DRAGON_F32, true><<<(unsigned)tiles, 256, 0, st>>>(a) : quant_tile_kernel<DRAGON_BF16, true><<<(unsigned)tiles, 256, 0, st>>>(a);
    else f32 ? quant_tile_kernel<DRAGON_F32, false><<<(unsigned)tiles, 256, 0, st>>>(a) : quant_tile_kernel<DRAGON_BF16, false><<<(unsigned)tiles, 256, 0, st>>>(a);
    return cudaGetLastError();
  }
  a.n_blocks = (long long)sh.d[0] * a.col_blocks;
  if (vec) {
    const unsigned grid = (unsigned)std::min<long long>((a.n_blocks + kQuantBlocks - 1) / kQuantBlocks, 0x7fffffffLL);
    if (a.cols % 128 == 0) f32 ? quant_row_vec_kernel<DRAGON_F32, true><<<grid, 256, 0, st>>>(a) : quant_row_vec_kernel<DRAGON_BF16, true><<<grid, 256, 0, st>>>(a);
    else f32 ? quant_row_vec_kernel<DRAGON_F32, false><<<grid, 256, 0, st>>>(a) : quant_row_vec_kernel<DRAGON_BF16, false><<<grid, 256, 0, st>>>(a);
  } else {
    const unsigned grid = (unsigned)std::min<long long>((a.n_blocks + 8 * kTogether - 1) / (8 * kTogether), 0x7fffffffLL);
    f32 ? quant_row_kernel<DRAGON_F32><<<grid, 256, 0, st>>>(a) : quant_row_kernel<DRAGON_BF16><<<grid, 256, 0, st>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace dragon
