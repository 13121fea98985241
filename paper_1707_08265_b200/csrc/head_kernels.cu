// HeadNorm and Rotate: every head of a row over its root mean square, and turned by the row's position.
//
//   u = x / sqrt(mean(x^2) + eps) * g;  y = amplitude (a cos t - b sin t, b cos t + a sin t) over pairs (a, b) of u's first dims
//   elements, t = position * f_i.  Backwards, with d = the rotation by -t of dy:
//   dg = sum over rows and heads of d x r,  dx = r (d g) - x r^3 mean(d g x),  r = 1 / sqrt(mean(x^2) + eps).
//
// Angles: f_i / 2 pi is kept as a 64-bit fraction of a turn, so position * f_i modulo one turn is one wrapping integer product
// (no rounding grows with the position); its top 32 bits go through sincospi in fp32.  They are the same for every head of a
// row: a CTA computes those of its rows once, into shared memory.
//
// Bound: HBM (every element is read and written once).  A warp works on one row at a time: 8 elements a lane, a head in the next
// power of two of lanes, so that the head's sums are a few shuffles; the lane's angles stay in registers while the warp walks the
// row's heads.  Tensors of the same rows (queries and keys) are one launch.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

constexpr int kHeadThreads = 256, kHeadWarps = kHeadThreads / 32;
constexpr int kHeadRowsMost = kHeadWarps;       // rows of a tile: their angles are computed together
constexpr int kPairsMost = kMaxRotatedWidth / 2;

enum Pairing { P_NONE, P_NEIGHBOURS, P_LANES, P_ANY };   // where a lane finds the partners of its 8 elements

struct HeadJob {
  const void *x, *gain, *dy;
  void *u, *y;             // backwards: y receives dx
  float* dgain;            // partial rows [grid][width]
  int xt, gt, dyt, ut, yt;
  int round_u;             // u is rounded to bf16 before it is rotated
  int heads;
  float eps;
};
struct HeadArgs {
  HeadJob job[kHeadsPerLaunch];
  const int* pos;
  int *status_clear;
  int rows, width, dims, lanes;   // lanes: of a head, a power of two
  int tile;                // rows of a tile, a power of two
  float amplitude;
  unsigned long long freq[kPairsMost];   // turns per position, times 2^64
};

// (amplitude cos, amplitude sin) of pair i, where every lane finds those of its elements without a bank in common
__device__ __forceinline__ int place_of(int i) { return (i & 7) * (kPairsMost / 8 + 1) + (i >> 3); }
constexpr int kPlaces = 8 * (kPairsMost / 8 + 1);

// the angles of `rows` rows from r0 on
__device__ __forceinline__ void fill_angles(const HeadArgs& a, float2 (*cs)[kPlaces], int r0, int rows) {
  const int pairs = a.dims >> 1;
  for (int i = threadIdx.x; i < rows * pairs; i += kHeadThreads) {
    const int r = i / pairs, k = i - r * pairs;
    const unsigned long long turn = (unsigned long long)(long long)__ldg(a.pos + r0 + r) * a.freq[k];
    float s, c;
    sincospif((float)(int)(turn >> 32) * 0x1p-31f, &s, &c);
    cs[r][place_of(k)] = make_float2(a.amplitude * c, a.amplitude * s);
  }
}

// the angles of this lane's elements, from e0 of the head on: of its 4 pairs, or of the pairs that its 8 elements belong to.  An
// element behind dims gets (1, 0); the second of a pair gets minus its sine, so that x' = x c - partner s for both
template <int kPairing> __device__ __forceinline__ void load_angles(const float2* cs, int e0, int dims, float2* t) {
  const int half = dims >> 1;
  if (kPairing == P_NEIGHBOURS) {
#pragma unroll
    for (int p = 0; p < 4; ++p) t[p] = (e0 >> 1) + p < half ? cs[place_of((e0 >> 1) + p)] : make_float2(1.f, 0.f);
  } else if (kPairing != P_NONE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int at = e0 + e;
      t[e] = at < dims ? cs[place_of(at < half ? at : at - half)] : make_float2(1.f, 0.f);
      if (at >= half) t[e].y = -t[e].y;
    }
  }
}

// v: this lane's 8 elements; back: by the negative angle.  buf: 256 floats of this warp (P_ANY)
template <int kPairing, bool kBack> __device__ __forceinline__ void turn(float* v, const float2* t, int e0, int dims, int lane, float* buf) {
  const int half = dims >> 1;
  if (kPairing == P_NEIGHBOURS) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float c = t[p].x, s = kBack ? -t[p].y : t[p].y, p0 = v[2 * p], p1 = v[2 * p + 1];
      v[2 * p] = p0 * c - p1 * s;
      v[2 * p + 1] = p1 * c + p0 * s;
    }
  } else if (kPairing == P_LANES) {      // half a multiple of 8: the partners are the 8 elements of one other lane
    const int from = e0 < dims ? lane + (e0 < half ? half : -half) / 8 : lane;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float other = __shfl_sync(0xffffffffu, v[e], from);
      v[e] = v[e] * t[e].x + (kBack ? other : -other) * t[e].y;
    }
  } else if (kPairing == P_ANY) {
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 8; ++e) buf[lane * 8 + e] = v[e];
    __syncwarp();
    const float* head = buf + lane * 8 - e0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int at = e0 + e;
      const float other = at < dims ? head[at < half ? at + half : at - half] : 0.f;
      v[e] = v[e] * t[e].x + (kBack ? other : -other) * t[e].y;
    }
  }
}

__device__ __forceinline__ float sum_over_lanes(float v, int lanes) {
  for (int s = lanes >> 1; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
  return v;
}

// DT: the type of x, u and y (backwards: x, dy and dx), -1 for a mixture
template <int DT, int kPairing, bool kBack> __global__ void __launch_bounds__(kHeadThreads) head_kernel(const __grid_constant__ HeadArgs a) {
  constexpr int kUnroll = kBack ? 2 : 4;
  __shared__ float2 cs[kPairing == P_NONE ? 1 : kHeadRowsMost][kPlaces];
  __shared__ float buf[kPairing == P_ANY ? kHeadWarps : 1][256];
  __shared__ float sums[kBack ? kHeadWarps : 1][kMaxRotatedWidth];
  const HeadJob& jb = a.job[blockIdx.y];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (a.status_clear && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int l = lane & (a.lanes - 1), e0 = 8 * l;
  const bool active = e0 < a.width;
  const int per_warp = 32 / a.lanes, sub = lane / a.lanes;      // heads of one warp access
  const int groups = (jb.heads + per_warp - 1) / per_warp;
  const int side = kHeadWarps / a.tile, my_row = warp / side, my_side = warp - my_row * side;      // warps of a row
  const float inv_width = 1.f / (float)a.width;
  const bool norm = jb.gain != nullptr;
  float g[8], dg[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { g[e] = 1.f; dg[e] = 0.f; }
  if (norm && active) load_any<8>(jb.gain, jb.gt, (size_t)e0, g);
  for (long long r0 = (long long)blockIdx.x * a.tile; r0 < a.rows; r0 += (long long)gridDim.x * a.tile) {
    const int rows = (int)min((long long)a.tile, a.rows - r0);
    float2 t[kPairing == P_NONE ? 1 : 8];
    if (kPairing != P_NONE) {
      __syncthreads();
      fill_angles(a, cs, (int)r0, rows);
      __syncthreads();
    }
    if (my_row >= rows) continue;
    if (kPairing != P_NONE) load_angles<kPairing>(cs[my_row], e0, a.dims, t);
    const size_t row_at = (size_t)(r0 + my_row) * jb.heads * a.width + e0;
    for (int i0 = my_side; i0 < groups; i0 += side * kUnroll) {
      Raw<DT, 8> rx[kUnroll], rd[kUnroll];
      size_t at[kUnroll];
      bool ok[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int head = (i0 + k * side) * per_warp + sub;
        ok[k] = active && head < jb.heads;
        at[k] = row_at + (size_t)head * a.width;
        if (ok[k]) {
          if (!kBack || norm) rx[k].load(jb.x, jb.xt, at[k]);
          if (kBack) rd[k].load(jb.dy, jb.dyt, at[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        if (i0 + k * side >= groups) break;       // the whole warp
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
        if (ok[k] && (!kBack || norm)) rx[k].get(x);
        float inv = 1.f;
        if (!kBack) {
          if (norm) {
            float q = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) q += x[e] * x[e];
            inv = rsqrtf(sum_over_lanes(q, a.lanes) * inv_width + jb.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * g[e];
            if (jb.u && ok[k]) store_any<8>(jb.u, jb.ut, at[k], x);
            if (jb.round_u) {
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = bf16_rounded(x[e]);
            }
          }
          turn<kPairing, false>(x, t, e0, a.dims, lane, buf[kPairing == P_ANY ? warp : 0]);
          if (jb.y && ok[k]) { Raw<DT, 8> o; o.set(x); o.store(jb.y, jb.yt, at[k]); }
        } else {
          float d[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = 0.f;
          if (ok[k]) rd[k].get(d);
          turn<kPairing, true>(d, t, e0, a.dims, lane, buf[kPairing == P_ANY ? warp : 0]);
          if (norm) {
            float q = 0.f, m = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) { q += x[e] * x[e]; m += d[e] * g[e] * x[e]; }
            inv = rsqrtf(sum_over_lanes(q, a.lanes) * inv_width + jb.eps);
            const float c = inv * inv * inv * (sum_over_lanes(m, a.lanes) * inv_width);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              dg[e] += d[e] * x[e] * inv;
              d[e] = inv * d[e] * g[e] - x[e] * c;
            }
          }
          if (jb.y && ok[k]) { Raw<DT, 8> o; o.set(d); o.store(jb.y, jb.yt, at[k]); }
        }
      }
    }
  }
  if (kBack && jb.dgain) {      // the CTA's part of dg: lanes of the same elements, then the warps, in a fixed order
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      for (int s = a.lanes; s < 32; s <<= 1) dg[e] += __shfl_xor_sync(0xffffffffu, dg[e], s);
      if (lane < a.lanes && active) sums[warp][e0 + e] = dg[e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += kHeadThreads) {
      float t = 0.f;
      for (int w = 0; w < kHeadWarps; ++w) t += sums[w][c];
      jb.dgain[(size_t)blockIdx.x * a.width + c] = t;
    }
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// dg: the partial rows in a fixed order (in fp64), 32 columns a CTA
struct FinishArgs {
  const float* part[kHeadsPerLaunch];
  void* out[kHeadsPerLaunch];
  int type[kHeadsPerLaunch];
  int n, width;
};
__global__ void __launch_bounds__(1024) head_finish(const __grid_constant__ FinishArgs a) {
  __shared__ double sh[32][33];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float* part = a.part[blockIdx.y];
  double s = 0.0;
  if (c < a.width) {
    int i = slice;
    for (; i + 96 < a.n; i += 128) {
      const float v0 = part[(size_t)i * a.width + c], v1 = part[(size_t)(i + 32) * a.width + c], v2 = part[(size_t)(i + 64) * a.width + c], v3 = part[(size_t)(i + 96) * a.width + c];
      s += ((double)v0 + (double)v1) + ((double)v2 + (double)v3);
    }
    for (; i < a.n; i += 32) s += (double)part[(size_t)i * a.width + c];
  }
  sh[slice][lane] = s;
  __syncthreads();
  if (slice == 0 && c < a.width) {
    for (int k = 1; k < 32; ++k) s += sh[k][lane];
    const float v = (float)s;
    store_any<1>(a.out[blockIdx.y], a.type[blockIdx.y], (size_t)c, &v);
  }
}

// Rows of a tile: as many as leave four CTAs for every SM
int tile_rows(int64_t rows, int sm_count) {
  int t = kHeadRowsMost;
  while (t > 1 && rows < t * (4 * (int64_t)sm_count)) t /= 2;
  return t;
}

template <bool kBack, int DT> void launch_pairing(const HeadArgs& a, int pairing, dim3 grid, cudaStream_t st) {
  switch (pairing) {
    case P_NONE: head_kernel<DT, P_NONE, kBack><<<grid, kHeadThreads, 0, st>>>(a); break;
    case P_NEIGHBOURS: head_kernel<DT, P_NEIGHBOURS, kBack><<<grid, kHeadThreads, 0, st>>>(a); break;
    case P_LANES: head_kernel<DT, P_LANES, kBack><<<grid, kHeadThreads, 0, st>>>(a); break;
    default: head_kernel<DT, P_ANY, kBack><<<grid, kHeadThreads, 0, st>>>(a);
  }
}

template <bool kBack> cudaError_t launch(HeadArgs& a, const Step& s, int jobs, dim3 grid, cudaStream_t st) {
  const std::vector<double>& n = s.num;
  a.lanes = 1;
  while (a.lanes * 8 < a.width) a.lanes *= 2;
  int pairing = P_NONE;
  if (a.pos) {
    a.dims = (int)n[hn::DIMS];
    a.amplitude = (float)n[hn::AMPLITUDE];
    std::copy(s.freq.begin(), s.freq.end(), a.freq);
    pairing = n[hn::INTERLEAVED] != 0.0 ? P_NEIGHBOURS : a.dims % 16 == 0 ? P_LANES : P_ANY;
  }
  bool all[2] = {true, true};      // every tensor is f32, is bf16
  for (int j = 0; j < jobs; ++j) {
    const HeadJob& b = a.job[j];
    for (int t = 0; t < 2; ++t) {
      const int type = t ? DRAGON_BF16 : DRAGON_F32;
      all[t] &= (!b.x || b.xt == type) && (!b.y || b.yt == type) && (!kBack || b.dyt == type);
    }
  }
  if (all[1]) launch_pairing<kBack, DRAGON_BF16>(a, pairing, grid, st);
  else if (all[0]) launch_pairing<kBack, DRAGON_F32>(a, pairing, grid, st);
  else launch_pairing<kBack, -1>(a, pairing, grid, st);
  return cudaGetLastError();
}

}  // namespace

int head_bwd_partials(int64_t rows, int sm_count) {
  const int tile = tile_rows(rows, sm_count);
  return (int)std::min<int64_t>((rows + tile - 1) / tile, 4 * (int64_t)sm_count);
}

cudaError_t launch_head(const StepRun& r) {
  const Step& s = r.s;
  const Shape& sh = r.mems[s.rd[hd::X]].shape;
  HeadArgs a = {};
  a.width = (int)s.num[hn::WIDTH];
  a.rows = (int)sh.d[0];
  const int jobs = (int)s.rd.size() / hd::READS;
  bool rotated = false;
  for (int j = 0; j < jobs; ++j) {
    HeadJob& b = a.job[j];
    const int rd = hd::READS * j, wr = hd::WRITES * j;
    b.x = r.rd(rd + hd::X); b.xt = r.rd_type(rd + hd::X);
    b.gain = r.rd(rd + hd::GAIN); b.gt = r.rd_type(rd + hd::GAIN);
    b.u = r.wr(wr + hd::U); b.ut = r.wr_type(wr + hd::U);
    b.y = r.wr(wr + hd::Y); b.yt = r.wr_type(wr + hd::Y);
    rotated = b.y != nullptr;      // (steps are joined only where all of them rotate, or none does)
    if (!b.y) { b.y = b.u; b.yt = b.ut; b.u = nullptr; }      // the norm alone writes its result as the last step
    b.round_u = rotated && s.head_round[j] == DRAGON_BF16;
    b.eps = s.head_eps[j];
    b.heads = (int)(r.mems[s.rd[rd + hd::X]].shape.d[1] / a.width);
  }
  a.pos = rotated ? reinterpret_cast<const int*>(r.rd(hd::POS)) : nullptr;
  a.status_clear = r.status_clear;
  a.tile = tile_rows(a.rows, r.sm_count);
  return launch<false>(a, s, jobs, dim3((unsigned)((a.rows + (int64_t)a.tile - 1) / a.tile), jobs), reinterpret_cast<cudaStream_t>(r.stream));
}

cudaError_t launch_head_bwd(const StepRun& r) {
  const Step& s = r.s;
  const Shape& sh = r.mems[s.rd[hb::DY]].shape;
  HeadArgs a = {};
  FinishArgs f = {};
  a.width = f.width = (int)s.num[hn::WIDTH];
  a.rows = (int)sh.d[0];
  const int jobs = (int)s.rd.size() / hb::READS, grid = head_bwd_partials(a.rows, r.sm_count);
  int sums = 0;
  for (int j = 0; j < jobs; ++j) {
    HeadJob& b = a.job[j];
    const int rd = hb::READS * j, wr = hb::WRITES * j;
    b.x = r.rd(rd + hb::X); b.xt = r.rd_type(rd + hb::X);
    b.gain = r.rd(rd + hb::GAIN); b.gt = r.rd_type(rd + hb::GAIN);
    b.dy = r.rd(rd + hb::DY); b.dyt = r.rd_type(rd + hb::DY);
    b.y = r.wr(wr + hb::DX); b.yt = r.wr_type(wr + hb::DX);
    b.eps = s.head_eps[j];
    b.heads = (int)(r.mems[s.rd[rd + hb::DY]].shape.d[1] / a.width);
    if (s.wr[wr + hb::DGAIN] >= 0) {
      b.dgain = reinterpret_cast<float*>(r.ws + s.colpart_off) + (size_t)j * grid * a.width;
      f.part[sums] = b.dgain;
      f.out[sums] = r.wr(wr + hb::DGAIN);
      f.type[sums++] = r.wr_type(wr + hb::DGAIN);
    }
  }
  a.pos = reinterpret_cast<const int*>(r.rd(hb::POS));
  a.status_clear = r.status_clear;
  a.tile = tile_rows(a.rows, r.sm_count);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const cudaError_t e = launch<true>(a, s, jobs, dim3(grid, jobs), st);
  if (e != cudaSuccess || !sums) return e;
  f.n = grid;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((a.width + 31) / 32, sums);
  cfg.blockDim = dim3(1024);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, head_finish, f);
}

}  // namespace dragon
