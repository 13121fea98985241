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
// Bound: HBM (every element is read and written once).  8 elements a lane, a head in the next power of two of lanes, so that the
// head's sums are a few shuffles; four heads in flight per lane.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "device_util.h"
#include "plan.h"

namespace dragon {
cudaError_t launch_colsum_finish(const float* part, int n_part, int cols, void* out, int dtype, cudaStream_t st);

namespace {

constexpr int kHeadThreads = 256, kHeadWarps = kHeadThreads / 32;
constexpr int kHeadRowsMost = 8;       // rows of a tile: their angles are computed together
constexpr int kPairsMost = kMaxRotatedWidth / 2;

enum Pairing { P_NONE, P_NEIGHBOURS, P_LANES, P_ANY };   // where a lane finds the partners of its 8 elements

struct HeadArgs {
  const void *x, *gain, *dy;
  const int* pos;
  void *u, *y;             // backwards: y receives dx
  float* dgain;            // partial rows [grid][width]
  int *status_clear;
  int xt, gt, dyt, ut, yt;
  int round_u;             // u is rounded to bf16 before it is rotated
  int rows, heads, width, dims, lanes;   // lanes: of a head, a power of two
  int tile;                // rows of a tile
  float eps, amplitude;
  unsigned long long freq[kPairsMost];   // turns per position, times 2^64
};

// the angles of `rows` rows from r0 on: (amplitude cos, amplitude sin) of every pair
__device__ __forceinline__ void fill_angles(const HeadArgs& a, float2 (*cs)[kPairsMost], int r0, int rows) {
  const int pairs = a.dims >> 1;
  for (int i = threadIdx.x; i < rows * pairs; i += kHeadThreads) {
    const int r = i / pairs, k = i - r * pairs;
    const unsigned long long turn = (unsigned long long)(long long)__ldg(a.pos + r0 + r) * a.freq[k];
    float s, c;
    sincospif((float)(int)(turn >> 32) * 0x1p-31f, &s, &c);
    cs[r][k] = make_float2(a.amplitude * c, a.amplitude * s);
  }
}

// v: this lane's 8 elements (from element e0 of its head on); back: by the negative angle.  buf: 256 floats of this warp (P_ANY)
template <int kPairing> __device__ __forceinline__ void turn(float* v, const float2* cs, int e0, int dims, int lane, bool back, float* buf) {
  const int half = dims >> 1;
  if (kPairing == P_NEIGHBOURS) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int i = (e0 >> 1) + p;
      if (i < half) {
        const float c = cs[i].x, s = back ? -cs[i].y : cs[i].y, p0 = v[2 * p], p1 = v[2 * p + 1];
        v[2 * p] = p0 * c - p1 * s;
        v[2 * p + 1] = p1 * c + p0 * s;
      }
    }
  } else if (kPairing == P_LANES) {      // half a multiple of 8: the partners are the 8 elements of one other lane
    const bool first = e0 < half, in = e0 < dims;
    const int from = in ? lane + (first ? half : -half) / 8 : lane, i0 = first ? e0 : in ? e0 - half : 0;
    const bool minus = first != back;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float other = __shfl_sync(0xffffffffu, v[e], from);
      const float2 t = cs[i0 + e];
      if (in) v[e] = v[e] * t.x + (minus ? -other : other) * t.y;
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
      if (at < dims) {
        const bool first = at < half;
        const float2 t = cs[first ? at : at - half];
        const float other = head[first ? at + half : at - half];
        v[e] = v[e] * t.x + (first != back ? -other : other) * t.y;
      }
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
  __shared__ float2 cs[kPairing == P_NONE ? 1 : kHeadRowsMost][kPairsMost];
  __shared__ float buf[kPairing == P_ANY ? kHeadWarps : 1][256];
  __shared__ float sums[kBack ? kHeadWarps : 1][kMaxRotatedWidth];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int l = lane & (a.lanes - 1), e0 = 8 * l;
  const bool active = e0 < a.width;
  const int per_warp = 32 / a.lanes, sub = lane / a.lanes;      // heads of one warp access
  const int groups = (a.heads + per_warp - 1) / per_warp;
  const float inv_width = 1.f / (float)a.width;
  const bool norm = a.gain != nullptr;
  float g[8], dg[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { g[e] = 1.f; dg[e] = 0.f; }
  if (norm && active) load_any<8>(a.gain, a.gt, (size_t)e0, g);
  for (long long r0 = (long long)blockIdx.x * a.tile; r0 < a.rows; r0 += (long long)gridDim.x * a.tile) {
    const int rows = (int)min((long long)a.tile, a.rows - r0);
    if (kPairing != P_NONE) {
      __syncthreads();
      fill_angles(a, cs, (int)r0, rows);
      __syncthreads();
    }
    const int items = rows * groups;
    for (int it0 = warp; it0 < items; it0 += kHeadWarps * kUnroll) {
      Raw<DT, 8> rx[kUnroll], rd[kUnroll];
      size_t at[kUnroll];
      int row[kUnroll];
      bool ok[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int it = it0 + k * kHeadWarps;
        row[k] = it / groups;
        const int head = (it - row[k] * groups) * per_warp + sub;
        ok[k] = it < items && active && head < a.heads;
        at[k] = ((size_t)(r0 + row[k]) * a.heads + head) * a.width + e0;
        if (ok[k]) {
          if (!kBack || norm) rx[k].load(a.x, a.xt, at[k]);
          if (kBack) rd[k].load(a.dy, a.dyt, at[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        if (it0 + k * kHeadWarps >= items) break;       // the whole warp
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
            inv = rsqrtf(sum_over_lanes(q, a.lanes) * inv_width + a.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * g[e];
            if (a.u && ok[k]) store_any<8>(a.u, a.ut, at[k], x);
            if (a.round_u) {
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = bf16_rounded(x[e]);
            }
          }
          if (kPairing != P_NONE) turn<kPairing>(x, cs[row[k]], e0, a.dims, lane, false, buf[kPairing == P_ANY ? warp : 0]);
          if (a.y && ok[k]) { Raw<DT, 8> o; o.set(x); o.store(a.y, a.yt, at[k]); }
        } else {
          float d[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = 0.f;
          if (ok[k]) rd[k].get(d);
          if (kPairing != P_NONE) turn<kPairing>(d, cs[row[k]], e0, a.dims, lane, true, buf[kPairing == P_ANY ? warp : 0]);
          if (norm) {
            float q = 0.f, m = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) { q += x[e] * x[e]; m += d[e] * g[e] * x[e]; }
            inv = rsqrtf(sum_over_lanes(q, a.lanes) * inv_width + a.eps);
            const float c = inv * inv * inv * (sum_over_lanes(m, a.lanes) * inv_width);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              dg[e] += d[e] * x[e] * inv;
              d[e] = inv * d[e] * g[e] - x[e] * c;
            }
          }
          if (a.y && ok[k]) { Raw<DT, 8> o; o.set(d); o.store(a.y, a.yt, at[k]); }
        }
      }
    }
  }
  if (kBack && a.dgain) {      // the CTA's part of dg: lanes of the same elements, then the warps, in a fixed order
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      for (int s = a.lanes; s < 32; s <<= 1) dg[e] += __shfl_xor_sync(0xffffffffu, dg[e], s);
      if (lane < a.lanes && active) sums[warp][e0 + e] = dg[e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += kHeadThreads) {
      float t = 0.f;
      for (int w = 0; w < kHeadWarps; ++w) t += sums[w][c];
      a.dgain[(size_t)blockIdx.x * a.width + c] = t;
    }
  }
}

// Rows of a tile: as many as leave four CTAs for every SM
int tile_rows(int64_t rows, int sm_count) { return (int)std::min<int64_t>(kHeadRowsMost, std::max<int64_t>(1, rows / (4 * (int64_t)sm_count))); }

template <bool kBack, int DT> void launch_pairing(const HeadArgs& a, int pairing, int grid, cudaStream_t st) {
  switch (pairing) {
    case P_NONE: head_kernel<DT, P_NONE, kBack><<<grid, kHeadThreads, 0, st>>>(a); break;
    case P_NEIGHBOURS: head_kernel<DT, P_NEIGHBOURS, kBack><<<grid, kHeadThreads, 0, st>>>(a); break;
    case P_LANES: head_kernel<DT, P_LANES, kBack><<<grid, kHeadThreads, 0, st>>>(a); break;
    default: head_kernel<DT, P_ANY, kBack><<<grid, kHeadThreads, 0, st>>>(a);
  }
}

template <bool kBack> cudaError_t launch(HeadArgs& a, const Step& s, int grid, cudaStream_t st) {
  const std::vector<double>& n = s.num;
  a.eps = (float)n[hn::EPS];
  a.lanes = 1;
  while (a.lanes * 8 < a.width) a.lanes *= 2;
  int pairing = P_NONE;
  if (a.pos) {
    a.dims = (int)n[hn::DIMS];
    a.amplitude = (float)n[hn::AMPLITUDE];
    const long double two_pi = 6.283185307179586476925286766559005768L;
    for (int i = 0; i < a.dims / 2; ++i) {
      const long double f = std::pow((long double)n[hn::BASE], -2.0L * i / a.dims);
      long double keep = 0.0L;
      if (n[hn::ORIGINAL] > 0.0) {
        const long double turns = n[hn::ORIGINAL] * f / two_pi;
        keep = n[hn::HIGH] > n[hn::LOW] ? (turns - n[hn::LOW]) / (n[hn::HIGH] - n[hn::LOW]) : turns >= n[hn::LOW] ? 1.0L : 0.0L;
        keep = std::min(1.0L, std::max(0.0L, keep));
      }
      a.freq[i] = (unsigned long long)(f * (keep + (1.0L - keep) / (long double)n[hn::FACTOR]) / two_pi * 18446744073709551616.0L);
    }
    pairing = n[hn::INTERLEAVED] != 0.0 ? P_NEIGHBOURS : a.dims % 16 == 0 ? P_LANES : P_ANY;
  }
  const bool bf16 = (kBack && !a.x ? true : a.xt == DRAGON_BF16) && (!a.y || a.yt == DRAGON_BF16) && (!kBack || a.dyt == DRAGON_BF16);
  const bool f32 = (kBack && !a.x ? true : a.xt == DRAGON_F32) && (!a.y || a.yt == DRAGON_F32) && (!kBack || a.dyt == DRAGON_F32);
  if (bf16) launch_pairing<kBack, DRAGON_BF16>(a, pairing, grid, st);
  else if (f32) launch_pairing<kBack, DRAGON_F32>(a, pairing, grid, st);
  else launch_pairing<kBack, -1>(a, pairing, grid, st);
  return cudaGetLastError();
}

}  // namespace

int head_bwd_partials(int64_t rows, int64_t, int sm_count) {
  const int tile = tile_rows(rows, sm_count);
  return (int)std::min<int64_t>((rows + tile - 1) / tile, 4 * (int64_t)sm_count);
}

cudaError_t launch_head(const StepRun& r) {
  const Step& s = r.s;
  const Shape& sh = r.mems[s.rd[hd::X]].shape;
  HeadArgs a = {};
  a.x = r.rd(hd::X); a.xt = r.rd_type(hd::X);
  a.gain = r.rd(hd::GAIN); a.gt = r.rd_type(hd::GAIN);
  a.pos = reinterpret_cast<const int*>(r.rd(hd::POS));
  a.u = r.wr(hd::U); a.ut = r.wr_type(hd::U);
  a.y = r.wr(hd::Y); a.yt = r.wr_type(hd::Y);
  if (!a.pos) { a.y = a.u; a.yt = a.ut; a.u = nullptr; }      // the norm alone writes its result as the last step
  if (s.wr[hd::Y] < 0) a.pos = nullptr;
  if (!a.y) { a.y = a.u; a.yt = a.ut; a.u = nullptr; }
  a.round_u = a.pos && s.round_dtype == DRAGON_BF16;
  a.status_clear = r.status_clear;
  a.width = (int)s.num[hn::WIDTH];
  a.rows = (int)sh.d[0];
  a.heads = (int)(sh.d[1] / a.width);
  a.tile = tile_rows(a.rows, r.sm_count);
  return launch<false>(a, s, (int)((a.rows + (int64_t)a.tile - 1) / a.tile), reinterpret_cast<cudaStream_t>(r.stream));
}

cudaError_t launch_head_bwd(const StepRun& r) {
  const Step& s = r.s;
  const Shape& sh = r.mems[s.rd[hb::DY]].shape;
  HeadArgs a = {};
  a.x = r.rd(hb::X); a.xt = r.rd_type(hb::X);
  a.gain = r.rd(hb::GAIN); a.gt = r.rd_type(hb::GAIN);
  a.pos = reinterpret_cast<const int*>(r.rd(hb::POS));
  a.dy = r.rd(hb::DY); a.dyt = r.rd_type(hb::DY);
  a.y = r.wr(hb::DX); a.yt = r.wr_type(hb::DX);
  a.status_clear = r.status_clear;
  a.width = (int)s.num[hn::WIDTH];
  a.rows = (int)sh.d[0];
  a.heads = (int)(sh.d[1] / a.width);
  a.tile = tile_rows(a.rows, r.sm_count);
  if (s.wr[hb::DGAIN] >= 0) a.dgain = reinterpret_cast<float*>(r.ws + s.colpart_off);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const int grid = head_bwd_partials(a.rows, a.heads, r.sm_count);
  cudaError_t e = launch<true>(a, s, grid, st);
  if (e == cudaSuccess && a.dgain) e = launch_colsum_finish(a.dgain, grid, a.width, r.wr(hb::DGAIN), r.wr_type(hb::DGAIN), st);
  return e;
}

}  // namespace dragon
